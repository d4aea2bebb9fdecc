"""The operators behind the classifier without a GPU: what the C ABI refuses before any HIP call, and the oracle's own definitions."""
import numpy as np
import pytest
import torch

from paper_1805_12549_amd import binding as B
from tests import logits_oracle as O

P = 0x100000        # an address that is never read: every call here returns before the first HIP call


def logprobs_args(**kw):
    a = dict(logits=P, dtype=B.CG_F32, rows=4, classes=100, row_stride=100, temperature=1.0, labels=P, given=1, top=5, logprob=P, entropy=P, top_ids=P,
             top_logprobs=P, workspace=0, workspace_bytes=0)
    a.update(kw)
    return a


def forward_args(**kw):
    a = dict(logits=P, dtype=B.CG_F32, rows=4, classes=100, row_stride=100, temperature=1.0, top_ids=P, top_logits=P, top=5, labels=P, teacher_weight=0.5,
             label_weight=0.5, loss=P, stats=P, grad_loss=P, grad=P, grad_stride=100, workspace=0, workspace_bytes=0)
    a.update(kw)
    return a


def backward_args(**kw):
    a = forward_args(**kw)
    for k in ("loss", "workspace", "workspace_bytes"):
        a.pop(k)
    return a


LOGITS = [(dict(dtype=B.CG_I8), B.CG_EUNSUPPORTED), (dict(dtype=7), B.CG_EUNSUPPORTED), (dict(rows=-1), B.CG_EINVAL), (dict(classes=0), B.CG_EINVAL),
          (dict(classes=-3), B.CG_EINVAL), (dict(row_stride=-1), B.CG_EINVAL), (dict(row_stride=1 << 61), B.CG_EINVAL), (dict(temperature=0.0), B.CG_EINVAL),
          (dict(temperature=-1.0), B.CG_EINVAL), (dict(temperature=float("inf")), B.CG_EINVAL), (dict(temperature=float("nan")), B.CG_EINVAL),
          (dict(temperature=1e-42), B.CG_EINVAL), (dict(temperature=3.1e-39), B.CG_EINVAL), (dict(temperature=3e38), B.CG_EINVAL), (dict(logits=0), B.CG_EINVAL), (dict(logits=P + 2), B.CG_EINVAL),
          (dict(logits=P + 1, dtype=B.CG_BF16), B.CG_EINVAL)]
TEACHER = [(dict(top=-1), B.CG_EINVAL), (dict(top=129), B.CG_EUNSUPPORTED), (dict(top=0), B.CG_EINVAL), (dict(top_ids=0), B.CG_EINVAL),
           (dict(top_logits=0), B.CG_EINVAL), (dict(labels=0), B.CG_EINVAL), (dict(teacher_weight=float("nan")), B.CG_EINVAL),
           (dict(label_weight=float("inf")), B.CG_EINVAL), (dict(top_ids=P + 4), B.CG_EINVAL), (dict(labels=P + 4), B.CG_EINVAL),
           (dict(top_logits=P + 2), B.CG_EINVAL), (dict(grad_loss=P + 1), B.CG_EINVAL), (dict(stats=P + 2), B.CG_EINVAL), (dict(grad=P + 2), B.CG_EINVAL),
           (dict(grad_stride=99), B.CG_EINVAL), (dict(grad_stride=1 << 61), B.CG_EINVAL), (dict(grad_stride=104), B.CG_EINVAL)]


def refused(call, args, code):
    with pytest.raises(B.CGError) as e:
        call(**args)
    assert e.value.code == code and str(e.value)


@pytest.mark.parametrize("over,code", LOGITS + [(dict(given=-1), B.CG_EINVAL), (dict(top=101), B.CG_EINVAL), (dict(top=-1), B.CG_EINVAL),
                                                (dict(classes=1000, row_stride=1000, top=129), B.CG_EUNSUPPORTED), (dict(labels=0), B.CG_EINVAL),
                                                (dict(logprob=0), B.CG_EINVAL), (dict(top_ids=0), B.CG_EINVAL), (dict(top_logprobs=0), B.CG_EINVAL),
                                                (dict(labels=P + 4), B.CG_EINVAL), (dict(top_ids=P + 4), B.CG_EINVAL), (dict(entropy=P + 2), B.CG_EINVAL)])
def test_logprobs_refusals(over, code):
    refused(B.cg_logprobs, logprobs_args(**over), code)


@pytest.mark.parametrize("over,code", LOGITS + TEACHER + [(dict(loss=0), B.CG_EINVAL), (dict(loss=P + 2), B.CG_EINVAL)])
def test_distill_forward_refusals(over, code):
    refused(B.cg_distill_forward, forward_args(**over), code)


@pytest.mark.parametrize("over,code", LOGITS + TEACHER + [(dict(stats=0), B.CG_EINVAL), (dict(grad=0), B.CG_EINVAL)])
def test_distill_backward_refusals(over, code):
    refused(B.cg_distill_backward, backward_args(**over), code)


def test_no_rows_is_no_work():
    B.cg_logprobs(**logprobs_args(rows=0, logits=0, labels=0, logprob=0, entropy=0, top_ids=0, top_logprobs=0))
    B.cg_distill_forward(**forward_args(rows=0, logits=0, top_ids=0, top_logits=0, labels=0, loss=0, stats=0, grad=0, grad_loss=0))
    B.cg_distill_backward(**backward_args(rows=0, logits=0, top_ids=0, top_logits=0, labels=0, stats=0, grad=0, grad_loss=0))


def test_workspace_is_asked_for_where_it_is_needed():
    for rows, classes in ((1, 10), (1, 131072), (4, 1 << 20), (100000, 1000), (0, 5)):
        assert B.cg_logprobs_workspace_bytes(rows, classes, 20) < 1 << 28
        assert B.cg_distill_workspace_bytes(rows, classes) < 1 << 28
    for rows, classes in ((-1, 10), (1, 0), (1, -5)):
        assert B.cg_logprobs_workspace_bytes(rows, classes, 20) == 0 and B.cg_distill_workspace_bytes(rows, classes) == 0


def test_tensors_that_are_not_on_the_gpu_are_refused():
    z, ids = torch.zeros(2, 10), torch.zeros(2, 3, dtype=torch.int64)
    for call in (lambda: B.logprobs(z), lambda: B.distill(z, ids, torch.zeros(2, 3)), lambda: B.distill_backward(z, torch.zeros(2, 3), ids, torch.zeros(2, 3)),
                 lambda: B.logprobs(z.half())):
        with pytest.raises(B.CGError):
            call()


def test_oracle_against_torch():
    """The oracle's definitions against torch's own in 64 bits."""
    rng = np.random.default_rng(0)
    z = rng.standard_normal(50) * 3
    got = O.logprobs(z, [4, -1, 50], 50, 0.7)
    want = torch.log_softmax(torch.from_numpy(z) / 0.7, 0)
    assert np.allclose(got["logprob"][0][:1], want[4]) and got["logprob"][0][1] == 0 and np.isnan(got["logprob"][0][2])
    assert np.isclose(got["entropy"][0], -(want.exp() * want).sum())
    assert np.array_equal(got["top_ids"], want.argsort(descending=True).numpy())
    ids, t = np.array([3, 9, 3, -1]), np.array([1.0, 2.0, -0.5, 7.0])
    x = torch.from_numpy(z).requires_grad_()
    q = torch.softmax(torch.from_numpy(t[:3]) / 2, 0)
    loss = 1.5 * (q * (q.log() - torch.log_softmax(x / 2, 0)[torch.from_numpy(ids[:3])])).sum() - 0.3 * torch.log_softmax(x, 0)[9]
    loss.backward()
    (lv, _), (gv, _) = O.distill(z, ids, t, 9, 1.5, 0.3, 2.0)
    assert np.isclose(lv, loss.item()) and np.allclose(gv, x.grad.numpy())


def test_bounds_reject_a_planted_mistake():
    """A log probability off by one part in ten thousand, a gradient without the factor 1 / T: outside the bounds."""
    rng = np.random.default_rng(1)
    z = rng.standard_normal(1000) * 3
    value, bound = O.logprobs(z, [5], 0, 1.0)["logprob"]
    with pytest.raises(AssertionError):
        O.check(value * (1 + 1e-4), value, bound, "planted")
    _, (gv, gb) = O.distill(z, np.arange(8), np.arange(8.0), -1, 1.0, 0.0, 2.0)
    with pytest.raises(AssertionError):
        O.check(gv * 2, gv, O.rounded(gb, gv, 2), "planted")
