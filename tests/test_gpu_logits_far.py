"""Logits so far apart that their difference passes float32's range while the difference over the temperature does not."""
import numpy as np
import pytest
import torch

from paper_1805_12549_amd import binding as B
from tests import logits_oracle as O

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def far_rows(classes, dtype):
    """Rows whose logits reach from the type's lowest value to its greatest."""
    most = torch.finfo(TYPES[dtype]).max
    rng = np.random.default_rng(classes)
    z = torch.from_numpy(rng.uniform(-1, 1, (5, classes)).astype(np.float32)).cuda().mul_(most).to(TYPES[dtype]).clamp_(-most, most)
    z[0] = -most
    z[0, classes - 1] = most
    z[1] = most
    z[1, ::2] = -most
    z[2, 0], z[2, 1] = most, -most
    z[3, 1::3] = -float("inf")
    z[3, 0] = most
    z[4] = -most
    z[4, 2] = 0.75 * most
    return z


# temperatures at which the classes' shares are anything from one to equal; powers of two, whose quotients are exact
@pytest.mark.parametrize("temperature", [2.0, 3.0, 2.0 ** 20, 2.0 ** 119, 2.0 ** 122, 1.1 * 2.0 ** 124, 2.0 ** 126])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [3, 1000, 20001, 70001])
def test_far_logits(classes, dtype, temperature):
    z = far_rows(classes, dtype)
    rows, top = z.shape[0], min(20, classes)
    wide = z.double().cpu().numpy()
    t32 = float(np.float32(temperature))
    labels = np.tile(np.array([0, classes - 1, classes // 2]), (rows, 1))
    got = B.logprobs(z, torch.from_numpy(labels).cuda(), top=top, temperature=temperature)
    torch.cuda.synchronize()
    logprob, entropy, ids, alternatives = [g.cpu().numpy() for g in got]
    for r in range(rows):
        want = O.logprobs(wide[r], labels[r], top, t32)
        O.check(logprob[r], *want["logprob"], "row %d logprob" % r)
        O.check(entropy[r], *want["entropy"], "row %d entropy" % r)
        assert np.array_equal(ids[r], want["top_ids"]), r
        O.check(alternatives[r], *want["top_logprobs"], "row %d alternatives" % r)


# (a temperature above 2^122 makes gradients of denormal size, which are no part of this)
@pytest.mark.parametrize("temperature", [4.0, 2.0 ** 20, 2.0 ** 121])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [3, 1000, 20001, 70001])
def test_far_logits_and_a_far_teacher(classes, dtype, temperature):
    z = far_rows(classes, dtype)
    rows = z.shape[0]
    most = np.finfo(np.float32).max
    rng = np.random.default_rng(classes)
    ids = np.stack([rng.permutation(classes)[:3] for _ in range(rows)])
    ids[3] = 0                                                 # (a class that the mask leaves)
    t = (rng.uniform(-1, 1, (rows, 3)) * most).astype(np.float32)
    t[0], t[1] = (most, -most, 0), (-most, -most, most)
    wide = z.double().cpu().numpy()
    teacher = [torch.from_numpy(a).cuda() for a in (ids, t)]
    kw = dict(teacher_weight=0.125, temperature=temperature)
    up = torch.full((rows,), temperature, device="cuda")       # (the usual factor, so that gradients are of ordinary size)
    loss, stats, grad = B.distill(z, *teacher, grad=True, grad_loss=up, **kw)
    alone, stats2, _ = B.distill(z, *teacher, **kw)
    later = B.distill_backward(z, stats2, *teacher, grad_loss=up, **kw)
    torch.cuda.synchronize()
    for r in range(rows):
        (lv, lb), (gv, gb) = O.distill(wide[r], ids[r], t[r], -1, 0.125, 0.0, temperature, temperature)
        gb = O.rounded(gb, gv, z.element_size())
        for got in (loss, alone):
            O.check(got[r].item(), lv, lb, "row %d loss" % r)
        for got in (grad, later):
            O.check(got[r].double().cpu().numpy(), gv, gb, "row %d gradient" % r)


def test_a_teachers_entry_below_the_normal_range_holds_no_mass():
    """87.3 temperatures below the greatest one: such an entry asks for nothing, of a class that is ruled out neither; above that the loss is infinite."""
    z = torch.zeros((4, 1000), device="cuda")
    z[:, 7] = -float("inf")
    ids = torch.tensor([[3, 7]] * 4, device="cuda")
    t = torch.tensor([[0.0, -87.0], [0.0, -88.0], [5.0, -3.0e38], [0.0, -float("inf")]], device="cuda")
    for temperature in (1.0, 4.0):
        loss, _, grad = B.distill(z, ids, t * temperature if temperature == 1.0 else torch.where(t > -1e38, t * temperature, t), temperature=temperature, grad=True)
        assert loss[0].item() == float("inf")
        assert np.abs(loss[1:].cpu().numpy() - np.log(999.0)).max() <= (O.chain(1000) + 64) * O.U * np.log(999.0)
        assert torch.isfinite(grad).all() and (grad[1:, 7] == 0).all()
