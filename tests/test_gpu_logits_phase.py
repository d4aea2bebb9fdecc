"""Gradients of logits that begin off a 16-byte boundary: a new gradient lies as its logits do, row for row."""
import numpy as np
import pytest
import torch

from paper_1805_12549_amd import binding as B
from tests import logits_oracle as O

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("way", ["extension", "ctypes"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,pad", [(1, 1, 0), (1, 1001, 3), (4, 5, 0), (4, 1000, 0), (5, 1003, 0), (4, 1003, 6), (3, 50003, 0), (3, 50001, 2), (200, 20003, 0)])
def test_a_new_gradient_lies_as_its_logits(rows, classes, pad, dtype, way, monkeypatch):
    if way == "ctypes":
        monkeypatch.setattr(B, "_calls", None)
    elif B._calls is None:
        pytest.skip("the extension is not built")
    rng = np.random.default_rng(classes + pad)
    size = TYPES[dtype].itemsize
    ids = rng.integers(0, classes, (rows, 5))
    t = rng.standard_normal((rows, 5)).astype(np.float32)
    labels = rng.integers(0, classes, rows)
    teacher = [torch.from_numpy(a).cuda() for a in (ids, t, labels)]
    for offset in range(16 // size):
        buf = torch.full((offset + rows * (classes + pad),), float("nan"), dtype=TYPES[dtype], device="cuda")
        z = buf[offset:].as_strided((rows, classes), (classes + pad, 1))
        z.copy_(torch.from_numpy((2.5 * rng.standard_normal((rows, classes))).astype(np.float32)))
        kw = dict(label_weight=0.5, temperature=2.0)
        loss, stats, grad = B.distill(z, *teacher, grad=True, **kw)
        later = B.distill_backward(z, stats, *teacher, **kw)
        for g in (grad, later):
            assert g.shape == z.shape and g.dtype == z.dtype and g.stride(1) == 1 and not g._is_view()
            assert [g[r].data_ptr() % 16 for r in range(rows)] == [z[r].data_ptr() % 16 for r in range(rows)], "offset %d" % offset
            assert g.untyped_storage().nbytes() < (rows * classes + (rows + 1) * (16 // size)) * size
        wide = z.double().cpu().numpy()
        for r in (0, rows - 1):
            (lv, lb), (gv, gb) = O.distill(wide[r], ids[r], t[r], labels[r], 1.0, 0.5, 2.0)
            O.check(loss[r].item(), lv, lb, "loss")
            for g in (grad, later):
                O.check(g[r].double().cpu().numpy(), gv, O.rounded(gb, gv, size), "gradient, offset %d" % offset)


@pytest.mark.parametrize("way", ["extension", "ctypes"])
def test_no_rows_and_inference_mode(way, monkeypatch):
    if way == "ctypes":
        monkeypatch.setattr(B, "_calls", None)
    elif B._calls is None:
        pytest.skip("the extension is not built")
    z = torch.randn(3 * 1001 + 1, device="cuda")[1:].view(3, 1001)
    ids, t = torch.zeros((3, 2), dtype=torch.int64, device="cuda"), torch.zeros((3, 2), device="cuda")
    want = B.distill(z, ids, t, grad=True)[2]
    assert B.distill(z[:0], ids[:0], t[:0], grad=True)[2].shape == (0, 1001)
    with torch.inference_mode():
        got = B.distill(z, ids, t, grad=True)[2]
        assert got.is_inference() and got.data_ptr() % 16 == z.data_ptr() % 16 and torch.equal(got, want)
    # as it is used: into the backward pass of what made the logits
    leaf = torch.randn(3 * 1001 + 1, device="cuda", requires_grad=True)
    logits = (2 * leaf)[1:].view(3, 1001)
    logits.backward(B.distill(logits.detach(), ids, t, grad=True)[2])
    plain = leaf.detach().double().requires_grad_()
    q = torch.full((3, 2), 0.5, dtype=torch.float64, device="cuda")
    (-(q * torch.log_softmax((2 * plain)[1:].view(3, 1001), 1).gather(1, ids))).sum().backward()
    assert torch.allclose(leaf.grad.double(), plain.grad, rtol=1e-5, atol=1e-6)
