"""The operators behind the classifier on the GPU against their definitions in 64 bits (tests/logits_oracle.py)."""
import numpy as np
import pytest
import torch

from paper_1805_12549_amd import binding as B
from tests import logits_oracle as O

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
INF, NAN = float("inf"), float("nan")


def rows_of(rng, rows, classes, dtype, pad=0, offset=0, spread=2.5):
    """Logits as a view of a larger tensor: `pad` elements between rows, `offset` in front; the rest is NaN."""
    z = (rng.standard_normal((rows, classes)) * spread + 4 * rng.standard_normal((rows, 1))).astype(np.float32)
    buf = torch.full((offset + rows * (classes + pad),), NAN, device="cuda", dtype=TYPES[dtype])
    view = buf[offset:].as_strided((rows, classes), (classes + pad, 1)) if rows else buf.new_empty((0, classes))
    view.copy_(torch.from_numpy(z))
    return view


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int8), b.contiguous().view(torch.int8))


def wide(t):
    return t.float().cpu().numpy().astype(np.float64)


def check_logprobs(logits, labels, top, temperature=1.0, given_rows=None):
    got = B.logprobs(logits, None if labels is None else torch.from_numpy(labels).cuda(), top=top, temperature=temperature)
    torch.cuda.synchronize()
    logprob, entropy, ids, alternatives = [None if g is None else g.cpu().numpy() for g in got]
    z = wide(logits)
    for r in (range(len(z)) if given_rows is None else given_rows):
        want = O.logprobs(z[r], [] if labels is None else np.atleast_1d(labels[r]), top, temperature)
        where = "row %d of %s" % (r, tuple(logits.shape))
        if labels is not None:
            O.check(np.atleast_1d(logprob[r]), *want["logprob"], where + " logprob")
        O.check(entropy[r], *want["entropy"], where + " entropy")
        if top:
            assert np.array_equal(ids[r], want["top_ids"]), where
            O.check(alternatives[r], *want["top_logprobs"], where + " alternatives")
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,top", [(1, 1, 1), (3, 2, 2), (5, 7, 0), (4, 10, 10), (2, 63, 5), (2, 64, 64), (3, 65, 20), (2, 128, 128), (9, 255, 128),
                                              (4, 257, 1), (6, 1000, 5), (3, 1023, 128), (3, 2049, 128), (2, 4099, 20), (1, 8191, 3), (5, 16385, 64),
                                              (2, 50003, 20), (1, 131072, 128), (1, 262147, 20)])
def test_logprobs(rows, classes, top, dtype):
    rng = np.random.default_rng(rows * 1000003 + classes)
    labels = rng.integers(0, classes, (rows, 3))
    check_logprobs(rows_of(rng, rows, classes, dtype), labels, top, temperature=(1.0, 0.7, 2.5)[classes % 3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes,pad,offset", [(1000, 1, 0), (1001, 0, 3), (3001, 5, 1), (50000, 8, 2), (50001, 7, 5), (131, 0, 1), (5, 2, 1), (100000, 3, 7)])
def test_logprobs_of_rows_at_any_address(classes, pad, offset, dtype):
    rng = np.random.default_rng(classes + pad)
    check_logprobs(rows_of(rng, 5, classes, dtype, pad, offset), rng.integers(0, classes, (5,)), min(20, classes))


@pytest.mark.parametrize("rows", [2, 17, 300, 1025, 3001])
def test_logprobs_of_many_rows(rows):
    rng = np.random.default_rng(rows)
    check_logprobs(rows_of(rng, rows, 1000, "f32"), rng.integers(0, 1000, (rows, 1)), 5, given_rows=range(0, rows, 1 + rows // 40))
    check_logprobs(rows_of(rng, rows, 4103, "bf16"), rng.integers(0, 4103, (rows, 1)), 20, given_rows=range(0, rows, 1 + rows // 20))


def test_logprobs_of_one_row_many_times():
    """Rows at distance 0, as an expanded tensor has them."""
    rng = np.random.default_rng(5)
    one = rows_of(rng, 1, 5000, "bf16")
    check_logprobs(one.expand(7, 5000), rng.integers(0, 5000, (7,)), 9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [9, 1000, 5003, 70001])
def test_logprobs_of_special_rows(classes, dtype):
    rng = np.random.default_rng(classes)
    z = rows_of(rng, 16, classes, dtype)
    lowest = torch.finfo(TYPES[dtype]).min
    z[0] = -INF                                     # a mask that leaves nothing
    z[1, 1:] = -INF                                 # ... one class
    z[2, : classes - 1] = -INF                      # ... the last one
    z[3] = lowest                                   # masked by the type's lowest value throughout
    z[4, ::2] = lowest
    z[5, 3] = NAN
    z[6, classes - 1] = INF
    z[7] = NAN
    z[8] = 2.5                                      # all equal
    z[9] = 0.0
    z[9, ::3] = -0.0                                # 0 and -0 are equal
    z[10] = torch.arange(classes, device="cuda") % 7        # ties throughout
    z[11] = -torch.arange(classes, device="cuda").float()   # falling
    z[12] = torch.arange(classes, device="cuda").float() / 16       # rising
    z[13] += 1.0e4 if dtype == "f32" else 64.0      # a large offset
    z[14, torch.rand(classes, device="cuda") < 0.98] = -INF
    z[15] = -torch.finfo(TYPES[dtype]).max
    z[15, 4] = torch.finfo(TYPES[dtype]).max
    labels = rng.integers(0, classes, (16, 4))
    labels[:, 1] = -1
    labels[:, 2] = np.where(np.arange(16) % 2, classes, -100)
    labels[3, 2] = 2 ** 62
    labels[1, 0], labels[2, 0] = 0, 0
    check_logprobs(z, labels, min(9, classes), 0.5)
    check_logprobs(z, labels, min(128, classes))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes,top", [(50, 20), (300, 128), (1000, 20), (5003, 128), (131072, 20), (140001, 128)])
def test_logprobs_where_a_mask_leaves_few(classes, top, dtype):
    """Fewer classes than alternatives, as many and some more, at the row's ends and anywhere: the rest are ruled out ones, by index."""
    rng = np.random.default_rng(classes)
    left = [0, 1, 2, top - 1, top, top + 1, 2 * top, classes]
    z = rows_of(rng, 2 * len(left), classes, dtype)
    for r, n in enumerate(left * 2):
        n = min(n, classes)
        keep = rng.choice(classes, n, replace=False) if r < len(left) else np.r_[:n // 2, classes - (n - n // 2):classes]
        mask = torch.ones(classes, dtype=torch.bool, device="cuda")
        mask[torch.from_numpy(keep).cuda()] = False
        z[r, mask] = -INF
    check_logprobs(z, rng.integers(0, classes, (2 * len(left),)), top)


@pytest.mark.parametrize("classes", [1000, 40000, 131072])
def test_logprobs_where_one_lane_holds_the_alternatives(classes):
    """The greatest logits at a fixed distance from each other: whichever way a row is shared out, some lane holds many of them."""
    rng = np.random.default_rng(classes)
    z = rows_of(rng, 8, classes, "f32")
    for r, step in enumerate((1, 4, 8, 256, 512, 1024, 2048, 8192)):
        at = torch.arange(r % 3, classes, step, device="cuda")
        z[r, at] += 50 + torch.from_numpy(rng.permutation(len(at)).astype(np.float32)).cuda() / 64
    check_logprobs(z, None, 128)


@pytest.mark.parametrize("classes", [9, 1000])
@pytest.mark.parametrize("top", [9, 32, 33])
def test_logprobs_of_special_rows_among_many(classes, top):
    """Short rows in great numbers: NaN, infinities, ties and masks beside each other."""
    rng = np.random.default_rng(top)
    z = rows_of(rng, 8, classes, "f32")
    z[0] = -INF
    z[1, 1:] = -INF
    z[2, 3] = NAN
    z[3, classes - 1] = INF
    z[4] = 1.5
    z[5] = torch.finfo(torch.float32).min
    z[6] = torch.arange(classes, device="cuda") % 3
    many = z.repeat(100, 1)
    labels = rng.integers(-1, classes + 1, 800)
    labels[:8] = 0
    got = check_logprobs(many, labels, min(top, classes), given_rows=range(40))
    for t in got[1:]:
        assert same_bits(t, t[:8].repeat(100, *[1] * (t.dim() - 1)))


def test_one_row_of_two_to_the_31_less_one_classes():
    """The longest row: zeros but for a few classes, so that every value is known."""
    classes = 2 ** 31 - 1
    z = torch.zeros((1, classes), dtype=torch.bfloat16, device="cuda")
    at = [0, 7, 2 ** 30, classes - 2, classes - 1]
    z[0, at] = torch.tensor([20.0, 21.0, 22.0, 23.0, 24.0], dtype=torch.bfloat16, device="cuda")
    total = classes - 5 + sum(np.exp(v) for v in (20.0, 21.0, 22.0, 23.0, 24.0))
    label = torch.tensor([classes - 2], device="cuda")
    logprob, entropy, ids, alternatives = B.logprobs(z, label, top=7)
    assert ids[0].tolist() == at[::-1] + [1, 2]
    want = np.array([24.0, 23.0, 22.0, 21.0, 20.0, 0.0, 0.0]) - np.log(total)
    # (sums of whole numbers below 2^24 are exact; the five exponentials and each sum of parts round)
    assert np.abs(alternatives[0].cpu().numpy() - want).max() <= 200 * O.U * 24 and abs(logprob.item() - want[1]) <= 200 * O.U * 24
    t = torch.tensor([[1.0, 0.0]], device="cuda")
    ids = torch.tensor([[classes - 1, 5]], device="cuda")
    q = 1 / (1 + np.exp(-1.0))
    loss, stats, grad = B.distill(z, ids, t, label, label_weight=1.0, grad=True)
    assert abs(loss.item() - (q * (np.log(q) - want[0]) + (1 - q) * (np.log(1 - q) - want[6]) - want[1])) <= 600 * O.U * 24
    step = 2.0 ** -8 + 1e-5
    for v, x in ((0, 2 * np.exp(20) / total), (classes - 2, 2 * np.exp(23) / total - 1), (classes - 1, 2 * np.exp(24) / total - q), (5, 2 / total - (1 - q)),
                 (2 ** 31 - 100, 2 / total)):
        assert abs(grad[0, v].item() - x) <= step * abs(x) + 1e-5 * (v in (5, classes - 1, classes - 2)), v


def test_logprobs_leave_out_what_is_not_asked_for():
    z = rows_of(np.random.default_rng(1), 4, 777, "f32")
    assert [o is None for o in B.logprobs(z, entropy=False)] == [True] * 4
    logprob, entropy, ids, alternatives = B.logprobs(z, torch.zeros(4, 0, dtype=torch.int64, device="cuda"))
    assert logprob.shape == (4, 0) and entropy.shape == (4,) and ids is None and alternatives is None
    for out in B.logprobs(z[:0], torch.zeros(0, 2, dtype=torch.int64, device="cuda"), top=3):
        assert out.shape[0] == 0


def teacher_of(rng, rows, classes, top, absent=False, repeated=False):
    ids = np.stack([rng.permutation(classes)[:top] if classes < 100000 else rng.choice(classes, top, replace=False) for _ in range(rows)]).astype(np.int64)
    if repeated and top > 1:
        ids[:, 1::2] = ids[:, :1]
    if absent:
        ids[np.arange(top)[None, :] >= rng.integers(0, top + 1, (rows, 1))] = -1
    t = (3 * rng.standard_normal((rows, top)) + 9).astype(np.float32)
    labels = rng.integers(0, classes, rows)
    if absent:
        labels[rng.random(rows) < 0.3] = -100
    return ids.reshape(rows, top), t, labels


def check_distill(z, ids, t, labels, wt, wl, temperature, up=None, given_rows=None, in_place=False):
    """Loss, the gradient of the same call and that of a backward call."""
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    teacher = (dev(ids), dev(t), dev(labels))
    kw = dict(teacher_weight=wt, label_weight=wl, temperature=temperature)
    up_dev = dev(up)
    rows, classes = z.shape
    zw = wide(z)
    loss, stats, grad = B.distill(z, *teacher, grad=True, grad_loss=up_dev, **kw)
    alone, stats2, none = B.distill(z, *teacher, **kw)
    later = B.distill_backward(z, stats2, *teacher, grad_loss=up_dev, **kw)
    torch.cuda.synchronize()
    assert none is None and grad.shape == z.shape and grad.dtype == z.dtype
    got = [wide(loss), wide(grad), wide(alone), wide(later)]
    for r in (range(rows) if given_rows is None else given_rows):
        no = np.zeros(0)
        (lv, lb), (gv, gb) = O.distill(zw[r], no if ids is None else ids[r], no if t is None else t[r], -1 if labels is None else labels[r], wt, wl, temperature,
                                       1.0 if up is None else float(up[r]))
        gb = O.rounded(gb, np.where(np.isfinite(gv), gv, 0.0), z.element_size())
        where = "row %d of %s" % (r, tuple(z.shape))
        O.check(got[0][r], lv, lb, where + " loss")
        O.check(got[2][r], lv, lb, where + " loss alone")
        O.check(got[1][r], gv, gb, where + " gradient")
        O.check(got[3][r], gv, gb, where + " gradient of the backward call")
    if in_place:
        again = z.clone() if z.is_contiguous() else z
        same = B.distill(again, *teacher, grad=again, grad_loss=up_dev, **kw)
        assert same[2] is again and same_bits(same[0], loss) and same_bits(again, grad)
    return loss, grad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,top", [(1, 1, 1), (3, 2, 2), (5, 7, 3), (4, 10, 10), (2, 64, 64), (3, 65, 20), (2, 128, 128), (6, 1000, 16), (3, 1023, 128),
                                              (3, 2049, 7), (2, 4099, 50), (5, 16385, 64), (2, 50003, 20), (1, 131072, 128), (1, 262147, 20)])
@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_distill(rows, classes, top, temperature, dtype):
    rng = np.random.default_rng(rows * 1000003 + classes)
    up = rng.standard_normal(rows).astype(np.float32)
    check_distill(rows_of(rng, rows, classes, dtype), *teacher_of(rng, rows, classes, top), 0.5 * temperature ** 2, 0.5, temperature, up)


@pytest.mark.parametrize("wt,wl,temperature", [(1.0, 0.0, 1.0), (0.0, 1.0, 1.0), (2.0, 0.0, 0.5), (0.0, 0.7, 3.0), (0.0, 0.0, 1.0), (-1.0, 2.0, 4.0)])
@pytest.mark.parametrize("classes", [1000, 20001])
def test_distill_with_one_term(wt, wl, temperature, classes):
    rng = np.random.default_rng(classes)
    ids, t, labels = teacher_of(rng, 4, classes, 12)
    check_distill(rows_of(rng, 4, classes, "f32"), ids, t, labels, wt, wl, temperature)
    if wt == 0:
        check_distill(rows_of(rng, 4, classes, "bf16"), None, None, labels, wt, wl, temperature)
    if wl == 0:
        check_distill(rows_of(rng, 4, classes, "bf16"), ids, t, None, wt, wl, temperature)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes,pad,offset", [(1000, 1, 0), (1001, 0, 3), (3001, 5, 1), (50000, 8, 2), (50001, 7, 5), (131, 0, 1), (5, 2, 1), (100000, 3, 7)])
def test_distill_of_rows_at_any_address(classes, pad, offset, dtype):
    rng = np.random.default_rng(classes + pad)
    ids, t, labels = teacher_of(rng, 5, classes, min(33, classes), absent=True)
    check_distill(rows_of(rng, 5, classes, dtype, pad, offset), ids, t, labels, 0.5, 0.5, 1.0, rng.standard_normal(5).astype(np.float32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes,offset", [(1003, 0), (40001, 1)])
def test_distill_into_a_given_tensor_leaves_the_rest(classes, offset, dtype):
    rng = np.random.default_rng(classes)
    z = rows_of(rng, 6, classes, dtype, pad=2)
    ids, t, labels = teacher_of(rng, 6, classes, 11)
    teacher = [torch.from_numpy(a).cuda() for a in (ids, t, labels)]
    buf = torch.full((offset + 6 * (classes + 9),), 7.0, dtype=TYPES[dtype], device="cuda")
    view = buf[offset:].as_strided((5, classes), (classes + 9, 1))
    kw = dict(label_weight=0.5, temperature=2.0)
    loss, stats, want = B.distill(z, *teacher, grad=True, **kw)
    for call in (lambda: B.distill(z[:5], teacher[0][:5], teacher[1][:5], teacher[2][:5], grad=view, **kw),
                 lambda: B.distill_backward(z[:5], stats[:5], teacher[0][:5], teacher[1][:5], teacher[2][:5], grad=view, **kw)):
        buf.fill_(7.0)
        call()
        got = buf.clone()
        got[offset:].as_strided((5, classes), (classes + 9, 1)).fill_(7.0)
        assert bool((got == 7.0).all()), "elements beside the rows were written"
        # (rows of another alignment may be summed in another order: each side is off by its bound at most)
        for r in range(5):
            value, bound = O.distill(wide(z)[r], ids[r], t[r], labels[r], 1.0, 0.5, 2.0)[1]
            bound = O.rounded(bound, value, z.element_size())
            O.check(wide(view)[r], value, bound, "row %d of the given tensor" % r)
            O.check(wide(want)[r], value, bound, "row %d" % r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(5, 1000), (3, 50003), (70, 4099), (300, 777)])
def test_distill_in_place_of_the_logits(rows, classes, dtype):
    rng = np.random.default_rng(rows)
    ids, t, labels = teacher_of(rng, rows, classes, 17, absent=True, repeated=True)
    check_distill(rows_of(rng, rows, classes, dtype), ids, t, labels, 0.5, 0.5, 2.0, rng.standard_normal(rows).astype(np.float32),
                  given_rows=range(0, rows, 1 + rows // 10), in_place=True)


@pytest.mark.parametrize("rows", [2, 17, 300, 1025, 3001])
def test_distill_of_many_rows(rows):
    rng = np.random.default_rng(rows)
    for classes, dtype in ((1000, "f32"), (4103, "bf16")):
        ids, t, labels = teacher_of(rng, rows, classes, 16, absent=True)
        check_distill(rows_of(rng, rows, classes, dtype), ids, t, labels, 0.5, 0.5, 2.0, rng.standard_normal(rows).astype(np.float32),
                      given_rows=range(0, rows, 1 + rows // 20))


@pytest.mark.parametrize("rows,classes,dtype,top", [(4200, 100, "f32", 7), (700, 300, "f32", 100), (1500, 4100, "f32", 16), (600, 12001, "f32", 128),
                                                    (300, 70001, "bf16", 33), (300, 140001, "bf16", 40), (130, 70001, "f32", 20), (129, 66000, "f32", 3)])
def test_distill_of_rows_walked_in_turn(rows, classes, dtype, top):
    """More rows than there are workgroups, of every length that registers hold and longer ones; in place as well."""
    rng = np.random.default_rng(rows)
    z = rows_of(rng, rows, classes, dtype)
    ids = rng.integers(0, classes, (rows, top))
    ids[rng.random((rows, top)) < 0.1] = -1
    labels = rng.integers(-1, classes, rows)
    check_distill(z, ids, (3 * rng.standard_normal((rows, top))).astype(np.float32), labels, 0.5, 0.5, (1.0, 2.0)[rows % 2],
                  rng.standard_normal(rows).astype(np.float32), given_rows=[0, 1, rows // 2, rows - 2, rows - 1], in_place=True)


def special_rows(rng, classes, dtype):
    z = rows_of(rng, 20, classes, dtype)
    ids, t, labels = teacher_of(rng, 20, classes, 8)
    lowest = torch.finfo(TYPES[dtype]).min
    z[0] = -INF
    z[1, 1:] = -INF                     # (the teacher's classes are ruled out: an infinite loss)
    ids[2], labels[2] = -1, -1          # a padded row, with what it likes in it
    z[2] = NAN
    z[3] = lowest
    z[4, ::2] = lowest
    ids[4], labels[4] = 1 + 2 * (np.arange(8) % 4), 1      # (classes that have a probability)
    z[5, classes // 2] = NAN
    z[6, 0] = INF
    ids[7, 3] = classes                 # beyond the classes
    labels[8] = classes + 5
    ids[9, 1:] = ids[9, 0]              # one class, eight times
    labels[9] = ids[9, 0]
    t[10] = -INF                        # a teacher without mass
    t[11, 2:] = -INF
    z[11, torch.from_numpy(ids[11, 2:]).cuda()] = -INF      # ruled out on both sides
    t[12, 3] = NAN
    t[13, 3] = INF
    t[14] = t[14] - 1.0e4               # log probabilities or logits: any constant
    z[15] = 3.0
    z[16] += 1.0e4 if dtype == "f32" else 64.0
    ids[17, ::2] = -5
    labels[18] = -100
    z[19, ::3] = -INF
    ids[19], labels[19] = 1, 1
    return z, ids, t, labels


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [9, 1000, 5003, 70001])
@pytest.mark.parametrize("wt,wl,temperature", [(0.5, 0.5, 1.0), (4.0, 0.5, 2.0), (1.0, 0.0, 0.7), (0.0, 1.0, 1.0)])
def test_distill_of_special_rows(classes, wt, wl, temperature, dtype):
    check_distill(*special_rows(np.random.default_rng(classes), classes, dtype), wt, wl, temperature, in_place=True)


@pytest.mark.parametrize("classes", [9, 1000])
def test_distill_of_special_rows_among_many(classes):
    z, ids, t, labels = special_rows(np.random.default_rng(classes), classes, "f32")
    again = lambda a: np.tile(a, (30,) + (1,) * (a.ndim - 1))  # noqa: E731
    loss, grad = check_distill(z.repeat(30, 1), again(ids), again(t), again(labels), 0.5, 0.5, 2.0, given_rows=range(20), in_place=True)
    assert same_bits(loss, loss[:20].repeat(30)) and same_bits(grad, grad[:20].repeat(30, 1))


def test_distill_gradient_is_the_loss_difference():
    """Differences of the losses that the GPU returns, against the gradient that it returns: z +- h, with h = 2^-4 the difference quotient is off by
    h^2 / 6 times the third derivative (a sum of probabilities' third central moments: below 1 for each term's weight over T^3) and by the
    losses' own errors over 2 h."""
    rng = np.random.default_rng(11)
    classes, temperature, h = 37, 1.5, 2.0 ** -4
    z = rows_of(rng, 1, classes, "f32")
    ids, t, labels = teacher_of(rng, 1, classes, 9, repeated=True)
    moved = z.repeat(2 * classes, 1)
    at = torch.arange(classes, device="cuda")
    moved[at, at] += h
    moved[classes + at, at] -= h
    steps = wide(moved)
    dev = [torch.from_numpy(np.repeat(a, 2 * classes, 0)).cuda() for a in (ids, t, labels)]
    kw = dict(teacher_weight=2.0, label_weight=0.5, temperature=temperature)
    loss = wide(B.distill(moved, *dev, **kw)[0])
    grad = wide(B.distill(z, *[d[:1] for d in dev], grad=True, **kw)[2])[0]
    bounds = np.array([O.distill(s, ids[0], t[0], labels[0], 2.0, 0.5, temperature)[0][1] for s in steps])
    quotient = (loss[:classes] - loss[classes:]) / (steps[np.arange(classes), np.arange(classes)] - steps[classes + np.arange(classes), np.arange(classes)])
    grad_bound = O.distill(wide(z)[0], ids[0], t[0], labels[0], 2.0, 0.5, temperature)[1][1]
    assert (np.abs(quotient - grad) <= h * h / 6 * (2.0 / temperature ** 3 + 0.5) + (bounds[:classes] + bounds[classes:]) / (2 * h) + grad_bound).all()


def test_teacher_and_student_together():
    """As they are used: the network's logits, its answers, a teacher's top classes from the same operator, and the student's step on them."""
    rng = np.random.default_rng(3)
    classes, rows, top = 1000, 24, 32
    teacher, student = rows_of(rng, rows, classes, "f32", spread=4.0), rows_of(rng, rows, classes, "bf16")
    labels = teacher.argmax(1)
    _, _, ids, logp = check_logprobs(teacher, labels.cpu().numpy(), top)
    loss, grad = check_distill(student, ids.cpu().numpy(), logp.cpu().numpy(), labels.cpu().numpy(), 0.5, 0.5, 1.0)
    # against autograd, in 64 bits
    z = student.double().requires_grad_()
    q = torch.softmax(logp.double(), 1)
    want = 0.5 * (q * (q.log() - torch.log_softmax(z, 1).gather(1, ids))).sum(1) + 0.5 * torch.nn.functional.cross_entropy(z, labels, reduction="none")
    want.sum().backward()
    assert torch.allclose(loss.double(), want.detach(), rtol=1e-5, atol=1e-5)
    assert torch.allclose(grad.double(), z.grad, rtol=2.0 ** -8, atol=1e-6)


@pytest.mark.parametrize("rows,classes", [(3, 1000), (4, 90001), (600, 5000)])
def test_same_bits_on_other_streams_and_in_graphs(rows, classes):
    rng = np.random.default_rng(classes)
    z = rows_of(rng, rows, classes, "bf16")
    ids, t, labels = [torch.from_numpy(a).cuda() for a in teacher_of(rng, rows, classes, 20, absent=True)]
    kw = dict(teacher_weight=0.5, label_weight=0.5, temperature=2.0)

    def all_of_them():
        first = B.logprobs(z, labels, top=20)
        second = B.distill(z, ids, t, labels, grad=True, **kw)
        return [*first, *second, B.distill_backward(z, second[1], ids, t, labels, **kw)]

    same = lambda got, want: all(same_bits(g, w) for g, w in zip(got, want))  # noqa: E731
    want = all_of_them()
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(3):
        for s in side:
            with torch.cuda.stream(s):
                got.append(all_of_them())
    torch.cuda.synchronize()
    assert all(same(g, want) for g in got)
    graphs = []
    for s in side:
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                graphs.append((g, all_of_them()))
    torch.cuda.synchronize()
    for again in range(3):
        for g, out in graphs:
            for o in out:
                o.view(torch.int8).fill_(again)
            with torch.cuda.stream(side[again % 2]):
                g.replay()
            eager = all_of_them()
            torch.cuda.synchronize()
            assert same(out, want) and same(eager, want)


def test_rows_beyond_two_to_the_31_elements():
    """The last rows of a tensor of more than 2^31 elements."""
    classes, rows = 131072, 16400
    z = torch.zeros((rows, classes), dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(2)
    picked = [0, 1, rows - 2, rows - 1]
    for r in picked:
        z[r] = torch.from_numpy((2.5 * rng.standard_normal(classes)).astype(np.float32)).cuda()
    labels = rng.integers(0, classes, rows)
    check = z[picked]
    got = B.logprobs(z, torch.from_numpy(labels).cuda(), top=7)
    want = B.logprobs(check, torch.from_numpy(labels[picked]).cuda(), top=7)
    for g, w in zip(got, want):
        assert torch.allclose(g[picked], w, rtol=1e-5)
    ids, t, lab = [torch.from_numpy(a).cuda() for a in teacher_of(rng, 4, classes, 5)]
    many = [torch.zeros((rows,) + tuple(a.shape[1:]), dtype=a.dtype, device="cuda") for a in (ids, t, lab)]
    for m, a in zip(many, (ids, t, lab)):
        m[picked] = a
    got = B.distill(z, *many, label_weight=0.5, grad=z)
    want = B.distill(check, ids, t, lab, label_weight=0.5, grad=True)
    for g, w in zip(got, want):
        assert torch.allclose(g[picked].float(), w.float(), rtol=2.0 ** -7 if g.dtype == torch.bfloat16 else 1e-5, atol=1e-12)


def test_with_and_without_the_calls_extension(monkeypatch):
    """Both ways of marshalling: the same outputs, and their layouts too."""
    if B._calls is None:
        pytest.skip("the extension is not built")
    rng = np.random.default_rng(8)
    z = rows_of(rng, 5, 1003, "bf16", pad=3)
    ids, t, labels = [torch.from_numpy(a).cuda() for a in teacher_of(rng, 5, 1003, 20, absent=True)]
    up = torch.rand(5, device="cuda")

    def every():
        kw = dict(teacher_weight=2, label_weight=0.5, temperature=2.0)
        loss, stats, grad = B.distill(z, ids, t, labels, grad=True, grad_loss=up, **kw)
        into = torch.zeros_like(grad)
        assert B.distill(z, ids, t, labels, grad=into, **kw)[2] is into and B.distill_backward(z, stats, ids, t, labels, grad=into, grad_loss=up, **kw) is into
        return [*B.logprobs(z, labels, top=7, temperature=2), *B.logprobs(z, ids, entropy=False)[:1], loss, stats, grad, into,
                B.distill(z, None, None, labels, teacher_weight=0.0, label_weight=1.0)[0], B.distill_backward(z, stats, ids, t, labels, **kw)]

    want = every()
    assert B.distill(z, ids, t)[2] is None and B.distill(z, ids, t, grad=False)[2] is None
    calls = B._calls
    monkeypatch.setattr(B, "_calls", None)
    for w, g in zip(want, every()):
        assert w.shape == g.shape and w.stride() == g.stride() and w.dtype == g.dtype and same_bits(w, g)
    # the small outputs of a call share a block of memory and nothing else
    monkeypatch.setattr(B, "_calls", calls)
    with torch.inference_mode():
        assert all(o.is_inference() for o in B.logprobs(z, labels, top=7))
    outs = [*B.logprobs(z, labels, top=7), *B.distill(z, ids, t)[:2]]
    copies = [o.clone() for o in outs]
    for o, c in zip(outs, copies):
        o.fill_(3)
        assert all(same_bits(x, y) or x is o for x, y in zip(outs, copies))
        o.copy_(c)
    # what the extension leaves to Python
    assert calls.logprobs(z, labels, 2000, 1.0, True) is None and calls.logprobs(z.half(), None, 0, 1.0, True) is None
    assert calls.logprobs(z, labels.int(), 0, 1.0, True) is None and calls.logprobs(z.t(), None, 0, 1.0, True) is None
    assert isinstance(calls.logprobs(z, None, 0, -1.0, True), int)
    assert calls.distill(z, None, ids, t[:4], labels, 1.0, 0.0, 1.0, None, None) is None
    assert calls.distill(z, None, ids, t, None, 1.0, 0.0, "1", None, None) is None


def test_refusals_on_the_gpu():
    z = torch.zeros((4, 100), device="cuda")
    i64 = lambda *s: torch.zeros(s, dtype=torch.int64, device="cuda")  # noqa: E731
    f32 = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    bad = [lambda: B.logprobs(z.half()), lambda: B.logprobs(z[0]), lambda: B.logprobs(z.t()), lambda: B.logprobs(z, top=101), lambda: B.logprobs(z, top=-1),
           lambda: B.logprobs(z, i64(3)), lambda: B.logprobs(z, f32(4)), lambda: B.logprobs(z, i64(4).cpu()), lambda: B.logprobs(z, temperature=0.0),
           lambda: B.logprobs(z, temperature=NAN), lambda: B.logprobs(z, i64(4, 6)[:, ::2]), lambda: B.logprobs(torch.zeros((4, 500), device="cuda"), top=129),
           lambda: B.distill(z, i64(4, 3), None), lambda: B.distill(z, i64(4, 3), f32(4, 2)), lambda: B.distill(z, i64(3, 3), f32(3, 3)),
           lambda: B.distill(z, i64(4, 129), f32(4, 129)), lambda: B.distill(z, i64(4, 3), f32(4, 3), label_weight=1.0),
           lambda: B.distill(z, None, None), lambda: B.distill(z, i64(4, 3), f32(4, 3), teacher_weight=INF),
           lambda: B.distill(z, i64(4, 3), f32(4, 3), grad=f32(4, 99)), lambda: B.distill(z, i64(4, 3), f32(4, 3), grad=f32(1, 100).expand(4, 100)),
           lambda: B.distill(z, i64(4, 3), f32(4, 3), grad=True, grad_loss=f32(3)),
           lambda: B.distill_backward(z, f32(4, 2), i64(4, 3), f32(4, 3)), lambda: B.distill_backward(z, f32(4, 3), i64(4, 3), f32(4, 3), temperature=-1.0)]
    for k, call in enumerate(bad):
        with pytest.raises(B.CGError):
            call()
            pytest.fail("call %d was taken" % k)
