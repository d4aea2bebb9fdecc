"""The operators behind the classifier in 64 bits (numpy), from their definitions, each value with a bound on what 32-bit arithmetic may add.

The bounds count roundings of U = 2^-24, the half step of a 32-bit number.  With y = (z - m) / T the kernels round the difference, 1 / T and the product
(3 U |y|), scale by log2 e for the exponential (U |y| more, the constant's own rounding U |y|; v_exp_f32 and its like add a few U), and add terms in an
order in which no term passes more than V / 64 + 24 additions (at least 64 lanes share a row, whose sums meet pairwise, and segments of a row number
fewer than the terms that they spare a lane)."""
import numpy as np

U = 2.0 ** -24


def chain(classes):
    return classes / 64 + 24


def softmax_parts(z, temperature):
    """z float64 [V], some of it finite: y, p, log of the sum, and the bound on the error of a log probability's sum and of p, relative."""
    y = (z - z.max()) / temperature
    e = np.exp(y)
    s = e.sum()
    p = e / s
    ay = np.where(p > 0, np.abs(y), 0.0)
    # the sum, relative: its additions, and the errors of its terms weighted by their share
    sum_error = U * (chain(len(z)) + 4 + 6 * (p * ay).sum())
    return y, p, np.log(s), sum_error


def rank(z, top):
    """The `top` first classes by falling logit, equal ones by index."""
    return np.argsort(-z, kind="stable")[:top]


def logprobs(z, labels, top, temperature):
    """One row: dict of (value, bound) of logprob and entropy, top_ids, and (value, bound) of top_logprobs."""
    z = z.astype(np.float64)
    classes = len(z)
    labels = np.asarray(labels, np.int64)
    inside = (labels >= 0) & (labels < classes)
    if np.isnan(z).any() or (z == np.inf).any():
        nan = np.full(top, np.nan)
        return dict(logprob=(np.where(labels < 0, 0.0, np.nan), np.zeros(len(labels))), entropy=(np.nan, 0.0), top_ids=np.full(top, -1),
                    top_logprobs=(nan, np.zeros(top)))
    if (z == -np.inf).all():
        logp, bound, entropy, entropy_bound = np.full(classes, -np.inf), np.zeros(classes), 0.0, 0.0
    else:
        y, p, log_sum, sum_error = softmax_parts(z, temperature)
        ay = np.where(np.isfinite(y), np.abs(y), 0.0)
        logp = y - log_sum
        bound = sum_error + U * (4 * ay + 4 * abs(log_sum) + 4)
        held = p > 0
        entropy = -(p[held] * logp[held]).sum()
        a, b = (p[held] * ay[held]).sum(), (p[held] * ay[held] ** 2).sum()
        # log of the sum, and the moment over the sum: its additions, the division, its terms' errors
        entropy_bound = sum_error * (1 + a) + U * (4 * abs(log_sum) + 4 + (chain(classes) + 8) * a + 6 * b)
    ids = rank(z, top)
    safe = np.where(inside, labels, 0)
    return dict(logprob=(np.where(labels < 0, 0.0, np.where(inside, logp[safe], np.nan)), np.where(inside, bound[safe], 0.0)),
                entropy=(entropy, entropy_bound), top_ids=ids, top_logprobs=(logp[ids], bound[ids]))


def distill(z, top_ids, top_logits, label, teacher_weight, label_weight, temperature, up=1.0):
    """One row: ((loss, bound), (gradient, bound))."""
    z = z.astype(np.float64)
    classes = len(z)
    ids, t = np.asarray(top_ids, np.int64), np.asarray(top_logits).astype(np.float64)
    here = ids >= 0
    t = np.where(here, t, -np.inf)
    beyond = (ids >= classes).any()
    finite_teacher = here.any() and not (t[here] == -np.inf).all()
    taught = teacher_weight != 0 and (finite_teacher or beyond)
    labelled = label_weight != 0 and label >= 0
    zero = ((0.0, 0.0), (np.zeros(classes), np.zeros(classes)))
    if (z == -np.inf).all() or not (taught or labelled):
        return zero
    if (taught and (beyond or np.isnan(t[here]).any() or (t == np.inf).any())) or (labelled and label >= classes) or np.isnan(z).any() or (z == np.inf).any():
        return (np.nan, 0.0), (np.full(classes, np.nan), np.zeros(classes))
    loss = loss_bound = 0.0
    grad, grad_bound = np.zeros(classes), np.zeros(classes)
    if taught:
        ty = (t - t.max()) / temperature
        q = np.exp(ty)
        mass = q.sum()
        q = q / mass
        aty = np.where(np.isfinite(ty), np.abs(ty), 0.0)
        q_error = U * (6 * aty + 16 + 6 * (q * aty).sum())                     # relative
        y, p, log_sum, sum_error = softmax_parts(z, temperature)
        ay = np.where(np.isfinite(y), np.abs(y), 0.0)
        at = np.where(here, ids, 0)
        with np.errstate(invalid="ignore"):
            each = np.where(q > 0, ty - np.log(mass) - (y[at] - log_sum), 0.0)
        loss += teacher_weight * (q[q > 0] * each[q > 0]).sum()
        each_error = sum_error + U * (4 * ay[at] + 4 * abs(log_sum) + 4 * aty + 4 * abs(np.log(mass)) + 16) + q_error * np.where(np.isfinite(each), abs(each), 0.0)
        loss_bound += abs(teacher_weight) * (q * (each_error + 10 * U * np.where(np.isfinite(each), abs(each), 0.0))).sum()
        c = up * teacher_weight / temperature
        grad += c * p
        np.subtract.at(grad, at, c * q)
        grad_bound += abs(c) * p * (sum_error + U * (6 * ay + 12))
        np.add.at(grad_bound, at, abs(c) * q * (q_error + 136 * U))            # (up to 128 entries name one class)
    if labelled:
        y, p, log_sum, sum_error = softmax_parts(z, 1.0)
        ay = np.where(np.isfinite(y), np.abs(y), 0.0)
        loss += label_weight * (log_sum - y[label])
        loss_bound += abs(label_weight) * (sum_error + U * (4 * ay[label] + 4 * abs(log_sum) + 8))
        c = up * label_weight
        grad += c * p
        grad[label] -= c
        grad_bound += abs(c) * p * (sum_error + U * (6 * ay + 12))
        grad_bound[label] += 4 * U * abs(c)
    grad_bound += 2.0 ** -126                                                   # (denormal numbers may come out as 0)
    return (loss, loss_bound + 4 * U * abs(loss) if np.isfinite(loss) else 0.0), (grad, grad_bound)


def rounded(bound, value, dtype_bytes):
    """The bound of a value that is rounded to bf16 at the end as well: half a step, 2^-8 of it."""
    return bound + (2.0 ** -8 * (np.abs(value) + bound) if dtype_bytes == 2 else 0.0)


def check(got, value, bound, what):
    """got (float32 and the like) against value +- bound; NaN and infinities have to be the same (values beyond float32 are infinities of it)."""
    got, value, bound = np.asarray(got, np.float64), np.asarray(value, np.float64), np.asarray(bound, np.float64)
    value = np.where(np.abs(value) >= 2.0 ** 128, np.copysign(np.inf, value), value)
    assert got.shape == value.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(value)), what + ": NaN in other places"
    infinite = np.isinf(value)
    assert np.array_equal(got[infinite], value[infinite]), what + ": infinities"
    fine = np.isfinite(value)
    off = np.abs(got[fine] - value[fine])
    over = off > np.broadcast_to(bound, value.shape)[fine]
    assert not over.any(), "%s: off by %.3g where %.3g is allowed" % (what, off[over].max(), np.broadcast_to(bound, value.shape)[fine][over][off[over].argmax()])
