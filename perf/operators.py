"""What is done with a network's logits: log probabilities with entropy and top alternatives, and the
distillation loss from a teacher's top logits with its gradient, as cases that can be timed.

A case is a dict of plain values.  `listed()` gives the fixed ones, `draw(rng)` one more from the same
ranges, `prepare(case, seed)` what a program holds before the call, `run(state)` one pass through an operator,
`work(case)` the bytes and operations the pass cannot do without and `exact(case, seed)` its outputs from
the definition in 64 bits.  Where `own` is false `run` computes the operators from elementary torch operations
in 32 bits, where it is true it calls the library.

Logits are normal with a spread of 2.5 and an offset per row; a teacher's classes stand out in the
student's row as they do in a half-trained network.  `masked` is the share of the classes that are ruled out
(-inf), `pad` the elements between rows.
"""
import math

import torch

own = False

_DTYPES = {"f32": (torch.float32, 4), "bf16": (torch.bfloat16, 2)}


def _logprobs(name, rows, classes, dtype, **kw):
    case = dict(kind="logprobs", name=name, rows=rows, classes=classes, dtype=dtype, pad=0, given=1, top=0, temperature=1.0, masked=0.0)
    case.update(kw)
    return case


def _distill(name, rows, classes, dtype, mode, **kw):
    case = dict(kind="distill", name=name, rows=rows, classes=classes, dtype=dtype, mode=mode, pad=0, top=16, temperature=1.0,
                teacher_weight=0.5, label_weight=0.5, absent=False)
    case.update(kw)
    return case


def listed():
    return [
        # one image's answer: the classifier's own logits, its label and the five best classes
        _logprobs("answer 1x1000 f32", 1, 1000, "f32", top=5),
        # an evaluation batch of the benchmark's network: top-1 / top-5 errors, entropies
        _logprobs("answers 256x1000 f32", 256, 1000, "f32", top=5),
        # one token of a language model, with its alternatives, at a sampling temperature
        _logprobs("token 1x131072 bf16", 1, 131072, "bf16", top=20, temperature=0.7),
        # a decoding batch: an odd vocabulary in padded rows, some of it ruled out, several candidates each
        _logprobs("tokens 48x130077 bf16", 48, 130077, "bf16", pad=3, given=4, top=20, masked=0.1),
        # a prompt scored: every token's log probability, odd rows without gaps
        _logprobs("prompt 2048x50003 bf16", 2048, 50003, "bf16"),
        # a teacher's top classes written down for training
        _logprobs("teacher 4096x131072 bf16", 4096, 131072, "bf16", given=0, top=64),
        # the training step of the method's classifier: both terms at equal weight, no temperature
        _distill("step 128x1000 f32", 128, 1000, "f32", "step"),
        # the loss alone, as in validation, at a temperature: two softmaxes of one row
        _distill("validation 512x32768 bf16", 512, 32768, "bf16", "forward", temperature=2.0, top=32),
        # few rows of a large vocabulary: the row has to be shared out
        _distill("step 7x200003 f32", 7, 200003, "f32", "step", temperature=2.0, top=64),
        # forward, later backward with what came from above: ragged teacher lists, rows without a label, odd rows
        _distill("pair 1024x50003 bf16", 1024, 50003, "bf16", "pair", absent=True, top=50),
        # the same in 32 bits, at a temperature
        _distill("pair 2048x32000 f32", 2048, 32000, "f32", "pair", temperature=2.0, label_weight=0.3, teacher_weight=2.8),
        # a training step over a large vocabulary: loss and gradient in one call
        _distill("step 4096x131072 bf16", 4096, 131072, "bf16", "step", top=64, label_weight=0.0, teacher_weight=1.0),
    ]


def _spread(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16", "bf16"])
    classes = _spread(rng, 2, 200003)
    rows = _spread(rng, 1, min(8192, (1 << 29) // _DTYPES[dtype][1] // classes))
    kw = dict(pad=rng.choice([0, 0, 1, 5, 16]), temperature=rng.choice([1.0, 1.0, 0.7, 2.0, 3.5]))
    if rng.random() < 0.5:
        case = _logprobs("", rows, classes, dtype, given=rng.choice([0, 1, 1, 3]), top=min(rng.choice([0, 1, 5, 20, 64, 128]), classes),
                         masked=rng.choice([0.0, 0.0, 0.3, 0.9]), **kw)
    else:
        case = _distill("", rows, classes, dtype, rng.choice(["forward", "step", "step", "pair"]), top=min(_spread(rng, 1, 128), classes),
                        teacher_weight=rng.choice([1.0, 0.5, 4.0]), label_weight=rng.choice([0.0, 0.5, 1.0]), absent=rng.random() < 0.5, **kw)
    del case["name"]
    return case


def prepare(case, seed):
    rows, classes, top = case["rows"], case["classes"], case["top"]
    dtype = _DTYPES[case["dtype"]][0]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.randn(rows, classes + case["pad"], device="cuda", generator=g)
    z.mul_(2.5).add_(4.0 * torch.randn(rows, 1, device="cuda", generator=g))
    s = dict(case)
    if case["kind"] == "logprobs":
        if case["masked"]:
            z.masked_fill_(torch.rand(z.shape, device="cuda", generator=g) < case["masked"], -math.inf)
        s["labels"] = torch.randint(0, classes, (rows, case["given"]), device="cuda", generator=g) if case["given"] else None
        s["logits"] = z.to(dtype)[:, :classes]
        return s
    # the teacher's classes: all different, spread over the row; its first ones are the likeliest
    first = torch.randint(0, classes, (rows, 1), device="cuda", generator=g)
    ids = (first + torch.arange(top, device="cuda") * max(1, classes // top)) % classes
    order = torch.arange(top, device="cuda", dtype=torch.float32)
    z.scatter_add_(1, ids, (10.0 - 0.1 * order).expand(rows, top).contiguous())
    s["top_logits"] = 12.0 - 0.15 * order + torch.randn(rows, top, device="cuda", generator=g)
    s["labels"] = ids[:, 0].clone()
    s["logits"] = z.to(dtype)[:, :classes]
    if case["absent"]:
        held = torch.randint(0, top + 1, (rows, 1), device="cuda", generator=g)
        ids = torch.where(torch.arange(top, device="cuda") < held, ids, -1)
        s["labels"][torch.rand(rows, device="cuda", generator=g) < 0.25] = -100
    s["top_ids"] = ids
    s["grad_loss"] = torch.rand(rows, device="cuda", generator=g) / rows
    return s


def _weights(s):
    return dict(temperature=s["temperature"], teacher_weight=s["teacher_weight"], label_weight=s["label_weight"])


def run(s):
    if own:
        from paper_1805_12549_amd import binding as B
        if s["kind"] == "logprobs":
            logprob, entropy, top_ids, top_logprobs = B.logprobs(s["logits"], s["labels"], top=s["top"], temperature=s["temperature"])
            return dict(logprob=logprob, entropy=entropy, top_ids=top_ids, top_logprobs=top_logprobs)
        teacher = (s["top_ids"], s["top_logits"], s["labels"])
        if s["mode"] == "forward":
            return dict(loss=B.distill(s["logits"], *teacher, **_weights(s))[0])
        if s["mode"] == "step":
            loss, _, grad = B.distill(s["logits"], *teacher, grad=True, grad_loss=s["grad_loss"], **_weights(s))
            return dict(loss=loss, grad=grad)
        loss, stats, _ = B.distill(s["logits"], *teacher, **_weights(s))
        return dict(loss=loss, grad=B.distill_backward(s["logits"], stats, *teacher, grad_loss=s["grad_loss"], **_weights(s)))
    return _plain_logprobs(s) if s["kind"] == "logprobs" else _plain_distill(s)


def _softmax_parts(z, temperature):
    """Per row: (z - max) / temperature, its exponential and the logarithm of that one's sum."""
    most = z.amax(1, keepdim=True)
    y = (z - torch.where(most == -math.inf, 0.0, most)) / temperature
    e = torch.exp(y)
    return y, e, torch.log(e.sum(1, keepdim=True))


def _plain_logprobs(s):
    z = s["logits"].float()
    y, e, log_sum = _softmax_parts(z, s["temperature"])
    some = torch.isfinite(log_sum)
    out = dict(logprob=None, top_ids=None, top_logprobs=None)
    out["entropy"] = torch.where(some, log_sum - torch.where(e > 0, e * y, 0.0).sum(1, keepdim=True) / torch.exp(log_sum), 0.0)[:, 0]
    if s["labels"] is not None:
        out["logprob"] = torch.where(some, y.gather(1, s["labels"]) - log_sum, -math.inf)
    if s["top"]:
        # keys that order like the logits and, where those are equal, by index
        bits = (z + 0.0).view(torch.int32).to(torch.int64)
        bits = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
        keys = bits * (1 << 32) - torch.arange(z.shape[1], device=z.device)
        out["top_ids"] = -keys.topk(s["top"], dim=1, sorted=True).values % (1 << 32)
        out["top_logprobs"] = torch.where(some, y.gather(1, out["top_ids"]) - log_sum, -math.inf)
    return out


def _plain_distill(s):
    z, temperature = s["logits"].float(), s["temperature"]
    classes = z.shape[1]
    # the teacher's distribution over its classes
    held = s["top_ids"] >= 0
    ids = s["top_ids"].clamp(min=0)
    t = torch.where(held, s["top_logits"], -math.inf)
    most = t.amax(1, keepdim=True)
    t = (t - torch.where(most == -math.inf, 0.0, most)) / temperature
    q = torch.exp(t)
    mass = q.sum(1, keepdim=True)
    any_q = mass > 0
    mass = torch.where(any_q, mass, 1.0)
    q = q / mass
    labelled = (s["labels"] >= 0).unsqueeze(1)
    label = s["labels"].clamp(min=0).unsqueeze(1)
    # loss
    y, e, log_sum = _softmax_parts(z, temperature)
    soft = torch.where(q > 0, q * ((t - torch.log(mass)) - (y.gather(1, ids) - log_sum)), 0.0).sum(1)
    y1, e1, log_sum1 = (y, e, log_sum) if temperature == 1.0 else _softmax_parts(z, 1.0)
    hard = torch.where(labelled, log_sum1 - y1.gather(1, label), 0.0)[:, 0]
    out = dict(loss=s["label_weight"] * hard + s["teacher_weight"] * soft)
    if s["mode"] == "forward":
        return out
    # gradient
    up = s["grad_loss"].unsqueeze(1)
    wt = torch.where(any_q, up * (s["teacher_weight"] / temperature), 0.0)
    wl = torch.where(labelled, up * s["label_weight"], 0.0)
    grad = e * (wt / torch.exp(log_sum)) + e1 * (wl / torch.exp(log_sum1))
    grad.scatter_add_(1, ids, -wt * q)
    grad.scatter_add_(1, label, -wl)
    out["grad"] = grad.to(s["logits"].dtype)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    rows, classes = s["logits"].shape
    parts = []
    step = max(1, (1 << 26) // classes)          # rows at a time
    for r in range(0, rows, step):
        one = {k: v[r:r + step] if isinstance(v, torch.Tensor) else v for k, v in s.items()}
        parts.append(_exact_logprobs(one) if case["kind"] == "logprobs" else _exact_distill(one))
    return {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_logprobs(s):
    z = s["logits"].double()
    logp = z / s["temperature"]
    logp = logp - torch.logsumexp(logp, 1, keepdim=True)
    logp[(z == -math.inf).all(1)] = -math.inf
    out = dict(entropy=-torch.special.xlogy(logp.exp(), logp.exp()).sum(1), logprob=None, top_ids=None, top_logprobs=None)
    if s["labels"] is not None:
        out["logprob"] = logp.gather(1, s["labels"])
    if s["top"]:
        out["top_ids"] = z.sort(dim=1, descending=True, stable=True).indices[:, :s["top"]]
        out["top_logprobs"] = logp.gather(1, out["top_ids"])
    return out


def _exact_distill(s):
    z, k = s["logits"].double(), s["temperature"]
    n, classes = z.shape
    row = torch.arange(n, device=z.device)
    # the teacher's distribution over all classes, and one for the label
    q = torch.zeros_like(z)
    for j in range(s["top_ids"].shape[1]):
        at = s["top_ids"][:, j]
        weight = torch.exp((s["top_logits"][:, j].double() - s["top_logits"].double().amax(1)) / k)
        q.index_put_((row, at.clamp(min=0)), torch.where(at >= 0, weight, 0.0), accumulate=True)
    mass = q.sum(1, keepdim=True)
    q = q / torch.where(mass > 0, mass, 1.0)
    one = torch.zeros_like(z)
    one[row, s["labels"].clamp(min=0)] = (s["labels"] >= 0).double()
    logp, logp1 = torch.log_softmax(z / k, 1), torch.log_softmax(z, 1)
    loss = s["teacher_weight"] * (torch.special.xlogy(q, q) - q * logp).sum(1) - s["label_weight"] * (one * logp1).sum(1)
    if s["mode"] == "forward":
        return dict(loss=loss)
    grad = s["teacher_weight"] / k * (logp.exp() * q.sum(1, keepdim=True) - q) + s["label_weight"] * (logp1.exp() * one.sum(1, keepdim=True) - one)
    return dict(loss=loss, grad=grad * s["grad_loss"].double().unsqueeze(1))


def work(case):
    rows, classes, top, size = case["rows"], case["classes"], case["top"], _DTYPES[case["dtype"]][1]
    n = rows * classes
    if case["kind"] == "logprobs":
        # difference, exponential, sum; product and sum of the entropy
        return dict(bytes=n * size + rows * (12 * case["given"] + 4 + 12 * top), flops=5 * n)
    sums = 2 if case["temperature"] != 1.0 and case["label_weight"] else 1
    forward = rows * (12 * top + 8 + 4)
    if case["mode"] == "forward":
        return dict(bytes=n * size + forward, flops=3 * n * sums)
    # a gradient's element: an exponential again, a product with the row's factor, a sum of the two terms
    reads = 2 if case["mode"] == "pair" else 1
    return dict(bytes=(reads + 1) * n * size + reads * forward + 4 * rows, flops=n * sums * 6)
