"""Losses over a vocabulary, as cases to measure: the softmax layer with its cross-entropy and all
gradients without keeping the logits, the largest logits of a row (a teacher's side of
distillation), and distillation from them.

``run`` computes a case in its plain form (elementary torch operations in 32 bits, one rounding at
the end) or, with ``own`` set, through ``paper_1909_09010_b200.binding``.  ``exact`` gives the same
outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
IGNORE = -100


def listed():
    return [
        # how likely is this word: one word of one stream, 10,000 words: the smallest call, all latency
        dict(name="loss_one_word", op="linear_loss", dtype="bf16", rows=1, n_in=1024, vocab=10000,
             bias=True, weighted=False, grad=False),
        # scoring 8 streams with the 267,735-word softmax layer in 32 bits: one read of the table
        dict(name="loss_scores_8", op="linear_loss", dtype="f32", rows=8, n_in=512, vocab=267735,
             bias=True, weighted=False, grad=False),
        # evaluation of the 100,000-word, 1024-wide model on held-out text
        dict(name="loss_eval", op="linear_loss", dtype="bf16", rows=2048, n_in=1024, vocab=100000,
             bias=True, weighted=False, grad=False),
        # training step of that softmax layer: the largest
        dict(name="train_softmax", op="linear_loss", dtype="bf16", rows=2048, n_in=1024, vocab=100000,
             bias=True, weighted=False, grad=True),
        # training step of the 267,735-word, 512-wide softmax layer, rows weighted, odd vocabulary
        dict(name="train_267k", op="linear_loss", dtype="bf16", rows=1024, n_in=512, vocab=267735,
             bias=True, weighted=True, grad=True),
        # 32-bit training on a ragged batch and odd widths
        dict(name="train_odd_f32", op="linear_loss", dtype="f32", rows=1003, n_in=515, vocab=10007,
             bias=True, weighted=True, grad=True),
        # the next words that one stream may take, 267,735 words
        dict(name="top_one", op="top", dtype="bf16", rows=1, vocab=267735, k=16, temperature=1.0),
        # a teacher's lists for a training batch, 267,735 words
        dict(name="top_267k", op="top", dtype="bf16", rows=2048, vocab=267735, k=64, temperature=2.0),
        # the same for a 10,000-word teacher in 32 bits
        dict(name="top_10k", op="top", dtype="f32", rows=515, vocab=10000, k=32, temperature=1.0),
        # distillation of a 1,000-word model, lists that count as the whole distribution: all latency
        dict(name="distill_small", op="distill", dtype="f32", rows=64, vocab=1000, k=8, temperature=1.0,
             rest=False, hard=0.0, weighted=False),
        # distillation of the 267,735-word model, the words outside the list as one class
        dict(name="distill_267k", op="distill", dtype="bf16", rows=2048, vocab=267735, k=64,
             temperature=2.0, rest=True, hard=0.0, weighted=False),
        # soft and hard targets together, 33,278 words in 32 bits, ragged batch
        dict(name="distill_hard", op="distill", dtype="f32", rows=1003, vocab=33278, k=50,
             temperature=3.0, rest=False, hard=0.3, weighted=True),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over its logarithm: odd as it comes, or a
    multiple of 8 or 128 half of the time."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    step = rng.choice([1, 1, 8, 128])
    return min(high, max(low, (v // step) * step if v >= step else v))


def draw(rng):
    op = rng.choice(["linear_loss", "linear_loss", "top", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    rows, vocab = _spread(rng, 1, 2048), _spread(rng, 1000, 267735)
    if op == "linear_loss":
        n_in = _spread(rng, 64, 1024)
        while rows * n_in * vocab > (5e10 if dtype == "f32" else 2e11):
            rows = max(1, rows // 2)
        return dict(op=op, dtype=dtype, rows=rows, n_in=n_in, vocab=vocab, bias=rng.random() < 0.8,
                    weighted=rng.random() < 0.5, grad=rng.random() < 0.7)
    temperature = rng.choice([1.0, 1.5, 2.0, 4.0])
    if dtype == "f32":
        rows = max(1, rows // 2)
    if op == "top":
        return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, k=_spread(rng, 1, 128), temperature=temperature)
    return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, k=_spread(rng, 1, 128), temperature=temperature,
                rest=rng.random() < 0.5, hard=rng.choice([0.0, 0.0, 0.25, 0.5]), weighted=rng.random() < 0.5)


def _top_of(rows, k):
    """(values, indices) of the k largest of each row, the lower index first among equal ones."""
    bits = rows.float().view(torch.int32).to(torch.int64)
    order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)        # as the values, and whole numbers
    best = torch.topk(order * (1 << 31) - torch.arange(rows.shape[1], device=rows.device), k, dim=1).values
    index = (-best) % (1 << 31)
    return rows.gather(1, index), index


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 2654435761 % (1 << 31))
    t, n, v = DTYPES[case["dtype"]], case["rows"], case["vocab"]

    def normal(*shape, scale=1.0):
        return torch.empty(shape, dtype=t, device="cuda").normal_(0.0, scale, generator=g)

    state = dict(case=case)
    if case["op"] == "top":
        state.update(logits=normal(n, v, scale=3.0))
        return state
    targets = torch.randint(0, v, (n,), device="cuda", generator=g)
    skipped = torch.rand((n,), device="cuda", generator=g) < 0.1          # padding of ragged batches
    state.update(targets=torch.where(skipped, IGNORE, targets) if n > 1 else targets, scale=1.0 / n,
                 weight=torch.rand((n,), device="cuda", generator=g) + 0.5 if case["weighted"] else None)
    if case["op"] == "linear_loss":
        state.update(x=normal(n, case["n_in"]), w=normal(v, case["n_in"], scale=2.0 * case["n_in"] ** -0.5),
                     bias=normal(v, scale=0.5) if case["bias"] else None)
        return state
    # the student's logits are the teacher's with noise
    student = normal(n, v, scale=2.5)
    values, index, lse = [], [], []
    for a in range(0, n, 256):
        rows = student[a:a + 256].float()
        teacher = (1.2 * rows + torch.empty_like(rows).normal_(0.0, 1.5, generator=g)).to(t)
        top = _top_of(teacher, case["k"])
        values.append(top[0])
        index.append(top[1])
        lse.append(torch.logsumexp(teacher.float() / case["temperature"], 1))
    state.update(logits=student, teacher=torch.cat(values), index=torch.cat(index),
                 teacher_lse=torch.cat(lse) if case["rest"] else None)
    return state


def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)(state, case, case["op"])


def _run_own(s, case, op):
    from paper_1909_09010_b200 import binding
    ops = binding.local_ops()
    if op == "linear_loss":
        return ops.linear_cross_entropy(s["x"], s["w"], s["targets"], bias=s["bias"], ignore_index=IGNORE,
                                        row_weight=s["weight"], scale=s["scale"], want_grad=case["grad"])
    if op == "top":
        return ops.top_logits(s["logits"], case["k"], temperature=case["temperature"])
    return ops.distillation(s["logits"], s["teacher"], s["index"], teacher_lse=s["teacher_lse"],
                            temperature=case["temperature"], targets=s["targets"], hard_weight=case["hard"],
                            ignore_index=IGNORE, row_weight=s["weight"], scale=s["scale"])


def _row_weights(s):
    valid = s["targets"] != IGNORE
    weight = valid.float() * s["scale"]
    return torch.where(valid, s["targets"], 0), weight if s["weight"] is None else weight * s["weight"]


def _softmax(u):
    """(exp(u) / sum, log sum) of each row."""
    top = u.amax(1, keepdim=True)
    e = torch.exp(u - top)
    total = e.sum(1, keepdim=True)
    return e / total, (top + torch.log(total)).squeeze(1)


def _run_plain(s, case, op):
    t = DTYPES[case["dtype"]]
    if op == "top":
        x = s["logits"].to(torch.float32, copy=True)
        lse = _softmax(x / case["temperature"])[1]
        values, index = [], []
        for _ in range(case["k"]):                       # the largest one, lowest index first, is taken out
            top, at = x.max(1, keepdim=True)
            values.append(top)
            index.append(at)
            x.scatter_(1, at, -math.inf)
        return torch.cat(values, 1).to(t), torch.cat(index, 1), lse
    rows = torch.arange(case["rows"], device="cuda")
    at, weight = _row_weights(s)
    if op == "linear_loss":
        x, w = s["x"].float(), s["w"].float()
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        d, lse = _softmax(z)
        loss = weight * (lse - z[rows, at])
        if not case["grad"]:
            return loss, lse
        d[rows, at] -= 1
        d = d * weight[:, None]
        grads = ((d @ w).to(t), (d.t() @ x).to(t))
        return (loss, lse, *grads) if s["bias"] is None else (loss, lse, *grads, d.sum(0).to(t))
    T, h = case["temperature"], case["hard"]
    x, a = s["logits"].float(), s["teacher"].float() / T
    p, lse = _softmax(x / T)
    log_p = (x / T).gather(1, s["index"]) - lse[:, None]
    log_q = a - (_softmax(a)[1] if s["teacher_lse"] is None else s["teacher_lse"])[:, None]
    q = torch.exp(log_q)
    loss = (q * (log_q - log_p)).sum(1)
    d = p.clone()
    if s["teacher_lse"] is not None:
        q_rest = torch.clamp(1 - q.sum(1, dtype=torch.float64), min=0).float()
        p_rest = p.scatter(1, s["index"], 0.0).sum(1)
        loss = loss + torch.where(q_rest > 0, q_rest * (torch.log(q_rest) - torch.log(p_rest)), 0.0)
        d = d * (1 - q_rest / p_rest)[:, None]
        d.scatter_(1, s["index"], p.gather(1, s["index"]))
    d.scatter_add_(1, s["index"], -q)
    loss, d = T * T * loss, T * d
    if h > 0:
        p1, lse1 = _softmax(x)
        p1[rows, at] -= 1
        loss = (1 - h) * loss + h * (lse1 - x[rows, at])
        d = (1 - h) * d + h * p1
    return weight * loss, lse, (d * weight[:, None]).to(t)


def work(case):
    b, n, v = SIZE[case["dtype"]], case["rows"], case["vocab"]
    if case["op"] == "linear_loss":
        table = v * (case["n_in"] + case["bias"]) + n * case["n_in"]
        times = 2 if case["grad"] else 1                 # operands, and as many gradients
        return {"bytes": float(b * table * times + 20 * n), "flops": (6.0 if case["grad"] else 2.0) * n * v * case["n_in"]}
    if case["op"] == "top":
        return {"bytes": float(b * n * v + n * (case["k"] * (b + 8) + 4)), "flops": 4.0 * n * v}
    return {"bytes": float(2 * b * n * v + n * (case["k"] * (b + 8) + 24)), "flops": 6.0 * n * v}


def exact(case, seed):
    s = prepare(case, seed)
    d, op = torch.float64, case["op"]
    if op == "top":
        lse = torch.cat([torch.logsumexp(r.to(d) / case["temperature"], 1) for r in s["logits"].split(256)])
        values, index = zip(*(_top_of(r, case["k"]) for r in s["logits"].split(256)))
        return torch.cat(values).to(d), torch.cat(index), lse
    counted = s["targets"] != IGNORE
    weight = s["scale"] * counted.to(d) * (1.0 if s["weight"] is None else s["weight"].to(d))
    at = s["targets"].clamp(min=0)[:, None]
    one = torch.ones_like(at, dtype=d)
    if op == "linear_loss":
        x, w = s["x"].to(d), s["w"].to(d)
        z = torch.einsum("ni,vi->nv", x, w)
        if s["bias"] is not None:
            z += s["bias"].to(d)
        lse = torch.logsumexp(z, 1)
        loss = weight * (lse - z.gather(1, at)[:, 0])
        if not case["grad"]:
            return loss, lse
        z.sub_(lse[:, None]).exp_().scatter_add_(1, at, -one).mul_(weight[:, None])
        grads = (torch.einsum("nv,vi->ni", z, w), torch.einsum("nv,ni->vi", z, x))
        return (loss, lse, *grads) if s["bias"] is None else (loss, lse, *grads, torch.einsum("nv->v", z))
    T, h, index = case["temperature"], case["hard"], s["index"]
    losses, lses, grads = [], [], []
    for rows in torch.arange(case["rows"], device="cuda").split(256):
        x, a, ix = s["logits"][rows].to(d), s["teacher"][rows].to(d) / T, index[rows]
        lse = torch.logsumexp(x / T, 1, keepdim=True)
        log_q = torch.log_softmax(a, 1) if s["teacher_lse"] is None else a - s["teacher_lse"][rows].to(d)[:, None]
        q, log_p = log_q.exp(), (x / T).gather(1, ix) - lse
        soft = torch.sum(q * (log_q - log_p), 1)
        grad = torch.exp(x / T - lse)
        if s["teacher_lse"] is not None:
            listed_p = grad.gather(1, ix)
            q_rest = (1 - q.sum(1)).clamp(min=0)
            log_rest = torch.logsumexp((x / T).scatter(1, ix, -math.inf), 1) - lse[:, 0]
            soft += torch.special.xlogy(q_rest, q_rest) - q_rest * log_rest
            grad *= (1 - q_rest * torch.exp(-log_rest))[:, None]
            grad.scatter_(1, ix, listed_p)
        grad.scatter_add_(1, ix, -q)
        total, grad = (1 - h) * T * T * soft, (1 - h) * T * grad
        if h > 0:
            lse1 = torch.logsumexp(x, 1, keepdim=True)
            total += h * (lse1 - x.gather(1, at[rows]))[:, 0]
            grad += h * torch.exp(x - lse1)
            grad.scatter_add_(1, at[rows], -h * one[rows])
        losses.append(weight[rows] * total)
        lses.append(lse[:, 0])
        grads.append(grad.mul_(weight[rows][:, None]))
    return torch.cat(losses), torch.cat(lses), torch.cat(grads)
