"""The operators of a worker's local training step, as cases to measure: a linear layer with its
epilogue and its two gradients, the cross-entropy over a vocabulary with its gradient, and the
gradient norm and clipping over a worker's tensors.

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
        # one word of one stream through a 1024-wide layer: the smallest call, all latency
        dict(name="forward_one_token", op="forward", dtype="bf16", rows=1, n_in=1024, n_out=4096,
             act="gelu", bias=True, residual=False, keep_z=False),
        # next-word scores of 8 streams over the 267,735-word softmax table: one read of the table
        dict(name="forward_scores_8", op="forward", dtype="f32", rows=8, n_in=512, n_out=267735,
             act="none", bias=True, residual=False, keep_z=False),
        # the widening half of a 512-wide feed-forward block in training: z is kept for the gradient
        dict(name="forward_block", op="forward", dtype="bf16", rows=4096, n_in=512, n_out=2048,
             act="gelu", bias=True, residual=False, keep_z=True),
        # softmax layer of the 100,000-word, 1024-wide model over a training batch: the largest
        dict(name="forward_softmax", op="forward", dtype="bf16", rows=2048, n_in=1024, n_out=100000,
             act="none", bias=True, residual=False, keep_z=False),
        # gradient through the narrowing half of that block, with the derivative of the activation
        dict(name="input_grad_block", op="input_grad", dtype="bf16", rows=4096, n_in=2048, n_out=512,
             act="gelu", residual=False, want_dx=False),
        # 32-bit training on a ragged batch and odd widths, with the residual branch's gradient
        dict(name="input_grad_odd", op="input_grad", dtype="f32", rows=1003, n_in=515, n_out=1027,
             act="silu", residual=True, want_dx=True),
        # weight gradient of a 1024-wide block, 32-bit result as the optimiser's buffer takes it
        dict(name="weight_grad_block", op="weight_grad", dtype="bf16", grad="f32", rows=8192,
             n_in=1024, n_out=4096, bias=True),
        # the same in 32 bits throughout, 512-wide
        dict(name="weight_grad_f32", op="weight_grad", dtype="f32", grad="f32", rows=2048,
             n_in=512, n_out=2048, bias=True),
        # four workers of the 1,000-word, 128-wide two-layer model: all launch latency
        dict(name="clip_small", op="clip", dtype="f32", workers=4, vocab=1000, width=128, layers=2,
             clip=10.0, scale=0.05),
        # four workers of the 100,000-word, 1024-wide four-layer model, bf16 gradients
        dict(name="clip_large", op="clip", dtype="bf16", workers=4, vocab=100000, width=1024, layers=4,
             clip=10.0, scale=0.01),
        # loss of a 10,000-word model over a batch of 512 words in 32 bits
        dict(name="loss_10k", op="loss", dtype="f32", rows=512, vocab=10000, weighted=False),
        # loss of the 267,735-word model over a training batch, rows weighted
        dict(name="loss_267k", op="loss", dtype="bf16", rows=2048, vocab=267735, weighted=True),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over its logarithm: odd as it comes, or a
    multiple of 8 or 128 half of the time."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    step = rng.choice([1, 1, 8, 128])
    return min(high, max(low, (v // step) * step if v >= step else v))


def draw(rng):
    op = rng.choice(["forward", "forward", "input_grad", "weight_grad", "clip", "loss"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    act = rng.choice(["none", "relu", "gelu", "silu", "tanh", "sigmoid"])
    if op in ("forward", "input_grad", "weight_grad"):
        rows, n_in, n_out = _spread(rng, 1, 8192), _spread(rng, 64, 4096), _spread(rng, 64, 4096)
        if op == "forward" and rng.random() < 0.25:          # a softmax layer
            rows, n_in, n_out = _spread(rng, 1, 1024), _spread(rng, 128, 1024), _spread(rng, 10000, 267735)
        if op == "forward":
            return dict(op=op, dtype=dtype, rows=rows, n_in=n_in, n_out=n_out, act=act,
                        bias=rng.random() < 0.8, residual=rng.random() < 0.3, keep_z=rng.random() < 0.5)
        if op == "input_grad":
            return dict(op=op, dtype=dtype, rows=rows, n_in=n_in, n_out=n_out, act=act,
                        residual=rng.random() < 0.5, want_dx=rng.random() < 0.5)
        return dict(op=op, dtype=dtype, grad=rng.choice(["f32", dtype]), rows=rows, n_in=n_in,
                    n_out=n_out, bias=rng.random() < 0.8)
    if op == "clip":
        return dict(op=op, dtype=dtype, workers=rng.randint(1, 8), vocab=_spread(rng, 1000, 50000),
                    width=_spread(rng, 64, 1024), layers=rng.randint(1, 4), clip=10.0,
                    scale=rng.choice([0.05, 0.01, 1e-6]))
    return dict(op=op, dtype=dtype, rows=_spread(rng, 1, 2048), vocab=_spread(rng, 1000, 267735),
                weighted=rng.random() < 0.5)


def _tensors(case):
    """Shapes of one worker's tensors: embedding, per layer two gate matrices and a bias, softmax."""
    v, h = case["vocab"], case["width"]
    shapes = [(v, h)]
    for _ in range(case["layers"]):
        shapes += [(4 * h, h), (4 * h, h), (4 * h,)]
    return shapes + [(v, h), (v,)]


def _row_length(case):
    n = sum(math.prod(s) for s in _tensors(case))
    return n, (n + 31) // 32 * 32


def _make(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 2654435761 % (1 << 31))
    t = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.empty(shape, dtype=t, device="cuda").normal_(0.0, scale, generator=g)

    op = case["op"]
    if op == "forward":
        n, i, o = case["rows"], case["n_in"], case["n_out"]
        return dict(x=normal(n, i), w=normal(o, i, scale=i ** -0.5),
                    bias=normal(o, scale=0.1) if case["bias"] else None,
                    residual=normal(n, o) if case["residual"] else None)
    if op == "input_grad":
        n, i, o = case["rows"], case["n_in"], case["n_out"]
        return dict(dz=normal(n, o, scale=1e-3), w=normal(o, i, scale=i ** -0.5), z=normal(n, i),
                    residual=normal(n, i, scale=1e-3) if case["residual"] else None)
    if op == "weight_grad":
        n, i, o = case["rows"], case["n_in"], case["n_out"]
        return dict(dz=normal(n, o, scale=1e-3), x=normal(n, i))
    if op == "clip":
        return dict(grads=[[normal(*s, scale=case["scale"] * (1.0 + 0.25 * k)) for s in _tensors(case)]
                           for k in range(case["workers"])])
    n, v = case["rows"], case["vocab"]
    targets = torch.randint(0, v, (n,), device="cuda", generator=g)
    skipped = torch.rand((n,), device="cuda", generator=g) < 0.1          # padding of ragged batches
    targets = torch.where(skipped, IGNORE, targets)
    weight = torch.rand((n,), device="cuda", generator=g) + 0.5 if case["weighted"] else None
    return dict(logits=normal(n, v, scale=2.0), targets=targets, weight=weight, scale=1.0 / n)


def prepare(case, seed):
    state = _make(case, seed)
    state["case"] = case
    if case["op"] == "clip":
        # the optimiser's gradient buffer [workers][ld]: every worker's tensors one after another
        n, ld = _row_length(case)
        state["flat"] = torch.zeros((case["workers"], ld), device="cuda")
        if own:
            from paper_1909_09010_b200 import binding
            entries = []
            for k, tensors in enumerate(state["grads"]):
                at = 0
                for t in tensors:
                    entries.append((t, state["flat"][k, at:at + t.numel()].view(t.shape), k))
                    at += t.numel()
            state["plan"] = binding.GradClip(entries, groups=case["workers"])
    return state


def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)(state, case, case["op"])


def _run_own(s, case, op):
    from paper_1909_09010_b200 import binding
    if op == "clip":
        return dict(norms=s["plan"].clip(case["clip"]), flat=s["flat"])
    ops = binding.local_ops()
    if op == "forward":
        return ops.linear_forward(s["x"], s["w"], bias=s["bias"], residual=s["residual"],
                                  activation=case["act"], keep_z=case["keep_z"])
    if op == "input_grad":
        return ops.linear_backward_input(s["dz"], s["w"], residual=s["residual"], z_prev=s["z"],
                                         activation=case["act"], want_dx=case["want_dx"])
    if op == "weight_grad":
        return ops.linear_backward_weight(s["dz"], s["x"], grad_dtype=DTYPES[case["grad"]],
                                          want_bias=case["bias"])
    return ops.cross_entropy(s["logits"], s["targets"], ignore_index=IGNORE, row_weight=s["weight"],
                             scale=s["scale"])


def _act(z, name):
    if name == "none":
        return z
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.7071067811865476))
    if name == "silu":
        return z * torch.sigmoid(z)
    return torch.tanh(z) if name == "tanh" else torch.sigmoid(z)


def _act_grad(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.7071067811865476)) + z * torch.exp(-0.5 * z * z) * 0.3989422804014327
    if name == "tanh":
        return 1 - torch.tanh(z) ** 2
    s = torch.sigmoid(z)
    return s * (1 - s) if name == "sigmoid" else s * (1 + z * (1 - s))


def _run_plain(s, case, op):
    t = DTYPES[case["dtype"]]
    if op == "forward":
        z = s["x"].float() @ s["w"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return (y.to(t), z.to(t)) if case["keep_z"] else y.to(t)
    if op == "input_grad":
        dx = s["dz"].float() @ s["w"].float()
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        dzp = dx * _act_grad(s["z"].float(), case["act"])
        return (dx.to(t), dzp.to(t)) if case["want_dx"] else dzp.to(t)
    if op == "weight_grad":
        dz = s["dz"].float()
        dw = (dz.t() @ s["x"].float()).to(DTYPES[case["grad"]])
        return (dw, dz.sum(0).to(DTYPES[case["grad"]])) if case["bias"] else dw
    if op == "clip":
        norms = []
        for k, tensors in enumerate(s["grads"]):
            row = torch.cat([g.reshape(-1) for g in tensors]).float()
            norm = torch.sqrt(torch.sum(row * row))
            s["flat"][k, :row.numel()] = row * (case["clip"] / torch.clamp(norm, min=case["clip"]))
            norms.append(norm)
        return dict(norms=torch.stack(norms), flat=s["flat"])
    x = s["logits"].float()
    rows = torch.arange(x.shape[0], device=x.device)
    valid = s["targets"] != IGNORE
    at = torch.where(valid, s["targets"], 0)
    weight = valid.float() * s["scale"]
    if s["weight"] is not None:
        weight = weight * s["weight"]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    loss = weight * (lse - x[rows, at])
    d = e / total
    d[rows, at] -= 1
    return loss, lse, (d * weight[:, None]).to(t)


def work(case):
    b, op = SIZE[case["dtype"]], case["op"]
    if op in ("forward", "input_grad", "weight_grad"):
        n, i, o = case["rows"], case["n_in"], case["n_out"]
        flops = 2.0 * n * i * o
        if op == "forward":
            outs = 1 + case["keep_z"] + case["residual"]
            return {"bytes": b * (n * i + o * i + n * o * outs + o * case["bias"]), "flops": flops}
        if op == "input_grad":
            outs = 2 + case["want_dx"] + case["residual"]
            return {"bytes": b * (n * o + o * i + n * i * outs), "flops": flops}
        return {"bytes": b * (n * o + n * i) + SIZE[case["grad"]] * (o * i + o * case["bias"]), "flops": flops}
    if op == "clip":
        n = _row_length(case)[0] * case["workers"]
        return {"bytes": n * (b + 4.0), "flops": 3.0 * n}
    n = case["rows"] * case["vocab"]
    return {"bytes": 2.0 * b * n + 24.0 * case["rows"], "flops": 6.0 * n}


def exact(case, seed):
    s = _make(case, seed)
    op, d = case["op"], torch.float64
    sqrt2, sqrt2pi = math.sqrt(2.0), math.sqrt(2.0 * math.pi)
    value = {"none": lambda z: z, "relu": lambda z: torch.where(z > 0, z, torch.zeros_like(z)),
             "gelu": lambda z: z * torch.special.erfc(-z / sqrt2) / 2,
             "silu": lambda z: z / (1 + torch.exp(-z)), "tanh": torch.tanh,
             "sigmoid": lambda z: 1 / (1 + torch.exp(-z))}
    slope = {"none": torch.ones_like, "relu": lambda z: torch.heaviside(z, torch.zeros_like(z)),
             "gelu": lambda z: torch.special.erfc(-z / sqrt2) / 2 + z * torch.exp(-z * z / 2) / sqrt2pi,
             "silu": lambda z: (1 + torch.exp(-z) * (1 + z)) / (1 + torch.exp(-z)) ** 2,
             "tanh": lambda z: 1 / torch.cosh(z) ** 2,
             "sigmoid": lambda z: torch.exp(-z) / (1 + torch.exp(-z)) ** 2}
    if op == "forward":
        z = torch.einsum("ni,oi->no", s["x"].to(d), s["w"].to(d))
        z = z if s["bias"] is None else z + s["bias"].to(d)[None, :]
        y = value[case["act"]](z)
        y = y if s["residual"] is None else y + s["residual"].to(d)
        return (y, z) if case["keep_z"] else y
    if op == "input_grad":
        dx = torch.einsum("no,oi->ni", s["dz"].to(d), s["w"].to(d))
        dx = dx if s["residual"] is None else dx + s["residual"].to(d)
        dzp = dx * slope[case["act"]](s["z"].to(d))
        return (dx, dzp) if case["want_dx"] else dzp
    if op == "weight_grad":
        dw = torch.einsum("no,ni->oi", s["dz"].to(d), s["x"].to(d))
        return (dw, torch.einsum("no->o", s["dz"].to(d))) if case["bias"] else dw
    if op == "clip":
        norms, (n, ld) = [], _row_length(case)
        flat = torch.zeros((case["workers"], ld), dtype=d, device="cuda")
        for k, tensors in enumerate(s["grads"]):
            norm = math.sqrt(sum(float(torch.linalg.vector_norm(g.to(d))) ** 2 for g in tensors))
            flat[k, :n] = torch.cat([g.to(d).flatten() for g in tensors]) * min(1.0, case["clip"] / norm)
            norms.append(norm)
        return dict(norms=torch.tensor(norms, dtype=d), flat=flat)
    x = s["logits"].to(d)
    lse = torch.logsumexp(x, 1)
    counted = s["targets"] != IGNORE
    weight = (torch.ones_like(lse) if s["weight"] is None else s["weight"].to(d)) * s["scale"] * counted
    at = s["targets"].clamp(min=0)[:, None]
    loss = weight * (lse - x.gather(1, at)[:, 0])
    x.sub_(lse[:, None]).exp_()
    x.scatter_add_(1, at, -torch.ones_like(at, dtype=d))
    return loss, lse, x.mul_(weight[:, None])
