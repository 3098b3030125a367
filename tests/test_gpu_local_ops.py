"""The operators of a worker's local step (linear layer and its gradients, cross-entropy, gradient
norm and clipping) against plain 64-bit formulas."""
import math

import numpy as np
import pytest
import torch

from paper_1909_09010_b200 import binding

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
ROUND = {BF: 2.0 ** -8, F: 2.0 ** -22}       # one rounding to nearest, with room for a tie that flips
ACTS = ["none", "relu", "gelu", "silu", "tanh", "sigmoid"]


@pytest.fixture(scope="module")
def ops():
    return binding.local_ops(0)


def rnd(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def lay(t, how):
    """The same values in another layout: as it is, rows padded to an odd stride, or off alignment."""
    if t is None or how == "plain":
        return t
    if t.dim() == 1:
        if how == "padded":
            return t
        buf = torch.full((t.numel() + 1,), math.nan, dtype=t.dtype, device=t.device)
        buf[1:] = t
        return buf[1:]
    r, c = t.shape
    pad, off = {"padded": (24, 0), "odd": (5, 3)}[how]
    buf = torch.full((r * (c + pad) + off,), math.nan, dtype=t.dtype, device=t.device)
    v = buf[off:].view(r, c + pad)[:, :c]
    v.copy_(t)
    return v


def act64(z, name):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * torch.special.erfc(-z / 2 ** 0.5) / 2,
            "silu": lambda: z * torch.sigmoid(z), "tanh": lambda: torch.tanh(z),
            "sigmoid": lambda: torch.sigmoid(z)}[name]()


def slope64(z, name):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(),
            "gelu": lambda: torch.special.erfc(-z / 2 ** 0.5) / 2 + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
            "silu": lambda: s * (1 + z * (1 - s)), "tanh": lambda: 1 - torch.tanh(z) ** 2,
            "sigmoid": lambda: s * (1 - s)}[name]()


def sum_error(a, b, k):
    """Bound on the error of an fp32 sum of k products in any order, each step off by at most one
    unit in the last place (2^-23) of a partial sum: a, b are |A|, |B| as matrices."""
    return (k + 8) * 2.0 ** -23 * (a @ b)


def check(got, ref, tol, dtype, what):
    assert got.dtype is dtype and got.shape == ref.shape
    err = (got.double() - ref).abs()
    bad = ~(err <= tol + ROUND[dtype] * ref.abs())
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float(err.max()):.3g}"
    n = float(ref.norm())
    if n > 0 and ref.numel() >= 64:
        # 2-norm: rounding to bf16 gives 2^-8 / sqrt(12) .. 2^-9; fp32 sums stay near 1e-6 however long
        assert float((got.double() - ref).norm()) / n < (3e-3 if dtype is BF else 3e-6), what


SHAPES = [(1, 1, 1), (1, 64, 8), (2, 1024, 4096), (3, 5, 7), (8, 512, 1001), (16, 96, 333), (17, 129, 65),
          (33, 64, 2048), (64, 512, 128), (100, 1024, 1000), (128, 64, 256), (130, 200, 515), (257, 512, 384),
          (512, 2048, 136), (1003, 515, 1027), (300, 4099, 264), (2049, 256, 1032)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_linear_forward(ops, dtype, rows, n_in, n_out):
    g = gen(rows * 7 + n_in * 3 + n_out)
    for i, act in enumerate(ACTS):
        how = ["plain", "padded", "odd"][(i + rows) % 3]
        x, w = rnd(g, (rows, n_in), dtype), rnd(g, (n_out, n_in), dtype, n_in ** -0.5)
        bias = rnd(g, (n_out,), dtype, 0.5) if i % 2 == 0 else None
        res = rnd(g, (rows, n_out), dtype) if i % 3 == 0 else None
        out = lay(torch.zeros((rows, n_out), dtype=dtype, device="cuda"), how)
        got = ops.linear_forward(lay(x, how), lay(w, how), bias=lay(bias, how), residual=lay(res, how),
                                 activation=act, keep_z=i != 1, out=out)
        z = x.double() @ w.double().t()
        tol = sum_error(x.double().abs(), w.double().abs().t(), n_in)
        if bias is not None:
            z = z + bias.double()
        y = act64(z, act)
        more = 1.25 * tol + 1e-6 * (1 + z.abs())
        if res is not None:
            more = more + 2.0 ** -23 * (y.abs() + res.double().abs())
            y = y + res.double()
        if i != 1:
            check(got[1], z, tol + 2.0 ** -23 * z.abs(), dtype, f"z {act} {how}")
            got = got[0]
        check(got, y, more, dtype, f"y {act} {how}")
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_linear_backward_input(ops, dtype, rows, n_in, n_out):
    g = gen(rows * 11 + n_in + n_out * 5)
    for i, act in enumerate(ACTS):
        how = ["plain", "padded", "odd"][(i + rows) % 3]
        dz, w = rnd(g, (rows, n_out), dtype, 1e-2), rnd(g, (n_out, n_in), dtype, n_in ** -0.5)
        z = rnd(g, (rows, n_in), dtype, 1.5) if i != 0 else None
        res = rnd(g, (rows, n_in), dtype, 1e-2) if i % 2 == 0 else None
        got = ops.linear_backward_input(lay(dz, how), lay(w, how), residual=lay(res, how), z_prev=lay(z, how),
                                        activation=act, want_dx=i % 3 == 1)
        dx = dz.double() @ w.double()
        tol = sum_error(dz.double().abs(), w.double().abs(), n_out)
        if res is not None:
            tol = tol + 2.0 ** -23 * (dx.abs() + res.double().abs())
            dx = dx + res.double()
        if z is None:
            check(got, dx, tol, dtype, f"dx {how}")
            continue
        if i % 3 == 1:
            check(got[0], dx, tol, dtype, f"dx {act} {how}")
            got = got[1]
        zd = z.double()
        check(got, dx * slope64(zd, act), 1.25 * tol + dx.abs() * 1e-6 * (1 + zd.abs()), dtype, f"dz_prev {act} {how}")
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES + [(20000, 64, 72), (9001, 512, 8)])
def test_linear_backward_weight(ops, dtype, rows, n_in, n_out):
    g = gen(rows + n_in * 13 + n_out)
    for i, (grad, accumulate, how) in enumerate([(F, False, "plain"), (F, True, "odd"), (BF, False, "padded"),
                                                 (BF, True, "plain")]):
        if grad is BF and dtype is F and accumulate:
            how = "odd"
        dz, x = rnd(g, (rows, n_out), dtype, 1e-2), rnd(g, (rows, n_in), dtype)
        dw0, db0 = rnd(g, (n_out, n_in), grad, 0.1), rnd(g, (n_out,), grad, 0.1)
        dw, db = lay(dw0.clone(), how), lay(db0.clone(), how)
        ops.linear_backward_weight(lay(dz, how), lay(x, how), dw_out=dw, dbias_out=db, accumulate=accumulate)
        ref, rb = dz.double().t() @ x.double(), dz.double().sum(0)
        tol = sum_error(dz.double().abs().t(), x.double().abs(), rows)
        tb = (rows + 8) * 2.0 ** -23 * dz.double().abs().sum(0)
        if accumulate:
            tol, tb = tol + 2.0 ** -23 * (ref.abs() + dw0.double().abs()), tb + 2.0 ** -23 * (rb.abs() + db0.double().abs())
            ref, rb = ref + dw0.double(), rb + db0.double()
        check(dw, ref, tol, grad, f"dw {grad} {how}")
        check(db, rb, tb, grad, f"dbias {grad} {how}")
        again = ops.linear_backward_weight(dz, x, grad_dtype=grad)
        once = ops.linear_backward_weight(dz, x, grad_dtype=grad)
        assert all(torch.equal(p, q) for p, q in zip(again, once)), "two calls give different bits"
    only = ops.linear_backward_weight(dz, x, want_bias=False)
    assert torch.equal(only, ops.linear_backward_weight(dz, x)[0])
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
def test_linear_writes_nothing_outside(ops, dtype):
    """Padding between the rows of every output, and what lies before and after, stays as it was."""
    g = gen(3)
    for rows, n_in, n_out in [(5, 40, 21), (131, 64, 259), (300, 136, 130)]:
        x, w, dz = rnd(g, (rows, n_in), dtype), rnd(g, (n_out, n_in), dtype), rnd(g, (rows, n_out), dtype)
        for r, c, call in [(rows, n_out, lambda o: ops.linear_forward(x, w, out=o)),
                           (rows, n_in, lambda o: ops.linear_backward_input(dz, w, dx_out=o)),
                           (n_out, n_in, lambda o: ops.linear_backward_weight(dz, x, dw_out=o, want_bias=False))]:
            for pad, off in [(0, 8), (16, 16), (7, 5)]:
                buf = torch.full((off + r * (c + pad) + 64,), 777.0, dtype=dtype, device="cuda")
                view = buf[off:off + r * (c + pad)].view(r, c + pad)
                call(view[:, :c])
                assert bool((view[:, c:] == 777).all()) and bool((buf[:off] == 777).all())
                assert bool((buf[off + r * (c + pad):] == 777).all())
                assert not bool((view[:, :c] == 777).all())


@pytest.mark.parametrize("dtype", [BF, F])
def test_linear_empty(ops, dtype):
    e = lambda *s: torch.ones(s, dtype=dtype, device="cuda")                        # noqa: E731
    bias = torch.tensor([1.0, -2.0, 0.5], dtype=dtype, device="cuda")
    y, z = ops.linear_forward(e(4, 0), e(3, 0), bias=bias, residual=e(4, 3), activation="relu", keep_z=True)
    assert torch.equal(z, bias.expand(4, 3)) and torch.equal(y, torch.relu(bias).expand(4, 3) + 1)
    assert ops.linear_forward(e(0, 8), e(3, 8), bias=bias).shape == (0, 3)
    assert ops.linear_forward(e(2, 8), e(0, 8)).shape == (2, 0)
    assert torch.equal(ops.linear_backward_input(e(2, 0), e(0, 5), residual=e(2, 5)), e(2, 5))
    assert ops.linear_backward_input(e(0, 3), e(3, 5)).shape == (0, 5)
    dw, db = ops.linear_backward_weight(e(0, 3), e(0, 5))
    assert not bool(dw.any()) and not bool(db.any())
    keep_w, keep_b = e(3, 5), e(3)
    ops.linear_backward_weight(e(0, 3), e(0, 5), dw_out=keep_w, dbias_out=keep_b, accumulate=True)
    assert torch.equal(keep_w, e(3, 5)) and torch.equal(keep_b, e(3))
    dw, db = ops.linear_backward_weight(e(4, 3), e(4, 0))
    assert dw.shape == (3, 0) and torch.equal(db, 4 * e(3))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows", [4, 200])
def test_linear_not_finite_stays_in_its_row(ops, dtype, rows):
    g = gen(9)
    x, w = rnd(g, (rows, 320), dtype), rnd(g, (160, 320), dtype, 0.1)
    clean = ops.linear_forward(x, w)
    bad = x.clone()
    bad[1, 7], bad[2, 300] = math.inf, math.nan
    y = ops.linear_forward(bad, w)
    assert not bool(torch.isfinite(y[1:3]).any())
    rest = [0] + list(range(3, rows))
    assert torch.equal(y[rest], clean[rest])
    # large and tiny operands: products across the whole exponent range stay what they are
    big = torch.full((rows, 8), 3.0e38, dtype=dtype, device="cuda")
    small = torch.full((16, 8), 2.0 ** -126, dtype=dtype, device="cuda")
    got = ops.linear_forward(big, small).double()
    ref = 8 * float(big[0, 0].double()) * 2.0 ** -126
    assert float((got - ref).abs().max()) <= ROUND[dtype] * ref


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("act", ACTS)
def test_activation_values_and_slopes(ops, dtype, act):
    """The whole range of an activation through an identity matrix, its slope, and infinities."""
    z = torch.linspace(-30, 30, 24_000, device="cuda").to(dtype).view(-1, 16)
    eye = torch.eye(16, dtype=dtype, device="cuda")
    y = ops.linear_forward(z, eye, activation=act)
    check(y, act64(z.double(), act), 1e-6 * (1 + z.double().abs()), dtype, act)
    dy = torch.ones_like(z)
    s = slope64(z.double(), act)
    for got in (ops.activation_backward(dy, z, act), ops.linear_backward_input(dy, eye, z_prev=z, activation=act)):
        check(got, s, 1e-6 * (1 + z.double().abs()), dtype, f"slope of {act}")
    place = dy.clone()
    assert torch.equal(ops.activation_backward(place, z, act, out=place), ops.activation_backward(dy, z, act))
    ends = torch.tensor([[-math.inf, math.inf, -1e30, 1e30, 0.0, -0.0, 100.5, -100.5]], dtype=dtype, device="cuda")
    limits = {"none": [1, 1, 1, 1, 1, 1, 1, 1], "relu": [0, 1, 0, 1, 0, 0, 1, 0], "gelu": [0, 1, 0, 1, .5, .5, 1, 0],
              "silu": [0, 1, 0, 1, .5, .5, 1, 0], "tanh": [0, 0, 0, 0, 1, 1, 0, 0],
              "sigmoid": [0, 0, 0, 0, .25, .25, 0, 0]}[act]
    got = ops.activation_backward(torch.ones_like(ends), ends, act).double().cpu()
    assert float((got - torch.tensor([limits]).double()).abs().max()) < 1e-30
    nan = torch.full((1, 8), math.nan, dtype=dtype, device="cuda")
    if act != "none":
        assert bool(torch.isnan(ops.activation_backward(torch.ones_like(nan), nan, act)).all())


def test_linear_gradients_against_differences(ops):
    """Sum of c * y over a two-layer residual block: gradients of the calls against central
    differences of the calls' own forward values."""
    g = gen(21)
    n, d, h = 6, 24, 40
    x, w1, b1 = rnd(g, (n, d), F), rnd(g, (h, d), F, 0.3), rnd(g, (h,), F, 0.3)
    w2, b2, c = rnd(g, (d, h), F, 0.3), rnd(g, (d,), F, 0.3), rnd(g, (n, d), F)

    def value(x, w1, b1, w2, b2):
        y1 = ops.linear_forward(x, w1, bias=b1, activation="gelu")
        return float((ops.linear_forward(y1, w2, bias=b2, residual=x).double() * c.double()).sum())

    y1, z1 = ops.linear_forward(x, w1, bias=b1, activation="gelu", keep_z=True)
    dw2, db2 = ops.linear_backward_weight(c, y1)
    dz1 = ops.linear_backward_input(c, w2, z_prev=z1, activation="gelu")
    dw1, db1 = ops.linear_backward_weight(dz1, x)
    dx = ops.linear_backward_input(dz1, w1, residual=c)
    args = [x, w1, b1, w2, b2]
    step = 2.0 ** -6
    for i, grad in enumerate([dx, dw1, db1, dw2, db2]):
        flat = grad.reshape(-1)
        for j in range(0, flat.numel(), max(1, flat.numel() // 12)):
            v = []
            for s in (step, -step):
                moved = [t.clone() for t in args]
                moved[i].view(-1)[j] += s
                v.append(value(*moved))
            # third derivatives here are below ~60 per argument: truncation step^2/6 * 60 = 2.5e-3;
            # 2 sums of ~1e2 terms of size 1 off by 1e-6 each, over 2 * step: below 1e-2
            assert abs((v[0] - v[1]) / (2 * step) - float(flat[j])) < 1.3e-2


def test_linear_on_another_stream_and_in_a_graph(ops):
    g = gen(5)
    x, w, b = rnd(g, (300, 256), BF), rnd(g, (520, 256), BF), rnd(g, (520,), BF)
    ref = ops.linear_forward(x, w, bias=b, activation="silu")
    xf, wf = rnd(g, (300, 131), F), rnd(g, (77, 131), F)
    reff = ops.linear_forward(xf, wf)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out, outf = torch.empty_like(ref), torch.empty_like(reff)
    ops.linear_forward(x, w, bias=b, activation="silu", out=out, stream=side)
    ops.linear_forward(xf, wf, out=outf, stream=side)
    side.synchronize()
    assert torch.equal(out, ref) and torch.equal(outf, reff)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.linear_forward(x, w, bias=b, activation="silu", out=out)
        ops.linear_forward(xf, wf, out=outf)
        dw, db = ops.linear_backward_weight(out, x)
    x.mul_(0.5)
    xf.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ops.linear_forward(x, w, bias=b, activation="silu"))
    assert torch.equal(outf, ops.linear_forward(xf, wf))
    assert torch.equal(dw, ops.linear_backward_weight(out, x)[0])


# ---------------------------------------------------------------------------------- cross-entropy
def loss64(x, t, ignore, weight, scale):
    x = x.double()
    lse = torch.logsumexp(x, 1)
    on = t != ignore
    s = torch.full_like(lse, scale) if weight is None else weight.double() * scale
    s = s * on
    at = torch.where(on, t, 0)
    loss = torch.where(on, s * (lse - x[torch.arange(x.shape[0]), at]), 0.0)
    d = torch.exp(x - lse[:, None])
    d[torch.arange(x.shape[0]), at] -= 1
    return loss, lse, torch.where(on[:, None], d * s[:, None], 0.0), s


def check_loss(got, x, t, ignore, weight, scale, dtype):
    loss, lse, d, s = loss64(x, t, ignore, weight, scale)
    # logits below 100 in size: exponents off by 100 * 2^-23 at most, a sum by less, the log by 2^-22
    assert float((got[1].double() - lse).abs().max()) <= 2e-5 + 1e-6 * float(lse.abs().max())
    assert bool(((got[0].double() - loss).abs() <= s.abs() * (2e-5 + 2e-6 * x.double().abs().max()) + 1e-6 * loss.abs()).all())
    if len(got) == 3:
        err = (got[2].double() - d).abs()
        p = d.abs() + s.abs()[:, None] * 1e-7
        assert bool((err <= ROUND[dtype] * d.abs() + 3e-5 * p).all()), float(err.max())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (5, 31), (4, 256), (700, 1000), (64, 4097), (9, 10000),
                                        (40, 33278), (7, 50003), (3, 131072), (5, 267735), (300, 20011)])
def test_cross_entropy(ops, dtype, rows, vocab):
    g = gen(rows + vocab)
    for how, weighted in [("plain", False), ("odd", True), ("padded", True)]:
        x = rnd(g, (rows, vocab), dtype, 4.0)
        t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        if rows > 2:
            t[1], t[2] = 5 - 100 - 5, vocab - 1
        w = torch.rand((rows,), generator=g, device="cuda") + 0.1 if weighted else None
        scale = 1.0 / rows
        src = lay(x, how)
        got = ops.cross_entropy(src, t, row_weight=w, scale=scale)
        check_loss(got, x, t, -100, w, scale, dtype)
        only = ops.cross_entropy(src, t, row_weight=w, scale=scale, want_grad=False)
        assert torch.equal(only[0], got[0]) and torch.equal(only[1], got[1])
        out = lay(torch.zeros_like(x), {"plain": "odd", "odd": "padded", "padded": "plain"}[how])
        ops.cross_entropy(src, t, row_weight=w, scale=scale, dlogits_out=out)
        assert torch.equal(out, got[2])
        assert ops.cross_entropy(src, t, row_weight=w, scale=scale, dlogits_out=src)[2] is src
        assert torch.equal(src, got[2]), "in place"
        if how != "plain":
            rest = src.as_strided((rows - 1, src.stride(0) - vocab), (src.stride(0), 1), src.storage_offset() + vocab)
            assert bool(torch.isnan(rest).all()), "padding was written"
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("vocab", [7, 1000, 30001, 150000])
def test_cross_entropy_masked_and_not_finite(ops, dtype, vocab):
    g = gen(vocab)
    x = rnd(g, (10, vocab), dtype, 2.0)
    low = torch.finfo(dtype).min
    x[0, 1:] = -math.inf                       # one word left
    x[1, :] = -math.inf                        # none left
    x[2, vocab // 2:] = -math.inf
    x[3, :] = math.nan                         # ignored
    x[4, 3] = math.nan
    x[5, 2] = math.inf
    x[6, 1:] = low
    x[7, :] = low
    x[8, 0] = -math.inf                        # the target itself cannot occur
    t = torch.tensor([0, 1, 1, -7, 0, 0, 0, 2, 0, 3], device="cuda")
    loss, lse, d = ops.cross_entropy(x, t, ignore_index=-7, scale=0.5)
    assert float(loss[0]) == 0 and float(lse[0]) == float(x[0, 0]) and not bool(d[0].any())
    assert float(lse[1]) == -math.inf and float(loss[1]) == math.inf and not bool(d[1].any())
    assert not bool(d[2, vocab // 2:].any())
    assert float(loss[3]) == 0 and not bool(d[3].any())
    for r in (4, 5):
        assert math.isnan(float(loss[r])) and math.isnan(float(lse[r])) and bool(torch.isnan(d[r]).all())
    assert float(loss[6]) == 0 and not bool(d[6].any())
    assert abs(float(loss[7]) - 0.5 * math.log(vocab)) <= 2.0 ** -22 * abs(low)
    assert abs(float(d[7, 0]) - 0.5 / vocab) <= 0.5 / vocab * 2.0 ** -7
    assert float(loss[8]) == math.inf and bool(torch.isfinite(d[8]).all())
    for r in (2, 9):
        check_loss([v[r:r + 1] for v in (loss, lse, d)], x[r:r + 1], t[r:r + 1], -7, None, 0.5, dtype)
    assert ops.device_status() == 0
    zero = ops.cross_entropy(x, t, row_weight=torch.zeros(10, device="cuda"), ignore_index=-7)
    assert not bool(zero[0].any()) and not bool(zero[2].any())


def test_cross_entropy_target_outside(ops):
    x = torch.randn((3, 500), device="cuda")
    t = torch.tensor([1, 500, -1], device="cuda")
    loss, lse, d = ops.cross_entropy(x, t)
    assert ops.device_status() == binding.ERR_INVALID_ARG and ops.device_status() == 0
    assert bool(torch.isnan(loss[1:]).all()) and not bool(d[1:].any()) and bool(torch.isfinite(lse).all())
    check_loss([loss[:1], lse[:1], d[:1]], x[:1], t[:1], -100, None, 1.0, F)


def test_cross_entropy_gradient_against_differences(ops):
    g = gen(4)
    x = rnd(g, (3, 40), F, 2.0)
    t = torch.tensor([4, 39, 0], device="cuda")
    d = ops.cross_entropy(x, t)[2]
    h = 2.0 ** -5
    for r in range(3):
        for v in range(0, 40, 3):
            a, b = x.clone(), x.clone()
            a[r, v] += h
            b[r, v] -= h
            num = (float(ops.cross_entropy(a, t)[0][r]) - float(ops.cross_entropy(b, t)[0][r])) / (2 * h)
            # |third derivative| <= 1/8: h^2/6/8 = 2.1e-5; two losses near 5 off by 1e-6 over 2h: 3.2e-5
            assert abs(num - float(d[r, v])) < 6e-5


# ----------------------------------------------------------------------------- norms and clipping
def entries_of(g, dtypes, shapes, groups, scale, outs):
    rows = []
    for k in range(groups):
        for i, s in enumerate(shapes):
            dt = dtypes[(k + i) % len(dtypes)]
            t = rnd(g, s, dt, scale * (k + 1))
            how = outs[(k + 2 * i) % len(outs)]
            out = None if how == "none" else t if how == "place" else torch.full(
                s, 9.0, dtype=dt if how == "same" else F, device="cuda")
            rows.append((t, out, k))
    return rows


@pytest.mark.parametrize("max_norm", [1.0, 1e6, 0.0])
@pytest.mark.parametrize("dtypes", [[F], [BF], [BF, F]])
@pytest.mark.parametrize("groups,shapes", [(1, [(1,)]), (1, [(5, 7), (100_003,), ()]), (3, [(0,), (64, 33), (8192,), (8193,)]),
                                           (5, [(1000, 128), (512, 128), (3,), (128,)]), (2, [(3_000_001,), (17, 5)]),
                                           (40, [(9,), (2, 2)])])
def test_norms_and_clip(max_norm, dtypes, groups, shapes):
    g = gen(groups + len(shapes))
    entries = entries_of(g, dtypes, shapes, groups, 0.1, ["f32", "same", "none", "place"])
    g.manual_seed(1)
    order = torch.randperm(len(entries), generator=torch.Generator().manual_seed(groups)).tolist()
    entries = [entries[i] for i in order]
    before = [t.clone() for t, _, _ in entries]
    clip = binding.GradClip(entries, groups=groups)
    norms = clip.norms()
    ref = torch.zeros(groups, dtype=torch.float64)
    for t, (_, _, k) in zip(before, entries):
        ref[k] += float((t.double() ** 2).sum())
    ref = ref.sqrt()
    # double sums, one rounding to fp32
    assert bool(((norms.cpu().double() - ref).abs() <= 2.0 ** -23 * ref).all())
    assert torch.equal(clip.clip(max_norm), norms)
    for t, (grad, out, k) in zip(before, entries):
        if out is None:
            continue
        n32 = float(norms[k])
        c = max_norm / max(n32, max_norm) if max_norm > 0 else 1.0
        want = t.double() * c
        # the factor is rounded once, the product once, and once more to the output's type
        tol = (2.0 ** -22 + (ROUND[BF] if out.dtype is BF else 0)) * want.abs() + 2.0 ** -133
        assert bool(((out.double() - want).abs() <= tol).all())
        if out is not grad:
            assert torch.equal(grad, t)
    clip.destroy()


def test_clip_strided_rows_and_offsets():
    """Gradients inside rows of a larger buffer, transposed ones, outs inside an optimiser's rows."""
    g = gen(8)
    big = rnd(g, (40, 260), F)
    flat = torch.full((2, 40 * 100 + 77 * 3 + 30), 5.0, device="cuda")
    views = [big[:, 3:103], rnd(g, (3, 77), BF).t(), rnd(g, (11,), BF)[1:], big[7:9, 200:210].t()]
    outs, at = [], 1
    for v in views[:3]:
        n = v.numel()
        outs.append(flat[1, at:at + n].view(v.t().shape).t() if v.dim() == 2 and v.stride(0) == 1 else flat[1, at:at + n].view(v.shape))
        at += n
    outs.append(torch.zeros((2, 10), device="cuda").t())
    clip = binding.GradClip([(v, o, 0) for v, o in zip(views, outs)])
    norm = float(clip.clip(2.0)[0])
    ref = math.sqrt(sum(float((v.double() ** 2).sum()) for v in views))
    assert abs(norm - ref) <= 2.0 ** -23 * ref
    for v, o in zip(views, outs):
        assert torch.allclose(o.double(), v.double() * (2.0 / norm), rtol=2.0 ** -22, atol=0)
    assert bool((flat[0] == 5).all()) and float(flat[1, 0]) == 5 and bool((flat[1, at:] == 5).all())
    with pytest.raises(ValueError):
        binding.GradClip([(torch.zeros((4, 4, 4), device="cuda")[:, :2, :2], None, 0)])


def test_clip_not_finite_group_gives_zeros():
    for bad in (math.inf, -math.inf, math.nan):
        a, b = torch.randn(5000, device="cuda"), torch.randn(5000, device="cuda").to(BF)
        a[4999] = bad
        oa, ob = torch.ones_like(a), torch.ones_like(b)
        clip = binding.GradClip([(a, oa, 0), (b, ob, 1)], groups=2)
        norms = clip.clip(1.0)
        assert not math.isfinite(float(norms[0])) and math.isfinite(float(norms[1]))
        assert not bool(oa.any()) and bool((ob != 0).any())
    # squares beyond the fp32 range: the norm itself is representable
    a = torch.full((100,), 1e30, device="cuda")
    tiny = torch.full((100,), 1e-30, device="cuda")
    oa, ot = torch.zeros_like(a), torch.zeros_like(tiny)
    clip = binding.GradClip([(a, oa, 0), (tiny, ot, 1)], groups=2)
    norms = clip.clip(1.0).cpu()
    assert abs(float(norms[0]) - 1e31) < 1e25 and abs(float(norms[1]) - 1e-29) < 1e-35
    assert abs(float(oa[0]) - 0.1) < 1e-6 and torch.equal(ot, tiny)


def test_clip_same_bits_new_tensors_and_graph():
    g = gen(2)
    make = lambda: [(rnd(g, s, F, 0.1), torch.zeros(s, device="cuda"), i % 2)                     # noqa: E731
                    for i, s in enumerate([(400, 300), (50_000,), (7,), (123, 45)])]
    first, second = make(), make()
    clip = binding.GradClip(first, groups=2)
    n1 = clip.clip(0.5)
    out1 = [o.clone() for _, o, _ in first]
    for _ in range(3):
        assert torch.equal(clip.clip(0.5), n1)
        assert all(torch.equal(o, p) for (_, o, _), p in zip(first, out1))
    clip.set_tensors(second[:3])
    n2 = clip.clip(0.5)
    ref = [math.sqrt(sum(float((t.double() ** 2).sum()) for t, _, k in second[:3] if k == j)) for j in range(2)]
    assert np.allclose(n2.cpu().numpy(), ref, rtol=1e-6)
    norms = torch.zeros(2, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        clip.clip(0.5, norms_out=norms)
    second[0][0].mul_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(norms, clip.norms())
    clip.set_tensors([])
    assert not bool(clip.clip(1.0).any())


# ------------------------------------------------------------------------------------- refusals
def test_refusals(ops):
    x, w = torch.zeros((4, 8), device="cuda"), torch.zeros((6, 8), device="cuda")
    for call in [lambda: ops.linear_forward(x, w[:, :7]), lambda: ops.linear_forward(x, w.to(BF)),
                 lambda: ops.linear_forward(x, w.cpu()), lambda: ops.linear_forward(x.cpu(), w.cpu()),
                 lambda: ops.linear_forward(x, w, bias=torch.zeros(7, device="cuda")),
                 lambda: ops.linear_forward(x.t(), w[:, :4].t().contiguous()),
                 lambda: ops.linear_forward(x.half(), w.half()),
                 lambda: ops.linear_forward(x, w, activation="swish"),
                 lambda: ops.linear_forward(x[0], w), lambda: ops.linear_backward_input(x, w),
                 lambda: ops.linear_backward_input(x[:, :6], w, dz_out=torch.zeros((4, 8), device="cuda")),
                 lambda: ops.linear_backward_weight(x, w), lambda: ops.linear_backward_weight(x, x, accumulate=True),
                 lambda: ops.cross_entropy(x, torch.zeros(3, dtype=torch.int64, device="cuda")),
                 lambda: ops.cross_entropy(x, torch.zeros(4, dtype=torch.int32, device="cuda")),
                 lambda: binding.GradClip([(x, torch.zeros(4, 7, device="cuda"), 0)]),
                 lambda: binding.GradClip([(x.half(), None, 0)])]:
        with pytest.raises((ValueError, TypeError, KeyError)):
            call()
    L, h = binding.lib(), ops._h
    import ctypes
    p, q = x.data_ptr(), w.data_ptr()
    good = dict(rows=4, n_in=8, n_out=6, x=p, w=q, y=p, ld_x=8, ld_w=8, ld_y=8)
    for change in [dict(rows=-1), dict(x=None), dict(w=None), dict(y=None), dict(x=p + 1), dict(ld_x=7), dict(ld_y=5),
                   dict(dtype=2), dict(activation=6), dict(activation=-1), dict(ld_w=1 << 50)]:
        a = binding.LinearForwardArgs(**{**good, **change})
        assert L.gbmuf_linear_forward(h, ctypes.byref(a), None) == binding.ERR_INVALID_ARG, change
        assert L.gbmuf_last_error(None)
    a = binding.LinearForwardArgs(**{**good, "rows": 1 << 31})
    assert L.gbmuf_linear_forward(h, ctypes.byref(a), None) == binding.ERR_UNSUPPORTED
    assert L.gbmuf_linear_forward(None, ctypes.byref(a), None) == binding.ERR_INVALID_ARG
    assert L.gbmuf_linear_forward(h, None, None) == binding.ERR_INVALID_ARG
    for change in [dict(vocab=0), dict(logits=None), dict(targets=None), dict(scale=math.nan), dict(dtype=3), dict(ld_logits=5),
                   dict(dlogits=p, ld_dlogits=12)]:
        a = binding.CrossEntropyArgs(**{**dict(rows=4, vocab=8, logits=p, targets=q, ld_logits=8, scale=1.0), **change})
        assert L.gbmuf_cross_entropy(h, ctypes.byref(a), None) == binding.ERR_INVALID_ARG, change
    for change in [dict(grad=None), dict(rows=-1), dict(group=1), dict(group=-1), dict(dtype=5), dict(ld_grad=3),
                   dict(out=p + 128, out_dtype=1, ld_out=8), dict(out=p, ld_out=9)]:
        t = (binding.GradTensor * 1)(binding.GradTensor(**{**dict(grad=p, rows=4, cols=8, ld_grad=8), **change}))
        out = ctypes.c_void_p()
        assert L.gbmuf_clip_create(0, 1, 1, t, ctypes.byref(out)) == binding.ERR_INVALID_ARG, change
        assert not out.value
    clip = binding.GradClip([(x, None, 0)])
    with pytest.raises(binding.GbmufError):
        clip.clip(math.nan)


# ------------------------------------------------------- products large enough for every launch shape
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,n_in,n_out", [(2048, 1024, 20000), (4096, 512, 2048), (8192, 4096, 1024),
                                             (64, 4096, 1024), (128, 4096, 1024), (16, 2048, 2048), (256, 1024, 30000),
                                             (8200, 264, 250), (1000, 4104, 1032), (33, 8192, 100)])
def test_linear_large(ops, dtype, rows, n_in, n_out):
    g = gen(rows + n_in + n_out)
    x, w, b = rnd(g, (rows, n_in), dtype), rnd(g, (n_out, n_in), dtype, n_in ** -0.5), rnd(g, (n_out,), dtype, 0.2)
    dz, res = rnd(g, (rows, n_out), dtype, 1e-2), rnd(g, (rows, n_in), dtype, 1e-2)
    xd, wd, dd = x.double(), w.double(), dz.double()
    y, z = ops.linear_forward(x, w, bias=b, activation="silu", keep_z=True)
    ref = xd @ wd.t() + b.double()
    tol = sum_error(xd.abs(), wd.abs().t(), n_in)
    check(z, ref, tol + 2.0 ** -23 * ref.abs(), dtype, "z")
    check(y, act64(ref, "silu"), 1.25 * tol + 1e-6 * (1 + ref.abs()), dtype, "y")
    dx, dp = ops.linear_backward_input(dz, w, residual=res, z_prev=x, activation="tanh", want_dx=True)
    ref = dd @ wd
    tol = sum_error(dd.abs(), wd.abs(), n_out) + 2.0 ** -23 * (ref.abs() + res.double().abs())
    ref = ref + res.double()
    check(dx, ref, tol, dtype, "dx")
    check(dp, ref * slope64(xd, "tanh"), 1.25 * tol + ref.abs() * 1e-6 * (1 + xd.abs()), dtype, "dz_prev")
    for grad in (F, BF):
        dw, db = ops.linear_backward_weight(dz, x, grad_dtype=grad)
        check(dw, dd.t() @ xd, sum_error(dd.abs().t(), xd.abs(), rows), grad, "dw")
        check(db, dd.sum(0), (rows + 8) * 2.0 ** -23 * dd.abs().sum(0), grad, "dbias")
    assert ops.device_status() == 0


def test_two_streams_at_once(ops):
    """Calls on two streams share the handle; results are those of calls one after the other."""
    g = gen(77)
    jobs = []
    for i in range(2):
        x, w = rnd(g, (700 + i, 515), F), rnd(g, (333, 515), F)
        logits, t = rnd(g, (40, 50_001), BF, 3.0), torch.randint(0, 50_001, (40,), generator=g, device="cuda")
        jobs.append((x, w, logits, t))
    ref = [(ops.linear_forward(x, w, activation="gelu"), *ops.cross_entropy(l, t)) for x, w, l, t in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, (x, w, l, t) in zip(streams, jobs):
            with torch.cuda.stream(s):
                got.append((ops.linear_forward(x, w, activation="gelu"), *ops.cross_entropy(l, t)))
        torch.cuda.synchronize()
        for a, b in zip(got, ref):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
