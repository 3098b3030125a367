"""The softmax layer with its cross-entropy and gradients, without the logits in memory
(``linear_cross_entropy``), against plain 64-bit formulas."""
import ctypes
import math

import pytest
import torch

from paper_1909_09010_b200 import binding

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F: 2.0 ** -24}        # half a step, relative
IGNORE = -100


@pytest.fixture(scope="module")
def ops():
    return binding.local_ops(0)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rnd(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


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


def problem(g, rows, n_in, vocab, dtype, bias=True, weighted=True, spread=2.0):
    x, w = rnd(g, (rows, n_in), dtype), rnd(g, (vocab, n_in), dtype, spread * max(n_in, 1) ** -0.5)
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    if rows > 2:
        t[torch.rand(rows, device="cuda", generator=g) < 0.15] = IGNORE
    return (x, w, t, rnd(g, (vocab,), dtype, 0.5) if bias else None,
            torch.rand(rows, device="cuda", generator=g) + 0.5 if weighted else None)


def reference(x, w, t, bias, weight, scale):
    """Values, and bounds on the error of what the call computes.

    z: an fp32 sum of n_in products, each step off by at most one unit 2^-23 of a partial sum, and the bias.
    lse: as far off as the worst z; its exponentials by 2^-21 and the rounding of their exponents; a running
    sum has at most vocab / 8 additions (a thread takes every fourth strip, two words at a time), the joins fewer.
    d: relative to p, the sum of both; rounded to the operands' type (three bf16 parts: 2^-23)."""
    x, w = x.double(), w.double()
    n_in, vocab = x.shape[1], w.shape[0]
    z = x @ w.t()
    ez = (n_in + 8) * 2.0 ** -23 * (x.abs() @ w.abs().t())
    if bias is not None:
        z = z + bias.double()
        ez = ez + 2.0 ** -23 * (z.abs() + bias.double().abs())
    lse = torch.logsumexp(z, 1)
    elog = (ez.nan_to_num(0, 0, 0).amax(1) if vocab else 0) + 2.0 ** -20 + (vocab / 8 + 64) * 2.0 ** -24
    valid = t != IGNORE
    s = scale * valid.double() * (1 if weight is None else weight.double())
    at = torch.where(valid, t, 0)[:, None]
    zt = z.gather(1, at)[:, 0]
    loss = torch.where(s == 0, 0.0, s * (lse - zt))
    eloss = s.abs() * (elog + ez.gather(1, at)[:, 0] + 2.0 ** -22 * (lse.abs() + zt.abs()))
    p = torch.exp(z - lse[:, None])
    d = torch.where((s == 0)[:, None], 0.0, s[:, None] * (p - torch.zeros_like(p).scatter_(1, at, 1.0)))
    ed = s.abs()[:, None] * p * (ez + elog[:, None] + 2.0 ** -20 + 2.0 ** -23 * (z - lse[:, None]).abs())
    return dict(z=z, lse=lse, else_=elog + 2.0 ** -23 * lse.abs(), loss=loss, eloss=eloss, d=d, ed=ed, x=x, w=w)


def inside(got, ref, tol, dtype, what):
    assert got.dtype is dtype and got.shape == ref.shape, what
    err = (got.double() - ref).abs()
    bad = ~(err <= tol + HALF[dtype] * (ref.abs() + tol))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float(err.max()):.3g}"


def close(got, ref, dtype, what):
    """2-norm.  bf16: two roundings (d and the result), each 2^-8 / sqrt(12) to 2^-9 or so; fp32: exponents of a few
    tens rounded at 2^-24, sums of products at about 1e-6."""
    n = float(ref.norm())
    if n > 0 and ref.numel() >= 64:
        assert float((got.double() - ref).norm()) / n < (2.0 ** -8 if dtype is BF else 2.0 ** -17), what


def check(got, R, dtype, grad_dtype, what, bias=True, before=None):
    inside(got[0], R["loss"], R["eloss"], F, what + " loss")
    inside(got[1], R["lse"], R["else_"], F, what + " lse")
    if len(got) == 2:
        return
    rows, vocab = R["d"].shape
    d, ed = R["d"], R["ed"]
    ed_rounded = ed + (HALF[BF] if dtype is BF else 2.0 ** -23) * (d.abs() + ed)
    dx = d @ R["w"]
    inside(got[2], dx, ed_rounded @ R["w"].abs() + (vocab + 8) * 2.0 ** -23 * (d.abs() @ R["w"].abs()), dtype, what + " dx")
    close(got[2], dx, dtype, what + " dx")
    if len(got) == 3:
        return
    a, b = (0, 0) if before is None else (before[0].double(), before[1].double())
    dw = d.t() @ R["x"] + a
    more = 0 if before is None else 2.0 ** -23 * dw.abs()
    inside(got[3], dw, ed_rounded.t() @ R["x"].abs() + (rows + 8) * 2.0 ** -23 * (d.abs().t() @ R["x"].abs()) + more,
           grad_dtype, what + " dw")
    if before is None:
        close(got[3], dw, BF if BF in (dtype, grad_dtype) else F, what + " dw")
    if bias:
        db = d.sum(0) + b
        inside(got[4], db, ed.sum(0) + (rows + 8) * 2.0 ** -23 * d.abs().sum(0) + 2.0 ** -23 * db.abs(), grad_dtype,
               what + " dbias")


SHAPES = [(1, 1, 1), (1, 1024, 1000), (2, 8, 64), (3, 5, 7), (17, 129, 333), (64, 64, 256), (130, 200, 1515),
          (257, 512, 2048), (300, 70, 4099), (1003, 515, 1027), (2049, 256, 1032), (128, 8, 20011), (5, 320, 40_001)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,n_in,vocab", SHAPES)
def test_values_and_gradients(ops, dtype, rows, n_in, vocab):
    g = gen(rows * 7 + n_in * 3 + vocab)
    for i, how in enumerate(["plain", "padded", "odd"]):
        bias, weighted = i != 1, i != 2
        x, w, t, b, rw = problem(g, rows, n_in, vocab, dtype, bias, weighted)
        scale = [1.0 / rows, 1.0, -0.5][i]
        R = reference(x, w, t, b, rw, scale)
        args = (lay(x, how), lay(w, how), t, lay(b, how))
        kw = dict(row_weight=rw, scale=scale)
        check(ops.linear_cross_entropy(*args, want_grad=False, **kw), R, dtype, dtype, f"{how} values")
        check(ops.linear_cross_entropy(*args, **kw), R, dtype, dtype, how, bias)
        # pieces: small, odd, and the last one short
        piece = [64, max(1, vocab // 3 + 1), max(1, min(vocab - 1, 1000))][i]
        gd = F if i != 1 else dtype
        dx = lay(torch.zeros((rows, n_in), dtype=dtype, device="cuda"), how)
        dw = lay(torch.zeros((vocab, n_in), dtype=gd, device="cuda"), how)
        got = ops.linear_cross_entropy(*args, piece=piece, dx_out=dx, dw_out=dw, **kw)
        assert got[2] is dx and got[3] is dw
        check(got, R, dtype, gd, f"{how} piece {piece}", bias)
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,n_in,vocab", [(300, 40, 7), (70, 24, 1), (8, 520, 3001), (9, 64, 5000), (16, 72, 2500), (17, 72, 2500),
                                             (4, 1000, 40_000), (2000, 24, 33), (33, 2056, 96)])
def test_few_rows_few_words(ops, dtype, rows, n_in, vocab):
    """On both sides of the rules for a few rows, and tiles wider than the vocabulary or the batch."""
    x, w, t, b, rw = problem(gen(rows + vocab), rows, n_in, vocab, dtype)
    R = reference(x, w, t, b, rw, 0.5)
    for how in ("plain", "odd"):
        got = ops.linear_cross_entropy(lay(x, how), lay(w, how), t, lay(b, how), row_weight=rw, scale=0.5)
        check(got, R, dtype, dtype, how)
        alone = ops.linear_cross_entropy(lay(x, how), lay(w, how), t, lay(b, how), row_weight=rw, scale=0.5, want_grad=False)
        check(alone, R, dtype, dtype, how)
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,n_in,vocab,piece", [(495, 170, 3, 1), (4, 3, 9, 2), (40, 7, 33, 16), (100, 8, 65, 64), (12, 40, 21, 5)])
def test_pieces_of_a_single_word(ops, dtype, rows, n_in, vocab, piece):
    """A piece of one word may be aligned where its matrix is not: it is packed like the others."""
    x, w, t, b, rw = problem(gen(rows + vocab), rows, n_in, vocab, dtype)
    R = reference(x, w, t, b, rw, 0.3)
    for how in ("plain", "padded", "odd"):
        got = ops.linear_cross_entropy(lay(x, how), lay(w, how), t, lay(b, how), row_weight=rw, scale=0.3, piece=piece)
        check(got, R, dtype, dtype, how)
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows", [3, 200])
def test_masks_of_the_lowest_value(ops, dtype, rows):
    """A bias of the type's lowest value: words that hardly occur, or a mask that leaves nothing (all words equal)."""
    g = gen(rows)
    n_in, vocab = 32, 700
    x, w, t, b, rw = problem(g, rows, n_in, vocab, dtype)
    lowest = torch.finfo(dtype).min
    some = torch.where(torch.rand(vocab, device="cuda", generator=g) < 0.5, lowest, b.float()).to(dtype)
    some[t[t != IGNORE]] = 0.0
    for bias in (some, torch.full_like(b, lowest)):
        z = x.double() @ w.double().t() + bias.double()
        top = z.amax(1, keepdim=True)
        if float(bias.max()) == lowest:
            z = torch.zeros_like(z)                        # lowest plus anything of this size is lowest
            top = torch.full_like(top, lowest)
        else:
            z, top = z - top, top
        lse = torch.logsumexp(z, 1, keepdim=True)
        valid = t != IGNORE
        at = torch.where(valid, t, 0)[:, None]
        s = torch.where(valid, rw.double(), 0.0)
        loss = s * (lse - z.gather(1, at))[:, 0]
        d = s[:, None] * (torch.exp(z - lse) - torch.zeros_like(z).scatter_(1, at, 1.0))
        got = ops.linear_cross_entropy(x, w, t, bias, row_weight=rw, grad_dtype=F, piece=256)
        # logits of a few units off by 1e-6, as their exponentials and sums
        assert float((got[0].double() - loss).abs().max()) <= 1e-5 * (1 + float(loss.abs().max()))
        assert float((got[1].double() - (top + lse)[:, 0]).abs().max()) <= 1e-5 * (1 + float((top + lse).abs().max()))
        assert float((got[4].double() - d.sum(0)).abs().max()) <= 1e-5 * (1 + float(d.abs().sum(0).max()))
        dw = d.t() @ x.double()
        assert float((got[3].double() - dw).norm()) <= (2.0 ** -8 if dtype is BF else 2.0 ** -17) * float(dw.norm())
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
def test_accumulate_and_single_gradients(ops, dtype):
    g = gen(5)
    x, w, t, b, rw = problem(g, 150, 96, 777, dtype)
    R = reference(x, w, t, b, rw, 0.25)
    for gd in (BF, F):
        before = rnd(g, (777, 96), gd, 0.1), rnd(g, (777,), gd, 0.1)
        dw, db = before[0].clone(), before[1].clone()
        got = ops.linear_cross_entropy(x, w, t, b, row_weight=rw, scale=0.25, dw_out=dw, dbias_out=db, accumulate=True,
                                       piece=300)
        assert got[3] is dw and got[4] is db
        check(got, R, dtype, gd, f"accumulate {gd}", before=before)
    only = ops.linear_cross_entropy(x, w, t, b, row_weight=rw, scale=0.25, want_weight_grad=False, piece=300)
    assert len(only) == 3 and torch.equal(only[2], got[2])
    # without dx: the C call with one result at a time
    h, L = ops._h, binding.lib()
    for which in ("dw", "dbias"):
        out = torch.zeros((777, 96) if which == "dw" else (777,), device="cuda")
        a = binding.LinearCrossEntropyArgs(
            rows=150, n_in=96, vocab=777, x=x.data_ptr(), w=w.data_ptr(), bias=b.data_ptr(), targets=t.data_ptr(),
            row_weight=rw.data_ptr(), ld_x=96, ld_w=96, ld_dw=96, ignore_index=IGNORE, dtype=binding._dtype_code(x),
            grad_dtype=binding.F32, scale=0.25, **{which: out.data_ptr()})
        need = ctypes.c_int64()
        assert L.gbmuf_linear_cross_entropy_workspace(h, ctypes.byref(a), ctypes.byref(need)) == 0
        work = torch.empty(need.value, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = work.data_ptr(), need.value
        assert L.gbmuf_linear_cross_entropy(h, ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == 0
        whole = ops.linear_cross_entropy(x, w, t, b, row_weight=rw, scale=0.25, grad_dtype=F)
        assert torch.equal(out, whole[3] if which == "dw" else whole[4])


@pytest.mark.parametrize("dtype", [BF, F])
def test_words_that_cannot_occur_ignored_rows_and_nan(ops, dtype):
    g = gen(8)
    rows, n_in, vocab = 70, 40, 600
    x, w, t, b, _ = problem(g, rows, n_in, vocab, dtype, weighted=False)
    never = torch.rand(vocab, device="cuda", generator=g) < 0.4
    never[t[t != IGNORE]] = False
    t[3], never[17] = 17, True                             # the target itself cannot occur
    weight = torch.ones(rows, device="cuda")
    weight[5] = 0.0
    b[never] = -math.inf
    for piece in (0, 100):
        got = ops.linear_cross_entropy(x, w, t, b, row_weight=weight, piece=piece, grad_dtype=F)
        R = reference(x, w, t, b, weight, 1.0)
        assert float(got[0][3]) == math.inf
        ok = torch.arange(rows, device="cuda") != 3
        R["eloss"] = torch.where(ok, R["eloss"].nan_to_num(0, 0, 0), 0.0)
        inside(got[0][ok], R["loss"][ok], R["eloss"][ok], F, "loss")
        R["ed"] = R["ed"].nan_to_num(0, 0, 0)
        R["d"] = R["d"].nan_to_num(0, 0, 0)
        R["d"][3, 17] = -1.0
        tol = R["ed"] + (HALF[BF] if dtype is BF else 2.0 ** -23) * (R["d"].abs() + R["ed"])
        dw = R["d"].t() @ R["x"]
        inside(got[3], dw, tol.t() @ R["x"].abs() + (rows + 8) * 2.0 ** -23 * (R["d"].abs().t() @ R["x"].abs()), F, "dw")
        assert bool((got[3][never & (torch.arange(vocab, device="cuda") != 17)] == 0).all())
        assert bool((got[0][t == IGNORE] == 0).all()) and float(got[0][5]) == 0
        assert bool((got[2][5] == 0).all()) and bool((got[2][t == IGNORE] == 0).all())
    # no word at all: loss inf, zero gradient
    none = ops.linear_cross_entropy(x, w, t, torch.full_like(b, -math.inf), piece=200)
    valid = t != IGNORE
    assert bool((none[0][valid] == math.inf).all()) and bool((none[0][~valid] == 0).all())
    assert bool((none[1] == -math.inf).all()) and all(bool((n == 0).all()) for n in none[2:])
    # NaN and +inf stay in their rows (dw and dbias have every row in every sum)
    x2 = x.clone()
    x2[9, 1] = math.nan
    w2 = w.clone()
    first = ops.linear_cross_entropy(x, w, t, None, piece=128)
    second = ops.linear_cross_entropy(x2, w2, t, None, piece=128)
    rest = torch.arange(rows, device="cuda") != 9
    for a, c in zip(first[:3], second[:3]):
        assert torch.equal(a[rest], c[rest])
    if t[9] != IGNORE:
        assert bool(second[0][9].isnan()) and bool(second[2][9].isnan().all())
    assert bool(second[1][9].isnan())
    b3 = torch.zeros_like(b)
    b3[44] = math.inf
    third = ops.linear_cross_entropy(x, w, t, b3)
    assert bool(third[1].isnan().all()) and bool(third[0][valid].isnan().all())
    assert ops.device_status() == 0


def test_target_outside(ops):
    g = gen(9)
    x, w, t, b, _ = problem(g, 40, 24, 100, BF, weighted=False)
    good = ops.linear_cross_entropy(x, w, t, b)
    t2 = t.clone()
    for word in (100, -1, 2 ** 40, 127):
        t2[7] = word
        got = ops.linear_cross_entropy(x, w, t2, b)
        assert bool(got[0][7].isnan()) and bool((got[2][7] == 0).all()) and torch.equal(got[1], good[1])
        rest = torch.arange(40, device="cuda") != 7
        assert torch.equal(got[0][rest], good[0][rest]) and torch.equal(got[2][rest], good[2][rest])
        assert ops.device_status() == binding.ERR_INVALID_ARG
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
def test_empty(ops, dtype):
    w, b = rnd(gen(1), (50, 12), dtype), rnd(gen(2), (50,), dtype)
    none = torch.zeros((0,), dtype=torch.int64, device="cuda")
    got = ops.linear_cross_entropy(torch.zeros((0, 12), dtype=dtype, device="cuda"), w, none, b, grad_dtype=F,
                                   dw_out=torch.ones((50, 12), device="cuda"))
    assert got[0].shape == (0,) and got[2].shape == (0, 12)
    assert bool((got[3] == 0).all()) and bool((got[4] == 0).all())
    dw, db = torch.ones((50, 12), device="cuda"), torch.ones(50, device="cuda")
    ops.linear_cross_entropy(torch.zeros((0, 12), dtype=dtype, device="cuda"), w, none, b, dw_out=dw, dbias_out=db,
                             accumulate=True)
    assert bool((dw == 1).all()) and bool((db == 1).all())
    # no input at all: the logits are the bias
    t = torch.tensor([3, 49, IGNORE], device="cuda")
    x0, w0 = torch.zeros((3, 0), dtype=dtype, device="cuda"), torch.zeros((50, 0), dtype=dtype, device="cuda")
    R = reference(x0, w0, t, b, None, 1.0)
    check(ops.linear_cross_entropy(x0, w0, t, b, piece=32), R, dtype, dtype, "no input")
    with pytest.raises(binding.GbmufError):
        ops.linear_cross_entropy(torch.zeros((3, 12), dtype=dtype, device="cuda"), w[:0], t)
    assert ops.device_status() == 0


def test_gradients_against_differences(ops):
    g = gen(12)
    rows, n_in, vocab = 24, 20, 300
    x, w, t, b, rw = problem(g, rows, n_in, vocab, F)

    def objective(x, w, b):
        z = x.double() @ w.double().t() + b.double()
        keep = t != IGNORE
        per = rw.double() * (torch.logsumexp(z, 1) - z.gather(1, torch.where(keep, t, 0)[:, None])[:, 0])
        return float(torch.where(keep, per, 0.0).sum()) * 0.125

    loss, _, dx, dw, db = ops.linear_cross_entropy(x, w, t, b, row_weight=rw, scale=0.125, piece=128)
    assert abs(float(loss.double().sum()) - objective(x, w, b)) < 1e-4
    for i, grad in enumerate((dx, dw, db)):
        for turn in range(4):
            step = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)
            h = 1e-5
            at = [a.double() for a in (x, w, b)]
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * step, at[i] - h * step
            slope = (objective(*up) - objective(*down)) / (2 * h)
            # central differences: h^2 of third derivatives, 1e-16 / h of cancellation; fp32 gradients 1e-5
            assert abs(slope - float((grad.double() * step).sum())) < 1e-5 * (1 + float((grad.double() * step).abs().sum()))


@pytest.mark.parametrize("dtype", [BF, F])
def test_nothing_outside_is_written_and_bits_repeat(ops, dtype):
    g = gen(13)
    rows, n_in, vocab = 77, 50, 1203
    x, w, t, b, rw = problem(g, rows, n_in, vocab, dtype)
    bufs = []
    for r, c in ((rows, n_in), (vocab, n_in)):
        bufs.append(torch.full((r + 2, c + 7), 7.0, dtype=dtype, device="cuda"))
    db = torch.full((vocab + 2,), 7.0, dtype=dtype, device="cuda")
    first = None
    for _ in range(3):
        got = ops.linear_cross_entropy(x, w, t, b, row_weight=rw, dx_out=bufs[0][1:-1, 3:-4], dw_out=bufs[1][1:-1, 3:-4],
                                       dbias_out=db[1:-1], piece=500)
        now = [a.clone() for a in got]
        assert first is None or all(torch.equal(a, c) for a, c in zip(first, now))
        first = now
    for buf in bufs:
        edge = torch.ones_like(buf, dtype=torch.bool)
        edge[1:-1, 3:-4] = False
        assert bool((buf[edge] == 7).all())
    assert float(db[0]) == 7 and float(db[-1]) == 7
    assert all(torch.equal(a, c) for a, c in zip(first, ops.linear_cross_entropy(x, w, t, b, row_weight=rw, piece=500)))


def test_on_other_streams_and_in_graphs(ops):
    g = gen(14)
    x, w, t, b, rw = problem(g, 200, 128, 5000, BF)
    want = ops.linear_cross_entropy(x, w, t, b, row_weight=rw, piece=1024)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for got in (ops.linear_cross_entropy(x, w, t, b, row_weight=rw, piece=1024, stream=side),
                ops.linear_cross_entropy(x, w, t, b, row_weight=rw, piece=1024, stream=side.cuda_stream)):
        side.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, got))
    graphs, outs, xs = [], [], [x.clone(), x.flip(0).contiguous()]
    for xi in xs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(ops.linear_cross_entropy(xi, w, t, b, row_weight=rw, piece=1024))
        graphs.append(gr)
    for i in (0, 1, 0, 1):
        graphs[i].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, outs[0]))
    flipped = ops.linear_cross_entropy(xs[1], w, t, b, row_weight=rw, piece=1024)
    assert all(torch.equal(a, c) for a, c in zip(flipped, outs[1]))
    assert ops.device_status() == 0


@pytest.mark.parametrize("rows,n_in,vocab", [(2048, 512, 30_011), (4000, 136, 9000), (40_000, 16, 300)])
def test_large(ops, rows, n_in, vocab):
    """Several launches of the statistics, the library's own pieces."""
    x, w, t, b, rw = problem(gen(rows), rows, n_in, vocab, BF)
    got = ops.linear_cross_entropy(x, w, t, b, row_weight=rw, scale=1.0 / rows)
    check(got, reference(x, w, t, b, rw, 1.0 / rows), BF, BF, "large")
    assert ops.device_status() == 0


def test_refusals(ops):
    g = gen(15)
    x, w, t, b, rw = problem(g, 6, 8, 10, BF)
    bad = [dict(x=x.half()), dict(w=w[:, :7]), dict(w=w.float()), dict(targets=t[:5]), dict(targets=t.int()), dict(bias=b[:9]),
           dict(bias=b.float()), dict(row_weight=rw.double()), dict(x=x.cpu()), dict(x=x.t().contiguous().t()),
           dict(dx_out=torch.zeros((6, 8), device="cuda")), dict(dw_out=torch.zeros((10, 7), dtype=BF, device="cuda")),
           dict(dw_out=torch.zeros((10, 8), dtype=BF, device="cuda"), grad_dtype=F), dict(accumulate=True),
           dict(dbias_out=torch.zeros(10, dtype=BF, device="cuda"), bias=None), dict(want_grad=False, dx_out=x.clone()),
           dict(want_weight_grad=False, dw_out=w.clone()), dict(grad_dtype=torch.float16)]
    for change in bad:
        args = dict(x=x, w=w, targets=t, bias=b, row_weight=rw)
        args.update(change)
        with pytest.raises((ValueError, TypeError)):
            ops.linear_cross_entropy(**args)
    with pytest.raises(binding.GbmufError):
        ops.linear_cross_entropy(x, w, t, b, piece=-1)
    with pytest.raises(binding.GbmufError):
        ops.linear_cross_entropy(x, w, t, b, scale=math.nan)
    # too small a workspace, none, and one off alignment
    L = binding.lib()
    work = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    a = binding.LinearCrossEntropyArgs(rows=6, n_in=8, vocab=10, x=x.data_ptr(), w=w.data_ptr(), targets=t.data_ptr(), ld_x=8,
                                       ld_w=8, dtype=binding.BF16, grad_dtype=binding.BF16, scale=1.0)
    need = ctypes.c_int64()
    assert L.gbmuf_linear_cross_entropy_workspace(ops._h, ctypes.byref(a), ctypes.byref(need)) == 0 and need.value > 0
    for p, n in ((0, need.value), (work.data_ptr(), need.value - 1), (work.data_ptr() + 16, need.value)):
        a.workspace, a.workspace_bytes = p, n
        assert L.gbmuf_linear_cross_entropy(ops._h, ctypes.byref(a), None) == binding.ERR_INVALID_ARG
        assert b"workspace" in L.gbmuf_last_error(None)
    assert ops.device_status() == 0


def test_weights_past_two_to_the_31(ops):
    """270,001 words of 8,000 bf16: the last words' gradients."""
    g = gen(16)
    rows, n_in, vocab = 40, 8000, 270_001
    x = rnd(g, (rows, n_in), BF)
    w = torch.empty((vocab, n_in), dtype=BF, device="cuda").normal_(0.0, 2.0 * n_in ** -0.5, generator=g)
    t = torch.randint(vocab - 50, vocab, (rows,), device="cuda", generator=g)
    loss, lse, dx, dw = ops.linear_cross_entropy(x, w, t, scale=1.0 / rows)
    z = torch.cat([x.double() @ part.double().t() for part in w.split(30_000)], 1)
    ref = torch.logsumexp(z, 1)
    # z: an fp32 sum of 8,000 products, each step off by at most 2^-23 of a partial sum
    ez = 8008 * 2.0 ** -23 * float((x.double().abs() @ w[-500:].double().abs().t()).max())
    assert float((lse.double() - ref).abs().max()) <= ez + 1e-2
    assert float((loss.double() * rows - (ref - z.gather(1, t[:, None])[:, 0])).abs().max()) <= 2 * ez + 1e-2
    d = (torch.exp(z - ref[:, None]) - torch.zeros_like(z).scatter_(1, t[:, None], 1.0)) / rows
    for words in (slice(0, 300), slice(vocab - 300, vocab)):
        exact = d[:, words].t() @ x.double()
        assert float((dw[words].double() - exact).norm()) <= 2.0 ** -7 * float(exact.norm())
    exact = torch.zeros((rows, n_in), dtype=torch.float64, device="cuda")
    for a in range(0, vocab, 30_000):
        exact += d[:, a:a + 30_000] @ w[a:a + 30_000].double()
    close(dx, exact, BF, "dx")
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,piece", [(3, 0), (300, 0), (142, 1500)])
def test_the_scale_is_a_factor_of_finished_sums(ops, dtype, rows, piece):
    """A mean's 1 / rows takes no digits from the gradients: they are those of scale 1, multiplied once."""
    g = gen(91)
    x, w, t, b, weight = problem(g, rows, 200, 4001, dtype, weighted=rows == 142)
    scale = torch.tensor(1.0 / rows, dtype=F).item()
    one, got = (ops.linear_cross_entropy(x, w, t, b, ignore_index=IGNORE, row_weight=weight, scale=s, grad_dtype=F,
                                         piece=piece) for s in (1.0, scale))
    for i, what in ((3, "dw"), (4, "dbias")) + (((2, "dx"),) if dtype is F else ()):
        assert torch.equal(got[i], one[i] * scale), what
    assert ops.device_status() == 0


def test_a_mean_over_any_rows_is_as_exact_as_a_sum(ops):
    """bf16, p small beside a target's 1: of d / scale a target's -1 + p, p < 2^-9, is rounded to -1 and so off by p, the
    others by half a step.  1 / 300 rounded to bf16 is 2.1e-3 off; dw, projected on the exact one, must not be."""
    g = gen(92)
    rows, n_in, vocab = 300, 256, 20000
    x, w, t, b, _ = problem(g, rows, n_in, vocab, BF, weighted=False, spread=0.25)
    R = reference(x, w, t, b, None, 1.0 / rows)
    got = ops.linear_cross_entropy(x, w, t, b, ignore_index=IGNORE, scale=1.0 / rows, grad_dtype=F)
    p = torch.exp(R["z"] - R["lse"][:, None]) * (t != IGNORE)[:, None] / rows
    valid = (t != IGNORE).nonzero()[:, 0]
    off = HALF[BF] * p
    off[valid, t[valid]] = p[valid, t[valid]]
    assert float(off[valid, t[valid]].max()) * rows < 2.0 ** -9
    exact = R["d"].t() @ R["x"]
    bound = float(((off + R["ed"]).t() @ R["x"].abs()).norm() / exact.norm()) + rows * 2.0 ** -23
    assert bound < 1e-3
    mean = float((got[3].double() * exact).sum() / exact.square().sum())
    assert abs(mean - 1) < bound, (mean, bound)
    assert ops.device_status() == 0


@pytest.mark.parametrize("rows,n_in,vocab,piece", [(1, 64, 1000, 0), (1, 70, 4001, 1000), (2, 1024, 5003, 0), (5, 33, 20_000, 0),
                                                  (9, 512, 3001, 0), (31, 515, 1027, 300), (32, 256, 40_001, 0)])
def test_few_rows_have_two_parts(ops, rows, n_in, vocab, piece):
    """bf16, up to 32 rows: d is taken as two bf16 parts, the second one of what the first one's rounding left, so it is
    off by half a step of half a step; dw and dbias are asked for in fp32."""
    g = gen(rows + n_in + vocab)
    x, w, t, b, rw = problem(g, rows, n_in, vocab, BF)
    R = reference(x, w, t, b, rw, 1.0 / rows)
    d, ed = R["d"], R["ed"]
    er = ed + HALF[BF] ** 2 * (d.abs() + ed)
    for how in ("plain", "odd"):
        got = ops.linear_cross_entropy(lay(x, how), lay(w, how), t, lay(b, how), ignore_index=IGNORE, row_weight=rw,
                                       scale=1.0 / rows, grad_dtype=F, piece=piece)
        inside(got[0], R["loss"], R["eloss"], F, "loss")
        inside(got[2], d @ R["w"], er @ R["w"].abs() + (vocab + 8) * 2.0 ** -23 * (d.abs() @ R["w"].abs()), BF, "dx")
        inside(got[3], d.t() @ R["x"], er.t() @ R["x"].abs() + (2 * rows + 8) * 2.0 ** -23 * (d.abs().t() @ R["x"].abs()), F, "dw")
        inside(got[4], d.sum(0), ed.sum(0) + (rows + 8) * 2.0 ** -23 * d.abs().sum(0), F, "dbias")
    assert ops.device_status() == 0
