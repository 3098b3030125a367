"""The largest logits of a row (``top_logits``) and distillation from them (``distillation``) against plain
64-bit formulas."""
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
    if how == "plain":
        return t
    r, c = t.shape
    pad, off = {"padded": (24, 0), "odd": (5, 3)}[how]
    fill = -7 if t.dtype is torch.int64 else math.nan
    buf = torch.full((r * (c + pad) + off,), fill, dtype=t.dtype, device=t.device)
    v = buf[off:].view(r, c + pad)[:, :c]
    v.copy_(t)
    return v


# ---------------------------------------------------------------------------------------- the largest logits
def largest(x, k):
    """Indices of the k largest, NaN first, lower indices first among equal ones."""
    key = torch.where(x.isnan(), math.inf, x.double() + 0.0)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    nan_first = torch.sort(x.gather(1, order).isnan().int(), dim=1, descending=True, stable=True).indices
    return order.gather(1, nan_first)[:, :k]


def lse_tolerance(lse, vocab):
    # exponentials 2^-21 and the rounding of their exponents; at most vocab / 8 additions in a running sum
    return 2.0 ** -20 + (vocab / 8 + 64) * 2.0 ** -24 + 2.0 ** -22 * lse.abs()


def check_top(ops, x, k, T=1.0, how="plain", **kw):
    values, index, lse = ops.top_logits(lay(x, how), k, temperature=T, **kw)
    want = largest(x, k)
    assert torch.equal(index, want)
    got = values.view(torch.int16 if x.dtype is BF else torch.int32)
    assert torch.equal(got, x.gather(1, want).view(got.dtype))
    ref = torch.logsumexp(x.double() / T, 1)
    finite = ~(x.isnan() | (x == math.inf)).any(1)
    assert bool(lse[~finite].isnan().all())
    empty = finite & (ref == -math.inf)
    assert bool((lse[empty] == -math.inf).all())
    some = finite & ~empty
    assert bool(((lse[some].double() - ref[some]).abs() <= lse_tolerance(ref[some], x.shape[1])).all())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (5, 256), (40, 300), (9, 1000), (700, 2048), (1, 2049), (2, 4100),
                                        (33, 10_000), (600, 5003), (7, 50_001), (1, 267_735), (300, 33_278), (40, 267_735)])
def test_top(ops, dtype, rows, vocab):
    g = gen(rows + vocab)
    for i, k in enumerate([1, 2, 16, 65, 256]):
        if k <= vocab:
            check_top(ops, rnd(g, (rows, vocab), dtype, 3.0), k, [1.0, 2.0, 0.5][i % 3], ["plain", "padded", "odd"][(i + rows) % 3])
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,vocab", [(6, 1500), (2, 9000), (400, 8195)])
def test_top_of_hard_rows(ops, dtype, rows, vocab):
    """Equal values, rising and falling rows, few values, masked words, infinities, NaN."""
    g = gen(vocab)
    ramp = torch.arange(vocab, device="cuda", dtype=torch.float32)
    base = rnd(g, (rows, vocab), dtype)
    cases = [torch.zeros_like(base), torch.full_like(base, -math.inf), ramp.expand(rows, -1).to(dtype).contiguous(),
             (-ramp).expand(rows, -1).to(dtype).contiguous(), torch.randint(0, 3, base.shape, device="cuda", generator=g).to(dtype),
             torch.where(torch.rand(base.shape, device="cuda", generator=g) < 0.999, -math.inf, base.float()).to(dtype),
             torch.where(torch.rand(base.shape, device="cuda", generator=g) < 0.01, math.inf, base.float()).to(dtype),
             torch.where(torch.rand(base.shape, device="cuda", generator=g) < 0.02, math.nan, base.float()).to(dtype),
             torch.full_like(base, math.nan), torch.full_like(base, torch.finfo(dtype).min),
             torch.where(torch.rand(base.shape, device="cuda", generator=g) < 0.5, -0.0, 0.0).to(dtype), base * 1e-40]
    last = torch.zeros_like(base)
    last[:, -1] = 1.0
    cases += [last, torch.sort(base, dim=1).values]
    for x in cases:
        for k in (1, 50, 256):
            check_top(ops, x, k)
    assert ops.device_status() == 0


def test_top_results_handed_in_streams_graphs(ops):
    g = gen(3)
    x = rnd(g, (20, 5000), BF)
    want = ops.top_logits(x, 10)
    values, index = torch.full((22, 14), 9.0, dtype=BF, device="cuda"), torch.full((22, 13), 9, device="cuda")
    lse = torch.zeros(20, device="cuda")
    got = ops.top_logits(x, 10, values_out=values[1:-1, 2:-2], index_out=index[1:-1, 1:-2], lse_out=lse)
    assert got[2] is lse and all(torch.equal(a, b) for a, b in zip(got, want))
    assert int((values == 9).sum()) >= 22 * 14 - 200 and int((index != 9).sum()) <= 200
    assert bool((index[0] == 9).all()) and bool((index[:, 0] == 9).all()) and bool((index[:, -2:] == 9).all())
    assert len(ops.top_logits(x, 10, want_lse=False)) == 2
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = ops.top_logits(x, 10, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want))
    graphs = []
    for xi in (x, x.flip(1).contiguous()):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = ops.top_logits(xi, 10)
        graphs.append((gr, out, xi))
    for gr, _, _ in graphs + graphs:
        gr.replay()
    torch.cuda.synchronize()
    for _, out, xi in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, ops.top_logits(xi, 10)))
    empty = ops.top_logits(torch.zeros((0, 50), device="cuda"), 3)
    assert empty[0].shape == (0, 3) and empty[2].shape == (0,)
    assert ops.device_status() == 0


def test_top_refusals(ops):
    x = torch.zeros((4, 20), device="cuda")
    for args, kw in [((x, 0), {}), ((x, 257), {}), ((x.half(), 3), {}), ((x[0], 3), {}), ((x.cpu(), 3), {}), ((x.t(), 3), {}),
                     ((x, 3), dict(values_out=torch.zeros((4, 2), device="cuda"))),
                     ((x, 3), dict(index_out=torch.zeros((4, 3), dtype=torch.int32, device="cuda"))),
                     ((x, 3), dict(lse_out=torch.zeros(5, device="cuda")))]:
        with pytest.raises((ValueError, TypeError)):
            ops.top_logits(*args, **kw)
    for args, kw in [((x, 21), {}), ((x, 3), dict(temperature=0.0)), ((x, 3), dict(temperature=math.nan)),
                     ((x, 3), dict(temperature=2000.0)), ((x[:, :0], 3), {})]:
        with pytest.raises(binding.GbmufError):
            ops.top_logits(*args, **kw)


# ---------------------------------------------------------------------------------------- distillation
def lists(g, x, k, T, teacher_dtype, noise=1.5):
    """A teacher near the student: its k largest logits, their words, its log-sum-exp."""
    teacher = (1.1 * x.double().clamp(-1e4, 1e4) + noise * torch.randn(x.shape, generator=g, device="cuda").double()).to(teacher_dtype)
    index = torch.sort(teacher.double(), dim=1, descending=True, stable=True).indices[:, :k].contiguous()
    return teacher.gather(1, index), index, torch.logsumexp(teacher.double() / T, 1).float()


def reference(x, t, ix, tlse, T, targets, h, weight, scale):
    """Loss, lse and gradient, and bounds on the error of what the call computes.  Entries that are not there have a
    logit of -inf (and any valid index).

    p: exponentials 2^-21, their exponents' rounding, running sums of at most vocab / 8 additions (ep relative);
    q: an exponential of a difference rounded to fp32 (eq); q_r: the q's errors."""
    x, t = x.double(), t.double()
    rows, vocab = x.shape
    # relative to the row's largest logit: with the type's lowest value in every place, log sum exp itself holds no
    # digit of log(vocab), in 64 bits either
    high = x.amax(1, keepdim=True)
    high = torch.where(high.isfinite(), high, 0.0)
    x = x - high
    u, a = x / T, t / T
    there = t != -math.inf
    lse = torch.logsumexp(u, 1, keepdim=True)
    log_q = a - (torch.logsumexp(a, 1, keepdim=True) if tlse is None else tlse.double()[:, None])
    q = torch.where(there, log_q.exp(), 0.0)
    log_q = torch.where(there, log_q, 0.0)
    lp = torch.where(there, u.gather(1, ix) - lse, 0.0)
    p = torch.exp(u - lse)
    Q = torch.zeros_like(p).scatter_add_(1, ix, q)
    listed = torch.zeros_like(p).scatter_add_(1, ix, there.double()) > 0
    soft = torch.where(q > 0, q * (log_q - lp), 0.0).sum(1)
    mass = q.sum(1)
    off = (u.amax(1, keepdim=True) - u).abs().nan_to_num(0, 0, 0)
    ep = 2.0 ** -19 + (vocab / 8 + 64) * 2.0 ** -24 + 2.0 ** -22 * off
    eq = 2.0 ** -21 + 2.0 ** -22 * (log_q.abs() + (0 if tlse is not None else 4))
    spread = 2.0 ** -21 * (log_q.abs() + lp.abs()) + ep.amin(1, keepdim=True)
    esoft = (q * (eq * (1 + (log_q - lp).abs().nan_to_num(0, 0, 0)) + spread.nan_to_num(0, 0, 0))).sum(1)
    d = p * mass[:, None] - Q
    ed = p * (mass[:, None] * ep + (q * eq).sum(1, keepdim=True)) + torch.zeros_like(p).scatter_add_(1, ix, q * eq)
    if tlse is not None:
        rest = listed.sum(1) < vocab
        q_r = torch.where(rest, (1 - mass).clamp(min=0), 0.0)
        p_r = torch.where(listed, 0.0, p).sum(1)
        log_pr = torch.logsumexp(torch.where(listed, -math.inf, u), 1) - lse[:, 0]
        soft = soft + torch.where(q_r > 0, q_r * (q_r.log() - log_pr), 0.0)
        eqr = (q * eq).sum(1) + 2.0 ** -23
        esoft = esoft + torch.where(rest, eqr * (2 + (eqr + q_r).log().abs() + log_pr.abs()), 0.0) + \
            q_r * (ep.amin(1) + 2.0 ** -21 * log_pr.abs().nan_to_num(0, 0, 0))
        share = torch.where(p_r > 0, q_r / p_r, 0.0)[:, None]
        more = torch.where(rest & (p_r > 0), eqr / p_r, 0.0)[:, None]
        d = torch.where(listed, p * (mass + q_r)[:, None] - Q, p * ((mass + q_r)[:, None] - share))
        ed = ed + p * (eqr + q_r)[:, None] * ep + torch.where(listed, 0.0, p * (share * 2 * ep + more))
    loss, eloss = (1 - h) * T * T * soft, (1 - h) * T * T * esoft
    d, ed = (1 - h) * T * d, (1 - h) * T * ed
    s = scale * (torch.ones(rows, device="cuda").double() if weight is None else weight.double())
    if targets is not None:
        s = torch.where(targets == IGNORE, 0.0, s)
        if h > 0:
            at = torch.where(targets == IGNORE, 0, targets)[:, None]
            lse1 = torch.logsumexp(x, 1, keepdim=True)
            xt = x.gather(1, at)
            p1 = torch.exp(x - lse1)
            ep1 = 2.0 ** -19 + (vocab / 8 + 64) * 2.0 ** -24 + 2.0 ** -22 * off * T
            loss = loss + h * (lse1 - xt)[:, 0]
            eloss = eloss + h * (ep1.amin(1) + 2.0 ** -22 * (x.amax(1) - xt[:, 0]).abs())
            d = d + h * (p1 - torch.zeros_like(p).scatter_(1, at, 1.0))
            ed = ed + h * (p1 * ep1 + torch.zeros_like(p).scatter_(1, at, 2.0 ** -23))
    zero = (s == 0)[:, None]
    return dict(loss=torch.where(s == 0, 0.0, s * loss), eloss=s.abs() * (eloss + 2.0 ** -22 * loss.abs()), lse=lse[:, 0] + high[:, 0] / T,
                d=torch.where(zero, 0.0, s[:, None] * d), ed=s.abs()[:, None] * (ed + 2.0 ** -22 * d.abs()))


def check(got, R, dtype, vocab, what):
    def inside(name, value, ref, tol, kind):
        assert value.dtype is kind and value.shape == ref.shape
        err = (value.double() - ref).abs()
        bad = ~(err <= tol + HALF[kind] * (ref.abs() + tol)) & ~(value.double() == ref)     # equal infinities
        assert not bad.any(), f"{what} {name}: {int(bad.sum())} of {bad.numel()} outside, worst {float(err.max()):.3g}"
    inside("lse", got[1], R["lse"], lse_tolerance(R["lse"], vocab), F)
    inside("loss", got[0], R["loss"], R["eloss"], F)
    if len(got) > 2:
        inside("gradient", got[2], R["d"], R["ed"], dtype)


SETTINGS = [dict(T=1.0, rest=False, h=0.0), dict(T=2.0, rest=True, h=0.0), dict(T=1.0, rest=True, h=0.3),
            dict(T=3.0, rest=False, h=0.5), dict(T=1.5, rest=True, h=0.25), dict(T=0.5, rest=True, h=1.0)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 5), (6, 64), (30, 256), (65, 1000), (40, 2048), (1, 2049), (3, 4100), (33, 10_000),
                                        (310, 6007), (5, 50_001), (600, 33_278), (2, 267_735), (150, 131_071)])
def test_distillation(ops, dtype, rows, vocab):
    g = gen(rows * 3 + vocab)
    for i, c in enumerate(SETTINGS):
        k = min(vocab, [1, 8, 50, 64, 256, 33][i])
        how = ["plain", "padded", "odd"][(i + rows) % 3]
        x = rnd(g, (rows, vocab), dtype, 2.5)
        t, ix, tlse = lists(g, x, k, c["T"], [BF, F][i % 2])
        targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
        targets[::3] = ix[::3, 0]                          # some targets are in the list
        if rows > 2:
            targets[torch.rand(rows, device="cuda", generator=g) < 0.15] = IGNORE
        weight = torch.rand(rows, device="cuda", generator=g) + 0.5 if i % 2 else None
        given = targets if c["h"] > 0 or i % 2 else None
        R = reference(x, t, ix, tlse if c["rest"] else None, c["T"], given, c["h"], weight, 0.25)
        kw = dict(teacher_lse=tlse if c["rest"] else None, temperature=c["T"], targets=given, hard_weight=c["h"], row_weight=weight,
                  scale=0.25)
        got = ops.distillation(lay(x, how), lay(t, how), lay(ix, how), dlogits_out=lay(torch.zeros_like(x), how), **kw)
        check(got, R, dtype, vocab, f"{i} {how}")
        place = lay(x.clone(), how)
        inplace = ops.distillation(place, t, ix, dlogits_out=place, **kw)
        assert inplace[2] is place and all(torch.equal(a, b) for a, b in zip(got, inplace))
        alone = ops.distillation(x, t, ix, want_grad=False, **kw)
        check(alone, R, dtype, vocab, f"{i} loss alone")
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("vocab", [700, 5000])
def test_distillation_short_lists_and_words_that_come_twice(ops, dtype, vocab):
    g = gen(vocab)
    rows, k = 40, 24
    x = rnd(g, (rows, vocab), dtype, 2.0)
    t, ix, tlse = lists(g, x, k, 2.0, F)
    # entries that are not there: index -1, or a logit of -inf; row 4 has none at all
    gone = torch.rand((rows, k), device="cuda", generator=g) < 0.3
    gone[4] = True
    how = torch.rand((rows, k), device="cuda", generator=g) < 0.5
    given_ix = torch.where(gone & how, -1, ix)
    given_t = torch.where(gone & ~how, -math.inf, t)
    ref_t = torch.where(gone, -math.inf, t)
    for rest in (False, True):
        R = reference(x, ref_t, ix, tlse if rest else None, 2.0, None, 0.0, None, 1.0)
        if not rest:                                       # no entry: nothing to learn
            for name in ("loss", "eloss", "d", "ed"):
                R[name][4] = 0.0
        got = ops.distillation(x, given_t, given_ix, teacher_lse=tlse if rest else None, temperature=2.0)
        check(got, R, dtype, vocab, f"short lists {rest}")
    # the same words again and again, in one thread's pieces, with targets among them
    ix2 = ix.clone()
    ix2[:, 5], ix2[:, 9], ix2[:, 20] = ix[:, 3], ix[:, 3], ix[:, 7]
    ix2[11] = 17
    ix2[12] = (torch.arange(k, device="cuda") % 3) + 8 * torch.arange(k, device="cuda").div(3, rounding_mode="floor")
    targets = ix2[:, 9].clone()
    for rest in (False, True):
        kw = dict(temperature=2.0, targets=targets, hard_weight=0.5)
        R = reference(x, t, ix2, tlse if rest else None, 2.0, targets, 0.5, None, 1.0)
        first = ops.distillation(x, t, ix2, teacher_lse=tlse if rest else None, **kw)
        check(first, R, dtype, vocab, f"twice {rest}")
        for _ in range(5):
            assert all(torch.equal(a, b) for a, b in zip(first, ops.distillation(x, t, ix2, teacher_lse=tlse if rest else None, **kw)))
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("vocab", [9, 1200, 6000])
def test_distillation_masked_and_not_finite(ops, dtype, vocab):
    g = gen(vocab + 1)
    rows, k = 12, 8
    x = rnd(g, (rows, vocab), dtype, 2.0)
    t, ix, tlse = lists(g, x, k, 1.0, dtype)
    x[0, ix[0, 2]] = -math.inf                             # cannot occur, but the teacher says it does: loss inf
    never = torch.rand(vocab, device="cuda", generator=g) < 0.5
    never[ix[1]] = False
    x[1, never] = -math.inf                                # words outside the list that cannot occur
    x[2] = -math.inf                                       # nothing can
    x[3, vocab // 2] = math.nan
    x[4, vocab - 1] = math.inf
    t[5, 1] = math.nan
    x[6] = torch.finfo(dtype).min                          # equal, and at the lowest value
    keep = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    keep[ix[7]] = True
    x[7, ~keep] = -math.inf                                # no word outside the list can occur: P_r = 0
    x[8] += 1e4                                            # a large common offset
    weight = torch.ones(rows, device="cuda")
    weight[9] = 0.0
    x[9] = math.nan                                        # and is ignored
    for rest in (False, True):
        got = ops.distillation(x, t, ix, teacher_lse=tlse if rest else None, row_weight=weight)
        R = reference(x, t, ix, tlse if rest else None, 1.0, None, 0.0, weight, 1.0)
        assert float(got[0][0]) == math.inf and bool(got[2][0].isfinite().all())
        assert float(got[0][2]) == math.inf and float(got[1][2]) == -math.inf and bool((got[2][2] == 0).all())
        for r in (3, 4):
            assert bool(got[0][r].isnan()) and bool(got[1][r].isnan()) and bool(got[2][r].isnan().all())
        assert bool(got[0][5].isnan()) and bool(got[2][5].isnan().all()) and bool(got[1][5].isfinite())
        if rest and float((1 - torch.exp(t[7].double() - tlse[7].double()).sum())) > 1e-5:
            assert float(got[0][7]) == math.inf and bool(got[2][7].isfinite().all())
        assert float(got[0][9]) == 0 and bool((got[2][9] == 0).all())
        rows_left = [1, 6, 8, 10, 11] + ([] if rest else [7])
        if rest and dtype is F:
            rows_left.remove(8)                            # the teacher's list was made before the offset: fp32 rounds it
        pick = torch.tensor(rows_left, device="cuda")
        check([v[pick] for v in got], {n: v[pick] for n, v in R.items()}, dtype, vocab, f"rest {rest}")
    assert ops.device_status() == 0
    bad = ix.clone()
    for word in (vocab, -2, 2 ** 40):
        bad[10, 3] = word
        got2 = ops.distillation(x, t, bad, row_weight=weight)
        assert bool(got2[0][10].isnan()) and bool((got2[2][10] == 0).all())
        assert torch.equal(got2[2][11], ops.distillation(x, t, ix, row_weight=weight)[2][11])
        assert ops.device_status() == binding.ERR_INVALID_ARG
    targets = torch.zeros(rows, dtype=torch.int64, device="cuda")
    targets[11] = vocab
    got3 = ops.distillation(x, t, ix, targets=targets, row_weight=weight)
    assert bool(got3[0][11].isnan()) and bool((got3[2][11] == 0).all()) and ops.device_status() == binding.ERR_INVALID_ARG
    assert ops.device_status() == 0


def test_distillation_gradient_against_differences(ops):
    g = gen(21)
    rows, vocab, k = 9, 400, 12
    x = rnd(g, (rows, vocab), F, 1.5)
    for T, rest, h in ((1.0, True, 0.0), (2.5, True, 0.4), (2.0, False, 0.2)):
        t, ix, tlse = lists(g, x, k, T, F)
        targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
        loss, _, d = ops.distillation(x, t, ix, teacher_lse=tlse if rest else None, temperature=T, targets=targets, hard_weight=h)

        def objective(y):
            u = y / T
            lse = torch.logsumexp(u, 1, keepdim=True)
            a = t.double() / T
            lq = a - (tlse.double()[:, None] if rest else torch.logsumexp(a, 1, keepdim=True))
            total = (lq.exp() * (lq - (u.gather(1, ix) - lse))).sum(1)
            if rest:
                q_r = (1 - lq.exp().sum(1)).clamp(min=0)
                total = total + q_r * (q_r.log() - (torch.logsumexp(u.scatter(1, ix, -math.inf), 1) - lse[:, 0]))
            hard = torch.logsumexp(y, 1) - y.gather(1, targets[:, None])[:, 0]
            return float(((1 - h) * T * T * total + h * hard).sum())

        y = x.double()
        assert abs(float(loss.double().sum()) - objective(y)) < 1e-4
        for _ in range(4):
            step = torch.randn(y.shape, generator=g, device="cuda", dtype=torch.float64)
            slope = (objective(y + 1e-5 * step) - objective(y - 1e-5 * step)) / 2e-5
            # central differences: 1e-10 of third derivatives, 1e-16 / 1e-5 of cancellation; fp32 gradients 1e-5
            assert abs(slope - float((d.double() * step).sum())) < 1e-5 * (1 + float((d.double() * step).abs().sum()))
    assert ops.device_status() == 0


def test_distillation_streams_graphs_and_repeats(ops):
    g = gen(22)
    x = rnd(g, (500, 9001), BF, 2.0)
    t, ix, tlse = lists(g, x, 40, 2.0, BF)
    call = lambda a, **kw: ops.distillation(a, t, ix, teacher_lse=tlse, temperature=2.0, **kw)      # noqa: E731
    want = call(x)
    for _ in range(10):
        assert all(torch.equal(a, b) for a, b in zip(want, call(x)))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = call(x, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graphs = []
    for xi in (x, x.flip(0).contiguous()):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = call(xi)
        graphs.append((gr, out, xi))
    for gr, _, _ in graphs + graphs:
        gr.replay()
    torch.cuda.synchronize()
    for _, out, xi in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, call(xi)))
    none = ops.distillation(x[:0], t[:0], ix[:0])
    assert none[0].shape == (0,) and none[2].shape == (0, 9001)
    assert ops.device_status() == 0


def test_teacher_to_student(ops):
    """The operators in a row: a teacher's lists, a student's scores, the mixed loss, the layer's gradients."""
    g = gen(23)
    rows, width, vocab, T, h = 96, 64, 3001, 2.0, 0.3
    x = rnd(g, (rows, width), F)
    w_teacher, w = rnd(g, (vocab, width), F, 0.3), rnd(g, (vocab, width), F, 0.3)
    targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    t, ix, tlse = ops.top_logits(ops.linear_forward(x, w_teacher), 32, temperature=T)
    scores = ops.linear_forward(x, w)
    loss, _, d = ops.distillation(scores, t, ix, teacher_lse=tlse, temperature=T, targets=targets, hard_weight=h,
                                  scale=1.0 / rows, dlogits_out=scores)
    dw = ops.linear_backward_weight(d, x, want_bias=False)
    wd = w.double().requires_grad_()
    teacher = x.double() @ w_teacher.double().t() / T
    s = x.double() @ wd.t()
    q = torch.softmax(teacher, 1).gather(1, ix)
    lp = torch.log_softmax(s / T, 1)
    q_r = 1 - q.sum(1)
    lr = torch.logsumexp(lp.scatter(1, ix, -math.inf), 1)
    soft = (q * (q.log() - lp.gather(1, ix))).sum(1) + q_r * (q_r.log() - lr)
    total = ((1 - h) * T * T * soft - h * torch.log_softmax(s, 1).gather(1, targets[:, None])[:, 0]).mean()
    total.backward()
    total = total.detach()
    # fp32 throughout: logits of about 3 off by 1e-6, probabilities by as much, relative
    assert abs(float(loss.sum()) - float(total)) < 1e-4
    assert float((dw.double() - wd.grad).norm() / wd.grad.norm()) < 1e-5
    assert ops.device_status() == 0


def test_distillation_refusals(ops):
    x = torch.zeros((4, 20), device="cuda")
    t, ix = torch.zeros((4, 3), device="cuda"), torch.zeros((4, 3), dtype=torch.int64, device="cuda")
    for change in [dict(logits=x.half()), dict(teacher_logits=t.half()), dict(teacher_logits=t[:3]), dict(teacher_index=ix.int()),
                   dict(teacher_index=ix[:, :2]), dict(teacher_lse=torch.zeros(3, device="cuda")), dict(row_weight=torch.zeros(4)),
                   dict(targets=torch.zeros(4, device="cuda")), dict(dlogits_out=x.bfloat16()), dict(teacher_logits=t.cpu())]:
        args = dict(logits=x, teacher_logits=t, teacher_index=ix)
        args.update(change)
        with pytest.raises((ValueError, TypeError)):
            ops.distillation(**args)
    targets = torch.zeros(4, dtype=torch.int64, device="cuda")
    for kw in [dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.inf), dict(hard_weight=0.5),
               dict(hard_weight=1.5, targets=targets), dict(hard_weight=-0.1, targets=targets), dict(scale=math.nan),
               dict(hard_weight=math.nan, targets=targets)]:
        with pytest.raises(binding.GbmufError):
            ops.distillation(x, t, ix, **kw)
    with pytest.raises(binding.GbmufError):
        ops.distillation(x, torch.zeros((4, 257), device="cuda"), torch.zeros((4, 257), dtype=torch.int64, device="cuda"))
    with pytest.raises(binding.GbmufError):
        ops.distillation(x, t[:, :0], ix[:, :0])
    assert ops.device_status() == 0


def test_two_streams_at_once(ops):
    """All three operators on two streams side by side, again and again, give the bits of one after another."""
    g = gen(31)
    jobs = []
    for rows, vocab, dtype in ((300, 20_011, BF), (150, 9_001, F)):
        x = rnd(g, (rows, vocab), dtype, 2.0)
        t, ix, tlse = lists(g, x, 30, 2.0, dtype)
        h, w, b = rnd(g, (rows, 72), dtype), rnd(g, (vocab, 72), dtype, 0.2), rnd(g, (vocab,), dtype)
        targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
        jobs.append(lambda x=x, t=t, ix=ix, tlse=tlse, h=h, w=w, b=b, targets=targets: (
            *ops.top_logits(x, 20), *ops.distillation(x, t, ix, teacher_lse=tlse, temperature=2.0, targets=targets, hard_weight=0.2),
            *ops.linear_cross_entropy(h, w, targets, b, piece=4000)))
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results = []
    for _ in range(10):
        for job, s in zip(jobs, streams):
            with torch.cuda.stream(s):
                results.append(job())
    torch.cuda.synchronize()
    for i, got in enumerate(results):
        assert all(torch.equal(a, b) for a, b in zip(want[i % 2], got))
    assert ops.device_status() == 0


@pytest.mark.parametrize("rows,vocab", [(1, 2_000_003), (2, 700_001)])
def test_very_long_rows(ops, rows, vocab):
    """Rows of many chunks: groups of several chunks in the largest logits, every slice fetched twice in distillation."""
    g = gen(vocab)
    for dtype in (BF, F):
        x = rnd(g, (rows, vocab), dtype, 2.0)
        check_top(ops, x, 100)
        t, ix, tlse = lists(g, x, 40, 2.0, dtype)
        R = reference(x, t, ix, tlse, 2.0, None, 0.0, None, 1.0)
        check(ops.distillation(x, t, ix, teacher_lse=tlse, temperature=2.0), R, dtype, vocab, "long")
    many = rnd(g, (40, 400_003), F, 2.0)                   # a block to a row: more chunks than groups
    check_top(ops, many.repeat(8, 1), 64)
    assert ops.device_status() == 0


def test_logits_past_two_to_the_31(ops):
    """8,100 x 267,735 bf16 logits: the last rows, in place."""
    g = gen(41)
    rows, vocab, k = 8100, 267_735, 20
    x = torch.empty((rows, vocab), dtype=BF, device="cuda").normal_(0.0, 2.0, generator=g)
    last = x[-40:].clone()
    values, index, lse = ops.top_logits(x, k, temperature=2.0)
    want = largest(last, k)
    assert torch.equal(index[-40:], want) and torch.equal(values[-40:], last.gather(1, want))
    t = values.float() + 0.5
    out = ops.distillation(x, t, index, temperature=2.0, dlogits_out=x)
    R = reference(last, t[-40:], index[-40:], None, 2.0, None, 0.0, None, 1.0)
    check([v[-40:] for v in out], R, BF, vocab, "last rows")
    assert ops.device_status() == 0
