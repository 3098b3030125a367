"""Gradients of ``linear_cross_entropy`` that are not off to one side; batches that take several launches of the statistics."""
import pytest
import torch

from paper_1909_09010_b200 import binding
from test_gpu_linear_loss import BF, F, HALF, IGNORE, check, gen, lay, problem, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    return binding.local_ops(0)


@pytest.mark.parametrize("rows,n_in,vocab,piece", [(33, 64, 4001, 0), (300, 200, 4001, 1500), (513, 72, 10_000, 0), (140_001, 8, 100, 0)])
@pytest.mark.parametrize("value", [1.0 / 300, 1.0 / 513, 0.7, 3e-30])
def test_equal_weights_are_a_scale(ops, rows, n_in, vocab, piece, value):
    """The same call written twice: the same weight for all rows, or as their scale; a mask divided by its count, or rows
    without a target.  bf16, where the gradient of the logits is rounded: a weight within it would be rounded the same
    way in every row (1 / 300 is 2.1e-3 off), so it must not be there; the bits are the same."""
    value = torch.tensor(value, dtype=F).item()
    x, w, t, b, _ = problem(gen(rows + n_in), rows, n_in, vocab, BF, weighted=False)
    kw = dict(ignore_index=IGNORE, grad_dtype=F, piece=piece)
    want = ops.linear_cross_entropy(x, w, t, b, scale=value, **kw)
    got = ops.linear_cross_entropy(x, w, t, b, row_weight=torch.full((rows,), value, device="cuda"), **kw)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    # rows that are not counted have any weight
    mask = torch.where(t == IGNORE, 1e9, value)
    assert all(torch.equal(a, c) for a, c in zip(ops.linear_cross_entropy(x, w, t, b, row_weight=mask, **kw), want))
    # and the mask itself: weight 0 instead of a target that is ignored
    mask, there = torch.where(t == IGNORE, 0.0, value), torch.where(t == IGNORE, 3, t)
    assert all(torch.equal(a, c) for a, c in zip(ops.linear_cross_entropy(x, w, there, b, row_weight=mask, **kw), want))
    assert ops.device_status() == 0


def along(got, exact):
    """What part of `exact` is in `got`: 1 where errors go to all sides."""
    return float((got.double() * exact).sum() / exact.square().sum())


def off_along(p, p_target, at, ed, part):
    """How far the rounding of d to bf16 may move that number; part: what an element of d does to it.  With a target's
    factor of 1 and p < 2^-9, -1 + p is rounded to -1, off by p.  The others are off by half a step of p at most, to either
    side: by Hoeffding's inequality 8 times the root of the squares' sum is passed with probability 2 e^-32.  ed: before."""
    target = float((p_target[:, None] * part.gather(1, at).abs()).sum())
    return target + 8 * HALF[BF] * float((p * part).square().sum()) ** 0.5 + float((ed * part.abs()).sum())


@pytest.mark.parametrize("rows", [33, 300])
@pytest.mark.parametrize("masked", [False, True])
def test_a_weighted_mean_is_as_exact_as_a_sum(ops, rows, masked):
    """scale 1, weights 1 / count: 1 / 300 rounded to bf16 is 2.1e-3 off; the gradients must not be."""
    g = gen(rows)
    n_in, vocab = 256, 20_000
    x, w, t, b, _ = problem(g, rows, n_in, vocab, BF, weighted=False, spread=0.25)
    weight = torch.full((rows,), 1.0 / 300, device="cuda")
    if masked:
        weight = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.6, weight, 0.0)
    R = reference(x, w, t, b, weight, 1.0)
    s = weight.double() * (t != IGNORE)
    at = torch.where(s > 0, t, 0)[:, None]
    p = torch.exp(R["z"] - R["lse"][:, None]) * s[:, None]
    p_target = p.gather(1, at)[:, 0]
    assert float(p_target.max()) < 2.0 ** -9 * float(s.max())
    got = ops.linear_cross_entropy(x, w, t, b, ignore_index=IGNORE, row_weight=weight, grad_dtype=F)
    dx, dw = R["d"] @ R["w"], R["d"].t() @ R["x"]
    for grad, exact, part in ((got[2], dx, dx @ R["w"].t()), (got[3], dw, R["x"] @ dw.t())):
        total = exact.square().sum()
        # fp32 sums of `rows` products, or of words by 16 in the accumulator
        bound = off_along(p, p_target, at, R["ed"], part / total) + (rows + vocab // 16) * 2.0 ** -23
        if grad.dtype is BF:
            bound += 8 * HALF[BF] * float(exact.pow(4).sum().sqrt() / total)
        assert bound < 1.5e-3                              # well below 2.1e-3
        assert abs(along(grad, exact) - 1) < bound, (along(grad, exact), bound)
    assert ops.device_status() == 0


def test_weights_of_any_size(ops):
    """Weights that differ by many powers of ten, negative ones, a scale that takes their size back."""
    g = gen(77)
    rows, n_in, vocab = 100, 96, 3001
    x, w, t, b, _ = problem(g, rows, n_in, vocab, BF, weighted=False)
    weight = 10.0 ** (8 * torch.rand(rows, device="cuda", generator=g) - 4)
    weight = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.3, -weight, weight)
    for factor, scale in ((1.0, 1.0), (1e20, 1e-20), (1e-20, 1e20), (-1e4, 1e-3)):
        R = reference(x, w, t, b, weight * factor, scale)
        got = ops.linear_cross_entropy(x, w, t, b, ignore_index=IGNORE, row_weight=weight * factor, scale=scale, grad_dtype=F, piece=1000)
        check(got, R, BF, F, f"{factor} {scale}")
    # no row counts
    none = ops.linear_cross_entropy(x, w, torch.full_like(t, IGNORE), b, ignore_index=IGNORE, row_weight=weight)
    assert all(bool((a == 0).all()) for a in (none[0], *none[2:]))
    assert ops.device_status() == 0


def test_long_sums_over_the_vocabulary(ops):
    """dx of bf16 operands, 120,011 words in a piece.  The tensor cores' accumulator cuts every addition towards zero, so a
    sum that stayed in it would make each target's term smaller, by 2^-24 on average and 2^-23 at most every 16 words.
    Sums leave it after 2,048 words."""
    g = gen(120)
    rows, n_in, vocab = 1024, 4096, 120_011
    x, w, t, _, _ = problem(g, rows, n_in, vocab, BF, bias=False, weighted=False, spread=0.25)
    w = w - w.float().mean(0).to(BF)
    got = ops.linear_cross_entropy(x, w, t, None, ignore_index=IGNORE, piece=vocab)[2]
    wd = w.double()
    z = x.double() @ wd.t()
    valid = t != IGNORE
    at = torch.where(valid, t, 0)[:, None]
    p = torch.softmax(z, 1) * valid[:, None]
    p_target = p.gather(1, at)[:, 0]
    assert float(p_target.max()) < 2.0 ** -9
    d = p.scatter_add(1, at, -valid[:, None].double())
    exact = d @ wd
    total = float(exact.square().sum())
    ed = p * ((n_in / 16 + 8) * 2.0 ** -23 * z.abs().max() + 2.0 ** -20)
    bound = 128 * 2.0 ** -23 + off_along(p, p_target, at, ed, (exact @ wd.t()) / total)
    bound += 8 * HALF[BF] * float(exact.pow(4).sum().sqrt()) / total
    assert bound < 6e-5
    assert abs(along(got, exact) - 1) < bound, (along(got, exact), bound)
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype,rows,n_in,vocab,piece,how", [
    (BF, 4000, 136, 3001, 1000, "odd"), (BF, 4001, 33, 2100, 300, "odd"), (F, 4000, 136, 2500, 700, "plain"), (F, 4100, 72, 2500, 0, "odd"),
    (F, 20_000, 16, 300, 128, "plain"), (BF, 20_011, 16, 600, 256, "odd")])
def test_several_launches_of_the_statistics(ops, dtype, rows, n_in, vocab, piece, how):
    """Rows whose tiles do not fill the GPU evenly, with weights that are packed a piece at a time."""
    x, w, t, b, rw = problem(gen(rows + vocab), rows, n_in, vocab, dtype)
    R = reference(x, w, t, b, rw, 0.5)
    args = (lay(x, how), lay(w, how), t, lay(b, how))
    check(ops.linear_cross_entropy(*args, row_weight=rw, scale=0.5, piece=piece), R, dtype, dtype, how)
    check(ops.linear_cross_entropy(*args, row_weight=rw, scale=0.5, piece=piece, want_grad=False), R, dtype, dtype, how + " values")
    assert ops.device_status() == 0


def test_graphs_take_the_weights_they_find(ops):
    """A captured step, replayed after its weights, targets and inputs have changed, on another stream too."""
    g = gen(5)
    x, w, t, b, rw = problem(g, 300, 72, 3001, BF)
    call = lambda **kw: ops.linear_cross_entropy(x, w, t, b, row_weight=rw, scale=0.1, piece=1000, **kw)      # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for turn in range(4):
        rw.copy_(torch.rand(300, device="cuda", generator=g) * 10.0 ** (3 * turn - 4))
        t.copy_(torch.randint(0, 3001, (300,), device="cuda", generator=g))
        x.copy_(x.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        got = [a.clone() for a in out]
        assert all(torch.equal(a, c) for a, c in zip(got, call()))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        other = call(stream=side)
        side.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, other))
        check(got, reference(x, w, t, b, rw, 0.1), BF, BF, f"turn {turn}")
    assert ops.device_status() == 0
