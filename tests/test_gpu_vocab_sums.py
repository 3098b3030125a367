"""Sums over a vocabulary word by word: what a long row's slices, chunks and unaligned ends leave out or count twice,
and what NaN does to them."""
import math

import pytest
import torch

from paper_1909_09010_b200 import binding
from test_gpu_vocab_ops import BF, F, check_top, gen, lay, lists, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    return binding.local_ops(0)


# rows: clusters of 8, 4, 2 blocks to a row, and a block to a row or several
SIZES = [(3, 1), (2, 300), (5, 2048), (1, 2049), (6, 4100), (30, 10_007), (70, 20_011), (140, 33_278), (320, 9001), (600, 2050),
         (20, 267_735), (60, 131_071), (130, 100_003), (310, 40_001)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_every_word_counts_once(ops, dtype, rows, vocab):
    """Equal logits c: every exponential is 1, so the sums are whole numbers below 2^24 and exact, and lse = c / T + log V to
    the logarithm's 2^-24 or so of 13 and one rounding; one word too few would be 1 / V = 3.7e-6."""
    for how, c, T in (("plain", 0.0, 1.0), ("odd", 1.5, 2.0), ("padded", -1.0, 0.5)):
        want = c / T + math.log(vocab)
        tol = 2.0 ** -23 * (1 + abs(c / T) + math.log(vocab))
        assert tol < 0.6 / vocab or vocab < 1000
        x = lay(torch.full((rows, vocab), c, dtype=dtype, device="cuda"), how)
        k = min(vocab, 40)
        values, index, lse = ops.top_logits(x, k, temperature=T)
        assert float((lse.double() - want).abs().max()) <= tol
        assert torch.equal(index, torch.arange(k, device="cuda").expand(rows, k)) and bool((values == c).all())
        # a list of words all over the row, words that come twice among them
        g = gen(vocab)
        ix = torch.randint(0, vocab, (rows, k), device="cuda", generator=g)
        ix[:, 0], ix[:, -1] = vocab - 1, 0
        t = torch.zeros((rows, k), device="cuda")
        teacher = torch.full((rows,), math.log(4.0 * k), device="cuda")          # q = 1 / (4 k) each, 3 / 4 outside
        for grad in (False, True):
            got = ops.distillation(x, t, ix, teacher_lse=teacher, temperature=T, want_grad=grad)
            assert float((got[1].double() - want).abs().max()) <= tol
            # sum q (log q + log V) + q_r (log q_r + log V - log(words outside))
            distinct = torch.tensor([len(set(r)) for r in ix.tolist()], device="cuda", dtype=torch.float64)
            outside = vocab - distinct
            soft = 0.25 * (math.log(vocab) - math.log(4 * k))
            soft = soft + torch.where(outside > 0, 0.75 * (math.log(0.75) + math.log(vocab) - outside.clamp(min=1).log()), 0.0)
            # q: 2^-22 of each; products with logarithms of at most 13
            assert float((got[0].double() - T * T * soft).abs().max()) <= T * T * 2.0 ** -20 * (1 + math.log(vocab))
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,vocab,piece", [(1, 10_007, 0), (8, 3001, 0), (16, 4100, 0), (40, 9001, 1000), (300, 5003, 64), (4000, 1515, 500),
                                              (4000, 2100, 0), (20_000, 700, 300)])
def test_every_word_counts_once_in_the_softmax_layer(ops, dtype, rows, vocab, piece):
    """As above, with weights of 0: the statistics of few rows, of one launch and of several, of every piece."""
    x, w = torch.ones((rows, 40), dtype=dtype, device="cuda"), torch.zeros((vocab, 40), dtype=dtype, device="cuda")
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=gen(rows))
    for how in ("plain", "odd"):
        loss, lse, _, _, db = ops.linear_cross_entropy(lay(x, how), lay(w, how), t, torch.full((vocab,), 0.5, dtype=dtype, device="cuda"),
                                                       piece=piece, grad_dtype=F)
        tol = 2.0 ** -23 * (2 + math.log(vocab))
        assert tol < 0.5 / vocab
        assert float((lse.double() - 0.5 - math.log(vocab)).abs().max()) <= tol
        assert float((loss.double() - math.log(vocab)).abs().max()) <= tol
        want = rows / vocab - torch.bincount(t, minlength=vocab).double()
        assert float((db.double() - want).abs().max()) <= rows * 2.0 ** -23 * (8 + 2 * rows / vocab)
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,vocab", [s for s in SIZES if s[1] >= 300])
def test_sums_of_few_additions(ops, dtype, rows, vocab):
    """Each of 256 threads has four running sums, so one has vocab / 1024 additions at most (a warp's or a block's short
    row 64), and the joins fewer than 64; exponentials 2^-20 with their exponents' rounding."""
    x = rnd(gen(rows + vocab), (rows, vocab), dtype, 2.0)
    for how, T in (("odd", 1.0), ("plain", 2.0)):
        ref = torch.logsumexp(x.double() / T, 1)
        tol = 2.0 ** -20 + (vocab / 1024 + 64) * 2.0 ** -24 + 2.0 ** -23 * ref.abs()
        lse = ops.top_logits(lay(x, how), 20, temperature=T)[2]
        assert bool(((lse.double() - ref).abs() <= tol).all())
        t, ix, tlse = lists(gen(1), x, 20, T, F)
        for grad in (False, True):
            lse = ops.distillation(lay(x, how), t, ix, teacher_lse=tlse, temperature=T, want_grad=grad)[1]
            assert bool(((lse.double() - ref).abs() <= tol).all())
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,vocab", [(30, 20_011), (70, 20_011), (140, 40_001), (320, 20_011), (25, 267_735)])
def test_the_largest_at_every_edge(ops, dtype, rows, vocab):
    """The largest logits where slices of a cluster, chunks of 16 KB, pieces of 16 bytes and the row begin and end."""
    each = 128 // torch.finfo(dtype).bits
    places = {0, 1, each - 1, each, vocab - 1, vocab - 2, vocab - each, vocab - each - 1}
    for split in (1, 2, 4, 8):
        for part in range(split + 1):
            places |= {vocab // each * part // split * each + i for i in range(-each, 2 * each)}
    for chunk in range(0, vocab, 1024 * each):
        places |= {chunk + i for i in (-1, 0, 1, each - 1, each)}
    places = sorted(p for p in places if 0 <= p < vocab)
    x = rnd(gen(rows), (rows, vocab), dtype)
    for start in range(0, len(places), rows):
        y = x.clone()
        for row, place in enumerate(places[start:start + rows]):
            y[row, place] = 50.0
            y[row, (place + 1) % vocab] = 49.0
        for how in ("plain", "odd"):
            check_top(ops, y, 3, how=how)
    assert ops.device_status() == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("vocab", [40, 1500, 9001])
def test_nan_whatever_the_list_is(ops, dtype, vocab):
    """NaN or +inf in a student's row, or a NaN of the teacher's, its log-sum-exp among them, gives NaN: with a list without
    entries and with a list that holds every word that can occur too."""
    g = gen(vocab)
    rows, k = 8, 30
    x = rnd(g, (rows, vocab), dtype)
    t, ix, tlse = lists(g, x, k, 1.0, F)
    targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    never = torch.ones((rows, vocab), dtype=torch.bool, device="cuda").scatter_(1, ix, False)
    for value in (math.nan, math.inf):
        for hard in (0.0, 0.4, 1.0):
            kw = dict(targets=targets, hard_weight=hard) if hard else {}
            for given_lse in (None, tlse):
                bad = x.clone()
                bad[2, vocab // 2] = value
                empty = ix.clone()
                empty[2] = -1
                loss, lse, d = ops.distillation(bad, t, empty, teacher_lse=given_lse, **kw)
                assert bool(loss[2].isnan()) and bool(lse[2].isnan()) and bool(d[2].isnan().all()), (value, hard)
                bad = torch.where(never, -math.inf, x.float()).to(dtype)         # no word outside the list can occur
                bad[2, ix[2, 3]] = value
                kw2 = dict(kw, targets=ix[:, 1].contiguous()) if hard else {}
                loss, lse, d = ops.distillation(bad, t, ix, teacher_lse=given_lse, **kw2)
                assert bool(loss[2].isnan()) and bool(lse[2].isnan()) and bool(d[2].isnan().all()), (value, hard)
                assert bool(d[3].isfinite().all())
    nan_lse = tlse.clone()
    nan_lse[5] = math.nan
    empty = ix.clone()
    empty[5] = -1
    nan_list = t.clone()
    nan_list[5, 2] = math.nan
    for hard in (0.0, 0.4, 1.0):
        kw = dict(targets=targets, hard_weight=hard) if hard else {}
        for lists_, index, lse_ in ((t, ix, nan_lse), (t, empty, nan_lse), (nan_list, ix, tlse), (nan_list, ix, None)):
            loss, lse, d = ops.distillation(x, lists_, index, teacher_lse=lse_, **kw)
            assert bool(loss[5].isnan()) and bool(d[5].isnan().all()) and bool(lse.isfinite().all())
            rest = torch.arange(rows, device="cuda") != 5
            assert bool(loss[rest].isfinite().all()) and bool(d[rest].isfinite().all())
    assert ops.device_status() == 0
