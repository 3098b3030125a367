"""Sums over a vocabulary: what NaN does to them."""
import math

import pytest
import torch

from paper_1909_09010_b200 import binding
from test_gpu_vocab_ops import BF, F, gen, lists, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    return binding.local_ops(0)


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
