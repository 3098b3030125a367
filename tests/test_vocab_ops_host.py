"""The vocabulary operators without a GPU: struct layouts, refusals, and which stream the binding's calls allocate
on and run on."""
import ctypes
import math

import pytest
import torch

from paper_1909_09010_b200 import binding
from test_local_ops_streams import CALLER, SIDE, world                           # noqa: F401 (a fixture)


def offsets(cls):
    return {name: getattr(cls, name).offset for name, _ in cls._fields_}


def test_argument_blocks_have_the_layout_of_the_header():
    c = offsets(binding.LinearCrossEntropyArgs)
    assert (c["vocab"], c["x"], c["targets"], c["loss"], c["dx"], c["dbias"], c["ld_x"], c["piece"], c["dtype"], c["accumulate"],
            c["scale"], c["workspace"]) == (16, 24, 48, 64, 80, 96, 104, 144, 152, 160, 164, 168)
    assert ctypes.sizeof(binding.LinearCrossEntropyArgs) == 184
    t = offsets(binding.TopLogitsArgs)
    assert (t["logits"], t["lse"], t["ld_logits"], t["dtype"], t["k"], t["temperature"]) == (16, 40, 48, 72, 76, 80)
    assert ctypes.sizeof(binding.TopLogitsArgs) == 88
    d = offsets(binding.DistillationArgs)
    assert (d["logits"], d["teacher_lse"], d["loss"], d["dlogits"], d["ld_logits"], d["ignore_index"], d["dtype"], d["k"],
            d["temperature"], d["scale"]) == (16, 40, 64, 80, 88, 120, 128, 136, 140, 148)
    assert ctypes.sizeof(binding.DistillationArgs) == 152


@pytest.mark.parametrize("cls", [binding.LinearCrossEntropyArgs, binding.TopLogitsArgs, binding.DistillationArgs])
def test_packed_arguments_are_the_bytes_of_the_structure(cls):
    values = [0.25 if t is ctypes.c_float else i + 1 for i, (_, t) in enumerate(cls._fields_)]
    assert binding._packer(cls)(*values) == bytes(cls(*values))


def test_refusals_without_a_gpu():
    L, bad = binding.lib(), binding.ERR_INVALID_ARG
    n = ctypes.c_int64()
    a = binding.LinearCrossEntropyArgs(rows=1, n_in=1, vocab=1)
    assert L.gbmuf_linear_cross_entropy(None, None, None) == bad and L.gbmuf_linear_cross_entropy(None, ctypes.byref(a), None) == bad
    assert L.gbmuf_linear_cross_entropy_workspace(None, ctypes.byref(a), ctypes.byref(n)) == bad
    assert L.gbmuf_linear_cross_entropy_workspace(None, ctypes.byref(a), None) == bad
    t = binding.TopLogitsArgs(rows=1, vocab=1, k=1, temperature=1.0)
    assert L.gbmuf_top_logits(None, None, None) == bad and L.gbmuf_top_logits(None, ctypes.byref(t), None) == bad
    d = binding.DistillationArgs(rows=1, vocab=1, k=1, temperature=1.0)
    assert L.gbmuf_distillation(None, None, None) == bad and L.gbmuf_distillation(None, ctypes.byref(d), None) == bad
    assert b"NULL" in L.gbmuf_last_error(None)


# A handle that is never looked into: what comes before any call of the driver.
@pytest.fixture
def handle():
    block = ctypes.create_string_buffer(4096)
    return block, ctypes.addressof(block)


def refused(call, handle, args, status, text, **change):
    for name, value in change.items():
        setattr(args, name, value)
    assert call(handle[1], ctypes.byref(args), None) == status
    assert text in binding.lib().gbmuf_last_error(None).decode()


def test_arguments_are_checked_before_the_gpu(handle):
    L, bad, big = binding.lib(), binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    p = 4096

    def layer():
        return binding.LinearCrossEntropyArgs(rows=4, n_in=8, vocab=10, x=p, w=p, targets=p, loss=p, lse=p, ld_x=8, ld_w=8, ld_dx=8,
                                              ld_dw=8, scale=1.0)
    for status, text, change in [
            (bad, "negative", dict(rows=-1)), (bad, "negative", dict(vocab=-1)), (big, "2^31", dict(vocab=1 << 31)),
            (big, "2^31", dict(n_in=1 << 31)), (bad, "vocab", dict(vocab=0)), (bad, "dtype", dict(dtype=2)), (bad, "dtype", dict(grad_dtype=-1)),
            (bad, "scale", dict(scale=math.nan)), (bad, "piece", dict(piece=-5)), (bad, "x is NULL", dict(x=None)), (bad, "w is NULL", dict(w=None)),
            (bad, "x is not aligned", dict(x=p + 2)), (bad, "w has a row stride", dict(ld_w=7)), (bad, "dx has a row stride", dict(dx=p, ld_dx=3)),
            (bad, "dw is not aligned", dict(dw=p + 1)), (bad, "dbias is not aligned", dict(dbias=p + 2)), (bad, "bias is not aligned", dict(bias=p + 3)),
            (bad, "targets is NULL", dict(targets=None)), (bad, "targets is not aligned", dict(targets=p + 4)),
            (bad, "row_weight", dict(row_weight=p + 1)), (bad, "lse", dict(lse=p + 2)), (bad, "2^56", dict(ld_w=1 << 60))]:
        refused(L.gbmuf_linear_cross_entropy, handle, layer(), status, text, **change)

    def top():
        return binding.TopLogitsArgs(rows=4, vocab=10, logits=p, values=p, index=p, lse=p, ld_logits=10, ld_values=3, ld_index=3, k=3, temperature=1.0)
    for status, text, change in [
            (bad, "negative", dict(vocab=-1)), (big, "2^31", dict(rows=1 << 31)), (bad, "vocab", dict(vocab=0)), (bad, "dtype", dict(dtype=7)),
            (bad, "k must be 1", dict(k=0)), (big, "k must be at most 256", dict(k=257)), (bad, "k must be at most vocab", dict(k=11, ld_values=11, ld_index=11)),
            (bad, "temperature", dict(temperature=0.0)), (bad, "temperature", dict(temperature=math.inf)), (bad, "logits is NULL", dict(logits=None)),
            (bad, "values is NULL", dict(values=None)), (bad, "index is NULL", dict(index=None)), (bad, "index is not aligned", dict(index=p + 4)),
            (bad, "index has a row stride", dict(ld_index=2)), (bad, "values has a row stride", dict(ld_values=2)), (bad, "lse", dict(lse=p + 1))]:
        refused(L.gbmuf_top_logits, handle, top(), status, text, **change)

    def distil():
        return binding.DistillationArgs(rows=4, vocab=10, logits=p, teacher_logits=p, teacher_index=p, loss=p, lse=p, dlogits=2 * p, ld_logits=10,
                                        ld_teacher=3, ld_index=3, ld_dlogits=10, k=3, temperature=1.0, scale=1.0)
    for status, text, change in [
            (bad, "negative", dict(rows=-2)), (bad, "teacher_dtype", dict(teacher_dtype=3)), (big, "k must be at most", dict(k=300)),
            (bad, "temperature", dict(temperature=-1.0)), (bad, "hard_weight must", dict(hard_weight=1.5)), (bad, "hard_weight must", dict(hard_weight=math.nan)),
            (bad, "needs targets", dict(hard_weight=0.5)), (bad, "scale", dict(scale=math.nan)), (bad, "logits is NULL", dict(logits=None)),
            (bad, "teacher_logits is NULL", dict(teacher_logits=None)), (bad, "teacher_index is NULL", dict(teacher_index=None)),
            (bad, "teacher_index has a row stride", dict(ld_index=1)), (bad, "dlogits has a row stride", dict(ld_dlogits=9)),
            (bad, "in place", dict(dlogits=p, ld_dlogits=12)), (bad, "targets is not aligned", dict(targets=p + 4)),
            (bad, "teacher_lse", dict(teacher_lse=p + 2))]:
        refused(L.gbmuf_distillation, handle, distil(), status, text, **change)


def calls(w):
    x, m, dz = torch.ones(20, 12), torch.ones(7, 12), torch.ones(20, 7)
    t = torch.zeros(20, dtype=torch.int64)
    tops, index = torch.ones(20, 3), torch.zeros((20, 3), dtype=torch.int64)
    ops = w.LocalOps
    return [lambda s: ops.linear_cross_entropy(x, m, t, bias=torch.ones(7), stream=s),
            lambda s: ops.linear_cross_entropy(x, m, t, want_grad=False, stream=s),
            lambda s: ops.top_logits(dz, 3, stream=s), lambda s: ops.distillation(dz, tops, index, stream=s)]


@pytest.mark.parametrize("i", range(4))
@pytest.mark.parametrize("as_handle", [False, True])
def test_results_and_workspace_belong_to_the_stream_of_the_call(world, i, as_handle):          # noqa: F811
    results = calls(world)[i](SIDE if as_handle else world.side)
    assert world.ran == [SIDE] and world.current == CALLER
    assert world.made and all(s == SIDE for _, s in world.made), "allocated on another stream than the call's"
    assert all(any(t is r for t, _ in world.made) for r in results)
    assert sorted(id(t) for t, s in world.recorded if s == CALLER) == sorted(id(r) for r in results)


@pytest.mark.parametrize("i", range(4))
def test_without_a_stream_everything_is_on_the_current_one(world, i):                          # noqa: F811
    calls(world)[i](None)
    assert world.ran == [CALLER] and all(s == CALLER for _, s in world.made) and not world.recorded
