"""The C ABI of the local-step operators without a GPU: struct layouts and refusals that need none."""
import ctypes

import pytest

from paper_1909_09010_b200 import binding


def offsets(cls):
    return {name: getattr(cls, name).offset for name, _ in cls._fields_}


def test_argument_blocks_have_the_layout_of_the_header():
    f = offsets(binding.LinearForwardArgs)
    assert (f["rows"], f["x"], f["y"], f["ld_x"], f["ld_z"], f["dtype"], f["activation"], f["workspace"]) == \
        (0, 24, 56, 72, 104, 112, 116, 120) and ctypes.sizeof(binding.LinearForwardArgs) == 136
    i = offsets(binding.LinearBackwardInputArgs)
    assert (i["dz"], i["dx"], i["ld_dz"], i["ld_dz_prev"], i["dtype"], i["workspace"]) == (24, 56, 72, 112, 120, 128)
    assert ctypes.sizeof(binding.LinearBackwardInputArgs) == 144
    w = offsets(binding.LinearBackwardWeightArgs)
    assert (w["dz"], w["dbias"], w["ld_dz"], w["dtype"], w["reserved"], w["workspace"]) == (24, 48, 56, 80, 92, 96)
    assert ctypes.sizeof(binding.LinearBackwardWeightArgs) == 112
    c = offsets(binding.CrossEntropyArgs)
    assert (c["vocab"], c["logits"], c["dlogits"], c["ld_logits"], c["ignore_index"], c["dtype"], c["scale"]) == \
        (8, 16, 56, 64, 80, 88, 92) and ctypes.sizeof(binding.CrossEntropyArgs) == 96
    g = offsets(binding.GradTensor)
    assert (g["out"], g["rows"], g["ld_out"], g["dtype"], g["group"]) == (8, 16, 40, 48, 56)
    assert ctypes.sizeof(binding.GradTensor) == 64


@pytest.mark.parametrize("cls,values", [
    (binding.LinearForwardArgs, [3, 4, 5, 6, 7, 0, 8, 9, 0, 10, 11, 12, 13, 14, 1, 2, 0, 0]),
    (binding.CrossEntropyArgs, [2, 3, 4, 5, 0, 6, 7, 8, 9, 10, -100, 1, 0.25])])
def test_packed_arguments_are_the_bytes_of_the_structure(cls, values):
    assert binding._packer(cls)(*values) == bytes(cls(*[v or None if t is ctypes.c_void_p else v
                                                        for v, (_, t) in zip(values, cls._fields_)]))


def test_refusals_without_a_gpu():
    L, bad = binding.lib(), binding.ERR_INVALID_ARG
    h, n = ctypes.c_void_p(), ctypes.c_int64()
    assert L.gbmuf_ops_create(0, None) == bad and L.gbmuf_ops_create(-1, ctypes.byref(h)) == bad
    assert b"negative" in L.gbmuf_last_error(None)
    a = binding.LinearForwardArgs(rows=1, n_in=1, n_out=1)
    for name in ("forward", "backward_input", "backward_weight"):
        assert getattr(L, "gbmuf_linear_" + name)(None, ctypes.byref(a), None) == bad
        assert getattr(L, "gbmuf_linear_" + name)(None, None, None) == bad
        assert getattr(L, "gbmuf_linear_" + name + "_workspace")(None, ctypes.byref(a), ctypes.byref(n)) == bad
        assert getattr(L, "gbmuf_linear_" + name + "_workspace")(None, ctypes.byref(a), None) == bad
    assert L.gbmuf_activation_backward(None, 1, 1, 0, 0, None, 1, None, 1, None, 1, None) == bad
    assert L.gbmuf_cross_entropy(None, None, None) == bad
    assert L.gbmuf_clip_create(0, 0, 0, None, ctypes.byref(h)) == bad          # no group
    assert L.gbmuf_clip_create(0, 1, 0, None, None) == bad
    assert L.gbmuf_clip_set_tensors(None, 0, None) == bad
    assert L.gbmuf_clip_norms(None, None, None) == bad and L.gbmuf_clip_scale(None, 1.0, None, None) == bad
    assert L.gbmuf_ops_device_status(None, None, None) == bad and L.gbmuf_clip_device_status(None, None, None) == bad
    assert not h.value
    assert L.gbmuf_ops_destroy(None) == binding.GBMUF_OK and L.gbmuf_clip_destroy(None) == binding.GBMUF_OK
