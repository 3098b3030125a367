"""Thin ctypes binding of ``libgbmuf.so``: argument marshalling only, same names as the C ABI.

Every step of the synchronisation round runs in the CUDA library.  PyTorch is used here only to
hand over device pointers and the current stream.  If the library is missing this module raises;
there is no other implementation to fall back to.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

from . import build as _build

GBMUF_OK = 0
ERR_INVALID_ARG, ERR_BAD_STATE, ERR_ALLOC, ERR_CUDA, ERR_TIMEOUT, ERR_UNSUPPORTED = 1, 2, 3, 4, 5, 6
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "BAD_STATE", 3: "ALLOC", 4: "CUDA", 5: "TIMEOUT",
                6: "UNSUPPORTED"}
F32, BF16 = 0, 1
MODE_BMUF, MODE_MA = 0, 1

EXPORTS = ["gbmuf_create", "gbmuf_set_partition", "gbmuf_init", "gbmuf_local_perturb",
           "gbmuf_sync_round", "gbmuf_get_neighbors", "gbmuf_final_average", "gbmuf_device_status",
           "gbmuf_set_tuning", "gbmuf_get_launch_info", "gbmuf_last_error", "gbmuf_destroy",
           "gbmuf_sync_round_noalloc", "gbmuf_sync_round_host", "gbmuf_host_create",
           "gbmuf_host_sync_round", "gbmuf_host_destroy", "gbmuf_local_adagrad",
           "gbmuf_selftest_wait_timeout", "gbmuf_selftest_divide", "gbmuf_peer_create", "gbmuf_peer_set_partition",
           "gbmuf_peer_sync_round", "gbmuf_peer_device_status", "gbmuf_peer_destroy",
           "gbmuf_ops_create", "gbmuf_ops_device_status", "gbmuf_ops_destroy",
           "gbmuf_linear_forward_workspace", "gbmuf_linear_forward",
           "gbmuf_linear_backward_input_workspace", "gbmuf_linear_backward_input",
           "gbmuf_linear_backward_weight_workspace", "gbmuf_linear_backward_weight",
           "gbmuf_activation_backward", "gbmuf_cross_entropy", "gbmuf_linear_cross_entropy_workspace",
           "gbmuf_linear_cross_entropy", "gbmuf_top_logits", "gbmuf_distillation", "gbmuf_clip_create",
           "gbmuf_clip_set_tensors", "gbmuf_clip_norms", "gbmuf_clip_scale", "gbmuf_clip_device_status",
           "gbmuf_clip_selftest_wait_timeout", "gbmuf_clip_destroy"]
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, "tanh": 4, "sigmoid": 5}


class Config(ctypes.Structure):
    """Mirror of ``gbmuf_config``."""
    _fields_ = [("K", ctypes.c_int32), ("N", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("p", ctypes.c_int32), ("q", ctypes.c_int32), ("eta", ctypes.c_float),
                ("zeta", ctypes.c_float), ("mode", ctypes.c_int32), ("theta_dtype", ctypes.c_int32),
                ("seed", ctypes.c_uint64), ("device", ctypes.c_int32), ("comp_base", ctypes.c_int32),
                ("elem_base", ctypes.c_int64)]


def _fields(spec: str):
    """ctypes fields from "type name name, type name ..." (i: int32, l: int64, f: float, p: pointer)."""
    types = {"i": ctypes.c_int32, "l": ctypes.c_int64, "f": ctypes.c_float, "p": ctypes.c_void_p}
    return [(name, types[part.split()[0]]) for part in spec.split(",") for name in part.split()[1:]]


def _packer(cls):
    """Packs the fields of a ctypes structure, in order, into its bytes: a tenth of the time that
    filling the structure takes, which for the smallest calls is longer than the GPU's part."""
    code = {ctypes.c_int32: "i", ctypes.c_int64: "q", ctypes.c_float: "f", ctypes.c_void_p: "P"}
    packer = struct.Struct("@" + "".join(code[t] for _, t in cls._fields_) + "0q")
    assert packer.size == ctypes.sizeof(cls)
    return packer.pack


class LinearForwardArgs(ctypes.Structure):
    """Mirror of ``gbmuf_linear_forward_args``."""
    _fields_ = _fields("l rows n_in n_out, p x w bias residual y z, l ld_x ld_w ld_residual ld_y ld_z, "
                       "i dtype activation, p workspace, l workspace_bytes")


class LinearBackwardInputArgs(ctypes.Structure):
    """Mirror of ``gbmuf_linear_backward_input_args``."""
    _fields_ = _fields("l rows n_in n_out, p dz w residual z_prev dx dz_prev, "
                       "l ld_dz ld_w ld_residual ld_z_prev ld_dx ld_dz_prev, i dtype activation, "
                       "p workspace, l workspace_bytes")


class LinearBackwardWeightArgs(ctypes.Structure):
    """Mirror of ``gbmuf_linear_backward_weight_args``."""
    _fields_ = _fields("l rows n_in n_out, p dz x dw dbias, l ld_dz ld_x ld_dw, "
                       "i dtype grad_dtype accumulate reserved, p workspace, l workspace_bytes")


class CrossEntropyArgs(ctypes.Structure):
    """Mirror of ``gbmuf_cross_entropy_args``."""
    _fields_ = _fields("l rows vocab, p logits targets row_weight loss lse dlogits, "
                       "l ld_logits ld_dlogits ignore_index, i dtype, f scale")


class LinearCrossEntropyArgs(ctypes.Structure):
    """Mirror of ``gbmuf_linear_cross_entropy_args``."""
    _fields_ = _fields("l rows n_in vocab, p x w bias targets row_weight loss lse dx dw dbias, "
                       "l ld_x ld_w ld_dx ld_dw ignore_index piece, i dtype grad_dtype accumulate, f scale, "
                       "p workspace, l workspace_bytes")


class TopLogitsArgs(ctypes.Structure):
    """Mirror of ``gbmuf_top_logits_args``."""
    _fields_ = _fields("l rows vocab, p logits values index lse, l ld_logits ld_values ld_index, i dtype k, "
                       "f temperature, i reserved")


class DistillationArgs(ctypes.Structure):
    """Mirror of ``gbmuf_distillation_args``."""
    _fields_ = _fields("l rows vocab, p logits teacher_logits teacher_index teacher_lse targets row_weight loss lse "
                       "dlogits, l ld_logits ld_teacher ld_index ld_dlogits ignore_index, i dtype teacher_dtype k, "
                       "f temperature hard_weight scale")


class GradTensor(ctypes.Structure):
    """Mirror of ``gbmuf_grad_tensor``."""
    _fields_ = _fields("p grad out, l rows cols ld_grad ld_out, i dtype out_dtype group reserved")


class GbmufError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"gbmuf status {status} ({STATUS_NAMES.get(status, '?')}): {message}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library.  Raises if it is not built: there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_1909_09010_b200.build` "
                           "(nvcc, sm_100a).  There is no CPU or other fallback.")
    L = ctypes.CDLL(path)
    i32, i64, u64, f32, vp = (ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float,
                              ctypes.c_void_p)
    L.gbmuf_create.argtypes = [ctypes.POINTER(Config), vp, vp, vp, ctypes.POINTER(vp)]
    L.gbmuf_set_partition.argtypes = [vp, i32, vp, vp]
    L.gbmuf_init.argtypes = [vp, vp, vp]
    L.gbmuf_local_perturb.argtypes = [vp, u64, f32, f32, i32, vp]
    L.gbmuf_local_adagrad.argtypes = [vp, vp, vp, f32, f32, f32, vp, vp]
    L.gbmuf_sync_round.argtypes = [vp, u64, vp, vp]
    L.gbmuf_get_neighbors.argtypes = [vp, u64, vp]
    L.gbmuf_final_average.argtypes = [vp, vp, vp]
    L.gbmuf_device_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
    L.gbmuf_set_tuning.argtypes = [vp, i32, i32, i32, i32, i32]
    L.gbmuf_get_launch_info.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i32),
                                        ctypes.POINTER(i32), ctypes.POINTER(i32),
                                        ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.gbmuf_sync_round_noalloc.argtypes = [ctypes.POINTER(Config), vp, vp, vp, i32, vp, vp, u64, vp,
                                           ctypes.POINTER(i32)]
    L.gbmuf_sync_round_host.argtypes = [ctypes.POINTER(Config), vp, vp, vp, i32, vp, vp, u64, i64]
    L.gbmuf_host_create.argtypes = [ctypes.POINTER(Config), i32, vp, i64, i32, ctypes.POINTER(vp)]
    L.gbmuf_host_sync_round.argtypes = [vp, vp, vp, vp, vp, u64]
    L.gbmuf_host_destroy.argtypes = [vp]
    L.gbmuf_selftest_wait_timeout.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_double)]
    L.gbmuf_selftest_divide.argtypes = [vp, i32, vp, ctypes.POINTER(u64), ctypes.POINTER(ctypes.c_uint32)]
    L.gbmuf_peer_create.argtypes = [ctypes.POINTER(Config), i32, vp, vp, vp, ctypes.POINTER(vp)]
    L.gbmuf_peer_set_partition.argtypes = [vp, i32, vp, vp]
    L.gbmuf_peer_sync_round.argtypes = [vp, u64, vp, i32, vp]
    L.gbmuf_peer_device_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
    L.gbmuf_peer_destroy.argtypes = [vp]
    L.gbmuf_ops_create.argtypes = [i32, ctypes.POINTER(vp)]
    L.gbmuf_ops_device_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
    L.gbmuf_ops_destroy.argtypes = [vp]
    for name in ("forward", "backward_input", "backward_weight"):
        getattr(L, "gbmuf_linear_" + name).argtypes = [vp, vp, vp]
        getattr(L, "gbmuf_linear_" + name + "_workspace").argtypes = [vp, vp, vp]
    L.gbmuf_activation_backward.argtypes = [vp, i64, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp]
    L.gbmuf_cross_entropy.argtypes = [vp, vp, vp]
    L.gbmuf_linear_cross_entropy_workspace.argtypes = [vp, vp, vp]
    L.gbmuf_linear_cross_entropy.argtypes = [vp, vp, vp]
    L.gbmuf_top_logits.argtypes = [vp, vp, vp]
    L.gbmuf_distillation.argtypes = [vp, vp, vp]
    L.gbmuf_clip_create.argtypes = [i32, i32, i64, vp, ctypes.POINTER(vp)]
    L.gbmuf_clip_set_tensors.argtypes = [vp, i64, vp]
    L.gbmuf_clip_norms.argtypes = [vp, vp, vp]
    L.gbmuf_clip_scale.argtypes = [vp, f32, vp, vp]
    L.gbmuf_clip_device_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
    L.gbmuf_clip_selftest_wait_timeout.argtypes = [vp, vp]
    L.gbmuf_clip_destroy.argtypes = [vp]
    L.gbmuf_last_error.argtypes = [vp]
    L.gbmuf_last_error.restype = ctypes.c_char_p
    L.gbmuf_destroy.argtypes = [vp]
    for name in EXPORTS:
        if name != "gbmuf_last_error":
            getattr(L, name).restype = i32
    _lib = L
    return L


def _ptr(t) -> int:
    """Device (torch tensor) or host (numpy array) address; None -> NULL."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        assert t.flags["C_CONTIGUOUS"]
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


def sync_round_noalloc(theta, omega, delta, offsets, rnd, *, K, N, ld, p, q, eta, zeta, seed=0,
                       mode=MODE_BMUF, theta_dtype=F32, device=0, comp_base=0, elem_base=0,
                       comp_mask=None, stream=None, want_status=False):
    """``gbmuf_sync_round_noalloc``: one round without a context and without any allocation by the
    library (its tables live in a fixed array of the loaded library).  For callers that cannot
    allocate device memory where they synchronise.  Calls on one GPU share that array: keep them
    on one stream.  Returns the device status word if ``want_status`` (this waits for the stream).
    """
    cfg = Config(K, N, ld, p, q, eta, zeta, mode, theta_dtype, seed, device, comp_base, elem_base)
    off = np.ascontiguousarray(offsets, dtype=np.int64)
    mask = None if comp_mask is None else np.ascontiguousarray(comp_mask, dtype=np.uint8)
    word = ctypes.c_int32(-1)
    st = lib().gbmuf_sync_round_noalloc(ctypes.byref(cfg), _ptr(theta), _ptr(omega), _ptr(delta),
                                        off.shape[0] - 1, _ptr(off), _ptr(mask), rnd,
                                        _stream(stream), ctypes.byref(word) if want_status else None)
    if st != GBMUF_OK:
        raise GbmufError(st, lib().gbmuf_last_error(None).decode())
    return word.value if want_status else None


def sync_round_host(theta, omega, delta, offsets, rnd, *, K, N, ld, p, q, eta, zeta, seed=0,
                    mode=MODE_BMUF, theta_dtype=F32, device=0, comp_base=0, elem_base=0,
                    comp_mask=None, chunk_cols=0):
    """``gbmuf_sync_round_host``: one round over HOST arrays [K][ld] (numpy arrays or CPU torch
    tensors, ideally page-locked), streamed through the GPU in column chunks.  Synchronous."""
    cfg = Config(K, N, ld, p, q, eta, zeta, mode, theta_dtype, seed, device, comp_base, elem_base)
    off = np.ascontiguousarray(offsets, dtype=np.int64)
    mask = None if comp_mask is None else np.ascontiguousarray(comp_mask, dtype=np.uint8)
    st = lib().gbmuf_sync_round_host(ctypes.byref(cfg), _ptr(theta), _ptr(omega), _ptr(delta),
                                     off.shape[0] - 1, _ptr(off), _ptr(mask), rnd, chunk_cols)
    if st != GBMUF_OK:
        raise GbmufError(st, lib().gbmuf_last_error(None).decode())


class GbmufHost:
    """``gbmuf_host_*``: rounds over HOST arrays [K][ld] with the device chunk buffers, streams and
    chunk tables kept across rounds (``sync_round_host`` sets them up and frees them per call)."""

    def __init__(self, offsets, *, K, N, ld, p, q, eta, zeta, seed=0, mode=MODE_BMUF, theta_dtype=F32,
                 device=0, comp_base=0, elem_base=0, chunk_cols=0, row_copies=False):
        self._h = ctypes.c_void_p()
        cfg = Config(K, N, ld, p, q, eta, zeta, mode, theta_dtype, seed, device, comp_base, elem_base)
        off = np.ascontiguousarray(offsets, dtype=np.int64)
        self.m = off.shape[0] - 1
        st = lib().gbmuf_host_create(ctypes.byref(cfg), self.m, _ptr(off), chunk_cols,
                                     1 if row_copies else 0, ctypes.byref(self._h))
        if st != GBMUF_OK:
            raise GbmufError(st, lib().gbmuf_last_error(None).decode())

    def sync_round(self, theta, omega, delta, rnd, comp_mask=None):
        mask = None if comp_mask is None else np.ascontiguousarray(comp_mask, dtype=np.uint8)
        if mask is not None and mask.shape[0] != self.m:
            raise ValueError("comp_mask must have one entry per component")
        st = lib().gbmuf_host_sync_round(self._h, _ptr(theta), _ptr(omega), _ptr(delta), _ptr(mask), rnd)
        if st != GBMUF_OK:
            raise GbmufError(st, lib().gbmuf_last_error(None).decode())

    def destroy(self):
        if self._h:
            lib().gbmuf_host_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class GbmufPeer:
    """One worker of the one-worker-per-GPU form.  ``theta_bufs[b][j]`` is buffer b (0/1) of worker j
    (tensors or raw device addresses; entry ``rank`` is this worker's own memory)."""

    def __init__(self, rank, theta_bufs, omega, delta, *, K, N, ld, p, q, eta, zeta, seed=0,
                 mode=MODE_BMUF, theta_dtype=F32, device=0, comp_base=0):
        self._h = ctypes.c_void_p()
        self.cfg = Config(K, N, ld, p, q, eta, zeta, mode, theta_dtype, seed, device, comp_base, 0)
        self._keep = (theta_bufs, omega, delta)
        addr = [(t if isinstance(t, int) else t.data_ptr()) for b in (0, 1) for t in theta_bufs[b]]
        arr = (ctypes.c_void_p * (2 * K))(*addr)
        st = lib().gbmuf_peer_create(ctypes.byref(self.cfg), rank, arr, _ptr(omega), _ptr(delta),
                                     ctypes.byref(self._h))
        if st != GBMUF_OK:
            raise GbmufError(st, lib().gbmuf_last_error(None).decode())
        self.m = 0

    def _check(self, st):
        if st != GBMUF_OK:
            raise GbmufError(st, lib().gbmuf_last_error(None).decode())

    def set_partition(self, offsets, periods=None):
        off = np.ascontiguousarray(offsets, dtype=np.int64)
        per = None if periods is None else np.ascontiguousarray(periods, dtype=np.int32)
        self._check(lib().gbmuf_peer_set_partition(self._h, off.shape[0] - 1, _ptr(off), _ptr(per)))
        self.m = off.shape[0] - 1

    def sync_round(self, rnd, read_buffer, comp_mask=None, stream=None):
        mask = None if comp_mask is None else np.ascontiguousarray(comp_mask, dtype=np.uint8)
        self._check(lib().gbmuf_peer_sync_round(self._h, rnd, _ptr(mask), read_buffer, _stream(stream)))

    def device_status(self, stream=None) -> int:
        v = ctypes.c_int32(-1)
        self._check(lib().gbmuf_peer_device_status(self._h, _stream(stream), ctypes.byref(v)))
        return v.value

    def destroy(self):
        if self._h:
            lib().gbmuf_peer_destroy(self._h)
            self._h = ctypes.c_void_p()
            self._keep = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class Gbmuf:
    """One context: K replicas [K][ld] in caller-owned device tensors theta / omega / delta."""

    def __init__(self, theta, omega, delta, *, K, N, ld, p, q, eta, zeta, seed=0, mode=MODE_BMUF,
                 theta_dtype=F32, device=0, comp_base=0, elem_base=0):
        self._h = ctypes.c_void_p()
        self.cfg = Config(K, N, ld, p, q, eta, zeta, mode, theta_dtype, seed, device, comp_base,
                          elem_base)
        self._keep = (theta, omega, delta)
        self.m = 0
        st = lib().gbmuf_create(ctypes.byref(self.cfg), _ptr(theta), _ptr(omega), _ptr(delta),
                                ctypes.byref(self._h))
        if st != GBMUF_OK:
            raise GbmufError(st, lib().gbmuf_last_error(None).decode())

    def _check(self, st: int):
        if st != GBMUF_OK:
            raise GbmufError(st, lib().gbmuf_last_error(self._h).decode())

    def set_partition(self, offsets, periods=None):
        off = np.ascontiguousarray(offsets, dtype=np.int64)
        per = None if periods is None else np.ascontiguousarray(periods, dtype=np.int32)
        m = off.shape[0] - 1
        if per is not None and per.shape[0] != m:
            raise ValueError("periods must have one entry per component")
        self._check(lib().gbmuf_set_partition(self._h, m, _ptr(off), _ptr(per)))
        self.m = m

    def init(self, theta0, stream=None):
        self._check(lib().gbmuf_init(self._h, _ptr(theta0), _stream(stream)))

    def local_perturb(self, step, lr, sigma, nsteps=1, stream=None):
        self._check(lib().gbmuf_local_perturb(self._h, step, lr, sigma, nsteps, _stream(stream)))

    def local_adagrad(self, grad, accum, lr, eps=0.0, clip_norm=0.0, clip_mask=None, stream=None):
        mask = None
        if clip_mask is not None:
            mask = np.ascontiguousarray(clip_mask, dtype=np.uint8)
            if mask.shape[0] != self.m:
                raise ValueError("clip_mask must have one entry per component")
        self._check(lib().gbmuf_local_adagrad(self._h, _ptr(grad), _ptr(accum), lr, eps, clip_norm,
                                              _ptr(mask), _stream(stream)))

    def sync_round(self, rnd, comp_mask=None, stream=None):
        mask = None
        if comp_mask is not None:
            mask = np.ascontiguousarray(comp_mask, dtype=np.uint8)
            if mask.shape[0] != self.m:
                raise ValueError("comp_mask must have one entry per component")
        self._check(lib().gbmuf_sync_round(self._h, rnd, _ptr(mask), _stream(stream)))

    def get_neighbors(self, rnd) -> np.ndarray:
        out = np.full((self.cfg.K, self.m, self.cfg.q), -1, dtype=np.int32)
        self._check(lib().gbmuf_get_neighbors(self._h, rnd, _ptr(out)))
        return out

    def final_average(self, out, stream=None):
        """The returned model of Algorithm 1.  Also the point where a training run ends, so the
        device status word is read here (this waits for the stream): a bounded device-side wait
        that expired in any earlier round would otherwise go unnoticed."""
        self._check(lib().gbmuf_final_average(self._h, _ptr(out), _stream(stream)))
        self.raise_on_device_error(stream)

    def raise_on_device_error(self, stream=None):
        """Reads (and clears) the device status word; raises if a kernel reported a failure."""
        word = self.device_status(stream)
        if word != GBMUF_OK:
            raise GbmufError(word, "a device-side wait expired in an earlier call on this context; "
                                   "theta, omega and Delta are unspecified")

    def device_status(self, stream=None) -> int:
        v = ctypes.c_int32(-1)
        self._check(lib().gbmuf_device_status(self._h, _stream(stream), ctypes.byref(v)))
        return v.value

    def selftest_wait_timeout(self, stream=None) -> float:
        """Lets a bounded device-side wait expire on purpose; returns the kernel's duration (s)."""
        sec = ctypes.c_double(0.0)
        self._check(lib().gbmuf_selftest_wait_timeout(self._h, _stream(stream), ctypes.byref(sec)))
        return sec.value

    def selftest_divide(self, divisor: int, stream=None) -> tuple[int, int]:
        """Compares the kernels' averaging division with the plain division over all 2^32
        dividends; returns (number of differing patterns, smallest differing pattern)."""
        bad, first = ctypes.c_uint64(0), ctypes.c_uint32(0)
        self._check(lib().gbmuf_selftest_divide(self._h, divisor, _stream(stream), ctypes.byref(bad),
                                                ctypes.byref(first)))
        return bad.value, first.value

    def set_tuning(self, consumer_threads=0, tile_elems=0, theta_stages=0, ring_slots=0, flags=0):
        self._check(lib().gbmuf_set_tuning(self._h, consumer_threads, tile_elems, theta_stages,
                                           ring_slots, flags))

    def launch_info(self) -> dict:
        tiles = ctypes.c_int64()
        g, b, s, t, st = (ctypes.c_int32() for _ in range(5))
        self._check(lib().gbmuf_get_launch_info(self._h, ctypes.byref(tiles), ctypes.byref(g),
                                                ctypes.byref(b), ctypes.byref(s), ctypes.byref(t),
                                                ctypes.byref(st)))
        return {"tiles": tiles.value, "grid": g.value, "block": b.value, "smem_bytes": s.value,
                "tile_elems": t.value, "stages": st.value,
                "variant": "tmem" if st.value == 0 else "tmem-window" if st.value < 0
                else "smem-window" if st.value >= 1000 else "smem"}

    def last_error(self) -> str:
        return lib().gbmuf_last_error(self._h).decode()

    def destroy(self, check_status=True):
        """Frees the context.  Reads the device status word first (unless told not to) and raises
        after freeing if an earlier round reported a failure nobody has looked at."""
        if self._h:
            word = GBMUF_OK
            if check_status:
                try:
                    word = self.device_status()
                except Exception:
                    word = GBMUF_OK
            st = lib().gbmuf_destroy(self._h)
            self._h = ctypes.c_void_p()
            self._keep = None
            if st != GBMUF_OK:
                raise GbmufError(st, "destroy failed")
            if word != GBMUF_OK:
                raise GbmufError(word, "a device-side wait expired in an earlier call on this context "
                                       "and was never read; its results were unspecified")

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ------------------------------------------------------------------------------------------------
# The operators of a worker's local step
# ------------------------------------------------------------------------------------------------
_pack_forward = _packer(LinearForwardArgs)
_pack_backward_input = _packer(LinearBackwardInputArgs)
_pack_backward_weight = _packer(LinearBackwardWeightArgs)
_pack_cross_entropy = _packer(CrossEntropyArgs)
_pack_linear_cross_entropy = _packer(LinearCrossEntropyArgs)
_pack_top_logits = _packer(TopLogitsArgs)
_pack_distillation = _packer(DistillationArgs)


def _dtype_code(t) -> int:
    import torch
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float32:
        return F32
    raise TypeError(f"tensors are float32 or bfloat16, not {t.dtype}")


def _matrix(name, t, shape, dtype, device):
    """(address, row stride) of a matrix of the given shape, type and device; (0, 0) for None."""
    if t is None:
        return 0, 0
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, not {list(t.shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{device}")
    ld, step = t.stride()
    if step != 1 and shape[1] > 1 and shape[0] > 0:
        raise ValueError(f"{name} must have its columns next to one another")
    return t.data_ptr(), ld if shape[0] > 1 else shape[1]


def _result(name, given, like, shape, dtype, device):
    """(tensor, address, row stride) of a result: the one handed in, or a new one on like's device."""
    if given is None:
        t = like.new_empty(shape) if dtype is like.dtype else like.new_empty(shape, dtype=dtype)
        return t, t.data_ptr(), shape[1]
    return (given, *_matrix(name, given, shape, dtype, device))


def _vector(name, t, n, dtype, device):
    if t is None:
        return 0
    if t.shape != (n,):
        raise ValueError(f"{name} must be [{n}], not {list(t.shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{device}")
    if n > 1 and t.stride(0) != 1:
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _two_dims(name, t):
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix")
    return t.shape


class _OnDevice:
    """What LocalOps and GradClip share: the library, errors, streams."""

    def _open(self, device):
        import torch
        self._torch = torch
        self._L = lib()
        self._h = ctypes.c_void_p()
        self.device = device
        # the address of the current stream without building a torch Stream object around it
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                                   lambda d: torch.cuda.current_stream(d).cuda_stream)

    def _check(self, st):
        if st != GBMUF_OK:
            raise GbmufError(st, self._L.gbmuf_last_error(None).decode())

    def _on(self, stream):
        if stream is None:
            return self._raw_stream(self.device)
        return getattr(stream, "cuda_stream", stream)

    def _on_stream(self, stream, given, call, *args):
        """``call(*args)`` with ``stream`` as torch's current one: what it allocates (results, workspace)
        then comes from memory whose earlier uses are ordered before the call.  New results (not among
        ``given``) may be used, and dropped, on the caller's stream."""
        torch = self._torch
        if not hasattr(stream, "cuda_stream"):                      # a handle; 1 and 0 name the same stream
            stream = torch.cuda.ExternalStream(0 if stream == 1 else stream, device=self.device)
        caller = torch.cuda.current_stream(self.device)
        if stream.device.index != self.device:
            raise ValueError(f"stream is on {stream.device}, not on cuda:{self.device}")
        with torch.cuda.stream(stream):
            results = call(*args)
        for t in results if isinstance(results, tuple) else (results,):
            if not any(t is g for g in given):
                t.record_stream(caller)
        return results


class LocalOps(_OnDevice):
    """``gbmuf_ops_*``: linear layers with their gradients and the loss, on one device.  Tensors are
    torch tensors on it; autograd does not see the calls (results have no history, whatever the
    arguments' ``requires_grad`` says).  ``stream`` (default: the current one of the device) is where a call runs and
    where torch allocates what it needs: results that are not handed in, and the workspace.  Tensors
    handed in that were last used on another stream are the caller's to guard, and a result has to
    be waited for before another stream reads it, as for any torch operation."""

    _loss_bytes = {}                                             # workspace sizes of linear_cross_entropy

    def __init__(self, device=0):
        self._open(device)
        self._check(self._L.gbmuf_ops_create(device, ctypes.byref(self._h)))

    def _linear(self, call, query, pack, fields, in_place, like):
        """Runs a linear-layer call.  in_place: its operands are aligned bf16, no workspace."""
        if in_place:
            args = pack(*fields, 0, 0)
        else:
            args, need = pack(*fields, 0, 0), ctypes.c_int64()
            self._check(query(self._h, args, ctypes.byref(need)))
            if need.value:
                work = self._torch.empty(need.value, dtype=self._torch.uint8, device=like.device)
                args = pack(*fields, work.data_ptr(), need.value)
        st = call(self._h, args, self._raw_stream(self.device))
        if st != GBMUF_OK:
            self._check(st)

    def linear_forward(self, x, w, bias=None, residual=None, activation="none", keep_z=False, out=None,
                       z_out=None, stream=None):
        """``gbmuf_linear_forward``: y = act(x w^T + bias) + residual; with ``keep_z`` (or ``z_out``)
        returns (y, z), z = x w^T + bias.  x [rows][n_in], w [n_out][n_in]."""
        if stream is not None:
            return self._on_stream(stream, (out, z_out), self.linear_forward, x, w, bias, residual, activation,
                                   keep_z, out, z_out)
        rows, n_in = _two_dims("x", x)
        n_out = _two_dims("w", w)[0]
        dtype, dev, shape = x.dtype, self.device, (rows, n_out)
        code = _dtype_code(x)
        px, lx = _matrix("x", x, (rows, n_in), dtype, dev)
        pw, lw = _matrix("w", w, (n_out, n_in), dtype, dev)
        pb = _vector("bias", bias, n_out, dtype, dev)
        pr, lr = _matrix("residual", residual, shape, dtype, dev)
        act = ACTIVATIONS[activation]
        y, py, ly = _result("out", out, x, shape, dtype, dev)
        z, pz, lz = _result("z_out", z_out, x, shape, dtype, dev) if keep_z or z_out is not None else (None, 0, 0)
        self._linear(self._L.gbmuf_linear_forward, self._L.gbmuf_linear_forward_workspace, _pack_forward,
                     (rows, n_in, n_out, px, pw, pb, pr, py, pz, lx, lw, lr, ly, lz, code, act),
                     code == BF16 and not ((px | pw) & 15 or (lx | lw) & 7), x)
        return y if z is None else (y, z)

    def linear_backward_input(self, dz, w, residual=None, z_prev=None, activation="none", want_dx=None,
                              dx_out=None, dz_out=None, stream=None):
        """``gbmuf_linear_backward_input``: dx = dz w + residual, and with ``z_prev`` also
        dz_prev = dx * act'(z_prev).  Returns dx without ``z_prev``; dz_prev with it, or
        (dx, dz_prev) if ``want_dx`` or ``dx_out``."""
        if stream is not None:
            return self._on_stream(stream, (dx_out, dz_out), self.linear_backward_input, dz, w, residual, z_prev,
                                   activation, want_dx, dx_out, dz_out)
        rows, n_out = _two_dims("dz", dz)
        n_in = _two_dims("w", w)[1]
        dtype, dev, shape = dz.dtype, self.device, (rows, n_in)
        code = _dtype_code(dz)
        pd, ldd = _matrix("dz", dz, (rows, n_out), dtype, dev)
        pw, lw = _matrix("w", w, (n_out, n_in), dtype, dev)
        pr, lr = _matrix("residual", residual, shape, dtype, dev)
        pz, lz = _matrix("z_prev", z_prev, shape, dtype, dev)
        act = ACTIVATIONS[activation]
        if z_prev is None and dz_out is not None:
            raise ValueError("dz_out needs z_prev")
        dx = dp = None
        px = lx = pp = lp = 0
        if want_dx or z_prev is None or dx_out is not None:
            dx, px, lx = _result("dx_out", dx_out, dz, shape, dtype, dev)
        if z_prev is not None:
            dp, pp, lp = _result("dz_out", dz_out, dz, shape, dtype, dev)
        self._linear(self._L.gbmuf_linear_backward_input, self._L.gbmuf_linear_backward_input_workspace,
                     _pack_backward_input,
                     (rows, n_in, n_out, pd, pw, pr, pz, px, pp, ldd, lw, lr, lz, lx, lp, code, act),
                     code == BF16 and not ((pd | pw) & 15 or (ldd | lw) & 7), dz)
        return dx if dp is None else (dp if dx is None else (dx, dp))

    def linear_backward_weight(self, dz, x, grad_dtype=None, want_bias=True, dw_out=None, dbias_out=None,
                               accumulate=False, stream=None):
        """``gbmuf_linear_backward_weight``: dw = dz^T x and dbias = sum over the rows of dz, in
        ``grad_dtype`` (default: the operands' type); with ``accumulate`` added to ``dw_out`` and
        ``dbias_out``.  Returns dw, or (dw, dbias) if ``want_bias`` or ``dbias_out``."""
        if stream is not None:
            return self._on_stream(stream, (dw_out, dbias_out), self.linear_backward_weight, dz, x, grad_dtype,
                                   want_bias, dw_out, dbias_out, accumulate)
        rows, n_out = _two_dims("dz", dz)
        n_in = _two_dims("x", x)[1]
        dtype, dev, shape = dz.dtype, self.device, (n_out, n_in)
        code = _dtype_code(dz)
        pd, ldd = _matrix("dz", dz, (rows, n_out), dtype, dev)
        px, lx = _matrix("x", x, (rows, n_in), dtype, dev)
        if dw_out is not None:
            if grad_dtype is not None and dw_out.dtype is not grad_dtype:
                raise TypeError(f"dw_out must be {grad_dtype}, not {dw_out.dtype}")
            grad_dtype = dw_out.dtype
        elif grad_dtype is None:
            grad_dtype = dtype
        if accumulate and (dw_out is None or (want_bias and dbias_out is None)):
            raise ValueError("accumulate adds to dw_out and dbias_out: hand them in")
        dw, pw, lw = _result("dw_out", dw_out, dz, shape, grad_dtype, dev)
        db = dbias_out if dbias_out is not None else (
            dz.new_empty((n_out,), dtype=grad_dtype) if want_bias else None)
        pb = _vector("dbias_out", db, n_out, grad_dtype, dev)
        self._linear(self._L.gbmuf_linear_backward_weight, self._L.gbmuf_linear_backward_weight_workspace,
                     _pack_backward_weight,
                     (rows, n_in, n_out, pd, px, pw, pb, ldd, lx, lw, code, _dtype_code(dw),
                      1 if accumulate else 0, 0),
                     code == BF16 and not ((pd | px) & 15 or (ldd | lx) & 7), dz)
        return dw if db is None else (dw, db)

    def activation_backward(self, dy, z, activation, out=None, stream=None):
        """``gbmuf_activation_backward``: dy * act'(z); ``out`` may be dy."""
        if stream is not None:
            return self._on_stream(stream, (out,), self.activation_backward, dy, z, activation, out)
        shape = _two_dims("dy", dy)
        rows, cols = shape
        dtype, dev = dy.dtype, self.device
        code = _dtype_code(dy)
        py, ly = _matrix("dy", dy, shape, dtype, dev)
        pz, lz = _matrix("z", z, shape, dtype, dev)
        act = ACTIVATIONS[activation]
        dz = out if out is not None else dy.new_empty(shape)
        po, lo = _matrix("out", dz, shape, dtype, dev)
        self._check(self._L.gbmuf_activation_backward(self._h, rows, cols, code, act, py, ly, pz, lz, po, lo,
                                                      self._raw_stream(self.device)))
        return dz

    def cross_entropy(self, logits, targets, ignore_index=-100, row_weight=None, scale=1.0,
                      want_grad=True, dlogits_out=None, stream=None):
        """``gbmuf_cross_entropy``: (loss, lse, dlogits), or (loss, lse) without ``want_grad``.  loss
        and lse are float32 [rows]; ``dlogits_out`` may be the logits."""
        if stream is not None:
            return self._on_stream(stream, (dlogits_out,), self.cross_entropy, logits, targets, ignore_index,
                                   row_weight, scale, want_grad, dlogits_out)
        torch = self._torch
        shape = _two_dims("logits", logits)
        rows, vocab = shape
        dtype, dev = logits.dtype, self.device
        code = _dtype_code(logits)
        pl, ll = _matrix("logits", logits, shape, dtype, dev)
        pt = _vector("targets", targets, rows, torch.int64, dev)
        pw = _vector("row_weight", row_weight, rows, torch.float32, dev)
        d, pd, ldd = None, 0, 0
        if want_grad or dlogits_out is not None:
            d, pd, ldd = _result("dlogits_out", dlogits_out, logits, shape, dtype, dev)
        loss = logits.new_empty((rows,), dtype=torch.float32)
        lse = logits.new_empty((rows,), dtype=torch.float32)
        args = _pack_cross_entropy(rows, vocab, pl, pt, pw, loss.data_ptr(), lse.data_ptr(), pd, ll, ldd,
                                   ignore_index, code, scale)
        st = self._L.gbmuf_cross_entropy(self._h, args, self._raw_stream(self.device))
        if st != GBMUF_OK:
            self._check(st)
        return (loss, lse) if d is None else (loss, lse, d)

    def linear_cross_entropy(self, x, w, targets, bias=None, ignore_index=-100, row_weight=None, scale=1.0,
                             want_grad=True, want_weight_grad=True, grad_dtype=None, dx_out=None, dw_out=None,
                             dbias_out=None, accumulate=False, piece=0, stream=None):
        """``gbmuf_linear_cross_entropy``: the softmax layer x w^T + bias and its cross-entropy without the
        logits in memory.  Returns (loss, lse) without ``want_grad``; else (loss, lse, dx), followed with
        ``want_weight_grad`` by dw and, with a bias, dbias, in ``grad_dtype`` (default: the operands' type);
        with ``accumulate`` those are added to ``dw_out`` and ``dbias_out``.  loss and lse are float32 [rows].
        ``piece``: words of the vocabulary whose gradient is in memory at a time (0: the library's choice)."""
        if stream is not None:
            return self._on_stream(stream, (dx_out, dw_out, dbias_out), self.linear_cross_entropy, x, w, targets,
                                   bias, ignore_index, row_weight, scale, want_grad, want_weight_grad, grad_dtype,
                                   dx_out, dw_out, dbias_out, accumulate, piece)
        torch = self._torch
        rows, n_in = _two_dims("x", x)
        vocab = _two_dims("w", w)[0]
        dtype, dev = x.dtype, self.device
        code = _dtype_code(x)
        px, lx = _matrix("x", x, (rows, n_in), dtype, dev)
        pw, lw = _matrix("w", w, (vocab, n_in), dtype, dev)
        pb = _vector("bias", bias, vocab, dtype, dev)
        pt = _vector("targets", targets, rows, torch.int64, dev)
        pr = _vector("row_weight", row_weight, rows, torch.float32, dev)
        if not want_grad and not (dx_out is None and dw_out is None and dbias_out is None):
            raise ValueError("dx_out, dw_out and dbias_out need want_grad")
        if not want_weight_grad and not (dw_out is None and dbias_out is None):
            raise ValueError("dw_out and dbias_out need want_weight_grad")
        if dbias_out is not None and bias is None:
            raise ValueError("dbias_out needs a bias")
        weights = want_grad and want_weight_grad
        for name, t in (("dw_out", dw_out), ("dbias_out", dbias_out)):
            if t is None:
                continue
            if grad_dtype is None:
                grad_dtype = t.dtype
            elif t.dtype is not grad_dtype:
                raise TypeError(f"{name} must be {grad_dtype}, not {t.dtype}")
        if grad_dtype is None:
            grad_dtype = dtype
        if accumulate and weights and (dw_out is None or (bias is not None and dbias_out is None)):
            raise ValueError("accumulate adds to dw_out and dbias_out: hand them in")
        results, pdx, ldx, pdw, ldw, pdb, grad_code = [], 0, 0, 0, 0, 0, code
        if want_grad:
            dx, pdx, ldx = _result("dx_out", dx_out, x, (rows, n_in), dtype, dev)
            results.append(dx)
        if weights:
            dw, pdw, ldw = _result("dw_out", dw_out, x, (vocab, n_in), grad_dtype, dev)
            grad_code = _dtype_code(dw)
            results.append(dw)
            if bias is not None:
                db = dbias_out if dbias_out is not None else x.new_empty((vocab,), dtype=grad_dtype)
                pdb = _vector("dbias_out", db, vocab, grad_dtype, dev)
                results.append(db)
        loss = x.new_empty((rows,), dtype=torch.float32)
        lse = x.new_empty((rows,), dtype=torch.float32)
        fields = (rows, n_in, vocab, px, pw, pb, pt, pr, loss.data_ptr(), lse.data_ptr(), pdx, pdw, pdb, lx, lw, ldx,
                  ldw, ignore_index, piece, code, grad_code, 1 if accumulate else 0, scale)
        # the bytes follow from sizes, types, alignment and which results there are
        key = (dev, rows, n_in, vocab, code, px & 15, pw & 15, lx, lw, piece, pdx != 0, pdw != 0, pdb != 0, pr != 0)
        need = self._loss_bytes.get(key)
        if need is None:
            answer = ctypes.c_int64()
            self._check(self._L.gbmuf_linear_cross_entropy_workspace(
                self._h, _pack_linear_cross_entropy(*fields, 0, 0), ctypes.byref(answer)))
            if len(self._loss_bytes) >= 256:
                self._loss_bytes.clear()
            need = self._loss_bytes[key] = answer.value
        work = torch.empty(need, dtype=torch.uint8, device=x.device)
        args = _pack_linear_cross_entropy(*fields, work.data_ptr() if need else 0, need)
        st = self._L.gbmuf_linear_cross_entropy(self._h, args, self._raw_stream(dev))
        if st != GBMUF_OK:
            self._check(st)
        return (loss, lse, *results)

    def top_logits(self, logits, k, temperature=1.0, want_lse=True, values_out=None, index_out=None, lse_out=None,
                   stream=None):
        """``gbmuf_top_logits``: (values, index, lse) of the k largest logits of each row, largest first, lower
        indices first among equal ones; (values, index) without ``want_lse``.  index is int64, lse (float32) the
        log-sum-exp of the row over the temperature."""
        if stream is not None:
            return self._on_stream(stream, (values_out, index_out, lse_out), self.top_logits, logits, k, temperature,
                                   want_lse, values_out, index_out, lse_out)
        torch = self._torch
        shape = _two_dims("logits", logits)
        rows, vocab = shape
        dtype, dev = logits.dtype, self.device
        code = _dtype_code(logits)
        pl, ll = _matrix("logits", logits, shape, dtype, dev)
        if not 1 <= k <= 256:
            raise ValueError("k must be 1 .. 256")
        values, pv, lv = _result("values_out", values_out, logits, (rows, k), dtype, dev)
        index, pi, li = _result("index_out", index_out, logits, (rows, k), torch.int64, dev)
        lse = lse_out
        if lse is None and want_lse:
            lse = logits.new_empty((rows,), dtype=torch.float32)
        args = _pack_top_logits(rows, vocab, pl, pv, pi, _vector("lse_out", lse, rows, torch.float32, dev), ll, lv, li, code,
                                k, temperature, 0)
        self._check(self._L.gbmuf_top_logits(self._h, args, self._raw_stream(dev)))
        return (values, index) if lse is None else (values, index, lse)

    def distillation(self, logits, teacher_logits, teacher_index, teacher_lse=None, temperature=1.0, targets=None,
                     hard_weight=0.0, ignore_index=-100, row_weight=None, scale=1.0, want_grad=True, dlogits_out=None,
                     stream=None):
        """``gbmuf_distillation``: (loss, lse, dlogits), or (loss, lse) without ``want_grad``: the loss of a
        student's logits against a teacher's largest ones (as :meth:`top_logits` gives them), mixed with the
        cross-entropy of ``targets`` by ``hard_weight``.  ``dlogits_out`` may be the logits."""
        if stream is not None:
            return self._on_stream(stream, (dlogits_out,), self.distillation, logits, teacher_logits, teacher_index,
                                   teacher_lse, temperature, targets, hard_weight, ignore_index, row_weight, scale,
                                   want_grad, dlogits_out)
        torch = self._torch
        shape = _two_dims("logits", logits)
        rows, vocab = shape
        k = _two_dims("teacher_logits", teacher_logits)[1]
        dtype, dev = logits.dtype, self.device
        code = _dtype_code(logits)
        pl, ll = _matrix("logits", logits, shape, dtype, dev)
        teacher_code = _dtype_code(teacher_logits)
        px, lx = _matrix("teacher_logits", teacher_logits, (rows, k), teacher_logits.dtype, dev)
        pi, li = _matrix("teacher_index", teacher_index, (rows, k), torch.int64, dev)
        pe = _vector("teacher_lse", teacher_lse, rows, torch.float32, dev)
        pt = _vector("targets", targets, rows, torch.int64, dev)
        pw = _vector("row_weight", row_weight, rows, torch.float32, dev)
        d, pd, ldd = None, 0, 0
        if want_grad or dlogits_out is not None:
            d, pd, ldd = _result("dlogits_out", dlogits_out, logits, shape, dtype, dev)
        loss = logits.new_empty((rows,), dtype=torch.float32)
        lse = logits.new_empty((rows,), dtype=torch.float32)
        args = _pack_distillation(rows, vocab, pl, px, pi, pe, pt, pw, loss.data_ptr(), lse.data_ptr(), pd, ll, lx, li,
                                  ldd, ignore_index, code, teacher_code, k, temperature, hard_weight, scale)
        self._check(self._L.gbmuf_distillation(self._h, args, self._raw_stream(dev)))
        return (loss, lse) if d is None else (loss, lse, d)

    def device_status(self, stream=None) -> int:
        """Waits for the stream; reads and clears the status word."""
        v = ctypes.c_int32(-1)
        self._check(self._L.gbmuf_ops_device_status(self._h, self._on(stream), ctypes.byref(v)))
        return v.value

    def destroy(self):
        if self._h:
            self._L.gbmuf_ops_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


_local_ops = {}


def local_ops(device=None) -> LocalOps:
    """The process's :class:`LocalOps` of a device (default: the current one)."""
    if device is None:
        import torch
        device = torch.cuda.current_device()
    ops = _local_ops.get(device)
    if ops is None:
        ops = _local_ops[device] = LocalOps(device)
    return ops


def _rows_cols(name, t):
    """A tensor as rows of elements that follow one another: (rows, cols, row stride)."""
    dims = [(n, s) for n, s in zip(t.shape, t.stride()) if n != 1]
    if t.numel() == 0 or not dims:
        return 1, t.numel(), max(1, t.numel())
    cols, inner = 1, 1
    while dims and dims[-1][1] == inner:
        cols *= dims[-1][0]
        inner = cols
        dims.pop()
    rows, ld = 1, cols
    if dims:
        rows, ld = dims[-1]
        dims.pop()
        while dims and dims[-1][1] == ld * rows:
            rows *= dims.pop()[0]
    if dims or ld < cols:
        raise ValueError(f"{name} must be rows of elements that follow one another, with one stride")
    return rows, cols, ld


class GradClip(_OnDevice):
    """``gbmuf_clip_*``: the gradient norm of each group (a worker) over a list of tensors, and the
    clipped copies.  entries: (gradient, out or None, group); gradient float32 or bfloat16, out of
    the same shape in float32 or the gradient's type (or the gradient itself)."""

    def __init__(self, entries, groups=1, device=None):
        entries = list(entries)
        if device is None:
            import torch
            device = entries[0][0].get_device() if entries else torch.cuda.current_device()
        self._open(device)
        self.groups = groups
        arr = self._table(entries)
        self._check(self._L.gbmuf_clip_create(device, groups, len(entries), arr, ctypes.byref(self._h)))
        self._keep = entries

    def _table(self, entries):
        arr = (GradTensor * len(entries))()
        for i, (g, out, group) in enumerate(entries):
            for name, t in (("gradient", g), ("out", out)):
                if t is not None and (t.device.type != "cuda" or t.device.index != self.device):
                    raise ValueError(f"{name} {i} is on {t.device}, not on cuda:{self.device}")
            if out is not None and out.shape != g.shape:
                raise ValueError(f"out {i} must have its gradient's shape")
            # dimensions in the order of memory, the same for both (a transposed pair is fine)
            order = sorted(range(g.dim()), key=lambda d: -g.stride(d))
            g = g.permute(order)
            rows, cols, ld = _rows_cols(f"gradient {i}", g)
            ld_out = 0
            if out is not None:
                out = out.permute(order)
                r2, c2, ld_out = _rows_cols(f"out {i}", out)
                if (r2, c2) != (rows, cols):       # one of the two is whole: cut it like the other
                    if r2 * c2 != rows * cols or 1 not in (r2, rows):
                        raise ValueError(f"out {i} and its gradient have rows of different lengths")
                    if r2 == 1:
                        ld_out = cols
                    else:
                        rows, cols, ld = r2, c2, c2
            arr[i] = GradTensor(g.data_ptr(), None if out is None else out.data_ptr(), rows, cols, ld,
                                ld_out, _dtype_code(g), 0 if out is None else _dtype_code(out), group, 0)
        return arr

    def set_tensors(self, entries):
        """New tensors (and groups) for the same number of groups; waits for this handle's work.  A graph
        recorded before goes on with the tensors of then, which the caller keeps alive for it."""
        entries = list(entries)
        self._check(self._L.gbmuf_clip_set_tensors(self._h, len(entries), self._table(entries)))
        self._keep = entries

    def _norms(self, out):
        if out is None:
            return self._torch.empty(self.groups, dtype=self._torch.float32, device=f"cuda:{self.device}")
        if out.dtype is not self._torch.float32 or out.dim() != 1 or out.shape[0] != self.groups \
                or out.device.type != "cuda" or out.device.index != self.device \
                or (self.groups > 1 and out.stride(0) != 1):
            raise ValueError(f"norms_out must be contiguous float32 [{self.groups}] on cuda:{self.device}")
        return out

    def norms(self, norms_out=None, stream=None):
        """``gbmuf_clip_norms``: float32 [groups].  ``stream`` as for :class:`LocalOps`."""
        if stream is not None:
            return self._on_stream(stream, (norms_out,), self.norms, norms_out)
        norms = self._norms(norms_out)
        self._check(self._L.gbmuf_clip_norms(self._h, norms.data_ptr(), self._raw_stream(self.device)))
        return norms

    def clip(self, max_norm, norms_out=None, stream=None):
        """``gbmuf_clip_scale``: writes every entry's out; returns the norms before clipping.  ``stream`` as
        for :class:`LocalOps`."""
        if stream is not None:
            return self._on_stream(stream, (norms_out,), self.clip, max_norm, norms_out)
        norms = self._norms(norms_out)
        self._check(self._L.gbmuf_clip_scale(self._h, max_norm, norms.data_ptr(), self._raw_stream(self.device)))
        return norms

    def device_status(self, stream=None) -> int:
        """Waits for the stream; reads and clears the status word."""
        v = ctypes.c_int32(-1)
        self._check(self._L.gbmuf_clip_device_status(self._h, self._on(stream), ctypes.byref(v)))
        return v.value

    def selftest_wait_timeout(self, stream=None):
        """``gbmuf_clip_selftest_wait_timeout``: a wait that expires, after which ``device_status`` says so."""
        self._check(self._L.gbmuf_clip_selftest_wait_timeout(self._h, self._on(stream)))

    def destroy(self):
        if self._h:
            self._L.gbmuf_clip_destroy(self._h)
            self._h = ctypes.c_void_p()
            self._keep = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
