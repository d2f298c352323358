"""Thin ctypes binding of ``libhccs.so``: argument marshalling only.

Every function mirrors the C entry point of the same name in ``include/hccs.h``
and raises :class:`HccsError` on a non-zero status.  Tensors are torch tensors
(device memory and streams come from PyTorch); nothing here computes.
There is no fallback: if the compiled library is missing, importing fails.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "csrc", "libhccs.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_02292_b200.build` "
                      "(needs nvcc); there is no CPU implementation to fall back to")

_lib = ctypes.CDLL(LIB_PATH)

HCCS_OK = 0
HCCS_ERR_INVALID_ARG = 1
HCCS_ERR_CONSTRAINT = 2
HCCS_ERR_NOT_UPLOADED = 3
HCCS_ERR_UNSUPPORTED = 4
HCCS_ERR_CUDA = 5
HCCS_ERR_DEVICE_TIMEOUT = 6
HCCS_ERR_DEVICE_INDEX = 7

HCCS_OUT_U8 = 0
HCCS_OUT_U16 = 1
HCCS_RECIP_DIV = 0
HCCS_RECIP_CLB = 2
HCCS_CAUSAL = 4
HCCS_RECIP_REAL = 8

HCCS_I32, HCCS_F32, HCCS_BF16, HCCS_F16 = 0, 1, 2, 3
HCCS_ROPE_NONE, HCCS_ROPE_LINEAR, HCCS_ROPE_BASE, HCCS_ROPE_WAVELENGTH, HCCS_ROPE_DIMENSION = 0, 1, 2, 3, 4
HCCS_MAX_CACHE_HEADS = 256
HCCS_MAX_CACHE_KEYS = 131072
HCCS_MAX_ROT_DIM = 128
HCCS_MAX_AXES = 4
HCCS_AXES_SECTIONS, HCCS_AXES_TURNS = 0, 1

EXPORTS = ("hccs_create", "hccs_destroy", "hccs_params_check", "hccs_params_upload", "hccs_forward",
           "hccs_forward_keylen", "hccs_forward_host",
           "hccs_attention_fused", "hccs_attention_fused_keylen", "hccs_attention_fused_f32", "hccs_attention_fused_i8", "hccs_device_status", "hccs_last_cuda_error", "hccs_status_string",
           "hccs_launch_count", "hccs_forward_static_scratch", "hccs_calibrate", "hccs_debug_wait_timeout",
           "hccs_rope_frequencies", "hccs_cache_write", "hccs_cache_read", "hccs_params_upload_wide", "hccs_attention_cached",
           "hccs_rope_axes", "hccs_cache_write_axes", "hccs_states_write", "hccs_attention_cross")

_vp, _i32, _u32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32

_lib.hccs_create.argtypes = [ctypes.POINTER(_vp), ctypes.c_int]
_lib.hccs_create.restype = ctypes.c_int
_lib.hccs_destroy.argtypes = [_vp]
_lib.hccs_destroy.restype = ctypes.c_int
_lib.hccs_params_upload.argtypes = [_vp, _vp, _i32, _i32, _i32, ctypes.POINTER(_i32), _vp]
_lib.hccs_params_upload.restype = ctypes.c_int
_lib.hccs_params_check.argtypes = [_vp, _i32, _i32, ctypes.POINTER(_i32)]
_lib.hccs_params_check.restype = ctypes.c_int
_lib.hccs_forward.argtypes = [_vp, _vp, _vp, _i32, _i32, _i32, _i32, _u32, _vp]
_lib.hccs_forward.restype = ctypes.c_int
_lib.hccs_forward_keylen.argtypes = [_vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _u32, _vp]
_lib.hccs_forward_keylen.restype = ctypes.c_int
_lib.hccs_forward_host.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _u32, _vp]
_lib.hccs_forward_host.restype = ctypes.c_int
_lib.hccs_attention_fused.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32,
                                      _u32, _vp]
_lib.hccs_attention_fused.restype = ctypes.c_int
_lib.hccs_attention_fused_keylen.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32,
                                             _u32, _vp]
_lib.hccs_attention_fused_keylen.restype = ctypes.c_int
_lib.hccs_attention_fused_f32.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32,
                                          _u32, _vp]
_lib.hccs_attention_fused_f32.restype = ctypes.c_int
_lib.hccs_attention_fused_i8.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _i32, _i32, _i32, _i32, _i32,
                                         _u32, _vp]
_lib.hccs_attention_fused_i8.restype = ctypes.c_int
_lib.hccs_device_status.argtypes = [_vp, ctypes.POINTER(_u32), _vp]
_lib.hccs_device_status.restype = ctypes.c_int
_lib.hccs_last_cuda_error.argtypes = [_vp]
_lib.hccs_last_cuda_error.restype = _i32
_lib.hccs_status_string.argtypes = [ctypes.c_int]
_lib.hccs_status_string.restype = ctypes.c_char_p
_lib.hccs_launch_count.argtypes = [_vp]
_lib.hccs_launch_count.restype = ctypes.c_uint64
_lib.hccs_debug_wait_timeout.argtypes = [_vp, _i32, ctypes.c_int64, _vp]
_lib.hccs_debug_wait_timeout.restype = ctypes.c_int


_lib.hccs_forward_static_scratch.argtypes = [_vp, _i32, _i32, _i32, _vp, _vp, _i32, _i32, _i32, _i32, _u32,
                                             ctypes.POINTER(_u32), _vp]
_lib.hccs_forward_static_scratch.restype = ctypes.c_int


class Rope(ctypes.Structure):
    """``hccs_rope_t``: rotary frequencies in radians per position, one per pair of rotated dims."""
    _fields_ = [("rot_dim", _i32), ("interleaved", _i32), ("scale", ctypes.c_double),
                ("freq", ctypes.c_double * (HCCS_MAX_ROT_DIM // 2))]

    def __init__(self, freq=(), interleaved: bool = False, scale: float = 1.0):
        freq = [float(f) for f in freq]
        if len(freq) > HCCS_MAX_ROT_DIM // 2:
            raise ValueError(f"at most {HCCS_MAX_ROT_DIM // 2} frequencies, got {len(freq)}")
        super().__init__(2 * len(freq), int(bool(interleaved)), float(scale))
        for i, f in enumerate(freq):
            self.freq[i] = f


class RopeAxes(ctypes.Structure):
    """``hccs_rope_axes_t``: frequencies and, per pair of rotated dims, the axis whose positions turn it."""
    _fields_ = [("rope", Rope), ("num_axes", _i32), ("axis", ctypes.c_uint8 * (HCCS_MAX_ROT_DIM // 2))]

    def __init__(self, freq=(), axis=(), interleaved: bool = False, scale: float = 1.0, num_axes: int | None = None):
        axis = [int(x) for x in axis]
        if len(axis) != len(freq):
            raise ValueError(f"{len(freq)} frequencies and {len(axis)} axes: there is one of each per pair")
        count = max(axis, default=0) + 1 if num_axes is None else int(num_axes)
        if not 1 <= count <= HCCS_MAX_AXES or any(not 0 <= x < count for x in axis):
            raise ValueError(f"axes are numbered 0 to {HCCS_MAX_AXES - 1} at most")
        super().__init__(Rope(freq, interleaved, scale), count)
        for i, x in enumerate(axis):
            self.axis[i] = x


class _RopeScaling(ctypes.Structure):
    _fields_ = [("kind", _i32), ("factor", ctypes.c_double), ("low", ctypes.c_double), ("high", ctypes.c_double),
                ("original_len", ctypes.c_double)]


_i64 = ctypes.c_int64
_lib.hccs_rope_frequencies.argtypes = [ctypes.POINTER(Rope), _i32, _i32, ctypes.c_double, ctypes.POINTER(_RopeScaling)]
_lib.hccs_rope_frequencies.restype = ctypes.c_int
_lib.hccs_cache_write.argtypes = [_vp, _vp, _vp, _vp, ctypes.c_int, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                  _i32, _i32, _i32, _i32, _i32, _i32, _vp]
_lib.hccs_cache_write.restype = ctypes.c_int
_lib.hccs_cache_read.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_int, _i32, _i32, _i32, _i32, _i32, _i32,
                                 _i32, _i32, _vp]
_lib.hccs_cache_read.restype = ctypes.c_int
_lib.hccs_params_upload_wide.argtypes = [_vp, _vp, _i32, _i32, ctypes.POINTER(_i32), _vp]
_lib.hccs_params_upload_wide.restype = ctypes.c_int
_lib.hccs_attention_cached.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _i32, _vp, _vp, ctypes.c_int,
                                       _i32, _i32, _i32, _i32, _i32, _i32, _i32, _i32, _i32, _i32, _u32, _vp]
_lib.hccs_attention_cached.restype = ctypes.c_int


def hccs_rope_frequencies(rot_dim: int, base: float = 10000.0, interleaved: bool = False, kind: int = HCCS_ROPE_NONE,
                          factor: float = 1.0, low: float = 1.0, high: float = 4.0, original_len: float = 8192.0) -> Rope:
    """A :class:`Rope` with the frequencies base^(-2i/rot_dim), changed for longer contexts as ``kind`` says."""
    rope = Rope()
    sc = _RopeScaling(int(kind), float(factor), float(low), float(high), float(original_len))
    st = _lib.hccs_rope_frequencies(ctypes.byref(rope), int(rot_dim), int(bool(interleaved)), float(base), ctypes.byref(sc))
    if st != HCCS_OK:
        raise HccsError(st, "hccs_rope_frequencies")
    return rope


_lib.hccs_rope_axes.argtypes = [ctypes.POINTER(RopeAxes), _i32, _i32, ctypes.c_double, ctypes.POINTER(_RopeScaling), _vp, _i32, _i32, _i32]
_lib.hccs_rope_axes.restype = ctypes.c_int
_lib.hccs_cache_write_axes.argtypes = [_vp, _vp, _vp, _vp, ctypes.c_int, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _vp, _vp,
                                       _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _i32, _vp]
_lib.hccs_cache_write_axes.restype = ctypes.c_int
_lib.hccs_states_write.argtypes = [_vp, _vp, _vp, _vp, ctypes.c_int, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _vp,
                                   _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _vp]
_lib.hccs_states_write.restype = ctypes.c_int
_lib.hccs_attention_cross.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, ctypes.c_int,
                                      _i32, _i32, _i32, _i32, _i32, _i32, _i32, _i32, _u32, _vp]
_lib.hccs_attention_cross.restype = ctypes.c_int


def hccs_rope_axes(rot_dim: int, pairs, base: float = 10000.0, interleaved: bool = False, order: int = HCCS_AXES_SECTIONS,
                   restart: bool = False, kind: int = HCCS_ROPE_NONE, factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                   original_len: float = 8192.0) -> RopeAxes:
    """A :class:`RopeAxes` whose axis x has ``pairs[x]`` of the rot_dim / 2 pairs, dealt out in sections or in turns, with the
    frequencies of :func:`hccs_rope_frequencies` over all pairs, or (``restart``) over each axis's own."""
    axes = RopeAxes()
    count = np.ascontiguousarray(pairs, dtype=np.int32).reshape(-1)
    sc = _RopeScaling(int(kind), float(factor), float(low), float(high), float(original_len))
    st = _lib.hccs_rope_axes(ctypes.byref(axes), int(rot_dim), int(bool(interleaved)), float(base), ctypes.byref(sc),
                             count.ctypes.data_as(_vp), count.size, int(order), int(bool(restart)))
    if st != HCCS_OK:
        raise HccsError(st, "hccs_rope_axes")
    return axes


class _CalibGrid(ctypes.Structure):
    _fields_ = [(k, _i32) for k in ("D_lo", "D_hi", "D_step", "S_lo", "S_hi", "S_step", "B_step")]


_lib.hccs_calibrate.argtypes = [_vp, _i32, _i32, _i32, _i32, ctypes.c_double, ctypes.POINTER(_CalibGrid), _vp, _vp, _vp]
_lib.hccs_calibrate.restype = ctypes.c_int


def hccs_calibrate(logits, alpha: float, grid, stream=None):
    """Grid-scan calibration of every head on device logits [B,H,Lq,Lk]; grid = (D_lo, D_hi, D_step,
    S_lo, S_hi, S_step, B_step).  Returns (theta int32 [H,3], kl float64 [H])."""
    B, H, Lq, Lk = logits.shape
    _check_tensor(logits, "logits", 1)
    g = _CalibGrid(*[int(v) for v in grid])
    best = np.zeros((H, 3), dtype=np.int32)
    kl = np.zeros(H, dtype=np.float64)
    st = _lib.hccs_calibrate(_ptr(logits), B, H, Lq, Lk, float(alpha), ctypes.byref(g),
                             best.ctypes.data_as(_vp), kl.ctypes.data_as(_vp), _stream_ptr(stream))
    if st != HCCS_OK:
        raise HccsError(st, "hccs_calibrate")
    return best, kl


def hccs_status_string(status: int) -> str:
    return _lib.hccs_status_string(int(status)).decode()


class HccsError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = int(status)
        super().__init__(f"{where}: {hccs_status_string(status)}{(' ' + detail) if detail else ''}")


def _stream_ptr(stream):
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    if isinstance(stream, int):
        return _vp(stream)
    return _vp(stream.cuda_stream)


def _ptr(t):
    return _vp(t.data_ptr()) if t is not None else _vp(0)


def hccs_params_check(params, n_design: int):
    """(status, bad_head) of the host-side admissibility check; needs no GPU."""
    arr = np.ascontiguousarray(params, dtype=np.int32).reshape(-1, 3)
    bad = _i32(-1)
    st = _lib.hccs_params_check(arr.ctypes.data_as(_vp), arr.shape[0], int(n_design), ctypes.byref(bad))
    return int(st), int(bad.value)


class Context:
    """Owns one ``hccs_ctx_t`` (created on ``device``) and exposes the entry points as methods."""

    def __init__(self, device: int = 0):
        h = _vp()
        st = _lib.hccs_create(ctypes.byref(h), int(device))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_create")
        self._h = h
        self.device = int(device)

    def close(self):
        if getattr(self, "_h", None):
            _lib.hccs_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- hccs_params_upload
    def hccs_params_upload(self, params, n_design: int, out_shift: int = 0, stream=None) -> None:
        arr = np.ascontiguousarray(params, dtype=np.int32).reshape(-1, 3)
        bad = _i32(-1)
        st = _lib.hccs_params_upload(self._h, arr.ctypes.data_as(_vp), arr.shape[0], int(n_design),
                                     int(out_shift), ctypes.byref(bad), _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_params_upload", f"(head {bad.value})" if bad.value >= 0 else "")

    # -- hccs_forward
    def hccs_forward(self, logits, probs, flags: int = 0, stream=None) -> None:
        B, H, Lq, Lk = logits.shape
        _check_tensor(logits, "logits", 1)
        _check_tensor(probs, "probs", 2 if flags & HCCS_OUT_U16 else 1, logits.shape)
        st = _lib.hccs_forward(self._h, _ptr(logits), _ptr(probs), B, H, Lq, Lk, int(flags),
                               _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_forward")

    # -- hccs_forward_keylen
    def hccs_forward_keylen(self, logits, probs, key_len, flags: int = 0, stream=None) -> None:
        B, H, Lq, Lk = logits.shape
        _check_tensor(logits, "logits", 1)
        _check_tensor(probs, "probs", 2 if flags & HCCS_OUT_U16 else 1, logits.shape)
        _check_tensor(key_len, "key_len", 4, (B,))
        st = _lib.hccs_forward_keylen(self._h, _ptr(logits), _ptr(probs), _ptr(key_len), B, H, Lq, Lk,
                                      int(flags), _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_forward_keylen")

    # -- hccs_forward_host
    def hccs_forward_host(self, logits_host, probs_host, logits_staging, probs_staging,
                          flags: int = 0, stream=None) -> None:
        B, H, Lq, Lk = logits_host.shape
        osz = 2 if flags & HCCS_OUT_U16 else 1
        _check_tensor(logits_host, "logits_host", 1, device="cpu")
        _check_tensor(probs_host, "probs_host", osz, logits_host.shape, device="cpu")
        _check_tensor(logits_staging, "logits_staging", 1, logits_host.shape)
        _check_tensor(probs_staging, "probs_staging", osz, logits_host.shape)
        st = _lib.hccs_forward_host(self._h, _ptr(logits_host), _ptr(probs_host), _ptr(logits_staging),
                                    _ptr(probs_staging), B, H, Lq, Lk, int(flags), _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_forward_host")

    # -- hccs_attention_fused
    def hccs_attention_fused(self, Q, K, V, O, requant_mult, requant_shift: int, flags: int = 0,
                             stream=None) -> None:
        B, H, L, d = Q.shape
        for name, t in (("Q", Q), ("K", K), ("V", V)):
            _check_tensor(t, name, 1, Q.shape)
        _check_tensor(O, "O", 4, Q.shape)
        mult = np.ascontiguousarray(requant_mult, dtype=np.int32).reshape(-1)
        if mult.size != H:
            raise ValueError("requant_mult must have H entries")
        st = _lib.hccs_attention_fused(self._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(O),
                                       mult.ctypes.data_as(_vp), int(requant_shift), B, H, L, d,
                                       int(flags), _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_attention_fused")

    # -- hccs_attention_fused_keylen
    def hccs_attention_fused_keylen(self, Q, K, V, O, key_len, requant_mult, requant_shift: int,
                                    flags: int = 0, stream=None) -> None:
        B, H, L, d = Q.shape
        for name, t in (("Q", Q), ("K", K), ("V", V)):
            _check_tensor(t, name, 1, Q.shape)
        _check_tensor(O, "O", 4, Q.shape)
        _check_tensor(key_len, "key_len", 4, (B,))
        mult = np.ascontiguousarray(requant_mult, dtype=np.int32).reshape(-1)
        if mult.size != H:
            raise ValueError("requant_mult must have H entries")
        st = _lib.hccs_attention_fused_keylen(self._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(key_len),
                                              mult.ctypes.data_as(_vp), int(requant_shift), B, H, L, d,
                                              int(flags), _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_attention_fused_keylen")

    # -- hccs_attention_fused_f32
    def hccs_attention_fused_f32(self, Q, K, V, O, out_scale, requant_mult, requant_shift: int,
                                 flags: int = 0, stream=None) -> None:
        B, H, L, d = Q.shape
        for name, t in (("Q", Q), ("K", K), ("V", V)):
            _check_tensor(t, name, 1, Q.shape)
        _check_tensor(O, "O", 4, Q.shape)
        mult = np.ascontiguousarray(requant_mult, dtype=np.int32).reshape(-1)
        scale = np.ascontiguousarray(out_scale, dtype=np.float32).reshape(-1)
        if mult.size != H or scale.size != H:
            raise ValueError("requant_mult and out_scale must have H entries")
        st = _lib.hccs_attention_fused_f32(self._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(O),
                                           scale.ctypes.data_as(_vp), mult.ctypes.data_as(_vp),
                                           int(requant_shift), B, H, L, d, int(flags), _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_attention_fused_f32")

    # -- hccs_attention_fused_i8
    def hccs_attention_fused_i8(self, Q, K, V, O, out_mult, out_shift: int, requant_mult, requant_shift: int,
                                flags: int = 0, stream=None) -> None:
        B, H, L, d = Q.shape
        for name, t in (("Q", Q), ("K", K), ("V", V)):
            _check_tensor(t, name, 1, Q.shape)
        _check_tensor(O, "O", 1, Q.shape)
        mult = np.ascontiguousarray(requant_mult, dtype=np.int32).reshape(-1)
        omult = np.ascontiguousarray(out_mult, dtype=np.int32).reshape(-1)
        if mult.size != H or omult.size != H:
            raise ValueError("requant_mult and out_mult must have H entries")
        st = _lib.hccs_attention_fused_i8(self._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), omult.ctypes.data_as(_vp),
                                          int(out_shift), mult.ctypes.data_as(_vp), int(requant_shift), B, H, L, d,
                                          int(flags), _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_attention_fused_i8")

    # -- hccs_params_upload_wide
    def hccs_params_upload_wide(self, params, n_design: int, stream=None) -> None:
        arr = np.ascontiguousarray(params, dtype=np.int32).reshape(-1, 3)
        bad = _i32(-1)
        st = _lib.hccs_params_upload_wide(self._h, arr.ctypes.data_as(_vp), arr.shape[0], int(n_design),
                                          ctypes.byref(bad), _raw_stream(self.device) if stream is None else _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_params_upload_wide", f"(head {bad.value})" if bad.value >= 0 else "")

    # -- hccs_cache_write
    def hccs_cache_write(self, q, k, v, q8, k_pages, v_pages, positions, slots, q_step, k_step, v_step,
                         rope: Rope | None = None, stream=None) -> None:
        """Rotates and quantises tokens: q [T,Hq,d] to q8, k and v [T,Hkv,d] into the pools at ``slots``.  q (with q8 and
        q_step) may be None, or k and v (with the pools, the slots and their steps).  q, k and v may be views whose tokens
        are any multiple of 16 bytes apart."""
        (some, T, d, Hq, Hkv, pages, size, qp, kp, vp, q8p, kpp, vpp, slotp, qs, ks, vs, q_stride, k_stride,
         v_stride) = self._paged_tokens(q, k, v, q8, k_pages, v_pages, slots, q_step, k_step, v_step)
        dev, posp, ropep = self.device, None, _rotation(rope, Rope)
        if positions is not None:
            if positions.get_device() != dev or positions.dtype not in _I32 or positions.shape != (T,) or not positions.is_contiguous():
                self._explain(positions, "positions", 4, (T,))
            posp = positions.data_ptr()
        st = _lib.hccs_cache_write(self._h, qp, kp, vp, _type_of(some), q_stride, k_stride, v_stride, posp, slotp,
                                   ropep, qs, ks, vs, q8p, kpp, vpp, T, Hq, Hkv, d, pages, size,
                                   _raw_stream(dev) if stream is None else _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_cache_write")

    # -- hccs_cache_write_axes
    def hccs_cache_write_axes(self, q, k, v, q8, k_pages, v_pages, positions, slots, q_step, k_step, v_step,
                              rope: RopeAxes | None = None, stream=None) -> None:
        """:meth:`hccs_cache_write` with positions [axes,T] (int32, any strides: the transpose of [T,axes] as well)."""
        (some, T, d, Hq, Hkv, pages, size, qp, kp, vp, q8p, kpp, vpp, slotp, qs, ks, vs, q_stride, k_stride,
         v_stride) = self._paged_tokens(q, k, v, q8, k_pages, v_pages, slots, q_step, k_step, v_step)
        ropep = _rotation(rope, RopeAxes)
        posp, axis_stride, token_stride = self._axes(positions, rope, T)
        st = _lib.hccs_cache_write_axes(self._h, qp, kp, vp, _type_of(some), q_stride, k_stride, v_stride, posp, axis_stride, token_stride,
                                        slotp, ropep, qs, ks, vs, q8p, kpp, vpp, T, Hq, Hkv, d, pages,
                                        size, _raw_stream(self.device) if stream is None else _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_cache_write_axes")

    def _paged_tokens(self, q, k, v, q8, k_pages, v_pages, slots, q_step, k_step, v_step):
        """What the two cache writes hand to the library."""
        some = q if q is not None else k
        if some is None:
            raise ValueError("q or k and v must be given")
        if (k is None) != (v is None):
            raise ValueError("k and v go together")
        T, _, d = some.shape
        Hq = Hkv = pages = size = 0
        qp = kp = vp = q8p = kpp = vpp = slotp = qs = ks = vs = None
        q_stride = k_stride = v_stride = 0
        dev, dtype = self.device, some.dtype
        if q is not None:
            if q8 is None:
                raise ValueError("q8 must be given with q")
            Hq = q.shape[1]
            if q8.get_device() != dev or q8.shape != q.shape or q8.dtype not in _I8 or not q8.is_contiguous():
                self._explain(q8, "q8", 1, q.shape)
            qp, q8p, qs = q.data_ptr(), q8.data_ptr(), _floats(q_step, "q_step", Hq)
            q_stride = self._tokens(q, "q", some)
        if k is not None:
            if k_pages is None or v_pages is None or slots is None:
                raise ValueError("k_pages, v_pages and slots must be given with k and v")
            shape = k.shape
            Hkv = shape[1]
            pages, _, size, _ = pool = k_pages.shape
            if v.dtype != dtype or v.shape != shape:
                raise ValueError("k and v must have one shape and type")
            k_stride, v_stride = self._tokens(k, "k", some), self._tokens(v, "v", some)
            if (k_pages.get_device() != dev or v_pages.get_device() != dev or slots.get_device() != dev or pool[1] != Hkv or pool[3] != d
                    or v_pages.shape != pool or k_pages.dtype not in _I8 or v_pages.dtype not in _I8 or slots.dtype not in _I64
                    or slots.shape != (T,) or not k_pages.is_contiguous() or not v_pages.is_contiguous() or not slots.is_contiguous()):
                self._explain(k_pages, "k_pages", 1, (pages, Hkv, size, d))
                self._explain(v_pages, "v_pages", 1, pool)
                self._explain(slots, "slots", 8, (T,))
            kp, vp, kpp, vpp, slotp = k.data_ptr(), v.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), slots.data_ptr()
            ks, vs = _floats(k_step, "k_step", Hkv), _floats(v_step, "v_step", Hkv)
        return (some, T, d, Hq, Hkv, pages, size, qp, kp, vp, q8p, kpp, vpp, slotp, qs, ks, vs, q_stride, k_stride, v_stride)

    def _axes(self, positions, rope, T):
        """(address, stride of the axes, stride of the tokens) of positions [axes,T]."""
        if positions is None:
            return None, 0, 0
        shape = positions.shape
        if positions.get_device() != self.device or positions.dtype not in _I32 or len(shape) != 2 or shape[1] != T:
            # (a copy, since any strides will do; and a first call's types are known from here on)
            self._explain(positions if positions.get_device() != self.device else positions.contiguous(), "positions", 4,
                          (shape[0] if len(shape) else 0, T))
        if rope is not None and shape[0] < rope.num_axes:
            raise ValueError(f"positions have {shape[0]} axes, the rotation {rope.num_axes}")
        return positions.data_ptr(), *positions.stride()

    # -- hccs_states_write
    def hccs_states_write(self, q, k, v, q8, k8, v8, positions, q_step, k_step, v_step, rope: RopeAxes | None = None, stream=None) -> None:
        """Rotates (by positions [axes,T], any strides) and quantises tokens q [T,Hq,d], k and v [T,Hkv,d] into dense tensors:
        q8, k8 and v8 are [T,heads,d], or [B,heads,L,d] with B*L = T (as ``hccs_attention_fused`` reads them).  q (with q8
        and q_step) may be None, or k and v (with theirs)."""
        some, out = (q, q8) if q is not None else (k, k8)
        if some is None:
            raise ValueError("q or k and v must be given")
        if (k is None) != (v is None):
            raise ValueError("k and v go together")
        if q is not None and q8 is None:
            raise ValueError("q8 must be given with q")
        if k is not None and (k8 is None or v8 is None):
            raise ValueError("k8 and v8 must be given with k and v")
        T, _, d = some.shape
        heads_first = out.ndim == 4
        L = out.shape[2] if heads_first else 1
        if heads_first and out.shape[0] * L != T:
            raise ValueError(f"[B,heads,L,d] of {tuple(out.shape)} does not hold {T} tokens")

        def dense(t, name, heads):
            shape = (T // L if L else 0, heads, L, d) if heads_first else (T, heads, d)
            if t.get_device() != self.device or t.shape != shape or t.dtype not in _I8 or not t.is_contiguous():
                self._explain(t, name, 1, shape)
            return t.data_ptr()

        Hq = Hkv = 0
        qp = kp = vp = q8p = k8p = v8p = qs = ks = vs = None
        q_stride = k_stride = v_stride = 0
        if q is not None:
            Hq = q.shape[1]
            qp, q8p, qs, q_stride = q.data_ptr(), dense(q8, "q8", Hq), _floats(q_step, "q_step", Hq), self._tokens(q, "q", some)
        if k is not None:
            Hkv = k.shape[1]
            if v.dtype != some.dtype or v.shape != k.shape:
                raise ValueError("k and v must have one shape and type")
            k_stride, v_stride = self._tokens(k, "k", some), self._tokens(v, "v", some)
            kp, vp, k8p, v8p = k.data_ptr(), v.data_ptr(), dense(k8, "k8", Hkv), dense(v8, "v8", Hkv)
            ks, vs = _floats(k_step, "k_step", Hkv), _floats(v_step, "v_step", Hkv)
        ropep = _rotation(rope, RopeAxes)
        posp, axis_stride, token_stride = self._axes(positions, rope, T)
        st = _lib.hccs_states_write(self._h, qp, kp, vp, _type_of(some), q_stride, k_stride, v_stride, posp, axis_stride, token_stride,
                                    ropep, qs, ks, vs, q8p, k8p, v8p, T, max(L, 1), Hq, Hkv, d,
                                    _raw_stream(self.device) if stream is None else _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_states_write")

    # -- hccs_cache_read
    def hccs_cache_read(self, k_pages, v_pages, page_table, out_start, k_out, v_out, k_step, v_step, max_len: int,
                        stream=None) -> None:
        """Values of the sequences of ``page_table`` [B,max_pages]: token j of sequence b to row out_start[b] + j of k_out and
        v_out [rows,Hkv,d] (either may be None)."""
        pages, Hkv, size, d = k_pages.shape
        B, max_pages = page_table.shape
        some = k_out if k_out is not None else v_out
        if some is None:
            raise ValueError("k_out or v_out must be given")
        rows = some.shape[0]
        out = []
        for name, t in (("k_out", k_out), ("v_out", v_out)):
            if t is not None and t.dtype != some.dtype:
                raise ValueError("k_out and v_out must have one type")
            out.append(None if t is None else self._output(t, name, (rows, Hkv, d)))
        st = _lib.hccs_cache_read(self._h, self._check(k_pages, "k_pages", 1), self._check(v_pages, "v_pages", 1, k_pages.shape),
                                  self._check(page_table, "page_table", 4), self._check(out_start, "out_start", 4, (B + 1,)),
                                  _floats(k_step, "k_step", Hkv), _floats(v_step, "v_step", Hkv), out[0], out[1], _type_of(some),
                                  B, max_pages, max_len, rows, Hkv, d, pages, size,
                                  _raw_stream(self.device) if stream is None else _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_cache_read")

    # -- hccs_attention_cached
    def hccs_attention_cached(self, Q, k_pages, v_pages, page_table, q_start, kv_len, O, requant_mult, requant_shift: int,
                              max_q: int, max_kv: int, tree_mask=None, out_scale=None, flags: int = 0, stream=None) -> None:
        """HCCS attention of the new tokens Q [T,Hq,d] over the cache.  O [T,Hq,d] is int32 (no out_scale), or float32,
        bfloat16 or float16."""
        T, Hq, d = shape = Q.shape
        pages, Hkv, size, dk = pool = k_pages.shape
        B, max_pages = page_table.shape
        dev = self.device
        if dk != d:
            raise ValueError(f"the cache holds heads of {dk}, Q of {d}")
        if (Q.get_device() != dev or k_pages.get_device() != dev or v_pages.get_device() != dev or page_table.get_device() != dev
                or q_start.get_device() != dev or kv_len.get_device() != dev or O.get_device() != dev or Q.dtype not in _I8
                or k_pages.dtype not in _I8 or v_pages.dtype not in _I8 or page_table.dtype not in _I32
                or q_start.dtype not in _I32 or kv_len.dtype not in _I32 or v_pages.shape != pool or O.shape != shape
                or q_start.shape != (B + 1,) or kv_len.shape != (B,) or not Q.is_contiguous() or not k_pages.is_contiguous()
                or not v_pages.is_contiguous() or not page_table.is_contiguous() or not q_start.is_contiguous()
                or not kv_len.is_contiguous() or not O.is_contiguous()):
            self._explain(Q, "Q", 1)
            self._explain(k_pages, "k_pages", 1)
            self._explain(v_pages, "v_pages", 1, pool)
            self._explain(page_table, "page_table", 4)
            self._explain(q_start, "q_start", 4, (B + 1,))
            self._explain(kv_len, "kv_len", 4, (B,))
            self._output(O, "O", shape)
        words, treep = 0, None
        if tree_mask is not None:
            words = tree_mask.shape[-1]
            if tree_mask.get_device() != dev or tree_mask.dtype not in _I32 or tree_mask.shape != (T, words) or not tree_mask.is_contiguous():
                self._explain(tree_mask, "tree_mask", 4, (T, words))
            if words < 1:                      # (an empty tensor has no address, and none means causal)
                raise ValueError("tree_mask must have a word or more per token")
            treep = tree_mask.data_ptr()
        st = _lib.hccs_attention_cached(
            self._h, Q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), q_start.data_ptr(), kv_len.data_ptr(),
            treep, words, _ints(requant_mult, "requant_mult", Hq), requant_shift,
            None if out_scale is None else _floats(out_scale, "out_scale", Hq), O.data_ptr(), _type_of(O), T, B, Hq, Hkv, d, max_pages,
            pages, size, max_q, max_kv, flags, _raw_stream(dev) if stream is None else _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_attention_cached")

    # -- hccs_attention_cross
    def hccs_attention_cross(self, Q, K, V, q_start, k_start, k_len, O, requant_mult, requant_shift: int, max_q: int, max_kv: int,
                             key_range=None, out_scale=None, flags: int = 0, stream=None) -> None:
        """HCCS attention of the queries Q [T,Hq,d] to the states K and V [S,Hkv,d] (int8; views whose keys are a multiple of 16
        bytes apart as well).  O [T,Hq,d] is int32 (no out_scale), or float32, bfloat16 or float16."""
        T, Hq, d = shape = Q.shape
        S, Hkv, dk = K.shape
        B = k_len.shape[0]
        dev = self.device
        if dk != d:
            raise ValueError(f"the states have heads of {dk}, Q of {d}")
        if (Q.get_device() != dev or q_start.get_device() != dev or k_start.get_device() != dev or k_len.get_device() != dev
                or O.get_device() != dev or Q.dtype not in _I8 or q_start.dtype not in _I32 or k_start.dtype not in _I32
                or k_len.dtype not in _I32 or O.shape != shape or q_start.shape != (B + 1,) or k_start.shape != (B,) or k_len.shape != (B,)
                or not Q.is_contiguous() or not q_start.is_contiguous() or not k_start.is_contiguous() or not k_len.is_contiguous()
                or not O.is_contiguous()):
            self._explain(Q, "Q", 1)
            self._explain(q_start, "q_start", 4, (B + 1,))
            self._explain(k_start, "k_start", 4, (B,))
            self._explain(k_len, "k_len", 4, (B,))
            self._output(O, "O", shape)
        k_stride, v_stride = self._states(K, "K", K), self._states(V, "V", K)
        rangep = None
        if key_range is not None:
            if key_range.get_device() != dev or key_range.dtype not in _I32 or key_range.shape != (T, 2) or not key_range.is_contiguous():
                self._explain(key_range, "key_range", 4, (T, 2))
            rangep = key_range.data_ptr()
        st = _lib.hccs_attention_cross(
            self._h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), k_stride, v_stride, q_start.data_ptr(), k_start.data_ptr(), k_len.data_ptr(),
            rangep, _ints(requant_mult, "requant_mult", Hq), requant_shift, None if out_scale is None else _floats(out_scale, "out_scale", Hq),
            O.data_ptr(), _type_of(O), T, S, B, Hq, Hkv, d, max_q, max_kv, flags, _raw_stream(dev) if stream is None else _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_attention_cross")

    # The cache calls run on the context's device: on its current stream, with tensors that live there.  They are made
    # for every token of every layer, so their checks take the short way and build a message only where one is due.
    def _explain(self, t, name, itemsize, shape=None):
        """Raises with what is wrong with a tensor, if it is this one."""
        if t.get_device() != self.device:
            raise ValueError(f"{name} must live on cuda:{self.device}, not {t.device}")
        _check_tensor(t, name, itemsize, shape)
        if t.dtype not in _WHOLE[itemsize]:
            import torch                       # whoever misses a type fills the sets before it judges: threads do not wait for each other
            _I8.update((torch.int8, torch.uint8))
            _I32.update((torch.int32, torch.uint32))
            _I64.update((torch.int64, torch.uint64))
            if t.dtype not in _WHOLE[itemsize]:
                raise ValueError(f"{name} must hold integers, not {t.dtype}")

    def _check(self, t, name, itemsize, shape=None) -> int:
        """The address of a tensor of integers of the context's device that passes."""
        if t.get_device() != self.device or not t.is_contiguous() or t.dtype not in _WHOLE[itemsize] or (shape is not None and t.shape != shape):
            self._explain(t, name, itemsize, shape)
        return t.data_ptr()

    def _output(self, t, name, shape) -> int:
        """The address of an output tensor (its type goes to the library, which knows which it takes)."""
        if t.get_device() != self.device:
            raise ValueError(f"{name} must live on cuda:{self.device}, not {t.device}")
        _check_tensor(t, name, t.element_size(), shape)
        return t.data_ptr()

    def _tokens(self, t, name, some) -> int:
        """Elements between the tokens of a [T, heads, d] view that is contiguous inside a token."""
        if t.get_device() != self.device:
            raise ValueError(f"{name} must live on cuda:{self.device}, not {t.device}")
        T, heads, d = t.shape
        if t is not some:
            n, _, dim = some.shape
            if t.dtype != some.dtype or T != n or d != dim:
                raise ValueError(f"{name} must be [{n}, heads, {dim}] of {some.dtype}, got {tuple(t.shape)} of {t.dtype}")
        a, b, c = t.stride()
        if T and heads and (c != 1 or (heads > 1 and b != d)):
            raise ValueError(f"{name} must be contiguous inside a token")
        return a if T > 1 else 0

    def _states(self, t, name, like) -> int:
        """Bytes between the keys of int8 states [S, heads, d] that are contiguous inside a key."""
        shape = t.shape
        if t.get_device() != self.device or t.dtype not in _I8 or (t is not like and shape != like.shape):
            self._explain(t if t.get_device() != self.device or t.is_contiguous() else t.contiguous(), name, 1, like.shape)
        S, heads, d = shape
        a, b, c = t.stride()
        if S and heads and (c != 1 or (heads > 1 and b != d)):
            raise ValueError(f"{name} must be contiguous inside a key")
        return a if S > 1 else heads * d

    # -- hccs_device_status / hccs_last_cuda_error / hccs_launch_count
    def hccs_device_status(self, stream=None) -> int:
        w = _u32(0)
        st = _lib.hccs_device_status(self._h, ctypes.byref(w), _stream_ptr(stream))
        if st not in (HCCS_OK, HCCS_ERR_DEVICE_TIMEOUT, HCCS_ERR_DEVICE_INDEX):
            raise HccsError(st, "hccs_device_status")
        return int(w.value)

    # -- hccs_debug_wait_timeout
    def hccs_debug_wait_timeout(self, mode: int, limit_cycles: int, stream=None) -> None:
        st = _lib.hccs_debug_wait_timeout(self._h, int(mode), int(limit_cycles), _stream_ptr(stream))
        if st != HCCS_OK:
            raise HccsError(st, "hccs_debug_wait_timeout")

    def hccs_last_cuda_error(self) -> int:
        return int(_lib.hccs_last_cuda_error(self._h))

    def hccs_launch_count(self) -> int:
        return int(_lib.hccs_launch_count(self._h))


def hccs_forward_static_scratch(params, n_design: int, logits, probs, flags: int = 0, out_shift: int = 0,
                                check_timeout: bool = False, stream=None) -> int:
    """hccs_forward without a context and without any allocation inside the library: for callers
    that may not allocate device memory.  Runs on the current device; ``logits``/``probs`` are the
    caller's tensors.  With ``check_timeout`` the call synchronises and returns the status word."""
    arr = np.ascontiguousarray(params, dtype=np.int32).reshape(-1, 3)
    B, H, Lq, Lk = logits.shape
    _check_tensor(logits, "logits", 1)
    _check_tensor(probs, "probs", 2 if flags & HCCS_OUT_U16 else 1, logits.shape)
    word = _u32(0)
    st = _lib.hccs_forward_static_scratch(arr.ctypes.data_as(_vp), arr.shape[0], int(n_design),
                                          int(out_shift), _ptr(logits), _ptr(probs), B, H, Lq, Lk,
                                          int(flags), ctypes.byref(word) if check_timeout else None,
                                          _stream_ptr(stream))
    if st != HCCS_OK:
        raise HccsError(st, "hccs_forward_static_scratch")
    return int(word.value)


_TYPES = {}
_I8, _I32, _I64 = set(), set(), set()      # integer types by their size, filled on first use
_WHOLE = {1: _I8, 4: _I32, 8: _I64}


# torch is imported on first use: the host-only calls do without it.
def _raw_stream(device):
    """The handle of a device's current stream (torch's own short way where it has one)."""
    global _raw_stream
    import torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
    return _raw_stream(device)


def _type_of(t) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        import torch
        _TYPES.update({torch.int32: HCCS_I32, torch.float32: HCCS_F32, torch.bfloat16: HCCS_BF16, torch.float16: HCCS_F16})
        if t.dtype not in _TYPES:
            raise ValueError(f"int32, float32, bfloat16 or float16 is wanted, got {t.dtype}")
        kind = _TYPES[t.dtype]
    return kind


# The library reads a rotation by the layout of the call's own kind.
def _rotation(rope, kind):
    if rope is None:
        return None
    if not isinstance(rope, kind):
        raise ValueError(f"rope must be a {kind.__name__}, not a {type(rope).__name__}")
    return ctypes.byref(rope)


# Host arrays go to the library as the bytes of their values (it copies them before it returns).
_NP_F32, _NP_I32 = np.dtype(np.float32), np.dtype(np.int32)


def _bytes(v, name, n, dtype) -> bytes:
    arr = v if type(v) is np.ndarray and v.dtype is dtype else np.asarray(v, dtype=dtype)
    if arr.size != n:
        raise ValueError(f"{name} must have {n} entries, got {arr.size}")
    return arr.tobytes()


def _floats(v, name, n) -> bytes:
    return _bytes(v, name, n, _NP_F32)


def _ints(v, name, n) -> bytes:
    return _bytes(v, name, n, _NP_I32)


def _check_tensor(t, name, itemsize, shape=None, device="cuda"):
    if t.device.type != device:
        raise ValueError(f"{name} must live on {device}, not {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.element_size() != itemsize:
        raise ValueError(f"{name} must have {itemsize}-byte elements, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def raw():
    """The underlying ``ctypes.CDLL`` (for tests that call the C ABI with bad arguments)."""
    return _lib
