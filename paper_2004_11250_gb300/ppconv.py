"""Python binding of the C-ABI library (``include/ppconv.h``), by ctypes.

Same names as the C entry points; each wrapper only marshals arguments
(numpy arrays for host data, integers or torch tensors for device pointers,
``torch.cuda.Stream``/int/None for streams) and raises ``PPError`` on a
non-zero status.  Every step of the computation runs in the compiled library.
Importing this module loads ``_build/libppconv.so`` and fails loudly if it has
not been built (``paper_2004_11250_gb300.build.build()``).
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

from .build import LIB as _LIB_PATH

if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: build it with paper_2004_11250_gb300.build.build() "
                      "(or __graft_entry__.build()); there is no fallback path")

lib = ctypes.CDLL(_LIB_PATH)

PP_OK = 0
PP_ERR_INVALID_ARG = 1
PP_ERR_BAD_PATTERN_SET = 2
PP_ERR_TAP_NOT_IN_PATTERN = 3
PP_ERR_PRUNED_NONZERO = 4
PP_ERR_PATTERN_ID_MISMATCH = 5
PP_ERR_UNSUPPORTED = 6
PP_ERR_CUDA = 7
PP_ERR_OOM = 8

PP_KERNEL_AUTO = 0
PP_KERNEL_TMEM = 1
PP_KERNEL_REGISTER = 2
PP_KERNEL_TC = 3
PP_KERNEL_TC_FLAT = 4
PP_KERNEL_DIRECT = 5

PP_WAIT_POLLS = 1 << 18

PP_PROBE_FFMA = 0
PP_PROBE_MMA_TF32 = 1
PP_PROBE_MMA_F16 = 2

PP_PRECISION_TF32X3 = 0
PP_PRECISION_F16X3 = 1
PP_FLAT_PAIRED = 256  # or-ed into a flat-kernel split: CTA pairs over two filter blocks

PP_STATUS_TIMEOUT = 1
PP_STATUS_F16_RANGE = 2

PP_ADD_SKIP = 1
PP_RELU = 2
PP_POOL2 = 4

PP_F32 = 0
PP_F16 = 1
PP_BF16 = 2

PP_ATTN_CAUSAL = 1

PP_CACHE_BAD_PAGE = 1
PP_CACHE_BAD_LENGTH = 2
PP_CACHE_BAD_SLOT = 4
PP_CACHE_TIMEOUT = 8
PP_CACHE_NOT_FINITE = 16

_P = ctypes.c_void_p
_I = ctypes.c_int
_I64 = ctypes.c_int64
_F = ctypes.c_float
_PP = ctypes.POINTER(ctypes.c_void_p)

_SIGS = {
    "pp_status_string": ([_I], ctypes.c_char_p),
    "pp_version": ([], _I),
    "pp_pack_layer": ([_P, _P, _P, _I, _I, _I, _P, _PP], _I),
    "pp_packed_info": ([_P, _P, _P, _P, _P], _I),
    "pp_packed_arrays": ([_P, _PP, _PP, _PP, _PP, _PP, _PP], _I),
    "pp_unpack_layer": ([_P, _P, _P], _I),
    "pp_fold_batchnorm": ([_P, _P, _P, _P, _P, _P, ctypes.c_float, _I, _I], _I),
    "pp_packed_destroy": ([_P], None),
    "pp_layer_create": ([_P, _P, _P, _PP], _I),
    "pp_layer_info": ([_P, _P, _P, _P], _I),
    "pp_conv_forward": ([_P, _P, _P, _P, _I, _I, _I, _I, _P], _I),
    "pp_conv_forward_noalloc": ([_P, _P, _P, _P, _I, _I, _I, _I, _P], _I),
    "pp_layer_set_kernel": ([_P, _I], _I),
    "pp_layer_set_output_order": ([_P, _P, _P], _I),
    "pp_layer_set_precision": ([_P, _I, ctypes.c_float, _P], _I),
    "pp_layer_precision": ([_P, _P, _P], _I),
    "pp_permute_input_channels": ([_P, _P, _P, _I, _I, _P, _P, _P, _P], _I),
    "pp_layer_kernel": ([_P, _P], _I),
    "pp_layer_device_status": ([_P, _P], _I),
    "pp_wait_probe": ([ctypes.c_longlong, _P, _P], _I),
    "pp_peak_probe": ([_I, ctypes.c_longlong, _P, _P, _P], _I),
    "pp_layer_autotune": ([_P, _I, _I, _I, _I, _P], _I),
    "pp_layer_flat_geometry": ([_P, _I, _I, _I, _I, _P, _P], _I),
    "pp_layer_pin_flat_geometry": ([_P, _I, _I, _I, _I, _I, _I], _I),
    "pp_layer_destroy": ([_P], None),
    "pp_dense_create": ([_P, _P, _I, _I, _P, _PP], _I),
    "pp_dense_forward": ([_P, _P, _P, _P, _I, _I, _I, _I, _P], _I),
    "pp_dense_info": ([_P, _P, _P], _I),
    "pp_dense_device_status": ([_P, _P], _I),
    "pp_dense_destroy": ([_P], None),
    "pp_net_create": ([_I, _I, _I, _I, _PP], _I),
    "pp_net_add_conv": ([_P, _P, _I, _I], _I),
    "pp_net_add_dense": ([_P, _P, _I, _I], _I),
    "pp_net_finalize": ([_P], _I),
    "pp_net_output_shape": ([_P, _P, _P, _P, _P], _I),
    "pp_net_use_graph": ([_P, _I], _I),
    "pp_net_run": ([_P, _P, _P, _P], _I),
    "pp_net_run_host": ([_P, _P, _P, _P], _I),
    "pp_net_destroy": ([_P], None),
    "pp_rope_create": ([_I, _I, _P, _P, _I, _I, _P, _PP], _I),
    "pp_rope_destroy": ([_P], None),
    "pp_qk_rotate": ([_P, _I, _I, _P, _F, _P, _I64, _I64, _I, _P, _P, _P, _I64, _I64, _I, _P, _P, _P], _I),
    "pp_cache_create": ([_I, _I, _I, _I, _I, _P, _P, _P, _P, _PP], _I),
    "pp_cache8_create": ([_I, _I, _I, _I, _I, _P, _P, _P, _P, _PP], _I),
    "pp_cache_destroy": ([_P], None),
    "pp_cache_device_status": ([_P, _P], _I),
    "pp_qkv_store": ([_P, _P, _I, _P, _P, _F, _P, _I64, _I64, _I, _P, _P, _P, _I64, _I64, _P, _P, _I64, _I64, _P], _I),
    "pp_cache_summarize": ([_P, _P, _I, _P], _I),
    "pp_cache_select": ([_P, _I, _P, _I64, _I64, _I, _I, _P, _P, _I, _P, _I, _I, _I, _I, _P, _P], _I),
    "pp_cache_append": ([_P, _I, _P, _I64, _I64, _P, _I64, _I64, _I, _P, _P, _I, _P, _P], _I),
    "pp_cache_read": ([_P, _I, _I, _P, _P, _I, _P, _P, _P, _P], _I),
    "pp_attn_window": ([_P, _I, _P, _I64, _I64, _I, _I, _P, _P, _I, _P, _F, _I, _I, _I, _P, _P, _P], _I),
    "pp_attn_forward": ([_P, _I, _P, _I64, _I64, _I, _I, _P, _P, _I, _P, _F, _I, _P, _I, _P, _P, _P], _I),
}
for _name, (_args, _res) in _SIGS.items():
    _fn = getattr(lib, _name)
    _fn.argtypes = _args
    _fn.restype = _res


class PPError(RuntimeError):
    def __init__(self, code: int, where: str = ""):
        super().__init__(f"{where}: {pp_status_string(code)} ({code})")
        self.code = code


def pp_fold_batchnorm(w, bias, gamma, beta, mean, var, eps=1e-5):
    """Batch normalisation after the conv folded into (w [Co][Ci][3][3] or [Co][Ci][9], bias [Co] or None):
    returns new fp32 arrays (w in the shape given, bias [Co])."""
    import numpy as np
    w2 = np.array(w, dtype=np.float32, order="C", copy=True)
    Co, Ci = w2.shape[0], w2.shape[1]
    b2 = np.zeros(Co, np.float32) if bias is None else np.array(bias, dtype=np.float32, copy=True)
    arrs = [np.ascontiguousarray(a, dtype=np.float32) for a in (gamma, beta, mean, var)]
    for a in arrs:
        if a.shape != (Co,):
            raise ValueError("batch-norm parameters must have shape [Co]")
    _check(lib.pp_fold_batchnorm(w2.ctypes.data, b2.ctypes.data, *[a.ctypes.data for a in arrs], float(eps), Co, Ci),
           "pp_fold_batchnorm")
    return w2, b2


def pp_permute_input_channels(w, mask, layout, pattern_ids=None):
    """(w, mask, ids) with input channel c of the result = original channel layout[c]; ids None if not given."""
    w = _host(w, np.float32)
    Co, Ci = w.shape[0], w.shape[1]
    w = w.reshape(Co, Ci, 9)
    mask = _host(mask, np.uint8)
    ids = _host(pattern_ids, np.uint8)
    lay = _host(layout, np.int32)
    if mask.shape != (Co, Ci) or lay.shape != (Ci,) or (ids is not None and ids.shape != (Co, Ci)):
        raise PPError(PP_ERR_INVALID_ARG, "pp_permute_input_channels shapes")
    w2 = np.empty_like(w)
    m2 = np.empty_like(mask)
    i2 = None if ids is None else np.empty_like(ids)
    _check(lib.pp_permute_input_channels(_hp(w), _hp(mask), _hp(ids), Co, Ci, _hp(lay), _hp(w2), _hp(m2), _hp(i2)),
           "pp_permute_input_channels")
    return w2, m2, i2


def pp_status_string(code: int) -> str:
    return lib.pp_status_string(code).decode()


def pp_version() -> int:
    return lib.pp_version()


def _check(st: int, where: str):
    if st != PP_OK:
        raise PPError(st, where)


def _host(a, dtype):
    return None if a is None else np.ascontiguousarray(a, dtype=dtype)


def _hp(a):
    return None if a is None else a.ctypes.data


def _dp(t) -> Optional[int]:
    """Device pointer of a torch tensor or an int; None stays NULL."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(s) -> Optional[int]:
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return s.cuda_stream


# ------------------------------------------------------------------ packer


def pp_pack_layer(w, mask, pattern_taps, pattern_ids=None) -> int:
    """Pack a pruned layer; returns an opaque handle (free with pp_packed_destroy)."""
    w = _host(w, np.float32)
    Co, Ci = w.shape[0], w.shape[1]
    w = w.reshape(Co, Ci, 9)
    mask = _host(mask, np.uint8)
    taps = _host(pattern_taps, np.uint8)
    ids = _host(pattern_ids, np.uint8)
    if mask.shape != (Co, Ci) or taps.ndim != 2 or taps.shape[1] != 4 or (ids is not None and ids.shape != (Co, Ci)):
        raise PPError(PP_ERR_INVALID_ARG, "pp_pack_layer shapes")
    out = ctypes.c_void_p()
    _check(lib.pp_pack_layer(_hp(w), _hp(mask), _hp(taps), taps.shape[0], Co, Ci, _hp(ids), ctypes.byref(out)),
           "pp_pack_layer")
    return out.value


def pp_packed_info(pk):
    nk, co, ci, p = _I64(), _I(), _I(), _I()
    _check(lib.pp_packed_info(pk, ctypes.byref(nk), ctypes.byref(co), ctypes.byref(ci), ctypes.byref(p)),
           "pp_packed_info")
    return nk.value, co.value, ci.value, p.value


def pp_packed_arrays(pk) -> dict:
    """Copies of the stored arrays: perm, kptr, kidx, kpat, kw [nk][4], taps [P][4]."""
    nk, Co, Ci, P = pp_packed_info(pk)
    ptrs = [ctypes.c_void_p() for _ in range(6)]
    _check(lib.pp_packed_arrays(pk, *[ctypes.byref(p) for p in ptrs]), "pp_packed_arrays")

    def view(ptr, ctype, n, dtype):
        if n == 0:
            return np.zeros(0, dtype)
        buf = (ctype * n).from_address(ptr.value)
        return np.frombuffer(buf, dtype=dtype, count=n).copy()

    return {
        "perm": view(ptrs[0], ctypes.c_int32, Co, np.int32),
        "kptr": view(ptrs[1], ctypes.c_int32, Co + 1, np.int32),
        "kidx": view(ptrs[2], ctypes.c_int32, nk, np.int32),
        "kpat": view(ptrs[3], ctypes.c_uint8, nk, np.uint8),
        "kw": view(ptrs[4], ctypes.c_float, 4 * nk, np.float32).reshape(nk, 4),
        "taps": view(ptrs[5], ctypes.c_uint8, 4 * P, np.uint8).reshape(P, 4),
    }


def pp_unpack_layer(pk):
    nk, Co, Ci, P = pp_packed_info(pk)
    w = np.empty((Co, Ci, 9), np.float32)
    mask = np.empty((Co, Ci), np.uint8)
    _check(lib.pp_unpack_layer(pk, _hp(w), _hp(mask)), "pp_unpack_layer")
    return w, mask


def pp_packed_destroy(pk):
    lib.pp_packed_destroy(pk)


# ------------------------------------------------------------------ device layers


def pp_layer_create(pk, bias=None, stream=None) -> int:
    b = _host(bias, np.float32)
    out = ctypes.c_void_p()
    _check(lib.pp_layer_create(pk, _hp(b), _stream(stream), ctypes.byref(out)), "pp_layer_create")
    return out.value


def pp_layer_info(layer):
    co, ci, nb = _I(), _I(), _I64()
    _check(lib.pp_layer_info(layer, ctypes.byref(co), ctypes.byref(ci), ctypes.byref(nb)), "pp_layer_info")
    return co.value, ci.value, nb.value


def pp_conv_forward(layer, x, y, skip, N, H, W, flags, stream=None):
    _check(lib.pp_conv_forward(layer, _dp(x), _dp(y), _dp(skip), N, H, W, flags, _stream(stream)),
           "pp_conv_forward")


def pp_conv_forward_noalloc(layer, x, y, skip, N, H, W, flags, stream=None):
    """pp_conv_forward through the flat tensor-core kernel, whose split reduction needs no workspace (no device allocation)."""
    _check(lib.pp_conv_forward_noalloc(layer, _dp(x), _dp(y), _dp(skip), N, H, W, flags, _stream(stream)),
           "pp_conv_forward_noalloc")


def pp_layer_set_kernel(layer, kernel: int):
    _check(lib.pp_layer_set_kernel(layer, kernel), "pp_layer_set_kernel")


def pp_layer_set_output_order(layer, order=None, stream=None):
    """order[o] = output channel of original filter o (None: original order); see the header."""
    o = _host(order, np.int32)
    _check(lib.pp_layer_set_output_order(layer, _hp(o), _stream(stream)), "pp_layer_set_output_order")


def pp_layer_set_precision(layer, precision: int, input_bound: float = 0.0, stream=None):
    """PP_PRECISION_TF32X3 or PP_PRECISION_F16X3 for the tensor-core kernels (see the header)."""
    _check(lib.pp_layer_set_precision(layer, precision, float(input_bound), _stream(stream)), "pp_layer_set_precision")


def pp_layer_precision(layer):
    """(precision, input scale)."""
    p, sc = _I(), ctypes.c_float()
    _check(lib.pp_layer_precision(layer, ctypes.byref(p), ctypes.byref(sc)), "pp_layer_precision")
    return p.value, sc.value


def pp_layer_kernel(layer) -> int:
    k = _I()
    _check(lib.pp_layer_kernel(layer, ctypes.byref(k)), "pp_layer_kernel")
    return k.value


def pp_layer_autotune(layer, N, H, W, flags, stream=None):
    _check(lib.pp_layer_autotune(layer, N, H, W, flags, _stream(stream)), "pp_layer_autotune")


def pp_layer_flat_geometry(layer, N, H, W, flags):
    """(R, S) pinned for the flat tensor-core kernel at this shape, (0, 0) if none."""
    R, S = _I(), _I()
    _check(lib.pp_layer_flat_geometry(layer, N, H, W, flags, ctypes.byref(R), ctypes.byref(S)), "pp_layer_flat_geometry")
    return R.value, S.value


def pp_layer_pin_flat_geometry(layer, N, H, W, flags, R, S):
    _check(lib.pp_layer_pin_flat_geometry(layer, N, H, W, flags, R, S), "pp_layer_pin_flat_geometry")


def pp_layer_device_status(layer) -> int:
    v = _I()
    _check(lib.pp_layer_device_status(layer, ctypes.byref(v)), "pp_layer_device_status")
    return v.value


def pp_wait_probe(polls: int):
    """(gave_up, elapsed_ns) of `polls` polls of an mbarrier that nothing completes (see the header)."""
    g, ns = _I(), ctypes.c_longlong()
    _check(lib.pp_wait_probe(polls, ctypes.byref(g), ctypes.byref(ns)), "pp_wait_probe")
    return g.value, ns.value


def pp_peak_probe(kind: int, iters: int):
    """(TFLOP/s, SM MHz, ms) of one launch of a peak-rate probe (PP_PROBE_*; see the header)."""
    tf, mhz, ms = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
    _check(lib.pp_peak_probe(kind, iters, ctypes.byref(tf), ctypes.byref(mhz), ctypes.byref(ms)), "pp_peak_probe")
    return tf.value, mhz.value, ms.value


def pp_layer_destroy(layer):
    lib.pp_layer_destroy(layer)


def pp_dense_create(w, bias=None, stream=None) -> int:
    w = _host(w, np.float32)
    Co, Ci = w.shape[0], w.shape[1]
    b = _host(bias, np.float32)
    out = ctypes.c_void_p()
    _check(lib.pp_dense_create(_hp(w.reshape(Co, Ci, 9)), _hp(b), Co, Ci, _stream(stream), ctypes.byref(out)),
           "pp_dense_create")
    return out.value


def pp_dense_forward(layer, x, y, skip, N, H, W, flags, stream=None):
    _check(lib.pp_dense_forward(layer, _dp(x), _dp(y), _dp(skip), N, H, W, flags, _stream(stream)),
           "pp_dense_forward")


def pp_dense_info(layer):
    co, ci = _I(), _I()
    _check(lib.pp_dense_info(layer, ctypes.byref(co), ctypes.byref(ci)), "pp_dense_info")
    return co.value, ci.value


def pp_dense_device_status(layer) -> int:
    v = _I()
    _check(lib.pp_dense_device_status(layer, ctypes.byref(v)), "pp_dense_device_status")
    return v.value


def pp_dense_destroy(layer):
    lib.pp_dense_destroy(layer)


# ------------------------------------------------------------------ network


def pp_net_create(N, C, H, W) -> int:
    out = ctypes.c_void_p()
    _check(lib.pp_net_create(N, C, H, W, ctypes.byref(out)), "pp_net_create")
    return out.value


def pp_net_add_conv(net, layer, flags, skip_from=-1):
    _check(lib.pp_net_add_conv(net, layer, flags, skip_from), "pp_net_add_conv")


def pp_net_add_dense(net, layer, flags, skip_from=-1):
    _check(lib.pp_net_add_dense(net, layer, flags, skip_from), "pp_net_add_dense")


def pp_net_finalize(net):
    _check(lib.pp_net_finalize(net), "pp_net_finalize")


def pp_net_output_shape(net):
    v = [_I() for _ in range(4)]
    _check(lib.pp_net_output_shape(net, *[ctypes.byref(a) for a in v]), "pp_net_output_shape")
    return tuple(a.value for a in v)


def pp_net_use_graph(net, enable: bool):
    _check(lib.pp_net_use_graph(net, 1 if enable else 0), "pp_net_use_graph")


def pp_net_run(net, x, y, stream=None):
    _check(lib.pp_net_run(net, _dp(x), _dp(y), _stream(stream)), "pp_net_run")


def pp_net_run_host(net, x_host, y_host, stream=None):
    """x_host / y_host: host buffers (numpy arrays or pinned CPU torch tensors)."""
    xp = x_host.data_ptr() if hasattr(x_host, "data_ptr") else x_host.ctypes.data
    yp = y_host.data_ptr() if hasattr(y_host, "data_ptr") else y_host.ctypes.data
    _check(lib.pp_net_run_host(net, xp, yp, _stream(stream)), "pp_net_run_host")


def pp_net_destroy(net):
    lib.pp_net_destroy(net)


# ------------------------------------------------------------------ decoder operators


class _Types:
    """torch's types and the library's codes of them, made at the first use (the convolutions need no torch)."""

    def __init__(self):
        import torch
        self.code = {torch.float32: PP_F32, torch.float16: PP_F16, torch.bfloat16: PP_BF16}
        self.f32, self.i32, self.i8 = torch.float32, torch.int32, torch.int8


_types: Optional[_Types] = None


def _torch_types() -> _Types:
    global _types
    if _types is None:
        _types = _Types()
    return _types


def _dtype(t) -> int:
    """The library's code of a tensor's type; PP_ERR_INVALID_ARG for types it does not take."""
    try:
        return _torch_types().code[t.dtype]
    except KeyError:
        raise PPError(PP_ERR_INVALID_ARG, f"dtype {t.dtype}") from None


def _heads(t, dtype, T, D):
    """(pointer, token stride, head stride, heads) of a view [T][heads][D] of torch type dtype; None is no heads."""
    if t is None:
        return None, 0, 0, 0
    try:
        (t0, h, d), (ts, hs, ds) = t.shape, t.stride()
        if t0 == T and d == D and ds == 1 and t.dtype is dtype and t.is_cuda:
            return t.data_ptr(), ts, hs, h
    except ValueError:  # not three axes
        pass
    raise PPError(PP_ERR_INVALID_ARG, "a token tensor is [T][heads][D] of the call's type on the GPU, dense in D")


def _dense(t, shape, dtype, where):
    """Pointer of a dense tensor of this shape and torch type on the GPU; None stays NULL."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise PPError(PP_ERR_INVALID_ARG, f"{where}: expected a dense {dtype} of {tuple(shape)} on the GPU")
    return t.data_ptr()


class Rope(int):
    """A rotation plan's handle with what the binding checks shapes by."""
    D: int
    axes: int


class Cache(int):
    """A cache's handle with what the binding checks shapes by; it keeps the pools alive."""
    dtype: object
    shape: tuple


def pp_rope_create(D, axis, freq, axes=1, interleaved=False, stream=None) -> Rope:
    """axis and freq [pairs]: pair j turns by position[axis[j]] * freq[j] (axis None: all 0)."""
    f = _host(freq, np.float64)
    a = _host(axis, np.uint8)
    if f.ndim != 1 or (a is not None and a.shape != f.shape):
        raise PPError(PP_ERR_INVALID_ARG, "pp_rope_create shapes")
    out = ctypes.c_void_p()
    _check(lib.pp_rope_create(D, len(f), _hp(a), _hp(f), axes, 1 if interleaved else 0, _stream(stream),
                              ctypes.byref(out)), "pp_rope_create")
    r = Rope(out.value)
    r.D, r.axes = D, axes
    return r


def pp_rope_destroy(rope):
    lib.pp_rope_destroy(rope)


def pp_qk_rotate(rope, pos, eps, q, qw, q_out, k, kw, k_out, stream=None):
    """q [T][Hq][D], k [T][Hk][D] (either may be None) normalised and rotated into q_out, k_out; pos [axes][T] int32."""
    x = q if q is not None else k
    T, D, code, y = x.shape[0], rope.D, _dtype(x), _torch_types()
    dt = x.dtype
    qp, qt, qh, Hq = _heads(q, dt, T, D)
    kp, kt, kh, Hk = _heads(k, dt, T, D)
    _check(lib.pp_qk_rotate(rope, code, T, _dense(pos, (rope.axes, T), y.i32, "pos"), eps, qp, qt, qh, Hq,
                            _dense(qw, (D,), y.f32, "qw"), None if q is None else _dense(q_out, q.shape, dt, "q_out"), kp,
                            kt, kh, Hk, _dense(kw, (D,), y.f32, "kw"),
                            None if k is None else _dense(k_out, k.shape, dt, "k_out"), _stream(stream)),
           "pp_qk_rotate")


def pp_cache_create(k, v, codes=None, scales=None) -> Cache:
    """k, v: pools [pages][H][page][D]; codes [pages][H][2][D] int8 and scales [pages][H] fp32 of the page summaries."""
    if k.dim() != 4:
        raise PPError(PP_ERR_INVALID_ARG, "pp_cache_create shapes")
    pages, H, page, D = k.shape
    y = _torch_types()
    out = ctypes.c_void_p()
    _check(lib.pp_cache_create(_dtype(k), pages, page, H, D, _dense(k, k.shape, k.dtype, "k"),
                               _dense(v, k.shape, k.dtype, "v"), _dense(codes, (pages, H, 2, D), y.i8, "codes"),
                               _dense(scales, (pages, H), y.f32, "scales"), ctypes.byref(out)), "pp_cache_create")
    c = Cache(out.value)
    c.dtype, c.shape, c.pools = k.dtype, (pages, H, page, D), (k, v, codes, scales)
    return c


def pp_cache8_create(k, v, k_scales, v_scales, dtype) -> Cache:
    """A cache in 8 bits: codes k, v [pages][H][page][D] int8, scales [pages][H] fp32; dtype: torch type of its tokens."""
    y = _torch_types()
    if k.dim() != 4 or dtype not in y.code:
        raise PPError(PP_ERR_INVALID_ARG, "pp_cache8_create shapes and dtype")
    pages, H, page, D = k.shape
    out = ctypes.c_void_p()
    _check(lib.pp_cache8_create(y.code[dtype], pages, page, H, D, _dense(k, k.shape, y.i8, "k"), _dense(v, k.shape, y.i8, "v"),
                                _dense(k_scales, (pages, H), y.f32, "k_scales"), _dense(v_scales, (pages, H), y.f32, "v_scales"),
                                ctypes.byref(out)), "pp_cache8_create")
    c = Cache(out.value)
    c.dtype, c.shape, c.pools = dtype, (pages, H, page, D), (k, v, k_scales, v_scales)
    return c


def pp_cache_destroy(cache):
    lib.pp_cache_destroy(cache)


def pp_cache_device_status(cache) -> int:
    """Bits PP_CACHE_* of what the calls met since the last read (synchronous)."""
    v = _I()
    _check(lib.pp_cache_device_status(cache, ctypes.byref(v)), "pp_cache_device_status")
    return v.value


def pp_qkv_store(rope, cache, pos, slots, eps, q, qw, q_out, k, kw, v, stream=None):
    """pp_qk_rotate with the keys, and the values as they are, stored to slots [T] (int32) of the cache."""
    D, dt, y = rope.D, cache.dtype, _torch_types()
    H, shape = cache.shape[1], k.shape
    T = shape[0]
    kt, kh, kd = k.stride()
    vt, vh, vd = v.stride()
    if not (shape == v.shape == (T, H, D) and k.dtype is dt and v.dtype is dt and kd == 1 and vd == 1 and k.is_cuda and v.is_cuda):
        raise PPError(PP_ERR_INVALID_ARG, "pp_qkv_store: k and v are [T][the cache's heads][D] of its type on the GPU, dense in D")
    qp, qt, qh, Hq = _heads(q, dt, T, D)
    _check(lib.pp_qkv_store(rope, cache, T, _dense(pos, (rope.axes, T), y.i32, "pos"), _dense(slots, (T,), y.i32, "slots"),
                            eps, qp, qt, qh, Hq, _dense(qw, (D,), y.f32, "qw"),
                            None if q is None else _dense(q_out, q.shape, dt, "q_out"), k.data_ptr(), kt, kh,
                            _dense(kw, (D,), y.f32, "kw"), v.data_ptr(), vt, vh, _stream(stream)), "pp_qkv_store")


def pp_cache_summarize(cache, ids, stream=None):
    """Summaries of the full pages ids [n] (int32) into the cache's codes and scales."""
    n = ids.shape[0]
    _check(lib.pp_cache_summarize(cache, _dense(ids, (n,), _torch_types().i32, "ids"), n, _stream(stream)),
           "pp_cache_summarize")


def _sequences(q, cache, starts, table, lens, y):
    """The arguments that pp_cache_select and the attention calls share: tokens, queries, sequences."""
    T = q.shape[0]
    qp, qt, qh, Hq = _heads(q, cache.dtype, T, cache.shape[3])
    return (cache, T, qp, qt, qh, Hq, *_tables(starts, table, lens, y.i32))


def _tables(starts, table, lens, i32):
    """(sequences, starts, table, width, lens) as the calls take them.  A small call is the host's, so its checks are in one place."""
    B, width = table.shape
    first = None if starts is None else _dense(starts, (B + 1,), i32, "starts")
    if (lens is not None and table.dtype is i32 and lens.dtype is i32 and lens.shape == (B,) and table.is_cuda and lens.is_cuda and
            table.is_contiguous() and lens.is_contiguous()):
        return B, first, table.data_ptr(), width, lens.data_ptr()
    return B, first, _dense(table, (B, width), i32, "table"), width, _dense(lens, (B,), i32, "lens")


def pp_cache_select(cache, q, starts, table, lens, flags, first, last, sel, stream=None):
    """The pages of each token and cache head worth reading, into sel [T][H][keep] (int32); see the header."""
    keep, y = sel.shape[2], _torch_types()
    _check(lib.pp_cache_select(*_sequences(q, cache, starts, table, lens, y), flags, first, last, keep,
                               _dense(sel, (q.shape[0], cache.shape[1], keep), y.i32, "sel"), _stream(stream)),
           "pp_cache_select")


def pp_attn_forward(cache, q, starts, table, lens, scale, flags, sel, out, lse=None, stream=None):
    """Attention of q [T][Hq][D] over the cache into out; sel None: every visible page.  lse [T][Hq] fp32 or None."""
    (T, Hq, _), y = q.shape, _torch_types()
    keep = 0 if sel is None else sel.shape[2]
    _check(lib.pp_attn_forward(*_sequences(q, cache, starts, table, lens, y), scale, flags,
                               _dense(sel, (T, cache.shape[1], keep), y.i32, "sel"), keep,
                               _dense(out, q.shape, q.dtype, "out"), _dense(lse, (T, Hq), y.f32, "lse"),
                               _stream(stream)), "pp_attn_forward")


def pp_attn_window(cache, q, starts, table, lens, scale, flags, window, sinks, out, lse=None, stream=None):
    """pp_attn_forward where a token sees its last `window` keys and the first `sinks` ones."""
    (T, Hq, _), y = q.shape, _torch_types()
    _check(lib.pp_attn_window(*_sequences(q, cache, starts, table, lens, y), scale, flags, window, sinks,
                              _dense(out, q.shape, q.dtype, "out"), _dense(lse, (T, Hq), y.f32, "lse"), _stream(stream)),
           "pp_attn_window")


def pp_cache_append(cache, k, v, starts, table, lens, stream=None):
    """New tokens k, v [T][H][D] of the sequences into a cache in 8 bits: the last ones of lens[b] keys each."""
    shape, dt, (_, H, _, D) = k.shape, cache.dtype, cache.shape
    kt, kh, kd = k.stride()
    vt, vh, vd = v.stride()
    T = shape[0]
    if not (shape == v.shape == (T, H, D) and k.dtype is dt and v.dtype is dt and kd == 1 and vd == 1 and k.is_cuda and v.is_cuda):
        raise PPError(PP_ERR_INVALID_ARG, "pp_cache_append: k and v are [T][the cache's heads][D] of its type on the GPU, dense in D")
    _check(lib.pp_cache_append(cache, T, k.data_ptr(), kt, kh, v.data_ptr(), vt, vh,
                               *_tables(starts, table, lens, (_types or _torch_types()).i32), _stream(stream)), "pp_cache_append")


def pp_cache_read(cache, starts, table, lens, k_out, v_out, stream=None):
    """The sequences' last keys and values of a cache in 8 bits into k_out, v_out [T][H][D] (either may be None)."""
    x = k_out if k_out is not None else v_out
    if x is None:
        raise PPError(PP_ERR_INVALID_ARG, "pp_cache_read: nothing to read into")
    T, dt, (_, H, _, D) = x.shape[0], cache.dtype, cache.shape
    B, s, t, width, n = _tables(starts, table, lens, (_types or _torch_types()).i32)
    _check(lib.pp_cache_read(cache, T, B, s, t, width, n, _dense(k_out, (T, H, D), dt, "k_out"),
                             _dense(v_out, (T, H, D), dt, "v_out"), _stream(stream)), "pp_cache_read")
