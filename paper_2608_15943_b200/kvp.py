"""Binding of the C-ABI library (``include/kvp.h``): argument marshalling only, in ctypes and (the per-step calls) in the native
module ``_pack``.

Every function takes torch tensors (device memory, streams) and passes raw pointers and sizes to
the entry point of the same name; all computation happens in the library's CUDA kernels.  Importing
this module loads ``libkvp.so`` and raises if it has not been built -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvp.so")
for _so in (LIB_PATH, os.path.join(_HERE, "_pack.so")):
    if not os.path.exists(_so):
        raise ImportError(f"{_so} is missing: run `python -m paper_2608_15943_b200.build` (nvcc, sm_100a)")
lib = C.CDLL(LIB_PATH)

from . import _pack  # noqa: E402

OK, ERR_INVALID_ARG, ERR_BAD_DONOR, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(7)
PLAN_STOP_ON_NO_IMPROVE, PLAN_STAGE_LOCAL_DONOR = 1, 2
STOP_TOLERANCE, STOP_BUDGET, STOP_EXHAUSTED, STOP_NO_IMPROVE = range(4)
PLACE_ARCH_BALANCED, PLACE_UNIFORM, PLACE_BIPOLAR = range(3)
OP_PROJ_FWD, OP_PROJ_BWD, OP_ATTN_FWD, OP_ATTN_BWD, OP_DECODE = range(5)
BF16, F32 = 0, 1   # dtype of the activations / weights in the caller's memory (kvp_shape.dtype, kvp_decode_desc.dtype)

EXPORTS = ["kvp_status_string", "kvp_device_status", "kvp_launch_count", "kvp_set_timing_events", "kvp_set_gemm_pair_mode", "kvp_selftest_bounded_wait_pair",
           "kvp_timing_events_used", "kvp_plan", "kvp_layer_flops", "kvp_sim_1f1b", "kvp_workspace_bytes",
           "kvp_proj_fwd", "kvp_proj_bwd", "kvp_proj_bwd_range", "kvp_out_proj_fwd", "kvp_out_proj_bwd", "kvp_attn_fwd", "kvp_attn_bwd",
           "kvp_gemm", "kvp_rmsnorm", "kvp_rope", "kvp_swiglu", "kvp_add", "kvp_decode_workspace_bytes", "kvp_cache_append",
           "kvp_decode", "kvp_decode_static", "kvp_selftest_bounded_wait",
           "kvp_cache_append_tokens", "kvp_decode8", "kvp_decode8_workspace_bytes",
           "kvp_attn_chunk", "kvp_attn_chunk_workspace_bytes",
           "kvp_pages_workspace_bytes", "kvp_pages_copy", "kvp_pages_fork", "kvp_pages_resize", "kvp_pages_trim", "kvp_pages_compact"]


class KvpError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


lib.kvp_status_string.restype = C.c_char_p
lib.kvp_status_string.argtypes = [C.c_int]


def status_string(status: int) -> str:
    return lib.kvp_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise KvpError(status, where)


def device_status() -> int:
    """Synchronises and returns the library's device status (OK or ERR_TIMEOUT / ERR_CUDA)."""
    lib.kvp_device_status.restype = C.c_int
    return int(lib.kvp_device_status())


# torch's stream object is built anew for every look at it (4.4 us a call, half of what a small operator's whole call
# took); its handle alone takes 0.2 us where this torch offers it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream() -> int:
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(_device())
    # Without a device the entry points still validate their arguments (and fail before any launch).
    if not torch.cuda.is_available():
        return 0
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


# Host arrays of the entry points are passed as packed bytes.  Packed natively: four pointers 0.1 us instead of 0.7, a
# donor map of four layers 0.1 instead of 1.0.  (The per-step calls pack theirs in _pack's own functions.)
_ptr_array = _pack.pointers    # tensors (None: a null pointer), one per layer; what a list lacks of so many entries is a null pointer
_donors = _pack.donors


def _map(sizes, donor):
    """Donor map of a call, and how many entries its lists need.  One that is too short goes on with a layer without a donor, which
    the entry points refuse before they read a list."""
    d, layers = _donors(donor), max(getattr(sizes, "L", 0), 0)
    return (d, layers) if len(d) >= 4 * layers else (d + b"\xff" * 4, 0)


def _i32_array(xs: Sequence[int]):
    return (C.c_int32 * len(xs))(*map(int, xs))


def _u64_array(xs: Sequence[int]):
    return (C.c_uint64 * len(xs))(*[int(x) for x in xs])


# ------------------------------------------------------------------------------------------
# gemm
# ------------------------------------------------------------------------------------------
lib.kvp_gemm.restype = C.c_int
lib.kvp_gemm.argtypes = [C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_int64, C.c_int,
                         C.c_void_p, C.c_int64, C.c_int, C.c_void_p]


def gemm(a: torch.Tensor, b: torch.Tensor, c: torch.Tensor, a_mn: bool = False, b_mn: bool = False) -> torch.Tensor:
    """c[M,N] = A B.  a is stored [M,K] (a_mn False) or [K,M]; b is stored [N,K] (b_mn False) or
    [K,N]; c is bf16 or fp32, row-major."""
    status = _pack.gemm(a, b, c, a_mn, b_mn, _stream())
    if status is not NotImplemented:
        _check(status, "kvp_gemm")
        return c
    M, N = c.shape
    K = a.shape[0] if a_mn else a.shape[1]
    _check(lib.kvp_gemm(M, N, K, a.data_ptr(), a.stride(0), int(a_mn), b.data_ptr(), b.stride(0), int(b_mn),
                        c.data_ptr(), c.stride(0), int(c.dtype == torch.float32), _stream()), "kvp_gemm")
    return c


# ------------------------------------------------------------------------------------------
# element-wise stage operators
# ------------------------------------------------------------------------------------------
lib.kvp_rmsnorm.restype = C.c_int
lib.kvp_rmsnorm.argtypes = [C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p]
lib.kvp_rope.restype = C.c_int
lib.kvp_rope.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_int32, C.c_void_p, C.c_void_p]
lib.kvp_swiglu.restype = C.c_int
lib.kvp_swiglu.argtypes = [C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
lib.kvp_add.restype = C.c_int
lib.kvp_add.argtypes = [C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]


def rmsnorm(x: torch.Tensor, w: torch.Tensor, eps: float, y: torch.Tensor) -> torch.Tensor:
    """kvp_rmsnorm: y[T,D] = x / sqrt(mean(x^2) + eps) * w (bf16)."""
    status = _pack.rmsnorm(x, w, eps, y, _stream())
    if status is not NotImplemented:
        _check(status, "kvp_rmsnorm")
        return y
    T, D = x.shape
    _check(lib.kvp_rmsnorm(T, D, x.data_ptr(), w.data_ptr(), float(eps), y.data_ptr(), _stream()), "kvp_rmsnorm")
    return y


def rope(x: torch.Tensor, theta: float = 10000.0, pos0: int = 0) -> torch.Tensor:
    """kvp_rope: in place on x [B,S,H,dh] (bf16)."""
    status = _pack.rope(x, theta, pos0, _stream())
    if status is not NotImplemented:
        _check(status, "kvp_rope")
        return x
    B, S, H, dh = x.shape
    _check(lib.kvp_rope(B, S, H, dh, float(theta), int(pos0), x.data_ptr(), _stream()), "kvp_rope")
    return x


def swiglu(gate: torch.Tensor, up: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
    """kvp_swiglu: out = silu(gate) * up (bf16, same shapes)."""
    status = _pack.swiglu(gate, up, out, _stream())
    if status is not NotImplemented:
        _check(status, "kvp_swiglu")
        return out
    _check(lib.kvp_swiglu(gate.numel(), gate.data_ptr(), up.data_ptr(), out.data_ptr(), _stream()), "kvp_swiglu")
    return out


def add(a: torch.Tensor, b: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
    """kvp_add: out = a + b (bf16, same shapes)."""
    status = _pack.add(a, b, out, _stream())
    if status is not NotImplemented:
        _check(status, "kvp_add")
        return out
    _check(lib.kvp_add(a.numel(), a.data_ptr(), b.data_ptr(), out.data_ptr(), _stream()), "kvp_add")
    return out


# ------------------------------------------------------------------------------------------
# planner (host)
# ------------------------------------------------------------------------------------------
class _PlanIn(C.Structure):
    _fields_ = [("L", C.c_int32), ("P", C.c_int32), ("stage_begin", C.POINTER(C.c_int32)),
                ("f_full", C.POINTER(C.c_uint64)), ("f_share", C.POINTER(C.c_uint64)),
                ("stage_extra", C.POINTER(C.c_uint64)), ("eps_num", C.c_uint32), ("eps_den", C.c_uint32),
                ("max_conv", C.c_int32), ("flags", C.c_uint32), ("alpha_num", C.c_uint32), ("alpha_den", C.c_uint32),
                ("placement", C.c_int32)]


class _PlanOut(C.Structure):
    _fields_ = [("z", C.POINTER(C.c_uint8)), ("donor", C.POINTER(C.c_int32)), ("stage_flops", C.POINTER(C.c_uint64)),
                ("stage_ratio", C.POINTER(C.c_double)), ("fir_num", C.c_uint64), ("fir_den", C.c_uint64),
                ("fir", C.c_double), ("n_conv", C.c_int32), ("stop_reason", C.c_int32)]


class _ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("h", "f", "a", "g", "dh", "s", "vocab", "causal_half")]


lib.kvp_plan.restype = C.c_int
lib.kvp_plan.argtypes = [C.POINTER(_PlanIn), C.POINTER(_PlanOut)]
lib.kvp_layer_flops.restype = C.c_int
lib.kvp_layer_flops.argtypes = [C.POINTER(_ModelDesc), C.POINTER(C.c_uint64), C.POINTER(C.c_uint64),
                                C.POINTER(C.c_uint64)]


def plan(stage_begin, f_full, f_share, stage_extra, eps=(0, 1), max_conv=0, stop_on_no_improve=False,
         stage_local_donor=False, alpha=None, placement=PLACE_ARCH_BALANCED) -> dict:
    """kvp_plan (Algorithm 1).  Returns dict(z, donor, stage, stage_ratio, fir_num, fir_den, fir,
    n_conv, stop_reason)."""
    P = len(stage_begin) - 1
    L = len(f_full)
    sb, ff, fs, ex = _i32_array(stage_begin), _u64_array(f_full), _u64_array(f_share), _u64_array(stage_extra)
    z = (C.c_uint8 * L)()
    donor = (C.c_int32 * L)()
    st = (C.c_uint64 * P)()
    ratio = (C.c_double * P)()
    flags = (PLAN_STOP_ON_NO_IMPROVE if stop_on_no_improve else 0) | (PLAN_STAGE_LOCAL_DONOR if stage_local_donor else 0)
    an, ad = alpha if alpha else (0, 1)
    pin = _PlanIn(L, P, sb, ff, fs, ex, eps[0], eps[1], max_conv, flags, an, ad, placement)
    pout = _PlanOut(z, donor, st, ratio, 0, 0, 0.0, 0, 0)
    _check(lib.kvp_plan(C.byref(pin), C.byref(pout)), "kvp_plan")
    return dict(z=list(z), donor=list(donor), stage=list(st), stage_ratio=list(ratio), fir_num=pout.fir_num,
                fir_den=pout.fir_den, fir=pout.fir, n_conv=pout.n_conv, stop_reason=pout.stop_reason)


def layer_flops(h, f, a, g, dh, s, vocab, causal_half=True):
    """kvp_layer_flops -> (f_full, f_share, f_lm_head), per token, forward."""
    m = _ModelDesc(h, f, a, g, dh, s, vocab, int(causal_half))
    o = [C.c_uint64() for _ in range(3)]
    _check(lib.kvp_layer_flops(C.byref(m), *[C.byref(x) for x in o]), "kvp_layer_flops")
    return tuple(int(x.value) for x in o)


class _SimOut(C.Structure):
    _fields_ = [("makespan", C.c_int64), ("idle", C.POINTER(C.c_int64))]


lib.kvp_sim_1f1b.restype = C.c_int
lib.kvp_sim_1f1b.argtypes = [C.c_int32, C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.POINTER(_SimOut)]


def sim_1f1b(t_fwd, t_bwd, M):
    """kvp_sim_1f1b -> (makespan, idle[P]) for per-stage forward / backward times (integers) and M micro-batches."""
    P = len(t_fwd)
    tf = (C.c_int64 * P)(*[int(x) for x in t_fwd])
    tb = (C.c_int64 * len(t_bwd))(*[int(x) for x in t_bwd])
    idle = (C.c_int64 * max(P, 1))()
    out = _SimOut(0, idle)
    _check(lib.kvp_sim_1f1b(P if len(t_bwd) == P else -1, int(M), tf, tb, C.byref(out)), "kvp_sim_1f1b")
    return int(out.makespan), [int(x) for x in idle[:P]]


# ------------------------------------------------------------------------------------------
# training / prefill path
# ------------------------------------------------------------------------------------------
class Shape(C.Structure):
    """kvp_shape."""
    _fields_ = [(n, C.c_int32) for n in ("L", "B", "S", "D", "Hq", "Hkv", "dh", "dtype")]

    def __init__(self, L, B, S, D, Hq, Hkv, dh, dtype=0):
        super().__init__(L, B, S, D, Hq, Hkv, dh, dtype)


_PP = C.c_void_p    # a host array: packed bytes, or a ctypes array
lib.kvp_workspace_bytes.restype = C.c_size_t
lib.kvp_workspace_bytes.argtypes = [C.c_int, C.POINTER(Shape), C.c_void_p]
lib.kvp_proj_fwd.restype = C.c_int
lib.kvp_proj_fwd.argtypes = [C.POINTER(Shape), C.c_void_p] + [_PP] * 7 + [C.c_void_p, C.c_size_t, C.c_void_p]
lib.kvp_proj_bwd.restype = C.c_int
lib.kvp_proj_bwd.argtypes = [C.POINTER(Shape), C.c_void_p] + [_PP] * 11 + [C.c_void_p, C.c_size_t, C.c_void_p]
lib.kvp_proj_bwd_range.restype = C.c_int
lib.kvp_proj_bwd_range.argtypes = [C.POINTER(Shape), C.c_void_p] + [_PP] * 11 + [C.c_int, C.c_int, C.c_void_p, C.c_size_t,
                                                                                          C.c_void_p]
lib.kvp_out_proj_fwd.restype = C.c_int
lib.kvp_out_proj_fwd.argtypes = [C.POINTER(Shape)] + [_PP] * 3 + [C.c_void_p]
lib.kvp_out_proj_bwd.restype = C.c_int
lib.kvp_out_proj_bwd.argtypes = [C.POINTER(Shape)] + [_PP] * 5 + [C.c_void_p]
lib.kvp_attn_fwd.restype = C.c_int
lib.kvp_attn_fwd.argtypes = [C.POINTER(Shape), C.c_void_p, C.c_int, C.c_float] + [_PP] * 5 + \
    [C.c_void_p, C.c_size_t, C.c_void_p]
lib.kvp_attn_bwd.restype = C.c_int
lib.kvp_attn_bwd.argtypes = [C.POINTER(Shape), C.c_void_p, C.c_int, C.c_float] + [_PP] * 9 + \
    [C.c_void_p, C.c_size_t, C.c_void_p]


def workspace_bytes(op: int, shape: Shape, donor) -> int:
    return int(lib.kvp_workspace_bytes(op, C.byref(shape), _map(shape, donor)[0]))


def _ws(ws: Optional[torch.Tensor]):
    return (0, 0) if ws is None else (ws.data_ptr(), ws.nbytes)


def proj_fwd(shape, donor, x, wq, wk, wv, q, k, v, ws=None):
    status = _pack.proj_fwd(shape, donor, x, wq, wk, wv, q, k, v, ws, _stream())
    if status is not NotImplemented:
        return _check(status, "kvp_proj_fwd")
    d, n = _map(shape, donor)
    p, size = _ws(ws)
    _check(lib.kvp_proj_fwd(C.byref(shape), d, _ptr_array(x, n), _ptr_array(wq, n), _ptr_array(wk, n),
                            _ptr_array(wv, n), _ptr_array(q, n), _ptr_array(k, n), _ptr_array(v, n), p, size, _stream()),
           "kvp_proj_fwd")


def proj_bwd(shape, donor, x, wq, wk, wv, dq, dk_sum, dv_sum, dwq, dwk, dwv, dx, ws, layer_begin=None, layer_end=None):
    """kvp_proj_bwd, or kvp_proj_bwd_range when a layer range is given."""
    if layer_begin is None and layer_end is None:
        status = _pack.proj_bwd(shape, donor, x, wq, wk, wv, dq, dk_sum, dv_sum, dwq, dwk, dwv, dx, ws, _stream())
        if status is not NotImplemented:
            return _check(status, "kvp_proj_bwd")
    d, n = _map(shape, donor)
    p, size = _ws(ws)
    args = (C.byref(shape), d, _ptr_array(x, n), _ptr_array(wq, n), _ptr_array(wk, n), _ptr_array(wv, n),
            _ptr_array(dq, n), _ptr_array(dk_sum, n), _ptr_array(dv_sum, n), _ptr_array(dwq, n), _ptr_array(dwk, n), _ptr_array(dwv, n),
            _ptr_array(dx, n))
    if layer_begin is None and layer_end is None:
        _check(lib.kvp_proj_bwd(*args, p, size, _stream()), "kvp_proj_bwd")
    else:
        _check(lib.kvp_proj_bwd_range(*args, int(layer_begin or 0), shape.L if layer_end is None else int(layer_end), p, size,
                                      _stream()), "kvp_proj_bwd_range")


def out_proj_fwd(shape, o, wo, y):
    status = _pack.out_proj_fwd(shape, o, wo, y, _stream())
    if status is not NotImplemented:
        return _check(status, "kvp_out_proj_fwd")
    _check(lib.kvp_out_proj_fwd(C.byref(shape), _ptr_array(o, -1), _ptr_array(wo, -1), _ptr_array(y, -1), _stream()),
           "kvp_out_proj_fwd")


def out_proj_bwd(shape, o, wo, dy, d_o, dwo):
    status = _pack.out_proj_bwd(shape, o, wo, dy, d_o, dwo, _stream())
    if status is not NotImplemented:
        return _check(status, "kvp_out_proj_bwd")
    _check(lib.kvp_out_proj_bwd(C.byref(shape), _ptr_array(o, -1), _ptr_array(wo, -1), _ptr_array(dy, -1), _ptr_array(d_o, -1),
                                _ptr_array(dwo, -1), _stream()), "kvp_out_proj_bwd")


def attn_fwd(shape, donor, q, k, v, o, lse, causal=True, scale=0.0, ws=None):
    status = _pack.attn_fwd(shape, donor, causal, scale, q, k, v, o, lse, ws, _stream())
    if status is not NotImplemented:
        return _check(status, "kvp_attn_fwd")
    d, n = _map(shape, donor)
    p, size = _ws(ws)
    _check(lib.kvp_attn_fwd(C.byref(shape), d, int(causal), float(scale), _ptr_array(q, n),
                            _ptr_array(k, n), _ptr_array(v, n), _ptr_array(o, n), _ptr_array(lse, n), p, size, _stream()),
           "kvp_attn_fwd")


def attn_bwd(shape, donor, q, k, v, o, d_o, lse, dq, dk_sum, dv_sum, ws, causal=True, scale=0.0):
    status = _pack.attn_bwd(shape, donor, causal, scale, q, k, v, o, d_o, lse, dq, dk_sum, dv_sum, ws, _stream())
    if status is not NotImplemented:
        return _check(status, "kvp_attn_bwd")
    d, n = _map(shape, donor)
    p, size = _ws(ws)
    _check(lib.kvp_attn_bwd(C.byref(shape), d, int(causal), float(scale), _ptr_array(q, n),
                            _ptr_array(k, n), _ptr_array(v, n), _ptr_array(o, n), _ptr_array(d_o, n), _ptr_array(lse, n),
                            _ptr_array(dq, n), _ptr_array(dk_sum, n), _ptr_array(dv_sum, n), p, size, _stream()), "kvp_attn_bwd")


# ------------------------------------------------------------------------------------------
# decode over the shared paged cache
# ------------------------------------------------------------------------------------------
class DecodeDesc(C.Structure):
    """kvp_decode_desc."""
    _fields_ = [(n, C.c_int32) for n in ("L", "B", "Hq", "Hkv", "dh", "page_size", "max_pages", "n_pages",
                                         "num_splits", "dtype")]

    def __init__(self, L, B, Hq, Hkv, dh, page_size, max_pages, n_pages, num_splits=0, dtype=0):
        super().__init__(L, B, Hq, Hkv, dh, page_size, max_pages, n_pages, num_splits, dtype)


lib.kvp_decode_workspace_bytes.restype = C.c_size_t
lib.kvp_decode_workspace_bytes.argtypes = [C.POINTER(DecodeDesc), C.c_void_p]
lib.kvp_cache_append.restype = C.c_int
lib.kvp_cache_append.argtypes = [C.POINTER(DecodeDesc), C.c_void_p] + [_PP] * 4 + \
    [C.c_void_p, C.c_void_p, C.c_void_p]
lib.kvp_decode.restype = C.c_int
lib.kvp_decode.argtypes = [C.POINTER(DecodeDesc), C.c_void_p, C.c_float] + [_PP] * 3 + \
    [C.c_void_p, C.c_void_p] + [_PP] * 2 + [C.c_int, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]


# The calls above and below go through _pack where their arguments are plain tensors, lists and numbers, through ctypes otherwise.
_pack.bind([C.cast(getattr(lib, "kvp_" + n), C.c_void_p).value for n in (
    "gemm", "rmsnorm", "rope", "swiglu", "add", "proj_fwd", "proj_bwd", "out_proj_fwd", "out_proj_bwd", "attn_fwd", "attn_bwd",
    "cache_append", "decode")], Shape, DecodeDesc)


def decode_workspace_bytes(desc: DecodeDesc, donor) -> int:
    d, entries = _map(desc, donor)
    return int(lib.kvp_decode_workspace_bytes(C.byref(desc), d)) if entries else 0


def cache_append(desc, donor, k_new, v_new, k_cache, v_cache, block_table, lengths):
    status = _pack.cache_append(desc, donor, k_new, v_new, k_cache, v_cache, block_table, lengths, _stream())
    if status is not NotImplemented:
        return _check(status, "kvp_cache_append")
    d, n = _map(desc, donor)
    _check(lib.kvp_cache_append(C.byref(desc), d, _ptr_array(k_new, n), _ptr_array(v_new, n),
                                _ptr_array(k_cache, n), _ptr_array(v_cache, n), block_table.data_ptr(),
                                lengths.data_ptr(), _stream()), "kvp_cache_append")


def decode(desc, donor, q, k_cache, v_cache, block_table, lengths, o, lse, ws, scale=0.0, layer_begin=0,
           layer_end=None):
    status = _pack.decode(desc, donor, scale, q, k_cache, v_cache, block_table, lengths, o, lse, layer_begin, layer_end, ws, _stream())
    if status is not NotImplemented:
        return _check(status, "kvp_decode")
    d, n = _map(desc, donor)
    p, size = _ws(ws)
    _check(lib.kvp_decode(C.byref(desc), d, float(scale), _ptr_array(q, n), _ptr_array(k_cache, n),
                          _ptr_array(v_cache, n), block_table.data_ptr(), lengths.data_ptr(), _ptr_array(o, n),
                          _ptr_array(lse, n), layer_begin, desc.L if layer_end is None else layer_end, p, size, _stream()),
           "kvp_decode")


# ------------------------------------------------------------------------------------------
# benchmark bookkeeping
# ------------------------------------------------------------------------------------------
KERNEL_GEMM, KERNEL_ATTN_FWD, KERNEL_ATTN_BWD, KERNEL_DECODE, KERNEL_ATTN_BWD_AUX = range(5)
lib.kvp_launch_count.restype = C.c_ulonglong
lib.kvp_set_timing_events.restype = C.c_int
lib.kvp_set_timing_events.argtypes = [C.c_int, _PP, _PP, C.c_int]
lib.kvp_timing_events_used.restype = C.c_int
lib.kvp_timing_events_used.argtypes = [C.c_int]


def launch_count() -> int:
    return int(lib.kvp_launch_count())


lib.kvp_set_gemm_pair_mode.restype = None
lib.kvp_set_gemm_pair_mode.argtypes = [C.c_int]


def set_gemm_pair_mode(mode: int) -> None:
    """kvp_set_gemm_pair_mode: 1 = the kernel that suits the sizes (default), 0 = single-CTA tiles everywhere,
    2 = 256 x 256 tiles on CTA pairs everywhere."""
    lib.kvp_set_gemm_pair_mode(int(mode))


class KernelTimer:
    """Records CUDA events around up to n launches of one of the library's kernels and returns the
    per-launch durations in milliseconds."""

    def __init__(self, kernel: int, n: int):
        self.kernel, self.n = kernel, n
        self.starts = [torch.cuda.Event(enable_timing=True) for _ in range(n)]
        self.stops = [torch.cuda.Event(enable_timing=True) for _ in range(n)]
        for e in self.starts + self.stops:
            e.record()            # torch creates the underlying event lazily, on first record
        torch.cuda.synchronize()
        self._a = (C.c_void_p * n)(*[e.cuda_event for e in self.starts])
        self._b = (C.c_void_p * n)(*[e.cuda_event for e in self.stops])

    def __enter__(self):
        _check(lib.kvp_set_timing_events(self.kernel, self._a, self._b, self.n), "kvp_set_timing_events")
        return self

    def __exit__(self, *exc):
        self.used = int(lib.kvp_timing_events_used(self.kernel))
        lib.kvp_set_timing_events(self.kernel, None, None, 0)

    def durations_ms(self):
        torch.cuda.synchronize()
        return [self.starts[i].elapsed_time(self.stops[i]) for i in range(self.used)]


lib.kvp_selftest_bounded_wait.restype = C.c_int
lib.kvp_selftest_bounded_wait.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p]


lib.kvp_selftest_bounded_wait_pair.restype = C.c_int
lib.kvp_selftest_bounded_wait_pair.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p]


def selftest_bounded_wait_pair(scratch: torch.Tensor):
    """kvp_selftest_bounded_wait_pair: the same self-test on the CTA-pair GEMM kernel (scratch of at least 768 KiB)."""
    _check(lib.kvp_selftest_bounded_wait_pair(scratch.data_ptr(), scratch.numel() * scratch.element_size(), _stream()),
           "kvp_selftest_bounded_wait_pair")


def selftest_bounded_wait(scratch: torch.Tensor):
    """kvp_selftest_bounded_wait: enqueue the GEMM whose ring-stage arrival is withheld once; afterwards
    device_status() returns ERR_TIMEOUT once and the library stays usable."""
    _check(lib.kvp_selftest_bounded_wait(scratch.data_ptr(), scratch.numel() * scratch.element_size(), _stream()),
           "kvp_selftest_bounded_wait")


# ------------------------------------------------------------------------------------------
# decode without a workspace: scratch lives in a fixed array inside the library
# ------------------------------------------------------------------------------------------
ERR_STATIC_SCRATCH = 7
DECODE_STATIC_SCRATCH_BYTES = 16 << 20
lib.kvp_decode_static.restype = C.c_int
lib.kvp_decode_static.argtypes = [C.POINTER(DecodeDesc), C.c_void_p, C.c_float] + [_PP] * 3 + \
    [C.c_void_p, C.c_void_p] + [_PP] * 2 + [C.c_int, C.c_int, C.c_void_p]


def decode_static(desc, donor, q, k_cache, v_cache, block_table, lengths, o, lse, scale=0.0, layer_begin=0,
                  layer_end=None):
    """kvp_decode_static: same results as `decode`, for callers that cannot allocate device memory
    (no workspace tensor is passed and the library allocates nothing).  Raises KvpError with
    ERR_STATIC_SCRATCH when the request does not fit the built-in DECODE_STATIC_SCRATCH_BYTES array.
    Calls share that array, so do not let two of them overlap on the GPU."""
    d, n = _map(desc, donor)
    _check(lib.kvp_decode_static(C.byref(desc), d, float(scale), _ptr_array(q, n), _ptr_array(k_cache, n),
                                 _ptr_array(v_cache, n), block_table.data_ptr(), lengths.data_ptr(), _ptr_array(o, n),
                                 _ptr_array(lse, n), layer_begin, desc.L if layer_end is None else layer_end, _stream()),
           "kvp_decode_static")


# ------------------------------------------------------------------------------------------
# tokens with rotary positions into the paged cache; the cache held in 8 bits
# ------------------------------------------------------------------------------------------
CACHE_BLOCK = 16     # tokens that share a scale
lib.kvp_cache_append_tokens.restype = C.c_int
lib.kvp_cache_append_tokens.argtypes = [C.POINTER(DecodeDesc), C.c_void_p, C.c_int32, C.c_void_p, C.c_float] + [_PP] * 8 + [C.c_void_p] * 3
lib.kvp_decode8_workspace_bytes.restype = C.c_size_t
lib.kvp_decode8_workspace_bytes.argtypes = [C.POINTER(DecodeDesc), C.c_void_p]
lib.kvp_decode8.restype = C.c_int
lib.kvp_decode8.argtypes = [C.POINTER(DecodeDesc), C.c_void_p, C.c_float] + [_PP] * 5 + [C.c_void_p, C.c_void_p] + [_PP] * 2 + \
    [C.c_int, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
_pack.bind_cache([C.cast(getattr(lib, "kvp_" + n), C.c_void_p).value for n in ("cache_append_tokens", "decode8")])

_I32, _CODES, _SCALES = (torch.int32,), (torch.float8_e4m3fn, torch.uint8), (torch.float8_e8m0fnu, torch.uint8)


def _call_place():
    """Device that a call runs on (-2: there is none, and the library refuses the call or fails to launch) and its stream."""
    if _raw_stream is not None and torch.cuda.is_initialized():
        device = _device()
        return device, _raw_stream(device)
    return (_device() if torch.cuda.is_available() else -2), _stream()


def _fit(what: str, t, dtypes, numel: int, device: int) -> None:
    """The library sees pointers alone: what a tensor has to be besides is looked at here."""
    if t.dtype not in dtypes:
        raise ValueError(f"{what} is {t.dtype}: {' or '.join(map(str, dtypes))} is wanted")
    if t.numel() != numel:
        raise ValueError(f"{what} has {t.numel()} elements {tuple(t.shape)}: {numel} are wanted")
    if not t.is_contiguous():
        raise ValueError(f"{what} has strides {t.stride()}: a contiguous tensor is wanted")
    if device != -2 and (not t.is_cuda or t.get_device() != device):
        raise ValueError(f"{what} is on {t.device}: the call runs on cuda:{device}")


def _fit_layers(what, ts, dtypes, numel, layers, device) -> None:
    for l in layers:
        if l < len(ts) and ts[l] is not None:      # (missing ones are the library's to refuse)
            _fit(f"{what}[{l}]", ts[l], dtypes, numel, device)


def _layer_range(desc, donor, begin=0, end=None):
    """Layers of a call and their donors, as far as the map is one (the library refuses it otherwise)."""
    n = min(max(desc.L, 0), len(donor))
    layers = range(max(begin, 0), n if end is None else min(end, n))
    return layers, sorted({int(donor[l]) for l in layers if 0 <= int(donor[l]) <= l})


def _io(desc):
    return (torch.float32,) if desc.dtype == F32 else (torch.bfloat16,)


def cache_append_tokens(desc, donor, k_new, v_new, k_cache, v_cache, block_table, lengths, first=None, theta=0.0, q=None, q_out=None,
                        k_scale=None, v_scale=None):
    """kvp_cache_append_tokens: the rows k_new[l], v_new[l] [T, Hkv, dh] (owner layers) go into the pages of their sequences, K
    rotated by the token's position where theta is not 0, and q[l] [T, Hq, dh] rotated by the same positions goes to q_out[l].
    Sequence b has rows first[b] .. first[b+1]-1 (int32 [B + 1]; None: one token each, T == B) at the positions before lengths[b].
    With k_scale, v_scale (uint8 or float8_e8m0fnu [n_pages, Hkv, page_size / 16]) the cache holds float8_e4m3fn numbers.
    Tensors are contiguous, of the documented sizes, on the current device: ValueError otherwise."""
    device, stream = _call_place()
    status = _pack.cache_append_tokens(desc, donor, k_new, v_new, k_cache, v_cache, block_table, lengths, first, theta, q, q_out, k_scale, v_scale,
                                       device, stream)
    if status is not NotImplemented:
        return _check(status, "kvp_cache_append_tokens")
    layers, owners = _layer_range(desc, donor)
    T = next((int(t.shape[0]) if t.dim() else 0 for t in k_new if t is not None), 0)
    if T == 0 and any(l >= len(ts) or ts[l] is None for ts in (k_new, v_new) for l in owners):
        _check(ERR_INVALID_ARG, "kvp_cache_append_tokens")     # (by their addresses the library cannot tell missing rows from none)
    rows, io = desc.n_pages * desc.Hkv * desc.page_size, _io(desc)
    held = (torch.bfloat16,) if k_scale is None else _CODES
    for what, ts, dtypes, numel, of in (("k_new", k_new, io, T * desc.Hkv * desc.dh, owners), ("v_new", v_new, io, T * desc.Hkv * desc.dh, owners),
                                        ("k_cache", k_cache, held, rows * desc.dh, owners), ("v_cache", v_cache, held, rows * desc.dh, owners),
                                        ("q", q, io, T * desc.Hq * desc.dh, layers), ("q_out", q_out, io, T * desc.Hq * desc.dh, layers),
                                        ("k_scale", k_scale, _SCALES, rows // CACHE_BLOCK, owners), ("v_scale", v_scale, _SCALES, rows // CACHE_BLOCK, owners)):
        if ts is not None:
            _fit_layers(what, ts, dtypes, numel, of, device)
    for what, t, numel in (("block_table", block_table, desc.B * desc.max_pages), ("lengths", lengths, desc.B), ("first", first, desc.B + 1)):
        if t is not None:
            _fit(what, t, _I32, numel, device)
    d, n = _map(desc, donor)
    array = lambda ts: None if ts is None else _ptr_array(ts, n)
    _check(lib.kvp_cache_append_tokens(C.byref(desc), d, T, _ptr(first), float(theta), array(q), array(q_out), array(k_new), array(v_new),
                                       array(k_cache), array(v_cache), array(k_scale), array(v_scale), _ptr(block_table), _ptr(lengths), stream),
           "kvp_cache_append_tokens")


def decode8_workspace_bytes(desc: DecodeDesc, donor) -> int:
    """kvp_decode8_workspace_bytes: enough for any layer range."""
    d, entries = _map(desc, donor)
    return int(lib.kvp_decode8_workspace_bytes(C.byref(desc), d)) if entries else 0


def decode8(desc, donor, q, k_cache, v_cache, k_scale, v_scale, block_table, lengths, o, lse, ws, scale=0.0, layer_begin=0, layer_end=None):
    """kvp_decode8: decode attention over the cache held in 8 bits, as cache_append_tokens with scales leaves it.  Arguments as for
    decode; a sequence of length 0 has output 0 and LSE -infinity.  Tensors are contiguous, of the documented sizes, on the
    current device: ValueError otherwise."""
    device, stream = _call_place()
    status = _pack.decode8(desc, donor, scale, q, k_cache, v_cache, k_scale, v_scale, block_table, lengths, o, lse, layer_begin, layer_end, ws, device,
                           stream)
    if status is not NotImplemented:
        return _check(status, "kvp_decode8")
    end = desc.L if layer_end is None else int(layer_end)
    layers, owners = _layer_range(desc, donor, int(layer_begin), end)
    rows, io = desc.n_pages * desc.Hkv * desc.page_size, _io(desc)
    for what, ts, dtypes, numel, of in (("q", q, io, desc.B * desc.Hq * desc.dh, layers), ("o", o, io, desc.B * desc.Hq * desc.dh, layers),
                                        ("lse", lse, (torch.float32,), desc.B * desc.Hq, layers),
                                        ("k_cache", k_cache, _CODES, rows * desc.dh, owners), ("v_cache", v_cache, _CODES, rows * desc.dh, owners),
                                        ("k_scale", k_scale, _SCALES, rows // CACHE_BLOCK, owners), ("v_scale", v_scale, _SCALES, rows // CACHE_BLOCK, owners)):
        _fit_layers(what, ts, dtypes, numel, of, device)
    _fit("block_table", block_table, _I32, desc.B * desc.max_pages, device)
    _fit("lengths", lengths, _I32, desc.B, device)
    if ws is not None:
        _fit("ws", ws, (ws.dtype,), ws.numel(), device)
    d, n = _map(desc, donor)
    p, size = _ws(ws)
    _check(lib.kvp_decode8(C.byref(desc), d, float(scale), _ptr_array(q, n), _ptr_array(k_cache, n), _ptr_array(v_cache, n), _ptr_array(k_scale, n),
                           _ptr_array(v_scale, n), block_table.data_ptr(), lengths.data_ptr(), _ptr_array(o, n), _ptr_array(lse, n), int(layer_begin), end, p,
                           size, stream), "kvp_decode8")


# ------------------------------------------------------------------------------------------
# attention of new tokens over the paged cache
# ------------------------------------------------------------------------------------------
lib.kvp_attn_chunk_workspace_bytes.restype = C.c_size_t
lib.kvp_attn_chunk_workspace_bytes.argtypes = [C.POINTER(DecodeDesc), C.c_void_p, C.c_int32]
lib.kvp_attn_chunk.restype = C.c_int
lib.kvp_attn_chunk.argtypes = [C.POINTER(DecodeDesc), C.c_void_p, C.c_int32, C.c_void_p, C.c_float, C.c_int32, C.c_int32] + [_PP] * 5 + \
    [C.c_void_p, C.c_void_p] + [_PP] * 2 + [C.c_int, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]


def attn_chunk_workspace_bytes(desc: DecodeDesc, donor, T: int) -> int:
    """kvp_attn_chunk_workspace_bytes: enough for any layer range and for T rows or fewer."""
    d, entries = _map(desc, donor)
    return int(lib.kvp_attn_chunk_workspace_bytes(C.byref(desc), d, int(T))) if entries else 0


def _fit_pools(desc, k_cache, v_cache, k_scale, v_scale, owners, device) -> None:
    rows, held = desc.n_pages * desc.Hkv * desc.page_size, (torch.bfloat16,) if k_scale is None else _CODES
    for what, ts, dtypes, numel in (("k_cache", k_cache, held, rows * desc.dh), ("v_cache", v_cache, held, rows * desc.dh),
                                    ("k_scale", k_scale, _SCALES, rows // CACHE_BLOCK), ("v_scale", v_scale, _SCALES, rows // CACHE_BLOCK)):
        if ts is not None:
            _fit_layers(what, ts, dtypes, numel, owners, device)


def attn_chunk(desc, donor, q, k_cache, v_cache, block_table, lengths, o, lse, ws, first=None, scale=0.0, window=0, sinks=0, k_scale=None, v_scale=None,
               layer_begin=0, layer_end=None):
    """kvp_attn_chunk: attention of the rows q[l] [T, Hq, dh] over the paged cache that their tokens are in already, into o[l] and the
    log-sum-exp lse[l] [T, Hq].  Sequence b has rows first[b] .. first[b+1]-1 (int32 [B + 1]; None: one token each, T == B) at the
    positions before lengths[b]; a row sees the tokens up to its own, with window > 0 the last `window` of them and the first `sinks`
    alone.  With k_scale, v_scale the cache is the 8-bit one.  ws: attn_chunk_workspace_bytes.  Tensors are contiguous, of the
    documented sizes, on the current device: ValueError otherwise."""
    device, stream = _call_place()
    status = _pack.attn_chunk(desc, donor, q, k_cache, v_cache, block_table, lengths, o, lse, ws, first, scale, window, sinks, k_scale, v_scale, layer_begin,
                              layer_end, device, stream)
    if status is not NotImplemented:
        return _check(status, "kvp_attn_chunk")
    end = desc.L if layer_end is None else int(layer_end)
    layers, owners = _layer_range(desc, donor, int(layer_begin), end)
    T = next((int(q[l].shape[0]) if q[l].dim() else 0 for l in layers if l < len(q) and q[l] is not None), 0)
    if T == 0 and any(l >= len(ts) or ts[l] is None for ts in (q, o, lse) for l in layers):
        _check(ERR_INVALID_ARG, "kvp_attn_chunk")     # (by their addresses the library cannot tell missing rows from none)
    io = _io(desc)
    for what, ts, dtypes, numel in (("q", q, io, T * desc.Hq * desc.dh), ("o", o, io, T * desc.Hq * desc.dh), ("lse", lse, (torch.float32,), T * desc.Hq)):
        _fit_layers(what, ts, dtypes, numel, layers, device)
    _fit_pools(desc, k_cache, v_cache, k_scale, v_scale, owners, device)
    for what, t, numel in (("block_table", block_table, desc.B * desc.max_pages), ("lengths", lengths, desc.B), ("first", first, desc.B + 1)):
        if t is not None:
            _fit(what, t, _I32, numel, device)
    if ws is not None:
        _fit("ws", ws, (ws.dtype,), ws.numel(), device)
    d, n = _map(desc, donor)
    array = lambda ts: None if ts is None else _ptr_array(ts, n)
    p, size = _ws(ws)
    _check(lib.kvp_attn_chunk(C.byref(desc), d, T, _ptr(first), float(scale), int(window), int(sinks), _ptr_array(q, n), _ptr_array(k_cache, n),
                              _ptr_array(v_cache, n), array(k_scale), array(v_scale), _ptr(block_table), _ptr(lengths), _ptr_array(o, n),
                              _ptr_array(lse, n), int(layer_begin), end, p, size, stream), "kvp_attn_chunk")


# ------------------------------------------------------------------------------------------
# pages of the cache
# ------------------------------------------------------------------------------------------
_POOLS = [_PP] * 4
lib.kvp_pages_workspace_bytes.restype = C.c_size_t
lib.kvp_pages_workspace_bytes.argtypes = [C.POINTER(DecodeDesc)]
lib.kvp_pages_copy.restype = C.c_int
lib.kvp_pages_copy.argtypes = [C.POINTER(DecodeDesc), C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p] + _POOLS + [C.c_void_p]
lib.kvp_pages_fork.restype = C.c_int
lib.kvp_pages_fork.argtypes = [C.POINTER(DecodeDesc)] + [C.c_void_p] * 5 + [C.c_size_t, C.c_void_p]
lib.kvp_pages_resize.restype = C.c_int
lib.kvp_pages_resize.argtypes = [C.POINTER(DecodeDesc)] + [C.c_void_p] * 7 + [C.c_size_t] + _POOLS + [C.c_void_p]
lib.kvp_pages_trim.restype = C.c_int
lib.kvp_pages_trim.argtypes = [C.POINTER(DecodeDesc), C.c_int32, C.c_int32] + [C.c_void_p] * 4
lib.kvp_pages_compact.restype = C.c_int
lib.kvp_pages_compact.argtypes = [C.POINTER(DecodeDesc)] + [C.c_void_p] * 6 + [C.c_size_t] + _POOLS + [C.c_void_p]


def pages_workspace_bytes(desc: DecodeDesc) -> int:
    """kvp_pages_workspace_bytes: enough for each of the calls below."""
    return int(lib.kvp_pages_workspace_bytes(C.byref(desc)))


def _fit_book(desc, device, ws=None, **tensors) -> None:
    sizes = dict(block_table=desc.B * desc.max_pages, refs=desc.n_pages, lacking=1, used=1)
    for what, t in tensors.items():
        if t is not None:
            _fit(what, t, _I32, sizes.get(what, desc.B), device)
    if ws is not None:
        _fit("ws", ws, (ws.dtype,), ws.numel(), device)


def _pool_arrays(desc, donor, k_cache, v_cache, k_scale, v_scale, device):
    _fit_pools(desc, k_cache, v_cache, k_scale, v_scale, _layer_range(desc, donor)[1], device)
    d, n = _map(desc, donor)
    return d, [None if ts is None else _ptr_array(ts, n) for ts in (k_cache, v_cache, k_scale, v_scale)]


def pages_copy(desc, donor, src, dst, k_cache, v_cache, k_scale=None, v_scale=None):
    """kvp_pages_copy: the pages src[i] go to dst[i] (int32, as many), in all owner layers.  No page may be the target of two, nor a
    target and a source.  Tensors of these calls are contiguous, of the documented sizes, on the current device: ValueError otherwise."""
    device, stream = _call_place()
    status = _pack.pages_copy(desc, donor, src, dst, k_cache, v_cache, k_scale, v_scale, device, stream)
    if status is not NotImplemented:
        return _check(status, "kvp_pages_copy")
    n = src.numel()
    _fit("src", src, _I32, n, device)
    _fit("dst", dst, _I32, n, device)
    d, pools = _pool_arrays(desc, donor, k_cache, v_cache, k_scale, v_scale, device)
    _check(lib.kvp_pages_copy(C.byref(desc), d, n, _ptr(src), _ptr(dst), *pools, stream), "kvp_pages_copy")


def pages_fork(desc, parent, refs, block_table, lengths, ws):
    """kvp_pages_fork: row b goes on from what row parent[b] was (its own number: it stays; -1: it ends).  Pages are shared, none is
    copied; refs, block_table and lengths are updated in place."""
    device, stream = _call_place()
    status = _pack.pages_fork(desc, parent, refs, block_table, lengths, ws, device, stream)
    if status is not NotImplemented:
        return _check(status, "kvp_pages_fork")
    _fit_book(desc, device, ws, parent=parent, refs=refs, block_table=block_table, lengths=lengths)
    p, size = _ws(ws)
    _check(lib.kvp_pages_fork(C.byref(desc), _ptr(parent), _ptr(refs), _ptr(block_table), _ptr(lengths), p, size, stream), "kvp_pages_fork")


def pages_resize(desc, donor, new_lengths, refs, block_table, lengths, lacking, ws, k_cache, v_cache, k_scale=None, v_scale=None):
    """kvp_pages_resize: rows grow and shrink to new_lengths; a row that grows inside a shared page gets a copy of it,
    one that grows inside a place without a page gets one there.  lacking (int32
    [1]) receives 0, or what is short (then nothing is changed): the pages lacking, -1 for a length out of range."""
    device, stream = _call_place()
    status = _pack.pages_resize(desc, donor, new_lengths, refs, block_table, lengths, lacking, ws, k_cache, v_cache, k_scale, v_scale, device, stream)
    if status is not NotImplemented:
        return _check(status, "kvp_pages_resize")
    _fit_book(desc, device, ws, new_lengths=new_lengths, refs=refs, block_table=block_table, lengths=lengths, lacking=lacking)
    d, pools = _pool_arrays(desc, donor, k_cache, v_cache, k_scale, v_scale, device)
    p, size = _ws(ws)
    _check(lib.kvp_pages_resize(C.byref(desc), d, _ptr(new_lengths), _ptr(refs), _ptr(block_table), _ptr(lengths), _ptr(lacking), p, size, *pools, stream),
           "kvp_pages_resize")


def pages_trim(desc, window, sinks, refs, block_table, lengths):
    """kvp_pages_trim: frees the pages that no later token sees with this window and so many first tokens."""
    device, stream = _call_place()
    status = _pack.pages_trim(desc, window, sinks, refs, block_table, lengths, device, stream)
    if status is not NotImplemented:
        return _check(status, "kvp_pages_trim")
    _fit_book(desc, device, refs=refs, block_table=block_table, lengths=lengths)
    _check(lib.kvp_pages_trim(C.byref(desc), int(window), int(sinks), _ptr(refs), _ptr(block_table), _ptr(lengths), stream), "kvp_pages_trim")


def pages_compact(desc, donor, refs, block_table, lengths, used, ws, k_cache, v_cache, k_scale=None, v_scale=None):
    """kvp_pages_compact: the used pages become pages 0 .. used-1; used (int32 [1]) receives their number."""
    device, stream = _call_place()
    status = _pack.pages_compact(desc, donor, refs, block_table, lengths, used, ws, k_cache, v_cache, k_scale, v_scale, device, stream)
    if status is not NotImplemented:
        return _check(status, "kvp_pages_compact")
    _fit_book(desc, device, ws, refs=refs, block_table=block_table, lengths=lengths, used=used)
    d, pools = _pool_arrays(desc, donor, k_cache, v_cache, k_scale, v_scale, device)
    p, size = _ws(ws)
    _check(lib.kvp_pages_compact(C.byref(desc), d, _ptr(refs), _ptr(block_table), _ptr(lengths), _ptr(used), p, size, *pools, stream), "kvp_pages_compact")


_pack.bind_pages([C.cast(getattr(lib, "kvp_" + n), C.c_void_p).value for n in ("attn_chunk", "pages_copy", "pages_fork", "pages_resize", "pages_trim", "pages_compact")])
