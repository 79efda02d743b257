"""Thin ctypes binding of libdpool (include/dpool.h).

Argument marshalling only: every step of the decode runs in the library's
HIP kernels, the pool and the router run in its C++ host code.  torch
tensors supply device pointers and the current HIP stream.  There is no
fallback: if libdpool.so is missing or fails to load, every call raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# DPOOL_LIB selects another build of the same library (the host-sanitizer
# build of build_sanitize.py, for the CPU tests)
LIB_PATH = os.environ.get("DPOOL_LIB") or os.path.join(_PKG, "libdpool.so")

DP_OK = 0
DP_EIO = -5
DP_ENOMEM = -12
DP_EINVAL = -22
DP_ENOTSUP = -95
KV_BF16, KV_FP8_E4M3, KV_FP8_E4M3_BLOCK = 0, 1, 2
OUT_BF16, OUT_FP32 = 0, 1

# every function the header declares
EXPORTS = (
    "dp_last_error", "dp_version",
    "kv_pool_create", "kv_pool_info", "kv_pool_alloc_seq", "kv_pool_free_seq", "kv_pool_destroy",
    "route_default_params", "route_init", "route_requests", "route_on_response",
    "route_adapt_default_params", "route_adapt_threshold", "dp_cost_model",
    "paged_decode_workspace_size", "paged_decode_partition_tokens", "paged_decode_attention",
    "paged_decode_attention_noalloc", "window_decode_workspace_size", "window_decode_attention",
    "kv_cache_append", "chunked_prefill_attention", "window_prefill_attention", "kv_tables_step", "qk_norm_rope_append",
    "qk_norm_rope_append_scaled",
    "tree_decode_workspace_size", "tree_decode_attention", "kv_cache_accept", "dp_hbm_read_probe",
)


class DpoolError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libdpool error {code}: {msg}")
        self.code = code


class PoolConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype_bytes", ctypes.c_int32), ("block_size", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("c_max", ctypes.c_int64), ("m_gpu_bytes", ctypes.c_double), ("util", ctypes.c_double),
                ("m_model_bytes", ctypes.c_double)]


class RouteParams(ctypes.Structure):
    _fields_ = [("b_short", ctypes.c_double), ("beta", ctypes.c_double), ("gamma", ctypes.c_double),
                ("c0", ctypes.c_double), ("c_min", ctypes.c_double), ("spill_theta", ctypes.c_double)]


class CatState(ctypes.Structure):
    _fields_ = [("c_hat", ctypes.c_double), ("sigma", ctypes.c_double)]


class PoolState(ctypes.Structure):
    _fields_ = [("c_max", ctypes.c_int64), ("capacity", ctypes.c_int64), ("in_flight", ctypes.c_int64)]


class PoolSignals(ctypes.Structure):
    _fields_ = [("admitted", ctypes.c_int64), ("preempted", ctypes.c_int64), ("oom", ctypes.c_int64),
                ("rejected", ctypes.c_int64)]


class AdaptParams(ctypes.Structure):
    _fields_ = [("w_preempt", ctypes.c_double), ("w_oom", ctypes.c_double), ("w_reject", ctypes.c_double),
                ("target", ctypes.c_double), ("step", ctypes.c_double), ("b_min", ctypes.c_double),
                ("b_max", ctypes.c_double)]


class CostResult(ctypes.Structure):
    _fields_ = [("g_homo", ctypes.c_int64), ("g_dual", ctypes.c_int64), ("rho", ctypes.c_double),
                ("savings_formula", ctypes.c_double), ("savings_fleet", ctypes.c_double)]


class DecodeShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("max_blocks_per_seq", ctypes.c_int32), ("max_context_len", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("partition_tokens", ctypes.c_int32), ("workgroups_per_cu", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("num_blocks", ctypes.c_int64)]


class PrefillShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("max_blocks_per_seq", ctypes.c_int32), ("max_context_len", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("query_tile", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("total_q", ctypes.c_int64), ("num_blocks", ctypes.c_int64)]


class TablesShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("block_size", ctypes.c_int32), ("max_blocks_per_seq", ctypes.c_int32),
                ("mask_words", ctypes.c_int32), ("total_rows", ctypes.c_int64), ("num_blocks", ctypes.c_int64),
                ("reserved", ctypes.c_int64)]


class QKShape(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("kv_dtype", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("reserved", ctypes.c_int32), ("rows", ctypes.c_int64),
                ("num_blocks", ctypes.c_int64), ("n_positions", ctypes.c_int64), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


class TreeShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("max_blocks_per_seq", ctypes.c_int32), ("max_context_len", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("mask_words", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("total_q", ctypes.c_int64), ("num_blocks", ctypes.c_int64)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libdpool.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_08075_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        c_i32p, c_i64p, c_i8p = (ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int64),
                                 ctypes.POINTER(ctypes.c_int8))
        L.dp_last_error.restype = ctypes.c_char_p
        L.dp_version.restype = ctypes.c_char_p
        L.kv_pool_create.argtypes = [ctypes.POINTER(PoolConfig), ctypes.c_uint64, ctypes.POINTER(ctypes.c_void_p)]
        L.kv_pool_info.argtypes = [ctypes.c_void_p, c_i64p, c_i64p, c_i64p, c_i64p, c_i64p]
        L.kv_pool_alloc_seq.argtypes = [ctypes.c_void_p, ctypes.c_int64, c_i32p]
        L.kv_pool_free_seq.argtypes = [ctypes.c_void_p, c_i32p, ctypes.c_int64]
        L.kv_pool_destroy.argtypes = [ctypes.c_void_p]
        L.kv_pool_destroy.restype = None
        L.route_default_params.argtypes = [ctypes.POINTER(RouteParams)]
        L.route_init.argtypes = [ctypes.POINTER(RouteParams), ctypes.POINTER(CatState), ctypes.c_int32]
        L.route_requests.argtypes = [ctypes.POINTER(RouteParams), ctypes.POINTER(CatState), ctypes.c_int32,
                                     ctypes.POINTER(PoolState), c_i64p, c_i32p, c_i64p, ctypes.c_int64, c_i8p, c_i64p]
        L.route_on_response.argtypes = [ctypes.POINTER(RouteParams), ctypes.POINTER(CatState), ctypes.c_int32,
                                        ctypes.c_int32, ctypes.c_int64, ctypes.c_int64]
        L.route_adapt_default_params.argtypes = [ctypes.POINTER(AdaptParams)]
        L.route_adapt_threshold.argtypes = [ctypes.POINTER(AdaptParams), ctypes.POINTER(PoolSignals),
                                            ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)]
        L.dp_cost_model.argtypes = [ctypes.c_double] * 4 + [ctypes.POINTER(CostResult)]
        L.paged_decode_workspace_size.argtypes = [ctypes.POINTER(DecodeShape)]
        L.paged_decode_workspace_size.restype = ctypes.c_size_t
        L.paged_decode_partition_tokens.argtypes = [ctypes.POINTER(DecodeShape)]
        L.paged_decode_partition_tokens.restype = ctypes.c_int32
        L.paged_decode_attention.argtypes = [ctypes.c_void_p] * 5 + [ctypes.c_float] + [ctypes.c_void_p] * 3 + [
            ctypes.POINTER(DecodeShape), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.paged_decode_attention_noalloc.argtypes = [ctypes.c_void_p] * 5 + [ctypes.c_float] + [
            ctypes.c_void_p] * 3 + [ctypes.POINTER(DecodeShape), ctypes.c_void_p]
        L.window_decode_workspace_size.argtypes = [ctypes.POINTER(DecodeShape), ctypes.c_int32, ctypes.c_int32]
        L.window_decode_workspace_size.restype = ctypes.c_size_t
        L.window_decode_attention.argtypes = [ctypes.c_void_p] * 5 + [ctypes.c_float] + [ctypes.c_int32] * 2 + [
            ctypes.c_void_p] * 3 + [ctypes.POINTER(DecodeShape), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.kv_cache_append.argtypes = [ctypes.c_void_p] * 8 + [ctypes.POINTER(DecodeShape), ctypes.c_void_p]
        L.chunked_prefill_attention.argtypes = [ctypes.c_void_p] * 6 + [ctypes.c_float] + [ctypes.c_void_p] * 3 + [
            ctypes.POINTER(PrefillShape), ctypes.c_void_p]
        L.window_prefill_attention.argtypes = [ctypes.c_void_p] * 6 + [ctypes.c_float] + [ctypes.c_int32] * 2 + [
            ctypes.c_void_p] * 3 + [ctypes.POINTER(PrefillShape), ctypes.c_void_p]
        L.kv_tables_step.argtypes = [ctypes.c_void_p] * 15 + [ctypes.POINTER(TablesShape), ctypes.c_void_p]
        L.qk_norm_rope_append.argtypes = [ctypes.c_void_p] * 5 + [ctypes.c_float] + [ctypes.c_void_p] * 8 + [
            ctypes.POINTER(QKShape), ctypes.c_void_p]
        L.qk_norm_rope_append_scaled.argtypes = L.qk_norm_rope_append.argtypes
        L.tree_decode_workspace_size.argtypes = [ctypes.POINTER(TreeShape)]
        L.tree_decode_workspace_size.restype = ctypes.c_size_t
        L.tree_decode_attention.argtypes = [ctypes.c_void_p] * 7 + [ctypes.c_float] + [ctypes.c_void_p] * 3 + [
            ctypes.POINTER(TreeShape), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.kv_cache_accept.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int32] + [ctypes.c_void_p] * 5 + [
            ctypes.c_int32, ctypes.c_void_p, ctypes.POINTER(TreeShape), ctypes.c_void_p]
        L.dp_hbm_read_probe.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int64,
                                        ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        _lib = L
    return _lib


def last_error() -> str:
    return lib().dp_last_error().decode()


def check(rc: int) -> int:
    if rc != DP_OK:
        raise DpoolError(rc, last_error())
    return rc


def version() -> str:
    return lib().dp_version().decode()


def _ptr(a: np.ndarray, ctype):
    return a.ctypes.data_as(ctypes.POINTER(ctype))


# ---------------------------------------------------------------- KV pool

@dataclass
class PoolInfo:
    m_seq_bytes: int
    n_seq: int
    blocks_per_seq: int
    num_blocks: int
    free_blocks: int


class KVPool:
    """Owner of a dp_kv_pool handle (host memory)."""

    def __init__(self, n_layers, n_kv_heads, head_dim, dtype_bytes, c_max, m_gpu_bytes, util, m_model_bytes,
                 block_size=16, seed=0):
        cfg = PoolConfig(n_layers, n_kv_heads, head_dim, dtype_bytes, block_size, 0, c_max, m_gpu_bytes, util,
                         m_model_bytes)
        h = ctypes.c_void_p()
        check(lib().kv_pool_create(ctypes.byref(cfg), ctypes.c_uint64(seed), ctypes.byref(h)))
        self._h = h
        self.block_size = block_size

    def info(self) -> PoolInfo:
        vals = [ctypes.c_int64() for _ in range(5)]
        check(lib().kv_pool_info(self._h, *[ctypes.byref(v) for v in vals]))
        return PoolInfo(*[v.value for v in vals])

    def alloc_seq(self, n_tokens: int) -> np.ndarray:
        n = -(-n_tokens // self.block_size) if n_tokens > 0 else 0
        out = np.empty(max(n, 1), dtype=np.int32)
        check(lib().kv_pool_alloc_seq(self._h, n_tokens, _ptr(out, ctypes.c_int32)))
        return out[:n]

    def free_seq(self, ids) -> None:
        ids = np.ascontiguousarray(ids, dtype=np.int32)
        check(lib().kv_pool_free_seq(self._h, _ptr(ids, ctypes.c_int32), len(ids)))

    def close(self):
        if self._h:
            lib().kv_pool_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------- router

def default_route_params() -> RouteParams:
    p = RouteParams()
    check(lib().route_default_params(ctypes.byref(p)))
    return p


def make_categories(params: RouteParams, n_cats: int):
    cats = (CatState * n_cats)()
    check(lib().route_init(ctypes.byref(params), cats, n_cats))
    return cats


def make_pools(short_c_max, short_capacity, long_c_max, long_capacity):
    pools = (PoolState * 2)()
    pools[0] = PoolState(short_c_max, short_capacity, 0)
    pools[1] = PoolState(long_c_max, long_capacity, 0)
    return pools


def route_requests(params, cats, pools, req_bytes, req_cat, req_max_out):
    """Route a batch in order; returns (pool ids int8 [n], L_total int64 [n])."""
    b = np.ascontiguousarray(req_bytes, dtype=np.int64)
    k = np.ascontiguousarray(req_cat, dtype=np.int32)
    m = np.ascontiguousarray(req_max_out, dtype=np.int64)
    n = len(b)
    if len(k) != n or len(m) != n:
        raise ValueError("request arrays differ in length")
    out_p = np.empty(max(n, 1), dtype=np.int8)
    out_l = np.empty(max(n, 1), dtype=np.int64)
    check(lib().route_requests(ctypes.byref(params), cats, len(cats), pools, _ptr(b, ctypes.c_int64),
                               _ptr(k, ctypes.c_int32), _ptr(m, ctypes.c_int64), n, _ptr(out_p, ctypes.c_int8),
                               _ptr(out_l, ctypes.c_int64)))
    return out_p[:n], out_l[:n]


def route_on_response(params, cats, cat: int, req_bytes: int, prompt_tokens: int) -> None:
    check(lib().route_on_response(ctypes.byref(params), cats, len(cats), cat, req_bytes, prompt_tokens))


def default_adapt_params() -> AdaptParams:
    p = AdaptParams()
    check(lib().route_adapt_default_params(ctypes.byref(p)))
    return p


def adapt_threshold(params: AdaptParams, short_signals, long_signals, b_short: float):
    """One control step; signals are (admitted, preempted, oom, rejected).  Returns (b_short, action)."""
    sig = (PoolSignals * 2)(PoolSignals(*short_signals), PoolSignals(*long_signals))
    b = ctypes.c_double(float(b_short))
    act = ctypes.c_int32(0)
    check(lib().route_adapt_threshold(ctypes.byref(params), sig, ctypes.byref(b), ctypes.byref(act)))
    return b.value, act.value


# ---------------------------------------------------------------- cost model

def cost_model(lam: float, alpha: float, mu_short: float, mu_long: float) -> CostResult:
    """Sec. 3 fleet sizing and savings (include/dpool.h, dp_cost_model)."""
    out = CostResult()
    check(lib().dp_cost_model(float(lam), float(alpha), float(mu_short), float(mu_long), ctypes.byref(out)))
    return out


# ---------------------------------------------------------------- decode

def _kv_dtype(kv_fp8, block_scales):
    return KV_FP8_E4M3_BLOCK if block_scales else KV_FP8_E4M3 if kv_fp8 else KV_BF16


def decode_shape(batch, n_q_heads, n_kv_heads, max_blocks_per_seq, max_context_len, num_blocks, kv_fp8=False,
                 out_fp32=False, partition_tokens=0, workgroups_per_cu=0, head_dim=128, block_size=16,
                 block_scales=False) -> DecodeShape:
    """block_scales: an e4m3 cache with a scale for each block and head (window_decode_attention)."""
    return DecodeShape(batch, n_q_heads, n_kv_heads, head_dim, block_size, max_blocks_per_seq, max_context_len,
                       _kv_dtype(kv_fp8, block_scales), OUT_FP32 if out_fp32 else OUT_BF16, partition_tokens,
                       workgroups_per_cu, 0, num_blocks)


def workspace_size(shape: DecodeShape) -> int:
    return int(lib().paged_decode_workspace_size(ctypes.byref(shape)))


def partition_tokens(shape: DecodeShape) -> int:
    return int(lib().paged_decode_partition_tokens(ctypes.byref(shape)))


_partition_tokens = partition_tokens


def _stream_ptr(stream):
    if stream is None:
        import torch
        # torch's current stream of its current device, without the Stream
        # object that torch.cuda.current_stream() builds (0.2 us, 2.7 with it:
        # more than half of a small call's time on the host)
        try:
            if torch.cuda.is_initialized():
                return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:  # (torch does not promise these two names)
            pass
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _stream_here(stream, dev):
    """_stream_ptr, for tensors on device dev, which has to be the current one, where the launch goes."""
    import torch
    if dev < 0:
        raise ValueError("tensors must all be on the current device")
    try:
        if dev == torch._C._cuda_getDevice() and stream is None:
            return torch._C._cuda_getCurrentRawStream(dev)
    except AttributeError:  # (as in _stream_ptr)
        pass
    if dev != torch.cuda.current_device():
        raise ValueError(f"tensors on device {dev}: they must be on the current device")
    return _stream_ptr(stream)


_types = None


def _element_types():
    """The element types that may hold bf16 values, e4m3 codes and exponent bytes (as such or as their bits); int32,
    int64 and float32."""
    global _types
    if _types is None:
        import torch
        some = lambda *names: frozenset(getattr(torch, n) for n in names if hasattr(torch, n))  # noqa: E731
        _types = (some("bfloat16", "int16", "uint16"), some("float8_e4m3fn", "uint8", "int8"),
                  some("float8_e8m0fnu", "uint8", "int8"), torch.int32, torch.int64, torch.float32)
    return _types


def _ws(workspace):
    if workspace is None:
        return None, 0
    return workspace.data_ptr(), workspace.nbytes


def paged_decode_attention(q, k_blocks, v_blocks, block_tables, context_lens, scale, out, shape: DecodeShape,
                           workspace=None, k_scale=None, v_scale=None, stream=None) -> None:
    """Enqueue the decode on `stream` (default: torch's current stream).  All tensors are
    device tensors laid out as include/dpool.h documents; nothing is copied or converted.
    The workspace must have been zero-filled before its first use."""
    ws_ptr, ws_bytes = _ws(workspace)
    check(lib().paged_decode_attention(
        q.data_ptr(), k_blocks.data_ptr(), v_blocks.data_ptr(), block_tables.data_ptr(), context_lens.data_ptr(),
        float(scale), k_scale.data_ptr() if k_scale is not None else None,
        v_scale.data_ptr() if v_scale is not None else None, out.data_ptr(), ctypes.byref(shape), ws_ptr, ws_bytes,
        _stream_ptr(stream)))


def paged_decode_attention_noalloc(q, k_blocks, v_blocks, block_tables, context_lens, scale, out,
                                   shape: DecodeShape, k_scale=None, v_scale=None, stream=None) -> None:
    """Enqueue the decode without a workspace (the library's fixed per-GPU scratch;
    include/dpool.h, paged_decode_attention_noalloc)."""
    check(lib().paged_decode_attention_noalloc(
        q.data_ptr(), k_blocks.data_ptr(), v_blocks.data_ptr(), block_tables.data_ptr(), context_lens.data_ptr(),
        float(scale), k_scale.data_ptr() if k_scale is not None else None,
        v_scale.data_ptr() if v_scale is not None else None, out.data_ptr(), ctypes.byref(shape),
        _stream_ptr(stream)))


def window_workspace_size(shape: DecodeShape, window, n_sink=0) -> int:
    return int(lib().window_decode_workspace_size(ctypes.byref(shape), window, n_sink))


def _check_window(q, k_blocks, v_blocks, block_tables, lens, out, shape, rows, k_scale, v_scale, more=None,
                  more_dtype=None) -> int:
    """Refuses tensors with gaps, of other types than the shape's, with fewer elements than it asks for, or apart.
    more: the workspace, or the row offsets (of more_dtype).  Returns the tensors' device."""
    # (written out: half of what a loop takes on the host)
    if not (q.is_contiguous() and k_blocks.is_contiguous() and v_blocks.is_contiguous() and block_tables.is_contiguous()
            and lens.is_contiguous() and out.is_contiguous()):
        raise ValueError("q, caches, block tables, lengths and out must be contiguous")
    bf16, codes, exponents, int32, _, float32 = _element_types()
    kv, batch, heads = shape.kv_dtype, shape.batch, shape.n_kv_heads
    cache = codes if kv else bf16
    if q.dtype not in bf16 or k_blocks.dtype not in cache or v_blocks.dtype not in cache:
        raise ValueError(f"q is bf16 and the caches are {'e4m3' if kv else 'bf16'}, not {q.dtype}, {k_blocks.dtype} and "
                         f"{v_blocks.dtype}")
    if block_tables.dtype is not int32 or lens.dtype is not int32:
        raise ValueError("block tables and lengths are int32")
    if out.dtype is not float32 if shape.out_dtype else out.dtype not in bf16:
        raise ValueError(f"out is {'fp32' if shape.out_dtype else 'bf16'}, not {out.dtype}")
    tiles = shape.num_blocks * heads
    size, width = tiles * 2048, rows * shape.n_q_heads * 128  # (a tile: 16 tokens of 128 dimensions)
    if (q.numel() < width or out.numel() < width or k_blocks.numel() < size or v_blocks.numel() < size
            or block_tables.numel() < batch * shape.max_blocks_per_seq or lens.numel() < batch):
        raise ValueError("q, caches, block tables, lengths or out have fewer elements than the shape")
    dev = q.get_device()
    here = (dev >= 0 and k_blocks.get_device() == dev and v_blocks.get_device() == dev
            and block_tables.get_device() == dev and lens.get_device() == dev and out.get_device() == dev)
    if k_scale is not None and v_scale is not None:
        if (k_scale.dtype not in exponents or v_scale.dtype not in exponents) if kv == KV_FP8_E4M3_BLOCK else (
                k_scale.dtype is not float32 or v_scale.dtype is not float32):
            raise ValueError("scales are fp32 for each head, or one exponent byte for each block and head")
        if not (k_scale.is_contiguous() and v_scale.is_contiguous()):
            raise ValueError("scales must be contiguous")
        size = tiles if kv == KV_FP8_E4M3_BLOCK else heads
        if k_scale.numel() < size or v_scale.numel() < size:
            raise ValueError(f"scales have {k_scale.numel()} and {v_scale.numel()} elements, the shape asks for {size}")
        here = here and k_scale.get_device() == dev and v_scale.get_device() == dev
    if more is not None:
        if more_dtype is not None and (more.dtype is not more_dtype or more.numel() <= batch):
            raise ValueError("q_start is int32 and has an element more than the batch")
        if not more.is_contiguous():
            raise ValueError("workspace and q_start must be contiguous")
        here = here and more.get_device() == dev
    if not here:
        raise ValueError("tensors must all be on the current device")
    return dev


def window_decode_attention(q, k_blocks, v_blocks, block_tables, context_lens, scale, window, n_sink, out,
                            shape: DecodeShape, workspace=None, k_scale=None, v_scale=None, stream=None) -> None:
    """Enqueue the decode over a sliding window and the first n_sink tokens, or over block scales
    (include/dpool.h, window_decode_attention).  Tensors, the workspace among them, have to be contiguous, of the
    shape's element types (or integers of their size, for bf16, e4m3 and exponents), at least as large as it says and
    on the current device (ValueError otherwise)."""
    dev = _check_window(q, k_blocks, v_blocks, block_tables, context_lens, out, shape, shape.batch, k_scale, v_scale,
                        workspace)
    ws_ptr, ws_bytes = _ws(workspace)
    check(lib().window_decode_attention(
        q.data_ptr(), k_blocks.data_ptr(), v_blocks.data_ptr(), block_tables.data_ptr(), context_lens.data_ptr(),
        float(scale), window, n_sink, k_scale.data_ptr() if k_scale is not None else None,
        v_scale.data_ptr() if v_scale is not None else None, out.data_ptr(), ctypes.byref(shape), ws_ptr, ws_bytes,
        _stream_here(stream, dev)))


def kv_cache_append(k_new, v_new, k_blocks, v_blocks, block_tables, positions, shape: DecodeShape, k_scale=None,
                    v_scale=None, stream=None) -> None:
    """Enqueue the append of one token per sequence (include/dpool.h, kv_cache_append)."""
    check(lib().kv_cache_append(
        k_new.data_ptr(), v_new.data_ptr(), k_blocks.data_ptr(), v_blocks.data_ptr(), block_tables.data_ptr(),
        positions.data_ptr(), k_scale.data_ptr() if k_scale is not None else None,
        v_scale.data_ptr() if v_scale is not None else None, ctypes.byref(shape), _stream_ptr(stream)))


def prefill_shape(batch, n_q_heads, n_kv_heads, max_blocks_per_seq, max_context_len, num_blocks, total_q,
                  kv_fp8=False, out_fp32=False, query_tile=0, head_dim=128, block_size=16,
                  block_scales=False) -> PrefillShape:
    """block_scales: an e4m3 cache with a scale for each block and head (window_prefill_attention)."""
    return PrefillShape(batch, n_q_heads, n_kv_heads, head_dim, block_size, max_blocks_per_seq, max_context_len,
                        _kv_dtype(kv_fp8, block_scales), OUT_FP32 if out_fp32 else OUT_BF16, query_tile, 0,
                        total_q, num_blocks)


def chunked_prefill_attention(q, k_blocks, v_blocks, block_tables, context_lens, q_start, scale, out,
                              shape: PrefillShape, k_scale=None, v_scale=None, stream=None) -> None:
    """Enqueue the chunked-prefill attention (include/dpool.h, chunked_prefill_attention)."""
    check(lib().chunked_prefill_attention(
        q.data_ptr(), k_blocks.data_ptr(), v_blocks.data_ptr(), block_tables.data_ptr(), context_lens.data_ptr(),
        q_start.data_ptr(), float(scale), k_scale.data_ptr() if k_scale is not None else None,
        v_scale.data_ptr() if v_scale is not None else None, out.data_ptr(), ctypes.byref(shape),
        _stream_ptr(stream)))


def window_prefill_attention(q, k_blocks, v_blocks, block_tables, context_lens, q_start, scale, window, n_sink, out,
                             shape: PrefillShape, k_scale=None, v_scale=None, stream=None) -> None:
    """Enqueue the chunked prefill over a sliding window and the first n_sink tokens, or over block scales
    (include/dpool.h, window_prefill_attention).  Tensors have to be contiguous, of the shape's element types (or
    integers of their size, for bf16, e4m3 and exponents), at least as large as it says and on the current device
    (ValueError otherwise)."""
    dev = _check_window(q, k_blocks, v_blocks, block_tables, context_lens, out, shape, shape.total_q, k_scale, v_scale,
                        q_start, _element_types()[3])
    check(lib().window_prefill_attention(
        q.data_ptr(), k_blocks.data_ptr(), v_blocks.data_ptr(), block_tables.data_ptr(), context_lens.data_ptr(),
        q_start.data_ptr(), float(scale), window, n_sink, k_scale.data_ptr() if k_scale is not None else None,
        v_scale.data_ptr() if v_scale is not None else None, out.data_ptr(), ctypes.byref(shape),
        _stream_here(stream, dev)))


# ---------------------------------------------------------------- a step that verifies drafted tokens

def tables_shape(batch, max_blocks_per_seq, num_blocks, total_rows, mask_words=0, block_size=16) -> TablesShape:
    return TablesShape(batch, block_size, max_blocks_per_seq, mask_words, total_rows, num_blocks, 0)


def kv_tables_step(context_lens, n_owned, new_tokens, free_ids, free_state, block_tables, context_lens_out,
                   n_owned_out, free_state_out, q_start, slots, positions, granted, shape: TablesShape, parents=None,
                   tree_mask=None, stream=None) -> None:
    """Enqueue one step of the block tables (include/dpool.h, kv_tables_step); new_tokens -1 ends a sequence, -2 one
    whose entries below 0 hold no block."""
    check(lib().kv_tables_step(
        context_lens.data_ptr(), n_owned.data_ptr(), new_tokens.data_ptr(),
        parents.data_ptr() if parents is not None else None, free_ids.data_ptr(), free_state.data_ptr(),
        block_tables.data_ptr(), context_lens_out.data_ptr(), n_owned_out.data_ptr(), free_state_out.data_ptr(),
        q_start.data_ptr(), slots.data_ptr(), positions.data_ptr(), granted.data_ptr(),
        tree_mask.data_ptr() if tree_mask is not None else None, ctypes.byref(shape), _stream_ptr(stream)))


def qk_shape(rows, n_q_heads, n_kv_heads, num_blocks, n_positions, rotary_dim=128, interleaved=False, kv_fp8=False,
             q_stride=None, k_stride=None, v_stride=None, head_dim=128, block_size=16,
             block_scales=False) -> QKShape:
    """Strides in elements from one row to the next; None: rows lie next to each other.
    block_scales: the shape is one of qk_norm_rope_append_scaled."""
    return QKShape(n_q_heads, n_kv_heads, head_dim, block_size, _kv_dtype(kv_fp8, block_scales), rotary_dim,
                   int(interleaved), 0, rows, num_blocks, n_positions,
                   n_q_heads * head_dim if q_stride is None else q_stride,
                   n_kv_heads * head_dim if k_stride is None else k_stride,
                   n_kv_heads * head_dim if v_stride is None else v_stride)


def _check_rows(name, t, n, heads, head_dim, stride) -> None:
    """Refuses a tensor whose n rows of heads * head_dim values do not lie `stride` elements apart."""
    if t.numel() == 0:
        return
    width, inner, rows = heads * head_dim, 1, 1
    for size, step in zip(reversed(t.shape), reversed(t.stride())):
        if inner >= width and rows >= n:  # (further rows are not read, whatever lies between them)
            return
        if size != 1 and step != (inner if inner < width else stride * rows):
            raise ValueError(f"{name} has strides {tuple(t.stride())}, the shape's rows of {width} lie {stride} apart")
        if inner < width:
            inner *= size
        else:
            rows *= size


def _check_qkv(q, k, v, q_out, shape) -> None:
    qs, ks, vs = shape.q_stride, shape.k_stride, shape.v_stride
    # ([rows, heads, 128] is compared first, all three at once: 0.5 us of the host)
    if (q.stride(), k.stride(), v.stride()) != ((qs, 128, 1), (ks, 128, 1), (vs, 128, 1)):
        _check_rows("q", q, shape.rows, shape.n_q_heads, shape.head_dim, qs)
        _check_rows("k", k, shape.rows, shape.n_kv_heads, shape.head_dim, ks)
        _check_rows("v", v, shape.rows, shape.n_kv_heads, shape.head_dim, vs)
    if not q_out.is_contiguous():
        raise ValueError("q_out must be contiguous")


def qk_norm_rope_append(q, k, v, cos_sin, positions, slots, q_out, k_blocks, v_blocks, shape: QKShape, q_weight=None,
                        k_weight=None, eps=1e-6, k_scale=None, v_scale=None, stream=None) -> None:
    """Enqueue norm, rotation and cache write of the new tokens (include/dpool.h, qk_norm_rope_append).

    The rows of q, k and v have to lie as far apart as the shape says, q_out
    has to be contiguous (ValueError otherwise)."""
    _check_qkv(q, k, v, q_out, shape)
    check(lib().qk_norm_rope_append(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), q_weight.data_ptr() if q_weight is not None else None,
        k_weight.data_ptr() if k_weight is not None else None, float(eps),
        cos_sin.data_ptr() if cos_sin is not None else None, positions.data_ptr(), slots.data_ptr(),
        q_out.data_ptr(), k_blocks.data_ptr(), v_blocks.data_ptr(),
        k_scale.data_ptr() if k_scale is not None else None, v_scale.data_ptr() if v_scale is not None else None,
        ctypes.byref(shape), _stream_ptr(stream)))


def qk_norm_rope_append_scaled(q, k, v, cos_sin, positions, slots, q_out, k_blocks, v_blocks, k_scale, v_scale,
                               shape: QKShape, q_weight=None, k_weight=None, eps=1e-6, stream=None) -> None:
    """Enqueue norm, rotation and the write into a cache with block scales (include/dpool.h,
    qk_norm_rope_append_scaled); k_scale and v_scale, one byte each, are updated with it.

    q and q_out may be None where the shape has no query heads.  Rows as for
    qk_norm_rope_append; all other tensors have to be contiguous.  Element types
    as the names say, or integers of their size for bf16, e4m3 and exponents
    (int32 positions, int64 slots, fp32 cos_sin); at least as many elements as
    the shape asks for; all on the current device (ValueError)."""
    rows, cells = shape.rows, shape.num_blocks * shape.n_kv_heads
    width, size = rows * shape.n_kv_heads * 128, cells * 2048  # (a tile: 16 tokens of 128 dimensions)
    bf16, codes, exponents, int32, int64, float32 = _element_types()
    dev = k.get_device()
    here = dev >= 0
    if q is None:
        _check_rows("k", k, rows, shape.n_kv_heads, shape.head_dim, shape.k_stride)
        _check_rows("v", v, rows, shape.n_kv_heads, shape.head_dim, shape.v_stride)
    else:
        if q_out is None:
            raise ValueError("q_out is missing")
        _check_qkv(q, k, v, q_out, shape)
        q_width = rows * shape.n_q_heads * 128
        if q.dtype not in bf16 or q_out.dtype not in bf16:
            raise ValueError("q and q_out are bf16")
        if q.numel() < q_width or q_out.numel() < q_width:
            raise ValueError("q or q_out has fewer elements than the shape")
        here = here and q.get_device() == dev and q_out.get_device() == dev
    if not (k_blocks.is_contiguous() and v_blocks.is_contiguous() and k_scale.is_contiguous()
            and v_scale.is_contiguous() and positions.is_contiguous() and slots.is_contiguous()):
        raise ValueError("caches, scales, positions and slots must be contiguous")
    if k.dtype not in bf16 or v.dtype not in bf16 or k_blocks.dtype not in codes or v_blocks.dtype not in codes:
        raise ValueError("k and v are bf16, the caches e4m3")
    if k_scale.dtype not in exponents or v_scale.dtype not in exponents:
        raise ValueError("k_scale and v_scale hold one exponent byte for each block and head")
    if positions.dtype is not int32 or slots.dtype is not int64:
        raise ValueError("positions are int32, slots int64")
    if (k.numel() < width or v.numel() < width or k_blocks.numel() < size or v_blocks.numel() < size
            or k_scale.numel() < cells or v_scale.numel() < cells or positions.numel() < rows or slots.numel() < rows):
        raise ValueError("k, v, caches, scales, positions or slots have fewer elements than the shape")
    here = (here and v.get_device() == dev and k_blocks.get_device() == dev and v_blocks.get_device() == dev
            and k_scale.get_device() == dev and v_scale.get_device() == dev and positions.get_device() == dev
            and slots.get_device() == dev)
    if cos_sin is not None:
        if (cos_sin.dtype is not float32 or not cos_sin.is_contiguous()
                or cos_sin.numel() < shape.n_positions * shape.rotary_dim):
            raise ValueError("cos_sin is fp32, contiguous and has a row for each position")
        here = here and cos_sin.get_device() == dev
    for w in (q_weight, k_weight):
        if w is not None:
            if w.dtype not in bf16 or not w.is_contiguous() or w.numel() < 128:
                raise ValueError("q_weight and k_weight are bf16, contiguous and have 128 elements")
            here = here and w.get_device() == dev
    if not here:
        raise ValueError("tensors must all be on the current device")
    check(lib().qk_norm_rope_append_scaled(
        q.data_ptr() if q is not None else None, k.data_ptr(), v.data_ptr(),
        q_weight.data_ptr() if q_weight is not None else None, k_weight.data_ptr() if k_weight is not None else None,
        float(eps), cos_sin.data_ptr() if cos_sin is not None else None, positions.data_ptr(), slots.data_ptr(),
        q_out.data_ptr() if q_out is not None else None, k_blocks.data_ptr(), v_blocks.data_ptr(), k_scale.data_ptr(),
        v_scale.data_ptr(), ctypes.byref(shape), _stream_here(stream, dev)))


def tree_shape(batch, n_q_heads, n_kv_heads, max_blocks_per_seq, max_context_len, num_blocks, total_q, mask_words=1,
               kv_fp8=False, head_dim=128, block_size=16) -> TreeShape:
    return TreeShape(batch, n_q_heads, n_kv_heads, head_dim, block_size, max_blocks_per_seq, max_context_len,
                     KV_FP8_E4M3 if kv_fp8 else KV_BF16, mask_words, 0, total_q, num_blocks)


def tree_workspace_size(shape: TreeShape) -> int:
    return int(lib().tree_decode_workspace_size(ctypes.byref(shape)))


def tree_decode_attention(q, k_blocks, v_blocks, block_tables, context_lens, q_start, tree_mask, scale, out,
                          shape: TreeShape, workspace, k_scale=None, v_scale=None, stream=None) -> None:
    """Enqueue the attention of drafted trees (include/dpool.h, tree_decode_attention)."""
    ws_ptr, ws_bytes = _ws(workspace)
    check(lib().tree_decode_attention(
        q.data_ptr(), k_blocks.data_ptr(), v_blocks.data_ptr(), block_tables.data_ptr(), context_lens.data_ptr(),
        q_start.data_ptr(), tree_mask.data_ptr(), float(scale), k_scale.data_ptr() if k_scale is not None else None,
        v_scale.data_ptr() if v_scale is not None else None, out.data_ptr(), ctypes.byref(shape), ws_ptr, ws_bytes,
        _stream_ptr(stream)))


class CacheLayers:
    """The K and V caches of several layers, as kv_cache_accept takes them (keeps the tensors alive)."""

    def __init__(self, k_layers, v_layers):
        if len(k_layers) != len(v_layers):
            raise ValueError("as many K as V caches")
        if not all(t.is_contiguous() for t in (*k_layers, *v_layers)):
            raise ValueError("caches must be contiguous")
        self.tensors = (list(k_layers), list(v_layers))
        self.n = len(k_layers)
        self.k, self.v = ((ctypes.c_void_p * self.n)(*[t.data_ptr() for t in ts]) for ts in self.tensors)


def kv_cache_accept(layers: CacheLayers, block_tables, context_lens, q_start, accepted, n_accepted, context_lens_out,
                    shape: TreeShape, stream=None) -> None:
    """Enqueue the move of the accepted drafts, accepted [batch, max_accept] (include/dpool.h, kv_cache_accept)."""
    if accepted.dim() != 2 or not accepted.is_contiguous():
        raise ValueError("accepted must be a contiguous [batch, max_accept] tensor")
    check(lib().kv_cache_accept(
        layers.k, layers.v, layers.n, block_tables.data_ptr(), context_lens.data_ptr(), q_start.data_ptr(),
        accepted.data_ptr(), n_accepted.data_ptr(), accepted.shape[1], context_lens_out.data_ptr(),
        ctypes.byref(shape), _stream_ptr(stream)))


def hbm_read_probe(buf, workgroups, sink, tile_ids=None, stream=None) -> None:
    """Enqueue one read of `buf` (contiguous, or its 4 KiB tiles in `tile_ids` order)."""
    nbytes = buf.numel() * buf.element_size()
    check(lib().dp_hbm_read_probe(buf.data_ptr(), nbytes, tile_ids.data_ptr() if tile_ids is not None else None,
                                  tile_ids.numel() if tile_ids is not None else 0, int(workgroups), sink.data_ptr(),
                                  sink.numel() * sink.element_size(), _stream_ptr(stream)))


class PagedDecoder:
    """Holds one decode shape and its workspace; calling it enqueues the decode.

    Device memory for the workspace comes from torch's allocator once, at
    construction, zero-filled as the library requires; each call only marshals
    pointers into paged_decode_attention.
    """

    def __init__(self, batch, n_q_heads, n_kv_heads, max_blocks_per_seq, max_context_len, num_blocks,
                 kv_fp8=False, out_fp32=False, partition_tokens=0, workgroups_per_cu=0, device="cuda"):
        import torch
        self.shape = decode_shape(batch, n_q_heads, n_kv_heads, max_blocks_per_seq, max_context_len, num_blocks,
                                  kv_fp8, out_fp32, partition_tokens, workgroups_per_cu)
        self.partition_tokens = _partition_tokens(self.shape)
        if self.partition_tokens <= 0:
            raise DpoolError(DP_EINVAL, last_error())
        ws = workspace_size(self.shape)
        self.workspace = torch.zeros(ws, dtype=torch.uint8, device=device) if ws else None
        self.out_dtype = torch.float32 if out_fp32 else torch.bfloat16

    def new_out(self, device="cuda"):
        import torch
        s = self.shape
        return torch.empty((s.batch, s.n_q_heads, s.head_dim), dtype=self.out_dtype, device=device)

    def __call__(self, q, k_blocks, v_blocks, block_tables, context_lens, scale, out, k_scale=None, v_scale=None,
                 stream=None):
        paged_decode_attention(q, k_blocks, v_blocks, block_tables, context_lens, scale, out, self.shape,
                               self.workspace, k_scale, v_scale, stream)
        return out


class WindowDecoder:
    """Holds one decode shape with its window and its workspace; calling it enqueues the decode.

    window, n_sink: the query sees the `window` tokens up to its own, and the
    first n_sink; None: the whole context.  block_scales: the e4m3 cache has a
    scale for each block and head.  Device memory for the workspace comes from
    torch's allocator once, at construction, zero-filled as the library requires.
    """

    def __init__(self, batch, n_q_heads, n_kv_heads, max_blocks_per_seq, max_context_len, num_blocks, window=None,
                 n_sink=0, kv_fp8=False, block_scales=False, out_fp32=False, partition_tokens=0, workgroups_per_cu=0,
                 device="cuda"):
        import torch
        self.shape = decode_shape(batch, n_q_heads, n_kv_heads, max_blocks_per_seq, max_context_len, num_blocks,
                                  kv_fp8, out_fp32, partition_tokens, workgroups_per_cu, block_scales=block_scales)
        self.window = max(max_context_len, 1) if window is None else window
        self.n_sink = n_sink
        ws = window_workspace_size(self.shape, self.window, n_sink)
        if ws == 0:
            raise DpoolError(DP_EINVAL, last_error())
        self.workspace = torch.zeros(ws, dtype=torch.uint8, device=device)
        self.out_dtype = torch.float32 if out_fp32 else torch.bfloat16

    def new_out(self, device="cuda"):
        import torch
        s = self.shape
        return torch.empty((s.batch, s.n_q_heads, s.head_dim), dtype=self.out_dtype, device=device)

    def __call__(self, q, k_blocks, v_blocks, block_tables, context_lens, scale, out, k_scale=None, v_scale=None,
                 stream=None):
        window_decode_attention(q, k_blocks, v_blocks, block_tables, context_lens, scale, self.window, self.n_sink,
                                out, self.shape, self.workspace, k_scale, v_scale, stream)
        return out


class TreeDecoder:
    """Holds one tree-attention shape and its workspace; calling it enqueues the attention.

    Device memory for the workspace comes from torch's allocator once, at
    construction; each call only marshals pointers into tree_decode_attention.
    """

    def __init__(self, batch, n_q_heads, n_kv_heads, max_blocks_per_seq, max_context_len, num_blocks, total_q,
                 mask_words=1, kv_fp8=False, device="cuda"):
        import torch
        self.shape = tree_shape(batch, n_q_heads, n_kv_heads, max_blocks_per_seq, max_context_len, num_blocks,
                                total_q, mask_words, kv_fp8)
        ws = tree_workspace_size(self.shape)
        if ws == 0:
            raise DpoolError(DP_EINVAL, last_error())
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=device)

    def new_out(self, device="cuda"):
        import torch
        s = self.shape
        return torch.empty((s.total_q, s.n_q_heads, s.head_dim), dtype=torch.bfloat16, device=device)

    def __call__(self, q, k_blocks, v_blocks, block_tables, context_lens, q_start, tree_mask, scale, out, k_scale=None,
                 v_scale=None, stream=None):
        tree_decode_attention(q, k_blocks, v_blocks, block_tables, context_lens, q_start, tree_mask, scale, out,
                              self.shape, self.workspace, k_scale, v_scale, stream)
        return out
