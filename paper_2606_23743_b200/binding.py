"""Thin ctypes binding over the C ABI declared in include/sva.h.

Argument marshalling only: every step of the path runs in the CUDA kernels.  torch is used
for device memory and streams.  There is no CPU fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libsva.so")
_lib = None

SVA_OK = 0
SVA_BF16, SVA_FP8_E4M3 = 0, 1
SVA_DEV_BAD_INDEX, SVA_DEV_TIMEOUT, SVA_DEV_NO_PAGES = 1, 2, 4

EXPORTS = [
    "sva_select_max_nnz", "sva_select_workspace_bytes", "sva_block_select",
    "sva_block_sparse_attn_fwd", "sva_dense_attn_fwd", "sva_block_sparse_attn_fwd_simt",
    "sva_quantize_qk_fp8", "sva_status_string", "sva_block_select_noalloc", "sva_attn_workspace_bytes",
    "sva_attn_prepare_v", "sva_block_sparse_attn_fwd_prepared", "sva_gather_tokens", "sva_scatter_tokens",
    "sva_attn_one_call_workspace_bytes", "sva_quantize_qk_fp4", "sva_block_sparse_attn_fwd_fp4", "sva_attn_remainder_workspace_bytes", "sva_block_sparse_attn_remainder_fwd", "sva_smooth_workspace_bytes", "sva_quantize_qk_fp8_smooth_k", "sva_block_select_pooled", "sva_qk_norm_rope_pool", "sva_pool_qk",
    "sva_quantize_rows_fp8", "sva_quantize_tiles_fp8", "sva_linear_fp8", "sva_rope", "sva_rope_steps", "sva_kv_cache_write",
    "sva_kv_cache_read", "sva_kv_cache_append", "sva_cached_attn_workspace_bytes", "sva_cached_attn_fwd", "sva_cross_attn_workspace_bytes",
    "sva_cross_attn_fwd", "sva_kv_pages_copy", "sva_kv_pages_take", "sva_kv_pages_fork", "sva_kv_pages_free",
    "sva_kv_pages_compact_workspace_bytes", "sva_kv_pages_compact",
]
DEBUG_EXPORTS = ["sva_debug_set_prof_buffer", "sva_debug_set_mode", "sva_debug_set_wait_limit", "sva_debug_last_choice"]
NOALLOC_SCRATCH_BYTES = 16 << 20


class Problem(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("N", C.c_int32), ("d", C.c_int32),
                ("block", C.c_int32),
                ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3),
                ("v_stride", C.c_int64 * 3), ("o_stride", C.c_int64 * 3),
                ("softmax_scale", C.c_float), ("qk_dtype", C.c_int32)]


class Select(C.Structure):
    _fields_ = [("mode", C.c_int32), ("k", C.c_int32), ("mass", C.c_float),
                ("win_t", C.c_int32), ("win_s", C.c_int32), ("blocks_per_frame", C.c_int32)]


class Linear(C.Structure):
    _fields_ = [("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32), ("act", C.c_int32),
                ("x_stride", C.c_int64), ("w_stride", C.c_int64), ("out_stride", C.c_int64), ("residual_stride", C.c_int64),
                ("x8_stride", C.c_int64), ("w8_stride", C.c_int64), ("x_scale_stride", C.c_int64), ("w_scale_stride", C.c_int64)]
    # bytes of the three calls' tensors (make_linear, if they are on the GPU)
    rows = tiles = (float("inf"),) * 3
    product = (float("inf"),) * 7
    gaps = {}


class Rope(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hk", C.c_int32), ("N", C.c_int32), ("d", C.c_int32),
                ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("axis_pairs", C.c_int32 * 3), ("inverse", C.c_int32),
                ("factor", C.c_float), ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3),
                ("q_out_stride", C.c_int64 * 3), ("k_out_stride", C.c_int64 * 3), ("pos_stride", C.c_int64 * 2)]
    sizes = (float("inf"),) * 5                            # bytes of the call's tensors (make_rope, if they are on the GPU)
    gaps = {}


class KvCache(C.Structure):
    _fields_ = [("H", C.c_int32), ("d", C.c_int32), ("page", C.c_int32), ("pages", C.c_int32), ("format", C.c_int32),
                ("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("k_sf", C.c_void_p), ("v_sf", C.c_void_p)]
    # the tensors behind the pointers, whether they are on the GPU, on which (-1: none, or on several), and (H, d) (make_kv_cache)
    arrays, on_gpu, device, heads = None, False, -1, None


class CachedAttn(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("M", C.c_int32), ("max_pages", C.c_int32), ("causal", C.c_int32), ("softmax_scale", C.c_float),
                ("table_stride", C.c_int64), ("q_stride", C.c_int64 * 3), ("o_stride", C.c_int64 * 3)]
    # the cache that it was made for, q's shape, q's, o's and the table's strides (make_cached_attn)
    cache = shape = strides = table = None


class CrossAttn(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hk", C.c_int32), ("N", C.c_int32), ("S", C.c_int32), ("d", C.c_int32),
                ("softmax_scale", C.c_float), ("mask_stride", C.c_int64), ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3),
                ("v_stride", C.c_int64 * 3), ("o_stride", C.c_int64 * 3)]
    shapes = strides = None                                # of q, k, v, o (make_cross_attn)


class SvaError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: status {status} ({status_string(status)})")


def lib():
    """Loads libsva.so (built in-tree by paper_2606_23743_b200.build). Raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: run `python -m paper_2606_23743_b200.build` "
                               "(there is no fallback path)")
        L = C.CDLL(_LIB_PATH)
        vp = C.c_void_p
        L.sva_select_max_nnz.restype = C.c_int64
        L.sva_select_max_nnz.argtypes = [C.POINTER(Problem), C.POINTER(Select)]
        L.sva_select_workspace_bytes.restype = C.c_size_t
        L.sva_select_workspace_bytes.argtypes = [C.POINTER(Problem), C.POINTER(Select)]
        L.sva_block_select.restype = C.c_int
        L.sva_block_select.argtypes = [C.POINTER(Problem), C.POINTER(Select), vp, vp, vp, vp, vp, vp,
                                       vp, vp, C.c_size_t, vp]
        L.sva_block_select_noalloc.restype = C.c_int
        L.sva_block_select_noalloc.argtypes = [C.POINTER(Problem), C.POINTER(Select), vp, vp, vp, vp, vp, vp,
                                               vp, vp]
        L.sva_attn_one_call_workspace_bytes.restype = C.c_size_t
        L.sva_attn_one_call_workspace_bytes.argtypes = [C.POINTER(Problem)]
        L.sva_attn_workspace_bytes.restype = C.c_size_t
        L.sva_attn_workspace_bytes.argtypes = [C.POINTER(Problem)]
        L.sva_block_sparse_attn_fwd.restype = C.c_int
        L.sva_block_sparse_attn_fwd.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                                C.c_size_t, vp]
        L.sva_block_sparse_attn_fwd_simt.restype = C.c_int
        L.sva_block_sparse_attn_fwd_simt.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.sva_dense_attn_fwd.restype = C.c_int
        L.sva_dense_attn_fwd.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.sva_attn_remainder_workspace_bytes.restype = C.c_size_t
        L.sva_attn_remainder_workspace_bytes.argtypes = [C.POINTER(Problem), C.c_int32]
        L.sva_block_sparse_attn_remainder_fwd.restype = C.c_int
        L.sva_block_sparse_attn_remainder_fwd.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_int32, vp,
                                                          C.c_size_t, vp]
        L.sva_attn_prepare_v.restype = C.c_int
        L.sva_attn_prepare_v.argtypes = [C.POINTER(Problem), vp, vp, C.c_size_t, vp]
        L.sva_block_sparse_attn_fwd_prepared.restype = C.c_int
        L.sva_block_sparse_attn_fwd_prepared.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        for fn in (L.sva_gather_tokens, L.sva_scatter_tokens):
            fn.restype = C.c_int
            fn.argtypes = [vp, C.POINTER(C.c_int64), vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                           C.c_int32, vp, C.POINTER(C.c_int64), vp, vp]
        L.sva_quantize_qk_fp8.restype = C.c_int
        L.sva_quantize_qk_fp8.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, vp]
        L.sva_quantize_qk_fp4.restype = C.c_int
        L.sva_quantize_qk_fp4.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.sva_block_sparse_attn_fwd_fp4.restype = C.c_int
        L.sva_block_sparse_attn_fwd_fp4.argtypes = [C.POINTER(Problem)] + [vp] * 13 + [C.c_size_t, vp]
        L.sva_smooth_workspace_bytes.restype = C.c_size_t
        L.sva_smooth_workspace_bytes.argtypes = [C.POINTER(Problem)]
        L.sva_quantize_qk_fp8_smooth_k.restype = C.c_int
        L.sva_quantize_qk_fp8_smooth_k.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.sva_pool_qk.restype = C.c_int
        L.sva_pool_qk.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, vp]
        L.sva_block_select_pooled.restype = C.c_int
        L.sva_block_select_pooled.argtypes = [C.POINTER(Problem), C.POINTER(Select), vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.sva_qk_norm_rope_pool.restype = C.c_int
        L.sva_qk_norm_rope_pool.argtypes = [C.POINTER(Problem), vp, vp, vp, vp, vp, vp, C.c_float, vp, vp, vp, vp, vp, vp,
                                            vp, vp, vp]
        L.sva_quantize_rows_fp8.restype = C.c_int
        L.sva_quantize_rows_fp8.argtypes = [C.POINTER(Linear), vp, vp, vp, vp]
        L.sva_quantize_tiles_fp8.restype = C.c_int
        L.sva_quantize_tiles_fp8.argtypes = [C.POINTER(Linear), vp, vp, vp, vp]
        L.sva_linear_fp8.restype = C.c_int
        L.sva_linear_fp8.argtypes = [C.POINTER(Linear), vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.sva_rope.restype = C.c_int
        L.sva_rope.argtypes = [C.POINTER(Rope), vp, vp, vp, vp, vp, vp, vp]
        L.sva_rope_steps.restype = C.c_int
        L.sva_rope_steps.argtypes = [C.c_int32, C.POINTER(C.c_int32), C.c_double, C.c_int32, C.c_double, C.c_double, C.c_double,
                                     C.c_double, C.POINTER(C.c_uint64), C.POINTER(C.c_float)]
        i64p = C.POINTER(C.c_int64)
        L.sva_kv_cache_write.restype = C.c_int
        L.sva_kv_cache_write.argtypes = [C.POINTER(KvCache), vp, vp, i64p, i64p, C.c_int32, C.c_int32, vp, vp, vp]
        L.sva_kv_cache_read.restype = C.c_int
        L.sva_kv_cache_read.argtypes = [C.POINTER(KvCache), vp, C.c_int64, C.c_int32, vp, C.c_int32, C.c_int32, vp, vp, i64p, i64p,
                                        vp, vp]
        cache, i32, i64 = C.POINTER(KvCache), C.c_int32, C.c_int64
        L.sva_kv_cache_append.restype = C.c_int
        L.sva_kv_cache_append.argtypes = [cache, vp, vp, i64p, i64p, i32, i32, vp, i64, i32, vp, vp, vp, vp]
        L.sva_cached_attn_workspace_bytes.restype = C.c_size_t
        L.sva_cached_attn_workspace_bytes.argtypes = [cache, C.POINTER(CachedAttn)]
        L.sva_cached_attn_fwd.restype = C.c_int
        L.sva_cached_attn_fwd.argtypes = [cache, C.POINTER(CachedAttn)] + [vp] * 8 + [C.c_size_t, vp]
        L.sva_cross_attn_workspace_bytes.restype = C.c_size_t
        L.sva_cross_attn_workspace_bytes.argtypes = [C.POINTER(CrossAttn)]
        L.sva_cross_attn_fwd.restype = C.c_int
        L.sva_cross_attn_fwd.argtypes = [C.POINTER(CrossAttn)] + [vp] * 9 + [C.c_size_t, vp]
        L.sva_kv_pages_copy.restype = C.c_int
        L.sva_kv_pages_copy.argtypes = [cache, vp, vp, i32, vp, vp]
        L.sva_kv_pages_take.restype = C.c_int
        L.sva_kv_pages_take.argtypes = [cache, vp, vp, i64, i32, i32, vp, vp, vp, vp]
        for fn in (L.sva_kv_pages_fork, L.sva_kv_pages_free):
            fn.restype = C.c_int
            fn.argtypes = [cache, vp, vp, i64, i32, i32, vp, vp, vp, i32, vp, vp]
        L.sva_kv_pages_compact_workspace_bytes.restype = C.c_size_t
        L.sva_kv_pages_compact_workspace_bytes.argtypes = [cache]
        L.sva_kv_pages_compact.restype = C.c_int
        L.sva_kv_pages_compact.argtypes = [cache, vp, vp, i64, i32, i32, vp, vp, vp, C.c_size_t, vp]
        # test and tuning aids (include/sva_debug.h): process-global settings
        L.sva_debug_set_prof_buffer.restype = None
        L.sva_debug_set_prof_buffer.argtypes = [vp]
        L.sva_debug_set_mode.restype = None
        L.sva_debug_set_mode.argtypes = [C.c_int]
        L.sva_debug_set_wait_limit.restype = C.c_int
        L.sva_debug_set_wait_limit.argtypes = [C.c_longlong]
        L.sva_debug_last_choice.restype = C.c_int
        L.sva_debug_last_choice.argtypes = []
        L.sva_status_string.restype = C.c_char_p
        L.sva_status_string.argtypes = [C.c_int]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().sva_status_string(int(status)).decode()


def _ptr(t):
    return t.data_ptr() if t is not None else None              # (the functions' argument types make it a void*)


# torch.cuda.current_stream() builds a Stream object, 2 us of the 14 us that the two calls of a small clip spend in Python; the
# shorter way is not part of torch's public interface, and a torch without it gets the public one.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream():
    """The current stream of the current device, as a pointer."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


@functools.lru_cache(maxsize=1024)
def _stride_array(s):
    assert len(s) == 4 and s[3] == 1, "tensors are [B,H,N,d] with d contiguous"
    return (C.c_int64 * 3)(*s[:3])


def _strides(t):
    """b, h, n strides as the C ABI takes them (read only: tensors of equal strides share the array)."""
    return _stride_array(t.stride())


def _strides_any(t):
    """The same for a tensor that may hold nothing (torch gives such a one any strides)."""
    s = t.stride()
    return _stride_array(s) if s[3] == 1 or t.numel() else _stride_array((0, 0, 0, 1))


def make_problem(q, k, v, o, N: int, block: int, scale: float = 0.0, fp8: bool = False) -> Problem:
    """q,k,v,o: [B,H,n_alloc,d] device tensors (d contiguous); N = valid tokens <= n_alloc."""
    B, H, _, d = q.shape
    p = Problem()
    p.B, p.H, p.N, p.d, p.block = B, H, N, d, block
    p.q_stride, p.k_stride = _strides(q), _strides(k)
    p.v_stride = _strides(v) if v is not None else _strides(q)
    p.o_stride = _strides(o) if o is not None else _strides(q)
    p.softmax_scale = scale
    p.qk_dtype = SVA_FP8_E4M3 if fp8 else SVA_BF16
    return p


def make_select(mode: int, k: int, mass: float = 1.0, win_t: int = -1, win_s: int = -1,
                blocks_per_frame: int = 0) -> Select:
    return Select(mode, k, mass, win_t, win_s, blocks_per_frame)


def select_max_nnz(p: Problem, s: Select) -> int:
    return int(lib().sva_select_max_nnz(C.byref(p), C.byref(s)))


def select_workspace_bytes(p: Problem, s: Select) -> int:
    return int(lib().sva_select_workspace_bytes(C.byref(p), C.byref(s)))


def block_select(p: Problem, s: Select, q, k, row_ptr, col_idx, workspace, q_scale=None, k_scale=None,
                 block_scores=None) -> None:
    rc = lib().sva_block_select(C.byref(p), C.byref(s), _ptr(q), _ptr(k), _ptr(q_scale), _ptr(k_scale),
                                _ptr(row_ptr), _ptr(col_idx), _ptr(block_scores), _ptr(workspace),
                                workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_block_select")


def block_select_noalloc(p: Problem, s: Select, q, k, row_ptr, col_idx, q_scale=None, k_scale=None,
                         block_scores=None) -> None:
    """sva_block_select for callers that cannot allocate: the scratch is the library's built-in
    device array (NOALLOC_SCRATCH_BYTES); raises SvaError(status 6) when the problem needs more.
    Calls share that array, so calls that could overlap on the GPU must be serialised."""
    rc = lib().sva_block_select_noalloc(C.byref(p), C.byref(s), _ptr(q), _ptr(k), _ptr(q_scale),
                                        _ptr(k_scale), _ptr(row_ptr), _ptr(col_idx), _ptr(block_scores),
                                        _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_block_select_noalloc")


def attn_workspace_bytes(p: Problem) -> int:
    return int(lib().sva_attn_workspace_bytes(C.byref(p)))


def _ws_bytes(ws):
    return ws.numel() * ws.element_size() if ws is not None else 0


def block_sparse_attn_fwd_simt(p: Problem, q, k, v, row_ptr, col_idx, o, lse=None, status=None, q_scale=None,
                               k_scale=None) -> None:
    """The diagnostic CUDA-core twin (row_ptr None = dense)."""
    rc = lib().sva_block_sparse_attn_fwd_simt(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(q_scale),
                                              _ptr(k_scale), _ptr(row_ptr), _ptr(col_idx), _ptr(o),
                                              _ptr(lse), _ptr(status), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_block_sparse_attn_fwd_simt")


def block_sparse_attn_fwd(p: Problem, q, k, v, row_ptr, col_idx, o, lse=None, status=None, q_scale=None,
                          k_scale=None, simt: bool = False, workspace=None) -> None:
    if simt:
        return block_sparse_attn_fwd_simt(p, q, k, v, row_ptr, col_idx, o, lse, status, q_scale, k_scale)
    rc = lib().sva_block_sparse_attn_fwd(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(q_scale),
                                         _ptr(k_scale), _ptr(row_ptr), _ptr(col_idx), _ptr(o), _ptr(lse),
                                         _ptr(status), _ptr(workspace), _ws_bytes(workspace), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_block_sparse_attn_fwd")


def dense_attn_fwd(p: Problem, q, k, v, o, lse=None, status=None, q_scale=None, k_scale=None,
                   workspace=None) -> None:
    rc = lib().sva_dense_attn_fwd(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(q_scale), _ptr(k_scale),
                                  _ptr(o), _ptr(lse), _ptr(status), _ptr(workspace), _ws_bytes(workspace),
                                  _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_dense_attn_fwd")


def attn_prepare_v(p: Problem, v, workspace) -> None:
    """First half of the bf16 tensor-core path: V -> tiled transposed copy in `workspace` (on the current stream)."""
    rc = lib().sva_attn_prepare_v(C.byref(p), _ptr(v), _ptr(workspace), _ws_bytes(workspace), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_attn_prepare_v")


def block_sparse_attn_fwd_prepared(p: Problem, q, k, row_ptr, col_idx, o, lse=None, status=None,
                                   workspace=None, q_scale=None, k_scale=None) -> None:
    """Second half: the attention kernel alone on a workspace that attn_prepare_v filled (row_ptr None = dense)."""
    rc = lib().sva_block_sparse_attn_fwd_prepared(C.byref(p), _ptr(q), _ptr(k), _ptr(q_scale), _ptr(k_scale),
                                                  _ptr(row_ptr), _ptr(col_idx), _ptr(o), _ptr(lse), _ptr(status),
                                                  _ptr(workspace), _ws_bytes(workspace), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_block_sparse_attn_fwd_prepared")


def _token_move(name, src, token_idx, dst, status):
    Bq, Hq, n_src, d = src.shape
    assert token_idx.dim() == 2 and token_idx.shape[0] == Bq and token_idx.dtype is torch.int32 and token_idx.is_contiguous(), "token_idx is [B,M] int32"
    M = token_idx.shape[1]
    n_full, n_part = (dst.shape[2], n_src) if name == "sva_scatter_tokens" else (n_src, dst.shape[2])
    assert n_part >= M and dst.shape[:2] == (Bq, Hq) and dst.shape[3] == d and src.dtype is dst.dtype, "src, dst are [B,H,*,d] of one type"
    rc = getattr(lib(), name)(_ptr(src), _strides(src), _ptr(token_idx), Bq, Hq, M, n_full, d, src.element_size(),
                              _ptr(dst), _strides(dst), _ptr(status), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, name)


def gather_tokens(src, token_idx, dst, status=None) -> None:
    """dst[b,h,m,:] = src[b,h,token_idx[b,m],:]; src [B,H,N,d], token_idx [B,M] int32, dst [B,H,>=M,d]."""
    _token_move("sva_gather_tokens", src, token_idx, dst, status)


def scatter_tokens(src, token_idx, dst, status=None) -> None:
    """dst[b,h,token_idx[b,m],:] = src[b,h,m,:]; the other rows of dst keep their contents."""
    _token_move("sva_scatter_tokens", src, token_idx, dst, status)


def quantize_qk_fp8(p: Problem, q, k, q8, k8, q_scale, k_scale) -> None:
    rc = lib().sva_quantize_qk_fp8(C.byref(p), _ptr(q), _ptr(k), _ptr(q8), _ptr(k8), _ptr(q_scale),
                                   _ptr(k_scale), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_quantize_qk_fp8")


def smooth_workspace_bytes(p: Problem) -> int:
    return int(lib().sva_smooth_workspace_bytes(C.byref(p)))


def quantize_qk_fp8_smooth_k(p: Problem, q, k, q8, k8, q_scale, k_scale, k_mean, lse_shift, workspace) -> None:
    rc = lib().sva_quantize_qk_fp8_smooth_k(C.byref(p), _ptr(q), _ptr(k), _ptr(q8), _ptr(k8), _ptr(q_scale),
                                            _ptr(k_scale), _ptr(k_mean), _ptr(lse_shift), _ptr(workspace),
                                            C.c_size_t(_ws_bytes(workspace)), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_quantize_qk_fp8_smooth_k")


def block_select_pooled(p: Problem, s: Select, q_mean, k_mean, row_ptr, col_idx, workspace, block_scores=None) -> None:
    rc = lib().sva_block_select_pooled(C.byref(p), C.byref(s), _ptr(q_mean), _ptr(k_mean), _ptr(row_ptr), _ptr(col_idx),
                                       _ptr(block_scores), _ptr(workspace), C.c_size_t(_ws_bytes(workspace)), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_block_select_pooled")


def qk_norm_rope_pool(p: Problem, q, k, g_q, g_k, cos_table, sin_table, eps, q_out, k_out, q_mean=None, k_mean=None,
                      q8=None, k8=None, q_scale=None, k_scale=None) -> None:
    rc = lib().sva_qk_norm_rope_pool(C.byref(p), _ptr(q), _ptr(k), _ptr(g_q), _ptr(g_k), _ptr(cos_table),
                                     _ptr(sin_table), C.c_float(eps), _ptr(q_out), _ptr(k_out), _ptr(q_mean),
                                     _ptr(k_mean), _ptr(q8), _ptr(k8), _ptr(q_scale), _ptr(k_scale), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_qk_norm_rope_pool")


def pool_qk(p: Problem, q, k, q_mean, k_mean, q_scale=None, k_scale=None) -> None:
    rc = lib().sva_pool_qk(C.byref(p), _ptr(q), _ptr(k), _ptr(q_scale), _ptr(k_scale), _ptr(q_mean), _ptr(k_mean),
                           _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_pool_qk")


def debug_set_prof_buffer(buf) -> None:
    """Cycle counter of the attention kernel (include/sva_debug.h): a zeroed device int64 tensor of >= 320
    entries, entry 319 receives the cycle count of the longest CTA of later launches; None switches it off."""
    lib().sva_debug_set_prof_buffer(_ptr(buf))


def debug_set_mode(bits: int) -> None:
    """Kernel behaviour switches of later launches (include/sva_debug.h); 0 = normal."""
    lib().sva_debug_set_mode(int(bits))


def debug_set_wait_limit(cycles: int) -> None:
    """SM cycles a device-side wait may last before its CTA gives up; <= 0 restores the default."""
    if lib().sva_debug_set_wait_limit(C.c_longlong(int(cycles))) != 0:
        raise RuntimeError("sva_debug_set_wait_limit failed")


def debug_last_choice() -> int:
    """Which form the last linear, rotary or cache call chose (include/sva_debug.h)."""
    return lib().sva_debug_last_choice()


def attn_remainder_workspace_bytes(p: Problem, order: int = 0) -> int:
    return int(lib().sva_attn_remainder_workspace_bytes(C.byref(p), int(order)))


def block_sparse_attn_remainder_fwd(p: Problem, q, k, v, row_ptr, col_idx, o, lse=None, status=None, order: int = 0,
                                    workspace=None, block_scores=None) -> None:
    """Exact attention over the kept blocks plus the approximate remainder of the dropped ones (order 0: block means;
    order 1: plus the first-order term, which needs the routing's score matrix)."""
    rc = lib().sva_block_sparse_attn_remainder_fwd(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(row_ptr), _ptr(col_idx),
                                                   _ptr(block_scores), _ptr(o), _ptr(lse), _ptr(status), int(order),
                                                   _ptr(workspace), _ws_bytes(workspace), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_block_sparse_attn_remainder_fwd")


def quantize_qk_fp4(p: Problem, q, k, q4, k4, q_sf, k_sf, q_g, k_g, workspace) -> None:
    """Block-scaled 4-bit codes, e4m3 block scales (MMA tile order) and per-(b,h) fp32 scales of Q and K."""
    rc = lib().sva_quantize_qk_fp4(C.byref(p), _ptr(q), _ptr(k), _ptr(q4), _ptr(k4), _ptr(q_sf), _ptr(k_sf), _ptr(q_g),
                                   _ptr(k_g), _ptr(workspace), _ws_bytes(workspace), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_quantize_qk_fp4")


def block_sparse_attn_fwd_fp4(p: Problem, q4, k4, q_sf, k_sf, q_g, k_g, v, row_ptr, col_idx, o, lse=None, status=None,
                              workspace=None) -> None:
    """Attention over 4-bit block-scaled Q and K (row_ptr None = dense)."""
    rc = lib().sva_block_sparse_attn_fwd_fp4(C.byref(p), _ptr(q4), _ptr(k4), _ptr(q_sf), _ptr(k_sf), _ptr(q_g), _ptr(k_g),
                                             _ptr(v), _ptr(row_ptr), _ptr(col_idx), _ptr(o), _ptr(lse), _ptr(status),
                                             _ptr(workspace), _ws_bytes(workspace), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_block_sparse_attn_fwd_fp4")


def attn_one_call_workspace_bytes(p: Problem) -> int:
    """Workspace the one-call attention entry points need (e4m3 Q/K: just the row counters and tile lists)."""
    return int(lib().sva_attn_one_call_workspace_bytes(C.byref(p)))


ACTIVATIONS = {"none": 0, "gelu": 1, "silu": 2}
ROPE_LAYOUTS = {"interleaved": 0, "half": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}
CACHE_FORMATS = {"e4m3": 0, "fp4": 1, "e4m3_page": 8}


# A call's tensors are those that its plan was made from, or others like them: their sizes are compared, where the plan's have gaps their strides too, and
# what the plan has not seen is looked at.  (Strides and devices of every tensor again would be a third of what a small call takes in Python.)
_NOT_THE_PLANS = "tensors on the GPU, no smaller than those that the plan was made for"


def _gaps(**tensors):
    """The strides (of more than one row) of the tensors that reach further than their bytes."""
    found = {}
    for name, t in tensors.items():
        if t is None or t.is_contiguous():
            continue
        shape, strides, reach, size = t.shape, t.stride(), 1, 1
        for n, s in zip(shape, strides):
            reach += (n - 1) * s
            size *= n
        if reach > size > 0:
            found[name] = [(i, s) for i, (n, s) in enumerate(zip(shape, strides)) if n > 1]
    return found


def _same_gaps(gaps, **tensors):
    for name, t in tensors.items():
        assert t is None or all(t.stride(i) == s for i, s in gaps.get(name, ())), f"{name} has other strides than the plan's"


def _row_stride(t, what):
    assert t.dim() == 2 and t.stride(1) == 1, f"{what} is a matrix with contiguous rows"
    return t.stride(0)


def _holds_whole_pieces(codes, K: int) -> bool:
    """Whether a matrix of codes has room for rows of whole 16-byte pieces, as the quantisers write them.  (Of several rows the C side sees the
    stride; a single one may carry any.)"""
    row, rows, stride = -(-K // 16) * 16, codes.shape[0], codes.stride(0)
    end = codes.storage_offset() + (rows - 1) * stride + row
    return rows == 0 or (rows > 1 or codes.shape[1] >= row or stride >= row) and end <= codes.untyped_storage().nbytes()


def make_linear(x=None, x8=None, x_scale=None, w8=None, w_scale=None, out=None, act: str = "none", residual=None, w=None, K: int = 0) -> Linear:
    """A linear layer y = x w^T: x [M,K] bf16, x8 [M,>=K] codes, x_scale [ceil(K/128),M] fp32, w [N,K] bf16, w8 [N,>=K] codes,
    w_scale [ceil(N/128),ceil(K/128)] fp32, out and residual [M,N] bf16.  What a call does not use may be left out; K is taken from x or
    w, or given.  Codes that are written (x8 beside x, w8 beside w) have room for rows of whole 16-byte pieces."""
    p = Linear()
    rows = x if x is not None else x8
    p.M = rows.shape[0] if rows is not None else 0
    p.K = K or (x.shape[1] if x is not None else w.shape[1] if w is not None else 0)
    cols = w8 if w8 is not None else w
    p.N = cols.shape[0] if cols is not None else 0
    p.act = ACTIVATIONS[act]
    for name, t in (("x", x), ("w", w), ("out", out), ("residual", residual), ("x8", x8), ("w8", w8), ("x_scale", x_scale),
                    ("w_scale", w_scale)):
        if t is not None:
            # (a matrix of one row may carry any stride: its row's length, rounded up, will do)
            stride = _row_stride(t, name)
            setattr(p, name + "_stride", stride if t.shape[0] > 1 else -(-t.shape[1] // 16) * 16)
    for t, shape in ((x, (p.M, p.K)), (out, (p.M, p.N)), (residual, (p.M, p.N)), (w, (p.N, p.K))):
        assert t is None or tuple(t.shape) == shape and t.dtype == torch.bfloat16, "bf16 matrices of matching sizes"
    for t, n in ((x8, p.M), (w8, p.N)):
        assert t is None or t.shape[0] == n and t.shape[1] >= p.K and t.element_size() == 1, "codes are bytes, a row for each row"
    for given, codes in ((x, x8), (w, w8)):
        assert given is None or codes is None or _holds_whole_pieces(codes, p.K), "codes that are written are rows of whole 16-byte pieces"
    groups = -(-p.K // 128)
    for t, shape in ((x_scale, (groups, p.M)), (w_scale, (-(-p.N // 128), groups))):
        assert t is None or t.dtype == torch.float32 and t.shape[0] == shape[0] and t.shape[1] >= shape[1], "fp32 scales, one per block of 128"
    tensors = (x, x8, x_scale, w, w8, w_scale, out, residual)
    if all([t is None or t.is_cuda for t in tensors]):
        a, b, c, d, e, f, g, h = [0 if t is None else t.nbytes for t in tensors]
        p.rows, p.tiles, p.product = (a, b, c), (d, e, f), (b, c, e, f, g, h, 4 * p.N)
    p.gaps = _gaps(x=x, x8=x8, x_scale=x_scale, w=w, w8=w8, w_scale=w_scale, out=out, residual=residual)
    return p


def quantize_rows_fp8(p: Linear, x, x8, x_scale) -> None:
    """Activations to e4m3 codes, a scale per token and 128 inputs."""
    a, b, c = p.rows
    assert x.nbytes >= a and x8.nbytes >= b and x_scale.nbytes >= c, _NOT_THE_PLANS
    if p.gaps:
        _same_gaps(p.gaps, x=x, x8=x8, x_scale=x_scale)
    rc = (_lib or lib()).sva_quantize_rows_fp8(p, x.data_ptr(), x8.data_ptr(), x_scale.data_ptr(), _stream())
    if rc:
        raise SvaError(rc, "sva_quantize_rows_fp8")


def quantize_tiles_fp8(p: Linear, w, w8, w_scale) -> None:
    """Weights to e4m3 codes, a scale per tile of 128 x 128."""
    a, b, c = p.tiles
    assert w.nbytes >= a and w8.nbytes >= b and w_scale.nbytes >= c, _NOT_THE_PLANS
    if p.gaps:
        _same_gaps(p.gaps, w=w, w8=w8, w_scale=w_scale)
    rc = lib().sva_quantize_tiles_fp8(C.byref(p), _ptr(w), _ptr(w8), _ptr(w_scale), _stream())
    if rc != SVA_OK:
        raise SvaError(rc, "sva_quantize_tiles_fp8")


def linear_fp8(p: Linear, x8, x_scale, w8, w_scale, out, bias=None, residual=None, status=None) -> None:
    """out = bf16(act(x w^T + bias) + residual) from codes and scales."""
    a, b, c, d, e, f, g = p.product
    assert x8.nbytes >= a and x_scale.nbytes >= b and w8.nbytes >= c and w_scale.nbytes >= d and out.nbytes >= e and \
        (residual is None or residual.nbytes >= f) and (status is None or status.is_cuda), _NOT_THE_PLANS
    assert bias is None or bias.is_cuda and bias.dtype is torch.float32 and bias.nbytes == g and bias.is_contiguous(), "bias is [N] fp32"
    if p.gaps:
        _same_gaps(p.gaps, x8=x8, x_scale=x_scale, w8=w8, w_scale=w_scale, out=out, residual=residual)
    rc = (_lib or lib()).sva_linear_fp8(p, x8.data_ptr(), x_scale.data_ptr(), w8.data_ptr(), w_scale.data_ptr(), out.data_ptr(),
                                        None if bias is None else bias.data_ptr(), None if residual is None else residual.data_ptr(),
                                        None if status is None else status.data_ptr(), _stream())
    if rc:
        raise SvaError(rc, "sva_linear_fp8")


def rope_steps(rotary_dim: int, axis_pairs=None, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained_length: float = 1.0,
               beta_fast: float = 32.0, beta_slow: float = 1.0, device=None):
    """The frequency ladder of rope(): (steps, an int64 tensor of rotary_dim/2 fractions of a turn; the factor on cos and sin)."""
    pairs = list(axis_pairs or [rotary_dim // 2])
    steps, out = (C.c_uint64 * max(1, rotary_dim // 2))(), C.c_float()
    rc = lib().sva_rope_steps(rotary_dim, (C.c_int32 * 3)(*(pairs + [0, 0])[:3]), base, ROPE_SCALINGS[scaling], factor, trained_length,
                              beta_fast, beta_slow, steps, C.byref(out))
    if rc != SVA_OK:
        raise SvaError(rc, "sva_rope_steps")
    return torch.tensor(list(steps), dtype=torch.int64, device=device), out.value


def make_rope(q, k, q_out, k_out, positions, rotary_dim: int, layout: str = "interleaved", axis_pairs=None, factor: float = 1.0,
              inverse: bool = False) -> Rope:
    """q [B,Hq,N,d], k [B,Hk,N,d] (or None) and where they go; positions [axes, B or 1, N] int32."""
    p = Rope()
    p.B, p.Hq, p.N, p.d = q.shape
    p.Hk = k.shape[1] if k is not None else 0
    p.rotary_dim, p.layout, p.inverse, p.factor = rotary_dim, ROPE_LAYOUTS[layout], int(inverse), factor
    pairs = list(axis_pairs or [rotary_dim // 2])
    p.axis_pairs = (C.c_int32 * 3)(*(pairs + [0, 0])[:3])
    assert len(pairs) <= 3 and positions.dtype == torch.int32 and positions.dim() == 3 and positions.shape[0] >= len(pairs) and \
        positions.shape[1] in (1, p.B) and positions.shape[2] == p.N and (p.N <= 1 or positions.stride(2) == 1), "positions are [axes, B or 1, N] int32"
    p.pos_stride = (C.c_int64 * 2)(positions.stride(0), positions.stride(1) if positions.shape[1] > 1 else 0)
    p.q_stride, p.q_out_stride = _strides(q), _strides(q_out)
    assert q_out.shape == q.shape and q.dtype == q_out.dtype == torch.bfloat16
    if k is not None:
        assert k.shape == (p.B, p.Hk, p.N, p.d) and k_out.shape == k.shape and k.dtype == k_out.dtype == torch.bfloat16
        p.k_stride, p.k_out_stride = _strides(k), _strides(k_out)
    if q.is_cuda and q_out.is_cuda and positions.is_cuda and (k is None or k.is_cuda and k_out.is_cuda):
        p.sizes = q.nbytes, 4 * rotary_dim, positions.nbytes, q_out.nbytes, 0 if k is None else k.nbytes
    p.gaps = _gaps(q=q, k=k, positions=positions, q_out=q_out, k_out=k_out)
    return p


def rope(p: Rope, q, k, steps, positions, q_out, k_out) -> None:
    """Rotary positions of q and k (k None: q alone)."""
    a, b, c, d, e = p.sizes
    assert q.nbytes >= a and steps.nbytes >= b and positions.nbytes >= c and q_out.nbytes >= d and steps.is_cuda and \
        (k is None or k_out is None or k.nbytes >= e and k_out.nbytes >= e), _NOT_THE_PLANS
    if p.gaps:
        _same_gaps(p.gaps, q=q, k=k, positions=positions, q_out=q_out, k_out=k_out)
    rc = (_lib or lib()).sva_rope(p, q.data_ptr(), None if k is None else k.data_ptr(), steps.data_ptr(), positions.data_ptr(),
                                  q_out.data_ptr(), None if k_out is None else k_out.data_ptr(), _stream())
    if rc:
        raise SvaError(rc, "sva_rope")


def make_kv_cache(k, v, format: str = "e4m3") -> KvCache:
    """A cache over its arrays: k and v are [codes, scale] (e4m3, e4m3_page) or [codes, scale, sf] (fp4), codes [pages,H,page,d or d/2] bytes,
    scale [pages,H,page] fp32 (e4m3_page: [pages,H]), sf [pages,H,page,d/16] bytes, all contiguous.  The arrays are kept alive."""
    c = KvCache()
    c.format = CACHE_FORMATS[format]
    c.pages, c.H, c.page, row = k[0].shape
    c.d = row * 2 if format == "fp4" else row
    shapes = [(c.pages, c.H, c.page, row), (c.pages, c.H) if format == "e4m3_page" else (c.pages, c.H, c.page), (c.pages, c.H, c.page, c.d // 16)]
    for arrays in (k, v):
        assert len(arrays) == (3 if format == "fp4" else 2)
        for t, shape, size in zip(arrays, shapes, (1, 4, 1)):
            assert tuple(t.shape) == shape and t.is_contiguous() and t.element_size() == size, "contiguous arrays of the cache's sizes"
    c.k_codes, c.v_codes, c.k_scale, c.v_scale = _ptr(k[0]), _ptr(v[0]), _ptr(k[1]), _ptr(v[1])
    if format == "fp4":
        c.k_sf, c.v_sf = _ptr(k[2]), _ptr(v[2])
    c.arrays, c.on_gpu, c.heads = (tuple(k), tuple(v)), all(t.is_cuda for t in (*k, *v)), (c.H, c.d)
    c.device = k[0].get_device() if len({t.get_device() for t in (*k, *v)}) == 1 else -1
    return c


def kv_cache_write(c: KvCache, k, v, slots, status=None) -> None:
    """k, v [B,H,T,d] bf16 into the slots [B,T] int32 (negative: left out)."""
    shape = Bq, H, T, d = k.shape
    assert H == c.H and d == c.d and v.shape == shape and k.dtype is v.dtype is torch.bfloat16, "k, v are [B,H,T,d] bf16"
    assert slots.shape == (Bq, T) and slots.dtype is torch.int32 and slots.is_contiguous(), "slots are [B,T] int32"
    assert c.on_gpu and k.is_cuda and v.is_cuda and slots.is_cuda and (status is None or status.is_cuda), "the cache and its tensors are on the GPU"
    rc = (_lib or lib()).sva_kv_cache_write(c, k.data_ptr(), v.data_ptr(), _strides(k), _strides(v), Bq, T, slots.data_ptr(),
                                            None if status is None else status.data_ptr(), _stream())
    if rc:
        raise SvaError(rc, "sva_kv_cache_write")


def kv_cache_read(c: KvCache, page_table, lengths, k, v, status=None) -> None:
    """Each sequence's first rows, from its pages, into k, v [B,H,N,d] bf16; rows from lengths[b] on become zeros."""
    shape = Bq, H, N, d = k.shape
    assert H == c.H and d == c.d and v.shape == shape and k.dtype is v.dtype is torch.bfloat16, "k, v are [B,H,N,d] bf16"
    rows, most = page_table.shape
    stride, inner = page_table.stride()
    assert rows == Bq and page_table.dtype is torch.int32 and inner == 1, "page_table is [B,pages] int32"
    assert lengths.shape == (Bq,) and lengths.dtype is torch.int32 and lengths.is_contiguous(), "lengths is [B] int32"
    assert c.on_gpu and page_table.is_cuda and lengths.is_cuda and k.is_cuda and v.is_cuda and (status is None or status.is_cuda), "the cache and its tensors are on the GPU"
    rc = (_lib or lib()).sva_kv_cache_read(c, page_table.data_ptr(), stride, most, lengths.data_ptr(), Bq, N, k.data_ptr(), v.data_ptr(),
                                           _strides(k), _strides(v), None if status is None else status.data_ptr(), _stream())
    if rc:
        raise SvaError(rc, "sva_kv_cache_read")


_NOT_ON_GPU = "the cache and its tensors are on the current GPU"


def _table(page_table, rows):
    """Row stride and entries per row of a page table."""
    n, most = page_table.shape
    stride, inner = page_table.stride()
    assert n == rows and page_table.dtype is _I32 and (inner == 1 or most == 1), "page_table is [rows,pages] int32"
    return stride, most


_I32, _BF16 = torch.int32, torch.bfloat16


def _int32s(t, n, what, device):
    assert t.shape == (n,) and t.dtype is _I32 and t.is_contiguous() and t.get_device() == device, f"{what} are {n} int32, side by side, on the GPU"
    return t.data_ptr()


def _all_on(device, *tensors):
    """Whether the tensors (or None) are on that GPU, and it is the current one: kernels run there."""
    for t in tensors:
        if t is not None and t.get_device() != device:
            return False
    return device >= 0 and device == _raw_device()


def kv_cache_append(c: KvCache, k, v, page_table, lengths, counts=None, status=None) -> None:
    """k, v [B,H,T,d] bf16 behind the lengths [B] tokens that the sequences hold in their pages (the first counts [B] of each; None: all T).
    The cache's format is e4m3_page; `lengths` stays as it is."""
    shape = Bq, H, T, d = k.shape
    assert (H, d) == c.heads and v.shape == shape and k.dtype is v.dtype is _BF16, "k, v are [B,H,T,d] bf16"
    stride, most = _table(page_table, Bq)
    dev = c.device
    assert _all_on(dev, k, v, page_table, status), _NOT_ON_GPU
    rc = (_lib or lib()).sva_kv_cache_append(c, k.data_ptr(), v.data_ptr(), _strides_any(k), _strides_any(v), Bq, T, page_table.data_ptr(), stride, most,
                                             _int32s(lengths, Bq, "lengths", dev), None if counts is None else _int32s(counts, Bq, "counts", dev),
                                             None if status is None else status.data_ptr(), _stream())
    if rc:
        raise SvaError(rc, "sva_kv_cache_append")


def make_cached_attn(c: KvCache, q, o, page_table, causal: bool = False, scale: float = 0.0) -> CachedAttn:
    """Attention of q [B,Hq,M,d] over the cache (Hq a multiple of its heads), into o; page_table [B,pages] int32."""
    p = CachedAttn()
    p.B, p.Hq, p.M, d = q.shape
    assert d == c.d and p.Hq % c.H == 0 and o.shape == q.shape and q.dtype is o.dtype is _BF16, \
        "q, o are [B,Hq,M,d] bf16 with the cache's d and a multiple of its heads"
    p.table_stride, p.max_pages = _table(page_table, p.B)
    p.causal, p.softmax_scale, p.cache = int(causal), scale, c
    p.q_stride, p.o_stride = _strides_any(q), _strides_any(o)
    p.shape, p.strides, p.table = q.shape, (q.stride(), o.stride()), (page_table.shape, page_table.stride())
    return p


def cached_attn_workspace_bytes(p: CachedAttn) -> int:
    return int(lib().sva_cached_attn_workspace_bytes(C.byref(p.cache), C.byref(p)))


def cached_attn_fwd(p: CachedAttn, q, page_table, lengths, o, counts=None, lse=None, status=None, workspace=None) -> None:
    """o = attention of each sequence's counts [B] queries (None: all M) over its lengths [B] cached tokens; lse [B,Hq,M] fp32."""
    assert q.shape == p.shape == o.shape and q.dtype is o.dtype is _BF16 and (q.stride(), o.stride()) == p.strides, \
        "q, o are bf16 and of the sizes and strides that the plan was made for"
    assert (page_table.shape, page_table.stride()) == p.table and page_table.dtype is _I32, "page_table is int32 and of the plan's sizes and strides"
    assert lse is None or lse.shape == p.shape[:3] and lse.dtype is torch.float32 and lse.is_contiguous(), "lse is [B,Hq,M] fp32"
    dev = p.cache.device
    assert _all_on(dev, q, o, page_table, lse, status, workspace), _NOT_ON_GPU
    rc = (_lib or lib()).sva_cached_attn_fwd(p.cache, p, q.data_ptr(), page_table.data_ptr(), _int32s(lengths, p.shape[0], "lengths", dev),
                                             None if counts is None else _int32s(counts, p.shape[0], "counts", dev), o.data_ptr(),
                                             None if lse is None else lse.data_ptr(), None if status is None else status.data_ptr(),
                                             None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes, _stream())
    if rc:
        raise SvaError(rc, "sva_cached_attn_fwd")


def make_cross_attn(q, k, v, o, scale: float = 0.0) -> CrossAttn:
    """Attention of q [B,Hq,N,d] over an encoder's k, v [B,Hk,S,d] (Hq a multiple of Hk), into o; all bf16."""
    p = CrossAttn()
    p.B, p.Hq, p.N, p.d = q.shape
    p.Hk, p.S = k.shape[1], k.shape[2]
    assert k.shape == v.shape == (p.B, p.Hk, p.S, p.d) and o.shape == q.shape and p.Hk > 0 and p.Hq % p.Hk == 0, \
        "q, o are [B,Hq,N,d], k, v [B,Hk,S,d], Hq a multiple of Hk"
    assert q.dtype is k.dtype is v.dtype is o.dtype is torch.bfloat16, "q, k, v, o are bf16"
    p.softmax_scale, p.mask_stride = scale, p.S
    p.q_stride, p.k_stride, p.v_stride, p.o_stride = _strides_any(q), _strides_any(k), _strides_any(v), _strides_any(o)
    p.shapes, p.strides = (q.shape, k.shape), (q.stride(), k.stride(), v.stride(), o.stride())
    return p


def cross_attn_workspace_bytes(p: CrossAttn) -> int:
    return int(lib().sva_cross_attn_workspace_bytes(C.byref(p)))


def cross_attn_fwd(p: CrossAttn, q, k, v, o, lengths=None, key_mask=None, lse=None, status=None, workspace=None) -> None:
    """o = attention over the first lengths [B] keys (None: all S) that key_mask [B,S] (bool or bytes, None: all) does not leave out."""
    of_q, of_k = p.shapes
    assert q.shape == of_q == o.shape and k.shape == of_k == v.shape and q.dtype is k.dtype is v.dtype is o.dtype is _BF16 and \
        (q.stride(), k.stride(), v.stride(), o.stride()) == p.strides, "q, k, v, o are bf16 and of the sizes and strides that the plan was made for"
    if key_mask is not None:
        assert key_mask.shape == (of_k[0], of_k[2]) and key_mask.element_size() == 1 and (of_k[2] <= 1 or key_mask.stride(1) == 1), \
            "key_mask is [B,S] bytes"
        if of_k[0] > 1 and key_mask.stride(0) != p.mask_stride:              # (a plan is not changed by its calls: others may share it)
            p = CrossAttn.from_buffer_copy(p)
            p.mask_stride = key_mask.stride(0)
    assert lse is None or lse.shape == of_q[:3] and lse.dtype is torch.float32 and lse.is_contiguous(), "lse is [B,Hq,N] fp32"
    dev = q.get_device()
    assert _all_on(dev, k, v, o, key_mask, lse, status, workspace), "tensors are on the current GPU"
    rc = (_lib or lib()).sva_cross_attn_fwd(p, q.data_ptr(), k.data_ptr(), v.data_ptr(), None if lengths is None else _int32s(lengths, of_q[0], "lengths", dev),
                                            None if key_mask is None else key_mask.data_ptr(), o.data_ptr(), None if lse is None else lse.data_ptr(),
                                            None if status is None else status.data_ptr(), None if workspace is None else workspace.data_ptr(),
                                            0 if workspace is None else workspace.nbytes, _stream())
    if rc:
        raise SvaError(rc, "sva_cross_attn_fwd")


def kv_pages_copy(c: KvCache, src, dst, status=None) -> None:
    """Page dst[i] becomes page src[i] (int32; negative: left out)."""
    n = src.shape[0]
    assert _all_on(c.device, status), _NOT_ON_GPU
    rc = (_lib or lib()).sva_kv_pages_copy(c, _int32s(src, n, "src", c.device), _int32s(dst, n, "dst", c.device), n, _ptr(status), _stream())
    if rc:
        raise SvaError(rc, "sva_kv_pages_copy")


def _pool(c, refs, page_table, status):
    rows = page_table.shape[0]
    stride, most = _table(page_table, rows)
    assert _all_on(c.device, page_table, status), _NOT_ON_GPU
    return _int32s(refs, c.pages, "refs", c.device), page_table.data_ptr(), stride, rows, most


def kv_pages_take(c: KvCache, refs, page_table, lengths, counts, status=None) -> None:
    """Every row of page_table gets the pages for counts [rows] tokens behind its lengths [rows]: the free ones of the lowest ids."""
    pool = _pool(c, refs, page_table, status)
    rc = (_lib or lib()).sva_kv_pages_take(c, *pool, _int32s(lengths, pool[3], "lengths", c.device), _int32s(counts, pool[3], "counts", c.device), _ptr(status), _stream())
    if rc:
        raise SvaError(rc, "sva_kv_pages_take")


def kv_pages_fork(c: KvCache, refs, page_table, lengths, parents, children, status=None) -> None:
    """Row children[i] becomes a copy of row parents[i]: full pages shared, a partly filled last one copied to a page of its own.  Children
    hold nothing before, come once and are no parents of the call."""
    pool, n = _pool(c, refs, page_table, status), parents.shape[0]
    rc = (_lib or lib()).sva_kv_pages_fork(c, *pool, _int32s(lengths, pool[3], "lengths", c.device), _int32s(parents, n, "parents", c.device),
                                           _int32s(children, n, "children", c.device), n, _ptr(status), _stream())
    if rc:
        raise SvaError(rc, "sva_kv_pages_fork")


def kv_pages_free(c: KvCache, refs, page_table, lengths, rows, keep=None, status=None) -> None:
    """Gives back the pages of these rows behind their first keep [n] tokens (None: all of them)."""
    pool, n = _pool(c, refs, page_table, status), rows.shape[0]
    rc = (_lib or lib()).sva_kv_pages_free(c, *pool, _int32s(lengths, pool[3], "lengths", c.device), _int32s(rows, n, "rows", c.device),
                                           None if keep is None else _int32s(keep, n, "keep", c.device), n, _ptr(status), _stream())
    if rc:
        raise SvaError(rc, "sva_kv_pages_free")


def kv_pages_compact_workspace_bytes(c: KvCache) -> int:
    return int(lib().sva_kv_pages_compact_workspace_bytes(C.byref(c)))


def kv_pages_compact(c: KvCache, refs, page_table, workspace, live=None, status=None) -> None:
    """The pages in use move to the lowest ids; refs and page_table follow, live [1] int32 becomes their number."""
    pool = _pool(c, refs, page_table, status)
    assert workspace.get_device() == c.device, _NOT_ON_GPU
    rc = (_lib or lib()).sva_kv_pages_compact(c, *pool, None if live is None else _int32s(live, 1, "live", c.device), _ptr(status), _ptr(workspace),
                                              _ws_bytes(workspace), _stream())
    if rc:
        raise SvaError(rc, "sva_kv_pages_compact")
