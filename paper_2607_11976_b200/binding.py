"""ctypes binding of liblt_indexer.so: same names as the C ABI, argument marshalling only.

Every function takes torch CUDA tensors (used purely as device memory), passes
their pointers and sizes to the library and returns.  No arithmetic of the
method happens here, and there is no fallback: if the library is missing the
first call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

from . import build as _build

LT_DTYPE_F32, LT_DTYPE_BF16, LT_DTYPE_E4M3 = 0, 1, 2
LT_PATH_AUTO, LT_PATH_FUSED, LT_PATH_GENERIC, LT_PATH_FUSED_ABS = 0, 1, 2, 3
LT_OK = 0
LT_STATUS_TIMEOUT, LT_STATUS_FALLBACK, LT_STATUS_BOUNDS, LT_STATUS_SHORT = 1, 2, 4, 8
LT_DEBUG_SKIP_ONE_KTILE, LT_DEBUG_SKIP_SAMPLE_KTILE = 1, 2
LT_MAX_TOPK = 8192
LT_PAGE_KEYS, LT_KV4_GROUP = 64, 32

_DTYPE_CODES = {"f32": LT_DTYPE_F32, "bf16": LT_DTYPE_BF16, "e4m3": LT_DTYPE_E4M3}


class LtError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what} failed: {code} ({strerror(code)})")
        self.code = code


class Tunables(ctypes.Structure):
    """Mirror of `lt_tunables`; zero fields mean "default"."""

    _fields_ = [("path", ctypes.c_int), ("cap_mult", ctypes.c_int), ("sample_mult", ctypes.c_int),
                ("segment_tiles", ctypes.c_int), ("grid", ctypes.c_int), ("sample_rank", ctypes.c_int),
                ("wait_limit_us", ctypes.c_int), ("debug_flags", ctypes.c_int)]


_lib = None
_lib_path = None


def library_path() -> str:
    """The build `load()` opens: `use_library()`'s choice, else $LT_INDEXER_LIB, else the in-tree release build."""
    return _lib_path or os.environ.get("LT_INDEXER_LIB") or _build.LIB_PATH


def use_library(path: Optional[str]) -> None:
    """Selects which build of the library `load()` opens (None: the release build).  Used by the tests
    that run the bounds-checking build (`build.build(debug_bounds=True)`)."""
    global _lib, _lib_path
    _lib_path = path
    _lib = None


def load() -> ctypes.CDLL:
    """Loads the shared library (built in-tree by `build.build()`); raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: run `python -m paper_2607_11976_b200.build` (needs nvcc); "
                           "there is no CPU or PyTorch fallback for this path")
    lib = ctypes.CDLL(path)
    vp, fp, ip, i, sz = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.lt_indexer_topk.argtypes = [vp, fp, vp, fp, i, i, i, i, i, i, ip, fp, vp]
    lib.lt_indexer_topk.restype = i
    lib.lt_indexer_topk_ex.argtypes = [i, vp, fp, vp, fp, i, i, i, i, i, i, ip, fp, vp, sz, ctypes.POINTER(Tunables), vp]
    lib.lt_indexer_topk_ex.restype = i
    lib.lt_indexer_topk_workspace_bytes.argtypes = [i, i, i, i, i, i, ctypes.POINTER(Tunables)]
    lib.lt_indexer_topk_workspace_bytes.restype = sz
    lib.lt_indexer_topk_sampled.argtypes = [i, vp, fp, vp, fp, i, i, i, i, i, i, ip, i, ip, fp, vp, sz, ctypes.POINTER(Tunables), vp]
    lib.lt_indexer_topk_sampled.restype = i
    lib.lt_indexer_topk_sampled_workspace_bytes.argtypes = [i, i, i, i, i, i, i, ctypes.POINTER(Tunables)]
    lib.lt_indexer_topk_sampled_workspace_bytes.restype = sz
    lib.lt_indexer_topk_paged.argtypes = [i, vp, fp, vp, fp, ip, i, ctypes.c_longlong, i, i, i, i, i, i, ip, fp, vp, sz,
                                          ctypes.POINTER(Tunables), vp]
    lib.lt_indexer_topk_paged.restype = i
    lib.lt_indexer_topk_paged_workspace_bytes.argtypes = [i, i, i, i, i, i, ctypes.POINTER(Tunables)]
    lib.lt_indexer_topk_paged_workspace_bytes.restype = sz
    lib.lt_topk_frequent.argtypes = [ip, i, i, i, i, ip, ip, vp, sz, vp]
    lib.lt_topk_frequent.restype = i
    lib.lt_topk_frequent_workspace_bytes.argtypes = [i]
    lib.lt_topk_frequent_workspace_bytes.restype = sz
    lib.lt_knn_topk.argtypes = [i, vp, vp, i, i, i, i, ip, fp, vp, sz, ctypes.POINTER(Tunables), vp]
    lib.lt_knn_topk.restype = i
    lib.lt_knn_topk_workspace_bytes.argtypes = [i, i, i, i, i, ctypes.POINTER(Tunables)]
    lib.lt_knn_topk_workspace_bytes.restype = sz
    lib.lt_knn_scores.argtypes = [i, vp, vp, i, i, i, i, i, fp, vp]
    lib.lt_knn_scores.restype = i
    lib.lt_dsa_union_mask.argtypes = [ip, i, i, i, i, ip, ip, vp, vp]
    lib.lt_dsa_union_mask.restype = i
    lib.lt_indexer_sample_plan.argtypes = [i, i, i, ctypes.POINTER(Tunables), ctypes.POINTER(ctypes.c_int)]
    lib.lt_indexer_sample_plan.restype = i
    lib.lt_indexer_scores.argtypes = [i, vp, fp, vp, fp, i, i, i, i, i, i, i, fp, i, vp]
    lib.lt_indexer_scores.restype = i
    lib.lt_unfused_topk.argtypes = [i, vp, fp, vp, fp, i, i, i, i, i, i, ip, fp, fp, sz, i, vp]
    lib.lt_unfused_topk.restype = i
    lib.lt_indexer_topk_static.argtypes = [i, vp, fp, vp, fp, i, i, i, i, i, i, ip, fp, vp]
    lib.lt_indexer_topk_static.restype = i
    lib.lt_read_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int), vp]
    lib.lt_read_status.restype = i
    lib.lt_indexer_topk_static_max_keys.restype = i
    lib.lt_read_status_static.argtypes = [ctypes.POINTER(ctypes.c_int), vp]
    lib.lt_read_status_static.restype = i
    lib.lt_debug_wait_timeout.argtypes = [i, ip, vp]
    lib.lt_debug_wait_timeout.restype = i
    lib.lt_debug_umma_stream.argtypes = [i, i, ip, vp]
    lib.lt_debug_umma_stream.restype = i
    lib.lt_indexer_topk_strided.argtypes = [i, vp, fp, vp, ctypes.c_longlong, fp, i, i, i, i, i, i, ip, fp, vp, sz,
                                            ctypes.POINTER(Tunables), vp]
    lib.lt_indexer_topk_strided.restype = i
    ll, fl, tun = ctypes.c_longlong, ctypes.c_float, ctypes.POINTER(Tunables)
    lib.lt_kv4_page_bytes.argtypes = [i, i]
    lib.lt_kv4_page_bytes.restype = sz
    lib.lt_page_tables.argtypes = [ip, ip, ip, i, i, i, i, ip, ip, ip, ip, ip, ip, vp]
    lib.lt_page_tables.restype = i
    lib.lt_kv4_append.argtypes = [i, vp, vp, ll, ll, ip, i, i, i, vp, ll, vp]
    lib.lt_kv4_append.restype = i
    lib.lt_kv4_read.argtypes = [i, vp, ll, ip, i, i, i, vp, vp, vp]
    lib.lt_kv4_read.restype = i
    lib.lt_kv4_attention.argtypes = [i, vp, ll, vp, ll, ip, i, ip, ip, i, i, i, i, i, i, fl, vp, fp, vp, sz, tun, vp]
    lib.lt_kv4_attention.restype = i
    lib.lt_kv4_attention_topk.argtypes = [i, vp, ll, vp, ll, ip, i, ip, ip, ip, i, i, i, i, i, i, fl, vp, fp, vp, sz, tun, vp]
    lib.lt_kv4_attention_topk.restype = i
    lib.lt_kv4_attention_workspace_bytes.argtypes = [i, i, i, i, i, i]
    lib.lt_kv4_attention_workspace_bytes.restype = sz
    lib.lt_launch_count.restype = ctypes.c_ulonglong
    lib.lt_set_profiling.argtypes = [i]
    lib.lt_set_profiling.restype = i
    lib.lt_read_phase_ms.argtypes = [ctypes.POINTER(ctypes.c_float), vp]
    lib.lt_read_phase_ms.restype = i
    lib.lt_strerror.argtypes = [i]
    lib.lt_strerror.restype = ctypes.c_char_p
    lib.lt_last_cuda_error.restype = i
    lib.lt_version.restype = i
    lib.lt_shutdown.restype = None
    _lib = lib
    return lib


def strerror(code: int) -> str:
    return load().lt_strerror(code).decode()


def dtype_code(dtype) -> int:
    return _DTYPE_CODES[dtype] if isinstance(dtype, str) else int(dtype)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    return t.data_ptr()  # (the functions' argtypes make pointers of plain integers)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    # the current stream's handle without building a Stream object, which costs as much as a kernel launch
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _check(code: int, what: str) -> None:
    if code != LT_OK:
        extra = f" (cudaError {load().lt_last_cuda_error()})" if code == -4 else ""
        raise LtError(code, what + extra)


def _shape(q: torch.Tensor, k: torch.Tensor):
    T, H, D = q.shape
    N, D2 = k.shape
    if D2 != D:
        raise ValueError("q and k disagree on D")
    return T, N, H, D


def lt_indexer_topk_workspace_bytes(dtype, T: int, N: int, H: int, D: int, topk: int,
                                    tunables: Optional[Tunables] = None) -> int:
    return int(load().lt_indexer_topk_workspace_bytes(dtype_code(dtype), T, N, H, D, topk,
                                                      ctypes.byref(tunables) if tunables else None))


def lt_indexer_sample_plan(N: int, topk: int, causal_offset: int, tunables: Optional[Tunables] = None):
    """(sample size, stride, rank) the fused path uses for this problem; host-only."""
    buf = (ctypes.c_int * 3)()
    _check(load().lt_indexer_sample_plan(N, topk, causal_offset, ctypes.byref(tunables) if tunables else None, buf),
           "lt_indexer_sample_plan")
    return tuple(buf)


def lt_indexer_topk(q, w, k, k_scale, topk: int, causal_offset: int, out_idx, out_score=None, stream=None) -> None:
    """13-argument C entry point: dtype inferred from k_scale (None -> bf16, else e4m3)."""
    T, N, H, D = _shape(q, k)
    _check(load().lt_indexer_topk(_ptr(q), _ptr(w), _ptr(k), _ptr(k_scale), T, N, H, D, topk, causal_offset,
                                  _ptr(out_idx), _ptr(out_score), _stream(stream)), "lt_indexer_topk")


def lt_indexer_topk_ex(dtype, q, w, k, k_scale, topk: int, causal_offset: int, out_idx, out_score, workspace,
                       tunables: Optional[Tunables] = None, stream=None) -> None:
    T, N, H, D = _shape(q, k)
    _check(load().lt_indexer_topk_ex(dtype_code(dtype), _ptr(q), _ptr(w), _ptr(k), _ptr(k_scale), T, N, H, D, topk,
                                     causal_offset, _ptr(out_idx), _ptr(out_score), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(),
                                     ctypes.byref(tunables) if tunables else None, _stream(stream)), "lt_indexer_topk_ex")


def lt_indexer_topk_strided(dtype, q, w, k_view, k_scale, topk: int, causal_offset: int, out_idx, out_score, workspace,
                            tunables: Optional[Tunables] = None, stream=None) -> None:
    """lt_indexer_topk_ex over a row-strided key view: `k_view` is an [N, D] CUDA tensor whose rows are
    `k_view.stride(0)` elements apart (inner stride 1), e.g. `cache[:, :D]` of a wider cache."""
    T, H, D = q.shape
    N, D2 = k_view.shape
    if D2 != D or k_view.stride(1) != 1 or not k_view.is_cuda:
        raise ValueError("expected an [N, D] CUDA view with unit inner stride")
    _check(load().lt_indexer_topk_strided(dtype_code(dtype), _ptr(q), _ptr(w), k_view.data_ptr(),
                                          int(k_view.stride(0)), _ptr(k_scale), T, N, H, D, topk, causal_offset,
                                          _ptr(out_idx), _ptr(out_score), _ptr(workspace),
                                          workspace.numel() * workspace.element_size(),
                                          ctypes.byref(tunables) if tunables else None, _stream(stream)),
           "lt_indexer_topk_strided")


def lt_indexer_topk_sampled_workspace_bytes(dtype, T: int, N: int, H: int, D: int, topk: int, n_sample: int,
                                            tunables: Optional[Tunables] = None) -> int:
    return int(load().lt_indexer_topk_sampled_workspace_bytes(dtype_code(dtype), T, N, H, D, topk, n_sample,
                                                              ctypes.byref(tunables) if tunables else None))


def lt_indexer_topk_sampled(dtype, q, w, k, k_scale, topk: int, causal_offset: int, sample_idx, out_idx, out_score, workspace,
                            tunables: Optional[Tunables] = None, stream=None) -> None:
    """lt_indexer_topk_ex with a caller-provided sample (int32 device tensor of key positions)."""
    T, N, H, D = _shape(q, k)
    _check(load().lt_indexer_topk_sampled(dtype_code(dtype), _ptr(q), _ptr(w), _ptr(k), _ptr(k_scale), T, N, H, D, topk,
                                          causal_offset, _ptr(sample_idx), sample_idx.numel(), _ptr(out_idx), _ptr(out_score),
                                          _ptr(workspace), workspace.numel() * workspace.element_size(),
                                          ctypes.byref(tunables) if tunables else None, _stream(stream)),
           "lt_indexer_topk_sampled")


def lt_indexer_topk_paged_workspace_bytes(dtype, T: int, N: int, H: int, D: int, topk: int,
                                          tunables: Optional[Tunables] = None) -> int:
    return int(load().lt_indexer_topk_paged_workspace_bytes(dtype_code(dtype), T, N, H, D, topk,
                                                            ctypes.byref(tunables) if tunables else None))


def lt_indexer_topk_paged(dtype, q, w, k_pool, k_scale_pool, page_table, N: int, topk: int, causal_offset: int, out_idx,
                          out_score, workspace, tunables: Optional[Tunables] = None, stream=None) -> None:
    """lt_indexer_topk_ex over a paged key cache: k_pool [pool_rows, D], page_table int32 [n_pages] (pages of 64 keys)."""
    T, H, D = q.shape
    pool_rows, D2 = k_pool.shape
    if D2 != D:
        raise ValueError("q and k_pool disagree on D")
    _check(load().lt_indexer_topk_paged(dtype_code(dtype), _ptr(q), _ptr(w), _ptr(k_pool), _ptr(k_scale_pool), _ptr(page_table),
                                        page_table.numel(), pool_rows, T, N, H, D, topk, causal_offset, _ptr(out_idx),
                                        _ptr(out_score), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                        ctypes.byref(tunables) if tunables else None, _stream(stream)), "lt_indexer_topk_paged")


def lt_topk_frequent_workspace_bytes(N: int) -> int:
    return int(load().lt_topk_frequent_workspace_bytes(N))


def lt_topk_frequent(idx, N: int, out_pos, out_count, workspace, stream=None) -> None:
    """out_pos (int32 device tensor of n_out elements) = the most frequent positions of the [T, topk] matrix idx."""
    T, topk = idx.shape
    _check(load().lt_topk_frequent(_ptr(idx), T, topk, N, out_pos.numel(), _ptr(out_pos), _ptr(out_count), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)), "lt_topk_frequent")


def lt_knn_topk_workspace_bytes(T: int, N: int, D: int, topk: int, tunables: Optional[Tunables] = None) -> int:
    return int(load().lt_knn_topk_workspace_bytes(LT_DTYPE_BF16, T, N, D, topk, ctypes.byref(tunables) if tunables else None))


def lt_knn_topk(q, x, topk: int, out_idx, out_score, workspace, tunables: Optional[Tunables] = None, stream=None) -> None:
    """Exact top-k inner products of the bf16 queries q [T, D] over the bf16 corpus x [N, D]."""
    T, D = q.shape
    N, D2 = x.shape
    if D2 != D:
        raise ValueError("q and x disagree on D")
    _check(load().lt_knn_topk(LT_DTYPE_BF16, _ptr(q), _ptr(x), T, N, D, topk, _ptr(out_idx), _ptr(out_score), _ptr(workspace),
                              workspace.numel() * workspace.element_size(), ctypes.byref(tunables) if tunables else None,
                              _stream(stream)), "lt_knn_topk")


def lt_knn_scores(q, x, row_begin: int, row_end: int, out_scores, stream=None) -> None:
    T, D = q.shape
    N = x.shape[0]
    _check(load().lt_knn_scores(LT_DTYPE_BF16, _ptr(q), _ptr(x), T, N, D, row_begin, row_end, _ptr(out_scores), _stream(stream)),
           "lt_knn_scores")


def lt_dsa_union_mask(idx, N: int, group: int, union_pos, union_len, member_mask, stream=None) -> None:
    """LiteDSA union list + membership masks of consecutive groups of `group` rows of the [T, topk] matrix idx."""
    T, topk = idx.shape
    _check(load().lt_dsa_union_mask(_ptr(idx), T, topk, N, group, _ptr(union_pos), _ptr(union_len), _ptr(member_mask),
                                    _stream(stream)), "lt_dsa_union_mask")


# ---------------------------------------------------------------------------------------------
# serving step over a key-value cache held in 4 bits
# ---------------------------------------------------------------------------------------------

# (Calls of a decode step take a few microseconds on the GPU: what is asked of the tensors here is asked once.)
_I32, _U8 = torch.int32, torch.uint8


def _device() -> int:
    """The current CUDA device, where the library launches (-2 before there is any)."""
    return torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -2


def _dense(t: torch.Tensor, dtype, dev: int) -> int:
    """Pointer of a dense tensor of the dtype on the current device."""
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"expected a contiguous tensor of {dtype} on the current CUDA device")
    return t.data_ptr()


def _rows(t: torch.Tensor, dtype, dev: int) -> tuple:
    """(pointer, T, H, D, row stride in elements) of a [T, H, D] view whose heads are dense."""
    T, H, D = t.shape
    row, head, one = t.stride()
    if one != 1 or (head != D and H > 1) or t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"expected a [T, H, D] tensor of {dtype} with dense heads on the current CUDA device")
    return t.data_ptr(), T, H, D, row if T > 1 else H * D


def _value_type(dtype) -> tuple:
    """(the library's code, torch's type) of the values of a call."""
    code = _DTYPE_CODES[dtype] if dtype in _DTYPE_CODES else int(dtype)
    return code, torch.float32 if code == LT_DTYPE_F32 else torch.bfloat16


def _pool(pool: torch.Tensor, dev: int) -> tuple:
    """(pointer, pages, key-value heads, D) of a pool uint8 [pages, Hkv, 64, D + D / 8]."""
    pages, Hkv, keys, row = pool.shape
    if keys != LT_PAGE_KEYS or row % 9 != 0:
        raise ValueError("expected a pool uint8 [pages, Hkv, 64, D + D / 8]")
    return _dense(pool, _U8, dev), pages, Hkv, row // 9 * 8


def lt_kv4_page_bytes(Hkv: int, D: int) -> int:
    return int(load().lt_kv4_page_bytes(Hkv, D))


def alloc_kv4_pool(pages: int, Hkv: int, D: int, device="cuda") -> torch.Tensor:
    """An empty pool: uint8 [pages, Hkv, 64, D + D / 8], the shape that the calls below take Hkv and D from."""
    if lt_kv4_page_bytes(Hkv, D) == 0:
        raise ValueError("unsupported Hkv or D")
    return torch.empty((pages, Hkv, LT_PAGE_KEYS, D + D // 8), dtype=torch.uint8, device=device)


def lt_page_tables(context_len, new_len, free_pages, page_table, total_len, query_start, slot_map, position, status,
                   stream=None) -> None:
    """Block tables, slot map and positions of a step: int32 CUDA tensors context_len [B], new_len [B], free_pages
    [n_free], page_table [B, max_pages] (in and out), total_len [B], query_start [B + 1], slot_map [T], position [T],
    status [8]."""
    dev, B, T = _device(), context_len.numel(), slot_map.numel()
    rows, max_pages = page_table.shape
    if (rows != B or new_len.numel() != B or total_len.numel() != B or query_start.numel() != B + 1 or position.numel() != T or
            status.numel() < 8):
        raise ValueError("the tables disagree on the number of requests or tokens")
    n_free = 0 if free_pages is None else free_pages.numel()
    code = load().lt_page_tables(_dense(context_len, _I32, dev), _dense(new_len, _I32, dev), _dense(free_pages, _I32, dev) if n_free else None,
                                 n_free, B, max_pages, T, _dense(page_table, _I32, dev), _dense(total_len, _I32, dev),
                                 _dense(query_start, _I32, dev), _dense(slot_map, _I32, dev), _dense(position, _I32, dev), _dense(status, _I32, dev),
                                 _stream(stream))
    if code:
        _check(code, "lt_page_tables")


def lt_kv4_append(dtype, k, v, slot_map, pool, stream=None) -> None:
    """Quantises k, v [T, Hkv, D] (rows may be strided) into the slots of the pool."""
    dev = _device()
    code, values = _value_type(dtype)
    pool_ptr, pages, Hkv, D = _pool(pool, dev)
    k_ptr, T, H, d, k_row = _rows(k, values, dev)
    v_ptr, vT, vH, vd, v_row = _rows(v, values, dev)
    if vT != T or H != Hkv or vH != Hkv or d != D or vd != D or slot_map.numel() != T:
        raise ValueError("k, v, slot_map and pool disagree")
    code = load().lt_kv4_append(code, k_ptr, v_ptr, k_row, v_row, _dense(slot_map, _I32, dev), T, Hkv, D, pool_ptr, pages,
                                _stream(stream))
    if code:
        _check(code, "lt_kv4_append")


def lt_kv4_read(dtype, pool, slots, k_out, v_out, stream=None) -> None:
    """Values of the slots as k_out, v_out [n, Hkv, D]."""
    dev = _device()
    code, values = _value_type(dtype)
    pool_ptr, pages, Hkv, D = _pool(pool, dev)
    n = slots.numel()
    shape = k_out.shape
    if shape != (n, Hkv, D) or v_out.shape != shape:
        raise ValueError("slots, outputs and pool disagree")
    code = load().lt_kv4_read(code, pool_ptr, pages, _dense(slots, _I32, dev), n, Hkv, D, _dense(k_out, values, dev), _dense(v_out, values, dev),
                              _stream(stream))
    if code:
        _check(code, "lt_kv4_read")


def lt_kv4_attention_workspace_bytes(dtype, T: int, B: int, Hq: int, Hkv: int, D: int) -> int:
    return int(load().lt_kv4_attention_workspace_bytes(dtype_code(dtype), T, B, Hq, Hkv, D))


def _attention_args(dtype, q, pool, page_table, query_start, context_len, out, out_lse, workspace):
    """The arguments of both forms: (dtype .. context_len), (B, T, Hq, Hkv, D), (out, lse), (workspace, bytes), device."""
    dev = _device()
    code, values = _value_type(dtype)
    pool_ptr, pages, Hkv, D = _pool(pool, dev)
    q_ptr, T, Hq, d, q_row = _rows(q, values, dev)
    B = context_len.numel()
    rows, max_pages = page_table.shape
    if (d != D or rows != B or out.shape != q.shape or query_start.numel() != B + 1 or
            (out_lse is not None and out_lse.numel() != T * Hq)):
        raise ValueError("q, pool, tables and outputs disagree")
    return ((code, q_ptr, q_row, pool_ptr, pages, _dense(page_table, _I32, dev), max_pages, _dense(query_start, _I32, dev),
             _dense(context_len, _I32, dev)), (B, T, Hq, Hkv, D),
            (_dense(out, values, dev), None if out_lse is None else _dense(out_lse, torch.float32, dev)),
            (_dense(workspace, _U8, dev), workspace.numel()), dev)


def lt_kv4_attention(dtype, q, pool, page_table, query_start, context_len, scale: float, out, out_lse, workspace,
                     max_new: int = 0, tunables: Optional[Tunables] = None, stream=None) -> None:
    """Causal attention of q [T, Hq, D] over the requests' pages (out [T, Hq, D], out_lse fp32 [T, Hq] or None)."""
    inputs, sizes, outputs, scratch, _ = _attention_args(dtype, q, pool, page_table, query_start, context_len, out, out_lse, workspace)
    code = load().lt_kv4_attention(*inputs, *sizes, max_new, scale, *outputs, *scratch,
                                   ctypes.byref(tunables) if tunables else None, _stream(stream))
    if code:
        _check(code, "lt_kv4_attention")


def lt_kv4_attention_topk(dtype, q, pool, page_table, query_start, context_len, idx, scale: float, out, out_lse, workspace,
                          tunables: Optional[Tunables] = None, stream=None) -> None:
    """The same over the positions idx [T, topk] (int32, as lt_indexer_topk_paged writes them)."""
    inputs, sizes, outputs, scratch, dev = _attention_args(dtype, q, pool, page_table, query_start, context_len, out, out_lse, workspace)
    T, topk = idx.shape
    if T != sizes[1]:
        raise ValueError("expected idx [T, topk]")
    code = load().lt_kv4_attention_topk(*inputs, _dense(idx, _I32, dev), topk, *sizes, scale, *outputs, *scratch,
                                        ctypes.byref(tunables) if tunables else None, _stream(stream))
    if code:
        _check(code, "lt_kv4_attention_topk")


def lt_indexer_scores(dtype, q, w, k, k_scale, causal_offset: int, row_begin: int, row_end: int, out_scores,
                      path: int = LT_PATH_AUTO, stream=None) -> None:
    T, N, H, D = _shape(q, k)
    _check(load().lt_indexer_scores(dtype_code(dtype), _ptr(q), _ptr(w), _ptr(k), _ptr(k_scale), T, N, H, D, causal_offset,
                                    row_begin, row_end, _ptr(out_scores), path, _stream(stream)), "lt_indexer_scores")


def lt_unfused_topk(dtype, q, w, k, k_scale, topk: int, causal_offset: int, out_idx, out_score, score_buf,
                    path: int = LT_PATH_AUTO, stream=None) -> None:
    T, N, H, D = _shape(q, k)
    _check(load().lt_unfused_topk(dtype_code(dtype), _ptr(q), _ptr(w), _ptr(k), _ptr(k_scale), T, N, H, D, topk,
                                  causal_offset, _ptr(out_idx), _ptr(out_score), _ptr(score_buf),
                                  score_buf.numel() * score_buf.element_size(), path, _stream(stream)), "lt_unfused_topk")


def lt_indexer_topk_static(dtype, q, w, k, k_scale, topk: int, causal_offset: int, out_idx, out_score=None, stream=None) -> None:
    """Allocation-free entry point: same result as lt_indexer_topk_ex, scratch inside the library
    (16 MiB per GPU, one score row must fit: N <= 4,194,240).  Calls that may overlap on the GPU race."""
    T, N, H, D = _shape(q, k)
    _check(load().lt_indexer_topk_static(dtype_code(dtype), _ptr(q), _ptr(w), _ptr(k), _ptr(k_scale), T, N, H, D, topk,
                                         causal_offset, _ptr(out_idx), _ptr(out_score), _stream(stream)),
           "lt_indexer_topk_static")


def lt_read_status(workspace=None, stream=None) -> list:
    """Synchronises the stream and returns the 8-int status block of a workspace
    (None: the library-owned workspace of lt_indexer_topk)."""
    buf = (ctypes.c_int * 8)()
    _check(load().lt_read_status(_ptr(workspace), buf, _stream(stream)), "lt_read_status")
    return list(buf)


def lt_read_status_static(stream=None) -> list:
    """The status block of the last lt_indexer_topk_static call on the current device."""
    buf = (ctypes.c_int * 8)()
    _check(load().lt_read_status_static(buf, _stream(stream)), "lt_read_status_static")
    return list(buf)


def lt_debug_wait_timeout(limit_us: int, result2, stream=None) -> None:
    """Runs the bounded-wait probe: result2 (int32 CUDA tensor of 2) receives (wait result, abort flag)."""
    _check(load().lt_debug_wait_timeout(int(limit_us), _ptr(result2), _stream(stream)), "lt_debug_wait_timeout")


def lt_debug_umma_stream(pair: bool, iters: int, status, stream=None) -> None:
    """Enqueues one launch of the bare FP8 UMMA stream; status: zeroed int32 CUDA tensor of 1."""
    _check(load().lt_debug_umma_stream(1 if pair else 0, int(iters), _ptr(status), _stream(stream)), "lt_debug_umma_stream")


def lt_launch_count() -> int:
    return int(load().lt_launch_count())


def lt_set_profiling(enable: bool) -> None:
    _check(load().lt_set_profiling(1 if enable else 0), "lt_set_profiling")


def lt_read_phase_ms(stream=None) -> list:
    """Device ms of [sample scoring, sample statistics, fused scan, final select, fallback]."""
    buf = (ctypes.c_float * 5)()
    _check(load().lt_read_phase_ms(buf, _stream(stream)), "lt_read_phase_ms")
    return list(buf)


# ---------------------------------------------------------------------------------------------
# device-memory helpers (plumbing only)
# ---------------------------------------------------------------------------------------------

def to_device(inp, device="cuda"):
    """Uploads a workload (numpy storage codes) as torch tensors: (q, w, k, k_scale)."""
    def up(a):
        return None if a is None else torch.from_numpy(a).to(device)

    if inp.dtype == "bf16":
        q = torch.from_numpy(inp.q.view("int16")).to(device).view(torch.bfloat16)
        k = torch.from_numpy(inp.k.view("int16")).to(device).view(torch.bfloat16)
    else:
        q, k = up(inp.q), up(inp.k)
    return q, up(inp.w), k, up(inp.k_scale)


def alloc_workspace(dtype, T, N, H, D, topk, tunables: Optional[Tunables] = None, device="cuda") -> torch.Tensor:
    nbytes = lt_indexer_topk_workspace_bytes(dtype, T, N, H, D, topk, tunables)
    if nbytes == 0:
        raise ValueError("invalid problem for lt_indexer_topk_workspace_bytes")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)
