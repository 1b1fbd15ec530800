"""Thin ctypes binding of libkl.so: the same names as include/kl.h, argument marshalling only.

PyTorch appears here for device memory and streams alone (arenas, KV cache, token / logit buffers); every step
of the decode path runs inside the library's kernels.  There is no fallback: if the library is missing this
module raises at load time.
"""
from __future__ import annotations

import ctypes as C
import struct
from pathlib import Path

import torch

_LIB_PATH = Path(__file__).resolve().parent / "libkl.so"

KL_OK = 0
KL_ERR_INVALID_ARG = -1
KL_ERR_UNSUPPORTED_SHAPE = -2
KL_ERR_NOT_LOADED = -3
KL_ERR_CUDA = -4
KL_ERR_SYNC_TIMEOUT = -5
KL_ERR_OUT_OF_RANGE = -6
KL_ERR_TOO_LARGE = -7
KL_STATIC_ARGMAX_MAX_BATCH = 256
KL_MODE_LOOPED = 0
KL_MODE_PER_LAYER = 1
KL_MODE_PER_STAGE = 2

TENSOR_IDS = {"embed": 0, "wq": 1, "wk": 2, "wv": 3, "wo": 4, "wgate": 5, "wup": 6, "wdown": 7,
              "norm1": 8, "norm2": 9, "norm_f": 10, "lm_head": 11, "bq": 12, "bk": 13, "bv": 14, "router": 15}
KL_FLAG_QKV_BIAS = 1
KL_FLAG_NO_STASH = 2
KL_KV_BF16 = 0
KL_KV_E4M3 = 1
KL_F32 = 0
KL_BF16 = 1

# every symbol include/kl.h declares
EXPORTS = ("kl_workspace_bytes", "kl_create", "kl_load_weights", "kl_kv_cache_bytes", "kl_set_mode", "kl_decode_step",
           "kl_decode_step_host", "kl_argmax_advance", "kl_read_hidden", "kl_last_status", "kl_launch_count",
           "kl_set_wait_limit_ns", "kl_debug_skip_signal_once", "kl_status_string", "kl_destroy", "kl_profile_enable",
           "kl_profile_read", "kl_set_trace", "kl_set_tensor_core_attention", "kl_stash_mode", "kl_argmax_advance_static", "kl_set_batched_path",
           "kl_set_dependent_launch", "kl_decode_greedy_host", "kl_decode_greedy", "kl_decode_greedy_tokens",
           "kl_decode_greedy_tokens_host", "kl_debug_set_step", "kl_debug_set_jitter", "kl_load_expert_weights",
           "kl_paged_append", "kl_paged_read", "kl_paged_workspace_bytes", "kl_paged_select", "kl_paged_attention", "kl_paged_step_bytes",
           "kl_decode_step_paged")


class ModelDesc(C.Structure):
    _fields_ = [("n_layers", C.c_uint32), ("hidden", C.c_uint32), ("n_q_heads", C.c_uint32),
                ("n_kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("ffn", C.c_uint32), ("vocab", C.c_uint32),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("max_batch", C.c_uint32),
                ("max_ctx", C.c_uint32), ("flags", C.c_uint32), ("n_experts", C.c_uint32), ("top_k", C.c_uint32)]


class PagedCacheDesc(C.Structure):
    _fields_ = [("n_kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("page_size", C.c_uint32), ("n_pages", C.c_uint32),
                ("kv_type", C.c_uint32), ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("row_stride", C.c_int64),
                ("k_d", C.c_void_p), ("v_d", C.c_void_p), ("k_exp_d", C.c_void_p), ("v_exp_d", C.c_void_p), ("bounds_d", C.c_void_p)]


class PagedSeqs(C.Structure):
    _fields_ = [("positions_d", C.c_void_p), ("page_table_d", C.c_void_p), ("table_stride", C.c_int64), ("table_pages", C.c_uint32),
                ("n_seqs", C.c_uint32)]


_PACK_SEQS = struct.Struct("@PPqII").pack   # a PagedSeqs as bytes: building the ctypes object costs more than the rest of a call


_lib = None


def lib():
    """Loads libkl.so (built in-tree by paper_2410_23668_b200.build / __graft_entry__.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not _LIB_PATH.exists():
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2410_23668_b200.build` "
                           "(there is no CPU or PyTorch fallback for the decode path)")
    l = C.CDLL(str(_LIB_PATH))
    vp, u32, i32 = C.c_void_p, C.c_uint32, C.c_int32
    l.kl_workspace_bytes.argtypes = [C.POINTER(ModelDesc), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
    l.kl_workspace_bytes.restype = i32
    l.kl_create.argtypes = [C.POINTER(ModelDesc), vp, vp, C.POINTER(vp)]
    l.kl_create.restype = i32
    l.kl_load_weights.argtypes = [vp, C.c_int, C.c_int, vp, C.c_size_t, vp]
    l.kl_load_weights.restype = i32
    l.kl_load_expert_weights.argtypes = [vp, C.c_int, C.c_int, C.c_int, vp, C.c_size_t, vp]
    l.kl_load_expert_weights.restype = i32
    l.kl_kv_cache_bytes.argtypes = [vp, u32]
    l.kl_kv_cache_bytes.restype = C.c_size_t
    l.kl_set_mode.argtypes = [vp, C.c_int]
    l.kl_set_mode.restype = i32
    l.kl_decode_step.argtypes = [vp, vp, vp, vp, vp, u32, vp]
    l.kl_decode_step.restype = i32
    l.kl_decode_step_host.argtypes = [vp, vp, vp, vp, vp, u32, vp]
    l.kl_decode_step_host.restype = i32
    l.kl_decode_greedy_host.argtypes = [vp, vp, vp, vp, vp, u32, vp]
    l.kl_decode_greedy_host.restype = i32
    l.kl_decode_greedy.argtypes = [vp, vp, vp, vp, vp, u32, C.c_int, vp]
    l.kl_decode_greedy.restype = i32
    l.kl_decode_greedy_tokens.argtypes = [vp, vp, vp, vp, vp, vp, u32, u32, C.c_int, vp]
    l.kl_decode_greedy_tokens.restype = i32
    l.kl_decode_greedy_tokens_host.argtypes = [vp, i32, i32, vp, vp, u32, vp]
    l.kl_decode_greedy_tokens_host.restype = i32
    l.kl_argmax_advance.argtypes = [vp, vp, vp, vp, u32, vp]
    l.kl_argmax_advance.restype = i32
    l.kl_argmax_advance_static.argtypes = [vp, u32, vp, vp, u32, vp]
    l.kl_argmax_advance_static.restype = i32
    l.kl_read_hidden.argtypes = [vp, vp, u32, vp]
    l.kl_read_hidden.restype = i32
    l.kl_last_status.argtypes = [vp]
    l.kl_last_status.restype = i32
    l.kl_launch_count.argtypes = [vp]
    l.kl_launch_count.restype = C.c_uint64
    l.kl_set_wait_limit_ns.argtypes = [vp, C.c_uint64]
    l.kl_set_wait_limit_ns.restype = i32
    l.kl_debug_skip_signal_once.argtypes = [vp, C.c_int]
    l.kl_debug_skip_signal_once.restype = i32
    l.kl_debug_set_jitter.argtypes = [vp, u32, u32]
    l.kl_debug_set_jitter.restype = i32
    l.kl_debug_set_step.argtypes = [vp, u32, C.POINTER(u32)]
    l.kl_debug_set_step.restype = i32
    l.kl_profile_enable.argtypes = [vp, u32]
    l.kl_profile_enable.restype = i32
    l.kl_profile_read.argtypes = [vp, C.POINTER(u32), C.POINTER(C.c_float), C.POINTER(C.c_float)]
    l.kl_profile_read.restype = i32
    l.kl_set_trace.argtypes = [vp, vp, C.POINTER(u32), C.POINTER(u32), C.POINTER(u32)]
    l.kl_set_trace.restype = i32
    l.kl_set_tensor_core_attention.argtypes = [vp, C.c_int]
    l.kl_set_tensor_core_attention.restype = i32
    l.kl_stash_mode.argtypes = [vp]
    l.kl_stash_mode.restype = C.c_int
    l.kl_set_batched_path.argtypes = [vp, C.c_int]
    l.kl_set_batched_path.restype = i32
    l.kl_set_dependent_launch.argtypes = [vp, C.c_int]
    l.kl_set_dependent_launch.restype = i32
    pc, ps, i64 = vp, vp, C.c_int64   # kl_paged_cache *, kl_paged_seqs * (a ctypes structure by reference, or its bytes)
    l.kl_paged_append.argtypes = [pc, ps, vp, u32, vp, vp, C.c_int, i64, i64, vp, vp]
    l.kl_paged_append.restype = i32
    l.kl_paged_read.argtypes = [pc, ps, vp, u32, vp, vp, C.c_int, i64, i64, vp, vp]
    l.kl_paged_read.restype = i32
    l.kl_paged_workspace_bytes.argtypes = [pc, u32, u32, u32, C.POINTER(C.c_size_t)]
    l.kl_paged_workspace_bytes.restype = i32
    l.kl_paged_select.argtypes = [pc, ps, vp, C.c_int, i64, u32, u32, u32, u32, vp, vp, C.c_size_t, vp, vp]
    l.kl_paged_select.restype = i32
    l.kl_paged_attention.argtypes = [pc, ps, vp, vp, C.c_int, i64, i64, u32, C.c_float, u32, vp, u32, vp, vp, C.c_size_t, vp, vp]
    l.kl_paged_attention.restype = i32
    l.kl_paged_step_bytes.argtypes = [vp, pc, u32, u32, u32, C.POINTER(C.c_size_t)]
    l.kl_paged_step_bytes.restype = i32
    l.kl_decode_step_paged.argtypes = [vp, vp, vp, vp, vp, i64, u32, u32, vp, u32, vp, C.c_size_t, vp]
    l.kl_decode_step_paged.restype = i32
    l.kl_status_string.argtypes = [i32]
    l.kl_status_string.restype = C.c_char_p
    l.kl_destroy.argtypes = [vp]
    l.kl_destroy.restype = None
    _lib = l
    return l


class KlError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {kl_status_string(code)} ({code})")


def kl_status_string(code: int) -> str:
    return lib().kl_status_string(code).decode()


def _check(code: int, where: str) -> None:
    if code != KL_OK:
        raise KlError(code, where)


def make_desc(shape, max_batch: int, max_ctx: int, stash: bool = True) -> ModelDesc:
    return ModelDesc(shape.n_layers, shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.ffn,
                     shape.vocab, float(shape.rms_eps), float(shape.rope_theta), max_batch, max_ctx,
                     (KL_FLAG_QKV_BIAS if getattr(shape, "qkv_bias", False) else 0) | (0 if stash else KL_FLAG_NO_STASH),
                     int(getattr(shape, "n_experts", 0) or 0), int(getattr(shape, "top_k", 0) or 0))


def kl_workspace_bytes(desc: ModelDesc) -> tuple[int, int]:
    w, s = C.c_size_t(), C.c_size_t()
    _check(lib().kl_workspace_bytes(C.byref(desc), C.byref(w), C.byref(s)), "kl_workspace_bytes")
    return w.value, s.value


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _stream_ptr(stream) -> int:
    return 0 if stream is None else int(stream.cuda_stream)


def kl_argmax_advance_static(logits_d, tokens_d, positions_d, batch: int, stream=None) -> None:
    """Sampling block without a handle: scratch in a fixed array inside the library, nothing is allocated."""
    _check(lib().kl_argmax_advance_static(_ptr(logits_d), int(logits_d.shape[-1]), _ptr(tokens_d), _ptr(positions_d), batch,
                                          _stream_ptr(stream)), "kl_argmax_advance_static")


class PagedCache:
    """A paged key-value cache over tensors of the caller: k and v [n_pages, n_kv_heads, page_size, head_dim], bf16, or
    e4m3 codes (torch.float8_e4m3fn or uint8) with k_exp and v_exp uint8 [n_pages, n_kv_heads, page_size]; bounds
    (optional) bf16 [n_pages, n_kv_heads, 2, head_dim].  k and v may be permuted views, e.g. of a [n_pages, page_size,
    n_kv_heads, head_dim] tensor, as long as a row is contiguous and both have the same strides.  For page selection alone
    k and v may be None (then page_size and kv_type say what bounds does not).  The tensors must stay alive and in place."""

    def __init__(self, k, v, k_exp=None, v_exp=None, bounds=None, page_size=None, kv_type=None):
        self.tensors = (k, v, k_exp, v_exp, bounds)
        where = "PagedCache"
        d = PagedCacheDesc()
        if k is None:
            _need(v is None and bounds is not None and page_size is not None and kv_type is not None, where)
            d.n_pages, d.n_kv_heads, _, d.head_dim = bounds.shape
            d.page_size, d.kv_type = page_size, kv_type
        else:
            _need(k.dim() == 4 and k.shape == v.shape and k.stride(3) == 1 and v.stride(3) == 1 and k.dtype == v.dtype, where)
            strides = [[0 if t.shape[i] == 1 else t.stride(i) for i in range(3)] for t in (k, v)]   # of a single page or head: anything
            _need(strides[0] == strides[1], where)
            d.n_pages, d.n_kv_heads, d.page_size, d.head_dim = k.shape
            d.page_stride, d.head_stride, d.row_stride = strides[0]
            d.kv_type = KL_KV_BF16 if k.dtype == torch.bfloat16 else KL_KV_E4M3
            _need(k.dtype in (torch.bfloat16, torch.uint8, torch.float8_e4m3fn), where)
            if d.kv_type == KL_KV_E4M3:
                for e in (k_exp, v_exp):
                    _need(e is not None and e.dtype == torch.uint8 and e.shape == k.shape[:3] and e.is_contiguous(), where)
        if bounds is not None:
            _need(bounds.dtype == torch.bfloat16 and bounds.is_contiguous() and
                  tuple(bounds.shape) == (d.n_pages, d.n_kv_heads, 2, d.head_dim), where)
        d.k_d, d.v_d, d.k_exp_d, d.v_exp_d, d.bounds_d = (_ptr(t) or None for t in self.tensors)
        self.device = (bounds if k is None else k).device
        _need(all(t is None or t.device == self.device for t in self.tensors), where)
        self.desc = d
        self._index = self.device.index if self.device.type == "cuda" else -1
        self._ref = C.byref(d)

    @classmethod
    def allocate(cls, n_pages: int, n_kv_heads: int, page_size: int, head_dim: int, kv_type: int = KL_KV_BF16, bounds: bool = False,
                 device="cuda"):
        """A zeroed pool of its own."""
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        dt = torch.bfloat16 if kv_type == KL_KV_BF16 else torch.float8_e4m3fn
        k, v = torch.zeros(shape, dtype=dt, device=device), torch.zeros(shape, dtype=dt, device=device)
        ke = ve = b = None
        if kv_type == KL_KV_E4M3:
            ke, ve = (torch.zeros(shape[:3], dtype=torch.uint8, device=device) for _ in range(2))
        if bounds:
            b = torch.zeros(n_pages, n_kv_heads, 2, head_dim, dtype=torch.bfloat16, device=device)
        return cls(k, v, ke, ve, b)


def _need(ok: bool, where: str) -> None:
    if not ok:
        raise KlError(KL_ERR_INVALID_ARG, where)


_ROW_TYPES = {torch.float32: KL_F32, torch.bfloat16: KL_BF16}
_I32, _U8, _F32 = torch.int32, torch.uint8, torch.float32


def _here(cache: PagedCache) -> int:
    """Index of the device the cache lives on if that is the current one (the library launches there); -2 otherwise."""
    i = cache._index
    return i if i >= 0 and i == torch.cuda.current_device() else -2


def _paged_seqs(dev: int, positions, page_table, where: str):
    """The sequences of a call as the bytes of a kl_paged_seqs, and their number."""
    n, pages = page_table.shape
    stride, one = page_table.stride()
    _need(positions.dtype is _I32 and page_table.dtype is _I32 and one == 1 and positions.numel() == n and positions.is_contiguous() and
          positions.get_device() == dev and page_table.get_device() == dev, where)
    return _PACK_SEQS(positions.data_ptr(), page_table.data_ptr(), stride if n > 1 else max(stride, pages), pages, n), n


def _flag(dev: int, status, where: str) -> int:
    if status is None:
        return 0
    _need(status.dtype is _I32 and status.get_device() == dev and status.numel() >= 1, where)
    return status.data_ptr()


def _paged_rows(fn: str, call, cache: PagedCache, k, v, positions, page_table, row_starts, status, stream) -> None:
    dev, d = _here(cache), cache.desc
    rows, heads, width = shape = k.shape
    k_row, k_head, k_one = k.stride()
    v_row, v_head, v_one = v.stride()
    t = _ROW_TYPES.get(k.dtype)
    _need(t is not None and v.dtype is k.dtype and v.shape == shape and heads == d.n_kv_heads and width == d.head_dim and k_one == 1 and v_one == 1 and
          (heads == 1 or (k_head == width and v_head == width)) and k.get_device() == dev and v.get_device() == dev, fn)
    seqs, n = _paged_seqs(dev, positions, page_table, fn)
    starts = 0
    if row_starts is not None:
        _need(row_starts.dtype is _I32 and row_starts.is_contiguous() and row_starts.numel() == n + 1 and row_starts.get_device() == dev, fn)
        starts = row_starts.data_ptr()
    rc = call(cache._ref, seqs, starts, rows, k.data_ptr(), v.data_ptr(), t, k_row, v_row, _flag(dev, status, fn),
              0 if stream is None else stream.cuda_stream)
    if rc:
        raise KlError(rc, fn)


def kl_paged_append(cache: PagedCache, k_rows, v_rows, positions, page_table, row_starts=None, status=None, stream=None) -> None:
    """New rows [n_rows, n_kv_heads, head_dim] (bf16 or fp32; rows may be strided) into the pages; positions int32 [n_seqs],
    page_table int32 [n_seqs, pages], row_starts int32 [n_seqs + 1] or None (one row per sequence)."""
    _paged_rows("kl_paged_append", (_lib or lib()).kl_paged_append, cache, k_rows, v_rows, positions, page_table, row_starts, status, stream)


def kl_paged_read(cache: PagedCache, k_out, v_out, positions, page_table, row_starts=None, status=None, stream=None) -> None:
    """The rows that kl_paged_append with the same arguments would write, copied out."""
    _paged_rows("kl_paged_read", (_lib or lib()).kl_paged_read, cache, k_out, v_out, positions, page_table, row_starts, status, stream)


def kl_paged_workspace_bytes(cache: PagedCache, n_q_heads: int, n_seqs: int, table_pages: int) -> int:
    b = C.c_size_t()
    _check(lib().kl_paged_workspace_bytes(cache._ref, n_q_heads, n_seqs, table_pages, C.byref(b)), "kl_paged_workspace_bytes")
    return b.value


def _paged_queries(cache: PagedCache, dev: int, q, n: int, where: str):
    """(row type, row stride, query heads) of q [n, n_q_heads, head_dim]."""
    rows, heads, width = q.shape
    row, head, one = q.stride()
    t = _ROW_TYPES.get(q.dtype)
    _need(t is not None and rows == n and width == cache.desc.head_dim and one == 1 and (head == width or heads == 1) and q.get_device() == dev, where)
    return t, row, heads


def kl_paged_select(cache: PagedCache, q, positions, page_table, selected, workspace, keep_first: int = 1, keep_last: int = 1, status=None,
                    stream=None) -> None:
    """q [n_seqs, n_q_heads, head_dim] -> selected int32 [n_seqs, n_kv_heads, n_select]."""
    fn = "kl_paged_select"
    dev = _here(cache)
    seqs, n = _paged_seqs(dev, positions, page_table, fn)
    t, row, heads = _paged_queries(cache, dev, q, n, fn)
    s_n, s_h, n_select = selected.shape
    _need(selected.dtype is _I32 and selected.is_contiguous() and s_n == n and s_h == cache.desc.n_kv_heads and workspace.dtype is _U8 and
          workspace.is_contiguous() and 0 <= keep_first < 1 << 31 and 0 <= keep_last < 1 << 31 and selected.get_device() == dev and workspace.get_device() == dev, fn)
    rc = (_lib or lib()).kl_paged_select(cache._ref, seqs, q.data_ptr(), t, row, heads, keep_first, keep_last, n_select, selected.data_ptr(),
                                         workspace.data_ptr(), workspace.numel(), _flag(dev, status, fn), 0 if stream is None else stream.cuda_stream)
    if rc:
        raise KlError(rc, fn)


def kl_paged_attention(cache: PagedCache, q, out, positions, page_table, workspace, scale: float = 0.0, window: int = 0, selected=None, lse=None,
                       status=None, stream=None) -> None:
    """q, out [n_seqs, n_q_heads, head_dim] of one type; selected int32 [n_seqs, n_kv_heads, n_select]; lse fp32 [n_seqs, n_q_heads]."""
    fn = "kl_paged_attention"
    dev = _here(cache)
    seqs, n = _paged_seqs(dev, positions, page_table, fn)
    t, row, heads = _paged_queries(cache, dev, q, n, fn)
    t_out, out_row, out_heads = _paged_queries(cache, dev, out, n, fn)
    _need(t_out == t and out_heads == heads and workspace.dtype is _U8 and workspace.is_contiguous() and 0 <= window < 1 << 31 and
          workspace.get_device() == dev, fn)
    n_select = sel = lse_d = 0
    if selected is not None:
        s_n, s_h, n_select = selected.shape
        _need(selected.dtype is _I32 and selected.is_contiguous() and s_n == n and s_h == cache.desc.n_kv_heads and n_select > 0 and
              selected.get_device() == dev, fn)
        sel = selected.data_ptr()
    if lse is not None:
        _need(lse.dtype is _F32 and lse.is_contiguous() and lse.shape == (n, heads) and lse.get_device() == dev, fn)
        lse_d = lse.data_ptr()
    rc = (_lib or lib()).kl_paged_attention(cache._ref, seqs, q.data_ptr(), out.data_ptr(), t, row, out_row, heads, scale, window, sel, n_select, lse_d,
                                            workspace.data_ptr(), workspace.numel(), _flag(dev, status, fn), 0 if stream is None else stream.cuda_stream)
    if rc:
        raise KlError(rc, fn)


class Decoder:
    """One model instance on the current CUDA device.  Owns the two arenas as torch uint8 tensors."""

    def __init__(self, shape, max_batch: int, max_ctx: int, device="cuda", stash: bool = True):
        import torch
        self.torch = torch
        self.shape = shape
        self.max_batch, self.max_ctx = max_batch, max_ctx
        self.desc = make_desc(shape, max_batch, max_ctx, stash)
        wb, sb = kl_workspace_bytes(self.desc)
        self.weight_bytes, self.scratch_bytes = wb, sb
        self.weight_arena = torch.empty(wb, dtype=torch.uint8, device=device)
        self.scratch_arena = torch.empty(sb, dtype=torch.uint8, device=device)
        h = C.c_void_p()
        _check(lib().kl_create(C.byref(self.desc), _ptr(self.weight_arena), _ptr(self.scratch_arena), C.byref(h)), "kl_create")
        self.handle = h

    def close(self) -> None:
        if getattr(self, "handle", None):
            lib().kl_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the C-ABI calls, same names
    def kl_load_weights(self, name: str, layer: int, tensor, stream=None) -> None:
        t = tensor.contiguous()
        assert t.dtype == self.torch.bfloat16
        if "_e" in name:   # an expert's matrix of a mixture-of-experts layer: wgate_e<i>, wup_e<i>, wdown_e<i>
            stem, expert = name.rsplit("_e", 1)
            _check(lib().kl_load_expert_weights(self.handle, TENSOR_IDS[stem], layer, int(expert), _ptr(t), t.numel() * 2,
                                                _stream_ptr(stream)), f"kl_load_expert_weights({name}, {layer})")
        else:
            _check(lib().kl_load_weights(self.handle, TENSOR_IDS[name], layer, _ptr(t), t.numel() * 2, _stream_ptr(stream)),
                   f"kl_load_weights({name}, {layer})")
        if t.device.type == "cpu":
            self.torch.cuda.synchronize()  # pageable source must outlive the copy

    def kl_kv_cache_bytes(self, batch: int) -> int:
        return int(lib().kl_kv_cache_bytes(self.handle, batch))

    def kl_set_mode(self, mode: int) -> None:
        _check(lib().kl_set_mode(self.handle, mode), "kl_set_mode")

    def kl_decode_step(self, tokens_d, positions_d, kv_cache_d, logits_d, batch: int, stream=None) -> None:
        _check(lib().kl_decode_step(self.handle, _ptr(tokens_d), _ptr(positions_d), _ptr(kv_cache_d), _ptr(logits_d),
                                    batch, _stream_ptr(stream)), "kl_decode_step")

    def kl_decode_step_host(self, tokens_h, positions_h, kv_cache_d, logits_h, batch: int, stream=None) -> None:
        _check(lib().kl_decode_step_host(self.handle, _ptr(tokens_h), _ptr(positions_h), _ptr(kv_cache_d),
                                         _ptr(logits_h), batch, _stream_ptr(stream)), "kl_decode_step_host")

    def kl_decode_greedy(self, tokens_d, positions_d, kv_cache_d, logits_d, batch: int, restart: bool, stream=None) -> None:
        _check(lib().kl_decode_greedy(self.handle, _ptr(tokens_d), _ptr(positions_d), _ptr(kv_cache_d), _ptr(logits_d),
                                      batch, 1 if restart else 0, _stream_ptr(stream)), "kl_decode_greedy")

    def kl_decode_greedy_tokens(self, tokens_d, positions_d, kv_cache_d, logits_d, out_tokens_d, n_tokens: int, batch: int,
                                restart: bool, stream=None) -> None:
        _check(lib().kl_decode_greedy_tokens(self.handle, _ptr(tokens_d), _ptr(positions_d), _ptr(kv_cache_d), _ptr(logits_d),
                                             _ptr(out_tokens_d), n_tokens, batch, 1 if restart else 0, _stream_ptr(stream)),
               "kl_decode_greedy_tokens")

    def kl_decode_greedy_tokens_host(self, token: int, position: int, kv_cache_d, out_tokens_h, n_tokens: int, stream=None) -> None:
        _check(lib().kl_decode_greedy_tokens_host(self.handle, token, position, _ptr(kv_cache_d), _ptr(out_tokens_h), n_tokens,
                                                  _stream_ptr(stream)), "kl_decode_greedy_tokens_host")

    def kl_decode_greedy_host(self, tokens_h, positions_h, kv_cache_d, next_tokens_h, batch: int, stream=None) -> None:
        _check(lib().kl_decode_greedy_host(self.handle, _ptr(tokens_h), _ptr(positions_h), _ptr(kv_cache_d),
                                           _ptr(next_tokens_h), batch, _stream_ptr(stream)), "kl_decode_greedy_host")

    def kl_paged_step_bytes(self, cache: PagedCache, batch: int, table_pages: int, n_select: int = 0) -> int:
        b = C.c_size_t()
        _check(lib().kl_paged_step_bytes(self.handle, cache._ref, batch, table_pages, n_select, C.byref(b)), "kl_paged_step_bytes")
        return b.value

    def kl_decode_step_paged(self, tokens_d, positions_d, caches, page_table_d, logits_d, workspace_d, n_select: int = 0, stream=None) -> None:
        """caches: one PagedCache per layer; page_table_d int32 [batch, pages]."""
        fn = "kl_decode_step_paged"
        batch, pages = page_table_d.shape
        _need(len(caches) == self.shape.n_layers and tokens_d.numel() == batch and positions_d.numel() == batch and tokens_d.dtype is _I32 and
              positions_d.dtype is _I32 and page_table_d.dtype is _I32 and page_table_d.stride(1) == 1 and logits_d.dtype is _F32 and
              logits_d.numel() == batch * self.shape.vocab and logits_d.is_contiguous() and tokens_d.is_contiguous() and
              positions_d.is_contiguous() and workspace_d.dtype is _U8 and workspace_d.is_contiguous() and 0 <= n_select < 1 << 31, fn)
        dev = self.weight_arena.get_device()   # the library launches on the current device, and its weights lie there
        _need(dev >= 0 and dev == torch.cuda.current_device() and all(c._index == dev for c in caches) and
              all(t.get_device() == dev for t in (tokens_d, positions_d, page_table_d, logits_d, workspace_d)), fn)
        layers = (PagedCacheDesc * len(caches))(*(c.desc for c in caches))
        stride = page_table_d.stride(0) if batch > 1 else max(page_table_d.stride(0), pages)
        _check(lib().kl_decode_step_paged(self.handle, _ptr(tokens_d), _ptr(positions_d), C.addressof(layers), _ptr(page_table_d), stride, pages,
                                          n_select, _ptr(logits_d), batch, _ptr(workspace_d), workspace_d.numel(), _stream_ptr(stream)), fn)

    def kl_argmax_advance(self, logits_d, tokens_d, positions_d, batch: int, stream=None) -> None:
        _check(lib().kl_argmax_advance(self.handle, _ptr(logits_d), _ptr(tokens_d), _ptr(positions_d), batch,
                                       _stream_ptr(stream)), "kl_argmax_advance")

    def kl_read_hidden(self, hidden_d, batch: int, stream=None) -> None:
        _check(lib().kl_read_hidden(self.handle, _ptr(hidden_d), batch, _stream_ptr(stream)), "kl_read_hidden")

    def kl_last_status(self) -> int:
        return int(lib().kl_last_status(self.handle))

    def kl_launch_count(self) -> int:
        return int(lib().kl_launch_count(self.handle))

    def kl_profile_enable(self, capacity: int) -> None:
        _check(lib().kl_profile_enable(self.handle, capacity), "kl_profile_enable")

    def kl_profile_read(self, n: int) -> tuple[list[float], list[float]]:
        cnt = C.c_uint32(n)
        dec, cls = (C.c_float * n)(), (C.c_float * n)()
        _check(lib().kl_profile_read(self.handle, C.byref(cnt), dec, cls), "kl_profile_read")
        return list(dec[:cnt.value]), list(cls[:cnt.value])

    def kl_set_trace(self, trace_d=None) -> tuple[int, int, int]:
        a, b, c = C.c_uint32(), C.c_uint32(), C.c_uint32()
        _check(lib().kl_set_trace(self.handle, _ptr(trace_d), C.byref(a), C.byref(b), C.byref(c)), "kl_set_trace")
        return a.value, b.value, c.value

    def kl_stash_mode(self) -> int:
        return int(lib().kl_stash_mode(self.handle))

    def kl_set_tensor_core_attention(self, on: bool) -> None:
        _check(lib().kl_set_tensor_core_attention(self.handle, 1 if on else 0), "kl_set_tensor_core_attention")

    def kl_set_batched_path(self, on: bool) -> None:
        _check(lib().kl_set_batched_path(self.handle, 1 if on else 0), "kl_set_batched_path")

    def kl_set_dependent_launch(self, on: bool) -> None:
        _check(lib().kl_set_dependent_launch(self.handle, 1 if on else 0), "kl_set_dependent_launch")

    def kl_set_wait_limit_ns(self, ns: int) -> None:
        _check(lib().kl_set_wait_limit_ns(self.handle, ns), "kl_set_wait_limit_ns")

    def kl_debug_skip_signal_once(self, stage: int) -> None:
        _check(lib().kl_debug_skip_signal_once(self.handle, stage), "kl_debug_skip_signal_once")

    def kl_debug_set_jitter(self, seed: int, max_ns: int) -> None:
        _check(lib().kl_debug_set_jitter(self.handle, seed, max_ns), "kl_debug_set_jitter")

    def kl_debug_set_step(self, step: int | None = None) -> int:
        """Sets the step counter behind the tags (None: only queries); returns the step number at which it wraps."""
        w = C.c_uint32()
        _check(lib().kl_debug_set_step(self.handle, 0xffffffff if step is None else step, C.byref(w)), "kl_debug_set_step")
        return w.value

    # -- marshalling helpers
    def load_model(self, layer_weights, globals_, stream=None) -> None:
        """layer_weights(l) -> dict of bf16 tensors; globals_: dict with embed, norm_f, lm_head."""
        for l in range(self.shape.n_layers):
            for name, t in layer_weights(l).items():
                self.kl_load_weights(name, l, t, stream)
        for name in ("embed", "norm_f", "lm_head"):
            self.kl_load_weights(name, -1, globals_[name], stream)
        self.torch.cuda.synchronize()
