"""ctypes binding of the calls around the paged key/value cache (include/shareprefill.h): argument marshalling.

These calls read device memory by lengths that are themselves on the device, so the tensors' types, sizes and devices are
checked here: a buffer of another size than the geometry says would be read past its end.  A call goes to the current stream
of the tensors' device.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import _check, lib

SP_PLAN_OK, SP_PLAN_BAD_LENGTH, SP_PLAN_TOO_LONG, SP_PLAN_NO_ROOM, SP_PLAN_NO_PAGES = range(5)


class SpCacheShape(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("stride_page", ctypes.c_int64), ("stride_token", ctypes.c_int64),
                ("stride_head", ctypes.c_int64)]


class SpRopeShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_tokens", "n_q_heads", "n_kv_heads", "head_dim", "rotary_dim",
                                              "interleaved")] + \
               [(n, ctypes.c_int64) for n in ("q_stride_t", "q_stride_h", "k_stride_t", "k_stride_h", "v_stride_t",
                                              "v_stride_h", "qo_stride_t", "qo_stride_h", "ko_stride_t", "ko_stride_h")] + \
               [("eps", ctypes.c_float)]


class SpStepShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_requests", "n_tokens", "n_q_heads", "max_new", "max_pages",
                                              "mask_words")] + \
               [(n, ctypes.c_int64) for n in ("q_stride_t", "q_stride_h", "o_stride_t", "o_stride_h")] + \
               [("softmax_scale", ctypes.c_float)]


def declare(L):
    """Argument types of the calls, for lib()."""
    vp = ctypes.c_void_p
    i32, i64, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    cache, rope, step = (ctypes.POINTER(c) for c in (SpCacheShape, SpRopeShape, SpStepShape))
    L.sp_cache_plan_workspace_bytes.restype = ctypes.c_int
    L.sp_cache_plan_workspace_bytes.argtypes = [i32, ctypes.POINTER(size)]
    L.sp_cache_plan.restype = ctypes.c_int
    L.sp_cache_plan.argtypes = [i32] * 4 + [vp] * 5 + [i32, vp, vp, i32] + [vp] * 9 + [size, vp]
    L.sp_qk_norm_rope.restype = ctypes.c_int
    L.sp_qk_norm_rope.argtypes = [rope] + [vp] * 9 + [cache] + [vp] * 4
    L.sp_cache_attn_workspace_bytes.restype = ctypes.c_int
    L.sp_cache_attn_workspace_bytes.argtypes = [step, cache, ctypes.POINTER(size)]
    L.sp_cache_attn.restype = ctypes.c_int
    L.sp_cache_attn.argtypes = [step, cache] + [vp] * 10 + [size, vp]
    L.sp_cache_accept.restype = ctypes.c_int
    L.sp_cache_accept.argtypes = [cache, i32, i64, vp, vp, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp]


_I32, _F32, _BF16, _U8, _I64 = torch.int32, torch.float32, torch.bfloat16, torch.uint8, torch.int64


def _dev(t, dtype, n: int, device: int, name: str):
    """Address of a contiguous tensor on `device` of at least n elements of `dtype`; None stays None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < n or t.get_device() != device or device < 0 or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous tensor of {n} or more {dtype} elements on the call's device is needed, got "
                         f"{tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _mask(t, n: int, device: int, name: str):
    """64-bit words: torch.int64, whose bits they are, or torch.uint64."""
    return _dev(t, _I64 if t is None or t.dtype is _I64 else torch.uint64, n, device, name)


def _rows(t, shape, strides, device: int, name: str):
    """Address of a bf16 tensor on `device` of this shape and these strides, its last dimension contiguous."""
    if t.dtype is not _BF16 or t.get_device() != device or device < 0 or t.shape != shape or t.stride() != strides and (
            t.stride(-1) != 1 or any(a > 1 and b != c for a, b, c in zip(shape, t.stride(), strides))):
        raise ValueError(f"{name}: a bf16 tensor of shape {shape} and strides {strides} on the call's device is needed, got "
                         f"{tuple(t.shape)} {tuple(t.stride())} {t.dtype} on {t.device}")
    return t.data_ptr()


# The current stream's handle without a Stream object around it: 0.06 us of a call's 9 instead of 2.5.
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device  # 0.05 us instead of 0.2; a tensor is there


def _call(fn, device: int, *args):
    """fn(*args, stream) on the current stream of `device`."""
    if device == _current_device():
        _check(fn(*args, _stream_of(device)))
    else:
        with torch.cuda.device(device):
            _check(fn(*args, _stream_of(device)))


def cache_shape_of(cache) -> SpCacheShape:
    """sp_cache_shape of a cache tensor [pages][page_size][hkv][d] (any strides, d contiguous): of the keys' and the values'."""
    assert cache.dim() == 4 and cache.stride(3) == 1
    s = SpCacheShape()
    s.n_pages, s.page_size, s.n_kv_heads, s.head_dim = cache.shape
    s.stride_page, s.stride_token, s.stride_head = cache.stride(0), cache.stride(1), cache.stride(2)
    return s


def rope_shape_of(q, k, v, q_out, k_out, rotary_dim: int, interleaved: bool = False, eps: float = 1e-6) -> SpRopeShape:
    """sp_rope_shape for token-major tensors q, q_out [tokens][hq][d], k, v, k_out [tokens][hkv][d] (any strides, d
    contiguous); v and k_out may be None."""
    v, k_out = k if v is None else v, k if k_out is None else k_out
    assert all(x.dim() == 3 and x.stride(2) == 1 for x in (q, k, v, q_out, k_out))
    s = SpRopeShape()
    s.n_tokens, s.n_q_heads, s.head_dim = q.shape
    s.n_kv_heads, s.rotary_dim, s.interleaved, s.eps = k.shape[1], rotary_dim, 1 if interleaved else 0, eps
    s.q_stride_t, s.q_stride_h = q.stride(0), q.stride(1)
    s.k_stride_t, s.k_stride_h = k.stride(0), k.stride(1)
    s.v_stride_t, s.v_stride_h = v.stride(0), v.stride(1)
    s.qo_stride_t, s.qo_stride_h = q_out.stride(0), q_out.stride(1)
    s.ko_stride_t, s.ko_stride_h = k_out.stride(0), k_out.stride(1)
    return s


def step_shape_of(q, o, block_table, max_new: int, mask_words: int = 0, softmax_scale: float = 0.0) -> SpStepShape:
    """sp_step_shape for packed tokens q, o [tokens][hq][d] (any strides, d contiguous) and block_table [requests][pages]."""
    assert q.dim() == 3 and o.dim() == 3 and q.stride(2) == 1 and o.stride(2) == 1
    s = SpStepShape()
    s.n_requests, s.max_pages = block_table.shape
    s.n_tokens, s.n_q_heads = q.shape[0], q.shape[1]
    s.max_new, s.mask_words, s.softmax_scale = max_new, mask_words, softmax_scale
    s.q_stride_t, s.q_stride_h = q.stride(0), q.stride(1)
    s.o_stride_t, s.o_stride_h = o.stride(0), o.stride(1)
    return s


def _cache_rows(s: SpCacheShape, cache, device: int, name: str):
    return _rows(cache, (s.n_pages, s.page_size, s.n_kv_heads, s.head_dim), (s.stride_page, s.stride_token, s.stride_head, 1),
                 device, name)


def sp_cache_plan_workspace_bytes(n_requests: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().sp_cache_plan_workspace_bytes(n_requests, ctypes.byref(n)))
    return int(n.value)


def sp_cache_plan(ctx_len, new_len, n_held, block_table, free_pages, n_free, page_size: int, parents, n_held_out, n_free_out,
                  tok_start, seq_len, positions, slots, status, tree_mask, workspace):
    """block_table [requests][max_pages]; max_tokens is the length of positions and slots; tree_mask [max_tokens][words] or None."""
    (n, width), dev = block_table.shape, block_table.get_device()
    tokens, words = positions.numel(), 0 if tree_mask is None else tree_mask.shape[1]
    _call(lib().sp_cache_plan, dev, n, tokens, page_size, width, _dev(ctx_len, _I32, n, dev, "ctx_len"),
          _dev(new_len, _I32, n, dev, "new_len"), _dev(n_held, _I32, n, dev, "n_held"),
          _dev(block_table, _I32, n * width, dev, "block_table"), _dev(free_pages, _I32, 0, dev, "free_pages"),
          free_pages.numel(), _dev(n_free, _I32, 1, dev, "n_free"), _dev(parents, _I32, tokens, dev, "parents"), words,
          _dev(n_held_out, _I32, n, dev, "n_held_out"), _dev(n_free_out, _I32, 1, dev, "n_free_out"),
          _dev(tok_start, _I32, n + 1, dev, "tok_start"), _dev(seq_len, _I32, n, dev, "seq_len"),
          _dev(positions, _I32, tokens, dev, "positions"), _dev(slots, _I32, tokens, dev, "slots"),
          _dev(status, _I32, n, dev, "status"), _mask(tree_mask, tokens * words, dev, "tree_mask"),
          _dev(workspace, _U8, 0, dev, "workspace"), workspace.numel())


def sp_qk_norm_rope(shape: SpRopeShape, q, k, v, q_weight, k_weight, inv_freq, positions, q_out, k_out, cache=None,
                    k_cache=None, v_cache=None, slots=None):
    """cache: the sp_cache_shape of k_cache and v_cache, or None."""
    s, c, dev = shape, cache, q.get_device()
    n, d = s.n_tokens, s.head_dim
    qs, ks = (n, s.n_q_heads, d), (n, s.n_kv_heads, d)
    if s.rotary_dim and (inv_freq is None or positions is None):
        raise ValueError("rotary_dim needs inv_freq and positions")
    at_v = at_kc = at_vc = at_slots = at_c = None
    if c is not None:
        if v is None or k_cache is None or v_cache is None or slots is None:
            raise ValueError("a cache needs v, k_cache, v_cache and slots")
        at_c = ctypes.byref(c)
        at_v = _rows(v, ks, (s.v_stride_t, s.v_stride_h, 1), dev, "v")
        at_kc, at_vc = _cache_rows(c, k_cache, dev, "k_cache"), _cache_rows(c, v_cache, dev, "v_cache")
        at_slots = _dev(slots, _I32, n, dev, "slots")
    _call(lib().sp_qk_norm_rope, dev, ctypes.byref(s), _rows(q, qs, (s.q_stride_t, s.q_stride_h, 1), dev, "q"),
          _rows(k, ks, (s.k_stride_t, s.k_stride_h, 1), dev, "k"), at_v, _dev(q_weight, _BF16, d, dev, "q_weight"),
          _dev(k_weight, _BF16, d, dev, "k_weight"), _dev(inv_freq, _F32, s.rotary_dim // 2, dev, "inv_freq"),
          _dev(positions, _I32, n, dev, "positions"), _rows(q_out, qs, (s.qo_stride_t, s.qo_stride_h, 1), dev, "q_out"),
          None if k_out is None else _rows(k_out, ks, (s.ko_stride_t, s.ko_stride_h, 1), dev, "k_out"), at_c, at_kc, at_vc, at_slots)


def sp_cache_attn_workspace_bytes(shape: SpStepShape, cache: SpCacheShape) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().sp_cache_attn_workspace_bytes(ctypes.byref(shape), ctypes.byref(cache), ctypes.byref(n)))
    return int(n.value)


def sp_cache_attn(shape: SpStepShape, cache: SpCacheShape, q, k_cache, v_cache, block_table, seq_len, tok_start, tree_mask, o,
                  lse, workspace):
    """tree_mask None with mask_words 0; lse None: not wanted."""
    s, dev = shape, q.get_device()
    if tree_mask is not None and tree_mask.shape[-1] != s.mask_words:
        raise ValueError(f"tree_mask has {tree_mask.shape[-1]} words a token, the shape {s.mask_words}")
    n, rows = s.n_requests, (s.n_tokens, s.n_q_heads, cache.head_dim)
    _call(lib().sp_cache_attn, dev, ctypes.byref(s), ctypes.byref(cache), _rows(q, rows, (s.q_stride_t, s.q_stride_h, 1), dev, "q"),
          _cache_rows(cache, k_cache, dev, "k_cache"), _cache_rows(cache, v_cache, dev, "v_cache"),
          _dev(block_table, _I32, n * s.max_pages, dev, "block_table"), _dev(seq_len, _I32, n, dev, "seq_len"),
          _dev(tok_start, _I32, n + 1, dev, "tok_start"), _mask(tree_mask, s.n_tokens * s.mask_words, dev, "tree_mask"),
          _rows(o, rows, (s.o_stride_t, s.o_stride_h, 1), dev, "o"), _dev(lse, _F32, s.n_tokens * s.n_q_heads, dev, "lse"),
          _dev(workspace, _U8, 0, dev, "workspace"), workspace.numel())


def sp_cache_accept(cache: SpCacheShape, k_cache, v_cache, block_table, ctx_len, seq_len, path, n_accepted, ctx_out=None):
    """k_cache, v_cache: [layers][pages][page_size][hkv][d], or one layer's four dimensions; path [requests][max_accept]."""
    dev, dims, c = k_cache.get_device(), k_cache.dim(), cache
    layers, stride = (1, 0) if dims == 4 else (k_cache.shape[0], k_cache.stride(0))
    (n, width), most = block_table.shape, path.shape[1]
    if v_cache.dim() != dims or dims == 5 and (v_cache.shape[0] != layers or layers > 1 and v_cache.stride(0) != stride):
        raise ValueError("k_cache and v_cache need one geometry")
    shape, strides = (c.n_pages, c.page_size, c.n_kv_heads, c.head_dim), (c.stride_page, c.stride_token, c.stride_head, 1)
    if dims == 5:  # (a layer's view of its own, to look at, would cost a microsecond)
        shape, strides = (layers, *shape), (stride, *strides)
    at = _rows(k_cache, shape, strides, dev, "k_cache"), _rows(v_cache, shape, strides, dev, "v_cache")
    _call(lib().sp_cache_accept, dev, ctypes.byref(cache), layers, stride, at[0], at[1], n, width,
          _dev(block_table, _I32, n * width, dev, "block_table"), _dev(ctx_len, _I32, n, dev, "ctx_len"),
          _dev(seq_len, _I32, n, dev, "seq_len"), most, _dev(path, _I32, n * most, dev, "path"),
          _dev(n_accepted, _I32, n, dev, "n_accepted"), _dev(ctx_out, _I32, n, dev, "ctx_out"))
