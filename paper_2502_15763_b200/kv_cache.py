"""Binding of the KV-cache calls: keys and values in pages, written, read back and attended to.

`hos_kv_cache` checks a cache's tensors once and returns the handle that the other calls take.  The
batch is the same three device tensors everywhere (int32): `tok_off` [n_seq + 1], the packed new
tokens of every sequence; `kv_len` [n_seq], its tokens in the cache, the new ones included;
`page_table` [n_seq][>= pages], its pages in order.
"""
from __future__ import annotations

import ctypes as C
import math

from .binding import HosError, _torch, lib

HOS_KV_SAME, HOS_KV_E4M3, HOS_KV_INT8 = 0, 1, 2


class _KvCache(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("type", C.c_int32), ("format", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("page_stride", C.c_int64),
                ("scale_page_stride", C.c_int64)]


class _KvBatch(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("n_tokens", C.c_int32), ("max_new", C.c_int32), ("max_pages", C.c_int32),
                ("tok_off", C.c_void_p), ("kv_len", C.c_void_p), ("page_table", C.c_void_p), ("table_stride", C.c_int64)]


class KvCache:
    """Handle of a paged cache: its tensors, checked, and the C description of them.

    `status` (int32, one word per sequence of the largest batch so far) collects the HOS_ST_* bits of the
    calls made with this handle until `status.zero_()`."""

    def __init__(self, k, v, k_scale, v_scale, dtype):
        torch = _torch()
        formats = {torch.float8_e4m3fn: HOS_KV_E4M3, torch.int8: HOS_KV_INT8}
        types = {torch.bfloat16: 0, torch.float16: 1}
        for t, what in ((k, "k"), (v, "v")):
            if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 4):
                raise TypeError(f"{what}: expected a CUDA tensor [n_pages][n_kv_heads][page_size][head_dim]")
        if v.shape != k.shape or v.dtype != k.dtype or v.device != k.device or v.stride() != k.stride():
            raise ValueError("k and v must agree in shape, type, device and strides")
        self.format = formats.get(k.dtype, HOS_KV_SAME)
        dtype = dtype if dtype is not None else k.dtype
        if dtype not in types:
            raise TypeError("dtype: bfloat16 or float16 (give it for an 8-bit cache)")
        if self.format == HOS_KV_SAME and k.dtype != dtype:
            raise TypeError(f"k, v: expected {dtype}, float8_e4m3fn or int8")
        n_pages, n_kv, page, dim = k.shape
        if tuple(k.stride()[1:]) != (page * dim, dim, 1):
            raise ValueError("k, v: only the pages may be strided")
        scale_stride = 0
        if self.format != HOS_KV_SAME:
            for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
                if not (isinstance(t, torch.Tensor) and t.device == k.device and t.dtype == torch.float32):
                    raise TypeError(f"{what}: expected a CUDA tensor of float32")
                if tuple(t.shape) != (n_pages, n_kv, page) or tuple(t.stride()[1:]) != (page, 1):
                    raise ValueError(f"{what}: expected [n_pages][n_kv_heads][page_size], strided by pages only")
            if k_scale.stride(0) != v_scale.stride(0):
                raise ValueError("k_scale and v_scale must have the same strides")
            scale_stride = k_scale.stride(0)
        elif k_scale is not None or v_scale is not None:
            raise ValueError("scales belong to an 8-bit cache")
        self._torch, self._lib, self._index = torch, lib(), k.get_device()
        self._raw_stream = torch._C._cuda_getCurrentRawStream
        self.k, self.v, self.k_scale, self.v_scale, self.dtype = k, v, k_scale, v_scale, dtype
        self.n_kv_heads, self.page_size, self.head_dim, self.device = n_kv, page, dim, k.device
        self._status_len = 256
        self.status = torch.zeros((self._status_len,), dtype=torch.int32, device=k.device)
        # a page's stride means nothing where there is one page
        dense = n_kv * page * dim
        self._c = _KvCache(n_pages, page, n_kv, dim, types[dtype], self.format, k.data_ptr(), v.data_ptr(),
                           k_scale.data_ptr() if k_scale is not None else None,
                           v_scale.data_ptr() if v_scale is not None else None,
                           k.stride(0) if n_pages > 1 else dense, scale_stride if n_pages > 1 else 0)
        self._ref = C.byref(self._c)
        self._default_scale = 1.0 / math.sqrt(dim)
        self._ws_bytes = {}                            # heads -> workspace size

    # The checks below run in every call of a serving loop: straight-line code, no repeated look-ups.
    def _batch(self, tok_off, kv_len, page_table, n_tokens, max_new):
        i32, dev = self._torch.int32, self._index
        if not (tok_off.dtype is i32 and kv_len.dtype is i32 and page_table.dtype is i32 and tok_off.get_device() == dev
                and kv_len.get_device() == dev and page_table.get_device() == dev):
            raise TypeError("tok_off, kv_len, page_table: expected int32 tensors on the cache's device")
        if tok_off.dim() != 1 or kv_len.dim() != 1 or page_table.dim() != 2:
            raise ValueError("tok_off and kv_len must have one dimension, page_table two")
        n_seq, width = page_table.shape
        if tok_off.shape[0] != n_seq + 1 or kv_len.shape[0] != n_seq:
            raise ValueError("tok_off must have n_seq + 1 entries, kv_len n_seq, page_table n_seq rows")
        row, col = page_table.stride()
        if (col != 1 and width > 1) or not tok_off.is_contiguous() or not kv_len.is_contiguous():
            raise ValueError("tok_off, kv_len and the rows of page_table must be dense")
        if n_seq > self._status_len:
            self._grow_status(n_seq)
        return _KvBatch(n_seq, n_tokens, max_new, width, tok_off.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(),
                        row if n_seq > 1 else width)

    def _grow_status(self, n_seq):
        old = self.status
        self._status_len = 2 * n_seq
        self.status = self._torch.zeros((self._status_len,), dtype=self._torch.int32, device=self.device)
        self.status[:old.shape[0]] = old

    def _rows(self, t, what):
        """Strides of a [tokens][heads][head_dim] tensor of the cache's type; its shape and strides checked."""
        if t.dtype is not self.dtype or t.get_device() != self._index:
            raise TypeError(f"{what}: expected a tensor of {self.dtype} on the cache's device")
        if t.dim() != 3 or t.shape[2] != self.head_dim:
            raise ValueError(f"{what}: expected [tokens][heads][{self.head_dim}]")
        tok, head, one = t.stride()
        if one != 1:
            raise ValueError(f"{what}: the elements of a head must be dense")
        return tok, head


def hos_kv_cache(k, v, k_scale=None, v_scale=None, dtype=None) -> KvCache:
    """Handle of the cache in tensors k, v [n_pages][n_kv_heads][page_size][head_dim]: bfloat16 or float16, or
    float8_e4m3fn or int8 with float32 scales [n_pages][n_kv_heads][page_size] and the `dtype` of the
    queries and outputs.  The tensors stay the caller's; the handle keeps them alive."""
    return KvCache(k, v, k_scale, v_scale, dtype)


def hos_kv_append(cache: KvCache, k, v, tok_off, kv_len, page_table):
    """Writes the new tokens' k and v [n_tokens][n_kv_heads][head_dim] (strided views are fine) to their
    places, quantised to the cache's format.  Returns {'status': the handle's words}."""
    k_tok, k_head = cache._rows(k, "k")
    v_tok, v_head = cache._rows(v, "v")
    n_tok = k.shape[0]
    if k.shape[1] != cache.n_kv_heads or v.shape[1] != cache.n_kv_heads or v.shape[0] != n_tok:
        raise ValueError("k and v must be [n_tokens][n_kv_heads][head_dim]")
    b = cache._batch(tok_off, kv_len, page_table, n_tok, n_tok)
    rc = cache._lib.hos_kv_append(cache._ref, C.byref(b), k.data_ptr(), v.data_ptr(), k_tok, k_head, v_tok, v_head,
                                  cache.status.data_ptr(), cache._raw_stream(cache._index))
    if rc:
        raise HosError(rc, "hos_kv_append")
    return {"status": cache.status}


def hos_kv_read(cache: KvCache, tok_off, kv_len, page_table, n_tokens: int, out=None):
    """The batch's tokens (the last tok_off[s+1] - tok_off[s] of sequence s; n_tokens in all) from the cache,
    dequantised: {'k', 'v': [n_tokens][n_kv_heads][head_dim], 'status'}.  out: optional dense (k, v) to write into."""
    shape = (int(n_tokens), cache.n_kv_heads, cache.head_dim)
    if out is None:
        k, v = cache.k.new_empty(shape, dtype=cache.dtype), cache.k.new_empty(shape, dtype=cache.dtype)
    else:
        k, v = out
        cache._rows(k, "out")
        cache._rows(v, "out")
        if tuple(k.shape) != shape or tuple(v.shape) != shape or not (k.is_contiguous() and v.is_contiguous()):
            raise ValueError("out tensors must be dense [n_tokens][n_kv_heads][head_dim]")
    b = cache._batch(tok_off, kv_len, page_table, shape[0], shape[0])
    rc = cache._lib.hos_kv_read(cache._ref, C.byref(b), k.data_ptr(), v.data_ptr(), cache.status.data_ptr(),
                                cache._raw_stream(cache._index))
    if rc:
        raise HosError(rc, "hos_kv_read")
    return {"k": k, "v": v, "status": cache.status}


def hos_paged_attention(q, cache: KvCache, tok_off, kv_len, page_table, max_new: int, sm_scale=None, causal: bool = True,
                        window: int = 0, want_lse: bool = False, out=None, ws=None):
    """Attention of the batch's new tokens, q [n_tokens][n_heads][head_dim], to their sequences in the cache (which
    already holds the new tokens' own keys and values): {'out': like q, dense, 'lse': float32 [n_tokens][n_heads]
    or None, 'status'}.

    max_new: no sequence has more new tokens.  sm_scale: default 1 / sqrt(head_dim).  window > 0: a token sees
    the last `window` tokens up to itself.  out, ws: optional output tensor and workspace."""
    torch, L = cache._torch, cache._lib
    q_tok, q_head = cache._rows(q, "q")
    n_tok, heads, dim = q.shape
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        o_tok, o_head = heads * dim, dim
    else:
        o_tok, o_head = cache._rows(out, "out")
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    lse = q.new_empty((n_tok, heads), dtype=torch.float32) if want_lse else None
    b = cache._batch(tok_off, kv_len, page_table, n_tok, int(max_new))
    need = cache._ws_bytes.get(heads)
    if need is None:
        need = cache._ws_bytes[heads] = max(L.hos_paged_attention_workspace_bytes(cache._ref, C.byref(b), heads), 256)
    if ws is None or ws.numel() < need:
        ws = q.new_empty(need, dtype=torch.uint8)
    rc = L.hos_paged_attention(cache._ref, C.byref(b), q.data_ptr(), q_tok, q_head, heads,
                               cache._default_scale if sm_scale is None else sm_scale, causal, window, out.data_ptr(), o_tok,
                               o_head, lse.data_ptr() if want_lse else None, cache.status.data_ptr(), ws.data_ptr(), need,
                               cache._raw_stream(cache._index))
    if rc:
        raise HosError(rc, "hos_paged_attention")
    return {"out": out, "lse": lse, "status": cache.status}
