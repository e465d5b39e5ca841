"""Binding of the KV-cache calls: keys and values in pages, written, read back and attended to.

The calls have no backward pass: tensors that require grad are refused while gradients are on.  They are plain
functions, not registered operators, so dispatch modes and tracing do not see them.

`hos_kv_cache` checks a cache's tensors once and returns the handle that the other calls take.  The
batch is the same three device tensors everywhere (int32): `tok_off` [n_seq + 1], the packed new
tokens of every sequence; `kv_len` [n_seq], its tokens in the cache, the new ones included;
`page_table` [n_seq][>= pages], its pages in order.
"""
from __future__ import annotations

import ctypes as C
import importlib.util

from .binding import HosError, _torch, lib

HOS_KV_SAME, HOS_KV_E4M3, HOS_KV_INT8 = 0, 1, 2


STATUS_TOO_SHORT = 1                # of the compiled binding, not an error: more sequences than status words

_binding = _append = _read = _attention = None


def binding():
    """The compiled half of this module (_kv, built first if its source is newer), tied to the loaded library."""
    global _binding, _append, _read, _attention
    if _binding is None:
        from . import _build
        import torch  # noqa: F401  (its libraries have to be loaded first)
        L = lib()
        spec = importlib.util.spec_from_file_location("_kv", _build.build_binding())
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        m.init(*(C.cast(getattr(L, n), C.c_void_p).value for n in (
            "hos_kv_append", "hos_kv_read", "hos_paged_attention", "hos_paged_attention_workspace_bytes")))
        _binding, _append, _read, _attention = m, m.append, m.read, m.attention
    return _binding


class _KvCache(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("type", C.c_int32), ("format", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("page_stride", C.c_int64),
                ("scale_page_stride", C.c_int64)]


class _KvBatch(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("n_tokens", C.c_int32), ("max_new", C.c_int32), ("max_pages", C.c_int32),
                ("tok_off", C.c_void_p), ("kv_len", C.c_void_p), ("page_table", C.c_void_p), ("table_stride", C.c_int64)]


def _strided(t, want):
    """Whether t has these strides; that of a dimension of one means nothing."""
    return all(n == 1 or s == w for n, s, w in zip(t.shape[1:], t.stride()[1:], want))


class KvCache:
    """Handle of a paged cache: its tensors, checked, and the C description of them.

    `status` (int32, one word per sequence of the largest batch so far, 1,024 or the number of pages at least)
    collects the HOS_ST_* bits of the calls made with this handle until `status.zero_()`, on whatever streams and
    in whatever graphs they run."""

    def __init__(self, k, v, k_scale, v_scale, dtype):
        torch = _torch()
        formats = {torch.float8_e4m3fn: HOS_KV_E4M3, torch.int8: HOS_KV_INT8}
        types = {torch.bfloat16: 0, torch.float16: 1}
        for t, what in ((k, "k"), (v, "v")):
            if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 4):
                raise TypeError(f"{what}: expected a CUDA tensor [n_pages][n_kv_heads][page_size][head_dim]")
        if v.shape != k.shape or v.dtype != k.dtype or v.device != k.device or (k.shape[0] > 1 and v.stride(0) != k.stride(0)):
            raise ValueError("k and v must agree in shape, type, device and strides")
        self.format = formats.get(k.dtype, HOS_KV_SAME)
        dtype = dtype if dtype is not None else k.dtype
        if dtype not in types:
            raise TypeError("dtype: bfloat16 or float16 (give it for an 8-bit cache)")
        if self.format == HOS_KV_SAME and k.dtype != dtype:
            raise TypeError(f"k, v: expected {dtype}, float8_e4m3fn or int8")
        n_pages, n_kv, page, dim = k.shape
        if not (_strided(k, (page * dim, dim, 1)) and _strided(v, (page * dim, dim, 1))):
            raise ValueError("k, v: only the pages may be strided")
        if n_pages > 1 and k.stride(0) < n_kv * page * dim:      # 0, an expanded page, would mean densely packed pages below
            raise ValueError("k, v: pages must not overlap")
        scale_stride = 0
        if self.format != HOS_KV_SAME:
            for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
                if not (isinstance(t, torch.Tensor) and t.device == k.device and t.dtype == torch.float32):
                    raise TypeError(f"{what}: expected a CUDA tensor of float32")
                if tuple(t.shape) != (n_pages, n_kv, page) or not _strided(t, (page, 1)):
                    raise ValueError(f"{what}: expected [n_pages][n_kv_heads][page_size], strided by pages only")
            if n_pages > 1 and k_scale.stride(0) != v_scale.stride(0):
                raise ValueError("k_scale and v_scale must have the same strides")
            if n_pages > 1 and k_scale.stride(0) < n_kv * page:
                raise ValueError("k_scale, v_scale: pages must not overlap")
            scale_stride = k_scale.stride(0)
        elif k_scale is not None or v_scale is not None:
            raise ValueError("scales belong to an 8-bit cache")
        self.k, self.v, self.k_scale, self.v_scale, self.dtype = k, v, k_scale, v_scale, dtype
        self.n_kv_heads, self.page_size, self.head_dim, self.device = n_kv, page, dim, k.device
        self._earlier = []                 # shorter words, which calls in flight and captured graphs may still write to
        # a page's stride means nothing where there is one page
        dense = n_kv * page * dim
        self._c = _KvCache(n_pages, page, n_kv, dim, types[dtype], self.format, k.data_ptr(), v.data_ptr(),
                           k_scale.data_ptr() if k_scale is not None else None,
                           v_scale.data_ptr() if v_scale is not None else None,
                           k.stride(0) if n_pages > 1 else dense, scale_stride if n_pages > 1 else 0)
        self._h = binding().cache(C.addressof(self._c), k.get_device())
        self._new_status(max(1024, n_pages))

    def _new_status(self, n):
        torch = _torch()
        self._status = torch.zeros((n,), dtype=torch.int32, device=self.device)
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(self.device).synchronize()      # calls on other streams find zeros
        binding().set_status(self._h, self._status)

    def _grow_status(self, n_seq):
        if _torch().cuda.is_current_stream_capturing():               # words made here would be zeroed by every replay
            raise RuntimeError(f"{n_seq} sequences, status words for {self._status.shape[0]}: "
                               "make a call with the largest batch before a graph is captured")
        self._earlier.append(self._status)
        self._new_status(2 * n_seq)

    @property
    def status(self):
        if self._earlier:
            torch = _torch()
            torch.cuda.synchronize(self.device)
            for old in self._earlier:
                self._status[:old.shape[0]] |= old
                old.zero_()
            torch.cuda.synchronize(self.device)
        return self._status


def hos_kv_cache(k, v, k_scale=None, v_scale=None, dtype=None) -> KvCache:
    """Handle of the cache in tensors k, v [n_pages][n_kv_heads][page_size][head_dim]: bfloat16 or float16, or
    float8_e4m3fn or int8 with float32 scales [n_pages][n_kv_heads][page_size] and the `dtype` of the
    queries and outputs.  The tensors stay the caller's; the handle keeps them alive."""
    return KvCache(k, v, k_scale, v_scale, dtype)


def hos_kv_append(cache: KvCache, k, v, tok_off, kv_len, page_table):
    """Writes the new tokens' k and v [n_tokens][n_kv_heads][head_dim] (strided views are fine) to their
    places, quantised to the cache's format.  Returns {'status': the handle's words}."""
    rc = _append(cache._h, k, v, tok_off, kv_len, page_table)
    if rc == STATUS_TOO_SHORT:
        cache._grow_status(kv_len.shape[0])
        rc = _append(cache._h, k, v, tok_off, kv_len, page_table)
    if rc:
        raise HosError(rc, "hos_kv_append")
    return {"status": cache._status}


def hos_kv_read(cache: KvCache, tok_off, kv_len, page_table, n_tokens: int, out=None):
    """The batch's tokens (the last tok_off[s+1] - tok_off[s] of sequence s; n_tokens in all) from the cache,
    dequantised: {'k', 'v': [n_tokens][n_kv_heads][head_dim], 'status'}.  out: optional dense (k, v) to write into."""
    ok, ov = (None, None) if out is None else out
    rc, k, v = _read(cache._h, tok_off, kv_len, page_table, n_tokens, ok, ov)
    if rc == STATUS_TOO_SHORT:
        cache._grow_status(kv_len.shape[0])
        rc, k, v = _read(cache._h, tok_off, kv_len, page_table, n_tokens, ok, ov)
    if rc:
        raise HosError(rc, "hos_kv_read")
    return {"k": k, "v": v, "status": cache._status}


def hos_paged_attention(q, cache: KvCache, tok_off, kv_len, page_table, max_new: int, sm_scale=None, causal: bool = True,
                        window: int = 0, want_lse: bool = False, out=None, ws=None):
    """Attention of the batch's new tokens, q [n_tokens][n_heads][head_dim], to their sequences in the cache (which
    already holds the new tokens' own keys and values): {'out': like q, dense, 'lse': float32 [n_tokens][n_heads]
    or None, 'status'}.

    max_new: no sequence has more new tokens.  sm_scale: default 1 / sqrt(head_dim).  window > 0: a token sees
    the last `window` tokens up to itself.  out, ws: optional output tensor and workspace."""
    rc, o, lse = _attention(cache._h, q, tok_off, kv_len, page_table, max_new, sm_scale, causal, window, want_lse, out, ws)
    if rc == STATUS_TOO_SHORT:
        cache._grow_status(kv_len.shape[0])
        rc, o, lse = _attention(cache._h, q, tok_off, kv_len, page_table, max_new, sm_scale, causal, window, want_lse, out, ws)
    if rc:
        raise HosError(rc, "hos_paged_attention")
    return {"out": o, "lse": lse, "status": cache._status}
