"""Binding of the calls on a cache's pages and on drafted tokens.

Whose pages are whose is three int32 tensors: `refs` [n_pages], the number of page-table entries that hold each page
(0: free); `page_table` [n_seq][pages]; `kv_len` [n_seq].  A pool begins as zeros.  `hos_kv_resize`, `hos_kv_fork` and
`hos_kv_compact` return the new state as tensors of their own, or write it to `out` = (refs, page_table, kv_len), which
for hos_kv_resize and hos_kv_compact may be the old ones (and must not overlap with them otherwise).  A drafted decode round:

    r = hos_kv_resize(refs, table, kv_len, kv_len + 1 + drafts, page_size)
    hos_kv_copy_pages(caches, r["src"], r["dst"], r["count"])        # pages that were shared and are about to be written
    ...                                                              # append and attend, layer by layer
    v = hos_verify_drafts(tokens, target, draft, tok_off, u_accept, u_sample, kv_len=r["kv_len"])
    r = hos_kv_resize(r["refs"], r["page_table"], r["kv_len"], v["new_len"], page_size)

Everything stays on the device, so a round can be captured into a graph.  Like the other calls of the cache these are plain
functions without a backward pass.  The results of a call lie in one allocation: whoever keeps one of them (the status, say) keeps
the memory of all, the table and a workspace of up to 12 bytes a page and 12 a sequence included, and torch.save writes all of it;
clone what is kept for long.
"""
from __future__ import annotations

from . import kv_cache
from .binding import HosError
from .kv_cache import STATUS_TOO_SHORT, KvCache


def _compiled():
    return kv_cache._binding or kv_cache.binding()


def _checked(r, where):
    if type(r) is int:
        raise HosError(r, where)
    return r


def hos_kv_resize(refs, page_table, kv_len, new_len, page_size: int, out=None):
    """Sequences get the lengths new_len [n_seq]: pages past the new ends are given up, the lowest-numbered free ones
    taken; a sequence that grows inside a page which others hold as well gets one of its own for it.

    Returns the new state {'refs', 'page_table', 'kv_len'}, the page copies to be made before the next append
    {'src', 'dst': int32 [n_seq], 'count': int32 [1]} and 'status' [n_seq] (HOS_ST_PAGES: too few free pages, the
    sequence and all growing ones after it keep their lengths; HOS_ST_INVALID: a length or a page number out of range, or a
    page given up whose count comes out below zero)."""
    return _checked(_compiled().resize(refs, page_table, kv_len, new_len, page_size, out), "hos_kv_resize")


def hos_kv_fork(refs, page_table, kv_len, parent, page_size: int, out=None):
    """Sequence i of the new state holds what sequence parent[i] of the old one holds (-1: nothing); any number of them.

    Returns {'refs', 'page_table', 'kv_len', 'status' [len(parent)]}; in `out` only refs may be the old tensor."""
    return _checked(_compiled().fork(refs, page_table, kv_len, parent, page_size, out), "hos_kv_fork")


def hos_kv_compact(refs, page_table, kv_len, page_size: int, out=None):
    """Moves the pages in use to the front of the pool.

    Returns {'refs', 'page_table', 'kv_len' (the tensor that was given), 'src', 'dst': int32 [n_pages], 'count': int32 [1], 'status' [n_seq]}
    (HOS_ST_INVALID: a length out of range, or the sequence holds a page that refs says is free)."""
    return _checked(_compiled().compact(refs, page_table, kv_len, None, page_size, out), "hos_kv_compact")


def hos_kv_copy_pages(caches, src, dst, count=None, source=None):
    """Copies pages src[i] to pages dst[i] (int32) of a cache, or of several layers' caches in one call: keys, values, scales.

    count: int32 [1] on the device, only the first of them.  source: the cache or caches to read from, if they are others.
    A page must not be written twice, nor written and read.  Returns {'status'}: words of the first cache's handle, one
    for each i (HOS_ST_INVALID: a page number out of range)."""
    caches = [caches] if isinstance(caches, KvCache) else list(caches)
    source = caches if source is None else [source] if isinstance(source, KvCache) else list(source)
    try:
        to, of = [c._h for c in caches], [c._h for c in source]
    except AttributeError:
        raise TypeError("caches, source: expected handles made by hos_kv_cache") from None
    call = _compiled().copy_pages
    rc = call(to, of, src, dst, count)
    if rc == STATUS_TOO_SHORT:
        caches[0]._grow_status(src.shape[0])
        rc = call(to, of, src, dst, count)
    if rc:
        raise HosError(rc, "hos_kv_copy_pages")
    return {"status": caches[0]._status}


def hos_verify_drafts(tokens, target, draft, tok_off, u_accept, u_sample, kv_len=None):
    """Which drafted tokens the target keeps, and the token after them.

    tokens: int32 [n_tokens], packed by tok_off [n_seq + 1] as in the round's attention call: of every sequence the token it
    had, then its drafts.  target, draft: probabilities [n_tokens][vocab] (float32, bfloat16 or float16; rows may be strided):
    row r of target is the distribution after token r, row r of draft the one that tokens[r + 1] was drawn from; draft None: the
    drafts were not drawn.  u_accept [n_tokens], u_sample [n_seq]: float32 in [0, 1).  Rows of target and draft whose addresses
    differ modulo 16 bytes are read more slowly (by a tenth to a half).

    Returns int32 {'accepted' [n_seq], 'next' [n_seq], 'tokens' [n_tokens]: the accepted drafts, next, then -1 (rows of no
    sequence are not written), 'new_len' [n_seq]: kv_len without the drafts that were not accepted, or None, 'status' [n_seq]}."""
    return _checked(_compiled().verify(tokens, target, draft, tok_off, u_accept, u_sample, kv_len), "hos_verify_drafts")
