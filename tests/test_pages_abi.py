"""Host-side checks of the calls on pages and drafts: they come before any CUDA call, so they are testable without a device."""
import ctypes as C

import pytest

import paper_2502_15763_b200 as hos
from paper_2502_15763_b200.kv_cache import _KvCache

I32, P, I64 = C.c_int32, C.c_void_p, C.c_int64


class Pages(C.Structure):
    _fields_ = [("n_pages", I32), ("page_size", I32), ("n_seq", I32), ("max_pages", I32), ("refs", P), ("kv_len", P), ("page_table", P), ("table_stride", I64)]


class Moves(C.Structure):
    _fields_ = [("src", P), ("dst", P), ("count", P)]


class Drafts(C.Structure):
    _fields_ = [("n_seq", I32), ("n_tokens", I32), ("vocab", I32), ("type", I32), ("tok_off", P), ("tokens", P), ("target", P), ("draft", P),
                ("target_stride", I64), ("draft_stride", I64), ("u_accept", P), ("u_sample", P), ("kv_len", P), ("accepted", P), ("next", P),
                ("out_tokens", P), ("new_len", P), ("status", P)]


STATE = dict(n_pages=100, page_size=16, n_seq=4, max_pages=8, refs=4096, kv_len=8192, page_table=12288, table_stride=8)
OTHER = dict(STATE, refs=4096 * 8, kv_len=8192 * 8, page_table=12288 * 8)
MOVES = dict(src=256, dst=512, count=768)


def call(name, a=None, b=None, moves=None, change=1024, ws=1 << 20, ws_bytes=0):
    L = hos.lib()
    x, y, m = Pages(**{**STATE, **(a or {})}), Pages(**{**OTHER, **(b or {})}), Moves(**{**MOVES, **(moves or {})})
    if name == "resize":
        return L.hos_kv_resize(C.byref(x), change, C.byref(y), C.byref(m), None, ws, ws_bytes, None)
    if name == "fork":
        return L.hos_kv_fork(C.byref(x), change, C.byref(y), None, None)
    return L.hos_kv_compact(C.byref(x), C.byref(y), C.byref(m), None, ws, ws_bytes, None)


CALLS = ["resize", "fork", "compact"]


@pytest.mark.parametrize("name", ["resize", "compact"])
def test_good_arguments_get_as_far_as_the_workspace(name):
    L = hos.lib()
    need = getattr(L, f"hos_kv_{name}_workspace_bytes")(C.byref(Pages(**STATE)))
    assert need > 0 and need % 256 == 0
    assert call(name) == -2 and call(name, ws=None, ws_bytes=need) == -2
    assert call(name, ws_bytes=need - 1) == -2 and call(name, ws=(1 << 20) + 128, ws_bytes=need) == -2


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("change,code", [
    (dict(n_pages=0), -1), (dict(n_pages=-1), -1), (dict(page_size=0), -1), (dict(n_seq=-1), -1), (dict(max_pages=-1), -1), (dict(refs=None), -1),
    (dict(page_table=None), -1), (dict(table_stride=7), -1), (dict(n_pages=(1 << 24) + 1), -4), (dict(n_seq=(1 << 18) + 1), -4),
    (dict(page_size=1 << 28), -4), (dict(max_pages=1 << 27, table_stride=1 << 27), -4)])
def test_state_refusals(name, change, code):
    assert call(name, a=change, b=change) == code
    if code == -1 and set(change) <= {"refs", "page_table", "table_stride"}:
        assert call(name, a=change) == -1 and call(name, b=change) == -1


def test_states_that_do_not_belong_together():
    for name in CALLS:
        for change in (dict(n_pages=99), dict(page_size=32), dict(max_pages=7)):
            assert call(name, b=change) == -1
    assert call("resize", b=dict(n_seq=5)) == -1 and call("compact", b=dict(n_seq=3)) == -1
    # the table in its own place, but with rows elsewhere
    for name in ("resize", "compact"):
        assert call(name, b=dict(page_table=STATE["page_table"], table_stride=9)) == -1
        assert call(name, b=dict(page_table=STATE["page_table"])) == -2
    assert call("fork", b=dict(page_table=STATE["page_table"])) == -1 and call("fork", b=dict(kv_len=STATE["kv_len"])) == -1


def test_null_arguments():
    L = hos.lib()
    x, m = Pages(**STATE), Moves(**MOVES)
    assert L.hos_kv_resize(None, 1024, C.byref(x), C.byref(m), None, None, 0, None) == -1
    assert L.hos_kv_resize(C.byref(x), 1024, None, C.byref(m), None, None, 0, None) == -1
    assert L.hos_kv_resize(C.byref(x), 1024, C.byref(x), None, None, None, 0, None) == -1
    assert L.hos_kv_fork(None, 1024, C.byref(x), None, None) == -1 and L.hos_kv_compact(C.byref(x), None, C.byref(m), None, None, 0, None) == -1
    for name in ("resize", "compact"):
        assert getattr(L, f"hos_kv_{name}_workspace_bytes")(None) == 0
    assert call("resize", change=None) == -1 and call("fork", change=None) == -1
    for k in MOVES:
        assert call("resize", moves={k: None}) == -1 and call("compact", moves={k: None}) == -1
    assert call("resize", a=dict(kv_len=None)) == -1 and call("resize", b=dict(kv_len=None)) == -1 and call("compact", a=dict(kv_len=None)) == -1
    assert call("compact", b=dict(kv_len=None)) == -2


CACHE = dict(n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, type=0, format=0, k=4096, v=8192, k_scale=None, v_scale=None, page_stride=0,
             scale_page_stride=0)


def copy(to=None, of=None, layers=1, src=256, dst=256, n=0):
    a, b = ((_KvCache * 2)(_KvCache(**CACHE), _KvCache(**{**CACHE, **(x or {})})) for x in (to, of))
    at = C.sizeof(_KvCache) if layers == 1 else 0
    return hos.lib().hos_kv_copy_pages(C.addressof(a) + at, C.addressof(b) + at, layers, src, dst, None, n, None, None)


@pytest.mark.parametrize("change,code", [
    (dict(k=None), -1), (dict(n_pages=0), -1), (dict(n_kv_heads=0), -1), (dict(type=2), -1), (dict(format=3), -1), (dict(format=1), -1),
    (dict(head_dim=96), -4), (dict(page_size=8), -4), (dict(page_size=24), -4), (dict(page_stride=100), -1), (dict(page_stride=2 * 16 * 64 + 4), -1),
    (dict(k=4100), -1), (dict(format=2, k_scale=256, v_scale=260), -1), (dict(format=2, k_scale=256, v_scale=256, scale_page_stride=34), -1),
    (dict(n_kv_heads=1 << 20), -4)])
def test_copy_refusals(change, code):
    assert copy() == 0 and copy(layers=2) == 0
    assert copy(to=change, of=change) == code
    assert copy(of=change) == code and copy(to=change) == code


def test_copies_between_caches_that_differ():
    for change in (dict(page_size=32), dict(n_kv_heads=1), dict(head_dim=128), dict(type=1), dict(format=2, k_scale=256, v_scale=256)):
        assert copy(to=change) == -1 and copy(of=change) == -1
        assert copy(to=change, of=change, layers=2) == -1
    assert copy(to=dict(n_pages=5)) == 0 and copy(to=dict(n_pages=5), layers=2) == -1
    assert copy(layers=0) == -1 and copy(n=-1) == -1 and copy(n=1, src=None) == -1 and copy(n=1, dst=None) == -1
    assert hos.lib().hos_kv_copy_pages(None, None, 1, 256, 256, None, 0, None, None) == -1


DRAFTS = dict(n_seq=1, n_tokens=2, vocab=10, type=2, tok_off=256, tokens=256, target=256, draft=256, target_stride=10, draft_stride=10, u_accept=256,
              u_sample=256, kv_len=256, accepted=256, next=256, out_tokens=256, new_len=256, status=256)


@pytest.mark.parametrize("change,code", [
    (dict(n_seq=-1), -1), (dict(n_tokens=-1), -1), (dict(vocab=0), -1), (dict(type=3), -1), (dict(type=-1), -1), (dict(tok_off=None), -1),
    (dict(tokens=None), -1), (dict(target=None), -1), (dict(u_accept=None), -1), (dict(u_sample=None), -1), (dict(accepted=None), -1), (dict(next=None), -1),
    (dict(out_tokens=None), -1), (dict(kv_len=None), -1), (dict(new_len=None), -1), (dict(target=258), -1), (dict(draft=257), -1),
    (dict(type=0, target=257), -1), (dict(target_stride=-1), -1), (dict(draft_stride=-1), -1), (dict(n_seq=(1 << 18) + 1), -4), (dict(vocab=(1 << 30) + 1), -4),
    (dict(n_seq=0), 0)])
def test_draft_refusals(change, code):
    d = Drafts(**{**DRAFTS, **change})
    assert hos.lib().hos_verify_drafts(C.byref(d), None) == code


def test_no_drafts_argument():
    assert hos.lib().hos_verify_drafts(None, None) == -1
