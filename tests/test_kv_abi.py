"""Host-side checks of the KV-cache calls: they come before any CUDA call, so they are testable without a device."""
import ctypes as C

import pytest

import paper_2502_15763_b200 as hos
from paper_2502_15763_b200.kv_cache import _KvBatch, _KvCache

GOOD = dict(n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, type=0, format=0, k=4096, v=8192, k_scale=None, v_scale=None,
            page_stride=0, scale_page_stride=0)
BATCH = dict(n_seq=1, n_tokens=1, max_new=1, max_pages=2, tok_off=256, kv_len=256, page_table=256, table_stride=2)


def attention(cache=GOOD, batch=BATCH, heads=4, scale=1.0, window=0, q=4096, out=4096, q_strides=(256, 64), ws=None, ws_bytes=0):
    c, b = _KvCache(**{**GOOD, **cache}), _KvBatch(**{**BATCH, **batch})
    return hos.lib().hos_paged_attention(C.byref(c), C.byref(b), q, *q_strides, heads, scale, 1, window, out, 256, 64, None, None, ws,
                                         ws_bytes, None)


def test_null_arguments():
    L = hos.lib()
    c, b = _KvCache(**GOOD), _KvBatch(**BATCH)
    assert L.hos_kv_append(None, None, None, None, 0, 0, 0, 0, None, None) == -1
    assert L.hos_kv_append(C.byref(c), None, None, None, 0, 0, 0, 0, None, None) == -1
    assert L.hos_kv_append(C.byref(c), C.byref(b), None, None, 0, 0, 0, 0, None, None) == -1
    assert L.hos_kv_read(C.byref(c), C.byref(b), None, None, None, None) == -1
    assert L.hos_paged_attention_workspace_bytes(None, None, 4) == 0


@pytest.mark.parametrize("change,code", [
    (dict(k=None), -1), (dict(n_pages=0), -1), (dict(n_kv_heads=0), -1), (dict(type=2), -1), (dict(format=3), -1), (dict(format=1), -1),
    (dict(head_dim=96), -4), (dict(page_size=8), -4), (dict(page_size=24), -4), (dict(page_size=512), -4),
    (dict(page_stride=100), -1), (dict(page_stride=2 * 16 * 64 + 4), -1), (dict(k=4100), -1),
    (dict(format=2, k_scale=256, v_scale=260), -1), (dict(format=2, k_scale=256, v_scale=256, scale_page_stride=34), -1),
    (dict(n_kv_heads=1 << 26), -4)])
def test_cache_refusals(change, code):
    assert attention(cache=change) == code


@pytest.mark.parametrize("change,code", [
    (dict(n_seq=-1), -1), (dict(n_tokens=-1), -1), (dict(max_new=0), -1), (dict(tok_off=None), -1), (dict(page_table=None), -1),
    (dict(table_stride=1), -1), (dict(max_pages=1 << 27, table_stride=1 << 27), -4), (dict(n_tokens=0), 0), (dict(n_seq=0), 0)])
def test_batch_refusals(change, code):
    assert attention(batch=change) == code


def test_attention_refusals():
    assert attention(heads=3) == -1 and attention(heads=0) == -1
    assert attention(window=-1) == -1
    assert attention(scale=float("nan")) == -1 and attention(scale=float("inf")) == -1
    assert attention(q=None) == -1 and attention(q=4104) == -1 and attention(q_strides=(256, 60)) == -1
    assert attention() == -2                                          # no workspace
    assert attention(ws=4096 + 128, ws_bytes=1 << 40) == -2           # not 256-byte aligned
    need = hos.lib().hos_paged_attention_workspace_bytes(C.byref(_KvCache(**GOOD)), C.byref(_KvBatch(**BATCH)), 4)
    assert need > 0 and attention(ws=4096, ws_bytes=need - 1) == -2
    assert attention(batch=dict(n_tokens=1 << 30), heads=4) == -4


def test_group_division_is_exact():
    """The kernels divide row numbers by the group size with a multiplication; its constants are the host's."""
    for d in list(range(1, 300)) + [1000, 4097, 65535, 1 << 20]:
        shift = 0
        while (1 << shift) < d:
            shift += 1
        magic = (((1 << shift) - d) << 32) // d + 1
        assert magic < 1 << 32
        for n in {0, 1, d - 1, d, d + 1, 7 * d - 1, 7 * d, (1 << 31) - 1, ((1 << 31) - 1) // d * d, ((1 << 31) - 1) // d * d - 1} - {-1}:
            assert (n + (n * magic >> 32)) >> shift == n // d
