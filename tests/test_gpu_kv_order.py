"""Calls that follow one another without a wait on the host, in batches that take both attention kernels: an attention call sees
everything that the append just before it wrote, and a call's workspace is its own until its pieces are joined."""
import pytest
import torch

from tests import kv_reference as R
from tests.test_gpu_kv_cache import make_cache

pytestmark = pytest.mark.gpu

PAIRS = [(1, 900 + 37 * s) for s in range(40)] + [(300, 800), (77, 77), (513, 2000), (1, 5000)]


@pytest.mark.parametrize("fmt", ["same", "int8"])
def test_attention_right_after_a_large_append(fmt):
    import paper_2502_15763_b200 as hos
    page, hk, hq, d, dt = 32, 4, 16, 128, torch.bfloat16
    off, kv_len, table, n_pages = R.make_batch(PAIRS, page, 0, 1)
    full = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), kv_len.cumsum(0).to(torch.int32)])
    total, n_tok, most = int(kv_len.sum()), sum(n for n, _ in PAIRS), max(n for n, _ in PAIRS)
    cache = hos.hos_kv_cache(*make_cache(n_pages, hk, page, d, dt, fmt, 2), dtype=dt)
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn((n_tok, hq, d), generator=g, device="cuda", dtype=dt)
    fills = [tuple(torch.randn((total, hk, d), generator=g, device="cuda", dtype=dt) for _ in range(2)) for _ in range(4)]
    want = []
    for k, v in fills:                                          # everything in the cache is written anew
        hos.hos_kv_append(cache, k, v, full, kv_len, table)
        torch.cuda.synchronize()
        want.append(hos.hos_paged_attention(q, cache, off, kv_len, table, most)["out"])
        torch.cuda.synchronize()
    assert not torch.equal(want[0], want[1])
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    got = []
    for i in range(40):
        k, v = fills[i % 4]
        hos.hos_kv_append(cache, k, v, full, kv_len, table)
        got.append(hos.hos_paged_attention(q, cache, off, kv_len, table, most, ws=ws)["out"])
    torch.cuda.synchronize()
    assert int(cache.status.abs().sum()) == 0
    for i, o in enumerate(got):
        assert torch.equal(o.view(torch.int16), want[i % 4].view(torch.int16)), i


def test_calls_that_share_a_workspace():
    """Two batches in turn, one of them all decodes, with the same workspace."""
    import paper_2502_15763_b200 as hos
    page, hk, hq, d, dt = 64, 8, 32, 64, torch.float16
    off, kv_len, table, n_pages = R.make_batch(PAIRS, page, 0, 5)
    off1, len1, table1, n_pages1 = R.make_batch([(1, 3000)] * 16, page, 0, 6)
    cache = hos.hos_kv_cache(*make_cache(max(n_pages, n_pages1), hk, page, d, dt, "same", 7), dtype=dt)
    g = torch.Generator(device="cuda").manual_seed(8)
    q = torch.randn((sum(n for n, _ in PAIRS), hq, d), generator=g, device="cuda", dtype=dt)
    calls = [lambda ws: hos.hos_paged_attention(q, cache, off, kv_len, table, 513, ws=ws, window=700)["out"],
             lambda ws: hos.hos_paged_attention(q[:16], cache, off1, len1, table1, 1, ws=ws)["out"]]
    want = []
    for call in calls:
        want.append(call(None))
        torch.cuda.synchronize()
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    got = [calls[i % 2](ws) for i in range(60)]
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert torch.equal(o.view(torch.int16), want[i % 2].view(torch.int16)), i
