"""Status words of a cache handle: no bit is lost between streams, graphs and batches of growing size."""
import pytest
import torch

from tests import kv_reference as R
from tests.test_gpu_kv_cache import make_cache

pytestmark = pytest.mark.gpu

LONG = 40_000_000                                                # cycles of a kernel that does nothing: about 20 ms


def setup():
    import paper_2502_15763_b200 as hos
    off, kv_len, table, n_pages = R.make_batch([(1, 20), (1, 40), (1, 5)], 16, 0, 1)
    bad = table.clone()
    bad[1, 1] = n_pages + 7                                      # no such page
    tensors = make_cache(n_pages, 2, 16, 64, torch.bfloat16, "same", 2)
    q = torch.randn((3, 4, 64), device="cuda").bfloat16()
    hos.hos_paged_attention(q, hos.hos_kv_cache(*tensors), off, kv_len, table, 1)      # everything is loaded
    torch.cuda.synchronize()
    return hos, tensors, q, off, kv_len, table, bad


def many(n):
    """A batch of n sequences, of which only the first has anything."""
    off = torch.ones(n + 1, dtype=torch.int32, device="cuda")
    off[0] = 0
    kv_len = torch.zeros(n, dtype=torch.int32, device="cuda")
    kv_len[0] = 1
    return off, kv_len, torch.zeros((n, 1), dtype=torch.int32, device="cuda")


def test_a_handle_may_be_used_on_another_stream_at_once():
    hos, tensors, q, off, kv_len, table, bad = setup()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(one):
        del_me = torch.zeros(4096, dtype=torch.int32, device="cuda")               # memory of this stream's for the words
        torch.cuda.synchronize()
        del del_me
        torch.cuda._sleep(LONG)
        cache = hos.hos_kv_cache(*tensors)
    with torch.cuda.stream(two):
        hos.hos_paged_attention(q, cache, off, kv_len, bad, 1)
    torch.cuda.synchronize()
    assert cache.status[:3].tolist() == [0, hos.HOS_ST_INVALID, 0]


@pytest.mark.parametrize("n", [1500, 9000])
def test_bits_of_calls_in_flight_survive_a_larger_batch(n):
    hos, tensors, q, off, kv_len, table, bad = setup()
    cache = hos.hos_kv_cache(*tensors)
    big = many(n)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
        hos.hos_paged_attention(q, cache, off, kv_len, bad, 1)
    r = hos.hos_paged_attention(q[:1], cache, *big, 1)
    torch.cuda.synchronize()
    assert r["status"].shape[0] >= n
    assert cache.status[:3].tolist() == [0, hos.HOS_ST_INVALID, 0] and cache.status.shape[0] >= n
    cache.status.zero_()
    assert int(cache.status.abs().sum()) == 0


def test_graphs_captured_before_a_larger_batch_still_report():
    hos, tensors, q, off, kv_len, table, bad = setup()
    cache = hos.hos_kv_cache(*tensors)
    live = table.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        hos.hos_paged_attention(q, cache, off, kv_len, live, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hos.hos_paged_attention(q, cache, off, kv_len, live, 1)
    hos.hos_paged_attention(q[:1], cache, *many(5000), 1)
    graph.replay()
    torch.cuda.synchronize()
    assert int(cache.status.abs().sum()) == 0
    live.copy_(bad)
    graph.replay()
    torch.cuda.synchronize()
    assert cache.status[:3].tolist() == [0, hos.HOS_ST_INVALID, 0]
    cache.status.zero_()
    live.copy_(table)
    graph.replay()
    assert int(cache.status.abs().sum()) == 0


def test_a_larger_batch_within_a_capture_is_refused():
    hos, tensors, q, off, kv_len, table, bad = setup()
    cache = hos.hos_kv_cache(*tensors)
    big = many(4000)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="before a graph is captured"):
        with torch.cuda.graph(graph):
            hos.hos_paged_attention(q[:1], cache, *big, 1)
    torch.cuda.synchronize()
    hos.hos_paged_attention(q[:1], cache, *big, 1)               # outside it works, and then inside too
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = hos.hos_paged_attention(q[:1], cache, *big, 1)["out"]
    graph.replay()
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out).all()) and int(cache.status.abs().sum()) == 0


def test_the_words_outlive_calls_on_other_streams():
    """A handle dropped while a call on another stream is in flight: its words are not handed out before that call is done."""
    hos, tensors, q, off, kv_len, table, bad = setup()
    cache = hos.hos_kv_cache(*tensors)
    at = cache.status.data_ptr()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
        hos.hos_paged_attention(q, cache, off, kv_len, bad, 1)
    n = cache.status.shape[0]
    del cache
    taken = [torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(8)]
    assert all(t.data_ptr() != at for t in taken)
    torch.cuda.synchronize()
    assert all(int(t.abs().sum()) == 0 for t in taken)
