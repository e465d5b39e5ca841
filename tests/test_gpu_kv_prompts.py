"""Prompts and chunks with many whole tiles a CTA, against the 64-bit statement: the ring, the scale buffers and the queries of the
chunk kernel go round many times, over tiles of one, two and many steps and over tiles of 128 rows between tiles of 256."""
import pytest

from tests.test_gpu_kv_cache import check_attention

pytestmark = pytest.mark.gpu

# (new tokens, tokens): about 50 list steps a CTA with 40 KV heads
MIXED = [(1000, 1000), (100, 100), (513, 600), (129, 129), (64, 900), (700, 700), (20, 140), (257, 257), (1100, 1300), (90, 1500), (128, 128)]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["same", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_many_tiles_a_cta(dt, fmt, d):
    check_attention(MIXED, 40, 40, d, dt, fmt, 32, seed=21)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("n", [90, 200, 250, 380, 900])
def test_prompts_of_one_length(n, fmt):
    """Tiles of n rows at most: one step, two steps, and three to eight, all whole."""
    check_attention([(n, n)] * 24, 24, 24, 128, "bf16", fmt, 64, seed=n)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_grouped_chunks_behind_contexts(fmt):
    check_attention([(60, 2000), (31, 500), (200, 3000), (17, 1000), (100, 700)] * 3, 128, 16, 128, "f16", fmt, 16, seed=22)
    check_attention([(60, 2000), (31, 500), (200, 3000), (17, 1000), (100, 700)] * 3, 128, 16, 64, "bf16", fmt, 128, window=600, seed=23)


@pytest.mark.parametrize("fmt", ["same", "e4m3"])
def test_whole_prompts_again_and_again(fmt):
    """Back-to-back calls, each beginning while the one before drains; nothing is reported and every call gives the same."""
    import torch
    import paper_2502_15763_b200 as hos
    from tests import kv_reference as R
    from tests.test_gpu_kv_cache import make_cache
    pairs = [(384, 384)] * 8 + [(700, 700)] * 4
    off, kv_len, table, n_pages = R.make_batch(pairs, 64, 0, 3)
    cache = hos.hos_kv_cache(*make_cache(n_pages, 32, 64, 128, torch.bfloat16, fmt, 4), dtype=torch.bfloat16)
    q = torch.randn((sum(n for n, _ in pairs), 32, 128), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).bfloat16()
    first = hos.hos_paged_attention(q, cache, off, kv_len, table, 700)["out"]
    outs = [hos.hos_paged_attention(q, cache, off, kv_len, table, 700)["out"] for _ in range(60)]
    torch.cuda.synchronize()
    assert int(cache.status.abs().sum()) == 0
    for o in outs:
        assert torch.equal(o.view(torch.int16), first.view(torch.int16))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_prompts_beside_other_traffic(fmt, d):
    """Copies on another stream make loads and stores slow: same outputs, no status."""
    import torch
    import paper_2502_15763_b200 as hos
    from tests import kv_reference as R
    from tests.test_gpu_kv_cache import make_cache
    pairs = [(384, 384)] * 6 + [(100, 900)] * 6 + [(640, 640)] * 4
    off, kv_len, table, n_pages = R.make_batch(pairs, 32, 0, 3)
    cache = hos.hos_kv_cache(*make_cache(n_pages, 32, 32, d, torch.bfloat16, fmt, 4), dtype=torch.bfloat16)
    q = torch.randn((sum(n for n, _ in pairs), 32, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).bfloat16()
    first = hos.hos_paged_attention(q, cache, off, kv_len, table, 640)["out"]
    a, b = (torch.empty(1 << 30, dtype=torch.uint8, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(60):
            b.copy_(a)
    outs = [hos.hos_paged_attention(q, cache, off, kv_len, table, 640)["out"] for _ in range(40)]
    torch.cuda.synchronize()
    assert int(cache.status.abs().sum()) == 0
    for o in outs:
        assert torch.equal(o.view(torch.int16), first.view(torch.int16))
