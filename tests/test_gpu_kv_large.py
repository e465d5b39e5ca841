"""Caches whose pages lie further apart than 32 bits count, and batches whose largest number of new tokens is misstated."""
import pytest
import torch

from tests import kv_reference as R
from tests.test_gpu_kv_cache import ODD, check_attention, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["same", "int8"])
def test_page_offsets_beyond_32_bits(fmt):
    import paper_2502_15763_b200 as hos
    page, hk, hq, d, dt = 64, 2, 8, 64, torch.bfloat16
    pairs = [(1, 100), (40, 120), (150, 250)]
    off, kv_len, table, n_pages = R.make_batch(pairs, page, 0, 1)
    near = make_cache(n_pages, hk, page, d, dt, fmt, 2)
    per, s_per = hk * page * d, hk * page
    stride, s_stride = (2 ** 31 + 4096) // (n_pages - 1) // 64 * 64 * 4, 2 ** 31 // (n_pages - 1) // 64 * 64 + 64   # the last pages past 2^33, 2^31
    assert stride * (n_pages - 1) > 2 ** 32 and s_stride * (n_pages - 1) > 2 ** 30
    buf = torch.empty(stride * (n_pages - 1) + 2 * per, dtype=near[0].dtype, device="cuda")
    shape, strides = (n_pages, hk, page, d), (stride, page * d, d, 1)
    far = [buf.as_strided(shape, strides), buf[per:].as_strided(shape, strides), None, None]
    if fmt != "same":
        s_buf = torch.empty(s_stride * (n_pages - 1) + 2 * s_per, dtype=torch.float32, device="cuda")
        far[2:] = [s_buf[i * s_per:].as_strided(shape[:3], (s_stride, page, 1)) for i in (0, 1)]
    for a, b in zip(far, near):
        if a is not None:
            a.copy_(b)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn((sum(n for n, _ in pairs), n, d), generator=g, device="cuda", dtype=dt) for n in (hq, hk, hk))
    got = []
    for c in (near, far):
        cache = hos.hos_kv_cache(*c, dtype=dt)
        hos.hos_kv_append(cache, k, v, off, kv_len, table)
        r = hos.hos_paged_attention(q, cache, off, kv_len, table, 150, want_lse=True)
        back = hos.hos_kv_read(cache, off, kv_len, table, q.shape[0])
        torch.cuda.synchronize()
        assert int(cache.status.abs().sum()) == 0
        got.append((r["out"], r["lse"], back["k"], back["v"]))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    for a, b in zip(far, near):
        assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("max_new", [1, 2, 17, 100000])
@pytest.mark.parametrize("fmt", ["same", "e4m3"])
def test_a_misstated_largest_number_of_new_tokens_costs_time_only(max_new, fmt):
    check_attention(ODD + [(300, 300)], 4, 2, 64, "bf16", fmt, 32, max_new=max_new, seed=51)
    check_attention([(200, 500)], 16, 2, 128, "f16", fmt, 64, max_new=max_new, seed=52)
