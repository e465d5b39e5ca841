"""Tensors of unusual strides, sizes and origins as arguments of the KV-cache calls."""
import math

import pytest
import torch

from tests import kv_reference as R
from tests.test_gpu_kv_cache import make_cache

pytestmark = pytest.mark.gpu


def hos():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2502_15763_b200 as h
    return h


def test_pages_that_overlap_are_refused():
    """An expanded page has the stride 0, which the C interface takes for densely packed pages: memory past the tensor."""
    h = hos()
    k, v, ks, vs = make_cache(4, 2, 16, 64, torch.bfloat16, "int8", 1)
    same, same_v = (torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for bad, bad_v in ((same[:1].expand(4, -1, -1, -1), same_v[:1].expand(4, -1, -1, -1)),
                       (same.as_strided((4, 2, 16, 64), (1024, 1024, 64, 1)), same_v.as_strided((4, 2, 16, 64), (1024, 1024, 64, 1)))):
        with pytest.raises(ValueError, match="overlap"):
            h.hos_kv_cache(bad, bad_v)
    with pytest.raises(ValueError, match="overlap"):
        h.hos_kv_cache(k, v, ks[:1].expand(4, -1, -1), vs[:1].expand(4, -1, -1), dtype=torch.bfloat16)
    # one page has no neighbour to overlap with
    h.hos_kv_cache(same[:1].expand(1, -1, -1, -1), same_v[:1])


def odd_strides(x, tok, head):
    """x [tokens][heads][d] with these strides, in a buffer of its own that begins on 16 bytes."""
    buf = torch.full(((x.shape[0] - 1) * tok + (x.shape[1] - 1) * head + x.shape[2] + 64,), 7.0, dtype=x.dtype, device=x.device)
    y = buf.as_strided(x.shape, (tok, head, 1))
    y.copy_(x)
    return y


@pytest.mark.parametrize("n,heads,kv_heads,tok,head", [(1, 4, 4, 259, 64), (1, 1, 1, 1, 3), (5, 1, 1, 72, 5), (30, 1, 1, 64, 1), (1, 8, 2, 13, 72)])
def test_strides_of_a_single_token_or_head_mean_nothing(n, heads, kv_heads, tok, head):
    h = hos()
    d, page, t, dt = 64, 16, 50, torch.bfloat16
    off, kv_len, table, n_pages = R.make_batch([(n, t)], page, 1, 1)
    k, v, ks, vs = make_cache(n_pages, kv_heads, page, d, dt, "int8", 2)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, nk, nv = (torch.randn((n, hd, d), generator=g, device="cuda").to(dt) for hd in (heads, kv_heads, kv_heads))

    def step(odd):
        cache = h.hos_kv_cache(*(x.clone() for x in (k, v, ks, vs)), dtype=dt)
        a, b, c = (odd_strides(x, tok, head) if odd and x.shape[1] == q.shape[1] else x for x in (q, nk, nv))
        out = odd_strides(torch.zeros_like(q), tok, head) if odd else None
        h.hos_kv_append(cache, b, c, off, kv_len, table)
        r = h.hos_paged_attention(a, cache, off, kv_len, table, n, out=out)
        torch.cuda.synchronize()
        assert int(cache.status.abs().sum()) == 0
        return r["out"], cache
    want, c1 = step(False)
    got, c2 = step(True)
    assert torch.equal(got, want) and torch.equal(c1.k, c2.k) and torch.equal(c1.v_scale, c2.v_scale)


@pytest.mark.parametrize("fmt", ["same", "e4m3"])
def test_strides_of_a_single_kv_head_or_page_mean_nothing(fmt):
    h = hos()
    for n_pages, strides, s_strides in ((4, (1024, 13, 64, 1), (16, 3, 1)), (1, (5, 1024, 64, 1), (9, 16, 1)), (1, (3, 1, 64, 1), (1, 1, 1))):
        k, v, ks, vs = make_cache(n_pages, 1, 16, 64, torch.float16, fmt, 2)
        off, kv_len, table, _ = R.make_batch([(1, 16 * n_pages - 2)], 16, 0, 1)
        table.clamp_(0, n_pages - 1)
        q = torch.randn((1, 2, 64), device="cuda").half()
        want = h.hos_paged_attention(q, h.hos_kv_cache(k, v, ks, vs, dtype=torch.float16), off, kv_len, table, 1)["out"]
        odd = h.hos_kv_cache(k.as_strided(k.shape, strides), v, None if ks is None else ks.as_strided(ks.shape, s_strides), vs, dtype=torch.float16)
        got = h.hos_paged_attention(q, odd, off, kv_len, table, 1)["out"]
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_tensors_that_require_grad():
    """There is no backward pass: with gradients on they are refused instead of answered without a graph."""
    h = hos()
    off, kv_len, table, n_pages = R.make_batch([(2, 20)], 16, 0, 1)
    cache = h.hos_kv_cache(*make_cache(n_pages, 2, 16, 64, torch.bfloat16, "same", 2))
    q, k, v = (torch.randn((2, n, 64), device="cuda").bfloat16() for n in (4, 2, 2))
    want = h.hos_paged_attention(q, cache, off, kv_len, table, 2)["out"]
    g = q.clone().requires_grad_()
    with pytest.raises(ValueError, match="q requires grad"):
        h.hos_paged_attention(g, cache, off, kv_len, table, 2)
    with pytest.raises(ValueError, match="k requires grad"):
        h.hos_kv_append(cache, k.clone().requires_grad_(), v, off, kv_len, table)
    with pytest.raises(ValueError, match="v requires grad"):
        h.hos_kv_append(cache, k, v.clone().requires_grad_() * 1, off, kv_len, table)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            assert torch.equal(h.hos_paged_attention(g, cache, off, kv_len, table, 2)["out"], want)
    assert torch.equal(h.hos_paged_attention(g.detach(), cache, off, kv_len, table, 2)["out"], want)


def test_tokens_of_no_sequence_read_as_zero():
    h = hos()
    for d, fmt in ((64, "same"), (128, "int8")):
        cache = h.hos_kv_cache(*make_cache(3, 2, 16, d, torch.float16, fmt, 2), dtype=torch.float16)
        empty = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((1,), (0,), (0, 2))]
        out = [torch.full((7, 2, d), 5.0, dtype=torch.float16, device="cuda") for _ in range(2)]
        r = h.hos_kv_read(cache, *empty, 7, out=out)
        assert bool((r["k"] == 0).all()) and bool((r["v"] == 0).all())
        # a batch whose sequences begin after the first token and end before the last
        off = torch.tensor([2, 4], dtype=torch.int32, device="cuda")
        kv_len, table = torch.tensor([20], dtype=torch.int32, device="cuda"), torch.tensor([[2, 0]], dtype=torch.int32, device="cuda")
        r = h.hos_kv_read(cache, off, kv_len, table, 7, out=[t.fill_(5.0) for t in out])
        for x in (r["k"], r["v"]):
            assert bool((x[[0, 1, 4, 5, 6]] == 0).all()) and bool((x[2:4] != 0).any())


def test_an_expanded_output_is_refused():
    """Its rows would be written to one place by several blocks at once; the check comes before any launch."""
    h = hos()
    off, kv_len, table, n_pages = R.make_batch([(2, 20)], 16, 0, 1)
    cache = h.hos_kv_cache(*make_cache(n_pages, 2, 16, 64, torch.bfloat16, "same", 2))
    q = torch.randn((2, 4, 64), device="cuda").bfloat16()
    for out in (torch.zeros_like(q[:1]).expand(2, 4, 64), torch.zeros_like(q[:, :1]).expand(2, 4, 64)):
        with pytest.raises(ValueError, match="expanded"):
            h.hos_paged_attention(q, cache, off, kv_len, table, 2, out=out)
    one = torch.zeros((1, 1, 64), dtype=q.dtype, device="cuda").expand(1, 4, 64)
    with pytest.raises(ValueError, match="expanded"):
        h.hos_paged_attention(q[:1], cache, off, kv_len, table, 2, out=one)
    wide = q[:1].expand(2, 4, 64)                                # an expanded query is fine
    got = h.hos_paged_attention(wide, cache, off, kv_len, table, 2)["out"]
    assert torch.equal(got, h.hos_paged_attention(wide.contiguous(), cache, off, kv_len, table, 2)["out"])
