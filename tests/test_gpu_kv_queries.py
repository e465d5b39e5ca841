"""bf16 queries on 8-bit caches, whose products are of fp16 numbers: no element of a query loses bits that count.

Bounds as for the other attention tests, with e = (head_dim + 4) 2^-24 sum |q k| sm_scale + 2^-31 max |q| sum |k| sm_scale:
elements of a row far below its largest are rounded to within 2^-31 of that."""
import math

import pytest
import torch

from tests import kv_reference as R
from tests.test_gpu_kv_cache import make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,group", [(1, 2), (150, 2), (3, 12)])
@pytest.mark.parametrize("top", [2.0 ** -30, 2.0 ** -6, 2.0 ** -5, 2.0 ** -3, 0.1, 1.0, 50.0, 64.0, 3e4, 2.0 ** 90])
def test_small_elements_beside_a_large_one(top, n, group, d, fmt):
    """Each row's largest element meets zeros in every key; the score comes from elements 2^-9 to 2^-20 of it."""
    import paper_2502_15763_b200 as hos
    page, t, hk, dt = 32, 400, 2, torch.bfloat16
    pairs = [(n, t)]
    off, kv_len, table, n_pages = R.make_batch(pairs, page, 0, 1)
    k, v, ks, vs = make_cache(n_pages, hk, page, d, dt, fmt, 2)
    k.view(torch.uint8)[..., 5] = 0
    g = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn((n, hk * group, d), generator=g, device="cuda") * torch.exp2(-9 - 11 * torch.rand((n, hk * group, 1), generator=g, device="cuda"))
    size = q.abs().mean(-1, keepdim=True)
    q[..., 5] = 1.0
    sm = float(2.0 / math.sqrt(d) / (size.median() * top))      # scores of a few units
    q = (q.double() * top).to(dt)
    r = hos.hos_paged_attention(q, hos.hos_kv_cache(k, v, ks, vs, dtype=dt), off, kv_len, table, n, sm_scale=sm, want_lse=True)
    want, lse, mag, dot = R.attention(q, k, v, ks, vs, pairs, off, table, page, sm, True, 0)
    k_sum = max(float(R.sequence(k, ks, table[0], t, page).abs().sum(-1).max()), 0.0)
    e = (d + 4) * 2.0 ** -24 * dot + 2.0 ** -31 * q.double().abs().amax(-1) * k_sum * sm
    far = (r["lse"].double() - lse).abs() / (e + 2.0 ** -20 + 2.0 ** -22 * lse.abs())
    assert float(far.max()) <= 1.0, float(far.max())
    u = 2.0 ** -8
    bound = u * want.abs() + (2.0 ** -11 + 2.0 ** -18 + 2 * e[..., None]) * (1 + u) * mag + 2.0 ** -24
    worst = float(((r["out"].double() - want).abs() / bound).max())
    assert worst <= 1.0, worst
