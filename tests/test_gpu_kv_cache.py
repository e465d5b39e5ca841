"""Paged KV cache on the GPU: append, read back and attention against plain 64-bit statements.

Codes, scales and values read back have to be equal bit for bit (every step is an IEEE operation in 32 bits).
Attention is held to bounds that follow from the arithmetic, element by element, with u the unit roundoff of
the output's type (2^-8 bf16, 2^-11 fp16) and A = sum_j w_j |v_j|:
  - the output is rounded once: u |out|;
  - the weights are rounded to 16 bits before the product with the values: u_w A, u_w = 2^-8 for a bf16
    cache, else 2^-11;
  - a score is a 32-bit sum of head_dim products, so it is off by at most (head_dim + 4) 2^-24 sum |q k| sm_scale =: e;
    weights and their sum are off by a factor of 1 + 2 e, and 2^-18 covers the 32-bit sums and exponentials.
lse: e + 2^-20 + 2^-22 |lse|."""
import math

import pytest
import torch

from tests import kv_reference as R

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CODES = {"same": None, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def hos():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2502_15763_b200 as h
    return h


def make_cache(n_pages, hk, page, d, dt, fmt, seed, interleaved=False):
    """Random cache tensors (k, v, k_scale, v_scale); interleaved: a page's k and v lie next to each other."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n_pages, 2, hk, page, d), generator=g, device="cuda", dtype=dt)
    if CODES[fmt] is None:
        return (x[:, 0], x[:, 1], None, None) if interleaved else (x[:, 0].contiguous(), x[:, 1].contiguous(), None, None)
    c, s = R.quantise(x, CODES[fmt])
    if interleaved:
        return c[:, 0], c[:, 1], s[:, 0], s[:, 1]
    c8 = c.view(torch.uint8)
    return (c8[:, 0].contiguous().view(c.dtype), c8[:, 1].contiguous().view(c.dtype), s[:, 0].contiguous(), s[:, 1].contiguous())


def poison(cache, pairs, table, page):
    """NaN in every row that holds no token of a sequence."""
    k, v, ks, vs = cache
    used = torch.zeros((k.shape[0], page), dtype=torch.bool, device="cuda")
    for s, (_, t) in enumerate(pairs):
        for i in range(-(-t // page)):
            used[table[s, i], :min(page, t - i * page)] = True
    free = (~used)[:, None, :].expand(k.shape[:3])
    for x in (k, v):
        if x.dtype == torch.float8_e4m3fn:
            x.view(torch.uint8)[free] = 0x7F
        elif x.dtype == torch.int8:
            x[free] = -128
        else:
            x[free] = math.nan
    for x in (ks, vs):
        if x is not None:
            x[free] = math.nan


def check_attention(pairs, hq, hk, d, dt, fmt, page, causal=True, window=0, sm_scale=None, seed=0, q_gain=1.5, interleaved=False,
                    strided=False, max_new=None, dirty=True):
    h = hos()
    dtype = TYPES[dt]
    off, kv_len, table, n_pages = R.make_batch(pairs, page, 2, seed)
    cache = make_cache(n_pages, hk, page, d, dtype, fmt, seed + 1, interleaved)
    if dirty:
        poison(cache, pairs, table, page)
    n_tok = sum(n for n, _ in pairs)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    big = torch.randn((max(n_tok, 1), hq + 3, d + 8 if strided else d), generator=g, device="cuda", dtype=dtype).mul_(q_gain)
    q = big[:n_tok, 1:1 + hq, :d] if strided else big[:n_tok, :hq].contiguous()
    handle = h.hos_kv_cache(*cache, dtype=dtype)
    out = torch.full((n_tok, hq, 2 * d), 7.0, dtype=dtype, device="cuda")[..., :d] if strided else None
    most = max(n for n, _ in pairs) if max_new is None else max_new
    r = h.hos_paged_attention(q, handle, off, kv_len, table, most, sm_scale=sm_scale, causal=causal, window=window, want_lse=True, out=out)
    torch.cuda.synchronize()
    assert int(r["status"].abs().sum()) == 0
    scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    want, lse, mag, dot = R.attention(q, *cache, pairs, off, table, page, scale, causal, window)
    u = 2.0 ** -8 if dt == "bf16" else 2.0 ** -11
    uw = 2.0 ** -8 if dt == "bf16" and fmt == "same" else 2.0 ** -11
    e = (d + 4) * 2.0 ** -24 * dot
    got = r["out"].to(torch.float64)
    assert bool(torch.isfinite(got).all())
    bound = u * want.abs() + (uw + 2.0 ** -18 + 2 * e[..., None]) * (1 + u) * mag + 2.0 ** -24
    worst = float(((got - want).abs() / bound).max()) if n_tok else 0.0
    assert worst <= 1.0, worst
    empty = lse == -math.inf
    assert torch.equal(empty, r["lse"] == -math.inf)
    assert bool((r["out"][empty] == 0).all())
    far = (r["lse"].to(torch.float64) - lse).abs() / (e + 2.0 ** -20 + 2.0 ** -22 * lse.abs())
    assert not n_tok or float(far[~empty].max() if (~empty).any() else 0.0) <= 1.0
    if strided:
        assert bool((out.as_strided((n_tok, hq, d), (hq * 2 * d, 2 * d, 1), d) == 7.0).all())     # the gaps are untouched
    return r


# (new tokens, tokens in the cache): no tokens, no keys, more new tokens than the cache holds (rows that see
# nothing), lengths on both sides of the page and tile sizes
ODD = [(1, 1), (0, 5), (1, 17), (0, 0), (3, 3), (5, 2), (1, 0), (7, 130), (40, 300), (1, 1000), (129, 513), (2, 256), (16, 16)]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["same", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 8])
def test_attention_odd_batches(dt, fmt, d, group):
    check_attention(ODD, 2 * group, 2, d, dt, fmt, 16 if group == 1 else 64, seed=group)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("fmt", ["same", "int8"])
def test_attention_page_sizes(page, fmt):
    check_attention(ODD + [(300, 300)], 4, 2, 128, "bf16", fmt, page, seed=page)


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 37), (False, 100), (True, 5000), (False, 1)])
@pytest.mark.parametrize("fmt", ["same", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_masks(causal, window, fmt, d):
    check_attention(ODD + [(200, 900)], 8, 2, d, "f16", fmt, 32, causal=causal, window=window, seed=5)


@pytest.mark.parametrize("fmt", ["same", "e4m3", "int8"])
def test_attention_strides_and_interleaved_pages(fmt):
    check_attention(ODD, 6, 2, 64, "bf16", fmt, 32, seed=3, interleaved=True, strided=True)
    check_attention(ODD, 4, 4, 128, "f16", fmt, 128, seed=4, interleaved=True, strided=True)


@pytest.mark.parametrize("pairs,hq,hk", [([(1, 20000)], 8, 8), ([(1, 9001), (1, 3)], 32, 2), ([(2, 30000)], 5, 1),
                                         ([(17, 12345)], 16, 2), ([(300, 8000), (1, 8000)], 8, 1)])
@pytest.mark.parametrize("fmt", ["same", "int8"])
def test_attention_long_contexts(pairs, hq, hk, fmt):
    check_attention(pairs, hq, hk, 128, "bf16", fmt, 64, seed=9, dirty=False)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513])
def test_attention_prompt_lengths(n):
    check_attention([(n, n), (n, 2 * n + 1)], 2, 1, 128, "bf16", "same", 16, seed=n)
    check_attention([(n, n), (n, 2 * n + 1)], 3, 1, 64, "f16", "e4m3", 32, seed=n)


@pytest.mark.parametrize("n_seq", [1, 31, 33, 257, 1100])
def test_attention_many_sequences(n_seq):
    pairs = [((7 * s) % 3 if s % 5 else 1 + s % 40, 40 + (s * 37) % 90) for s in range(n_seq)]
    check_attention(pairs, 2, 1, 64, "bf16", "same", 16, seed=n_seq)


@pytest.mark.parametrize("gain,scale", [(40.0, None), (1e-3, None), (3.0, -0.5), (1.0, 0.0), (4.0, 2.0)])
@pytest.mark.parametrize("dt,fmt", [("bf16", "same"), ("bf16", "e4m3"), ("f16", "int8")])
def test_attention_score_ranges(gain, scale, dt, fmt):
    """Very peaked and flat softmaxes; negative and zero scales."""
    check_attention([(1, 500), (90, 400)], 4, 2, 128, dt, fmt, 64, sm_scale=scale, q_gain=gain, seed=11)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("n", [1, 150])
def test_attention_scales_of_any_size(dt, n):
    """Tokens whose values differ in size by many powers of ten keep their weight."""
    h = hos()
    page, d, t = 32, 128, 333
    pairs = [(n, t)]
    off, kv_len, table, n_pages = R.make_batch(pairs, page, 0, 1)
    k, v, ks, vs = make_cache(n_pages, 2, page, d, TYPES[dt], "e4m3", 2)
    for lo in (-3.0, 2.0):                                      # about 1e-6 .. 1 and 1e-1 .. 1e5 before the product with a code
        vs2 = 10.0 ** (lo + 3.0 * torch.sin(torch.arange(vs.numel(), device="cuda", dtype=torch.float32))).view_as(vs) * 1e-3
        q = torch.randn((n, 4, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(TYPES[dt])
        r = h.hos_paged_attention(q, h.hos_kv_cache(k, v, ks, vs2, dtype=TYPES[dt]), off, kv_len, table, n)
        want, _, mag, dot = R.attention(q, k, v, ks, vs2, pairs, off, table, page, d ** -0.5, True, 0)
        u = 2.0 ** -8 if dt == "bf16" else 2.0 ** -11
        bound = u * want.abs() + (2.0 ** -11 + 2.0 ** -18 + 2 * (d + 4) * 2.0 ** -24 * dot[..., None]) * (1 + u) * mag + 2.0 ** -24
        assert float(((r["out"].double() - want).abs() / bound).max()) <= 1.0


def test_attention_repeats_bit_for_bit_and_on_any_stream():
    h = hos()
    pairs = [(1, 3000), (1, 10), (60, 700), (1, 1)]
    off, kv_len, table, n_pages = R.make_batch(pairs, 32, 1, 0)
    cache = make_cache(n_pages, 2, 32, 128, torch.bfloat16, "same", 1)
    handle = h.hos_kv_cache(*cache)
    q = torch.randn((sum(n for n, _ in pairs), 8, 128), device="cuda").bfloat16()
    first = h.hos_paged_attention(q, handle, off, kv_len, table, 60, want_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = h.hos_paged_attention(q, handle, off, kv_len, table, 60, want_lse=True)
        third = h.hos_paged_attention(q, handle, off, kv_len, table, 60)
    torch.cuda.synchronize()
    for r in (second, third):
        assert torch.equal(r["out"], first["out"])
    assert torch.equal(second["lse"], first["lse"]) and third["lse"] is None


def test_calls_are_graph_capturable():
    h = hos()
    pairs = [(1, 300), (1, 77)]
    off, kv_len, table, n_pages = R.make_batch(pairs, 16, 0, 0)
    k, v, ks, vs = make_cache(n_pages, 2, 16, 64, torch.float16, "int8", 1)
    handle = h.hos_kv_cache(k, v, ks, vs, dtype=torch.float16)
    q, nk, nv = (torch.randn((2, n, 64), device="cuda").half() for n in (4, 2, 2))

    def step():
        h.hos_kv_append(handle, nk, nv, off, kv_len, table)
        return h.hos_paged_attention(q, handle, off, kv_len, table, 1)["out"]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = step().clone()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    got.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


# --- append and read ---------------------------------------------------------------------------

def awkward(n, heads, d, dtype, seed):
    """New vectors of every kind: ordinary, zero, tiny, huge, one element only."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, heads, d), generator=g, device="cuda") * torch.exp(2 * torch.randn((n, heads, 1), generator=g, device="cuda"))
    flat = x.view(-1, d)
    for i, f in ((0, 0.0), (1, 1e-6), (2, 3e4), (3, 1e-36 if dtype == torch.bfloat16 else 6e-8)):
        if i < flat.shape[0]:
            flat[i] *= f
    if flat.shape[0] > 4:
        flat[4] = 0.0
        flat[4, d - 1] = -3.0
    return x.to(dtype)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["same", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hk,page", [(1, 16), (3, 256), (17, 32), (40, 64)])
def test_append_and_read(dt, fmt, d, hk, page):
    h = hos()
    dtype = TYPES[dt]
    pairs = [(1, 1), (0, 9), (5, 2), (16, 16), (1, 300), (33, 290), (0, 0), (2, 257)]
    off, kv_len, table, n_pages = R.make_batch(pairs, page, 3, hk)
    cache = make_cache(n_pages, hk, page, d, dtype, fmt, 7, interleaved=hk == 3)
    want = [None if t is None else t.clone() for t in cache]
    n_tok = sum(n for n, _ in pairs)
    qkv = torch.cat([awkward(n_tok, hk, d, dtype, s) for s in (1, 2, 3)], dim=1)
    nk, nv = qkv[:, hk:2 * hk], qkv[:, 2 * hk:]
    handle = h.hos_kv_cache(*cache, dtype=dtype)
    r = h.hos_kv_append(handle, nk, nv, off, kv_len, table)
    assert int(r["status"].abs().sum()) == 0
    full_off = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), kv_len.cumsum(0).to(torch.int32)])
    back = h.hos_kv_read(handle, full_off, kv_len, table, int(kv_len.sum()))
    part = h.hos_kv_read(handle, off, kv_len, table, n_tok)
    torch.cuda.synchronize()
    raw = [t.view(torch.uint8) if t is not None and t.element_size() == 1 else t for t in want]
    for s, (n, t) in enumerate(pairs):
        for i in range(n):
            pos = t - n + i
            if pos < 0:
                continue
            page_id, row = int(table[s, pos // page]), pos % page
            for x, at in ((nk, 0), (nv, 1)):
                vec = x[int(off[s]) + i]
                if CODES[fmt] is None:
                    raw[at][page_id, :, row] = vec
                else:
                    c, sc = R.quantise(vec, CODES[fmt])
                    raw[at][page_id, :, row] = c.view(torch.uint8)
                    raw[at + 2][page_id, :, row] = sc
    for got, exp in zip(cache, want):
        assert (got is None) == (exp is None)
        if got is not None:
            a, b = (t.contiguous().view(torch.uint8) for t in (got, exp))
            assert torch.equal(a, b)
    for name, x, sc in (("k", want[0], want[2]), ("v", want[1], want[3])):
        at = 0
        for s, (n, t) in enumerate(pairs):
            pages = table[s, :-(-t // page)].long()
            val = (x.view(torch.uint8)[pages].view(x.dtype) if x.element_size() == 1 else x[pages]).float()
            if sc is not None:
                val = val * sc[pages][..., None]
            val = val.to(dtype).permute(0, 2, 1, 3).reshape(-1, hk, d)[:t]
            assert torch.equal(back[name][at:at + t], val)
            first = max(0, n - t)
            a = int(off[s])
            assert bool((part[name][a:a + min(n, first)] == 0).all())
            assert torch.equal(part[name][a + first:a + n], val[max(0, t - n):])
            at += t


@pytest.mark.parametrize("fmt", ["same", "e4m3", "int8"])
def test_non_finite_vectors_read_back_as_nan(fmt):
    h = hos()
    off, kv_len, table, n_pages = R.make_batch([(4, 4)], 16, 0, 0)
    cache = make_cache(n_pages, 2, 16, 64, torch.float16, fmt, 1)
    x = torch.randn((4, 2, 64), device="cuda").half()
    x[0, 0, 3], x[1, 1, 63], x[2, 0, 0] = math.nan, math.inf, -math.inf
    handle = h.hos_kv_cache(*cache, dtype=torch.float16)
    h.hos_kv_append(handle, x, x, off, kv_len, table)
    r = h.hos_kv_read(handle, off, kv_len, table, 4)
    torch.cuda.synchronize()
    for name in ("k", "v"):
        if fmt == "same":
            assert torch.equal(r[name].view(torch.int16), x.view(torch.int16))
            continue
        bad = torch.isnan(r[name]).all(-1)
        assert bad.tolist() == [[True, False], [False, True], [True, False], [False, False]]
        assert bool(torch.isfinite(r[name][~bad]).all())


# --- problems in the data, refusals ------------------------------------------------------------

def test_data_problems_set_status_and_leave_others_alone():
    h = hos()
    pairs = [(1, 40), (2, 50), (1, 33), (3, 64)]
    off, kv_len, table, n_pages = R.make_batch(pairs, 16, 0, 0)
    cache = make_cache(n_pages, 1, 16, 64, torch.bfloat16, "same", 1)
    handle = h.hos_kv_cache(*cache)
    q = torch.randn((7, 2, 64), device="cuda").bfloat16()
    good = h.hos_paged_attention(q, handle, off, kv_len, table, 3)["out"].clone()
    bad_table, bad_len = table.clone(), kv_len.clone()
    bad_table[1, 3] = n_pages                                    # one past the pool
    bad_len[2] = 16 * table.shape[1] + 1                         # longer than its row of the table
    for call in (lambda: h.hos_paged_attention(q, handle, off, bad_len, bad_table, 3)["out"],
                 lambda: h.hos_kv_read(handle, off, bad_len, bad_table, 7)["k"],
                 lambda: h.hos_kv_append(handle, torch.zeros((7, 1, 64), dtype=torch.bfloat16, device="cuda"),
                                         torch.zeros((7, 1, 64), dtype=torch.bfloat16, device="cuda"), off, bad_len, bad_table)):
        handle.status.zero_()
        before = cache[0].clone()
        got = call()
        torch.cuda.synchronize()
        assert handle.status[:4].tolist() == [0, h.HOS_ST_INVALID, h.HOS_ST_INVALID, 0]
        if isinstance(got, torch.Tensor) and got.shape == good.shape:
            keep = [0, 4, 5, 6]
            assert torch.equal(got[keep], good[keep])
        if isinstance(got, dict):
            changed = (cache[0] != before).any(-1).sum()
            assert int(changed) <= 1 + 2 + 3
    handle.status.zero_()
    bad_off = off.clone()
    bad_off[4] = 99                                              # past the packed tokens
    h.hos_paged_attention(q, handle, bad_off, kv_len, table, 3)
    torch.cuda.synchronize()
    assert handle.status[:4].tolist() == [0, 0, 0, h.HOS_ST_INVALID]


def test_refusals():
    h = hos()
    off, kv_len, table, n_pages = R.make_batch([(1, 5)], 16, 0, 0)
    k, v, ks, vs = make_cache(n_pages, 2, 16, 64, torch.bfloat16, "int8", 1)
    z = torch.zeros
    with pytest.raises(TypeError):
        h.hos_kv_cache(k, v, ks, vs)                             # the type of the queries is not known
    with pytest.raises(TypeError):
        h.hos_kv_cache(k, v, None, None, dtype=torch.bfloat16)   # codes without scales
    with pytest.raises(ValueError):
        h.hos_kv_cache(k, v[:, :1], ks, vs, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        h.hos_kv_cache(k.float(), v.float())
    handle = h.hos_kv_cache(k, v, ks, vs, dtype=torch.bfloat16)
    q = z((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        h.hos_paged_attention(q.half(), handle, off, kv_len, table, 1)
    with pytest.raises(ValueError):
        h.hos_paged_attention(z((1, 4, 128), dtype=torch.bfloat16, device="cuda"), handle, off, kv_len, table, 1)
    with pytest.raises(TypeError):
        h.hos_paged_attention(q, handle, off.long(), kv_len, table, 1)
    with pytest.raises(ValueError):
        h.hos_paged_attention(q, handle, off[:1], kv_len, table, 1)
    for heads in (3, 1):                                         # not a multiple of the KV heads
        with pytest.raises(h.HosError) as e:
            h.hos_paged_attention(z((1, heads, 64), dtype=torch.bfloat16, device="cuda"), handle, off, kv_len, table, 1)
        assert e.value.code == -1
    for kw in (dict(window=-1), dict(sm_scale=math.inf), dict(max_new=0)):
        with pytest.raises(h.HosError) as e:
            h.hos_paged_attention(q, handle, off, kv_len, table, **{"max_new": 1, **kw})
        assert e.value.code == -1
    wide = z((1, 4, 68), dtype=torch.bfloat16, device="cuda")[..., 4:]   # rows that do not start on 16 bytes
    with pytest.raises(h.HosError) as e:
        h.hos_paged_attention(wide, handle, off, kv_len, table, 1)
    assert e.value.code == -1
    for shape in ((3, 2, 16, 96), (3, 2, 8, 64), (3, 2, 48, 64)):
        odd = h.hos_kv_cache(z(shape, dtype=torch.float16, device="cuda"), z(shape, dtype=torch.float16, device="cuda"))
        with pytest.raises(h.HosError) as e:
            h.hos_kv_read(odd, off, kv_len, table, 1)
        assert e.value.code == -4
    with pytest.raises(ValueError):
        h.hos_kv_append(handle, z((1, 2, 64), dtype=torch.bfloat16, device="cuda"), z((2, 2, 64), dtype=torch.bfloat16, device="cuda"),
                        off, kv_len, table)
    # an empty batch is nothing to do
    none = z((0,), dtype=torch.int32, device="cuda")
    r = h.hos_paged_attention(q[:0], handle, z((1,), dtype=torch.int32, device="cuda"), none, z((0, 1), dtype=torch.int32, device="cuda"), 0)
    assert r["out"].shape == (0, 4, 64)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("n", [1, 150])
@pytest.mark.parametrize("fmt", ["same", "e4m3", "int8"])
def test_a_non_finite_value_is_not_lost(bad, where, n, fmt):
    """Every row that sees a NaN or infinity (in every column position of a step) has a non-finite output."""
    h = hos()
    t, page, d = 300, 32, 128
    off, kv_len, table, n_pages = R.make_batch([(n, t)], page, 0, 1)
    q = torch.randn((n, 2, d), device="cuda").bfloat16()
    x = torch.randn((t, 1, d), device="cuda").bfloat16()
    first = torch.zeros(2, dtype=torch.int32, device="cuda")
    first[1] = t
    for j in (0, 1, 2, 3, 5, 9, 13, 64, 127, 128, 149):
        cache = make_cache(n_pages, 1, page, d, torch.bfloat16, fmt, 2)
        handle = h.hos_kv_cache(*cache, dtype=torch.bfloat16)
        y = x.clone()
        y[j, 0, 7] = bad
        h.hos_kv_append(handle, y if where == "k" else x, y if where == "v" else x, first, kv_len, table)
        out = h.hos_paged_attention(q, handle, off, kv_len, table, n)["out"]
        # -infinity as a score is a weight of zero: only an 8-bit cache, whose whole vector is NaN then, has to show it;
        # an infinite score may have either sign
        if fmt == "same" and where == "k" and not math.isnan(bad):
            s = (q[:, :, 7].float() * bad) > 0
            seen = ~torch.isfinite(out).all(-1)
            assert bool(seen[s].all())
        else:
            assert not bool(torch.isfinite(out).all(-1).any())
