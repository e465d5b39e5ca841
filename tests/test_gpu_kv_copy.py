"""Copies of whole pages: the bytes of keys, values and scales arrive, and nothing else changes."""
import random

import pytest
import torch

from tests.test_gpu_kv_cache import make_cache

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def hos():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2502_15763_b200 as h
    return h


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def raw(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16) if t.element_size() == 2 else t.view(torch.int32)


def tensors(n_pages, heads, page, d, dt, fmt, seed, strided=False):
    """k, v, k_scale, v_scale (or None); strided: pages lie apart, with room behind each that must stay as it is."""
    out = make_cache(n_pages, heads, page, d, dt, fmt, seed)
    if not strided:
        return list(out)
    wide = []
    for t in out:
        if t is None:
            wide.append(None)
            continue
        buf = torch.zeros((n_pages, t[0].numel() + 32), dtype=torch.uint8 if t.element_size() == 1 else t.dtype, device="cuda")
        buf = buf.view(t.dtype) if t.element_size() == 1 else buf
        view = buf.as_strided(t.shape, (t[0].numel() + 32,) + tuple(t.stride()[1:]))
        raw(view).copy_(raw(t))
        wide.append(view)
    return wide


def check(n_pages, heads, page, d, fmt, src, dst, dt="bf16", layers=1, count=None, other=None, strided=False):
    h = hos()
    caches = [tensors(n_pages, heads, page, d, DT[dt], fmt, 10 + l, strided and l % 2 == 0) for l in range(layers)]
    froms = caches if other is None else [tensors(other, heads, page, d, DT[dt], fmt, 90 + l, strided and l % 2 == 1) for l in range(layers)]
    handles = [h.hos_kv_cache(*t, dtype=DT[dt]) for t in caches]
    sources = None if other is None else [h.hos_kv_cache(*t, dtype=DT[dt]) for t in froms]
    want = [[None if t is None else raw(t).clone() for t in c] for c in caches]
    n = len(src) if count is None else min(len(src), max(0, count))
    for w, f in zip(want, froms):
        for a, t in zip(w, f):
            if a is not None:
                for i in range(n):
                    if 0 <= src[i] < (other or n_pages) and 0 <= dst[i] < n_pages:
                        a[dst[i]] = raw(t)[src[i]]
    one = layers == 1 and count is None
    h.hos_kv_copy_pages(handles[0] if one else handles, dev(src), dev(dst), None if count is None else dev([count]),
                        sources[0] if one and sources else sources)
    torch.cuda.synchronize()
    for c, w in zip(caches, want):
        for t, a in zip(c, w):
            assert t is None or torch.equal(raw(t), a)
            if t is not None and not t.is_contiguous() and n_pages > 1:                       # the room between pages
                gap = t[0].numel()
                buf = raw(t.as_strided((n_pages, gap + 32), (gap + 32, 1)) if t.element_size() > 1 else t.view(torch.uint8).as_strided((n_pages, gap + 32), (gap + 32, 1)))
                assert int(buf[:-1, gap:].abs().sum()) == 0
    bad = [i for i in range(n) if not (0 <= src[i] < (other or n_pages) and 0 <= dst[i] < n_pages)]
    status = handles[0].status
    assert [i for i, x in enumerate(status.tolist()) if x] == bad and all(int(status[i]) == h.HOS_ST_INVALID for i in bad)


@pytest.mark.parametrize("fmt", ["same", "e4m3", "int8"])
@pytest.mark.parametrize("heads,page,d", [(1, 16, 64), (2, 16, 128), (3, 32, 64), (8, 128, 128), (5, 256, 128), (33, 64, 64)])
@pytest.mark.parametrize("moves", [1, 2, 37])
def test_copy(fmt, heads, page, d, moves):
    r = random.Random(moves + heads)
    both = r.sample(range(2 * moves + 5), 2 * moves)
    check(2 * moves + 5, heads, page, d, fmt, both[:moves], both[moves:], dt=["bf16", "f16"][moves % 2])


@pytest.mark.parametrize("layers", [2, 3, 80, 128, 129, 300])
@pytest.mark.parametrize("fmt", ["same", "int8"])
def test_copy_of_many_layers(layers, fmt):
    check(9, 2, 16, 64, fmt, [1, 8, 0], [4, 2, 7], layers=layers, strided=True)


@pytest.mark.parametrize("count", [-3, 0, 1, 4, 5, 100])
def test_copy_with_the_count_on_the_device(count):
    check(12, 2, 32, 64, "e4m3", [0, 1, 2, 3, -1], [11, 10, 9, 8, -1], layers=2, count=count)


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("fmt", ["same", "e4m3"])
def test_copy_from_another_cache(strided, fmt):
    check(6, 3, 16, 128, fmt, [30, 0, 17, 4], [0, 5, 2, 4], other=31, strided=strided)
    check(6, 3, 16, 128, fmt, [30, 30, 17, 17], [0, 5, 2, 4], layers=3, other=31, strided=strided)


def test_one_page_to_many():
    check(40, 2, 16, 64, "int8", [7] * 30, list(range(10, 40)))


def test_pages_out_of_range():
    check(8, 2, 16, 64, "same", [0, -1, 8, 2, 3, 2 ** 31 - 1, -2 ** 31], [4, 5, 6, 8, -1, 7, 1])
    check(8, 2, 16, 64, "e4m3", [0, -1, 8], [4, 5, 6], layers=5)


def test_more_moves_than_status_words():
    h = hos()
    cache = h.hos_kv_cache(*tensors(4, 1, 16, 64, torch.bfloat16, "same", 1))
    h.hos_kv_copy_pages(cache, dev([0] * 3000 + [9]), dev([-1] * 3001))
    assert cache.status.shape[0] >= 3001 and int((cache.status != 0).sum()) == 3001


def test_no_moves():
    h = hos()
    cache = h.hos_kv_cache(*tensors(4, 1, 16, 64, torch.bfloat16, "same", 1))
    before = cache.k.clone()
    h.hos_kv_copy_pages(cache, dev([]), dev([]))
    torch.cuda.synchronize()
    assert torch.equal(cache.k, before)


def test_a_pool_beyond_32_bits():
    """Pages whose offsets need more than 32 bits, in elements and in bytes."""
    h = hos()
    page = torch.empty((2, 256, 128), dtype=torch.bfloat16)
    n = (5 << 30) // (page.numel() * 2)                          # 5 GiB each for keys and values
    k, v = (torch.zeros((n, 2, 256, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[n - 1].normal_()
    v[3].normal_()
    cache = h.hos_kv_cache(k, v)
    h.hos_kv_copy_pages(cache, dev([n - 1, 3]), dev([1, n - 2]))
    torch.cuda.synchronize()
    assert torch.equal(k[1], k[n - 1]) and torch.equal(v[n - 2], v[3]) and bool((v[1] == 0).all()) and bool((k[n - 2] == 0).all())
    assert float(k[1].abs().max()) > 0


def test_captured_with_its_resize():
    """The moves of a resize are made by the copy behind it, replay after replay."""
    h = hos()
    k, v, ks, vs = make_cache(12, 2, 16, 64, torch.bfloat16, "int8", 3)
    cache = h.hos_kv_cache(k, v, ks, vs, dtype=torch.bfloat16)
    refs, lens, table = dev([3] + [0] * 11), dev([5, 5, 5]), dev([[0, -1], [0, -1], [0, -1]])
    new = dev([5, 5, 5])
    first = raw(k[0]).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = h.hos_kv_resize(refs, table, lens, new, 16, out=(refs, table, lens))
        h.hos_kv_copy_pages(cache, r["src"], r["dst"], r["count"])
    graph.replay()
    assert r["count"].tolist() == [0] and table.tolist() == [[0, -1]] * 3
    new.copy_(dev([6, 5, 7]))
    graph.replay()
    torch.cuda.synchronize()
    assert table.tolist() == [[1, -1], [0, -1], [2, -1]] and refs.tolist() == [1, 1, 1] + [0] * 9
    assert torch.equal(raw(k[1]), first) and torch.equal(raw(k[2]), first)
    graph.replay()
    assert r["count"].tolist() == [0] and int(cache.status.abs().sum()) == 0


def test_refusals():
    h = hos()
    a = h.hos_kv_cache(*tensors(4, 2, 16, 64, torch.bfloat16, "same", 1))
    others = [h.hos_kv_cache(*tensors(4, *s, torch.bfloat16, f, 1), dtype=torch.bfloat16) for s, f in (((1, 16, 64), "same"), ((2, 32, 64), "same"),
                                                                                                  ((2, 16, 128), "same"), ((2, 16, 64), "int8"))]
    others.append(h.hos_kv_cache(*tensors(4, 2, 16, 64, torch.float16, "same", 1)))
    one = dev([0])
    for o in others:
        with pytest.raises(ValueError, match="same heads"):
            h.hos_kv_copy_pages([a, o], one, one)
        with pytest.raises(ValueError, match="same heads"):
            h.hos_kv_copy_pages(a, one, one, source=o)
    with pytest.raises(ValueError, match="number of pages"):
        h.hos_kv_copy_pages([a, h.hos_kv_cache(*tensors(5, 2, 16, 64, torch.bfloat16, "same", 1))], one, one)
    for src, dst, count, kind in ((one.long(), one, None, TypeError), (one.cpu(), one, None, TypeError), (one, dev([0, 1]), None, ValueError), (one, one, dev([1, 1]), ValueError),
                                  (one, one, one.float(), TypeError), ([0], one, None, TypeError), (dev([[0]]), dev([[0]]), None, ValueError)):
        with pytest.raises(kind):
            h.hos_kv_copy_pages(a, src, dst, count)
    for bad in ([a.k], [None], [a, 3]):
        with pytest.raises(TypeError):
            h.hos_kv_copy_pages(bad, one, one)
    for bad, src in (([], None), ([a], [a, a])):
        with pytest.raises(ValueError):
            h.hos_kv_copy_pages(bad, one, one, source=src)
