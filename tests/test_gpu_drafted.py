"""The page and draft operators as they are used together: a client's schedule with drafted tokens, samples of one prompt."""
import math

import numpy as np
import pytest
import torch

from tests import kv_reference as K
from tests.test_gpu_kv_cache import CODES, make_cache

pytestmark = pytest.mark.gpu


def schedule(client=1):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2502_15763_b200 import replay as R
    from workload import workload
    w = workload("c0")
    p, o = (x[0] for x in w.lengths())
    return w, p, o, *R.client_schedule(p, o, w.n_clients, w.batch_cap, w.kv_budget, w.cost_model, client)


@pytest.mark.parametrize("fmt,heads,kv_heads,d,page,drafts", [("int8", 8, 2, 64, 16, 4), ("e4m3", 4, 4, 128, 128, 1), ("same", 4, 1, 64, 32, 7)])
def test_what_the_pages_hold_is_what_was_kept(fmt, heads, kv_heads, d, page, drafts):
    from paper_2502_15763_b200 import drafted as D
    w, p, o, recs, queue = schedule()
    held, calls = {}, [0]

    def watch(requests, x, off, kept, client):
        starts = off.tolist()
        for s, (r, k) in enumerate(zip(requests, kept)):
            mine = x[starts[s]:starts[s] + k]
            held.setdefault(r, []).append((mine[:, heads:heads + kv_heads], mine[:, heads + kv_heads:]))
        calls[0] += 1
        if calls[0] % 5:
            return
        lengths, refs = client.kv_len.tolist(), torch.zeros_like(client.refs)
        assert lengths == [sum(len(k) for k, _ in held[r]) for r in client.requests] + [0] * (client.rows - len(client.requests))
        for s, r in enumerate(client.requests):
            refs[client.table[s, :-(-lengths[s] // page)].long()] += 1
            for i in range(2):
                new = torch.cat([kv[i] for kv in held[r]])
                want = new.double() if CODES[fmt] is None else K.values(*K.quantise(new, CODES[fmt]))
                for cache in client.caches:
                    store, scale = ((cache.k, cache.k_scale), (cache.v, cache.v_scale))[i]
                    assert torch.equal(K.sequence(store, scale, client.table[s], lengths[s], page), want)
        assert torch.equal(refs, client.refs)

    r = D.replay(p, o, recs, queue, w.batch_cap, w.kv_budget, drafts=drafts, vocab=500, heads=heads, kv_heads=kv_heads, head_dim=d, page=page, fmt=fmt, layers=2,
                 compact_every=2, max_iters=90, watch=watch)
    assert calls[0] > 20 and r["rounds"] < r["iterations"] and 0 < r["accepted"] < r["drafts"] and r["tokens"] > 0


def test_a_whole_schedule():
    """Every request makes its tokens; without drafts there is a round for every decode iteration."""
    from paper_2502_15763_b200 import drafted as D
    w, p, o, recs, queue = schedule(0)
    decodes = int((recs["kind_n"] >> 31 == 0).sum())
    for drafts, agree in ((0, 0.5), (3, 1.0), (5, 0.3)):
        r = D.replay(p, o, recs, queue, w.batch_cap, w.kv_budget, drafts=drafts, agree=agree, vocab=300, heads=2, kv_heads=1, head_dim=64, page=16,
                     fmt="same", compact_every=5)
        assert r["iterations"] == len(recs) and r["tokens"] == int(o[queue].sum()) and r["most_pages"] <= r["pages"]
        assert r["rounds"] == decodes if drafts == 0 else r["rounds"] < decodes
        assert agree < 1.0 or r["accepted"] == r["drafts"]


def test_a_wrong_trace_and_none():
    from paper_2502_15763_b200 import ITER_REC_DTYPE, drafted as D
    w, p, o, recs, queue = schedule(0)
    more = dict(vocab=50, heads=2, kv_heads=1, head_dim=64, fmt="same", max_iters=10)
    wrong = recs.copy()
    wrong["tokens"][0] += 1
    with pytest.raises(RuntimeError, match="iteration 0"):
        D.replay(p, o, wrong, queue, w.batch_cap, w.kv_budget, **more)
    r = D.replay(p, o, np.zeros(0, dtype=ITER_REC_DTYPE), queue, w.batch_cap, w.kv_budget, **more)
    assert r["iterations"] == r["rounds"] == r["tokens"] == 0


@pytest.mark.parametrize("fmt", ["same", "int8"])
@pytest.mark.parametrize("page,length", [(16, 37), (32, 64), (16, 16), (128, 5)])
def test_samples_of_one_prompt(fmt, page, length):
    """A prompt is appended once, forked into five samples, and each goes on with tokens of its own: what they attend to is what five
    caches of their own would hold, bit for bit; once they are gone all pages are free."""
    import paper_2502_15763_b200 as h
    dt, hk, hq, d, n = torch.bfloat16, 2, 4, 64, 5
    k, v, ks, vs = make_cache(40, hk, page, d, dt, fmt, 1)
    cache = h.hos_kv_cache(k, v, ks, vs, dtype=dt)
    g = torch.Generator(device="cuda").manual_seed(length)

    def dev(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    width = 12
    state = dev([0] * 40), torch.full((1, width), -1, dtype=torch.int32, device="cuda"), dev([0])
    r = h.hos_kv_resize(*state, dev([length]), page)
    x = torch.randn((length, hq + 2 * hk, d), generator=g, device="cuda").to(dt)
    h.hos_kv_append(cache, x[:, hq:hq + hk], x[:, hq + hk:], dev([0, length]), r["kv_len"], r["page_table"])
    r = h.hos_kv_fork(r["refs"], r["page_table"], r["kv_len"], dev([0] * n), page)
    apart = h.hos_kv_cache(*make_cache(n * width, hk, page, d, dt, fmt, 2), dtype=dt)       # every sample on pages of its own
    own_table = torch.arange(n * width, dtype=torch.int32, device="cuda").view(n, width)
    full = x.repeat(n, 1, 1)
    h.hos_kv_append(apart, full[:, hq:hq + hk], full[:, hq + hk:], dev([i * length for i in range(n + 1)]), dev([length] * n), own_table)
    for step in range(2 * page + 3):
        r = h.hos_kv_resize(r["refs"], r["page_table"], r["kv_len"], r["kv_len"] + 1, page)
        assert int(r["count"]) == (n - 1 if step == 0 and length % page else 0)
        h.hos_kv_copy_pages(cache, r["src"], r["dst"], r["count"])
        y = torch.randn((n, hq + 2 * hk, d), generator=g, device="cuda").to(dt)
        off = dev(list(range(n + 1)))
        outs = []
        for c, table in ((cache, r["page_table"]), (apart, own_table)):
            h.hos_kv_append(c, y[:, hq:hq + hk], y[:, hq + hk:], off, r["kv_len"], table)
            outs.append(h.hos_paged_attention(y[:, :hq], c, off, r["kv_len"], table, 1, want_lse=True))
        assert torch.equal(outs[0]["out"], outs[1]["out"]) and torch.equal(outs[0]["lse"], outs[1]["lse"])
        if step == page:                                         # the pool is moved together in between
            r = h.hos_kv_compact(r["refs"], r["page_table"], r["kv_len"], page)
            h.hos_kv_copy_pages(cache, r["src"], r["dst"], r["count"])
    shared = length // page
    assert int(r["refs"].sum()) == n * math.ceil((length + 2 * page + 3) / page) and int((r["refs"] == n).sum()) == shared
    r = h.hos_kv_fork(r["refs"], r["page_table"], r["kv_len"], dev([3, -1, 3]), page)
    assert r["refs"].max() == 2 and r["kv_len"].tolist() == [length + 2 * page + 3, 0, length + 2 * page + 3]
    r = h.hos_kv_resize(r["refs"], r["page_table"], r["kv_len"], dev([0, 0, 0]), page)
    assert int(r["refs"].abs().sum()) == 0 and int(cache.status.abs().sum()) == 0
