"""A scheduled client's iterations run on the KV-cache operators: every iteration agrees with its trace record, and what the
cache holds at the end of a prefill and some decode rounds gives the attention that the formulas give."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,heads,kv_heads,page", [("int8", 16, 2, 128), ("same", 4, 4, 16)])
def test_replay_follows_the_trace(fmt, heads, kv_heads, page):
    import torch
    assert torch.cuda.is_available()
    from paper_2502_15763_b200 import replay as R
    from workload import workload
    w = workload("c0")
    p, o = (x[0] for x in w.lengths())
    recs, queue = R.client_schedule(p, o, w.n_clients, w.batch_cap, w.kv_budget, w.cost_model, 1)
    assert len(queue) > 0 and len(recs) > 300
    r = R.replay(p, o, recs, queue, w.batch_cap, w.kv_budget, heads=heads, kv_heads=kv_heads, head_dim=64, page=page, fmt=fmt, repeat=0)
    assert len(r["us"]) == len(recs) and r["most_pages"] <= r["n_pages"]
    # every request was prefilled once and decoded o times
    assert int(r["tokens"][r["prefill"]].sum()) == int(p[queue].sum())
    assert int(r["n"][~r["prefill"]].sum()) == int(o[queue].sum())
    timed = R.replay(p, o, recs, queue, w.batch_cap, w.kv_budget, heads=heads, kv_heads=kv_heads, head_dim=64, page=page, fmt=fmt, max_iters=30,
                     repeat=2)
    f = R.fit(timed, 2)
    assert f["iterations"] == 30 and (timed["us"] > 0).all() and np.isfinite(f["decode_us_per_kv_token"])


def test_replay_notices_a_wrong_trace():
    from paper_2502_15763_b200 import replay as R
    from workload import workload
    w = workload("c0")
    p, o = (x[0] for x in w.lengths())
    recs, queue = R.client_schedule(p, o, w.n_clients, w.batch_cap, w.kv_budget, w.cost_model, 0)
    recs = recs.copy()
    recs["tokens"][5] += 1
    with pytest.raises(RuntimeError, match="iteration 5"):
        R.replay(p, o, recs, queue, w.batch_cap, w.kv_budget, heads=2, kv_heads=1, head_dim=64, fmt="same", max_iters=10, repeat=0)


def test_a_client_without_requests():
    """Nothing to run is no error: empty arrays, no fit."""
    from paper_2502_15763_b200 import ITER_REC_DTYPE, replay as R
    from workload import workload
    w = workload("c0")
    p, o = (x[0] for x in w.lengths())
    none = np.zeros(0, dtype=ITER_REC_DTYPE)
    for queue, most in ((np.zeros(0, dtype=np.int64), None), (np.arange(3), 0)):
        r = R.replay(p, o, none, queue, w.batch_cap, w.kv_budget, heads=2, kv_heads=1, head_dim=64, fmt="same", max_iters=most, repeat=0)
        assert len(r["us"]) == len(r["n"]) == len(r["tokens"]) == 0 and r["most_pages"] == 0
        f = R.fit(r, 80)
        assert f["iterations"] == 0 and f["median_decode_us"] is None and "decode_kv_div" not in f
    # a workload of one request on four clients leaves three of them without any
    recs, queue = R.client_schedule(p[:1], o[:1], w.n_clients, w.batch_cap, w.kv_budget, w.cost_model, 3)
    r = R.replay(p[:1], o[:1], recs, queue, w.batch_cap, w.kv_budget, heads=2, kv_heads=1, head_dim=64, fmt="same", repeat=0)
    assert len(r["us"]) == len(recs)


@pytest.mark.parametrize("fmt", ["same", "int8"])
def test_every_timed_layer_has_a_cache_of_its_own(fmt, monkeypatch):
    """The layers of a timed iteration must not find each other's keys and values on the chip; all of them hold the same."""
    import torch
    from paper_2502_15763_b200 import replay as R
    from workload import workload
    made, make = [], R.hos_kv_cache

    def recorded(*args, **kw):
        made.append(make(*args, **kw))
        return made[-1]
    monkeypatch.setattr(R, "hos_kv_cache", recorded)
    w = workload("c0")
    p, o = (x[0] for x in w.lengths())
    recs, queue = R.client_schedule(p, o, w.n_clients, w.batch_cap, w.kv_budget, w.cost_model, 1)
    r = R.replay(p, o, recs, queue, w.batch_cap, w.kv_budget, heads=8, kv_heads=2, head_dim=64, page=32, fmt=fmt, max_iters=6, repeat=5)
    assert (r["us"] > 0).all() and len(made) == 5
    assert len({c.k.data_ptr() for c in made}) == 5
    one = R.cache_bytes(w.batch_cap, w.kv_budget, 2, 64, 32, fmt)
    for c in made:
        assert sum(t.numel() * t.element_size() for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None) == one
        assert torch.equal(c.k.view(torch.uint8), made[0].k.view(torch.uint8)) and torch.equal(c.v.view(torch.uint8), made[0].v.view(torch.uint8))
    assert bool(made[0].k.view(torch.uint8).any())


@pytest.mark.parametrize("fmt,heads,kv_heads,d,page", [("int8", 8, 2, 64, 32), ("e4m3", 8, 8, 128, 128), ("same", 4, 1, 64, 16)])
def test_replay_holds_and_attends_to_what_was_appended(fmt, heads, kv_heads, d, page):
    """After prefills and decode rounds, what the pages of the running requests hold is what was appended, bit for bit, and the outputs
    are the formulas' on that (bounds as in the tests of attention, with the unit roundoffs of bf16 and of the weights)."""
    import math
    import torch
    from paper_2502_15763_b200 import replay as R
    from tests import kv_reference as K
    from tests.test_gpu_kv_cache import CODES
    from workload import workload
    w = workload("c0")
    p, o = (x[0] for x in w.lengths())
    recs, queue = R.client_schedule(p, o, w.n_clients, w.batch_cap, w.kv_budget, w.cost_model, 1)
    held, checked = {}, []                                        # request -> its appended keys and values, call by call

    def watch(it, requests, x, cache, off, kv_len, table, out):
        starts = off.tolist()
        for s, r in enumerate(requests):
            mine = x[starts[s]:starts[s + 1]]
            held.setdefault(r, []).append((mine[:, heads:heads + kv_heads], mine[:, heads + kv_heads:]))
        prefill = bool(recs[it]["kind_n"] >> 31)
        if not (prefill and len(checked) % 2 == 0 or not prefill and it % 7 == 0):
            return
        checked.append(prefill)
        lengths = kv_len.tolist()
        assert lengths == [sum(len(k) for k, _ in held[r]) for r in requests]
        for s, r in enumerate(requests):
            for i, (store, scale) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
                new = torch.cat([kv[i] for kv in held[r]])
                want = new.double() if CODES[fmt] is None else K.values(*K.quantise(new, CODES[fmt]))
                assert torch.equal(K.sequence(store, scale, table[s], lengths[s], page), want)
        pairs = [(b - a, t) for a, b, t in zip(starts, starts[1:], lengths)]
        want, _, mag, dot = K.attention(x[:, :heads], cache.k, cache.v, cache.k_scale, cache.v_scale, pairs, off, table, page, 1 / math.sqrt(d), True, 0)
        u, uw = 2.0 ** -8, 2.0 ** -8 if fmt == "same" else 2.0 ** -11
        e = (d + 4) * 2.0 ** -24 * dot
        bound = u * want.abs() + (uw + 2.0 ** -18 + 2 * e[..., None]) * (1 + u) * mag + 2.0 ** -24
        assert float(((out.double() - want).abs() / bound).max()) <= 1.0, it

    R.replay(p, o, recs, queue, w.batch_cap, w.kv_budget, heads=heads, kv_heads=kv_heads, head_dim=d, page=page, fmt=fmt, max_iters=60, repeat=0,
             watch=watch)
    assert any(checked) and not all(checked)
