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
