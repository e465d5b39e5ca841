"""How a trace falls into prefills and stretches of decode iterations without a change of the batch."""
import numpy as np

from paper_2502_15763_b200 import ITER_REC_DTYPE
from paper_2502_15763_b200.drafted import stretches


def trace(*kinds):
    """p: a prefill; d: a decode iteration after which nobody is done; e: one after which somebody is."""
    recs = np.zeros(len(kinds), dtype=ITER_REC_DTYPE)
    for rec, kind in zip(recs, kinds):
        rec["kind_n"] = 3 | (1 << 31 if kind == "p" else 0)
        rec["aux"] = {"p": 7, "d": 0, "e": 2}[kind]
    return recs


def test_stretches():
    assert stretches(trace()) == []
    assert stretches(trace(*"p")) == [(True, [0])]
    assert stretches(trace(*"pddedepd")) == [(True, [0]), (False, [1, 2, 3]), (False, [4, 5]), (True, [6]), (False, [7])]
    assert stretches(trace(*"ppede")) == [(True, [0]), (True, [1]), (False, [2]), (False, [3, 4])]


def test_every_iteration_is_in_one_stretch():
    rng = np.random.default_rng(0)
    for n in (1, 10, 200):
        recs = trace(*rng.choice(list("pddde"), n))
        of = stretches(recs)
        assert [i for _, s in of for i in s] == list(range(n))
        assert all(len(s) == 1 for prefill, s in of if prefill)
        assert all(int(recs[i]["aux"]) == 0 for prefill, s in of if not prefill for i in s[:-1])
