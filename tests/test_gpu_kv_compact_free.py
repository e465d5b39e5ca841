"""Pages that a sequence holds although their counts say that they are free, wherever they lie: hos_kv_compact reports each such sequence."""
import random

import pytest
import torch

from tests import pages_reference as P
from tests.test_gpu_kv_pages import Pool, dev, hos

pytestmark = pytest.mark.gpu


def expected(pool, rows):
    refs, table, src, dst, status = P.compact(pool.refs, rows, pool.lens, pool.ps, pool.entries)
    cap = pool.entries * pool.ps
    for s, n in enumerate(pool.lens):
        if 0 <= n <= cap and any(0 <= p < pool.n_pages and not pool.refs[p] for p in rows[s][:P.held(n, pool.ps)]):
            status[s] |= P.INVALID
    return refs, table, src, dst, status


def check(pool, in_place):
    refs, table, lens = pool.device(padded=1)
    want = expected(pool, table.tolist())
    r = hos().hos_kv_compact(refs, table, lens, pool.ps, out=(refs, table, lens) if in_place else None)
    assert r["status"].tolist() == want[4]
    assert r["refs"].tolist() == want[0] and r["count"].tolist() == [len(want[2])]
    n = len(want[2])
    assert r["src"].tolist()[:n] == want[2] and r["dst"].tolist()[:n] == want[3]
    got = r["page_table"].tolist()
    for s, length in enumerate(pool.lens):
        used = P.held(length, pool.ps) if in_place else pool.entries
        assert got[s][:used] == want[1][s][:used]
    return want


@pytest.mark.parametrize("n_seq,page,entries", [(1, 16, 8), (12, 16, 30), (40, 16, 60), (40, 16, 700), (300, 4, 90), (1200, 4, 40)])
@pytest.mark.parametrize("in_place", [False, True])
def test_held_pages_that_are_free(n_seq, page, entries, in_place):
    """Below the pages that stay, among the holes that others move to, and behind them; in any entry of a row."""
    for seed in range(4):
        r = random.Random(100 * n_seq + seed)
        pool = Pool(seed, n_seq, page, 7 * page, (0, 3, 70, 4000)[seed], shared=0.2, entries=entries)
        n_live = sum(1 for x in pool.refs if x)
        low, high = [p for p in range(n_live) if not pool.refs[p]], [p for p in range(n_live, pool.n_pages) if not pool.refs[p]]
        bad = 0
        for s in range(n_seq):
            held = P.held(pool.lens[s], page)
            if held and r.random() < 0.3:
                pages = low if r.random() < 0.7 and low else high or low
                if pages:
                    pool.rows[s][r.randrange(held)] = r.choice(pages)
                    bad += 1
        status = check(pool, in_place)[4]
        assert sum(x == P.INVALID for x in status) == bad


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n_pages", [33, 1000, 9000, 70001])
def test_every_free_page_held_by_a_sequence_of_its_own(n_pages, in_place):
    """Each page in a row of one: exactly the rows of the free ones are reported, at every place of a group of pages."""
    r = random.Random(n_pages)
    pool = Pool(1, 1, 1, 0, 0)
    pool.n_pages, pool.entries = n_pages, 1
    pool.refs = [int(r.random() < 0.6) for _ in range(n_pages)]
    pool.rows, pool.lens = [[p] for p in range(n_pages)], [1] * n_pages
    assert check(pool, in_place)[4] == [0 if x else P.INVALID for x in pool.refs]


def test_nothing_is_in_use():
    """All pages are free, and rows hold some of them."""
    pool = Pool(3, 20, 16, 200, 5)
    pool.refs = [0] * pool.n_pages
    for in_place in (False, True):
        assert check(pool, in_place)[4] == [P.INVALID if n else 0 for n in pool.lens]
