"""Pages that are given up more often than their counts say: every sequence that gives such a page up is reported, whatever the order."""
import random

import pytest
import torch

from tests import pages_reference as P
from tests.test_gpu_kv_pages import Pool, dev, hos

pytestmark = pytest.mark.gpu


def expected(pool, new, rows):
    """The state is that of the step-by-step statement; the givers of a page whose count falls below zero are all reported."""
    refs, table, lens, src, dst, status = P.resize(pool.refs, rows, pool.lens, new, pool.ps, pool.entries)
    cap, count, given = pool.entries * pool.ps, list(pool.refs), []
    for s, (a, b) in enumerate(zip(pool.lens, new)):
        pages = [p for p in rows[s][P.held(b, pool.ps):P.held(a, pool.ps)] if 0 <= p < pool.n_pages] if 0 <= b < a <= cap else []
        given.append(pages)
        for p in pages:
            count[p] -= 1
    for s, pages in enumerate(given):
        if any(count[p] < 0 for p in pages):
            status[s] |= P.INVALID
    return refs, table, lens, src, dst, status


def check(pool, new, in_place):
    refs, table, lens = pool.device(padded=1)
    rows = table.tolist()
    want = expected(pool, new, rows)
    r = hos().hos_kv_resize(refs, table, lens, dev(new), pool.ps, out=(refs, table, lens) if in_place else None)
    assert r["status"].tolist() == want[5]
    assert r["refs"].tolist() == want[0] and r["kv_len"].tolist() == want[2]
    n = len(want[3])
    assert r["count"].tolist() == [n] and r["src"].tolist()[:n] == want[3] and r["dst"].tolist()[:n] == want[4]
    if in_place:
        for s, row in enumerate(want[1]):
            used = max(P.held(x, pool.ps) if 0 <= x <= pool.entries * pool.ps else pool.entries for x in (pool.lens[s], want[2][s]))
            row[used:] = rows[s][used:]
    assert r["page_table"].tolist() == want[1]
    return want[5]


@pytest.mark.parametrize("entries", [6, 3000])
@pytest.mark.parametrize("in_place", [False, True])
def test_one_page_given_up_by_several(entries, in_place):
    """Counts of 0 to 3, up to four givers, holders that keep it; pages twice in one row."""
    pool = Pool(1, 1, 16, 0, 0)
    pool.n_pages, pool.entries = 12, entries
    pool.refs = [0, 1, 2, 3, 2, 1, 1, 0, 1, 0, 0, 0]
    held = [[1, 0], [1, 2], [2, 3], [3, 3], [3, 2], [4, 5], [5, 4], [6], [6, 8], [8, 8], [0, 7]]
    keep = [0, 0, 0, 0, 0, 1, 1, 1, 0, 2, 0]                     # pages that stay
    pool.rows = [row + [-1] * (entries - len(row)) for row in held]
    pool.lens, new = [16 * len(row) for row in held], [16 * n for n in keep]
    status = check(pool, new, in_place)
    # 0: given up twice; 1: twice, held once; 2: three times, held twice; 3: four times; 4, 5: once each; 6, 8: once
    assert status == [4, 4, 4, 4, 4, 0, 0, 0, 0, 0, 4]


@pytest.mark.parametrize("n_seq,page,spare", [(7, 16, 3), (40, 16, 200), (130, 16, 9000), (1100, 4, 500), (1100, 4, 9000), (20000, 4, 9000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_counts_that_are_too_small(n_seq, page, spare, in_place):
    """Random states some of whose counts are lowered, some of whose sequences shrink."""
    for seed in range(3):
        r = random.Random(seed)
        pool = Pool(seed + 40, n_seq, page, 5 * page, spare, shared=0.6, entries=12)
        pool.refs = [x - (r.random() < 0.2) * r.randrange(1, 3) if x else 0 for x in pool.refs]
        pool.refs = [max(x, 0) for x in pool.refs]
        # nobody grows from inside a page: how often that is shared is not known where counts are wrong
        new = [r.choice([0, max(0, n - page), n // 2, n if n % page else n + page]) for n in pool.lens]
        new = [min(n, 12 * page) for n in new]
        new = [n if n <= a or a % page == 0 else a for n, a in zip(new, pool.lens)]
        status = check(pool, new, in_place)
        assert n_seq < 100 or status.count(P.INVALID) > 3


def test_the_status_is_that_of_every_run():
    """In a graph, replayed, and on two streams: the same words."""
    h = hos()
    pool = Pool(2, 600, 16, 100, 9000, shared=0.7, entries=40)
    pool.refs = [min(x, 1) for x in pool.refs]
    new = [0 if s % 3 else n for s, n in enumerate(pool.lens)]
    given = (*pool.device(), dev(new))
    want = expected(pool, new, given[1].tolist())[5]
    assert want.count(P.INVALID) > 50
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = h.hos_kv_resize(*given, 16)
    for _ in range(20):
        graph.replay()
        assert r["status"].tolist() == want
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(10):
        for st in streams:
            with torch.cuda.stream(st):
                got.append(h.hos_kv_resize(*given, 16))
    torch.cuda.synchronize()
    assert all(x["status"].tolist() == want for x in got)
