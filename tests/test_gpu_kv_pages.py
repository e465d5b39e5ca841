"""Resize, fork and compact against the same written out step by step; whole numbers, so everything has to be equal."""
import random

import pytest
import torch

from tests import pages_reference as P

pytestmark = pytest.mark.gpu


def hos():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2502_15763_b200 as h
    return h


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    """A consistent state with shared pages, in Python and on the device."""

    def __init__(self, seed, n_seq, page_size, longest, spare, shared=0.3, entries=None):
        r = random.Random(seed)
        self.ps, used, rows, lens = page_size, 0, [], []
        for s in range(n_seq):
            if rows and r.random() < shared:
                p = r.randrange(len(rows))
                keep = r.randrange(len(rows[p]) + 1)
                row, n = list(rows[p][:keep]), min(lens[p], keep * page_size)
                if keep and r.random() < 0.3:
                    n = max((keep - 1) * page_size + 1, n - r.randrange(page_size))
                if r.random() < 0.5:
                    n = max(n, keep * page_size)
                    more = r.randrange(longest // 2 + 1)
                    fresh = P.held(n + more, page_size) - keep
                    row, n = row + list(range(used, used + fresh)), n + more
                    used += fresh
            else:
                n = r.choice([0, 1, page_size, page_size + 1, r.randrange(longest + 1)])
                row = list(range(used, used + P.held(n, page_size)))
                used += len(row)
            rows.append(row)
            lens.append(n)
        self.n_pages = max(1, used + spare)
        order = list(range(self.n_pages))
        r.shuffle(order)
        self.entries = entries or max([len(x) for x in rows] + [1]) + 3
        self.lens = lens
        self.rows = [[order[p] for p in row] + [-1] * (self.entries - len(row)) for row in rows]
        self.refs = [0] * self.n_pages
        for row in self.rows:
            for p in row:
                if p >= 0:
                    self.refs[p] += 1
        assert all(P.held(n, page_size) == sum(1 for p in row if p >= 0) for n, row in zip(lens, self.rows))

    def device(self, padded=0, dirt=None):
        table = torch.full((len(self.rows), self.entries + padded), -7, dtype=torch.int32, device="cuda")
        if self.rows:
            t = dev(self.rows)
            if dirt is not None:
                t = torch.where(t < 0, dirt, t)
            table[:, :self.entries] = t
        return dev(self.refs), table[:, :self.entries], dev(self.lens)

    def targets(self, seed, most):
        r, cap = random.Random(seed), self.entries * self.ps
        return [min(cap, max(0, r.choice([0, n, n + 1, n + 5, n - 1, n - self.ps, n + self.ps, r.randrange(cap + 1) if most else n]))) for n in self.lens]


def check_resize(pool, new, in_place=False, padded=0, dirt=None):
    h = hos()
    refs, table, lens = pool.device(padded, dirt)
    keep = [x.clone() for x in (refs, table, lens)]
    rows = table.tolist()
    r = h.hos_kv_resize(refs, table, lens, dev(new), pool.ps, out=(refs, table, lens) if in_place else None)
    w_refs, w_rows, w_lens, src, dst, status = P.resize(pool.refs, rows, pool.lens, new, pool.ps, pool.entries)
    assert r["status"].tolist() == status
    assert r["kv_len"].tolist() == w_lens
    assert r["count"].tolist() == [len(src)]
    n = len(rows)
    assert r["src"].tolist() == src + [-1] * (n - len(src)) and r["dst"].tolist() == dst + [-1] * (n - len(dst))
    assert r["refs"].tolist() == w_refs
    got = r["page_table"].tolist()
    if in_place:                                               # entries that were not held before or after stay
        for s in range(n):
            used = max(P.held(x, pool.ps) if 0 <= x <= pool.entries * pool.ps else pool.entries for x in (pool.lens[s], w_lens[s]))
            w_rows[s][used:] = rows[s][used:]
        assert r["refs"].data_ptr() == refs.data_ptr() and r["page_table"].data_ptr() == table.data_ptr()
    else:
        assert all(torch.equal(a, b) for a, b in zip(keep, (refs, table, lens)))
    assert got == w_rows
    if padded and in_place:
        assert bool((table.as_strided((n, pool.entries + padded), (pool.entries + padded, 1))[:, pool.entries:] == -7).all())
    return r


SIZES = [(1, 1), (1, 16), (2, 128), (7, 16), (16, 128), (33, 7), (130, 16), (300, 32), (1100, 16)]


@pytest.mark.parametrize("n_seq,page", SIZES)
@pytest.mark.parametrize("spare", [0, 3, 4000])
@pytest.mark.parametrize("in_place", [False, True])
def test_resize(n_seq, page, spare, in_place):
    for seed in range(3):
        pool = Pool(seed, n_seq, page, 40 * page if n_seq < 200 else 6 * page, spare)
        check_resize(pool, pool.targets(seed, seed > 0), in_place, padded=seed * 3, dirt=[None, 99999999, 0][seed])


@pytest.mark.parametrize("spare", [0, 1, 5, 11, 40])
def test_resize_runs_out_of_pages(spare):
    """The first sequence without its pages and all growing ones after it keep their lengths; shrinking ones do not."""
    for seed in range(4):
        pool = Pool(100 + seed, 24, 16, 300, spare, shared=0.5)
        r = random.Random(seed)
        new = [r.choice([n, n + 1, n + 40, max(0, n - 30)]) for n in pool.lens]
        new = [min(n, pool.entries * 16) for n in new]
        check_resize(pool, new, in_place=bool(seed % 2))


@pytest.mark.parametrize("n_seq,length,fits", [(9, 20, True), (9, 20, False), (40, 33, True), (1100, 17, True)])
def test_resize_of_sequences_that_share_their_last_page(n_seq, length, fits):
    """Everybody grows inside one page: all but the last get a copy; if one stays, the last gets one, too."""
    page, pool = 16, Pool(1, 1, 16, 1, 0, entries=4)
    have = P.held(length, page)
    pool.rows = [list(range(have)) + [-1] * (4 - have) for _ in range(n_seq)]
    pool.lens, pool.n_pages = [length] * n_seq, have + (n_seq if fits else n_seq // 2)
    pool.refs = [n_seq] * have + [0] * (pool.n_pages - have)
    for new in ([length + 1] * n_seq, [length] + [length + 1] * (n_seq - 1), [length + 1] * (n_seq - 1) + [length], [0] + [length + 2] * (n_seq - 1),
                [length + 1] * (n_seq - 1) + [0], [length - 1] * n_seq):
        r = check_resize(pool, new)
        if fits and new == [length + 1] * n_seq:
            assert int(r["count"]) == n_seq - 1 and int(r["page_table"][n_seq - 1, have - 1]) == have - 1


def test_resize_nothing_and_everything():
    pool = Pool(3, 50, 16, 500, 10)
    check_resize(pool, list(pool.lens))
    r = check_resize(pool, [0] * 50)
    assert int(r["refs"].abs().sum()) == 0 and bool((r["page_table"] == -1).all())
    h = hos()
    empty = h.hos_kv_resize(dev([0, 2]), torch.zeros((0, 4), dtype=torch.int32, device="cuda"), dev([]), dev([]), 16)
    assert empty["refs"].tolist() == [0, 2] and empty["count"].tolist() == [0] and empty["page_table"].shape == (0, 4)
    none = h.hos_kv_resize(dev([0, 0]), torch.zeros((3, 0), dtype=torch.int32, device="cuda"), dev([0, 0, 0]), dev([0, 1, 0]), 16)
    assert none["status"].tolist() == [0, h.HOS_ST_INVALID, 0] and none["kv_len"].tolist() == [0, 0, 0]


@pytest.mark.parametrize("in_place", [False, True])
def test_resize_with_bad_data(in_place):
    """Lengths out of range, page numbers out of range, pages given up more often than they are held."""
    pool = Pool(5, 20, 16, 300, 30, shared=0.0)
    new = pool.targets(1, True)
    pool.lens[2], new[3], new[4], pool.lens[6] = -1, -5, pool.entries * 16 + 1, 2 ** 31 - 1
    pool.lens[8], new[8] = 40, 3
    pool.rows[8] = [pool.n_pages, -3, 2 ** 31 - 1] + [-1] * (pool.entries - 3)
    pool.lens[9], new[9] = 17, 18
    pool.rows[9] = [0, pool.n_pages + 5] + [-1] * (pool.entries - 2)
    free = [p for p, r in enumerate(pool.refs) if r == 0]
    pool.lens[10], new[10] = 20, 0
    pool.rows[10] = [free[0], free[1]] + [-1] * (pool.entries - 2)
    check_resize(pool, new, in_place)


def check_fork(pool, parent, refs_in_place=False, padded=0):
    h = hos()
    refs, table, lens = pool.device(padded)
    out = None
    if refs_in_place:
        wide = torch.full((len(parent), pool.entries + 2), -9, dtype=torch.int32, device="cuda")
        out = (refs, wide[:, :pool.entries], torch.empty(len(parent), dtype=torch.int32, device="cuda"))
    r = h.hos_kv_fork(refs, table, lens, dev(parent), pool.ps, out=out)
    w_refs, w_rows, w_lens, status = P.fork(pool.refs, pool.rows, pool.lens, parent, pool.ps, pool.entries)
    assert r["status"].tolist() == status and r["kv_len"].tolist() == w_lens
    assert r["refs"].tolist() == w_refs and r["page_table"].tolist() == w_rows
    if refs_in_place:
        assert bool((wide[:, pool.entries:] == -9).all())
    else:
        assert refs.tolist() == pool.refs
    return r


@pytest.mark.parametrize("n_seq,page", SIZES)
@pytest.mark.parametrize("kind", ["same", "samples", "beams", "none", "thin"])
def test_fork(n_seq, page, kind):
    pool = Pool(n_seq, n_seq, page, 30 * page if n_seq < 200 else 5 * page, 5)
    r = random.Random(n_seq)
    parent = {"same": list(range(n_seq)), "samples": [i // 4 for i in range(4 * n_seq)], "beams": [r.randrange(n_seq) for _ in range(n_seq)],
              "none": [-1] * 3, "thin": [s for s in range(n_seq) if r.random() < 0.5]}[kind]
    check_fork(pool, parent)
    check_fork(pool, parent, refs_in_place=True, padded=1)
    if kind == "thin":
        check_fork(pool, [])


def test_fork_with_bad_data():
    pool = Pool(2, 12, 16, 200, 4, shared=0.0)
    pool.lens[3], pool.lens[4] = -2, pool.entries * 16 + 1
    pool.lens[5] = 40
    pool.rows[5] = [-1, pool.n_pages, 0] + [-1] * (pool.entries - 3)
    r = check_fork(pool, [0, 3, 4, 5, 5, 12, -2, 2 ** 31 - 1, -2 ** 31, -1, 1])
    assert r["status"].tolist() == [0, 4, 4, 4, 4, 4, 4, 4, 4, 0, 0]


def check_compact(pool, in_place=False, padded=0, dirt=None):
    h = hos()
    refs, table, lens = pool.device(padded, dirt)
    rows = table.tolist()
    r = h.hos_kv_compact(refs, table, lens, pool.ps, out=(refs, table, lens) if in_place else None)
    w_refs, w_rows, src, dst, status = P.compact(pool.refs, rows, pool.lens, pool.ps, pool.entries)
    fill = [-1] * (pool.n_pages - len(src))
    assert r["status"].tolist() == status and r["count"].tolist() == [len(src)]
    assert r["src"].tolist() == src + fill and r["dst"].tolist() == dst + fill
    assert r["refs"].tolist() == w_refs and r["kv_len"].tolist() == pool.lens
    if in_place:
        for s, n in enumerate(pool.lens):
            used = P.held(n, pool.ps) if 0 <= n <= pool.entries * pool.ps else pool.entries
            w_rows[s][used:] = rows[s][used:]
    assert r["page_table"].tolist() == w_rows
    return r


@pytest.mark.parametrize("n_seq,page", SIZES)
@pytest.mark.parametrize("spare", [0, 1, 40, 70000])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(n_seq, page, spare, in_place):
    pool = Pool(n_seq + 7, n_seq, page, 30 * page if n_seq < 200 else 5 * page, spare)
    r = check_compact(pool, in_place, padded=2, dirt=0 if in_place else None)
    n = sum(1 for x in pool.refs if x)
    assert bool((r["refs"][:n] > 0).all()) and int(r["refs"][n:].abs().sum()) == 0


def test_compact_with_bad_data():
    for in_place in (False, True):
        pool = Pool(2, 12, 16, 200, 60, shared=0.0)
        pool.lens[3], pool.lens[4] = -2, pool.entries * 16 + 1
        pool.lens[5] = 70
        n_live = sum(1 for r in pool.refs if r)
        stray = [p for p in range(n_live, pool.n_pages) if not pool.refs[p]]
        pool.rows[5] = [-1, pool.n_pages, stray[0], stray[-1], 0] + [-1] * (pool.entries - 5)
        check_compact(pool, in_place)
    empty = Pool(1, 3, 16, 0, 5)
    empty.refs, empty.lens, empty.rows = [0] * empty.n_pages, [0] * 3, [[-1] * empty.entries] * 3
    check_compact(empty)


@pytest.mark.parametrize("n_seq,shared", [(2000, 0.0), (1100, 0.3), (40000, 0.2)])
def test_more_sequences_than_threads(n_seq, shared):
    """One block with several sequences a thread; sixteen of them."""
    pool = Pool(n_seq, n_seq, 4, 4, 700 if n_seq < 6000 else 9000, shared=shared, entries=2 if shared == 0.0 else None)
    new = pool.targets(1, True)
    for in_place in (False, True):
        check_resize(pool, new, in_place)
        check_compact(pool, in_place)
    r = random.Random(n_seq)
    check_fork(pool, [r.randrange(n_seq) for _ in range(n_seq)])
    check_fork(pool, [r.randrange(-1, n_seq) for _ in range(3 * n_seq // 2)], refs_in_place=True)


def test_compacting_a_million_pages_in_place():
    pool = Pool(4, 30, 1, 60000, 0, shared=0.0)
    more = 1_100_000 - pool.n_pages
    r = random.Random(1)
    at = sorted(r.sample(range(1_100_000), pool.n_pages))
    pool.rows = [[at[p] if p >= 0 else -1 for p in row] for row in pool.rows]
    pool.refs, pool.n_pages = [0] * 1_100_000, pool.n_pages + more
    for row in pool.rows:
        for p in row:
            if p >= 0:
                pool.refs[p] += 1
    check_compact(pool, True)
    check_compact(pool, False)


def test_a_million_pages():
    """Numbers beyond 16 bits, rows of many pieces; a sequence that takes nearly everything."""
    h = hos()
    n, entries = 1_000_003, 70_001
    refs = torch.zeros(n, dtype=torch.int32, device="cuda")
    table = torch.full((20, entries), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(20, dtype=torch.int32, device="cuda")
    new = torch.tensor([(i * 3701 + 1) * 16 for i in range(18)] + [70_000 * 16 + 3, 5], dtype=torch.int32, device="cuda")
    r = h.hos_kv_resize(refs, table, lens, new, 16)
    need = (new.cpu() + 15) // 16
    assert int(r["status"].abs().sum()) == 0 and int(r["refs"].sum()) == int(need.sum())
    first = 0
    for s in range(20):                                          # lowest numbers first, in order
        k = int(need[s])
        assert torch.equal(r["page_table"][s, :k], torch.arange(first, first + k, dtype=torch.int32, device="cuda"))
        assert bool((r["page_table"][s, k:] == -1).all())
        first += k
    drop = new.clone()
    drop[::2] = 0
    r2 = h.hos_kv_resize(r["refs"], r["page_table"], r["kv_len"], drop, 16)
    r3 = h.hos_kv_compact(r2["refs"], r2["page_table"], r2["kv_len"], 16)
    live = int(((drop.cpu() + 15) // 16).sum())
    assert int(r3["refs"][:live].sum()) == live == int(r3["refs"].sum())
    mine = r3["page_table"][r3["page_table"] >= 0]
    assert torch.equal(mine.sort().values, torch.arange(live, dtype=torch.int32, device="cuda"))
    for s in range(1, 20, 2):                                    # what a sequence holds is moved in its place
        k = int(need[s])
        to = dict(zip(r3["src"][:int(r3["count"])].tolist(), r3["dst"][:int(r3["count"])].tolist()))
        assert [to.get(p, p) for p in r2["page_table"][s, :k].tolist()] == r3["page_table"][s, :k].tolist()


@pytest.mark.parametrize("more", [20, 700])
def test_captured_and_on_other_streams(more):
    """In place, replayed: every replay is one more round.  Two calls at once on two streams have workspaces of their own.  By one block
    and by sixteen."""
    h = hos()
    pool = Pool(9, 16, 16, 200, 300)
    pool.entries += more
    pool.rows = [row + [-1] * more for row in pool.rows]
    refs, table, lens = pool.device()
    one = torch.ones_like(lens)
    new = torch.empty_like(lens)

    def step():
        torch.add(lens, one, out=new)
        return h.hos_kv_resize(refs, table, lens, new, 16, out=(refs, table, lens))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = step()
    state = (pool.refs, pool.rows, pool.lens)
    for _ in range(40):
        graph.replay()
        want = P.resize(*state, [n + 1 for n in state[2]], 16, pool.entries)
        state = want[:3]
        assert refs.tolist() == state[0] and table.tolist() == state[1] and lens.tolist() == state[2]
        assert r["count"].tolist() == [len(want[3])] and r["status"].tolist() == want[5]
    pools = [Pool(50 + i, 64, 16, 400, 50, entries=more + 60) for i in range(2)]
    given = [(p.device(), dev(p.targets(i, True)), p.targets(i, True)) for i, p in enumerate(pools)]
    streams, got = [torch.cuda.Stream() for _ in pools], []
    torch.cuda.synchronize()
    for _ in range(20):
        for st, (d, new, _) in zip(streams, given):
            with torch.cuda.stream(st):
                got.append(h.hos_kv_resize(*d, new, 16))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        p = pools[i % 2]
        want = P.resize(p.refs, p.rows, p.lens, given[i % 2][2], 16, p.entries)
        assert r["refs"].tolist() == want[0] and r["page_table"].tolist() == want[1]


@pytest.mark.parametrize("entries", [40, 600])
def test_a_chain_of_calls_in_one_graph(entries):
    """Resize, fork, compact and resize again, each on what the one before left, replayed on other states."""
    h = hos()
    pools = [Pool(70 + i, 40, 16, 300, 60, entries=entries) for i in range(4)]
    r = random.Random(3)
    parent = [r.randrange(-1, 40) for _ in range(50)]
    news = [(p.targets(1, False), [r.choice([0, 3, 20]) for _ in range(50)]) for p in pools]
    n = max(p.n_pages for p in pools)
    for p in pools:
        p.refs += [0] * (n - p.n_pages)
        p.n_pages = n
    refs, table, lens = pools[0].device()
    new, add, par = dev(news[0][0]), dev(news[0][1]), dev(parent)
    h.hos_kv_fork(refs, table, lens, par, 16)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = h.hos_kv_resize(refs, table, lens, new, 16)
        b = h.hos_kv_fork(a["refs"], a["page_table"], a["kv_len"], par, 16)
        c = h.hos_kv_compact(b["refs"], b["page_table"], b["kv_len"], 16)
        d = h.hos_kv_resize(c["refs"], c["page_table"], c["kv_len"], c["kv_len"] + add, 16)
    for i in (0, 2, 1, 3, 3, 0):
        p = pools[i]
        for x, y in zip((refs, table, lens, new, add), (*p.device(), dev(news[i][0]), dev(news[i][1]))):
            x.copy_(y)
        graph.replay()
        w = P.resize(p.refs, p.rows, p.lens, news[i][0], 16, entries)
        w = P.fork(*w[:3], parent, 16, entries)
        k = P.compact(*w[:3], 16, entries)
        w = P.resize(k[0], k[1], w[2], [x + y for x, y in zip(w[2], news[i][1])], 16, entries)
        assert d["refs"].tolist() == w[0] and d["page_table"].tolist() == w[1] and d["kv_len"].tolist() == w[2]
        assert d["src"].tolist()[:len(w[3])] == w[3] and d["status"].tolist() == w[5]


def test_refusals():
    h = hos()
    pool = Pool(1, 4, 16, 100, 3)
    refs, table, lens = pool.device()
    ok = dev(pool.lens)
    for bad, kind in ((lambda: h.hos_kv_resize(refs.long(), table, lens, ok, 16), TypeError), (lambda: h.hos_kv_resize(refs.cpu(), table, lens, ok, 16), TypeError),
                      (lambda: h.hos_kv_resize(refs, table.cpu(), lens, ok, 16), TypeError), (lambda: h.hos_kv_resize(refs, table, lens, ok.float(), 16), TypeError),
                      (lambda: h.hos_kv_resize(refs, table, lens, ok[:3], 16), ValueError), (lambda: h.hos_kv_resize(refs, table[:3], lens, ok, 16), ValueError),
                      (lambda: h.hos_kv_resize(refs, table[:1].expand(4, -1), lens, ok, 16), ValueError),
                      (lambda: h.hos_kv_resize(refs, table.t().contiguous().t(), lens, ok, 16), ValueError), (lambda: h.hos_kv_resize(refs, table, lens, ok, 0), ValueError),
                      (lambda: h.hos_kv_resize(refs[::2], table, lens, ok, 16), ValueError), (lambda: h.hos_kv_resize(refs[:0], table, lens, ok, 16), h.HosError),
                      (lambda: h.hos_kv_resize(refs, table, lens, ok, 16, out=(refs, table)), TypeError),
                      (lambda: h.hos_kv_resize(refs, table, lens, ok, 16, out=(refs, table[:, :-1].contiguous(), lens)), ValueError),
                      (lambda: h.hos_kv_fork(refs, table, lens, ok, 16, out=(refs, table, lens)), h.HosError),
                      (lambda: h.hos_kv_fork(refs, table, lens, ok, 16, out=(refs, table.clone(), lens)), h.HosError),
                      (lambda: h.hos_kv_resize(refs, table, lens, ok, 1 << 30), h.HosError), (lambda: h.hos_kv_compact([1], table, lens, 16), TypeError)):
        with pytest.raises(kind):
            bad()
    assert refs.tolist() == pool.refs and table.tolist() == pool.rows
