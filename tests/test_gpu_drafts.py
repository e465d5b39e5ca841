"""Drafted tokens against the same in plain Python and 64 bits: whole numbers, so everything has to be equal.

Sums of up to 10^5 weights in 64 bits, added in another order, differ by 10^-11 of their total at the very most; a random
number falls so near to the end of a token's share in one draw out of 10^6 of the largest here, and the inputs are fixed by their seeds."""
import math
import random

import pytest
import torch

from tests import pages_reference as P

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def hos():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2502_15763_b200 as h
    return h


def make(drafts, vocab, dt, seed, lookup=False, sharp=3.0, close=0.8):
    """Probabilities, tokens drawn from the draft's, random numbers; drafts: per sequence, -1 for one without tokens."""
    g = torch.Generator().manual_seed(seed)
    off = [0]
    for k in drafts:
        off.append(off[-1] + k + 1)
    n = off[-1]
    logits = sharp * torch.randn((n, vocab), generator=g)
    q = torch.softmax(logits + close * torch.randn((n, vocab), generator=g), -1)
    target, draft = torch.softmax(logits, -1).to(DT[dt]), q.to(DT[dt])
    tokens = torch.zeros(n + 1, dtype=torch.int32)
    if n:
        tokens[1:] = torch.multinomial(q, 1, generator=g)[:, 0].to(torch.int32)
    return target, None if lookup else draft, tokens[:n], torch.tensor(off, dtype=torch.int32), torch.rand(n, generator=g), torch.rand(len(drafts), generator=g)


def strided(t, pad, shift):
    buf = torch.full((t.shape[0] * (t.shape[1] + pad) + 64,), 0.5, dtype=t.dtype, device="cuda")
    view = buf[shift:].as_strided(t.shape, (t.shape[1] + pad, 1), shift)
    view.copy_(t)
    return view


def check(target, draft, tokens, off, ua, us, pad=(0, 0), shift=(0, 0), with_len=True):
    h = hos()
    n_seq, n = len(off) - 1, len(tokens)
    accepted, nxt, out, status = P.verify(tokens.tolist(), target.double(), None if draft is None else draft.double(), off.tolist(), ua.double().tolist(),
                                          us.double().tolist(), target.shape[1])
    kv_len = torch.arange(n_seq, dtype=torch.int32) * 7 + 40
    t = strided(target, pad[0], shift[0]) if pad[0] or shift[0] else target.cuda()
    d = None if draft is None else strided(draft, pad[1], shift[1]) if pad[1] or shift[1] else draft.cuda()
    r = h.hos_verify_drafts(tokens.cuda(), t, d, off.cuda(), ua.cuda(), us.cuda(), kv_len=kv_len.cuda() if with_len else None)
    assert r["status"].tolist() == status
    assert r["accepted"].tolist() == accepted
    assert r["next"].tolist() == nxt
    got = r["tokens"].tolist()
    assert all(w is None or w == g for w, g in zip(out, got)) and len(got) == n
    if with_len:
        k = [b - a - 1 if 0 <= a < b <= n else 0 for a, b in zip(off.tolist(), off.tolist()[1:])]
        assert r["new_len"].tolist() == [int(kv_len[s]) - k[s] + accepted[s] for s in range(n_seq)]
    else:
        assert r["new_len"] is None
    return accepted, nxt


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 511, 1000, 4099, 32000])
@pytest.mark.parametrize("lookup", [False, True])
def test_batches(dt, vocab, lookup):
    r = random.Random(vocab)
    for n_seq, most in ((1, 4), (5, 1), (40, 6), (3, 0)):
        drafts = [r.randrange(most + 1) if n_seq > 1 else most for _ in range(n_seq)]
        accepted, _ = check(*make(drafts, vocab, dt, vocab + n_seq, lookup), with_len=n_seq != 5)
        if n_seq == 40 and vocab > 30 and not lookup:
            assert any(a == k for a, k in zip(accepted, drafts) if k) and any(a < k for a, k in zip(accepted, drafts))


@pytest.mark.parametrize("vocab", [50257, 128000, 151937])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_large_vocabularies(vocab, dt):
    check(*make([2, 0, 5], vocab, dt, 3))
    check(*make([3], vocab, dt, 4, lookup=True, sharp=8.0))


@pytest.mark.parametrize("n_seq", [1, 2, 7, 30, 149, 600])
def test_many_sequences(n_seq):
    check(*make([s % 4 for s in range(n_seq)], 2000, "f32", n_seq))


@pytest.mark.parametrize("n_seq,vocab,dt", [(20, 20011, "f32"), (64, 9000, "bf16"), (140, 4100, "f32"), (310, 4500, "f16")])
def test_one_to_eight_blocks_a_sequence(n_seq, vocab, dt):
    check(*make([s % 3 for s in range(n_seq)], vocab, dt, n_seq))
    check(*make([s % 2 for s in range(n_seq)], vocab, dt, n_seq + 1, lookup=True))


@pytest.mark.parametrize("dt", ["f32", "f16"])
@pytest.mark.parametrize("pad,shift", [((1, 1), (0, 0)), ((3, 0), (1, 0)), ((0, 5), (0, 3)), ((8, 8), (4, 4)), ((7, 2), (5, 6))])
@pytest.mark.parametrize("vocab", [5, 1003, 8000])
def test_rows_of_any_alignment(dt, pad, shift, vocab):
    check(*make([3, 0, 5, 2, 1], vocab, dt, 8), pad=pad, shift=shift)


@pytest.mark.parametrize("k", [31, 32, 33, 64, 70, 200])
def test_many_drafts(k):
    """All accepted, and one not accepted anywhere among them."""
    target, draft, tokens, off, ua, us = make([k, 1, k], 64, "f32", k)
    draft.copy_(target)                                          # u q < p wherever u < 1 and p > 0
    accepted, _ = check(target, draft, tokens, off, ua, us)
    assert accepted[0] == k
    for stop in {0, 1, 30, 31, 32, k - 2, k - 1}:
        if 0 <= stop < k:
            u = ua.clone()
            u[stop] = 2.0
            accepted, _ = check(target, draft, tokens, off, u, us)
            assert accepted[0] == stop and accepted[2] == k


def test_sequences_without_tokens_or_drafts():
    check(*make([-1, 3, -1, -1, 0, 2, -1], 100, "f32", 1))
    check(*make([-1, -1], 100, "f32", 1))
    h = hos()
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    r = h.hos_verify_drafts(empty, torch.zeros((0, 9), device="cuda"), None, torch.zeros(1, dtype=torch.int32, device="cuda"), empty.float(), empty.float(), empty)
    assert r["accepted"].shape == r["next"].shape == r["tokens"].shape == r["new_len"].shape == (0,)


def test_a_rejected_draft_leaves_nothing():
    """p = q everywhere and a draft rejected by its number: the target's own row is drawn from."""
    target, draft, tokens, off, ua, us = make([2, 2, 2, 0], 777, "f32", 2)
    draft.copy_(target)
    ua[0], ua[4] = 1.5, math.inf
    accepted, _ = check(target, draft, tokens, off, ua, us)
    assert accepted[:2] == [0, 1]
    draft.mul_(1.25)                                             # q > p everywhere
    ua[:] = 0.9
    accepted, _ = check(target, draft, tokens, off, ua, us)
    assert accepted[:3] == [0, 0, 0]
    lookup = torch.zeros_like(target)                            # all of p at the draft that was looked up
    lookup[torch.arange(len(tokens)), tokens.long().roll(-1)] = 0.75
    ua[:] = 0.8
    check(lookup, None, tokens, off, ua, us)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_one_token_has_everything(dt):
    target, draft, tokens, off, ua, us = make([3, 3, 3, 0, 1], 300, dt, 5)
    best = target.float().argmax(-1)
    sure = torch.zeros_like(target)
    sure[torch.arange(len(best)), best] = 1.0
    tokens[1:] = best[:-1].to(torch.int32)
    tokens[6] = (tokens[6] + 1) % 300
    accepted, nxt = check(sure, draft, tokens, off, ua, us)
    assert accepted == [3, 1, 3, 0, 1] and nxt == [int(best[i]) for i in (3, 5, 11, 12, 14)]
    check(sure, None, tokens, off, ua, us)


@pytest.mark.parametrize("dt,vocab,share", [("f32", 90, 0.05), ("f32", 20000, 0.0002), ("bf16", 20000, 0.0002), ("f16", 4099, 0.001)])
def test_strange_entries(dt, vocab, share):
    """A few of them in large rows, anywhere."""
    for seed in range(4):
        target, draft, tokens, off, ua, us = make([4, 1, 0, 6, 2], vocab, dt, 40 + seed)
        g = torch.Generator().manual_seed(seed)
        for t, more in ((target, (math.inf, -math.inf, math.nan, -2.0, 0.0)), (draft, (math.inf, -math.inf, math.nan, -2.0, 0.0))):
            for x in more:
                t[torch.rand(t.shape, generator=g) < share] = x
        check(target, draft if seed % 2 else None, tokens, off, ua, us)


def test_strange_probabilities():
    """Zeros, negative entries, infinities and NaN count as nothing, in the target, the draft and at the draft's place."""
    for seed in range(6):
        target, draft, tokens, off, ua, us = make([4, 1, 0, 6, 2], 90, "f32", 20 + seed)
        g = torch.Generator().manual_seed(seed)
        for t in (target, draft):
            for x in (0.0, -0.5, math.inf, -math.inf, math.nan, 1e-42, 3e38):
                t[torch.rand(t.shape, generator=g) < 0.05] = x
        check(target, draft if seed % 2 else None, tokens, off, ua, us)
    target[:] = 0.0
    _, nxt = check(target, draft, tokens, off, ua, us)
    assert nxt == [-1] * 5
    target[:] = math.nan
    check(target, None, tokens, off, ua, us)
    target[4] = 0.0
    target[4, 89] = 1e-45                                        # the one entry that counts is the last, and tiny
    assert check(target, draft.fill_(0.0), tokens, off, ua.fill_(0.0), us)[1][1] == -1


def test_random_numbers_at_the_ends():
    target, draft, tokens, off, ua, us = make([2] * 7, 400, "f32", 6)
    for x in (0.0, 1.0, 1.0 - 2.0 ** -24, 2.0, -1.0, math.nan, math.inf):
        check(target, draft, tokens, off, ua, torch.full_like(us, x))
        check(target, draft, tokens, off, torch.full_like(ua, x), us)
    flat = torch.full((4, 1024), 2.0 ** -10)                     # shares end exactly at multiples of 2^-10
    off = torch.arange(5, dtype=torch.int32)
    _, nxt = check(flat, None, torch.zeros(4, dtype=torch.int32), off, torch.zeros(4), torch.tensor([0.0, 0.25, 0.5 - 2.0 ** -24, 1023 / 1024]))
    assert nxt == [0, 256, 511, 1023]


def test_small_differences_are_not_lost():
    """p - q of numbers of very different size is taken in 64 bits."""
    p, q = torch.zeros((2, 4)), torch.zeros((2, 4))
    p[0], q[0] = torch.tensor([0.5, 2.0 ** -30, 0.25, 0.0]), torch.tensor([0.5 + 2.0 ** -24, 2.0 ** -60, 0.25, 0.0])
    q[0, 3] = 0.25
    accepted, nxt = check(p, q, torch.tensor([0, 3], dtype=torch.int32), torch.tensor([0, 2], dtype=torch.int32), torch.zeros(2), torch.tensor([0.99]))
    assert (accepted, nxt) == ([0], [1])


def test_drafts_out_of_range():
    target, draft, tokens, off, ua, us = make([3, 3, 3, 3], 50, "f32", 7)
    draft.copy_(target)
    tokens[1], tokens[6], tokens[11] = 50, -1, 2 ** 31 - 1
    accepted, _ = check(target, draft, tokens, off, ua, us)
    assert accepted == [0, 1, 2, 3]
    check(target, None, tokens, off, ua, us)


def test_offsets_out_of_range():
    target, draft, tokens, off, ua, us = make([2, 2, 2, 2, 2], 60, "f32", 9)
    for bad in ([0, 3, 6, 9, 12, 16], [0, 3, 2, 9, 12, 15], [-1, 3, 6, 9, 12, 15], [0, 3, 6, 2 ** 31 - 1, 12, 15], [2, 3, 6, 9, 12, 13]):
        check(target, draft, tokens, torch.tensor(bad, dtype=torch.int32), ua, us)


def test_rows_beyond_32_bits():
    h = hos()
    vocab, n = 1 << 20, 2200                                     # 4.6 GB of 16-bit rows, the last ones beyond 2^31 elements
    target = torch.zeros((n, vocab), dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, 2, n - 3, n], dtype=torch.int32, device="cuda")
    tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
    target[n - 3, 77] = target[n - 2, vocab - 1] = 0.75
    target[n - 1, vocab - 2] = 1.0
    tokens[n - 2], tokens[n - 1] = 77, vocab - 1
    target[0, 5], target[1, 6], target[2, 9] = 0.5, 1.0, 1.0
    r = h.hos_verify_drafts(tokens, target, None, off, torch.full((n,), 0.5, device="cuda"), torch.zeros(3, device="cuda"))
    assert r["accepted"].tolist() == [0, 0, 2] and r["next"].tolist() == [5, 9, vocab - 2]


def test_captured_and_on_other_streams():
    h = hos()
    sets = [make([3, 1, 4, 0], 3001, "f32", 30 + i) for i in range(4)]
    want = [P.verify(t.tolist(), p.double(), q.double(), o.tolist(), a.double().tolist(), s.double().tolist(), 3001) for p, q, t, o, a, s in sets]
    given = [[x.cuda() for x in s] for s in sets]

    def call(p, q, t, o, a, s):
        return h.hos_verify_drafts(t, p, q, o, a, s)
    live = [x.clone() for x in given[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = call(*live)
    for i in (0, 2, 1, 3, 0):
        for x, y in zip(live, given[i]):
            x.copy_(y)
        graph.replay()
        assert (r["accepted"].tolist(), r["next"].tolist(), r["tokens"].tolist()) == want[i][:3]
    streams, got = [torch.cuda.Stream() for _ in sets], []
    torch.cuda.synchronize()
    for _ in range(10):
        for st, s in zip(streams, given):
            with torch.cuda.stream(st):
                got.append(call(*s))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        assert (r["accepted"].tolist(), r["next"].tolist()) == want[i % 4][:2]


def test_refusals():
    h = hos()
    p, q, t, o, a, s = (x.cuda() for x in make([2, 2], 30, "f32", 1))
    for args, kind in (((t, p.double(), q, o, a, s), TypeError), ((t, p.cpu(), q, o, a, s), TypeError), ((t, p, q.half(), o, a, s), TypeError),
                       ((t.long(), p, q, o, a, s), TypeError), ((t, p, q, o.long(), a, s), TypeError), ((t, p, q, o, a.double(), s), TypeError),
                       ((t[:-1], p, q, o, a, s), ValueError), ((t, p, q[:, :-1], o, a, s), ValueError), ((t, p, q, o, a[:-1], s), ValueError),
                       ((t, p, q, o, a, s[:1]), ValueError), ((t, p[0], q, o, a, s), ValueError), ((t, p.t().contiguous().t(), q, o, a, s), ValueError),
                       ((t, p[:, :0], None, o, a, s), ValueError), ((t, p, q, o[:0], a, s), ValueError), ((t, None, q, o, a, s), TypeError),
                       ((t, p, q, o, a, s, o), ValueError), ((t.cpu(), p, q, o, a, s), TypeError)):
        with pytest.raises(kind):
            h.hos_verify_drafts(*args)
    g = p.clone().requires_grad_()
    with pytest.raises(ValueError, match="target requires grad"):
        h.hos_verify_drafts(t, g, q, o, a, s)
    with pytest.raises(ValueError, match="draft requires grad"):
        h.hos_verify_drafts(t, p, g, o, a, s)
    want = h.hos_verify_drafts(t, p, q, o, a, s)
    with torch.no_grad():
        r = h.hos_verify_drafts(t, g, q, o, a, s)
    assert torch.equal(r["tokens"], want["tokens"])
