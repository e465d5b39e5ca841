"""Where the random number falls on the end of a token's share, or behind all of them.

The token is the least v whose sum is beyond u times the whole, sums good to 2^-40 of the whole: any v of positive weight whose share, widened
by that at both ends, holds u times the whole will do.  From u = 1 on it is the last v of positive weight, without a tolerance."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def hos():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2502_15763_b200 as h
    return h


def weights(p, q):
    """Of 64-bit rows; q may be None."""
    w = torch.where((p > 0) & (p < math.inf), p, torch.zeros_like(p))
    return w if q is None else (w - torch.where(q > 0, q, torch.zeros_like(q))).clamp_min(0.0)


def fits(w, u, v):
    """Whether v is an answer for a random number below 1."""
    if not (0 <= v < len(w) and float(w[v]) > 0.0):
        return False
    before, whole = math.fsum(w[:v].tolist()), math.fsum(w.tolist())
    t, tol = max(u, 0.0) * whole, 2.0 ** -40 * whole
    return before - tol <= t < before + float(w[v]) + tol


def draw(target, u, draft=None):
    """One draw a row; with a draft, after it was not accepted (of two tokens a sequence; infinity times q is below no p)."""
    n, vocab = target.shape
    target = target.cuda()
    if draft is None:
        off, tokens, ua = torch.arange(n + 1), torch.zeros(n), torch.zeros(n)
    else:
        off, tokens, ua = 2 * torch.arange(n + 1), torch.zeros(2 * n), torch.full((2 * n,), math.inf)
        target = torch.stack([target, torch.zeros_like(target)], 1).view(2 * n, vocab)
        draft = torch.stack([draft.cuda(), torch.zeros_like(draft.cuda())], 1).view(2 * n, vocab)
    r = hos().hos_verify_drafts(tokens.int().cuda(), target, draft, off.int().cuda(), ua.cuda(), torch.tensor(u, dtype=torch.float32).cuda())
    assert r["status"].tolist() == [0] * n and r["accepted"].tolist() == [0] * n
    return r["next"].tolist()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,n", [(40000, 1), (50257, 3), (40000, 40), (70000, 300)])
@pytest.mark.parametrize("with_draft", [False, True])
def test_a_number_at_the_end_of_a_share_behind_zeros(dt, vocab, n, with_draft):
    """1 + 2^-52 + 2^-53 is rounded up, so the sum before the last of them seems to lie beyond the number: the zero before it is no token."""
    target = torch.zeros((n, vocab), dtype=DT[dt])
    for s in range(n):
        a = 0 if s % 2 == 0 else (vocab // 3) // 8 * 8 + s
        target[s, a], target[s, a + 1], target[s, a + 9], target[s, vocab - 1] = 1.0, 2.0 ** -52, 2.0 ** -53, 1.0
    draft = None
    if with_draft:
        draft = torch.full_like(target, 0.25)
        draft[target > 0] = 0.0
    got = draw(target, [0.5] * n, draft)
    for s in range(n):
        assert fits(weights(target[s].double(), None if draft is None else draft[s].double()), 0.5, got[s]), (s, got[s])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,n", [(700, 40), (2000, 60), (9000, 30), (40000, 9), (128000, 4)])
@pytest.mark.parametrize("u", [1.0, 1.5, math.inf])
@pytest.mark.parametrize("with_draft", [False, True])
def test_from_one_on_the_last_token_that_has_any(dt, vocab, n, u, with_draft):
    """However little the last one has."""
    g = torch.Generator().manual_seed(vocab)
    target = (torch.rand((n, vocab), generator=g) * (torch.rand((n, vocab), generator=g) < 0.5)).to(DT[dt])
    last = [vocab - 1 - 3 * s for s in range(n)]
    for s in range(n):
        target[s, last[s]:] = 0.0
        target[s, last[s]] = (1e-14, 1e-20, 3e-16, 1.0)[s % 4]
    draft = None
    if with_draft:
        draft = torch.full_like(target, 0.125)
        draft[target > 0] *= 0.5
        for s in range(n):
            draft[s, last[s]] = 0.0
    assert draw(target, [u] * n, draft) == last
