"""Sums of many weights and differences of numbers of very different size, at borders that a 32-bit sum or difference would miss.

The sums are good to 2^-40 of the whole.  The borders here are 2^-38 to 2^-32 of the whole away from the number, so the token is determined; 32-bit
sums of n terms are off by up to n 2^-24, and a difference rounded to 32 bits by 2^-25 of itself."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def hos():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2502_15763_b200 as h
    return h


def draw(target, u, draft=None, lookup=None, pad=(0, 0)):
    """One draw a row of target [n][vocab].  With a draft's rows, or looked-up tokens `lookup` [n], after that draft was not accepted."""
    n, vocab = target.shape
    per = 1 if draft is None and lookup is None else 2
    rows = torch.zeros((2, n * per, vocab + max(pad)), dtype=target.dtype, device="cuda")
    t, q = (rows[i].view(-1)[:n * per * (vocab + pad[i])].view(n * per, vocab + pad[i])[:, :vocab] for i in range(2))
    t[::per] = target.cuda()
    if draft is not None:
        q[::per] = draft.cuda()
    tokens = torch.zeros(n * per, dtype=torch.int32)
    if lookup is not None:
        tokens[1::2] = torch.as_tensor(lookup, dtype=torch.int32)
    off = per * torch.arange(n + 1, dtype=torch.int32)
    r = hos().hos_verify_drafts(tokens.cuda(), t, None if draft is None else q, off.cuda(), torch.full((n * per,), float("inf"), device="cuda"),
                                torch.as_tensor(u, dtype=torch.float32).cuda())
    assert r["status"].tolist() == [0] * n and r["accepted"].tolist() == [0] * n
    return r["next"].tolist()


SHAPES = [(5, 1), (500, 3), (4100, 200), (20000, 1), (20000, 40), (64000, 1), (64000, 5), (40000, 300)]        # tokens a half, sequences


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("half,n", SHAPES)
def test_differences_that_32_bits_cannot_hold(dt, half, n):
    """The second half's weights are each 2^-30 smaller than the first's, so half of the sum lies before the end of the first half; rounded to
    32 bits all are equal, and the sum up to there is not beyond it.  Distance: 2^-32 of the whole."""
    one = 1024.0
    p = torch.full((n, 2 * half), one, dtype=DT[dt])
    q = torch.zeros_like(p)
    q[:, half:] = one * 2.0 ** -30
    assert float(p[0, -1]) - float(q[0, -1]) < one and float(torch.tensor(one) - q[0, -1].float()) == one
    assert draw(p, [0.5] * n, q) == [half - 1] * n
    assert draw(p, [0.5] * n, q, pad=(1, 0)) == [half - 1] * n                   # rows that are not aligned alike


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("half,n", SHAPES)
@pytest.mark.parametrize("kind", ["all accepted", "drawn", "looked up"])
def test_two_halves_and_a_little_more(dt, half, n, kind):
    """The same weights twice, in another order, and something tiny before them or behind them: half of the sum is just before the end of the
    first ones, or just behind it."""
    g = torch.Generator().manual_seed(half + n)
    w = (2048.0 * torch.rand((n, half), generator=g) + 1.0).to(DT[dt])       # the tiny ones are no zeros in 16 bits then
    less = (torch.rand((n, half), generator=g)).to(DT[dt]) if kind == "drawn" else None
    order = torch.stack([torch.randperm(half, generator=g) for _ in range(n)])
    p = torch.zeros((n, 2 * half + 3), dtype=DT[dt])
    q = torch.zeros_like(p) if kind == "drawn" else None
    for row, x in ((p, w), (q, less)):
        if x is not None:
            row[:, 1:half + 1], row[:, half + 1:2 * half + 1] = x, x.gather(1, order)
    whole = 2.0 * (w.double() - (less.double() if less is not None else 0.0)).sum(1)
    late = torch.arange(n) % 2 == 1
    tiny = (whole * 2.0 ** -35).to(DT[dt])
    assert bool(((tiny.double() / whole > 2.0 ** -37) & (tiny.double() / whole < 2.0 ** -33)).all())
    p[~late, 0], p[late, 2 * half + 2] = tiny[~late], tiny[late]
    lookup = None
    if kind == "looked up":                                     # all of the rest of p lies at the token that is not drawn
        p[:, 2 * half + 1] = 50.0
        lookup = [2 * half + 1] * n
    want = [half + 1 if x else half for x in late.tolist()]
    assert draw(p, [0.5] * n, q, lookup) == want
    if kind == "drawn":
        assert draw(p, [0.5] * n, q, pad=(0, 3)) == want


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,n", [(70000, 300), (30000, 600), (1 << 20, 1), (1 << 20, 6), (200001, 40)])
@pytest.mark.parametrize("kind", ["all accepted", "drawn", "looked up"])
def test_segments_that_are_searched_in_several_steps(dt, vocab, n, kind):
    """Dense rows, numbers all over (0, 1)."""
    g = torch.Generator(device="cuda").manual_seed(vocab + n)
    p, q = ((torch.rand((n, vocab), generator=g, device="cuda") + 0.1).to(DT[dt]) for _ in range(2))
    u = ((torch.arange(n, device="cuda") + torch.rand(n, generator=g, device="cuda")) / n).clamp(1e-6, 1.0 - 2.0 ** -20)
    lookup = torch.randint(0, vocab, (n,), generator=g, device="cuda").tolist()
    w = p.double()
    if kind == "drawn":
        w = (w - q.double()).clamp_min(0.0)
    elif kind == "looked up":
        w[torch.arange(n, device="cuda"), torch.tensor(lookup, device="cuda")] = 0.0
    c = w.cumsum(1)
    t = u.double() * c[:, -1]
    want = torch.searchsorted(c, t[:, None], right=True)[:, 0]
    near = ((c - t[:, None]).abs().amin(1) < 1e-9 * c[:, -1]).tolist()
    assert sum(near) <= 2                                       # a border every 10^-6 of the whole at the least
    args = [q if kind == "drawn" else None, lookup if kind == "looked up" else None]
    for got in [draw(p, u, *args)] + ([draw(p, u, *args, pad=(1, 2))] if n < 50 and kind == "drawn" else []):
        assert all(a == b or skip for a, b, skip in zip(got, want.tolist(), near))
