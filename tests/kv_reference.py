"""Plain 64-bit statement of the paged-cache operators, sequence by sequence, for the GPU tests.

Written from the formulas in include/hos.h; nothing of the package is used here."""
import math

import torch

TOP = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}


def make_batch(pairs, page, n_spare, seed, device="cuda", fill=-1):
    """tok_off, kv_len, page_table (pages in random order, unused entries `fill`) and the number of pages."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-t // page) for _, t in pairs]
    n_pages = max(1, sum(need) + n_spare)
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(pairs), max(1, max(need)) + 1), fill, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    off = torch.tensor([0] + [n for n, _ in pairs]).cumsum(0).to(torch.int32)
    kv_len = torch.tensor([t for _, t in pairs], dtype=torch.int32)
    return off.to(device), kv_len.to(device), table.to(device), n_pages


def quantise(x, code):
    """Codes and scales along the last axis, each step rounded to 32 bits."""
    x = x.float()
    a = x.abs().amax(-1).clamp_min(1e-30)
    top = torch.tensor(TOP[code], dtype=torch.float32, device=x.device)
    y = x * (a.reciprocal() * top)[..., None]
    return (y.round().to(code) if code == torch.int8 else y.to(code)), a * top.reciprocal()


def values(codes, scale):
    """[...] codes -> 64-bit values."""
    x = codes.to(torch.float32).to(torch.float64)
    return x if scale is None else x * scale.to(torch.float64)[..., None]


def sequence(cache, scale, table_row, length, page):
    """[length][n_kv][head_dim] of one sequence in 64 bits."""
    if length == 0:
        return torch.zeros((0, cache.shape[1], cache.shape[3]), dtype=torch.float64, device=cache.device)
    pages = table_row[:-(-length // page)].long()
    raw = cache.view(torch.uint8)[pages].view(cache.dtype) if cache.element_size() == 1 else cache[pages]
    x = values(raw, None if scale is None else scale[pages])
    return x.permute(0, 2, 1, 3).reshape(-1, cache.shape[1], cache.shape[3])[:length]


def attention(q, k, v, k_scale, v_scale, pairs, off, table, page, sm_scale, causal, window):
    """out, lse and the two quantities the error bounds need: sum_j w_j |v_j| and the largest
    sum_d |q_d k_jd| * sm_scale of each row."""
    n_tok, hq, d = q.shape
    hk = k.shape[1]
    dev = q.device
    out = torch.zeros((n_tok, hq, d), dtype=torch.float64, device=dev)
    mag = torch.zeros_like(out)
    lse = torch.full((n_tok, hq), -math.inf, dtype=torch.float64, device=dev)
    dot = torch.zeros((n_tok, hq), dtype=torch.float64, device=dev)
    for s, (n, t) in enumerate(pairs):
        if n == 0 or t == 0:
            continue
        ks, vs = sequence(k, k_scale, table[s], t, page), sequence(v, v_scale, table[s], t, page)
        a = int(off[s])
        pos = torch.arange(t - n, t, device=dev)[:, None]
        j = torch.arange(t, device=dev)[None, :]
        see = torch.ones((n, t), dtype=torch.bool, device=dev)
        if causal:
            see &= j <= pos
        if window:
            see &= j > pos - window
        for h in range(hq):
            qq, kk, vv = q[a:a + n, h].to(torch.float64), ks[:, h // (hq // hk)], vs[:, h // (hq // hk)]
            x = (qq @ kk.T * sm_scale).masked_fill(~see, -math.inf)
            e = torch.logsumexp(x, -1)
            w = torch.where(see.any(-1, keepdim=True), torch.exp(x - torch.where(e == -math.inf, 0.0, e)[:, None]), 0.0)
            out[a:a + n, h], mag[a:a + n, h], lse[a:a + n, h] = w @ vv, w @ vv.abs(), e
            dot[a:a + n, h] = ((qq.abs() @ kk.abs().T) * abs(sm_scale)).masked_fill(~see, 0.0).amax(-1)
    return out, lse, mag, dot
