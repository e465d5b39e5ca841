"""What is measured of the KV-cache operators: append, read back, and attention over the paged cache.

Every case describes one batch of sequences of one inference client: how many, how long, the head layout, the page
size and how the cache holds its values.  The plain forms are elementary torch operations in 32 bits; with `own`
set, `run` makes the calls of this package instead.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CODES = {"e4m3": (torch.float8_e4m3fn, 448.0), "int8": (torch.int8, 127.0)}
LEAST = 1e-30                    # smallest magnitude a quantised vector is scaled to

BASE = {"fmt": "same", "dtype": "bf16", "dim": 128, "page": 128, "window": 0, "causal": True, "decodes": 0,
        "ctx_mid": 0, "ctx_sigma": 0.0, "ctx_max": 4096, "new_mid": 1, "new_sigma": 0.0, "new_max": 4096, "mix": 0}


def _case(name, op, **more):
    return {**BASE, "name": name, "op": op, **more}


def listed():
    return [
        # one decode round of a 16-slot client, 64 heads spread over 8 devices: the latency of a write
        _case("append_round_16", "append", fmt="int8", n_seq=16, heads=8, kv_heads=8, ctx_mid=250, ctx_sigma=0.4, mix=1),
        # a prefill stage of long prompts on an undivided 64-head model: the rate of a write
        _case("append_prompts_8k", "append", fmt="e4m3", n_seq=22, heads=64, kv_heads=64, page=16, new_mid=300,
              new_sigma=0.6, new_max=4096, mix=2),
        # one short request handed on to another client
        _case("read_one_request", "read", fmt="e4m3", dtype="f16", n_seq=1, heads=8, kv_heads=8, dim=64, page=32,
              new_mid=333, mix=3),
        # everything a 16-slot client of 32,768 KV tokens holds
        _case("read_client_32k", "read", fmt="int8", n_seq=16, heads=64, kv_heads=64, new_mid=2000, new_sigma=0.2, mix=4),
        # a lone request in its decode phase: latency
        _case("decode_one", "attend", n_seq=1, heads=8, kv_heads=8, page=16, ctx_mid=250, mix=5),
        # a decode round of a full 16-slot client, 64 heads of their own KV
        _case("decode_16", "attend", n_seq=16, heads=64, kv_heads=64, ctx_mid=1900, ctx_sigma=0.4, mix=6),
        # a decode round of a 128-slot client near its 262,144 KV tokens, grouped heads, 8-bit cache
        _case("decode_128_int8", "attend", fmt="int8", n_seq=128, heads=64, kv_heads=8, page=16, ctx_mid=1700,
              ctx_sigma=0.6, ctx_max=6000, mix=7),
        # two requests with very long contexts: few rows, the split over the keys counts
        _case("decode_2_long", "attend", fmt="e4m3", dtype="f16", n_seq=2, heads=32, kv_heads=8, dim=64, page=64,
              ctx_mid=131000, ctx_sigma=0.1, ctx_max=150000, mix=8),
        # the longest prompt of the scale-out workload, prefilled whole, 64 heads of their own KV
        _case("prefill_4096", "attend", n_seq=1, heads=64, kv_heads=64, new_mid=4096, mix=9),
        # a prefill stage of short prompts with grouped heads
        _case("prefill_short_32", "attend", dtype="f16", n_seq=32, heads=64, kv_heads=8, page=16, new_mid=120,
              new_sigma=0.4, new_max=512, mix=10),
        # a chunk of an odd number of new tokens behind a long context, 8-bit cache
        _case("chunk_509_of_16k", "attend", fmt="e4m3", n_seq=1, heads=64, kv_heads=8, page=64, ctx_mid=15991,
              ctx_max=16384, new_mid=509, mix=11),
        # chunks and decodes in one call, sliding window, small heads
        _case("mixed_window", "attend", dtype="f16", n_seq=14, decodes=12, heads=32, kv_heads=8, dim=64, page=32,
              window=1000, ctx_mid=1500, ctx_sigma=0.5, new_mid=500, new_sigma=0.3, new_max=1024, mix=12),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "attend"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    group = rng.choice([1, 1, 4, 5, 8]) if op == "attend" else 1
    c = {**BASE, "op": op, "fmt": rng.choice(["same", "e4m3", "int8"]), "dtype": rng.choice(["bf16", "f16"]),
         "dim": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 64, 128, 256]), "kv_heads": kv_heads,
         "heads": kv_heads * group, "mix": rng.randrange(1 << 30)}
    if op != "attend":
        c["n_seq"] = _spread(rng, 1, 64)
        c["ctx_mid"] = _spread(rng, 1, 2000) if op == "append" else 0
        c["ctx_sigma"], c["new_sigma"] = 0.5, rng.choice([0.0, 0.5])
        c["new_mid"] = rng.choice([1, _spread(rng, 2, max(3, 260000 // (c["n_seq"] * kv_heads)))])
        return c
    c["window"] = rng.choice([0, 0, 0, _spread(rng, 64, 4000)])
    c["causal"] = rng.random() < 0.9
    if rng.random() < 0.5:                                   # decode rounds
        c["n_seq"] = _spread(rng, 1, 128)
        most = min(100000, 300000 // c["n_seq"], 1500000 // (c["n_seq"] * kv_heads))
        c["ctx_mid"], c["ctx_max"] = _spread(rng, 8, max(9, most // 3)), max(9, most)
        c["ctx_sigma"], c["new_mid"] = 0.6, rng.choice([1, 1, 1, 3])
    else:                                                    # chunks, alone or among decodes
        c["n_seq"] = _spread(rng, 1, 24)
        most = int((1.2e9 / (c["n_seq"] * c["heads"])) ** 0.5)
        c["new_mid"] = _spread(rng, 2, max(3, min(2048, most // 3)))
        c["new_max"] = min(4096, 2 * c["new_mid"])
        c["ctx_mid"] = rng.choice([0, _spread(rng, 1, max(2, most // 2))])
        c["ctx_max"], c["ctx_sigma"], c["new_sigma"] = max(1, most), 0.5, 0.4
        c["decodes"] = rng.choice([0, 0, c["n_seq"] // 2])
    return c


def lengths(case):
    """[(new tokens, tokens in the cache after them)] of the batch: log-normals like the scheduler's workloads."""
    r = random.Random(case["mix"])

    def one(mid, sigma, most):
        return min(most, int(round(mid * math.exp(sigma * r.gauss(0.0, 1.0)))))

    pairs = [(one(case["ctx_mid"], case["ctx_sigma"], case["ctx_max"]),
              1 if s < case["decodes"] else max(1, one(case["new_mid"], case["new_sigma"], case["new_max"])))
             for s in range(case["n_seq"])]
    return [(new, ctx + new) for ctx, new in pairs]


def _quantise(x, fmt):
    """Codes and scales of vectors along the last axis, in 32 bits."""
    code, top = CODES[fmt]
    x = x.float()
    a = x.abs().amax(-1).clamp_min(LEAST)
    y = x * (top / a)[..., None]
    return (y.round().to(code) if fmt == "int8" else y.to(code)), a / top


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt, hk, d, ps = DTYPES[case["dtype"]], case["kv_heads"], case["dim"], case["page"]
    pairs = lengths(case)
    new, total = [n for n, _ in pairs], [t for _, t in pairs]
    per_seq = [-(-t // ps) for t in total]
    n_pages, widest, n_tok = sum(per_seq) + 3, max(1, max(per_seq)), sum(new)
    # pages were handed out in no particular order
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    used = torch.arange(widest, device=dev)[None, :] < torch.tensor(per_seq, device=dev)[:, None]
    table = torch.zeros((len(pairs), widest), dtype=torch.int32, device=dev)
    table[used] = order[:int(used.sum())]
    off = torch.tensor([0] + new, device=dev).cumsum(0).to(torch.int32)
    gain = torch.exp(0.3 * torch.randn((hk, 1, d), generator=gen, device=dev)).to(dt)     # channels differ in size

    def pool():
        return torch.randn((n_pages, hk, ps, d), generator=gen, device=dev, dtype=dt).mul_(gain)

    def fresh(h):
        return torch.randn((n_tok, h, d), generator=gen, device=dev, dtype=dt)

    s = {"case": case, "off": off, "kv_len": torch.tensor(total, dtype=torch.int32, device=dev), "table": table,
         "n_tok": n_tok, "max_new": max(new), "max_kv": max(total), "k_scale": None, "v_scale": None}
    if case["fmt"] == "same":
        s["k"], s["v"] = pool(), pool()
    else:
        (s["k"], s["k_scale"]), (s["v"], s["v_scale"]) = _quantise(pool(), case["fmt"]), _quantise(pool(), case["fmt"])
    if case["op"] == "append":
        # the new keys and values are slices of one projection's output, as a model hands them over
        qkv = torch.randn((n_tok, case["heads"] + 2 * hk, d), generator=gen, device=dev, dtype=dt)
        s["new_k"], s["new_v"] = qkv[:, case["heads"]:case["heads"] + hk], qkv[:, case["heads"] + hk:]
    if case["op"] == "attend":
        s["q"] = fresh(case["heads"]).mul_(2.0)
    if own:
        import paper_2502_15763_b200 as hos
        s["hos"] = hos
        s["cache"] = hos.hos_kv_cache(s["k"], s["v"], s["k_scale"], s["v_scale"], dtype=dt)
    return s


def run(s):
    case = s["case"]
    if own:
        hos = s["hos"]
        if case["op"] == "append":
            hos.hos_kv_append(s["cache"], s["new_k"], s["new_v"], s["off"], s["kv_len"], s["table"])
            return {n: s[n] for n in ("k", "v", "k_scale", "v_scale") if s[n] is not None}
        if case["op"] == "read":
            r = hos.hos_kv_read(s["cache"], s["off"], s["kv_len"], s["table"], s["n_tok"])
            return {"k": r["k"], "v": r["v"]}
        r = hos.hos_paged_attention(s["q"], s["cache"], s["off"], s["kv_len"], s["table"], s["max_new"],
                                    causal=case["causal"], window=case["window"], want_lse=True)
        return {"out": r["out"], "lse": r["lse"]}
    if case["op"] == "append":
        return _append(s)
    return _read(s) if case["op"] == "read" else _attend(s)


def _places(s):
    """Sequence, page and row in the page of every new token."""
    tok = torch.arange(s["n_tok"], device=s["off"].device, dtype=torch.int32)
    seq = torch.bucketize(tok, s["off"][1:], right=True)
    pos = s["kv_len"][seq] - (s["off"][seq + 1] - tok)
    ps = s["case"]["page"]
    return seq, pos, s["table"][seq, pos // ps].long(), (pos % ps).long()


def _append(s):
    _, _, page, row = _places(s)
    out = {}
    if s["k_scale"] is None:
        s["k"][page, :, row] = s["new_k"]
        s["v"][page, :, row] = s["new_v"]
        return {"k": s["k"], "v": s["v"]}
    kc, ks = _quantise(s["new_k"], s["case"]["fmt"])
    vc, vs = _quantise(s["new_v"], s["case"]["fmt"])
    s["k"].view(torch.uint8)[page, :, row] = kc.view(torch.uint8)
    s["v"].view(torch.uint8)[page, :, row] = vc.view(torch.uint8)
    s["k_scale"][page, :, row] = ks
    s["v_scale"][page, :, row] = vs
    out.update(k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return out


def _read(s):
    _, _, page, row = _places(s)
    dt = DTYPES[s["case"]["dtype"]]
    if s["k_scale"] is None:
        return {"k": s["k"][page, :, row], "v": s["v"][page, :, row]}
    k = s["k"].view(torch.uint8)[page, :, row].view(s["k"].dtype).float() * s["k_scale"][page, :, row][..., None]
    v = s["v"].view(torch.uint8)[page, :, row].view(s["v"].dtype).float() * s["v_scale"][page, :, row][..., None]
    return {"k": k.to(dt), "v": v.to(dt)}


def _padded(s, codes, scale):
    """[n_seq][kv_heads][longest][dim] in 32 bits; rows past a sequence's end are zero."""
    c = s["case"]
    t = s["table"].long()
    x = codes.view(torch.uint8)[t].view(codes.dtype).float() if scale is not None else codes[t].float()
    if scale is not None:
        x = x * scale[t][..., None]
    x = x.transpose(1, 2).reshape(t.shape[0], c["kv_heads"], -1, c["dim"])[:, :, :s["max_kv"]]
    there = torch.arange(x.shape[2], device=x.device)[None, :] < s["kv_len"][:, None]
    return x.masked_fill(~there[:, None, :, None], 0.0)


def _attend(s):
    c = s["case"]
    b, hk, g, d, nq = len(s["kv_len"]), c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"], s["max_new"]
    off, n_new = s["off"][:-1], s["off"][1:] - s["off"][:-1]
    k, v = _padded(s, s["k"], s["k_scale"]), _padded(s, s["v"], s["v_scale"])
    at = torch.arange(nq, device=k.device, dtype=torch.int32)
    q = s["q"].float()[(off[:, None] + at).clamp_max(s["n_tok"] - 1)]                       # [b][nq][heads][d]
    q = q.view(b, nq, hk, g, d).permute(0, 2, 3, 1, 4).reshape(b, hk, g * nq, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(b, hk, g, nq, -1)
    j = torch.arange(k.shape[2], device=k.device, dtype=torch.int32)
    pos = (s["kv_len"] - n_new)[:, None] + at                                               # [b][nq]
    see = j < s["kv_len"][:, None, None]
    if c["causal"]:
        see = see & (j <= pos[..., None])
    if c["window"]:
        see = see & (j > pos[..., None] - c["window"])
    x.masked_fill_(~see[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = x.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hk, g * nq, -1), v).view(b, hk, g, nq, d) / torch.where(l == 0, 1.0, l)
    lse = (m + l.log()).squeeze(-1)
    tok = torch.arange(s["n_tok"], device=k.device, dtype=torch.int32)
    seq = torch.bucketize(tok, s["off"][1:], right=True)
    i = (tok - off[seq]).long()
    out = o.permute(0, 3, 1, 2, 4)[seq, i].reshape(s["n_tok"], c["heads"], d)
    return {"out": out.to(DTYPES[c["dtype"]]), "lse": lse.permute(0, 3, 1, 2)[seq, i].reshape(s["n_tok"], c["heads"])}


def work(case):
    pairs = lengths(case)
    hk, hq, d = case["kv_heads"], case["heads"], case["dim"]
    vec = 2 * d if case["fmt"] == "same" else d + 4                      # bytes of one cached vector
    n_tok = sum(n for n, _ in pairs)
    if case["op"] != "attend":
        return {"bytes": 2 * n_tok * hk * (2 * d + vec), "flops": 0}
    w = case["window"] or 1 << 30
    if case["causal"]:
        seen = sum(sum(min(w, p + 1) for p in range(t - n, t)) for n, t in pairs)
    else:
        seen = sum(sum(min(t, t - 1 - p + w) for p in range(t - n, t)) for n, t in pairs)
    keys = sum(t - max(0, t - n - w + 1) for n, t in pairs)
    return {"bytes": 2 * keys * hk * vec + n_tok * hq * (4 * d + 4), "flops": 4 * d * hq * seen}


def _round_e4m3(y):
    """Nearest e4m3 value (ties to even) of a 64-bit number of magnitude up to 448: 4 significant bits, none below 2^-9."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    pairs, ps, d = lengths(case), case["page"], case["dim"]
    f64 = torch.float64
    starts = [int(v) for v in s["off"].tolist()]

    def cached(name, q, t):
        """[kv_heads][t][dim] of sequence q in 64 bits."""
        pages = s["table"][q, :-(-t // ps)].long()
        x = s[name].view(torch.uint8)[pages].view(s[name].dtype) if case["fmt"] != "same" else s[name][pages]
        x = x.to(torch.float32).to(f64)
        if case["fmt"] != "same":
            x = x * s[name + "_scale"][pages].to(f64)[..., None]
        return x.permute(1, 0, 2, 3).reshape(case["kv_heads"], -1, d)[:, :t]

    if case["op"] == "append":
        out = {}
        for name in ("k", "v"):
            cache = s[name]
            if case["fmt"] == "same":
                want, scale = cache.to(f64), None
            else:
                want, scale = (cache.to(torch.float32).to(f64) if case["fmt"] == "e4m3" else None), s[name + "_scale"].to(f64)
            for q, (n, t) in enumerate(pairs):
                x = s["new_" + name][starts[q]:starts[q] + n].to(f64)                        # [n][kv_heads][d]
                pos = torch.arange(t - n, t, device=x.device)
                page, row = s["table"][q][pos // ps].long(), pos % ps
                if scale is None:
                    want[page, :, row] = x
                    continue
                top = CODES[case["fmt"]][1]
                sc = x.abs().amax(-1).clamp_min(LEAST) / top
                scale[page, :, row] = sc
                if want is not None:
                    want[page, :, row] = _round_e4m3(x / sc[..., None])
            out[name] = want
            if scale is not None:
                out[name + "_scale"] = scale
        return out
    if case["op"] == "read":
        both = {}
        for name in ("k", "v"):
            both[name] = torch.cat([cached(name, q, t)[:, t - n:].transpose(0, 1) for q, (n, t) in enumerate(pairs)])
        return both
    g = case["heads"] // case["kv_heads"]
    outs, lses = [], []
    for q, (n, t) in enumerate(pairs):
        k, v = cached("k", q, t), cached("v", q, t)
        j = torch.arange(t, device=k.device)
        o = torch.empty((n, case["heads"], d), dtype=f64, device=k.device)
        e = torch.empty((n, case["heads"]), dtype=f64, device=k.device)
        for h in range(case["heads"]):
            for a in range(0, n, 4096):
                rows = s["q"][starts[q] + a:starts[q] + min(n, a + 4096), h].to(f64)
                z = rows @ k[h // g].T / math.sqrt(d)
                pos = torch.arange(t - n + a, t - n + a + len(rows), device=k.device)[:, None]
                hide = (j > pos) if case["causal"] else torch.zeros_like(z, dtype=torch.bool)
                if case["window"]:
                    hide = hide | (j <= pos - case["window"])
                z = z.masked_fill(hide, -math.inf)
                le = torch.logsumexp(z, -1)
                o[a:a + len(rows), h] = torch.exp(z - le[:, None]) @ v[h // g]
                e[a:a + len(rows), h] = le
        outs.append(o)
        lses.append(e)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
