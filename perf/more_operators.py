"""What is measured of the operators on a cache's pages and on drafted tokens.

`resize` takes, shares out and frees pages as sequences change length, `fork` gives sequences to several successors,
`compact` moves the pages in use together, `copy` moves the pages' contents, `verify` holds drafted tokens against
the target's probabilities.  The plain forms are elementary torch operations; with `own` set, `run` makes the calls of
this package instead.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

PAGES = {"page": 128, "n_seq": 16, "spare": 0.3, "len_mid": 500, "len_sigma": 0.5, "len_max": 4096, "shared": 0.0, "mix": 0}
RESIZE = {**PAGES, "op": "resize", "grow": 1, "cut": 0.0, "drop": 0.0, "admit": 0.0}
FORK = {**PAGES, "op": "fork", "out_seq": 16, "kind": "samples"}
COMPACT = {**PAGES, "op": "compact"}
COPY = {"op": "copy", "fmt": "same", "dtype": "bf16", "dim": 128, "page": 128, "kv_heads": 8, "layers": 1, "moves": 1, "pages": 8,
        "order": "any", "mix": 0}
VERIFY = {"op": "verify", "dtype": "f32", "vocab": 32000, "n_seq": 1, "drafts": 4, "ragged": False, "draft_probs": True, "mix": 0}


def listed():
    return [
        # a decode round of a 16-slot client, one more token each: latency
        {**RESIZE, "name": "resize_round_16", "mix": 1},
        # a drafted round of a 128-slot client with pages of 16: some cut back, some retired, some admitted, some sharing a prompt
        {**RESIZE, "name": "resize_drafts_128", "page": 16, "n_seq": 128, "len_mid": 1500, "len_max": 8192, "shared": 0.3, "grow": 5, "cut": 0.3,
         "drop": 0.05, "admit": 0.05, "mix": 2},
        # four prompts answered four times each
        {**FORK, "name": "fork_samples_16", "n_seq": 4, "len_mid": 700, "mix": 3},
        # beams of 128 long sequences are reordered, some of them twice and some not at all
        {**FORK, "name": "fork_beams_128", "page": 16, "n_seq": 128, "out_seq": 128, "len_mid": 6000, "len_max": 16384, "shared": 0.3,
         "kind": "beams", "mix": 4},
        # the pool of a 16-slot client after an afternoon
        {**COMPACT, "name": "compact_256", "spare": 1.0, "mix": 5},
        # a pool of about 100,000 pages of 16 tokens, half of them free
        {**COMPACT, "name": "compact_100k", "page": 16, "n_seq": 256, "len_mid": 2500, "len_max": 16384, "shared": 0.2, "spare": 1.0, "mix": 6},
        # the last page of three sequences that were forked from one, in one layer's cache: latency
        {**COPY, "name": "copy_forked_3", "fmt": "int8", "page": 16, "moves": 3, "pages": 64, "mix": 7},
        # the pages that a compaction moves, of four layers with e4m3 caches
        {**COPY, "name": "copy_compacted_e4m3", "fmt": "e4m3", "dtype": "f16", "page": 16, "layers": 4, "moves": 2501, "pages": 6000,
         "order": "compact", "mix": 8},
        # the last pages of 16 forked sequences, of all 80 layers
        {**COPY, "name": "copy_forked_80_layers", "layers": 80, "moves": 16, "pages": 48, "mix": 9},
        # a lone request with four drafts: latency
        {**VERIFY, "name": "verify_one", "mix": 10},
        # a full 128-slot client, 128,000 tokens to choose from
        {**VERIFY, "name": "verify_128", "vocab": 128000, "n_seq": 128, "mix": 11},
        # drafts that were looked up instead of drawn, none to seven a request, odd vocabulary, 16 bits
        {**VERIFY, "name": "verify_lookup_33", "dtype": "bf16", "vocab": 50257, "n_seq": 33, "drafts": 7, "ragged": True, "draft_probs": False,
         "mix": 12},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["resize", "fork", "compact", "copy", "copy", "verify", "verify", "verify"])
    mix = rng.randrange(1 << 30)
    if op == "copy":
        c = {**COPY, "fmt": rng.choice(["same", "e4m3", "int8"]), "dtype": rng.choice(["bf16", "f16"]), "dim": rng.choice([64, 128, 128]),
             "page": rng.choice([16, 32, 64, 128, 256]), "kv_heads": rng.choice([1, 2, 3, 8, 8, 16]), "layers": _spread(rng, 1, 90),
             "order": rng.choice(["any", "any", "compact"]), "mix": mix}
        one = 2 * c["page"] * c["kv_heads"] * c["dim"] * (2 if c["fmt"] == "same" else 1)
        c["moves"] = _spread(rng, 1, max(2, min(4000, 600_000_000 // (one * c["layers"]))))
        c["pages"] = 2 * c["moves"] + rng.randrange(1, 50)
        return c
    if op == "verify":
        c = {**VERIFY, "dtype": rng.choice(["f32", "f32", "bf16", "f16"]), "vocab": _spread(rng, 100, 160000), "drafts": rng.choice([1, 2, 3, 4, 5, 8, 16]),
             "ragged": rng.random() < 0.5, "draft_probs": rng.random() < 0.7, "mix": mix}
        c["n_seq"] = _spread(rng, 1, max(2, min(256, 82_000_000 // (c["vocab"] * (c["drafts"] + 1)))))
        return c
    c = {**PAGES, "page": rng.choice([16, 16, 32, 64, 128, 256]), "n_seq": _spread(rng, 4, 300), "spare": rng.choice([0.02, 0.3, 1.0]),
         "len_sigma": rng.choice([0.3, 0.8]), "shared": rng.choice([0.0, 0.3, 0.6]), "mix": mix}
    c["len_max"] = 1024 * c["page"]
    c["len_mid"] = _spread(rng, 20, 300 * c["page"])
    if op == "resize":
        return {**RESIZE, **c, "grow": rng.choice([1, 1, 2, 5, 9, 100]), "cut": rng.choice([0.0, 0.4]), "drop": rng.choice([0.0, 0.1, 0.9]),
                "admit": rng.choice([0.0, 0.1, 0.5])}
    if op == "fork":
        return {**FORK, **c, "kind": rng.choice(["samples", "beams", "thin"]), "out_seq": _spread(rng, 1, 300)}
    return {**COMPACT, **c}


# ---------------------------------------------------------------------------------------------- pages

def _state(case, r):
    """Rows of the table, lengths and the number of pages, as a client comes to have them: lengths log-normal, pages in no
    particular order, some sequences forked from the one before them (all pages but the own end shared)."""
    ps, rows, lens = case["page"], [], []
    for s in range(case["n_seq"]):
        n = max(1, min(case["len_max"], int(round(case["len_mid"] * math.exp(case["len_sigma"] * r.gauss(0.0, 1.0))))))
        lens.append(n)
        rows.append(None)
    used = 0
    for s in range(case["n_seq"]):
        if s and r.random() < case["shared"]:
            row = list(rows[s - 1])
            if r.random() < 0.5:                             # forked just now: the last page is shared, too
                rows[s], lens[s] = row, lens[s - 1]
                continue
            keep = len(row) - 1                              # forked earlier: it has an end of its own by now
            lens[s] = min(case["len_max"], keep * ps + 1 + r.randrange(2 * ps))
            rows[s] = row[:keep]
        else:
            rows[s] = []
        while len(rows[s]) < -(-lens[s] // ps):
            rows[s].append(used)
            used += 1
    n_pages = used + max(5, int(case["spare"] * used))
    order = list(range(n_pages))
    r.shuffle(order)
    return [[order[p] for p in row] for row in rows], lens, n_pages


def _sizes(case):
    """Rows, lengths and pages for work(): they depend on the case alone."""
    return _state(case, random.Random(case["mix"]))


def _targets(case, lens, r):
    """New lengths of a round: most grow, some are cut back, retired, or come in anew (then they were empty before)."""
    new = []
    for s, n in enumerate(lens):
        x = r.random()
        if s and x < case["drop"]:                           # the first one stays
            new.append(0)
        elif r.random() < case["cut"]:
            new.append(max(0, n - r.randrange(1, 2 * case["page"])))
        else:
            new.append(min(case["len_max"] + 100, n + case["grow"]))
    return new


def _parents(case, r):
    n, m = case["n_seq"], case["out_seq"]
    if case["kind"] == "samples":
        return [i * n // m for i in range(m)] if m >= n else list(range(m))
    if case["kind"] == "thin":                               # finished sequences leave, the others move up
        alive = [s for s in range(n) if r.random() < 0.7]
        return (alive + [-1] * m)[:m]
    return [r.randrange(n) if r.random() < 0.5 else i % n for i in range(m)]


def _pages_state(case, seed):
    """Everything on the host: the case gives the sizes, the seed the order of pages and what happens in the round."""
    rows, lens, n_pages = _sizes(case)
    r = random.Random(seed * 1_000_003 + case["mix"])
    order = list(range(n_pages))
    r.shuffle(order)
    rows = [[order[p] for p in row] for row in rows]
    new = None
    if case["op"] == "resize":
        for s in range(len(rows)):                           # requests that are admitted in this round: empty rows so far
            if r.random() < case["admit"]:
                rows[s], lens[s] = [], 0
        new = _targets(case, lens, r)
        for s in range(len(rows)):
            if not rows[s]:
                new[s] = 1 + r.randrange(max(1, case["len_mid"]))
    refs = [0] * n_pages
    for row in rows:
        for p in row:
            refs[p] += 1
    width = -(-(case["len_max"] + 100) // case["page"])
    return rows, lens, n_pages, refs, width, new, (_parents(case, r) if case["op"] == "fork" else None)


def _prepare_pages(case, seed):
    rows, lens, n_pages, refs, width, new, parent = _pages_state(case, seed)
    dev = torch.device("cuda")
    table = torch.full((len(rows), width), -1, dtype=torch.int32)
    for s, row in enumerate(rows):
        table[s, :len(row)] = torch.tensor(row, dtype=torch.int32)
    s = {"case": case, "refs": torch.tensor(refs, dtype=torch.int32, device=dev), "table": table.to(dev), "page": case["page"],
         "kv_len": torch.tensor(lens, dtype=torch.int32, device=dev), "n_pages": n_pages, "width": width}
    if new is not None:
        s["new_len"] = torch.tensor(new, dtype=torch.int32, device=dev)
    if parent is not None:
        s["parent"] = torch.tensor(parent, dtype=torch.int32, device=dev)
    return s


def _resize(s):
    ps, n, dev = s["page"], s["n_pages"], s["refs"].device
    table, old, new = s["table"].long(), s["kv_len"].long(), s["new_len"].long()
    b, width = table.shape
    have, need = (old + ps - 1) // ps, (new + ps - 1) // ps
    col, seq = torch.arange(width, device=dev), torch.arange(b, device=dev)
    refs = torch.cat([s["refs"].long(), torch.zeros(1, dtype=torch.long, device=dev)])           # one place more, for what has none
    gone = (col >= need[:, None]) & (col < have[:, None])
    refs.scatter_add_(0, torch.where(gone, table, n).view(-1), -gone.long().view(-1))
    refs[n] = 0
    grow = new > old
    inside = grow & (old % ps != 0)
    last = torch.where(inside, table.gather(1, (have - 1).clamp_min(0)[:, None])[:, 0], n)
    growers = torch.zeros(n + 1, dtype=torch.long, device=dev).scatter_add_(0, last, inside.long())
    latest = torch.full((n + 1,), -1, dtype=torch.long, device=dev).scatter_reduce_(0, last, seq, "amax")
    own_page = inside & (refs[last] > 1) & ~((growers[last] == refs[last]) & (latest[last] == seq))
    takes = own_page.long() + torch.where(grow, need - have, 0)
    upto = takes.cumsum(0)
    base = upto - takes
    free = refs[:n] == 0
    rank = free.long().cumsum(0) - 1
    n_free = free.long().sum()
    queue = torch.full((n + 1,), -1, dtype=torch.long, device=dev).scatter_(0, torch.where(free, rank, n), torch.arange(n, device=dev))
    fits = grow & (upto <= n_free)
    own_page = own_page & fits
    refs.scatter_add_(0, torch.where(own_page, last, n), -own_page.long())
    at = col - have[:, None] + own_page.long()[:, None]                                          # which of the pages taken
    fresh = fits[:, None] & (((col == have[:, None] - 1) & own_page[:, None]) | ((col >= have[:, None]) & (col < need[:, None])))
    got = queue[torch.where(fresh, (base[:, None] + at).clamp(0, n), n)]
    kept = col < torch.where(new < old, need, have)[:, None]
    out = torch.where(fresh, got, torch.where(kept, table, -1))
    refs.scatter_(0, torch.where(fresh, got, n).view(-1), 1)
    order = own_page.long().cumsum(0) - 1
    place = torch.where(own_page, order, b)
    src = torch.full((b + 1,), -1, dtype=torch.long, device=dev).scatter_(0, place, last)[:b]
    dst = torch.full((b + 1,), -1, dtype=torch.long, device=dev).scatter_(0, place, queue[torch.where(own_page, base.clamp(0, n), n)])[:b]
    i32 = torch.int32
    return {"refs": refs[:n].to(i32), "page_table": out.to(i32), "kv_len": torch.where(grow & ~fits, old, new).to(i32), "src": src.to(i32),
            "dst": dst.to(i32), "count": own_page.sum().to(i32).view(1)}


def _fork(s):
    ps, n, dev = s["page"], s["n_pages"], s["refs"].device
    table, old, parent = s["table"].long(), s["kv_len"].long(), s["parent"].long()
    b, width = table.shape
    col = torch.arange(width, device=dev)
    there = parent >= 0
    children = torch.zeros(b + 1, dtype=torch.long, device=dev).scatter_add_(0, torch.where(there, parent, b), there.long())[:b]
    held = col < ((old + ps - 1) // ps)[:, None]
    refs = torch.cat([s["refs"].long(), torch.zeros(1, dtype=torch.long, device=dev)])
    refs.scatter_add_(0, torch.where(held, table, n).view(-1), torch.where(held, children[:, None] - 1, 0).view(-1))
    up = parent.clamp_min(0)
    out = torch.where(there[:, None] & held[up], table[up], -1)
    return {"refs": refs[:n].to(torch.int32), "page_table": out.to(torch.int32), "kv_len": torch.where(there, old[up], 0).to(torch.int32)}


def _compact(s):
    ps, n, dev = s["page"], s["n_pages"], s["refs"].device
    table, old = s["table"].long(), s["kv_len"].long()
    refs, pages = s["refs"].long(), torch.arange(n, device=dev)
    live = refs != 0
    n_live = live.long().sum()
    late, hole = live & (pages >= n_live), ~live & (pages < n_live)
    count = late.long().sum()
    none = torch.full((n + 1,), -1, dtype=torch.long, device=dev)
    src = none.clone().scatter_(0, torch.where(late, late.long().cumsum(0) - 1, n), pages)[:n]
    dst = none.clone().scatter_(0, torch.where(hole, hole.long().cumsum(0) - 1, n), pages)[:n]
    moved = torch.arange(n, device=dev) < count
    src, dst = torch.where(moved, src, -1), torch.where(moved, dst, -1)
    to = torch.arange(n + 1, device=dev).scatter_(0, torch.where(moved, src, n), dst)
    out = torch.zeros(n + 1, dtype=torch.long, device=dev).scatter_(0, torch.where(live, to[:n], n), refs)[:n]
    held = torch.arange(table.shape[1], device=dev) < ((old + ps - 1) // ps)[:, None]
    i32 = torch.int32
    return {"refs": out.to(i32), "page_table": torch.where(held, to[table.clamp_min(0)], -1).to(i32), "src": src.to(i32), "dst": dst.to(i32),
            "count": count.to(i32).view(1)}


# ----------------------------------------------------------------------------------------------- copy

def _moves(case, r):
    n, m = case["pages"], case["moves"]
    if case["order"] == "compact":                           # both ascending, from the upper part to the lower
        cut = n // 2
        return sorted(r.sample(range(cut, n), m)), sorted(r.sample(range(cut), m))
    both = r.sample(range(n), 2 * m)
    return both[:m], both[m:]


def _prepare_copy(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    src, dst = _moves(case, random.Random(seed * 1_000_003 + case["mix"]))
    dt = DTYPES[case["dtype"]]
    shape = (case["layers"], case["pages"], case["kv_heads"], case["page"], case["dim"])
    cache = {}                                               # the caches of all layers, cut from one allocation a kind
    for name in ("k", "v"):
        if case["fmt"] == "same":
            cache[name] = torch.randn(shape, generator=gen, device=dev, dtype=dt)
        elif case["fmt"] == "int8":
            cache[name] = torch.randint(-127, 128, shape, generator=gen, device=dev, dtype=torch.int8)
        else:
            cache[name] = torch.empty(shape, device=dev, dtype=torch.float8_e4m3fn)
            for layer in cache[name]:
                layer.copy_(torch.randn(shape[1:], generator=gen, device=dev, dtype=dt).mul_(100.0))
        if case["fmt"] != "same":
            cache[name + "_scale"] = torch.rand(shape[:4], generator=gen, device=dev) * 0.01
    s = {"case": case, "src": torch.tensor(src, dtype=torch.int32, device=dev), "dst": torch.tensor(dst, dtype=torch.int32, device=dev),
         "cache": cache, "layers": [{n: t[i] for n, t in cache.items()} for i in range(case["layers"])]}
    if own:
        import paper_2502_15763_b200 as hos
        s["hos"] = hos
        s["caches"] = [hos.hos_kv_cache(x["k"], x["v"], x.get("k_scale"), x.get("v_scale"), dtype=dt) for x in s["layers"]]
    return s


def _copy(s):
    src, dst = s["src"].long(), s["dst"].long()
    for layer in s["layers"]:
        for t in layer.values():
            raw = t.view(torch.uint8) if t.element_size() == 1 else t
            raw[dst] = raw[src]
    return s["cache"]


# --------------------------------------------------------------------------------------------- verify

def _drafts(case):
    """Drafts of every sequence."""
    r = random.Random(case["mix"])
    return [r.randrange(case["drafts"] + 1) if case["ragged"] else case["drafts"] for _ in range(case["n_seq"])]


def _prepare_verify(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    k = _drafts(case)
    n, v, dt = sum(k) + len(k), case["vocab"], DTYPES[case["dtype"]]
    starts = [0]
    for x in k:
        starts.append(starts[-1] + x + 1)
    off = torch.tensor(starts, dtype=torch.int32, device=dev)
    target = torch.empty((n, v), dtype=dt, device=dev)
    draft = torch.empty((n, v), dtype=dt, device=dev) if case["draft_probs"] else None
    tokens = torch.zeros((n,), dtype=torch.int32, device=dev)
    for s in range(len(k)):
        rows = slice(starts[s], starts[s + 1])
        logits = 3.0 * torch.randn((k[s] + 1, v), generator=gen, device=dev)
        guess = logits + 0.8 * torch.randn((k[s] + 1, v), generator=gen, device=dev)
        if s % 4 == 1:                                       # sampled from the likeliest tokens only
            least = logits.topk(min(50, v), dim=-1).values[:, -1:]
            logits = torch.where(logits < least, -math.inf, logits)
        if s % 8 == 3:                                       # not sampled at all: the likeliest token has everything
            logits = torch.where(logits < logits.amax(-1, keepdim=True), -math.inf, logits)
        target[rows] = torch.softmax(logits, -1).to(dt)
        q = torch.softmax(guess, -1)
        if draft is not None:
            draft[rows] = q.to(dt)
            pick = (q / torch.empty_like(q).exponential_(generator=gen)).argmax(-1)
        else:
            pick = torch.where(torch.rand(k[s] + 1, generator=gen, device=dev) < 0.7, logits.argmax(-1), guess.argmax(-1))
        tokens[rows][1:] = pick[:-1].to(torch.int32)
    s = {"case": case, "off": off, "target": target, "draft": draft, "tokens": tokens, "u_accept": torch.rand((n,), generator=gen, device=dev),
         "u_sample": torch.rand((len(k),), generator=gen, device=dev), "most": max(k),
         "kv_len": torch.tensor([100 + 3 * i + x + 1 for i, x in enumerate(k)], dtype=torch.int32, device=dev)}
    return s


def _verify(s):
    dev, n_seq = s["target"].device, s["off"].shape[0] - 1
    off = s["off"].long()
    k = off[1:] - off[:-1] - 1
    n = s["target"].shape[0]
    if s["most"]:
        i = torch.arange(s["most"], device=dev)
        row = (off[:-1, None] + i).clamp_max(n - 1)
        token = s["tokens"].long()[(row + 1).clamp_max(n - 1)]
        p = s["target"][row, token].double()
        q = s["draft"][row, token].double() if s["draft"] is not None else torch.ones_like(p)
        good = (s["u_accept"].double()[row] * q < p) & (i < k[:, None])
        accepted = good.long().cumprod(1).sum(1)
    else:
        accepted = torch.zeros_like(k)
    at = off[:-1] + accepted
    rejected = (accepted < k)[:, None]
    p = s["target"][at].double()
    if s["draft"] is not None:
        q = s["draft"][at].double()
    else:
        q = torch.zeros_like(p).scatter_(1, s["tokens"].long()[(at + 1).clamp_max(n - 1)][:, None], 2.0)     # more than any p
    w = torch.where(rejected, (p - q).clamp_min(0.0), p)
    w = torch.where((w.sum(1, keepdim=True) > 0) | ~rejected, w, p)
    c = w.cumsum(1)
    nxt = (c <= s["u_sample"].double()[:, None] * c[:, -1:]).sum(1)
    tok = torch.arange(n, device=dev)
    seq = torch.bucketize(tok, off[1:], right=True)
    j = tok - off[seq]
    out = torch.where(j < accepted[seq], s["tokens"].long()[(tok + 1).clamp_max(n - 1)], torch.where(j == accepted[seq], nxt[seq], -1))
    i32 = torch.int32
    return {"accepted": accepted.to(i32), "next": nxt.to(i32), "tokens": out.to(i32), "new_len": (s["kv_len"].long() - k + accepted).to(i32)}


# ------------------------------------------------------------------------------------------- together

def prepare(case, seed):
    s = _prepare_copy(case, seed) if case["op"] == "copy" else _prepare_verify(case, seed) if case["op"] == "verify" else _prepare_pages(case, seed)
    if own:
        import paper_2502_15763_b200 as hos
        s["hos"] = hos
    return s


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"resize": _resize, "fork": _fork, "compact": _compact, "copy": _copy, "verify": _verify}[op](s)
    hos = s["hos"]
    if op == "copy":
        hos.hos_kv_copy_pages(s["caches"], s["src"], s["dst"])
        return s["cache"]
    if op == "verify":
        r = hos.hos_verify_drafts(s["tokens"], s["target"], s["draft"], s["off"], s["u_accept"], s["u_sample"], kv_len=s["kv_len"])
        return {n: r[n] for n in ("accepted", "next", "tokens", "new_len")}
    if op == "resize":
        r = hos.hos_kv_resize(s["refs"], s["table"], s["kv_len"], s["new_len"], s["page"])
        return {n: r[n] for n in ("refs", "page_table", "kv_len", "src", "dst", "count")}
    if op == "fork":
        r = hos.hos_kv_fork(s["refs"], s["table"], s["kv_len"], s["parent"], s["page"])
        return {n: r[n] for n in ("refs", "page_table", "kv_len")}
    r = hos.hos_kv_compact(s["refs"], s["table"], s["kv_len"], s["page"])
    return {n: r[n] for n in ("refs", "page_table", "src", "dst", "count")}


def work(case):
    if case["op"] == "copy":
        vec = 2 * case["dim"] if case["fmt"] == "same" else case["dim"] + 4
        return {"bytes": 2 * 2 * case["moves"] * case["layers"] * case["kv_heads"] * case["page"] * vec, "flops": 0}
    if case["op"] == "verify":
        size = 4 if case["dtype"] == "f32" else 2
        # one row of the target each, and one of the draft where not all was accepted (about three drafts in four are)
        rows = sum(1 + (1 - 0.75 ** k if case["draft_probs"] else 0) for k in _drafts(case))
        return {"bytes": int(rows * case["vocab"] * size), "flops": int(2 * rows * case["vocab"])}
    rows, _, n_pages = _sizes(case)
    width = -(-(case["len_max"] + 100) // case["page"])
    held = sum(len(r) for r in rows)
    out = case["out_seq"] if case["op"] == "fork" else len(rows)
    lists = {"resize": 2 * len(rows), "fork": 0, "compact": 2 * n_pages}[case["op"]]
    return {"bytes": 4 * (2 * n_pages + held + out * width + lists), "flops": 0}


# ---------------------------------------------------------------------------------------------- exact

def _exact_resize(rows, lens, refs, new, ps, width):
    refs, rows, lens, src, dst = list(refs), [list(r) for r in rows], list(lens), [], []
    pages = [-(-n // ps) for n in new]
    for s, n in enumerate(new):
        while len(rows[s]) > pages[s]:
            refs[rows[s].pop()] -= 1
    left = [p for p, r in enumerate(refs) if r == 0]
    at, stuck = 0, False
    for s, n in enumerate(new):
        if n <= lens[s]:
            lens[s] = n
            continue
        split = lens[s] % ps != 0 and refs[rows[s][-1]] > 1
        takes = int(split) + pages[s] - len(rows[s])
        if stuck or at + takes > len(left):
            stuck = True
            continue
        mine = left[at:at + takes]
        at += takes
        for p in mine:
            refs[p] = 1
        if split:
            src.append(rows[s][-1])
            dst.append(mine[0])
            refs[src[-1]] -= 1
            rows[s][-1] = mine.pop(0)
        rows[s] += mine
        lens[s] = n
    return refs, rows, lens, src, dst


def exact(case, seed):
    i32, dev = torch.int32, torch.device("cuda")
    if case["op"] == "copy":
        s = _prepare_copy(case, seed)
        src, dst = s["src"].tolist(), s["dst"].tolist()
        if len(src) * case["layers"] > 12000:                # one small copy after the other takes too long
            return None
        for layer in s["layers"]:
            for t in layer.values():
                for a, b in zip(src, dst):
                    t[b].copy_(t[a])
        return s["cache"]
    if case["op"] == "verify":
        s = _prepare_verify(case, seed)
        starts, tokens, u, us = s["off"].tolist(), s["tokens"].tolist(), s["u_accept"].tolist(), s["u_sample"].tolist()
        out = {"accepted": [], "next": [], "tokens": [], "new_len": []}
        for q in range(case["n_seq"]):
            a, k = starts[q], starts[q + 1] - starts[q] - 1
            p = s["target"][a:a + k + 1].to(torch.float64).cpu()
            d = s["draft"][a:a + k + 1].to(torch.float64).cpu() if s["draft"] is not None else None
            j = 0
            while j < k and u[a + j] * (float(d[j, tokens[a + j + 1]]) if d is not None else 1.0) < float(p[j, tokens[a + j + 1]]):
                j += 1
            w = p[j].clone()
            if j < k:
                if d is not None:
                    w -= d[j]
                    w[w < 0] = 0.0
                else:
                    w[tokens[a + j + 1]] = 0.0
                if float(w.sum()) == 0.0:
                    w = p[j].clone()
            c = torch.cumsum(w, 0)
            pick = int(torch.searchsorted(c, torch.tensor([us[q] * float(c[-1])], dtype=torch.float64), right=True))
            out["accepted"].append(j)
            out["next"].append(pick)
            out["tokens"] += tokens[a + 1:a + 1 + j] + [pick] + [-1] * (k - j)
            out["new_len"].append(int(s["kv_len"][q]) - k + j)
        return {n: torch.tensor(x, dtype=i32, device=dev) for n, x in out.items()}
    rows, lens, n_pages, refs, width, new, parent = _pages_state(case, seed)
    ps, more = case["page"], {}
    if case["op"] == "resize":
        refs, rows, lens, src, dst = _exact_resize(rows, lens, refs, new, ps, width)
        more = {"kv_len": lens, "src": src + [-1] * (len(rows) - len(src)), "dst": dst + [-1] * (len(rows) - len(dst)), "count": [len(src)]}
    elif case["op"] == "fork":
        rows, lens = [list(rows[p]) if p >= 0 else [] for p in parent], [lens[p] if p >= 0 else 0 for p in parent]
        refs = [0] * n_pages
        for row in rows:
            for p in row:
                refs[p] += 1
        more = {"kv_len": lens}
    else:
        n_live = sum(1 for x in refs if x)
        src = [p for p in range(n_live, n_pages) if refs[p]]
        dst = [p for p in range(n_live) if not refs[p]]
        to = dict(zip(src, dst))
        for a, b in to.items():
            refs[b], refs[a] = refs[a], 0
        rows = [[to.get(p, p) for p in row] for row in rows]
        fill = [-1] * (n_pages - len(src))
        more = {"src": src + fill, "dst": dst + fill, "count": [len(src)]}
    table = torch.full((len(rows), width), -1, dtype=i32)
    for s, row in enumerate(rows):
        table[s, :len(row)] = torch.tensor(row, dtype=i32)
    r = {"refs": torch.tensor(refs, dtype=i32, device=dev), "page_table": table.to(dev)}
    r.update({n: torch.tensor(x, dtype=i32, device=dev) for n, x in more.items()})
    return r
