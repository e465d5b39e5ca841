"""Replays one client's schedule on the KV-cache operators and fits the cost model's token terms to what they take.

The scheduler's cost model has a term in the prompt tokens of a prefill and one in the KV tokens of a decode round
(a decode iteration lasts decode_fixed_us + decode_per_seq_us * B + sum KV / decode_kv_div).  This command schedules a
workload (offline packing, online simulation), takes the iteration trace of one client, and runs every iteration's KV
work for real: requests are admitted into a paged cache, their prompts' keys and values are appended and attended to in one
ragged call, decode rounds append and attend with one token per running request, retired requests give their pages back.
Every iteration is held against its trace record and timed (the two calls as a graph of several layers, each with a cache of its
own as in a model, so that a layer's keys and values come from memory and not from what the layer before left on the chip; the
host's side stays out of the figures), and the times are fitted by least squares.

    python -m paper_2502_15763_b200.replay --workload c0 --client 0 --heads 64 --kv-heads 8 --format int8 --layers 80
"""
from __future__ import annotations

import argparse
import json

import numpy as np

from . import (HOS_QUEUE_SORTED, ITER_REC_DTYPE, hos_kv_append, hos_kv_cache, hos_offline_pack, hos_online_simulate,
               hos_paged_attention, hos_trace_fill, hos_trace_offsets)
from .binding import view_struct


def client_schedule(p, o, n_clients, batch_cap, kv_budget, cost_model, client, lam_q16=1 << 16):
    """Trace records of one client of a single instance, and its requests in queue order."""
    import torch
    dp, do = (torch.from_numpy(np.ascontiguousarray(x[None].astype(np.int32))).cuda() for x in (p, o))
    args = (dp, do, n_clients, batch_cap, kv_budget, cost_model)
    assign = hos_offline_pack(*args)["assign"]
    lam = torch.tensor([lam_q16], dtype=torch.int64).to(torch.int32).cuda()
    sim = hos_online_simulate(*args, assign, lam, queue_order=HOS_QUEUE_SORTED, keep_events=True)
    off = hos_trace_offsets(sim["cres"])
    trace = torch.empty((int(off[-1]), ITER_REC_DTYPE.itemsize), dtype=torch.uint8, device="cuda")
    hos_trace_fill(*args, 1, sim, trace, off)
    if int(sim["status"].abs().sum()):
        raise RuntimeError("the simulation reported a problem: status bits set")
    recs = view_struct(trace, ITER_REC_DTYPE)[int(off[client]):int(off[client + 1])]
    mine = np.flatnonzero(assign[0].cpu().numpy() == client)
    total = p[mine].astype(np.int64) + o[mine]
    return recs, mine[np.lexsort((mine, -total))]


class PagePool:
    """Free pages of a cache; a request holds the pages of all its tokens from admission to retirement."""

    def __init__(self, n_pages, page_size):
        self.free, self.page_size = list(range(n_pages))[::-1], page_size

    def take(self, tokens):
        return [self.free.pop() for _ in range(-(-tokens // self.page_size))]

    def give(self, pages):
        self.free.extend(pages)


def device_us(steps):
    """Device time of one of `steps`, from a graph of them."""
    import torch
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for step in steps:
            step()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    graph.replay()
    start.record()
    graph.replay()
    end.record()
    torch.cuda.synchronize()
    return start.elapsed_time(end) * 1000.0 / len(steps)


def cache_bytes(batch_cap, kv_budget, kv_heads, head_dim, page, fmt):
    """Memory of one layer's cache in replay()."""
    vector = 2 * head_dim if fmt == "same" else head_dim + 4
    return 2 * (-(-kv_budget // page) + batch_cap) * kv_heads * page * vector


def replay(p, o, recs, queue, batch_cap, kv_budget, heads=64, kv_heads=8, head_dim=128, page=128, fmt="int8", max_iters=None,
           repeat=8, seed=0, watch=None):
    """Runs the records' KV work; returns per-iteration arrays (kind, n, tokens, us) and the pages' high-water mark.  The times
    are device times of one of `repeat` layers, each with a cache of its own (of the same pages); repeat = 0 runs every
    iteration once, untimed.  watch(iteration, requests, x, cache, tok_off, kv_len, page_table, out): called after each
    iteration with what one layer got ([token][queries, keys, values]) and gave."""
    import torch
    dt = torch.bfloat16
    # every running request may leave one page part empty
    n_pages = -(-kv_budget // page) + batch_cap
    shape = (n_pages, kv_heads, page, head_dim)
    store = {"same": dt, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[fmt]

    def layer():
        k, v = (torch.zeros(shape, dtype=torch.uint8 if fmt != "same" else dt, device="cuda").view(store) for _ in range(2))
        ks, vs = (torch.zeros(shape[:3], device="cuda") if fmt != "same" else None for _ in range(2))
        return hos_kv_cache(k, v, ks, vs, dtype=dt)

    caches = [layer() for _ in range(max(repeat, 1))]
    pool, running, most_pages = PagePool(n_pages, page), [], 0          # running: [request, tokens in the cache, steps left, pages]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    longest = int(p[queue].max()) if len(queue) else 1
    qkv = torch.randn((max(batch_cap, 1) * longest, heads + 2 * kv_heads, head_dim), generator=gen, device="cuda", dtype=dt)
    us, out = [], []
    for it, rec in enumerate(recs if max_iters is None else recs[:max_iters]):
        prefill = bool(rec["kind_n"] >> 31)
        n = int(rec["kind_n"] & 0x7FFFFFFF)
        if prefill:
            first = int(rec["aux"])
            batch = [[int(r), int(p[r]), int(o[r]), pool.take(int(p[r]) + int(o[r]))] for r in queue[first:first + n]]
            running += batch
            new = [b[1] for b in batch]
            seen = sum(new)
        else:
            batch = running
            seen = sum(b[1] for b in batch)
            new = [1] * len(batch)
            for b in batch:
                b[1] += 1
        if len(batch) != n or seen != int(rec["tokens"]):
            raise RuntimeError(f"iteration {it}: {len(batch)} requests, {seen} tokens; the trace says {n} and {int(rec['tokens'])}")
        most_pages = max(most_pages, n_pages - len(pool.free))
        width = max(len(b[3]) for b in batch)
        table = torch.tensor([b[3] + [0] * (width - len(b[3])) for b in batch], dtype=torch.int32).cuda()
        off = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
        kv_len = torch.tensor([b[1] for b in batch], dtype=torch.int32).cuda()
        x = qkv[:sum(new)]

        def step(cache=caches[0]):
            hos_kv_append(cache, x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], off, kv_len, table)
            return hos_paged_attention(x[:, :heads], cache, off, kv_len, table, max(new))["out"]

        got = step()
        us.append(device_us([lambda c=c: step(c) for c in caches]) if repeat else 0.0)
        if watch is not None:
            watch(it, [b[0] for b in batch], x, caches[0], off, kv_len, table, got)
        out.append((prefill, n, seen))
        if not prefill:
            done = [b for b in running if (b.__setitem__(2, b[2] - 1) or b[2] == 0)]
            if len(done) != int(rec["aux"]):
                raise RuntimeError(f"iteration {it}: {len(done)} requests are done; the trace says {int(rec['aux'])}")
            for b in done:
                pool.give(b[3])
            running = [b for b in running if b[2] > 0]
    torch.cuda.synchronize()
    if any(int(c.status.abs().sum()) for c in caches):
        raise RuntimeError("the cache calls reported a problem: status bits set")
    kind, n, tokens = np.array(out, dtype=np.int64).reshape(-1, 3).T
    return dict(prefill=kind.astype(bool), n=n, tokens=tokens, us=np.array(us, dtype=float), most_pages=most_pages, n_pages=n_pages)


def fit(r, layers):
    """Least squares: prefill us = a + b * sum p, decode us = c + d * B + e * sum KV, per layer and for `layers` of them."""
    def solve(mask, cols):
        if mask.sum() < cols.shape[1] + 2:
            return None
        return np.linalg.lstsq(cols[mask], r["us"][mask], rcond=None)[0]

    one = np.ones(len(r["us"]))
    pre = solve(r["prefill"], np.stack([one, r["tokens"]], 1))
    dec = solve(~r["prefill"], np.stack([one, r["n"], r["tokens"]], 1))
    res = dict(iterations=int(len(r["us"])), prefills=int(r["prefill"].sum()), most_pages=int(r["most_pages"]), pages=int(r["n_pages"]),
               median_decode_us=float(np.median(r["us"][~r["prefill"]])) if (~r["prefill"]).any() else None)
    if pre is not None:
        res["prefill_us_per_token"] = float(pre[1] * layers)
    if dec is not None:
        res["decode_us_per_kv_token"] = float(dec[2] * layers)
        res["decode_kv_div"] = float(1.0 / (dec[2] * layers)) if dec[2] > 0 else None
    return res


def main(argv=None):
    import torch
    from workload import workload
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="c0")
    ap.add_argument("--instance", type=int, default=0)
    ap.add_argument("--client", type=int, default=0)
    ap.add_argument("--heads", type=int, default=64)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--page", type=int, default=128)
    ap.add_argument("--format", default="int8", choices=("same", "e4m3", "int8"))
    ap.add_argument("--layers", type=int, default=80, help="layers of the model; as many as fit are run and timed")
    ap.add_argument("--iters", type=int, default=None)
    a = ap.parse_args(argv)
    w = workload(a.workload).subset(a.instance, 1)
    p, o = (x[0] for x in w.lengths())
    recs, queue = client_schedule(p, o, w.n_clients, w.batch_cap, w.kv_budget, w.cost_model, a.client)
    one = cache_bytes(w.batch_cap, w.kv_budget, a.kv_heads, a.head_dim, a.page, a.format)
    run = max(1, min(a.layers, int(0.6 * torch.cuda.mem_get_info()[0]) // one))
    r = replay(p, o, recs, queue, w.batch_cap, w.kv_budget, a.heads, a.kv_heads, a.head_dim, a.page, a.format, a.iters, repeat=run)
    print(json.dumps({"workload": a.workload, "client": a.client, "layers": a.layers, "layers_run": run, **fit(r, a.layers)}))


if __name__ == "__main__":
    main()
