"""Replays one client's schedule with drafted tokens, its pages kept on the device.

Where `replay` takes a decode iteration of the trace for what it is, one token per running request, this command gets the
same tokens in fewer rounds: a draft model proposes a few tokens per request, one round appends and attends to all of them,
and what the target does not accept is taken back.  Between two changes of the batch (a prefill, a request that is done) every request
makes as many tokens as the trace's iterations in between, so each such stretch is held against its trace records.
The pages live on the device: requests are admitted, grow and give back by hos_kv_resize, finished ones leave by hos_kv_fork (the others
move up), pages that are shared and about to be written are copied, and after some stretches the pool is compacted.
Target and draft probabilities are synthetic: random ones that agree to a given degree.

    python -m paper_2502_15763_b200.drafted --workload c0 --client 0 --drafts 4 --agree 0.7
"""
from __future__ import annotations

import argparse
import json

import numpy as np

from . import (hos_kv_append, hos_kv_cache, hos_kv_compact, hos_kv_copy_pages, hos_kv_fork, hos_kv_resize, hos_paged_attention,
               hos_verify_drafts)
from .replay import client_schedule


def stretches(recs):
    """The trace as [(records of one prefill)] and [(decode records without a change of the batch in between)]."""
    out = []
    for i, rec in enumerate(recs):
        prefill = bool(rec["kind_n"] >> 31)
        if not prefill and out and not out[-1][0] and not int(recs[i - 1]["aux"]):
            out[-1][1].append(i)
        else:
            out.append((prefill, [i]))
    return out


class Client:
    """The running requests' pages (row s of the state is the s-th running request) and the layers' caches."""

    def __init__(self, batch_cap, kv_budget, drafts, kv_heads, head_dim, page, fmt, layers):
        import torch
        dt = torch.bfloat16
        self.page, self.rows, self.requests = page, max(batch_cap, 1), []
        # every request may leave a page part empty, and drafts lie beyond the budget until they are taken back
        n_pages = -(-kv_budget // page) + self.rows * (1 + -(-(drafts + 1) // page))
        shape, self.caches = (n_pages, kv_heads, page, head_dim), []
        store = {"same": dt, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[fmt]
        for _ in range(layers):
            k, v = (torch.zeros(shape, dtype=torch.uint8 if fmt != "same" else dt, device="cuda").view(store) for _ in range(2))
            ks, vs = (torch.zeros(shape[:3], device="cuda") if fmt != "same" else None for _ in range(2))
            self.caches.append(hos_kv_cache(k, v, ks, vs, dtype=dt))
        width = -(-(kv_budget + drafts + 1) // page)
        self.refs = torch.zeros((n_pages,), dtype=torch.int32, device="cuda")
        self.table = torch.full((self.rows, width), -1, dtype=torch.int32, device="cuda")
        self.kv_len = torch.zeros((self.rows,), dtype=torch.int32, device="cuda")
        self.most_pages, self.n_pages = 0, n_pages

    def _take(self, r, what):
        if int(r["status"].abs().sum()):
            raise RuntimeError(f"{what}: status bits set")
        self.refs, self.table, self.kv_len = r["refs"], r["page_table"], r["kv_len"]
        self.most_pages = max(self.most_pages, int((self.refs > 0).sum()))

    def resize(self, new_len):
        r = hos_kv_resize(self.refs, self.table, self.kv_len, new_len, self.page, out=(self.refs, self.table, self.kv_len))
        hos_kv_copy_pages(self.caches, r["src"], r["dst"], r["count"])
        self._take(r, "hos_kv_resize")

    def drop(self, keep):
        """Only rows `keep` stay, in this order."""
        import torch
        parent = torch.tensor(keep + [-1] * (self.rows - len(keep)), dtype=torch.int32).cuda()
        self._take(hos_kv_fork(self.refs, self.table, self.kv_len, parent, self.page), "hos_kv_fork")

    def compact(self):
        r = hos_kv_compact(self.refs, self.table, self.kv_len, self.page, out=(self.refs, self.table, self.kv_len))
        hos_kv_copy_pages(self.caches, r["src"], r["dst"], r["count"])
        self._take(r, "hos_kv_compact")

    def attend(self, x, heads, kv_heads, rows, new):
        """Appends and attends with the new tokens of these rows in every layer; the last layer's outputs and the offsets."""
        import torch
        off = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
        at = torch.tensor(rows, dtype=torch.int64).cuda()
        kv_len, table = self.kv_len[at], self.table[at]
        for cache in self.caches:
            hos_kv_append(cache, x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], off, kv_len, table)
            out = hos_paged_attention(x[:, :heads], cache, off, kv_len, table, max(new))["out"]
        return out, off, kv_len, table


def probabilities(n, vocab, agree, gen):
    """Target's and draft's probabilities, n rows each: the draft's are the target's to the degree `agree`, and others besides."""
    import torch
    target, other = (torch.softmax(3.0 * torch.randn((n, vocab), generator=gen, device="cuda"), -1) for _ in range(2))
    return target, agree * target + (1.0 - agree) * other


def replay(p, o, recs, queue, batch_cap, kv_budget, drafts=4, agree=0.7, vocab=32000, heads=64, kv_heads=8, head_dim=128, page=128, fmt="int8",
           layers=1, compact_every=8, max_iters=None, seed=0, watch=None):
    """Runs the records' work with drafted tokens; returns what it took.  watch(requests, x, off, kept, client): called after each prefill and
    round with the requests, their new tokens' [queries, keys, values], how many of each stay, and the state."""
    import torch
    client = Client(batch_cap, kv_budget, drafts, kv_heads, head_dim, page, fmt, layers)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    running, rounds, made, proposed, taken, iterations, since = [], 0, 0, 0, 0, 0, 0    # running: [request, tokens it still makes]
    for prefill, of in stretches(recs if max_iters is None else recs[:max_iters]):
        rec, iterations = recs[of[0]], iterations + len(of)
        n = int(rec["kind_n"] & 0x7FFFFFFF)
        lens = client.kv_len.tolist()
        if prefill:
            first = int(rec["aux"])
            batch, new = [int(r) for r in queue[first:first + n]], [int(p[r]) for r in queue[first:first + n]]
            rows = list(range(len(running), len(running) + len(batch)))
            if len(batch) != n or sum(new) != int(rec["tokens"]):
                raise RuntimeError(f"iteration {of[0]}: {len(batch)} requests, {sum(new)} tokens; the trace says {n} and {int(rec['tokens'])}")
            for row, tokens in zip(rows, new):
                lens[row] = tokens
            client.resize(torch.tensor(lens, dtype=torch.int32).cuda())
            x = torch.randn((sum(new), heads + 2 * kv_heads, head_dim), generator=gen, device="cuda", dtype=torch.bfloat16)
            _, off, _, _ = client.attend(x, heads, kv_heads, rows, new)
            running += [[r, int(o[r])] for r in batch]
            client.requests = [r for r, _ in running]
            if watch is not None:
                watch(batch, x, off, new, client)
            continue
        if len(running) != n or sum(lens) != int(rec["tokens"]):
            raise RuntimeError(f"iteration {of[0]}: {len(running)} requests, {sum(lens)} tokens; the trace says {n} and {int(rec['tokens'])}")
        left = [len(of)] * n
        while any(left):
            rows = [s for s in range(n) if left[s]]
            new = [min(drafts, left[s] - 1) + 1 for s in rows]
            lens = client.kv_len.tolist()
            for s, k in zip(rows, new):
                lens[s] += k
            client.resize(torch.tensor(lens, dtype=torch.int32).cuda())
            total = sum(new)
            x = torch.randn((total, heads + 2 * kv_heads, head_dim), generator=gen, device="cuda", dtype=torch.bfloat16)
            _, off, kv_len, _ = client.attend(x, heads, kv_heads, rows, new)
            target, draft = probabilities(total, vocab, agree, gen)
            tokens = torch.zeros((total,), dtype=torch.int32, device="cuda")
            tokens[1:] = torch.multinomial(draft, 1, generator=gen)[:-1, 0].to(torch.int32)
            v = hos_verify_drafts(tokens, target, draft, off, torch.rand((total,), generator=gen, device="cuda"),
                                  torch.rand((len(rows),), generator=gen, device="cuda"), kv_len=kv_len)
            if int(v["status"].abs().sum()):
                raise RuntimeError("hos_verify_drafts: status bits set")
            after = client.kv_len.clone()
            after[torch.tensor(rows, dtype=torch.int64).cuda()] = v["new_len"]
            client.resize(after)
            kept = [1 + a for a in v["accepted"].tolist()]
            for s, k in zip(rows, kept):
                left[s] -= k
                running[s][1] -= k
            rounds, made, proposed, taken = rounds + 1, made + sum(kept), proposed + total - len(rows), taken + sum(kept) - len(rows)
            if watch is not None:
                watch([running[s][0] for s in rows], x, off, kept, client)
        stay = [s for s in range(n) if running[s][1]]
        if n - len(stay) != int(recs[of[-1]]["aux"]):
            raise RuntimeError(f"iteration {of[-1]}: {n - len(stay)} requests are done; the trace says {int(recs[of[-1]]['aux'])}")
        if len(stay) < n:
            client.drop(stay)
            running = [running[s] for s in stay]
            client.requests = [r for r, _ in running]
        since += 1
        if compact_every and since % compact_every == 0:
            client.compact()
    torch.cuda.synchronize()
    if any(int(c.status.abs().sum()) for c in client.caches):
        raise RuntimeError("the cache calls reported a problem: status bits set")
    return dict(iterations=iterations, rounds=rounds, tokens=made, drafts=proposed, accepted=taken, most_pages=client.most_pages, pages=client.n_pages)


def main(argv=None):
    from workload import workload
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="c0")
    ap.add_argument("--instance", type=int, default=0)
    ap.add_argument("--client", type=int, default=0)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--agree", type=float, default=0.7)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--heads", type=int, default=64)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--page", type=int, default=128)
    ap.add_argument("--format", default="int8", choices=("same", "e4m3", "int8"))
    ap.add_argument("--layers", type=int, default=1)
    ap.add_argument("--iters", type=int, default=None)
    a = ap.parse_args(argv)
    w = workload(a.workload).subset(a.instance, 1)
    p, o = (x[0] for x in w.lengths())
    recs, queue = client_schedule(p, o, w.n_clients, w.batch_cap, w.kv_budget, w.cost_model, a.client)
    r = replay(p, o, recs, queue, w.batch_cap, w.kv_budget, a.drafts, a.agree, a.vocab, a.heads, a.kv_heads, a.head_dim, a.page, a.format, a.layers,
               max_iters=a.iters)
    r["accepted_share"] = r["accepted"] / r["drafts"] if r["drafts"] else None
    print(json.dumps({"workload": a.workload, "client": a.client, "drafts_a_round": a.drafts, **r}))


if __name__ == "__main__":
    main()
