"""The page and draft operators, one step after the other, in plain Python and 64 bits, for the tests.

Written from include/hos.h; nothing of the package is used here."""
import math

INVALID, PAGES = 4, 16


def held(n, page_size):
    return -(-n // page_size)


def resize(refs, rows, lens, new, page_size, n_entries):
    """rows: full rows of the table (n_entries each).  Returns refs, rows, lens, src, dst, status; -1 after a row's pages."""
    refs, rows, lens = list(refs), [list(r) for r in rows], list(lens)
    n_pages, cap = len(refs), n_entries * page_size
    status, src, dst = [0] * len(rows), [], []
    ok = [0 <= a <= cap and 0 <= b <= cap for a, b in zip(lens, new)]
    for s, good in enumerate(ok):
        if not good:
            status[s] = INVALID
            continue
        for j in range(held(new[s], page_size), held(lens[s], page_size)):
            p = rows[s][j]
            if 0 <= p < n_pages:
                if refs[p] <= 0:
                    status[s] |= INVALID
                refs[p] -= 1
            else:
                status[s] |= INVALID
    free, at, stuck = [p for p, r in enumerate(refs) if r == 0], 0, False
    for s, good in enumerate(ok):
        if not good:
            continue
        have, need = held(lens[s], page_size), held(new[s], page_size)
        if new[s] <= lens[s]:
            rows[s] = rows[s][:need] + [-1] * (n_entries - need)
            lens[s] = new[s]
            continue
        split = False
        if lens[s] % page_size:
            p = rows[s][have - 1]
            if not 0 <= p < n_pages:
                status[s] |= INVALID
            else:
                split = refs[p] > 1
        takes = need - have + split
        if stuck or at + takes > len(free):
            stuck = True
            status[s] |= PAGES
            rows[s] = rows[s][:have] + [-1] * (n_entries - have)
            continue
        mine = free[at:at + takes]
        at += takes
        for p in mine:
            refs[p] = 1
        kept = rows[s][:have]
        if split:
            src.append(kept[-1])
            dst.append(mine[0])
            refs[kept[-1]] -= 1
            kept[-1] = mine.pop(0)
        rows[s] = kept + mine + [-1] * (n_entries - need)
        lens[s] = new[s]
    return refs, rows, lens, src, dst, status


def fork(refs, rows, lens, parent, page_size, n_entries):
    n_pages, cap = len(refs), n_entries * page_size
    out, out_len, status, kids = [], [], [], [0] * len(rows)
    for s in parent:
        bad = s < -1 or s >= len(rows) or (s >= 0 and not 0 <= lens[s] <= cap)
        n = held(lens[s], page_size) if s >= 0 and not bad else 0
        row = list(rows[s][:n]) if n else []
        out.append(row + [-1] * (n_entries - n))
        out_len.append(lens[s] if s >= 0 and not bad else 0)
        status.append(INVALID if bad or any(not 0 <= p < n_pages for p in row) else 0)
        if s >= 0 and not bad:
            kids[s] += 1
    refs = list(refs)
    for s, row in enumerate(rows):
        if 0 <= lens[s] <= cap:
            for p in row[:held(lens[s], page_size)]:
                if 0 <= p < n_pages:
                    refs[p] += kids[s] - 1
    return refs, out, out_len, status


def compact(refs, rows, lens, page_size, n_entries):
    n_pages, cap = len(refs), n_entries * page_size
    n_live = sum(1 for r in refs if r)
    src = [p for p in range(n_live, n_pages) if refs[p]]
    dst = [p for p in range(n_live) if not refs[p]]
    to, new_refs = dict(zip(src, dst)), list(refs)
    for a, b in to.items():
        new_refs[b], new_refs[a] = refs[a], 0
    out, status = [], []
    for s, row in enumerate(rows):
        if not 0 <= lens[s] <= cap:
            out.append(list(row))
            status.append(INVALID)
            continue
        n = held(lens[s], page_size)
        out.append([to.get(p, p) for p in row[:n]] + [-1] * (n_entries - n))
        status.append(INVALID if any(not 0 <= p < n_pages or (p >= n_live and not refs[p]) for p in row[:n]) else 0)
    return new_refs, out, src, dst, status


def verify(tokens, target, draft, off, u_accept, u_sample, vocab):
    """target, draft: 64-bit CPU tensors (draft may be None).  accepted, next, out, status; out is None where no sequence owns the row, or
    (offsets that descend) two do."""
    import torch

    def counted(row):
        return torch.where((row > 0) & (row < math.inf), row, torch.zeros_like(row))

    def of_draft(row):
        return torch.where(row > 0, row, torch.zeros_like(row))

    n_tok, n_seq = len(tokens), len(off) - 1
    accepted, nxt, out, status, owners = [0] * n_seq, [-1] * n_seq, [None] * n_tok, [0] * n_seq, [0] * n_tok
    for s in range(n_seq):
        a, b = off[s], off[s + 1]
        if a < 0 or b < a or b > n_tok:
            status[s] = INVALID
            continue
        if a == b:
            continue
        k, j = b - a - 1, 0
        while j < k:
            d = tokens[a + j + 1]
            if not 0 <= d < vocab:
                status[s] = INVALID
                break
            p = float(counted(target[a + j, d:d + 1])[0])
            q = 1.0 if draft is None else float(of_draft(draft[a + j, d:d + 1])[0])
            if not u_accept[a + j] * q < p:
                break
            j += 1
        p = counted(target[a + j])
        w = p.clone()
        if j < k:
            if draft is not None:
                w = (p - of_draft(draft[a + j])).clamp_min(0.0)
            elif 0 <= tokens[a + j + 1] < vocab:
                w[tokens[a + j + 1]] = 0.0
            if not bool((w > 0).any()):
                w = p
        pick = -1
        if bool((w > 0).any()):
            c = w.cumsum(0)
            u = u_sample[s]
            beyond = (c > (u * float(c[-1]) if u > 0 else 0.0)).nonzero()
            pick = int(beyond[0]) if len(beyond) else int((w > 0).nonzero()[-1])
        else:
            status[s] |= INVALID
        accepted[s], nxt[s] = j, pick
        for i in range(k + 1):
            out[a + i] = tokens[a + i + 1] if i < j else pick if i == j else -1
            owners[a + i] += 1
    return accepted, nxt, [x if n == 1 else None for x, n in zip(out, owners)], status
