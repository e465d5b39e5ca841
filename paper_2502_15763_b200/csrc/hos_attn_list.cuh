// The work list of an attention call: steps of STEP tokens, in the order (sequence, KV head, tile of ROWS
// rows, step).  Rows of a sequence and KV head are its new tokens times the query heads of the group,
// token by token.  Nothing is stored: a worker finds its place in the list from the lengths alone.
//
// A tile costs a worker more than its steps (queries in, result out), so it counts START steps more: these
// come first and hold no work.  A share that begins among them begins with the tile's first real step,
// one that ends among them ends before the tile.
#pragma once

#include "hos_kv.cuh"

namespace hos {

__device__ __forceinline__ long long warp_scan_i64(long long v) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long w = __shfl_up_sync(FULL, v, d);
        if (lane_id() >= d) v += w;
    }
    return v;
}

template <int ROWS, int STEP, int START> struct AttnList {
    const AttnView& a;
    int min_rows, max_rows;                    // sequences with rows in (min_rows, max_rows] are in the list

    struct Tile { int k0, kb, ke, steps, rows; };   // steps from k0 on; tokens [kb, ke) are seen by some row
    struct Cursor {
        int seq, head, tile, tiles, step;
        int at;                                // where the tile begins in the list, relative to the share's begin
        SeqInfo q;
        Tile t;
    };

    __device__ __forceinline__ Tile tile_of(const SeqInfo& q, int tile) const {
        Tile t;
        const int first = tile * ROWS, total = q.n * a.group;
        t.rows = min(ROWS, total - first);
        const int base = q.len - q.n;
        t.ke = a.causal ? min(q.len, base + by_group(a, first + t.rows - 1) + 1) : q.len;
        t.ke = max(t.ke, 0);
        t.kb = min(first_seen(a, base + by_group(a, first)), t.ke);
        t.k0 = t.kb & ~(STEP - 1);
        t.steps = max(1, (t.ke - t.k0 + STEP - 1) / STEP);
        return t;
    }
    __device__ __forceinline__ int tiles_of(const SeqInfo& q) const { return (q.n * a.group + ROWS - 1) / ROWS; }
    __device__ __forceinline__ bool has(const SeqInfo& q) const {
        const long long r = (long long)q.n * a.group;
        return r > min_rows && r <= max_rows;
    }

    // Length in the list of one KV head of this lane's sequence (called by the whole warp; q.n = 0 for none).  Sequences
    // of more than 16 tiles are summed by all lanes together.
    __device__ __forceinline__ long long steps_of(const SeqInfo& q) const {
        long long sum = 0;
        const int nt = has(q) ? tiles_of(q) : 0;
        if (nt > 0 && nt <= 16)
            for (int t = 0; t < nt; ++t) sum += tile_of(q, t).steps + START;
        for (unsigned big = __ballot_sync(FULL, nt > 16); big; big &= big - 1) {
            const int l = __ffs(big) - 1;
            SeqInfo b;
            b.off = 0;
            b.n = __shfl_sync(FULL, q.n, l);
            b.len = __shfl_sync(FULL, q.len, l);
            const int n = tiles_of(b);
            unsigned long long part = 0;
            for (int t = lane_id(); t < n; t += 32) part += (unsigned long long)(tile_of(b, t).steps + START);
            part = warp_sum_u64(part);
            if (lane_id() == l) sum = (long long)part;
        }
        return sum;
    }
    __device__ __forceinline__ SeqInfo lane_seq(int s, bool flag) const {
        SeqInfo q{0, 0, 0};
        if (s < a.kv.n_seq) q = load_seq(a.kv, s, flag);
        return q;
    }

    // Length of the whole list; `flag`: report sequences with bad offsets or lengths; `mine`: this lane's of the first 32
    // sequences, for locate().
    __device__ __forceinline__ long long total(bool flag, long long& mine) const {
        mine = steps_of(lane_seq(lane_id(), flag));
        long long sum = mine;
        for (int s0 = 32; s0 < a.kv.n_seq; s0 += 32) sum += steps_of(lane_seq(s0 + lane_id(), flag));
        return (long long)warp_sum_u64((unsigned long long)sum) * a.kv.n_kv;
    }

    // The real steps of the cursor's tile below this one belong to a share of `length`.
    __device__ __forceinline__ int end_of(const Cursor& c, int length) const { return min(c.t.steps, length - c.at - START); }
    // To the next tile; false if none of its steps belong to the share.
    __device__ __forceinline__ bool next(Cursor& c, int length) const {
        c.at += START + c.t.steps;
        if (c.at + START >= length) return false;
        c.step = 0;
        if (++c.tile == c.tiles) {
            c.tile = 0;
            if (++c.head == a.kv.n_kv) {
                c.head = 0;
                do {
                    if (++c.seq >= a.kv.n_seq) { c.seq = a.kv.n_seq - 1; break; }
                    c.q = load_seq(a.kv, c.seq, false);
                } while (!has(c.q));
                c.tiles = tiles_of(c.q);
            }
        }
        c.t = tile_of(c.q, c.tile);
        return true;
    }

    // Place number `at` (below the total) of the list; called by the whole warp.
    __device__ __forceinline__ Cursor locate(long long at, long long mine) const {
        Cursor c;
        long long before = 0, per_head = 1;
        c.seq = 0;
        for (int s0 = 0; s0 < a.kv.n_seq; s0 += 32) {
            const long long steps = s0 == 0 ? mine : steps_of(lane_seq(s0 + lane_id(), false));
            const long long scan = warp_scan_i64(steps * a.kv.n_kv);
            const unsigned hit = __ballot_sync(FULL, before + scan > at);
            if (hit) {
                const int l = __ffs(hit) - 1;
                c.seq = s0 + l;
                per_head = __shfl_sync(FULL, steps, l);
                before += __shfl_sync(FULL, scan, l) - per_head * a.kv.n_kv;
                break;
            }
            before += __shfl_sync(FULL, scan, 31);
        }
        c.q = load_seq(a.kv, c.seq, false);
        c.tiles = tiles_of(c.q);
        long long rest = at - before;
        c.head = (int)(rest / per_head);
        rest -= (long long)c.head * per_head;
        c.tile = 0;
        for (int t0 = 0; t0 < c.tiles; t0 += 32) {
            const int steps = t0 + lane_id() < c.tiles ? tile_of(c.q, t0 + lane_id()).steps + START : 0;
            const long long scan = warp_scan_i64(steps);
            const unsigned hit = __ballot_sync(FULL, scan > rest);
            if (hit) {
                const int l = __ffs(hit) - 1;
                c.tile = t0 + l;
                rest -= __shfl_sync(FULL, scan - steps, l);
                break;
            }
            rest -= __shfl_sync(FULL, scan, 31);
        }
        c.t = tile_of(c.q, c.tile);
        c.at = -(int)rest;
        c.step = max(0, (int)rest - START);
        return c;
    }
};

}  // namespace hos
