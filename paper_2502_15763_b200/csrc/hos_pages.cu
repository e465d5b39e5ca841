// The pages of a cache: who holds which, and their contents from one place to another.
//
// The tables (counts, rows, lengths; tens of kilobytes to a few megabytes) are a matter of latency: each of the three kernels is
// three or four phases of dependent reads with a barrier of everybody in between.  So each is one launch by one block, or by one cluster
// of 16 whose barrier is in hardware and whose blocks exchange their sums through shared memory; a barrier through global memory or a
// launch a phase would cost 1-2 us each.  What bounds them: for small states the reads, block barriers and counters of a
// phase (0.6-1.2 us each); for large ones the 16 SMs' own rate (a row's entries 32 at a time, instructions as much as bytes).
// One B200, device time: 16 sequences of 33 entries resized 5.0 us, 128 of 519 with 11,612 pages 9.9, 4 forked into 16 3.4, 128 rows of
// 1,031 reordered 7.4, 136 pages compacted 4.6, 79,796 pages under 256 rows of 1,031 13.8.
// The contents are a matter of bandwidth: each byte once in and once out, 6.6-6.7 TB/s (see k_kv_copy_pages).
#include <algorithm>

#include "hos_cluster.cuh"
#include "hos_kv_kernels.h"
#include "hos_kv.cuh"
#include "hos_pages_kernels.h"

namespace hos {
namespace {

// 256, 512 and 1,024 threads, us: 16 sequences resized 4.9, 5.2, 6.1; 128 9.6, 9.9, 11.2; 4 forked 3.3, 3.4, 3.9; 128 7.5, 7.5, 8.0; 136 pages
// compacted 4.5, 4.6, 5.4; 79,796 15.8, 13.8, 13.8; 256 rows of 1,000 entries grown in place 26, 11, 10.  (A barrier of 1,024 threads takes
// 100-160 cycles, and what all warps do alike adds up.)
constexpr int THREADS = 512, WARPS = THREADS / 32;

struct Range { int first, last; };
// The part of n things that falls to this block.
__device__ __forceinline__ Range block_part(int n) {
    const int each = (n + cluster_size() - 1) / cluster_size(), a = min(cluster_rank() * each, n);
    return Range{a, min(a + each, n)};
}
// The same in whole groups of 32: the k-th group of the pool is one warp's.
__device__ __forceinline__ Range block_part_of_groups(int n) {
    const Range g = block_part((n + 31) / 32);
    return Range{min(32 * g.first, n), min(32 * g.last, n)};
}
// A warp's part of the block's pages: whole groups of 32 but for the last one.
__device__ __forceinline__ Range warp_part(Range block) {
    const int each = ((block.last - block.first + WARPS - 1) / WARPS + 31) & ~31, a = min(block.first + warp_id() * each, block.last);
    return Range{a, min(a + each, block.last)};
}
// Of a block's warps, the one of this lane's number.
__device__ __forceinline__ int of_lane(const int* of_warps) { return lane_id() < WARPS ? of_warps[lane_id()] : 0; }
__device__ __forceinline__ unsigned lanes_before() { return (1u << lane_id()) - 1u; }

// Numbers of pages are added up in 32 bits.  What sequences ask for may be more than that holds; every sum stops at PLENTY, which no pool has
// (min(a + b, PLENTY) is associative for numbers from 0 to PLENTY, and 32 of them are below 2^31).
constexpr int PLENTY = 1 << 25;
__device__ __forceinline__ int sum_of_warp(int v) { return (int)__reduce_add_sync(FULL, (unsigned)v); }
__device__ __forceinline__ int sum_before_lane(int v) {
    int s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(FULL, s, d);
        if (lane_id() >= d) s = min(s + o, PLENTY);
    }
    s = __shfl_up_sync(FULL, s, 1);
    return lane_id() == 0 ? 0 : s;
}

// What the blocks tell one another: one warp of each writes its sums to all the others' boards before a barrier of the cluster (read from
// theirs after it, by all warps of all blocks at once, took 2 us).
constexpr int MOST_BLOCKS = 16;
struct Shares { int4 before, all; };
__device__ __forceinline__ void tell(int4* board, const int4& mine) {
    if (lane_id() < cluster_size()) write_to_block(board + cluster_rank(), lane_id(), mine);
}
__device__ __forceinline__ Shares heard(const int4* board) {
    const int rank = cluster_rank(), n = cluster_size();
    const int4 v = lane_id() < n ? board[lane_id()] : make_int4(0, 0, 0, 0);
    if (n == 1) return Shares{make_int4(0, 0, 0, 0), board[0]};
    Shares s;
    const bool b = lane_id() < rank;
    s.all = make_int4(min(sum_of_warp(v.x), PLENTY), sum_of_warp(v.y), sum_of_warp(v.z), sum_of_warp(v.w));
    s.before = make_int4(min(sum_of_warp(b ? v.x : 0), PLENTY), sum_of_warp(b ? v.y : 0), sum_of_warp(b ? v.z : 0), sum_of_warp(b ? v.w : 0));
    return s;
}

__device__ __forceinline__ bool is_page(const PagesView& p, int page) { return (unsigned)page < (unsigned)p.n_pages; }
__device__ __forceinline__ bool is_length(const PagesView& p, int len) { return len >= 0 && len <= (long long)p.max_pages * p.page_size; }
__device__ __forceinline__ int pages_of(const PagesView& p, int len) { return (int)(((unsigned)len + (unsigned)p.page_size - 1u) / (unsigned)p.page_size); }
__device__ __forceinline__ void flag(const PagesView& p, int s) {
    if (p.status) atomicOr(p.status + s, HOS_ST_INVALID);
}

// A warp's pages in groups of 32, as masks of those whose count is zero.  The loads of AHEAD groups are on their way at once; the masks
// of the first 32 groups stay with the lanes, lane g has group g: a pool of up to 16,384 pages a block is read once, and what is
// counted in it takes one step instead of one a group (a group is some 50 instructions of all warps).
constexpr int AHEAD = 8;
struct FreeMasks {
    Range part;
    unsigned kept;                                     // of group lane_id()
    __device__ __forceinline__ int group_first(int g) const { return part.first + 32 * g; }
    __device__ __forceinline__ unsigned load(const int32_t* refs, int g) const {
        const int i = group_first(g) + lane_id();
        return __ballot_sync(FULL, i < part.last && __ldcg(refs + i) == 0);
    }
    __device__ __forceinline__ void read(const int32_t* refs) {
        kept = 0;
        for (int g0 = 0; g0 < 32 && group_first(g0) < part.last; g0 += AHEAD) {
            int r[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int i = group_first(g0 + k) + lane_id();
                r[k] = i < part.last ? __ldcg(refs + i) : 1;
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const unsigned m = __ballot_sync(FULL, r[k] == 0);
                if (g0 + k == lane_id()) kept = m;
            }
        }
    }
    // Sum over the groups of f(first page, mask).
    template <typename F> __device__ __forceinline__ int sum(const int32_t* refs, F&& f) const {
        const int mine = group_first(lane_id());
        int n = sum_of_warp(mine < part.last ? f(mine, kept) : 0);
        for (int g = 32; group_first(g) < part.last; ++g) n += f(group_first(g), load(refs, g));
        return n;
    }
    // f(first page, mask) by the whole warp, group by group, until it returns false
    template <typename F> __device__ __forceinline__ void each(const int32_t* refs, F&& f) const {
        for (int g = 0; group_first(g) < part.last; ++g)
            if (!f(group_first(g), g < 32 ? __shfl_sync(FULL, kept, g) : load(refs, g))) return;
    }
    __device__ __forceinline__ unsigned there(int i0) const { return part.last - i0 >= 32 ? FULL : (1u << (part.last - i0)) - 1u; }
};

__device__ __forceinline__ void copy_counts(const PagesView& p, Range pages) {
    if (p.refs == p.refs_in) return;
    for (int i0 = pages.first + (int)threadIdx.x; i0 < pages.last; i0 += AHEAD * THREADS) {
        int r[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i0 + k * THREADS < pages.last) r[k] = p.refs_in[i0 + k * THREADS];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i0 + k * THREADS < pages.last) p.refs[i0 + k * THREADS] = r[k];
    }
}

// 32 x EACH entries of a row from `first` on, by a warp: all loads before the stores (the compiler cannot know that the tables are apart).
constexpr int EACH = 8, PIECE = 32 * EACH;
struct Piece { int e[EACH]; };
__device__ __forceinline__ Piece load_piece(const int32_t* row, int first, int last) {
    Piece x;
    if (first >= last) {                               // behind what a row holds: most pieces of a wide table
#pragma unroll
        for (int k = 0; k < EACH; ++k) x.e[k] = -1;
        return x;
    }
    const int left = last - first - lane_id();
    const int32_t* at = row + (first + lane_id());
#pragma unroll
    for (int k = 0; k < EACH; ++k) x.e[k] = 32 * k < left ? at[32 * k] : -1;
    return x;
}
__device__ __forceinline__ void store_piece(int32_t* row, int first, int last, const Piece& x) {
    const int left = last - first - lane_id();
    int32_t* at = row + (first + lane_id());
#pragma unroll
    for (int k = 0; k < EACH; ++k)
        if (32 * k < left) at[32 * k] = x.e[k];
}

// Part of a row to be gone through: of sequence `seq`, entries first to last - 1.
struct RowWork { int seq, first, last, from; };
// A list of row parts that the threads of a block make together and its warps go through, piece by piece: the next piece's entries
// are on their way while one is worked on, the first already before a barrier of the blocks where there is one in between.
struct RowList {
    RowWork row[THREADS];
    int n, pieces;                                     // row parts; pieces of the longest (at least)

    __device__ __forceinline__ void begin(int at_least) {
        if (threadIdx.x == 0) n = 0, pieces = at_least;
        __syncthreads();
    }
    __device__ __forceinline__ void add(const RowWork& r) {
        row[atomicAdd(&n, 1)] = r;
        const int need = (r.last - r.first + PIECE - 1) / PIECE;
        if (need > 1) atomicMax(&pieces, need);
    }
};
struct Cursor { int r, c; Piece next; };               // of a warp: its next piece, c of row part r
// load(row part, first entry)
template <typename L> __device__ __forceinline__ Cursor first_piece(const RowList& list, L&& load) {
    __syncthreads();
    Cursor at;
    const int pieces = list.pieces;
    at.r = pieces ? warp_id() / pieces : list.n;
    at.c = warp_id() - at.r * pieces;
    if (at.r < list.n) at.next = load(list.row[at.r], list.row[at.r].first + at.c * PIECE);
    return at;
}
// work(row part, first entry, piece)
template <typename L, typename W> __device__ __forceinline__ void all_pieces(const RowList& list, Cursor at, L&& load, W&& work) {
    const int rows = list.n, pieces = list.pieces;
    if (at.r >= rows) return;
    const int step_rows = WARPS / pieces, step = WARPS - step_rows * pieces;
    RowWork now = list.row[at.r];
    while (true) {
        const int j = now.first + at.c * PIECE;
        const RowWork then = now;
        const Piece x = at.next;
        at.r += step_rows;
        at.c += step;
        if (at.c >= pieces) at.c -= pieces, ++at.r;
        const bool more = at.r < rows;
        if (more) {
            now = list.row[at.r];
            at.next = load(now, now.first + at.c * PIECE);
        }
        work(then, j, x);
        if (!more) return;
    }
}

// ---- resize ------------------------------------------------------------------------------------------------------------
constexpr int GROWS = 1 << 30, SPLITS = 1 << 29, TAKES = SPLITS - 1;
constexpr int LACKING = 1 << 26;                       // beside a number of free pages, of each of up to 16 blocks

struct Change {
    int old, now;
    bool valid;
    bool inside;               // it grows from the inside of `page`, as the table has it (looked at late: it is still on its way)
    int page;
};
__device__ __forceinline__ Change change_of(const PagesView& p, int s) {
    Change c;
    c.old = p.len_in[s];
    c.now = p.change[s];
    c.valid = is_length(p, c.old) && is_length(p, c.now);
    const unsigned at = (unsigned)c.old / (unsigned)p.page_size;
    c.inside = c.valid && c.now > c.old && at * (unsigned)p.page_size != (unsigned)c.old;
    c.page = c.inside ? p.table_in[(long long)s * p.in_stride + at] : -1;
    return c;
}

// Why the result is that of one sequence after the other: counts only fall in the first step, so that which of the pages that
// sequences grow from are shared is known after it; of a page's holders that grow, all get a copy but the last of them, if nobody else
// holds it (two atomics a holder: how many, and the last); then sums over the sequences give each its place among the free pages, taken
// by number, and the first that is short is the first whose sum is beyond them, as all sums after it are.
__global__ void __launch_bounds__(THREADS, 1) k_kv_resize(const __grid_constant__ PagesView p) {
    __shared__ int4 board[MOST_BLOCKS];
    __shared__ int of_warp[3][WARPS];
    __shared__ bool lacking;                           // something was given up here that is no page, or that nobody held any more
    __shared__ RowList stay, go;
    pdl_launch_dependents();
    pdl_wait();
    const Range seqs = block_part(p.n_seq), pages = block_part(p.n_pages);
    const int tid = (int)threadIdx.x;
    const bool in_place = p.table == p.table_in;
    auto old_row = [&](const RowWork& r, int j) { return load_piece(p.table_in + (long long)r.seq * p.in_stride, j, r.last); };
    auto keep = [&](const RowWork& r, int j, const Piece& x) { store_piece(p.table + (long long)r.seq * p.out_stride, j, p.max_pages, x); };
    auto give_up = [&](const RowWork& r, int j, const Piece& x) {
        int was[EACH];                                 // all on their way before the first is looked at
#pragma unroll
        for (int k = 0; k < EACH; ++k) was[k] = is_page(p, x.e[k]) ? atomicSub(p.refs + x.e[k], 1) : 32 * k < r.last - j - lane_id() ? 0 : 1;
        bool bad = false;
#pragma unroll
        for (int k = 0; k < EACH; ++k) bad |= was[k] <= 0;
        if (bad) lacking = true;
    };
    auto list_of_gone = [&](const Change& c, int s) {
        if (c.valid && c.now < c.old) {
            const int have = pages_of(p, c.old), need = pages_of(p, c.now);
            if (need < have) go.add(RowWork{s, need, have, 0});
        }
    };
    // the new counts begin as the old ones; what is known of shared pages that are grown from, as nothing; rows of tables apart are copied
    // as far as they stay
    Change first = {0, 0, false, false, -1};           // of this thread's first sequence
    if (seqs.first + tid < seqs.last) first = change_of(p, seqs.first + tid);
    copy_counts(p, pages);
    if (tid == 0) lacking = false;
    go.begin(1);
    for (int s0 = seqs.first; s0 < seqs.last; s0 += THREADS) {
        stay.begin((p.max_pages + PIECE - 1) / PIECE);
        const int s = s0 + tid;
        Change c = first;
        if (s0 > seqs.first) c = s < seqs.last ? change_of(p, s) : Change{0, 0, false, false, -1};
        if (s < seqs.last) {
            if (!in_place) stay.add(RowWork{s, 0, c.valid ? pages_of(p, min(c.old, c.now)) : p.max_pages, 0});
            if (s0 == seqs.first) list_of_gone(c, s);
            p.src[s] = p.dst[s] = -1;
        }
        Cursor kept;
        if (!in_place) kept = first_piece(stay, old_row);
        const int holders = is_page(p, c.page) && s < seqs.last ? p.refs_in[c.page] : 0;
        if (!in_place) all_pieces(stay, kept, old_row, keep);
        if (s < seqs.last) {
            if (p.status) p.status[s] = c.valid && (!c.inside || is_page(p, c.page)) ? 0 : HOS_ST_INVALID;
            if (holders > 1) p.growers[c.page] = 0, p.latest[c.page] = -1;
        }
        if (s0 + THREADS < seqs.last) __syncthreads();
    }
    Cursor gone = first_piece(go, old_row);
    cluster_or_block_sync();
    // pages given up; how many sequences grow from the inside of a shared page, and the last of them
    for (int s0 = seqs.first; s0 < seqs.last; s0 += THREADS) {
        const int s = s0 + tid;
        if (s0 > seqs.first) {
            __syncthreads();
            go.begin(1);
        }
        if (s < seqs.last) {
            const Change c = s0 == seqs.first ? first : change_of(p, s);
            if (is_page(p, c.page) && __ldcg(p.refs_in + c.page) > 1) {
                atomicAdd(p.growers + c.page, 1);
                atomicMax(p.latest + c.page, s);
            }
            if (s0 > seqs.first) list_of_gone(c, s);
        }
        if (s0 > seqs.first) gone = first_piece(go, old_row);
        all_pieces(go, gone, old_row, give_up);
    }
    cluster_or_block_sync();
    // how many pages are free; what each sequence takes, with sums in order
    int holders = 0, growers = 0, latest = 0;          // of the page that this thread's first sequence grows from
    if (is_page(p, first.page)) {
        holders = __ldcg(p.refs + first.page);
        growers = __ldcg(p.growers + first.page);      // nothing, where there is but one holder: not looked at then
        latest = __ldcg(p.latest + first.page);
    }
    FreeMasks masks{warp_part(pages), 0};
    masks.read(p.refs);
    const int n_free = masks.sum(p.refs, [&](int, unsigned m) { return __popc(m); });
    if (lane_id() == 0) of_warp[2][warp_id()] = n_free;
    int sum_takes = 0, sum_splits = 0;
    ResizePlan of_first = {0, 0, 0};
    for (int s0 = seqs.first; s0 < seqs.last; s0 += THREADS) {
        const int s = s0 + tid;
        ResizePlan plan = {0, 0, 0};
        if (s < seqs.last) {
            const Change c = s0 == seqs.first ? first : change_of(p, s);
            if (c.valid && c.now > c.old) {
                plan.takes = GROWS | min(pages_of(p, c.now) - pages_of(p, c.old), PLENTY - 1);
                if (s0 > seqs.first && is_page(p, c.page)) {
                    holders = __ldcg(p.refs + c.page);
                    growers = __ldcg(p.growers + c.page);
                    latest = __ldcg(p.latest + c.page);
                }
                if (is_page(p, c.page) && holders > 1 && !(growers == holders && latest == s)) plan.takes = (plan.takes + 1) | SPLITS;
            }
        }
        const unsigned split = __ballot_sync(FULL, plan.takes & SPLITS);
        const int before = sum_before_lane(plan.takes & TAKES), all = min(before + (plan.takes & TAKES), PLENTY);
        if (lane_id() == 31) of_warp[0][warp_id()] = all, of_warp[1][warp_id()] = __popc(split);
        __syncthreads();
        const int t = of_lane(of_warp[0]), u = of_lane(of_warp[1]);
        const bool b = lane_id() < warp_id();
        plan.before = min(sum_takes + min(sum_of_warp(b ? t : 0), PLENTY) + before, PLENTY);
        plan.splits_before = sum_splits + sum_of_warp(b ? u : 0) + __popc(split & lanes_before());
        sum_takes = min(sum_takes + min(sum_of_warp(t), PLENTY), PLENTY);
        sum_splits += sum_of_warp(u);
        if (s0 == seqs.first) of_first = plan;
        else if (s < seqs.last) p.plan[s] = plan;
        if (s0 + THREADS < seqs.last) __syncthreads();
    }
    __syncthreads();
    const int free_of_lane = of_lane(of_warp[2]);
    if (warp_id() == 0) {
        const int all = sum_of_warp(free_of_lane);
        tell(board, make_int4(sum_takes, sum_splits, all + (lacking ? LACKING : 0), 0));
    }
    cluster_or_block_sync();
    const Shares shares = heard(board);
    const int wanted = shares.all.x, free = shares.all.z & (LACKING - 1);
    const bool anybody_lacking = shares.all.z >= LACKING;
    if (tid == 0 && cluster_rank() == 0 && wanted <= free) *p.count = shares.all.y;
    // Rows in place lose what was given up.  And if something was given up in vain, everybody who gave up a page whose count has come out below
    // zero is told: which of its holders came last in time says nothing.  (Entry by entry, since little code counts for more than its
    // speed: the instructions come from memory, too.  Cleared before the barrier, with the counts, it took 0.1-0.2 us less.)
    if (in_place || anybody_lacking)
        for (int s0 = seqs.first; s0 < seqs.last; s0 += THREADS) {
            if (seqs.last - seqs.first > THREADS) {    // else the list is still that of the only chunk
                __syncthreads();
                go.begin(1);
                if (s0 + tid < seqs.last) list_of_gone(s0 == seqs.first ? first : change_of(p, s0 + tid), s0 + tid);
                __syncthreads();
            }
            for (int i = warp_id(); i < go.n; i += WARPS) {
                const RowWork r = go.row[i];
#pragma unroll 1
                for (int j = r.first + lane_id(); j < r.last; j += 32) {
                    if (anybody_lacking) {
                        const int page = p.table_in[(long long)r.seq * p.in_stride + j];
                        if (!is_page(p, page) || __ldcg(p.refs + page) < 0) flag(p, r.seq);
                    }
                    if (in_place) p.table[(long long)r.seq * p.out_stride + j] = -1;
                }
            }
        }
    // the free pages in order, as many as are taken
    int at = (shares.before.z & (LACKING - 1)) + sum_of_warp(lane_id() < warp_id() ? free_of_lane : 0);
    if (at < wanted)
        masks.each(p.refs, [&](int i0, unsigned m) {
            const int k = at + __popc(m & lanes_before());
            if ((m >> lane_id() & 1u) && k < wanted) p.queue[k] = i0 + lane_id();
            at += __popc(m);
            return at < wanted;
        });
    cluster_or_block_sync();
    // lengths, and the pages that rows get
    auto taken = [&](const RowWork& r, int j) { return load_piece(p.queue + r.from, j, r.last); };
    for (int s0 = seqs.first; s0 < seqs.last; s0 += THREADS) {
        go.begin(1);
        const int s = s0 + tid;
        if (s < seqs.last) {
            const Change c = s0 == seqs.first ? first : change_of(p, s);
            const ResizePlan plan = s0 == seqs.first ? of_first : p.plan[s];
            const int base = min(shares.before.x + plan.before, PLENTY), takes = plan.takes & TAKES, splits = shares.before.y + plan.splits_before;
            const bool short_of = (plan.takes & GROWS) && base + takes > free;
            if (short_of) {
                // the first sequence whose pages are not there: the splits before it are those that are made
                if (base <= free) *p.count = splits;
                if (p.status) atomicOr(p.status + s, HOS_ST_PAGES);
            } else if (takes) {
                const int split = (plan.takes & SPLITS) != 0, have = pages_of(p, c.old);
                go.add(RowWork{s, have - split, pages_of(p, c.now), base - (have - split)});
                if (split) {
                    atomicSub(p.refs + c.page, 1);
                    p.src[splits] = c.page;
                    p.dst[splits] = __ldcg(p.queue + base);
                }
            }
            p.len[s] = c.valid && !short_of ? c.now : c.old;
        }
        all_pieces(go, first_piece(go, taken), taken, [&](const RowWork& r, int j, const Piece& x) {
#pragma unroll
            for (int k = 0; k < EACH; ++k)
                if (x.e[k] >= 0) p.refs[x.e[k]] = 1;
            store_piece(p.table + (long long)r.seq * p.out_stride, j, r.last, x);
        });
        if (s0 + THREADS < seqs.last) __syncthreads();
    }
}

// ---- fork --------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ int parent_of(const PagesView& p, int i, int* len) {
    const int s = p.change[i];
    *len = 0;
    if (s == -1) return -1;
    if (s < 0 || s >= p.n_seq) return -2;
    const int n = p.len_in[s];
    if (!is_length(p, n)) return -2;
    *len = n;
    return s;
}

// A row of s is read once for each of its children, and once more, with an atomic an entry, if it has not exactly one.
__global__ void __launch_bounds__(THREADS, 1) k_kv_fork(const __grid_constant__ PagesView p) {
    __shared__ int children[THREADS];
    __shared__ RowList list, held;
    pdl_launch_dependents();
    pdl_wait();
    const Range seqs = block_part(p.n_seq), outs = block_part(p.n_out);
    const int tid = (int)threadIdx.x;
    auto row_of_parent = [&](const RowWork& r, int j) { return load_piece(p.table_in + (long long)r.from * p.in_stride, j, r.last); };
    auto row = [&](const RowWork& r, int j) { return load_piece(p.table_in + (long long)r.seq * p.in_stride, j, r.last); };
    copy_counts(p, block_part(p.n_pages));
    for (int i0 = outs.first; i0 < outs.last; i0 += THREADS) {
        list.begin((p.max_pages + PIECE - 1) / PIECE);
        const int i = i0 + tid;
        if (i < outs.last) {
            int len;
            const int s = parent_of(p, i, &len);
            p.len[i] = len;
            if (p.status) p.status[i] = s == -2 ? HOS_ST_INVALID : 0;
            list.add(RowWork{i, 0, pages_of(p, len), s});
        }
        all_pieces(list, first_piece(list, row_of_parent), row_of_parent, [&](const RowWork& r, int j, const Piece& x) {
            bool bad = false;
#pragma unroll
            for (int k = 0; k < EACH; ++k) bad |= 32 * k < r.last - j - lane_id() && !is_page(p, x.e[k]);
            if (bad) flag(p, r.seq);
            store_piece(p.table + (long long)r.seq * p.out_stride, j, p.max_pages, x);
        });
        if (i0 + THREADS < outs.last) __syncthreads();
    }
    // the counts: every block looks through all parents for its own sequences' children
    for (int s0 = seqs.first; s0 == seqs.first || s0 < seqs.last; s0 += THREADS) {
        if (s0 > seqs.first) __syncthreads();
        children[tid] = 0;
        held.begin(1);
        for (int i0 = tid; i0 < p.n_out; i0 += AHEAD * THREADS) {
            int s[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) s[k] = i0 + k * THREADS < p.n_out ? p.change[i0 + k * THREADS] : -1;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (s[k] >= s0 && s[k] < min(s0 + THREADS, seqs.last)) atomicAdd(children + s[k] - s0, 1);
        }
        const int len = s0 + tid < seqs.last ? p.len_in[s0 + tid] : -1;
        __syncthreads();
        const int more = children[tid] - 1;
        if (is_length(p, len) && len > 0 && more != 0) held.add(RowWork{s0 + tid, 0, pages_of(p, len), more});
        const Cursor at = first_piece(held, row);
        if (s0 == seqs.first) cluster_or_block_sync();         // the counts have been copied
        all_pieces(held, at, row, [&](const RowWork& r, int, const Piece& x) {
#pragma unroll
            for (int k = 0; k < EACH; ++k)
                if (is_page(p, x.e[k])) atomicAdd(p.refs + x.e[k], r.from);
        });
    }
}

// ---- compact -----------------------------------------------------------------------------------------------------------
// With n pages in use there are as many of them from n on as there are free ones below n; both are numbered in order, and the k-th goes to the
// k-th.  A table entry finds its new page by two reads: its place among the moves, and where that one goes.  Where it stays, the first read is of
// its group's mask of free pages instead: whether the page is in use has to be known of every entry, and the counts change under a call in place.
__global__ void __launch_bounds__(THREADS, 1) k_kv_compact(const __grid_constant__ PagesView p) {
    __shared__ int4 live[MOST_BLOCKS], others[MOST_BLOCKS];
    __shared__ int of_warp[3][WARPS];
    __shared__ RowList list;
    pdl_launch_dependents();
    pdl_wait();
    cluster_begun_arrive();
    const Range seqs = block_part(p.n_seq), pages = block_part_of_groups(p.n_pages);
    const int tid = (int)threadIdx.x;
    const bool in_place = p.table == p.table_in;
    auto row = [&](const RowWork& r, int j) { return load_piece(p.table_in + (long long)r.seq * p.in_stride, j, r.last); };
    auto list_row = [&](int s, int len) {
        const bool valid = is_length(p, len);
        if (valid || !in_place) list.add(RowWork{s, 0, valid ? pages_of(p, len) : p.max_pages, valid});
    };
    FreeMasks masks{warp_part(pages), 0};
    masks.read(p.refs_in);
    const int n = masks.sum(p.refs_in, [&](int i0, unsigned m) { return __popc(masks.there(i0) & ~m); });
    if (lane_id() == 0) of_warp[0][warp_id()] = n;
    copy_counts(p, pages);
    const int first_len = seqs.first + tid < seqs.last ? p.len_in[seqs.first + tid] : 0;
    for (int s = seqs.first + tid; s < seqs.last; s += THREADS)
        if (p.status) p.status[s] = is_length(p, s == seqs.first + tid ? first_len : p.len_in[s]) ? 0 : HOS_ST_INVALID;
    cluster_begun_wait();
    __syncthreads();
    if (warp_id() == 0) {
        const int all = sum_of_warp(of_lane(of_warp[0]));
        tell(live, make_int4(0, 0, 0, all));
    }
    cluster_or_block_sync();
    const int n_live = heard(live).all.w;
    // pages in use behind the first n_live, and free ones among those: as many of the one as of the other
    auto behind = [&](int i0) { return i0 >= n_live ? FULL : n_live - i0 >= 32 ? 0u : FULL << (n_live - i0); };
    const int late = masks.sum(p.refs_in, [&](int i0, unsigned m) { return __popc(masks.there(i0) & ~m & behind(i0)); });
    const int hole = masks.sum(p.refs_in, [&](int i0, unsigned m) { return __popc(m & ~behind(i0)); });
    if (lane_id() == 0) of_warp[1][warp_id()] = late, of_warp[2][warp_id()] = hole;
    __syncthreads();
    const int late_of_lane = of_lane(of_warp[1]), hole_of_lane = of_lane(of_warp[2]);
    if (warp_id() == 0) {
        const int a = sum_of_warp(late_of_lane), b = sum_of_warp(hole_of_lane);
        tell(others, make_int4(0, a, b, 0));
    }
    cluster_or_block_sync();
    const Shares shares = heard(others);
    const bool b = lane_id() < warp_id();
    int late_at = shares.before.y + sum_of_warp(b ? late_of_lane : 0), hole_at = shares.before.z + sum_of_warp(b ? hole_of_lane : 0);
    const int count = shares.all.y;
    masks.each(p.refs_in, [&](int i0, unsigned m) {
        const int i = i0 + lane_id();
        const unsigned a = masks.there(i0) & ~m & behind(i0), h = m & ~behind(i0), me = 1u << lane_id();
        const int k = late_at + __popc(a & lanes_before());
        if (a & me) p.src[k] = i;
        if (h & me) p.dst[hole_at + __popc(h & lanes_before())] = i;
        if (i >= n_live && i < masks.part.last) p.growers[i] = a & me ? k : -1;
        if (i0 < n_live && lane_id() == 0) p.growers[i0 >> 5] = (int)m;        // below the places: i0 / 32 < n_live
        late_at += __popc(a);
        hole_at += __popc(h);
        return true;
    });
    for (int i = max(count, pages.first) + tid; i < pages.last; i += THREADS) p.src[i] = p.dst[i] = -1;
    if (tid == 0 && cluster_rank() == 0) *p.count = count;
    list.begin(in_place ? 1 : (p.max_pages + PIECE - 1) / PIECE);
    if (seqs.first + tid < seqs.last) list_row(seqs.first + tid, first_len);
    Cursor at = first_piece(list, row);
    cluster_or_block_sync();
    // a move, whose count goes along: its numbers come while the rows are worked on
    const int step = cluster_size() * THREADS, move = cluster_rank() * THREADS + tid;
    int from = 0, to = 0;
    if (move < count) from = __ldcg(p.src + move), to = __ldcg(p.dst + move);
    for (int s0 = seqs.first; s0 < seqs.last; s0 += THREADS) {
        if (s0 > seqs.first) {
            __syncthreads();
            list.begin(in_place ? 1 : (p.max_pages + PIECE - 1) / PIECE);
            if (s0 + tid < seqs.last) list_row(s0 + tid, p.len_in[s0 + tid]);
            at = first_piece(list, row);
        }
        all_pieces(list, at, row, [&](const RowWork& r, int j, Piece x) {
            if (r.from && j < r.last) {
                int word[EACH];                        // its place among the moves (-1: free), or which pages of its group are free
                bool bad = false;
#pragma unroll
                for (int k = 0; k < EACH; ++k) word[k] = is_page(p, x.e[k]) ? p.growers[x.e[k] < n_live ? x.e[k] >> 5 : x.e[k]] : -1;
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    const bool stays = x.e[k] < n_live, wrong = stays ? word[k] >> (x.e[k] & 31) & 1 : word[k] < 0;
                    bad |= wrong && 32 * k < r.last - j - lane_id();
                    if (!stays && word[k] >= 0) x.e[k] = __ldcg(p.dst + word[k]);
                }
                if (bad) flag(p, r.seq);
            }
            store_piece(p.table + (long long)r.seq * p.out_stride, j, in_place ? r.last : p.max_pages, x);
        });
    }
    for (int k = move; k < count; k += step) {
        if (k > move) from = __ldcg(p.src + k), to = __ldcg(p.dst + k);
        const int refs = p.refs_in[from];
        p.refs[to] = refs;
        p.refs[from] = 0;
    }
}

// ---- copy --------------------------------------------------------------------------------------------------------------
// HBM is the bound: 676 MB of e4m3 pages (2,501 moves of 33 KB a side, four layers) 102 us, 1.34 GB of bf16 ones 200 us, 6.6 and 6.7 TB/s, as
// fast as a plain copy of that size.
// A unit is 16 KB of a page's keys or values, with the scales of the 8-bit ones (1/16 or 1/32 of that); a thread has four
// accesses of 16 bytes on the way.  Units are counted on by a block's stride in three digits (unit of a page, move, layer), without divisions.
constexpr int COPY_THREADS = 256, COPY_UNIT = COPY_THREADS * 64;

// The layers come as kernel parameters.  Room for 128 of them, 12 KB, costs a call 2.5 us on the host more than for 4.
template <int LAYERS> struct CopyView {
    CopyCall call;
    CopyLayer layer[LAYERS];
};

template <int LAYERS> __global__ void __launch_bounds__(COPY_THREADS) k_kv_copy_pages(const __grid_constant__ CopyView<LAYERS> view) {
    const CopyCall& c = view.call;
    pdl_launch_dependents();
    pdl_wait();
    const int n = c.count ? max(0, min(c.n_moves, __ldg(c.count))) : c.n_moves;
    if (n == 0) return;
    const int units = 2 * ((c.bytes + COPY_UNIT - 1) / COPY_UNIT);
    const int step = (int)gridDim.x % units, step_moves = (int)gridDim.x / units % n, step_layers = (int)gridDim.x / units / n;
    int unit = (int)blockIdx.x % units, move = (int)blockIdx.x / units % n, layer = (int)blockIdx.x / units / n;
    const int scale_at = (int)threadIdx.x * 16;
    while (layer < c.n_layers) {
        const int from = __ldg(c.src + move), to = __ldg(c.dst + move);
        const CopyLayer& l = view.layer[layer];
        if ((unsigned)from < (unsigned)c.from_pages && (unsigned)to < (unsigned)c.to_pages) {
            const int v = unit & 1, at = (unit >> 1) * COPY_UNIT;              // keys and values in turn
            const int left = c.bytes - at - (int)threadIdx.x * 16;
            const unsigned char* a = l.from[v] + from * l.from_stride[0] + (at + (int)threadIdx.x * 16);
            unsigned char* b = l.to[v] + to * l.to_stride[0] + (at + (int)threadIdx.x * 16);
            uint4 x[4], s;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i * COPY_THREADS * 16 < left) x[i] = __ldg(reinterpret_cast<const uint4*>(a + i * COPY_THREADS * 16));
            const int scale_first = at >> c.scale_shift, scale_last = min(c.scale_bytes, (at + COPY_UNIT) >> c.scale_shift);
            const bool scale = scale_first + scale_at < scale_last;
            if (scale) s = __ldg(reinterpret_cast<const uint4*>(l.from[2 + v] + from * l.from_stride[1] + scale_first + scale_at));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i * COPY_THREADS * 16 < left) *reinterpret_cast<uint4*>(b + i * COPY_THREADS * 16) = x[i];
            if (scale) *reinterpret_cast<uint4*>(l.to[2 + v] + to * l.to_stride[1] + scale_first + scale_at) = s;
        } else if (threadIdx.x == 0 && unit == 0 && layer == 0 && c.status) {
            atomicOr(c.status + move, HOS_ST_INVALID);
        }
        unit += step;
        move += step_moves;
        layer += step_layers;
        if (unit >= units) unit -= units, ++move;
        if (move >= n) move -= n, ++layer;
    }
}

// A small state by one block, whose own barrier is enough; any other by a cluster of 16, the most there are (its barriers take 0.5-1 us
// each, one block 0.1-0.15 us for a thousand entries).  One block, 2, 4, 8, 16, us: 16 sequences of 33 entries 5.0, 6.4, 6.5, 6.6, 6.8, of 1,024
// (16,384 entries, mostly empty) 6.0, 7.1, 6.9, 6.6, 6.8 (resize); 128 of 519, 11,612 pages 18, 15, 11, 10, 9.9 (resize); 4 forked into 16 3.4, 3.8, 3.7,
// 3.7, 3.8, 128 of 1,031 38, 23, 14, 9.8, 7.4 (fork); 136 pages 4.6, 5.6, 5.6, 5.7, 5.8, 79,796 172, 82, 38, 20, 14 (compact).  A resize in
// place does not go through the entries that stay, but is counted by them all the same: 16 rows of 1,024 take 6.5 us in place, of 33 4.8.
constexpr long long SMALL_STATE = 8192;
template <void (*KERNEL)(PagesView)> cudaError_t launch_tables(const char* name, const PagesView& p, cudaStream_t st) {
    const long long rows = p.n_seq > p.n_out ? p.n_seq : p.n_out;
    const int blocks = p.n_pages + rows * p.max_pages <= SMALL_STATE ? 1 : MOST_BLOCKS;
    static std::atomic<unsigned long long> asked{0};
    if (blocks > 8) {
        const cudaError_t e = ask_for_large_clusters(reinterpret_cast<const void*>(KERNEL), asked);
        if (e != cudaSuccess) return e;
    }
    return launch_clusters(name, KERNEL, blocks, blocks, THREADS, st, p);
}

}  // namespace

cudaError_t launch_kv_resize(const PagesView& p, cudaStream_t st) { return launch_tables<k_kv_resize>("k_kv_resize", p, st); }
cudaError_t launch_kv_fork(const PagesView& p, cudaStream_t st) { return launch_tables<k_kv_fork>("k_kv_fork", p, st); }
cudaError_t launch_kv_compact(const PagesView& p, cudaStream_t st) { return launch_tables<k_kv_compact>("k_kv_compact", p, st); }

// A block a unit, as far as 256 an SM go, where all moves are there (16 moves of 80 layers, 1.34 GB, with 8, 32 and 256 blocks an SM: 224, 208
// and 200 us, 6.7 TB/s).  Where their number is on the device it is mostly small or nothing, and blocks without work cost more
// than that (none of 128 moves: 1.9, 5.5 and 40 us; one: 9.8, 10.5, 45): 8 an SM then, which takes 225 us for the 1.34 GB and 113 instead of 101 for
// the 676 MB above.
cudaError_t launch_kv_copy_pages(const CopyCall& c, const CopyLayer* layers, cudaStream_t st) {
    const long long units = 2ll * ((c.bytes + COPY_UNIT - 1) / COPY_UNIT);
    const long long blocks = std::min<long long>(units * c.n_moves * c.n_layers, ATTN_SMS * (c.count ? 8 : 256));
    auto launch = [&](auto most) {
        CopyView<decltype(most)::value> view;
        view.call = c;
        std::copy(layers, layers + c.n_layers, view.layer);
        launch_hook("k_kv_copy_pages", 0, st);
        const cudaError_t e = launch_early(k_kv_copy_pages<decltype(most)::value>, dim3((unsigned)blocks), COPY_THREADS, 0, st, view);
        launch_hook("k_kv_copy_pages", 1, st);
        return e;
    };
    return c.n_layers <= 4 ? launch(IntTag<4>{}) : c.n_layers <= 32 ? launch(IntTag<32>{}) : launch(IntTag<COPY_LAYERS>{});
}

}  // namespace hos
