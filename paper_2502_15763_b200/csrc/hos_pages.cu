// The pages of a cache: who holds which, and their contents from one place to another.
#include <algorithm>

#include "hos_cluster.cuh"
#include "hos_kv_kernels.h"
#include "hos_kv.cuh"
#include "hos_pages_kernels.h"

namespace hos {
namespace {

constexpr int THREADS = 1024, WARPS = THREADS / 32;

// Sum of `v` over the threads before this one in the block, and over all of it.  Contains barriers.
__device__ __forceinline__ unsigned long long block_before(unsigned long long v, unsigned long long* scratch, unsigned long long* all) {
    unsigned long long s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(FULL, s, d);
        if (lane_id() >= d) s += o;
    }
    __syncthreads();
    if (lane_id() == 31) scratch[warp_id()] = s;
    __syncthreads();
    unsigned long long w = scratch[lane_id()];
    const unsigned long long mine = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(FULL, w, d);
        if (lane_id() >= d) w += o;
    }
    *all = __shfl_sync(FULL, w, 31);
    return s - v + __shfl_sync(FULL, w - mine, warp_id());
}

// Sums of a value of every block: of those before this one, and of all.  `mine` is in shared memory, written by one thread
// of each block before the last cluster_sync.
struct Shares { unsigned long long before, all; };
__device__ __forceinline__ Shares shares_of(const unsigned long long* mine) {
    Shares s{0, 0};
    const int rank = cluster_rank(), n = cluster_size();
    const unsigned long long v = lane_id() < n ? read_of_block(mine, lane_id()) : 0;
    s.all = warp_sum_u64(v);
    s.before = warp_sum_u64(lane_id() < rank ? v : 0);
    return s;
}

struct Range { int first, last; };
// The part of n things that falls to this block.
__device__ __forceinline__ Range block_part(int n) {
    const int each = (n + cluster_size() - 1) / cluster_size(), a = min(cluster_rank() * each, n);
    return Range{a, min(a + each, n)};
}
// A warp's part of the block's pages: whole groups of 32 but for the last one.
__device__ __forceinline__ Range warp_part(Range block) {
    const int each = ((block.last - block.first + WARPS - 1) / WARPS + 31) & ~31, a = min(block.first + warp_id() * each, block.last);
    return Range{a, min(a + each, block.last)};
}
__device__ __forceinline__ unsigned lanes_before() { return (1u << lane_id()) - 1u; }

__device__ __forceinline__ bool is_page(const PagesView& p, int page) { return (unsigned)page < (unsigned)p.n_pages; }
__device__ __forceinline__ bool is_length(const PagesView& p, int len) { return len >= 0 && len <= (long long)p.max_pages * p.page_size; }
__device__ __forceinline__ int pages_of(const PagesView& p, int len) { return (int)(((long long)len + p.page_size - 1) / p.page_size); }
__device__ __forceinline__ void flag(const PagesView& p, int s) {
    if (p.status) atomicOr(p.status + s, HOS_ST_INVALID);
}

// Rows are gone through in pieces of PIECE entries, one a warp.
constexpr int PIECE = 128;
template <typename F> __device__ __forceinline__ void for_each_piece(const PagesView& p, Range rows, F&& f) {
    const int pieces = max(1, (p.max_pages + PIECE - 1) / PIECE);
    const long long n = (long long)(rows.last - rows.first) * pieces;
    for (long long i = warp_id(); i < n; i += WARPS) {
        const int s = rows.first + (int)(i / pieces), first = (int)(i % pieces) * PIECE;
        f(s, first, min(first + PIECE, p.max_pages));
    }
}

// ---- resize ------------------------------------------------------------------------------------------------------------
constexpr unsigned long long GROWS = 1ull << 63, SPLITS = 1ull << 62, ONE_SPLIT = 1ull << 43, TAKES = ONE_SPLIT - 1;

struct Change { int old, now; bool valid; };
__device__ __forceinline__ Change change_of(const PagesView& p, int s) {
    Change c;
    c.old = p.len_in[s];
    c.now = p.change[s];
    c.valid = is_length(p, c.old) && is_length(p, c.now);
    return c;
}
// The page that a sequence grows from the inside of; -1: none.
__device__ __forceinline__ int grown_page(const PagesView& p, int s, const Change& c) {
    if (!c.valid || c.now <= c.old || c.old % p.page_size == 0) return -1;
    const int page = p.table_in[(long long)s * p.in_stride + c.old / p.page_size];
    return is_page(p, page) ? page : -2;
}

__global__ void __launch_bounds__(THREADS, 1) k_kv_resize(const __grid_constant__ PagesView p) {
    __shared__ unsigned long long scratch[WARPS], mine[2], warp_free[WARPS];
    pdl_launch_dependents();
    pdl_wait();
    const Range seqs = block_part(p.n_seq), pages = block_part(p.n_pages);
    const Range part = warp_part(pages);
    const int tid = (int)threadIdx.x;
    // the new counts begin as the old ones; what is known of pages that are grown from, as nothing
    if (p.refs != p.refs_in)
        for (int i = pages.first + tid; i < pages.last; i += THREADS) p.refs[i] = p.refs_in[i];
    for (int s = seqs.first + tid; s < seqs.last; s += THREADS) {
        const Change c = change_of(p, s);
        p.src[s] = p.dst[s] = -1;
        const int page = grown_page(p, s, c);
        if (page >= 0) p.growers[page] = 0, p.latest[page] = -1;
        if (p.status) p.status[s] = c.valid && page != -2 ? 0 : HOS_ST_INVALID;
    }
    cluster_sync();
    // pages given up; how many sequences grow from the inside of a page, and the last of them
    for (int s = seqs.first + warp_id(); s < seqs.last; s += WARPS) {
        const Change c = change_of(p, s);
        if (!c.valid) continue;
        for (int j = pages_of(p, c.now) + lane_id(); j < pages_of(p, c.old); j += 32) {
            const int page = p.table_in[(long long)s * p.in_stride + j];
            if (!is_page(p, page) || atomicSub(p.refs + page, 1) <= 0) flag(p, s);
        }
        const int page = lane_id() == 0 ? grown_page(p, s, c) : -1;
        if (page >= 0) {
            atomicAdd(p.growers + page, 1);
            atomicMax(p.latest + page, s);
        }
    }
    cluster_sync();
    // what each sequence takes, with sums in order; how many pages are free
    unsigned long long sum = 0;
    for (int s0 = seqs.first; s0 < seqs.last; s0 += THREADS) {
        const int s = s0 + tid;
        unsigned long long takes = 0, flags = 0;
        ResizePlan plan{0, 0, 0};
        if (s < seqs.last) {
            const Change c = change_of(p, s);
            plan.have = c.valid ? pages_of(p, c.old) : p.max_pages;
            plan.need = c.valid ? pages_of(p, c.now) : p.max_pages;
            if (c.valid && c.now > c.old) {
                flags = GROWS;
                takes = min(plan.need - plan.have, p.n_pages + 1);
                const int page = grown_page(p, s, c);
                if (page >= 0) {
                    const int refs = __ldcg(p.refs + page);
                    if (refs > 1 && !(__ldcg(p.growers + page) == refs && __ldcg(p.latest + page) == s)) {
                        flags |= SPLITS;
                        takes += ONE_SPLIT + 1;
                    }
                }
            }
        }
        unsigned long long all;
        plan.before = sum + block_before(takes, scratch, &all) + flags;
        if (s < seqs.last) p.plan[s] = plan;
        sum += all;
    }
    unsigned n_free = 0;
    for (int i0 = part.first; i0 < part.last; i0 += 32) {
        const int i = i0 + lane_id();
        n_free += __popc(__ballot_sync(FULL, i < part.last && __ldcg(p.refs + i) == 0));
    }
    if (lane_id() == 0) warp_free[warp_id()] = n_free;
    __syncthreads();
    if (warp_id() == 0) {
        const unsigned long long all = warp_sum_u64(warp_free[lane_id()]);
        if (lane_id() == 0) mine[0] = sum, mine[1] = all;
    }
    cluster_sync();
    const Shares takes = shares_of(mine), free = shares_of(mine + 1);
    // the free pages in order, as many as are taken
    const unsigned long long wanted = takes.all & TAKES;
    unsigned long long at = free.before + warp_sum_u64(lane_id() < warp_id() ? warp_free[lane_id()] : 0);
    for (int i0 = part.first; i0 < part.last && at < wanted; i0 += 32) {
        const int i = i0 + lane_id();
        const bool is_free = i < part.last && __ldcg(p.refs + i) == 0;
        const unsigned m = __ballot_sync(FULL, is_free);
        const unsigned long long k = at + __popc(m & lanes_before());
        if (is_free && k < wanted) p.queue[k] = i;
        at += __popc(m);
    }
    cluster_sync();
    // rows
    const bool in_place = p.table == p.table_in;
    if (tid == 0 && cluster_rank() == 0 && (takes.all & TAKES) <= free.all) *p.count = (int)(takes.all >> 43);
    for_each_piece(p, seqs, [&](int s, int first, int last) {
        const ResizePlan plan = p.plan[s];
        const unsigned long long before = takes.before + (plan.before & ~(GROWS | SPLITS)), base = before & TAKES;
        const int split = (plan.before & SPLITS) != 0;
        const unsigned long long mine = plan.before & GROWS ? (unsigned long long)min(plan.need - plan.have, p.n_pages + 1) + split : 0;
        const bool short_of = (plan.before & GROWS) && base + mine > free.all;
        const int have = plan.have, need = short_of ? have : plan.need, kept = min(have, need), splits_at = split && !short_of ? have - 1 : -1;
        const int32_t* in = p.table_in + (long long)s * p.in_stride;
        int32_t* out = p.table + (long long)s * p.out_stride;
        int a = first, b = last;
        if (in_place) a = max(a, splits_at >= 0 ? splits_at : kept), b = min(b, max(have, need));
        for (int j = a + lane_id(); j < b; j += 32) {
            int e = -1;
            if (j == splits_at || (j >= have && j < need)) {
                e = __ldcg(p.queue + base + (j == splits_at ? 0 : split + j - have));
                p.refs[e] = 1;
            } else if (j < kept) {
                e = in[j];
            }
            if (j == splits_at) {
                const int k = (int)(before >> 43), page = in[j];
                atomicSub(p.refs + page, 1);
                p.src[k] = page;
                p.dst[k] = e;
            }
            out[j] = e;
        }
        if (first == 0 && lane_id() == 0) {
            // the first sequence whose pages are not there: the splits before it are those that are made
            if (short_of && base <= free.all) *p.count = (int)(before >> 43);
            if (short_of && p.status) atomicOr(p.status + s, HOS_ST_PAGES);
            if (!(plan.before & GROWS) || !short_of) {
                const Change c = change_of(p, s);
                p.len[s] = c.valid ? c.now : c.old;
            } else if (p.len != p.len_in) {
                p.len[s] = p.len_in[s];
            }
        }
    });
}

// ---- fork --------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ int parent_of(const PagesView& p, int i) {
    const int s = p.change[i];
    return s >= 0 && s < p.n_seq && is_length(p, p.len_in[s]) ? s : s == -1 ? -1 : -2;
}

__global__ void __launch_bounds__(THREADS, 1) k_kv_fork(const __grid_constant__ PagesView p) {
    pdl_launch_dependents();
    pdl_wait();
    const Range seqs = block_part(p.n_seq), outs = block_part(p.n_out), pages = block_part(p.n_pages);
    const int tid = (int)threadIdx.x;
    if (p.refs != p.refs_in)
        for (int i = pages.first + tid; i < pages.last; i += THREADS) p.refs[i] = p.refs_in[i];
    for (int s = seqs.first + tid; s < seqs.last; s += THREADS) p.children[s] = 0;
    for (int i = outs.first + tid; i < outs.last; i += THREADS) {
        const int s = parent_of(p, i);
        p.len[i] = s >= 0 ? p.len_in[s] : 0;
        if (p.status) p.status[i] = s == -2 ? HOS_ST_INVALID : 0;
    }
    cluster_sync();
    for (int i = outs.first + tid; i < outs.last; i += THREADS) {
        const int s = parent_of(p, i);
        if (s >= 0) atomicAdd(p.children + s, 1);
    }
    for_each_piece(p, outs, [&](int i, int first, int last) {
        const int s = parent_of(p, i), have = s >= 0 ? pages_of(p, p.len_in[s]) : 0;
        for (int j = first + lane_id(); j < last; j += 32) {
            int e = -1;
            if (j < have) {
                e = p.table_in[(long long)s * p.in_stride + j];
                if (!is_page(p, e)) flag(p, i);
            }
            p.table[(long long)i * p.out_stride + j] = e;
        }
    });
    cluster_sync();
    for_each_piece(p, seqs, [&](int s, int first, int last) {
        const int more = __ldcg(p.children + s) - 1, len = p.len_in[s];
        if (more == 0 || !is_length(p, len)) return;
        for (int j = first + lane_id(); j < min(last, pages_of(p, len)); j += 32) {
            const int page = p.table_in[(long long)s * p.in_stride + j];
            if (is_page(p, page)) atomicAdd(p.refs + page, more);
        }
    });
}

// ---- compact -----------------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(THREADS, 1) k_kv_compact(const __grid_constant__ PagesView p) {
    __shared__ unsigned long long mine[3], warp_live[WARPS], warp_late[WARPS], warp_hole[WARPS];
    pdl_launch_dependents();
    pdl_wait();
    const Range seqs = block_part(p.n_seq), pages = block_part(p.n_pages);
    const Range part = warp_part(pages);
    const int tid = (int)threadIdx.x;
    unsigned n = 0;
    for (int i0 = part.first; i0 < part.last; i0 += 32) {
        const int i = i0 + lane_id();
        n += __popc(__ballot_sync(FULL, i < part.last && p.refs_in[i] != 0));
    }
    if (lane_id() == 0) warp_live[warp_id()] = n;
    __syncthreads();
    if (warp_id() == 0) {
        const unsigned long long all = warp_sum_u64(warp_live[lane_id()]);
        if (lane_id() == 0) mine[0] = all;
    }
    cluster_sync();
    const int n_live = (int)shares_of(mine).all;
    // pages in use behind the first n_live, and free ones among those: as many of the one as of the other
    unsigned late = 0, hole = 0;
    for (int i0 = part.first; i0 < part.last; i0 += 32) {
        const int i = i0 + lane_id();
        const bool there = i < part.last, live = there && p.refs_in[i] != 0;
        late += __popc(__ballot_sync(FULL, live && i >= n_live));
        hole += __popc(__ballot_sync(FULL, there && !live && i < n_live));
    }
    if (lane_id() == 0) warp_late[warp_id()] = late, warp_hole[warp_id()] = hole;
    __syncthreads();
    if (warp_id() == 0) {
        const unsigned long long a = warp_sum_u64(warp_late[lane_id()]), b = warp_sum_u64(warp_hole[lane_id()]);
        if (lane_id() == 0) mine[1] = a, mine[2] = b;
    }
    cluster_sync();
    const Shares lates = shares_of(mine + 1), holes = shares_of(mine + 2);
    int late_at = (int)(lates.before + warp_sum_u64(lane_id() < warp_id() ? warp_late[lane_id()] : 0));
    int hole_at = (int)(holes.before + warp_sum_u64(lane_id() < warp_id() ? warp_hole[lane_id()] : 0));
    const int count = (int)lates.all;
    for (int i0 = part.first; i0 < part.last; i0 += 32) {
        const int i = i0 + lane_id();
        const bool there = i < part.last;
        const int refs = there ? p.refs_in[i] : 0;
        const bool is_late = refs != 0 && i >= n_live, is_hole = there && refs == 0 && i < n_live;
        const unsigned a = __ballot_sync(FULL, is_late), b = __ballot_sync(FULL, is_hole);
        if (is_late) p.src[late_at + __popc(a & lanes_before())] = i;
        if (is_hole) p.dst[hole_at + __popc(b & lanes_before())] = i;
        if (there && i >= n_live) p.growers[i] = is_late ? late_at + __popc(a & lanes_before()) : -1;
        if (there && i >= count) p.src[i] = p.dst[i] = -1;
        if (there && p.refs != p.refs_in) p.refs[i] = refs;
        late_at += __popc(a);
        hole_at += __popc(b);
    }
    if (tid == 0 && cluster_rank() == 0) *p.count = count;
    for (int s = seqs.first + tid; s < seqs.last; s += THREADS)
        if (p.status) p.status[s] = is_length(p, p.len_in[s]) ? 0 : HOS_ST_INVALID;
    cluster_sync();
    for (int k = cluster_rank() * THREADS + tid; k < count; k += cluster_size() * THREADS) {
        const int a = __ldcg(p.src + k), b = __ldcg(p.dst + k);
        const int refs = p.refs_in[a];
        p.refs[b] = refs;
        p.refs[a] = 0;
    }
    const bool in_place = p.table == p.table_in;
    for_each_piece(p, seqs, [&](int s, int first, int last) {
        const int len = p.len_in[s];
        const bool valid = is_length(p, len);
        const int have = valid ? pages_of(p, len) : p.max_pages;
        for (int j = first + lane_id(); j < (in_place ? min(last, have) : last); j += 32) {
            int e = -1;
            if (j < have) {
                e = p.table_in[(long long)s * p.in_stride + j];
                if (valid) {
                    const bool ok = is_page(p, e);
                    const int k = ok && e >= n_live ? __ldcg(p.growers + e) : -1;
                    if (!ok || (e >= n_live && k < 0)) flag(p, s);
                    if (k >= 0) e = __ldcg(p.dst + k);
                }
            }
            p.table[(long long)s * p.out_stride + j] = e;
        }
    });
}

// ---- copy --------------------------------------------------------------------------------------------------------------
constexpr int COPY_THREADS = 256, COPY_UNIT = COPY_THREADS * 64;

__global__ void __launch_bounds__(COPY_THREADS) k_kv_copy_pages(const __grid_constant__ CopyView c) {
    pdl_launch_dependents();
    pdl_wait();
    const int n = c.count ? max(0, min(c.n_moves, __ldg(c.count))) : c.n_moves;
    // a page of k or v is so many units, its scales one each as far as they go
    const int units = (c.bytes + COPY_UNIT - 1) / COPY_UNIT, scale_units = (c.scale_bytes + COPY_UNIT - 1) / COPY_UNIT, per = 2 * (units + scale_units);
    const long long total = (long long)n * c.n_layers * per;
    for (long long u = blockIdx.x; u < total; u += gridDim.x) {
        const int which = (int)(u % per), move = (int)(u / per % n), layer = (int)(u / per / n);
        const int from = __ldg(c.src + move), to = __ldg(c.dst + move);
        if ((unsigned)from >= (unsigned)c.from_pages || (unsigned)to >= (unsigned)c.to_pages) {
            if (threadIdx.x == 0 && which == 0 && layer == 0 && c.status) atomicOr(c.status + move, HOS_ST_INVALID);
            continue;
        }
        const bool scales = which >= 2 * units;
        const int w = scales ? which - 2 * units : which, each = scales ? scale_units : units;
        const int array = (scales ? 2 : 0) + w / each, at = w % each * COPY_UNIT, end = min(scales ? c.scale_bytes : c.bytes, at + COPY_UNIT);
        const CopyLayer& l = c.layer[layer];
        const unsigned char* a = l.from[array] + from * l.from_stride[scales];
        unsigned char* b = l.to[array] + to * l.to_stride[scales];
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int o = at + (i * COPY_THREADS + (int)threadIdx.x) * 16;
            if (o < end) x[i] = *reinterpret_cast<const uint4*>(a + o);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int o = at + (i * COPY_THREADS + (int)threadIdx.x) * 16;
            if (o < end) *reinterpret_cast<uint4*>(b + o) = x[i];
        }
    }
}

template <typename K> cudaError_t launch_cluster(const char* name, K kernel, int blocks, const PagesView& p, cudaStream_t st) {
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)blocks;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    launch_hook(name, 0, st);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
    launch_hook(name, 1, st);
    return e;
}

}  // namespace

cudaError_t launch_kv_resize(const PagesView& p, cudaStream_t st) { return launch_cluster("k_kv_resize", k_kv_resize, 1, p, st); }
cudaError_t launch_kv_fork(const PagesView& p, cudaStream_t st) { return launch_cluster("k_kv_fork", k_kv_fork, 1, p, st); }
cudaError_t launch_kv_compact(const PagesView& p, cudaStream_t st) { return launch_cluster("k_kv_compact", k_kv_compact, 1, p, st); }

cudaError_t launch_kv_copy_pages(const CopyView& c, cudaStream_t st) {
    const long long per = 2 * ((c.bytes + COPY_UNIT - 1) / COPY_UNIT + (c.scale_bytes + COPY_UNIT - 1) / COPY_UNIT);
    const long long blocks = std::min<long long>(per * c.n_moves * c.n_layers, 148 * 8);
    launch_hook("k_kv_copy_pages", 0, st);
    const cudaError_t e = launch_early(k_kv_copy_pages, dim3((unsigned)blocks), COPY_THREADS, 0, st, c);
    launch_hook("k_kv_copy_pages", 1, st);
    return e;
}

}  // namespace hos
