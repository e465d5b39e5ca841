// Drafted tokens against the target's probabilities.
//
// Of all the rows only one a sequence is read whole: that of the first draft which is not accepted, or the last one.  A cluster
// of blocks takes a sequence.  Each block finds that row for itself (two scattered reads a draft, 32 drafts at once), then each of
// its warps adds up the weights of a contiguous segment of the vocabulary in 64 bits; the blocks' sums are exchanged through
// shared memory, and the one that the random number falls into goes once more through the segment that it falls into, in order.
// Sums are kept in 64 bits because the token is found by comparing them: with 128,000 shares of 10^-5 an error of 10^-7
// would move their ends by a hundredth.
// Bound: latency where there are few sequences (six dependent steps: offsets, drafts, their probabilities, the row, the blocks' sums,
// the segment); where there are many, HBM for 32-bit entries, instructions for 16-bit ones (ten a pair; the bf16 form spills 16 bytes at its 64
// registers).  One B200: one sequence of 32,000 32-bit entries 4.6 us, 33 of 50,257 bf16 ones 6.8; 128 of 128,000 32-bit ones, four drafts (129 MB),
// 27 us, 4.8 TB/s: a single wave of blocks, not even over the SMs, whose first and last steps are not hidden behind the reads; 800 of them
// with one draft 122 us, 6.7 TB/s, of bf16 ones 81, 5.0, of fp16 ones 78, 5.2.
// Two forms go entry by entry.  Where a looked-up draft is not accepted, the warp whose segment holds it adds that up again: 128 of 128,000 bf16
// entries 18.6 us against 14.2 for an accepted one, 800 84 against 61, in 32 bits 126 against 85.  Rows of p and q that are not aligned alike:
// 128 of 128,000 31 us in 32 bits (23 where they are), 26 in bf16 (18), 800 134 (122) and 113 (81).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hos_cluster.cuh"
#include "hos_kv.cuh"
#include "hos_kv_kernels.h"
#include "hos_pages_kernels.h"

namespace hos {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32, BLOCKS_PER_SM = 4, MOST_BLOCKS = 16;

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ bool counts(float x) { return x > 0.0f && x < __int_as_float(0x7F800000); }
// What a probability of the target counts for: nothing, unless it is positive and finite; of the draft: nothing, if it is negative or NaN.
__device__ __forceinline__ float target_of(float x) { return counts(x) ? x : 0.0f; }
__device__ __forceinline__ float draft_of(float x) { return fmaxf(x, 0.0f); }

// 16 bytes of a row.
template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    uint4 w;
    __device__ __forceinline__ float at(int i) const;
};
template <> __device__ __forceinline__ float Vec<float>::at(int i) const {
    return __uint_as_float(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w);
}
__device__ __forceinline__ uint32_t pair_of(const uint4& w, int i) { return i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w; }
template <> __device__ __forceinline__ float Vec<__half>::at(int i) const {
    const float2 f = Pair<__half>::unpack(pair_of(w, i));
    return i & 1 ? f.y : f.x;
}
template <> __device__ __forceinline__ float Vec<__nv_bfloat16>::at(int i) const {
    const float2 f = Pair<__nv_bfloat16>::unpack(pair_of(w, i));
    return i & 1 ? f.y : f.x;
}

// The weights that the next token is drawn by: of entry v, max(p - q, 0) in 64 bits; q null: p, but nothing at `banned`.
template <typename T> struct Weights {
    const T *p, *q;
    int banned;
    __device__ __forceinline__ double at(int v) const {
        const double x = target_of(as_float(__ldg(p + v)));
        if (!q) return v == banned ? 0.0 : x;
        return fmax(x - (double)draft_of(as_float(__ldg(q + v))), 0.0);
    }
    // K weights from `a` on, as far as [a, b) goes.
    template <int K> __device__ __forceinline__ void run(int a, int b, bool wide, double (&x)[K]) const {
        constexpr int N = Vec<T>::N;
        if (K >= N && wide && b - a >= K && ((reinterpret_cast<uintptr_t>(p + a)) & 15) == 0) {
            Vec<T> u[(K + N - 1) / N], v[(K + N - 1) / N];
#pragma unroll
            for (int k = 0; k < K / N; ++k) {
                u[k].w = __ldg(reinterpret_cast<const uint4*>(p + a) + k);
                v[k].w = q ? __ldg(reinterpret_cast<const uint4*>(q + a) + k) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
                x[k] = a + k == banned ? 0.0 : fmax((double)target_of(u[k / N].at(k % N)) - (double)draft_of(v[k / N].at(k % N)), 0.0);
            return;
        }
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] = a + k < b ? at(a + k) : 0.0;
    }
    // Sum over [a, b) by one warp; where they can be read 16 bytes at a time from `a` on, in both rows.  A difference x - y > 0 is
    // d + e exactly, d rounded to 32 bits and e = (x - d) - y (Dekker, 1971); with the larger of x and y in the place of x both are
    // zero where nothing is left.  The d are added up in 64 bits; the e, below 2^-24 of them, 16 or 32 in 32 bits first, which leaves 2^-43 of the
    // sum.  So a conversion and a 64-bit sum are left of two and three (they go at a fraction of the others' rate).  An infinity or a NaN that
    // does not fall out by itself makes the sum one: the caller looks.
    template <bool Q> __device__ __forceinline__ double sum_wide(int a, int b) const {
        constexpr int N = Vec<T>::N, AHEAD = 4;
        double s[2] = {0.0, 0.0};
        const int whole = a + (b - a) / N * N;
        for (int i0 = a + lane_id() * N; i0 < whole; i0 += 32 * N * AHEAD) {
            Vec<T> x[AHEAD], y[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int i = i0 + k * 32 * N;
                x[k].w = y[k].w = make_uint4(0, 0, 0, 0);
                if (i < whole) {
                    x[k].w = __ldg(reinterpret_cast<const uint4*>(p + i));
                    if (Q) y[k].w = __ldg(reinterpret_cast<const uint4*>(q + i));
                }
            }
            float small = 0.0f;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (i0 - lane_id() * N + k * 32 * N >= whole) break;       // the end of the warp's
                const int out = banned - (i0 + k * 32 * N);        // which of these is the banned one
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (Q) {
                        const float u = draft_of(y[k].at(j)), v = fmaxf(x[k].at(j), u), d = v - u;
                        s[j & 1] += (double)d;
                        small += (v - d) - u;
                    } else {
                        s[j & 1] += (double)fmaxf(x[k].at(j), 0.0f);
                    }
                }
                if (!Q && (unsigned)out < (unsigned)N) return __longlong_as_double(0x7FF8000000000000ll);      // not by this way
            }
            if (Q) s[0] += (double)small;
        }
        const int i = whole + lane_id();
        if (i < b) s[0] += at(i);
        return s[0] + s[1];
    }
    __device__ __forceinline__ double sum_plain(int a, int b) const {
        double s = 0.0;
#pragma unroll 8
        for (int i = a + lane_id(); i < b; i += 32) s += at(i);
        return s;
    }
    // Of the whole warp.
    __device__ __forceinline__ double sum(int a, int b, bool wide) const {
        double s = !wide ? sum_plain(a, b) : q ? sum_wide<true>(a, b) : sum_wide<false>(a, b);
        if (wide && __any_sync(FULL, !(s < __longlong_as_double(0x7FF0000000000000ll)))) s = sum_plain(a, b);
        return s;
    }
};

__device__ __forceinline__ double warp_sum_double(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(FULL, v, d);
    return v;
}
__device__ __forceinline__ double warp_sum_upto(double v) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const double o = __shfl_up_sync(FULL, v, d);
        if (lane_id() >= d) v += o;
    }
    return v;
}
// The first lane whose sum `upto` is beyond t; if there is none (rounding, or a t that is the whole sum), the last one that has
// anything itself; -1: nobody has.
__device__ __forceinline__ int first_beyond(double upto, double own, double t) {
    const unsigned beyond = __ballot_sync(FULL, own > 0.0 && upto > t), some = __ballot_sync(FULL, own > 0.0);
    return beyond ? __ffs(beyond) - 1 : 31 - __clz(some);
}

struct Verdict {
    int off, n, accepted, flags;                     // the sequence's tokens; drafts accepted; status bits
};

// The drafts of a sequence, in order, until one is not accepted.  All lanes of a warp.
template <typename T> __device__ __forceinline__ Verdict judge(const hos_drafts& d, int s) {
    Verdict r{__ldg(d.tok_off + s), 0, 0, 0};
    const int end = __ldg(d.tok_off + s + 1);
    r.n = end - r.off;
    if (r.off < 0 || end < r.off || end > d.n_tokens) {
        r.n = 0;
        r.flags = HOS_ST_INVALID;
    }
    const int k = r.n - 1;
    for (int i0 = 0; i0 < k; i0 += 32) {
        const int i = i0 + lane_id();
        bool good = false, strange = false;
        if (i < k) {
            const long long row = r.off + i;
            const int token = __ldg(d.tokens + row + 1);
            const float u = __ldg(d.u_accept + row);
            strange = (unsigned)token >= (unsigned)d.vocab;
            if (!strange) {
                const float p = target_of(as_float(static_cast<const T*>(d.target)[row * d.target_stride + token]));
                const float q = d.draft ? draft_of(as_float(static_cast<const T*>(d.draft)[row * d.draft_stride + token])) : 1.0f;
                good = (double)u * (double)q < (double)p;
            }
        }
        const unsigned m = __ballot_sync(FULL, good);
        const unsigned odd = __ballot_sync(FULL, strange);
        const int run = __ffs(~m) - 1;                 // -1: all 32 accepted
        if (run < 0) {
            r.accepted += 32;
            continue;
        }
        r.accepted += run;
        if (odd >> run & 1u) r.flags = HOS_ST_INVALID;
        break;
    }
    return r;
}

// The first entry of [a, b) up to which the weights add up to more than `left` (or the last one that has any) is the next token.  By a
// whole block, RUN neighbours a thread, all loads at once (32 neighbours a warp at a time would take a scan for each 32: 3 us more).
template <int RUN, typename T>
__device__ __forceinline__ void search(const hos_drafts& d, int s, long long row, const Weights<T>& w, int a, int b, bool wide, double left, double* sums) {
    for (int i0 = a; i0 < b; i0 += THREADS * RUN) {
        const int first = i0 + (int)threadIdx.x * RUN;
        double x[RUN], mine = 0.0;
        w.template run<RUN>(first, b, wide, x);
#pragma unroll
        for (int k = 0; k < RUN; ++k) mine += x[k];
        const double upto_lane = warp_sum_upto(mine);
        __syncthreads();
        if (lane_id() == 31) sums[warp_id()] = upto_lane;
        __syncthreads();
        const double own = lane_id() < WARPS ? sums[lane_id()] : 0.0, upto = warp_sum_upto(own), all = __shfl_sync(FULL, upto, 31);
        const int in = first_beyond(upto, own, left);
        if (in == warp_id()) {                         // should `left` lie behind all of this, the last one so far
            double rest = left - __shfl_sync(FULL, upto - own, in);
            if (first_beyond(upto_lane, mine, rest) == lane_id()) {
                rest -= upto_lane - mine;
                int pick = -1;
                bool found = false;
#pragma unroll
                for (int k = 0; k < RUN; ++k) {
                    if (x[k] > 0.0 && !found) {        // only weights decide: rounded sums may have left a rest below zero
                        pick = first + k;
                        found = x[k] > rest;
                    }
                    rest -= x[k];
                }
                d.next[s] = d.out_tokens[row] = pick;
            }
        }
        if (all > left) return;
        left -= all;
    }
}

template <typename T> __global__ void __launch_bounds__(THREADS, BLOCKS_PER_SM) k_verify_drafts(const __grid_constant__ hos_drafts d) {
    __shared__ Verdict verdict;
    __shared__ double sums[WARPS], board[2][MOST_BLOCKS];  // of this block's warps; of all blocks, in each pass
    pdl_launch_dependents();
    pdl_wait();
    const int blocks = cluster_size(), rank = cluster_rank(), s = (int)blockIdx.x / blocks;
    cluster_begun_arrive();
    if (warp_id() == 0) {
        const Verdict v = judge<T>(d, s);
        if (lane_id() == 0) verdict = v;
    }
    __syncthreads();
    const Verdict v = verdict;
    const int k = v.n - 1;
    if (rank == 0) {
        for (int i = (int)threadIdx.x; i < v.n; i += THREADS)
            if (i != v.accepted) d.out_tokens[v.off + i] = i < v.accepted ? __ldg(d.tokens + v.off + i + 1) : -1;
        if (threadIdx.x == 0) {
            d.accepted[s] = v.accepted;
            if (d.new_len) d.new_len[s] = __ldg(d.kv_len + s) - (k > 0 ? k - v.accepted : 0);
            if (v.n == 0) d.next[s] = -1;
            if (d.status) d.status[s] = v.flags;
        }
    }
    cluster_begun_wait();
    if (v.n == 0) return;                              // the whole cluster
    const bool rejected = v.accepted < k;
    const long long row = v.off + v.accepted;
    Weights<T> w{static_cast<const T*>(d.target) + row * d.target_stride, nullptr, -1};
    if (rejected && d.draft) w.q = static_cast<const T*>(d.draft) + row * d.draft_stride;
    if (rejected && !d.draft) w.banned = __ldg(d.tokens + row + 1);
    // segments begin on 16 bytes of p, the first at 0, and end with the row
    constexpr int N = Vec<T>::N;
    const int head = (int)((16 - (reinterpret_cast<uintptr_t>(w.p) & 15)) & 15) / (int)sizeof(T);
    const bool wide = !w.q || ((reinterpret_cast<uintptr_t>(w.p) ^ reinterpret_cast<uintptr_t>(w.q)) & 15) == 0;
    const long long each = ((d.vocab + blocks * WARPS - 1) / (blocks * WARPS) + N - 1) / N * N;
    auto edge = [&](int i) { return i == 0 ? 0 : (int)min(head + i * each, (long long)d.vocab); };
    const int segment = rank * WARPS + warp_id(), a = edge(segment), b = edge(segment + 1);
    const float u = __ldg(d.u_sample + s);
    for (int pass = 0;; ++pass) {                      // a second one only if nothing is left of p - q
        const int from = min(b, max(a, head));
        double sum = w.sum(from, b, wide);
        if (a + lane_id() < from) sum += w.at(a + lane_id());
        sum = warp_sum_double(sum);
        if (lane_id() == 0) sums[warp_id()] = sum;
        __syncthreads();
        double own = lane_id() < WARPS ? sums[lane_id()] : 0.0, upto = warp_sum_upto(own);
        const double mine = __shfl_sync(FULL, upto, 31);
        if ((int)threadIdx.x < blocks) write_to_block(&board[pass][rank], (int)threadIdx.x, mine);
        cluster_or_block_sync();
        const double of_block = lane_id() < blocks ? board[pass][lane_id()] : 0.0;
        const double upto_block = warp_sum_upto(of_block);
        const double all = __shfl_sync(FULL, upto_block, 31);
        if (!(all > 0.0)) {
            if (rejected && pass == 0) {
                w.q = nullptr;
                w.banned = -1;
                continue;
            }
            if (rank == 0 && threadIdx.x == 0) {
                d.next[s] = d.out_tokens[row] = -1;
                if (d.status) d.status[s] = v.flags | HOS_ST_INVALID;
            }
            return;
        }
        // from 1 on beyond all sums, however they are rounded: the last token that has anything
        const double t = u >= 1.0f ? __longlong_as_double(0x7FF0000000000000ll) : u > 0.0f ? (double)u * all : 0.0;
        const int block = first_beyond(upto_block, of_block, t);
        if (block == rank) {
            double left = t - __shfl_sync(FULL, upto_block - of_block, block);
            const int warp = first_beyond(upto, own, left);
            left -= __shfl_sync(FULL, upto - own, warp);
            const int from = edge(rank * WARPS + warp), to = edge(rank * WARPS + warp + 1);
            // one neighbour a thread where that is enough (one sequence of 32,000 entries: 4.6 us, with 8 neighbours 5.6)
            if (to - from <= THREADS) search<1>(d, s, row, w, from, to, wide, left, sums);
            else search<8>(d, s, row, w, from, to, wide, left, sums);
        }
        return;
    }
}

// As many blocks a sequence as there is room for at once, with 1,000 entries each at least and, room or not, 64,000 at most; up to 16, but
// those only where two an SM are enough (clusters of 16 do not fill the groups of SMs that they have to stay in).  One, 2, 4, 8, 16, us, p and q in
// 32 bits: one sequence of 32,000 entries 9.7, 7.7, 6.3, 6.1, 5.1; of 128,000 21, 15, 9.4, 7.7, 6.6; 40 of those 28, 17, 13, 12, 13; 100 of them
// 40, 25, 19, 20, 27; 296 of them 59, 50 (6.1 TB/s), 56, 57, 76; 800 134, 121 (6.8 TB/s), 120, 129, 186.  With 512 threads, two blocks an SM and up
// to 8 a sequence: 5.7, 7.4, 12, 19, 47 and 120.
template <typename T> cudaError_t verify(const hos_drafts& d, cudaStream_t st) {
    int blocks = MOST_BLOCKS;
    auto room = [&] { return (long long)d.n_seq * blocks <= ATTN_SMS * (blocks > 8 ? 2 : BLOCKS_PER_SM); };
    while (blocks > 1 && (d.vocab < 1000 * blocks || (!room() && d.vocab <= 64000 * (blocks / 2)))) blocks >>= 1;
    static std::atomic<unsigned long long> asked{0};
    if (blocks > 8) {
        const cudaError_t e = ask_for_large_clusters(reinterpret_cast<const void*>(&k_verify_drafts<T>), asked);
        if (e != cudaSuccess) return e;
    }
    return launch_clusters("k_verify_drafts", k_verify_drafts<T>, d.n_seq * blocks, blocks, THREADS, st, d);
}

}  // namespace

cudaError_t launch_verify_drafts(const hos_drafts& d, cudaStream_t st) {
    if (d.type == HOS_TYPE_FP32) return verify<float>(d, st);
    return d.type == HOS_TYPE_BF16 ? verify<__nv_bfloat16>(d, st) : verify<__half>(d, st);
}

}  // namespace hos
