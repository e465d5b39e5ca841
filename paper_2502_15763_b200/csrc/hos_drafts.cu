// Drafted tokens against the target's probabilities.
//
// Of all the rows only one a sequence is read whole: that of the first draft which is not accepted, or the last one.  A cluster
// of blocks takes a sequence.  Each block finds that row for itself (two scattered reads a draft, 32 drafts at once), then each of
// its warps adds up the weights of a contiguous segment of the vocabulary in 64 bits; the segments' sums are exchanged through
// shared memory, and the one that the random number falls into is gone through once more, in order.
// Bound: HBM where there are many sequences, latency of four dependent reads where there are few.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hos_cluster.cuh"
#include "hos_kv.cuh"
#include "hos_kv_kernels.h"
#include "hos_pages_kernels.h"

namespace hos {
namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32, MOST_BLOCKS = 16;

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
// What a probability counts for: nothing, unless it is positive and finite.
__device__ __forceinline__ float counted(float x) { return x > 0.0f && x < __int_as_float(0x7F800000) ? x : 0.0f; }

__device__ __forceinline__ double warp_sum_double(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(FULL, v, d);
    return v;
}

// The weights that the next token is drawn by: of entry v, max(p - q, 0) in 64 bits; q null: p, but nothing at `banned`.
template <typename T> struct Weights {
    const T *p, *q;
    int banned;
    __device__ __forceinline__ double at(int v) const {
        const double x = counted(as_float(p[v]));
        if (!q) return v == banned ? 0.0 : x;
        return fmax(x - (double)counted(as_float(q[v])), 0.0);
    }
};

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
                const float p = counted(as_float(static_cast<const T*>(d.target)[row * d.target_stride + token]));
                const float q = d.draft ? counted(as_float(static_cast<const T*>(d.draft)[row * d.draft_stride + token])) : 1.0f;
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

template <typename T> __global__ void __launch_bounds__(THREADS) k_verify_drafts(const __grid_constant__ hos_drafts d) {
    __shared__ Verdict verdict;
    __shared__ double sums[WARPS], before[MOST_BLOCKS * WARPS + 1];
    pdl_launch_dependents();
    pdl_wait();
    const int blocks = cluster_size(), rank = cluster_rank(), s = (int)blockIdx.x / blocks;
    if (warp_id() == 0) {
        const Verdict v = judge<T>(d, s);
        if (lane_id() == 0) verdict = v;
    }
    __syncthreads();
    const Verdict v = verdict;
    const int k = v.n - 1;
    const bool rejected = v.accepted < k;
    int next = -1;
    if (v.n > 0) {                                     // the same for the whole cluster
        const long long row = v.off + v.accepted;
        Weights<T> w{static_cast<const T*>(d.target) + row * d.target_stride, nullptr, -1};
        if (rejected && d.draft) w.q = static_cast<const T*>(d.draft) + row * d.draft_stride;
        if (rejected && !d.draft) w.banned = __ldg(d.tokens + row + 1);
        const int each = (d.vocab + blocks * WARPS - 1) / (blocks * WARPS);
        const long long first = (long long)(rank * WARPS + warp_id()) * each;
        const int a = (int)min(first, (long long)d.vocab), b = (int)min(first + each, (long long)d.vocab);
        double all = 0.0;
        for (int pass = 0; pass < 2; ++pass) {         // a second one only if nothing is left of p - q
            double sum = 0.0;
#pragma unroll 8
            for (int i = a + lane_id(); i < b; i += 32) sum += w.at(i);
            sum = warp_sum_double(sum);
            if (lane_id() == 0) sums[warp_id()] = sum;
            cluster_sync();
            if (warp_id() == 0) {                      // sums of the segments before each, in order
                double base = 0.0;
                for (int i0 = 0; i0 < blocks * WARPS; i0 += 32) {
                    const int i = i0 + lane_id();
                    const double mine = i < blocks * WARPS ? __longlong_as_double((long long)read_of_block(sums + i % WARPS, i / WARPS)) : 0.0;
                    double x = mine;
#pragma unroll
                    for (int dd = 1; dd < 32; dd <<= 1) {
                        const double o = __shfl_up_sync(FULL, x, dd);
                        if (lane_id() >= dd) x += o;
                    }
                    if (i < blocks * WARPS) before[i + 1] = base + x;
                    base += __shfl_sync(FULL, x, 31);
                }
                if (lane_id() == 0) before[0] = 0.0;
            }
            __syncthreads();
            all = before[blocks * WARPS];
            cluster_sync();                            // nobody's sums are written or gone before all have been read
            if (all > 0.0 || !rejected || pass == 1) break;
            w.q = nullptr;
            w.banned = -1;
        }
        if (all > 0.0) {
            const float u = __ldg(d.u_sample + s);
            const double t = u > 0.0f ? (double)u * all : 0.0;
            // the first segment whose end is beyond t; if rounding or a u from 1 on leaves none, the last one that has anything
            const int mine = rank * WARPS + warp_id();
            int segment = -1, last = 0;
            for (int i0 = 0; i0 < blocks * WARPS && segment < 0; i0 += 32) {
                const int i = i0 + lane_id();
                const bool in = i < blocks * WARPS;
                const unsigned beyond = __ballot_sync(FULL, in && before[i + 1] > t), some = __ballot_sync(FULL, in && before[i + 1] > before[i]);
                if (beyond) segment = i0 + __ffs(beyond) - 1;
                else if (some) last = i0 + 31 - __clz(some);
            }
            if (segment < 0) segment = last;
            if (segment == mine) {
                double c = before[mine];
                int pick = -1, positive = -1;
                for (int i0 = a; i0 < b && pick < 0; i0 += 32) {
                    const int i = i0 + lane_id();
                    const double x = i < b ? w.at(i) : 0.0;
                    double sum = x;
#pragma unroll
                    for (int dd = 1; dd < 32; dd <<= 1) {
                        const double o = __shfl_up_sync(FULL, sum, dd);
                        if (lane_id() >= dd) sum += o;
                    }
                    const unsigned beyond = __ballot_sync(FULL, x > 0.0 && c + sum > t), some = __ballot_sync(FULL, x > 0.0);
                    if (beyond) pick = i0 + __ffs(beyond) - 1;
                    else if (some) positive = i0 + 31 - __clz(some);
                    c += __shfl_sync(FULL, sum, 31);
                }
                next = pick >= 0 ? pick : positive;
                if (lane_id() == 0) {
                    d.next[s] = next;
                    d.out_tokens[row] = next;
                }
            }
        }
        if (rank == 0) {
            if (!(all > 0.0) && threadIdx.x == 0) {
                d.next[s] = -1;
                d.out_tokens[row] = -1;
            }
            for (int i = (int)threadIdx.x; i < v.n; i += THREADS)
                if (i != v.accepted) d.out_tokens[v.off + i] = i < v.accepted ? __ldg(d.tokens + v.off + i + 1) : -1;
        }
        if (rank == 0 && threadIdx.x == 0 && d.status) d.status[s] = v.flags | (all > 0.0 ? 0 : HOS_ST_INVALID);
    } else if (rank == 0 && threadIdx.x == 0) {
        d.next[s] = -1;
        if (d.status) d.status[s] = v.flags;
    }
    if (rank == 0 && threadIdx.x == 0) {
        d.accepted[s] = v.accepted;
        if (d.new_len) d.new_len[s] = __ldg(d.kv_len + s) - (k > 0 ? k - v.accepted : 0);
    }
}

template <typename T> cudaError_t verify(const hos_drafts& d, cudaStream_t st) {
    const int blocks = 1;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)blocks;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(d.n_seq * blocks));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    launch_hook("k_verify_drafts", 0, st);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_verify_drafts<T>, d);
    launch_hook("k_verify_drafts", 1, st);
    return e;
}

}  // namespace

cudaError_t launch_verify_drafts(const hos_drafts& d, cudaStream_t st) {
    if (d.type == HOS_TYPE_FP32) return verify<float>(d, st);
    return d.type == HOS_TYPE_BF16 ? verify<__nv_bfloat16>(d, st) : verify<__half>(d, st);
}

}  // namespace hos
