// Second half of an attention call: the pieces of split tiles become outputs.
//
// A piece holds, per row, the unnormalised output, the reference m and the normaliser l of its tokens (exponents
// in base 2), so out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i with m = max_i m_i.  Pieces are added in list
// order.  Launched so that it may start while the attention kernel drains.
#include "hos_kernels.h"
#include "hos_kv.cuh"

namespace hos {
namespace {

// Worker w's record, if it has one, names the tile that begins in its share and ends in a later one's: the pieces are slot 1
// of w and slot 0 of the workers up to `last`.  A block looks through the records of every gridDim.x-th worker; its 16 warps
// take rows, and where there are fewer rows than warps several warps share a row's pieces.  D / 4 lanes read a piece's row.
constexpr int WARPS = 16, BLOCKS = 4 * ATTN_SMS;
template <typename T, int D, int ROWS>
__global__ void __launch_bounds__(WARPS * 32) k_attn_combine(const __grid_constant__ AttnView a, const Partial* __restrict__ meta, const int workers,
                                                            const RowState* __restrict__ state, const float* __restrict__ part) {
    constexpr int LANES = D / 4, PER = 32 / LANES;                     // pieces that a warp reads at once
    __shared__ float4 sum_o[WARPS][LANES];
    __shared__ float sum_l[WARPS];
    const int lane = lane_id(), warp = warp_id(), sub = lane / LANES;
    pdl_wait();
    for (int w0 = blockIdx.x; w0 < workers; w0 += 32 * gridDim.x) {
        // 32 records at a time
        const int wl = w0 + lane * (int)gridDim.x;
        Partial mine{0, 0, 0, -1};
        if (wl < workers) mine = meta[wl];
        for (unsigned some = __ballot_sync(FULL, mine.last >= 0); some; some &= some - 1) {
            const int src = __ffs(some) - 1, w = w0 + src * (int)gridDim.x;
            const int seq = __shfl_sync(FULL, mine.seq, src), head = __shfl_sync(FULL, mine.head, src);
            const int tile = __shfl_sync(FULL, mine.tile, src), n = __shfl_sync(FULL, mine.last, src) - w + 1;
            const SeqInfo q = load_seq(a.kv, seq, false);
            const int rows = min(ROWS, q.n * a.group - tile * ROWS);
            const int shares = rows > 8 ? 1 : rows > 4 ? 2 : rows > 2 ? 4 : rows == 2 ? 8 : 16;   // warps a row
            const int row = warp / shares, share = warp % shares;
            const bool busy = row < rows;
            auto slot = [&](int i) { return (long long)(i == 0 ? 2 * w + 1 : 2 * (w + i)) * ROWS + row; };
            float m = -INFINITY, l = 0.0f;
            float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (busy) {
                for (int i = lane; i < n; i += 32) m = fmaxf(m, state[slot(i)].m);
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL, m, d));
                const float ms = m == -INFINITY ? 0.0f : m;
                // pieces share * PER + sub, + shares * PER, ...
#pragma unroll 4
                for (int i = share * PER + sub; i < n; i += shares * PER) {
                    const RowState st = state[slot(i)];
                    const float4 v = reinterpret_cast<const float4*>(part + slot(i) * D)[lane % LANES];
                    const float by = exp2f(st.m - ms);
                    if (lane % LANES == 0) l += st.l * by;
                    o.x += by * v.x; o.y += by * v.y; o.z += by * v.z; o.w += by * v.w;
                }
                if (PER == 2) {
                    o.x += __shfl_xor_sync(FULL, o.x, 16); o.y += __shfl_xor_sync(FULL, o.y, 16);
                    o.z += __shfl_xor_sync(FULL, o.z, 16); o.w += __shfl_xor_sync(FULL, o.w, 16);
                    l += __shfl_xor_sync(FULL, l, 16);
                }
                if (lane < LANES) sum_o[warp][lane] = o;
                if (lane == 0) sum_l[warp] = l;
            }
            __syncthreads();
            if (busy && share == 0) {
                l = 0.0f;
                for (int k = 0; k < shares; ++k) l += sum_l[warp + k];
                const float by = l == 0.0f ? 0.0f : 1.0f / l;
                const int r = tile * ROWS + row, i = by_group(a, r), tok = q.off + i, hd = head * a.group + r - i * a.group;
                if (lane < LANES) {
                    o = sum_o[warp][lane];
                    for (int k = 1; k < shares; ++k) {
                        const float4 v = sum_o[warp + k][lane];
                        o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
                    }
                    T* dst = reinterpret_cast<T*>(a.out) + (long long)tok * a.o_tok + (long long)hd * a.o_head;
                    reinterpret_cast<uint2*>(dst)[lane] = make_uint2(Pair<T>::pack(o.x * by, o.y * by), Pair<T>::pack(o.z * by, o.w * by));
                }
                if (a.lse && lane == 0)
                    a.lse[(long long)tok * a.n_heads + hd] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
            }
            __syncthreads();
        }
    }
}

// The same for the chunk kernel's tiles of 256 rows, whose pieces are few: a warp takes four rows, whose loads do not wait for one
// another, and goes through the pieces with a running maximum.
constexpr int BIG_ROWS = 256, BIG_WARPS = 8, BIG_SPAN = 4 * BIG_WARPS;
template <typename T, int D>
__global__ void __launch_bounds__(BIG_WARPS * 32) k_attn_combine_tiles(const __grid_constant__ AttnView a, const Partial* __restrict__ meta,
                                                                      const RowState* __restrict__ state, const float* __restrict__ part) {
    constexpr int PER = D / 32;                // elements a lane
    const int lane = lane_id(), w = blockIdx.x;
    pdl_wait();
    const Partial p = meta[w];
    if (p.last < 0) return;
    const SeqInfo q = load_seq(a.kv, p.seq, false);
    const int rows = min(BIG_ROWS, q.n * a.group - p.tile * BIG_ROWS), r0 = blockIdx.y * BIG_SPAN + warp_id() * 4;
    if (r0 >= rows) return;
    float m[4], l[4], o[4][PER];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        m[k] = -INFINITY;
        l[k] = 0.0f;
#pragma unroll
        for (int e = 0; e < PER; ++e) o[k][e] = 0.0f;
    }
    const int n = p.last - w + 1;
#pragma unroll 2
    for (int i = 0; i < n; ++i) {
        // rows past the tile's end have room in the workspace, too; what they hold is not used
        const long long at = (long long)(i == 0 ? 2 * w + 1 : 2 * (w + i)) * BIG_ROWS + r0;
        RowState st[4];
        float v[4][PER];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            st[k] = state[at + k];
            const float* src = part + (at + k) * D + lane * PER;
            if (PER == 4) {
                const float4 f = *reinterpret_cast<const float4*>(src);
                v[k][0] = f.x; v[k][1] = f.y; v[k][PER - 2] = f.z; v[k][PER - 1] = f.w;
            } else {
                const float2 f = *reinterpret_cast<const float2*>(src);
                v[k][0] = f.x; v[k][1] = f.y;
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float mn = fmaxf(m[k], st[k].m), ms = mn == -INFINITY ? 0.0f : mn;
            const float old = exp2f(m[k] - ms), by = exp2f(st[k].m - ms);
            m[k] = mn;
            l[k] = l[k] * old + st[k].l * by;
#pragma unroll
            for (int e = 0; e < PER; ++e) o[k][e] = o[k][e] * old + v[k][e] * by;
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (r0 + k >= rows) break;
        const float by = l[k] == 0.0f ? 0.0f : 1.0f / l[k];
        const int r = p.tile * BIG_ROWS + r0 + k, i = by_group(a, r), tok = q.off + i, hd = p.head * a.group + r - i * a.group;
        T* dst = reinterpret_cast<T*>(a.out) + (long long)tok * a.o_tok + (long long)hd * a.o_head + lane * PER;
        if (PER == 4)
            *reinterpret_cast<uint2*>(dst) = make_uint2(Pair<T>::pack(o[k][0] * by, o[k][1] * by), Pair<T>::pack(o[k][PER - 2] * by, o[k][PER - 1] * by));
        else
            *reinterpret_cast<uint32_t*>(dst) = Pair<T>::pack(o[k][0] * by, o[k][1] * by);
        if (a.lse && lane == 0)
            a.lse[(long long)tok * a.n_heads + hd] = l[k] == 0.0f ? -INFINITY : (m[k] + log2f(l[k])) * 0.69314718055994530942f;
    }
}

template <typename T, int D, int ROWS>
cudaError_t run(const AttnView& a, int workers, const Partial* meta, const RowState* state, const float* part, cudaStream_t st) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    constexpr bool BIG = ROWS == BIG_ROWS;
    cfg.gridDim = BIG ? dim3((unsigned)workers, BIG_ROWS / BIG_SPAN) : dim3((unsigned)(workers < BLOCKS ? workers : BLOCKS));
    cfg.blockDim = dim3((BIG ? BIG_WARPS : WARPS) * 32);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    launch_hook("k_attn_combine", 0, st);
    cudaError_t e;
    if constexpr (BIG) e = cudaLaunchKernelEx(&cfg, k_attn_combine_tiles<T, D>, a, meta, state, part);
    else e = cudaLaunchKernelEx(&cfg, k_attn_combine<T, D, ROWS>, a, meta, workers, state, part);
    launch_hook("k_attn_combine", 1, st);
    return e;
}
template <typename T, int D>
cudaError_t with_rows(const AttnView& a, int rows, int workers, const Partial* meta, const RowState* state, const float* part,
                      cudaStream_t st) {
    if (rows == 8) return run<T, D, 8>(a, workers, meta, state, part, st);
    return rows == 16 ? run<T, D, 16>(a, workers, meta, state, part, st) : run<T, D, 256>(a, workers, meta, state, part, st);
}
template <typename T>
cudaError_t with_dim(const AttnView& a, int rows, int workers, const Partial* meta, const RowState* state, const float* part,
                     cudaStream_t st) {
    return a.kv.head_dim == 64 ? with_rows<T, 64>(a, rows, workers, meta, state, part, st)
                               : with_rows<T, 128>(a, rows, workers, meta, state, part, st);
}

}  // namespace

cudaError_t launch_attn_combine(const AttnView& a, int type, int rows, int workers, const Partial* meta, const RowState* state,
                                const float* part, cudaStream_t st) {
    return type == HOS_TYPE_BF16 ? with_dim<__nv_bfloat16>(a, rows, workers, meta, state, part, st)
                                 : with_dim<__half>(a, rows, workers, meta, state, part, st);
}

}  // namespace hos
