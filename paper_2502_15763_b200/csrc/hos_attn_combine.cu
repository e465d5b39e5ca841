// Second half of an attention call: the pieces of split tiles become outputs.
//
// A piece holds, per row, the unnormalised output, the maximum m and the normaliser l of its tokens (exponents
// in base 2), so out = sum_i 2^(mt_i - m) o_i / sum_i 2^(m_i - m) l_i with m = max_i m_i.  Pieces are added in list
// order.  Launched so that it may start while the attention kernel drains.
#include "hos_kernels.h"
#include "hos_kv.cuh"

namespace hos {
namespace {

// Joins the pieces of the tiles that the workers' shares cut: block (w, y) has rows 16 y .. 16 y + 15 of the tile that begins in worker
// w's share and ends in a later one's; the pieces are slot 1 of w and slot 0 of the workers up to `last`.
constexpr int COMBINE_WARPS = 8;
template <typename T, int D, int ROWS>
__global__ void __launch_bounds__(COMBINE_WARPS * 32) k_attn_combine(const __grid_constant__ AttnView a, const Partial* __restrict__ meta,
                                                                    const RowState* __restrict__ state,
                                                                    const float* __restrict__ part) {
    pdl_wait();
    const int w = (int)blockIdx.x;
    const Partial p = meta[w];
    if (p.last < 0) return;
    constexpr int PER = D / 32;                // elements a lane
    const SeqInfo q = load_seq(a.kv, p.seq, false);
    const int rows = min(min(ROWS, q.n * a.group - p.tile * ROWS), (int)(blockIdx.y + 1) * 16);
    for (int r = blockIdx.y * 16 + warp_id(); r < rows; r += COMBINE_WARPS) {
        // row state i of the pieces: slot 2w + 1, then 2(w + 1), 2(w + 2), ...
        auto slot = [&](int i) { return (long long)(i == 0 ? 2 * w + 1 : 2 * (w + i)) * ROWS + r; };
        const int n = p.last - w + 1;
        float m = -INFINITY;
        for (int i = lane_id(); i < n; i += 32) m = fmaxf(m, state[slot(i)].m);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL, m, d));
        const float ms = m == -INFINITY ? 0.0f : m;
        float l = 0.0f, o[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) o[i] = 0.0f;
        for (int i0 = 0; i0 < n; i0 += 32) {
            float by = 0.0f;
            if (i0 + lane_id() < n) {
                const RowState st = state[slot(i0 + lane_id())];
                l += st.l * exp2f(st.m - ms);
                by = st.mt == -INFINITY ? 0.0f : exp2f(st.mt - ms);
            }
            const int some = min(32, n - i0);
#pragma unroll 8
            for (int i = 0; i < some; ++i) {
                const float b = __shfl_sync(FULL, by, i);
                const float* src = part + slot(i0 + i) * D + lane_id() * PER;
                if (PER == 4) {
                    const float4 v = *reinterpret_cast<const float4*>(src);
                    o[0] += b * v.x; o[1] += b * v.y; o[PER - 2] += b * v.z; o[PER - 1] += b * v.w;
                } else {
                    const float2 v = *reinterpret_cast<const float2*>(src);
                    o[0] += b * v.x; o[1] += b * v.y;
                }
            }
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(FULL, l, d);
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
        const int row = p.tile * ROWS + r, tok = q.off + row / a.group, hd = p.head * a.group + row % a.group;
        T* dst = reinterpret_cast<T*>(a.out) + (long long)tok * a.o_tok + (long long)hd * a.o_head + lane_id() * PER;
        if (PER == 4)
            *reinterpret_cast<uint2*>(dst) = make_uint2(Pair<T>::pack(o[0] * by, o[1] * by), Pair<T>::pack(o[PER - 2] * by, o[PER - 1] * by));
        else
            *reinterpret_cast<uint32_t*>(dst) = Pair<T>::pack(o[0] * by, o[1] * by);
        if (a.lse && lane_id() == 0)
            a.lse[(long long)tok * a.n_heads + hd] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
    }
}

template <typename T, int D, int ROWS>
cudaError_t run(const AttnView& a, int workers, const Partial* meta, const RowState* state, const float* part, cudaStream_t st) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)workers, (ROWS + 15) / 16);
    cfg.blockDim = dim3(COMBINE_WARPS * 32);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    launch_hook("k_attn_combine", 0, st);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_attn_combine<T, D, ROWS>, a, meta, state, part);
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
