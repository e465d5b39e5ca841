// Second half of an attention call: the pieces of split tiles become outputs.
//
// A piece holds, per row, the unnormalised output, the reference m and the normaliser l of its tokens (exponents
// in base 2), so out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i with m = max_i m_i.  Pieces are added in list
// order.  Launched so that it may start while the attention kernel drains.  Bound by the latency of two or three dependent loads:
// 5-7 us for the row kernel's pieces, 8 us for 294 pieces of 256 rows (40 MB).
#include "hos_kv_kernels.h"
#include "hos_kv.cuh"

namespace hos {
namespace {

// Worker w's record, if it has one, names the tile that begins in its share and ends in a later one's: the pieces are slot 1
// of w and slot 0 of the workers up to `last`.  One kernel joins both kinds of tiles: first come the blocks of the row
// kernel's records, one each, then those of the chunk kernel's, four each.
constexpr int WARPS = 16, BIG_ROWS = ATTN_CHUNK_ROWS, BIG_BLOCKS = BIG_ROWS / (4 * WARPS);

// A tile of 8 or 16 rows, maybe many pieces: the warps take rows, and where there are fewer rows than warps several warps share a
// row's pieces.  D / 4 lanes read a piece's row.
template <typename T, int D, int ROWS>
__device__ __forceinline__ void join_rows(const AttnView& a, const AttnWs& ws, int w) {
    constexpr int LANES = D / 4, PER = 32 / LANES;                     // pieces that a warp reads at once
    __shared__ float4 sum_o[WARPS][LANES];
    __shared__ float sum_l[WARPS];
    const int lane = lane_id(), warp = warp_id(), sub = lane / LANES;
    const Partial p = ws.meta[w];
    if (p.last < 0) return;
    const SeqInfo q = load_seq(a.kv, p.seq, false);
    const int n = p.last - w + 1, rows = min(ROWS, q.n * a.group - p.tile * ROWS);
    const int shares = rows > 8 ? 1 : rows > 4 ? 2 : rows > 2 ? 4 : rows == 2 ? 8 : 16;   // warps a row
    const int row = warp / shares, share = warp % shares;
    const bool busy = row < rows;
    auto slot = [&](int i) { return (long long)(i == 0 ? 2 * w + 1 : 2 * (w + i)) * ROWS + row; };
    float m = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (busy) {
        for (int i = lane; i < n; i += 32) m = fmaxf(m, ws.state[slot(i)].m);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL, m, d));
        const float ms = m == -INFINITY ? 0.0f : m;
        // pieces share * PER + sub, + shares * PER, ...
#pragma unroll 4
        for (int i = share * PER + sub; i < n; i += shares * PER) {
            const RowState st = ws.state[slot(i)];
            const float4 v = reinterpret_cast<const float4*>(ws.part + slot(i) * D)[lane % LANES];
            const float by = exp2f(st.m - ms);
            if (lane % LANES == 0) l += st.l * by;
            o.x += by * v.x; o.y += by * v.y; o.z += by * v.z; o.w += by * v.w;
        }
        if (PER == 2) {
            __syncwarp();
            o.x += __shfl_xor_sync(FULL, o.x, 16); o.y += __shfl_xor_sync(FULL, o.y, 16);
            o.z += __shfl_xor_sync(FULL, o.z, 16); o.w += __shfl_xor_sync(FULL, o.w, 16);
            l += __shfl_xor_sync(FULL, l, 16);
        }
        if (lane < LANES) sum_o[warp][lane] = o;
        if (lane == 0) sum_l[warp] = l;
    }
    __syncthreads();
    if (!busy || share != 0) return;
    l = 0.0f;
    for (int k = 0; k < shares; ++k) l += sum_l[warp + k];
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
    const int r = p.tile * ROWS + row, i = by_group(a, r), tok = q.off + i, hd = p.head * a.group + r - i * a.group;
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
        a.lse[(long long)tok * a.n_heads + hd] = row_lse(m, l);
}

// A quarter of a tile of 256 rows, mostly of two or three pieces, which hold four columns of every row together: a warp takes four
// rows, eight lanes to each, and goes through the pieces with a running maximum; its loads do not wait for one another.
template <typename T, int D>
__device__ __forceinline__ void join_tile(const AttnView& a, const AttnWs& ws, int w, int quarter) {
    constexpr int PER = D / 32;                // groups of four columns a lane: g, g + 8, ...
    const int lane = lane_id(), g = lane >> 2;
    const Partial p = ws.meta[w];
    if (p.last < 0) return;
    const SeqInfo q = load_seq(a.kv, p.seq, false);
    const int rows = min(BIG_ROWS, q.n * a.group - p.tile * BIG_ROWS), row = (quarter * WARPS + warp_id()) * 4 + (lane & 3);
    float m = -INFINITY, l = 0.0f;
    float4 o[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const int n = row < rows ? p.last - w + 1 : 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const long long slot = i == 0 ? 2 * w + 1 : 2 * (w + i);
        const RowState st = ws.state[slot * BIG_ROWS + row];
        const float4* src = reinterpret_cast<const float4*>(ws.part) + slot * (BIG_ROWS * D / 4) + row;
        float4 v[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = src[(g + 8 * e) * BIG_ROWS];
        const float mn = fmaxf(m, st.m), ms = mn == -INFINITY ? 0.0f : mn;
        const float old = exp2f(m - ms), by = exp2f(st.m - ms);
        m = mn;
        l = l * old + st.l * by;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            o[e].x = o[e].x * old + v[e].x * by; o[e].y = o[e].y * old + v[e].y * by;
            o[e].z = o[e].z * old + v[e].z * by; o[e].w = o[e].w * old + v[e].w * by;
        }
    }
    if (row >= rows) return;
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
    const int r = p.tile * BIG_ROWS + row, i = by_group(a, r), tok = q.off + i, hd = p.head * a.group + r - i * a.group;
    T* dst = reinterpret_cast<T*>(a.out) + (long long)tok * a.o_tok + (long long)hd * a.o_head;
#pragma unroll
    for (int e = 0; e < PER; ++e)
        reinterpret_cast<uint2*>(dst)[g + 8 * e] = make_uint2(Pair<T>::pack(o[e].x * by, o[e].y * by), Pair<T>::pack(o[e].z * by, o[e].w * by));
    if (a.lse && g == 0)
        a.lse[(long long)tok * a.n_heads + hd] = row_lse(m, l);
}

template <typename T, int D, int ROWS>
__global__ void __launch_bounds__(WARPS * 32) k_attn_combine(const __grid_constant__ AttnView a, const AttnWs rows, const int row_workers,
                                                            const AttnWs tiles) {
    pdl_launch_dependents();
    pdl_wait();
    const int b = (int)blockIdx.x;
    if (b < row_workers) join_rows<T, D, ROWS>(a, rows, b);
    else join_tile<T, D>(a, tiles, (b - row_workers) / BIG_BLOCKS, (b - row_workers) % BIG_BLOCKS);
}

template <typename T, int D, int ROWS>
cudaError_t run(const AttnView& a, bool chunks, const AttnWs& chunk_ws, int row_workers, const AttnWs& row_ws, cudaStream_t st) {
    launch_hook("k_attn_combine", 0, st);
    const cudaError_t e = launch_early(k_attn_combine<T, D, ROWS>, dim3((unsigned)(row_workers + (chunks ? ATTN_SMS * BIG_BLOCKS : 0))), WARPS * 32, 0, st,
                                       a, row_ws, row_workers, chunk_ws);
    launch_hook("k_attn_combine", 1, st);
    return e;
}

}  // namespace

cudaError_t launch_attn_combine(const AttnView& a, int type, bool chunks, const AttnWs& chunk_ws, int tile_rows, int row_workers,
                                const AttnWs& row_ws, cudaStream_t st) {
    return kv_dispatch(type, HOS_KV_SAME, a.kv.head_dim, [&](auto t, auto f, auto d) {
        using T = typename decltype(t)::type;
        (void)f;
        return tile_rows == 8 ? run<T, decltype(d)::value, 8>(a, chunks, chunk_ws, row_workers, row_ws, st)
                              : run<T, decltype(d)::value, 16>(a, chunks, chunk_ws, row_workers, row_ws, st);
    });
}

}  // namespace hos
