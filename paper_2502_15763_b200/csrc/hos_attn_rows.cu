// Attention of few query rows per sequence and KV head (decode rounds, short chunks) to the paged cache.
//
// What bounds it: the cache is read once, 2 * head_dim multiply-adds per cached element and 16 rows at
// most, so HBM.  The kernel is built to keep loads in flight and nothing else:
//   - The work is a list of steps of 16 tokens (sequence, KV head, tile of 8 or 16 rows, step).  Every WARP
//     takes an equal, contiguous share of the list, whatever the lengths are; there is no barrier
//     wider than a warp.  A tile cut by the ends of a share leaves a partial result (unnormalised output,
//     maximum, normaliser) in the workspace, and k_attn_combine joins the pieces in list order, so the
//     result does not depend on which warp finished first.
//   - A warp copies its next steps into its own ring in shared memory (16-byte asynchronous copies), over
//     the ends of tiles and sequences, while it works on the current one.
//   - Rows are the query heads of a group times the new tokens.  Both products are 16x8x16 matrix
//     instructions with the rows as the 8 columns: S^T = K Q^T (16 tokens x 8 rows) and O^T += V^T P^T
//     (16 of head_dim x 8 rows), so a tile of 8 rows wastes nothing.  The k index of the first product and the
//     row index of the second may be permuted freely (the same way on both sides), so each lane reads its
//     operands as whole 16-byte chunks of K and V rows; nothing is transposed but pairs of V rows (one byte
//     permute a register) and the weights (one 8x8 exchange a half step).
//   - 8-bit codes become fp16 exactly; K's scale multiplies the score, V's scale joins the exponent of
//     the weight (w_j = exp2(x_j + log2 vs_j - max of that)), so no weight under- or overflows fp16
//     whatever the scales are.
#include "hos_attn_list.cuh"
#include "hos_kernels.h"
#include "hos_kv.cuh"

namespace hos {
namespace {

constexpr int STEP = 16, WARPS = 4;
constexpr int MIN_STEPS = 2;                  // a worker's smallest share; fewer and the joining costs more than it saves

template <typename T, int FMT, int D, int NB> struct Cfg {
    static constexpr bool Q8 = FMT != HOS_KV_SAME;
    static constexpr int ROWS = 8 * NB;
    static constexpr int ROW_BYTES = Q8 ? D : 2 * D;
    static constexpr int CHUNKS = ROW_BYTES / 16;
    static constexpr int KV_BYTES = STEP * ROW_BYTES;
    static constexpr int STAGE = 2 * KV_BYTES + (Q8 ? 2 * STEP * 4 : 0);
    // CTAs of four warps on an SM, and the ring of each warp: as many bytes as fit
    static constexpr int CTAS = !Q8 && D == 128 ? 2 : NB == 1 ? 4 : 2;
    static constexpr int STAGES = (int)(SMEM_LIMIT / CTAS - 1024) / (WARPS * STAGE) < 8 ? (int)(SMEM_LIMIT / CTAS - 1024) / (WARPS * STAGE) : 8;
    static constexpr int SMEM = WARPS * STAGES * STAGE;
};
// A row's weights are 2^(x - (maximum - LIFT)): in fp16 the largest is 2^14, so that small ones keep their bits
// down to 2^-28 of it.
template <typename M> constexpr float LIFT = std::is_same<M, __half>::value ? 14.0f : 0.0f;
template <typename T, int FMT> struct MatType { using type = __half; };
template <typename T> struct MatType<T, HOS_KV_SAME> { using type = T; };

// Where chunk c of row r of a step lies in its row: spreads both access patterns (eight lanes reading four
// chunks of two neighbouring rows; the same chunk pair of every second row) over the banks.
template <int CHUNKS> __device__ __forceinline__ int swizzle(int r) {
    return CHUNKS == 4 ? (r >> 1) & 3 : (((r >> 1) & 1) << 1) | ((((r >> 2) ^ r) & 1) << 2);
}

// Transposes an 8x8 matrix of 16-bit elements held as one pair a lane (lane / 4: row, lane % 4: pair of columns).
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// Over the eight lanes of a column of 8x8 results.
__device__ __forceinline__ float column_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(FULL, v, 4));
    v = fmaxf(v, __shfl_xor_sync(FULL, v, 8));
    return fmaxf(v, __shfl_xor_sync(FULL, v, 16));
}
__device__ __forceinline__ float column_sum(float v) {
    v += __shfl_xor_sync(FULL, v, 4);
    v += __shfl_xor_sync(FULL, v, 8);
    return v + __shfl_xor_sync(FULL, v, 16);
}

template <typename T, int FMT, int D, int NB>
__global__ void __launch_bounds__(WARPS * 32, Cfg<T, FMT, D, NB>::CTAS)
k_attn_rows(const __grid_constant__ AttnView a, const int max_rows, Partial* __restrict__ meta,
            RowState* __restrict__ state, float* __restrict__ part) {
    using C = Cfg<T, FMT, D, NB>;
    using M = typename MatType<T, FMT>::type;
    using List = AttnList<C::ROWS, STEP>;
    using Cursor = typename List::Cursor;
    constexpr int ROWS = C::ROWS;
    constexpr int KS = D / 16;                 // matrix instructions along head_dim, and tiles of O^T
    extern __shared__ __align__(128) unsigned char smem[];
    const int lane = lane_id(), g = lane >> 2, t4 = lane & 3;
    const int workers = (int)gridDim.x * WARPS;
    const int w = warp_id() * (int)gridDim.x + (int)blockIdx.x;
    pdl_launch_dependents();

    // this warp's share of the list
    const List list{a, 0, max_rows};
    const long long total = list.total(w == 0);
    const int active = (int)min((long long)workers, (total + MIN_STEPS - 1) / MIN_STEPS);
    if (w >= active) {
        if (lane == 0) meta[w].last = -1;
        return;
    }
    const long long lo = total * w / active, hi = total * (w + 1) / active;
    Cursor cons = list.locate(lo);
    Cursor prod = cons;
    int to_issue = (int)(hi - lo);
    const uint32_t ring = smem_u32(smem) + warp_id() * C::STAGES * C::STAGE;

    // --- copies -------------------------------------------------------------------------------
    int pages = 0, pages_at = -1;              // this lane's entry of 32 cached page numbers, and the first one's index
    auto issue = [&](int stage) {
        if (to_issue > 0) {
            --to_issue;
            const int j0 = prod.t.k0 + prod.step * STEP;
            const int pi = j0 >> a.kv.page_shift;
            if (pages_at < 0 || pi >= pages_at + 32) {
                pages_at = pi;
                pages = -1;
                if (pi + lane <= (prod.t.ke - 1) >> a.kv.page_shift && prod.t.ke > 0) {
                    pages = __ldg(a.kv.table + (long long)prod.seq * a.kv.table_stride + pi + lane);
                    if ((unsigned)pages >= (unsigned)a.kv.n_pages) {
                        pages = -1;
                        if (a.kv.status) atomicOr(a.kv.status + prod.seq, HOS_ST_INVALID);
                    }
                }
            }
            const int page = __shfl_sync(FULL, pages, pi - pages_at);
            const int row0 = j0 & ((1 << a.kv.page_shift) - 1);
            const long long e = page_elem(a.kv, max(page, 0), prod.head, row0) * (C::Q8 ? 1 : 2);
            const unsigned char* ksrc = a.kv.k + e;
            const unsigned char* vsrc = a.kv.v + e;
            const uint32_t kd = ring + stage * C::STAGE, vd = kd + C::KV_BYTES;
#pragma unroll
            for (int it = 0; it < STEP * C::CHUNKS / 32; ++it) {
                const int id = it * 32 + lane, r = id / C::CHUNKS, c = id % C::CHUNKS;
                const bool real = page >= 0 && j0 + r >= prod.t.kb && j0 + r < prod.t.ke;
                const uint32_t dst = r * C::ROW_BYTES + ((c ^ swizzle<C::CHUNKS>(r)) * 16);
                cp_async16(kd + dst, ksrc + (long long)id * 16, real);
                cp_async16(vd + dst, vsrc + (long long)id * 16, real);
            }
            if (C::Q8 && lane < 8) {
                const long long se = scale_elem(a.kv, max(page, 0), prod.head, row0) + (lane & 3) * 4;
                cp_async16(vd + C::KV_BYTES + lane * 16, (lane < 4 ? a.kv.k_scale : a.kv.v_scale) + se, page >= 0);
            }
            if (++prod.step == prod.t.steps && to_issue > 0) {
                list.next(prod);
                pages_at = -1;
            }
        }
        cp_async_commit();
    };
#pragma unroll 1
    for (int i = 0; i < C::STAGES - 1; ++i) issue(i);

    // --- the rows of the current tile ---------------------------------------------------------
    // as columns of a product: row nb * 8 + g when read, rows nb * 8 + 2 * t4 + {0, 1} of the results
    uint32_t bq[KS][NB][2];
    float o[KS][NB][4];
    float m[NB][2], l[NB][2], mt[NB][2], qmul[NB][2];
    int see_lo[NB][2], see_hi[NB][2];          // visible tokens
    const int f = swizzle<C::CHUNKS>(g);
    const uint32_t k_at = g * C::ROW_BYTES + (t4 ^ (f & 3)) * 16, k_x = (f & 4) * 16;

    auto begin = [&]() {
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][nb][j] = 0.0f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int r = cons.tile * ROWS + nb * 8 + g;
            const bool there = nb * 8 + g < cons.t.rows;
            const int i = r / a.group, hd = cons.head * a.group + r % a.group;
            const T* src = reinterpret_cast<const T*>(a.q) + (long long)(cons.q.off + i) * a.q_tok + (long long)hd * a.q_head;
            uint32_t x[2 * KS];
#pragma unroll
            for (int c = 0; c < KS / 2; ++c) {
                // lane t4's chunks: 8 elements at (c * 4 + t4) * 8, or with 8-bit keys pairs of them (16 elements)
                const int d = C::Q8 ? ((c >> 1) * 4 + t4) * 16 + (c & 1) * 8 : (c * 4 + t4) * 8;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (there) v = __ldg(reinterpret_cast<const uint4*>(src + d));
                x[4 * c] = v.x; x[4 * c + 1] = v.y; x[4 * c + 2] = v.z; x[4 * c + 3] = v.w;
            }
            float mul = a.scale_log2;
            if (C::Q8 && !std::is_same<T, __half>::value) {
                // bf16 queries meet fp16 keys: a power of two per row brings the row into fp16's range
                // (exact but for elements 2^-38 of the row's largest)
                float top = 0.0f;
#pragma unroll
                for (int i2 = 0; i2 < 2 * KS; ++i2) {
                    const float2 v = Pair<T>::unpack(x[i2]);
                    top = fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y)));
                }
                top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
                top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
                const int ex = (int)(__float_as_uint(top) >> 23);            // biased; top >= 0
                // top * 2^(140 - ex) is in [2^13, 2^14); rows of zeros, denormals or non-finite values stay
                const int sh = ex >= 27 && ex < 254 ? 140 - ex : 0;
                const float up = __uint_as_float((uint32_t)(127 + sh) << 23);
                mul *= __uint_as_float((uint32_t)(127 - sh) << 23);
#pragma unroll
                for (int i2 = 0; i2 < 2 * KS; ++i2) {
                    const float2 v = Pair<T>::unpack(x[i2]);
                    x[i2] = Pair<__half>::pack(v.x * up, v.y * up);
                }
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) { bq[ks][nb][0] = x[2 * ks]; bq[ks][nb][1] = x[2 * ks + 1]; }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r2 = cons.tile * ROWS + nb * 8 + 2 * t4 + e;
                const int pos = cons.q.len - cons.q.n + r2 / a.group;
                see_hi[nb][e] = nb * 8 + 2 * t4 + e < cons.t.rows ? (a.causal ? min(cons.q.len, pos + 1) : cons.q.len) : 0;
                see_lo[nb][e] = a.window > 0 ? max(0, pos - a.window + 1) : 0;
                qmul[nb][e] = __shfl_sync(FULL, mul, (2 * t4 + e) * 4);
                m[nb][e] = mt[nb][e] = -INFINITY;
                l[nb][e] = 0.0f;
            }
        }
    };

    // Tiles 4 q .. 4 q + 3 of O^T are eight consecutive elements of head_dim in this lane.
    auto dim_of = [&](int q) { return C::Q8 && D == 128 ? g * 16 + q * 8 : q * 64 + g * 8; };
    bool open_end = false;
    int seg_first = cons.step;                 // the step of the tile this warp began with
    auto finish = [&](long long unit) {
        const bool whole_start = seg_first == 0, whole_end = cons.step == cons.t.steps - 1;
        const bool whole = whole_start && whole_end;
        const int slot = 2 * w + (whole_start ? 1 : 0);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float sum = column_sum(l[nb][e]);
                const int in_tile = nb * 8 + 2 * t4 + e;
                if (in_tile >= cons.t.rows) continue;
                if (whole) {
                    const int r = cons.tile * ROWS + in_tile;
                    const int tok = cons.q.off + r / a.group, hd = cons.head * a.group + r % a.group;
                    float by = sum == 0.0f ? 0.0f : 1.0f / sum;
                    if (C::Q8 && sum != 0.0f) by *= exp2f(mt[nb][e] - m[nb][e]);
                    T* dst = reinterpret_cast<T*>(a.out) + (long long)tok * a.o_tok + (long long)hd * a.o_head;
#pragma unroll
                    for (int q = 0; q < KS / 4; ++q) {
                        uint32_t v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = Pair<T>::pack(o[4 * q + i][nb][e] * by, o[4 * q + i][nb][2 + e] * by);
                        *reinterpret_cast<uint4*>(dst + dim_of(q)) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                    if (a.lse && g == 0)
                        a.lse[(long long)tok * a.n_heads + hd] =
                            sum == 0.0f ? -INFINITY : (m[nb][e] + log2f(sum)) * 0.69314718055994530942f;
                } else {
                    const long long r = (long long)slot * ROWS + in_tile;
#pragma unroll
                    for (int q = 0; q < KS / 4; ++q)
#pragma unroll
                        for (int i = 0; i < 4; i += 2)
                            *reinterpret_cast<float4*>(part + r * D + dim_of(q) + 2 * i) =
                                make_float4(o[4 * q + i][nb][e], o[4 * q + i][nb][2 + e], o[4 * q + i + 1][nb][e], o[4 * q + i + 1][nb][2 + e]);
                    if (g == 0) state[r] = RowState{m[nb][e], sum, C::Q8 ? mt[nb][e] : m[nb][e], 0.0f};
                }
            }
        if (!whole && whole_start && lane == 0) {
            const long long end = unit + (cons.t.steps - cons.step);      // one past the tile's last step
            meta[w] = Partial{cons.seq, cons.head, cons.tile, (int)((end * active - 1) / total)};
        }
        open_end = whole_start && !whole_end;
    };

    begin();
    int stage = 0;
#pragma unroll 1
    for (long long unit = lo; unit < hi; ++unit) {
        cp_async_wait<C::STAGES - 2>();
        __syncwarp();
        issue(stage == 0 ? C::STAGES - 1 : stage - 1);
        const uint32_t kd = ring + stage * C::STAGE, vd = kd + C::KV_BYTES;
        if (++stage == C::STAGES) stage = 0;

        // scores: x[nb][0..1] token g, x[nb][2..3] token g + 8, rows nb * 8 + 2 * t4 + {0, 1}
        float x[NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[nb][j] = 0.0f;
#pragma unroll
        for (int c = 0; c < C::CHUNKS / 4; ++c) {
            const uint4 v0 = lds128(kd + k_at + ((c * 64) ^ k_x)), v1 = lds128(kd + 8 * C::ROW_BYTES + k_at + ((c * 64) ^ k_x));
            const uint32_t w0[4] = {v0.x, v0.y, v0.z, v0.w}, w1[4] = {v1.x, v1.y, v1.z, v1.w};
            if (!C::Q8) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t ak[4] = {w0[2 * i], w1[2 * i], w0[2 * i + 1], w1[2 * i + 1]};
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma16816<M>(x[nb], ak, bq[2 * c + i][nb][0], bq[2 * c + i][nb][1]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t ak[4] = {codes_to_half2<FMT>(w0[i]), codes_to_half2<FMT>(w1[i]), codes_to_half2<FMT>(w0[i] >> 16),
                                            codes_to_half2<FMT>(w1[i] >> 16)};
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma16816<M>(x[nb], ak, bq[(4 * c + i) % KS][nb][0], bq[(4 * c + i) % KS][nb][1]);
                }
            }
        }
        const int j0 = cons.t.k0 + cons.step * STEP;
        float ks[2] = {1.0f, 1.0f}, lv[2] = {0.0f, 0.0f};      // of tokens g and g + 8: K's scale, log2 of V's
        if (C::Q8) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                ks[i] = lds32f(vd + C::KV_BYTES + (g + 8 * i) * 4);
                lv[i] = __log2f(lds32f(vd + C::KV_BYTES + (STEP + g + 8 * i) * 4));
            }
        }
        float shrink[NB][2];
        uint32_t bp[NB][2];
        bool moved = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int e = j & 1, tok = j0 + g + 8 * (j >> 1);
                x[nb][j] *= C::Q8 ? qmul[nb][e] * ks[j >> 1] : a.scale_log2;
                if (tok < see_lo[nb][e] || tok >= see_hi[nb][e]) x[nb][j] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float top = column_max(fmaxf(x[nb][e], x[nb][2 + e]));
                const float mn = fmaxf(m[nb][e], C::Q8 ? top : top - LIFT<M>), ms = mn == -INFINITY ? 0.0f : mn;
                shrink[nb][e] = exp2_fast(m[nb][e] - ms);
                m[nb][e] = mn;
                p[e] = exp2_fast(x[nb][e] - ms);
                p[2 + e] = exp2_fast(x[nb][2 + e] - ms);
                l[nb][e] = l[nb][e] * shrink[nb][e] + (p[e] + p[2 + e]);
                if (C::Q8) {
                    const float y0 = x[nb][e] == -INFINITY ? -INFINITY : x[nb][e] + lv[0];
                    const float y1 = x[nb][2 + e] == -INFINITY ? -INFINITY : x[nb][2 + e] + lv[1];
                    const float yn = fmaxf(mt[nb][e], column_max(fmaxf(y0, y1)) - LIFT<M>), ys = yn == -INFINITY ? 0.0f : yn;
                    shrink[nb][e] = exp2_fast(mt[nb][e] - ys);
                    mt[nb][e] = yn;
                    p[e] = exp2_fast(y0 - ys);
                    p[2 + e] = exp2_fast(y1 - ys);
                }
                moved |= shrink[nb][e] != 1.0f;
            }
            bp[nb][0] = transpose8x8(Pair<M>::pack(p[0], p[1]));
            bp[nb][1] = transpose8x8(Pair<M>::pack(p[2], p[3]));
        }
        if (__any_sync(FULL, moved)) {
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[i][nb][j] *= shrink[nb][j & 1];
        }
        // O^T += V^T P^T: this lane's rows of V are tokens 2 * t4 + {0, 1, 8, 9}
        if (!C::Q8) {
#pragma unroll
            for (int half = 0; half < D / 64; ++half) {
                uint4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 2 * t4 + (i & 1) + (i >> 1) * 8;
                    v[i] = lds128(vd + r * C::ROW_BYTES + ((g ^ swizzle<C::CHUNKS>(r)) + half * 8) * 16);
                }
                const uint32_t vw[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w},
                                           {v[2].x, v[2].y, v[2].z, v[2].w}, {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t av[4] = {__byte_perm(vw[0][i], vw[1][i], 0x5410), __byte_perm(vw[0][i], vw[1][i], 0x7632),
                                            __byte_perm(vw[2][i], vw[3][i], 0x5410), __byte_perm(vw[2][i], vw[3][i], 0x7632)};
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma16816<M>(o[half * 4 + i][nb], av, bp[nb][0], bp[nb][1]);
                }
            }
        } else {
            constexpr int WORDS = D / 32;      // 32-bit words of a lane's codes per V row
            uint32_t vw[4][WORDS];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 2 * t4 + (i & 1) + (i >> 1) * 8;
                const int sw = swizzle<C::CHUNKS>(r);
                if (D == 128) {
                    const uint4 v = lds128(vd + r * C::ROW_BYTES + (g ^ sw) * 16);
                    vw[i][0] = v.x; vw[i][1] = v.y; vw[i][WORDS - 2] = v.z; vw[i][WORDS - 1] = v.w;
                } else {
                    const uint2 v = lds64(vd + r * C::ROW_BYTES + ((g >> 1) ^ sw) * 16 + (g & 1) * 8);
                    vw[i][0] = v.x; vw[i][1] = v.y;
                }
            }
#pragma unroll
            for (int i = 0; i < WORDS; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t x0 = __byte_perm(vw[0][i], vw[1][i], k ? 0x7362 : 0x5140);
                    const uint32_t x1 = __byte_perm(vw[2][i], vw[3][i], k ? 0x7362 : 0x5140);
                    const uint32_t av[4] = {codes_to_half2<FMT>(x0), codes_to_half2<FMT>(x0 >> 16), codes_to_half2<FMT>(x1), codes_to_half2<FMT>(x1 >> 16)};
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma16816<M>(o[2 * i + k][nb], av, bp[nb][0], bp[nb][1]);
                }
        }
        const bool tile_done = cons.step == cons.t.steps - 1;
        if (tile_done || unit + 1 == hi) {
            finish(unit);
            if (unit + 1 < hi) {
                list.next(cons);
                seg_first = 0;
                begin();
            }
        } else {
            ++cons.step;
        }
    }
    if (!open_end && lane == 0) meta[w].last = -1;
    cp_async_wait<0>();
}

template <typename T, int FMT, int D, int NB>
cudaError_t run(const AttnView& a, int max_rows, Partial* meta, RowState* state, float* part, cudaStream_t st) {
    using C = Cfg<T, FMT, D, NB>;
    static_assert(C::CTAS * C::ROWS <= ATTN_ROWS_PER_SM / WARPS, "workspace");
    const void* f = reinterpret_cast<const void*>(&k_attn_rows<T, FMT, D, NB>);
    cudaError_t e = allow_max_dynamic_smem(f);
    if (e != cudaSuccess) return e;
    const int ctas = 148 * C::CTAS;
    launch_hook("k_attn_rows", 0, st);
    k_attn_rows<T, FMT, D, NB><<<ctas, WARPS * 32, C::SMEM, st>>>(a, max_rows, meta, state, part);
    launch_hook("k_attn_rows", 1, st);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    return launch_attn_combine(a, std::is_same<T, __half>::value ? HOS_TYPE_FP16 : HOS_TYPE_BF16, C::ROWS, ctas * WARPS, meta,
                               state, part, st);
}

}  // namespace

cudaError_t launch_attn_rows(const AttnView& a, int type, int format, int tile_rows, int max_rows, Partial* meta, RowState* state,
                             float* part, cudaStream_t st) {
    return kv_dispatch(type, format, a.kv.head_dim, [&](auto t, auto f, auto d) {
        using T = typename decltype(t)::type;
        return tile_rows == 8 ? run<T, decltype(f)::value, decltype(d)::value, 1>(a, max_rows, meta, state, part, st)
                              : run<T, decltype(f)::value, decltype(d)::value, 2>(a, max_rows, meta, state, part, st);
    });
}

}  // namespace hos
