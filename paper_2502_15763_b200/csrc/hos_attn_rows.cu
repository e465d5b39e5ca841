// Attention of few query rows per sequence and KV head (decode rounds, short chunks) to the paged cache.
//
// What bounds it: the cache is read once, 2 * head_dim multiply-adds per cached element and 16 rows at
// most, so HBM.  The kernel is built to keep loads in flight and nothing else:
//   - The work is a list of steps of 16 tokens (sequence, KV head, tile of 16 rows, step).  Every WARP
//     takes an equal, contiguous share of the list, whatever the lengths are; there is no barrier
//     wider than a warp.  A tile cut by the ends of a share leaves a partial result (unnormalised output,
//     maximum, normaliser) in the workspace, and k_attn_combine joins the pieces in list order, so the
//     result does not depend on which warp finished first.
//   - A warp copies its next steps into its own ring in shared memory (16-byte asynchronous copies), over
//     the ends of tiles and sequences, while it works on the current one.
//   - Rows are the query heads of a group times the new tokens.  S = Q K^T and O += P V are 16x8x16 matrix
//     instructions.  The k index of the first product and the column index of the second may be
//     permuted freely (the same way on both sides), so each lane reads its operands as whole 16-byte
//     chunks of K and V rows; nothing is transposed but pairs of V rows (one byte permute a register).
//   - 8-bit codes become fp16 exactly; K's scale multiplies the score, V's scale joins the exponent of
//     the weight (w_j = exp2(x_j + log2 vs_j - max of that)), so no weight under- or overflows fp16
//     whatever the scales are.
#include "hos_attn_list.cuh"
#include "hos_kernels.h"
#include "hos_kv.cuh"

namespace hos {
namespace {

constexpr int ROWS = 16, STEP = 16, WARPS = 4;
using List = AttnList<ROWS, STEP>;
using Cursor = List::Cursor;
constexpr int MIN_STEPS = 2;                  // a worker's smallest share; fewer and the joining costs more than it saves

template <typename T, int FMT, int D> struct Cfg {
    static constexpr bool Q8 = FMT != HOS_KV_SAME;
    static constexpr int ROW_BYTES = Q8 ? D : 2 * D;
    static constexpr int CHUNKS = ROW_BYTES / 16;
    static constexpr int KV_BYTES = STEP * ROW_BYTES;
    static constexpr int STAGE = 2 * KV_BYTES + (Q8 ? 2 * STEP * 4 : 0);
    static constexpr int STAGES = Q8 ? (D == 128 ? 5 : 8) : (D == 128 ? 3 : 6);
    static constexpr int CTAS = Q8 ? 2 : 2;
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

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(WARPS * 32, Cfg<T, FMT, D>::CTAS)
k_attn_rows(const __grid_constant__ AttnView a, const int max_rows, Partial* __restrict__ meta,
            RowState* __restrict__ state, float* __restrict__ part) {
    using C = Cfg<T, FMT, D>;
    using M = typename MatType<T, FMT>::type;
    constexpr int KS = D / 16;                 // matrix instructions along head_dim
    constexpr int NT = D / 8;                  // column tiles of the output
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
    uint32_t aq[KS][4];
    float o[NT][4];
    float m[2], l[2], mt[2], qmul[2];          // [0]: row g, [1]: row g + 8
    int see_lo[2], see_hi[2];                  // visible tokens of the two rows
    const int f = swizzle<C::CHUNKS>(g);
    const uint32_t k_at = g * C::ROW_BYTES + (t4 ^ (f & 3)) * 16, k_x = (f & 4) * 16;

    auto begin = [&]() {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            m[h] = mt[h] = -INFINITY;
            l[h] = 0.0f;
            const int r = cons.tile * ROWS + g + 8 * h;
            const bool there = g + 8 * h < cons.t.rows;
            const int i = r / a.group, hd = cons.head * a.group + r % a.group;
            const int pos = cons.q.len - cons.q.n + i;
            see_hi[h] = there ? (a.causal ? min(cons.q.len, pos + 1) : cons.q.len) : 0;
            see_lo[h] = a.window > 0 ? max(0, pos - a.window + 1) : 0;
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
            qmul[h] = a.scale_log2;
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
                qmul[h] = a.scale_log2 * __uint_as_float((uint32_t)(127 - sh) << 23);
#pragma unroll
                for (int i2 = 0; i2 < 2 * KS; ++i2) {
                    const float2 v = Pair<T>::unpack(x[i2]);
                    x[i2] = Pair<__half>::pack(v.x * up, v.y * up);
                }
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) { aq[ks][h] = x[2 * ks]; aq[ks][2 + h] = x[2 * ks + 1]; }
        }
    };

    // Output column tile i, column 2 * t4 + cc of this lane: which element of head_dim.
    auto dim_of = [&](int i, int cc) {
        return C::Q8 && D == 128 ? (2 * t4 + cc) * 16 + i : (i >> 3) * 64 + (2 * t4 + cc) * 8 + (i & 7);
    };
    bool open_end = false;
    int seg_first = cons.step;                 // the step of the tile this warp began with
    auto finish = [&](long long unit) {
        const bool whole_start = seg_first == 0, whole_end = cons.step == cons.t.steps - 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(FULL, l[h], 1);
            l[h] += __shfl_xor_sync(FULL, l[h], 2);
        }
        if (whole_start && whole_end) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (g + 8 * h >= cons.t.rows) continue;
                const int r = cons.tile * ROWS + g + 8 * h;
                const int tok = cons.q.off + r / a.group, hd = cons.head * a.group + r % a.group;
                float by = l[h] == 0.0f ? 0.0f : 1.0f / l[h];
                if (C::Q8 && l[h] != 0.0f) by *= exp2f(mt[h] - m[h]);
                T* dst = reinterpret_cast<T*>(a.out) + (long long)tok * a.o_tok + (long long)hd * a.o_head;
#pragma unroll
                for (int cc = 0; cc < 2; ++cc)
#pragma unroll
                    for (int i = 0; i < NT; i += 8) {
                        uint4 v;
                        v.x = Pair<T>::pack(o[i][2 * h + cc] * by, o[i + 1][2 * h + cc] * by);
                        v.y = Pair<T>::pack(o[i + 2][2 * h + cc] * by, o[i + 3][2 * h + cc] * by);
                        v.z = Pair<T>::pack(o[i + 4][2 * h + cc] * by, o[i + 5][2 * h + cc] * by);
                        v.w = Pair<T>::pack(o[i + 6][2 * h + cc] * by, o[i + 7][2 * h + cc] * by);
                        *reinterpret_cast<uint4*>(dst + dim_of(i, cc)) = v;
                    }
                if (a.lse && t4 == 0)
                    a.lse[(long long)tok * a.n_heads + hd] =
                        l[h] == 0.0f ? -INFINITY : (m[h] + log2f(l[h])) * 0.69314718055994530942f;
            }
            return;
        }
        const int slot = 2 * w + (whole_start ? 1 : 0);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (g + 8 * h >= cons.t.rows) continue;
            const long long r = (long long)slot * ROWS + g + 8 * h;
            float* dst = part + r * D;
#pragma unroll
            for (int cc = 0; cc < 2; ++cc)
#pragma unroll
                for (int i = 0; i < NT; i += 4)
                    *reinterpret_cast<float4*>(dst + dim_of(i, cc)) =
                        make_float4(o[i][2 * h + cc], o[i + 1][2 * h + cc], o[i + 2][2 * h + cc], o[i + 3][2 * h + cc]);
            if (t4 == 0) state[r] = RowState{m[h], l[h], C::Q8 ? mt[h] : m[h], 0.0f};
        }
        if (whole_start && lane == 0) {
            const long long end = unit + (cons.t.steps - cons.step);      // one past the tile's last step
            meta[w] = Partial{cons.seq, cons.head, cons.tile, (int)((end * active - 1) / total)};
        }
        open_end = whole_start;
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

        // scores of 16 tokens: x[nt][0..1] row g, x[nt][2..3] row g + 8, tokens nt * 8 + 2 * t4 + {0, 1}
        float x[2][4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[nt][j] = 0.0f;
            const uint32_t at = kd + nt * 8 * C::ROW_BYTES + k_at;
#pragma unroll
            for (int c = 0; c < C::CHUNKS / 4; ++c) {
                const uint4 v = lds128(at + ((c * 64) ^ k_x));
                const uint32_t wv[4] = {v.x, v.y, v.z, v.w};
                if (!C::Q8) {
                    mma16816<M>(x[nt], aq[2 * c], wv[0], wv[1]);
                    mma16816<M>(x[nt], aq[2 * c + 1], wv[2], wv[3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        mma16816<M>(x[nt], aq[(4 * c + i) % KS], codes_to_half2<FMT>(wv[i]), codes_to_half2<FMT>(wv[i] >> 16));
                }
            }
        }
        const int j0 = cons.t.k0 + cons.step * STEP;
        const bool edge = j0 < see_lo[0] || j0 + STEP > see_hi[0] || j0 < see_lo[1] || j0 + STEP > see_hi[1];
        float vs[2][2];                        // log2 of V's scales
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            float ks0 = 1.0f, ks1 = 1.0f;
            if (C::Q8) {
                const uint2 kk = lds64(vd + C::KV_BYTES + (nt * 8 + 2 * t4) * 4);
                const uint2 vv = lds64(vd + C::KV_BYTES + STEP * 4 + (nt * 8 + 2 * t4) * 4);
                ks0 = __uint_as_float(kk.x); ks1 = __uint_as_float(kk.y);
                vs[nt][0] = __log2f(__uint_as_float(vv.x)); vs[nt][1] = __log2f(__uint_as_float(vv.y));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int h = j >> 1;
                x[nt][j] *= C::Q8 ? qmul[h] * ((j & 1) ? ks1 : ks0) : a.scale_log2;
                const int tok = j0 + nt * 8 + 2 * t4 + (j & 1);
                if (edge && (tok < see_lo[h] || tok >= see_hi[h])) x[nt][j] = -INFINITY;
            }
        }
        float shrink[2];
        uint32_t ap[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float top = fmaxf(fmaxf(x[0][2 * h], x[0][2 * h + 1]), fmaxf(x[1][2 * h], x[1][2 * h + 1]));
            top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
            top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
            const float mn = fmaxf(m[h], C::Q8 ? top : top - LIFT<M>), ms = mn == -INFINITY ? 0.0f : mn;
            shrink[h] = exp2_fast(m[h] - ms);
            m[h] = mn;
            float p[4], sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) { p[i] = exp2_fast(x[i >> 1][2 * h + (i & 1)] - ms); sum += p[i]; }
            l[h] = l[h] * shrink[h] + sum;
            if (C::Q8) {
                float y[4], ty = -INFINITY;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float xi = x[i >> 1][2 * h + (i & 1)];
                    y[i] = xi == -INFINITY ? xi : xi + vs[i >> 1][i & 1];
                    ty = fmaxf(ty, y[i]);
                }
                ty = fmaxf(ty, __shfl_xor_sync(FULL, ty, 1));
                ty = fmaxf(ty, __shfl_xor_sync(FULL, ty, 2));
                const float yn = fmaxf(mt[h], ty - LIFT<M>), ys = yn == -INFINITY ? 0.0f : yn;
                shrink[h] = exp2_fast(mt[h] - ys);
                mt[h] = yn;
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = exp2_fast(y[i] - ys);
            }
            ap[h] = Pair<M>::pack(p[0], p[1]);
            ap[2 + h] = Pair<M>::pack(p[2], p[3]);
        }
        if (__any_sync(FULL, shrink[0] != 1.0f || shrink[1] != 1.0f)) {
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                o[i][0] *= shrink[0]; o[i][1] *= shrink[0];
                o[i][2] *= shrink[1]; o[i][3] *= shrink[1];
            }
        }
        // O += P V: this lane's rows of V are tokens 2 * t4 + {0, 1, 8, 9}
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
                    mma16816<M>(o[half * 8 + 2 * i], ap, __byte_perm(vw[0][i], vw[1][i], 0x5410), __byte_perm(vw[2][i], vw[3][i], 0x5410));
                    mma16816<M>(o[half * 8 + 2 * i + 1], ap, __byte_perm(vw[0][i], vw[1][i], 0x7632), __byte_perm(vw[2][i], vw[3][i], 0x7632));
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
            for (int i = 0; i < WORDS; ++i) {
                const uint32_t x0 = __byte_perm(vw[0][i], vw[1][i], 0x5140), y0 = __byte_perm(vw[0][i], vw[1][i], 0x7362);
                const uint32_t x1 = __byte_perm(vw[2][i], vw[3][i], 0x5140), y1 = __byte_perm(vw[2][i], vw[3][i], 0x7362);
                mma16816<M>(o[4 * i], ap, codes_to_half2<FMT>(x0), codes_to_half2<FMT>(x1));
                mma16816<M>(o[4 * i + 1], ap, codes_to_half2<FMT>(x0 >> 16), codes_to_half2<FMT>(x1 >> 16));
                mma16816<M>(o[4 * i + 2], ap, codes_to_half2<FMT>(y0), codes_to_half2<FMT>(y1));
                mma16816<M>(o[4 * i + 3], ap, codes_to_half2<FMT>(y0 >> 16), codes_to_half2<FMT>(y1 >> 16));
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

template <typename T, int FMT, int D>
cudaError_t run(const AttnView& a, int max_rows, Partial* meta, RowState* state, float* part, cudaStream_t st) {
    using C = Cfg<T, FMT, D>;
    const void* f = reinterpret_cast<const void*>(&k_attn_rows<T, FMT, D>);
    cudaError_t e = allow_max_dynamic_smem(f);
    if (e != cudaSuccess) return e;
    const int ctas = attn_rows_workers() / WARPS;
    launch_hook("k_attn_rows", 0, st);
    k_attn_rows<T, FMT, D><<<ctas, WARPS * 32, C::SMEM, st>>>(a, max_rows, meta, state, part);
    launch_hook("k_attn_rows", 1, st);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    return launch_attn_combine(a, std::is_same<T, __half>::value ? HOS_TYPE_FP16 : HOS_TYPE_BF16, ROWS, attn_rows_workers(), meta,
                               state, part, st);
}

}  // namespace

// Two CTAs of four warps on each of 148 SMs.
int attn_rows_workers() { return 148 * 2 * WARPS; }

cudaError_t launch_attn_rows(const AttnView& a, int type, int format, int max_rows, Partial* meta, RowState* state,
                             float* part, cudaStream_t st) {
    return kv_dispatch(type, format, a.kv.head_dim, [&](auto t, auto f, auto d) {
        return run<typename decltype(t)::type, decltype(f)::value, decltype(d)::value>(a, max_rows, meta, state, part, st);
    });
}

}  // namespace hos
