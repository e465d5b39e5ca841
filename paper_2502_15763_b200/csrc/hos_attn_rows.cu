// Attention of few query rows per sequence and KV head (decode rounds, short chunks) to the paged cache.
//
// What bounds it: the cache is read once, 2 * head_dim multiply-adds per cached element and 16 rows at
// most, so HBM.  The kernel is built to keep loads in flight and nothing else:
//   - The work is a list of steps of 16 or 32 tokens (sequence, KV head, tile of 8 or 16 rows, step).  Every CTA
//     of four warps takes an equal, contiguous share of the list, whatever the lengths are; within a tile the
//     steps go round the warps, which meet only at the tile's end to add up their parts.  A tile cut by
//     the ends of a share leaves a partial result (unnormalised output, reference, normaliser) in the
//     workspace, and k_attn_combine joins the pieces in list order, so the result does not depend on which
//     CTA finished first.
//   - A warp copies its next steps into its own ring in shared memory (16-byte asynchronous copies), over
//     the ends of tiles and sequences, while it works on the current one.
//   - Rows are the query heads of a group times the new tokens.  Both products are 16x8x16 matrix
//     instructions with the rows as the 8 columns: S^T = K Q^T (16 tokens x 8 rows) and O^T += V^T P^T
//     (16 of head_dim x 8 rows), so a tile of 8 rows wastes nothing.  The k index of the first product and the
//     row index of the second may be permuted freely (the same way on both sides), so each lane reads its
//     operands as whole 16-byte chunks of K and V rows; nothing is transposed but pairs of V rows (one byte
//     permute a register) and the weights (one 8x8 exchange a half step).
//   - 8-bit codes become fp16 exactly; K's scale multiplies the score, V's scale joins the exponent of
//     the weight (w_j = 2^(x_j + log2 vs_j - m), m the maximum of that), so no weight under- or overflows fp16
//     whatever the scales are; the normaliser is sum w_j / vs_j.
//
// Measured on one B200, k_attn_combine included: 32,463 tokens of 64 bf16 KV heads of 128 in 16 sequences (1.06 GB) 168 us,
// 6.3 TB/s; 265,813 tokens of 8 int8 heads in 128 sequences (566 MB) 111 us, 5.1 TB/s; 282,150 tokens of 8 e4m3 heads of
// 64 in 2 sequences (307 MB) 62 us, 5.0 TB/s.  16-bit caches are bound by HBM, 8-bit ones by the work of a step (turning codes into
// fp16, the reductions) that 12 warps an SM hide only in part: 56 % of the issue slots are used.  One share a
// warp instead of one a CTA left four times the pieces and took 125 and 83 us for the last two.
#include "hos_attn_list.cuh"
#include "hos_kv_kernels.h"
#include "hos_kv.cuh"

namespace hos {
namespace {

constexpr int WARPS = 4;

template <typename T, int FMT, int D, int NB> struct Cfg {
    static constexpr bool Q8 = FMT != HOS_KV_SAME;
    static constexpr int ROWS = 8 * NB;
    static constexpr int ROW_BYTES = Q8 ? D : 2 * D;
    static constexpr int CHUNKS = ROW_BYTES / 16;
    // Steps of 32 tokens share the reductions over tokens; with rows of 256 bytes their ring would leave too few warps.
    static constexpr int SUB = ROW_BYTES > 128 ? 1 : 2, STEP = 16 * SUB;
    static constexpr int KV_BYTES = STEP * ROW_BYTES;
    static constexpr int STAGE = 2 * KV_BYTES + (Q8 ? 2 * STEP * 4 : 0);
    // CTAs on an SM, and the ring of each warp: as many bytes as fit
    static constexpr int CTAS = SUB == 1 || NB == 2 ? 2 : 3;
    static constexpr int FIT = (int)(SMEM_LIMIT / CTAS - 2048) / (WARPS * STAGE), STAGES = FIT < 8 ? FIT : 8;
    static constexpr int SMEM = WARPS * STAGES * STAGE;
};
constexpr int MIN_STEPS = WARPS;              // a CTA's smallest share
// What a tile's begin and end cost, in steps.  128 int8 decodes (1,024 tiles of about 65 steps of 32 tokens): 113 us with 4, 108 with 8, 112 with 16;
// 16 bf16 decodes (1,024 tiles of about 127 steps of 16): 173 us with 4, 172 with 16, 170 with 24.
template <int SUB> constexpr int TILE_STEPS = SUB == 2 ? 8 : 24;
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
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
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
k_attn_rows(const __grid_constant__ AttnView a, const int max_rows, const bool beside, Partial* __restrict__ meta,
            RowState* __restrict__ state, float* __restrict__ part) {
    using C = Cfg<T, FMT, D, NB>;
    using M = typename MatType<T, FMT>::type;
    constexpr int STEP = C::STEP, SUB = C::SUB;
    using List = AttnList<C::ROWS, STEP, TILE_STEPS<SUB>>;
    using Cursor = typename List::Cursor;
    constexpr int ROWS = C::ROWS;
    constexpr int KS = D / 16;                 // matrix instructions along head_dim, and tiles of O^T
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ RowState warp_state[WARPS][ROWS];
    const int lane = lane_id(), warp = warp_id(), g = lane >> 2, t4 = lane & 3;
    const int w = (int)blockIdx.x;
    pdl_launch_dependents();
    // Beside the chunk kernel there is nothing of it to wait for until the end, and what came before is complete: that kernel
    // lets this one start only after its own wait for it, in every CTA (it has to stay so).  The fence drops what this
    // SM's L1 may still hold from before.
    if (beside) __threadfence();
    else pdl_wait();

    // this CTA's share of the list
    const List list{a, 0, max_rows};
    long long mine;
    const long long total = list.total(w == 0 && warp == 0, mine);
    const int active = (int)min((long long)gridDim.x, (total + MIN_STEPS - 1) / MIN_STEPS);
    if (w >= active) {
        if (threadIdx.x == 0) meta[w].last = -1;
        pdl_wait();
        return;
    }
    const long long lo = total * w / active;
    const int share = (int)(total * (w + 1) / active - lo);
    Cursor cons = list.locate(lo, mine);
    // where the copies are: this warp's steps of a tile, every fourth one, then the next tile
    Cursor prod = cons;
    int prod_end = list.end_of(prod, share);
    bool prod_more = prod.step < prod_end;
    prod.step += warp;
    const uint32_t ring = smem_u32(smem) + warp * C::STAGES * C::STAGE;

    // --- copies -------------------------------------------------------------------------------
    int pages = 0, pages_at = -1;              // this lane's entry of 32 cached page numbers, and the first one's index
    constexpr int PASSES = 16 * C::CHUNKS / 32, PERIOD = C::CHUNKS / 4;        // copies of 512 bytes for 16 rows; for 8
    uint32_t dst_at[PERIOD];                   // where this lane's chunk goes: the layout repeats every 8 rows
#pragma unroll
    for (int i = 0; i < PERIOD; ++i) {
        const int id = i * 32 + lane, r = id / C::CHUNKS, c = id % C::CHUNKS;
        dst_at[i] = r * C::ROW_BYTES + ((c ^ swizzle<C::CHUNKS>(r)) * 16);
    }
    auto dst_of = [&](int i) { return dst_at[i % PERIOD] + (i / PERIOD) * 8 * C::ROW_BYTES; };
    auto settle = [&]() {                      // to this warp's next step, if it has one
        while (prod_more && prod.step >= prod_end) {
            prod_more = list.next(prod, share);
            prod_end = list.end_of(prod, share);
            prod.step = warp;
            pages_at = -1;
        }
    };
    settle();
    auto issue = [&](int stage) {
        if (prod_more) {
            const int j0 = prod.t.k0 + prod.step * STEP;
            const int pi = j0 >> a.kv.page_shift;
            // a step of 32 tokens may be two pages of 16
            if (pages_at < 0 || ((j0 + STEP - 1) >> a.kv.page_shift) >= pages_at + 32) {
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
            const uint32_t kd = ring + stage * C::STAGE, vd = kd + C::KV_BYTES;
            int page = -1;
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) {
                const int js = j0 + 16 * sub, row0 = js & ((1 << a.kv.page_shift) - 1);
                if (sub == 0 || a.kv.page_shift == 4) page = __shfl_sync(FULL, pages, (js >> a.kv.page_shift) - pages_at);
                const long long e = page_elem(a.kv, max(page, 0), prod.head, row0) * (C::Q8 ? 1 : 2) + lane * 16;
                const unsigned char* ksrc = a.kv.k + e;
                const unsigned char* vsrc = a.kv.v + e;
                const uint32_t ks = kd + sub * 16 * C::ROW_BYTES, vs = ks + C::KV_BYTES;
                if (page >= 0 && js >= prod.t.kb && js + 16 <= prod.t.ke) {
#pragma unroll
                    for (int i = 0; i < PASSES; ++i) {
                        cp_async16(ks + dst_of(i), ksrc + i * 512);
                        cp_async16(vs + dst_of(i), vsrc + i * 512);
                    }
                } else {                       // tokens that no row sees become zeros, whatever memory holds
#pragma unroll
                    for (int i = 0; i < PASSES; ++i) {
                        const int j = js + (i * 32 + lane) / C::CHUNKS;
                        const bool real = page >= 0 && j >= prod.t.kb && j < prod.t.ke;
                        cp_async16(ks + dst_of(i), ksrc + i * 512, real);
                        cp_async16(vs + dst_of(i), vsrc + i * 512, real);
                    }
                }
            }
            if (C::Q8) {                       // scales, four tokens a lane: K's by the first eight lanes, V's by the next
                static_assert(!C::Q8 || SUB == 2, "");
                const int js = j0 + (lane & 7) * 4, at = __shfl_sync(FULL, pages, (js >> a.kv.page_shift) - pages_at);
                if (lane < 16) {
                    const long long se = scale_elem(a.kv, max(at, 0), prod.head, js & ((1 << a.kv.page_shift) - 1));
                    cp_async16(vd + C::KV_BYTES + lane * 16, (lane < 8 ? a.kv.k_scale : a.kv.v_scale) + se, at >= 0);
                }
            }
            prod.step += WARPS;
            settle();
        }
        cp_async_commit();
    };
#pragma unroll 1
    for (int i = 0; i < C::STAGES - 1; ++i) issue(i);

    // --- the rows of the current tile ---------------------------------------------------------
    // as columns of a product: row nb * 8 + g when read, rows nb * 8 + 2 * t4 + {0, 1} of the results
    uint32_t bq[KS][NB][2];
    float o[KS][NB][4];
    float m[NB][2], l[NB][2], qmul[NB][2];     // m: the exponents' reference, the running maximum - LIFT
    int see_lo[NB][2], see_hi[NB][2];          // visible tokens
    int all_lo = 0, all_hi = 0;                // tokens that every row of the tile sees
    const int f = swizzle<C::CHUNKS>(g);
    const uint32_t k_at = g * C::ROW_BYTES + (t4 ^ (f & 3)) * 16, k_x = (f & 4) * 16;

    auto begin = [&]() {
        {
            const int first = cons.q.len - cons.q.n + by_group(a, cons.tile * ROWS);
            const int last = cons.q.len - cons.q.n + by_group(a, cons.tile * ROWS + cons.t.rows - 1);
            all_hi = a.causal ? min(cons.q.len, first + 1) : cons.q.len;
            all_lo = first_seen(a, last);
        }
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
            const int i = by_group(a, r), hd = cons.head * a.group + r - i * a.group;
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
                // bf16 queries meet fp16 keys: a power of two per row brings the row into fp16's range.  Elements down to
                // 2^-30 of the row's largest are exact, smaller ones rounded to within 2^-38 of it.
                float top = 0.0f;
#pragma unroll
                for (int i2 = 0; i2 < 2 * KS; ++i2) {
                    const float2 v = Pair<T>::unpack(x[i2]);
                    top = fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y)));
                }
                top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
                top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
                const int ex = (int)(__float_as_uint(top) >> 23);            // biased; top >= 0
                // top * 2^(140 - ex) is in [2^13, 2^14); rows of zeros, of nothing above 2^-100 and non-finite ones stay
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
                const int pos = cons.q.len - cons.q.n + by_group(a, r2);
                // columns past the tile see everything that its rows do; they are not written
                const bool real = nb * 8 + 2 * t4 + e < cons.t.rows;
                see_hi[nb][e] = real && a.causal ? min(cons.q.len, pos + 1) : cons.q.len;
                see_lo[nb][e] = real ? first_seen(a, pos) : 0;
                qmul[nb][e] = __shfl_sync(FULL, mul, (2 * t4 + e) * 4);
                m[nb][e] = -INFINITY;
                l[nb][e] = 0.0f;
            }
        }
    };

    int stage = 0;
    // Element of head_dim of this lane's first value of tile i of O^T (the second one's is the next).
    auto dim_of = [&](int i) { return C::Q8 && D == 128 ? g * 16 + i * 2 : (i >> 2) * 64 + g * 8 + (i & 3) * 2; };
    bool open_end = false;
    // The four warps' parts of a tile are added up: warp k ends with tiles OWN k .. OWN k + OWN - 1 of O^T and writes them.
    // What it has of the others' tiles goes through its stage that was read last (nothing is on its way there).
    auto finish = [&](bool whole_start, bool whole_end, long long end) {
        constexpr int OWN = KS / WARPS;
        const bool whole = whole_start && whole_end;
        auto buffer = [&](int k, int st) { return smem_u32(smem) + (k * C::STAGES + st) * C::STAGE + lane * (OWN * NB * 16); };
        __shared__ int free_stage[WARPS];
        const int free = stage == 0 ? C::STAGES - 1 : stage - 1;
        if (lane == 0) free_stage[warp] = free;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
            if (k == warp) continue;
            const uint32_t at = buffer(warp, free) + ((k - (k > warp ? 1 : 0)) * 32) * (OWN * NB * 16);
#pragma unroll
            for (int i = 0; i < OWN; ++i)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" :: "r"(at + (i * NB + nb) * 16), "f"(o[k * OWN + i][nb][0]),
                                 "f"(o[k * OWN + i][nb][1]), "f"(o[k * OWN + i][nb][2]), "f"(o[k * OWN + i][nb][3]) : "memory");
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float sum = column_sum(l[nb][e]);
                if (g == 0) warp_state[warp][nb * 8 + 2 * t4 + e] = RowState{m[nb][e], sum};
            }
        __syncthreads();
        float ref[NB][2], norm[NB][2], by[WARPS][NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = nb * 8 + 2 * t4 + e;
                float top = -INFINITY;
#pragma unroll
                for (int k = 0; k < WARPS; ++k) top = fmaxf(top, warp_state[k][r].m);
                const float ms = top == -INFINITY ? 0.0f : top;
                ref[nb][e] = top;
                norm[nb][e] = 0.0f;
#pragma unroll
                for (int k = 0; k < WARPS; ++k) {
                    by[k][nb][e] = exp2_fast(warp_state[k][r].m - ms);
                    norm[nb][e] = fmaf(warp_state[k][r].l, by[k][nb][e], norm[nb][e]);
                }
            }
        float own[OWN][NB][4];
#pragma unroll
        for (int i = 0; i < OWN; ++i)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int j = 0; j < 4; ++j) own[i][nb][j] = 0.0f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {      // in the order of the warps, whichever one adds
            if (k == warp) {
#pragma unroll
                for (int i = 0; i < OWN; ++i)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float v = o[i][nb][j];
#pragma unroll
                            for (int q = 1; q < WARPS; ++q) v = warp == q ? o[q * OWN + i][nb][j] : v;
                            own[i][nb][j] = fmaf(v, by[k][nb][j & 1], own[i][nb][j]);
                        }
            } else {
                const uint32_t at = buffer(k, free_stage[k]) + ((warp - (warp > k ? 1 : 0)) * 32) * (OWN * NB * 16);
#pragma unroll
                for (int i = 0; i < OWN; ++i)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        const uint4 v = lds<uint4>(at + (i * NB + nb) * 16);
                        own[i][nb][0] = fmaf(__uint_as_float(v.x), by[k][nb][0], own[i][nb][0]);
                        own[i][nb][1] = fmaf(__uint_as_float(v.y), by[k][nb][1], own[i][nb][1]);
                        own[i][nb][2] = fmaf(__uint_as_float(v.z), by[k][nb][0], own[i][nb][2]);
                        own[i][nb][3] = fmaf(__uint_as_float(v.w), by[k][nb][1], own[i][nb][3]);
                    }
            }
        }
        const int slot = 2 * w + (whole_start ? 1 : 0);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int in_tile = nb * 8 + 2 * t4 + e;
                if (in_tile >= cons.t.rows) continue;
                const int d0 = dim_of(warp * OWN);
                if (whole) {
                    const int r = cons.tile * ROWS + in_tile;
                    const int i = by_group(a, r), tok = cons.q.off + i, hd = cons.head * a.group + r - i * a.group;
                    const float inv = norm[nb][e] == 0.0f ? 0.0f : 1.0f / norm[nb][e];
                    T* dst = reinterpret_cast<T*>(a.out) + (long long)tok * a.o_tok + (long long)hd * a.o_head + d0;
                    uint32_t v[OWN];
#pragma unroll
                    for (int k = 0; k < OWN; ++k) v[k] = Pair<T>::pack(own[k][nb][e] * inv, own[k][nb][2 + e] * inv);
                    if (OWN == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(v[0], v[OWN - 1]);
                    else *reinterpret_cast<uint32_t*>(dst) = v[0];
                    if (a.lse && g == 0 && warp == 0)
                        a.lse[(long long)tok * a.n_heads + hd] = row_lse(ref[nb][e], norm[nb][e]);
                } else {
                    const long long r = (long long)slot * ROWS + in_tile;
                    float* dst = part + r * D + d0;
                    if (OWN == 2)
                        *reinterpret_cast<float4*>(dst) = make_float4(own[0][nb][e], own[0][nb][2 + e], own[OWN - 1][nb][e], own[OWN - 1][nb][2 + e]);
                    else
                        *reinterpret_cast<float2*>(dst) = make_float2(own[0][nb][e], own[0][nb][2 + e]);
                    if (g == 0 && warp == 0) state[r] = RowState{ref[nb][e], norm[nb][e]};
                }
            }
        if (!whole && whole_start && threadIdx.x == 0)
            meta[w] = Partial{cons.seq, cons.head, cons.tile, (int)((end * active - 1) / total)};
        open_end = whole_start && !whole_end;
        __syncthreads();                       // the buffers may be written again
    };

    for (bool more = cons.step < list.end_of(cons, share); more; more = list.next(cons, share)) {
        begin();
        const int first = cons.step, end = list.end_of(cons, share);
#pragma unroll 1
    for (int step = first + warp; step < end; step += WARPS) {
        cp_async_wait<C::STAGES - 2>();
        __syncwarp();
        issue(stage == 0 ? C::STAGES - 1 : stage - 1);
        const uint32_t kd = ring + stage * C::STAGE, vd = kd + C::KV_BYTES;
        if (++stage == C::STAGES) stage = 0;

        // scores: x[sub][nb][0..1] token g, x[sub][nb][2..3] token g + 8 of 16, rows nb * 8 + 2 * t4 + {0, 1}
        float x[SUB][NB][4];
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[sub][nb][j] = 0.0f;
            const uint32_t ka = kd + sub * 16 * C::ROW_BYTES + k_at;
#pragma unroll
            for (int c = 0; c < C::CHUNKS / 4; ++c) {
                const uint4 v0 = lds<uint4>(ka + ((c * 64) ^ k_x)), v1 = lds<uint4>(ka + 8 * C::ROW_BYTES + ((c * 64) ^ k_x));
                const uint32_t w0[4] = {v0.x, v0.y, v0.z, v0.w}, w1[4] = {v1.x, v1.y, v1.z, v1.w};
                if (!C::Q8) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t ak[4] = {w0[2 * i], w1[2 * i], w0[2 * i + 1], w1[2 * i + 1]};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) mma16816<M>(x[sub][nb], ak, bq[2 * c + i][nb][0], bq[2 * c + i][nb][1]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint2 h0 = codes_to_half4<FMT>(w0[i]), h1 = codes_to_half4<FMT>(w1[i]);
                        const uint32_t ak[4] = {h0.x, h1.x, h0.y, h1.y};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb)
                            mma16816<M>(x[sub][nb], ak, bq[(4 * c + i) % KS][nb][0], bq[(4 * c + i) % KS][nb][1]);
                    }
                }
            }
        }
        const int j0 = cons.t.k0 + step * STEP;
        const bool edge = j0 < all_lo || j0 + STEP > all_hi;
        // of tokens g and g + 8: K's scale; log2 of V's scale, which joins the exponent, and its inverse, which takes it out of
        // the normaliser again
        float iv[SUB][2];
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float ks = 1.0f, lv = 0.0f;
                iv[sub][i] = 1.0f;
                if (C::Q8) {
                    ks = lds<float>(vd + C::KV_BYTES + (16 * sub + g + 8 * i) * 4);
                    const float vs = lds<float>(vd + C::KV_BYTES + (STEP + 16 * sub + g + 8 * i) * 4);
                    const float v1 = vs < LEAST_V_SCALE ? LEAST_V_SCALE : vs;      // a NaN stays one
                    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(lv) : "f"(v1));
                    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(iv[sub][i]) : "f"(v1));
                }
                const int tok = j0 + 16 * sub + g + 8 * i;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float& v = x[sub][nb][2 * i + e];
                        v = C::Q8 ? fmaf(v, qmul[nb][e] * ks, lv) : v * a.scale_log2;
                        if (edge && (tok < see_lo[nb][e] || tok >= see_hi[nb][e])) v = -INFINITY;
                    }
                if (edge && (tok < cons.t.kb || tok >= cons.t.ke)) iv[sub][i] = 0.0f;      // its scale may be anything
            }
        float shrink[NB][2];
        uint32_t bp[SUB][NB][2];
        bool moved = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float p[SUB][4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = fmaxf(x[0][nb][e], x[0][nb][2 + e]);
                if (SUB == 2) top = fmaxf(top, fmaxf(x[SUB - 1][nb][e], x[SUB - 1][nb][2 + e]));
                top = column_max(top);
                const float mn = fmaxf(m[nb][e], top - LIFT<M>), ms = mn == -INFINITY ? 0.0f : mn;
                shrink[nb][e] = exp2_fast(m[nb][e] - ms);
                m[nb][e] = mn;
                float sum = 0.0f;
#pragma unroll
                for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        p[sub][2 * i + e] = exp2_fast(x[sub][nb][2 * i + e] - ms);
                        sum = C::Q8 ? fmaf(p[sub][2 * i + e], iv[sub][i], sum) : sum + p[sub][2 * i + e];
                    }
                l[nb][e] = fmaf(l[nb][e], shrink[nb][e], sum);
                moved |= shrink[nb][e] != 1.0f;
            }
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) {
                bp[sub][nb][0] = transpose8x8(Pair<M>::pack(p[sub][0], p[sub][1]));
                bp[sub][nb][1] = transpose8x8(Pair<M>::pack(p[sub][2], p[sub][3]));
            }
        }
        if (__any_sync(FULL, moved)) {
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[i][nb][j] *= shrink[nb][j & 1];
        }
        // O^T += V^T P^T: this lane's rows of V are tokens 2 * t4 + {0, 1, 8, 9} of 16
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
            const uint32_t va = vd + sub * 16 * C::ROW_BYTES;
            if (!C::Q8) {
#pragma unroll
                for (int half = 0; half < D / 64; ++half) {
                    uint4 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = 2 * t4 + (i & 1) + (i >> 1) * 8;
                        v[i] = lds<uint4>(va + r * C::ROW_BYTES + ((g ^ swizzle<C::CHUNKS>(r)) + half * 8) * 16);
                    }
                    const uint32_t vw[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w},
                                               {v[2].x, v[2].y, v[2].z, v[2].w}, {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t av[4] = {__byte_perm(vw[0][i], vw[1][i], 0x5410), __byte_perm(vw[0][i], vw[1][i], 0x7632),
                                                __byte_perm(vw[2][i], vw[3][i], 0x5410), __byte_perm(vw[2][i], vw[3][i], 0x7632)};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) mma16816<M>(o[half * 4 + i][nb], av, bp[sub][nb][0], bp[sub][nb][1]);
                    }
                }
            } else {
                constexpr int WORDS = D / 32;  // 32-bit words of a lane's codes per V row
                uint32_t vw[4][WORDS];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 2 * t4 + (i & 1) + (i >> 1) * 8;
                    const int sw = swizzle<C::CHUNKS>(r);
                    if (D == 128) {
                        const uint4 v = lds<uint4>(va + r * C::ROW_BYTES + (g ^ sw) * 16);
                        vw[i][0] = v.x; vw[i][1] = v.y; vw[i][WORDS - 2] = v.z; vw[i][WORDS - 1] = v.w;
                    } else {
                        const uint2 v = lds<uint2>(va + r * C::ROW_BYTES + ((g >> 1) ^ sw) * 16 + (g & 1) * 8);
                        vw[i][0] = v.x; vw[i][1] = v.y;
                    }
                }
#pragma unroll
                for (int i = 0; i < WORDS; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t x0 = __byte_perm(vw[0][i], vw[1][i], k ? 0x7362 : 0x5140);
                        const uint32_t x1 = __byte_perm(vw[2][i], vw[3][i], k ? 0x7362 : 0x5140);
                        const uint2 h0 = codes_to_half4<FMT>(x0), h1 = codes_to_half4<FMT>(x1);
                        const uint32_t av[4] = {h0.x, h0.y, h1.x, h1.y};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) mma16816<M>(o[2 * i + k][nb], av, bp[sub][nb][0], bp[sub][nb][1]);
                    }
            }
        }
    }
        __syncwarp();                          // every lane has read the stage that finish() may use
        finish(first == 0, end == cons.t.steps, lo + cons.at + TILE_STEPS<SUB> + cons.t.steps);
    }
    if (!open_end && threadIdx.x == 0) meta[w].last = -1;
    cp_async_wait<0>();
    pdl_wait();                                // the chunk kernel, if one was launched before, is done when this one is
}

template <typename T, int FMT, int D, int NB>
cudaError_t run(const AttnView& a, int max_rows, bool beside, const AttnWs& ws, int* workers, cudaStream_t st) {
    using C = Cfg<T, FMT, D, NB>;
    static_assert(C::CTAS <= ATTN_WORKERS_PER_SM && C::CTAS * C::ROWS <= ATTN_ROWS_PER_SM && C::STAGES >= 2, "");
    cudaError_t e = allow_max_dynamic_smem(reinterpret_cast<const void*>(&k_attn_rows<T, FMT, D, NB>));
    if (e != cudaSuccess) return e;
    const int ctas = ATTN_SMS * C::CTAS;
    *workers = ctas;
    launch_hook("k_attn_rows", 0, st);
    e = launch_early(k_attn_rows<T, FMT, D, NB>, dim3((unsigned)ctas), WARPS * 32, C::SMEM, st, a, max_rows, beside, ws.meta, ws.state, ws.part);
    launch_hook("k_attn_rows", 1, st);
    return e;
}

}  // namespace

// `beside`: the chunk kernel of the same call was launched just before, and this one may start while that runs (a CTA of it fits on
// an SM once the chunk kernel's has left it, so it fills that kernel's tail).
cudaError_t launch_attn_rows(const AttnView& a, int type, int format, int tile_rows, int max_rows, bool beside, const AttnWs& ws, int* workers,
                             cudaStream_t st) {
    return kv_dispatch(type, format, a.kv.head_dim, [&](auto t, auto f, auto d) {
        using T = typename decltype(t)::type;
        return tile_rows == 8 ? run<T, decltype(f)::value, decltype(d)::value, 1>(a, max_rows, beside, ws, workers, st)
                              : run<T, decltype(f)::value, decltype(d)::value, 2>(a, max_rows, beside, ws, workers, st);
    });
}

}  // namespace hos
