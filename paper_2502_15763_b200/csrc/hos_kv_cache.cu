// Keys and values into the pages of the cache (quantised on the way) and back out.
//
// Both kernels move each byte once: HBM is the bound, there is next to no arithmetic.  A block takes a few
// consecutive tokens and up to 16 heads: its warps look up the tokens' places together (two or three dependent
// loads, paid once a block), then the block goes through the vectors, heads first, so that neighbouring vectors
// lie together on the packed side and neighbouring tokens on the side of the pages.  A vector of head_dim
// elements is spread over head_dim / 16 lanes with 16 elements (32 bytes) each: the largest magnitude of a vector
// takes two or three shuffles, and a lane's 16 codes are one 16-byte access.
// Measured on one B200: 6,634 tokens of 64 heads of 128 appended as e4m3 (329 MB) 62 us, 5.3 TB/s; 31,896 tokens of 64 heads
// read back from int8 (1.58 GB) 265-271 us, 5.9 TB/s.
#include <initializer_list>

#include "hos_kv_kernels.h"
#include "hos_kv.cuh"

namespace hos {
namespace {

constexpr int WARPS = 8, MOST_TOKENS = 16, APPEND_TOKENS = 4, MOST_HEADS = KV_HEADS_A_BLOCK;
// Vectors that a thread has on the way at once; blocks an SM.  Few and many: reading 31,896 tokens of 64 int8 heads (1.6 GB) takes
// 331 us with 4 vectors and 4 blocks, 305 with 2 and 5, 265 with 1 and 7; appending 6,634 tokens of 64 heads as e4m3 (329 MB)
// took 66, 62 and 63 us (62 with the magnitudes compared two at a time and the final shape).
constexpr int APPEND_AHEAD = 2, APPEND_BLOCKS = 5, READ_AHEAD = 1, READ_BLOCKS = 7;

// The sequence that owns packed token t: the last one whose offset is <= t (offsets ascend).  All lanes
// probe at once, so 32 sequences fall in one step, 1,024 in two.
__device__ __forceinline__ int find_seq(const KvView& c, int t) {
    int lo = 0, n = c.n_seq;                       // answer in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) >> 5;
        const int at = lo + lane_id() * step;
        const bool le = lane_id() * step < n && __ldg(c.tok_off + at) <= t;
        const unsigned m = __ballot_sync(FULL, le);
        const int k = m ? 31 - __clz(m) : 0;
        const int left = n - k * step;
        lo += k * step;
        n = left < step ? left : step;
    }
    return lo;
}

// Page and row of packed token t; false if it has no valid place.
__device__ __forceinline__ bool find_place(const KvView& c, int t, int& page, int& row) {
    const int s = find_seq(c, t);
    const SeqInfo q = load_seq(c, s, lane_id() == 0);
    const int i = t - q.off;
    const int pos = q.len - q.n + i;
    if (i < 0 || i >= q.n || pos < 0) return false;
    page = __ldg(c.table + (long long)s * c.table_stride + (pos >> c.page_shift));
    row = pos & ((1 << c.page_shift) - 1);
    if ((unsigned)page >= (unsigned)c.n_pages) {
        if (lane_id() == 0 && c.status) atomicOr(c.status + s, HOS_ST_INVALID);
        return false;
    }
    return true;
}

struct Vec16 { uint32_t w[8]; };                   // 16 elements of 16 bits

// 32 bytes of a lane: one access (and a whole sector) where the addresses allow it.
__device__ __forceinline__ Vec16 load16(const void* p, bool wide) {
    Vec16 v;
    if (wide) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]), "=r"(v.w[7]) : "l"(p));
        return v;
    }
    const uint4* q = static_cast<const uint4*>(p);
    const uint4 a = __ldg(q), b = __ldg(q + 1);
    return Vec16{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ void store16(void* p, const Vec16& v, bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     :: "l"(p), "r"(v.w[0]), "r"(v.w[1]), "r"(v.w[2]), "r"(v.w[3]), "r"(v.w[4]), "r"(v.w[5]), "r"(v.w[6]), "r"(v.w[7]) : "memory");
        return;
    }
    uint4* q = static_cast<uint4*>(p);
    q[0] = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    q[1] = make_uint4(v.w[4], v.w[5], v.w[6], v.w[7]);
}

template <typename T, int FMT>
__device__ __forceinline__ uint4 quantise16(const Vec16& v, int lanes, float* scale) {
    constexpr float TOP = FMT == HOS_KV_E4M3 ? 448.0f : 127.0f;
    // magnitudes compared as 16-bit integers, two at a time: same order, and a NaN is larger than everything
    uint32_t tops[2] = {0, 0};
    float x[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = Pair<T>::unpack(v.w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
        tops[i & 1] = __vmaxu2(tops[i & 1], v.w[i] & 0x7FFF7FFFu);
    }
    const uint32_t both = __vmaxu2(tops[0], tops[1]);
    const float2 ends = Pair<T>::unpack(both);
    uint32_t top = max(__float_as_uint(1e-30f), max(__float_as_uint(ends.x), __float_as_uint(ends.y)));
    for (int d = lanes >> 1; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(FULL, top, d));
    const float a = __uint_as_float(top);
    const float inv = __fmul_rn(__frcp_rn(a), TOP);
    // a NaN or an infinity anywhere makes the scale NaN, and with it the whole vector
    *scale = top >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __fmul_rn(a, 1.0f / TOP);
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = __fmul_rn(x[4 * i + j], inv);
        if (FMT == HOS_KV_E4M3) {
            uint16_t lo, hi;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y[1]), "f"(y[0]));
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y[3]), "f"(y[2]));
            r[i] = (uint32_t)lo | ((uint32_t)hi << 16);
        } else {
            uint32_t b = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) b |= ((uint32_t)__float2int_rn(y[j]) & 0xFFu) << (8 * j);
            r[i] = b;
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

template <typename T, int FMT>
__device__ __forceinline__ Vec16 dequantise16(const uint4& c, float scale) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    Vec16 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint2 h = codes_to_half4<FMT>(w[i]);
        const float2 f = Pair<__half>::unpack(h.x), g = Pair<__half>::unpack(h.y);
        v.w[2 * i] = Pair<T>::pack(__fmul_rn(f.x, scale), __fmul_rn(f.y, scale));
        v.w[2 * i + 1] = Pair<T>::pack(__fmul_rn(g.x, scale), __fmul_rn(g.y, scale));
    }
    return v;
}

struct Place { int page, row; };                   // page -1: none

// What a block works on: `tokens` tokens from t0, heads h0 .. h0 + 2^head_shift - 1 (those below n_kv).
struct Work {
    int t0, tokens, h0, head_shift;
};
__device__ __forceinline__ Work block_work(const KvView& c, int tokens, int head_shift) {
    Work w;
    w.t0 = (int)blockIdx.x * tokens;
    w.tokens = min(tokens, c.n_tokens - w.t0);
    w.h0 = (int)blockIdx.y << head_shift;
    w.head_shift = head_shift;
    return w;
}
__device__ __forceinline__ void find_places(const KvView& c, const Work& w, Place* place) {
    for (int i = warp_id(); i < w.tokens; i += WARPS) {
        Place p{-1, 0};
        if (!find_place(c, w.t0 + i, p.page, p.row)) p.page = -1;
        if (lane_id() == 0) place[i] = p;
    }
}

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(WARPS * 32, APPEND_BLOCKS) k_kv_append(const __grid_constant__ KvView c, const T* __restrict__ k,
                                                         const T* __restrict__ v, long long k_tok, long long k_head,
                                                         long long v_tok, long long v_head, int tokens, int head_shift, bool wide) {
    constexpr int AHEAD = APPEND_AHEAD, LANES = D / 16, SPAN = WARPS * 32 / LANES;           // vectors that the block moves at once
    __shared__ Place place[MOST_TOKENS];
    const Work w = block_work(c, tokens, head_shift);
    pdl_launch_dependents();
    pdl_wait();
    const int at = ((int)threadIdx.x % LANES) * 16, per_side = w.tokens << head_shift;
    bool known = false;
    for (int id0 = (int)threadIdx.x / LANES; id0 - (int)threadIdx.x / LANES < 2 * per_side; id0 += AHEAD * SPAN) {
        Vec16 x[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int id = id0 + i * SPAN, side = id >= per_side, r = side ? id - per_side : id;
            const int h = w.h0 + (r & ((1 << head_shift) - 1));
            const long long t = w.t0 + (r >> head_shift);
            x[i] = Vec16{{0, 0, 0, 0, 0, 0, 0, 0}};
            if (id < 2 * per_side && h < c.n_kv) x[i] = load16((side ? v + t * v_tok + h * v_head : k + t * k_tok + h * k_head) + at, wide);
        }
        if (!known) {                              // the first loads are on their way meanwhile
            find_places(c, w, place);
            __syncthreads();
            known = true;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int id = id0 + i * SPAN, side = id >= per_side, r = side ? id - per_side : id;
            const int h = w.h0 + (r & ((1 << head_shift) - 1));
            uint4 codes = make_uint4(0, 0, 0, 0);
            float scale = 0.0f;
            if (FMT != HOS_KV_SAME) codes = quantise16<T, FMT>(x[i], LANES, &scale);
            if (id >= 2 * per_side || h >= c.n_kv) continue;
            const Place p = place[r >> head_shift];
            if (p.page < 0) continue;
            const long long e = page_elem(c, p.page, h, p.row) + at;
            if (FMT == HOS_KV_SAME) {
                store16((side ? c.v : c.k) + 2 * e, x[i], wide);
            } else {
                *reinterpret_cast<uint4*>((side ? c.v : c.k) + e) = codes;
                if (at == 0) (side ? c.v_scale : c.k_scale)[scale_elem(c, p.page, h, p.row)] = scale;
            }
        }
    }
}

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(WARPS * 32, READ_BLOCKS) k_kv_read(const __grid_constant__ KvView c, T* __restrict__ k, T* __restrict__ v,
                                                       int tokens, int head_shift, bool wide) {
    constexpr int AHEAD = READ_AHEAD, LANES = D / 16, SPAN = WARPS * 32 / LANES;
    __shared__ Place place[MOST_TOKENS];
    const Work w = block_work(c, tokens, head_shift);
    pdl_launch_dependents();
    pdl_wait();
    find_places(c, w, place);
    __syncthreads();
    const int at = ((int)threadIdx.x % LANES) * 16, per_side = w.tokens << head_shift;
    for (int id0 = (int)threadIdx.x / LANES; id0 < 2 * per_side; id0 += AHEAD * SPAN) {
        Vec16 x[AHEAD];
        uint4 codes[AHEAD];
        float scale[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int id = id0 + i * SPAN, side = id >= per_side, r = side ? id - per_side : id;
            const int h = w.h0 + (r & ((1 << head_shift) - 1));
            x[i] = Vec16{{0, 0, 0, 0, 0, 0, 0, 0}};
            codes[i] = make_uint4(0, 0, 0, 0);
            scale[i] = 0.0f;
            if (id >= 2 * per_side || h >= c.n_kv) continue;
            const Place p = place[r >> head_shift];
            if (p.page < 0) continue;
            const long long e = page_elem(c, p.page, h, p.row) + at;
            if (FMT == HOS_KV_SAME) {
                x[i] = load16((side ? c.v : c.k) + 2 * e, wide);
            } else {
                codes[i] = __ldg(reinterpret_cast<const uint4*>((side ? c.v : c.k) + e));
                scale[i] = __ldg((side ? c.v_scale : c.k_scale) + scale_elem(c, p.page, h, p.row));
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int id = id0 + i * SPAN, side = id >= per_side, r = side ? id - per_side : id;
            const int h = w.h0 + (r & ((1 << head_shift) - 1));
            if (id >= 2 * per_side || h >= c.n_kv) continue;
            if (FMT != HOS_KV_SAME) x[i] = dequantise16<T, FMT>(codes[i], scale[i]);
            store16((side ? v : k) + ((long long)(w.t0 + (r >> head_shift)) * c.n_kv + h) * D + at, x[i], wide);
        }
    }
}

bool multiples32(std::initializer_list<long long> bytes) {
    for (long long b : bytes)
        if (b % 32) return false;
    return true;
}
long long address(const void* p) { return static_cast<long long>(reinterpret_cast<uintptr_t>(p)); }

// Blocks of `most_tokens` tokens where there are enough of them to fill the device, else of fewer, for latency.
struct Shape { dim3 grid; int tokens, head_shift; };
Shape shape_of(const KvView& c, int most_tokens) {
    Shape s;
    s.head_shift = 0;
    while ((1 << s.head_shift) < c.n_kv && (1 << s.head_shift) < MOST_HEADS) ++s.head_shift;
    const long long rows = (c.n_kv + (1 << s.head_shift) - 1) >> s.head_shift;
    s.tokens = most_tokens;
    while (s.tokens > 1 && (c.n_tokens + s.tokens - 1) / s.tokens * rows < 4 * ATTN_SMS) s.tokens >>= 1;
    s.grid = dim3((unsigned)((c.n_tokens + s.tokens - 1) / s.tokens), (unsigned)rows);
    return s;
}

template <typename T, int FMT, int D>
cudaError_t append(const KvView& c, const void* k, const void* v, const long long (&st)[4], cudaStream_t stream) {
    // four tokens: all loads of a block are on their way at once, before the places are known
    const Shape s = shape_of(c, APPEND_TOKENS);
    const bool wide = multiples32({address(k), address(v), 2 * st[0], 2 * st[1], 2 * st[2], 2 * st[3]}) &&
                      (FMT != HOS_KV_SAME || multiples32({address(c.k), address(c.v), 2 * c.page_stride}));
    launch_hook("k_kv_append", 0, stream);
    const cudaError_t e = launch_early(k_kv_append<T, FMT, D>, s.grid, WARPS * 32, 0, stream, c, static_cast<const T*>(k), static_cast<const T*>(v), st[0],
                                       st[1], st[2], st[3], s.tokens, s.head_shift, wide);
    launch_hook("k_kv_append", 1, stream);
    return e;
}
template <typename T, int FMT, int D>
cudaError_t read(const KvView& c, void* k, void* v, cudaStream_t stream) {
    const Shape s = shape_of(c, MOST_TOKENS);
    const bool wide = multiples32({address(k), address(v)}) &&
                      (FMT != HOS_KV_SAME || multiples32({address(c.k), address(c.v), 2 * c.page_stride}));
    launch_hook("k_kv_read", 0, stream);
    const cudaError_t e = launch_early(k_kv_read<T, FMT, D>, s.grid, WARPS * 32, 0, stream, c, static_cast<T*>(k), static_cast<T*>(v), s.tokens, s.head_shift,
                                       wide);
    launch_hook("k_kv_read", 1, stream);
    return e;
}

}  // namespace

cudaError_t launch_kv_append(const KvView& c, int type, int format, const void* k, const void* v,
                             const long long (&st)[4], cudaStream_t stream) {
    return kv_dispatch(type, format, c.head_dim, [&](auto t, auto f, auto d) {
        return append<typename decltype(t)::type, decltype(f)::value, decltype(d)::value>(c, k, v, st, stream);
    });
}
cudaError_t launch_kv_read(const KvView& c, int type, int format, void* k, void* v, cudaStream_t stream) {
    return kv_dispatch(type, format, c.head_dim, [&](auto t, auto f, auto d) {
        return read<typename decltype(t)::type, decltype(f)::value, decltype(d)::value>(c, k, v, stream);
    });
}

}  // namespace hos
