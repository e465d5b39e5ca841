// Keys and values into the pages of the cache (quantised on the way) and back out.
//
// Both kernels move each byte once: HBM is the bound, there is next to no arithmetic.  One warp takes
// one token and HEADS_PER_WARP heads of it.  A vector of head_dim elements is spread over
// head_dim / 16 lanes with 16 elements (32 bytes) each, so a warp moves four (head_dim 128) or eight
// (64) vectors per instruction, the largest magnitude of a vector takes two or three shuffles, and a
// lane's 16 codes leave in one 16-byte store.
#include "hos_kernels.h"
#include "hos_kv.cuh"

namespace hos {
namespace {

constexpr int WARPS = 8;
constexpr int HEADS_PER_WARP = 16;

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

__device__ __forceinline__ Vec16 load16(const void* p) {
    const uint4* q = static_cast<const uint4*>(p);
    const uint4 a = __ldg(q), b = __ldg(q + 1);
    return Vec16{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ void store16(void* p, const Vec16& v) {
    uint4* q = static_cast<uint4*>(p);
    q[0] = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    q[1] = make_uint4(v.w[4], v.w[5], v.w[6], v.w[7]);
}

template <typename T, int FMT>
__device__ __forceinline__ uint4 quantise16(const Vec16& v, int lanes, float* scale) {
    constexpr float TOP = FMT == HOS_KV_E4M3 ? 448.0f : 127.0f;
    // magnitudes compared as integers: same order, and a NaN is larger than everything
    uint32_t top = __float_as_uint(1e-30f);
    float x[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = Pair<T>::unpack(v.w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
        top = max(top, max(__float_as_uint(f.x) & 0x7FFFFFFFu, __float_as_uint(f.y) & 0x7FFFFFFFu));
    }
    for (int d = lanes >> 1; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(FULL, top, d));
    const float a = __uint_as_float(top);
    const float inv = __fdiv_rn(TOP, a);
    // a NaN or an infinity anywhere makes the scale NaN, and with it the whole vector
    *scale = top >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __fdiv_rn(a, TOP);
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

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(WARPS * 32) k_kv_append(const __grid_constant__ KvView c, const T* __restrict__ k,
                                                         const T* __restrict__ v, long long k_tok, long long k_head,
                                                         long long v_tok, long long v_head) {
    constexpr int LANES = D / 16, PER = 32 / LANES, STEPS = HEADS_PER_WARP / PER;
    const long long t = (long long)blockIdx.x * WARPS + warp_id();
    if (t >= c.n_tokens) return;
    const int sub = lane_id() / LANES, at = (lane_id() % LANES) * 16;
    const int h0 = blockIdx.y * HEADS_PER_WARP;
    // the loads do not depend on the place, so they are issued before it is known
    Vec16 xk[STEPS], xv[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int h = h0 + i * PER + sub;
        if (h < c.n_kv) {
            xk[i] = load16(k + t * k_tok + h * k_head + at);
            xv[i] = load16(v + t * v_tok + h * v_head + at);
        } else {
            xk[i] = Vec16{{0, 0, 0, 0, 0, 0, 0, 0}};
            xv[i] = xk[i];
        }
    }
    int page, row;
    if (!find_place(c, (int)t, page, row)) return;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int h = h0 + i * PER + sub;
        const long long e = page_elem(c, page, h, row) + at;
        if (FMT == HOS_KV_SAME) {
            if (h < c.n_kv) {
                store16(c.k + 2 * e, xk[i]);
                store16(c.v + 2 * e, xv[i]);
            }
        } else {
            float sk, sv;
            const uint4 ck = quantise16<T, FMT>(xk[i], LANES, &sk);
            const uint4 cv = quantise16<T, FMT>(xv[i], LANES, &sv);
            if (h < c.n_kv) {
                *reinterpret_cast<uint4*>(c.k + e) = ck;
                *reinterpret_cast<uint4*>(c.v + e) = cv;
                if (at == 0) {
                    const long long se = scale_elem(c, page, h, row);
                    c.k_scale[se] = sk;
                    c.v_scale[se] = sv;
                }
            }
        }
    }
}

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(WARPS * 32) k_kv_read(const __grid_constant__ KvView c, T* __restrict__ k, T* __restrict__ v) {
    constexpr int LANES = D / 16, PER = 32 / LANES, STEPS = HEADS_PER_WARP / PER;
    const long long t = (long long)blockIdx.x * WARPS + warp_id();
    if (t >= c.n_tokens) return;
    const int sub = lane_id() / LANES, at = (lane_id() % LANES) * 16;
    const int h0 = blockIdx.y * HEADS_PER_WARP;
    int page = 0, row = 0;
    const bool there = find_place(c, (int)t, page, row);
    Vec16 xk[STEPS], xv[STEPS];
    uint4 ck[STEPS], cv[STEPS];
    float sk[STEPS], sv[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int h = h0 + i * PER + sub;
        const long long e = page_elem(c, page, h, row) + at;
        if (FMT == HOS_KV_SAME) {
            xk[i] = Vec16{{0, 0, 0, 0, 0, 0, 0, 0}};
            xv[i] = xk[i];
            if (there && h < c.n_kv) { xk[i] = load16(c.k + 2 * e); xv[i] = load16(c.v + 2 * e); }
        } else {
            ck[i] = make_uint4(0, 0, 0, 0);
            cv[i] = ck[i];
            sk[i] = sv[i] = 0.0f;
            if (there && h < c.n_kv) {
                ck[i] = __ldg(reinterpret_cast<const uint4*>(c.k + e));
                cv[i] = __ldg(reinterpret_cast<const uint4*>(c.v + e));
                const long long se = scale_elem(c, page, h, row);
                sk[i] = __ldg(c.k_scale + se);
                sv[i] = __ldg(c.v_scale + se);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int h = h0 + i * PER + sub;
        if (h >= c.n_kv) continue;
        const long long e = ((long long)t * c.n_kv + h) * D + at;
        if (FMT != HOS_KV_SAME) {
            xk[i] = dequantise16<T, FMT>(ck[i], sk[i]);
            xv[i] = dequantise16<T, FMT>(cv[i], sv[i]);
        }
        store16(k + e, xk[i]);
        store16(v + e, xv[i]);
    }
}

struct Grid { dim3 g; };
dim3 grid_of(const KvView& c) {
    return dim3((unsigned)((c.n_tokens + WARPS - 1) / WARPS), (unsigned)((c.n_kv + HEADS_PER_WARP - 1) / HEADS_PER_WARP));
}

template <typename T, int FMT, int D>
cudaError_t append(const KvView& c, const void* k, const void* v, const long long (&st)[4], cudaStream_t stream) {
    launch_hook("k_kv_append", 0, stream);
    k_kv_append<T, FMT, D><<<grid_of(c), WARPS * 32, 0, stream>>>(c, static_cast<const T*>(k), static_cast<const T*>(v),
                                                                  st[0], st[1], st[2], st[3]);
    launch_hook("k_kv_append", 1, stream);
    return cudaGetLastError();
}
template <typename T, int FMT, int D>
cudaError_t read(const KvView& c, void* k, void* v, cudaStream_t stream) {
    launch_hook("k_kv_read", 0, stream);
    k_kv_read<T, FMT, D><<<grid_of(c), WARPS * 32, 0, stream>>>(c, static_cast<T*>(k), static_cast<T*>(v));
    launch_hook("k_kv_read", 1, stream);
    return cudaGetLastError();
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
