// Shared pieces of the KV-cache kernels: the batch as a kernel sees it, places in the cache, the
// 8-bit formats, asynchronous copies and the 16-bit matrix instruction of the row kernel.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "hos.h"
#include "hos_common.cuh"

namespace hos {

// hos_kv_cache and hos_kv_batch with the defaults filled in; passed to kernels by value.
struct KvView {
    unsigned char *k, *v;
    float *k_scale, *v_scale;
    long long page_stride, scale_page_stride;        // elements
    const int32_t *tok_off, *kv_len, *table;
    long long table_stride;
    int32_t* status;
    int n_pages, page_shift, n_kv, head_dim;
    int n_seq, n_tokens, max_pages;
};

struct SeqInfo { int off, n, len; };

// A sequence's tokens and length.  Offsets outside the batch: no tokens; a length outside the page
// table: length 0.  Both set HOS_ST_INVALID (when `flag`).
__device__ __forceinline__ SeqInfo load_seq(const KvView& c, int s, bool flag) {
    SeqInfo q;
    q.off = __ldg(c.tok_off + s);
    const int end = __ldg(c.tok_off + s + 1);
    q.len = __ldg(c.kv_len + s);
    q.n = end - q.off;
    bool bad = false;
    if (q.off < 0 || end < q.off || end > c.n_tokens) { q.n = 0; bad = true; }
    if (q.len < 0 || q.len > ((long long)c.max_pages << c.page_shift)) { q.len = 0; bad = true; }
    if (bad && flag && c.status) atomicOr(c.status + s, HOS_ST_INVALID);
    return q;
}

// Row of k/v (in units of head_dim elements) or element of the scales is base(page) + local.
__device__ __forceinline__ long long page_elem(const KvView& c, int page, int head, int row) {
    return (long long)page * c.page_stride +
           ((long long)(((long long)head << c.page_shift) + row)) * c.head_dim;
}
__device__ __forceinline__ long long scale_elem(const KvView& c, int page, int head, int row) {
    return (long long)page * c.scale_page_stride + (((long long)head << c.page_shift) + row);
}

// 16-bit pairs.  T is __nv_bfloat16 or __half.
template <typename T> struct Pair;
template <> struct Pair<__half> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ float2 unpack(uint32_t x) {
        return __half22float2(*reinterpret_cast<const __half2*>(&x));
    }
};
template <> struct Pair<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ float2 unpack(uint32_t x) {
        return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
    }
};

// Four 8-bit codes -> two fp16 pairs (exact for both formats).
template <int FMT> __device__ __forceinline__ uint2 codes_to_half4(uint32_t x) {
    uint2 r;
    if (FMT == HOS_KV_E4M3) {
        asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }" : "=r"(r.x), "=r"(r.y) : "r"(x));
    } else {
        // 1024 + (code + 128) in fp16 is 0x6400 | (code ^ 0x80); subtracting 1152 is exact
        const uint32_t u = x ^ 0x80808080u;
        const uint32_t lo = __byte_perm(u, 0x64646464u, 0x4140), hi = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 off = __half2half2(__ushort_as_half(0x6480));
        const __half2 a = __hsub2(*reinterpret_cast<const __half2*>(&lo), off), b = __hsub2(*reinterpret_cast<const __half2*>(&hi), off);
        r = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    }
    return r;
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
// 16 bytes to shared memory without passing through registers; zeros where !real.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }
// Loads by shared-memory address, as ordinary memory reads (the compiler may move them between barriers).
template <typename V> __device__ __forceinline__ V lds(uint32_t a) { return *static_cast<const V*>(__cvta_shared_to_generic(a)); }

// exp2 with results below 2^-126 flushed; exp2(-inf) = 0.  Relative error about 2^-22.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// c[16][8] += a[16][16] b[16][8], 32-bit sums.
template <typename T> __device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Programmatic dependent launch: a kernel launched with the attribute may start while its predecessor
// drains.  The wait covers the direct predecessor only; that what came before it is complete as well follows
// from the predecessor's own wait, so every kernel waits in all its threads and on every way out, and before it
// touches memory.  The one exception is the row kernel beside the chunk kernel, which waits at its end.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Attention call as the kernels see it.
struct AttnView {
    KvView kv;
    const unsigned char* q;
    long long q_tok, q_head;                  // strides in elements
    unsigned char* out;
    long long o_tok, o_head;
    float* lse;
    int n_heads, group;
    uint32_t group_magic, group_shift;        // for by_group
    float scale_log2;                         // sm_scale * log2(e)
    int causal, window;
};

// n / group for 0 <= n < 2^31: with 2^shift the smallest power of two >= group and magic = floor(2^32 (2^shift - group) / group) + 1
// the quotient is (n + floor(n magic / 2^32)) >> shift (Granlund, Montgomery, "Division by invariant integers using
// multiplication", 1994).
__device__ __forceinline__ int by_group(const AttnView& a, int n) {
    return (int)(((uint32_t)n + __umulhi((uint32_t)n, a.group_magic)) >> a.group_shift);
}

// The first token that a row at position pos sees.  Positions below 0 (more new tokens than the cache holds) see what 0 sees
// there; so counted, the difference stays in 32 bits for every window.
__device__ __forceinline__ int first_seen(const AttnView& a, int pos) {
    return a.window > 0 ? max(0, max(pos, 0) - a.window + 1) : 0;
}

// Workspace of an attention call.  A worker (warp or CTA) owns a contiguous range of the call's work
// units; a tile that crosses the range's ends is left as a partial result: slot 0 if the tile began in an
// earlier worker's range, slot 1 if it begins here and ends later.
struct Partial {                              // per worker, what slot 1 holds
    int32_t seq, head, tile, last;            // last: the worker in whose range the tile ends; -1: slot unused
};
struct RowState { float m, l; };              // of one row: what its exponents (base 2) are relative to, and the sum of its weights

// A row's lse from its state.  The power of two of l joins m first: with an 8-bit cache m holds the lift and the log2 of V's scale, and
// log2 l as much with the other sign, so that their sum would keep the rounding of numbers around 20.  SMALL: m holds no scale and a
// lift of 7 at most, which costs no such bits (32 short prompts, fp16, in the chunk kernel: 70.9 us so, 71.5 otherwise).
template <bool SMALL = false> __device__ __forceinline__ float row_lse(float m, float l) {
    constexpr float LN2 = 0.69314718055994530942f;
    if (l == 0.0f) return -INFINITY;
    if (SMALL) return (m + log2f(l)) * LN2;
    const uint32_t bits = __float_as_uint(l);
    const int biased = (int)(bits >> 23);
    if (biased < 1 || biased > 254) return (m + log2f(l)) * LN2;          // denormal, infinite, NaN
    return ((m + (float)(biased - 127)) + log2f(__uint_as_float((bits & 0x7FFFFFu) | 0x3F800000u))) * LN2;
}

// The smallest V scale that the attention kernels tell from zero (a vector of values below 1e-21).
constexpr float LEAST_V_SCALE = 8.2718061e-25f;                       // 2^-80

// Calls f(type tag, format tag, head_dim tag) for the run-time combination.
template <typename T> struct TypeTag { using type = T; };
template <int N> struct IntTag { static constexpr int value = N; };
template <typename F> cudaError_t kv_dispatch(int type, int format, int head_dim, F&& f) {
    auto with_dim = [&](auto t, auto fm) {
        return head_dim == 64 ? f(t, fm, IntTag<64>{}) : f(t, fm, IntTag<128>{});
    };
    auto with_format = [&](auto t) {
        if (format == HOS_KV_E4M3) return with_dim(t, IntTag<HOS_KV_E4M3>{});
        if (format == HOS_KV_INT8) return with_dim(t, IntTag<HOS_KV_INT8>{});
        return with_dim(t, IntTag<HOS_KV_SAME>{});
    };
    return type == HOS_TYPE_BF16 ? with_format(TypeTag<__nv_bfloat16>{}) : with_format(TypeTag<__half>{});
}

}  // namespace hos
