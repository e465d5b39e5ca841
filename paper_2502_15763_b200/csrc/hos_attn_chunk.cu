// Attention of many query rows per sequence and KV head (prompts, chunks of new tokens) to the paged cache.
//
// The mathematics: with x = scale * log2(e) * q.k, a row keeps a reference m near its running maximum, l = sum 2^(x - m)
// and O = sum 2^(x - m) v; m moves (and O and l are rescaled) only when the maximum has grown by more than 2^8 -- the
// quotient O / l does not depend on m, and 2^8 is far inside every type's range -- so O is rescaled in the first few
// steps of a tile and hardly ever after.
//
// One CTA of 12 (16-bit cache) or 16 warps (8-bit cache) an SM works through an equal, contiguous share of the batch's
// steps of 128 tokens; a tile is two halves of 128 rows.  Both products run on tcgen05: S = Q K^T from shared memory
// into tensor memory (128 columns a half), O += P V with P from tensor memory, where it takes the place of S.
// While one half's S is turned into P by its four warps (one thread a row, no shuffles), the tensor cores have the other
// half's products.
//   warps 0-3, 4-7   softmax, output of half 0, 1
//   warp 8           K and V into a ring of shared memory by TMA, page by page
//   warp 9           issues the products
//   warps 10, 11     the rows of the next tile's queries, half 0, 1
//   warps 12-15      (8-bit cache) turn the codes of a stage into fp16, in place
// An 8-bit cache's K scale multiplies the score, its V scale joins the exponent: y_j = x_j + log2 vs_j, the weights 2^(y_j - m)
// meet the bare codes and are safe in fp16 whatever the scales are, and l = sum 2^(y_j - m) / vs_j.
//
// Measured on one B200, k_attn_combine included: 4,096 tokens, 64 heads of 128, bf16, causal: 334-344 us under the power cap
// (810 TFLOP/s); 509 tokens, 64 heads over 8, behind 15,991 in an e4m3 cache: 343-347 us; 32 prompts of 129
// tokens, 64 heads over 8, fp16: 69-71 us.  What bounds it: a half's chain of scores -> maximum -> exponentials -> products, which two
// halves hide from one another only in part: a step of 2 x 128 rows takes about 3,300 cycles, of which the tensor cores need 2,048 and
// the exponentials (16 a cycle and SM) 2,048; with an 8-bit cache about 5,300, since every thread reads three vectors
// of 128 scales from shared memory.  Work that short prompts cannot hide: a tile's queries in, its first score and its result out.
// (The first 96 of a step's 128 weights are handed over early, so that only a quarter of the second product waits for the last
// exponentials; with head_dim 128 a third half in flight would need more tensor memory than there is.)
//
// Waits by parity: a barrier must not be two phases past (or short of) the one waited for.  Why none is, by barrier:
//   kv_full    the products' warp waits in order, and a stage is refilled only after that warp has freed it; half 0's wait for V
//              (clear_v) comes after its score of the step, and the stage is freed only after its weights of the step
//   raw_full   the warps that convert wait in order, and the refill of a stage needs their arrivals on kv_full
//   kv_free    the copying warp waits in order, and a stage is freed again only after it has been refilled
//   q_full, q_free   one of each a tile, and either side needs the other's last one
//   s_full, o_done   a half's next score needs its weights of this step; its next output needs weights that come after this output
//   p_half, p_ready  a half's next weights need the score that is issued after the last ones were waited for
//   scales_full      filled again only after V of the step that read it was freed, which needs all weights of that step; a
//              half that skips tiles does not run ahead of it, since it waits for its own score first
//
// All waits are bounded: one that runs out sets HOS_ST_LIMIT and the CTA drains and returns.
#include <cuda.h>

#include "hos_attn_list.cuh"
#include "hos_kv_kernels.h"
#include "hos_kv.cuh"

namespace hos {
namespace {

constexpr int ROWS = ATTN_CHUNK_ROWS, STEP = 128, HALF = 128;
constexpr int TILE_STEPS = 2;                 // what a tile's begin and end cost, in steps
using List = AttnList<ROWS, STEP, TILE_STEPS>;
using Cursor = List::Cursor;
constexpr int FIRST_PART = 96;                // of a step's 128 weights a row, those whose product is issued before the rest is known
constexpr float GROWTH = 8.0f;                // log2 of how far a row's maximum may pass the one its reference was taken from
// The reference is the maximum - LIFT: fp16 weights start at 2^7 and end below 2^15, so that small ones keep their bits.
template <typename M> constexpr float LIFT = std::is_same<M, __half>::value ? 7.0f : 0.0f;

template <typename T, int FMT, int D> struct Cfg {
    static constexpr bool Q8 = FMT != HOS_KV_SAME;
    static constexpr int THREADS = Q8 ? 512 : 384;
    // Registers of the softmax warps and of the others: their sum must not pass what the CTA is launched with, or the wait for more
    // would not end.
    static constexpr int SOFTMAX_REGS = Q8 ? 184 : 200, OTHER_REGS = Q8 ? 72 : 104, LAUNCH_REGS = 65536 / THREADS / 8 * 8;
    static_assert(256 * SOFTMAX_REGS + (THREADS - 256) * OTHER_REGS <= THREADS * LAUNCH_REGS, "");
    static constexpr int TILE_BYTES = STEP * D * 2;            // K or V of a step, 16-bit
    static constexpr int Q_BYTES = HALF * D * 2;               // one half's queries
    static constexpr int STAGES = D == 128 ? 4 : 8;
    static constexpr int OUT_PIECE = Q8 ? 64 : 128;            // bytes of a row that a warp writes at once
    static constexpr int OUT_BYTES = 8 * 32 * OUT_PIECE;
    static constexpr int SCALE_BUFS = STAGES / 2 + 1;
    static constexpr int SCALES = Q8 ? SCALE_BUFS * 3 * STEP * 4 : 0;
    static constexpr bool Q_RANGE = Q8 && !std::is_same<T, __half>::value;   // bf16 queries become fp16: see Q_LIFT
    static constexpr int Q_SCALES = Q_RANGE ? 2 * ROWS * 4 : 0;
    static constexpr int HEAD = 1024;                          // barriers, the cursor, the tensor memory address
    static constexpr int SMEM = 1024 /*alignment*/ + HEAD + 2 * Q_BYTES + STAGES * TILE_BYTES + OUT_BYTES + SCALES + Q_SCALES;
    static_assert(SMEM <= (int)SMEM_LIMIT, "");
};
// bf16 queries meet the fp16 values of an 8-bit cache, lifted by 2^9, which the scales take back: a row whose largest element is in
// [2^-3, 2^6) then has it in [2^6, 2^15), and any other row is brought to [2^13, 2^14) by a power of two of its own, which
// costs its warp a multiplication a score.  Elements down to 2^-23 of the row's largest are exact, smaller ones rounded to
// within 2^-31 of it.
constexpr int Q_LIFT = 9;
template <typename T, int FMT> struct MatType { using type = __half; };
template <typename T> struct MatType<T, HOS_KV_SAME> { using type = T; };

// --- barriers ---------------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
constexpr long long WAIT_CYCLES = 4000000000ll;        // about two seconds
// The whole warp waits for the phase; false (for all lanes) after two seconds or once another role has given up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    if (__all_sync(FULL, bar_try(bar, parity))) return true;
    const uint32_t t0 = (uint32_t)(clock64() >> 16);
#pragma unroll 1
    for (;;) {
        if (__all_sync(FULL, bar_try(bar, parity))) return true;
        if ((uint32_t)(clock64() >> 16) - t0 > (uint32_t)(WAIT_CYCLES >> 16)) *gave_up = 1;
        if (__any_sync(FULL, *gave_up != 0)) return false;
    }
}
// The same for one wait at the end of a role, whatever the others do.
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!bar_try(bar, parity) && clock64() - t0 < WAIT_CYCLES) {}
}

// --- tcgen05 ----------------------------------------------------------------------------------
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
// D[128][N] (+)= A[128][16] B[N][16]^T, both in shared memory, A_STEP and B_STEP (16-byte units) past the descriptors' addresses.
// (Added in here so that the sums of every step of a product are not kept in registers.)
template <int A_STEP, int B_STEP> __device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{ .reg .pred p; .reg .b64 x, y; setp.ne.u32 p, %4, 0; add.s64 x, %1, %5; add.s64 y, %2, %6;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p; }"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "n"(A_STEP), "n"(B_STEP) : "memory");
}
// The same with A in tensor memory, A_STEP columns past its address.
template <int A_STEP, int B_STEP> __device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{ .reg .pred p; .reg .b32 x; .reg .b64 y; setp.ne.u32 p, %4, 0; add.u32 x, %1, %5; add.s64 y, %2, %6;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [x], y, %3, p; }"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "n"(A_STEP), "n"(B_STEP) : "memory");
}
// f(step tag) for FIRST .. END - 1
template <int FIRST, int END, typename F> __device__ __forceinline__ void each_step(F&& f) {
    if constexpr (FIRST < END) {
        f(IntTag<FIRST>{});
        each_step<FIRST + 1, END>(f);
    }
}
#define HOS_R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define HOS_W8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
// 32 columns of this thread's row of tensor memory.
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t* x) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : HOS_R8(x, 0), HOS_R8(x, 8), HOS_R8(x, 16), HOS_R8(x, 24) : "r"(addr));
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t* x) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : HOS_R8(x, 0), HOS_R8(x, 8) : "r"(addr));
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t* x) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 :: HOS_W8(x, 0), HOS_W8(x, 8), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory operands: rows of 128 bytes (64 elements along head_dim), the 16-byte chunk c of row r at c ^ (r & 7);
// a tile of head_dim 128 is two such blocks of 128 rows, one after the other.
constexpr int BLOCK_BYTES = 128 * 128;
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead_bytes) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(lead_bytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
constexpr uint32_t instr_desc(bool bf16, bool b_along_n, int n) {
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((b_along_n ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

// One lane of the (converged) warp; the compiler knows that it is one, so the operands of the matrix
// instructions stay in uniform registers.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p; }" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(FULL, x, 0); }

template <int N> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(N)); }
template <int N> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(N)); }

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Two 32-bit floats in one instruction.
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 f2_split(F2 x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void lds_f2x2(uint32_t addr, F2& a, F2& b) {
    asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "r"(addr));
}
__device__ __forceinline__ void st_shared16(uint32_t addr, const uint4& v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" :: "r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Named barrier of 128 threads (whole warps); true if `mine` holds in all of them.
__device__ __forceinline__ bool all_of_four_warps(bool mine) {
    uint32_t all;
    asm volatile("{ .reg .pred p, q; setp.ne.u32 p, %1, 0; bar.red.and.pred q, 1, 128, p; selp.u32 %0, 1, 0, q; }"
                 : "=r"(all) : "r"((uint32_t)mine) : "memory");
    return all != 0;
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

struct Shared {                                // in the first HEAD bytes
    uint64_t bars[48];
    Cursor first;
    long long lo, total, active;
    int share;                                 // steps of this CTA
    uint32_t tmem;
    int gave_up;
};
static_assert(sizeof(Shared) <= 1024, "");

struct Segment { int blocks; bool starts, ends; };   // steps of the current tile that are this CTA's; whether it has the first, the last

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(Cfg<T, FMT, D>::THREADS, 1)
k_attn_chunk(const __grid_constant__ AttnView a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
             const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap o_map, const bool q_tma, const bool o_tma,
             const int min_rows, Partial* __restrict__ meta, RowState* __restrict__ state, float* __restrict__ part) {
    using C = Cfg<T, FMT, D>;
    using M = typename MatType<T, FMT>::type;
    constexpr bool BF16 = std::is_same<M, __nv_bfloat16>::value;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    Shared& sh = *reinterpret_cast<Shared*>(base);
    volatile int* gave_up = &sh.gave_up;
    const uint32_t q_smem = smem_u32(base) + C::HEAD, ring = q_smem + 2 * C::Q_BYTES;
    const uint32_t out_buf = ring + C::STAGES * C::TILE_BYTES, scales = out_buf + C::OUT_BYTES;          // [buffer][scale log2(e) ks | log2 vs | 1 / vs][token]
    const uint32_t q_scales = scales + C::SCALES;                      // [tile parity][row]: what a row of queries was divided by
    const uint32_t bar0 = smem_u32(sh.bars);
    auto kv_full = [&](uint32_t i) { return bar0 + 8 * i; };
    auto kv_free = [&](uint32_t i) { return bar0 + 8 * (C::STAGES + i); };
    const uint32_t bar1 = bar0 + 16 * C::STAGES;
    auto q_full = [&](int h) { return bar1 + 8 * h; };
    auto q_free = [&](int h) { return bar1 + 16 + 8 * h; };
    auto s_full = [&](int h) { return bar1 + 32 + 8 * h; };
    auto p_ready = [&](int h) { return bar1 + 48 + 8 * h; };
    auto o_done = [&](int h) { return bar1 + 64 + 8 * h; };
    auto p_half = [&](int h) { return bar1 + 80 + 8 * h; };
    const uint32_t drain = bar1 + 96;
    auto raw_full = [&](uint32_t i) { return C::Q8 ? bar1 + 104 + 8 * i : kv_full(i); };   // what the copies report to
    auto scales_full = [&](uint32_t i) { return bar1 + 104 + 8 * (C::STAGES + i); };        // (8-bit cache) a step's scales
    static_assert(3 * C::STAGES + 13 + C::SCALE_BUFS <= sizeof(Shared::bars) / 8, "");
    const int warp = uniform(warp_id()), lane = lane_id(), w = (int)blockIdx.x;
    const List list{a, min_rows, 0x7FFFFFFF};
    // In this order: the row kernel of the same call starts on this signal and reads and writes at once what the kernels
    // before this one wrote and read.
    pdl_wait();
    pdl_launch_dependents();

    if (warp == 0) {
        long long mine;
        const long long total = list.total(w == 0, mine);
        const int active = (int)min((long long)gridDim.x, total);
        const long long lo = w < active ? total * w / active : 0, hi = w < active ? total * (w + 1) / active : 0;
        Cursor c = {};
        if (hi > lo) c = list.locate(lo, mine);
        if (lane == 0) {
            sh.first = c;
            sh.lo = lo;
            sh.share = (int)(hi - lo);
            sh.total = total;
            sh.active = active;
            sh.gave_up = 0;
            meta[w].last = -1;                 // until the softmax warps find a tile that begins here and ends in a later share
        }
    } else if (warp == 1 && lane == 0) {
        for (int i = 0; i < C::STAGES; ++i) {
            bar_init(kv_full(i), C::Q8 ? 4 : 1);
            bar_init(kv_free(i), 1);
            if (C::Q8) bar_init(raw_full(i), 1);
        }
        if (C::Q8)
            for (int i = 0; i < C::SCALE_BUFS; ++i) bar_init(scales_full(i), 4);
        for (int h = 0; h < 2; ++h) {
            bar_init(q_full(h), 1);
            bar_init(q_free(h), 1);
            bar_init(s_full(h), 1);
            bar_init(p_half(h), 4);
            bar_init(p_ready(h), 4);
            bar_init(o_done(h), 1);
        }
        bar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = (uint32_t)uniform((int)sh.tmem);
    const int share = sh.share;
    Cursor cur = sh.first;
    bool more = share > 0 && cur.step < list.end_of(cur, share);
    auto segment = [&]() {                                              // of the current tile
        Segment s;
        const int end = list.end_of(cur, share);
        s.blocks = end - cur.step;
        s.starts = cur.step == 0;
        s.ends = end == cur.t.steps;
        return s;
    };

    if (warp < 8) {
        // ================================ softmax and output ================================
        more_registers<C::SOFTMAX_REGS>();
        const int h = warp >> 2, row = (warp & 3) * 32 + lane;         // row of this half
        const uint32_t lane_at = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_tm = tmem + lane_at + h * 128, o_tm = tmem + lane_at + 256 + h * D;
        const float c = fmaxf(fabsf(a.scale_log2), 1.17549435e-38f);   // positive, so that masked scores stay -inf
        uint32_t s_phase = 0, o_phase = 0;
        uint32_t block = 0;                                           // steps this CTA has begun: ring item 2 * block is K
        uint32_t q_buf = 1;
        bool ok = true;
        // Rows of V outside the visible tokens may hold anything, and 0 * NaN is NaN: half 0's threads clear them before
        // either half's product (half 1's is issued later).
        auto clear_v = [&](int j0, uint32_t item) {
            const uint32_t stage = item % C::STAGES;
            if (!bar_wait(kv_full(stage), (item / C::STAGES) & 1, gave_up)) return false;
            if (j0 + row < cur.t.kb || j0 + row >= cur.t.ke) {
#pragma unroll 1
                for (int i = 0; i < D / 8; ++i)
                    st_shared16(ring + stage * C::TILE_BYTES + (i >> 3) * BLOCK_BYTES + row * 128 + (i & 7) * 16, make_uint4(0, 0, 0, 0));
            }
            fence_async_smem();
            return true;
        };
        for (; more && ok; more = list.next(cur, share)) {
            const Segment seg = segment();
            const bool active = cur.t.rows > h * HALF;
            q_buf ^= 1;
            if (!active) {
                block += seg.blocks;
                continue;
            }
            const int r = cur.tile * ROWS + h * HALF + row;
            const bool there = h * HALF + row < cur.t.rows;
            const int tok = by_group(a, r), hd = cur.head * a.group + r - tok * a.group;
            const int pos = cur.q.len - cur.q.n + tok;
            // rows past the tile see everything: no masking, and they are not written
            const int see_hi = !there ? 0x7FFFFFFF : a.causal ? min(cur.q.len, pos + 1) : cur.q.len;
            const int see_lo = there ? first_seen(a, pos) : 0;
            float m = -INFINITY, l = 0.0f;
#pragma unroll 1
            for (int b = 0; b < seg.blocks; ++b, ++block) {
                const int j0 = cur.t.k0 + (cur.step + b) * STEP;
                const int buf = C::Q8 ? (int)(block % C::SCALE_BUFS) : 0;
                if (!bar_wait(s_full(h), s_phase, gave_up)) { ok = false; break; }
                s_phase ^= 1;
                // The score follows from the step's scales (its K was reported full after them), so this is no wait in time: it makes
                // them visible.  K's own barrier would not do: its stage may be full of a later step's K by now.
                if (C::Q8 && !bar_wait(scales_full(buf), (block / C::SCALE_BUFS) & 1, gave_up)) { ok = false; break; }
                tc_fence_after();
                uint32_t s[128];
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_load32(s_tm + 32 * i, s + 32 * i);
                tmem_wait_load();
                float* x = reinterpret_cast<float*>(s);
                const uint32_t f_at = scales + buf * (3 * STEP * 4), lv_at = f_at + STEP * 4, iv_at = lv_at + STEP * 4;
                if (C::Q_RANGE) {
                    const float up = lds<float>(q_scales + (q_buf * ROWS + h * HALF + row) * 4);
                    if (__any_sync(FULL, up != 1.0f)) {
#pragma unroll
                        for (int i = 0; i < 128; ++i) x[i] *= up;
                    }
                }
                if (C::Q8) {
                    // y = x * (scale log2(e) ks) + log2 vs
#pragma unroll
                    for (int i = 0; i < 128; i += 4) {
                        F2 f0, f1, l0, l1;
                        lds_f2x2(f_at + 4 * i, f0, f1);
                        lds_f2x2(lv_at + 4 * i, l0, l1);
                        const float2 y0 = f2_split(f2_fma(f2(x[i], x[i + 1]), f0, l0)), y1 = f2_split(f2_fma(f2(x[i + 2], x[i + 3]), f1, l1));
                        x[i] = y0.x; x[i + 1] = y0.y; x[i + 2] = y1.x; x[i + 3] = y1.y;
                    }
                }
                if (__any_sync(FULL, j0 < see_lo || j0 + STEP > see_hi)) {
                    // only the 32 columns that some row's limits fall into are looked at one by one
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int first = see_lo - j0 - 32 * q, end = see_hi - j0 - 32 * q;
                        if (!__any_sync(FULL, first > 0 || end < 32)) continue;
                        const uint32_t below = end >= 32 ? FULL : (1u << max(end, 0)) - 1u;
                        const uint32_t keep = below & (first <= 0 ? FULL : first >= 32 ? 0u : FULL << first);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (!(keep & (1u << i))) x[32 * q + i] = -INFINITY;
                    }
                }
                float tops[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) tops[i] = fmaxf(x[2 * i], x[2 * i + 1]);
#pragma unroll
                for (int i = 8; i < 128; i += 2) tops[(i >> 1) & 3] = max3(tops[(i >> 1) & 3], x[i], x[i + 1]);
                float top = max3(fmaxf(tops[0], tops[1]), tops[2], tops[3]);
                if (!C::Q8) top *= c;
                if (b == 0) {
                    m = top - LIFT<M>;
                } else if (__any_sync(FULL, top > m + (GROWTH + LIFT<M>))) {
                    // the products up to the previous step are complete (this step's score was issued after them)
                    const float mn = fmaxf(m, top - LIFT<M>);
                    const float by = mn == -INFINITY ? 1.0f : exp2_fast(m - mn);
                    m = mn;
                    l *= by;
#pragma unroll 1
                    for (int i = 0; i < D / 16; ++i) {
                        uint32_t o[16];
                        tmem_load16(o_tm + 16 * i, o);
                        tmem_wait_load();
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * by);
                        tmem_store16(o_tm + 16 * i, o);
                    }
                }
                const float ms = m == -INFINITY ? 0.0f : m;
                const F2 c2 = f2(c, c), m2 = f2(-ms, -ms);
                F2 sums[2] = {0, 0};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t p[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const int j = 32 * q + 2 * i;
                        F2 e[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const F2 v = f2(x[j + 2 * k], x[j + 2 * k + 1]);
                            const float2 z = f2_split(C::Q8 ? f2_add(v, m2) : f2_fma(v, c2, m2));
                            const float2 w2 = make_float2(exp2_fast(z.x), exp2_fast(z.y));
                            p[i + k] = Pair<M>::pack(w2.x, w2.y);
                            e[k] = f2(w2.x, w2.y);
                        }
                        if (C::Q8) {
                            F2 iv0, iv1;
                            lds_f2x2(iv_at + 4 * j, iv0, iv1);
                            sums[0] = f2_fma(e[0], iv0, sums[0]);
                            sums[1] = f2_fma(e[1], iv1, sums[1]);
                        } else {
                            sums[0] = f2_add(sums[0], e[0]);
                            sums[1] = f2_add(sums[1], e[1]);
                        }
                    }
                    tmem_store16(s_tm + 16 * q, p);
                    if (q == FIRST_PART / 32 - 1) {
                        // these may be multiplied while the rest is worked out
                        if (!C::Q8 && h == 0 && (j0 < cur.t.kb || j0 + STEP > cur.t.ke)) {
                            ok = clear_v(j0, 2 * block + 1);
                            if (!ok) break;
                        }
                        tmem_wait_store();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive(p_half(h));
                    }
                }
                if (!ok) break;
                const float2 sum = f2_split(f2_add(sums[0], sums[1]));
                l += sum.x + sum.y;
                tmem_wait_store();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_ready(h));
            }
            if (!ok) break;
            // --- output ---
            if (!bar_wait(o_done(h), o_phase, gave_up)) { ok = false; break; }
            o_phase ^= 1;
            tc_fence_after();
            const bool whole = seg.starts && seg.ends;
            const int slot = 2 * w + (seg.starts ? 1 : 0);
            const float by = l == 0.0f ? 0.0f : 1.0f / l;
            // A lane has a row.  Whole tiles: PIECE bytes of each of the warp's 32 rows at a time go through shared memory, from where
            // they leave by TMA, or, where the rows are not all there or not a box of the output, eight (four) lanes to a row.
            constexpr int PIECE = C::OUT_PIECE, CHUNKS = PIECE / 16;
            const uint32_t buf_at = out_buf + warp * 32 * PIECE;
            auto place = [&](int r, int ch) { return buf_at + r * PIECE + (ch ^ (CHUNKS == 8 ? r & 7 : (r >> 1) & 3)) * 16; };
            if (whole) {
                const bool by_tma = o_tma && __all_sync(FULL, there);
                unsigned char* dst = a.out + 2 * ((long long)(cur.q.off + tok) * a.o_tok + (long long)hd * a.o_head);
#pragma unroll 1
                for (int i = 0; i < D / (PIECE / 2); ++i) {             // PIECE / 2 columns become PIECE bytes
                    uint32_t o[PIECE / 2];
#pragma unroll
                    for (int k = 0; k < PIECE / 64; ++k) tmem_load32(o_tm + i * (PIECE / 2) + 32 * k, o + 32 * k);
                    tmem_wait_load();
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");   // the buffer has been read
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < PIECE / 4; ++k) o[k] = Pair<T>::pack(__uint_as_float(o[2 * k]) * by, __uint_as_float(o[2 * k + 1]) * by);
#pragma unroll
                    for (int ch = 0; ch < CHUNKS; ++ch) st_shared16(place(lane, ch), make_uint4(o[4 * ch], o[4 * ch + 1], o[4 * ch + 2], o[4 * ch + 3]));
                    if (by_tma) {
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
                                         :: "l"(&o_map), "r"(i * (PIECE / 2)), "r"(hd), "r"(cur.q.off + tok), "r"(buf_at) : "memory");
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                    } else {
                        __syncwarp();
#pragma unroll
                        for (int k = 0; k < CHUNKS; ++k) {
                            const int r2 = k * (32 / CHUNKS) + lane / CHUNKS, ch = lane % CHUNKS;
                            unsigned char* to = reinterpret_cast<unsigned char*>(__shfl_sync(FULL, reinterpret_cast<unsigned long long>(there ? dst : nullptr), r2));
                            const uint4 x4 = lds<uint4>(place(r2, ch));
                            if (to) *reinterpret_cast<uint4*>(to + i * PIECE + ch * 16) = x4;
                        }
                        __syncwarp();
                    }
                }
            } else {
                // a piece: four columns of every row together, so that the lanes' 16 bytes lie next to each other
                float* dst = part + (long long)slot * ROWS * D + (h * HALF + row) * 4;
#pragma unroll 1
                for (int i = 0; i < D / 32; ++i) {
                    uint32_t o[32];
                    tmem_load32(o_tm + i * 32, o);
                    tmem_wait_load();
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        *reinterpret_cast<uint4*>(dst + (long long)(i * 8 + k) * (ROWS * 4)) = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                }
            }
            if (there) {
                if (whole) {
                    if (a.lse) a.lse[(long long)(cur.q.off + tok) * a.n_heads + hd] = row_lse<!C::Q8>(m, l);
                } else {
                    state[(long long)slot * ROWS + h * HALF + row] = RowState{m, l};
                }
            }
            if (!whole && seg.starts && h == 0 && row == 0) {
                const long long end = sh.lo + cur.at + TILE_STEPS + cur.t.steps;
                meta[w] = Partial{cur.seq, cur.head, cur.tile, (int)((end * sh.active - 1) / sh.total)};
            }
            tc_fence_before();
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else {
        fewer_registers<C::OTHER_REGS>();
        if (warp == 8) {
            // ================================ K and V by TMA ================================
            const int box = min(STEP, 1 << a.kv.page_shift), pieces = STEP / box;
            uint32_t item = 0;
            for (; more; more = list.next(cur, share)) {
                const Segment seg = segment();
                bool ok = true;
                for (int b = 0; b < seg.blocks && ok; ++b) {
                    const int j0 = cur.t.k0 + (cur.step + b) * STEP, j = j0 + lane * box;
                    int page = a.kv.n_pages;                            // past the pool: TMA fills with zeros
                    if (lane < pieces && j < cur.t.ke && j + box > cur.t.kb) {
                        const int p = __ldg(a.kv.table + (long long)cur.seq * a.kv.table_stride + (j >> a.kv.page_shift));
                        if ((unsigned)p < (unsigned)a.kv.n_pages) page = p;
                        else if (a.kv.status) atomicOr(a.kv.status + cur.seq, HOS_ST_INVALID);
                    }
                    for (int kv = 0; kv < 2; ++kv, ++item) {
                        const int stage = item % C::STAGES;
                        const uint32_t round = item / C::STAGES;
                        if (!bar_wait(kv_free(stage), (round & 1) ^ 1, gave_up)) { ok = false; break; }
                        if (lane == 0) bar_expect(raw_full(stage), C::Q8 ? C::TILE_BYTES / 2 : C::TILE_BYTES);
                        __syncwarp();
                        if (lane < pieces) {
                            // codes land in the second half of the stage that their fp16 values will fill
#pragma unroll
                            for (int half = 0; half < (C::Q8 ? 1 : D / 64); ++half)
                                asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                                             :: "r"(ring + stage * C::TILE_BYTES +
                                                    (C::Q8 ? C::TILE_BYTES / 2 + lane * box * D : half * BLOCK_BYTES + lane * box * 128)),
                                                "l"(kv ? &v_map : &k_map), "r"(half * 64), "r"(j & ((1 << a.kv.page_shift) - 1)), "r"(cur.head), "r"(page),
                                                "r"(raw_full(stage)) : "memory");
                        }
                    }
                }
                if (!ok) break;
            }
            // leave only when every copy has landed
            for (uint32_t i = item > C::STAGES ? item - C::STAGES : 0; i < item; ++i) bar_drain(raw_full(i % C::STAGES), (i / C::STAGES) & 1);
        } else if (warp == 9) {
            // ================================ the products ================================
            constexpr uint32_t QK = instr_desc(BF16, false, STEP), PV = instr_desc(BF16, true, D);
            uint32_t q_phase = 0, p_phase[2] = {0, 0};
            uint32_t item = 0;                                         // ring items consumed
            bool ok = true, issued = false;
            auto product_qk = [&](int h, int stage) {
                const uint64_t qa = smem_desc(q_smem + h * C::Q_BYTES, 16), kb = smem_desc(ring + stage * C::TILE_BYTES, 16);
                each_step<0, D / 16>([&](auto t) {
                    constexpr int k = decltype(t)::value, step = ((k >> 2) * BLOCK_BYTES + (k & 3) * 32) >> 4;
                    mma_ss<step, step>(tmem + h * 128, qa, kb, QK, k > 0);
                });
                tc_commit(s_full(h));
            };
            auto product_pv = [&](int h, int stage, bool add, auto part_of) {
                const uint64_t vb = smem_desc(ring + stage * C::TILE_BYTES, BLOCK_BYTES);
                constexpr bool first = decltype(part_of)::value == 0;
                each_step<first ? 0 : FIRST_PART / 16, (first ? FIRST_PART : STEP) / 16>([&](auto t) {
                    constexpr int k = decltype(t)::value;
                    mma_ts<8 * k, k * 16 * 128 / 16>(tmem + 256 + h * D, tmem + h * 128, vb, PV, add || k > 0);
                });
            };
            for (; more && ok; more = list.next(cur, share)) {
                const Segment seg = segment();
                const int halves = uniform(cur.t.rows > HALF ? 2 : 1), blocks = uniform(seg.blocks);
                for (int h = 0; h < 2 && ok; ++h) ok = bar_wait(q_full(h), q_phase, gave_up);
                q_phase ^= 1;
                if (ok) ok = bar_wait(kv_full(item % C::STAGES), (item / C::STAGES) & 1, gave_up);
                if (!ok) break;
                tc_fence_after();
                issued = true;
                if (elect_one()) {
                    for (int h = 0; h < halves; ++h) product_qk(h, item % C::STAGES);
                    tc_commit(kv_free(item % C::STAGES));
                    if (blocks == 1) { tc_commit(q_free(0)); tc_commit(q_free(1)); }
                }
                __syncwarp();
                for (int b = 0; b < blocks; ++b) {
                    const uint32_t vi = item + 1, ki = item + 2;
                    const bool more = b + 1 < blocks;
                    ok = bar_wait(kv_full(vi % C::STAGES), (vi / C::STAGES) & 1, gave_up);
                    if (ok && more) ok = bar_wait(kv_full(ki % C::STAGES), (ki / C::STAGES) & 1, gave_up);
                    if (!ok) break;
                    for (int h = 0; h < halves; ++h) {
                        // the weights come in two parts
                        ok = bar_wait(p_half(h), p_phase[h], gave_up);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) product_pv(h, vi % C::STAGES, b > 0, IntTag<0>{});
                        __syncwarp();
                        ok = bar_wait(p_ready(h), p_phase[h], gave_up);
                        if (!ok) break;
                        p_phase[h] ^= 1;
                        tc_fence_after();
                        if (elect_one()) {
                            product_pv(h, vi % C::STAGES, true, IntTag<1>{});
                            if (more) product_qk(h, ki % C::STAGES); else tc_commit(o_done(h));
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect_one()) {
                        tc_commit(kv_free(vi % C::STAGES));
                        if (more) tc_commit(kv_free(ki % C::STAGES));
                        if (b + 2 == blocks) { tc_commit(q_free(0)); tc_commit(q_free(1)); }
                    }
                    __syncwarp();
                    item += 2;
                }
            }
            // nothing of this warp's is in flight when the tensor memory is given back
            if (issued && elect_one()) {
                tc_commit(drain);
                bar_drain(drain, 0);
            }
            __syncwarp();
        } else if (warp == 10 || warp == 11) {
            // ================================ queries ================================
            constexpr int CH = D / 8;                                   // 16-byte chunks of a row
            const int h = warp - 10;
            const uint32_t dst = q_smem + h * C::Q_BYTES;
            const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;   // the softmax works with |scale|
            uint32_t phase = 1, q_buf = 0, last = 2;                             // the first wait falls through
            for (; more; more = list.next(cur, share)) {
                const Segment seg = segment();
                if (!bar_wait(q_free(h), phase, gave_up)) break;
                phase ^= 1;
                if (q_tma) {
                    // a row is a token's query head: 128 rows are 128 / group whole tokens
                    if (lane == 0) {
                        bar_expect(q_full(h), C::Q_BYTES);
#pragma unroll
                        for (int half = 0; half < D / 64; ++half)
                            asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                                         :: "r"(dst + half * BLOCK_BYTES), "l"(&q_map), "r"(half * 64), "r"(cur.head * a.group),
                                            "r"(cur.q.off + by_group(a, cur.tile * ROWS + h * HALF)), "r"(q_full(h)) : "memory");
                    }
                    __syncwarp();
                    last = phase;
                    continue;
                }
                constexpr int BATCH = 8;                                // loads in flight
#pragma unroll 1
                for (int r0 = 0; r0 < HALF; r0 += 32) {
                  // lane l knows where row r0 + l is
                  const int pr = cur.tile * ROWS + h * HALF + r0 + lane, tok = by_group(a, pr), hd = cur.head * a.group + pr - tok * a.group;
                  const long long where = h * HALF + r0 + lane < cur.t.rows ? (long long)(cur.q.off + tok) * a.q_tok + (long long)hd * a.q_head : -1;
#pragma unroll 1
                  for (int i0 = 0; i0 < CH; i0 += BATCH) {
                    uint4 batch[BATCH];
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
                      const int id = (i0 + i) * 32 + lane;
                      const long long from = __shfl_sync(FULL, where, id / CH);
                      batch[i] = make_uint4(0, 0, 0, 0);
                      if (from >= 0) batch[i] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.q) + from + (id % CH) * 8));
                    }
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
                    const int id = (i0 + i) * 32 + lane, r = r0 + id / CH, ch = id % CH;
                    const uint4 v = batch[i];
                    uint32_t x[4] = {v.x ^ flip, v.y ^ flip, v.z ^ flip, v.w ^ flip};
                    if (C::Q_RANGE) {
                        // rows of zeros, of nothing above 2^-100 and non-finite ones get the lift alone
                        float2 f[4];
                        float top = 0.0f;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            f[k] = Pair<T>::unpack(x[k]);
                            top = fmaxf(top, fmaxf(fabsf(f[k].x), fabsf(f[k].y)));
                        }
#pragma unroll
                        for (int d = CH / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, d));
                        const int ex = (int)(__float_as_uint(top) >> 23);
                        const int sh = ex >= 27 && ex < 254 && (ex < 127 - 3 || ex >= 127 + 6) ? 140 - ex : Q_LIFT;
                        const float up = __uint_as_float((uint32_t)(127 + sh) << 23);
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[k] = Pair<__half>::pack(f[k].x * up, f[k].y * up);
                        if (ch == 0)
                            asm volatile("st.shared.f32 [%0], %1;" :: "r"(q_scales + (q_buf * ROWS + h * HALF + r) * 4),
                                         "f"(__uint_as_float((uint32_t)(127 + Q_LIFT - sh) << 23)) : "memory");
                    }
                    st_shared16(dst + (ch >> 3) * BLOCK_BYTES + r * 128 + ((ch & 7) ^ (r & 7)) * 16, make_uint4(x[0], x[1], x[2], x[3]));
                    }
                  }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) bar_arrive(q_full(h));
                q_buf ^= 1;
            }
            if (last < 2) bar_drain(q_full(h), last);                   // the last copy has landed
        } else if (C::Q8 && warp >= 12) {
            // ================================ K and V of an 8-bit cache ================================
            // The four warps take a tile's codes out of the second half of its stage, wait for one another, and fill the
            // stage with fp16 in the layout that the products read.
            constexpr int LANES = D / 16, PASSES = LANES, PER_PASS = 128 / LANES;
            const int tid = (int)threadIdx.x - 384, sub = tid % LANES, row0 = tid / LANES;
            const float c = fabsf(a.scale_log2) * (C::Q_RANGE ? 1.0f / (1 << Q_LIFT) : 1.0f);
            float ks = 0.0f, vs = 0.0f;
            bool seen = false;
            // this thread's token's scales, on their way while the step before is converted
            auto fetch_scales = [&]() {
                const int j = cur.t.k0 + cur.step * STEP + tid;
                seen = false;
                if (j < cur.t.kb || j >= cur.t.ke) return;
                const int p = __ldg(a.kv.table + (long long)cur.seq * a.kv.table_stride + (j >> a.kv.page_shift));
                if ((unsigned)p >= (unsigned)a.kv.n_pages) return;
                const long long e = scale_elem(a.kv, p, cur.head, j & ((1 << a.kv.page_shift) - 1));
                ks = __ldg(a.kv.k_scale + e);
                vs = __ldg(a.kv.v_scale + e);
                seen = true;
            };
            // Rows outside [first, end) become zeros.  A warp whose wait ran out still comes to the named barrier, which knows no limit:
            // the four warps vote there and leave together.
            auto convert = [&](uint32_t item, int first, int end, bool ok) {
                const uint32_t stage = item % C::STAGES, at = ring + stage * C::TILE_BYTES;
                ok = ok && bar_wait(raw_full(stage), (item / C::STAGES) & 1, gave_up);
                uint4 x[PASSES];
#pragma unroll
                for (int i = 0; i < PASSES; ++i) {
                    const int r = i * PER_PASS + row0;
                    x[i] = lds<uint4>(at + C::TILE_BYTES / 2 + r * D + sub * 16);
                    if (r < first || r >= end) x[i] = make_uint4(0, 0, 0, 0);
                }
                if (!all_of_four_warps(ok)) return false;
#pragma unroll
                for (int i = 0; i < PASSES; ++i) {
                    const int r = i * PER_PASS + row0;
                    const uint2 c0 = codes_to_half4<FMT>(x[i].x), c1 = codes_to_half4<FMT>(x[i].y);
                    const uint2 c2 = codes_to_half4<FMT>(x[i].z), c3 = codes_to_half4<FMT>(x[i].w);
                    const uint4 lo4 = make_uint4(c0.x, c0.y, c1.x, c1.y), hi4 = make_uint4(c2.x, c2.y, c3.x, c3.y);
                    // lanes 4-7 of a row go to the other block of the tile: they store their chunks the other way
                    // round, so that eight lanes always fill eight different chunk positions
                    const bool swap = sub & 4;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int ch = sub * 2 + (swap ? 1 - e : e);
                        st_shared16(at + (ch >> 3) * BLOCK_BYTES + r * 128 + ((ch & 7) ^ (r & 7)) * 16, (e == 0) != swap ? lo4 : hi4);
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) bar_arrive(kv_full(stage));
                return true;
            };
            if (more) fetch_scales();
            int end_step = list.end_of(cur, share);
            for (int block = 0; more; ++block) {
                const int j0 = cur.t.k0 + cur.step * STEP, first = cur.t.kb - j0, end = cur.t.ke - j0;
                const uint32_t item = 2 * block;
                // The buffer's last reader was done before the stage that V of this step will take was free, and K's
                // copy was issued after that.
                const bool ok = bar_wait(raw_full(item % C::STAGES), (item / C::STAGES) & 1, gave_up);
                const uint32_t sc = scales + (block % C::SCALE_BUFS) * (3 * STEP * 4) + tid * 4;
                const float v1 = fmaxf(vs, LEAST_V_SCALE);
                const float f = seen ? c * ks : 0.0f, lv = seen ? (vs != vs ? vs : __log2f(v1)) : -INFINITY, iv = seen ? 1.0f / v1 : 0.0f;
                asm volatile("st.shared.f32 [%0], %1;" :: "r"(sc), "f"(f) : "memory");
                asm volatile("st.shared.f32 [%0], %1;" :: "r"(sc + STEP * 4), "f"(lv) : "memory");
                asm volatile("st.shared.f32 [%0], %1;" :: "r"(sc + 2 * STEP * 4), "f"(iv) : "memory");
                __syncwarp();
                if (lane == 0) bar_arrive(scales_full(block % C::SCALE_BUFS));
                if (++cur.step == end_step) {
                    more = list.next(cur, share);
                    end_step = list.end_of(cur, share);
                }
                if (more) fetch_scales();
                if (!convert(item, first, end, ok) || !convert(item + 1, first, end, true)) break;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*gave_up && threadIdx.x == 0 && a.kv.status) {
        // whichever wait ran out: rows of any sequence in this share may be missing
        Cursor c = sh.first;
        do atomicOr(a.kv.status + c.seq, HOS_ST_LIMIT);
        while (list.next(c, share));
    }
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem));
}

// Tensor map of k or v: {head_dim, row in page, KV head, page}, boxes of 64 elements (8-bit: whole rows) by (part of) a page.
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                CUtensorMapFloatOOBfill);
EncodeTiled encoder() {
    static EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}
bool make_map(CUtensorMap* map, const KvView& c, void* base) {
    const EncodeTiled f = encoder();
    if (!f) return false;
    const int page = 1 << c.page_shift;
    const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)page, (cuuint64_t)c.n_kv, (cuuint64_t)c.n_pages};
    const cuuint64_t bytes = c.k_scale ? 1 : 2;
    const cuuint64_t strides[3] = {c.head_dim * bytes, (cuuint64_t)page * c.head_dim * bytes, (cuuint64_t)c.page_stride * bytes};
    const cuuint32_t box[4] = {bytes == 1 ? (cuuint32_t)c.head_dim : 64, (cuuint32_t)(page < STEP ? page : STEP), 1, 1}, one[4] = {1, 1, 1, 1};
    return f(map, bytes == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, base, dims, strides, box, one,
             CU_TENSOR_MAP_INTERLEAVE_NONE, bytes == 1 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows of queries or outputs: {head_dim, head, token}; a box is `columns` of `rows` consecutive rows of a KV head, token by token.
// False where these are no box (or the strides are none that a tensor map can hold, such as those of an expanded tensor).
bool make_rows_map(CUtensorMap* map, const AttnView& a, const unsigned char* base, long long tok, long long head, int columns, int rows) {
    const EncodeTiled f = encoder();
    const int heads = a.group < rows ? a.group : rows;
    if (!f || rows % heads || a.group % heads || head <= 0 || tok <= 0) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)a.kv.head_dim, (cuuint64_t)a.n_heads, (cuuint64_t)a.kv.n_tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)head * 2, (cuuint64_t)tok * 2};
    const cuuint32_t box[3] = {(cuuint32_t)columns, (cuuint32_t)heads, (cuuint32_t)(rows / heads)}, one[3] = {1, 1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<unsigned char*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
             columns == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int FMT, int D>
cudaError_t run(const AttnView& a, int min_rows, const AttnWs& ws, cudaStream_t st) {
    using C = Cfg<T, FMT, D>;
    cudaError_t e = allow_max_dynamic_smem(reinterpret_cast<const void*>(&k_attn_chunk<T, FMT, D>));
    if (e != cudaSuccess) return e;
    CUtensorMap km = {}, vm = {}, qm = {}, om = {};
    // Queries come by TMA where 128 rows are a box and nothing has to be done to them on the way; else by two warps.  (A tile's 128
    // rows begin at a whole token where the group divides 128.)
    const bool q_tma = !C::Q_RANGE && HALF % a.group == 0 && a.scale_log2 >= 0.0f && make_rows_map(&qm, a, a.q, a.q_tok, a.q_head, 64, HALF);
    const bool o_tma = make_rows_map(&om, a, a.out, a.o_tok, a.o_head, C::OUT_PIECE / 2, 32);
    if (!make_map(&km, a.kv, a.kv.k) || !make_map(&vm, a.kv, a.kv.v)) return cudaErrorInvalidValue;
    launch_hook("k_attn_chunk", 0, st);
    e = launch_early(k_attn_chunk<T, FMT, D>, dim3(ATTN_SMS), C::THREADS, C::SMEM, st, a, km, vm, qm, om, q_tma, o_tma, min_rows, ws.meta, ws.state,
                     ws.part);
    launch_hook("k_attn_chunk", 1, st);
    return e;
}

}  // namespace

cudaError_t launch_attn_chunk(const AttnView& a, int type, int format, int min_rows, const AttnWs& ws, cudaStream_t st) {
    return kv_dispatch(type, format, a.kv.head_dim, [&](auto t, auto f, auto d) {
        return run<typename decltype(t)::type, decltype(f)::value, decltype(d)::value>(a, min_rows, ws, st);
    });
}

}  // namespace hos
