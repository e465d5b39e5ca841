// C-ABI layer of the KV-cache calls: argument validation, workspace carving, kernel sequencing.
#include <cmath>

#include "hos_kv_kernels.h"
#include "hos_kv.cuh"

namespace {

using namespace hos;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool multiple16(long long elems, int bytes) { return (elems * bytes) % 16 == 0; }

int check_cache(const hos_kv_cache* c) {
    if (!c || !c->k || !c->v) return HOS_E_INVALID;
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->page_stride < 0 || c->scale_page_stride < 0) return HOS_E_INVALID;
    if (c->type != HOS_TYPE_BF16 && c->type != HOS_TYPE_FP16) return HOS_E_INVALID;
    if (c->format != HOS_KV_SAME && c->format != HOS_KV_E4M3 && c->format != HOS_KV_INT8) return HOS_E_INVALID;
    const bool coded = c->format != HOS_KV_SAME;
    if (coded && (!c->k_scale || !c->v_scale)) return HOS_E_INVALID;
    if (c->head_dim != 64 && c->head_dim != 128) return HOS_E_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return HOS_E_UNSUPPORTED;
    const long long rows = (long long)c->n_kv_heads * c->page_size;
    if (rows * c->head_dim >= (1ll << 31)) return HOS_E_UNSUPPORTED;
    if (c->page_stride && c->page_stride < rows * c->head_dim) return HOS_E_INVALID;
    if (coded && c->scale_page_stride && c->scale_page_stride < rows) return HOS_E_INVALID;
    if (!aligned16(c->k) || !aligned16(c->v) || !multiple16(c->page_stride, coded ? 1 : 2)) return HOS_E_INVALID;
    if (coded && (!aligned16(c->k_scale) || !aligned16(c->v_scale) || !multiple16(c->scale_page_stride, 4)))
        return HOS_E_INVALID;
    return HOS_OK;
}

int check_kv_batch(const hos_kv_cache* c, const hos_kv_batch* b) {
    if (!b || b->n_seq < 0 || b->n_tokens < 0 || b->max_new < 0 || b->max_pages < 0) return HOS_E_INVALID;
    if (b->n_seq == 0 || b->n_tokens == 0) return HOS_OK;
    if (!b->tok_off || !b->kv_len || (b->max_pages > 0 && !b->page_table) || b->max_new < 1) return HOS_E_INVALID;
    if (b->table_stride < b->max_pages) return HOS_E_INVALID;
    if ((long long)b->max_pages * c->page_size >= (1ll << 31) - 256) return HOS_E_UNSUPPORTED;   // positions are 32-bit
    return HOS_OK;
}

KvView view(const hos_kv_cache* c, const hos_kv_batch* b, int32_t* status) {
    KvView v;
    const long long rows = (long long)c->n_kv_heads * c->page_size;
    v.k = static_cast<unsigned char*>(c->k);
    v.v = static_cast<unsigned char*>(c->v);
    v.k_scale = c->format == HOS_KV_SAME ? nullptr : c->k_scale;
    v.v_scale = c->format == HOS_KV_SAME ? nullptr : c->v_scale;
    v.page_stride = c->page_stride ? c->page_stride : rows * c->head_dim;
    v.scale_page_stride = c->scale_page_stride ? c->scale_page_stride : rows;
    v.tok_off = b->tok_off;
    v.kv_len = b->kv_len;
    v.table = b->page_table;
    v.table_stride = b->table_stride;
    v.status = status;
    v.n_pages = c->n_pages;
    v.page_shift = 0;
    while ((1 << v.page_shift) < c->page_size) ++v.page_shift;
    v.n_kv = c->n_kv_heads;
    v.head_dim = c->head_dim;
    v.n_seq = b->n_seq;
    v.n_tokens = b->n_tokens;
    v.max_pages = b->max_pages;
    return v;
}

// An error is reported once: the runtime would hand it to the next call that asks for its last one, too.
inline int cuda_rc(cudaError_t e) {
    if (e == cudaSuccess) return HOS_OK;
    cudaGetLastError();
    return HOS_E_CUDA;
}

struct AttnSpace {
    AttnWs rows, chunks;
    size_t bytes;
};
AttnSpace carve_attention(int head_dim, void* ws) {
    AttnSpace s;
    unsigned char* base = static_cast<unsigned char*>(ws);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        unsigned char* p = base + off;
        off += (bytes + 255) & ~(size_t)255;
        return p;
    };
    auto carve = [&](size_t shares, size_t rows) {       // a share leaves two pieces at most
        AttnWs w;
        w.meta = reinterpret_cast<Partial*>(take(shares * sizeof(Partial)));
        w.state = reinterpret_cast<RowState*>(take(2 * rows * sizeof(RowState)));
        w.part = reinterpret_cast<float*>(take(2 * rows * (size_t)head_dim * 4));
        return w;
    };
    s.rows = carve((size_t)ATTN_SMS * ATTN_WORKERS_PER_SM, (size_t)ATTN_SMS * ATTN_ROWS_PER_SM);
    s.chunks = carve(ATTN_SMS, (size_t)ATTN_SMS * ATTN_CHUNK_ROWS);
    s.bytes = off;
    return s;
}

}  // namespace

extern "C" {

int hos_kv_append(const hos_kv_cache* c, const hos_kv_batch* b, const void* k, const void* v, int64_t k_tok_stride,
                  int64_t k_head_stride, int64_t v_tok_stride, int64_t v_head_stride, int32_t* status, void* stream) {
    int rc = check_cache(c);
    if (rc) return rc;
    if ((rc = check_kv_batch(c, b))) return rc;
    if (b->n_seq == 0 || b->n_tokens == 0) return HOS_OK;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return HOS_E_INVALID;
    if (c->n_kv_heads > KV_MOST_HEADS) return HOS_E_UNSUPPORTED;
    const long long st[4] = {k_tok_stride, k_head_stride, v_tok_stride, v_head_stride};
    for (long long s : st)
        if (!multiple16(s, 2)) return HOS_E_INVALID;
    return cuda_rc(launch_kv_append(view(c, b, status), c->type, c->format, k, v, st, static_cast<cudaStream_t>(stream)));
}

int hos_kv_read(const hos_kv_cache* c, const hos_kv_batch* b, void* k, void* v, int32_t* status, void* stream) {
    int rc = check_cache(c);
    if (rc) return rc;
    if ((rc = check_kv_batch(c, b))) return rc;
    if (b->n_tokens == 0) return HOS_OK;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return HOS_E_INVALID;
    if (c->n_kv_heads > KV_MOST_HEADS) return HOS_E_UNSUPPORTED;
    if (b->n_seq == 0) {                              // tokens of no sequence have no place, and read as zero
        const size_t bytes = (size_t)b->n_tokens * c->n_kv_heads * c->head_dim * 2;
        for (void* p : {k, v})
            if ((rc = cuda_rc(cudaMemsetAsync(p, 0, bytes, static_cast<cudaStream_t>(stream))))) return rc;
        return HOS_OK;
    }
    return cuda_rc(launch_kv_read(view(c, b, status), c->type, c->format, k, v, static_cast<cudaStream_t>(stream)));
}

size_t hos_paged_attention_workspace_bytes(const hos_kv_cache* c, const hos_kv_batch* b, int n_heads) {
    if (check_cache(c) || check_kv_batch(c, b) || n_heads < 1) return 0;
    return carve_attention(c->head_dim, nullptr).bytes;
}

int hos_paged_attention(const hos_kv_cache* c, const hos_kv_batch* b, const void* q, int64_t q_tok_stride,
                        int64_t q_head_stride, int n_heads, float sm_scale, int causal, int window, void* out,
                        int64_t out_tok_stride, int64_t out_head_stride, float* lse, int32_t* status, void* ws,
                        size_t ws_bytes, void* stream) {
    int rc = check_cache(c);
    if (rc) return rc;
    if ((rc = check_kv_batch(c, b))) return rc;
    if (n_heads < 1 || n_heads % c->n_kv_heads || window < 0 || !std::isfinite(sm_scale)) return HOS_E_INVALID;
    if ((long long)b->n_tokens * n_heads >= (1ll << 31) - 4096) return HOS_E_UNSUPPORTED;
    if (b->n_seq == 0 || b->n_tokens == 0) return HOS_OK;
    if (!q || !out || !aligned16(q) || !aligned16(out)) return HOS_E_INVALID;
    for (long long s : {(long long)q_tok_stride, (long long)q_head_stride, (long long)out_tok_stride, (long long)out_head_stride})
        if (!multiple16(s, 2)) return HOS_E_INVALID;
    const AttnSpace w = carve_attention(c->head_dim, ws);
    if (!ws || ws_bytes < w.bytes || (reinterpret_cast<uintptr_t>(ws) & 255)) return HOS_E_WORKSPACE;
    AttnView a;
    a.kv = view(c, b, status);
    a.q = static_cast<const unsigned char*>(q);
    a.q_tok = q_tok_stride;
    a.q_head = q_head_stride;
    a.out = static_cast<unsigned char*>(out);
    a.o_tok = out_tok_stride;
    a.o_head = out_head_stride;
    a.lse = lse;
    a.n_heads = n_heads;
    a.group = n_heads / c->n_kv_heads;
    a.group_shift = 0;
    while ((1ll << a.group_shift) < a.group) ++a.group_shift;
    a.group_magic = (uint32_t)((((1ull << a.group_shift) - a.group) << 32) / a.group + 1);
    a.scale_log2 = sm_scale * 1.44269504088896340736f;
    a.causal = causal != 0;
    a.window = window;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // A sequence has new tokens * group rows a KV head.  Up to 16: the row kernel, in tiles of 8 where that is enough for
    // all.  If there are larger ones, they go to the chunk kernel (all, if there is but one sequence), and the row kernel
    // keeps the single tokens: 8 rows, or 16 for groups above 8.
    const long long most = (long long)b->max_new * a.group;
    const bool chunks = most > 16, alone = b->n_seq == 1;
    const int tile = chunks ? (a.group <= 8 ? 8 : 16) : most <= 8 ? 8 : 16;
    int row_workers = 0;
    if (chunks && (rc = cuda_rc(launch_attn_chunk(a, c->type, c->format, alone ? 0 : tile, w.chunks, st)))) return rc;
    if (!(chunks && alone) && (rc = cuda_rc(launch_attn_rows(a, c->type, c->format, tile, chunks ? tile : 0x7FFFFFFF, chunks, w.rows,
                                                             &row_workers, st))))
        return rc;
    return cuda_rc(launch_attn_combine(a, c->type, chunks, w.chunks, tile, row_workers, w.rows, st));
}

}  // extern "C"
