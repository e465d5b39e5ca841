// C-ABI layer of the calls on a cache's pages and on drafted tokens: argument validation, workspace carving, launches.
#include <initializer_list>

#include "hos_pages_kernels.h"

namespace {

using namespace hos;

// Numbers of sequences and of pages add up in 32 bits (what is asked for may be more: its sums stop at 2^25, which no pool has).
constexpr int MOST_SEQS = 1 << 18, MOST_PAGES = 1 << 24;

inline int cuda_rc(cudaError_t e) {
    if (e == cudaSuccess) return HOS_OK;
    cudaGetLastError();                                              // reported once
    return HOS_E_CUDA;
}

// The sizes of a state (enough for a workspace's size); and that what they ask for is there, lengths only where `length` says so.
int check_sizes(const hos_kv_pages* p) {
    if (!p || p->n_pages < 1 || p->page_size < 1 || p->n_seq < 0 || p->max_pages < 0) return HOS_E_INVALID;
    if (p->n_pages > MOST_PAGES || p->n_seq > MOST_SEQS || (long long)p->max_pages * p->page_size >= (1ll << 31) - 256) return HOS_E_UNSUPPORTED;
    return HOS_OK;
}
int check_pages(const hos_kv_pages* p, bool length) {
    const int rc = check_sizes(p);
    if (rc) return rc;
    if (!p->refs || (p->n_seq > 0 && length && !p->kv_len)) return HOS_E_INVALID;
    if (p->n_seq > 0 && p->max_pages > 0 && (!p->page_table || p->table_stride < p->max_pages)) return HOS_E_INVALID;
    return HOS_OK;
}
bool same_shape(const hos_kv_pages* a, const hos_kv_pages* b) {
    return a->n_pages == b->n_pages && a->page_size == b->page_size && a->max_pages == b->max_pages;
}
// A table may be its own successor, but only row by row.
bool tables_agree(const hos_kv_pages* a, const hos_kv_pages* b) {
    return a->page_table != b->page_table || a->n_seq <= 1 || a->max_pages == 0 || a->table_stride == b->table_stride;
}
int check_moves(const hos_kv_moves* m) { return m && m->src && m->dst && m->count ? HOS_OK : HOS_E_INVALID; }

size_t carve(PagesView& v, bool resize, void* ws) {
    unsigned char* base = static_cast<unsigned char*>(ws);
    size_t off = 0;
    auto take = [&](size_t bytes) -> void* {
        void* p = base + off;
        off += (bytes + 255) & ~(size_t)255;
        return p;
    };
    const size_t pages = (size_t)v.n_pages * 4;
    v.growers = static_cast<int32_t*>(take(pages));
    if (!resize) return off;
    v.latest = static_cast<int32_t*>(take(pages));
    v.queue = static_cast<int32_t*>(take(pages));
    v.plan = static_cast<ResizePlan*>(take((size_t)v.n_seq * sizeof(ResizePlan)));
    return off;
}

PagesView view(const hos_kv_pages* in, const hos_kv_pages* out) {
    PagesView v = {};
    v.refs_in = in->refs;
    v.len_in = in->kv_len;
    v.table_in = in->page_table;
    v.refs = out->refs;
    v.len = out->kv_len;
    v.table = out->page_table;
    v.in_stride = in->table_stride;
    v.out_stride = out->table_stride;
    v.n_pages = in->n_pages;
    v.page_size = in->page_size;
    v.n_seq = in->n_seq;
    v.n_out = out->n_seq;
    v.max_pages = in->max_pages;
    return v;
}

size_t workspace(const hos_kv_pages* in, bool resize) {
    if (check_sizes(in)) return 0;
    PagesView v = {};
    v.n_pages = in->n_pages;
    v.n_seq = in->n_seq;
    return carve(v, resize, nullptr);
}
bool fits(size_t need, const void* ws, size_t ws_bytes) { return ws && ws_bytes >= need && (reinterpret_cast<uintptr_t>(ws) & 255) == 0; }

// Caches that pages can be copied between as they are, and the bytes of a page.
int check_layer(const hos_kv_cache* c) {
    if (!c->k || !c->v || c->n_pages < 1 || c->n_kv_heads < 1 || c->page_stride < 0 || c->scale_page_stride < 0) return HOS_E_INVALID;
    if (c->type != HOS_TYPE_BF16 && c->type != HOS_TYPE_FP16) return HOS_E_INVALID;
    if (c->format != HOS_KV_SAME && c->format != HOS_KV_E4M3 && c->format != HOS_KV_INT8) return HOS_E_INVALID;
    if (c->head_dim != 64 && c->head_dim != 128) return HOS_E_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return HOS_E_UNSUPPORTED;
    const bool coded = c->format != HOS_KV_SAME;
    const long long rows = (long long)c->n_kv_heads * c->page_size, bytes = coded ? 1 : 2;
    if (rows * c->head_dim * bytes >= (1ll << 30)) return HOS_E_UNSUPPORTED;
    if ((c->page_stride && c->page_stride < rows * c->head_dim) || (coded && c->scale_page_stride && c->scale_page_stride < rows)) return HOS_E_INVALID;
    uintptr_t bits = reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v) | (uintptr_t)(c->page_stride * bytes);
    if (coded) {
        if (!c->k_scale || !c->v_scale) return HOS_E_INVALID;
        bits |= reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale) | (uintptr_t)(c->scale_page_stride * 4);
    }
    return bits & 15 ? HOS_E_INVALID : HOS_OK;
}

}  // namespace

extern "C" {

size_t hos_kv_resize_workspace_bytes(const hos_kv_pages* in) { return workspace(in, true); }
size_t hos_kv_compact_workspace_bytes(const hos_kv_pages* in) { return workspace(in, false); }

int hos_kv_resize(const hos_kv_pages* in, const int32_t* new_len, const hos_kv_pages* out, const hos_kv_moves* moves, int32_t* status, void* ws,
                  size_t ws_bytes, void* stream) {
    int rc = check_pages(in, true);
    if (rc || (rc = check_pages(out, true))) return rc;
    if (!same_shape(in, out) || in->n_seq != out->n_seq || !tables_agree(in, out)) return HOS_E_INVALID;
    if ((in->n_seq > 0 && !new_len) || check_moves(moves)) return HOS_E_INVALID;
    PagesView v = view(in, out);
    if (!fits(carve(v, true, ws), ws, ws_bytes)) return HOS_E_WORKSPACE;
    v.change = new_len;
    v.src = moves->src;
    v.dst = moves->dst;
    v.count = moves->count;
    v.status = status;
    return cuda_rc(launch_kv_resize(v, static_cast<cudaStream_t>(stream)));
}

int hos_kv_fork(const hos_kv_pages* in, const int32_t* parent, const hos_kv_pages* out, int32_t* status, void* stream) {
    int rc = check_pages(in, true);
    if (rc || (rc = check_pages(out, true))) return rc;
    if (!same_shape(in, out) || (out->n_seq > 0 && !parent)) return HOS_E_INVALID;
    if (in->n_seq > 0 && out->n_seq > 0 && (in->kv_len == out->kv_len || (in->max_pages > 0 && in->page_table == out->page_table))) return HOS_E_INVALID;
    PagesView v = view(in, out);
    v.change = parent;
    v.status = status;
    return cuda_rc(launch_kv_fork(v, static_cast<cudaStream_t>(stream)));
}

int hos_kv_compact(const hos_kv_pages* in, const hos_kv_pages* out, const hos_kv_moves* moves, int32_t* status, void* ws, size_t ws_bytes,
                   void* stream) {
    int rc = check_pages(in, true);
    if (rc || (rc = check_pages(out, false))) return rc;
    if (!same_shape(in, out) || in->n_seq != out->n_seq || !tables_agree(in, out) || check_moves(moves)) return HOS_E_INVALID;
    PagesView v = view(in, out);
    if (!fits(carve(v, false, ws), ws, ws_bytes)) return HOS_E_WORKSPACE;
    v.src = moves->src;
    v.dst = moves->dst;
    v.count = moves->count;
    v.status = status;
    return cuda_rc(launch_kv_compact(v, static_cast<cudaStream_t>(stream)));
}

int hos_kv_copy_pages(const hos_kv_cache* to, const hos_kv_cache* from, int n_layers, const int32_t* src_page, const int32_t* dst_page,
                      const int32_t* count, int n_moves, int32_t* status, void* stream) {
    if (!to || !from || n_layers < 1 || n_moves < 0) return HOS_E_INVALID;
    for (int l = 0; l < n_layers; ++l)
        for (const hos_kv_cache* c : {to + l, from + l}) {
            const int rc = check_layer(c);
            if (rc) return rc;
            if (c->page_size != to->page_size || c->n_kv_heads != to->n_kv_heads || c->head_dim != to->head_dim || c->type != to->type ||
                c->format != to->format || to[l].n_pages != to->n_pages || from[l].n_pages != from->n_pages)
                return HOS_E_INVALID;
        }
    if (n_moves == 0) return HOS_OK;
    if (!src_page || !dst_page) return HOS_E_INVALID;
    const bool coded = to->format != HOS_KV_SAME;
    const long long rows = (long long)to->n_kv_heads * to->page_size, size = coded ? 1 : 2;
    CopyCall v;
    CopyLayer layers[COPY_LAYERS];
    v.src = src_page;
    v.dst = dst_page;
    v.count = count;
    v.status = status;
    v.n_moves = n_moves;
    v.from_pages = from->n_pages;
    v.to_pages = to->n_pages;
    v.bytes = (int)(rows * to->head_dim * size);
    v.scale_bytes = coded ? (int)(rows * 4) : 0;
    v.scale_shift = to->head_dim == 64 ? 4 : 5;
    for (int first = 0; first < n_layers; first += COPY_LAYERS) {
        v.n_layers = n_layers - first < COPY_LAYERS ? n_layers - first : COPY_LAYERS;
        for (int l = 0; l < v.n_layers; ++l) {
            const hos_kv_cache &a = from[first + l], &b = to[first + l];
            CopyLayer& w = layers[l];
            void* const as[4] = {a.k, a.v, a.k_scale, a.v_scale};
            void* const bs[4] = {b.k, b.v, b.k_scale, b.v_scale};
            for (int i = 0; i < 4; ++i) {
                w.from[i] = static_cast<const unsigned char*>(as[i]);
                w.to[i] = static_cast<unsigned char*>(bs[i]);
            }
            w.from_stride[0] = a.page_stride ? a.page_stride * size : v.bytes;
            w.to_stride[0] = b.page_stride ? b.page_stride * size : v.bytes;
            w.from_stride[1] = a.scale_page_stride ? a.scale_page_stride * 4 : v.scale_bytes;
            w.to_stride[1] = b.scale_page_stride ? b.scale_page_stride * 4 : v.scale_bytes;
        }
        const int rc = cuda_rc(launch_kv_copy_pages(v, layers, static_cast<cudaStream_t>(stream)));
        if (rc) return rc;
    }
    return HOS_OK;
}

int hos_verify_drafts(const hos_drafts* d, void* stream) {
    if (!d || d->n_seq < 0 || d->n_tokens < 0 || d->vocab < 1) return HOS_E_INVALID;
    if (d->type != HOS_TYPE_BF16 && d->type != HOS_TYPE_FP16 && d->type != HOS_TYPE_FP32) return HOS_E_INVALID;
    if (d->n_seq > MOST_SEQS || d->vocab > (1 << 30)) return HOS_E_UNSUPPORTED;
    if (d->n_seq == 0) return HOS_OK;
    if (!d->tok_off || !d->accepted || !d->next || !d->u_sample || !d->kv_len != !d->new_len) return HOS_E_INVALID;
    if (d->n_tokens > 0) {
        if (!d->tokens || !d->target || !d->u_accept || !d->out_tokens) return HOS_E_INVALID;
        if (d->target_stride < 0 || d->draft_stride < 0) return HOS_E_INVALID;
        const uintptr_t bits = reinterpret_cast<uintptr_t>(d->target) | reinterpret_cast<uintptr_t>(d->draft);
        if (bits & (d->type == HOS_TYPE_FP32 ? 3 : 1)) return HOS_E_INVALID;
    }
    return cuda_rc(launch_verify_drafts(*d, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
