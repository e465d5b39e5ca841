// Internal launch interface of the kernels on a cache's pages and on drafted tokens.
#pragma once

#include "hos_kernels.h"

namespace hos {

// What a sequence of hos_kv_resize goes through, worked out once.  `takes` counts the pages taken before it by the
// sequences of the same block, `splits` the pages among them that replace shared ones; the two top bits of splits say
// whether it grows and whether it is one of those itself.
struct ResizePlan {
    int32_t have, need;
    unsigned long long before;
};

// hos_kv_pages in and out, with their workspace; passed to kernels by value.
struct PagesView {
    const int32_t *refs_in, *len_in, *table_in;
    int32_t *refs, *len, *table;
    long long in_stride, out_stride;
    const int32_t* change;                 // new lengths, or parents
    int32_t *src, *dst, *count, *status;
    int n_pages, page_size, n_seq, n_out, max_pages;
    // workspace
    int32_t *growers, *latest, *queue;     // [n_pages]; queue: the free pages in order; hos_kv_compact: growers is a page's place among the moves
    ResizePlan* plan;                      // [n_seq]
    int32_t* children;                     // [n_seq]
};

cudaError_t launch_kv_resize(const PagesView& p, cudaStream_t st);
cudaError_t launch_kv_fork(const PagesView& p, cudaStream_t st);
cudaError_t launch_kv_compact(const PagesView& p, cudaStream_t st);

// Layers of a hos_kv_copy_pages call that one launch takes; kernel parameters may have 32,764 bytes.
constexpr int COPY_LAYERS = 128;
struct CopyLayer {
    const unsigned char* from[4];          // k, v, k_scale, v_scale
    unsigned char* to[4];
    long long from_stride[2], to_stride[2];        // bytes from page to page: of k and v, of their scales
};
struct CopyView {
    const int32_t *src, *dst, *count;
    int32_t* status;
    int n_moves, n_layers, from_pages, to_pages;
    int bytes, scale_bytes;                // of a page's k or v, of its scales (0: none)
    CopyLayer layer[COPY_LAYERS];
};
cudaError_t launch_kv_copy_pages(const CopyView& c, cudaStream_t st);

cudaError_t launch_verify_drafts(const hos_drafts& d, cudaStream_t st);

}  // namespace hos
