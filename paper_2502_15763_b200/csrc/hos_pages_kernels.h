// Internal launch interface of the kernels on a cache's pages and on drafted tokens.
#pragma once

#include <atomic>

#include "hos_kernels.h"

namespace hos {

// Clusters of more than 8 blocks have to be asked for, once a kernel and device; `asked` is the kernel's own.
inline cudaError_t ask_for_large_clusters(const void* kernel, std::atomic<unsigned long long>& asked) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 64 || !(asked.load() >> dev & 1))) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess && dev < 64) asked.fetch_or(1ull << dev);
    return e;
}

// `blocks` blocks in clusters of `cluster`, early (see launch_early).
template <typename... Params, typename... Args>
cudaError_t launch_clusters(const char* name, void (*kernel)(Params...), int blocks, int cluster, int threads, cudaStream_t st, const Args&... args) {
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    launch_hook(name, 0, st);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    launch_hook(name, 1, st);
    return e;
}

// What a sequence of hos_kv_resize takes (with flags: whether it grows, whether one of the pages replaces a shared one), and what those
// before it in its block take and replace.
struct ResizePlan { int32_t takes, before, splits_before; };

// hos_kv_pages in and out, with their workspace; passed to kernels by value.
struct PagesView {
    const int32_t *refs_in, *len_in, *table_in;
    int32_t *refs, *len, *table;
    long long in_stride, out_stride;
    const int32_t* change;                 // new lengths, or parents
    int32_t *src, *dst, *count, *status;
    int n_pages, page_size, n_seq, n_out, max_pages;
    // workspace
    int32_t *growers, *latest, *queue;     // [n_pages]; queue: the free pages in order; hos_kv_compact: growers is a page's place among the moves,
                                           // and before those the masks of free pages, 32 each
    ResizePlan* plan;                      // [n_seq]
};

cudaError_t launch_kv_resize(const PagesView& p, cudaStream_t st);
cudaError_t launch_kv_fork(const PagesView& p, cudaStream_t st);
cudaError_t launch_kv_compact(const PagesView& p, cudaStream_t st);

struct CopyLayer {
    const unsigned char* from[4];          // k, v, k_scale, v_scale
    unsigned char* to[4];
    long long from_stride[2], to_stride[2];        // bytes from page to page: of k and v, of their scales
};
struct CopyCall {
    const int32_t *src, *dst, *count;
    int32_t* status;
    int n_moves, n_layers, from_pages, to_pages;
    int bytes, scale_bytes;                // of a page's k or v, of its scales (0: none)
    int scale_shift;                       // log2 of the one over the other
};
constexpr int COPY_LAYERS = 128;           // that one launch takes
cudaError_t launch_kv_copy_pages(const CopyCall& c, const CopyLayer* layers, cudaStream_t st);

cudaError_t launch_verify_drafts(const hos_drafts& d, cudaStream_t st);

}  // namespace hos
