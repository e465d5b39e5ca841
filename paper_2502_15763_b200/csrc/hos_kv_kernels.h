// Internal launch interface of the KV-cache kernels.
#pragma once

#include "hos_kernels.h"

namespace hos {

// A launch that may begin while the kernel before it on the stream drains (programmatic dependent launch); the kernel waits for
// that one's end (pdl_wait) before it touches memory.  Saves the gap between two kernels of a few microseconds.
template <typename... Params, typename... Args>
cudaError_t launch_early(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t st, Args&&... args) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Args&&>(args)...);
}

// KV cache and attention over it (hos_kv_cache.cu, hos_attn_rows.cu).
struct KvView;
struct AttnView;
struct RowState;
struct Partial;
// Part of an attention call's workspace: the records and pieces of one kernel's split tiles.
struct AttnWs {
    Partial* meta;
    RowState* state;
    float* part;
};
// Append and read take up to 16 heads a block, and a grid's second dimension ends at 65,535.
constexpr int KV_HEADS_A_BLOCK = 16, KV_MOST_HEADS = 65535 * KV_HEADS_A_BLOCK;
cudaError_t launch_kv_append(const KvView& c, int type, int format, const void* k, const void* v,
                             const long long (&strides)[4], cudaStream_t st);
cudaError_t launch_kv_read(const KvView& c, int type, int format, void* k, void* v, cudaStream_t st);
// Work shares of the attention kernels on an SM: the row kernel's, at most, and the rows of all their tiles; the chunk kernel's
// one share and the rows of its tile.
constexpr int ATTN_SMS = 148, ATTN_WORKERS_PER_SM = 3, ATTN_ROWS_PER_SM = 32, ATTN_CHUNK_ROWS = 256;
cudaError_t launch_attn_rows(const AttnView& a, int type, int format, int tile_rows, int max_rows, bool beside, const AttnWs& ws, int* workers,
                             cudaStream_t st);
cudaError_t launch_attn_chunk(const AttnView& a, int type, int format, int min_rows, const AttnWs& ws, cudaStream_t st);
// Joins the pieces of the chunk kernel's tiles (with `chunks`) and of the row kernel's (with row_workers > 0, tiles of tile_rows).
cudaError_t launch_attn_combine(const AttnView& a, int type, bool chunks, const AttnWs& chunk_ws, int tile_rows, int row_workers,
                                const AttnWs& row_ws, cudaStream_t st);

}  // namespace hos
