// bqkv_launch.h -- launchers of the 4-bit cache's attention kernels, one translation unit per kernel
// family (internal to libbq).
#pragma once

#include <cuda_runtime.h>

#include "bq4_codebook.h"
#include "bqkv_rows.cuh"

namespace bqkvl {

// A launch with programmatic stream serialization: the kernel may become resident while the one before it ends, and waits
// (griddepcontrol.wait) for it before it touches global memory.  Behind a kernel that does not signal its dependents this is an
// ordinary launch.
template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(unsigned(threads), 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// Whether attend_rows is built for the cache's rows: head size, blocks per row, and pages of whole groups of 16 rows.
bool rows_shape(int dim, int block, int page);
size_t rows_partial_floats(int dim, int query_rows, int sms);    // partial results of its CTAs (one per SM) and their warps
cudaError_t launch_rows(int query_rows, int sms, const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, cudaStream_t stream);

// weights from softmax statistics and, where they were kept, scores
cudaError_t launch_weights(const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, float sm_log2, int max_len,
                           float* weights, int64_t weights_stride, cudaStream_t stream);

struct TilesCall {
    const void* q;
    int64_t q_stride;
    int bf16, q_heads;
    float sm_scale;
    void* out;
    float* weights;                        // null: none wanted, nor the three below
    int64_t weights_stride;
    int max_len;
    float4* stats;
    uint32_t* scaled;
    int* status;
};
cudaError_t launch_tiles(long long query_rows, const bqkvk::Cache& c, const bqkvk::Rows& rows, const TilesCall& t, const bq4_codebook& cb, cudaStream_t stream);

cudaError_t launch_evict(const bqkvk::Cache& c, float* weights, int64_t stride, int budget, int sinks, int recent, void* workspace, cudaStream_t stream);

}  // namespace bqkvl
