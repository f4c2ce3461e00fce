// bqkv_checks.h -- what the C ABI units of the 4-bit cache share: argument checks and the cache as the kernels see it (internal
// to libbq).
#pragma once

#include "../../include/bq4.h"
#include "bq_error.h"
#include "bqkv_kernels.cuh"

namespace bqkvc {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool is16(int dt) { return dt == BQ_F16 || dt == BQ_BF16; }
inline int log2_exact(int v) {
    int l = 0;
    while ((1 << l) < v) ++l;
    return ((1 << l) == v) ? l : -1;
}
inline int cuda_fail(cudaError_t e) {
    bql::set_last_cuda_error(cudaGetErrorString(e));
    return BQ_ERR_CUDA;
}

// The sizes of the cache description, without its pointers.
inline int check_sizes(const bqkv_cache* c) {
    if (!c) return BQ_ERR_NULL;
    if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 != 0) return BQ_ERR_SIZE;
    if (c->block < 8 || c->block % 8 != 0 || c->head_dim % c->block != 0) return BQ_ERR_BLOCK;
    if (c->kv_heads < 1 || c->kv_heads > 1024 || c->page < 1 || c->page > 65536 || c->n_pages < 1) return BQ_ERR_SIZE;
    if (int64_t(c->n_pages) * c->kv_heads >= (int64_t(1) << 31)) return BQ_ERR_SIZE;
    if (c->n_seq < 1 || c->n_seq > 65535 || c->max_pages < 1 || c->table_stride < c->max_pages) return BQ_ERR_SIZE;
    if (int64_t(c->max_pages) * c->page >= (int64_t(1) << 30)) return BQ_ERR_SIZE;
    return BQ_OK;
}

inline int check_cache(const bqkv_cache* c) {
    const int rc = check_sizes(c);
    if (rc != BQ_OK) return rc;
    if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->table || !c->lens) return BQ_ERR_NULL;
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16)) return BQ_ERR_SIZE;
    return BQ_OK;
}

inline int check_rows(const bqkv_cache* c, const int32_t* starts, int n_rows) {
    if (n_rows < 0 || n_rows > (1 << 27)) return BQ_ERR_SIZE;
    if (!starts && n_rows != c->n_seq) return BQ_ERR_SIZE;
    return BQ_OK;
}

inline bqkvk::Cache device_view(const bqkv_cache* c) {
    bqkvk::Cache d;
    d.k_codes = c->k_codes; d.v_codes = c->v_codes; d.k_scale = c->k_scale; d.v_scale = c->v_scale;
    d.table = c->table; d.lens = c->lens;
    d.n_pages = c->n_pages; d.heads = c->kv_heads; d.page = c->page; d.dim = c->head_dim; d.block = c->block;
    d.n_seq = c->n_seq; d.max_pages = c->max_pages; d.table_stride = c->table_stride;
    d.page_shift = log2_exact(c->page);
    d.chunk_shift = log2_exact(c->head_dim / 8);
    d.block_shift = log2_exact(c->block / 8);
    return d;
}

}  // namespace bqkvc
