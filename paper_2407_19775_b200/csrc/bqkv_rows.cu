// bqkv_rows.cu -- instances and launches of attend_rows.
#include "bqkv_rows_launch.cuh"

namespace bqkvl {

bool rows_shape(int dim, int block, int page) {
    if (page % 16 != 0) return false;
    return (dim == 64 && (block == 64 || block == 32)) || (dim == 128 && (block == 128 || block == 64 || block == 32));
}
size_t rows_partial_floats(int dim, int query_rows, int sms) {
    const size_t r = query_rows <= 8 ? 8 : 16;
    const int warps = query_rows > 8 ? bqkvk::RowsCfg<64, 1, 2>::kWarps : dim == 64 ? bqkvk::RowsCfg<64, 1, 1>::kWarps : bqkvk::RowsCfg<128, 1, 1>::kWarps;
    return size_t(sms) * (2 + warps) * (r * size_t(dim) + 2 * r);
}

cudaError_t launch_rows(int query_rows, int sms, const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, cudaStream_t st) {
    return query_rows <= 8 ? launch_nt<1, false>(sms, c, rows, a, cb, st) : launch_nt<2, false>(sms, c, rows, a, cb, st);
}

cudaError_t launch_weights(const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, float sm_log2, int max_len,
                           float* weights, int64_t weights_stride, cudaStream_t st) {
    constexpr int per_cta = bqkvk::kWeightThreads * bqkvk::kWeightSlots;
    const dim3 grid(unsigned((max_len + per_cta - 1) / per_cta), unsigned(c.heads), unsigned(c.n_seq));
    return launch_after(a.bf16 ? bqkvk::attend_rows_weights<bq4k::kBF16> : bqkvk::attend_rows_weights<bq4k::kF16>, grid, bqkvk::kWeightThreads, 0, st, c, rows, a, sm_log2, weights,
                        weights_stride, cb.tab);
}

}  // namespace bqkvl
