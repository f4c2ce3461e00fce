// bqkv_rows_parts.cu -- instances of attend_rows for calls whose slots are attended to in parts.
#include "bqkv_rows_launch.cuh"

namespace bqkvl {

cudaError_t launch_rows_part(int query_rows, int sms, const bqkvk::Cache& c, const bqkvk::PartRows& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, cudaStream_t st) {
    return query_rows <= 8 ? launch_nt<1, true>(sms, c, rows, a, cb, st) : launch_nt<2, true>(sms, c, rows, a, cb, st);
}

}  // namespace bqkvl
