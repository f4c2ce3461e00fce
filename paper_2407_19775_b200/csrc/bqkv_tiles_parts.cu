// bqkv_tiles_parts.cu -- instances of attend_tiles for calls whose slots are attended to in parts.
#include "bqkv_tiles_launch.cuh"

namespace bqkvl {

cudaError_t launch_tiles_parts(long long query_rows, const bqkvk::Cache& c, const bqkvk::PartRows& rows, const TilesCall& t, const bq4_codebook& cb, cudaStream_t st) {
    return launch_any<true>(query_rows, c, rows, t, cb, st);
}

}  // namespace bqkvl
