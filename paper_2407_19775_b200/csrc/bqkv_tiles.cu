// bqkv_tiles.cu -- instances and launches of attend_tiles and weights_tiles.
#include "bqkv_tiles_launch.cuh"

namespace bqkvl {

namespace {

template <int D, int NB>
cudaError_t weigh(const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::TilesArgs& a, const bq4_codebook& cb, const TilesCall& t, cudaStream_t st) {
    using Cfg = bqkvk::WeightsCfg<D, NB>;
    static bool opted[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> guard(g_lock);
        if (!opted[dev]) {
            e = cudaFuncSetAttribute(bqkvk::weights_tiles<D, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
            if (e != cudaSuccess) return e;
            opted[dev] = true;
        }
    }
    bqkvk::PairTable pairs;
    for (int i = 0; i < 16; ++i) pairs.half[i] = cb.half[i];
    const dim3 grid(unsigned((t.max_len + Cfg::kSlots - 1) / Cfg::kSlots), unsigned(c.heads), unsigned(c.n_seq));
    bqkvk::weights_tiles<D, NB><<<grid, Cfg::kThreads, Cfg::kSmem, st>>>(c, rows, a, t.weights, t.weights_stride, pairs);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_tiles(long long query_rows, const bqkvk::Cache& c, const bqkvk::Rows& rows, const TilesCall& t, const bq4_codebook& cb, cudaStream_t st) {
    return launch_any<false>(query_rows, c, rows, t, cb, st);
}

cudaError_t launch_tiles_weights(const bqkvk::Cache& c, const bqkvk::Rows& rows, const TilesCall& t, const bq4_codebook& cb, cudaStream_t st) {
    const bqkvk::TilesArgs a = args_of(c, t, cb);
    const int nb = c.dim / c.block;
    if (c.dim == 64) return nb == 1 ? weigh<64, 1>(c, rows, a, cb, t, st) : weigh<64, 2>(c, rows, a, cb, t, st);
    return nb == 1 ? weigh<128, 1>(c, rows, a, cb, t, st) : nb == 2 ? weigh<128, 2>(c, rows, a, cb, t, st) : weigh<128, 4>(c, rows, a, cb, t, st);
}

}  // namespace bqkvl
