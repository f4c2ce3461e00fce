// bqkv_tiles.cu -- instances and launches of attend_tiles.
#include "bqkv_launch.h"
#include "bqkv_tiles.cuh"

#include <mutex>

namespace bqkvl {

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_lock;

template <int D, int NB, bool SPLIT>
cudaError_t launch(long long query_rows, const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::TilesArgs& a, const bq4_codebook& cb, cudaStream_t st) {
    using Cfg = bqkvk::TilesCfg<D, NB, SPLIT>;
    static bool opted[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> guard(g_lock);
        if (!opted[dev]) {
            cudaFuncAttributes at;                                    // stage 0 starts within the first 5 KB
            e = cudaFuncGetAttributes(&at, bqkvk::attend_tiles<D, NB, SPLIT>);
            if (e != cudaSuccess) return e;
            if (at.sharedSizeBytes > 4096) return cudaErrorInvalidConfiguration;
            e = cudaFuncSetAttribute(bqkvk::attend_tiles<D, NB, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
            if (e != cudaSuccess) return e;
            opted[dev] = true;
        }
    }
    bqkvk::PairTable pairs;
    for (int i = 0; i < 16; ++i) pairs.half[i] = cb.half[i];
    const long long blocks = (query_rows + Cfg::kRowsPerCta - 1) / Cfg::kRowsPerCta;
    const dim3 grid(unsigned(c.heads), unsigned(c.n_seq), unsigned(blocks < 65535 ? blocks : 65535));
    bqkvk::attend_tiles<D, NB, SPLIT><<<grid, Cfg::kThreads, Cfg::kSmem, st>>>(c, rows, a, pairs);
    return cudaGetLastError();
}

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

template <int D, int NB>
cudaError_t both(long long query_rows, const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::TilesArgs& a, const bq4_codebook& cb, const TilesCall& t,
                 cudaStream_t st) {
    const cudaError_t e = a.bf16 ? launch<D, NB, false>(query_rows, c, rows, a, cb, st) : launch<D, NB, true>(query_rows, c, rows, a, cb, st);
    return e != cudaSuccess || !t.weights ? e : weigh<D, NB>(c, rows, a, cb, t, st);
}

}  // namespace

cudaError_t launch_tiles(long long query_rows, const bqkvk::Cache& c, const bqkvk::Rows& rows, const TilesCall& t, const bq4_codebook& cb, cudaStream_t st) {
    bqkvk::TilesArgs a = {};
    a.q = t.q; a.q_stride = t.q_stride; a.bf16 = t.bf16; a.q_heads = t.q_heads; a.group = t.q_heads / c.heads;
    a.score_scale = float((t.sm_scale < 0 ? -double(t.sm_scale) : double(t.sm_scale)) * 1.4426950408889634 / cb.unit);
    a.negate = t.sm_scale < 0;
    a.inv_unit = 1.0f / cb.unit;
    a.out = t.out; a.stats = t.stats; a.scaled = t.scaled; a.status = t.status;
    const int nb = c.dim / c.block;
    if (c.dim == 64) return nb == 1 ? both<64, 1>(query_rows, c, rows, a, cb, t, st) : both<64, 2>(query_rows, c, rows, a, cb, t, st);
    return nb == 1 ? both<128, 1>(query_rows, c, rows, a, cb, t, st)
                   : nb == 2 ? both<128, 2>(query_rows, c, rows, a, cb, t, st) : both<128, 4>(query_rows, c, rows, a, cb, t, st);
}

}  // namespace bqkvl
