// bqkv_tiles_launch.cuh -- the launch of attend_tiles, for the units that hold its instances (internal to libbq).
#pragma once

#include "bqkv_launch.h"
#include "bqkv_tiles.cuh"

#include <mutex>

namespace bqkvl {

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_lock;

template <int D, int NB, bool SPLIT, bool PARTS, typename R>
cudaError_t launch(long long query_rows, const bqkvk::Cache& c, const R& rows, const bqkvk::TilesArgs& a, const bq4_codebook& cb, cudaStream_t st) {
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
            e = cudaFuncGetAttributes(&at, bqkvk::attend_tiles<D, NB, SPLIT, PARTS>);
            if (e != cudaSuccess) return e;
            if (at.sharedSizeBytes > 4096) return cudaErrorInvalidConfiguration;
            e = cudaFuncSetAttribute(bqkvk::attend_tiles<D, NB, SPLIT, PARTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
            if (e != cudaSuccess) return e;
            opted[dev] = true;
        }
    }
    bqkvk::PairTable pairs;
    for (int i = 0; i < 16; ++i) pairs.half[i] = cb.half[i];
    const long long blocks = (query_rows + Cfg::kRowsPerCta - 1) / Cfg::kRowsPerCta;
    const long long most = 65535 / a.splits;
    const dim3 grid(unsigned(c.heads), unsigned(c.n_seq), unsigned((blocks < most ? blocks : most) * a.splits));
    if constexpr (PARTS) return launch_after(bqkvk::attend_tiles<D, NB, SPLIT, PARTS>, grid, Cfg::kThreads, Cfg::kSmem, st, c, rows, a, pairs);
    bqkvk::attend_tiles<D, NB, SPLIT, PARTS><<<grid, Cfg::kThreads, Cfg::kSmem, st>>>(c, rows, a, pairs);
    return cudaGetLastError();
}

bqkvk::TilesArgs args_of(const bqkvk::Cache& c, const TilesCall& t, const bq4_codebook& cb) {
    bqkvk::TilesArgs a = {};
    a.q = t.q; a.q_stride = t.q_stride; a.bf16 = t.bf16; a.q_heads = t.q_heads; a.group = t.q_heads / c.heads;
    a.score_scale = float((t.sm_scale < 0 ? -double(t.sm_scale) : double(t.sm_scale)) * 1.4426950408889634 / cb.unit);
    a.negate = t.sm_scale < 0;
    a.inv_unit = 1.0f / cb.unit;
    a.out = t.out; a.stats = t.stats; a.scaled = t.scaled; a.status = t.status;
    a.parts = t.parts; a.splits = t.splits; a.part_rows = t.part_rows;
    return a;
}

template <int D, int NB, bool PARTS, typename R>
cudaError_t launch_as(long long query_rows, const bqkvk::Cache& c, const R& rows, const bqkvk::TilesArgs& a, const bq4_codebook& cb, cudaStream_t st) {
    return a.bf16 ? launch<D, NB, false, PARTS>(query_rows, c, rows, a, cb, st) : launch<D, NB, true, PARTS>(query_rows, c, rows, a, cb, st);
}

template <bool PARTS, typename R>
cudaError_t launch_any(long long query_rows, const bqkvk::Cache& c, const R& rows, const TilesCall& t, const bq4_codebook& cb, cudaStream_t st) {
    const bqkvk::TilesArgs a = args_of(c, t, cb);
    const int nb = c.dim / c.block;
    if (c.dim == 64) return nb == 1 ? launch_as<64, 1, PARTS>(query_rows, c, rows, a, cb, st) : launch_as<64, 2, PARTS>(query_rows, c, rows, a, cb, st);
    return nb == 1 ? launch_as<128, 1, PARTS>(query_rows, c, rows, a, cb, st)
                   : nb == 2 ? launch_as<128, 2, PARTS>(query_rows, c, rows, a, cb, st) : launch_as<128, 4, PARTS>(query_rows, c, rows, a, cb, st);
}

}  // namespace

}  // namespace bqkvl
