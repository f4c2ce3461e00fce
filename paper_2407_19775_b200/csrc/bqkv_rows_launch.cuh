// bqkv_rows_launch.cuh -- the launch of attend_rows, for the units that hold its instances (internal to libbq).
#pragma once

#include "bqkv_launch.h"

#include <mutex>

namespace bqkvl {

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_lock;

template <int D, int NB, int NT, bool SPLIT, bool PARTS, typename R>
cudaError_t launch_as(int sms, const bqkvk::Cache& c, const R& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, cudaStream_t st) {
    using Cfg = bqkvk::RowsCfg<D, NB, NT>;
    static bool opted[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> guard(g_lock);
        if (!opted[dev]) {
            cudaFuncAttributes at;                                    // the rings below the table start within the first 6 KB
            e = cudaFuncGetAttributes(&at, bqkvk::attend_rows<D, NB, NT, SPLIT, PARTS>);
            if (e != cudaSuccess) return e;
            if (at.sharedSizeBytes > 6144 - 1024 - 256) return cudaErrorInvalidConfiguration;
            e = cudaFuncSetAttribute(bqkvk::attend_rows<D, NB, NT, SPLIT, PARTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
            if (e != cudaSuccess) return e;
            opted[dev] = true;
        }
    }
    bqkvk::PairTable pairs;
    for (int i = 0; i < 16; ++i) pairs.half[i] = cb.half[i];
    return launch_after(bqkvk::attend_rows<D, NB, NT, SPLIT, PARTS>, dim3(unsigned(sms)), Cfg::kWarps * 32, Cfg::kSmem, st, c, rows, a, pairs);
}

// fp16 outputs keep 11 bits, as many as a probability in one part has: they take two, 22 bits.  bf16 outputs keep 8.
template <int D, int NB, int NT, bool PARTS, typename R>
cudaError_t launch(int sms, const bqkvk::Cache& c, const R& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, cudaStream_t st) {
    return a.bf16 ? launch_as<D, NB, NT, false, PARTS>(sms, c, rows, a, cb, st) : launch_as<D, NB, NT, true, PARTS>(sms, c, rows, a, cb, st);
}

template <int NT, bool PARTS, typename R>
cudaError_t launch_nt(int sms, const bqkvk::Cache& c, const R& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, cudaStream_t st) {
    const int nb = c.dim / c.block;
    if (c.dim == 64) return nb == 1 ? launch<64, 1, NT, PARTS>(sms, c, rows, a, cb, st) : launch<64, 2, NT, PARTS>(sms, c, rows, a, cb, st);
    return nb == 1 ? launch<128, 1, NT, PARTS>(sms, c, rows, a, cb, st)
                   : nb == 2 ? launch<128, 2, NT, PARTS>(sms, c, rows, a, cb, st) : launch<128, 4, NT, PARTS>(sms, c, rows, a, cb, st);
}

}  // namespace

}  // namespace bqkvl
