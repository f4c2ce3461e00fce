// bqkv_rows.cu -- instances and launches of attend_rows.
#include "bqkv_launch.h"

#include <mutex>

namespace bqkvl {

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_lock;

template <int D, int NB, int NT, bool SPLIT>
cudaError_t launch_as(int sms, const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, cudaStream_t st) {
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
            e = cudaFuncGetAttributes(&at, bqkvk::attend_rows<D, NB, NT, SPLIT>);
            if (e != cudaSuccess) return e;
            if (at.sharedSizeBytes > 6144 - 1024 - 256) return cudaErrorInvalidConfiguration;
            e = cudaFuncSetAttribute(bqkvk::attend_rows<D, NB, NT, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
            if (e != cudaSuccess) return e;
            opted[dev] = true;
        }
    }
    bqkvk::PairTable pairs;
    for (int i = 0; i < 16; ++i) pairs.half[i] = cb.half[i];
    return launch_after(bqkvk::attend_rows<D, NB, NT, SPLIT>, dim3(unsigned(sms)), Cfg::kWarps * 32, Cfg::kSmem, st, c, rows, a, pairs);
}

// fp16 outputs keep 11 bits, as many as a probability in one part has: they take two, 22 bits.  bf16 outputs keep 8.
template <int D, int NB, int NT>
cudaError_t launch(int sms, const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, cudaStream_t st) {
    return a.bf16 ? launch_as<D, NB, NT, false>(sms, c, rows, a, cb, st) : launch_as<D, NB, NT, true>(sms, c, rows, a, cb, st);
}

template <int NT>
cudaError_t launch_nt(int sms, const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, cudaStream_t st) {
    const int nb = c.dim / c.block;
    if (c.dim == 64) return nb == 1 ? launch<64, 1, NT>(sms, c, rows, a, cb, st) : launch<64, 2, NT>(sms, c, rows, a, cb, st);
    return nb == 1 ? launch<128, 1, NT>(sms, c, rows, a, cb, st)
                   : nb == 2 ? launch<128, 2, NT>(sms, c, rows, a, cb, st) : launch<128, 4, NT>(sms, c, rows, a, cb, st);
}

}  // namespace

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
    return query_rows <= 8 ? launch_nt<1>(sms, c, rows, a, cb, st) : launch_nt<2>(sms, c, rows, a, cb, st);
}

cudaError_t launch_weights(const bqkvk::Cache& c, const bqkvk::Rows& rows, const bqkvk::RowsArgs& a, const bq4_codebook& cb, float sm_log2, int max_len,
                           float* weights, int64_t weights_stride, cudaStream_t st) {
    constexpr int per_cta = bqkvk::kWeightThreads * bqkvk::kWeightSlots;
    const dim3 grid(unsigned((max_len + per_cta - 1) / per_cta), unsigned(c.heads), unsigned(c.n_seq));
    return launch_after(a.bf16 ? bqkvk::attend_rows_weights<bq4k::kBF16> : bqkvk::attend_rows_weights<bq4k::kF16>, grid, bqkvk::kWeightThreads, 0, st, c, rows, a, sm_log2, weights,
                        weights_stride, cb.tab);
}

}  // namespace bqkvl
