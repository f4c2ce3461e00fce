// mmd_adapters.h -- launchers of the low-rank adapters' kernels (internal to libbq).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

struct mmd_weights;
namespace mmdk { struct AdaptArgs; }

namespace mmda {

// Who has which adapter, and the adapters themselves (the fields of mmd_adapters, checked by the host).
struct Adapters {
    const uint16_t* a;                     // [count][rank][K]
    const uint16_t* b;                     // [count][N][rank]
    const float* scale;                    // [count]
    int count, rank;
    const int32_t* ids;                    // of the sequences
    const int32_t* starts;                 // n_seq + 1, or null: one row per sequence
    int n_seq;
};

// The rows that the adapters see: as they are, or (gamma not null) h gamma rms, rounded to fp32 twice, with each row's rms.
struct Input {
    const uint16_t* x;
    const uint16_t* gamma;
    const float* rms;
    int M, K, N;
};

// How the first product is cut: `rows` rows of the call and K / chunks features to a CTA.
struct ShrinkPlan { int rows, chunks; };
ShrinkPlan shrink_plan(int M, int n_seq, int K, int rank);

// u[chunk][M][rank] = partial sums of x a^T over the chunk's features; rows without an adapter are not written.  row_id[M]: the rows'
// adapters, -1: none.
cudaError_t launch_shrink(bool bf16, const Input& in, const Adapters& ad, const ShrinkPlan& plan, float* u, int32_t* row_id, cudaStream_t stream);

// y[M][N] = narrow(y32 + scale (sum of the chunks of u) b^T), rows of y32 `ld` apart; y may be y32 (fp32 outputs, ld == N).
cudaError_t launch_expand(bool bf16, int M, int N, const Adapters& ad, const ShrinkPlan& plan, const float* u, const int32_t* row_id, const float* y32, int ld, void* y,
                          bool f32out, cudaStream_t stream);

// the CTA-pair product with the adapters' part added in its epilogue
cudaError_t launch_fused(const mmd_weights* w, const int8_t* qx, const float* sx, const void* sidex, void* y, int M, bool f32out, const mmdk::AdaptArgs& ad,
                         cudaStream_t stream);

}  // namespace mmda
