// mmd_adapters.h -- launchers of the low-rank adapters' kernels (internal to libbq).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

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

// The rows that the adapters see: as they are, or (gamma not null) narrow(narrow32(h gamma) rms) with each row's rms.
struct Input {
    const uint16_t* x;
    const uint16_t* gamma;
    const float* rms;
    int M, K;
};

// How the first product is cut: `rows` rows of the call and K / chunks features to a CTA.
struct ShrinkPlan { int rows, chunks; };
ShrinkPlan shrink_plan(int M, int n_seq, int K);

// u[chunk][M][rank] = partial sums of x a^T over the chunk's features; rows without an adapter are not written.
cudaError_t launch_shrink(bool bf16, const Input& in, const Adapters& ad, const ShrinkPlan& plan, float* u, cudaStream_t stream);
// y[M][N] = narrow(y32 + scale (sum of the chunks of u) b^T); y may be y32 (ydt fp32).  ydt: 0 fp32, 1 fp16, 2 bf16.
cudaError_t launch_expand(bool bf16, int M, int N, const Adapters& ad, int chunks, const float* u, const float* y32, void* y, int ydt, cudaStream_t stream);

}  // namespace mmda
