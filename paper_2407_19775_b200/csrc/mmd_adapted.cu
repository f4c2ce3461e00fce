// mmd_adapted.cu -- instances of gemm_tc2 whose epilogue adds low-rank adapters.
#include "mmd_adapters.h"
#include "mmd_launch.cuh"

namespace mmda {

cudaError_t launch_fused(const mmd_weights* w, const int8_t* qx, const float* sx, const void* sidex, void* y, int M, bool f32out, const mmdk::AdaptArgs& ad,
                         cudaStream_t stream) {
    CUtensorMap mqx;
    if (!make_map_kblocks(&mqx, qx, uint64_t(M), uint64_t(w->K), 128, mmdk::kPairStepBlocks)) return cudaErrorNotSupported;
    if (w->dtype == BQ_BF16)
        return f32out ? launch_tc2<mmdk::kBF16, mmdk::kF32, true>(w, mqx, sx, sidex, y, M, ad, stream) : launch_tc2<mmdk::kBF16, mmdk::kBF16, true>(w, mqx, sx, sidex, y, M, ad, stream);
    return f32out ? launch_tc2<mmdk::kF16, mmdk::kF32, true>(w, mqx, sx, sidex, y, M, ad, stream) : launch_tc2<mmdk::kF16, mmdk::kF16, true>(w, mqx, sx, sidex, y, M, ad, stream);
}

}  // namespace mmda
