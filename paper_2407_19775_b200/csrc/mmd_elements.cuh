// mmd_elements.cuh -- 16-bit elements as the kernels of the decomposed layers read and write them (sm_100a).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace mmdk {

enum { kF32 = 0, kF16 = 1, kBF16 = 2 };

template <int DT>
__device__ __forceinline__ float widen16(uint32_t bits16) {
    if constexpr (DT == kBF16) return __uint_as_float(bits16 << 16);
    else return __half2float(__ushort_as_half(static_cast<unsigned short>(bits16)));
}

template <int DT>
__device__ __forceinline__ void widen8(const uint4& w, float (&f)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = widen16<DT>(u[i] & 0xffffu);
        f[2 * i + 1] = widen16<DT>(u[i] >> 16);
    }
}

// a result narrowed to its type
template <int YDT>
__device__ __forceinline__ void store_y(void* y, size_t i, float v) {
    if constexpr (YDT == kF32) static_cast<float*>(y)[i] = v;
    else if constexpr (YDT == kBF16) static_cast<__nv_bfloat16*>(y)[i] = __float2bfloat16_rn(v);
    else static_cast<__half*>(y)[i] = __float2half_rn(v);
}

}  // namespace mmdk
