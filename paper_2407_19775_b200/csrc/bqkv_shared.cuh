// bqkv_shared.cuh -- the end of an attention whose slots were attended to in parts (the sequences' own and, in one or several parts, a
// prefix that they share): join_parts (sm_100a).
#pragma once

#include "bqkv_kernels.cuh"

namespace bqkvk {

// A warp per (row of the call, query head), D / 32 columns a lane.  With M the largest reference of the parts that saw a slot and
// f_i = 2^(m_i - M):  out = sum_i f_i sums_i / sum_i f_i l_i.  Parts are added in order, so the same call gives the same bits; those that saw
// nothing are not read.  Part 0 is of the sequence's own slots, the others of its prefix, if it has one; rows of no sequence are left alone.
// stats2 / stats4 (either may be null): reference and 1 / sum of the whole row, for the weights of the own slots.
// Bound by its bytes.
constexpr int kJoinThreads = 256, kMostParts = 32;

template <int DT, int D>
__global__ void __launch_bounds__(kJoinThreads)
join_parts(const PartRows shared, int n_own, int prefixes, int q_heads, int n_parts, const Parts parts, void* __restrict__ out, float2* __restrict__ stats2,
           float4* __restrict__ stats4) {
    constexpr int C = D / 32;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    const int lane = threadIdx.x & 31;
    const int upto = shared.starts ? min(__ldg(shared.starts + n_own), shared.n) : shared.n;
    const int p0 = shared.begin(0), p1 = shared.begin(prefixes);
    const int64_t rows = int64_t(upto) * q_heads, all = int64_t(shared.n) * q_heads;
    for (int64_t at = int64_t(blockIdx.x) * (kJoinThreads / 32) + (threadIdx.x >> 5); at < rows; at += int64_t(gridDim.x) * (kJoinThreads / 32)) {
        const int r = int(at / q_heads), n = r >= p0 && r < p1 ? n_parts : 1;
        const float2 ml = lane < n ? __ldcg(parts.softmax + int64_t(lane) * all + at) : make_float2(0.0f, 0.0f);
        const bool saw = ml.y != 0.0f;                                  // NaN too
        float top = saw ? ml.x : -INFINITY;
#pragma unroll
        for (int k = 16; k >= 1; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
        const float f = saw ? exp2f(ml.x - top) : 0.0f;
        float sum = 0.0f, o[C] = {};
        for (unsigned left = __ballot_sync(0xffffffffu, saw); left;) {  // two parts at a time: their loads together
            const int i = __ffs(left) - 1;
            left &= left - 1;
            const int j = left ? __ffs(left) - 1 : i;
            const bool two = left != 0;
            left &= left - 1;
            float x[C], y[C];
            const float* pi = parts.sums + (int64_t(i) * all + at) * D + lane * C;
            const float* pj = parts.sums + (int64_t(j) * all + at) * D + lane * C;
            if constexpr (C == 4) {
                const float4 a = __ldcg(reinterpret_cast<const float4*>(pi)), b = __ldcg(reinterpret_cast<const float4*>(pj));
                x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
                y[0] = b.x; y[1] = b.y; y[2] = b.z; y[3] = b.w;
            } else {
                const float2 a = __ldcg(reinterpret_cast<const float2*>(pi)), b = __ldcg(reinterpret_cast<const float2*>(pj));
                x[0] = a.x; x[1] = a.y;
                y[0] = b.x; y[1] = b.y;
            }
            const float fi = __shfl_sync(0xffffffffu, f, i), fj = two ? __shfl_sync(0xffffffffu, f, j) : 0.0f;
            sum = __fmaf_rn(__shfl_sync(0xffffffffu, ml.y, i), fi, sum);
            if (two) sum = __fmaf_rn(__shfl_sync(0xffffffffu, ml.y, j), fj, sum);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                o[c] = __fmaf_rn(x[c], fi, o[c]);
                if (two) o[c] = __fmaf_rn(y[c], fj, o[c]);
            }
        }
        const float inv = sum != 0.0f ? __fdiv_rn(1.0f, sum) : 0.0f;
        uint32_t w[C / 2];
#pragma unroll
        for (int c = 0; c < C; c += 2) {
            if constexpr (DT == kBF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[c / 2]) : "f"(o[c + 1] * inv), "f"(o[c] * inv));
            else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[c / 2]) : "f"(o[c + 1] * inv), "f"(o[c] * inv));
        }
        uint32_t* to = reinterpret_cast<uint32_t*>(out) + (at * D + lane * C) / 2;
        if constexpr (C == 4) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
        else *to = w[0];
        if (lane == 0) {
            const float ref = sum != 0.0f ? top : 0.0f;
            if (stats2) stats2[at] = make_float2(ref, inv);
            if (stats4) { stats4[at].x = ref; stats4[at].y = inv; }
        }
    }
}

}  // namespace bqkvk
