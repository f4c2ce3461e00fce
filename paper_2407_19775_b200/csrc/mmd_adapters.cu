// mmd_adapters.cu -- low-rank adapters of many sequences beside a shared decomposed projection (sm_100a):
//
//     y_r = (the decomposed layer's row, in fp32) + scale_a (x_r A_a^T) B_a^T,   a the adapter of row r's sequence
//
// in two kernels around the layer's product: `shrink` (u = x A^T, few numbers per row) and `expand`.  A decode step reads every
// adapter in use once (rank (K + N) 16-bit numbers each, 0.5 MB at rank 16 and 8192 features), which bounds it; for prompts the
// rows' own bytes do.
#include "mmd_adapters.h"

#include "bqkv_launch.h"
#include "mmd_elements.cuh"

namespace mmda {

namespace {

using mmdk::kBF16;
using mmdk::kF16;
using mmdk::kF32;

// The adapter of row r, found by the whole warp; -1: none.
__device__ __forceinline__ int adapter_of(const Adapters& ad, int r, int M) {
    int s = r;
    if (ad.starts) {
        s = bqkvk::last_begun(r, ad.n_seq, [&](int i) { return __ldg(ad.starts + i); });
        if (r >= __ldg(ad.starts + s + 1) || r < __ldg(ad.starts + s)) return -1;
    }
    const int id = __ldg(ad.ids + s);
    return id >= 0 && id < ad.count ? id : -1;
}

template <int DT>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (DT == kBF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight elements of the normed row.
template <int DT>
__device__ __forceinline__ uint4 normed(uint4 h, uint4 g, float rms) {
    float f[8], w[8];
    mmdk::widen8<DT>(h, f);
    mmdk::widen8<DT>(g, w);
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __fmul_rn(__fmul_rn(f[2 * i], w[2 * i]), rms), hi = __fmul_rn(__fmul_rn(f[2 * i + 1], w[2 * i + 1]), rms);
        if constexpr (DT == kBF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y[i]) : "f"(hi), "f"(lo));
        else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y[i]) : "f"(hi), "f"(lo));
    }
    return make_uint4(y[0], y[1], y[2], y[3]);
}

// ------------------------------------------------------------------------------------------
// shrink: u^T = A x^T by mma.sync m16n8k16: 16 ranks are the 16 rows, up to 8 rows of the call the 8 columns (tcgen05 has no shape this
// small, and the products are not what bounds it).  The order of k within a product does not matter as long as both operands have
// the same, so a lane takes eight consecutive features, 16 bytes, of its adapter row and of its activation row.
// A CTA has `rows` rows of the call and a chunk of the features; its warps share the chunk's steps of 32 and are added in order.
constexpr int kShrinkThreads = 256, kShrinkWarps = kShrinkThreads / 32;

template <int DT, int NT /* times 8 rows */, bool NORM>
__global__ void __launch_bounds__(kShrinkThreads)
shrink(const Input in, const Adapters ad, int rows, float* __restrict__ u) {
    __shared__ int id_of[8 * NT];
    __shared__ float red[kShrinkWarps][NT][4][32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int r0 = int(blockIdx.x) * rows, nr = min(rows, in.M - r0);
    for (int i = wid; i < 8 * NT; i += kShrinkWarps) {
        const int id = i < nr ? adapter_of(ad, r0 + i, in.M) : -1;
        if (lane == 0) id_of[i] = id;
    }
    __syncthreads();
    const int steps = (in.K + 31) / 32, s0 = int((long long)steps * blockIdx.y / gridDim.y), s1 = int((long long)steps * (blockIdx.y + 1) / gridDim.y);
    const int w0 = s0 + (s1 - s0) * wid / kShrinkWarps, w1 = s0 + (s1 - s0) * (wid + 1) / kShrinkWarps;
    float* const to = u + size_t(blockIdx.y) * in.M * ad.rank;
    for (int first = 0; first < nr; ++first) {
        const int id = id_of[first];
        bool fresh = id >= 0;
        for (int i = 0; i < first; ++i) fresh &= id_of[i] != id;        // the adapters of the block, each once
        if (!fresh) continue;
        const uint16_t* x[NT];
        float rms[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const bool mine = id_of[8 * n + g] == id;
            x[n] = mine ? in.x + size_t(r0 + 8 * n + g) * in.K + 8 * t : nullptr;
            rms[n] = NORM && mine ? __ldg(in.rms + r0 + 8 * n + g) : 0.0f;
        }
        for (int j0 = 0; j0 < ad.rank; j0 += 16) {
            const uint16_t* a0 = ad.a + (size_t(id) * ad.rank + j0 + g) * in.K + 8 * t;
            const uint16_t* a1 = a0 + size_t(8) * in.K;
            float acc[NT][4] = {};
#pragma unroll 4
            for (int s = w0; s < w1; ++s) {
                const int k = 32 * s;
                const bool there = k + 8 * t < in.K;                    // K is a multiple of 16
                const uint4 zero = make_uint4(0, 0, 0, 0);
                const uint4 p = there ? __ldg(reinterpret_cast<const uint4*>(a0 + k)) : zero, q = there ? __ldg(reinterpret_cast<const uint4*>(a1 + k)) : zero;
                uint4 gm = zero;
                if (NORM && there) gm = __ldg(reinterpret_cast<const uint4*>(in.gamma + k + 8 * t));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint4 v = there && x[n] ? __ldg(reinterpret_cast<const uint4*>(x[n] + k)) : zero;
                    if constexpr (NORM) v = normed<DT>(v, gm, rms[n]);
                    mma16<DT>(acc[n], p.x, q.x, p.y, q.y, v.x, v.y);
                    mma16<DT>(acc[n], p.z, q.z, p.w, q.w, v.z, v.w);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) red[wid][n][c][lane] = acc[n][c];
            __syncthreads();
            // fragment element c of lane l: rank (l >> 2) + 8 (c >> 1), row 2 (l & 3) + (c & 1)
            for (int i = threadIdx.x; i < 8 * NT * 16; i += kShrinkThreads) {
                const int j = i & 15, row = i >> 4, n = row >> 3, l = (j & 7) * 4 + ((row & 7) >> 1), c = (j >> 3) * 2 + (row & 1);
                if (id_of[row] != id) continue;
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < kShrinkWarps; ++w) sum += red[w][n][c][l];
                to[size_t(r0 + row) * ad.rank + j0 + j] = sum;
            }
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------------------------------------
// expand: a thread has two columns of kExpandRows rows; fp32 throughout, one rounding at the end.  Bound by its bytes: the adapters' b for
// single rows, y32 and y for many.
constexpr int kExpandThreads = 256;

template <int DT, int YDT, int ROWS>
__global__ void __launch_bounds__(kExpandThreads)
expand(const Adapters ad, int M, int N, int chunks, const float* __restrict__ u, const float* y32, void* y) {
    __shared__ int id_of[ROWS];
    extern __shared__ __align__(16) float v[];                          // [ROWS][rank]
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int r0 = int(blockIdx.x) * ROWS, nr = min(ROWS, M - r0);
    for (int i = wid; i < ROWS; i += kExpandThreads / 32) {
        const int id = i < nr ? adapter_of(ad, r0 + i, M) : -1;
        if (lane == 0) id_of[i] = id;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < nr * ad.rank; i += kExpandThreads) {
        const int id = id_of[i / ad.rank];
        float sum = 0.0f;
        if (id >= 0) {
            for (int c = 0; c < chunks; ++c) sum += u[(size_t(c) * M + r0) * ad.rank + i];
            sum *= __ldg(ad.scale + id);
        }
        v[i] = sum;
    }
    __syncthreads();
    const int n = (int(blockIdx.y) * kExpandThreads + int(threadIdx.x)) * 2;
    if (n >= N) return;
    const bool two = n + 1 < N;
    float acc[ROWS][2];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const size_t at = size_t(r0 + i) * N + n;
        acc[i][0] = i < nr ? y32[at] : 0.0f;
        acc[i][1] = i < nr && two ? y32[at + 1] : 0.0f;
    }
    for (int first = 0; first < nr; ++first) {
        const int id = id_of[first];
        bool fresh = id >= 0;
        for (int i = 0; i < first; ++i) fresh &= id_of[i] != id;
        if (!fresh) continue;
        const uint16_t* b = ad.b + (size_t(id) * N + n) * ad.rank;
        for (int j = 0; j < ad.rank; j += 8) {
            float p[8], q[8];
            mmdk::widen8<DT>(__ldg(reinterpret_cast<const uint4*>(b + j)), p);
            mmdk::widen8<DT>(two ? __ldg(reinterpret_cast<const uint4*>(b + ad.rank + j)) : make_uint4(0, 0, 0, 0), q);
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                if (id_of[i] != id) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float w = v[i * ad.rank + j + e];
                    acc[i][0] = __fmaf_rn(w, p[e], acc[i][0]);
                    acc[i][1] = __fmaf_rn(w, q[e], acc[i][1]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (i >= nr) continue;
        const size_t at = size_t(r0 + i) * N + n;
        mmdk::store_y<YDT>(y, at, acc[i][0]);
        if (two) mmdk::store_y<YDT>(y, at + 1, acc[i][1]);
    }
}

template <int DT, int YDT>
cudaError_t expand_as(int M, int N, const Adapters& ad, int chunks, const float* u, const float* y32, void* y, cudaStream_t st) {
    const unsigned cols = unsigned((N + 2 * kExpandThreads - 1) / (2 * kExpandThreads));
    if (M <= 256) return bqkvl::launch_after(expand<DT, YDT, 1>, dim3(unsigned(M), cols), kExpandThreads, size_t(ad.rank) * 4, st, ad, M, N, chunks, u, y32, y);
    return bqkvl::launch_after(expand<DT, YDT, 8>, dim3(unsigned((M + 7) / 8), cols), kExpandThreads, size_t(8 * ad.rank) * 4, st, ad, M, N, chunks, u, y32, y);
}

template <int DT, int NT>
cudaError_t shrink_as(const Input& in, const Adapters& ad, const ShrinkPlan& plan, float* u, cudaStream_t st) {
    const dim3 grid(unsigned((in.M + plan.rows - 1) / plan.rows), unsigned(plan.chunks));
    return bqkvl::launch_after(in.gamma ? shrink<DT, NT, true> : shrink<DT, NT, false>, grid, kShrinkThreads, 0, st, in, ad, plan.rows, u);
}

}  // namespace

// Single rows, each with an adapter of its own, go to a CTA each; prompts by 32 rows.  Features are cut until there are two CTAs for every
// SM, in chunks of 512 at least.
ShrinkPlan shrink_plan(int M, int n_seq, int K) {
    ShrinkPlan p;
    p.rows = M <= 256 && n_seq * 2 > M ? 1 : M <= 1024 ? 8 : 32;
    const int blocks = (M + p.rows - 1) / p.rows, most = K / 512 < 1 ? 1 : K / 512;
    p.chunks = blocks > 0 ? 2 * 148 / blocks : 1;
    if (p.chunks > 16) p.chunks = 16;
    if (p.chunks > most) p.chunks = most;
    if (p.chunks < 1) p.chunks = 1;
    return p;
}

cudaError_t launch_shrink(bool bf16, const Input& in, const Adapters& ad, const ShrinkPlan& plan, float* u, cudaStream_t st) {
    if (plan.rows <= 8) return bf16 ? shrink_as<kBF16, 1>(in, ad, plan, u, st) : shrink_as<kF16, 1>(in, ad, plan, u, st);
    return bf16 ? shrink_as<kBF16, 4>(in, ad, plan, u, st) : shrink_as<kF16, 4>(in, ad, plan, u, st);
}

cudaError_t launch_expand(bool bf16, int M, int N, const Adapters& ad, int chunks, const float* u, const float* y32, void* y, int ydt, cudaStream_t st) {
    if (ydt == kF32) return bf16 ? expand_as<kBF16, kF32>(M, N, ad, chunks, u, y32, y, st) : expand_as<kF16, kF32>(M, N, ad, chunks, u, y32, y, st);
    return bf16 ? expand_as<kBF16, kBF16>(M, N, ad, chunks, u, y32, y, st) : expand_as<kF16, kF16>(M, N, ad, chunks, u, y32, y, st);
}

}  // namespace mmda
