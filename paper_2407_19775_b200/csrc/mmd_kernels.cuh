// mmd_kernels.cuh -- device code of the mixed matrix decomposition (sm_100a).
//
//   rowquant      : per row absmax over the regular features, int8 codes, row scale and the
//                   16-bit side columns of the critical features.  One CTA per row.
//   gemm_general  : Y = fma(fp32(qx qw^T), sx sw, sidex sidew^T) with integer dot products
//                   (dp4a) for any M and N; the correctness path and the fallback.
//   gemm_tc       : the same on the 5th-generation tensor cores: TMA loads 128-byte-swizzled
//                   tiles into a 4-stage shared-memory ring, one thread issues tcgen05.mma
//                   (kind::i8 into an int32 accumulator in tensor memory, then kind::f16 for
//                   the side columns into a second, fp32 accumulator), four warps read both
//                   accumulators back with tcgen05.ld and apply the scales.
//
// Arithmetic contract (it is what makes the integer part bit-identical to the plain
// definition): 127 v is exact in fp32 for 16-bit v; one IEEE division; cvt.rni (ties to
// even); int32 sums are exact; the output is one fma and one round-to-nearest-even narrowing.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mmd_elements.cuh"
#include "tc_primitives.cuh"

namespace mmdk {

constexpr int kSidePad = 64;

// ------------------------------------------------------------------------------------------
// rowquant: one CTA of 256 threads per row.  A bit mask of the critical features sits in
// shared memory, one byte per 16-byte chunk of the row, so the regular path costs one byte
// load per eight elements.  The row is read twice (the second pass hits L1 / L2).
//
// The kernel is bound by instruction issue, so both passes are written for few instructions:
// the absmax pass works on the packed 16-bit patterns (the magnitudes of finite fp16 / bf16
// values order like their bit patterns: one mask and one two-lane unsigned max per pair), the
// code pass does its fp32 arithmetic two elements per instruction, rounds to an integer by
// adding 1.5 * 2^23 (round-to-nearest-even, the low byte of the sum's bit pattern is the int8
// code) and gathers the four low bytes of a word with byte permutes.  A chunk that holds a
// critical feature (rare) takes a slower masked path.
__device__ __forceinline__ uint64_t rq_pack2(float a, float b) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ uint64_t rq_mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t rq_fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t rq_add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint32_t rq_prmt(uint32_t a, uint32_t b, uint32_t sel) {
    uint32_t d;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(sel));
    return d;
}
// per-halfword unsigned maximum
__device__ __forceinline__ uint32_t rq_max_u16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// 0xffff in the halves of word j (elements 2j, 2j + 1 of the chunk) whose mask bit is clear
__device__ __forceinline__ uint32_t rq_keep_halves(uint32_t mk, int j) {
    return (((mk >> (2 * j)) & 1u) ? 0u : 0x0000ffffu) | (((mk >> (2 * j + 1)) & 1u) ? 0u : 0xffff0000u);
}
// 0xff in the bytes of code word h (elements 4h .. 4h + 3 of the chunk) whose mask bit is clear
__device__ __forceinline__ uint32_t rq_keep_bytes(uint32_t mk, int h) {
    uint32_t keep = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) keep |= ((mk >> (4 * h + i)) & 1u) ? 0u : (0xffu << (8 * i));
    return keep;
}

template <int DT>
__global__ void __launch_bounds__(256, 6)                        // six CTAs per SM: the row's second read then mostly hits L1 / L2 while others load
rowquant(const void* v, int R, int K, const int32_t* __restrict__ idx, int ko, int side_cols,
         int8_t* __restrict__ q_out, float* __restrict__ scale_out, void* __restrict__ side_out,
         int* __restrict__ zero_words, int n_zero_words /* counters of the product kernel that follows; may be none */) {
    extern __shared__ __align__(16) unsigned char mask[];       // K / 8 bytes
    __shared__ uint32_t red[8];
    // A product kernel launched behind this one with programmatic stream serialization may start its set-up and its
    // weight loads now; it waits (griddepcontrol.wait) for this grid's results before it reads them.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int nchunks = K / 8;
    for (int c = threadIdx.x; c < (nchunks + 3) / 4; c += 256) reinterpret_cast<uint32_t*>(mask)[c] = 0u;
    // This kernel is itself launched with programmatic stream serialization: behind a product kernel that lets its
    // dependents start early (a chain of layers) its CTAs are already resident when that kernel ends.  Everything it reads
    // from or writes to global memory comes after this wait for the kernels before it (the product kernel of the previous
    // call may still be reading the buffers written below).
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __syncthreads();
    if (blockIdx.x == 0)
        for (int j = threadIdx.x; j < n_zero_words; j += 256) zero_words[j] = 0;
    for (int j = threadIdx.x; j < ko; j += 256) {
        const int k = idx[j];
        atomicOr(reinterpret_cast<uint32_t*>(mask) + (k >> 5), 1u << (k & 31));
    }
    __syncthreads();

    for (int r = blockIdx.x; r < R; r += gridDim.x) {
        const uint4* row = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(v) + size_t(r) * K);
        uint32_t m2 = 0u;                                                       // two running maxima of 15-bit magnitudes
        for (int c0 = threadIdx.x; c0 < nchunks; c0 += 256 * 4) {               // four loads in flight per thread
            uint4 w[4];
            uint32_t mk[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int c = c0 + 256 * u;
                const bool in = c < nchunks;
                w[u] = in ? row[c] : make_uint4(0, 0, 0, 0);
                mk[u] = in ? uint32_t(mask[c]) : 0u;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint32_t x[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
                if (mk[u] != 0u) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] &= rq_keep_halves(mk[u], j);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) m2 = rq_max_u16x2(m2, x[j] & 0x7fff7fffu);
            }
        }
        m2 = max(m2 & 0xffffu, m2 >> 16);
#pragma unroll
        for (int s = 16; s >= 1; s >>= 1) m2 = max(m2, __shfl_xor_sync(0xffffffffu, m2, s));
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m2;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) m2 = max(m2, red[i]);
        const float a = widen16<DT>(m2);
        const float d = (a != 0.0f) ? a : 1.0f;
        if (threadIdx.x == 0) scale_out[r] = __fdiv_rn(a, 127.0f);
        // t = RN32(127 v / d).  n = 127 v is exact; for d within [2^-64, 2^64]: q0 = RN(n rc), e = n - d q0 (exact in one
        // fma), t = RN(q0 + e rc) from the approximate reciprocal rc (within 1 ulp of 1 / d).  q0 + e rc is within a relative
        // 2^-44 of n / d while a quotient with an 11-bit divisor that is not itself an fp32 stays a relative 2^-36 away from
        // every rounding boundary, so t is the IEEE quotient (the CPU tests check every pair of 16-bit significands with rc
        // off by up to 2 ulp).  Outside the window: the IEEE division.  d is the same for the whole CTA.
        const bool quick = (d >= 5.421010862427522e-20f) && (d <= 1.8446744073709552e19f);
        float rc;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rc) : "f"(d));
        constexpr float kMagic = 12582912.0f;                                   // 1.5 * 2^23: t + kMagic rounds t to an integer, ties to even
        const uint64_t c127 = rq_pack2(127.0f, 127.0f), rc2 = rq_pack2(rc, rc), nd2 = rq_pack2(-d, -d), magic2 = rq_pack2(kMagic, kMagic);

        uint2* qrow = reinterpret_cast<uint2*>(q_out + size_t(r) * K);
        for (int c = threadIdx.x; c < nchunks; c += 256) {
            const uint4 w = row[c];
            const uint32_t mk = mask[c];
            float f[8];
            widen8<DT>(w, f);
            uint32_t b[8];                                                      // bit patterns whose low byte is the code
            if (quick) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const uint64_t n2 = rq_mul2(rq_pack2(f[i], f[i + 1]), c127);
                    const uint64_t q0 = rq_mul2(n2, rc2);
                    const uint64_t t2 = rq_fma2(rq_fma2(nd2, q0, n2), rc2, q0);
                    const uint64_t s2 = rq_add2(t2, magic2);
                    b[i] = uint32_t(s2);
                    b[i + 1] = uint32_t(s2 >> 32);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(__fadd_rn(__fdiv_rn(__fmul_rn(f[i], 127.0f), d), kMagic));
            }
            uint32_t lo = rq_prmt(rq_prmt(b[0], b[1], 0x0040u), rq_prmt(b[2], b[3], 0x0040u), 0x5410u);
            uint32_t hi = rq_prmt(rq_prmt(b[4], b[5], 0x0040u), rq_prmt(b[6], b[7], 0x0040u), 0x5410u);
            if (mk != 0u) {                                                     // critical features hold no code
                lo &= rq_keep_bytes(mk, 0);
                hi &= rq_keep_bytes(mk, 1);
            }
            qrow[c] = make_uint2(lo, hi);
        }
        uint16_t* srow = static_cast<uint16_t*>(side_out) + size_t(r) * side_cols;
        const uint16_t* vrow = static_cast<const uint16_t*>(v) + size_t(r) * K;
        for (int j = threadIdx.x; j < side_cols; j += 256) srow[j] = (j < ko) ? vrow[idx[j]] : uint16_t(0);
        __syncthreads();                                         // red[] is reused by the next row
    }
}

// ------------------------------------------------------------------------------------------
// norm_rowquant: the residual's addition, the root-mean-square norm and the row operation in one
// pass.  Per row, with h = RN16(x + res) (or x), t_k = RN32(h_k g_k), r = 1 / sqrt(mean h^2 + eps):
//     y_k  = t_k r                                the normed row
//     a    = max over regular k of |t_k|          (y's absmax is a r)
//     q_k  = rint(RN32(RN32(127 t_k) / a))        = the codes of y: r divides out of 127 y / max|y|
//     scale = RN32(RN32(a / 127) r),  side_j = RN16(RN32(t r)) at the critical features
// so the codes do not wait for the sum of squares and do not depend on its rounding.
//
// A thread keeps its first kNormChunks chunks of eight elements in registers (16-bit pairs); rows
// longer than that are read again (h_out as this thread wrote it, or x).  Bound by its bytes: per
// element 2 (x) + 2 (res) in and 2 (h) + 1 (code) out.  Measured, 4096 x 6144 bf16 with a residual: 37 us, 4.8 TB/s (27 us at the
// copy rate); the exact quotients (a product with the reciprocal, corrected by two fused multiply-adds) are most of the rest.
constexpr int kNormChunks = 4;

// the bit patterns of RN16(a + b) for a pair of elements
template <int DT>
__device__ __forceinline__ uint32_t add_pair(uint32_t a, uint32_t b) {
    const float lo = __fadd_rn(widen16<DT>(a & 0xffffu), widen16<DT>(b & 0xffffu)), hi = __fadd_rn(widen16<DT>(a >> 16), widen16<DT>(b >> 16));
    if constexpr (DT == kBF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}

// The factors and side columns of the CTA's rows once more, where some row's squares left fp32's range (|h| above 2^64) or lost bits
// below it: the sum runs over h 2^-E, with 2^E the larger of the row's largest |h| and sqrt(eps), to a factor of two, and
//     rms = 2^-E / sqrt(mean (h 2^-E)^2 + eps 2^-2E).
// The same sums in the same order, so rows in range get the bits that they had.  Rare, and a call of its own behind all rows: a
// second sum within the loop over the rows took registers that cost every row (4096 x 6144 bf16: 42.3 us).
template <int DT, int THREADS>
__device__ __noinline__ void norm_far_rows(const uint16_t* h, const uint16_t* gamma, int R, int K, float eps, const int32_t* idx, int ko, int side_cols,
                                           const unsigned char* mask, float* red /* shared, one per warp */, float* scale_out, uint16_t* side_out,
                                           float* rms_out) {
    auto of_block = [&](float v, auto join) {
#pragma unroll
        for (int s = 16; s >= 1; s >>= 1) v = join(v, __shfl_xor_sync(0xffffffffu, v, s));
        __syncthreads();                                         // everyone has read what was there
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.0f;
        for (int i = 0; i < THREADS / 32; ++i) v = join(v, red[i]);
        return v;
    };
    auto larger = [](float p, float q) { return fmaxf(p, q); };
    auto exponent = [](float v) { return int(__float_as_uint(v) >> 23) - 127; };
    for (int r = blockIdx.x; r < R; r += gridDim.x) {
        const uint4* hrow = reinterpret_cast<const uint4*>(h + size_t(r) * K);
        float a = 0.0f, big = 0.0f, ss = 0.0f, f[8], g[8];
        for (int c = threadIdx.x; c < K / 8; c += THREADS) {
            widen8<DT>(hrow[c], f);
            widen8<DT>(reinterpret_cast<const uint4*>(gamma)[c], g);
            for (int i = 0; i < 8; ++i) {
                big = fmaxf(big, fabsf(f[i]));
                if (!((mask[c] >> i) & 1u)) a = fmaxf(a, fabsf(__fmul_rn(f[i], g[i])));
            }
        }
        a = of_block(a, larger);
        big = of_block(big, larger);
        const int e = min(max(max(exponent(big), eps > 0.0f ? exponent(eps) >> 1 : -126), -126), 126);
        const float up = __uint_as_float(uint32_t(127 - e) << 23);
        for (int c = threadIdx.x; c < K / 8; c += THREADS) {
            widen8<DT>(hrow[c], f);
            for (int i = 0; i < 8; ++i) {
                const float v = __fmul_rn(f[i], up);
                ss = __fmaf_rn(v, v, ss);
            }
        }
        ss = of_block(ss, [](float p, float q) { return __fadd_rn(p, q); });
        const float rms = __fdiv_rn(up, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, float(K)), __fmul_rn(__fmul_rn(eps, up), up))));
        if (threadIdx.x == 0) {
            scale_out[r] = __fmul_rn(__fdiv_rn(a, 127.0f), rms);
            if (rms_out) rms_out[r] = rms;
        }
        for (int j = threadIdx.x; j < ko; j += THREADS) {
            const int k = idx[j];
            const float v = __fmul_rn(__fmul_rn(widen16<DT>(h[size_t(r) * K + k]), widen16<DT>(gamma[k])), rms);
            if constexpr (DT == kBF16) side_out[size_t(r) * side_cols + j] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
            else side_out[size_t(r) * side_cols + j] = __half_as_ushort(__float2half_rn(v));
        }
    }
}

template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
norm_rowquant(const void* x, const void* res /* h_out may be either of the two */, const void* __restrict__ gamma, int R, int K, float eps,
              const int32_t* __restrict__ idx, int ko, int side_cols, uint16_t* h_out, int8_t* __restrict__ q_out, float* __restrict__ scale_out,
              void* __restrict__ side_out, float* __restrict__ rms_out /* may be null */) {
    extern __shared__ __align__(16) unsigned char mask[];       // K / 8 bytes
    __shared__ float red_a[THREADS / 32], red_s[THREADS / 32];
    __shared__ int far;                                         // some row's squares left the range
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) far = 0;
    const int nchunks = K / 8;
    for (int c = threadIdx.x; c < (nchunks + 3) / 4; c += THREADS) reinterpret_cast<uint32_t*>(mask)[c] = 0u;
    asm volatile("griddepcontrol.wait;" ::: "memory");          // nothing in global memory is touched before the kernels before this one are done
    __syncthreads();
    for (int j = threadIdx.x; j < ko; j += THREADS) {
        const int k = idx[j];
        atomicOr(reinterpret_cast<uint32_t*>(mask) + (k >> 5), 1u << (k & 31));
    }
    __syncthreads();
    const uint4* grow = reinterpret_cast<const uint4*>(gamma);
    for (int r = blockIdx.x; r < R; r += gridDim.x) {
        const uint4* xrow = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + size_t(r) * K);
        const uint4* rrow = res ? reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(res) + size_t(r) * K) : nullptr;
        uint4* hrow = h_out ? reinterpret_cast<uint4*>(h_out + size_t(r) * K) : nullptr;
        float a = 0.0f, ss = 0.0f;
        auto first = [&](int c, uint4 w, uint4 b) {              // one chunk of the first pass: h, its squares and |t|
            if (rrow) {
                w = make_uint4(add_pair<DT>(w.x, b.x), add_pair<DT>(w.y, b.y), add_pair<DT>(w.z, b.z), add_pair<DT>(w.w, b.w));
            }
            if (hrow) hrow[c] = w;
            float f[8], g[8];
            widen8<DT>(w, f);
            widen8<DT>(__ldg(grow + c), g);
            const uint32_t mk = mask[c];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                ss = __fmaf_rn(f[i], f[i], ss);
                const float t = fabsf(__fmul_rn(f[i], g[i]));
                a = fmaxf(a, ((mk >> i) & 1u) ? 0.0f : t);
            }
            return w;
        };
        uint4 keep[kNormChunks];
        {
            uint4 b[kNormChunks];
#pragma unroll
            for (int u = 0; u < kNormChunks; ++u) {              // all loads before the arithmetic
                const int c = threadIdx.x + THREADS * u;
                if (c < nchunks) {
                    keep[u] = __ldcs(xrow + c);                           // (not through the read-only path: h_out may be the same memory)
                    if (rrow) b[u] = __ldcs(rrow + c);
                }
            }
#pragma unroll
            for (int u = 0; u < kNormChunks; ++u) {
                const int c = threadIdx.x + THREADS * u;
                if (c < nchunks) keep[u] = first(c, keep[u], b[u]);
            }
        }
        for (int c = threadIdx.x + THREADS * kNormChunks; c < nchunks; c += THREADS) first(c, xrow[c], rrow ? rrow[c] : make_uint4(0, 0, 0, 0));
#pragma unroll
        for (int s = 16; s >= 1; s >>= 1) {
            a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, s));
            ss += __shfl_xor_sync(0xffffffffu, ss, s);
        }
        if ((threadIdx.x & 31) == 0) { red_a[threadIdx.x >> 5] = a; red_s[threadIdx.x >> 5] = ss; }
        __syncthreads();
        a = 0.0f;
        ss = 0.0f;
#pragma unroll
        for (int i = 0; i < THREADS / 32; ++i) { a = fmaxf(a, red_a[i]); ss += red_s[i]; }
        const float rms = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, float(K)), eps)));
        const float d = (a != 0.0f) ? a : 1.0f;
        if (threadIdx.x == 0) {
            scale_out[r] = __fmul_rn(__fdiv_rn(a, 127.0f), rms);
            if (rms_out) rms_out[r] = rms;
            // squares that overflowed, or a sum below 2^-90 (which lost bits) that no eps above 2^-100 covers
            if (!(ss < INFINITY) || (ss < 8.0779357e-28f && eps < 7.8886091e-31f)) far = 1;
        }
        // RN32(n / d) for n = RN32(127 t).  rc = RN(1 / d); q0 = RN(n rc) is within two units of the quotient, one correction
        // with the exact remainder makes it faithful, a second one correctly rounded (Markstein's theorem: a faithful quotient,
        // a correctly rounded reciprocal, the exact remainder).  Inside the window nothing that decides a code can underflow;
        // outside it the IEEE division.
        const bool quick = (d >= 5.421010862427522e-20f) && (d <= 1.8446744073709552e19f);
        const float rc = __frcp_rn(d);
        constexpr float kMagic = 12582912.0f;                                   // 1.5 * 2^23: rounds to an integer, ties to even
        const uint64_t c127 = rq_pack2(127.0f, 127.0f), rc2 = rq_pack2(rc, rc), nd2 = rq_pack2(-d, -d), magic2 = rq_pack2(kMagic, kMagic);
        uint2* qrow = reinterpret_cast<uint2*>(q_out + size_t(r) * K);
        auto second = [&](int c, const uint4& w) {
            float f[8], g[8];
            widen8<DT>(w, f);
            widen8<DT>(__ldg(grow + c), g);
            const uint32_t mk = mask[c];
            uint32_t b[8];                                                      // bit patterns whose low byte is the code
            if (quick) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const uint64_t n2 = rq_mul2(rq_mul2(rq_pack2(f[i], f[i + 1]), rq_pack2(g[i], g[i + 1])), c127);
                    const uint64_t q0 = rq_mul2(n2, rc2);
                    const uint64_t q1 = rq_fma2(rq_fma2(nd2, q0, n2), rc2, q0);
                    const uint64_t s2 = rq_add2(rq_fma2(rq_fma2(nd2, q1, n2), rc2, q1), magic2);
                    b[i] = uint32_t(s2);
                    b[i + 1] = uint32_t(s2 >> 32);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(__fadd_rn(__fdiv_rn(__fmul_rn(__fmul_rn(f[i], g[i]), 127.0f), d), kMagic));
            }
            uint32_t lo = rq_prmt(rq_prmt(b[0], b[1], 0x0040u), rq_prmt(b[2], b[3], 0x0040u), 0x5410u);
            uint32_t hi = rq_prmt(rq_prmt(b[4], b[5], 0x0040u), rq_prmt(b[6], b[7], 0x0040u), 0x5410u);
            if (mk != 0u) {                                                     // critical features hold no code
                lo &= rq_keep_bytes(mk, 0);
                hi &= rq_keep_bytes(mk, 1);
            }
            qrow[c] = make_uint2(lo, hi);
        };
#pragma unroll
        for (int u = 0; u < kNormChunks; ++u) {
            const int c = threadIdx.x + THREADS * u;
            if (c < nchunks) second(c, keep[u]);
        }
        const uint4* again = hrow ? hrow : xrow;
        for (int c = threadIdx.x + THREADS * kNormChunks; c < nchunks; c += THREADS) second(c, again[c]);
        uint16_t* srow = static_cast<uint16_t*>(side_out) + size_t(r) * side_cols;
        for (int j = threadIdx.x; j < side_cols; j += THREADS) {
            uint16_t out = 0;
            if (j < ko) {                                                       // another thread's h: written before the barrier above
                const int k = idx[j];
                const uint32_t e = (h_out ? h_out : static_cast<const uint16_t*>(x))[size_t(r) * K + k];
                const float v = __fmul_rn(__fmul_rn(widen16<DT>(e), widen16<DT>(static_cast<const uint16_t*>(gamma)[k])), rms);
                if constexpr (DT == kBF16) out = __bfloat16_as_ushort(__float2bfloat16_rn(v));
                else out = __half_as_ushort(__float2half_rn(v));
            }
            srow[j] = out;
        }
        __syncthreads();                                         // red_* are reused by the next row
    }
    if (far)
        norm_far_rows<DT, THREADS>(h_out ? h_out : static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(gamma), R, K, eps, idx, ko, side_cols, mask, red_s,
                                   scale_out, static_cast<uint16_t*>(side_out), rms_out);
}

// ------------------------------------------------------------------------------------------
// gemm_general: 64 x 64 outputs per CTA of 256 threads, 4 x 4 per thread (rows ty + 16 i,
// columns tx + 16 j), 64 features per step through shared memory, four int8 products per dp4a.
template <int XDT, int YDT>
__global__ void __launch_bounds__(256)
gemm_general(const int8_t* __restrict__ qx, const int8_t* __restrict__ qw, const float* __restrict__ sx, const float* __restrict__ sw,
             const void* __restrict__ sidex, const void* __restrict__ sidew, int side_cols, void* __restrict__ y, int M, int N, int K) {
    __shared__ uint32_t xs[64][17];
    __shared__ uint32_t ws[64][17];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
    int acc[4][4];
    float part[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) { acc[i][j] = 0; part[i][j] = 0.0f; }

    const int lr = threadIdx.x >> 2, lc = threadIdx.x & 3;       // this thread's 16-byte piece of the 64 x 64-byte tiles
    for (int k0 = 0; k0 < K; k0 += 64) {
        uint4 a = make_uint4(0, 0, 0, 0), b = make_uint4(0, 0, 0, 0);
        const int kk = k0 + lc * 16;
        if (kk < K) {
            if (m0 + lr < M) a = *reinterpret_cast<const uint4*>(qx + size_t(m0 + lr) * K + kk);
            if (n0 + lr < N) b = *reinterpret_cast<const uint4*>(qw + size_t(n0 + lr) * K + kk);
        }
        __syncthreads();
        xs[lr][lc * 4 + 0] = a.x; xs[lr][lc * 4 + 1] = a.y; xs[lr][lc * 4 + 2] = a.z; xs[lr][lc * 4 + 3] = a.w;
        ws[lr][lc * 4 + 0] = b.x; ws[lr][lc * 4 + 1] = b.y; ws[lr][lc * 4 + 2] = b.z; ws[lr][lc * 4 + 3] = b.w;
        __syncthreads();
#pragma unroll
        for (int kw = 0; kw < 16; ++kw) {
            int av[4], bv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { av[i] = int(xs[ty + 16 * i][kw]); bv[i] = int(ws[tx + 16 * i][kw]); }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(av[i], bv[j], acc[i][j]);
        }
    }
    // side columns: 16 per step, widened to fp32 in shared memory
    float* xf = reinterpret_cast<float*>(&xs[0][0]);
    float* wf = reinterpret_cast<float*>(&ws[0][0]);
    for (int k0 = 0; k0 < side_cols; k0 += 16) {
        __syncthreads();
        {
            const int row = threadIdx.x >> 2, c4 = (threadIdx.x & 3) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = k0 + c4 + e;
                float xv = 0.0f, wv = 0.0f;
                if (m0 + row < M) xv = mmdk::widen16<XDT>(static_cast<const uint16_t*>(sidex)[size_t(m0 + row) * side_cols + col]);
                if (n0 + row < N) wv = mmdk::widen16<XDT>(static_cast<const uint16_t*>(sidew)[size_t(n0 + row) * side_cols + col]);
                xf[row * 17 + c4 + e] = xv;
                wf[row * 17 + c4 + e] = wv;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            float av[4], bv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { av[i] = xf[(ty + 16 * i) * 17 + k]; bv[i] = wf[(tx + 16 * i) * 17 + k]; }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) part[i][j] = __fmaf_rn(av[i], bv[j], part[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + ty + 16 * i;
        if (m >= M) continue;
        const float sxm = sx[m];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = n0 + tx + 16 * j;
            if (n >= N) continue;
            const float s = __fmul_rn(sxm, sw[n]);
            store_y<YDT>(y, size_t(m) * N + n, __fmaf_rn(float(acc[i][j]), s, part[i][j]));
        }
    }
}

// ------------------------------------------------------------------------------------------
// gemm_tc: tensor-core kernel.
//
// One CTA computes a 128 x BN tile of Y.  192 threads: warp 0 issues the TMA loads, warp 1
// allocates tensor memory and issues the MMAs, warps 2-5 are the epilogue (warp w reads the
// 32 accumulator lanes of its quarter, w % 4).  A stage of the ring holds a 128-row tile of
// the activations and a BN-row tile of the weights, each row 128 bytes (128 int8 features,
// or 64 side columns of 16 bits), written by TMA with the 128-byte swizzle that the MMA's
// shared-memory descriptors name.  The int8 steps accumulate into columns [0, BN) of tensor
// memory as int32; the side steps into columns [BN, 2 BN) as fp32.
//
// Every wait is bounded: a wait that runs out records a code in *status, raises the CTA's
// abort flag and the kernel winds down (no further stores, tensor memory freed).
//
// Split K.  A call with one row of tiles over a narrow layer (a decode step) has fewer tiles
// than the GPU has SMs, and an SM streams weights from DRAM only as fast as the bytes it can
// keep in flight.  Such calls are launched in clusters of 2-4 CTAs along z: the CTAs of a
// cluster work on the same tile, each on its own share of the K steps (the side steps go to
// rank 0), and afterwards ranks 1.. write their int32 accumulators into rank 0's ring memory
// (distributed shared memory; the ring is free by then, which the first cluster barrier
// establishes), a second cluster barrier publishes them, and rank 0 adds them to its own and
// runs the epilogue.  Integer sums do not depend on the order, so the result is the same bits.

constexpr int kTcThreads = 192;
constexpr int kTcBM = 128;
constexpr int kTcRowBytes = 128;

// BM = rows of the MMA: 128, or 64 for calls with at most 64 activation rows (a decode step), whose ring stages then
// spend 8 KB instead of 16 KB on activations and hold more steps of the weight stream in flight.
// KPB = K blocks of 128 features one ring step (one TMA load per operand) brings: 1, or 2 for decode-size calls, where
// the pace is set by the number of loads rather than by their bytes.
template <int BN, int BM = kTcBM, int KPB = 1> struct TcCfg {
    static constexpr uint32_t kASlabBytes = BM * kTcRowBytes;                   // one K block of the activation tile
    static constexpr uint32_t kBSlabBytes = BN * kTcRowBytes;
    static constexpr uint32_t kABytes = KPB * kASlabBytes;
    static constexpr uint32_t kBBytes = KPB * kBSlabBytes;
    static constexpr uint32_t kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = (196608u / kStageBytes) > 12u ? 12 : int(196608u / kStageBytes);
    static constexpr uint32_t kTmemCols = (2 * BN <= 32) ? 32 : 2 * BN;          // a power of two >= 32
    static constexpr uint32_t kSmemBytes = kStages * kStageBytes + 1024 /* alignment slack */ + 2048 /* barriers, scales */;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address, in the cluster's shared window, of this CTA's shared address `addr` in CTA `rank`
__device__ __forceinline__ uint32_t map_to_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void st_cluster_u32(uint32_t cluster_addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}

template <int XDT, int YDT, int BN, int BM, int KPB>
__global__ void __launch_bounds__(kTcThreads, 1)
gemm_tc(const __grid_constant__ CUtensorMap map_qx, const __grid_constant__ CUtensorMap map_qw,
        const __grid_constant__ CUtensorMap map_sidex, const __grid_constant__ CUtensorMap map_sidew,
        const float* __restrict__ sx, const float* __restrict__ sw, void* __restrict__ y,
        int M, int N, int kblocks_all /* K blocks of 128 int8 features */, int sblocks_all /* side steps of 64 columns */,
        int n_tile_base /* first column tile of this launch */, int* status) {
    using Cfg = TcCfg<BN, BM, KPB>;
    constexpr uint32_t kTxMain = Cfg::kStageBytes;                              // bytes of an int8 step's two loads (boxes of BM and BN rows)
    constexpr uint32_t kTxSide = Cfg::kASlabBytes + Cfg::kBSlabBytes;           // bytes of a side step's two loads
    constexpr int S = Cfg::kStages;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;               // swizzled tiles need 1024-byte alignment
    unsigned char* ctrl = smem_raw + (tiles - smem_u32(smem_raw)) + S * Cfg::kStageBytes;
    const uint32_t full0 = smem_u32(ctrl);                                      // S barriers: tile landed
    const uint32_t empty0 = full0 + 8u * S;                                     // S barriers: tile consumed
    const uint32_t accbar = empty0 + 8u * S;                                    // accumulators complete
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl + 8 * (2 * S + 1));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 8 * (2 * S + 1) + 8);
    volatile int* peer_gave_up = reinterpret_cast<volatile int*>(ctrl + 8 * (2 * S + 1) + 12);   // split K: set in rank 0 by a rank that ran out of a wait
    static_assert(8 * (2 * S + 1) + 16 <= 256, "control words end before the column scales");
    float* sw_s = reinterpret_cast<float*>(ctrl + 256);                         // BN scales of this tile's columns

    // Kernels launched behind this one with programmatic stream serialization (the row kernel of the next call, or this
    // call's second launch for the tiles left over) may become resident as SMs free up; each waits for this grid to
    // complete before it touches global memory that this grid reads or writes.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int m0 = blockIdx.x * BM, n0 = (n_tile_base + int(blockIdx.y)) * BN;
    const uint32_t nsplit = cluster_size(), rank = cluster_rank();              // 1 and 0 without a cluster launch
    const int ksteps_all = (kblocks_all + KPB - 1) / KPB;                       // int8 ring steps of KPB K blocks each
    const int kb_lo = int((long(ksteps_all) * rank) / nsplit), kb_hi = int((long(ksteps_all) * (rank + 1)) / nsplit);
    const int kblocks = kb_hi - kb_lo;                                          // this CTA's share of the int8 steps
    const int sblocks = (rank == 0) ? sblocks_all : 0;
    const int steps = kblocks + sblocks;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(full0 + 8u * s, 1); mbar_init(empty0 + 8u * s, 1); }
        mbar_init(accbar, 1);
        *abort_flag = 0;
        *peer_gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(Cfg::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;
    // the load of one int8 step of one operand: KPB K blocks of `rows` rows from K block `step * KPB` on
    auto load_main = [&](uint32_t dst, const CUtensorMap* map, int row0, int step, uint32_t bar) {
        if constexpr (KPB == 1) tma_load_2d(dst, map, step * 128, row0, bar);
        else tma_load_3d(dst, map, row0, step * KPB, bar);                      // a K block past the end reads as zeros
    };

    if (warp == 0) {
        if (lane == 0) {
            // The first ring-full of weight tiles does not depend on the row kernel that runs before this one: their loads
            // go out at once; the activation tiles of those stages follow when that kernel's results are visible.
            const int pre = steps < S ? steps : S;
            for (int i = 0; i < pre; ++i) {
                const uint32_t b_dst = tiles + uint32_t(i) * Cfg::kStageBytes + Cfg::kABytes;
                mbar_expect_tx(full0 + 8u * i, i < kblocks ? kTxMain : kTxSide);
                if (i < kblocks) load_main(b_dst, &map_qw, n0, kb_lo + i, full0 + 8u * i);
                else tma_load_2d(b_dst, &map_sidew, (i - kblocks) * 64, n0, full0 + 8u * i);
            }
            asm volatile("griddepcontrol.wait;" ::: "memory");
            for (int i = 0; i < pre; ++i) {
                const uint32_t a_dst = tiles + uint32_t(i) * Cfg::kStageBytes;
                if (i < kblocks) load_main(a_dst, &map_qx, m0, kb_lo + i, full0 + 8u * i);
                else tma_load_2d(a_dst, &map_sidex, (i - kblocks) * 64, m0, full0 + 8u * i);
            }
            for (int i = pre; i < steps; ++i) {
                const int s = i % S;
                const uint32_t round = uint32_t(i / S);
                if (!mbar_wait(empty0 + 8u * s, (round & 1u) ^ 1u, abort_flag, status, 1)) break;
                const uint32_t a_dst = tiles + uint32_t(s) * Cfg::kStageBytes, b_dst = a_dst + Cfg::kABytes;
                mbar_expect_tx(full0 + 8u * s, i < kblocks ? kTxMain : kTxSide);
                if (i < kblocks) {
                    load_main(a_dst, &map_qx, m0, kb_lo + i, full0 + 8u * s);
                    load_main(b_dst, &map_qw, n0, kb_lo + i, full0 + 8u * s);
                } else {
                    tma_load_2d(a_dst, &map_sidex, (i - kblocks) * 64, m0, full0 + 8u * s);
                    tma_load_2d(b_dst, &map_sidew, (i - kblocks) * 64, n0, full0 + 8u * s);
                }
            }
        }
        __syncwarp();
        if (nsplit > 1) { cluster_sync_all(); cluster_sync_all(); }              // the two barriers of the exchange (see the epilogue)
    } else if (warp == 1) {
        if (elect_one()) {
            constexpr uint32_t idesc_i8 = umma_idesc(2, 1, BM, BN);                      // int32 <- int8 x int8
            constexpr uint32_t idesc_16 = umma_idesc(1, XDT == kBF16 ? 1u : 0u, BM, BN);        // fp32 <- 16-bit x 16-bit
            bool ok = true;
            for (int i = 0; i < steps && ok; ++i) {
                const int s = i % S;
                const uint32_t round = uint32_t(i / S);
                ok = mbar_wait(full0 + 8u * s, round & 1u, abort_flag, status, 2);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t a_src = tiles + uint32_t(s) * Cfg::kStageBytes, b_src = a_src + Cfg::kABytes;
                const uint64_t adesc = umma_smem_desc(a_src), bdesc = umma_smem_desc(b_src);
                if (i < kblocks) {
#pragma unroll
                    for (int j = 0; j < KPB; ++j) {
                        const uint64_t aj = umma_smem_desc(a_src + uint32_t(j) * Cfg::kASlabBytes), bj = umma_smem_desc(b_src + uint32_t(j) * Cfg::kBSlabBytes);
#pragma unroll
                        for (int k = 0; k < 4; ++k)                   // 32 int8 features = 32 bytes per MMA
                            umma_i8(tmem, aj + uint64_t(2 * k), bj + uint64_t(2 * k), idesc_i8, (i > 0 || j > 0 || k > 0) ? 1u : 0u);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)                       // 16 side columns = 32 bytes per MMA
                        umma_f16(tmem + uint32_t(BN), adesc + uint64_t(2 * k), bdesc + uint64_t(2 * k), idesc_16, (i > kblocks || k > 0) ? 1u : 0u);
                }
                umma_commit(empty0 + 8u * s);                         // the stage is free once these MMAs have read it
            }
            if (ok) umma_commit(accbar);
        }
        __syncwarp();
        if (nsplit > 1) { cluster_sync_all(); cluster_sync_all(); }
    } else {
        // epilogue: 128 threads, one accumulator row each
        const int et = threadIdx.x - 64;
        for (int c = et; c < BN; c += 128) sw_s[c] = (n0 + c < N) ? sw[n0 + c] : 0.0f;
        asm volatile("bar.sync 1, 128;" ::: "memory");
        asm volatile("griddepcontrol.wait;" ::: "memory");       // the activations' row scales come from the kernel before this one
        const int quarter = warp & 3;
        // a 128-row accumulator has row r in lane r; a 64-row one keeps rows 16 q .. 16 q + 15 in the first 16 lanes of
        // quarter q (the other lanes of the quarter hold nothing of it)
        const bool row_lane = (BM == 128) || lane < 16;
        const int m = row_lane ? m0 + quarter * (BM / 4) + lane : M;
        const float sxm = (m < M) ? sx[m] : 0.0f;
        bool ok = true;
        if (lane == 0) ok = mbar_wait(accbar, 0, abort_flag, status, 3);
        ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t lane_base = tmem + (uint32_t(quarter * 32) << 16);
        const uint32_t row_in_tile = uint32_t(quarter * (BM / 4) + lane);       // meaningful where row_lane holds
        constexpr uint32_t kPartBytes = uint32_t(BM) * BN * 4u;                  // one rank's accumulator, stored [column][row]
        if (nsplit > 1) {
            cluster_sync_all();                                                  // every CTA of the cluster is through its main loop: rank 0's ring is free
            if (rank > 0) {
#pragma unroll 1
                for (int c0 = 0; c0 < BN; c0 += 32) {
                    uint32_t ai[32];
                    tmem_ld32(lane_base + uint32_t(c0), ai);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                    if (ok && row_lane) {
                        const uint32_t dst = map_to_cta(tiles + (rank - 1u) * kPartBytes + uint32_t(c0) * BM * 4u + row_in_tile * 4u, 0);
#pragma unroll
                        for (int j = 0; j < 32; ++j) st_cluster_u32(dst + uint32_t(j) * BM * 4u, ai[j]);
                    }
                }
                // a rank whose wait ran out has no sums to give: it says so, and rank 0 then stores nothing for this tile
                if (!ok && lane == 0) st_cluster_u32(map_to_cta(smem_u32(const_cast<int*>(peer_gave_up)), 0), 1u);
            }
            cluster_sync_all();                                                  // the partial sums are in rank 0's shared memory
            if (rank == 0 && *peer_gave_up) ok = false;
        }
        if (ok && rank == 0) {
#pragma unroll 1
            for (int c0 = 0; c0 < BN; c0 += 32) {
                uint32_t ai[32], af[32];
                tmem_ld32(lane_base + uint32_t(c0), ai);
                if (sblocks > 0) tmem_ld32(lane_base + uint32_t(BN + c0), af);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                if (nsplit > 1 && row_lane) {
                    for (uint32_t r = 1; r < nsplit; ++r) {
                        const uint32_t src = tiles + (r - 1u) * kPartBytes + uint32_t(c0) * BM * 4u + row_in_tile * 4u;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            uint32_t v;
                            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(src + uint32_t(j) * BM * 4u) : "memory");
                            ai[j] += v;
                        }
                    }
                }
                float out[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const float s = __fmul_rn(sxm, sw_s[c0 + j]);
                    const float p = (sblocks > 0) ? __uint_as_float(af[j]) : 0.0f;
                    out[j] = __fmaf_rn(float(int(ai[j])), s, p);
                }
                if (m < M) {
                    const int n = n0 + c0;
                    if constexpr (YDT == kF32) {
                        float* dst = static_cast<float*>(y) + size_t(m) * N + n;
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            if (n + j < N) *reinterpret_cast<float4*>(dst + j) = make_float4(out[j], out[j + 1], out[j + 2], out[j + 3]);
                    } else {
                        uint16_t* dst = static_cast<uint16_t*>(y) + size_t(m) * N + n;
#pragma unroll
                        for (int j = 0; j < 32; j += 8) {
                            uint32_t pk[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if constexpr (YDT == kBF16) {
                                    const __nv_bfloat162 h = __floats2bfloat162_rn(out[j + 2 * e], out[j + 2 * e + 1]);
                                    pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                                } else {
                                    const __half2 h = __floats2half2_rn(out[j + 2 * e], out[j + 2 * e + 1]);
                                    pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                                }
                            }
                            if (n + j < N) *reinterpret_cast<uint4*>(dst + j) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                        }
                    }
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }

    __syncthreads();
    if (*abort_flag) {
        // copies that were issued but never waited for may still be landing in this CTA's
        // shared memory: give them time before the memory is handed to another CTA
        for (int i = 0; i < 64; ++i) __nanosleep(2000);
        __syncthreads();
    }
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Cfg::kTmemCols) : "memory");
    }
}


// ------------------------------------------------------------------------------------------
// gemm_sk: one row of tiles (a decode step, at most 64 activation rows) with the K steps of ALL
// tiles dealt out evenly over the CTAs of one launch ("stream K").
//
// gemm_tc gives every 128-column tile to one CTA, or to a cluster of 2-4 CTAs that share its K
// steps; with 64 tiles on 148 SMs either 84 SMs stream weights or 128 do.  Here the units of
// work (per tile: its int8 steps of two K blocks, then one unit for all of its side steps) are
// numbered across the tiles and CTA c takes units [c T / G, (c + 1) T / G): every SM streams the
// same number of bytes, whatever the number of tiles.  A CTA's range touches at most two tiles
// (the host launches at least as many CTAs as tiles); the part of a tile that a CTA computes is a
// "segment", accumulated in its own half of tensor memory, so the epilogue of the first segment
// runs under the loads and MMAs of the second.
//
// Tiles that several CTAs share are put together without anybody waiting: a CTA writes its
// segment's int32 sums (and, if it holds the tile's side unit, the fp32 side sums) to a slot of
// global scratch, fences, and takes a ticket from the tile's counter; the CTA whose ticket is
// the last one adds the other slots to its own sums, which are still in its tensor memory, and
// runs the epilogue.  Integer sums do not depend on the order and the side sums come from one
// CTA, so the result is the same bits as gemm_tc's.  The counters are zeroed by the row kernel
// that runs before every product.  Waits are bounded as in gemm_tc.
constexpr int kSkBN = 128, kSkBM = 64, kSkKPB = 2;

template <int XDT, int YDT>
__global__ void __launch_bounds__(kTcThreads, 1)
gemm_sk(const __grid_constant__ CUtensorMap map_qx, const __grid_constant__ CUtensorMap map_qw,
        const __grid_constant__ CUtensorMap map_sidex, const __grid_constant__ CUtensorMap map_sidew,
        const float* __restrict__ sx, const float* __restrict__ sw, void* __restrict__ y,
        int M, int N, int kblocks_all, int sblocks_all, int n_tiles, int maxparts,
        int* __restrict__ counters, int* __restrict__ part_acc, float* __restrict__ part_side, int* status) {
    using Cfg = TcCfg<kSkBN, kSkBM, kSkKPB>;
    constexpr int BN = kSkBN, BM = kSkBM, KPB = kSkKPB, S = Cfg::kStages;
    constexpr uint32_t kTxMain = Cfg::kStageBytes;
    constexpr uint32_t kTxSide = Cfg::kASlabBytes + Cfg::kBSlabBytes;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* ctrl = smem_raw + (tiles - smem_u32(smem_raw)) + S * Cfg::kStageBytes;
    const uint32_t full0 = smem_u32(ctrl);                                      // S barriers: tile landed
    const uint32_t empty0 = full0 + 8u * S;                                     // S barriers: tile consumed
    const uint32_t accbar0 = empty0 + 8u * S;                                   // 2 barriers: a segment's accumulators complete
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl + 8 * (2 * S + 2));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 8 * (2 * S + 2) + 8);
    volatile int* ticket = reinterpret_cast<volatile int*>(ctrl + 8 * (2 * S + 2) + 12);
    static_assert(8 * (2 * S + 2) + 16 <= 256, "control words end before the column scales");
    float* sw_s = reinterpret_cast<float*>(ctrl + 256);                         // 2 x BN scales: one set per segment

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ksteps = (kblocks_all + KPB - 1) / KPB;
    const int upt = ksteps + (sblocks_all > 0 ? 1 : 0);                         // units per tile
    const long long total = (long long)n_tiles * upt;
    const long long G = gridDim.x, c = blockIdx.x;
    const long long lo = total * c / G, hi = total * (c + 1) / G;               // this CTA's units
    const int t_first = int(lo / upt), t_last = int((hi - 1) / upt);
    const int nseg = (hi > lo) ? t_last - t_first + 1 : 0;                      // 0, 1 or 2

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(full0 + 8u * s, 1); mbar_init(empty0 + 8u * s, 1); }
        mbar_init(accbar0, 1);
        mbar_init(accbar0 + 8u, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;

    // ring steps of a unit: an int8 unit is one step, the side unit is sblocks_all steps
    auto steps_of = [&](long long g) -> int { return (int(g % upt) < ksteps) ? 1 : sblocks_all; };

    if (warp == 0) {
        if (lane == 0) {
            // The loads of one ring step: `side` < 0 is int8 step `kstep` of tile `t`, otherwise side step `side`.
            auto issue_b = [&](int s, int t, int kstep, int side) {
                const uint32_t b_dst = tiles + uint32_t(s) * Cfg::kStageBytes + Cfg::kABytes;
                if (side < 0) tma_load_3d(b_dst, &map_qw, t * BN, kstep * KPB, full0 + 8u * s);
                else tma_load_2d(b_dst, &map_sidew, side * 64, t * BN, full0 + 8u * s);
            };
            auto issue_a = [&](int s, int kstep, int side) {
                const uint32_t a_dst = tiles + uint32_t(s) * Cfg::kStageBytes;
                if (side < 0) tma_load_3d(a_dst, &map_qx, 0, kstep * KPB, full0 + 8u * s);
                else tma_load_2d(a_dst, &map_sidex, side * 64, 0, full0 + 8u * s);
            };
            // The first ring-full of weight tiles does not depend on the row kernel before this one.
            int it = 0;
            bool waited = false, ok = true;
            int pre_t[S], pre_k[S], pre_side[S], npre = 0;
            for (long long g = lo; g < hi && ok; ++g) {
                const int t = int(g / upt), u = int(g % upt);
                const int nst = steps_of(g);
                for (int j = 0; j < nst && ok; ++j, ++it) {
                    const int s = it % S;
                    const int kstep = (u < ksteps) ? u : 0, side = (u < ksteps) ? -1 : j;
                    if (it < S) {                                                    // ring not yet wrapped: weights now, activations after the wait
                        mbar_expect_tx(full0 + 8u * s, side < 0 ? kTxMain : kTxSide);
                        issue_b(s, t, kstep, side);
                        pre_t[npre] = t; pre_k[npre] = kstep; pre_side[npre] = side; ++npre;
                        continue;
                    }
                    if (!waited) {
                        asm volatile("griddepcontrol.wait;" ::: "memory");
                        for (int q = 0; q < npre; ++q) issue_a(q, pre_k[q], pre_side[q]);
                        waited = true;
                    }
                    ok = mbar_wait(empty0 + 8u * s, ((uint32_t(it / S) & 1u) ^ 1u), abort_flag, status, 1);
                    if (!ok) break;
                    mbar_expect_tx(full0 + 8u * s, side < 0 ? kTxMain : kTxSide);
                    issue_a(s, kstep, side);
                    issue_b(s, t, kstep, side);
                }
            }
            if (!waited) {
                asm volatile("griddepcontrol.wait;" ::: "memory");
                for (int q = 0; q < npre; ++q) issue_a(q, pre_k[q], pre_side[q]);
            }
            (void)pre_t;
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            constexpr uint32_t idesc_i8 = umma_idesc(2, 1, BM, BN);
            constexpr uint32_t idesc_16 = umma_idesc(1, XDT == kBF16 ? 1u : 0u, BM, BN);
            int it = 0;
            bool ok = true;
            for (int seg = 0; seg < nseg && ok; ++seg) {
                const int t = t_first + seg;
                const long long a = (lo > (long long)t * upt) ? lo : (long long)t * upt;
                const long long b = (hi < (long long)(t + 1) * upt) ? hi : (long long)(t + 1) * upt;
                const uint32_t tm = tmem + uint32_t(seg & 1) * 256u;
                bool first_i8 = true, first_side = true;
                for (long long g = a; g < b && ok; ++g) {
                    const int u = int(g % upt);
                    const int nst = steps_of(g);
                    for (int j = 0; j < nst && ok; ++j, ++it) {
                        const int s = it % S;
                        ok = mbar_wait(full0 + 8u * s, uint32_t(it / S) & 1u, abort_flag, status, 2);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t a_src = tiles + uint32_t(s) * Cfg::kStageBytes, b_src = a_src + Cfg::kABytes;
                        if (u < ksteps) {
#pragma unroll
                            for (int jj = 0; jj < KPB; ++jj) {
                                const uint64_t aj = umma_smem_desc(a_src + uint32_t(jj) * Cfg::kASlabBytes), bj = umma_smem_desc(b_src + uint32_t(jj) * Cfg::kBSlabBytes);
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    umma_i8(tm, aj + uint64_t(2 * k), bj + uint64_t(2 * k), idesc_i8, (first_i8 && jj == 0 && k == 0) ? 0u : 1u);
                            }
                            first_i8 = false;
                        } else {
                            const uint64_t adesc = umma_smem_desc(a_src), bdesc = umma_smem_desc(b_src);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                umma_f16(tm + uint32_t(BN), adesc + uint64_t(2 * k), bdesc + uint64_t(2 * k), idesc_16, (first_side && k == 0) ? 0u : 1u);
                            first_side = false;
                        }
                        umma_commit(empty0 + 8u * s);
                    }
                }
                if (ok) umma_commit(accbar0 + 8u * uint32_t(seg & 1));
            }
        }
        __syncwarp();
    } else {
        // epilogue: 128 threads; a 64-row accumulator keeps rows 16 q .. 16 q + 15 in the first 16 lanes of quarter q
        const int et = threadIdx.x - 64;
        const int quarter = warp & 3;
        const bool row_lane = lane < 16;
        const int m = row_lane ? quarter * 16 + lane : M;
        asm volatile("griddepcontrol.wait;" ::: "memory");       // row scales and the zeroed counters come from the kernel before this one
        const float sxm = (m < M) ? sx[m] : 0.0f;
        const uint32_t row_in_tile = uint32_t(quarter * 16 + lane);
        constexpr size_t kPart = size_t(BM) * BN;                                // values of one partial tile, stored [row][column]
        for (int seg = 0; seg < nseg; ++seg) {
            const int t = t_first + seg;
            const int n0 = t * BN;
            const long long ta = (long long)t * upt, tb = (long long)(t + 1) * upt;
            const long long a = lo > ta ? lo : ta, b = hi < tb ? hi : tb;
            const bool has_side = sblocks_all > 0 && b == tb;                    // the side unit is the tile's last
            const bool has_i8 = a < ta + ksteps;                                 // a segment of the side unit alone has no integer sums
            const int c_first = int(((ta + 1) * G + total - 1) / total) - 1, c_last = int((tb * G + total - 1) / total) - 1;
            const int parts = c_last - c_first + 1, mypart = int(c) - c_first;
            float* sws = sw_s + (seg & 1) * BN;
            for (int cc = et; cc < BN; cc += 128) sws[cc] = (n0 + cc < N) ? sw[n0 + cc] : 0.0f;
            asm volatile("bar.sync 1, 128;" ::: "memory");
            bool ok = true;
            if (lane == 0) ok = mbar_wait(accbar0 + 8u * uint32_t(seg & 1), 0, abort_flag, status, 3);
            ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t lane_base = tmem + uint32_t(seg & 1) * 256u + (uint32_t(quarter * 32) << 16);
            bool last = true;
            if (parts > 1) {
                // this segment's sums into its slot, then a ticket: the last one to arrive finishes the tile
                if (ok) {
#pragma unroll 1
                    for (int c0 = 0; c0 < BN; c0 += 32) {
                        uint32_t ai[32], af[32];
                        tmem_ld32(lane_base + uint32_t(c0), ai);
                        if (has_side) tmem_ld32(lane_base + uint32_t(BN + c0), af);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                        if (!has_i8) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) ai[j] = 0u;
                        }
                        if (row_lane) {
                            int* dst = part_acc + (size_t(t) * maxparts + mypart) * kPart + size_t(row_in_tile) * BN + c0;
#pragma unroll
                            for (int j = 0; j < 32; j += 4) *reinterpret_cast<uint4*>(dst + j) = make_uint4(ai[j], ai[j + 1], ai[j + 2], ai[j + 3]);
                            if (has_side) {
                                float* ds = part_side + size_t(t) * kPart + size_t(row_in_tile) * BN + c0;
#pragma unroll
                                for (int j = 0; j < 32; j += 4) *reinterpret_cast<uint4*>(ds + j) = make_uint4(af[j], af[j + 1], af[j + 2], af[j + 3]);
                            }
                        }
                    }
                    __threadfence();
                }
                asm volatile("bar.sync 1, 128;" ::: "memory");
                if (et == 0) *ticket = ok ? atomicAdd(counters + t, 1) : -1;      // a segment that gave up takes no ticket: the tile is then never finished
                asm volatile("bar.sync 1, 128;" ::: "memory");
                last = (*ticket == parts - 1);
                __threadfence();
            }
            if (ok && last) {
#pragma unroll 1
                for (int c0 = 0; c0 < BN; c0 += 32) {
                    uint32_t ai[32], af[32];
                    tmem_ld32(lane_base + uint32_t(c0), ai);
                    if (has_side) tmem_ld32(lane_base + uint32_t(BN + c0), af);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                    if (!has_i8) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) ai[j] = 0u;
                    }
                    if (parts > 1 && row_lane) {
                        for (int pp = 0; pp < parts; ++pp) {
                            if (pp == mypart) continue;
                            const int* src = part_acc + (size_t(t) * maxparts + pp) * kPart + size_t(row_in_tile) * BN + c0;
#pragma unroll
                            for (int j = 0; j < 32; j += 4) {
                                const uint4 v = __ldcg(reinterpret_cast<const uint4*>(src + j));
                                ai[j] += v.x; ai[j + 1] += v.y; ai[j + 2] += v.z; ai[j + 3] += v.w;
                            }
                        }
                        if (sblocks_all > 0 && !has_side) {
                            const float* ss = part_side + size_t(t) * kPart + size_t(row_in_tile) * BN + c0;
#pragma unroll
                            for (int j = 0; j < 32; j += 4) {
                                const uint4 v = __ldcg(reinterpret_cast<const uint4*>(ss + j));
                                af[j] = v.x; af[j + 1] = v.y; af[j + 2] = v.z; af[j + 3] = v.w;
                            }
                        }
                    }
                    float out[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const float sc = __fmul_rn(sxm, sws[c0 + j]);
                        const float pside = (sblocks_all > 0) ? __uint_as_float(af[j]) : 0.0f;
                        out[j] = __fmaf_rn(float(int(ai[j])), sc, pside);
                    }
                    if (m < M) {
                        const int n = n0 + c0;
                        if constexpr (YDT == kF32) {
                            float* dst = static_cast<float*>(y) + size_t(m) * N + n;
#pragma unroll
                            for (int j = 0; j < 32; j += 4)
                                if (n + j < N) *reinterpret_cast<float4*>(dst + j) = make_float4(out[j], out[j + 1], out[j + 2], out[j + 3]);
                        } else {
                            uint16_t* dst = static_cast<uint16_t*>(y) + size_t(m) * N + n;
#pragma unroll
                            for (int j = 0; j < 32; j += 8) {
                                uint32_t pk[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if constexpr (YDT == kBF16) {
                                        const __nv_bfloat162 h = __floats2bfloat162_rn(out[j + 2 * e], out[j + 2 * e + 1]);
                                        pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                                    } else {
                                        const __half2 h = __floats2half2_rn(out[j + 2 * e], out[j + 2 * e + 1]);
                                        pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                                    }
                                }
                                if (n + j < N) *reinterpret_cast<uint4*>(dst + j) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                            }
                        }
                    }
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }

    __syncthreads();
    if (*abort_flag) {
        for (int i = 0; i < 64; ++i) __nanosleep(2000);
        __syncthreads();
    }
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ------------------------------------------------------------------------------------------
// gemm_tcp: persistent tensor-core kernel for large products with at most kTcpSide critical
// features.
//
// One CTA per SM walks over 128 x 256 tiles (M-tile index fastest, so CTAs that run together
// share weight tiles in L2).  Tensor memory holds TWO int32 accumulators (2 x 256 columns):
// while the epilogue warps drain the accumulator of tile i, the MMA thread is already
// accumulating tile i + 1 into the other one, and the TMA thread runs ahead through the
// 4-stage ring, so set-up, the first load round trip and the epilogue no longer stop the
// tensor pipe between tiles.  With both accumulators taken by integer sums the side columns
// cannot use the tensor cores here; they are few, so the epilogue adds them with fp32 FMAs
// in ascending feature order (the same order as gemm_general), hidden under the next tile's
// MMAs.  Waits are bounded as in gemm_tc.

constexpr int kTcpBN = 256;
constexpr int kTcpStages = 4;
constexpr int kTcpSide = 16;                                   // most critical features this kernel takes
constexpr uint32_t kTcpStageBytes = (kTcBM + kTcpBN) * kTcRowBytes;
constexpr uint32_t kTcpCtrlBytes = 512;
constexpr uint32_t kTcpSwBytes = 2 * kTcpBN * 4;               // column scales, one copy per accumulator
constexpr uint32_t kTcpWoBytes = kTcpBN * kTcpSide * 4;        // side columns of the tile's weight rows, fp32
constexpr uint32_t kTcpSmemBytes = kTcpStages * kTcpStageBytes + 1024 + kTcpCtrlBytes + kTcpSwBytes + kTcpWoBytes;

template <int XDT, int YDT>
__global__ void __launch_bounds__(kTcThreads, 1)
gemm_tcp(const __grid_constant__ CUtensorMap map_qx, const __grid_constant__ CUtensorMap map_qw,
         const float* __restrict__ sx, const float* __restrict__ sw, const void* __restrict__ sidex, const void* __restrict__ sidew,
         int side_cols /* row pitch of the side matrices */, int ko /* critical features, <= kTcpSide */,
         void* __restrict__ y, int M, int N, int kblocks, int mtiles, int ntiles, int* status) {
    constexpr int S = kTcpStages;
    constexpr int BN = kTcpBN;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t tiles_sm = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* ctrl = smem_raw + (tiles_sm - smem_u32(smem_raw)) + S * kTcpStageBytes;
    const uint32_t full0 = smem_u32(ctrl);                                      // S: tile landed
    const uint32_t empty0 = full0 + 8u * S;                                     // S: tile consumed
    const uint32_t accf0 = empty0 + 8u * S;                                     // 2: accumulator complete
    const uint32_t acce0 = accf0 + 16u;                                         // 2: accumulator drained
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl + 8 * (2 * S + 4));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 8 * (2 * S + 4) + 8);
    volatile int* epi_ok = reinterpret_cast<volatile int*>(ctrl + 8 * (2 * S + 4) + 12);     // what the epilogue thread that waited found, for the other 127
    float* sw_s = reinterpret_cast<float*>(ctrl + kTcpCtrlBytes);               // [2][BN]
    float* wo_s = sw_s + 2 * BN;                                                // [BN][kTcpSide]

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int total_tiles = mtiles * ntiles;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(full0 + 8u * s, 1); mbar_init(empty0 + 8u * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(accf0 + 8u * b, 1); mbar_init(acce0 + 8u * b, 4); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2 * BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < total_tiles && ok; t += gridDim.x) {
                const int m0 = (t % mtiles) * kTcBM, n0 = (t / mtiles) * BN;
                for (int i = 0; i < kblocks; ++i, ++it) {
                    const uint32_t s = it % S, round = it / S;
                    ok = mbar_wait(empty0 + 8u * s, (round & 1u) ^ 1u, abort_flag, status, 1);
                    if (!ok) break;
                    const uint32_t a_dst = tiles_sm + s * kTcpStageBytes, b_dst = a_dst + kTcBM * kTcRowBytes;
                    mbar_expect_tx(full0 + 8u * s, kTcpStageBytes);
                    tma_load_2d(a_dst, &map_qx, i * 128, m0, full0 + 8u * s);
                    tma_load_2d(b_dst, &map_qw, i * 128, n0, full0 + 8u * s);
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            constexpr uint32_t idesc_i8 = umma_idesc(2, 1, kTcBM, BN);
            uint32_t it = 0, lt = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < total_tiles && ok; t += gridDim.x, ++lt) {
                const uint32_t buf = lt & 1u;
                ok = mbar_wait(acce0 + 8u * buf, ((lt >> 1) & 1u) ^ 1u, abort_flag, status, 4);    // the epilogue has drained this accumulator
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t d_tmem = tmem + buf * uint32_t(BN);
                for (int i = 0; i < kblocks; ++i, ++it) {
                    const uint32_t s = it % S, round = it / S;
                    ok = mbar_wait(full0 + 8u * s, round & 1u, abort_flag, status, 2);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t a_src = tiles_sm + s * kTcpStageBytes, b_src = a_src + kTcBM * kTcRowBytes;
                    const uint64_t adesc = umma_smem_desc(a_src), bdesc = umma_smem_desc(b_src);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        umma_i8(d_tmem, adesc + uint64_t(2 * k), bdesc + uint64_t(2 * k), idesc_i8, (i > 0 || k > 0) ? 1u : 0u);
                    umma_commit(empty0 + 8u * s);
                }
                if (ok) umma_commit(accf0 + 8u * buf);
            }
        }
        __syncwarp();
    } else {
        const int et = threadIdx.x - 64;
        const int quarter = warp & 3;
        const uint16_t* sxo = static_cast<const uint16_t*>(sidex);
        const uint16_t* swo = static_cast<const uint16_t*>(sidew);
        uint32_t lt = 0;
        bool ok = true;
        for (int t = blockIdx.x; t < total_tiles && ok; t += gridDim.x, ++lt) {
            const uint32_t buf = lt & 1u;
            const int m0 = (t % mtiles) * kTcBM, n0 = (t / mtiles) * BN;
            const int m = m0 + quarter * 32 + lane;
            // this tile's column scales and side columns; they are read while the MMAs of the tile still run
            float* sws = sw_s + buf * BN;
            for (int c = et; c < BN; c += 128) sws[c] = (n0 + c < N) ? sw[n0 + c] : 0.0f;
            float xo[kTcpSide];
#pragma unroll
            for (int j = 0; j < kTcpSide; ++j) xo[j] = 0.0f;
            if (ko > 0) {
                // side rows are at least 64 columns wide (128 bytes), so the first 16 columns are two aligned 16-byte loads
                for (int c = et; c < BN; c += 128) {
                    const int n = n0 + c;
                    float f[kTcpSide];
                    if (n < N) {
                        const uint4* src = reinterpret_cast<const uint4*>(swo + size_t(n) * side_cols);
                        float lo[8], hi[8];
                        widen8<XDT>(src[0], lo);
                        widen8<XDT>(src[1], hi);
#pragma unroll
                        for (int j = 0; j < 8; ++j) { f[j] = lo[j]; f[8 + j] = hi[j]; }
                    } else {
#pragma unroll
                        for (int j = 0; j < kTcpSide; ++j) f[j] = 0.0f;
                    }
#pragma unroll
                    for (int j = 0; j < kTcpSide; j += 4)
                        *reinterpret_cast<float4*>(wo_s + c * kTcpSide + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
                }
                if (m < M) {
                    const uint4* src = reinterpret_cast<const uint4*>(sxo + size_t(m) * side_cols);
                    float lo[8], hi[8];
                    widen8<XDT>(src[0], lo);
                    widen8<XDT>(src[1], hi);
#pragma unroll
                    for (int j = 0; j < 8; ++j) { xo[j] = lo[j]; xo[8 + j] = hi[j]; }
                }
            }
            const float sxm = (m < M) ? sx[m] : 0.0f;
            // one thread waits for the accumulator, with the bound; what it found reaches the other 127 through the
            // barrier that also publishes the scales above, so the four warps always take the same way
            if (et == 0) *epi_ok = mbar_wait(accf0 + 8u * buf, (lt >> 1) & 1u, abort_flag, status, 3) ? 1 : 0;
            asm volatile("bar.sync 1, 128;" ::: "memory");
            ok = (*epi_ok != 0);
            if (ok) (void)mbar_try(accf0 + 8u * buf, (lt >> 1) & 1u);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (ok) {
                const uint32_t lane_base = tmem + (uint32_t(quarter * 32) << 16) + buf * uint32_t(BN);
#pragma unroll 1
                for (int c0 = 0; c0 < BN; c0 += 32) {
                    uint32_t ai[32];
                    tmem_ld32(lane_base + uint32_t(c0), ai);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                    float out[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        float p = 0.0f;
                        if (ko > 0) {
                            const float4* wrow = reinterpret_cast<const float4*>(wo_s + (c0 + j) * kTcpSide);
#pragma unroll
                            for (int q = 0; q < kTcpSide / 4; ++q) {
                                if (q * 4 < ko) {
                                    const float4 wv = wrow[q];
                                    p = __fmaf_rn(xo[4 * q + 0], wv.x, p);
                                    p = __fmaf_rn(xo[4 * q + 1], wv.y, p);
                                    p = __fmaf_rn(xo[4 * q + 2], wv.z, p);
                                    p = __fmaf_rn(xo[4 * q + 3], wv.w, p);
                                }
                            }
                        }
                        out[j] = __fmaf_rn(float(int(ai[j])), __fmul_rn(sxm, sws[c0 + j]), p);
                    }
                    if (m < M) {
                        const int n = n0 + c0;
                        if constexpr (YDT == kF32) {
                            float* dst = static_cast<float*>(y) + size_t(m) * N + n;
#pragma unroll
                            for (int j = 0; j < 32; j += 4)
                                if (n + j < N) *reinterpret_cast<float4*>(dst + j) = make_float4(out[j], out[j + 1], out[j + 2], out[j + 3]);
                        } else {
                            uint16_t* dst = static_cast<uint16_t*>(y) + size_t(m) * N + n;
#pragma unroll
                            for (int j = 0; j < 32; j += 8) {
                                uint32_t pk[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if constexpr (YDT == kBF16) {
                                        const __nv_bfloat162 h = __floats2bfloat162_rn(out[j + 2 * e], out[j + 2 * e + 1]);
                                        pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                                    } else {
                                        const __half2 h = __floats2half2_rn(out[j + 2 * e], out[j + 2 * e + 1]);
                                        pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                                    }
                                }
                                if (n + j < N) *reinterpret_cast<uint4*>(dst + j) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                            }
                        }
                    }
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(acce0 + 8u * buf);         // this warp's quarter of the accumulator is free again
            }
            asm volatile("bar.sync 2, 128;" ::: "memory");             // wo_s is rewritten for the next tile
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }

    __syncthreads();
    if (*abort_flag) {
        for (int i = 0; i < 64; ++i) __nanosleep(2000);
        __syncthreads();
    }
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN) : "memory");
    }
}


// ------------------------------------------------------------------------------------------
// gemm_tc2: persistent kernel on CTA pairs (clusters of two, tcgen05 cta_group::2).
//
// The two SMs of a TPC share a 256 x 256 tile: each CTA loads its own 128 activation rows and
// only HALF of the weight rows (32 KB per K step of 128 features instead of 48 KB), and one
// thread of the even CTA issues MMAs of shape 256 x 256 x 32 that read both halves from the
// two shared memories and write each CTA's 128 rows into that CTA's own tensor memory.
// Otherwise as gemm_tcp: a ring (6 stages here), two accumulators per CTA, epilogue under the
// next tile's MMAs, side features by ordered fp32 FMAs.
//
// Barriers: "tile landed" lives in the even CTA and counts the bytes of both CTAs' loads (the
// odd CTA's TMA loads name the even CTA's barrier); "stage free" and "accumulator complete"
// are signalled in both CTAs by one multicast tcgen05.commit; "accumulator drained" lives in
// the even CTA and takes one arrival per epilogue warp of both CTAs.  No load is multicast.

constexpr int kPairStages = 3;
constexpr int kPairStepBlocks = 2;                                            // K blocks of 128 features one TMA load brings
constexpr uint32_t kPairSlabBytes = 128 * kTcRowBytes;                        // 128 rows x 128 features
constexpr uint32_t kPairHalfBytes = kPairStepBlocks * kPairSlabBytes;         // a stage's activations, or its weights
constexpr uint32_t kPairStageBytes = 2 * kPairHalfBytes;
constexpr uint32_t kPairSmemBytes = kPairStages * kPairStageBytes + 1024 + kTcpCtrlBytes + kTcpSwBytes + kTcpWoBytes;

__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// one load of a [K blocks][rows][128 bytes] box from a map that views the matrix as (128 bytes, rows, K / 128)
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int row, int kblock, uint32_t bar_cluster_addr) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(0), "r"(row), "r"(kblock), "r"(bar_cluster_addr) : "memory");
}
__device__ __forceinline__ void umma_i8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives on the barrier at this shared address in both CTAs of the pair once the MMAs issued so far are done
__device__ __forceinline__ void umma_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(uint16_t(3)) : "memory");
}

// Low-rank adapters of the rows (mmd_linear_adapted) in this kernel's epilogue: sum_j v_j B[n][j] is added to the outputs in fp32 before they
// are rounded, with v_j = scale u_j, u the sums over the chunks that the kernel before left.  A thread has a row; of the tile's 256 columns
// two (adapter, 16 ranks) pieces of B lie in shared memory as they are, 8 KB each, read by broadcast: those of the tile's first two
// adapters (rank 16), or both of the first one's (rank 32).  Rows of further adapters, where a tile has them, read B from global
// memory.  Fused multiply-adds on two columns at a time, hidden under the next tile's products (mma.sync is not: its products wait
// behind the tcgen05 ones that fill the pipe; 4900 x 6144 -> 16384 took twice as long with it).
struct AdaptArgs {
    const uint16_t* b;                     // [adapters][N][rank]
    const float* scale;                    // [adapters]
    const float* u;                        // [chunks][M][rank]
    const int32_t* row_id;                 // [M]: the rows' adapters, -1: none
    int rank, chunks;                      // rank 16 or 32
    size_t u_stride;                       // M rank
};
constexpr int kFusedRank = 32;
constexpr int kAdaptEpilogue = 256;                                             // epilogue threads: two for every row, half of the columns each
constexpr uint32_t kAdaptSlotBytes = kTcpBN * 16 * 2;
constexpr uint32_t kAdaptBytes = 2 * kAdaptSlotBytes + 128 * 4;                 // the two pieces, the rows' adapters
constexpr uint32_t kAdaptWoBytes = kTcpBN * kTcpSide * 2;                       // side columns as they are, to make room

// out[c] += sum_j v[j] B[c][j] of eight columns, their 16 ranks `pitch` bytes apart, from shared or global memory.  One warp has a scheduler to
// itself here, so the eight sums go on side by side.
template <int XDT, bool SHARED>
__device__ __forceinline__ void add_ranks16(float (&out)[8], const float (&v)[16], const unsigned char* b, size_t pitch) {
    uint64_t o[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = rq_pack2(out[2 * c], out[2 * c + 1]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint4 w[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const uint4* p = reinterpret_cast<const uint4*>(b + size_t(c) * pitch) + h;
            w[c] = SHARED ? *p : __ldg(p);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {                                   // words of two ranks
            uint64_t v0 = rq_pack2(v[8 * h + 2 * i], v[8 * h + 2 * i]), v1 = rq_pack2(v[8 * h + 2 * i + 1], v[8 * h + 2 * i + 1]);
            float lo[8], hi[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const uint32_t x = i == 0 ? w[c].x : i == 1 ? w[c].y : i == 2 ? w[c].z : w[c].w;
                lo[c] = widen16<XDT>(x & 0xffffu);
                hi[c] = widen16<XDT>(x >> 16);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = rq_fma2(v0, rq_pack2(lo[2 * c], lo[2 * c + 1]), o[c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = rq_fma2(v1, rq_pack2(hi[2 * c], hi[2 * c + 1]), o[c]);
        }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        out[2 * c] = __uint_as_float(uint32_t(o[c]));
        out[2 * c + 1] = __uint_as_float(uint32_t(o[c] >> 32));
    }
}

template <int XDT>
struct TileAdapter {
    int mine;                              // this thread's row's adapter
    int slot;                              // its first piece in shared memory, or -1
    float v[2][16];
    // The epilogue threads together: pieces into shared memory (published by the barrier behind the wait for the accumulator), this row's
    // values.
    __device__ __forceinline__ void begin(const AdaptArgs& ad, int et, int m, int row /* of the tile */, int M, int n0, int N, unsigned char* pieces) {
        int* ids = reinterpret_cast<int*>(pieces + 2 * kAdaptSlotBytes);
        mine = m < M ? __ldcg(ad.row_id + m) : -1;                     // (from L2: what other kernels of the call have written)
        if (et < 128) ids[row] = mine;
        asm volatile("bar.sync 3, %0;" ::"n"(kAdaptEpilogue) : "memory");
        int of[4], two[2] = {-1, -1};
#pragma unroll
        for (int k = 0; k < 4; ++k) of[k] = ids[32 * k + (et & 31)];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 3; k >= 0; --k) {                              // the lowest row wins
                const unsigned has = __ballot_sync(0xffffffffu, of[k] >= 0 && (i == 0 || of[k] != two[0]));
                const int id = __shfl_sync(0xffffffffu, of[k], has ? __ffs(has) - 1 : 0);
                if (has) two[i] = id;
            }
        const bool wide = ad.rank > 16;
        slot = mine < 0 ? -1 : mine == two[0] ? 0 : !wide && mine == two[1] ? 1 : -1;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int id = wide ? two[0] : two[i], j0 = wide ? 16 * i : 0;
            if (id < 0) continue;
            for (int c = et; c < kTcpBN; c += kAdaptEpilogue) {
                uint4 w[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
                if (n0 + c < N) {
                    const uint4* p = reinterpret_cast<const uint4*>(ad.b + (size_t(id) * size_t(N) + size_t(n0 + c)) * ad.rank + j0);
                    w[0] = __ldg(p);
                    w[1] = __ldg(p + 1);
                }
                uint4* to = reinterpret_cast<uint4*>(pieces + i * kAdaptSlotBytes + c * 32);
                to[0] = w[0];
                to[1] = w[1];
            }
        }
        const float scale = mine >= 0 ? __ldg(ad.scale + mine) : 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[i][j] = 0.0f;
            if (mine < 0 || (i == 1 && !wide)) continue;
            for (int k = 0; k < ad.chunks; ++k) {
                const float4* p = reinterpret_cast<const float4*>(ad.u + size_t(k) * ad.u_stride + size_t(m) * ad.rank + 16 * i);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 f = __ldcg(p + q);
                    v[i][4 * q] += f.x; v[i][4 * q + 1] += f.y; v[i][4 * q + 2] += f.z; v[i][4 * q + 3] += f.w;
                }
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) v[i][j] = __fmul_rn(scale, v[i][j]);
        }
    }
    // columns c0 .. c0 + 7 of the tile, which exist (N is a multiple of 8); the caller's warp meets behind it
    __device__ __forceinline__ void add(const AdaptArgs& ad, int c0, int n0, int N, const unsigned char* pieces, float (&out)[8]) const {
        if (mine < 0) return;
        if (slot >= 0) {
            add_ranks16<XDT, true>(out, v[0], pieces + slot * kAdaptSlotBytes + c0 * 32, 32);
            if (ad.rank > 16) add_ranks16<XDT, true>(out, v[1], pieces + kAdaptSlotBytes + c0 * 32, 32);
        } else {
            const unsigned char* p = reinterpret_cast<const unsigned char*>(ad.b + (size_t(mine) * size_t(N) + size_t(n0 + c0)) * ad.rank);
            add_ranks16<XDT, false>(out, v[0], p, size_t(ad.rank) * 2);
            if (ad.rank > 16) add_ranks16<XDT, false>(out, v[1], p + 32, size_t(ad.rank) * 2);
        }
    }
};

template <bool ADAPT> struct PairCfg {                                            // of gemm_tc2
    static constexpr int kThreads = ADAPT ? 64 + kAdaptEpilogue : kTcThreads;
    static constexpr uint32_t kSmem = ADAPT ? kPairSmemBytes - kTcpWoBytes + kAdaptWoBytes + kAdaptBytes : kPairSmemBytes;
};
static_assert(PairCfg<true>::kSmem <= 227 * 1024, "fits an SM");

// Scales and side columns of one tile's 256 weight rows into shared memory, and this thread's
// own activation row's side values into registers (epilogue threads, et = 0..127).
template <int XDT, bool RAW /* side columns as they are */, int THREADS>
__device__ __forceinline__ void stage_tile_side(int et, int n0, int N, int m, int M, int ko, int side_cols, const float* __restrict__ sw,
                                                const uint16_t* __restrict__ sxo, const uint16_t* __restrict__ swo, float* sws, float* wo_s,
                                                float (&xo)[kTcpSide]) {
    for (int c = et; c < kTcpBN; c += THREADS) sws[c] = (n0 + c < N) ? sw[n0 + c] : 0.0f;
#pragma unroll
    for (int j = 0; j < kTcpSide; ++j) xo[j] = 0.0f;
    if (ko > 0) {
        for (int c = et; c < kTcpBN; c += THREADS) {
            const int n = n0 + c;
            if constexpr (RAW) {
                uint4 w[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
                if (n < N) {
                    const uint4* src = reinterpret_cast<const uint4*>(swo + size_t(n) * side_cols);
                    w[0] = src[0];
                    w[1] = src[1];
                }
                uint4* to = reinterpret_cast<uint4*>(wo_s) + 2 * c;
                to[0] = w[0];
                to[1] = w[1];
                continue;
            }
            float f[kTcpSide];
            if (n < N) {
                const uint4* src = reinterpret_cast<const uint4*>(swo + size_t(n) * side_cols);
                float lo[8], hi[8];
                widen8<XDT>(src[0], lo);
                widen8<XDT>(src[1], hi);
#pragma unroll
                for (int j = 0; j < 8; ++j) { f[j] = lo[j]; f[8 + j] = hi[j]; }
            } else {
#pragma unroll
                for (int j = 0; j < kTcpSide; ++j) f[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < kTcpSide; j += 4)
                *reinterpret_cast<float4*>(wo_s + c * kTcpSide + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
        }
        if (m < M) {
            const uint4* src = reinterpret_cast<const uint4*>(sxo + size_t(m) * side_cols);
            float lo[8], hi[8];
            widen8<XDT>(src[0], lo);
            widen8<XDT>(src[1], hi);
#pragma unroll
            for (int j = 0; j < 8; ++j) { xo[j] = lo[j]; xo[8 + j] = hi[j]; }
        }
    }
}

// One accumulator row of 256 int32 sums -> scaled, side part added, narrowed, stored.
template <int YDT>
__device__ __forceinline__ void drain_row(uint32_t lane_base, float sxm, const float* sws, const float* wo_s, const float (&xo)[kTcpSide], int ko,
                                          void* __restrict__ y, int m, int M, int n0, int N) {
#pragma unroll 1
    for (int c0 = 0; c0 < kTcpBN; c0 += 32) {
        uint32_t ai[32];
        tmem_ld32(lane_base + uint32_t(c0), ai);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        float out[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            float p = 0.0f;
            if (ko > 0) {
                const float4* wrow = reinterpret_cast<const float4*>(wo_s + (c0 + j) * kTcpSide);
#pragma unroll
                for (int q = 0; q < kTcpSide / 4; ++q) {
                    if (q * 4 < ko) {
                        const float4 wv = wrow[q];
                        p = __fmaf_rn(xo[4 * q + 0], wv.x, p);
                        p = __fmaf_rn(xo[4 * q + 1], wv.y, p);
                        p = __fmaf_rn(xo[4 * q + 2], wv.z, p);
                        p = __fmaf_rn(xo[4 * q + 3], wv.w, p);
                    }
                }
            }
            out[j] = __fmaf_rn(float(int(ai[j])), __fmul_rn(sxm, sws[c0 + j]), p);
        }
        if (m < M) {
            const int n = n0 + c0;
            if constexpr (YDT == kF32) {
                float* dst = static_cast<float*>(y) + size_t(m) * N + n;
#pragma unroll
                for (int j = 0; j < 32; j += 4)
                    if (n + j < N) *reinterpret_cast<float4*>(dst + j) = make_float4(out[j], out[j + 1], out[j + 2], out[j + 3]);
            } else {
                uint16_t* dst = static_cast<uint16_t*>(y) + size_t(m) * N + n;
#pragma unroll
                for (int j = 0; j < 32; j += 8) {
                    uint32_t pk[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (YDT == kBF16) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(out[j + 2 * e], out[j + 2 * e + 1]);
                            pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                        } else {
                            const __half2 h = __floats2half2_rn(out[j + 2 * e], out[j + 2 * e + 1]);
                            pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                    }
                    if (n + j < N) *reinterpret_cast<uint4*>(dst + j) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                }
            }
        }
    }
}

// The same with the rows' adapters, eight columns at a time.
template <int XDT, int YDT>
__device__ __forceinline__ void drain_row_adapted(uint32_t lane_base, float sxm, const float* sws, const uint4* wo_s, const float (&xo)[kTcpSide], int ko,
                                                  void* __restrict__ y, int m, int M, int n0, int N, const AdaptArgs& ad, const TileAdapter<XDT>& ta,
                                                  const unsigned char* pieces, int first, int last /* columns */) {
#pragma unroll 1
    for (int c0 = first; c0 < last; c0 += 8) {
        uint32_t ai[8];
        tmem_ld8(lane_base + uint32_t(c0), ai);
        float p[8] = {};
        if (ko > 0) {
#pragma unroll
            for (int q = 0; q < kTcpSide / 8; ++q) {
                if (q * 8 < ko) {
                    uint4 w[8];
#pragma unroll
                    for (int c = 0; c < 8; ++c) w[c] = wo_s[2 * (c0 + c) + q];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const uint32_t x = i == 0 ? w[c].x : i == 1 ? w[c].y : i == 2 ? w[c].z : w[c].w;
                                p[c] = __fmaf_rn(xo[8 * q + 2 * i + e], widen16<XDT>(e ? x >> 16 : x & 0xffffu), p[c]);
                            }
                }
            }
        }
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        float out[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) out[c] = __fmaf_rn(float(int(ai[c])), __fmul_rn(sxm, sws[c0 + c]), p[c]);
        if (n0 + c0 < N) ta.add(ad, c0, n0, N, pieces, out);
        if (m < M && n0 + c0 < N) {
            if constexpr (YDT == kF32) {
                float4* dst = reinterpret_cast<float4*>(static_cast<float*>(y) + size_t(m) * N + n0 + c0);
                dst[0] = make_float4(out[0], out[1], out[2], out[3]);
                dst[1] = make_float4(out[4], out[5], out[6], out[7]);
            } else {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (YDT == kBF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[e]) : "f"(out[2 * e + 1]), "f"(out[2 * e]));
                    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[e]) : "f"(out[2 * e + 1]), "f"(out[2 * e]));
                }
                *reinterpret_cast<uint4*>(static_cast<uint16_t*>(y) + size_t(m) * N + n0 + c0) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        __syncwarp();
    }
}

template <int XDT, int YDT, bool ADAPT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairCfg<ADAPT>::kThreads, 1)
gemm_tc2(const __grid_constant__ CUtensorMap map_qx, const __grid_constant__ CUtensorMap map_qw /* boxes of 128 weight rows */,
         const float* __restrict__ sx, const float* __restrict__ sw, const void* __restrict__ sidex, const void* __restrict__ sidew,
         int side_cols, int ko, void* __restrict__ y, int M, int N, int kblocks, int mpairs /* tiles of 256 rows */, int ntiles, int* status,
         const __grid_constant__ AdaptArgs ad) {
    constexpr int S = kPairStages, EPI = PairCfg<ADAPT>::kThreads - 64;            // epilogue threads
    constexpr int BN = kTcpBN;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t tiles_sm = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* ctrl = smem_raw + (tiles_sm - smem_u32(smem_raw)) + S * kPairStageBytes;
    const uint32_t full0 = smem_u32(ctrl);                                      // S: tile landed (used in the even CTA)
    const uint32_t empty0 = full0 + 8u * S;                                     // S: stage free
    const uint32_t accf0 = empty0 + 8u * S;                                     // 2: accumulator complete
    const uint32_t acce0 = accf0 + 16u;                                         // 2: accumulator drained (used in the even CTA)
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl + 8 * (2 * S + 4));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 8 * (2 * S + 4) + 8);
    volatile int* epi_ok = reinterpret_cast<volatile int*>(ctrl + 8 * (2 * S + 4) + 12);
    float* sw_s = reinterpret_cast<float*>(ctrl + kTcpCtrlBytes);               // [2][BN]
    float* wo_s = sw_s + 2 * BN;                                                // [BN][kTcpSide]
    [[maybe_unused]] unsigned char* const pieces = reinterpret_cast<unsigned char*>(wo_s) + kAdaptWoBytes;      // of adapters

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
    const int total_tiles = mpairs * ntiles;
    const int ksteps = (kblocks + kPairStepBlocks - 1) / kPairStepBlocks;      // ring steps per tile

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(full0 + 8u * s, 1); mbar_init(empty0 + 8u * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(accf0 + 8u * b, 1); mbar_init(acce0 + 8u * b, 2 * EPI / 32); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2 * BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                                          // both CTAs' barriers exist before either signals the other
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int t = pair; t < total_tiles && ok; t += npairs) {
                const int m0 = (t % mpairs) * 256 + int(rank) * 128;             // this CTA's activation rows
                const int nb0 = (t / mpairs) * BN + int(rank) * 128;             // this CTA's half of the weight rows
                for (int i = 0; i < ksteps; ++i, ++it) {
                    const uint32_t s = it % S, round = it / S;
                    ok = mbar_wait(empty0 + 8u * s, (round & 1u) ^ 1u, abort_flag, status, 1);
                    if (!ok) break;
                    const uint32_t a_dst = tiles_sm + s * kPairStageBytes, b_dst = a_dst + kPairHalfBytes;
                    const uint32_t full_even = map_to_cta(full0 + 8u * s, 0);
                    if (rank == 0) mbar_expect_tx(full0 + 8u * s, 2 * kPairStageBytes);      // both CTAs' bytes
                    tma_load_3d_pair(a_dst, &map_qx, m0, i * kPairStepBlocks, full_even);     // a K block past the end reads as zeros
                    tma_load_3d_pair(b_dst, &map_qw, nb0, i * kPairStepBlocks, full_even);
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            constexpr uint32_t idesc_i8 = umma_idesc(2, 1, 256, BN);
            uint32_t it = 0, lt = 0;
            bool ok = true;
            for (int t = pair; t < total_tiles && ok; t += npairs, ++lt) {
                const uint32_t buf = lt & 1u;
                ok = mbar_wait(acce0 + 8u * buf, ((lt >> 1) & 1u) ^ 1u, abort_flag, status, 4);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t d_tmem = tmem + buf * uint32_t(BN);
                for (int i = 0; i < ksteps; ++i, ++it) {
                    const uint32_t s = it % S, round = it / S;
                    ok = mbar_wait(full0 + 8u * s, round & 1u, abort_flag, status, 2);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t a_src = tiles_sm + s * kPairStageBytes, b_src = a_src + kPairHalfBytes;
#pragma unroll
                    for (int j = 0; j < kPairStepBlocks; ++j) {
                        const uint64_t adesc = umma_smem_desc(a_src + uint32_t(j) * kPairSlabBytes), bdesc = umma_smem_desc(b_src + uint32_t(j) * kPairSlabBytes);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            umma_i8_pair(d_tmem, adesc + uint64_t(2 * k), bdesc + uint64_t(2 * k), idesc_i8, (i > 0 || j > 0 || k > 0) ? 1u : 0u);
                    }
                    umma_commit_pair(empty0 + 8u * s);
                }
                if (ok) umma_commit_pair(accf0 + 8u * buf);
            }
        }
        __syncwarp();
    } else {
        const int et = threadIdx.x - 64;
        const int quarter = warp & 3;
        const uint16_t* sxo = static_cast<const uint16_t*>(sidex);
        const uint16_t* swo = static_cast<const uint16_t*>(sidew);
        uint32_t lt = 0;
        bool ok = true;
        for (int t = pair; t < total_tiles && ok; t += npairs, ++lt) {
            const uint32_t buf = lt & 1u;
            const int m0 = (t % mpairs) * 256 + int(rank) * 128, n0 = (t / mpairs) * BN;
            const int m = m0 + quarter * 32 + lane;
            float* sws = sw_s + buf * BN;
            float xo[kTcpSide];
            stage_tile_side<XDT, ADAPT, EPI>(et, n0, N, m, M, ko, side_cols, sw, sxo, swo, sws, wo_s, xo);
            const float sxm = (m < M) ? sx[m] : 0.0f;
            [[maybe_unused]] TileAdapter<XDT> ta;
            if constexpr (ADAPT) ta.begin(ad, et, m, quarter * 32 + lane, M, n0, N, pieces);
            if (et == 0) *epi_ok = mbar_wait(accf0 + 8u * buf, (lt >> 1) & 1u, abort_flag, status, 3) ? 1 : 0;
            asm volatile("bar.sync 1, %0;" ::"n"(EPI) : "memory");
            ok = (*epi_ok != 0);
            if (ok) (void)mbar_try(accf0 + 8u * buf, (lt >> 1) & 1u);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (ok) {
                const uint32_t lane_base = tmem + (uint32_t(quarter * 32) << 16) + buf * uint32_t(BN);
                if constexpr (ADAPT) drain_row_adapted<XDT, YDT>(lane_base, sxm, sws, reinterpret_cast<const uint4*>(wo_s), xo, ko, y, m, M, n0, N, ad, ta, pieces,
                                                                    et < 128 ? 0 : BN / 2, et < 128 ? BN / 2 : BN);
                else drain_row<YDT>(lane_base, sxm, sws, wo_s, xo, ko, y, m, M, n0, N);
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_cta(acce0 + 8u * buf, 0));
            }
            asm volatile("bar.sync 2, %0;" ::"n"(EPI) : "memory");
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }

    __syncthreads();
    if (*abort_flag) {
        for (int i = 0; i < 64; ++i) __nanosleep(2000);
        __syncthreads();
    }
    cluster_sync_all();                                                          // neither CTA leaves while the other may still signal it
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN) : "memory");
    }
}

}  // namespace mmdk
