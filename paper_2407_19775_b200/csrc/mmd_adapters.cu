// mmd_adapters.cu -- low-rank adapters of many sequences beside a shared decomposed projection (sm_100a):
//
//     y_r = (the decomposed layer's row, in fp32) + scale_a (x_r A_a^T) B_a^T,   a the adapter of row r's sequence
//
// u = x A^T, few numbers per row, by `shrink` in front of the layer's product; the rest by `expand_rows` or `expand_tiles` behind it, which add
// to the layer's fp32 rows, or by the CTA-pair product itself (TileAdapter in mmd_kernels.cuh).  A decode step reads every adapter in use
// once (rank (K + N) 16-bit numbers each, 0.5 MB at rank 16 and 8192 features).
#include "mmd_adapters.h"

#include "bqkv_launch.h"
#include "mmd_elements.cuh"

namespace mmda {

namespace {

using mmdk::kBF16;
using mmdk::kF16;
using mmdk::kF32;

// Starts and ids are read from L2: shrink reads them before its wait for the kernels in front too, and behind it a line that lies in L1 from there
// would be the old one.  So are the rows and what the kernels of a call hand on to one another, which an SM reads once.
// The sequence of row r, found by the whole warp.
__device__ __forceinline__ int sequence_of(const Adapters& ad, int r) {
    return ad.starts ? bqkvk::last_begun(r, ad.n_seq, [&](int i) { return __ldcg(ad.starts + i); }) : r;
}
// The adapter of row r if it lies in sequence s, else -1; `in`: whether it does.
__device__ __forceinline__ int adapter_in(const Adapters& ad, int s, int r, bool& in) {
    const int id = __ldcg(ad.ids + s);
    in = !ad.starts || (__ldcg(ad.starts + s) <= r && r < __ldcg(ad.starts + s + 1));
    return in && id >= 0 && id < ad.count ? id : -1;
}
// The adapters of rows r0 + lane, from the sequence of the first of them on; rows from M on have none.
__device__ __forceinline__ int adapters_from(const Adapters& ad, int r0, int M) {
    const int r = r0 + int(threadIdx.x & 31);
    int s = sequence_of(ad, r0);
    if (!ad.starts) s = min(r, M - 1);
    else while (s + 1 < ad.n_seq && __ldcg(ad.starts + s + 1) <= r) ++s;
    bool in;
    const int id = adapter_in(ad, s, r, in);
    return r < M ? id : -1;
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

// Four numbers as two 16-bit parts: the pairs' first parts, then what they leave.
template <int XDT>
__device__ __forceinline__ uint4 two_parts(const float4& f) {
    uint4 w;
    if constexpr (XDT == kBF16) {
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.x) : "f"(f.y), "f"(f.x));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.y) : "f"(f.w), "f"(f.z));
        const float a = f.x - __uint_as_float(w.x << 16), b = f.y - __uint_as_float(w.x & 0xffff0000u);
        const float c = f.z - __uint_as_float(w.y << 16), d = f.w - __uint_as_float(w.y & 0xffff0000u);
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.z) : "f"(b), "f"(a));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.w) : "f"(d), "f"(c));
    } else {
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w.x) : "f"(f.y), "f"(f.x));
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w.y) : "f"(f.w), "f"(f.z));
        const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w.x)), q = __half22float2(*reinterpret_cast<const __half2*>(&w.y));
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w.z) : "f"(f.y - p.y), "f"(f.x - p.x));
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w.w) : "f"(f.w - q.y), "f"(f.z - q.x));
    }
    return w;
}

// Eight elements of the normed row as two 16-bit parts: the elements rounded, and what that leaves, rounded.  (The products take 16-bit operands; the
// first part alone, 2^-8 or 2^-11 of an element, was the largest error of fp32 outputs.  4900 rows of 6144, rank 16, cold 40 -> 44 us.)
template <int DT>
__device__ __forceinline__ void normed(uint4 h, uint4 g, float rms, uint4& first, uint4& rest) {
    float f[8], w[8];
    mmdk::widen8<DT>(h, f);
    mmdk::widen8<DT>(g, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __fmul_rn(__fmul_rn(f[i], w[i]), rms);
    const uint4 p = two_parts<DT>(make_float4(f[0], f[1], f[2], f[3])), q = two_parts<DT>(make_float4(f[4], f[5], f[6], f[7]));
    first = make_uint4(p.x, p.y, q.x, q.y);
    rest = make_uint4(p.z, p.w, q.z, q.w);
}

// ------------------------------------------------------------------------------------------
// shrink: u^T = A x^T by mma.sync m16n8k16: 16 ranks are the 16 rows, up to 8 rows of the call the 8 columns (tcgen05 has no shape this
// small, and the products are not what bounds it).  The order of k within a product does not matter as long as both operands have
// the same, so a lane takes eight consecutive features, 16 bytes, of its adapter row and of its activation row.
// A CTA has `rows` rows of the call and a chunk of the features; its warps share the chunk's steps of 32 and are added in order.  Up to
// 16 RT ranks go together, so that the rows are read once for them.  Measured, cold caches: 64 rows of 8192 with 38 adapters of rank 16 9.3 us
// (10 MB of A, and 10 of B asked for), 1224 rows of 2048 with 9 of rank 64 18.2 us (bound by the latency of lookups and loads: two steps a warp),
// 4900 rows of 6144 normed on the way, rank 16, 44 us (60 MB, 1.4 TB/s: norming, per element, is what a warp does most of the time).
constexpr int kShrinkThreads = 256, kShrinkWarps = kShrinkThreads / 32;

template <int DT, int NT /* times 8 rows */, int RT /* times 16 ranks */, bool NORM>
__global__ void __launch_bounds__(kShrinkThreads)
shrink(const Input in, const Adapters ad, int rows, float* __restrict__ u, int32_t* __restrict__ row_id) {
    __shared__ int id_of[32];
    __shared__ float red[kShrinkWarps][RT][NT][4][32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int r0 = int(blockIdx.x) * rows, nr = min(rows, in.M - r0);
    const int steps = (in.K + 31) / 32, s0 = int((long long)steps * blockIdx.y / gridDim.y), s1 = int((long long)steps * (blockIdx.y + 1) / gridDim.y);
    [[maybe_unused]] int early = 0;
    if (NT == 1 && rows == 1 && wid == 0) {
        // Under the kernel before: the row's sequence (checked again below), and this CTA's share of its adapter from memory into L2.  (Ids
        // that earlier kernels are still writing would only ask for another adapter.)
        early = sequence_of(ad, r0);
        bool mine;
        const int id = adapter_in(ad, early, r0, mine);
        if (id >= 0) {
            const uint32_t bytes = uint32_t(min(in.K, 32 * s1) - 32 * s0) * 2u;
            for (int j = lane; j < ad.rank; j += 32)
                asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(ad.a + (size_t(id) * ad.rank + j) * in.K + 32 * s0), "r"(bytes) : "memory");
            const size_t all = size_t(in.N) * ad.rank / 8;                // of b, in pieces of 16 bytes
            const size_t b0 = all * blockIdx.y / gridDim.y, b1 = all * (blockIdx.y + 1) / gridDim.y, each = (b1 - b0 + 31) / 32;
            const size_t from = b0 + each * lane, upto = min(from + each, b1);
            if (from < upto)
                asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(ad.b + size_t(id) * size_t(in.N) * ad.rank + from * 8), "r"(uint32_t(upto - from) * 16u) : "memory");
        }
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    if (wid == 0) {
        int id;
        if (NT == 1 && rows == 1) {
            bool same;
            id = adapter_in(ad, early, r0, same);
            if (!same) id = adapter_in(ad, sequence_of(ad, r0), r0, same);
            if (lane > 0) id = -1;
        } else {
            id = adapters_from(ad, r0, in.M);
            if (lane >= nr) id = -1;
        }
        id_of[lane] = id;
        if (lane < nr && blockIdx.y == 0) row_id[r0 + lane] = id;
    }
    __syncthreads();
    const int w0 = s0 + (s1 - s0) * wid / kShrinkWarps, w1 = s0 + (s1 - s0) * (wid + 1) / kShrinkWarps;
    float* const to = u + size_t(blockIdx.y) * in.M * ad.rank;
    const int all_ids = id_of[lane];
    for (unsigned todo = __ballot_sync(0xffffffffu, all_ids >= 0); todo;) {
        const int id = __shfl_sync(0xffffffffu, all_ids, __ffs(todo) - 1);
        const unsigned mask = __ballot_sync(0xffffffffu, all_ids == id);
        todo &= ~mask;
        const uint16_t* x[NT];
        float rms[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const bool mine = (mask >> (8 * n + g)) & 1u;
            x[n] = mine ? in.x + size_t(r0 + 8 * n + g) * in.K + 8 * t : nullptr;
            rms[n] = NORM && mine ? __ldcg(in.rms + r0 + 8 * n + g) : 0.0f;
        }
        for (int j0 = 0; j0 < ad.rank; j0 += 16 * RT) {
            const uint16_t* a0 = ad.a + (size_t(id) * ad.rank + j0 + g) * in.K + 8 * t;
            float acc[RT][NT][4] = {};
#pragma unroll(RT == 1 ? 4 : 2)
            for (int s = w0; s < w1; ++s) {
                const int k = 32 * s;
                const bool there = k + 8 * t < in.K;                    // K is a multiple of 16
                const uint4 zero = make_uint4(0, 0, 0, 0);
                uint4 p[RT], q[RT];
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const bool have = there && j0 + 16 * i < ad.rank;
                    p[i] = have ? __ldg(reinterpret_cast<const uint4*>(a0 + size_t(16 * i) * in.K + k)) : zero;
                    q[i] = have ? __ldg(reinterpret_cast<const uint4*>(a0 + size_t(16 * i + 8) * in.K + k)) : zero;
                }
                uint4 gm = zero;
                if (NORM && there) gm = __ldg(reinterpret_cast<const uint4*>(in.gamma + k + 8 * t));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint4 v = there && x[n] ? __ldcg(reinterpret_cast<const uint4*>(x[n] + k)) : zero;
                    [[maybe_unused]] uint4 rest;
                    if constexpr (NORM) normed<DT>(v, gm, rms[n], v, rest);
#pragma unroll
                    for (int i = 0; i < RT; ++i) {
                        mma16<DT>(acc[i][n], p[i].x, q[i].x, p[i].y, q[i].y, v.x, v.y);
                        mma16<DT>(acc[i][n], p[i].z, q[i].z, p[i].w, q[i].w, v.z, v.w);
                        if constexpr (NORM) {
                            mma16<DT>(acc[i][n], p[i].x, q[i].x, p[i].y, q[i].y, rest.x, rest.y);
                            mma16<DT>(acc[i][n], p[i].z, q[i].z, p[i].w, q[i].w, rest.z, rest.w);
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 4; ++c) red[wid][i][n][c][lane] = acc[i][n][c];
            __syncthreads();
            // fragment element c of lane l: rank (l >> 2) + 8 (c >> 1), row 2 (l & 3) + (c & 1)
            for (int i = threadIdx.x; i < 8 * NT * 16 * RT; i += kShrinkThreads) {
                const int j = i % (16 * RT), row = i / (16 * RT), n = row >> 3, l = (j & 7) * 4 + ((row & 7) >> 1), c = ((j >> 3) & 1) * 2 + (row & 1);
                if (!((mask >> row) & 1u) || j0 + j >= ad.rank) continue;
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < kShrinkWarps; ++w) sum += red[w][j >> 4][n][c][l];
                to[size_t(r0 + row) * ad.rank + j0 + j] = sum;
            }
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------------------------------------
// Four numbers as three bf16 parts, all of fp32's bits.
__device__ __forceinline__ void three_parts(const float4& f, uint2 (&part)[3]) {
    float x[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(part[i].x) : "f"(x[1]), "f"(x[0]));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(part[i].y) : "f"(x[3]), "f"(x[2]));
        x[0] -= __uint_as_float(part[i].x << 16); x[1] -= __uint_as_float(part[i].x & 0xffff0000u);
        x[2] -= __uint_as_float(part[i].y << 16); x[3] -= __uint_as_float(part[i].y & 0xffff0000u);
    }
}

// ------------------------------------------------------------------------------------------
// expand_tiles: a warp has 16 rows by 32 columns, a CTA 32 by 128; V B^T by mma.sync m16n8k16, V = scale u in two 16-bit parts, which the CTA
// leaves in shared memory first: bf16 16 bits, which outputs of 8 bits do not show; fp16 22 bits, after a power of two that takes the row's
// largest to 2^14 (V may leave fp16's range; what is 2^-39 of the row's largest is lost).  fp32 outputs of bf16 layers: fp32 in shared memory, all of
// whose bits go into three parts on the way to the products.  The rows' distinct adapters take turns, the others' rows zero meanwhile.  A
// thread loads four consecutive ranks (8 bytes) of B and of both parts of V (16 bytes); which ranks meet in a product does not matter as long as both
// sides agree.  Columns are dealt to the products so that a thread ends with four neighbours of a row: column 16 p + 4 t + 2 e + j is column
// 2 t + j of product 2 p + e.  Measured, 1224 rows x 2312, 9 adapters of rank 64, fp16, cold caches 18.8 us for 19 MB; 64 columns a warp 21.1, and with
// tf32 parts besides 24.2.  Bound by the latency of what a CTA reads in turn: lookups, partial sums, B.
constexpr int kExpandThreads = 256, kExpandRows = 32, kExpandCols = 128, kExpandWarpCols = 32;

template <int DT, int YDT>
__global__ void __launch_bounds__(kExpandThreads, 3)
expand_tiles(const Adapters ad, int M, int N, int chunks, const float* __restrict__ u, const int32_t* __restrict__ row_id, const float* y32, int ld, void* y) {
    constexpr int P = kExpandWarpCols / 16, B = 2 * P;                  // groups of 16 columns, products of 8
    extern __shared__ __align__(16) float vs[];                         // [kExpandRows][rank + 4]
    __shared__ int id_of[kExpandRows];
    [[maybe_unused]] __shared__ int top[kExpandRows];                   // a row's largest |V|, as bits
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int b0 = int(blockIdx.x) * kExpandRows, r0 = b0 + 16 * (wid & 1), c0 = int(blockIdx.y) * kExpandCols + kExpandWarpCols * (wid >> 1);
    const bool vec = (N & 3) == 0, vec32 = (ld & 3) == 0;
    float base[2][P][4];                                                // [8 rows][16 columns][column]
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int r = r0 + 8 * h + g, n = c0 + 16 * p + 4 * t;
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (r < M && n < N) {
                const float* q = y32 + size_t(r) * ld + n;
                if (vec32) v = __ldcg(reinterpret_cast<const float4*>(q));
                else v = make_float4(__ldcg(q), n + 1 < N ? __ldcg(q + 1) : 0.0f, n + 2 < N ? __ldcg(q + 2) : 0.0f, n + 3 < N ? __ldcg(q + 3) : 0.0f);
            }
            base[h][p][0] = v.x; base[h][p][1] = v.y; base[h][p][2] = v.z; base[h][p][3] = v.w;
        }
    constexpr bool kWhole = DT == kBF16 && YDT == kF32;                 // V as fp32, in three parts
    const int pitch = ad.rank + 4;
    if (wid == 0) {
        id_of[lane] = b0 + lane < M ? __ldcg(row_id + b0 + lane) : -1;
        if constexpr (DT != kBF16) top[lane] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kExpandRows * ad.rank / 4; i += kExpandThreads) {
        const int row = i / (ad.rank / 4), j = (i - row * (ad.rank / 4)) * 4, id = id_of[row];
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (id >= 0) {
            const float s = __ldg(ad.scale + id);
#pragma unroll 4
            for (int k = 0; k < chunks; ++k) {
                const float4 f = __ldcg(reinterpret_cast<const float4*>(u + (size_t(k) * M + b0 + row) * ad.rank + j));
                x.x += f.x; x.y += f.y; x.z += f.z; x.w += f.w;
            }
            x = make_float4(__fmul_rn(s, x.x), __fmul_rn(s, x.y), __fmul_rn(s, x.z), __fmul_rn(s, x.w));
        }
        if constexpr (kWhole) {
            *reinterpret_cast<float4*>(vs + row * pitch + j) = x;
        } else if constexpr (DT == kBF16) {
            *reinterpret_cast<uint4*>(vs + row * pitch + j) = two_parts<DT>(x);
        } else {
            *reinterpret_cast<float4*>(vs + row * pitch + j) = x;
            atomicMax(top + row, __float_as_int(fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(x.z), fabsf(x.w)))));
        }
    }
    __syncthreads();
    // 2^up: the power of two of a row
    [[maybe_unused]] auto up_of = [&](int row) { return 14 - max((top[row] >> 23) - 127, -100); };
    [[maybe_unused]] auto two_to = [](int e) { return __int_as_float((e + 127) << 23); };
    if constexpr (DT != kBF16) {
        for (int i = threadIdx.x; i < kExpandRows * ad.rank / 4; i += kExpandThreads) {      // a thread's own ones
            const int row = i / (ad.rank / 4), j = (i - row * (ad.rank / 4)) * 4;
            const float up = two_to(up_of(row));
            const float4 x = *reinterpret_cast<const float4*>(vs + row * pitch + j);
            *reinterpret_cast<uint4*>(vs + row * pitch + j) = two_parts<DT>(make_float4(x.x * up, x.y * up, x.z * up, x.w * up));
        }
        __syncthreads();
    }
    const int mine = id_of[16 * (wid & 1) + (lane & 15)];               // twice over the warp
    const unsigned with = __ballot_sync(0xffffffffu, mine >= 0) & 0xffffu;
    float d[B][4] = {};
    const float* const vrow = vs + (16 * (wid & 1) + g) * pitch + 4 * t;
    for (unsigned todo = c0 < N ? with : 0u; todo;) {
        const int id = __shfl_sync(0xffffffffu, mine, __ffs(todo) - 1);
        const unsigned mask = __ballot_sync(0xffffffffu, mine == id) & 0xffffu;
        todo &= ~mask;
        const bool in0 = (mask >> g) & 1u, in1 = (mask >> (8 + g)) & 1u;
#pragma unroll 2
        for (int j0 = 0; j0 < ad.rank; j0 += 16) {
            uint2 w[B];
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int n = c0 + 16 * (b >> 1) + 4 * (g >> 1) + 2 * (b & 1) + (g & 1);
                w[b] = n < N ? __ldg(reinterpret_cast<const uint2*>(ad.b + (size_t(id) * size_t(N) + size_t(n)) * ad.rank + j0 + 4 * t)) : make_uint2(0u, 0u);
            }
            if constexpr (kWhole) {
                const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                uint2 p[3], q[3];
                three_parts(in0 ? *reinterpret_cast<const float4*>(vrow + j0) : zero, p);
                three_parts(in1 ? *reinterpret_cast<const float4*>(vrow + 8 * pitch + j0) : zero, q);
#pragma unroll
                for (int b = 0; b < B; ++b)
#pragma unroll
                    for (int i = 2; i >= 0; --i) mma16<DT>(d[b], p[i].x, q[i].x, p[i].y, q[i].y, w[b].x, w[b].y);
            } else {
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                const uint4 p = in0 ? *reinterpret_cast<const uint4*>(vrow + j0) : zero, q = in1 ? *reinterpret_cast<const uint4*>(vrow + 8 * pitch + j0) : zero;
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    mma16<DT>(d[b], p.x, q.x, p.y, q.y, w[b].x, w[b].y);
                    mma16<DT>(d[b], p.z, q.z, p.w, q.w, w[b].x, w[b].y);
                }
            }
        }
    }
    [[maybe_unused]] float down[2];
    if constexpr (DT != kBF16) {
        for (int h = 0; h < 2; ++h) down[h] = two_to(-up_of(16 * (wid & 1) + 8 * h + g));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int r = r0 + 8 * h + g, n = c0 + 16 * p + 4 * t;
            if (r >= M || n >= N) continue;
            float* o = base[h][p];
            if ((with >> (8 * h + g)) & 1u) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = d[2 * p + (e >> 1)][2 * h + (e & 1)];
                    if constexpr (DT == kBF16) o[e] += x;
                    else o[e] = __fmaf_rn(x, down[h], o[e]);
                }
            }
            const size_t at = size_t(r) * N + n;
            if (vec) {
                // (a Y at any place, 16-bit and fp32: the general product's)
                if constexpr (YDT == kF32) {
                    float* q = static_cast<float*>(y) + at;
                    if ((reinterpret_cast<uintptr_t>(q) & 15u) == 0) *reinterpret_cast<float4*>(q) = make_float4(o[0], o[1], o[2], o[3]);
                    else { q[0] = o[0]; q[1] = o[1]; q[2] = o[2]; q[3] = o[3]; }
                } else {
                    uint2 z;
                    if constexpr (YDT == kBF16) {
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(z.x) : "f"(o[1]), "f"(o[0]));
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(z.y) : "f"(o[3]), "f"(o[2]));
                    } else {
                        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(z.x) : "f"(o[1]), "f"(o[0]));
                        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(z.y) : "f"(o[3]), "f"(o[2]));
                    }
                    uint16_t* q = static_cast<uint16_t*>(y) + at;
                    if ((reinterpret_cast<uintptr_t>(q) & 7u) == 0) *reinterpret_cast<uint2*>(q) = z;
                    else { q[0] = uint16_t(z.x); q[1] = uint16_t(z.x >> 16); q[2] = uint16_t(z.y); q[3] = uint16_t(z.y >> 16); }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) if (n + e < N) mmdk::store_y<YDT>(y, at + e, o[e]);
            }
        }
}

// expand_rows: for single rows, each with an adapter of its own (a product would work for one row of 16): a thread has two columns of a row, fp32
// throughout.  What it reads is on its way before the row's values are added up.  Bound by the adapters' B, which the kernel before has
// asked into L2: 64 rows x 8192 of 38 adapters of rank 16 7.9 us for 13 MB, cold.
template <int DT, int YDT>
__global__ void __launch_bounds__(kExpandThreads)
expand_rows(const Adapters ad, int M, int N, int chunks, const float* __restrict__ u, const int32_t* __restrict__ row_id, const float* y32, int ld, void* y) {
    __shared__ __align__(16) float v[256];                              // the largest rank
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int r = int(blockIdx.x), id = __ldcg(row_id + r);
    const int n = (int(blockIdx.y) * kExpandThreads + int(threadIdx.x)) * 2;
    const bool in = n < N, two = n + 1 < N;
    const size_t at = size_t(r) * N + (in ? n : 0), at32 = size_t(r) * ld + (in ? n : 0);
    float p = in ? __ldcg(y32 + at32) : 0.0f, q = two ? __ldcg(y32 + at32 + 1) : 0.0f;
    const uint4* b = reinterpret_cast<const uint4*>(ad.b + (size_t(max(id, 0)) * size_t(N) + size_t(in ? n : 0)) * ad.rank);
    const int pitch = two ? ad.rank / 8 : 0;
    auto ask = [&](int j, uint4 (&w)[4]) {                              // ranks j .. j + 15 of both columns
        w[0] = __ldg(b + j / 8); w[1] = __ldg(b + j / 8 + 1); w[2] = __ldg(b + pitch + j / 8); w[3] = __ldg(b + pitch + j / 8 + 1);
    };
    uint4 w[4] = {};
    if (id >= 0) ask(0, w);
    if (id >= 0 && threadIdx.x < ad.rank) {
        const float s = __ldg(ad.scale + id);
        float sum = 0.0f;
#pragma unroll 4
        for (int c = 0; c < chunks; ++c) sum += __ldcg(u + (size_t(c) * M + r) * ad.rank + threadIdx.x);
        v[threadIdx.x] = __fmul_rn(s, sum);
    }
    __syncthreads();
    if (!in) return;
    for (int j = 0; id >= 0 && j < ad.rank; j += 16) {
        uint4 next[4] = {};
        if (j + 16 < ad.rank) ask(j + 16, next);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float f[8], g[8];
            mmdk::widen8<DT>(w[h], f);
            mmdk::widen8<DT>(w[2 + h], g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p = __fmaf_rn(v[j + 8 * h + e], f[e], p);
                q = __fmaf_rn(v[j + 8 * h + e], g[e], q);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = next[e];
    }
    mmdk::store_y<YDT>(y, at, p);
    if (two) mmdk::store_y<YDT>(y, at + 1, q);
}

template <int DT, int YDT>
cudaError_t expand_as(int M, int N, const Adapters& ad, const ShrinkPlan& plan, const float* u, const int32_t* row_id, const float* y32, int ld, void* y, cudaStream_t st) {
    if (plan.rows == 1)
        return bqkvl::launch_after(expand_rows<DT, YDT>, dim3(unsigned(M), unsigned((N + 2 * kExpandThreads - 1) / (2 * kExpandThreads))), kExpandThreads, 0, st, ad, M, N,
                                   plan.chunks, u, row_id, y32, ld, y);
    return bqkvl::launch_after(expand_tiles<DT, YDT>, dim3(unsigned((M + kExpandRows - 1) / kExpandRows), unsigned((N + kExpandCols - 1) / kExpandCols)),
                               kExpandThreads, size_t(kExpandRows) * (ad.rank + 4) * 4, st, ad, M, N, plan.chunks, u, row_id, y32, ld, y);
}

template <int DT, int NT, int RT>
cudaError_t shrink_as(const Input& in, const Adapters& ad, const ShrinkPlan& plan, float* u, int32_t* row_id, cudaStream_t st) {
    const dim3 grid(unsigned((in.M + plan.rows - 1) / plan.rows), unsigned(plan.chunks));
    return bqkvl::launch_after(in.gamma ? shrink<DT, NT, RT, true> : shrink<DT, NT, RT, false>, grid, kShrinkThreads, 0, st, in, ad, plan.rows, u, row_id);
}

template <int DT>
cudaError_t shrink_any(const Input& in, const Adapters& ad, const ShrinkPlan& plan, float* u, int32_t* row_id, cudaStream_t st) {
    if (plan.rows <= 8) return ad.rank <= 16 ? shrink_as<DT, 1, 1>(in, ad, plan, u, row_id, st) : shrink_as<DT, 1, 4>(in, ad, plan, u, row_id, st);
    if (plan.rows <= 16) return shrink_as<DT, 2, 4>(in, ad, plan, u, row_id, st);
    return ad.rank <= 16 ? shrink_as<DT, 4, 1>(in, ad, plan, u, row_id, st) : shrink_as<DT, 4, 2>(in, ad, plan, u, row_id, st);
}

}  // namespace

// Single rows, each with an adapter of its own, go to a CTA each; prompts by 32 rows, or 16 with ranks above 32 (what the registers hold).
// Features are cut until there are four CTAs for every SM, in chunks of 512 at least.
ShrinkPlan shrink_plan(int M, int n_seq, int K, int rank) {
    ShrinkPlan p;
    p.rows = M <= 256 && n_seq * 2LL > M ? 1 : M <= 512 ? 8 : rank > 32 ? 16 : 32;
    const int blocks = (M + p.rows - 1) / p.rows, most = K / 512 < 1 ? 1 : K / 512;
    p.chunks = blocks > 0 ? 4 * 148 / blocks : 1;
    if (p.chunks > 16) p.chunks = 16;
    if (p.chunks > most) p.chunks = most;
    if (p.chunks < 1) p.chunks = 1;
    return p;
}

cudaError_t launch_shrink(bool bf16, const Input& in, const Adapters& ad, const ShrinkPlan& plan, float* u, int32_t* row_id, cudaStream_t st) {
    return bf16 ? shrink_any<kBF16>(in, ad, plan, u, row_id, st) : shrink_any<kF16>(in, ad, plan, u, row_id, st);
}

cudaError_t launch_expand(bool bf16, int M, int N, const Adapters& ad, const ShrinkPlan& plan, const float* u, const int32_t* row_id, const float* y32, int ld,
                          void* y, bool f32out, cudaStream_t st) {
    if (f32out) return bf16 ? expand_as<kBF16, kF32>(M, N, ad, plan, u, row_id, y32, ld, y, st) : expand_as<kF16, kF32>(M, N, ad, plan, u, row_id, y32, ld, y, st);
    return bf16 ? expand_as<kBF16, kBF16>(M, N, ad, plan, u, row_id, y32, ld, y, st) : expand_as<kF16, kF16>(M, N, ad, plan, u, row_id, y32, ld, y, st);
}

}  // namespace mmda
