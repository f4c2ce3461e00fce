// bqkv_shared.cuh -- the end of an attention whose slots were attended to in parts (the sequences' own and, in one or several parts, a
// prefix that they share): join_parts (sm_100a).
#pragma once

#include "bqkv_kernels.cuh"

namespace bqkvk {

// A warp per (row of the call, query head), D / 32 columns a lane.  With M the largest reference of the parts that saw a slot and
// f_i = 2^(m_i - M):  out = sum_i f_i sums_i / sum_i f_i l_i.  Parts are added in order, so the same call gives the same bits; those that saw
// nothing are not read.  Part 0 is of the sequence's own slots, the others of its prefix, if it has one; rows of no sequence are left alone.
// stats2 / stats4 (either may be null): reference and 1 / sum of the whole row, for the weights of the own slots.
// Bound by its bytes: 64 x 64 rows of 128 in 10 parts 8.3 us for 22 MB, cold.
constexpr int kJoinThreads = 256, kMostParts = 32;

template <int DT, int D>
__global__ void __launch_bounds__(kJoinThreads)
join_parts(const PartRows shared, int n_own, int prefixes, int q_heads, int n_parts, const Parts parts, void* __restrict__ out, float2* __restrict__ stats2,
           float4* __restrict__ stats4) {
    constexpr int C = D / 32;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    const int lane = threadIdx.x & 31;
    const int upto = shared.starts ? min(shared.starts[n_own], shared.n) : shared.n;
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

// ------------------------------------------------------------------------------------------
// attend_part_general: a part of the slots for head sizes, blocks and pages that the other kernels do not take.  attend_general dequantizes a slot
// once for every query row; here a CTA has eight query rows of a (sequence, cached head) -- row = query * group + head, as in the
// tiles kernel -- and takes 64 slots at a time for all of them.  Scores: a lane per slot, four warps on the words of its key, eight rows to
// each element that a lane has dequantized, the rows' elements broadcast from shared memory; the warps' sums are added in order.
// Softmax: a warp per row.  Outputs: a thread per byte of the value (two columns) and every G-th slot, eight rows again.  fp32
// throughout; natural units, as join_general wants them.  Bound by instructions and by the loads that they wait for.  Measured, head_dim 80 in
// blocks of 40, whole calls, attend_general on both sides | this: 11 single tokens of 8 cached heads of 2 behind 6298 slots 143 | 85 us, 9 sequences
// of up to 108 rows, 1 cached head of 7, behind 5 prefixes of up to 419 slots 227 | 124 us, 56 single tokens, 1 head of 5, behind 167 slots 34 | 33 us.
constexpr int kPartRows = 8, kPartSlots = 64, kPartThreads = 256;

template <int DT>
__global__ void __launch_bounds__(kPartThreads, 3)
attend_part_general(const Cache c, const PartRows rows, const void* __restrict__ q, int64_t q_stride, int q_heads, float sm_scale, int blocks /* per sequence */,
                    float* __restrict__ partial, int z0, int z_all, const __grid_constant__ bq4k::Tables4 tab) {
    constexpr int R = kPartRows, W = kPartThreads / 32;
    static_assert(R == 8 && W == 8 && kPartSlots == 64, "a warp per row; two halves of a tile, four warps each");
    __shared__ float thr[16], val[16];
    __shared__ __align__(16) float qs[256][R], ps[kPartSlots][R];
    __shared__ float sums[W][R][32], fade[R];
    __shared__ int limit[R];                                            // slots that each row sees
    __shared__ size_t row_of[2][kPartSlots];
    bq4k::fill_tables(tab, thr, val);
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, dim = c.dim, words = dim / 8, nb = dim / c.block, bytes = dim / 2;
    const int s = int(blockIdx.x) / blocks, h = blockIdx.y, group = q_heads / c.heads;
    const int r0 = rows.begin(s), n = rows.end(s) - r0, counted = c.counted(s), len = c.held(counted), first = rows.first(counted, len, n);
    const int64_t all = int64_t(max(n, 0)) * group;
    const int G = kPartThreads / bytes, col = tid % bytes, grp = tid / bytes, vb = 2 * col / c.block;     // G groups of a thread per byte; the rest idle
    const int half = wid >> 2, word0 = wid & 3;                         // this warp's half of a tile's slots, and every fourth word of them
    auto sees = [&](int64_t row) { return row < all ? min(max(first + int(row / group) + 1, 0), len) : 0; };       // slots 0 .. sees - 1
    for (int64_t b0 = int64_t(int(blockIdx.x) % blocks) * R; b0 < all; b0 += int64_t(blocks) * R) {
        const int seen = sees(b0 + wid);                                // of this warp's row
        const int sure = b0 + R <= all ? sees(b0) : 0, most = sees(min(b0 + R, all) - 1);       // of every row, of the block's last one
        const int tiles = (most + kPartSlots - 1) / kPartSlots;
        const int t0 = int((long long)tiles * blockIdx.z / gridDim.z), t1 = int((long long)tiles * (blockIdx.z + 1) / gridDim.z);
        auto look_up = [&](int t) {
            if (tid < kPartSlots && t < t1) row_of[t & 1][tid] = c.row(s, h, min(t * kPartSlots + tid, most - 1));
        };
        __syncthreads();                                                // the block before is done with shared memory
        {
            const int64_t row = b0 + wid;
            const int i = int(row / group);
            const size_t at = size_t(r0 + i) * size_t(q_stride) + size_t(h * group + int(row - int64_t(i) * group)) * dim;
            for (int d = lane; d < dim; d += 32) qs[d][wid] = row < all ? bq4k::load1<DT>(q, at + d) : 0.0f;
        }
        look_up(t0);
        if (lane == 0) limit[wid] = seen;
        float m = -INFINITY, l = 0.0f, o[R][2] = {};
        for (int t = t0; t < t1; ++t) {
            const int j0 = t * kPartSlots;
            __syncthreads();                                            // row_of is there; ps is free
            look_up(t + 1);
            {
                float x[R] = {};
                const size_t row = row_of[t & 1][half * 32 + lane];
                for (int w = word0; w < words; w += 4) {
                    const uint32_t u = reinterpret_cast<const uint32_t*>(c.k_codes)[row * words + w];
                    const float f = scale_of(c.k_scale, row * nb + (w * 8) / c.block);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float k = __fmul_rn(val[(u >> (4 * e)) & 15u], f);
                        const float4 a = *reinterpret_cast<const float4*>(&qs[w * 8 + e][0]), b = *reinterpret_cast<const float4*>(&qs[w * 8 + e][4]);
                        x[0] = __fmaf_rn(k, a.x, x[0]), x[1] = __fmaf_rn(k, a.y, x[1]), x[2] = __fmaf_rn(k, a.z, x[2]), x[3] = __fmaf_rn(k, a.w, x[3]);
                        x[4] = __fmaf_rn(k, b.x, x[4]), x[5] = __fmaf_rn(k, b.y, x[5]), x[6] = __fmaf_rn(k, b.z, x[6]), x[7] = __fmaf_rn(k, b.w, x[7]);
                    }
                }
#pragma unroll
                for (int r = 0; r < R; ++r) sums[wid][r][lane] = x[r];
            }
            __syncthreads();
            {
                float x[2], top = m, p[2], both;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    x[k] = sums[4 * k][wid][lane];
#pragma unroll
                    for (int w = 1; w < 4; ++w) x[k] += sums[4 * k + w][wid][lane];
                    x[k] = j0 + 32 * k + lane < seen ? __fmul_rn(x[k], sm_scale) : -INFINITY;
                    top = fmaxf(top, x[k]);
                }
#pragma unroll
                for (int k = 16; k >= 1; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
                const bool none = top == -INFINITY;                     // the row has seen nothing yet, or nothing but NaN
                const float f = none ? 1.0f : expf(m - top);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    p[k] = j0 + 32 * k + lane >= seen || (none && x[k] == top) ? 0.0f : expf(x[k] - top);
                    ps[32 * k + lane][wid] = p[k];
                }
                both = p[0] + p[1];
                if (lane == 0) fade[wid] = f;
                m = top;
#pragma unroll
                for (int k = 16; k >= 1; k >>= 1) both += __shfl_xor_sync(0xffffffffu, both, k);
                l = __fmaf_rn(l, f, both);
            }
            __syncthreads();
            if (grp < G) {
#pragma unroll
                for (int r = 0; r < R; ++r) o[r][0] *= fade[r], o[r][1] *= fade[r];
                const int slots = min(kPartSlots, most - j0);
                auto value = [&](int j, float& v0, float& v1) {
                    const size_t row = row_of[t & 1][j];
                    const uint32_t byte = c.v_codes[row * size_t(bytes) + col];
                    const float f = scale_of(c.v_scale, row * nb + vb);
                    v0 = __fmul_rn(val[byte & 15u], f), v1 = __fmul_rn(val[byte >> 4], f);
                };
                float v0, v1;
                if (j0 + slots <= sure) {
#pragma unroll 4
                    for (int j = grp; j < slots; j += G) {
                        value(j, v0, v1);
                        const float4 a = *reinterpret_cast<const float4*>(&ps[j][0]), b = *reinterpret_cast<const float4*>(&ps[j][4]);
                        const float p[R] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                        for (int r = 0; r < R; ++r) o[r][0] = __fmaf_rn(p[r], v0, o[r][0]), o[r][1] = __fmaf_rn(p[r], v1, o[r][1]);
                    }
                } else {                                                // some rows see less: what a masked slot holds stays out, NaN too
#pragma unroll 2
                    for (int j = grp; j < slots; j += G) {
                        value(j, v0, v1);
#pragma unroll
                        for (int r = 0; r < R; ++r)
                            if (j0 + j < limit[r]) o[r][0] = __fmaf_rn(ps[j][r], v0, o[r][0]), o[r][1] = __fmaf_rn(ps[j][r], v1, o[r][1]);
                    }
                }
            }
        }
        // the groups' sums, in order, a row at a time
        float* cols = &sums[0][0][0];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = b0 + r;
            if (row >= all) break;
            __syncthreads();
            if (grp < G) cols[grp * dim + 2 * col] = o[r][0], cols[grp * dim + 2 * col + 1] = o[r][1];
            __syncthreads();
            const int i = int(row / group);
            const size_t pair = size_t(r0 + i) * q_heads + h * group + int(row - int64_t(i) * group);
            float* part = partial + (pair * z_all + z0 + blockIdx.z) * (dim + 2);
            if (tid < dim) {
                float sum = 0.0f;
                for (int k = 0; k < G; ++k) sum += cols[k * dim + tid];
                part[tid] = sum;
            }
            if (wid == r && lane == 0) part[dim] = m, part[dim + 1] = l;
        }
    }
}

}  // namespace bqkvk
