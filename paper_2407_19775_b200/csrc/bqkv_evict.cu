// bqkv_evict.cu -- eviction from the 4-bit cache by accumulated attention weight: kernels and launch.
#include "bqkv_launch.h"

namespace bqkvk {

namespace {

// evict: one CTA per (sequence, head).
//
// Weights map to unsigned keys that order as they do (NaN to 0, below -inf).  The key of the
// last survivor is found by radix selection, eight bits a pass over the middle slots; slots above
// it stay, and of those equal to it the first `need`.  One ordered pass then lists the holes and
// the late survivors (the i-th hole takes the i-th late survivor), and the rows move: holes first
// (sources and destinations are disjoint), then the recent rows slide down in ascending order,
// a batch read before it is written (destinations lie below every source still to be read).
constexpr int kEvictThreads = 512;

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (!(w == w)) return 0u;
    const uint32_t b = __float_as_uint(w + 0.0f);                       // -0 counts as +0
    return (b >> 31) ? ~b : (b | 0x80000000u);
}

// exclusive prefix of `flag` over the CTA's threads; `total` its sum
__device__ __forceinline__ int cta_rank(bool flag, int* warp_sums, int& total) {
    const unsigned b = __ballot_sync(0xffffffffu, flag);
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    __syncthreads();
    if (lane == 0) warp_sums[w] = __popc(b);
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kEvictThreads / 32; ++i) {
        const int n = warp_sums[i];
        before += i < w ? n : 0;
        all += n;
    }
    total = all;
    return before + __popc(b & ((1u << lane) - 1u));
}

__device__ __forceinline__ void copy_row(const Cache& c, size_t dst, size_t src, int lane, int lanes) {
    const int words = c.dim / 8, nb = c.dim / c.block;
    for (int i = lane; i < words; i += lanes) {
        reinterpret_cast<uint32_t*>(c.k_codes)[dst * words + i] = reinterpret_cast<const uint32_t*>(c.k_codes)[src * words + i];
        reinterpret_cast<uint32_t*>(c.v_codes)[dst * words + i] = reinterpret_cast<const uint32_t*>(c.v_codes)[src * words + i];
    }
    for (int i = lane; i < nb; i += lanes) {
        c.k_scale[dst * nb + i] = c.k_scale[src * nb + i];
        c.v_scale[dst * nb + i] = c.v_scale[src * nb + i];
    }
}

__global__ void __launch_bounds__(kEvictThreads)
evict(const Cache c, float* __restrict__ weights, int64_t stride, int budget, int sinks, int recent, int32_t* __restrict__ lists) {
    __shared__ int hist[256], warp_sums[kEvictThreads / 32], pick[2];
    const int h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x;
    const int len = int(min(int64_t(c.len(s)), stride));
    if (len <= budget) return;
    float* w = weights + (size_t(s) * c.heads + h) * size_t(stride);
    const int lo = sinks, hi = len - recent, keep = budget - sinks - recent, edge = budget - recent;
    int32_t* holes = lists + (size_t(s) * c.heads + h) * 2 * size_t(budget);
    int32_t* late = holes + budget;

    uint32_t prefix = 0, mask = 0;
    int need = keep;                                                    // survivors still to be found among the keys that match the prefix
    for (int shift = 24; shift >= 0 && keep > 0; shift -= 8) {
        for (int i = tid; i < 256; i += kEvictThreads) hist[i] = 0;
        __syncthreads();
        for (int j = lo + tid; j < hi; j += kEvictThreads) {
            const uint32_t k = weight_key(w[j]);
            if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int b = 255, left = need;
            for (; b > 0 && hist[b] < left; --b) left -= hist[b];
            pick[0] = b;
            pick[1] = left;
        }
        __syncthreads();
        prefix |= uint32_t(pick[0]) << shift;
        mask |= 255u << shift;
        need = pick[1];
        __syncthreads();
    }
    int n_holes = 0, n_late = 0, n_equal = 0;
    for (int j0 = lo; j0 < hi; j0 += kEvictThreads) {
        const int j = j0 + tid;
        const bool in = j < hi;
        const uint32_t k = in ? weight_key(w[j]) : 0u;
        int total;
        const int rank = cta_rank(in && keep > 0 && k == prefix, warp_sums, total);
        const bool stays = in && keep > 0 && (k > prefix || (k == prefix && n_equal + rank < need));
        n_equal += total;
        const int rh = cta_rank(in && !stays && j < edge, warp_sums, total);
        if (in && !stays && j < edge) holes[n_holes + rh] = j;
        n_holes += total;
        const int rl = cta_rank(stays && j >= edge, warp_sums, total);
        if (stays && j >= edge) late[n_late + rl] = j;
        n_late += total;
    }
    __syncthreads();
    const int team = tid >> 4, lane = tid & 15;                         // sixteen threads move a row
    for (int i = team; i < n_holes; i += kEvictThreads / 16) {
        const int dst = holes[i], src = late[i];
        copy_row(c, c.row(s, h, dst), c.row(s, h, src), lane, 16);
        if (lane == 0) w[dst] = w[src];
    }
    __syncthreads();
    // the recent rows, 32 at a time: read, wait, write
    const int words = c.dim / 8, nb = c.dim / c.block;
    for (int i0 = 0; i0 < recent; i0 += kEvictThreads / 16) {
        const int i = i0 + team;
        uint32_t kw[2], vw[2];
        uint16_t ks[2], vs[2];
        float wt = 0.0f;
        const bool in = i < recent;
        const size_t src = in ? c.row(s, h, len - recent + i) : 0, dst = in ? c.row(s, h, edge + i) : 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int e = lane + 16 * u;
            if (in && e < words) {
                kw[u] = reinterpret_cast<const uint32_t*>(c.k_codes)[src * words + e];
                vw[u] = reinterpret_cast<const uint32_t*>(c.v_codes)[src * words + e];
            }
            if (in && e < nb) { ks[u] = c.k_scale[src * nb + e]; vs[u] = c.v_scale[src * nb + e]; }
        }
        if (in && lane == 0) wt = w[len - recent + i];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int e = lane + 16 * u;
            if (in && e < words) {
                reinterpret_cast<uint32_t*>(c.k_codes)[dst * words + e] = kw[u];
                reinterpret_cast<uint32_t*>(c.v_codes)[dst * words + e] = vw[u];
            }
            if (in && e < nb) { c.k_scale[dst * nb + e] = ks[u]; c.v_scale[dst * nb + e] = vs[u]; }
        }
        if (in && lane == 0) w[edge + i] = wt;
        __syncthreads();
    }
}

// lens after the heads of every sequence have read them
__global__ void __launch_bounds__(256) evict_lens(const Cache c, int64_t stride, int budget) {
    const int s = blockIdx.x * 256 + threadIdx.x;
    if (s < c.n_seq && int(min(int64_t(c.len(s)), stride)) > budget) c.lens[s] = budget;
}

}  // namespace

}  // namespace bqkvk

namespace bqkvl {

cudaError_t launch_evict(const bqkvk::Cache& c, float* weights, int64_t stride, int budget, int sinks, int recent, void* workspace, cudaStream_t st) {
    bqkvk::evict<<<dim3(unsigned(c.heads), unsigned(c.n_seq)), bqkvk::kEvictThreads, 0, st>>>(c, weights, stride, budget, sinks, recent,
                                                                                           static_cast<int32_t*>(workspace));
    bqkvk::evict_lens<<<unsigned((c.n_seq + 255) / 256), 256, 0, st>>>(c, stride, budget);
    return cudaGetLastError();
}

}  // namespace bqkvl
