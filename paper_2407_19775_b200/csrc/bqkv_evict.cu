// bqkv_evict.cu -- eviction from the 4-bit cache by accumulated attention weight: kernels and launch.
#include "bqkv_launch.h"

#include <mutex>

namespace bqkvk {

namespace {

// evict: one CTA per (sequence, head).
//
// Weights map to unsigned keys that order as they do (NaN to 0, below -inf); the keys of the middle slots are kept in shared
// memory where they fit.  The key of the last survivor is found by radix selection, eight bits a pass; the counters have eight
// copies, because the first pass meets few exponents and equal addresses of one warp are added one after the other.  Slots
// above that key stay, and of those equal to it the first `need`.  Each warp then owns a contiguous range of slots: it counts
// (equal keys; then holes and late survivors), one prefix over the warps, and it lists its own in order.  The i-th hole takes
// the i-th late survivor; the rows move: holes first (sources and destinations are disjoint), then the recent rows slide down
// in ascending order, a batch read before it is written (destinations lie below every source still to be read).
// Bound by latency: a chain of passes over a few slots per thread, with a barrier between them.  Measured: 32 sequences x 8 heads
// from 1025 slots to 1024, 64 of them recent: 21 us for 3 MB (256 CTAs on 148 SMs; one sequence 12 us); 8 x 8 from up to 32768 to 2048:
// 44 us in 64 CTAs, 44 MB at most (7 us by their bytes).
constexpr int kEvictThreads = 1024, kEvictWarps = kEvictThreads / 32;
constexpr int kCopies = 8;
constexpr int kKeysInShared = 40960;                                    // of the middle slots, 160 KB

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (!(w == w)) return 0u;
    const uint32_t b = __float_as_uint(w + 0.0f);                       // -0 counts as +0
    return (b >> 31) ? ~b : (b | 0x80000000u);
}

// Sum over the warps before this one of a per-warp count, and the total; all threads call it.
__device__ __forceinline__ int warps_before(int count, int* shared, int& total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    __syncthreads();
    if (lane == 0) shared[w] = count;
    __syncthreads();
    int v = shared[lane];                                               // 32 warps, one per lane
    int inc = v;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, inc, k);
        if (lane >= k) inc += o;
    }
    total = __shfl_sync(0xffffffffu, inc, 31);
    return __shfl_sync(0xffffffffu, inc - v, w);
}

__global__ void __launch_bounds__(kEvictThreads)
evict(const Cache c, float* __restrict__ weights, int64_t stride, int budget, int sinks, int recent, int keys_room, int32_t* __restrict__ lists) {
    extern __shared__ __align__(16) uint32_t kept_keys[];                 // later the rows of moves, sixteen bytes each
    __shared__ int hist[256 * kCopies], bins[256], sums[kEvictWarps], pick[2];
    const int h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int len = int(min(int64_t(c.len(s)), stride));
    if (len <= budget) return;
    float* w = weights + (size_t(s) * c.heads + h) * size_t(stride);
    const int lo = sinks, hi = len - recent, count = hi - lo, keep = budget - sinks - recent, edge = budget - recent;
    int32_t* holes = lists + (size_t(s) * c.heads + h) * 2 * size_t(budget);
    int32_t* late = holes + budget;
    const bool in_shared = count <= keys_room;
    if (in_shared)
        for (int i = tid; i < count; i += kEvictThreads) kept_keys[i] = weight_key(w[lo + i]);
    auto key_of = [&](int i) -> uint32_t { return in_shared ? kept_keys[i] : weight_key(w[lo + i]); };      // of middle slot lo + i

    uint32_t prefix = 0, mask = 0;
    int need = keep;                                                    // survivors still to be found among the keys that match the prefix
    for (int shift = 24; shift >= 0 && keep > 0; shift -= 8) {
        for (int i = tid; i < 256 * kCopies; i += kEvictThreads) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < count; i += kEvictThreads) {
            const uint32_t k = key_of(i);
            if ((k & mask) == prefix) atomicAdd(&hist[((k >> shift) & 255u) * kCopies + (tid & (kCopies - 1))], 1);
        }
        __syncthreads();
        // survivors with a larger digit than bin b: a suffix sum over the bins, 32 per warp
        if (tid < 256) {
            const int b = 255 - tid;                                    // from the top
            int n = 0;
#pragma unroll
            for (int k = 0; k < kCopies; ++k) n += hist[b * kCopies + k];
            int inc = n;
#pragma unroll
            for (int k = 1; k < 32; k <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, inc, k);
                if (lane >= k) inc += o;
            }
            bins[tid] = inc;
            if (lane == 31) sums[warp] = inc;
        }
        __syncthreads();
        if (tid < 256) {
            int before = 0;
            for (int k = 0; k < warp; ++k) before += sums[k];
            const int inc = before + bins[tid], ex = lane > 0 ? before + bins[tid - 1] : before;
            if (ex < need && need <= inc) { pick[0] = 255 - tid; pick[1] = need - ex; }
        }
        __syncthreads();
        prefix |= uint32_t(pick[0]) << shift;
        mask |= 255u << shift;
        need = pick[1];
    }
    // each warp's range of middle slots, a multiple of 32
    const int span = (count + kEvictThreads - 1) / kEvictThreads * 32, b0 = min(warp * span, count), b1 = min(b0 + span, count);
    int total, n_equal = 0;
    if (keep > 0)
        for (int i = b0 + lane; i < b1; i += 32) n_equal += key_of(i) == prefix;
    n_equal = __reduce_add_sync(0xffffffffu, n_equal);
    const int equal_before = warps_before(n_equal, sums, total);
    auto walk = [&](auto visit) {                                       // visit(slot, in, stays) for 32 slots at a time, in order
        int equal = equal_before;
        for (int i0 = b0; i0 < b1; i0 += 32) {
            const int i = i0 + lane;
            const bool in = i < b1;
            const uint32_t k = in ? key_of(i) : 0u;
            const bool same = in && keep > 0 && k == prefix;
            const unsigned m = __ballot_sync(0xffffffffu, same);
            const bool stays = in && keep > 0 && (k > prefix || (same && equal + __popc(m & ((1u << lane) - 1u)) < need));
            equal += __popc(m);
            visit(lo + i, in, stays);
        }
    };
    int my_holes = 0, my_late = 0;
    walk([&](int j, bool in, bool stays) {
        my_holes += __popc(__ballot_sync(0xffffffffu, in && !stays && j < edge));
        my_late += __popc(__ballot_sync(0xffffffffu, stays && j >= edge));
    });
    int n_holes;
    int hole_at = warps_before(my_holes, sums, n_holes);
    int late_at = warps_before(my_late, sums, total);
    walk([&](int j, bool in, bool stays) {
        const bool hole = in && !stays && j < edge, is_late = stays && j >= edge;
        const unsigned mh = __ballot_sync(0xffffffffu, hole), ml = __ballot_sync(0xffffffffu, is_late), below = (1u << lane) - 1u;
        if (hole) holes[hole_at + __popc(mh & below)] = j;
        if (is_late) late[late_at + __popc(ml & below)] = j;
        hole_at += __popc(mh);
        late_at += __popc(ml);
    });
    __syncthreads();
    const int team = tid >> 4, tl = tid & 15;                           // sixteen threads move a row
    // The rows of a batch of moves are looked up first, all at once (the keys' place in shared memory is free, or there is none:
    // then batches of 64), and four rows per team are read before they are written: the chain of dependent loads is what costs.
    __shared__ ulonglong2 few[64];
    ulonglong2* const moves = keys_room >= 4096 ? reinterpret_cast<ulonglong2*>(kept_keys) : few;
    const int batch = keys_room >= 4096 ? keys_room / 4 : 64;
    for (int m0 = 0; m0 < n_holes; m0 += batch) {
        const int n = min(batch, n_holes - m0);
        __syncthreads();
        for (int i = tid; i < n; i += kEvictThreads) {
            const int dst = holes[m0 + i], src = late[m0 + i];
            moves[i] = make_ulonglong2(c.row(s, h, dst), c.row(s, h, src));
            w[dst] = w[src];
        }
        __syncthreads();
        const int words_ = c.dim / 8, nb_ = c.dim / c.block;
        for (int i0 = team; i0 < n; i0 += 4 * (kEvictThreads / 16)) {
            for (int e = tl; e < words_; e += 16) {
                uint32_t kw[4], vw[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int i = i0 + u * (kEvictThreads / 16);
                    if (i < n) {
                        kw[u] = reinterpret_cast<const uint32_t*>(c.k_codes)[moves[i].y * words_ + e];
                        vw[u] = reinterpret_cast<const uint32_t*>(c.v_codes)[moves[i].y * words_ + e];
                    }
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int i = i0 + u * (kEvictThreads / 16);
                    if (i < n) {
                        reinterpret_cast<uint32_t*>(c.k_codes)[moves[i].x * words_ + e] = kw[u];
                        reinterpret_cast<uint32_t*>(c.v_codes)[moves[i].x * words_ + e] = vw[u];
                    }
                }
            }
            for (int e = tl; e < nb_; e += 16) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int i = i0 + u * (kEvictThreads / 16);
                    if (i < n) {
                        c.k_scale[moves[i].x * nb_ + e] = c.k_scale[moves[i].y * nb_ + e];
                        c.v_scale[moves[i].x * nb_ + e] = c.v_scale[moves[i].y * nb_ + e];
                    }
                }
            }
        }
    }
    __syncthreads();
    // the recent rows, 64 at a time: read, wait, write
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
            const int e = tl + 16 * u;
            if (in && e < words) {
                kw[u] = reinterpret_cast<const uint32_t*>(c.k_codes)[src * words + e];
                vw[u] = reinterpret_cast<const uint32_t*>(c.v_codes)[src * words + e];
            }
            if (in && e < nb) { ks[u] = c.k_scale[src * nb + e]; vs[u] = c.v_scale[src * nb + e]; }
        }
        if (in && tl == 0) wt = w[len - recent + i];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int e = tl + 16 * u;
            if (in && e < words) {
                reinterpret_cast<uint32_t*>(c.k_codes)[dst * words + e] = kw[u];
                reinterpret_cast<uint32_t*>(c.v_codes)[dst * words + e] = vw[u];
            }
            if (in && e < nb) { c.k_scale[dst * nb + e] = ks[u]; c.v_scale[dst * nb + e] = vs[u]; }
        }
        if (in && tl == 0) w[edge + i] = wt;
        __syncthreads();
    }
}

// lens after the heads of every sequence have read them
__global__ void __launch_bounds__(256) evict_lens(const Cache c, int64_t stride, int budget) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int s = blockIdx.x * 256 + threadIdx.x;
    if (s < c.n_seq && int(min(int64_t(c.len(s)), stride)) > budget) c.lens[s] = budget;
}

}  // namespace

}  // namespace bqkvk

namespace bqkvl {

cudaError_t launch_evict(const bqkvk::Cache& c, float* weights, int64_t stride, int budget, int sinks, int recent, void* workspace, cudaStream_t st) {
    static bool opted[64] = {};
    static std::mutex lock;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> guard(lock);
        if (!opted[dev]) {
            e = cudaFuncSetAttribute(bqkvk::evict, cudaFuncAttributeMaxDynamicSharedMemorySize, bqkvk::kKeysInShared * 4);
            if (e != cudaSuccess) return e;
            opted[dev] = true;
        }
    }
    // room for the keys of the longest sequence there can be, as far as it goes
    const long long most = (long long)c.max_pages * c.page < stride ? (long long)c.max_pages * c.page : stride;
    const int room = most <= bqkvk::kKeysInShared ? int(most) : bqkvk::kKeysInShared;
    e = launch_after(bqkvk::evict, dim3(unsigned(c.heads), unsigned(c.n_seq)), bqkvk::kEvictThreads, size_t(room) * 4, st, c, weights, stride, budget, sinks, recent,
                     room, static_cast<int32_t*>(workspace));
    if (e != cudaSuccess) return e;
    return launch_after(bqkvk::evict_lens, dim3(unsigned((c.n_seq + 255) / 256)), 256, 0, st, c, stride, budget);
}

}  // namespace bqkvl
