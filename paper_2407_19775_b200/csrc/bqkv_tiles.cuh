// bqkv_tiles.cuh -- attention of many query rows per cached head over the 4-bit cache (a prompt, or
// a chunk of one): attend_tiles (sm_100a, tcgen05).
//
// One CTA takes 256 query rows of a (sequence, cached head) -- rows of the group's heads interleaved,
// row = query * group + head -- as two tiles of 128, and walks over the visible slots, dequantizing 64
// and attending to 32 at a time:
//
//   warps 0-7    softmax, one thread per query row: scores from tensor memory, probabilities back
//                into it as fp16 (they take the place of the scores they came from)
//   warps 8-11   dequantize keys:   K  [64 slots][D], K-major, 128-byte swizzle, in shared memory
//   warps 12-15  dequantize values: V^T [D][64 slots], likewise
//   warp 16      one thread issues tcgen05.mma (kind::f16): S = Q K^T and O += P V, the A operand
//                (queries, probabilities) in tensor memory, so that shared memory feeds only K and V
//
// Scores have two buffers per row tile, so that the scores of the next 32 slots are there when a
// softmax ends.  Tensor memory (512 columns): queries 2 x D / 2, scores 2 x 2 x 32, outputs 2 x D.
//
// Exactness.  Queries are scaled by a power of two per row.  With one block per cached row the
// operands are the exact codebook values (in units that make them fp16 numbers) and the scales of
// the slot multiply scores and probabilities in fp32.  With several blocks per row a key is
// value * s with s the block's scale over a power of two common to the slot: 19 bits, split exactly
// into two fp16 numbers and two products; a value likewise for fp16 outputs, and rounded to its 11 bits
// for bf16 outputs (their own rounding is 8 times as large).  Probabilities enter the second product with
// 11 bits (bf16 outputs), or as two fp16 numbers (fp16 outputs, whose own rounding that would match).
// What enters the second product as fp16 is probability times value scale.  A row's reference R is the largest of
// score + log2(value scale) over the slots that it sees, so that the row's largest such product is 2^10 (up to 2^14 until the
// reference moves) and keeps its bits down to 2^-24, whatever scales other slots have, masked or of no weight.
// The softmax's sum, in fp32, holds 2^(score - R) without the scale: value scales count as 2^-80 at least in R, which bounds it.
//
// Measured (4 sequences, chunks up to 2048 tokens over as many cached, 8 x 4 heads, head_dim 128, bf16; 222 GFLOP counted
// for the slots each row sees): 404 us, 0.55 PFLOP/s, 3400 cycles per 64 slots and SM.  Of these the tensor cores work 1000, the
// exponentials take 1024 of the special-function pipe (16 a clock), and the warps issue 1650 instructions per scheduler:
// about 600 per softmax warp and 200 per dequantizing warp.  Bound by latency between these: each scheduler has two softmax
// and two dequantizing warps, which is what registers (104 and 88 a thread) and shared memory (the pair table and two stages)
// leave room for.  What it took, in the order of the gains: products issued behind elect.sync (a thread chosen by its lane
// number took 125 cycles per product, now about 35); the next tile's loads after the stage is handed over, not before; the softmax's registers
// (spilled ones go through an L1 that the shared memory has left little of); two score buffers.  A CTA begins and ends in
// about 21000 cycles (queries in, first tile, outputs), six times 64 slots.
// fp16 outputs: 455 us; with blocks of 64 487 us (bf16) and 560 us (fp16, 515 with values rounded to 11 bits and a third more error
// against 64 bits).
// Waits are bounded as in the product kernels.
#pragma once

#include "bqkv_rows.cuh"
#include "tc_primitives.cuh"

namespace bqkvk {

struct TilesArgs {
    const void* q;
    int64_t q_stride;
    int bf16, q_heads, group;
    float score_scale;                     // |sm_scale| log2(e) / unit, positive
    int negate;                            // sm_scale is negative: the queries' signs are flipped instead
    float inv_unit;
    void* out;
    float4* stats;                         // for the weights kernel: (reference, 1 / sum, factor of its scores, -) of every (row, query head), log2 units
    uint32_t* scaled;                      // and the row's scaled fp16 queries; both null where no weights are wanted
    int* status;
};

template <int D, int NB, bool SPLIT>
struct TilesCfg {
    static constexpr int kRowsPerCta = 256, kSlots = 64, kStep = 32;
    static constexpr int kSoftmaxWarps = 8, kThreads = 17 * 32;
    static constexpr uint32_t kKBytes = kSlots * D * 2, kVBytes = kSlots * D * 2;
    static constexpr uint32_t kStage = kKBytes * (NB > 1 ? 2 : 1) + kVBytes;      // keys (with several blocks: high and low parts), values
    static constexpr uint32_t kVLow = NB > 1 && SPLIT ? kVBytes : 0;   // low parts of the values, both stages' behind stage 1
    static constexpr int kTable = 256 * 256;
    static constexpr int kSmem = 2 * kTable + int(kStage + 2 * kVLow) - 1024;      // stage 0, the pair table at a multiple of 64 KB, stage 1
    static constexpr uint32_t kTmemQ = 0, kTmemS = D, kTmemO = D + 128;
    static constexpr uint32_t kTmemCols = 512;                         // D + 128 + 2 D, rounded up to a power of two
    static_assert(kSmem + 4096 <= 227 * 1024 && kStage <= 65536 - 4096 - 1024, "fits");
};

__device__ __forceinline__ void umma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void st_shared16(uint32_t at, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Whether all 128 threads that meet at the named barrier say so.
__device__ __forceinline__ bool all_of(int barrier, bool x) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %2, 0;\n\tbar.red.and.pred p, %1, 128, q;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(r) : "r"(barrier), "r"(uint32_t(x)) : "memory");
    return r != 0;
}
__device__ __forceinline__ float pow2_of(int e) {                     // 2^e; 0 below the normal numbers
    return e < -126 ? 0.0f : __uint_as_float(uint32_t(min(e, 127) + 127) << 23);
}

// A row of D 16-bit elements (pairs in out) as fp16 pairs whose largest magnitude lies in [2^14, 2^15), and the power of two
// that undoes that.  Exact down to 2^-29 of the largest.
template <int D>
__device__ __forceinline__ float scale_query(bool bf16, bool negate, uint32_t (&out)[D / 2]) {
    auto both = [&](uint32_t v, float& x, float& y) {
        x = bf16 ? __uint_as_float(v << 16) : __low2float(*reinterpret_cast<const __half2*>(&v));
        y = bf16 ? __uint_as_float(v & 0xffff0000u) : __high2float(*reinterpret_cast<const __half2*>(&v));
    };
    float big = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 2; ++i) {
        float x, y;
        both(out[i], x, y);
        big = fmaxf(big, fmaxf(fabsf(x), fabsf(y)));
    }
    const int up = min(max(14 - (int(__float_as_uint(big) >> 23) - 127), -126), 126);      // (a row of zeros: anything)
    const float f = __uint_as_float(uint32_t(up + 127) << 23) * (negate ? -1.0f : 1.0f);
#pragma unroll
    for (int i = 0; i < D / 2; ++i) {
        float x, y;
        both(out[i], x, y);
        out[i] = half2_of(x * f, y * f);
    }
    return __uint_as_float(uint32_t(127 - up) << 23);
}

template <int D, int NB, bool SPLIT /* probabilities, and values that are not exact, as two fp16 numbers */>
__global__ void __launch_bounds__(TilesCfg<D, NB, SPLIT>::kThreads, 1)
attend_tiles(const Cache c, const Rows rows, const TilesArgs a, const __grid_constant__ PairTable pairs) {
    using Cfg = TilesCfg<D, NB, SPLIT>;
    constexpr int BN = Cfg::kSlots, ST = Cfg::kStep;
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ __align__(16) float key_factor[2][BN], value_factor[2][BN];      // of the slots of a stage
    __shared__ __align__(16) __half rho[2][2][NB > 1 ? NB : 1][NB > 1 ? BN : 8];      // keys, values: a block's scale over what its slot's factor holds
    __shared__ uint16_t half[16];
    __shared__ __align__(8) uint64_t bars[17];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    // (a shuffle tells the compiler that the value is the same in all lanes: loop counts and addresses stay in uniform registers)
    auto uniform = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
    const int warp = uniform(int(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    const uint32_t low = uint32_t(__cvta_generic_to_shared(smem)), table = (low + 0xFFFFu) & 0xFFFF0000u;
    const uint32_t stage_at[2] = {(low + 1023u) & ~1023u, table + Cfg::kTable};
    [[maybe_unused]] const uint32_t v_low = stage_at[1] + Cfg::kStage;
    const uint32_t bar0 = uint32_t(__cvta_generic_to_shared(bars));
    const uint32_t kv_full = bar0, kv_empty = bar0 + 16, s_full = bar0 + 32 /* [row tile][buffer] */, p_ready = bar0 + 64 /* likewise */,
                   o_done = bar0 + 96 /* likewise */, q_ready = bar0 + 128;

    const int h = blockIdx.x, s = blockIdx.y;                          // blocks of rows last: those that see most slots start first
    const int r0 = uniform(rows.begin(s)), n = max(uniform(rows.end(s)) - r0, 0), counted = uniform(c.counted(s)), len = c.held(counted);
    const int at0 = counted - n;                                       // slot of the first row
    const uint32_t group = uint32_t(a.group), all_rows = uint32_t(n) * group;      // below 2^31: the caller sees to that

    if (threadIdx.x < 16) half[threadIdx.x] = pairs.half[threadIdx.x];
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mmdk::mbar_init(kv_full + 8u * i, 256);
            mmdk::mbar_init(kv_empty + 8u * i, 1);
            mmdk::mbar_init(s_full + 8u * i, 1);
            mmdk::mbar_init(s_full + 16u + 8u * i, 1);
            mmdk::mbar_init(p_ready + 8u * i, 128);
            mmdk::mbar_init(p_ready + 16u + 8u * i, 128);
            mmdk::mbar_init(o_done + 8u * i, 1);
            mmdk::mbar_init(o_done + 16u + 8u * i, 1);
        }
        mmdk::mbar_init(q_ready, 256);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 16) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(uint32_t(__cvta_generic_to_shared(&tmem_slot))), "r"(Cfg::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    if (warp >= Cfg::kSoftmaxWarps && warp < 16) {                     // the pair table: entry e, four lanes' copies per store
        for (int i = int(threadIdx.x) - 256; i < 256 * 8; i += 256) {
            const uint32_t e = uint32_t(i) >> 3, v = uint32_t(half[e & 15u]) | uint32_t(half[e >> 4]) << 16;
            *reinterpret_cast<uint4*>(smem + (table - low) + e * 256 + (i & 7) * 16) = make_uint4(v, v, v, v);
        }
    }
    tc_after();
    const uint32_t tmem = uint32_t(uniform(int(tmem_slot)));
    const uint32_t table_lane = table | uint32_t(lane) * 4u;
    auto pair_of = [&](uint32_t word, int byte) -> uint32_t {
        uint32_t v;
        asm("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(bq4k::prmt(word, table_lane, 0x7604u | uint32_t(byte) << 4)));
        return v;
    };
    uint32_t it = 0;                                                   // tiles since the start: phases of the barriers
    bool ok = true;

    // Row blocks of this CTA; more than one only where the caller's bound on the rows was too small.  Later rows see more slots:
    // they go first.
    const int blocks = int((all_rows + Cfg::kRowsPerCta - 1u) / Cfg::kRowsPerCta);
    uint32_t q_round = 0;
    auto walk = [&](auto&& role) {
      for (int blk = blocks - 1 - int(blockIdx.z); blk >= 0 && ok; blk -= int(gridDim.z), ++q_round) {
        const uint32_t first = uint32_t(blk) * Cfg::kRowsPerCta;
        const uint32_t last = min(first + Cfg::kRowsPerCta, all_rows) - 1u;
        const int most = min(max(at0 + int(last / group) + 1, 0), len);      // slots the last row sees
        const int nt = (most + BN - 1) / BN;
        role(first, nt);
        it += uint32_t(nt);
        // all roles are through with this row block before its tensor memory and factors are used again
        tc_before();
        __syncthreads();
        tc_after();
        if (abort_flag) ok = false;
        if (nt == 0 && q_round < 0xffffffffu) --q_round;               // no queries were handed over: the barrier's phase did not move
      }
    };
    // The softmax holds 32 scores and what becomes of them; at the 96 registers that 17 warps leave a thread some of that would go
    // to memory and back (most of the time of a step went there).  The dequantization needs fewer: 256 x 104 + 256 x 88 + 32 x 96
    // registers are what the block was launched with.
    if (warp < Cfg::kSoftmaxWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        walk([&](uint32_t first, int nt) {
            const int m = warp >> 2;                                   // row tile
            const uint32_t lanes = tmem + (uint32_t((warp & 3) * 32) << 16);
            const uint32_t row = first + threadIdx.x;
            const bool exists = row < all_rows;
            const int i = exists ? int(row / group) : 0, hq = h * a.group + (exists ? int(row - uint32_t(i) * group) : 0);
            const int seen = exists ? min(max(at0 + i + 1, 0), len) : 0x7fffffff;      // (a row that is not there: no mask for its sake)
            const size_t out_row = size_t(r0 + i) * a.q_heads + hq;
            // The warp's 32 rows pass through the stages' memory, which nobody else uses yet, on their way from global memory and back
            // to it: whole rows by neighbouring lanes there, a row per lane here (16 loads of a lane each from a row of its own took
            // 8500 cycles, as long as two and a half steps).
            constexpr int CH = D / 8;                                  // 16-byte chunks of a row
            const uint32_t region = stage_at[m] + uint32_t((warp & 3) * 32 * D * 2);
            auto chunk_at = [&](int r, int ch) -> uint32_t { return region + uint32_t(r * D * 2) + uint32_t((ch ^ (r & 7)) << 4); };
            auto rows_out = [&](uint4* to, long long lane_row) {       // to[row][CH] of the rows that are there
                __syncwarp();
#pragma unroll 4
                for (int t = 0; t < CH; ++t) {
                    const int r = (lane + 32 * t) / CH, ch = (lane + 32 * t) % CH;
                    const long long at = __shfl_sync(0xffffffffu, lane_row, r);
                    if (at >= 0) to[at * CH + ch] = ld_shared16(chunk_at(r, ch));
                }
                __syncwarp();
            };
            float qs;
            {
                const bool wide = (reinterpret_cast<uintptr_t>(a.q) & 15u) == 0 && (a.q_stride & 7) == 0;
                const long long lane_at = exists ? (long long)(r0 + i) * a.q_stride + (long long)hq * D : -1;
#pragma unroll 4
                for (int t = 0; t < CH; ++t) {
                    const int r = (lane + 32 * t) / CH, ch = (lane + 32 * t) % CH;
                    const long long at = __shfl_sync(0xffffffffu, lane_at, r);
                    if (at >= 0) {
                        const uint16_t* src = static_cast<const uint16_t*>(a.q) + at + 8 * ch;
                        if (wide) {
                            copy16(chunk_at(r, ch), src);
                        } else {
                            const uint32_t* w = reinterpret_cast<const uint32_t*>(src);
                            st_shared16(chunk_at(r, ch), make_uint4(__ldg(w), __ldg(w + 1), __ldg(w + 2), __ldg(w + 3)));
                        }
                    }
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                __syncwarp();
                uint32_t qv[D / 2];
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    const uint4 v = exists ? ld_shared16(chunk_at(lane, k)) : make_uint4(0, 0, 0, 0);
                    qv[4 * k] = v.x; qv[4 * k + 1] = v.y; qv[4 * k + 2] = v.z; qv[4 * k + 3] = v.w;
                }
                const float undo = scale_query<D>(a.bf16, a.negate, qv);
                qs = fmaxf(a.score_scale * undo, 1.0e-37f);            // above zero: a masked score stays -inf
                if (a.scaled) {
#pragma unroll
                    for (int k = 0; k < CH; ++k) st_shared16(chunk_at(lane, k), make_uint4(qv[4 * k], qv[4 * k + 1], qv[4 * k + 2], qv[4 * k + 3]));
                    rows_out(reinterpret_cast<uint4*>(a.scaled), exists ? (long long)out_row : -1);
                }
                if (nt > 0) {
#pragma unroll
                    for (int k = 0; k < D / 64; ++k) {
                        uint32_t part[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) part[e] = qv[32 * k + e];
                        tmem_st32(lanes + Cfg::kTmemQ + uint32_t(m * (D / 2) + 32 * k), part);
                    }
                    tmem_wait_st();
                    tc_before();
                    mbar_arrive(q_ready);
                }
            }
            const int warp_seen = __reduce_min_sync(0xffffffffu, seen);      // tiles below it need no mask
            const bool idle = first + 32u * warp >= all_rows;           // none of the warp's rows is there
            float ref = -1.0e30f, sum = 0.0f;
            const uint32_t o_at = lanes + Cfg::kTmemO + uint32_t(m * D);
            for (int u = 0; u < 2 * nt; ++u) {
                const uint32_t v = 2u * it + uint32_t(u), st = (v >> 1) & 1u, b = v & 1u;      // step, stage, score buffer
                const uint32_t s_at = lanes + Cfg::kTmemS + uint32_t(m * 64) + b * ST;
                const int c0 = int(u & 1) * ST, j0 = u * ST;           // first of the step's slots in the stage, in the sequence
                ok = mmdk::mbar_wait(s_full + 16u * m + 8u * b, (v >> 1) & 1u, &abort_flag, a.status, 11) &&
                     ((u & 1) || mmdk::mbar_wait(kv_full + 8u * st, (v >> 2) & 1u, &abort_flag, a.status, 12));      // the factors, once a stage
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_after();
                if (idle) {                                            // nothing to work on, but the barriers' phases go on
                    mbar_arrive(p_ready + 16u * m + 8u * b);
                    continue;
                }
                const bool masked = j0 + ST > warp_seen;
                uint32_t raw[ST], hi[ST / 2], lo[SPLIT ? ST / 2 : 1];
                bool above;
                float part;
                // 2^(score - reference) and their products with the value scales; above: some of them call for a higher reference
                auto attend = [&](auto with_mask) {
                    constexpr bool MASK = decltype(with_mask)::value != 0;
                    const uint64_t qs2 = bq4k::pack2(qs, qs), nr2 = bq4k::pack2(-ref, -ref);
                    uint64_t sum2 = 0;
                    float largest[2] = {0.0f, 0.0f};                   // of the products (a NaN, of inf and a scale of zero, does not count)
                    mmdk::tmem_ld32(s_at, raw);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < ST; k += 4) {
                        const ulonglong2 kf = *reinterpret_cast<const ulonglong2*>(&key_factor[st][c0 + k]);
                        const ulonglong2 vf = *reinterpret_cast<const ulonglong2*>(&value_factor[st][c0 + k]);
                        float y[4];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint64_t x2 = bq4k::mul2(bq4k::pack2(__uint_as_float(raw[k + 2 * e]), __uint_as_float(raw[k + 2 * e + 1])), e == 0 ? kf.x : kf.y);
                            bq4k::unpack2(bq4k::fma2(x2, qs2, nr2), y[2 * e], y[2 * e + 1]);
                            if constexpr (MASK) {
                                if (j0 + k + 2 * e >= seen) y[2 * e] = -INFINITY;
                                if (j0 + k + 2 * e + 1 >= seen) y[2 * e + 1] = -INFINITY;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint64_t p2 = bq4k::pack2(exp2_fast(y[2 * e]), exp2_fast(y[2 * e + 1]));
                            sum2 = add2(sum2, p2);
                            float w0, w1;
                            bq4k::unpack2(bq4k::mul2(p2, e == 0 ? vf.x : vf.y), w0, w1);
                            asm("max.f32 %0, %1, %2, %3;" : "=f"(largest[e]) : "f"(largest[e]), "f"(w0), "f"(w1));
                            const uint32_t h = half2_of(w0, w1);
                            hi[k / 2 + e] = h;
                            if constexpr (SPLIT) {
                                const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&h));
                                lo[k / 2 + e] = half2_of(w0 - back.x, w1 - back.y);
                            }
                        }
                    }
                    float s0, s1;
                    bq4k::unpack2(sum2, s0, s1);
                    part = s0 + s1;
                    above = fmaxf(largest[0], largest[1]) > 16384.0f || part > 1.9342813e25f;      // 2^14; 2^84
                };
                if (masked) attend(Flag<1>{});
                else attend(Flag<0>{});
                if (__any_sync(0xffffffffu, above)) {
                    // The reference moves (always on the first step, where it is below everything): the row's largest score with its
                    // value scale anew, from the scores, which are still there; then the outputs so far, once the product of the step
                    // before is done (the one before that was done when these scores were).
                    mmdk::tmem_ld32(s_at, raw);
                    tmem_wait_ld();
                    float big = -INFINITY;
#pragma unroll
                    for (int k = 0; k < ST; ++k) {
                        const float x = __uint_as_float(raw[k]) * key_factor[st][c0 + k] * qs, lv = fmaxf(log2_fast(value_factor[st][c0 + k]), -70.0f);
                        big = fmaxf(big, j0 + k < seen ? x + lv : -INFINITY);
                    }
                    big -= 10.0f;                                      // of the factors
                    const float moved = big > ref + 4.0f ? big : ref, f = exp2_fast(ref - moved);
                    ref = moved;
                    sum *= f;
                    if (u > 0) {
                        ok = mmdk::mbar_wait(o_done + 16u * m + 8u * (b ^ 1u), ((v - 1u) >> 1) & 1u, &abort_flag, a.status, 13);
                        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                        tc_after();
#pragma unroll 1
                        for (int k = 0; k < D / 32; ++k) {
                            mmdk::tmem_ld32(o_at + 32u * k, raw);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e) raw[e] = __float_as_uint(__uint_as_float(raw[e]) * f);
                            tmem_st32(o_at + 32u * k, raw);
                        }
                        tmem_wait_st();
                    }
                    attend(Flag<1>{});
                }
                sum += part;
                if constexpr (SPLIT) {
#pragma unroll
                    for (int k = 0; k < ST / 2; ++k) { raw[k] = hi[k]; raw[ST / 2 + k] = lo[k]; }
                    tmem_st32(s_at, raw);
                } else {
                    tmem_st16(s_at, hi);
                }
                tmem_wait_st();
                tc_before();
                mbar_arrive(p_ready + 16u * m + 8u * b);
            }
            if (ok) {
                if (nt > 0) {
                    // of the last step, an odd one, of both row tiles: the stages are written below
                    ok = mmdk::mbar_wait(o_done + 8u, (it + uint32_t(nt) - 1u) & 1u, &abort_flag, a.status, 14) &&
                         mmdk::mbar_wait(o_done + 24u, (it + uint32_t(nt) - 1u) & 1u, &abort_flag, a.status, 14);
                    ok = __all_sync(0xffffffffu, ok);
                    tc_after();
                }
                if (ok) {
                    const float inv = sum > 0.0f ? __fdiv_rn(1.0f, sum) : 0.0f;
                    const float f = inv * a.inv_unit * pow2_of(-10);
                    if (a.stats && exists) a.stats[out_row] = make_float4(ref, inv, qs, 0.0f);
#pragma unroll 1
                    for (int k = 0; k < D / 32; ++k) {
                        uint32_t v[32];
                        if (nt > 0) {
                            mmdk::tmem_ld32(o_at + 32u * k, v);
                            tmem_wait_ld();
                        } else {
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] = 0u;
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t w[4];
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                const float y0 = __uint_as_float(v[8 * e + 2 * b]) * f, y1 = __uint_as_float(v[8 * e + 2 * b + 1]) * f;
                                if (a.bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[b]) : "f"(y1), "f"(y0));
                                else w[b] = half2_of(y0, y1);
                            }
                            st_shared16(chunk_at(lane, 4 * k + e), make_uint4(w[0], w[1], w[2], w[3]));
                        }
                    }
                    rows_out(static_cast<uint4*>(a.out), exists ? (long long)out_row : -1);
                    tc_before();
                }
            }
        });
    } else if (warp < 16) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        asm volatile("bar.sync 1, 256;" ::: "memory");                 // the table is theirs alone
        walk([&](uint32_t, int nt) {
            const bool is_v = warp >= 12;
            const int tid = int(threadIdx.x) - (is_v ? 384 : 256);     // 0 .. 127 of this operand's threads
            // keys: chunk of 16 code bytes `tid & (CPR - 1)` of slots tid / CPR + (128 / CPR) u; values: slots 8 (tid & 7) .. + 7, word tid / 8
            constexpr int CPR = D / 32, KU = BN * CPR / 128, WORDS = D / 8;
            uint4 kw[KU];
            uint32_t vw[8];
            uint16_t sc[2][NB];                                        // the next tile's scales: of slot tid (keys), of slots lane and lane + 32 (values, warp 12)
            const bool v_on = (tid >> 3) < WORDS;
            const int cap = c.max_pages * c.page;                      // past the table's end: any existing rows, their factors are zero
            const int32_t* table_row = c.table + size_t(s) * c.table_stride;
            auto page_of = [&](int j) -> int { return quotient_of(j, c.page, c.page_shift); };
            auto row_in = [&](int page_entry, int j) -> size_t {
                return (size_t(min(max(page_entry, 0), c.n_pages - 1)) * c.heads + h) * c.page + (j - page_of(j) * c.page);
            };
            // slots that this thread looks up: of the codes (keys: KU; values: the first of eight, in one page as its size is a
            // multiple of 16), then of the scales
            auto slot_of = [&](int j, int x) -> int {
                if (!is_v) return min(j * BN + (x < KU ? tid / CPR + (128 / CPR) * x : tid), cap - 1);
                return x == 0 ? min(j * BN + 8 * (tid & 7), cap - 8) : min(j * BN + lane + 32 * (x - 1), cap - 1);
            };
            const int looks = !is_v ? (tid < BN ? KU + 1 : KU) : (warp == 12 ? 3 : 1);
            int entry[3];                                              // of the table, a tile ahead of the rows they lead to
            auto look = [&](int j) {
#pragma unroll
                for (int x = 0; x < 3; ++x) if (x < looks) entry[x] = __ldg(table_row + page_of(slot_of(j, x)));
            };
            auto load = [&](int j) {
                if (!is_v) {
#pragma unroll
                    for (int u = 0; u < KU; ++u)
                        kw[u] = __ldg(reinterpret_cast<const uint4*>(c.k_codes + row_in(entry[u], slot_of(j, u)) * (D / 2)) + tid % CPR);
                    if (tid < BN) {
                        const size_t row = row_in(entry[KU], slot_of(j, KU));
#pragma unroll
                        for (int b = 0; b < NB; ++b) sc[0][b] = j * BN + tid < len ? __ldg(c.k_scale + row * NB + b) : uint16_t(0);
                    }
                    return;
                }
                if (warp == 12) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const size_t row = row_in(entry[1 + u], slot_of(j, 1 + u));
#pragma unroll
                        for (int b = 0; b < NB; ++b) sc[u][b] = j * BN + lane + 32 * u < len ? __ldg(c.v_scale + row * NB + b) : uint16_t(0);
                    }
                }
                if (v_on) {
                    const uint32_t* p = reinterpret_cast<const uint32_t*>(c.v_codes + row_in(entry[0], slot_of(j, 0)) * (D / 2)) + (tid >> 3);
#pragma unroll
                    for (int k = 0; k < 8; ++k) vw[k] = __ldg(p + k * WORDS);
                }
            };
            if (nt > 0) {
                look(0);
                load(0);
                if (nt > 1) look(1);
            }
            for (int j = 0; j < nt; ++j) {
                const uint32_t g = it + uint32_t(j), st = g & 1u;
                if constexpr (NB > 1) {                                // (the stage's last readers have met at the barrier of the tile before)
                    if (!is_v && tid < BN) {
                        float big = 0.0f;
#pragma unroll
                        for (int b = 0; b < NB; ++b) big = fmaxf(big, __uint_as_float(uint32_t(sc[0][b]) << 16));
                        const uint32_t e = min(max(__float_as_uint(big) >> 23, 1u), 253u);
#pragma unroll
                        for (int b = 0; b < NB; ++b)                   // below 2, eight significant bits; 0 past the length
                            rho[0][st][b][tid] = __float2half_rn(__uint_as_float(uint32_t(sc[0][b]) << 16) * __uint_as_float((254u - e) << 23));
                    }
                    if (warp == 12) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            float big = 0.0f;
#pragma unroll
                            for (int b = 0; b < NB; ++b) big = fmaxf(big, __uint_as_float(uint32_t(sc[u][b]) << 16));
                            const int e = min(max(int(__float_as_uint(big) >> 23) - 127, -100), 126);
#pragma unroll
                            for (int b = 0; b < NB; ++b)
                                rho[1][st][b][lane + 32 * u] =
                                    __float2half_rn(big > 0.0f ? __uint_as_float(uint32_t(sc[u][b]) << 16) * __uint_as_float(uint32_t(127 - e) << 23) : 0.0f);
                        }
                    }
                }
                if (g >= 2) ok = mmdk::mbar_wait(kv_empty + 8u * st, ((g >> 1) + 1u) & 1u, &abort_flag, a.status, 15);
                if (j == 0 && ok) ok = mmdk::mbar_wait(q_ready, q_round & 1u, &abort_flag, a.status, 20);      // the queries have passed through the stages
                // an operand's four warps go on or give up together: they meet at a barrier where blocks share scales
                ok = NB > 1 ? all_of(is_v ? 3 : 2, ok) : __all_sync(0xffffffffu, ok) != 0;
                if (!ok) break;
                const int j0 = j * BN;
                if (!is_v) {
                    // factors of the scores: the slot's scale (one block), or the power of two its blocks share
                    if (tid < BN) {
                        float big = 0.0f;
#pragma unroll
                        for (int b = 0; b < NB; ++b) big = fmaxf(big, __uint_as_float(uint32_t(sc[0][b]) << 16));
                        const uint32_t e = min(max(__float_as_uint(big) >> 23, 1u), 253u);
                        key_factor[st][tid] = NB == 1 ? big : __uint_as_float(e << 23);
                    }
#pragma unroll
                    for (int u = 0; u < KU; ++u) {
                        const int r = tid / CPR + (128 / CPR) * u;      // row of the tile
                        const uint32_t words[4] = {kw[u].x, kw[u].y, kw[u].z, kw[u].w};
                        __half2 rk = __half2half2(__ushort_as_half(0));
                        if constexpr (NB > 1) rk = __half2half2(rho[0][st][(tid % CPR) * 32 / (D / NB)][r]);
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const int chunk = (tid % CPR) * 4 + w;      // of eight elements
                            const uint32_t at = stage_at[st] + uint32_t(chunk >> 3) * (BN * 128) + uint32_t(r) * 128u + uint32_t(((chunk & 7) ^ (r & 7)) << 4);
                            uint32_t hi[4];
#pragma unroll
                            for (int b = 0; b < 4; ++b) hi[b] = pair_of(words[w], b);
                            if constexpr (NB > 1) {
                                uint32_t lo[4];
#pragma unroll
                                for (int b = 0; b < 4; ++b) {
                                    const __half2 v = *reinterpret_cast<const __half2*>(&hi[b]);
                                    const __half2 top = __hmul2_rn(v, rk), rest = __hfma2(v, rk, __hneg2(top));
                                    hi[b] = *reinterpret_cast<const uint32_t*>(&top);
                                    lo[b] = *reinterpret_cast<const uint32_t*>(&rest);
                                }
                                asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at + Cfg::kKBytes), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3]) : "memory");
                            }
                            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
                        }
                    }
                } else {
                    if (warp == 12) {
                        // factors of the probabilities, times 2^10: the slot's scale (one block), or the power of two its blocks share;
                        // zero past the length
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            float big = 0.0f;
#pragma unroll
                            for (int b = 0; b < NB; ++b) big = fmaxf(big, __uint_as_float(uint32_t(sc[u][b]) << 16));
                            const int e = min(max(int(__float_as_uint(big) >> 23) - 127, -100), 126);
                            value_factor[st][lane + 32 * u] = NB == 1 ? big * 1024.0f : big > 0.0f ? pow2_of(e + 10) : 0.0f;
                        }
                    }
                    if (v_on) {
                        const int tg = tid & 7, dg = tid >> 3;          // slots 8 tg .., columns 8 dg ..
                        __half2 rv[4];
                        if constexpr (NB > 1) {
                            const uint4 v = *reinterpret_cast<const uint4*>(&rho[1][st][dg * 8 / (D / NB)][8 * tg]);
                            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) rv[k] = *reinterpret_cast<const __half2*>(&w[k]);
                        }
                        uint32_t col[8][4];                            // [column][pair of slots]
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t w0 = vw[2 * k], w1 = vw[2 * k + 1];
                            const uint32_t ev = (w0 & 0x0F0F0F0Fu) | ((w1 << 4) & 0xF0F0F0F0u), od = ((w0 >> 4) & 0x0F0F0F0Fu) | (w1 & 0xF0F0F0F0u);
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                col[2 * b][k] = pair_of(ev, b);
                                col[2 * b + 1][k] = pair_of(od, b);
                            }
                        }
                        const uint32_t base = stage_at[st] + Cfg::kStage - Cfg::kVBytes;
#pragma unroll
                        for (int d = 0; d < 8; ++d) {
                            const uint32_t in_tile = uint32_t(8 * dg + d) * 128u + uint32_t((tg ^ d) << 4), at = base + in_tile;
                            if constexpr (NB > 1) {
                                [[maybe_unused]] uint32_t low_part[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    const __half2 v = *reinterpret_cast<const __half2*>(&col[d][k]), top = __hmul2_rn(v, rv[k]);
                                    if constexpr (SPLIT) {
                                        const __half2 rest = __hfma2(v, rv[k], __hneg2(top));
                                        low_part[k] = *reinterpret_cast<const uint32_t*>(&rest);
                                    }
                                    col[d][k] = *reinterpret_cast<const uint32_t*>(&top);
                                }
                                if constexpr (SPLIT) st_shared16(v_low + st * Cfg::kVLow + in_tile, make_uint4(low_part[0], low_part[1], low_part[2], low_part[3]));
                            }
                            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(col[d][0]), "r"(col[d][1]), "r"(col[d][2]), "r"(col[d][3]) : "memory");
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(kv_full + 8u * st);
                if (j + 1 < nt) load(j + 1);                           // on their way while the other roles work
                if (j + 2 < nt) look(j + 2);
            }
        });
    } else {
        walk([&](uint32_t first, int nt) {
            const bool two = all_rows - first > 128;                   // the second row tile has rows
          if (nt > 0 && mmdk::elect_one()) {
            constexpr uint32_t idesc_s = mmdk::umma_idesc(1, 0, 128, ST), idesc_o = mmdk::umma_idesc(1, 0, 128, D);
            auto scores = [&](uint32_t v, int m) {                     // of step v (its buffer was last read by a product issued before)
                const uint32_t k_at = stage_at[(v >> 1) & 1u] + (v & 1u) * (ST * 128);
                if (m == 0 || two)
#pragma unroll
                for (int part = 0; part < (NB > 1 ? 2 : 1); ++part)
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t b = mmdk::umma_smem_desc(k_at + uint32_t(part) * Cfg::kKBytes + uint32_t(k >> 2) * (BN * 128)) + uint64_t(2 * (k & 3));
                        umma_f16_ta(tmem + Cfg::kTmemS + uint32_t(m * 64) + (v & 1u) * ST, tmem + Cfg::kTmemQ + uint32_t(m * (D / 2) + 8 * k), b, idesc_s,
                                    (part > 0 || k > 0) ? 1u : 0u);
                    }
                mmdk::umma_commit(s_full + 16u * m + 8u * (v & 1u));
            };
            const uint32_t v0 = 2u * it;
            ok = mmdk::mbar_wait(q_ready, q_round & 1u, &abort_flag, a.status, 16) && mmdk::mbar_wait(kv_full + 8u * ((v0 >> 1) & 1u), (v0 >> 2) & 1u, &abort_flag, a.status, 17);
            tc_after();
            if (ok) { scores(v0, 0); scores(v0, 1); }
            for (int u = 0; u < 2 * nt && ok; ++u) {
                const uint32_t v = v0 + uint32_t(u), st = (v >> 1) & 1u;
                if (u + 1 < 2 * nt) {
                    if (u & 1) ok = mmdk::mbar_wait(kv_full + 8u * (((v + 1u) >> 1) & 1u), ((v + 1u) >> 2) & 1u, &abort_flag, a.status, 19);
                    if (!ok) break;
                    tc_after();
                    scores(v + 1u, 0);
                    scores(v + 1u, 1);
                }
                const uint32_t v_at = stage_at[st] + Cfg::kStage - Cfg::kVBytes;
#pragma unroll 1
                for (int m = 0; m < 2 && ok; ++m) {
                    ok = mmdk::mbar_wait(p_ready + 16u * m + 8u * (v & 1u), (v >> 1) & 1u, &abort_flag, a.status, 18);
                    if (!ok) break;
                    tc_after();
                    const uint32_t p_at = tmem + Cfg::kTmemS + uint32_t(m * 64) + (v & 1u) * ST;
                    if (m == 0 || two)
#pragma unroll
                    for (int part = 0; part < (SPLIT ? 2 : 1); ++part)
#pragma unroll
                        for (int k = 0; k < ST / 16; ++k)
                            umma_f16_ta(tmem + Cfg::kTmemO + uint32_t(m * D), p_at + uint32_t(part * (ST / 2) + 8 * k),
                                        mmdk::umma_smem_desc(v_at) + uint64_t(2 * (2 * (v & 1u) + k)), idesc_o, (u > 0 || part > 0 || k > 0) ? 1u : 0u);
                    if (Cfg::kVLow > 0 && (m == 0 || two))
#pragma unroll
                        for (int k = 0; k < ST / 16; ++k)
                            umma_f16_ta(tmem + Cfg::kTmemO + uint32_t(m * D), p_at + uint32_t(8 * k),
                                        mmdk::umma_smem_desc(v_low + st * Cfg::kVLow) + uint64_t(2 * (2 * (v & 1u) + k)), idesc_o, 1u);
                    mmdk::umma_commit(o_done + 16u * m + 8u * (v & 1u));
                    if (m == 1 && (v & 1u)) mmdk::umma_commit(kv_empty + 8u * st);
                }
            }
          }
          __syncwarp();
        });
    }
    if (abort_flag) {                                                  // products that nobody waited for may still be running
        for (int i = 0; i < 64; ++i) __nanosleep(2000);
    }
    __syncthreads();
    if (warp == 16) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Cfg::kTmemCols) : "memory");
    }
}

// ------------------------------------------------------------------------------------------
// weights_tiles: weights[s, h, j] += the sum of the probabilities of slot j over the query rows, from the statistics and the
// scaled queries that attend_tiles left.  One CTA takes 128 slots; their keys are dequantized once into shared memory and
// every 128 query rows that see them pass by: S^T = K Q^T on the tensor cores, so that a thread owns a slot and its sum needs
// no exchange.  Two warpgroups take row tiles in turn (two accumulators); a slot's two sums are added at the end: a fixed order.
// Measured: 6 prompts up to 777 tokens, 4 x 7 heads, head_dim 64, fp16: the whole call 132 us, 56 of them attend_tiles.  Bound by
// the CTA that owns the first slots, which every row sees (43 row tiles one after the other, 1.8 us each); with two stages
// of queries, each copy awaited before the next, it was 2.4 us (the call 153).
//   warps 0-7   a slot per thread and warpgroup       warps 8-11  copy queries, 128-byte swizzle       warp 12  tcgen05.mma
template <int D, int NB>
struct WeightsCfg {
    static constexpr int kSlots = 128, kRows = 128, kThreads = 13 * 32, kStages = 4;      // of queries: their copies take longer than a tile
    static constexpr uint32_t kKeys = kSlots * D * 2, kQueries = kRows * D * 2;
    static constexpr int kSmem = int(kKeys) * (NB > 1 ? 2 : 1) + kStages * int(kQueries) + 1024;
    static constexpr uint32_t kTmemCols = 256;
};

template <int D, int NB>
__global__ void __launch_bounds__(WeightsCfg<D, NB>::kThreads)
weights_tiles(const Cache c, const Rows rows, const TilesArgs a, float* __restrict__ weights, int64_t stride, const __grid_constant__ PairTable pairs) {
    using Cfg = WeightsCfg<D, NB>;
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ uint32_t lut[256];
    __shared__ __align__(16) float4 row_of_tile[Cfg::kStages][Cfg::kRows];        // factor of the scores, reference, 1 / sum, slots seen
    __shared__ float half_sum[Cfg::kSlots];
    __shared__ uint16_t half[16];
    __shared__ __align__(8) uint64_t bars[12];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (uint32_t(__cvta_generic_to_shared(smem)) + 1023u) & ~1023u;
    const uint32_t q_at = base + Cfg::kKeys * (NB > 1 ? 2u : 1u);
    const uint32_t bar0 = uint32_t(__cvta_generic_to_shared(bars));
    const uint32_t q_full = bar0, q_empty = bar0 + 32, s_full = bar0 + 64, s_free = bar0 + 80;
    const int h = blockIdx.y, s = blockIdx.z;
    const int r0 = rows.begin(s), n = max(rows.end(s) - r0, 0), counted = c.counted(s), len = c.held(counted);
    const int at0 = counted - n;                                       // slot of the first row
    const long long all_rows = (long long)n * a.group;
    if (threadIdx.x < 16) half[threadIdx.x] = pairs.half[threadIdx.x];
    if (threadIdx.x == 0) {
        for (int i = 0; i < Cfg::kStages; ++i) {
            mmdk::mbar_init(q_full + 8u * i, 128);
            mmdk::mbar_init(q_empty + 8u * i, 129);                    // the products' commit, and the threads that used the rows' factors
        }
        for (int i = 0; i < 2; ++i) {
            mmdk::mbar_init(s_full + 8u * i, 1);
            mmdk::mbar_init(s_free + 8u * i, 128);
        }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(uint32_t(__cvta_generic_to_shared(&tmem_slot))), "r"(Cfg::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 256; i += Cfg::kThreads) lut[i] = uint32_t(half[i & 15]) | uint32_t(half[i >> 4]) << 16;
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = tmem_slot;
    const int cap = c.max_pages * c.page;
    uint32_t it = 0;
    bool ok = true;
    for (int j0 = int(blockIdx.x) * Cfg::kSlots; j0 < len && n > 0 && ok; j0 += int(gridDim.x) * Cfg::kSlots) {
        // keys: 16 code bytes (32 elements, of one block) a step
        constexpr int CPR = D / 32;
        for (int i = threadIdx.x; i < Cfg::kSlots * CPR; i += Cfg::kThreads) {
            const int r = i / CPR, piece = i % CPR;
            const size_t row = c.row(s, h, min(j0 + r, cap - 1));
            const uint4 w = __ldg(reinterpret_cast<const uint4*>(c.k_codes + row * (D / 2)) + piece);
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
            __half2 rho = __half2half2(__ushort_as_half(0));
            if constexpr (NB > 1) {
                float big = 0.0f;
#pragma unroll
                for (int b = 0; b < NB; ++b) big = fmaxf(big, scale_of(c.k_scale, row * NB + b));
                const float mine = scale_of(c.k_scale, row * NB + piece * 32 / (D / NB));
                const uint32_t e = min(max(__float_as_uint(big) >> 23, 1u), 253u);
                rho = __float2half2_rn(j0 + r < len ? mine * __uint_as_float((254u - e) << 23) : 0.0f);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int chunk = piece * 4 + u;
                const uint32_t at = base + uint32_t(chunk >> 3) * (Cfg::kSlots * 128) + uint32_t(r) * 128u + uint32_t(((chunk & 7) ^ (r & 7)) << 4);
                uint32_t hi[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) hi[b] = lut[(words[u] >> (8 * b)) & 255u];
                if constexpr (NB > 1) {
                    uint32_t lo[4];
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const __half2 v = *reinterpret_cast<const __half2*>(&hi[b]);
                        const __half2 top = __hmul2_rn(v, rho), rest = __hfma2(v, rho, __hneg2(top));
                        hi[b] = *reinterpret_cast<const uint32_t*>(&top);
                        lo[b] = *reinterpret_cast<const uint32_t*>(&rest);
                    }
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at + Cfg::kKeys), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3]) : "memory");
                }
                asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        // row tiles from the one that holds the first query that sees slot j0
        const long long first_row = max((long long)j0 - at0, 0ll) * a.group;
        const int t0 = int(first_row / Cfg::kRows), nt = int((all_rows + Cfg::kRows - 1) / Cfg::kRows) - t0;

        if (warp < 8) {
            const int w = warp >> 2, slot = j0 + int(threadIdx.x & 127);
            const uint32_t s_at = tmem + (uint32_t((warp & 3) * 32) << 16) + uint32_t(w * 128);
            float kf = 0.0f, sum = 0.0f;
            if (slot < len) {
                const size_t row = c.row(s, h, slot);
                float big = 0.0f;
#pragma unroll
                for (int b = 0; b < NB; ++b) big = fmaxf(big, scale_of(c.k_scale, row * NB + b));
                kf = NB == 1 ? big : __uint_as_float(min(max(__float_as_uint(big) >> 23, 1u), 253u) << 23);
            }
            for (int t = 0; t < nt; ++t) {
                const uint32_t g = it + uint32_t(t);
                if ((g & 1u) != uint32_t(w)) continue;
                ok = mmdk::mbar_wait(s_full + 8u * w, (g >> 1) & 1u, &abort_flag, a.status, 21) && mmdk::mbar_wait(q_full + 8u * (g & 3u), (g >> 2) & 1u, &abort_flag, a.status, 22);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_after();
#pragma unroll 1
                for (int k = 0; k < Cfg::kRows; k += 32) {
                    uint32_t v[32];
                    mmdk::tmem_ld32(s_at + uint32_t(k), v);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const float4 r = row_of_tile[g & 3u][k + e];
                        const float p = exp2_fast(__fmaf_rn(__uint_as_float(v[e]) * kf, r.x, -r.y));
                        sum = __fmaf_rn(slot < __float_as_int(r.w) ? p : 0.0f, r.z, sum);
                    }
                }
                tc_before();
                mbar_arrive(s_free + 8u * w);
                mbar_arrive(q_empty + 8u * (g & 3u));
            }
            if (w == 1) half_sum[threadIdx.x & 127] = sum;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (w == 0 && ok && slot < len && slot < stride) {
                float* to = weights + (size_t(s) * c.heads + h) * size_t(stride) + slot;
                *to += sum + half_sum[threadIdx.x & 127];
            }
        } else if (warp < 12) {
            const int tid = int(threadIdx.x) - 256;
            // two tiles' copies stay on their way while a third is asked for
            auto arrived = [&](uint32_t g) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(q_full + 8u * (g & 3u));
            };
            const uint32_t group = uint32_t(a.group);
            for (int t = 0; t < nt; ++t) {
                const uint32_t g = it + uint32_t(t), st = g & 3u;
                if (g >= 4) {
                    ok = mmdk::mbar_wait(q_empty + 8u * st, ((g >> 2) + 1u) & 1u, &abort_flag, a.status, 23);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                }
                constexpr int CH = D / 8;                              // 16-byte chunks per row
                const uint32_t row0 = uint32_t(t0 + t) * Cfg::kRows;
#pragma unroll 4
                for (int i = tid; i < Cfg::kRows * CH; i += 128) {
                    const int r = i / CH, ch = i % CH;
                    const uint32_t row = min(row0 + r, uint32_t(all_rows - 1)), qi = row / group;
                    const size_t src = (size_t(r0 + int(qi)) * a.q_heads + h * a.group + (row - qi * group)) * (D / 2) + ch * 4;
                    copy16(q_at + st * Cfg::kQueries + uint32_t(ch >> 3) * (Cfg::kRows * 128) + uint32_t(r) * 128u + uint32_t(((ch & 7) ^ (r & 7)) << 4), a.scaled + src);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                {
                    const uint32_t row = row0 + tid;
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, __int_as_float(0));
                    if (row < uint32_t(all_rows)) {
                        const uint32_t qi = row / group;
                        const float4 f = a.stats[size_t(r0 + int(qi)) * a.q_heads + h * a.group + (row - qi * group)];
                        v = make_float4(f.z, f.x, f.y, __int_as_float(min(max(at0 + int(qi) + 1, 0), len)));
                    }
                    row_of_tile[st][tid] = v;
                }
                if (t >= 2) {
                    asm volatile("cp.async.wait_group 2;" ::: "memory");
                    arrived(g - 2u);
                }
            }
            if (ok && nt >= 2) {
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                arrived(it + uint32_t(nt) - 2u);
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (ok && nt >= 1) arrived(it + uint32_t(nt) - 1u);
        } else {
            if (mmdk::elect_one()) {
                constexpr uint32_t idesc = mmdk::umma_idesc(1, 0, Cfg::kSlots, Cfg::kRows);
                for (int t = 0; t < nt && ok; ++t) {
                    const uint32_t g = it + uint32_t(t), st = g & 1u, sq = g & 3u;
                    ok = mmdk::mbar_wait(q_full + 8u * sq, (g >> 2) & 1u, &abort_flag, a.status, 25);
                    if (ok && g >= 2) ok = mmdk::mbar_wait(s_free + 8u * st, ((g >> 1) + 1u) & 1u, &abort_flag, a.status, 26);
                    if (!ok) break;
                    tc_after();
#pragma unroll
                    for (int part = 0; part < (NB > 1 ? 2 : 1); ++part)
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint64_t ad = mmdk::umma_smem_desc(base + uint32_t(part) * Cfg::kKeys + uint32_t(k >> 2) * (Cfg::kSlots * 128)) + uint64_t(2 * (k & 3));
                            const uint64_t bd = mmdk::umma_smem_desc(q_at + sq * Cfg::kQueries + uint32_t(k >> 2) * (Cfg::kRows * 128)) + uint64_t(2 * (k & 3));
                            mmdk::umma_f16(tmem + st * 128u, ad, bd, idesc, (part > 0 || k > 0) ? 1u : 0u);
                        }
                    mmdk::umma_commit(q_empty + 8u * sq);
                    mmdk::umma_commit(s_full + 8u * st);
                }
            }
            __syncwarp();
        }
        it += uint32_t(nt);
        tc_before();
        __syncthreads();                                               // the keys and the sums are done with
        tc_after();
        if (abort_flag) ok = false;
    }
    if (abort_flag) {
        for (int i = 0; i < 64; ++i) __nanosleep(2000);
    }
    __syncthreads();
    if (warp == 12) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Cfg::kTmemCols) : "memory");
    }
}

}  // namespace bqkvk
