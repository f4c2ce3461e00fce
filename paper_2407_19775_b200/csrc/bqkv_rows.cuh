// bqkv_rows.cuh -- attention of a few query rows per cached head over the 4-bit cache (a decode
// step): attend_rows, attend_rows_finish and attend_rows_weights (sm_100a).
//
// The step is bound by the stream of cache rows (D + 4 D / block bytes per token and head) as long
// as a token costs few instructions, so everything here is about instructions per cached element.
//
//   dequantize   a byte (two codes) is one lookup of a pair of fp16 values.  The 256 pairs sit in
//                shared memory once per lane, each lane in its own bank (no conflicts), 256 bytes
//                apart, so that ONE byte permute builds the address: code byte in byte 1, lane * 4 in
//                byte 0.  Two instructions per pair.
//   exact values the pairs hold value * unit, with the unit chosen on the host so that all sixteen
//                are fp16 numbers (the dynamic tree: integers up to 2000); the block scales never
//                touch them.  Scales of keys multiply the scores, one fp32 accumulator per block;
//                scales of values multiply the probabilities.
//   products     mma.sync m16n8k16 with the CACHE in the 16-row operand and up to eight query rows in
//                the 8-column one: S^T = K Q^T, O^T = V^T P^T.  tcgen05 has no shape for this (at
//                least 64 rows, operands through shared memory, while here the dequantized pairs are
//                already in registers), and tensor throughput is not what bounds the step.
//   transposes   V^T wants pairs of TOKENS of one column.  Two words of codes of two tokens give the
//                words of pairs with two shifts and two bitwise selects per 16 elements, before the
//                lookup.  P^T is the score fragment through movmatrix.
//   softmax      running reference per row, moved only when a score exceeds it by 8 (in log2).  A
//                token's value scale enters as 2^e vs' (1 <= vs' < 2): e joins the exponent before the
//                reference is subtracted, so that the fp16 probabilities cannot overflow and what they
//                lose is small against the row's largest product of probability and scale.
//   split        the tiles of 32 tokens of all (sequence, head) pairs, numbered in order, are dealt
//                out evenly over the warps of the grid (ragged batches stay balanced); a warp's range
//                starts and ends inside a pair at most once each, so it leaves at most two partial
//                results, which attend_rows_finish joins in warp order (no atomics).
#pragma once

#include "bqkv_kernels.cuh"

namespace bqkvk {

struct PairTable {                         // the sixteen values times `unit`, as fp16 bits
    uint16_t half[16];
};

struct RowsArgs {
    const void* q;
    int64_t q_stride;
    int bf16, q_heads, group;
    float score_scale;                     // sm_scale * log2(e) / unit
    float inv_unit;                        // of the values
    void* out;
    float* partial;                        // 2 slots per warp: [row][dim] sums, then [row] references and sums
    long long* prefix;                     // n_seq + 1: tiles before each sequence, written for attend_rows_finish
    float2* stats;                         // (reference, 1 / sum) of every (row, query head); may be null
    float* scores;                         // [n_seq, heads, score_rows, score_len] in log2 units; may be null
    int score_rows, score_len;
    int warps;                             // warps of the grid
};

template <int D, int NB, int NT>
struct RowsCfg {
    static constexpr int kRows = 8 * NT;                               // query rows a warp works on
    static constexpr int kWarps = NT == 1 ? 16 : 12;
    static constexpr int kTile = 32;                                   // tokens
    static constexpr int kRowBytes = D / 2;
    static constexpr int kCodes = kTile * kRowBytes;                   // bytes of one operand's codes in a stage
    static constexpr int kScales = kTile * NB * 2;
    static constexpr int kStage = 2 * kCodes + 2 * kScales;
    static constexpr int kStages = NT == 1 ? 2 : 3;
    static constexpr int kTable = 256 * 256;
    static constexpr int kSmem = kTable + kWarps * kStages * kStage;
    static constexpr int kSlot = kRows * D + 2 * kRows;                // floats of a partial result
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// Where the tiles of the call lie: the sequence of a tile and what is needed to walk on from there.
struct Walk {
    int s, h, rg, tile;                    // sequence, cached head, group of query rows, tile of the sequence
    int len, n, r0, tiles, groups;         // slots, rows of the call, first of them, tiles, groups of query rows
};

template <int ROWS, int TILE>
__device__ __forceinline__ void walk_load(const Cache& c, const Rows& rows, int group, Walk& w) {
    w.r0 = rows.begin(w.s);
    w.n = max(rows.end(w.s) - w.r0, 0);
    w.len = c.len(w.s);
    w.groups = (w.n * group + ROWS - 1) / ROWS;
    w.tiles = w.groups > 0 ? (w.len + TILE - 1) / TILE : 0;
}
template <int ROWS, int TILE>
__device__ __forceinline__ bool walk_next(const Cache& c, const Rows& rows, int group, Walk& w) {      // true when a new (head, row group) begins
    if (++w.tile < w.tiles) return false;
    w.tile = 0;
    if (++w.rg == w.groups) {
        w.rg = 0;
        if (++w.h == c.heads) {
            w.h = 0;
            do {
                if (++w.s >= c.n_seq) { w.s = c.n_seq; return true; }
                walk_load<ROWS, TILE>(c, rows, group, w);
            } while (w.tiles == 0);
        }
    }
    return true;
}

// Tiles before each sequence, by one CTA: the total is returned to all threads; with `find` the sequence that holds tile
// `find` of thread 0's choosing is looked for as well.  `base` receives the tiles before that sequence.
template <int ROWS, int TILE>
__device__ __forceinline__ long long count_tiles(const Cache& c, const Rows& rows, int group, long long* scratch /* shared, one per warp + 1 */,
                                                 long long* prefix /* global or null */) {
    long long total = 0;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = blockDim.x >> 5;
    for (int s0 = 0; s0 < c.n_seq; s0 += blockDim.x) {
        Walk w;
        w.s = s0 + threadIdx.x;
        long long t = 0;
        if (w.s < c.n_seq) {
            walk_load<ROWS, TILE>(c, rows, group, w);
            t = (long long)w.tiles * w.groups * c.heads;
        }
        long long inc = t;
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const long long o = __shfl_up_sync(0xffffffffu, inc, k);
            if (lane >= k) inc += o;
        }
        if (lane == 31) scratch[wid] = inc;
        __syncthreads();
        long long before = 0, all = 0;
        for (int i = 0; i < nw; ++i) {
            const long long v = scratch[i];
            before += i < wid ? v : 0;
            all += v;
        }
        if (prefix && w.s < c.n_seq) prefix[w.s] = total + before + inc - t;
        total += all;
        __syncthreads();
    }
    if (prefix && threadIdx.x == 0) prefix[c.n_seq] = total;
    return total;
}

// The warps that share T tiles: one tile each at least.  Warp w takes tiles [T w / W, T (w + 1) / W).
__device__ __forceinline__ long long active_warps(long long total, int warps) { return total < warps ? total : warps; }
__device__ __forceinline__ int owner_of(long long tile, long long total, long long warps) { return int(((tile + 1) * warps + total - 1) / total) - 1; }

template <int D, int NB, int NT>
__global__ void __launch_bounds__(RowsCfg<D, NB, NT>::kWarps * 32, 1)
attend_rows(const Cache c, const Rows rows, const RowsArgs a, const __grid_constant__ PairTable pairs) {
    using Cfg = RowsCfg<D, NB, NT>;
    constexpr int KS = D / 16;                                         // k steps of the scores = row tiles of the outputs
    constexpr int KSB = KS / NB;                                       // of one block
    extern __shared__ __align__(256) unsigned char smem[];
    __shared__ long long scratch[Cfg::kWarps + 1];
    __shared__ uint16_t half[16];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    if (threadIdx.x < 16) half[threadIdx.x] = pairs.half[threadIdx.x];
    const long long total = count_tiles<Cfg::kRows, Cfg::kTile>(c, rows, a.group, scratch, blockIdx.x == 0 ? a.prefix : nullptr);
    // consecutive warps of the order sit in different CTAs, so that little work still spreads over all SMs
    const long long W = active_warps(total, a.warps), me = (long long)wid * gridDim.x + blockIdx.x;
    if (blockIdx.x >= W) return;                                       // no warp of this CTA has any tile
    const long long lo = me < W ? total * me / W : 0, hi = me < W ? total * (me + 1) / W : 0;

    // the sequence that holds tile `lo`
    Walk ld = {};
    if (lo < hi) {
        long long left = lo;
        for (int s0 = 0;; s0 += 32) {                                  // 32 sequences a step; lo < total, so one holds it
            ld.s = s0 + lane;
            long long n = 0;
            if (ld.s < c.n_seq) {
                walk_load<Cfg::kRows, Cfg::kTile>(c, rows, a.group, ld);
                n = (long long)ld.tiles * ld.groups * c.heads;
            }
            long long inc = n;
#pragma unroll
            for (int k = 1; k < 32; k <<= 1) {
                const long long o = __shfl_up_sync(0xffffffffu, inc, k);
                if (lane >= k) inc += o;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, left < inc);
            if (hit) {
                const int w = __ffs(hit) - 1;
                ld.s = s0 + w;
                left -= __shfl_sync(0xffffffffu, inc - n, w);
                break;
            }
            left -= __shfl_sync(0xffffffffu, inc, 31);
        }
        walk_load<Cfg::kRows, Cfg::kTile>(c, rows, a.group, ld);
        ld.tile = int(left % ld.tiles);
        const int pair = int(left / ld.tiles);
        ld.rg = pair % ld.groups;
        ld.h = pair / ld.groups;
    }
    Walk cu = ld;

    const uint32_t table = uint32_t(__cvta_generic_to_shared(smem)), lane4 = uint32_t(lane) * 4u;
    const uint32_t ring = table + Cfg::kTable + uint32_t(wid) * Cfg::kStages * Cfg::kStage;
    auto pair_of = [&](uint32_t word, int byte) -> uint32_t {          // the fp16 pair of byte `byte` of a word of codes
        return *reinterpret_cast<const uint32_t*>(smem + bq4k::prmt(word, lane4, 0x5504u | uint32_t(byte) << 4));
    };
    // Where a row's 16-byte chunk sits in its region: xor-ed so that the fragment reads below meet no bank twice.
    auto chunk_at = [](int row, int chunk) -> uint32_t {
        return uint32_t(row * Cfg::kRowBytes + ((D == 128 ? chunk ^ ((row >> 1) & 3) : chunk ^ ((row >> 2) & 1)) << 4));
    };
    // Token, within its group of 16, of row i of the score fragment (i < 8; i + 8 is 8 further).  Chosen with the xor above:
    // the rows one key read covers (2, 4 or 8 of them) and the rows one value read covers (those of 2t, or of 2t + 1, for
    // t = 0..3) fall into different banks.
    auto token_of = [](int i) -> int {
        return D == 128 ? int((0x67235410u >> (4 * i)) & 7u) : int((0x53427160u >> (4 * i)) & 7u);
    };

    auto fetch = [&](const Walk& w, int stage) {
        const uint32_t st = ring + uint32_t(stage) * Cfg::kStage;
        const int j0 = w.tile * Cfg::kTile;
        constexpr int CPR = Cfg::kRowBytes / 16;                       // chunks per row
#pragma unroll
        for (int u = 0; u < 2; ++u) {                                  // 16 tokens lie in one page (its size is a multiple of 16)
            const int j = min(j0 + 16 * u, c.max_pages * c.page - 16); // past the table's end: any existing group, its scores are masked
            const size_t row = c.row(w.s, w.h, j);
#pragma unroll
            for (int k = 0; k < 16 * CPR; k += 32) {
                const int i = k + lane, r = i / CPR, ch = i % CPR;
                const uint32_t dst = st + chunk_at(16 * u + r, ch);
                copy16(dst, c.k_codes + row * Cfg::kRowBytes + size_t(i) * 16);
                copy16(dst + Cfg::kCodes, c.v_codes + row * Cfg::kRowBytes + size_t(i) * 16);
            }
            if (lane < 4 * NB) {
                const int i = lane % (2 * NB);
                const bool is_v = lane >= 2 * NB;
                const uint32_t dst = st + 2 * Cfg::kCodes + (is_v ? Cfg::kScales : 0) + uint32_t(u * 16 * NB * 2 + i * 16);
                copy16(dst, reinterpret_cast<const char*>(is_v ? c.v_scale : c.k_scale) + row * NB * 2 + size_t(i) * 16);
            }
        }
    };
    auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };

    uint32_t qf[NT][KS][2];                                            // query fragments
    float qs[NT][2];                                                   // factor of the scores of this thread's rows 2t, 2t + 1
    int seen[NT][2];                                                   // slots those rows see (0: no such row)
    float o[NT][KS][4], ref[NT][2], sum[NT][2];
    bool whole;                                                        // this warp has all tiles of the current pair

    auto begin = [&](const Walk& w) {                                  // the queries of a (sequence, head, row group)
        float mine[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = w.rg * Cfg::kRows + nt * 8 + g;              // row of the pair: query row r / group, head r % group
            const bool in = r < w.n * a.group;
            const int i = in ? r / a.group : 0, hq = w.h * a.group + (in ? r % a.group : 0);
            const uint32_t* q = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(a.q) + size_t(w.r0 + i) * size_t(a.q_stride) + size_t(hq) * D);
            uint32_t raw[KS][2];
            float big = 0.0f;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int k = 0; k < KSB; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {                      // byte 2k + e of this thread's piece of block b
                        const uint32_t v = in ? __ldg(q + (b * (D / NB) + t * (D / NB / 4)) / 2 + 2 * k + e) : 0u;
                        raw[b * KSB + k][e] = v;
                        const float x = a.bf16 ? __uint_as_float(v << 16) : __low2float(*reinterpret_cast<const __half2*>(&v));
                        const float y = a.bf16 ? __uint_as_float(v & 0xffff0000u) : __high2float(*reinterpret_cast<const __half2*>(&v));
                        big = fmaxf(big, fmaxf(fabsf(x), fabsf(y)));
                    }
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
            // A power of two brings the row's largest element to [2^14, 2^15): exact, down to 2^-29 of it.
            const int ex = big > 0.0f ? int(__float_as_uint(big) >> 23) - 127 : 0;
            const float up = ldexpf(1.0f, min(max(14 - ex, -126), 126));
            mine[nt] = in ? a.score_scale * ldexpf(1.0f, -min(max(14 - ex, -126), 126)) : 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t v = raw[k][e];
                    const float x = a.bf16 ? __uint_as_float(v << 16) : __low2float(*reinterpret_cast<const __half2*>(&v));
                    const float y = a.bf16 ? __uint_as_float(v & 0xffff0000u) : __high2float(*reinterpret_cast<const __half2*>(&v));
                    qf[nt][k][e] = half2_of(x * up, y * up);
                }
            const int last = in ? min(max(w.len - w.n + i + 1, 0), w.len) : 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {                              // this thread's score columns are rows 2t + e
                qs[nt][e] = __shfl_sync(0xffffffffu, mine[nt], 4 * (2 * t + e));
                seen[nt][e] = __shfl_sync(0xffffffffu, last, 4 * (2 * t + e));
                ref[nt][e] = -INFINITY;
                sum[nt][e] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][k][e] = 0.0f;
        }
    };

    // column of output row tile mt, this thread: pair (even, odd) starting here
    constexpr int PB = Cfg::kRowBytes / (8 * NB);                      // value bytes per thread, row and block: 8, 4 or 2
    auto column_of = [&](int mt) -> int { return (mt / PB) * (D / NB) + g * 2 * PB + 2 * (mt % PB); };

    // Ends the current pair: the final rows, or one of this warp's two partial slots.
    auto finish = [&](const Walk& w, bool from_start) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int k = 4; k <= 16; k <<= 1) sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], k);
            }
        if (whole) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = w.rg * Cfg::kRows + nt * 8 + 2 * t + e;
                    if (r >= w.n * a.group) continue;
                    const size_t at = size_t(w.r0 + r / a.group) * a.q_heads + w.h * a.group + r % a.group;
                    const float inv = sum[nt][e] > 0.0f ? __fdiv_rn(1.0f, sum[nt][e]) : 0.0f;
                    if (a.stats && g == 0) a.stats[at] = make_float2(ref[nt][e], inv);
                    const float f = inv * a.inv_unit;
                    uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + at * D);
#pragma unroll
                    for (int mt = 0; mt < KS; ++mt) {
                        const float x = o[nt][mt][e] * f, y = o[nt][mt][2 + e] * f;
                        uint32_t v;
                        if (a.bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(y), "f"(x));
                        else v = half2_of(x, y);
                        out[column_of(mt) / 2] = v;
                    }
                }
        } else {
            float* slot = a.partial + (size_t(me) * 2 + (from_start ? 1 : 0)) * Cfg::kSlot;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = nt * 8 + 2 * t + e;
#pragma unroll
                    for (int mt = 0; mt < KS; ++mt)
                        *reinterpret_cast<float2*>(slot + r * D + column_of(mt)) = make_float2(o[nt][mt][e], o[nt][mt][2 + e]);
                    if (g == 0) { slot[Cfg::kRows * D + r] = ref[nt][e]; slot[Cfg::kRows * D + Cfg::kRows + r] = sum[nt][e]; }
                }
        }
    };

    auto scale16 = [](uint32_t addr) -> float {
        uint16_t v;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
        return __uint_as_float(uint32_t(v) << 16);
    };

    auto compute = [&](const Walk& w, int stage) {
        const uint32_t st = ring + uint32_t(stage) * Cfg::kStage, ksc = st + 2 * Cfg::kCodes, vsc = ksc + Cfg::kScales;
        const int j0 = w.tile * Cfg::kTile;
        float sc[2][NT][4];                                            // scores: group u, tokens g (0, 1) and g + 8 (2, 3), rows 2t (0, 2) and 2t + 1 (1, 3)
        int tok[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int e = 0; e < 2; ++e) tok[u][e] = 16 * u + 8 * e + token_of(g);
            uint32_t kw[2][D / 32];                                    // this thread's codes of the two tokens: D / 8 bytes each
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    constexpr int PK = Cfg::kRowBytes / (4 * NB);      // bytes per thread and block: 16, 8 or 4
                    const int byte = b * (Cfg::kRowBytes / NB) + t * PK;
                    const uint32_t at = st + chunk_at(tok[u][e], byte >> 4) + uint32_t(byte & 15);
                    if constexpr (PK == 16) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(kw[e][0]), "=r"(kw[e][1]), "=r"(kw[e][2]), "=r"(kw[e][3]) : "r"(at));
                    else if constexpr (PK == 8) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(kw[e][2 * b]), "=r"(kw[e][2 * b + 1]) : "r"(at));
                    else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(kw[e][b]) : "r"(at));
                }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[u][nt][e] = 0.0f;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float acc[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[nt][e] = 0.0f;
#pragma unroll
                for (int k = 0; k < KSB; ++k) {
                    const int i = 2 * (b * KSB + k);                   // byte within the thread's D / 8
                    const uint32_t a0 = pair_of(kw[0][i >> 2], i & 3), a1 = pair_of(kw[1][i >> 2], i & 3);
                    const uint32_t a2 = pair_of(kw[0][i >> 2], (i & 3) + 1), a3 = pair_of(kw[1][i >> 2], (i & 3) + 1);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(acc[nt], a0, a1, a2, a3, qf[nt][b * KSB + k][0], qf[nt][b * KSB + k][1]);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float ks = scale16(ksc + uint32_t((tok[u][e] * NB + b) * 2));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        sc[u][nt][2 * e] = __fmaf_rn(acc[nt][2 * e], ks, sc[u][nt][2 * e]);
                        sc[u][nt][2 * e + 1] = __fmaf_rn(acc[nt][2 * e + 1], ks, sc[u][nt][2 * e + 1]);
                    }
                }
            }
        }
        // value scales: vs = 2^e vs'; a token past the length gets e = 0, vs' = 0 (its bytes may be anything)
        float vs[2][2][NB], ve[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bool in = j0 + tok[u][e] < w.len;
                uint32_t raw[NB], top = 0;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    uint16_t v;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(vsc + uint32_t((tok[u][e] * NB + b) * 2)));
                    raw[b] = in ? uint32_t(v) << 16 : 0u;
                    top = max(top, raw[b]);
                }
                const int ex = min(max(int(top >> 23) - 127, -100), 100);
                const float down = __uint_as_float(uint32_t(127 - ex) << 23);
                ve[u][e] = float(ex);
#pragma unroll
                for (int b = 0; b < NB; ++b) vs[u][e][b] = __fmul_rn(__uint_as_float(raw[b]), down);
            }
        // scores in log2 units, masked; the running reference
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + tok[u][e >> 1];
                    const float x = j < seen[nt][e & 1] ? __fmul_rn(sc[u][nt][e], qs[nt][e & 1]) : -INFINITY;
                    sc[u][nt][e] = x;
                    top[e & 1] = fmaxf(top[e & 1], x + ve[u][e >> 1]);
                }
            if (__any_sync(0xffffffffu, top[0] > ref[nt][0] + 8.0f || top[1] > ref[nt][1] + 8.0f)) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float m = fmaxf(top[e], ref[nt][e]);
#pragma unroll
                    for (int k = 4; k <= 16; k <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
                    const float f = ref[nt][e] == m ? 1.0f : exp2_fast(ref[nt][e] - m);      // 1 also where nothing is seen yet
                    ref[nt][e] = m;
                    sum[nt][e] *= f;
#pragma unroll
                    for (int mt = 0; mt < KS; ++mt) { o[nt][mt][e] *= f; o[nt][mt][2 + e] *= f; }
                }
            }
        }
        if (a.scores && w.len <= a.score_len && w.n * a.group <= a.score_rows) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = w.rg * Cfg::kRows + nt * 8 + 2 * t + e;
                    if (r >= w.n * a.group) continue;
                    float* dst = a.scores + ((size_t(w.s) * c.heads + w.h) * a.score_rows + r) * size_t(a.score_len) + j0;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        if (j0 + tok[u][0] < w.len) dst[tok[u][0]] = sc[u][nt][e];
                        if (j0 + tok[u][1] < w.len) dst[tok[u][1]] = sc[u][nt][2 + e];
                    }
                }
        }
        // probabilities and the second product, 16 tokens at a time
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t pf[NT][NB][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float r0 = ref[nt][0] == -INFINITY ? 0.0f : ref[nt][0], r1 = ref[nt][1] == -INFINITY ? 0.0f : ref[nt][1];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x0 = sc[u][nt][2 * e] - r0, x1 = sc[u][nt][2 * e + 1] - r1;
                    sum[nt][0] += exp2_fast(x0);
                    sum[nt][1] += exp2_fast(x1);
                    const float p0 = exp2_fast(x0 + ve[u][e]), p1 = exp2_fast(x1 + ve[u][e]);
#pragma unroll
                    for (int b = 0; b < NB; ++b) pf[nt][b][e] = transpose8x8(half2_of(__fmul_rn(p0, vs[u][e][b]), __fmul_rn(p1, vs[u][e][b])));
                }
            }
            // this thread's value codes: fragment tokens 2t, 2t + 1, 2t + 8, 2t + 9
            constexpr int VW = D / 64;                                 // words per row and thread
            uint32_t vw[4][VW];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * u + 8 * (r >> 1) + token_of(2 * t + (r & 1));
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const int byte = b * (Cfg::kRowBytes / NB) + g * PB;
                    const uint32_t at = st + Cfg::kCodes + chunk_at(row, byte >> 4) + uint32_t(byte & 15);
                    if constexpr (PB == 8) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(vw[r][0]), "=r"(vw[r][VW - 1]) : "r"(at));
                    else if constexpr (PB == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(vw[r][b]) : "r"(at));
                    else {
                        uint16_t h;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at));
                        if ((b & 1) == 0) vw[r][b >> 1] = h;
                        else vw[r][b >> 1] |= uint32_t(h) << 16;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                // bytes of two tokens' codes of one column: even columns from the low nibbles, odd ones from the high
                const uint32_t e0 = (vw[0][i] & 0x0F0F0F0Fu) | ((vw[1][i] << 4) & 0xF0F0F0F0u), o0 = ((vw[0][i] >> 4) & 0x0F0F0F0Fu) | (vw[1][i] & 0xF0F0F0F0u);
                const uint32_t e1 = (vw[2][i] & 0x0F0F0F0Fu) | ((vw[3][i] << 4) & 0xF0F0F0F0u), o1 = ((vw[2][i] >> 4) & 0x0F0F0F0Fu) | (vw[3][i] & 0xF0F0F0F0u);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int mt = 4 * i + k, b = mt / PB;
                    const uint32_t a0 = pair_of(e0, k), a1 = pair_of(o0, k), a2 = pair_of(e1, k), a3 = pair_of(o1, k);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][mt], a0, a1, a2, a3, pf[nt][b][0], pf[nt][b][1]);
                }
            }
        }
    };

    // ---- the pipeline: kStages - 1 tiles in flight ahead of the one being worked on
    long long fetched = lo;
    int st_in = 0, st_out = 0;
#pragma unroll
    for (int i = 0; i < Cfg::kStages - 1; ++i) {
        if (fetched < hi) {
            fetch(ld, st_in);
            walk_next<Cfg::kRows, Cfg::kTile>(c, rows, a.group, ld);
            ++fetched;
        }
        commit();
        st_in = st_in + 1 == Cfg::kStages ? 0 : st_in + 1;
    }
    bool fresh = false, from_start = cu.tile == 0;
    whole = from_start && lo + cu.tiles <= hi;
    if (lo < hi) begin(cu);
    // the pair table, under the first loads
    for (int i = threadIdx.x; i < 256 * 8; i += Cfg::kWarps * 32) {   // four lanes' copies of entry i / 8 per store
        const uint32_t e = uint32_t(i) >> 3, v = uint32_t(half[e & 15u]) | uint32_t(half[e >> 4]) << 16;
        *reinterpret_cast<uint4*>(smem + e * 256 + (i & 7) * 16) = make_uint4(v, v, v, v);
    }
    __syncthreads();
    for (long long i = lo; i < hi; ++i) {
        if (fresh) {
            from_start = cu.tile == 0;
            whole = from_start && i + cu.tiles <= hi;
            begin(cu);
            fresh = false;
        }
        if (fetched < hi) {
            fetch(ld, st_in);
            walk_next<Cfg::kRows, Cfg::kTile>(c, rows, a.group, ld);
            ++fetched;
        }
        commit();
        st_in = st_in + 1 == Cfg::kStages ? 0 : st_in + 1;
        asm volatile("cp.async.wait_group %0;" ::"n"(Cfg::kStages - 1) : "memory");
        __syncwarp();
        compute(cu, st_out);
        __syncwarp();
        st_out = st_out + 1 == Cfg::kStages ? 0 : st_out + 1;
        const bool last = i + 1 == hi || cu.tile + 1 == cu.tiles;
        if (last) finish(cu, from_start);
        fresh = walk_next<Cfg::kRows, Cfg::kTile>(c, rows, a.group, cu);
    }
}

// Joins the partial results of pairs that several warps shared, in warp order, and writes zeros for rows without any slot.
// One CTA of 128 threads per (sequence, head) and query row.
template <int D, int NT>
__global__ void __launch_bounds__(128)
attend_rows_finish(const Cache c, const Rows rows, const RowsArgs a) {
    constexpr int ROWS = 8 * NT, SLOT = ROWS * D + 2 * ROWS, TILE = 32;
    constexpr int LANES = D / 4, TEAMS = 128 / LANES;                  // a team adds every TEAMS-th part
    __shared__ float red[TEAMS][D];
    __shared__ float red_sum[TEAMS];
    Walk w;
    w.s = blockIdx.x / c.heads;
    w.h = blockIdx.x % c.heads;
    walk_load<ROWS, TILE>(c, rows, a.group, w);
    const long long total = a.prefix[c.n_seq], W = active_warps(total, a.warps);
    const int team = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    for (int r = blockIdx.y; r < w.n * a.group; r += gridDim.y) {
        const size_t at = size_t(w.r0 + r / a.group) * a.q_heads + w.h * a.group + r % a.group;
        if (w.tiles == 0) {
            if (threadIdx.x < D / 2) reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + at * D)[threadIdx.x] = 0u;
            if (a.stats && threadIdx.x == 0) a.stats[at] = make_float2(0.0f, 0.0f);
            continue;
        }
        const int rg = r / ROWS, rr = r % ROWS;
        const long long first = a.prefix[w.s] + ((long long)w.h * w.groups + rg) * w.tiles;
        const int w0 = owner_of(first, total, W), w1 = owner_of(first + w.tiles - 1, total, W);
        if (w0 == w1) continue;                                        // one warp had it all
        auto slot = [&](int i) -> const float* { return a.partial + (size_t(i) * 2 + (i == w0 ? 1 : 0)) * SLOT; };
        float m = -INFINITY;
        for (int i = w0 + int(threadIdx.x & 31); i <= w1; i += 32) m = fmaxf(m, slot(i)[ROWS * D + rr]);
#pragma unroll
        for (int k = 16; k >= 1; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
        const float mm = m == -INFINITY ? 0.0f : m;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float sum = 0.0f;
        for (int i = w0 + team; i <= w1; i += TEAMS) {
            const float* s = slot(i);
            const float f = exp2_fast(s[ROWS * D + rr] - mm);
            const float4 v = *reinterpret_cast<const float4*>(s + rr * D + 4 * lane);
            acc.x = __fmaf_rn(v.x, f, acc.x);
            acc.y = __fmaf_rn(v.y, f, acc.y);
            acc.z = __fmaf_rn(v.z, f, acc.z);
            acc.w = __fmaf_rn(v.w, f, acc.w);
            sum = __fmaf_rn(s[ROWS * D + ROWS + rr], f, sum);
        }
        *reinterpret_cast<float4*>(&red[team][4 * lane]) = acc;
        if (lane == 0) red_sum[team] = sum;
        __syncthreads();
        sum = 0.0f;
#pragma unroll
        for (int k = 0; k < TEAMS; ++k) sum += red_sum[k];
        const float inv = sum > 0.0f ? __fdiv_rn(1.0f, sum) : 0.0f, f = inv * a.inv_unit;
        if (threadIdx.x < D / 2) {
            float x = 0.0f, y = 0.0f;
#pragma unroll
            for (int k = 0; k < TEAMS; ++k) { x += red[k][2 * threadIdx.x]; y += red[k][2 * threadIdx.x + 1]; }
            x *= f;
            y *= f;
            uint32_t v;
            if (a.bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(y), "f"(x));
            else v = half2_of(x, y);
            reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + at * D)[threadIdx.x] = v;
        }
        if (a.stats && threadIdx.x == 0) a.stats[at] = make_float2(m, inv);
        __syncthreads();
    }
}

// weights[s, h, j] += sum over the rows of 2^(score - reference) / sum, rows in ascending order; a thread owns a slot.  Scores
// of sequences that the caller's bounds did not cover are computed again.
template <int DT>
__global__ void __launch_bounds__(128)
attend_rows_weights(const Cache c, const Rows rows, const RowsArgs a, float sm_log2, float* __restrict__ weights, int64_t stride,
                    const __grid_constant__ bq4k::Tables4 tab) {
    __shared__ float thr[16], val[16], qsm[256];
    __shared__ float2 st[32];
    bq4k::fill_tables(tab, thr, val);
    const int s = blockIdx.z, h = blockIdx.y;
    const int r0 = rows.begin(s), n = max(rows.end(s) - r0, 0), len_all = c.len(s);
    const int len = int(min(int64_t(len_all), stride)), nr = n * a.group;
    if (nr == 0) return;
    const bool stored = len_all <= a.score_len && nr <= a.score_rows;
    const float* sc = a.scores + (size_t(s) * c.heads + h) * a.score_rows * size_t(a.score_len);
    for (int j0 = blockIdx.x * 128; j0 < len; j0 += gridDim.x * 128) {
        const int j = j0 + int(threadIdx.x);
        float sum = 0.0f;
        for (int rb = 0; rb < nr; rb += 32) {
            __syncthreads();
            if (threadIdx.x < 32 && rb + threadIdx.x < nr) {
                const int r = rb + threadIdx.x;
                st[threadIdx.x] = a.stats[size_t(r0 + r / a.group) * a.q_heads + h * a.group + r % a.group];
            }
            __syncthreads();
            for (int r = rb; r < min(nr, rb + 32); ++r) {
                const float2 m = st[r - rb];
                if (stored) {
                    if (j < len && m.y > 0.0f) sum += exp2_fast(sc[size_t(r) * a.score_len + j] - m.x) * m.y;
                } else {
                    const int i = r / a.group;
                    __syncthreads();
                    for (int d = threadIdx.x; d < c.dim; d += 128)
                        qsm[d] = bq4k::load1<DT>(a.q, size_t(r0 + i) * size_t(a.q_stride) + size_t(h * a.group + r % a.group) * c.dim + d);
                    __syncthreads();
                    if (j < len && j < len_all - n + i + 1)
                        sum += exp2_fast(dot_row(c.k_codes, c.k_scale, c.row(s, h, j), c.dim, c.block, val, qsm) * sm_log2 - m.x) * m.y;
                }
            }
        }
        if (j < len) weights[(size_t(s) * c.heads + h) * size_t(stride) + j] += sum;
    }
}

}  // namespace bqkvk
