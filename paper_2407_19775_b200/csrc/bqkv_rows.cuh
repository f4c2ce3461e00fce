// bqkv_rows.cuh -- attention of a few query rows per cached head over the 4-bit cache (a decode
// step): attend_rows and attend_rows_weights (sm_100a).
//
// The step is bound by the stream of cache rows (D + 4 D / block bytes per token and head) as long
// as a token costs few instructions, so everything here is about instructions per cached element.
//
//   dequantize   a byte (two codes) is one lookup of a pair of fp16 values.  The 256 pairs sit in
//                shared memory once per lane, each lane in its own bank (no conflicts), 256 bytes
//                apart and from an address that is a multiple of 64 KB, so that ONE byte permute builds
//                the address: lane * 4 in byte 0, the code byte in byte 1, the table's place above.
//                Two instructions per pair.
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
//   softmax      running reference per row: 2^7 below the row's largest product of probability and
//                value scale when it is taken, moved only when a product exceeds it by 2^15.  The log2
//                of a token's (largest) value scale joins its score before the reference is taken, so
//                that what enters the second product as fp16 cannot overflow, and its smallest step
//                is 2^-31 of the row's largest: a context's many light tokens count.  The softmax's
//                sum, in fp32, holds 2^(score - reference) without the scale: value scales count as
//                2^-80 at least in the reference, which bounds it.
//   rounding     a product of probability and value scale enters as one fp16 number for bf16 outputs
//                (11 bits against their own 8), as two for fp16 outputs, whose own rounding one would
//                match.  Measured, 64 ragged sequences, fp16: 100.6 us with one (and a third more error
//                against 64 bits), 108.6 with two; 64 x 4 rows: 51.9 and 58.0.
//   split        the tiles of 32 tokens of all (sequence, head) pairs, numbered in order, are dealt
//                out evenly over the CTAs (one per SM) and, within a CTA, over its warps: ragged
//                batches stay balanced.  A range starts and ends inside a pair at most once each, so a
//                warp leaves at most two partial results, which its CTA joins in shared memory, and a
//                CTA two, which the last of a pair's CTAs to arrive (a ticket) joins; always in
//                ascending order, whoever does it, so the same call gives the same bits.
//
// Measured: 64 ragged sequences up to 8192 slots, 8 x 8 heads, head_dim 128, blocks of 64, bf16: 362 MB in 101 us, 3.6 TB/s; two
// sequences up to 131072 slots: 225 MB in 65 us, 3.5 TB/s.  That is 0.55 of the copy rate, bound by dependent latencies at three
// warps per scheduler: the pipe of the lookups is busy two thirds of the time, every second cycle issues, the memory is not
// waited for.  A short prompt's next token (1 x 500 slots): 11 us, launch and latency.
#pragma once

#include "bqkv_kernels.cuh"

namespace bqkvk {

// (a & mask) | (b & ~mask) in one instruction
__device__ __forceinline__ uint32_t select_bits(uint32_t a, uint32_t b, uint32_t mask) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xE4;" : "=r"(d) : "r"(a), "r"(b), "r"(mask));
    return d;
}

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
    float* partial;                        // 2 slots per CTA, then one per warp
    int* tickets;                          // one per CTA, zero between calls: parts of the pair it began that have arrived
    float2* stats;                         // (reference, 1 / sum) of every (row, query head); may be null
    float* scores;                         // [n_seq, heads, score_rows, score_len] in log2 units; may be null
    int score_rows, score_len;
};

template <int D, int NB, int NT>
struct RowsCfg {
    static constexpr int kRows = 8 * NT;                               // query rows a warp works on
    // Registers decide: 8 (16) accumulator fragments and the scheduling room that lets lookups of one product run under another.
    // Measured, 64 ragged sequences, D = 128, 8 rows: 16 warps 104 us, 12 warps 100 us, 8 warps 108 us; 16 rows: 12 warps 91 us,
    // 8 warps 84 us; D = 64, 8 rows: 16 warps 62 us, 12 warps 66 us.
    static constexpr int kWarps = NT == 2 ? 8 : D == 64 ? 16 : 12;
    static constexpr int kTile = 32;                                   // tokens
    static constexpr int kRowBytes = D / 2;
    static constexpr int kCodes = kTile * kRowBytes;                   // bytes of one operand's codes in a stage
    static constexpr int kScales = kTile * NB * 2;
    static constexpr int kStage = 2 * kCodes + 2 * kScales;
    static constexpr int kStages = 2;
    static constexpr int kRing = kStages * kStage;                     // a warp's
    static constexpr int kTable = 256 * 256;                           // from the first multiple of 64 KB of the shared address space on;
    static constexpr int kLowWarps = (kTable - 6144) / kRing < kWarps ? (kTable - 6144) / kRing : kWarps;      // the rings below it (6 KB: static shared memory)
    // A partial result: the accumulator fragments register by register (32 lanes each), then the rows' references and sums.
    static constexpr int kValues = kRows * D, kSlot = kValues + 2 * kRows;
    static constexpr int kLoop = 2 * kTable + (kWarps - kLowWarps) * kRing - 1024;                             // ... and above it; the space starts 1 KB in at least
    static constexpr int kJoin = 2 * kWarps * kSlot * 4;
    static constexpr int kSmem = kLoop > kJoin ? kLoop : kJoin;
    static_assert(kSmem + 5120 <= 227 * 1024, "fits an SM");
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {      // d = a b
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
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
__device__ __forceinline__ float log2_fast(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
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
    int first;                             // slot of the first row (negative: it and some behind it have none)
};

template <int ROWS, int TILE>
__device__ __forceinline__ void walk_load(const Cache& c, const Rows& rows, int group, Walk& w) {
    w.r0 = rows.begin(w.s);
    w.n = max(rows.end(w.s) - w.r0, 0);
    const int counted = c.counted(w.s);
    w.len = c.held(counted);
    w.first = counted - w.n;
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

// Where row r of a pair's row group goes, as (row of the call) * q_heads + query head; -1: there is no such row.
template <int ROWS>
__device__ __forceinline__ int64_t row_of(const RowsArgs& a, const Walk& w, int h_first /* w.h * group */, int r) {
    const int row = w.rg * ROWS + r;
    if (row >= w.n * a.group) return -1;
    if (row < a.group) return int64_t(w.r0) * a.q_heads + h_first + row;
    return int64_t(w.r0 + row / a.group) * a.q_heads + h_first + row % a.group;
}
// Columns col, col + 1 of a row from its sums: the final values (and, once, its statistics).
template <int D>
__device__ __forceinline__ void store_pair(const RowsArgs& a, int64_t at, int col, float m, float l, float x, float y) {
    if (at < 0) return;
    const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : 0.0f, f = inv * a.inv_unit;
    x *= f;
    y *= f;
    uint32_t v;
    if (a.bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(y), "f"(x));
    else v = half2_of(x, y);
    reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + at * D)[col / 2] = v;
    if (a.stats && col == 0) a.stats[at] = make_float2(m, inv);
}

template <int V> struct Flag { static constexpr int value = V; };

// Tiles and (head, row group) pairs of the whole call, counted by one CTA; `empty`: some sequence has rows but no slots.
template <int ROWS, int TILE>
__device__ __forceinline__ void count_tiles(const Cache& c, const Rows& rows, int group, int (*scratch)[2] /* shared, one per warp */, int& total, int& pairs,
                                            bool& empty) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = blockDim.x >> 5;
    total = pairs = 0;
    empty = false;
    for (int s0 = 0; s0 < c.n_seq; s0 += blockDim.x) {
        Walk w;
        w.s = s0 + threadIdx.x;
        int t = 0, p = 0;
        bool none = false;
        if (w.s < c.n_seq) {
            walk_load<ROWS, TILE>(c, rows, group, w);
            p = w.tiles > 0 ? w.groups * c.heads : 0;
            t = p * w.tiles;
            none = w.groups > 0 && w.tiles == 0;
        }
#pragma unroll
        for (int k = 16; k >= 1; k >>= 1) { t += __shfl_xor_sync(0xffffffffu, t, k); p += __shfl_xor_sync(0xffffffffu, p, k); }
        if (lane == 0) { scratch[wid][0] = t; scratch[wid][1] = p; }
        empty |= __syncthreads_or(none) != 0;
        for (int i = 0; i < nw; ++i) { total += scratch[i][0]; pairs += scratch[i][1]; }
        __syncthreads();
    }
}

// T units in n shares that differ by one at most: where share k begins, and the share that holds a unit.
struct Shares {
    int each, more;                        // `more` shares of each + 1 units come first
    __device__ __forceinline__ Shares(int total, int n) { each = total / n; more = total - each * n; }
    __device__ __forceinline__ int begin(int k) const { return k * each + min(k, more); }
    __device__ __forceinline__ int of(int unit) const {
        const int split = more * (each + 1);
        return unit < split ? unit / (each + 1) : more + (unit - split) / each;
    }
};

template <int D, int NB, int NT, bool SPLIT /* probabilities as two fp16 numbers */>
__global__ void __launch_bounds__(RowsCfg<D, NB, NT>::kWarps * 32, 1)
attend_rows(const Cache c, const Rows rows, const RowsArgs a, const __grid_constant__ PairTable pairs) {
    using Cfg = RowsCfg<D, NB, NT>;
    constexpr int KS = D / 16;                                         // k steps of the scores = row tiles of the outputs
    constexpr int KSB = KS / NB;                                       // of one block
    extern __shared__ __align__(256) unsigned char smem[];
    __shared__ int scratch[Cfg::kWarps][2];
    __shared__ uint16_t half[16];
    __shared__ Walk walks[Cfg::kWarps][2];                             // where this warp loads, and where it computes
    // What a warp leaves behind.  Slot 0: a pair it continued from the warp before (and ended, or not); slot 1: one it began
    // and did not end.  The walk and the first tile of the pair of either.
    struct Left { int has[2], ended, saved; Walk w[2]; int first[2]; };
    __shared__ Left lefts[Cfg::kWarps];
    __shared__ int4 chains[Cfg::kWarps + 1];                           // first warp, slot, last warp, whether the pair is whole
    __shared__ int n_chains, chain_at[2], chain_from[2], chain_parts[2];      // the last three: of the (at most two) pairs shared with other CTAs
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    if (threadIdx.x < 16) half[threadIdx.x] = pairs.half[threadIdx.x];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");                 // nothing in global memory is touched before the kernels before this one are done
    // Up to 32 sequences: one per lane, every warp for itself.  More: counted by the CTA, looked up again below.
    const bool by_lane = c.n_seq <= 32;
    Walk mine = {};
    int total, n_pairs, upto = 0;                                      // upto: tiles of the lanes' sequences up to this one
    bool empty;
    if (by_lane) {
        mine.s = lane;
        int p = 0;
        if (lane < c.n_seq) {
            walk_load<Cfg::kRows, Cfg::kTile>(c, rows, a.group, mine);
            p = mine.tiles > 0 ? mine.groups * c.heads : 0;
        }
        upto = p * mine.tiles;
        empty = __any_sync(0xffffffffu, mine.groups > 0 && mine.tiles == 0);
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, upto, k);
            if (lane >= k) upto += o;
            p += __shfl_xor_sync(0xffffffffu, p, k);
        }
        total = __shfl_sync(0xffffffffu, upto, 31);
        n_pairs = p;
    } else {
        count_tiles<Cfg::kRows, Cfg::kTile>(c, rows, a.group, scratch, total, n_pairs, empty);
    }
    if (empty)                                                         // rows of sequences without any slot: zeros
        for (int s = blockIdx.x; s < c.n_seq; s += gridDim.x) {
            const int r0 = rows.begin(s), n = rows.end(s) - r0;
            if (n <= 0 || c.len(s) > 0) continue;
            uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + size_t(r0) * a.q_heads * D);
            for (size_t i = threadIdx.x; i < size_t(n) * a.q_heads * (D / 2); i += Cfg::kWarps * 32) out[i] = 0u;
            if (a.stats)
                for (size_t i = threadIdx.x; i < size_t(n) * a.q_heads; i += Cfg::kWarps * 32) a.stats[size_t(r0) * a.q_heads + i] = make_float2(0.0f, 0.0f);
        }
    // All CTAs share the tiles where there is work for two rounds of all their warps.  Below that a pair goes to one CTA, or to
    // as many as it has tiles for one round of their warps: joining parts across CTAs (a fence, a ticket and a round of loads,
    // 3-4 us) costs more than a second tile per warp.
    int ctas = gridDim.x;
    if (total < 2 * Cfg::kWarps * ctas && n_pairs > 0 && n_pairs <= ctas) {
        const int each = total / (n_pairs * Cfg::kWarps), most = ctas / n_pairs;
        ctas = n_pairs * (each < 1 ? 1 : each < most ? each : most);
    }
    if (ctas > total) ctas = total;
    if (int(blockIdx.x) >= ctas) return;                               // a tile for every CTA at least
    const Shares of_ctas(total, ctas);
    const int cta_lo = of_ctas.begin(blockIdx.x), cta_n = of_ctas.begin(blockIdx.x + 1) - cta_lo;
    const int aw = min(cta_n, Cfg::kWarps);                            // warps with a tile
    const Shares of_warps(cta_n, aw);
    const int lo = cta_lo + of_warps.begin(min(wid, aw)), hi = cta_lo + of_warps.begin(min(wid + 1, aw));
    if (lane == 0) { lefts[wid].has[0] = lefts[wid].has[1] = lefts[wid].ended = lefts[wid].saved = 0; }

    Walk ld = {};
    if (lo < hi) {
        int left = lo;
        if (by_lane) {
            const int w = __ffs(__ballot_sync(0xffffffffu, lo < upto)) - 1;
            const int before = __shfl_up_sync(0xffffffffu, upto, 1);
            const int first = __shfl_sync(0xffffffffu, before, w);
            left -= w > 0 ? first : 0;
            ld.s = w;
            ld.len = __shfl_sync(0xffffffffu, mine.len, w);
            ld.first = __shfl_sync(0xffffffffu, mine.first, w);
            ld.n = __shfl_sync(0xffffffffu, mine.n, w);
            ld.r0 = __shfl_sync(0xffffffffu, mine.r0, w);
            ld.tiles = __shfl_sync(0xffffffffu, mine.tiles, w);
            ld.groups = __shfl_sync(0xffffffffu, mine.groups, w);
        } else {
            for (int s0 = 0;; s0 += 32) {                              // 32 sequences a step; lo < total, so one holds it
                ld.s = s0 + lane;
                int n = 0;
                if (ld.s < c.n_seq) {
                    walk_load<Cfg::kRows, Cfg::kTile>(c, rows, a.group, ld);
                    n = ld.tiles * ld.groups * c.heads;
                }
                int inc = n;
#pragma unroll
                for (int k = 1; k < 32; k <<= 1) {
                    const int o = __shfl_up_sync(0xffffffffu, inc, k);
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
        }
        const int pair = left / ld.tiles;
        ld.tile = left - pair * ld.tiles;
        ld.h = pair / ld.groups;
        ld.rg = pair - ld.h * ld.groups;
    }
    if (lane == 0) { walks[wid][0] = ld; walks[wid][1] = ld; }
    __syncwarp();
    const uint32_t low = uint32_t(__cvta_generic_to_shared(smem)), table = (low + 0xFFFFu) & 0xFFFF0000u, table_lane = table | uint32_t(lane) * 4u;
    const uint32_t ring = wid < Cfg::kLowWarps ? low + uint32_t(wid) * Cfg::kRing : table + Cfg::kTable + uint32_t(wid - Cfg::kLowWarps) * Cfg::kRing;
    auto pair_of = [&](uint32_t word, int byte) -> uint32_t {          // the fp16 pair of byte `byte` of a word of codes
        uint32_t v;
        asm("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(bq4k::prmt(word, table_lane, 0x7604u | uint32_t(byte) << 4)));
        return v;
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

    // The loading side: what a tile's address needs stays in registers, the rest of its walk in shared memory.
    constexpr int CPR = Cfg::kRowBytes / 16;                           // 16-byte chunks per row
    const uint32_t dst0 = chunk_at(lane / CPR, lane % CPR);            // the xor repeats every 8 rows: later chunks are a constant further
    const uint32_t page_codes = uint32_t(c.page) * Cfg::kRowBytes, page_scales = uint32_t(c.page) * NB * 2;
    const uint8_t* const k_lane = c.k_codes + lane * 16;
    const uint8_t* const v_lane = c.v_codes + lane * 16;
    // scales: lanes 0 .. 2 NB - 1 copy the keys' of 16 tokens, the next 2 NB the values'
    const bool s_lane = lane < 4 * NB, s_v = lane >= 2 * NB;
    const uint32_t s_i = uint32_t(s_v ? lane - 2 * NB : lane) * 16u, s_dst = 2 * Cfg::kCodes + (s_v ? Cfg::kScales : 0) + s_i;
    const char* const s_src = reinterpret_cast<const char*>(s_v ? c.v_scale : c.k_scale) + s_i;
    const bool whole_tiles = c.page % Cfg::kTile == 0;                 // a tile lies in one page
    const int last_group = c.max_pages * c.page - 16;
    int ld_tile = ld.tile, ld_tiles = ld.tiles, ld_h = ld.h;
    const int32_t* ld_table = c.table + size_t(ld.s) * c.table_stride;
    auto place = [&](int j, uint32_t& head_row) -> int {               // page and head of slot j, and its row in the page
        const int p = c.page_shift >= 0 ? j >> c.page_shift : j / c.page;
        const int pg = min(max(__ldg(ld_table + p), 0), c.n_pages - 1);
        head_row = uint32_t(pg) * uint32_t(c.heads) + uint32_t(ld_h);  // below 2^31: checked by the host
        return j - p * c.page;
    };
    const uint8_t *ks = nullptr, *vs = nullptr;                        // this lane's place in the current page
    const char* sc = nullptr;
    int in_page = 0;                                                   // slots left there
    auto point = [&](int j) {
        uint32_t hr;
        const int r = place(j, hr);
        const uint64_t at = uint64_t(hr) * page_codes + uint32_t(r) * uint32_t(Cfg::kRowBytes);
        ks = k_lane + at;
        vs = v_lane + at;
        sc = s_src + (uint64_t(hr) * page_scales + uint32_t(r) * uint32_t(NB * 2));
        in_page = c.page - r;
    };
    auto copy_group = [&](uint32_t st, int u, int off) {               // 16 tokens; off: groups from the pointers
#pragma unroll
        for (int k = 0; k < Cfg::kCodes / 1024; ++k) {
            copy16(st + dst0 + u * (Cfg::kCodes / 2) + k * 512, ks + off * (Cfg::kCodes / 2) + k * 512);
            copy16(st + dst0 + Cfg::kCodes + u * (Cfg::kCodes / 2) + k * 512, vs + off * (Cfg::kCodes / 2) + k * 512);
        }
        if (s_lane) copy16(st + s_dst + u * (Cfg::kScales / 2), sc + off * (Cfg::kScales / 2));
    };
    auto fetch = [&](uint32_t st) {
        if (in_page == 0) point(ld_tile * Cfg::kTile);
        if (whole_tiles) {
            copy_group(st, 0, 0);
            copy_group(st, 1, 1);
            ks += Cfg::kCodes;
            vs += Cfg::kCodes;
            sc += Cfg::kScales;
            in_page -= Cfg::kTile;
        } else {
            copy_group(st, 0, 0);
            point(min(ld_tile * Cfg::kTile + 16, last_group));         // past the table's end: any group, its scores are masked
            copy_group(st, 1, 0);
            in_page = 0;
        }
        if (++ld_tile == ld_tiles) {                                   // on to the next (head, row group, sequence)
            Walk w = walks[wid][0];
            __syncwarp();
            w.tile = w.tiles - 1;
            walk_next<Cfg::kRows, Cfg::kTile>(c, rows, a.group, w);
            if (lane == 0) walks[wid][0] = w;
            __syncwarp();
            ld_tile = 0;
            in_page = 0;
            ld_tiles = w.tiles;
            ld_h = w.h;
            ld_table = c.table + size_t(min(w.s, c.n_seq - 1)) * c.table_stride;
        }
    };
    auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };

    uint32_t qf[NT][KS][2];                                            // query fragments
    float qs[NT][2];                                                   // factor of the scores of this thread's rows 2t, 2t + 1
    int seen[NT][2];                                                   // slots those rows see (a row that does not exist: all)
    int all_see;                                                       // the smallest of the rows' counts
    float o[NT][KS][4], ref[NT][2], sum[NT][2];
    float* score_at = nullptr;                                         // where this pair's scores go, if they are wanted
    int score_rows = 0;
    auto begin = [&](const Walk& w) {                                  // the queries of a (sequence, head, row group)
        all_see = min(max(w.first + (w.rg * Cfg::kRows) / a.group + 1, 0), w.len);       // its first row sees the fewest
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
            const int ex = min(max(14 - (int(__float_as_uint(big) >> 23) - 127), -126), 126);       // (a row of zeros: anything)
            const float up = __uint_as_float(uint32_t(127 + ex) << 23);
            mine[nt] = in ? a.score_scale * __uint_as_float(uint32_t(127 - ex) << 23) : 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t v = raw[k][e];
                    const float x = a.bf16 ? __uint_as_float(v << 16) : __low2float(*reinterpret_cast<const __half2*>(&v));
                    const float y = a.bf16 ? __uint_as_float(v & 0xffff0000u) : __high2float(*reinterpret_cast<const __half2*>(&v));
                    qf[nt][k][e] = half2_of(x * up, y * up);
                }
            const int last = in ? min(max(w.first + i + 1, 0), w.len) : w.len;
#pragma unroll
            for (int e = 0; e < 2; ++e) {                              // this thread's score columns are rows 2t + e
                qs[nt][e] = __shfl_sync(0xffffffffu, mine[nt], 4 * (2 * t + e));
                seen[nt][e] = __shfl_sync(0xffffffffu, last, 4 * (2 * t + e));
                ref[nt][e] = -1.0e30f;                                 // finite, so that nothing below needs a case of its own
                sum[nt][e] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][k][e] = 0.0f;
        }
        const bool keep = a.scores && w.len <= a.score_len && w.n * a.group <= a.score_rows;
        score_rows = w.n * a.group - w.rg * Cfg::kRows;
        score_at = keep ? a.scores + ((size_t(w.s) * c.heads + w.h) * a.score_rows + w.rg * Cfg::kRows) * size_t(a.score_len) : nullptr;
    };

    // column of output row tile mt, this thread: pair (even, odd) starting here
    constexpr int PB = Cfg::kRowBytes / (8 * NB);                      // value bytes per thread, row and block: 8, 4 or 2
    auto column_of = [](int mt, int gg) -> int { return (mt / PB) * (D / NB) + gg * 2 * PB + 2 * (mt % PB); };
    auto save = [&](float* slot) {                                     // this warp's partial result
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int mt = 0; mt < KS; ++mt)
#pragma unroll
                for (int q = 0; q < 4; ++q) slot[((nt * KS + mt) * 4 + q) * 32 + lane] = o[nt][mt][q];
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (g == 0) {
                    slot[Cfg::kValues + nt * 8 + 2 * t + e] = ref[nt][e];
                    slot[Cfg::kValues + Cfg::kRows + nt * 8 + 2 * t + e] = sum[nt][e];
                }
        }
    };

    auto store_rows = [&](const Walk& w) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int64_t at = row_of<Cfg::kRows>(a, w, w.h * a.group, nt * 8 + 2 * t + e);
#pragma unroll
                for (int mt = 0; mt < KS; ++mt) store_pair<D>(a, at, column_of(mt, g), ref[nt][e], sum[nt][e], o[nt][mt][e], o[nt][mt][2 + e]);
            }
    };
    // The end of this warp's part of a pair: the final rows where it had all of it; a partial result otherwise, which stays in
    // registers unless the warp goes on (`more`) with another pair.
    auto finish = [&](const Walk& w, bool from_start, bool whole, int done, int next, bool more) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int k = 4; k <= 16; k <<= 1) sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], k);
            }
        if (whole) {
            store_rows(w);
            return;
        }
        if (lane == 0) {
            Left& l = lefts[wid];
            const int which = from_start ? 1 : 0;
            l.has[which] = 1;
            l.w[which] = w;
            l.first[which] = next - done;
            if (!from_start) { l.ended = done == w.tiles; l.saved = more; }
        }
        if (more) save(a.partial + (size_t(2) * gridDim.x + size_t(blockIdx.x) * Cfg::kWarps + wid) * Cfg::kSlot);
    };

    const int tg = token_of(g);                                        // this thread's tokens: tg and tg + 8
    // this thread's key codes of token tg, and value codes of fragment tokens 2t and 2t + 1 (8 further: 2t + 8, 2t + 9); rows
    // 8 further are a constant further, blocks of a row change the chunk
    constexpr int PK = Cfg::kRowBytes / (4 * NB);                      // key bytes per thread, row and block: 16, 8 or 4
    uint32_t k_at[NB], v_at[2][NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int kb = b * (Cfg::kRowBytes / NB) + t * PK, vb = b * (Cfg::kRowBytes / NB) + g * PB;
        k_at[b] = chunk_at(tg, kb >> 4) + uint32_t(kb & 15);
#pragma unroll
        for (int e = 0; e < 2; ++e) v_at[e][b] = uint32_t(Cfg::kCodes) + chunk_at(token_of(2 * t + e), vb >> 4) + uint32_t(vb & 15);
    }

    // A tile's scales, one token per lane: the keys' (as they are) and, of the values', the log2 of the token's largest one and
    // the blocks' relative to that.  compute() hands them to the lanes that hold the token's scores by shuffles.
    float lane_ks[NB], lane_lv, lane_vs[NB];
    auto scales = [&](uint32_t st, int j0, int len) {
        const uint32_t at = st + uint32_t(2 * Cfg::kCodes + lane * NB * 2);
        uint32_t kr[(NB + 1) / 2], vr[(NB + 1) / 2];                   // bf16 pairs (NB == 1: one in the low half)
        if constexpr (NB == 1) {
            uint16_t x, y;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at));
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(at + Cfg::kScales));
            kr[0] = x;
            vr[0] = y;
        } else {
#pragma unroll
            for (int i = 0; i < NB / 2; ++i) {
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(kr[i]) : "r"(at + 4 * i));
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(vr[i]) : "r"(at + Cfg::kScales + 4 * i));
            }
        }
        const bool in = j0 + lane < len;                               // past the length the bytes may be anything
        float top = 0.0f;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            lane_ks[b] = __uint_as_float(b & 1 ? kr[b / 2] & 0xffff0000u : kr[b / 2] << 16);
            const float v = __uint_as_float(b & 1 ? vr[b / 2] & 0xffff0000u : vr[b / 2] << 16);
            lane_vs[b] = in ? v : 0.0f;
            top = b == 0 ? lane_vs[0] : fmaxf(top, lane_vs[b]);
        }
        lane_lv = fmaxf(log2_fast(top), -126.0f);                      // a row of zeros: its codes' values are zeros
        if constexpr (NB > 1) {
            const float down = exp2_fast(-lane_lv);
#pragma unroll
            for (int b = 0; b < NB; ++b) lane_vs[b] = __fmul_rn(lane_vs[b], down);
        }
    };

    // A tile: the scores of its two groups of 16 tokens, one look at the running reference, then probabilities and outputs group
    // by group.  CARE: some row does not see all of the tile, or its scores are kept.
    auto compute = [&](uint32_t st, int j0, int len, auto care) {
        constexpr bool CARE = decltype(care)::value != 0;
        float sc[2][NT][4];                                            // group u: tokens tg (0, 1) and tg + 8 (2, 3), rows 2t (0, 2) and 2t + 1 (1, 3)
        float lv[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            auto of_token = [&](float v, int e) { return __shfl_sync(0xffffffffu, v, 16 * u + 8 * e + tg); };
            const uint32_t off = u * (Cfg::kCodes / 2);
            uint32_t kw[2][D / 32];                                    // codes of the two tokens: D / 8 bytes each
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const uint32_t at = st + k_at[b] + off + uint32_t(8 * e * Cfg::kRowBytes);
                    if constexpr (PK == 16) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(kw[e][0]), "=r"(kw[e][1]), "=r"(kw[e][2]), "=r"(kw[e][3]) : "r"(at));
                    else if constexpr (PK == 8) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(kw[e][2 * b]), "=r"(kw[e][2 * b + 1]) : "r"(at));
                    else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(kw[e][b]) : "r"(at));
                }
            lv[u][0] = of_token(lane_lv, 0);
            lv[u][1] = of_token(lane_lv, 1);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                // two chains of products where one block has them all: a chain's length is latency
                constexpr int CH = (NB == 1 && KSB >= 4) ? 2 : 1;
                float acc[CH][NT][4];
#pragma unroll
                for (int k = 0; k < KSB; ++k) {
                    const int i = 2 * (b * KSB + k);                   // byte within the thread's D / 8
                    const uint32_t a0 = pair_of(kw[0][i >> 2], i & 3), a1 = pair_of(kw[1][i >> 2], i & 3);
                    const uint32_t a2 = pair_of(kw[0][i >> 2], (i & 3) + 1), a3 = pair_of(kw[1][i >> 2], (i & 3) + 1);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (k < CH) mma_f16_first(acc[k % CH][nt], a0, a1, a2, a3, qf[nt][b * KSB + k][0], qf[nt][b * KSB + k][1]);
                        else mma_f16(acc[k % CH][nt], a0, a1, a2, a3, qf[nt][b * KSB + k][0], qf[nt][b * KSB + k][1]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float ks = of_token(lane_ks[b], e);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int q = 2 * e; q < 2 * e + 2; ++q) {
                            const float x = CH == 2 ? acc[0][nt][q] + acc[CH - 1][nt][q] : acc[0][nt][q];
                            sc[u][nt][q] = b == 0 ? __fmul_rn(x, ks) : __fmaf_rn(x, ks, sc[u][nt][q]);
                        }
                }
            }
            // in log2 units, masked
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    sc[u][nt][q] = __fmul_rn(sc[u][nt][q], qs[nt][q & 1]);
                    if (CARE && j0 + 16 * u + tg + 8 * (q >> 1) >= seen[nt][q & 1]) sc[u][nt][q] = -INFINITY;
                }
        }
        // the running reference: of the score with the value scale
        float lr[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) lr[u][e] = fmaxf(lv[u][e], -80.0f);
        bool above = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float top = fmaxf(fmaxf(sc[0][nt][e] + lr[0][0], sc[0][nt][2 + e] + lr[0][1]), fmaxf(sc[1][nt][e] + lr[1][0], sc[1][nt][2 + e] + lr[1][1]));
                above |= top > ref[nt][e] + 15.0f;
            }
        if (__any_sync(0xffffffffu, above)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float m = fmaxf(fmaxf(sc[0][nt][e] + lr[0][0], sc[0][nt][2 + e] + lr[0][1]), fmaxf(sc[1][nt][e] + lr[1][0], sc[1][nt][2 + e] + lr[1][1]));
                    m = fmaxf(m - 7.0f, ref[nt][e]);
#pragma unroll
                    for (int k = 4; k <= 16; k <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
                    const float f = exp2_fast(ref[nt][e] - m);
                    ref[nt][e] = m;
                    sum[nt][e] *= f;
#pragma unroll
                    for (int mt = 0; mt < KS; ++mt) { o[nt][mt][e] *= f; o[nt][mt][2 + e] *= f; }
                }
        }
        if (CARE && score_at) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (nt * 8 + 2 * t + e >= score_rows) continue;
                    float* dst = score_at + size_t(nt * 8 + 2 * t + e) * size_t(a.score_len) + j0 + tg;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        if (j0 + 16 * u + tg < len) dst[16 * u] = sc[u][nt][e];
                        if (j0 + 16 * u + tg + 8 < len) dst[16 * u + 8] = sc[u][nt][2 + e];
                    }
                }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            [[maybe_unused]] float rel[2][NB];                         // the blocks' value scales relative to the token's largest
            if constexpr (NB > 1) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e) rel[e][b] = __shfl_sync(0xffffffffu, lane_vs[b], 16 * u + 8 * e + tg);
            }
            constexpr int PARTS = SPLIT ? 2 : 1;
            uint32_t pf[PARTS][NT][NB][2];
            auto put = [&](int nt, int b, int e, float p0, float p1) {
                const uint32_t h = half2_of(p0, p1);
                pf[0][nt][b][e] = transpose8x8(h);
                if constexpr (SPLIT) {
                    const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&h));
                    pf[PARTS - 1][nt][b][e] = transpose8x8(half2_of(p0 - back.x, p1 - back.y));
                }
            };
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x0 = sc[u][nt][2 * e] - ref[nt][0], x1 = sc[u][nt][2 * e + 1] - ref[nt][1];
                    sum[nt][0] += exp2_fast(x0);
                    sum[nt][1] += exp2_fast(x1);
                    const float p0 = exp2_fast(x0 + lv[u][e]), p1 = exp2_fast(x1 + lv[u][e]);
                    if constexpr (NB == 1) put(nt, 0, e, p0, p1);
                    else {
#pragma unroll
                        for (int b = 0; b < NB; ++b) put(nt, b, e, __fmul_rn(p0, rel[e][b]), __fmul_rn(p1, rel[e][b]));
                    }
                }
            const uint32_t off = u * (Cfg::kCodes / 2);
            constexpr int VW = D / 64;                                 // words of value codes per row and thread
            uint32_t vw[4][VW];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const uint32_t at = st + v_at[r & 1][b] + off + uint32_t(8 * (r >> 1) * Cfg::kRowBytes);
                    if constexpr (PB == 8) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(vw[r][0]), "=r"(vw[r][VW - 1]) : "r"(at));
                    else if constexpr (PB == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(vw[r][b]) : "r"(at));
                    else {
                        uint16_t h;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at));
                        if ((b & 1) == 0) vw[r][b >> 1] = h;
                        else vw[r][b >> 1] |= uint32_t(h) << 16;
                    }
                }
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                // bytes of two tokens' codes of one column: even columns from the low nibbles, odd ones from the high
                const uint32_t e0 = select_bits(vw[0][i], vw[1][i] << 4, 0x0F0F0F0Fu), o0 = select_bits(vw[0][i] >> 4, vw[1][i], 0x0F0F0F0Fu);
                const uint32_t e1 = select_bits(vw[2][i], vw[3][i] << 4, 0x0F0F0F0Fu), o1 = select_bits(vw[2][i] >> 4, vw[3][i], 0x0F0F0F0Fu);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int mt = 4 * i + k, b = mt / PB;
                    const uint32_t a0 = pair_of(e0, k), a1 = pair_of(o0, k), a2 = pair_of(e1, k), a3 = pair_of(o1, k);
#pragma unroll
                    for (int part = 0; part < PARTS; ++part)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][mt], a0, a1, a2, a3, pf[part][nt][b][0], pf[part][nt][b][1]);
                }
            }
        }
    };

    // ---- the pipeline: kStages - 1 tiles in flight ahead of the one being worked on
    int left = hi - lo, to_fetch = left;
    uint32_t st_in = ring, st_out = ring;
    auto next_stage = [&](uint32_t st) { return st == ring ? st + Cfg::kStage : ring; };
#pragma unroll
    for (int i = 0; i < Cfg::kStages - 1; ++i) {
        if (to_fetch > 0) { fetch(st_in); --to_fetch; }
        commit();
        st_in = next_stage(st_in);
    }
    __syncthreads();                                                   // half[]
    // the pair table, under the first loads
    for (int i = threadIdx.x; i < 256 * 8; i += Cfg::kWarps * 32) {   // four lanes' copies of entry i / 8 per store
        const uint32_t e = uint32_t(i) >> 3, v = uint32_t(half[e & 15u]) | uint32_t(half[e >> 4]) << 16;
        *reinterpret_cast<uint4*>(smem + (table - low) + e * 256 + (i & 7) * 16) = make_uint4(v, v, v, v);
    }
    int tile = ld.tile, tiles = ld.tiles, len = ld.len;
    bool from_start = tile == 0, whole = from_start && tiles <= left;
    if (left > 0) begin(ld);
    __syncthreads();
    while (left > 0) {
        if (to_fetch > 0) { fetch(st_in); --to_fetch; }
        commit();
        st_in = next_stage(st_in);
        asm volatile("cp.async.wait_group %0;" ::"n"(Cfg::kStages - 1) : "memory");
        __syncwarp();
        scales(st_out, tile * Cfg::kTile, len);
        if (tile * Cfg::kTile + Cfg::kTile > all_see || score_at) compute(st_out, tile * Cfg::kTile, len, Flag<1>{});
        else compute(st_out, tile * Cfg::kTile, len, Flag<0>{});
        __syncwarp();
        st_out = next_stage(st_out);
        --left;
        ++tile;
        if (tile == tiles || left == 0) {
            Walk w = walks[wid][1];
            __syncwarp();
            finish(w, from_start, whole, tile, hi - left, left > 0);
            if (left > 0) {
                w.tile = w.tiles - 1;
                walk_next<Cfg::kRows, Cfg::kTile>(c, rows, a.group, w);
                if (lane == 0) walks[wid][1] = w;
                __syncwarp();
                tile = 0;
                tiles = w.tiles;
                len = w.len;
                from_start = true;
                whole = tiles <= left;
                begin(w);
            }
        }
    }

    // ---- pairs that several of this CTA's warps shared.  Parts still in registers go to shared memory (tables and rings are done
    // with), two slots per warp; one that a warp had to put away before it went on is in its slot of global memory.  A chain is
    // a pair's part of this CTA: the slot 1 of the warp that began it, or the slot 0 of warp 0 (begun in an earlier CTA), then
    // the slots 0 of the warps behind until one ends the pair.  All threads share all chains, a pair of columns of a row each.
    __syncthreads();
    float* const slots = reinterpret_cast<float*>(smem);
    const float* const saved = a.partial + (size_t(2) * gridDim.x + size_t(blockIdx.x) * Cfg::kWarps) * Cfg::kSlot;
    if (lo < hi) {
        const Left& l = lefts[wid];
        if (l.has[1]) save(slots + (2 * wid + 1) * Cfg::kSlot);
        else if (l.has[0] && !l.saved) save(slots + 2 * wid * Cfg::kSlot);
    }
    if (wid == 0) {                                                    // chain 0: begun in an earlier CTA, if any; then one per beginner
        const bool carried = lefts[0].has[0] != 0, heads = lane < aw && lefts[lane < Cfg::kWarps ? lane : 0].has[1] != 0;
        const unsigned hm = __ballot_sync(0xffffffffu, heads);
        auto chain = [&](int at, int first, int which) {
            int last = first;
            bool ended = which == 0 && lefts[first].ended;
            while (!ended && last + 1 < aw && lefts[last + 1].has[0]) { ++last; ended = lefts[last].ended != 0; }
            chains[at] = make_int4(first, which, last, which == 1 && ended);
            if (which == 0) chain_at[0] = first;
            else if (!ended) chain_at[1] = first;
        };
        if (lane == 0) { chain_at[0] = chain_at[1] = -1; n_chains = __popc(hm) + carried; }
        __syncwarp();
        if (lane == 0 && carried) chain(0, 0, 0);
        if (heads) chain(int(carried) + __popc(hm & ((1u << lane) - 1u)), lane, 1);
    }
    __syncthreads();
    constexpr int kItems = Cfg::kRows * (D / 2), kThreads = Cfg::kWarps * 32;
    const int joined = n_chains * kItems;
    for (int i = threadIdx.x; i < joined; i += kThreads) {
        const int4 ch = chains[i / kItems];
        const int ln = i & 31, e = (i >> 5) & 1, mt = (i >> 6) % KS, nt = (i % kItems) / (64 * KS);
        const int r = nt * 8 + 2 * (ln & 3) + e, at = ((nt * KS + mt) * 4 + e) * 32 + ln;
        float m = -1.0e30f, l = 0.0f, x = 0.0f, y = 0.0f;
        for (int k = ch.x; k <= ch.z; ++k) {
            const bool far = lefts[k].saved && !(k == ch.x && ch.y == 1);
            const float* p = far ? saved + size_t(k) * Cfg::kSlot : slots + (2 * k + (k == ch.x ? ch.y : 0)) * Cfg::kSlot;
            const float m2 = p[Cfg::kValues + r], top = fmaxf(m, m2), f = exp2_fast(m - top), f2 = exp2_fast(m2 - top);
            x = __fmaf_rn(p[at], f2, __fmul_rn(x, f));
            y = __fmaf_rn(p[at + 64], f2, __fmul_rn(y, f));
            l = __fmaf_rn(p[Cfg::kValues + Cfg::kRows + r], f2, __fmul_rn(l, f));
            m = top;
        }
        const int col = column_of(mt, ln >> 2);
        if (ch.w) {
            const Walk& w = lefts[ch.x].w[1];
            store_pair<D>(a, row_of<Cfg::kRows>(a, w, w.h * a.group, r), col, m, l, x, y);
        } else {                                                       // goes on in the next CTA, or came from the one before
            float* mine = a.partial + (size_t(2) * blockIdx.x + ch.y) * Cfg::kSlot;
            mine[at] = x;
            mine[at + 64] = y;
            if (col == 0) { mine[Cfg::kValues + r] = m; mine[Cfg::kValues + Cfg::kRows + r] = l; }
        }
    }
    const bool crosses[2] = {chain_at[0] >= 0, chain_at[1] >= 0};      // this CTA's part of a pair shared with other CTAs: continued, begun
    // Chains of CTAs: a ticket for each of this CTA's (at most two) parts; the last one of a pair's CTAs joins them.
    if (!crosses[0] && !crosses[1]) return;
    __syncthreads();
    if (threadIdx.x < 2 && crosses[threadIdx.x]) {
        __threadfence();                                               // the CTA's writes, ordered before it by the barrier, before the ticket
        const Left& l = lefts[chain_at[threadIdx.x]];
        const int t0 = l.first[threadIdx.x];
        const int c0 = threadIdx.x == 0 ? of_ctas.of(t0) : int(blockIdx.x), c1 = of_ctas.of(t0 + l.w[threadIdx.x].tiles - 1);
        const int all = atomicAdd(a.tickets + c0, 1) == c1 - c0;
        chain_from[threadIdx.x] = c0;
        chain_parts[threadIdx.x] = all ? c1 - c0 + 1 : 0;
        if (all) a.tickets[c0] = 0;
        __threadfence();
    }
    __syncthreads();
    for (int which = 0; which < 2; ++which) {
        if (!crosses[which] || chain_parts[which] == 0) continue;
        const int c0 = chain_from[which], n = chain_parts[which];
        const Walk& w = lefts[chain_at[which]].w[which];
        auto part = [&](int k) -> const float* { return a.partial + (size_t(2) * (c0 + k) + (k == 0 ? 1 : 0)) * Cfg::kSlot; };
        for (int i = threadIdx.x; i < kItems; i += kThreads) {
            const int ln = i & 31, e = (i >> 5) & 1, mt = (i >> 6) % KS, nt = i / (64 * KS);
            const int r = nt * 8 + 2 * (ln & 3) + e, at = ((nt * KS + mt) * 4 + e) * 32 + ln;
            float m = -1.0e30f, l = 0.0f, x = 0.0f, y = 0.0f;
            for (int k0 = 0; k0 < n; k0 += 8) {                        // eight parts' loads together
                float rm[8], rl[8], rx[8], ry[8], top = m;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float* p = part(min(k0 + k, n - 1));
                    rm[k] = k0 + k < n ? __ldcg(p + Cfg::kValues + r) : -1.0e30f;
                    rl[k] = k0 + k < n ? __ldcg(p + Cfg::kValues + Cfg::kRows + r) : 0.0f;
                    rx[k] = k0 + k < n ? __ldcg(p + at) : 0.0f;
                    ry[k] = k0 + k < n ? __ldcg(p + at + 64) : 0.0f;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) top = fmaxf(top, rm[k]);
                const float f = exp2_fast(m - top);
                l *= f;
                x *= f;
                y *= f;
                m = top;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float g2 = exp2_fast(rm[k] - m);
                    l = __fmaf_rn(rl[k], g2, l);
                    x = __fmaf_rn(rx[k], g2, x);
                    y = __fmaf_rn(ry[k], g2, y);
                }
            }
            store_pair<D>(a, row_of<Cfg::kRows>(a, w, w.h * a.group, r), column_of(mt, ln >> 2), m, l, x, y);
        }
    }
}

// weights[s, h, j] += sum over the rows of 2^(score - reference) / sum, rows in ascending order; a thread owns four slots, 128
// apart.  Scores of sequences that the caller's bounds did not cover are computed again.  Bound by latency: a chain of
// dependent loads (rows, length, statistics, scores) ends in one addition per slot, so the CTAs are to be there all at once
// (16 x 16 heads x 4100 slots: the call takes 35.3 us; 39.2 with a slot per thread and 3.6 waves of CTAs) and what does not depend is asked for first.
constexpr int kWeightSlots = 4, kWeightThreads = 128;

template <int DT>
__global__ void __launch_bounds__(kWeightThreads)
attend_rows_weights(const Cache c, const Rows rows, const RowsArgs a, float sm_log2, float* __restrict__ weights, int64_t stride,
                    const __grid_constant__ bq4k::Tables4 tab) {
    __shared__ float thr[16], val[16], qsm[256];
    __shared__ float2 st[32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int s = blockIdx.z, h = blockIdx.y;
    const int r0 = rows.begin(s), n = max(rows.end(s) - r0, 0), len_all = c.len(s), first = c.counted(s) - n;
    const int len = int(min(int64_t(len_all), stride)), nr = n * a.group;
    if (nr == 0) return;
    const bool stored = len_all <= a.score_len && nr <= a.score_rows;
    if (!stored) {
        bq4k::fill_tables(tab, thr, val);
        __syncthreads();
    }
    const float* sc = a.scores + (size_t(s) * c.heads + h) * a.score_rows * size_t(a.score_len);
    float* mine = weights + (size_t(s) * c.heads + h) * size_t(stride);
    for (int j0 = blockIdx.x * (kWeightThreads * kWeightSlots); j0 < len; j0 += gridDim.x * (kWeightThreads * kWeightSlots)) {
        const int j1 = j0 + int(threadIdx.x);
        float sum[kWeightSlots], before[kWeightSlots];
#pragma unroll
        for (int k = 0; k < kWeightSlots; ++k) {
            sum[k] = 0.0f;
            before[k] = j1 + kWeightThreads * k < len ? mine[j1 + kWeightThreads * k] : 0.0f;
        }
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
                    float x[kWeightSlots];
#pragma unroll
                    for (int k = 0; k < kWeightSlots; ++k) x[k] = j1 + kWeightThreads * k < len ? sc[size_t(r) * a.score_len + j1 + kWeightThreads * k] : -INFINITY;
#pragma unroll
                    for (int k = 0; k < kWeightSlots; ++k)
                        if (m.y > 0.0f) sum[k] += exp2_fast(x[k] - m.x) * m.y;
                } else {
                    const int i = r / a.group;
                    __syncthreads();
                    for (int d = threadIdx.x; d < c.dim; d += kWeightThreads)
                        qsm[d] = bq4k::load1<DT>(a.q, size_t(r0 + i) * size_t(a.q_stride) + size_t(h * a.group + r % a.group) * c.dim + d);
                    __syncthreads();
#pragma unroll
                    for (int k = 0; k < kWeightSlots; ++k) {
                        const int j = j1 + kWeightThreads * k;
                        if (j < len && j < first + i + 1)
                            sum[k] += exp2_fast(dot_row(c.k_codes, c.k_scale, c.row(s, h, j), c.dim, c.block, val, qsm) * sm_log2 - m.x) * m.y;
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kWeightSlots; ++k)
            if (j1 + kWeightThreads * k < len) mine[j1 + kWeightThreads * k] = before[k] + sum[k];
    }
}

}  // namespace bqkvk
