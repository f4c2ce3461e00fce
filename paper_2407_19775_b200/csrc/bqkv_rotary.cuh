// bqkv_rotary.cuh -- device code of the store with positions (sm_100a): queries and keys of a call are turned by their
// positions, the keys and values go into the 4-bit cache as append writes them.
//
// Pair i of a head's row turns by the angle position * f_i.  The host hands f_i down as turns per position in units of 2^-64,
// modulo a whole turn: position * f_i modulo a turn is then one wrapping 64-bit product, exact to position * 2^-65 turns however
// far the position (an fp32 angle of position 10^6 is off by 0.03 radian, an fp64 one by 10^-10).  sincospi takes it from there
// in 64 bits.
//
// A key's elements are turned in 64 bits and rounded once, to fp32: its codes are those of the correctly rounded row (a row that is
// 2^-24 off lands on another code wherever a quotient lies that near to a midpoint: one element in a few million).  Queries, which
// are rounded to 16 bits anyway, are turned in fp32.
#pragma once

#include "bqkv_kernels.cuh"

namespace bqkvk {

constexpr int kMostPairs = 128;                                         // half of the largest head_dim
constexpr int kTurnBatch = 32;                                          // rows that append_rotary looks up together, a lane each

struct Turns {
    uint64_t step[kMostPairs];                                          // turns per position, units of 2^-64
    uint8_t axis[kMostPairs];                                           // whose position turns the pair
    int pairs, interleaved;                                             // (2i, 2i + 1), or (i, i + pairs)
};

struct RotaryArgs {
    const uint16_t *q, *k, *v;
    uint16_t* q_out;
    int64_t q_stride, k_stride, v_stride, out_stride;
    const int32_t* positions;                                           // [axes][rows], or null: the rows' places as lens counts them
    int64_t axis_stride;
    int q_heads;
    int parts;                                                          // items that a row's heads are dealt out in
    int cuts, batch;                                                    // append_rotary: CTAs that share rows; rows looked up together
};

// A warp's walk over the (row, part) units of a call: the row's place, and its first slot row in the pools (of head 0).
struct TurnWalk {
    int unit, step, r, part, place;
    bool held, belongs;                                                 // there is a slot for it; it is a sequence's row at all
    size_t row0;
    __device__ __forceinline__ void look(const Cache& c, const Rows& rows, int parts) {
        r = unit / parts;
        part = unit - r * parts;
        held = belongs = false;
        row0 = 0;
        place = 0;
        if (r >= rows.n) return;
        const int s = rows.seq(r, c.n_seq), end = rows.end(s);
        belongs = r < end;
        place = c.counted(s) - (end - r);
        const int slot = c.slot(s, r, end);
        held = slot >= 0;
        if (held) row0 = c.row(s, 0, slot);
    }
};
__device__ __forceinline__ TurnWalk first_turn(const Cache& c, const Rows& rows, int parts) {
    TurnWalk w;
    w.unit = int(blockIdx.x) * (kStoreThreads / 32) + int(threadIdx.x >> 5);
    w.step = int(gridDim.x) * (kStoreThreads / 32);
    w.look(c, rows, parts);
    return w;
}

// cos and sin of a pair at a position
__device__ __forceinline__ double2 turn_of(uint64_t step, int position) {
    const int64_t turn = int64_t(step * uint64_t(int64_t(position)));   // of a whole one: [-1/2, 1/2)
    double2 cs;
    sincospi(double(turn) * 1.0842021724855044e-19 /* 2^-63 */, &cs.y, &cs.x);
    return cs;
}

template <int DT>
__device__ __forceinline__ uint32_t narrow2(float lo, float hi) {
    uint32_t d;
    if constexpr (DT == kBF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// ------------------------------------------------------------------------------------------
// append_rotary_any: any head size, block, alignment and number of turned elements.  A warp takes a (row, part): its turns once,
// into shared memory, then head by head of its part (queries, keys, values); an element per lane and step.  Bound by instructions: 11008 rows of 32
// queries, 8 keys and 8 values of 128 of which 64 elements turn, bf16, 246 us (the kernel below, which turns all of them, 64).
template <int DT>
__global__ void __launch_bounds__(kStoreThreads)
append_rotary_any(const Cache c, const Rows rows, const RotaryArgs a, const __grid_constant__ Turns turns, const __grid_constant__ bq4k::Tables4 tab) {
    constexpr int W = kStoreThreads / 32;
    __shared__ float thr[16], val[16];
    __shared__ double2 cs[W][kMostPairs];
    __shared__ float row_of_warp[W][2 * kMostPairs];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bq4k::fill_tables(tab, thr, val);
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, heads = a.q_heads + 2 * c.heads, rot = 2 * turns.pairs, nb = c.dim / c.block;
    float* const f = row_of_warp[wid];
    for (TurnWalk now = first_turn(c, rows, a.parts); now.r < rows.n; now.unit += now.step, now.look(c, rows, a.parts)) {
        if (!now.belongs) continue;
        __syncwarp();
        for (int i = lane; i < turns.pairs; i += 32) cs[wid][i] = turn_of(turns.step[i], a.positions ? a.positions[size_t(turns.axis[i]) * size_t(a.axis_stride) + now.r] : now.place);
        __syncwarp();
        const int h1 = int((long long)(now.part + 1) * heads / a.parts);
        for (int h = int((long long)now.part * heads / a.parts); h < h1; ++h) {
            const int kind = h < a.q_heads ? 0 : h < a.q_heads + c.heads ? 1 : 2;      // query, key, value
            if (kind > 0 && !now.held) break;
            const int hk = h - a.q_heads - (kind == 2 ? c.heads : 0);
            const uint16_t* x = kind == 0 ? a.q + int64_t(now.r) * a.q_stride + int64_t(h) * c.dim
                                          : (kind == 1 ? a.k + int64_t(now.r) * a.k_stride : a.v + int64_t(now.r) * a.v_stride) + int64_t(hk) * c.dim;
            for (int i = lane; i < c.dim; i += 32) f[i] = bq4k::load1<DT>(x, i);
            __syncwarp();
            if (kind < 2) {
                for (int i = lane; i < turns.pairs; i += 32) {
                    const int ia = turns.interleaved ? 2 * i : i, ib = turns.interleaved ? 2 * i + 1 : i + turns.pairs;
                    const float u = f[ia], v = f[ib];
                    const double2 t = cs[wid][i];
                    if (kind == 0) {
                        const float tc = float(t.x), ts = float(t.y);
                        f[ia] = __fmaf_rn(u, tc, -__fmul_rn(v, ts));
                        f[ib] = __fmaf_rn(v, tc, __fmul_rn(u, ts));
                    } else {
                        f[ia] = float(__fma_rn(double(u), t.x, -__dmul_rn(double(v), t.y)));
                        f[ib] = float(__fma_rn(double(v), t.x, __dmul_rn(double(u), t.y)));
                    }
                }
                __syncwarp();
            }
            if (kind == 0) {
                uint16_t* y = a.q_out + int64_t(now.r) * a.out_stride + int64_t(h) * c.dim;
                for (int i = lane; i < c.dim; i += 32) {
                    if (i < rot || y != x) bq4k::store1<DT>(y, i, f[i]);
                }
            } else {
                const size_t row = now.row0 + size_t(hk) * c.page;
                // a block's scale by the warp, then a word of eight codes to a lane
                for (int b = 0; b < nb; ++b) {
                    float m = 0.0f;
                    for (int i = lane; i < c.block; i += 32) m = fmaxf(m, fabsf(f[b * c.block + i]));
#pragma unroll
                    for (int s = 16; s >= 1; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
                    m = bq4k::block_scale<true>(m);
                    if (lane == 0) (kind == 2 ? c.v_scale : c.k_scale)[row * nb + b] = uint16_t(__float_as_uint(m) >> 16);
                    const float d = m != 0.0f ? m : 1.0f;
                    for (int i = lane; i < c.block; i += 32) f[b * c.block + i] = __fdiv_rn(f[b * c.block + i], d);
                }
                __syncwarp();
                for (int ch = lane; ch < c.dim / 8; ch += 32) {
                    uint32_t word = 0;
#pragma unroll
                    for (int u = 0; u < 8; ++u) word |= bq4k::search16(thr, f[ch * 8 + u]) << (4 * u);
                    reinterpret_cast<uint32_t*>(kind == 2 ? c.v_codes : c.k_codes)[row * (c.dim / 8) + ch] = word;
                }
            }
            __syncwarp();
        }
    }
}

// ------------------------------------------------------------------------------------------
// append_rotary: whole rows of 64 or 128 turned elements, blocks a power of two, everything 16-byte aligned.
//
// A lane has two chunks of eight elements of a head, those that turn with one another: chunks l and l + D / 16 (halves), or 2 l and
// 2 l + 1 (interleaved); D / 16 lanes make a head, 512 elements a step of the warp.  A lane's eight pairs are the same in every step, so
// their cos and sin are computed once per (row, part) by the warp, two pairs a lane, and stay in registers for the queries (fp32) and in
// shared memory for the keys (64 bits, laid out so that the lanes of a head meet no bank twice).  Steps of queries first, then of keys,
// then of values; the next step's chunks are on their way during a step's arithmetic.
// Measured: 11008 rows, 32 queries, 8 keys and 8 values of 128, bf16, 58 us cold for 237 MB (4.1 TB/s): issue 0.57 of the cycles, ALU 45 %, nothing
// else above a fifth; the queries by themselves 31 us (5.8 TB/s).  64 rows in a graph with the read-back 10.0 us, a single one 6.5.
// A key's elements are 24-bit numbers x; their quotients by a scale d of 8 significant bits come out right from the same one correction that
// 16-bit elements take: the first quotient is off by 2^-22, so what the correction rounds is off by 2^-44, while x / d lies 2^-33 (relative)
// or more from any midpoint m of two fp32 numbers, as x - m d is a multiple of 2^-33 and not 0 (m d has 25 bits at least).
template <int DT>
__device__ __forceinline__ void widen_pair(uint32_t w, float& lo, float& hi) {
    if constexpr (DT == kBF16) {
        lo = __uint_as_float(w << 16);
        hi = __uint_as_float(w & 0xffff0000u);
    } else {
        const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w));
        lo = p.x;
        hi = p.y;
    }
}

template <int DT, int D, bool HALVES, bool FOLDED>
__global__ void __launch_bounds__(kStoreThreads, 4)
append_rotary(const Cache c, const Rows rows, const RotaryArgs a, const __grid_constant__ Turns turns, const __grid_constant__ bq4k::Tables4 tab) {
    constexpr int W = kStoreThreads / 32, LPH = D / 16, HPS = 32 / LPH, PAIRS = D / 2;      // lanes per head, heads per step
    extern __shared__ __align__(16) double2 cs[];                       // [rows of a batch][PAIRS], pair 8 l + j at j LPH + l
    __shared__ float thr[16], val[16];
    __shared__ __align__(128) uint32_t ent[FOLDED ? bq4k::kFoldCells * 32 : 1];
    __shared__ size_t slot_row[kTurnBatch];                             // of a batch's rows: in the pools, of head 0
    __shared__ int place_of[kTurnBatch];                                // as lens counts it
    __shared__ uint8_t state_of[kTurnBatch];                            // 0: of no sequence; 1: without a slot; 2: with one
    uint32_t ent_lane = 0;
    if constexpr (FOLDED) {
        for (int i = threadIdx.x; i < bq4k::kFoldCells * 32; i += kStoreThreads) ent[i] = tab.entry[i >> 5];
        ent_lane = uint32_t(__cvta_generic_to_shared(ent)) + (threadIdx.x & 31) * 4u - bq4k::kFoldCellBase * 128u;
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bq4k::fill_tables(tab, thr, val);
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, l = lane % LPH;
    const int nq = (a.q_heads + HPS - 1) / HPS, nk = (c.heads + HPS - 1) / HPS;
    const int at_x = HALVES ? 8 * l : 16 * l, at_y = HALVES ? 8 * l + D / 2 : 16 * l + 8;      // of this lane's chunks in a turned row

    // The codes of this lane's two chunks, whose blocks reach over lanes of the head, and the blocks' scales.
    auto store = [&](uint32_t* codes, uint16_t* scale /* of the head's row */, bool halves, bool there, const float (&fx)[8], const float (&fy)[8]) {
        float ax = 0.0f, ay = 0.0f;
#pragma unroll
        for (int u = 0; u < 8; u += 2) {
            asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(ax) : "f"(ax), "f"(fx[u]), "f"(fx[u + 1]));
            asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(ay) : "f"(ay), "f"(fy[u]), "f"(fy[u + 1]));
        }
        const int lanes = halves ? min(c.block, D / 2) / 8 : c.block / 16;      // that share a block
        if (halves ? c.block == D : c.block > 8) ax = ay = fmaxf(ax, ay);
        for (int m = 1; m < lanes; m <<= 1) {
            ax = fmaxf(ax, __shfl_xor_sync(0xffffffffu, ax, m));
            ay = fmaxf(ay, __shfl_xor_sync(0xffffffffu, ay, m));
        }
        ax = bq4k::block_scale<true>(ax);
        ay = bq4k::block_scale<true>(ay);
        const float dx = ax != 0.0f ? ax : 1.0f, dy = ay != 0.0f ? ay : 1.0f;
        const bool quick = __all_sync(0xffffffffu, fminf(dx, dy) >= 5.421010862427522e-20f && fmaxf(dx, dy) <= 1.8446744073709552e19f);
        auto code = [&](const float (&f)[8], float d) -> uint32_t {
            float rc, xh[8];
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rc) : "f"(d));
            bq4k::quotients8(f, d, rc, quick, xh);
            uint32_t neg0 = 0, neg1 = 0;
            if constexpr (FOLDED) {
                neg0 = bq4k::sign_bytes_32(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                neg1 = bq4k::sign_bytes_32(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
            }
            return bq4k::codes8<FOLDED>(xh, ent_lane, tab.neg_limit, thr, neg0, neg1);
        };
        const uint32_t wx = code(fx, dx), wy = code(fy, dy);
        if (!there) return;
        const int cx = halves ? l : 2 * l, cy = halves ? l + LPH : 2 * l + 1, first = (1 << c.block_shift) - 1;      // chunks; a block's first has these bits clear
        if (halves) {
            codes[cx] = wx;
            codes[cy] = wy;
        } else {
            *reinterpret_cast<uint2*>(codes + cx) = make_uint2(wx, wy);
        }
        if ((cx & first) == 0) scale[cx >> c.block_shift] = uint16_t(__float_as_uint(ax) >> 16);
        if ((cy & first) == 0) scale[cy >> c.block_shift] = uint16_t(__float_as_uint(ay) >> 16);
    };

    const int scales_shift = (D == 128 ? 4 : 3) - c.block_shift;        // log2 of a row's scales
    // this CTA's rows, in batches; `cuts` CTAs share the steps of the same rows
    const int cut = int(blockIdx.x) % a.cuts, share = int(blockIdx.x) / a.cuts, shares = int(gridDim.x) / a.cuts;
    const int r_begin = int((long long)rows.n * share / shares), r_end = int((long long)rows.n * (share + 1) / shares);
    for (int base = r_begin; base < r_end; base += a.batch) {
        const int nb = min(a.batch, r_end - base);
        if (base != r_begin) __syncthreads();                           // the batch before is done with
        if (wid == 0) {                                                 // a lane looks up a row
            int s = rows.seq(base, c.n_seq);                            // of the first row; the others' lie behind it
            const int r = min(base + lane, rows.n - 1);
            if (rows.starts) {
                while (s + 1 < c.n_seq && rows.starts[s + 1] <= r) ++s;
            } else {
                s = r;
            }
            if (lane < nb) {
                const int end = rows.end(s), slot = c.slot(s, r, end);
                place_of[lane] = c.counted(s) - (end - r);
                state_of[lane] = r >= end ? 0 : slot < 0 ? 1 : 2;
                slot_row[lane] = slot < 0 ? 0 : c.row(s, 0, slot);
            }
            __syncwarp();
        }
        if (!a.positions) __syncthreads();
        static_assert(kStoreThreads % PAIRS == 0, "a thread's pair is the same in every row");
        {
            // (a constant for each lane is slow: once for all rows, and not for threads without a row)
            const int p = int(threadIdx.x) < nb * PAIRS ? threadIdx.x % PAIRS : 0;
            const uint64_t step = turns.step[p];
            const int32_t* const positions = a.positions ? a.positions + size_t(turns.axis[p]) * size_t(a.axis_stride) + base : nullptr;
            for (int row = threadIdx.x / PAIRS; row < nb; row += kStoreThreads / PAIRS)
                cs[row * PAIRS + (p & 7) * LPH + (p >> 3)] = turn_of(step, positions ? positions[row] : place_of[row]);
        }
        __syncthreads();
      // (row, part) items to the warps in turn: steps first, first + stride, ..
      const int stride = a.parts * a.cuts;
      for (int item = wid; item < nb * a.parts; item += W) {
        const int br = item / a.parts, r = base + br, part = (item - br * a.parts) * a.cuts + cut;
        if (state_of[br] == 0) continue;
        const double2* const mine = cs + br * PAIRS;
        // the queries' steps of this part, two of them on their way before anything is looked up
        const int hop = stride * HPS;                                   // heads from one to the next
        int h = part * HPS + lane / LPH;
        const uint16_t* from = a.q + int64_t(r) * a.q_stride + h * D;
        uint4 x[2] = {}, y[2] = {};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (h + i * hop < a.q_heads) {                              // (q_out may be q: not through the read-only path)
                x[i] = *reinterpret_cast<const uint4*>(from + i * hop * D + at_x);
                y[i] = *reinterpret_cast<const uint4*>(from + i * hop * D + at_y);
            }
        if (part < nq) {
            uint64_t c2[4], s2[4], n2[4];                               // of two pairs each
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double2 u = mine[2 * i * LPH + l], v = mine[(2 * i + 1) * LPH + l];
                c2[i] = bq4k::pack2(float(u.x), float(v.x));
                s2[i] = bq4k::pack2(float(u.y), float(v.y));
                n2[i] = bq4k::pack2(-float(u.y), -float(v.y));
            }
            uint16_t* to = a.q_out + int64_t(r) * a.out_stride + h * D;
            from += 2 * hop * D;
#pragma unroll 2
            for (int t = part; t < nq; t += stride, h += hop, from += hop * D, to += hop * D) {
                const uint32_t wx[4] = {x[0].x, x[0].y, x[0].z, x[0].w}, wy[4] = {y[0].x, y[0].y, y[0].z, y[0].w};
                x[0] = x[1];
                y[0] = y[1];
                if (h + 2 * hop < a.q_heads) {
                    x[1] = *reinterpret_cast<const uint4*>(from + at_x);
                    y[1] = *reinterpret_cast<const uint4*>(from + at_y);
                }
                uint32_t ox[4], oy[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x0, x1, y0, y1;
                    widen_pair<DT>(wx[i], x0, x1);
                    widen_pair<DT>(wy[i], y0, y1);
                    if constexpr (HALVES) {
                        const uint64_t x2 = bq4k::pack2(x0, x1), y2 = bq4k::pack2(y0, y1);
                        bq4k::unpack2(bq4k::fma2(x2, c2[i], bq4k::mul2(y2, n2[i])), x0, x1);
                        bq4k::unpack2(bq4k::fma2(y2, c2[i], bq4k::mul2(x2, s2[i])), y0, y1);
                        ox[i] = narrow2<DT>(x0, x1);
                        oy[i] = narrow2<DT>(y0, y1);
                    } else {                                            // a pair per word: pairs i (x) and 4 + i (y)
                        float ca, cb, sa, sb, k0, k1;
                        bq4k::unpack2(c2[i >> 1], k0, k1);
                        ca = i & 1 ? k1 : k0;
                        bq4k::unpack2(s2[i >> 1], k0, k1);
                        sa = i & 1 ? k1 : k0;
                        bq4k::unpack2(c2[2 + (i >> 1)], k0, k1);
                        cb = i & 1 ? k1 : k0;
                        bq4k::unpack2(s2[2 + (i >> 1)], k0, k1);
                        sb = i & 1 ? k1 : k0;
                        ox[i] = narrow2<DT>(__fmaf_rn(x0, ca, -__fmul_rn(x1, sa)), __fmaf_rn(x1, ca, __fmul_rn(x0, sa)));
                        oy[i] = narrow2<DT>(__fmaf_rn(y0, cb, -__fmul_rn(y1, sb)), __fmaf_rn(y1, cb, __fmul_rn(y0, sb)));
                    }
                }
                if (h < a.q_heads) {
                    *reinterpret_cast<uint4*>(to + at_x) = make_uint4(ox[0], ox[1], ox[2], ox[3]);
                    *reinterpret_cast<uint4*>(to + at_y) = make_uint4(oy[0], oy[1], oy[2], oy[3]);
                }
            }
        }
        if (state_of[br] < 2) continue;
        // keys, then values
#pragma unroll 1
        for (int is_v = 0; is_v < 2; ++is_v) {
            const int first = nq + is_v * nk, k0 = (part - first % stride + stride) % stride;      // this part's first step of them
            if (k0 >= nk) continue;
            const bool halves = HALVES || is_v;
            const int ax = halves ? 8 * l : at_x, ay = halves ? 8 * l + D / 2 : at_y;
            int hk = k0 * HPS + lane / LPH;
            const uint16_t* p = (is_v ? a.v + int64_t(r) * a.v_stride : a.k + int64_t(r) * a.k_stride) + hk * D;
            size_t row = slot_row[br] + size_t(hk) * c.page;
            uint4 u = make_uint4(0, 0, 0, 0), v = u;
            if (hk < c.heads) {
                u = *reinterpret_cast<const uint4*>(p + ax);
                v = *reinterpret_cast<const uint4*>(p + ay);
            }
#pragma unroll 1
            for (int t = k0; t < nk; t += stride) {
                const uint32_t wx[4] = {u.x, u.y, u.z, u.w}, wy[4] = {v.x, v.y, v.z, v.w};
                p += hop * D;
                if (hk + hop < c.heads) {
                    u = *reinterpret_cast<const uint4*>(p + ax);
                    v = *reinterpret_cast<const uint4*>(p + ay);
                }
                float fx[8], fy[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    widen_pair<DT>(wx[i], fx[2 * i], fx[2 * i + 1]);
                    widen_pair<DT>(wy[i], fy[2 * i], fy[2 * i + 1]);
                }
                if (!is_v) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const double2 cs2 = mine[j * LPH + l];
                        float& e = HALVES ? fx[j] : j < 4 ? fx[(2 * j) & 7] : fy[(2 * j) & 7];
                        float& f = HALVES ? fy[j] : j < 4 ? fx[(2 * j + 1) & 7] : fy[(2 * j + 1) & 7];
                        const double de = double(e), df = double(f);
                        e = float(__fma_rn(de, cs2.x, -__dmul_rn(df, cs2.y)));
                        f = float(__fma_rn(df, cs2.x, __dmul_rn(de, cs2.y)));
                    }
                }
                store(reinterpret_cast<uint32_t*>(is_v ? c.v_codes : c.k_codes) + row * (D / 8), (is_v ? c.v_scale : c.k_scale) + (row << scales_shift), halves, hk < c.heads, fx, fy);
                hk += hop;
                row += size_t(hop) * c.page;
            }
        }
      }
    }
}

}  // namespace bqkvk
