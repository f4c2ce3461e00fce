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
    int q_heads, parts;
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

// cos and sin of pair i at the warp's row
__device__ __forceinline__ double2 turn_of(const Turns& t, const RotaryArgs& a, const TurnWalk& w, int i) {
    const int p = a.positions ? __ldg(a.positions + size_t(t.axis[i]) * size_t(a.axis_stride) + w.r) : w.place;
    const int64_t turn = int64_t(t.step[i] * uint64_t(int64_t(p)));     // of a whole one: [-1/2, 1/2)
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
// into shared memory, then head by head of its part (queries, keys, values); an element per lane and step.
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
        for (int i = lane; i < turns.pairs; i += 32) cs[wid][i] = turn_of(turns, a, now, i);
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

}  // namespace bqkvk
