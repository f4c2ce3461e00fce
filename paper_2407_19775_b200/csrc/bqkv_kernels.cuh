// bqkv_kernels.cuh -- device code of the 4-bit key/value cache (sm_100a): the store and its
// inverse, eviction, and the general attention kernels (any head size, block and page).
//
// The codec is the one of bq4_kernels.cuh (bf16 scale rounded up, one IEEE quotient, the number
// of midpoints below it), so that a cache row holds the bits bq4_quantize_s16 writes.
#pragma once

#include "bq4_kernels.cuh"

namespace bqkvk {

using bq4k::kBF16;
using bq4k::kF16;

// The cache as the kernels see it; the same fields as bqkv_cache, checked by the host.
struct Cache {
    uint8_t* k_codes;
    uint8_t* v_codes;
    uint16_t* k_scale;
    uint16_t* v_scale;
    const int32_t* table;
    int32_t* lens;
    int n_pages, heads, page, dim, block, n_seq, max_pages, table_stride;
    int page_shift, chunk_shift, block_shift;        // log2 of page, dim / 8 (chunks of eight elements per row) and block / 8, or -1

    // Slots counted into a sequence, and those of them that the table has room for.  A row's place goes by the former: rows past
    // the table's end have none and are dropped, while the rows before them stay where they are.
    __device__ __forceinline__ int counted(int s) const { return max(lens[s], 0); }
    __device__ __forceinline__ int held(int count) const { return min(count, max_pages * page); }
    __device__ __forceinline__ int len(int s) const { return held(counted(s)); }
    // The slot of row r of a call, the rows of sequence s ending before row `end`; -1: none, because the row belongs to no sequence,
    // or the sequence has not that many slots, or the slot lies past the table's end.
    __device__ __forceinline__ int slot(int s, int r, int end) const {
        if (r >= end) return -1;
        const int j = counted(s) - (end - r);
        return j < max_pages * page ? max(j, -1) : -1;
    }
    // row number, in units of rows of one head, of slot j of sequence s in the pools of head h
    __device__ __forceinline__ size_t row(int s, int h, int j) const {
        const int p = page_shift >= 0 ? j >> page_shift : j / page;
        const int pg = min(max(table[size_t(s) * table_stride + p], 0), n_pages - 1);
        return (size_t(pg) * heads + h) * page + (j - p * page);
    }
};

// What the kernels in front may have written (pools, table, lens, starts, members, positions, queries) is read by ordinary loads everywhere, which see
// it behind griddepcontrol.wait.  The read-only path (__ldg, or const __restrict__) is for what does not change while a kernel is resident, and
// a kernel that starts early is resident while those in front of it still write.
__device__ __forceinline__ int quotient_of(int a, int b, int shift) { return shift >= 0 ? a >> shift : a / b; }

// The last s of 0 .. n - 1 with begin(s) <= r (empty sequences before it share its start), found by the whole warp: each step compares
// 32 evenly spaced ones, two steps for 1024 sequences.  The same r in all lanes.
template <typename Begin>
__device__ __forceinline__ int last_begun(int r, int n, Begin begin) {
    int lo = 0, hi = n;                                                 // begin(lo) <= r; begin(hi) > r or hi == n
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + step * int(threadIdx.x & 31);
        const unsigned le = __ballot_sync(0xffffffffu, at < hi && begin(at) <= r) | 1u;
        const int k = 31 - __clz(le);
        hi = min(hi, lo + step * (k + 1));
        lo += step * k;
    }
    return lo;
}

// The rows of a call.
struct Rows {
    const int32_t* starts;                 // n_seq + 1, or null: one row per sequence
    int n;
    __device__ __forceinline__ int begin(int s) const { return starts ? min(max(starts[s], 0), n) : s; }
    __device__ __forceinline__ int end(int s) const { return starts ? min(max(starts[s + 1], 0), n) : s + 1; }
    // The slot of the first of a sequence's `rows` rows: they are its last ones, and see the slots up to their own.
    __device__ __forceinline__ int first(int counted, int /* held */, int rows) const { return counted - rows; }
    // The sequence of row r.
    __device__ __forceinline__ int seq(int r, int n_seq) const {
        if (!starts) return r;
        return last_begun(r, n_seq, [this](int s) { return starts[s]; });
    }
};

// The same of a call whose slots are attended to in parts.  `shared`: the sequences here are prefixes, each shared by the call's sequences
// members[s] .. members[s + 1] - 1 (null: one prefix, all of the call's n_own sequences), whose rows all lie behind its slots.
struct PartRows {
    const int32_t* starts;
    int n, shared, n_own;
    const int32_t* members;
    __device__ __forceinline__ int first_member(int s) const {
        if (!shared) return s;
        return members ? min(max(members[s], 0), n_own) : s == 0 ? 0 : n_own;
    }
    __device__ __forceinline__ int begin(int s) const {
        const int at = first_member(s);
        return starts ? min(max(starts[at], 0), n) : at;
    }
    __device__ __forceinline__ int end(int s) const { return begin(s + 1); }
    __device__ __forceinline__ int first(int counted, int held, int rows) const { return shared ? held : counted - rows; }
};
template <bool PARTS> struct RowsOf { using type = Rows; };
template <> struct RowsOf<true> { using type = PartRows; };

// Where the partial results of a call whose slots are attended to in several parts go: of every (row, query head) and part the sums of
// probabilities times values, not yet divided, and (reference, sum) of the softmax, in log2 units.  A part that saw nothing has sum 0
// and no values.
struct Parts {
    float* sums;                           // [rows of the call * query heads][dim]
    float2* softmax;
    int beside;                            // runs beside the kernel before it, of the same call: see after_before()
};
// The kernels of such a call touch nothing of each other's, so the second may run on SMs that the first has left.  The first waits for the kernels
// before the call and lets its dependents start only then; the second need not wait for anything, as the first has, but it ends behind it,
// for the sake of the kernel that joins the parts and waits for the second alone.
__device__ __forceinline__ void after_before(const Parts& p) {
    if (!p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ void end_behind(const Parts& p) {
    if (p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
}

__device__ __forceinline__ float scale_of(const uint16_t* p, size_t i) { return __uint_as_float(uint32_t(p[i]) << 16); }

// ------------------------------------------------------------------------------------------
// append: a row of the call (its keys and its values) goes to `parts` warps, one for many rows, several for a decode step's
// few; a lane takes chunks of eight elements.  Finding a row (its sequence, its page) is a chain of dependent loads: a warp
// looks up its next row while it works on one.  Measured: 8 prompts up to 2048 tokens, 8 heads of 128, bf16: 57 MB (16-bit rows in, about
// a quarter of them out) in 36 us, 1.6 TB/s, four times what the bytes need; 29 instructions per element, of which the same exact codes
// take the tensor call (bq4_quantize_s16) a third of the time, so that it is this form of the walk that bounds it.  64 single
// rows: 2.7 us, launch and latency.
//
// LPB > 0: a block is LPB = block / 8 consecutive chunks (a power of two up to 32), its absmax a segmented shuffle.  LPB == 0
// (other blocks, e.g. 40): every chunk reads its whole block again from L1 for the absmax.  WIDE: rows are 16-byte aligned;
// otherwise element loads.  FOLDED: codes by the folded table (one lookup per element; its per-lane copies are worth filling
// for many rows); otherwise the 4-step search over the midpoints.
constexpr int kStoreThreads = 256;

// A warp's walk over the (row, part) units of a call: first slot row in the pools (of head 0), or no slot.
struct RowWalk {
    int unit, step, r, part;
    bool has;
    size_t row0;
    __device__ __forceinline__ void look(const Cache& c, const Rows& rows, int parts) {
        r = unit / parts;
        part = unit - r * parts;
        has = false;
        row0 = 0;
        if (r >= rows.n) return;
        const int s = rows.seq(r, c.n_seq);
        const int slot = c.slot(s, r, rows.end(s));
        has = slot >= 0;
        if (has) row0 = c.row(s, 0, slot);
    }
};
__device__ __forceinline__ RowWalk first_row(const Cache& c, const Rows& rows, int parts) {
    RowWalk w;
    w.unit = int(blockIdx.x) * (kStoreThreads / 32) + int(threadIdx.x >> 5);
    w.step = int(gridDim.x) * (kStoreThreads / 32);
    w.look(c, rows, parts);
    return w;
}

template <int DT, int LPB, bool WIDE, bool FOLDED>
__global__ void __launch_bounds__(kStoreThreads)
append(const Cache c, const Rows rows, const void* k, const void* v, int64_t k_stride, int64_t v_stride, int parts,
       const __grid_constant__ bq4k::Tables4 tab) {
    __shared__ float thr[16], val[16];
    __shared__ __align__(128) uint32_t ent[FOLDED ? bq4k::kFoldCells * 32 : 1];
    uint32_t ent_lane = 0;
    if constexpr (FOLDED) {
        for (int i = threadIdx.x; i < bq4k::kFoldCells * 32; i += kStoreThreads) ent[i] = tab.entry[i >> 5];
        ent_lane = uint32_t(__cvta_generic_to_shared(ent)) + (threadIdx.x & 31) * 4u - bq4k::kFoldCellBase * 128u;
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bq4k::fill_tables(tab, thr, val);
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    const int lane = threadIdx.x & 31;
    const int per_head = c.dim / 8, per_row = c.heads * per_head, cpb = c.block / 8, nb = c.dim / c.block;
    // steps of 32 chunks: the keys' first, then the values'; a part is a range of them.  The next step's chunk is loaded before
    // this one's arithmetic, across rows too.
    const int sp = (per_row + 31) / 32;
    auto chunk_of = [&](const RowWalk& w, int q, bool& in, bool& is_v) -> int {
        is_v = q >= sp;
        const int e = (is_v ? q - sp : q) * 32 + lane;
        in = e < per_row && w.has;
        return e < per_row ? e : 0;
    };
    auto load = [&](const RowWalk& w, bool is_v, int chunk, float (&f)[8]) {
        const size_t el = size_t(w.r) * size_t(is_v ? v_stride : k_stride) + size_t(chunk) * 8;
        if constexpr (WIDE) bq4k::load8<DT>(static_cast<const uint16_t*>(is_v ? v : k) + el, 0, f);
        else {
#pragma unroll
            for (int u = 0; u < 8; ++u) f[u] = bq4k::load1<DT>(is_v ? v : k, el + u);
        }
    };
    RowWalk now = first_row(c, rows, parts);
    float ahead[8] = {};
    bool in, is_v;
    if (now.r < rows.n) {
        const int e = chunk_of(now, now.part * 2 * sp / parts, in, is_v);
        load(now, is_v, e, ahead);
    }
    while (now.r < rows.n) {
        RowWalk next = now;
        next.unit += next.step;
        const int qa = now.part * 2 * sp / parts, q1 = (now.part + 1) * 2 * sp / parts;
        for (int q = qa; q < q1; ++q) {
            if (q + 1 == q1) next.look(c, rows, parts);                 // its first chunk is loaded below
            const int e = chunk_of(now, q, in, is_v);
            float f[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) f[u] = ahead[u];
            {
                bool in2, v2;
                if (q + 1 < q1) {
                    const int e2 = chunk_of(now, q + 1, in2, v2);
                    load(now, v2, e2, ahead);
                } else if (next.r < rows.n) {
                    const int e2 = chunk_of(next, next.part * 2 * sp / parts, in2, v2);
                    load(next, v2, e2, ahead);
                }
            }
            float a = 0.0f;
#pragma unroll
            for (int u = 0; u < 8; u += 2) asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(a) : "f"(a), "f"(f[u]), "f"(f[u + 1]));
            if constexpr (LPB > 0) {
#pragma unroll
                for (int m = 1; m < LPB; m <<= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, m));
            } else {
                const int b0 = quotient_of(e, cpb, c.block_shift) * cpb;
                for (int b = 0; b < cpb; ++b) {
                    float g[8];
                    load(now, is_v, b0 + b, g);
#pragma unroll
                    for (int u = 0; u < 8; ++u) a = fmaxf(a, fabsf(g[u]));
                }
            }
            a = bq4k::block_scale<true>(a);
            const float d = (a != 0.0f) ? a : 1.0f;
            const bool quick = __all_sync(0xffffffffu, (d >= 5.421010862427522e-20f) && (d <= 1.8446744073709552e19f));
            float rc, xh[8];
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rc) : "f"(d));
            bq4k::quotients8(f, d, rc, quick, xh);
            uint32_t neg0 = 0, neg1 = 0;
            if constexpr (FOLDED) {
                neg0 = bq4k::sign_bytes_32(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                neg1 = bq4k::sign_bytes_32(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
            }
            const uint32_t word = bq4k::codes8<FOLDED>(xh, ent_lane, tab.neg_limit, thr, neg0, neg1);
            if (in) {
                const int h = quotient_of(e, per_head, c.chunk_shift), ch = e - h * per_head, b = quotient_of(ch, cpb, c.block_shift);
                const size_t row = now.row0 + size_t(h) * c.page;
                reinterpret_cast<uint32_t*>(is_v ? c.v_codes : c.k_codes)[row * per_head + ch] = word;
                if (ch == b * cpb) (is_v ? c.v_scale : c.k_scale)[row * nb + b] = uint16_t(__float_as_uint(a) >> 16);
            }
        }
        now = next;
    }
}

// read: the inverse, rows dealt out likewise; eight elements per lane and step: 4 bytes of codes in, 16 out.  Bound by its bytes.
template <int DT, bool POW2 /* dim / 8 and block / 8 are powers of two */>
__global__ void __launch_bounds__(kStoreThreads)
read_rows(const Cache c, const Rows rows, void* __restrict__ k_out, void* __restrict__ v_out, int parts, const __grid_constant__ bq4k::Tables4 tab) {
    constexpr int U = 4;                                                // steps whose loads go out together
    __shared__ float thr[16], val[16];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bq4k::fill_tables(tab, thr, val);
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    const int lane = threadIdx.x & 31;
    const int per_head = c.dim / 8, per_row = c.heads * per_head, cpb = c.block / 8, nb = c.dim / c.block;
    const int sp = (per_row + 31) / 32;                                 // steps of 32 chunks: the keys' first, then the values'
    for (RowWalk now = first_row(c, rows, parts); now.r < rows.n;) {
        RowWalk next = now;
        next.unit += next.step;
        const int qa = now.part * 2 * sp / parts, q1 = (now.part + 1) * 2 * sp / parts;
        for (int q0 = qa; q0 < q1; q0 += U) {
            uint32_t w[U];
            uint16_t a16[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool is_v = q0 + u >= sp;
                const int e = (q0 + u - (is_v ? sp : 0)) * 32 + lane;
                w[u] = 0u;
                a16[u] = 0;
                if (q0 + u < q1 && e < per_row && now.has) {
                    const int h = POW2 ? e >> c.chunk_shift : e / per_head, ch = e - h * per_head, b = POW2 ? ch >> c.block_shift : ch / cpb;
                    const size_t row = now.row0 + size_t(h) * c.page;
                    w[u] = reinterpret_cast<const uint32_t*>(is_v ? c.v_codes : c.k_codes)[row * per_head + ch];
                    a16[u] = (is_v ? c.v_scale : c.k_scale)[row * nb + b];
                }
            }
            if (q0 == qa) next.look(c, rows, parts);                    // under these loads
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool is_v = q0 + u >= sp;
                const int e = (q0 + u - (is_v ? sp : 0)) * 32 + lane;
                if (q0 + u < q1 && e < per_row) {
                    const float a = __uint_as_float(uint32_t(a16[u]) << 16);        // a slot that does not exist: zeros
                    uint32_t y[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = __fmul_rn(val[(w[u] >> (8 * i)) & 15u], a), q = __fmul_rn(val[(w[u] >> (8 * i + 4)) & 15u], a);
                        if constexpr (DT == kBF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y[i]) : "f"(q), "f"(p));
                        else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y[i]) : "f"(q), "f"(p));
                    }
                    if (!now.has) y[0] = y[1] = y[2] = y[3] = 0u;
                    reinterpret_cast<uint4*>(is_v ? v_out : k_out)[size_t(now.r) * per_row + e] = make_uint4(y[0], y[1], y[2], y[3]);
                }
            }
        }
        now = next;
    }
}

// read_many: the same for many rows, bound by instructions as read_rows does it (16 per element), so written for few of them:
// a byte's two values are one 64-bit lookup in a table that every lane has for itself in its own pair of banks, 256 bytes per
// entry from a multiple of 64 KB on, so that one byte permute makes the address; sixteen elements per lane and step, one row's
// loads together.  One CTA per SM; filling the table (64 KB) is what few rows cannot afford.  dim / 16 and block / 16 powers
// of two, outputs 32-byte aligned (256-bit stores: whole sectors).  Measured: 31000 rows of 8 heads of 128: 41 us against 54 by
// read_rows (161 MB, 3.9 TB/s; writes, which are three quarters of it, bound it from 33 us on).
constexpr int kManyThreads = 1024, kManySmem = 2 * 65536 - 1024;

template <int DT>
__global__ void __launch_bounds__(kManyThreads, 1)
read_many(const Cache c, const Rows rows, void* __restrict__ k_out, void* __restrict__ v_out, const __grid_constant__ bq4k::Tables4 tab) {
    extern __shared__ __align__(16) unsigned char many_smem[];
    __shared__ float thr[16], val[16];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bq4k::fill_tables(tab, thr, val);
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // launched with programmatic serialization: the kernels before this one are done
    const int lane = threadIdx.x & 31;
    const uint32_t low = uint32_t(__cvta_generic_to_shared(many_smem)), table = (low + 0xFFFFu) & 0xFFFF0000u, table_lane = table | uint32_t(lane) * 8u;
    for (int i = threadIdx.x; i < 256 * 16; i += kManyThreads) {       // two lanes' copies per store
        const float x = val[(i >> 4) & 15], y = val[i >> 8];
        *reinterpret_cast<float4*>(many_smem + (table - low) + (i >> 4) * 256 + (i & 15) * 16) = make_float4(x, y, x, y);
    }
    __syncthreads();
    const int sh = c.chunk_shift - 1, per_head = c.dim / 16, per_row = c.heads * per_head, nb = c.dim / c.block, bsh = c.block_shift - 1;
    const int units = gridDim.x * (kManyThreads / 32);
    auto look = [&](int r, size_t& row0) -> bool {
        if (r >= rows.n) return false;
        const int s = rows.seq(r, c.n_seq);
        const int slot = c.slot(s, r, rows.end(s));
        if (slot < 0) return false;
        row0 = c.row(s, 0, slot);
        return true;
    };
    int r = int(blockIdx.x) * (kManyThreads / 32) + int(threadIdx.x >> 5);
    size_t row0 = 0;
    bool has = look(r, row0);
    while (r < rows.n) {
        size_t next0 = 0;
        bool next_has = false;
        for (int e0 = lane; e0 - lane < per_row; e0 += 64) {            // two steps of the keys and of the values
            uint2 w[4];
            uint16_t a16[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int e = e0 + (u & 1) * 32;
                w[u] = make_uint2(0u, 0u);
                a16[u] = 0;
                if (e < per_row && has) {
                    const int h = e >> sh, ch = e - (h << sh);
                    const size_t row = row0 + uint32_t(h * c.page);
                    w[u] = reinterpret_cast<const uint2*>(u >= 2 ? c.v_codes : c.k_codes)[row * uint32_t(per_head) + ch];
                    a16[u] = (u >= 2 ? c.v_scale : c.k_scale)[row * uint32_t(nb) + (ch >> bsh)];
                }
            }
            if (e0 == lane) next_has = look(r + units, next0);          // under these loads: a chain of loads of its own
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int e = e0 + (u & 1) * 32;
                if (e >= per_row) continue;
                const float a = __uint_as_float(uint32_t(a16[u]) << 16);
                uint32_t y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float p, q;
                    asm("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(p), "=f"(q) : "r"(bq4k::prmt(i < 4 ? w[u].x : w[u].y, table_lane, 0x7604u | uint32_t(i & 3) << 4)));
                    p = __fmul_rn(p, a);
                    q = __fmul_rn(q, a);
                    if constexpr (DT == kBF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y[i]) : "f"(q), "f"(p));
                    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y[i]) : "f"(q), "f"(p));
                }
                if (!has) {                                             // a slot that does not exist: zeros
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = 0u;
                }
                void* to = static_cast<char*>(u >= 2 ? v_out : k_out) + (size_t(r) * uint32_t(per_row) + e) * 32;
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]), "r"(y[4]),
                             "r"(y[5]), "r"(y[6]), "r"(y[7]) : "memory");
            }
        }
        r += units;
        row0 = next0;
        has = next_has;
    }
}

// ------------------------------------------------------------------------------------------
// attend_general: one CTA per (row of the call, query head), for head sizes and blocks the other kernels do not take.  Tiles of
// 256 slots: a thread takes one slot's score, the running maximum and sum follow, then a thread takes a byte of the value rows (two
// columns) of every G-th slot, G = 256 / (dim / 2); the G partial columns are added in order at the end.  fp32 throughout.
// Few rows over many slots are split over gridDim.z CTAs, whose partial results join_general adds in order.  Bound by latency and
// instructions (a lookup and a product per element, keys read once per query head).  lse (when not null) receives log of the
// softmax sum, for the weights kernel.  Measured, head_dim 80, 4 x 4 heads: 16 x 4000 slots 119 us, 2 x 32000 slots 126 us (1079 in
// one CTA per row and head).
constexpr int kGenThreads = 256;

__device__ __forceinline__ float dot_row(const uint8_t* codes, const uint16_t* scale, size_t row, int dim, int block, const float* val, const float* q) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(codes) + row * size_t(dim / 8);
    float x = 0.0f;
    for (int b = 0; b < dim / block; ++b) {
        float acc = 0.0f;
        for (int ch = b * block / 8; ch < (b + 1) * block / 8; ++ch) {
            const uint32_t u = w[ch];
#pragma unroll
            for (int e = 0; e < 8; ++e) acc = __fmaf_rn(val[(u >> (4 * e)) & 15u], q[ch * 8 + e], acc);
        }
        x = __fmaf_rn(acc, scale_of(scale, row * size_t(dim / block) + b), x);
    }
    return x;
}

template <int DT>
__global__ void __launch_bounds__(kGenThreads)
attend_general(const Cache c, const Rows rows, const void* __restrict__ q, int64_t q_stride, int q_heads, float sm_scale, void* __restrict__ out,
               float* __restrict__ lse, float* __restrict__ partial /* where gridDim.z > 1 */, const __grid_constant__ bq4k::Tables4 tab) {
    constexpr int W = kGenThreads / 32;
    __shared__ float thr[16], val[16], qs[256], ps[kGenThreads], red[2][W], cols[2][kGenThreads];
    __shared__ size_t row_of[kGenThreads];
    bq4k::fill_tables(tab, thr, val);
    const int tid = threadIdx.x, hq = blockIdx.y, h = hq / (q_heads / c.heads), nb = c.dim / c.block;
    const int bytes = c.dim / 2, G = kGenThreads / bytes, col = tid % bytes, grp = tid / bytes;      // G groups of a thread per byte; the rest idle
    const int vb = 2 * col / c.block;
    for (int r = blockIdx.x; r < rows.n; r += gridDim.x) {
        const int s = rows.seq(r, c.n_seq);
        const int end = rows.end(s), counted = c.counted(s);
        const int seen = r < end ? min(max(counted - (end - r) + 1, 0), c.held(counted)) : 0;      // slots 0 .. seen - 1
        __syncthreads();
        for (int d = tid; d < c.dim; d += kGenThreads) qs[d] = bq4k::load1<DT>(q, size_t(r) * size_t(q_stride) + size_t(hq) * c.dim + d);
        float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
        const long long tiles = (max(seen, 0) + kGenThreads - 1) / kGenThreads;
        const int lo = int(tiles * blockIdx.z / gridDim.z) * kGenThreads, hi = int(tiles * (blockIdx.z + 1) / gridDim.z) * kGenThreads;
        for (int t0 = lo; t0 < hi; t0 += kGenThreads) {
            __syncthreads();
            const int j = t0 + tid;
            float x = -INFINITY;
            if (j < seen) {
                const size_t row = c.row(s, h, j);
                row_of[tid] = row;
                x = __fmul_rn(dot_row(c.k_codes, c.k_scale, row, c.dim, c.block, val, qs), sm_scale);
            }
            float mx = x;
#pragma unroll
            for (int k = 16; k >= 1; k >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, k));
            if ((tid & 31) == 0) red[0][tid >> 5] = mx;
            __syncthreads();
            mx = m;
#pragma unroll
            for (int k = 0; k < W; ++k) mx = fmaxf(mx, red[0][k]);                    // finite: slot t0 is seen
            const float corr = expf(m - mx);                                          // 0 on the first tile
            float p = j < seen ? expf(x - mx) : 0.0f;
            ps[tid] = p;
            m = mx;
#pragma unroll
            for (int k = 16; k >= 1; k >>= 1) p += __shfl_xor_sync(0xffffffffu, p, k);
            if ((tid & 31) == 0) red[1][tid >> 5] = p;
            __syncthreads();
            l *= corr;
#pragma unroll
            for (int k = 0; k < W; ++k) l += red[1][k];
            if (grp < G) {
                const int n = min(kGenThreads, seen - t0);
                float a0 = 0.0f, a1 = 0.0f;
#pragma unroll 8
                for (int k = grp; k < n; k += G) {
                    const size_t row = row_of[k];
                    const uint32_t byte = c.v_codes[row * size_t(bytes) + col];
                    const float f = scale_of(c.v_scale, row * nb + vb);
                    a0 = __fmaf_rn(ps[k], __fmul_rn(val[byte & 15u], f), a0);
                    a1 = __fmaf_rn(ps[k], __fmul_rn(val[byte >> 4], f), a1);
                }
                o0 = __fmaf_rn(o0, corr, a0);
                o1 = __fmaf_rn(o1, corr, a1);
            }
        }
        __syncthreads();
        cols[0][tid] = o0;
        cols[1][tid] = o1;
        __syncthreads();
        const size_t pair = size_t(r) * q_heads + hq;
        float* part = partial + (pair * gridDim.z + blockIdx.z) * (c.dim + 2);
        for (int d = tid; d < c.dim; d += kGenThreads) {
            float o = 0.0f;
            for (int k = 0; k < G; ++k) o += cols[d & 1][k * bytes + d / 2];
            if (gridDim.z > 1) part[d] = o;
            else bq4k::store1<DT>(out, pair * c.dim + d, seen > 0 ? __fdiv_rn(o, l) : 0.0f);
        }
        if (tid == 0) {
            if (gridDim.z > 1) { part[c.dim] = m; part[c.dim + 1] = l; }
            else if (lse) lse[pair] = seen > 0 ? m + logf(l) : 0.0f;
        }
    }
}

// The partial results of attend_general's splits, one CTA per (row, query head): columns, then maximum and sum, per split.
// `prefixes` > 0: a row whose sequence shares one of them has `z_all` splits, the others the first `own` of them, and rows of no sequence none.
template <int DT>
__global__ void __launch_bounds__(128)
join_general(const PartRows rows, int n_own, int prefixes, int q_heads, int dim, int own, int z_all, const float* __restrict__ partial, void* __restrict__ out,
             float* __restrict__ lse) {
    for (int r = blockIdx.x; r < rows.n; r += gridDim.x) {
        int splits = z_all;
        if (prefixes > 0) {
            if (r >= (rows.starts ? rows.starts[n_own] : n_own) || (rows.starts && r < rows.starts[0])) continue;
            if (r < rows.begin(0) || r >= rows.begin(prefixes)) splits = own;
        }
        const size_t pair = size_t(r) * q_heads + blockIdx.y;
        const float* part = partial + pair * z_all * (dim + 2);
        float m = -INFINITY, l = 0.0f;
        bool any = false;                                               // a split that saw a slot has a sum of 1 at least, or NaN
        for (int z = 0; z < splits; ++z) {
            m = fmaxf(m, part[z * (dim + 2) + dim]);
            any |= part[z * (dim + 2) + dim + 1] != 0.0f;
        }
        for (int z = 0; any && z < splits; ++z) l = __fmaf_rn(part[z * (dim + 2) + dim + 1], expf(part[z * (dim + 2) + dim] - m), l);
        for (int d = threadIdx.x; d < dim; d += 128) {
            float o = 0.0f;
            for (int z = 0; any && z < splits; ++z) o = __fmaf_rn(part[z * (dim + 2) + d], expf(part[z * (dim + 2) + dim] - m), o);
            bq4k::store1<DT>(out, pair * dim + d, any ? __fdiv_rn(o, l) : 0.0f);
        }
        if (lse && threadIdx.x == 0) lse[pair] = any ? m + logf(l) : 0.0f;
    }
}

// weights_general: weights[s, h, j] += sum over the sequence's rows i and the group's query heads of exp(x - lse); a thread
// owns a slot and adds in ascending order of (row, query head).
template <int DT>
__global__ void __launch_bounds__(kGenThreads)
weights_general(const Cache c, const Rows rows, const void* __restrict__ q, int64_t q_stride, int q_heads, float sm_scale,
                const float* __restrict__ lse, float* __restrict__ weights, int64_t stride, const __grid_constant__ bq4k::Tables4 tab) {
    __shared__ float thr[16], val[16], qs[256];
    bq4k::fill_tables(tab, thr, val);
    const int s = blockIdx.z, h = blockIdx.y, g = q_heads / c.heads;
    const int r0 = rows.begin(s), n = rows.end(s) - r0;
    const int len = int(min(int64_t(c.len(s)), stride));
    const int first = c.counted(s) - n;                                 // slot of the first row
    for (int t0 = blockIdx.x * kGenThreads; t0 < len; t0 += gridDim.x * kGenThreads) {
        const int j = t0 + int(threadIdx.x);
        float sum = 0.0f;
        for (int i = 0; i < n; ++i) {
            const int seen = first + i + 1;
            if (t0 >= seen) continue;                                   // the same for the whole CTA
            for (int u = 0; u < g; ++u) {
                __syncthreads();
                for (int d = threadIdx.x; d < c.dim; d += kGenThreads)
                    qs[d] = bq4k::load1<DT>(q, size_t(r0 + i) * size_t(q_stride) + size_t(h * g + u) * c.dim + d);
                __syncthreads();
                if (j < seen && j < len) {
                    const float x = __fmul_rn(dot_row(c.k_codes, c.k_scale, c.row(s, h, j), c.dim, c.block, val, qs), sm_scale);
                    sum += expf(x - lse[size_t(r0 + i) * q_heads + h * g + u]);
                }
            }
        }
        if (j < len && n > 0) weights[(size_t(s) * c.heads + h) * size_t(stride) + j] += sum;
    }
}

}  // namespace bqkvk
