// bqkv_rotary.cu -- the C ABI of the store with positions (see include/bq4.h): the handle, argument checks and launches.
#include "../../include/bq4.h"
#include "bq4_codebook.h"
#include "bq_error.h"
#include "bqkv_checks.h"
#include "bqkv_launch.h"
#include "bqkv_rotary.cuh"

#include <cmath>
#include <new>

struct bqkv_rotary {
    bqkvk::Turns turns;                                                      // first: its steps are read back through the handle in tests
    int axes;
};

namespace {

using namespace bqkvc;

// Whether rows of `xn` bytes, xs apart, meet rows of `yn` bytes, ys apart (n rows of each; a pitch is at least its row's bytes).
// With equal pitches exactly; with others the whole ranges count.
bool rows_meet(const void* x, int64_t xs, int64_t xn, const void* y, int64_t ys, int64_t yn, int64_t n) {
    const int64_t d = reinterpret_cast<intptr_t>(y) - reinterpret_cast<intptr_t>(x), x1 = xs * (n - 1) + xn, y1 = ys * (n - 1) + yn;
    if (d >= x1 || -d >= y1) return false;
    if (xs != ys || n == 1) return true;
    const int64_t off = ((d % xs) + xs) % xs;                                // of y's rows behind the x row before them
    if (off < xn) {                                                          // the y row begins in an x row; is it one that exists?
        const int64_t i = (d - off) / xs;
        if (i + n - 1 >= 0 && i <= n - 1) return true;
    }
    if (off + yn > xs) {                                                     // the y row ends in the next one
        const int64_t i = (d - off) / xs + 1;
        if (i + n - 1 >= 0 && i <= n - 1) return true;
    }
    return false;
}

// f / (2 pi) modulo one in units of 2^-64, rounded: positions are whole numbers, so whole turns per position do not matter.  |f| = m 2^e with a
// 53-bit m, times 1 / (2 pi) in units of 2^-128, is exact but for that number's last unit (2^-112 turns at f = 65536); the bits above
// a turn are dropped from the whole product.  (A quotient in extended precision is off by up to 2^-54 turns there, 5e-7 radian 2^31 positions on.)
uint64_t turns_per_position(double f) {
    if (f == 0.0) return 0;
    constexpr uint64_t hi = 0x28be60db9391054aull, lo = 0x7f09d5f47d4d3770ull;                 // 1 / (2 pi)
    int e;
    const uint64_t m = uint64_t(std::ldexp(std::frexp(std::fabs(f), &e), 53));
    typedef unsigned __int128 u128;
    const u128 a = u128(m) * lo, b = u128(m) * hi + uint64_t(a >> 64);
    const uint64_t word[4] = {uint64_t(a), uint64_t(b), uint64_t(b >> 64), 0};                  // m / (2 pi), units of 2^-128
    const int shift = 64 + 53 - e;                                                              // down to units of 2^-64: 100 at least, as e <= 17
    auto bits_from = [&](int at) -> uint64_t {                                                  // 64 of them, the lowest at `at`
        if (at >= 192) return 0;
        const int w = at / 64, s = at % 64;
        return s == 0 ? word[w] : word[w] >> s | word[w + 1] << (64 - s);
    };
    const uint64_t turns = bits_from(shift) + (bits_from(shift - 1) & 1u);
    return f < 0.0 ? 0 - turns : turns;
}

template <int DT, int D, bool HALVES>
cudaError_t launch_whole(bool folded, unsigned grid, const bqkvk::Cache& d, const bqkvk::Rows& rows, const bqkvk::RotaryArgs& a, const bqkvk::Turns& t, const bq4_codebook& cb,
                         cudaStream_t st) {
    auto* const kernel = folded ? bqkvk::append_rotary<DT, D, HALVES, true> : bqkvk::append_rotary<DT, D, HALVES, false>;
    return bqkvl::launch_after(kernel, dim3(grid), bqkvk::kStoreThreads, size_t(a.batch) * (D / 2) * sizeof(double2), st, d, rows, a, t, cb.tab);
}

template <int DT>
cudaError_t launch(const bqkvk::Cache& d, const bqkvk::Rows& rows, bqkvk::RotaryArgs a, const bqkvk::Turns& t, const bq4_codebook& cb, cudaStream_t st) {
    constexpr int W = bqkvk::kStoreThreads / 32;
    const bool pow2 = (d.block & (d.block - 1)) == 0;
    const bool wide = aligned(a.k, 16) && aligned(a.v, 16) && a.k_stride % 8 == 0 && a.v_stride % 8 == 0 &&
                      (a.q_heads == 0 || (aligned(a.q, 16) && aligned(a.q_out, 16) && a.q_stride % 8 == 0 && a.out_stride % 8 == 0));
    if ((d.dim == 64 || d.dim == 128) && 2 * t.pairs == d.dim && pow2 && wide) {
        // A CTA for every place on the device (four per SM), each with a range of the rows, their items two to a row; fewer rows than that:
        // a row per CTA, and as many CTAs share its steps as there are places and steps for every warp of them.
        const int per_step = 512 / d.dim, steps = (a.q_heads + per_step - 1) / per_step + 2 * ((d.heads + per_step - 1) / per_step), places = 148 * 4;
        const bool many = rows.n >= places;
        a.cuts = 1;
        if (!many) while (a.cuts * 2 * rows.n <= places && a.cuts * W < steps) a.cuts *= 2;
        const int shares = many ? places : rows.n, most = (rows.n + shares - 1) / shares;
        a.parts = many ? 2 : W;
        const int batches = (most + bqkvk::kTurnBatch - 1) / bqkvk::kTurnBatch;
        a.batch = (most + batches - 1) / batches;
        const unsigned grid = unsigned(shares * a.cuts);
        const bool folded = rows.n >= 4 * places && cb.tab.folded;           // its table is filled once per CTA
        if (d.dim == 64) return t.interleaved ? launch_whole<DT, 64, false>(folded, grid, d, rows, a, t, cb, st) : launch_whole<DT, 64, true>(folded, grid, d, rows, a, t, cb, st);
        return t.interleaved ? launch_whole<DT, 128, false>(folded, grid, d, rows, a, t, cb, st) : launch_whole<DT, 128, true>(folded, grid, d, rows, a, t, cb, st);
    }
    const int heads = a.q_heads + 2 * d.heads;
    a.parts = 1;
    while (a.parts < 32 && a.parts * 2 <= heads && (long long)rows.n * a.parts < 148 * 32) a.parts *= 2;
    const long long want = ((long long)rows.n * a.parts + W - 1) / W;
    const unsigned grid = unsigned(want < 148 * 8 ? want : 148 * 8);
    return bqkvl::launch_after(bqkvk::append_rotary_any<DT>, dim3(grid), bqkvk::kStoreThreads, 0, st, d, rows, a, t, cb.tab);
}

}  // namespace

extern "C" {

int bqkv_make_rotary(int rotary_dim, const double* frequencies, const int32_t* axis_of_pair, int axes, int interleaved, bqkv_rotary** out) {
    if (!out) return BQ_ERR_NULL;
    *out = nullptr;
    if (rotary_dim < 2 || rotary_dim > 2 * bqkvk::kMostPairs || rotary_dim % 2 != 0 || axes < 1 || axes > 255) return BQ_ERR_SIZE;
    if (!frequencies || (axes > 1 && !axis_of_pair)) return BQ_ERR_NULL;
    for (int i = 0; i < rotary_dim / 2; ++i) {
        if (!(std::fabs(frequencies[i]) <= 65536.0)) return BQ_ERR_SIZE;     // NaN too
        if (axis_of_pair && (axis_of_pair[i] < 0 || axis_of_pair[i] >= axes)) return BQ_ERR_SIZE;
    }
    bqkv_rotary* r = new (std::nothrow) bqkv_rotary();
    if (!r) return BQ_ERR_CUDA;
    r->axes = axes;
    r->turns.pairs = rotary_dim / 2;
    r->turns.interleaved = interleaved != 0;
    for (int i = 0; i < rotary_dim / 2; ++i) {
        r->turns.step[i] = turns_per_position(frequencies[i]);
        r->turns.axis[i] = axis_of_pair ? uint8_t(axis_of_pair[i]) : 0;
    }
    *out = r;
    return BQ_OK;
}

int bqkv_free_rotary(bqkv_rotary* r) {
    delete r;
    return BQ_OK;
}

int bqkv_append_rotary(const bqkv_cache* c, const bq4_codebook* cb, const bqkv_rotary* rotary, const void* q, const void* k, const void* v, bq_dtype dt,
                       int64_t q_stride, int64_t k_stride, int64_t v_stride, int q_heads, const int32_t* positions, int64_t positions_stride,
                       const int32_t* starts, int n_rows, void* q_out, int64_t q_out_stride, void* cuda_stream) {
    if (!is16(dt)) return BQ_ERR_DTYPE;
    int rc = check_cache(c);
    if (rc == BQ_OK) rc = check_rows(c, starts, n_rows);
    if (rc != BQ_OK) return rc;
    if (!cb) return BQ_ERR_CODEBOOK;
    if (!rotary) return BQ_ERR_NULL;
    if (2 * rotary->turns.pairs > c->head_dim || q_heads < 0 || q_heads > 65535) return BQ_ERR_SIZE;
    if (n_rows == 0) return BQ_OK;
    if (!k || !v || (q_heads > 0 && (!q || !q_out))) return BQ_ERR_NULL;
    const int64_t row = int64_t(c->kv_heads) * c->head_dim, q_row = int64_t(q_heads) * c->head_dim;
    if (n_rows == 1) {                                                       // a single row's stride means nothing
        k_stride = v_stride = row;
        q_stride = q_out_stride = q_row;
    }
    if (k_stride < row || v_stride < row || !aligned(k, 2) || !aligned(v, 2)) return BQ_ERR_SIZE;
    if (positions && (!aligned(positions, 4) || (rotary->axes > 1 && positions_stride < n_rows))) return BQ_ERR_SIZE;
    if (q_heads > 0) {
        if (q_stride < q_row || q_out_stride < q_row || !aligned(q, 2) || !aligned(q_out, 2)) return BQ_ERR_SIZE;
        // a row is written while others are still to be read: q_out is q itself, or meets no input
        const bool in_place = q == q_out && q_stride == q_out_stride;
        if (!in_place && rows_meet(q, 2 * q_stride, 2 * q_row, q_out, 2 * q_out_stride, 2 * q_row, n_rows)) return BQ_ERR_SIZE;
        if (rows_meet(k, 2 * k_stride, 2 * row, q_out, 2 * q_out_stride, 2 * q_row, n_rows) ||
            rows_meet(v, 2 * v_stride, 2 * row, q_out, 2 * q_out_stride, 2 * q_row, n_rows))
            return BQ_ERR_SIZE;
    }
    const bqkvk::Cache d = device_view(c);
    const bqkvk::Rows rows{starts, n_rows};
    bqkvk::RotaryArgs a = {};
    a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v);
    a.q_out = static_cast<uint16_t*>(q_out);
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.out_stride = q_out_stride;
    a.positions = positions; a.axis_stride = positions_stride;
    a.q_heads = q_heads;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = dt == BQ_F16 ? launch<bq4k::kF16>(d, rows, a, rotary->turns, *cb, st) : launch<bq4k::kBF16>(d, rows, a, rotary->turns, *cb, st);
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

}  // extern "C"
