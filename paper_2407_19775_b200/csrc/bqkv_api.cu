// bqkv_api.cu -- the C ABI of the 4-bit key/value cache (see include/bq4.h): argument checks,
// workspace layout and the choice of kernel.
#include "../../include/bq4.h"
#include "bq4_codebook.h"
#include "bq_error.h"
#include "bqkv_checks.h"
#include "bqkv_launch.h"
#include "bqkv_shared.cuh"

#include <cmath>
#include <mutex>

namespace {

using namespace bqkvc;

constexpr int kMaxDevices = 64;
std::mutex g_lock;

constexpr size_t kWsAlign = 256;
constexpr size_t kHeader = 1024, kTickets = 256;                // the workspace of bqkv_attend: status word, tickets of the rows kernel; zero between calls

size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// Whether out (contiguous rows of `row` elements of two bytes) shares memory with some row of q.
bool overlaps(const void* q, int64_t q_stride, const void* out, int64_t row, int n) {
    const int64_t o0 = reinterpret_cast<intptr_t>(out) - reinterpret_cast<intptr_t>(q), o1 = o0 + 2 * row * n;      // bytes from q on
    const int64_t past = o0 - 2 * row;                                       // a row that begins beyond this one ends beyond o0
    const int64_t first = past < 0 ? 0 : past / (2 * q_stride) + 1;
    return first < n && 2 * q_stride * first < o1;
}

unsigned grid_of(long long want, long long cap) { return unsigned(want < 1 ? 1 : (want > cap ? cap : want)); }
constexpr long long kMaxGrid = 1 << 20;                          // rows beyond it are taken by the kernels' row loops

template <int DT, bool WIDE, bool FOLDED>
cudaError_t launch_append(int lpb, int parts, unsigned grid, cudaStream_t st, const bqkvk::Cache& d, const bqkvk::Rows& rows, const void* k, const void* v, int64_t ks,
                   int64_t vs, const bq4k::Tables4& tab) {
    constexpr int T = bqkvk::kStoreThreads;
    switch (lpb) {
        case 1: return bqkvl::launch_after(bqkvk::append<DT, 1, WIDE, FOLDED>, dim3(grid), T, 0, st, d, rows, k, v, ks, vs, parts, tab);
        case 2: return bqkvl::launch_after(bqkvk::append<DT, 2, WIDE, FOLDED>, dim3(grid), T, 0, st, d, rows, k, v, ks, vs, parts, tab);
        case 4: return bqkvl::launch_after(bqkvk::append<DT, 4, WIDE, FOLDED>, dim3(grid), T, 0, st, d, rows, k, v, ks, vs, parts, tab);
        case 8: return bqkvl::launch_after(bqkvk::append<DT, 8, WIDE, FOLDED>, dim3(grid), T, 0, st, d, rows, k, v, ks, vs, parts, tab);
        case 16: return bqkvl::launch_after(bqkvk::append<DT, 16, WIDE, FOLDED>, dim3(grid), T, 0, st, d, rows, k, v, ks, vs, parts, tab);
        case 32: return bqkvl::launch_after(bqkvk::append<DT, 32, WIDE, FOLDED>, dim3(grid), T, 0, st, d, rows, k, v, ks, vs, parts, tab);
        default: return bqkvl::launch_after(bqkvk::append<DT, 0, WIDE, FOLDED>, dim3(grid), T, 0, st, d, rows, k, v, ks, vs, parts, tab);
    }
}

template <int DT>
cudaError_t append_any(bool wide, bool folded, int lpb, int parts, unsigned grid, cudaStream_t st, const bqkvk::Cache& d, const bqkvk::Rows& rows, const void* k, const void* v,
                int64_t ks, int64_t vs, const bq4k::Tables4& tab) {
    if (wide && folded) return launch_append<DT, true, true>(lpb, parts, grid, st, d, rows, k, v, ks, vs, tab);
    if (wide) return launch_append<DT, true, false>(lpb, parts, grid, st, d, rows, k, v, ks, vs, tab);
    return launch_append<DT, false, false>(lpb, parts, grid, st, d, rows, k, v, ks, vs, tab);
}

// Rows go one to a warp, or in up to eight parts of whole 32-chunk steps where there are too few of them to fill the device;
// enough CTAs to fill it several times over, the row loops take what is left.
int store_parts(const bqkv_cache* c, int n_rows) {
    const int steps = (2 * c->kv_heads * (c->head_dim / 8) + 31) / 32;
    int parts = 1;
    while (parts < 8 && parts * 2 <= steps && (long long)n_rows * parts < 148 * 32) parts *= 2;
    return parts;
}
unsigned store_grid(int n_rows, int parts) {
    const long long units = (long long)n_rows * parts;
    return grid_of((units + bqkvk::kStoreThreads / 32 - 1) / (bqkvk::kStoreThreads / 32), 148 * 8);
}

constexpr int kManyRows = 148 * 32;              // a row for every warp of read_many's grid

template <int DT>
cudaError_t launch_read_many(const bqkvk::Cache& d, const bqkvk::Rows& rows, void* k, void* v, const bq4k::Tables4& tab, cudaStream_t st) {
    static bool opted[kMaxDevices] = {};
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> guard(g_lock);
        if (!opted[dev]) {
            e = cudaFuncSetAttribute(bqkvk::read_many<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, bqkvk::kManySmem);
            if (e != cudaSuccess) return e;
            opted[dev] = true;
        }
    }
    return bqkvl::launch_after(bqkvk::read_many<DT>, dim3(unsigned(sms)), bqkvk::kManyThreads, bqkvk::kManySmem, st, d, rows, k, v, tab);
}

int sm_count(int* sms) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

// What a call does, from its host arguments alone (bqkv_attend_workspace and bqkv_attend agree on it), and its workspace:
// the header; general path: log-sum-exp of every (row, query head); rows path: partial results and (for weights) the softmax
// statistics and the scores within the caller's bounds; tiles path, for weights: softmax
// statistics and the scaled queries.
struct AttendPlan {
    int path;                          // BQKV_PATH_GENERAL, _ROWS or _TILES
    int query_rows, max_len;           // rows per cached head and slots within the caller's bounds
    int splits;                        // general path: CTAs that share a (row, query head)
    size_t lse, partial, stats, scores, scaled, total;
};

constexpr int kMostQueryRows = 16;     // of a pass of the rows kernel: two of its 8-column operands
constexpr int kSizedSms = 148;         // the workspace is sized without asking the device; a larger one runs on this many SMs

// Whether the rows kernel is the faster one.  It reads the cache once per 16 query rows, but spreads that over every SM; the
// tile kernel reads once per 256 rows, and a (sequence, cached head, 256 rows) stays on one SM.  In units of what the tile
// kernel takes for 64 slots (1.4 us; it begins and ends in about 6 of them) an SM of the rows kernel takes 1/8 for 64 slots of
// 16 rows, and 18/8 to begin and join a chain of them.  Measured, 8 cached heads, head_dim 128 (blocks of 64), bf16, us, rows | tiles:
//   1 x 4096 slots: 64 rows 29 | 121, 256 rows 44 | 147;   1 x 32768: 256 rows 189 | 1086
//   16 x 1024: 48 rows 38 | 39, 128 rows 63 | 41;   16 x 8192: 128 rows 203 | 255, 256 rows 354 | 292
//   64 x 512: 48 rows 74 | 73, 128 rows 133 | 75;   64 x 4096: 96 rows 290 | 339, 192 rows 507 | 355
// fp16 takes both longer (two parts of a probability), the rows kernel by up to 18 %: 16 x 8192, 128 rows 236 | 264; 64 x 4096, 96 rows
// 338 | 346; where the sides are close the rule is off by up to 10 %: 64 x 512, 48 rows 83 | 75.
// With weights the rows kernel also writes every score, which is kept to one pass.
bool rows_faster(const bqkv_cache* c, int query_rows, int max_len, bool weights) {
    if (query_rows <= kMostQueryRows) return true;
    if (weights) return false;
    const long long pairs = (long long)c->n_seq * c->kv_heads, passes = (query_rows + kMostQueryRows - 1) / kMostQueryRows;
    const long long waves = (pairs * ((query_rows + 255) / 256) + kSizedSms - 1) / kSizedSms, steps = (max_len + 63) / 64;
    return pairs * passes * (18 + steps) < 8 * kSizedSms * waves * (6 + steps);
}

AttendPlan attend_plan(const bqkv_cache* c, int n_rows, int q_heads, int max_new, int max_len, bool weights, int path, int sms) {
    AttendPlan p = {};
    const int cap = c->max_pages * c->page;
    p.max_len = (max_len <= 0 || max_len > cap) ? cap : max_len;
    const int new_rows = max_new < n_rows ? max_new : n_rows;
    const long long qr = (long long)(new_rows < 1 ? 1 : new_rows) * (q_heads / c->kv_heads);
    p.query_rows = qr > (1 << 20) ? (1 << 20) : int(qr);
    // (the tile kernel counts query rows in 31 bits)
    const bool rows_ok = bqkvl::rows_shape(c->head_dim, c->block, c->page) && (long long)n_rows * q_heads < (1ll << 31);
    p.path = BQKV_PATH_GENERAL;
    // the rows kernel counts its tiles of 32 slots in 32 bits
    const long long row_groups = (long long)n_rows * (q_heads / c->kv_heads) / 8 + c->n_seq + n_rows;
    const bool countable = row_groups * c->kv_heads < (1ll << 31) / (cap / 32 + 1);
    if (path == BQKV_PATH_ROWS && !countable) path = BQKV_PATH_GENERAL;
    if (rows_ok && path != BQKV_PATH_GENERAL)
        p.path = path == BQKV_PATH_AUTO ? (countable && rows_faster(c, p.query_rows, p.max_len, weights) ? BQKV_PATH_ROWS : BQKV_PATH_TILES) : path;
    size_t at = kHeader;
    auto take = [&](size_t bytes) { const size_t o = at; at += round_up(bytes, kWsAlign); return o; };
    if (p.path == BQKV_PATH_GENERAL) {
        p.lse = take(weights ? size_t(n_rows) * q_heads * 4 : 0);
        // about four CTAs per SM (eight fit), a tile of 256 slots each at least
        const long long pairs = (long long)n_rows * q_heads, most = (p.max_len + bqkvk::kGenThreads - 1) / bqkvk::kGenThreads;
        const long long want = pairs > 0 ? 4 * kSizedSms / pairs : 1;
        p.splits = int(want < 1 ? 1 : want < most ? want : most);
        p.partial = take(p.splits > 1 ? size_t(pairs) * p.splits * (c->head_dim + 2) * 4 : 0);
    } else if (p.path == BQKV_PATH_TILES) {
        if (weights) {
            p.stats = take(size_t(n_rows) * q_heads * 16);
            p.scaled = take(size_t(n_rows) * q_heads * c->head_dim * 2);
        }
    } else {
        const int qrows = p.query_rows < kMostQueryRows ? p.query_rows : kMostQueryRows;
        p.partial = take(bqkvl::rows_partial_floats(c->head_dim, qrows, sms) * 4);
        if (weights) {
            p.stats = take(size_t(n_rows) * q_heads * 8);
            p.scores = take(size_t(c->n_seq) * c->kv_heads * p.query_rows * size_t(p.max_len) * 4);
        }
    }
    p.total = at;
    return p;
}

// A call whose sequences share prefixes: both sides' plans, the parts of the prefix side and the workspace behind the own side's.
struct SharedPlan {
    AttendPlan own, prefix;
    int prefix_parts;                  // of every (row, query head): with the own side's they are joined
    int own_blocks, prefix_blocks;     // general kernel: of eight query rows, per (sequence, cached head)
    size_t partial, sums, softmax, total;
};

// The parts of a prefix's slots, where the tile kernel takes them: as many CTAs share a block of 256 query rows as make the whole call
// shortest.  In microseconds, a CTA takes about 18 and 1.4 for 64 slots, and a part's sums are written and read at about 4 TB/s.
int tile_parts(long long blocks, int max_len, long long pairs, int dim, double* cost_out) {
    const long long steps = (max_len + 63) / 64;
    const double part = double(pairs) * dim * 8.0 / 4.0e6;
    int best = 1;
    double least = 1e30;
    for (int s = 1; s < bqkvk::kMostParts && (s == 1 || 2 * s <= steps); ++s) {
        const double cost = double((blocks * s + kSizedSms - 1) / kSizedSms) * (18.0 + 1.4 * double((steps + s - 1) / s)) + part * s;
        if (cost < least) { least = cost; best = s; }
    }
    *cost_out = least;
    return best;
}
// What the rows kernel takes for them: a walk over 32 slots of up to 16 rows by each of its warps, a pass for every 16 rows, and the joins of a
// pair that many CTAs share.  Measured, us, both kernels' whole calls with the own slots, rows | tiles (bf16, head_dim 128 where not said):
//   1 x 8192 slots, 8 heads: 64 rows 43 | 49, 128 rows 58 | 50;   1 x 2000: 16 rows 31 | 30, 256 rows 54 | 47;   1 x 16000, 1 head: 32 rows 60 | 35
//   5 x 3000, 8 heads: 26 rows 57 | 60;   3 x 16000, 16 heads of 64: 32 rows 106 | 174;   1 x 16000: 96 rows 91 | 83
double rows_cost(long long pairs, long long query_rows, int max_len) {
    const double passes = double((query_rows + kMostQueryRows - 1) / kMostQueryRows), chains = double(pairs) * passes;
    return 12.0 + (passes - 1.0) + 2.6 * chains * double((max_len + 31) / 32) / (kSizedSms * 8) + (chains < kSizedSms ? 0.3 * kSizedSms / chains : 0.0);
}

SharedPlan shared_plan(const bqkv_cache* c, const bqkv_cache* pc, int n_rows, int q_heads, int max_new, int max_len, int max_shared, int max_prefix, bool weights,
                       int path) {
    SharedPlan p = {};
    if (max_shared <= 0 || max_shared > n_rows) max_shared = n_rows;
    const int own_path = path == BQKV_PATH_GENERAL ? BQKV_PATH_GENERAL : BQKV_PATH_AUTO;
    p.own = attend_plan(c, n_rows, q_heads, max_new, max_len, weights, own_path, kSizedSms);
    p.prefix = attend_plan(pc, n_rows, q_heads, max_shared, max_prefix, false, path == BQKV_PATH_AUTO ? BQKV_PATH_TILES : path, kSizedSms);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += round_up(bytes, kWsAlign); return o; };
    const long long pairs = (long long)n_rows * q_heads;
    if (p.own.path == BQKV_PATH_GENERAL || p.prefix.path == BQKV_PATH_GENERAL) {      // both or none: their parts differ in form
        p.own = attend_plan(c, n_rows, q_heads, max_new, max_len, weights, BQKV_PATH_GENERAL, kSizedSms);
        p.prefix = attend_plan(pc, n_rows, q_heads, max_shared, max_prefix, false, BQKV_PATH_GENERAL, kSizedSms);
        // Blocks for as many rows as a sequence may have, but no more CTAs than fill the device many times over (a CTA takes further blocks in
        // turn).  Four CTAs per SM, 64 slots each at least; by the rows of the call where they are more than the bound says.
        auto parts_of = [&](const bqkv_cache* x, const AttendPlan& a, int* blocks) {
            const long long chains = (long long)x->n_seq * x->kv_heads, most_blocks = (kSizedSms * 64 + chains - 1) / chains;
            const long long need = (a.query_rows + bqkvk::kPartRows - 1) / bqkvk::kPartRows, by_rows = pairs / bqkvk::kPartRows;
            *blocks = int(need < 1 ? 1 : need < most_blocks ? need : most_blocks);
            const long long ctas = chains * *blocks > by_rows ? chains * *blocks : by_rows;
            const long long want = 4 * kSizedSms / ctas, most = (a.max_len + 63) / 64;
            return int(want < 1 ? 1 : want < most ? want : most < 1 ? 1 : most);
        };
        p.own.splits = parts_of(c, p.own, &p.own_blocks);
        p.prefix.splits = parts_of(pc, p.prefix, &p.prefix_blocks);
        at = p.own.total;
        p.prefix_parts = p.prefix.splits;
        p.partial = take(size_t(pairs) * (p.own.splits + p.prefix.splits) * (c->head_dim + 2) * 4);
        p.total = at;
        return p;
    }
    double cost = 0.0;
    // (the rows of a prefix as they are on average: the bound holds for the largest)
    const long long heads = (long long)pc->n_seq * pc->kv_heads, rows_each = ((n_rows + pc->n_seq - 1) / pc->n_seq) * (long long)(q_heads / c->kv_heads);
    const long long query_rows = rows_each < 1 ? 1 : rows_each < p.prefix.query_rows ? rows_each : p.prefix.query_rows;
    p.prefix_parts = tile_parts(heads * ((query_rows + 255) / 256), p.prefix.max_len, pairs, c->head_dim, &cost);
    if (path == BQKV_PATH_AUTO && rows_cost(heads, query_rows, p.prefix.max_len) < cost) {
        const AttendPlan rows = attend_plan(pc, n_rows, q_heads, max_shared, max_prefix, false, BQKV_PATH_ROWS, kSizedSms);
        if (rows.path == BQKV_PATH_ROWS) p.prefix = rows;
    }
    if (p.prefix.path == BQKV_PATH_ROWS) p.prefix_parts = 1;
    at = p.own.total;
    p.partial = take(p.prefix.path == BQKV_PATH_ROWS ? p.prefix.total - kHeader : 0);
    p.sums = take(size_t(pairs) * (1 + p.prefix_parts) * c->head_dim * 4);
    p.softmax = take(size_t(pairs) * (1 + p.prefix_parts) * 8);
    p.total = at;
    return p;
}

// What the two caches of such a call have in common.
int check_prefix(const bqkv_cache* c, const bqkv_cache* pc) {
    return pc->kv_heads == c->kv_heads && pc->head_dim == c->head_dim && pc->block == c->block ? BQ_OK : BQ_ERR_SIZE;
}

bqkvk::RowsArgs rows_args(const bqkv_cache* c, const bq4_codebook* cb, const void* q, int64_t q_stride, bq_dtype dt, int q_heads, float sm_scale, void* out) {
    bqkvk::RowsArgs a = {};
    a.q = q; a.q_stride = q_stride; a.bf16 = dt == BQ_BF16; a.q_heads = q_heads; a.group = q_heads / c->kv_heads;
    a.score_scale = float(double(sm_scale) * 1.4426950408889634 / cb->unit);
    a.inv_unit = 1.0f / cb->unit;
    a.out = out;
    return a;
}

int check_heads(const bqkv_cache* c, int q_heads) {
    return (q_heads < 1 || q_heads % c->kv_heads != 0 || q_heads / c->kv_heads > 1024 || q_heads > 65535) ? BQ_ERR_SIZE : BQ_OK;
}

}  // namespace

extern "C" {

int bqkv_append(const bqkv_cache* c, const bq4_codebook* cb, const void* k, const void* v, bq_dtype dt, int64_t k_stride, int64_t v_stride,
                const int32_t* starts, int n_rows, void* cuda_stream) {
    if (!is16(dt)) return BQ_ERR_DTYPE;
    int rc = check_cache(c);
    if (rc == BQ_OK) rc = check_rows(c, starts, n_rows);
    if (rc != BQ_OK) return rc;
    if (!cb) return BQ_ERR_CODEBOOK;
    if (n_rows == 0) return BQ_OK;
    if (!k || !v) return BQ_ERR_NULL;
    const int64_t row = int64_t(c->kv_heads) * c->head_dim;
    if (n_rows == 1) k_stride = v_stride = row;                              // a single row's stride means nothing
    if (k_stride < row || v_stride < row) return BQ_ERR_SIZE;
    if (!aligned(k, 2) || !aligned(v, 2)) return BQ_ERR_SIZE;
    const bool wide = aligned(k, 16) && aligned(v, 16) && k_stride % 8 == 0 && v_stride % 8 == 0;
    const bqkvk::Cache d = device_view(c);
    const bqkvk::Rows rows{starts, n_rows};
    const int lpb = log2_exact(c->block / 8) >= 0 ? c->block / 8 : 0;
    const int parts = store_parts(c, n_rows);
    const unsigned grid = store_grid(n_rows, parts);
    // the folded table is filled once per CTA (9 KB): worth it when a CTA has several rows to store
    const bool folded = cb->tab.folded && n_rows >= 148 * 8 * (bqkvk::kStoreThreads / 32) / 4;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = dt == BQ_F16 ? append_any<bq4k::kF16>(wide, folded, lpb, parts, grid, st, d, rows, k, v, k_stride, v_stride, cb->tab)
                                       : append_any<bq4k::kBF16>(wide, folded, lpb, parts, grid, st, d, rows, k, v, k_stride, v_stride, cb->tab);
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

int bqkv_read(const bqkv_cache* c, const bq4_codebook* cb, const int32_t* starts, int n_rows, void* k_out, void* v_out, bq_dtype dt, void* cuda_stream) {
    if (!is16(dt)) return BQ_ERR_DTYPE;
    int rc = check_cache(c);
    if (rc == BQ_OK) rc = check_rows(c, starts, n_rows);
    if (rc != BQ_OK) return rc;
    if (!cb) return BQ_ERR_CODEBOOK;
    if (n_rows == 0) return BQ_OK;
    if (!k_out || !v_out) return BQ_ERR_NULL;
    if (!aligned(k_out, 16) || !aligned(v_out, 16)) return BQ_ERR_SIZE;
    const bqkvk::Cache d = device_view(c);
    const bqkvk::Rows rows{starts, n_rows};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool pow2 = d.chunk_shift >= 0 && d.block_shift >= 0;
    if (pow2 && d.chunk_shift >= 1 && d.block_shift >= 1 && n_rows >= kManyRows && aligned(k_out, 32) && aligned(v_out, 32)) {
        const cudaError_t e = dt == BQ_F16 ? launch_read_many<bq4k::kF16>(d, rows, k_out, v_out, cb->tab, st) : launch_read_many<bq4k::kBF16>(d, rows, k_out, v_out, cb->tab, st);
        return e == cudaSuccess ? BQ_OK : cuda_fail(e);
    }
    const int parts = store_parts(c, n_rows);
    const unsigned grid = store_grid(n_rows, parts);
    constexpr int T = bqkvk::kStoreThreads;
    auto* const kernel = dt == BQ_F16 ? (pow2 ? bqkvk::read_rows<bq4k::kF16, true> : bqkvk::read_rows<bq4k::kF16, false>)
                                      : (pow2 ? bqkvk::read_rows<bq4k::kBF16, true> : bqkvk::read_rows<bq4k::kBF16, false>);
    const cudaError_t e = bqkvl::launch_after(kernel, dim3(grid), T, 0, st, d, rows, k_out, v_out, parts, cb->tab);
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

int bqkv_attend_workspace(const bqkv_cache* c, int n_rows, int q_heads, int max_new, int max_len, int with_weights, size_t* bytes) {
    if (!bytes) return BQ_ERR_NULL;
    int rc = check_sizes(c);
    if (rc == BQ_OK) rc = check_heads(c, q_heads);
    if (rc != BQ_OK) return rc;
    if (n_rows < 0 || max_new < 0) return BQ_ERR_SIZE;
    size_t most = 0;
    for (int path = BQKV_PATH_AUTO; path <= BQKV_PATH_TILES; ++path) {
        if (path == BQKV_PATH_ROWS && with_weights == 1) continue;          // every score of every row: only where it is asked for
        const AttendPlan p = attend_plan(c, n_rows, q_heads, max_new, max_len, with_weights != 0, path, kSizedSms);
        if (p.total > most) most = p.total;
    }
    *bytes = most;
    return BQ_OK;
}

int bqkv_attend(const bqkv_cache* c, const bq4_codebook* cb, const void* q, bq_dtype dt, int64_t q_stride, const int32_t* starts, int n_rows, int q_heads,
                int max_new, int max_len, float sm_scale, float* weights, int64_t weights_stride, void* out, void* workspace, size_t workspace_bytes,
                int path, void* cuda_stream) {
    if (!is16(dt)) return BQ_ERR_DTYPE;
    int rc = check_cache(c);
    if (rc == BQ_OK) rc = check_rows(c, starts, n_rows);
    if (rc == BQ_OK) rc = check_heads(c, q_heads);
    if (rc != BQ_OK) return rc;
    if (!cb) return BQ_ERR_CODEBOOK;
    if (max_new < 0 || !std::isfinite(sm_scale) || (weights && weights_stride < 0)) return BQ_ERR_SIZE;
    if (path < BQKV_PATH_AUTO || path > BQKV_PATH_TILES) return BQKV_ERR_PATH;
    if (n_rows == 0) return BQ_OK;
    if (!q || !out) return BQ_ERR_NULL;
    if (n_rows == 1) q_stride = int64_t(q_heads) * c->head_dim;             // a single row's stride means nothing
    if (q_stride < int64_t(q_heads) * c->head_dim) return BQ_ERR_SIZE;
    if (!aligned(q, 2) || !aligned(out, 16)) return BQ_ERR_SIZE;
    // in place a row's queries are read before it is written, but those of weights once more after that
    const int64_t row = int64_t(q_heads) * c->head_dim;
    if (overlaps(q, q_stride, out, row, n_rows) && (weights || q != out || q_stride != row)) return BQ_ERR_SIZE;
    int sms = kSizedSms;
    AttendPlan p = attend_plan(c, n_rows, q_heads, max_new, max_len, weights != nullptr, path, kSizedSms);
    if (p.path != BQKV_PATH_GENERAL && !(aligned(q, 4) && q_stride % 2 == 0)) {          // the other kernels read pairs of elements
        if (path != BQKV_PATH_AUTO) return BQKV_ERR_PATH;
        p = attend_plan(c, n_rows, q_heads, max_new, max_len, weights != nullptr, BQKV_PATH_GENERAL, kSizedSms);
    }
    if (path != BQKV_PATH_AUTO && p.path != path) return BQKV_ERR_PATH;
    if (!workspace || !aligned(workspace, kWsAlign) || workspace_bytes < p.total) return BQKV_ERR_WORKSPACE;
    const bqkvk::Cache d = device_view(c);
    const bqkvk::Rows rows{starts, n_rows};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(workspace);
    if (p.path != BQKV_PATH_GENERAL) {
        const double log2e = 1.4426950408889634;
        bqkvk::RowsArgs a = rows_args(c, cb, q, q_stride, dt, q_heads, sm_scale, out);
        cudaError_t e;
        if (p.path == BQKV_PATH_ROWS) {
            rc = sm_count(&sms);
            if (rc != BQ_OK) return rc;
            if (sms > kSizedSms) sms = kSizedSms;
            a.partial = reinterpret_cast<float*>(ws + p.partial);
            a.tickets = reinterpret_cast<int*>(ws + kTickets);
            if (weights) {
                a.stats = reinterpret_cast<float2*>(ws + p.stats);
                a.scores = reinterpret_cast<float*>(ws + p.scores);
                a.score_rows = p.query_rows;
                a.score_len = p.max_len;
            }
            e = bqkvl::launch_rows(p.query_rows < kMostQueryRows ? p.query_rows : kMostQueryRows, sms, d, rows, a, *cb, st);
            if (e == cudaSuccess && weights) e = bqkvl::launch_weights(d, rows, a, *cb, float(double(sm_scale) * log2e), p.max_len, weights, weights_stride, st);
        } else {
            bqkvl::TilesCall t = {q, q_stride, a.bf16, q_heads, sm_scale, out, weights, weights_stride, p.max_len, nullptr, nullptr, reinterpret_cast<int*>(ws), {}, 1, 0};
            if (weights) {
                t.stats = reinterpret_cast<float4*>(ws + p.stats);
                t.scaled = reinterpret_cast<uint32_t*>(ws + p.scaled);
            }
            e = bqkvl::launch_tiles(p.query_rows, d, rows, t, *cb, st);
            if (e == cudaSuccess && weights) e = bqkvl::launch_tiles_weights(d, rows, t, *cb, st);
        }
        return e == cudaSuccess ? BQ_OK : cuda_fail(e);
    }
    max_len = p.max_len;
    float* lse = weights ? reinterpret_cast<float*>(ws + p.lse) : nullptr;
    const dim3 grid(grid_of(n_rows, kMaxGrid), unsigned(q_heads), unsigned(p.splits));
    float* partial = reinterpret_cast<float*>(ws + p.partial);
    if (dt == BQ_F16) bqkvk::attend_general<bq4k::kF16><<<grid, bqkvk::kGenThreads, 0, st>>>(d, rows, q, q_stride, q_heads, sm_scale, out, lse, partial, cb->tab);
    else bqkvk::attend_general<bq4k::kBF16><<<grid, bqkvk::kGenThreads, 0, st>>>(d, rows, q, q_stride, q_heads, sm_scale, out, lse, partial, cb->tab);
    if (p.splits > 1) {
        const dim3 jgrid(grid.x, grid.y);
        const bqkvk::PartRows whole{starts, n_rows, 0, 0, nullptr};
        if (dt == BQ_F16) bqkvk::join_general<bq4k::kF16><<<jgrid, 128, 0, st>>>(whole, c->n_seq, 0, q_heads, c->head_dim, p.splits, p.splits, partial, out, lse);
        else bqkvk::join_general<bq4k::kBF16><<<jgrid, 128, 0, st>>>(whole, c->n_seq, 0, q_heads, c->head_dim, p.splits, p.splits, partial, out, lse);
    }
    if (weights) {
        const dim3 wgrid(grid_of((max_len + bqkvk::kGenThreads - 1) / bqkvk::kGenThreads, 65535), unsigned(c->kv_heads), unsigned(c->n_seq));
        if (dt == BQ_F16)
            bqkvk::weights_general<bq4k::kF16><<<wgrid, bqkvk::kGenThreads, 0, st>>>(d, rows, q, q_stride, q_heads, sm_scale, lse, weights, weights_stride, cb->tab);
        else
            bqkvk::weights_general<bq4k::kBF16><<<wgrid, bqkvk::kGenThreads, 0, st>>>(d, rows, q, q_stride, q_heads, sm_scale, lse, weights, weights_stride, cb->tab);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

int bqkv_attend_shared_workspace(const bqkv_cache* c, const bqkv_cache* prefix, int n_rows, int q_heads, int max_new, int max_len, int max_shared, int max_prefix,
                                 int with_weights, size_t* bytes) {
    if (!bytes) return BQ_ERR_NULL;
    int rc = check_sizes(c);
    if (rc == BQ_OK) rc = check_sizes(prefix);
    if (rc == BQ_OK) rc = check_prefix(c, prefix);
    if (rc == BQ_OK) rc = check_heads(c, q_heads);
    if (rc != BQ_OK) return rc;
    if (n_rows < 0 || max_new < 0) return BQ_ERR_SIZE;
    size_t most = 0;
    for (int path = BQKV_PATH_AUTO; path <= BQKV_PATH_TILES; ++path) {
        const SharedPlan p = shared_plan(c, prefix, n_rows, q_heads, max_new, max_len, max_shared, max_prefix, with_weights != 0, path);
        if (p.total > most) most = p.total;
    }
    *bytes = most;
    return BQ_OK;
}

int bqkv_attend_shared(const bqkv_cache* c, const bqkv_cache* prefix, const bq4_codebook* cb, const int32_t* members, const void* q, bq_dtype dt, int64_t q_stride,
                       const int32_t* starts, int n_rows, int q_heads, int max_new, int max_len, int max_shared, int max_prefix, float sm_scale, float* weights,
                       int64_t weights_stride, void* out, void* workspace, size_t workspace_bytes, int path, void* cuda_stream) {
    if (!is16(dt)) return BQ_ERR_DTYPE;
    int rc = check_cache(c);
    if (rc == BQ_OK) rc = check_cache(prefix);
    if (rc == BQ_OK) rc = check_prefix(c, prefix);
    if (rc == BQ_OK) rc = check_rows(c, starts, n_rows);
    if (rc == BQ_OK) rc = check_heads(c, q_heads);
    if (rc != BQ_OK) return rc;
    if (!cb) return BQ_ERR_CODEBOOK;
    if (max_new < 0 || !std::isfinite(sm_scale) || (weights && weights_stride < 0)) return BQ_ERR_SIZE;
    if (path < BQKV_PATH_AUTO || path > BQKV_PATH_TILES) return BQKV_ERR_PATH;
    if (!members && prefix->n_seq != 1) return BQ_ERR_NULL;                 // who shares which of them?
    if (n_rows == 0) return BQ_OK;
    if (!q || !out) return BQ_ERR_NULL;
    const int64_t row = int64_t(q_heads) * c->head_dim;
    if (n_rows == 1) q_stride = row;                                        // a single row's stride means nothing
    if (q_stride < row) return BQ_ERR_SIZE;
    if (!aligned(q, 2) || !aligned(out, 16)) return BQ_ERR_SIZE;
    // results are written behind the last reading of the queries, but for those of weights
    if (weights && overlaps(q, q_stride, out, row, n_rows)) return BQ_ERR_SIZE;
    SharedPlan p = shared_plan(c, prefix, n_rows, q_heads, max_new, max_len, max_shared, max_prefix, weights != nullptr, path);
    if (p.own.path != BQKV_PATH_GENERAL && !(aligned(q, 4) && q_stride % 2 == 0)) {      // the other kernels read pairs of elements
        if (path != BQKV_PATH_AUTO) return BQKV_ERR_PATH;
        p = shared_plan(c, prefix, n_rows, q_heads, max_new, max_len, max_shared, max_prefix, weights != nullptr, BQKV_PATH_GENERAL);
    }
    if (path != BQKV_PATH_AUTO && p.prefix.path != path) return BQKV_ERR_PATH;
    if (p.own.path == BQKV_PATH_GENERAL && overlaps(q, q_stride, out, row, n_rows) && (q != out || q_stride != row)) return BQ_ERR_SIZE;
    if (!workspace || !aligned(workspace, kWsAlign) || workspace_bytes < p.total) return BQKV_ERR_WORKSPACE;
    const bqkvk::Cache d = device_view(c), dp = device_view(prefix);
    const bqkvk::Rows rows{starts, n_rows};
    const bqkvk::PartRows own{starts, n_rows, 0, 0, nullptr}, shared{starts, n_rows, 1, c->n_seq, members};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(workspace);
    const int64_t pairs = int64_t(n_rows) * q_heads;
    if (p.own.path == BQKV_PATH_GENERAL) {
        const int all = p.own.splits + p.prefix.splits;
        float *lse = weights ? reinterpret_cast<float*>(ws + p.own.lse) : nullptr, *partial = reinterpret_cast<float*>(ws + p.partial);
        const unsigned grid_rows = grid_of(n_rows, kMaxGrid);
        auto* const kernel = dt == BQ_F16 ? bqkvk::attend_part_general<bq4k::kF16> : bqkvk::attend_part_general<bq4k::kBF16>;
        kernel<<<dim3(unsigned(c->n_seq) * p.own_blocks, unsigned(c->kv_heads), unsigned(p.own.splits)), bqkvk::kPartThreads, 0, st>>>(
            d, own, q, q_stride, q_heads, sm_scale, p.own_blocks, partial, 0, all, cb->tab);
        kernel<<<dim3(unsigned(prefix->n_seq) * p.prefix_blocks, unsigned(c->kv_heads), unsigned(p.prefix.splits)), bqkvk::kPartThreads, 0, st>>>(
            dp, shared, q, q_stride, q_heads, sm_scale, p.prefix_blocks, partial, p.own.splits, all, cb->tab);
        auto* const join = dt == BQ_F16 ? bqkvk::join_general<bq4k::kF16> : bqkvk::join_general<bq4k::kBF16>;
        join<<<dim3(grid_rows, unsigned(q_heads)), 128, 0, st>>>(shared, c->n_seq, prefix->n_seq, q_heads, c->head_dim, p.own.splits, all, partial, out, lse);
        if (weights) {
            const dim3 wgrid(grid_of((p.own.max_len + bqkvk::kGenThreads - 1) / bqkvk::kGenThreads, 65535), unsigned(c->kv_heads), unsigned(c->n_seq));
            auto* const weigh = dt == BQ_F16 ? bqkvk::weights_general<bq4k::kF16> : bqkvk::weights_general<bq4k::kBF16>;
            weigh<<<wgrid, bqkvk::kGenThreads, 0, st>>>(d, rows, q, q_stride, q_heads, sm_scale, lse, weights, weights_stride, cb->tab);
        }
        const cudaError_t e = cudaGetLastError();
        return e == cudaSuccess ? BQ_OK : cuda_fail(e);
    }
    int sms = 0;
    rc = sm_count(&sms);
    if (rc != BQ_OK) return rc;
    if (sms > kSizedSms) sms = kSizedSms;
    // part 0: the own slots; the prefix's parts behind it
    const bqkvk::Parts parts{reinterpret_cast<float*>(ws + p.sums), reinterpret_cast<float2*>(ws + p.softmax), 1};
    const bqkvk::Parts behind{parts.sums + pairs * c->head_dim, parts.softmax + pairs, 0};
    bqkvk::RowsArgs a = rows_args(c, cb, q, q_stride, dt, q_heads, sm_scale, out);
    a.tickets = reinterpret_cast<int*>(ws + kTickets);
    bqkvl::TilesCall t = {q, q_stride, a.bf16, q_heads, sm_scale, out, weights, weights_stride, p.own.max_len, nullptr, nullptr, reinterpret_cast<int*>(ws), parts, 1, pairs};
    float2* stats2 = nullptr;
    cudaError_t e;
    if (p.prefix.path == BQKV_PATH_ROWS) {
        bqkvk::RowsArgs b = a;
        b.partial = reinterpret_cast<float*>(ws + p.partial);
        b.parts = behind;
        e = bqkvl::launch_rows_part(p.prefix.query_rows < kMostQueryRows ? p.prefix.query_rows : kMostQueryRows, sms, dp, shared, b, *cb, st);
    } else {
        bqkvl::TilesCall b = t;
        b.weights = nullptr;
        b.max_len = p.prefix.max_len;
        b.parts = behind;
        b.splits = p.prefix_parts;
        e = bqkvl::launch_tiles_parts(p.prefix.query_rows, dp, shared, b, *cb, st);
    }
    if (e != cudaSuccess) return cuda_fail(e);
    if (p.own.path == BQKV_PATH_ROWS) {
        a.partial = reinterpret_cast<float*>(ws + p.own.partial);
        a.parts = parts;
        if (weights) {
            stats2 = a.stats = reinterpret_cast<float2*>(ws + p.own.stats);
            a.scores = reinterpret_cast<float*>(ws + p.own.scores);
            a.score_rows = p.own.query_rows;
            a.score_len = p.own.max_len;
        }
        e = bqkvl::launch_rows_part(p.own.query_rows < kMostQueryRows ? p.own.query_rows : kMostQueryRows, sms, d, own, a, *cb, st);
    } else {
        if (weights) {
            t.stats = reinterpret_cast<float4*>(ws + p.own.stats);
            t.scaled = reinterpret_cast<uint32_t*>(ws + p.own.scaled);
        }
        e = bqkvl::launch_tiles_parts(p.own.query_rows, d, own, t, *cb, st);
    }
    if (e != cudaSuccess) return cuda_fail(e);
    auto* const join = c->head_dim == 64 ? (dt == BQ_F16 ? bqkvk::join_parts<bq4k::kF16, 64> : bqkvk::join_parts<bq4k::kBF16, 64>)
                                         : (dt == BQ_F16 ? bqkvk::join_parts<bq4k::kF16, 128> : bqkvk::join_parts<bq4k::kBF16, 128>);
    const unsigned grid = grid_of((pairs + bqkvk::kJoinThreads / 32 - 1) / (bqkvk::kJoinThreads / 32), kSizedSms * 8);
    e = bqkvl::launch_after(join, dim3(grid), bqkvk::kJoinThreads, 0, st, shared, c->n_seq, prefix->n_seq, q_heads, 1 + p.prefix_parts, parts, out, stats2, t.stats);
    if (e == cudaSuccess && weights)
        e = p.own.path == BQKV_PATH_ROWS ? bqkvl::launch_weights(d, rows, a, *cb, float(double(sm_scale) * 1.4426950408889634), p.own.max_len, weights, weights_stride, st)
                                         : bqkvl::launch_tiles_weights(d, rows, t, *cb, st);
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

int bqkv_kernel_status(void* workspace, int* status_out) {
    if (!workspace || !status_out) return BQ_ERR_NULL;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(status_out, workspace, sizeof(int), cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && *status_out != 0) e = cudaMemset(workspace, 0, sizeof(int));
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

int bqkv_evict_workspace(const bqkv_cache* c, int budget, size_t* bytes) {
    if (!bytes) return BQ_ERR_NULL;
    const int rc = check_sizes(c);
    if (rc != BQ_OK) return rc;
    if (budget < 1) return BQ_ERR_SIZE;
    *bytes = round_up(size_t(c->n_seq) * c->kv_heads * 2 * size_t(budget) * 4, kWsAlign);
    return BQ_OK;
}

int bqkv_evict(const bqkv_cache* c, float* weights, int64_t weights_stride, int budget, int sinks, int recent, void* workspace, size_t workspace_bytes,
               void* cuda_stream) {
    const int rc = check_cache(c);
    if (rc != BQ_OK) return rc;
    if (budget < 1 || sinks < 0 || recent < 0 || int64_t(sinks) + recent > budget) return BQ_ERR_SIZE;
    if (!weights) return BQ_ERR_NULL;
    if (weights_stride < 1) return BQ_ERR_SIZE;
    size_t want = 0;
    bqkv_evict_workspace(c, budget, &want);
    if (!workspace || !aligned(workspace, kWsAlign) || workspace_bytes < want) return BQKV_ERR_WORKSPACE;
    if (int64_t(budget) >= int64_t(c->max_pages) * c->page) return BQ_OK;       // no sequence can exceed it
    const bqkvk::Cache d = device_view(c);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = bqkvl::launch_evict(d, weights, weights_stride, budget, sinks, recent, workspace, st);
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

}  // extern "C"
