// mmd_launch.cuh -- the handle of a decomposed matrix, tensor maps, and the choice and launches of the product kernels, for the units that
// hold their instances: mmd_api.cu (plain layers) and mmd_adapted.cu (gemm_tc2 with low-rank adapters) (internal to libbq).
#pragma once

#include "../../include/mmd.h"
#include "bq_error.h"
#include "mmd_kernels.cuh"

#include <cstring>
#include <mutex>
#include <new>

namespace {

constexpr size_t kWsAlign = 256;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
bool is16(int dt) { return dt == BQ_F16 || dt == BQ_BF16; }

// cuTensorMapEncodeTiled through the runtime's entry-point lookup (no link against the driver library)
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    // a function-local static is initialised once, under the language's own lock, however many threads arrive together
    static const EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) == cudaSuccess && qres == cudaDriverEntryPointSuccess)
            return reinterpret_cast<EncodeTiledFn>(p);
        return EncodeTiledFn(nullptr);
    }();
    return fn;
}

// Per-device facts that the launchers look up on first use (shared-memory opt-ins, how many clusters run at once) are
// kept in small tables indexed by the device ordinal and written under this lock: two host threads may issue their
// first call at the same time.  mmd_decompose refuses devices beyond the tables, so an index is always in range.
constexpr int kMaxDevices = 64;
std::mutex g_cache_lock;

// Row-major [rows, cols] matrix of 1- or 2-byte elements, tiles of box_rows x 128 bytes, 128-byte swizzle.
bool make_map(CUtensorMap* map, const void* base, int elem_bytes, uint64_t rows, uint64_t cols, uint32_t box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {cols, rows};
    const cuuint64_t strides[1] = {cols * uint64_t(elem_bytes)};
    const cuuint32_t box[2] = {cuuint32_t(128 / elem_bytes), box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUtensorMapDataType dt = (elem_bytes == 1) ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
    return fn(map, dt, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same matrix (K a multiple of 128, 1-byte elements) seen as (128 bytes, rows, K / 128): one load then brings
// `box_kblocks` K blocks of `box_rows` rows, laid out block after block, each with the 128-byte swizzle.
bool make_map_kblocks(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint32_t box_rows, uint32_t box_kblocks) {
    EncodeTiledFn fn = encode_fn();
    if (!fn || cols % 128 != 0) return false;
    const cuuint64_t dims[3] = {128, rows, cols / 128};
    const cuuint64_t strides[2] = {cols, 128};
    const cuuint32_t box[3] = {128, box_rows, box_kblocks};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int cuda_fail(cudaError_t e) {
    bql::set_last_cuda_error(cudaGetErrorString(e));
    return BQ_ERR_CUDA;
}

}  // namespace

struct mmd_weights {
    int N, K, ko, side_cols, dtype, device, sm_count;
    int rows;                    // of the matrix: N, but for a view whose product has more columns than that (see `linear`)
    void* blob;                  // q | scale | side | idx | status
    int8_t* q;
    float* scale;
    void* side;
    int32_t* idx;
    int* status;
    bool have_maps;
    CUtensorMap map_q[3], map_side[3];       // weight tiles of 256, 128 and 64 rows
    bool have_pair_map;                      // K a multiple of 128: the CTA-pair kernel's view of the codes
    CUtensorMap map_q_pair;                  // (128 bytes, rows, K / 128), boxes of 128 rows x 2 K blocks
};

namespace {

int bn_slot(int bn) { return bn == 256 ? 0 : (bn == 128 ? 1 : 2); }

// Rows of the activation tiles the one-tile-per-CTA kernel loads: a decode step's few rows need only half a tile.
int activation_box_rows(int M) { return M <= 64 ? 64 : 128; }

template <int XDT, int YDT, int BN, int BM, int KPB>
cudaError_t launch_tc_bm(const mmd_weights* w, const CUtensorMap& mqx, const CUtensorMap& msx, const float* sx, void* y, int M, int split,
                         cudaStream_t stream, int n_tile_base = 0, int n_tile_count = -1) {
    using Cfg = mmdk::TcCfg<BN, BM, KPB>;
    static bool opted[kMaxDevices] = {};
    static int max_clusters[kMaxDevices][5] = {};
    if (w->device < 0 || w->device >= kMaxDevices) return cudaErrorInvalidDevice;
    const int d = w->device;
    std::lock_guard<std::mutex> guard(g_cache_lock);              // held to the end: the tables are read on the way to the launch
    if (!opted[d]) {
        const cudaError_t e = cudaFuncSetAttribute(mmdk::gemm_tc<XDT, YDT, BN, BM, KPB>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(Cfg::kSmemBytes));
        if (e != cudaSuccess) return e;
        opted[d] = true;
    }
    int kblocks = (w->K + 127) / 128, sblocks = w->side_cols / 64;
    const int ksteps = (kblocks + KPB - 1) / KPB;
    const int slot = bn_slot(BN);
    CUtensorMap mqw = w->map_q[slot];
    if (KPB > 1 && !make_map_kblocks(&mqw, w->q, uint64_t(w->rows), uint64_t(w->K), BN, KPB)) return cudaErrorInvalidValue;
    int* status = w->status;
    int Mv = M, Nv = w->N;
    const float* swv = w->scale;
    // the ranks' partial sums must fit into rank 0's ring
    if (split > 1 && size_t(split - 1) * BM * BN * 4 > size_t(Cfg::kStages) * Cfg::kStageBytes) split = 1;
    if (split > ksteps) split = ksteps;
    if (split > 4) split = 4;                                    // the largest cluster the exchange is written for (and the table below holds)
    if (split < 1) split = 1;
    cudaLaunchConfig_t cfg = {};
    if (n_tile_count < 0) n_tile_count = (w->N + BN - 1) / BN - n_tile_base;
    cfg.blockDim = dim3(mmdk::kTcThreads, 1, 1);
    cfg.dynamicSmemBytes = Cfg::kSmemBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1;
    attr[1].val.clusterDim.y = 1;
    // The split is there to put one CTA on every SM at the same time.  A cluster's CTAs must sit in one GPC, so fewer
    // clusters of 3 or 4 fit on the device than its SM count suggests; a split whose clusters would not all run at once
    // (a second, nearly empty wave) is lowered until they do.
    const long clusters = long((M + BM - 1) / BM) * n_tile_count;
    for (; split > 1; --split) {
        if (max_clusters[d][split] == 0) {
            cfg.gridDim = dim3(1, unsigned(w->sm_count / split), unsigned(split));
            attr[1].val.clusterDim.z = unsigned(split);
            cfg.attrs = &attr[1];
            cfg.numAttrs = 1;
            int n = 0;
            const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, mmdk::gemm_tc<XDT, YDT, BN, BM, KPB>, &cfg);
            if (e != cudaSuccess) return e;
            max_clusters[d][split] = n > 0 ? n : -1;
        }
        if (clusters <= max_clusters[d][split]) break;
    }
    cfg.gridDim = dim3(unsigned((M + BM - 1) / BM), unsigned(n_tile_count), unsigned(split));
    // The row kernel launched just before lets this kernel start early (its set-up and first weight loads overlap the row
    // kernel); the kernel itself waits for the row kernel's results before it touches them.
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].val.clusterDim.z = unsigned(split);
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, mmdk::gemm_tc<XDT, YDT, BN, BM, KPB>, mqx, mqw, sblocks ? msx : mqx,
                              sblocks ? w->map_side[slot] : w->map_q[slot], sx, swv, y, Mv, Nv, kblocks, sblocks, n_tile_base, status);
}

// At most 64 activation rows: 64-row MMAs and 64-row activation boxes (the host's maps are made to match).
template <int XDT, int YDT, int BN>
cudaError_t launch_tc(const mmd_weights* w, const CUtensorMap& mqx, const CUtensorMap& msx, const float* sx, void* y, int M, int split,
                      cudaStream_t stream) {
    return activation_box_rows(M) == 64 ? launch_tc_bm<XDT, YDT, BN, 64, 1>(w, mqx, msx, sx, y, M, split, stream)
                                        : launch_tc_bm<XDT, YDT, BN, 128, 1>(w, mqx, msx, sx, y, M, split, stream);
}

// 128-column tiles with K a multiple of 128: two K blocks per load (decode-size calls and mid-size products).  `mqx2` is
// the activations' three-dimensional map with boxes of activation_box_rows(M) rows x 2 K blocks.
template <int XDT, int YDT>
cudaError_t launch_tc_decode(const mmd_weights* w, const CUtensorMap& mqx2, const CUtensorMap& msx, const float* sx, void* y, int M, int split,
                             cudaStream_t stream, int n_tile_base = 0, int n_tile_count = -1) {
    return activation_box_rows(M) == 64 ? launch_tc_bm<XDT, YDT, 128, 64, 2>(w, mqx2, msx, sx, y, M, split, stream, n_tile_base, n_tile_count)
                                        : launch_tc_bm<XDT, YDT, 128, 128, 2>(w, mqx2, msx, sx, y, M, split, stream, n_tile_base, n_tile_count);
}

template <int XDT, int YDT>
cudaError_t launch_tcp(const mmd_weights* w, const CUtensorMap& mqx, const float* sx, const void* sidex, void* y, int M, cudaStream_t stream) {
    static bool opted[kMaxDevices] = {};
    if (w->device < 0 || w->device >= kMaxDevices) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> guard(g_cache_lock);
        if (!opted[w->device]) {
            const cudaError_t e = cudaFuncSetAttribute(mmdk::gemm_tcp<XDT, YDT>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(mmdk::kTcpSmemBytes));
            if (e != cudaSuccess) return e;
            opted[w->device] = true;
        }
    }
    const int mtiles = (M + 127) / 128, ntiles = (w->N + mmdk::kTcpBN - 1) / mmdk::kTcpBN;
    const long total = long(mtiles) * ntiles;
    const unsigned grid = unsigned(total < w->sm_count ? total : w->sm_count);
    mmdk::gemm_tcp<XDT, YDT><<<grid, mmdk::kTcThreads, mmdk::kTcpSmemBytes, stream>>>(
        mqx, w->map_q[0], sx, w->scale, sidex, w->side, w->side_cols, w->ko, y, M, w->N, (w->K + 127) / 128, mtiles, ntiles, w->status);
    return cudaGetLastError();
}

template <int XDT, int YDT, bool ADAPT>
cudaError_t launch_tc2(const mmd_weights* w, const CUtensorMap& mqx, const float* sx, const void* sidex, void* y, int M, const mmdk::AdaptArgs& ad, cudaStream_t stream) {
    static bool opted[kMaxDevices] = {};
    static int max_pairs[kMaxDevices] = {};
    if (w->device < 0 || w->device >= kMaxDevices) return cudaErrorInvalidDevice;
    const int d = w->device;
    std::unique_lock<std::mutex> guard(g_cache_lock);
    if (!opted[d]) {
        cudaError_t e = cudaFuncSetAttribute(mmdk::gemm_tc2<XDT, YDT, ADAPT>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(mmdk::PairCfg<ADAPT>::kSmem));
        if (e != cudaSuccess) return e;
        // how many CTA pairs the device runs at once: the persistent grid must not exceed it
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(unsigned(w->sm_count & ~1), 1, 1);
        cfg.blockDim = dim3(mmdk::PairCfg<ADAPT>::kThreads, 1, 1);
        cfg.dynamicSmemBytes = mmdk::PairCfg<ADAPT>::kSmem;
        int n = 0;
        e = cudaOccupancyMaxActiveClusters(&n, mmdk::gemm_tc2<XDT, YDT, ADAPT>, &cfg);
        if (e != cudaSuccess) return e;
        if (n < 1) return cudaErrorInvalidConfiguration;
        max_pairs[d] = n;
        opted[d] = true;
    }
    const int pairs_at_once = max_pairs[d];
    guard.unlock();
    const int mpairs = (M + 255) / 256, ntiles = (w->N + mmdk::kTcpBN - 1) / mmdk::kTcpBN;
    const long total = long(mpairs) * ntiles;
    const unsigned pairs = unsigned(total < pairs_at_once ? total : pairs_at_once);
    mmdk::gemm_tc2<XDT, YDT, ADAPT><<<2 * pairs, mmdk::PairCfg<ADAPT>::kThreads, mmdk::PairCfg<ADAPT>::kSmem, stream>>>(
        mqx, w->map_q_pair, sx, w->scale, sidex, w->side, w->side_cols, w->ko, y, M, w->N, (w->K + 127) / 128, mpairs, ntiles, w->status, ad);
    return cudaGetLastError();
}

// Large products with few critical features take the persistent kernels.
bool wants_persistent(const mmd_weights* w, int M) {
    // from about half a wave of 128 x 256 tiles on: below that the one-tile-per-CTA kernel's narrower tiles fill the SMs better.
    // One row of tiles (a decode step) is bound by the weight stream, not by the tensor cores: it stays with that kernel too.
    return w->ko <= mmdk::kTcpSide && w->N >= 256 && M > 128 && long((M + 127) / 128) * ((w->N + 255) / 256) >= w->sm_count / 2;
}

template <int XDT, int YDT>
cudaError_t launch_tc_bn(const mmd_weights* w, const CUtensorMap& mqx, const CUtensorMap& msx, const int8_t* qx, const float* sx, void* y, int M,
                         cudaStream_t stream) {
    // The widest tile has the highest arithmetic intensity; when it would leave SMs without a
    // tile (few rows, as in a decode step, where the weights are read once and the kernel is
    // bound by that stream) narrower tiles put more CTAs on the weight stream.
    const long mt = (M + 127) / 128;
    if (w->N >= 256 && mt * ((w->N + 255) / 256) >= w->sm_count) return launch_tc<XDT, YDT, 256>(w, mqx, msx, sx, y, M, 1, stream);
    if (w->N >= 128 && mt * ((w->N + 127) / 128) >= w->sm_count) {
        CUtensorMap mqx2;                                                        // K a multiple of 128: two K blocks per load
        if (w->have_pair_map && make_map_kblocks(&mqx2, qx, uint64_t(M), uint64_t(w->K), uint32_t(activation_box_rows(M)), 2)) {
            // One row of tiles that does not fill whole waves (a decode step through a wide layer): the whole waves run one
            // tile per CTA, and the tiles left over share their K steps among 2-4 CTAs each, so that the last wave also
            // keeps about one CTA per SM on the weight stream instead of running at full length on a few SMs.
            const long tiles = (w->N + 127) / 128;
            const long rest = tiles % w->sm_count;
            if (mt == 1 && rest > 0 && rest <= w->sm_count / 2) {
                int split = int(w->sm_count / rest);
                if (split > 4) split = 4;
                while (split > 1 && (w->K + 255) / 256 < 4 * split) --split;    // at least 4 steps per CTA
                if (split > 1) {
                    const cudaError_t e = launch_tc_decode<XDT, YDT>(w, mqx2, msx, sx, y, M, 1, stream, 0, int(tiles - rest));
                    if (e != cudaSuccess) return e;
                    return launch_tc_decode<XDT, YDT>(w, mqx2, msx, sx, y, M, split, stream, int(tiles - rest), int(rest));
                }
            }
            return launch_tc_decode<XDT, YDT>(w, mqx2, msx, sx, y, M, 1, stream);
        }
        return launch_tc<XDT, YDT, 128>(w, mqx, msx, sx, y, M, 1, stream);
    }
    // One row of tiles (a decode step) streams every weight once from DRAM, and an SM streams only as fast as the bytes it
    // keeps in flight.  128-row weight tiles hold the most per CTA; when they leave SMs idle, 2-4 CTAs share each tile's K
    // steps (clusters along z) so that about one CTA per SM is streaming.
    if (mt == 1 && w->N >= 1024) {
        const long tiles = (w->N + 127) / 128;
        int split = int(w->sm_count / tiles);
        if (split > 4) split = 4;
        if (split < 1) split = 1;
        if (w->have_pair_map) {                                                  // K a multiple of 128: two K blocks per load
            while (split > 1 && (w->K + 255) / 256 < 4 * split) --split;        // at least 4 steps per CTA
            CUtensorMap mqx2;
            if (make_map_kblocks(&mqx2, qx, uint64_t(M), uint64_t(w->K), uint32_t(activation_box_rows(M)), 2))
                return launch_tc_decode<XDT, YDT>(w, mqx2, msx, sx, y, M, split, stream);
        }
        while (split > 1 && (w->K + 127) / 128 < 8 * split) --split;            // at least 8 steps per CTA
        return launch_tc<XDT, YDT, 128>(w, mqx, msx, sx, y, M, split, stream);
    }
    return launch_tc<XDT, YDT, 64>(w, mqx, msx, sx, y, M, 1, stream);
}

template <int XDT, int YDT>
cudaError_t launch_general(const mmd_weights* w, const int8_t* qx, const float* sx, const void* sidex, void* y, int M, cudaStream_t stream) {
    const dim3 grid(unsigned((w->N + 63) / 64), unsigned((M + 63) / 64));
    mmdk::gemm_general<XDT, YDT><<<grid, 256, 0, stream>>>(qx, w->q, sx, w->scale, sidex, w->side, w->side_cols, y, M, w->N, w->K);
    return cudaGetLastError();
}

// A product over rows that the row stage has decomposed.
struct Product {
    const int8_t* qx;
    const float* sx;
    const void* sidex;
    void* y;
    int M;
    bool use_tc, persistent, pairs;                                          // which kernel; persistent and pairs: of use_tc
};

// cudaErrorNotSupported: no tensor map for these operands
template <int XDT, int YDT>
cudaError_t product_as(const mmd_weights* w, const Product& p, cudaStream_t stream) {
    if (!p.use_tc) return launch_general<XDT, YDT>(w, p.qx, p.sx, p.sidex, p.y, p.M, stream);
    CUtensorMap mqx, msx;
    if (p.pairs) {
        if (!make_map_kblocks(&mqx, p.qx, uint64_t(p.M), uint64_t(w->K), 128, mmdk::kPairStepBlocks)) return cudaErrorNotSupported;
        return launch_tc2<XDT, YDT, false>(w, mqx, p.sx, p.sidex, p.y, p.M, mmdk::AdaptArgs{}, stream);
    }
    const uint32_t rows = p.persistent ? 128u : uint32_t(activation_box_rows(p.M));
    if (!make_map(&mqx, p.qx, 1, uint64_t(p.M), uint64_t(w->K), rows)) return cudaErrorNotSupported;
    if (p.persistent) return launch_tcp<XDT, YDT>(w, mqx, p.sx, p.sidex, p.y, p.M, stream);
    if (w->side_cols == 0) msx = mqx;
    else if (!make_map(&msx, p.sidex, 2, uint64_t(p.M), uint64_t(w->side_cols), rows)) return cudaErrorNotSupported;
    return launch_tc_bn<XDT, YDT>(w, mqx, msx, p.qx, p.sx, p.y, p.M, stream);
}

}  // namespace
