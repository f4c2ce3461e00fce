// mmd_api.cu -- the C ABI of the mixed matrix decomposition (see include/mmd.h): argument
// checks, the weight handle, the row stage and the choice of kernel.
#include "mmd_adapters.h"
#include "mmd_launch.cuh"
#include "mmd_selftest.cuh"

namespace {

constexpr int kMaxK = 262144;
constexpr int kMaxFeatures = 1024;

template <int DT>
cudaError_t launch_rowquant(const void* v, int R, int K, const int32_t* idx, int ko, int8_t* q, float* scale, void* side, int sm_count,
                            cudaStream_t stream, int* zero_words = nullptr, int n_zero_words = 0) {
    const size_t smem = round_up(size_t(K) / 8, 4);
    if (smem > 48 * 1024) return cudaErrorInvalidValue;          // K <= kMaxK keeps the mask within the default limit
    int grid = R;
    const int cap = sm_count * 16;
    if (grid > cap) grid = cap;
    // launched with programmatic stream serialization: the kernel waits (griddepcontrol.wait) for the kernels before it
    // before it touches global memory; behind a kernel that never signals its dependents this is an ordinary launch
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(grid), 1, 1);
    cfg.blockDim = dim3(256, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int side_cols = mmd_side_columns(ko);
    return cudaLaunchKernelEx(&cfg, mmdk::rowquant<DT>, v, R, K, idx, ko, side_cols, q, scale, side, zero_words, n_zero_words);
}

cudaError_t rowquant_any(int dt, const void* v, int R, int K, const int32_t* idx, int ko, int8_t* q, float* scale, void* side, int sm_count,
                         cudaStream_t stream, int* zero_words = nullptr, int n_zero_words = 0) {
    return dt == BQ_BF16 ? launch_rowquant<mmdk::kBF16>(v, R, K, idx, ko, q, scale, side, sm_count, stream, zero_words, n_zero_words)
                         : launch_rowquant<mmdk::kF16>(v, R, K, idx, ko, q, scale, side, sm_count, stream, zero_words, n_zero_words);
}

template <int DT, int THREADS>
cudaError_t launch_norm_t(const void* x, const void* res, const void* gamma, int R, int K, float eps, const int32_t* idx, int ko, void* h, int8_t* q,
                          float* scale, void* side, float* rms, int sm_count, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    const int cap = sm_count * 8;
    cfg.gridDim = dim3(unsigned(R < cap ? R : cap), 1, 1);
    cfg.blockDim = dim3(THREADS, 1, 1);
    cfg.dynamicSmemBytes = round_up(size_t(K) / 8, 4);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // as launch_rowquant
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, mmdk::norm_rowquant<DT, THREADS>, x, res, gamma, R, K, eps, idx, ko, mmd_side_columns(ko), static_cast<uint16_t*>(h), q,
                              scale, side, rms);
}

// A decode step's few rows cannot fill the device: four times the threads per row shorten the pass.
template <int DT>
cudaError_t launch_norm(const void* x, const void* res, const void* gamma, int R, int K, float eps, const int32_t* idx, int ko, void* h, int8_t* q,
                        float* scale, void* side, float* rms, int sm_count, cudaStream_t stream) {
    return R <= sm_count && K >= 4096 ? launch_norm_t<DT, 1024>(x, res, gamma, R, K, eps, idx, ko, h, q, scale, side, rms, sm_count, stream)
                                      : launch_norm_t<DT, 256>(x, res, gamma, R, K, eps, idx, ko, h, q, scale, side, rms, sm_count, stream);
}

cudaError_t norm_any(int dt, const void* x, const void* res, const void* gamma, int R, int K, float eps, const int32_t* idx, int ko, void* h, int8_t* q,
                     float* scale, void* side, float* rms /* of every row, or null */, int sm_count, cudaStream_t stream) {
    return dt == BQ_BF16 ? launch_norm<mmdk::kBF16>(x, res, gamma, R, K, eps, idx, ko, h, q, scale, side, rms, sm_count, stream)
                         : launch_norm<mmdk::kF16>(x, res, gamma, R, K, eps, idx, ko, h, q, scale, side, rms, sm_count, stream);
}

// The arguments the two norm calls share.
int check_norm(const void* x, const void* res, const void* gamma, const void* h_out, float eps, int R, int K) {
    if (!x || !gamma || (res && !h_out)) return BQ_ERR_NULL;
    if (!aligned(x, 16) || !aligned(res, 16) || !aligned(gamma, 16) || !aligned(h_out, 16)) return BQ_ERR_SIZE;
    // a row is written while later ones are still to be read: h_out is an input itself, or shares no memory with it
    const uint64_t bytes = uint64_t(R) * uint64_t(K) * 2;
    for (const void* in : {x, res}) {
        const uint64_t a = reinterpret_cast<uintptr_t>(in), b = reinterpret_cast<uintptr_t>(h_out);
        if (in && h_out && in != h_out && a < b + bytes && b < a + bytes) return BQ_ERR_SIZE;
    }
    return (eps >= 0.0f && eps < 3.0e38f) ? BQ_OK : BQ_ERR_SIZE;
}

int check_features(const int32_t* idx_host, int ko, int K) {
    if (ko < 0 || ko > kMaxFeatures || ko >= K) return MMD_ERR_FEATURES;
    if (ko > 0 && !idx_host) return BQ_ERR_NULL;
    for (int j = 0; j < ko; ++j) {
        if (idx_host[j] < 0 || idx_host[j] >= K) return MMD_ERR_FEATURES;
        if (j > 0 && idx_host[j] <= idx_host[j - 1]) return MMD_ERR_FEATURES;
    }
    return BQ_OK;
}

}  // namespace

namespace {

struct WsLayout { size_t q, scale, side, total; };

WsLayout ws_layout(const mmd_weights* w, int M) {
    WsLayout L;
    L.q = 0;
    L.scale = round_up(size_t(M) * w->K, kWsAlign);
    L.side = L.scale + round_up(size_t(M) * 4, kWsAlign);
    L.total = L.side + round_up(size_t(M) * w->side_cols * 2, kWsAlign);
    return L;
}

bool on_device(const mmd_weights* w) {
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == w->device;
}

// One row of tiles (a decode step of at most 64 rows) with the K steps of all tiles dealt out over one CTA per SM: the
// shape must have fewer 128-column tiles than SMs (so that a CTA's share touches at most two tiles) and the caller's
// workspace must have room, behind the decomposed activations, for the tiles' counters and partial sums.
struct SkPlan {
    bool ok;
    int n_tiles, grid, maxparts;
    size_t counters, acc, side, total;                     // offsets behind the base workspace, and the extra bytes
};

SkPlan sk_plan(const mmd_weights* w, int M) {
    SkPlan p = {};
    if (!w->have_maps || !w->have_pair_map || M < 1 || M > 64 || w->N < 1024 || w->N % 8 != 0) return p;
    p.n_tiles = (w->N + 127) / 128;
    if (p.n_tiles >= w->sm_count) return p;
    const long long ksteps = ((w->K + 127) / 128 + 1) / 2, upt = ksteps + (w->side_cols > 0 ? 1 : 0);
    const long long total = (long long)p.n_tiles * upt;
    if (ksteps < 8) return p;                              // too few steps per tile to be worth sharing
    const long long G = total < w->sm_count ? total : w->sm_count;
    p.grid = int(G);
    for (int t = 0; t < p.n_tiles; ++t) {
        const long long ta = (long long)t * upt, tb = ta + upt;
        const int c_first = int(((ta + 1) * G + total - 1) / total) - 1, c_last = int((tb * G + total - 1) / total) - 1;
        if (c_last - c_first + 1 > p.maxparts) p.maxparts = c_last - c_first + 1;
    }
    const size_t tile_values = size_t(64) * 128;
    p.counters = 0;
    p.acc = round_up(size_t(p.n_tiles) * 4, kWsAlign);
    p.side = p.acc + round_up(size_t(p.n_tiles) * p.maxparts * tile_values * 4, kWsAlign);
    p.total = p.side + (w->side_cols > 0 ? round_up(size_t(p.n_tiles) * tile_values * 4, kWsAlign) : 0);
    p.ok = true;
    return p;
}

template <int XDT, int YDT>
cudaError_t launch_sk(const mmd_weights* w, const SkPlan& p, const int8_t* qx, const void* sidex, const float* sx, void* y, int M, char* extra,
                      cudaStream_t stream) {
    using Cfg = mmdk::TcCfg<mmdk::kSkBN, mmdk::kSkBM, mmdk::kSkKPB>;
    static bool opted[kMaxDevices] = {};
    if (w->device < 0 || w->device >= kMaxDevices) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> guard(g_cache_lock);
        if (!opted[w->device]) {
            const cudaError_t e = cudaFuncSetAttribute(mmdk::gemm_sk<XDT, YDT>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(Cfg::kSmemBytes));
            if (e != cudaSuccess) return e;
            opted[w->device] = true;
        }
    }
    CUtensorMap mqx, mqw, msx;
    if (!make_map_kblocks(&mqx, qx, uint64_t(M), uint64_t(w->K), 64, mmdk::kSkKPB)) return cudaErrorInvalidValue;
    if (!make_map_kblocks(&mqw, w->q, uint64_t(w->N), uint64_t(w->K), mmdk::kSkBN, mmdk::kSkKPB)) return cudaErrorInvalidValue;
    if (w->side_cols > 0) {
        if (!make_map(&msx, sidex, 2, uint64_t(M), uint64_t(w->side_cols), 64)) return cudaErrorInvalidValue;
    } else {
        msx = mqx;
    }
    const int slot = bn_slot(mmdk::kSkBN);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(p.grid), 1, 1);
    cfg.blockDim = dim3(mmdk::kTcThreads, 1, 1);
    cfg.dynamicSmemBytes = Cfg::kSmemBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // starts under the row kernel; waits for it before reading its results
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, mmdk::gemm_sk<XDT, YDT>, mqx, mqw, msx, w->side_cols > 0 ? w->map_side[slot] : w->map_q[slot], sx,
                              static_cast<const float*>(w->scale), y, M, w->N, (w->K + 127) / 128, w->side_cols / 64, p.n_tiles, p.maxparts,
                              reinterpret_cast<int*>(extra + p.counters), reinterpret_cast<int*>(extra + p.acc),
                              reinterpret_cast<float*>(extra + p.side), w->status);
}

// What fills the workspace with the decomposed rows: the plain row kernel over X, or (gamma not null) the norm.
struct RowStage { const void *X, *residual, *gamma; void* h_out; float eps; };

// Whether the CTA-pair kernel adds the adapters in its epilogue: where it takes the product, for ranks whose pieces of B fit beside its stages.
// The layer's fp32 rows then need not go to memory and back.  Measured, 4914 rows, 6144 -> 16384, bf16, whole call behind the norm in a
// graph, cold, here | with the adapters added by a kernel behind the product: rank 16 459 | 594 us, fp32 outputs 523 | 671; rank 32 747 | 709, in a row
// 679 | 690.
bool fuses(const mmd_weights* w, int M, int rank, bool tc_ok, int path) {
    return tc_ok && (path == MMD_PATH_AUTO || path == MMD_PATH_TENSOR) && wants_persistent(w, M) && w->have_pair_map && rank <= mmdk::kFusedRank;
}

// Where the adapters' numbers lie behind the decomposed activations: the rows' rms (with a norm), the rows' adapters, the first product's
// partial sums and, where the adapters' part is added by a kernel of its own, the layer's rows in fp32 (fp32 outputs: in Y itself).
struct AdaptedLayout { size_t rms, row_id, u, y32, total; mmda::ShrinkPlan plan; };

AdaptedLayout adapted_layout(const mmd_weights* w, int M, int n_seq, int rank, bool y32) {
    AdaptedLayout L;
    L.plan = mmda::shrink_plan(M, n_seq, w->K, rank);
    L.rms = ws_layout(w, M).total;
    L.row_id = L.rms + round_up(size_t(M) * 4, kWsAlign);
    L.u = L.row_id + round_up(size_t(M) * 4, kWsAlign);
    L.y32 = L.u + round_up(size_t(L.plan.chunks) * M * rank * 4, kWsAlign);
    L.total = L.y32 + (y32 ? round_up(size_t(M) * round_up(size_t(w->N), 8) * 4, kWsAlign) : 0);
    return L;
}

int linear(const mmd_weights* w, const RowStage& rows, int M, void* Y, bq_dtype ydt, void* workspace, size_t workspace_bytes, int path, void* cuda_stream,
           const mmda::Adapters* ad = nullptr) {
    const void* X = rows.X;
    if (!w) return BQ_ERR_NULL;
    if (ydt != BQ_F32 && int(ydt) != w->dtype) return BQ_ERR_DTYPE;
    if (M < 0) return BQ_ERR_SIZE;
    if (path < MMD_PATH_AUTO || path > MMD_PATH_TENSOR_STREAMK) return MMD_ERR_PATH;
    if (M == 0) return BQ_OK;
    if (!X || !Y) return BQ_ERR_NULL;
    if (!aligned(X, 16) || !aligned(Y, ydt == BQ_F32 ? 4 : 2)) return BQ_ERR_SIZE;
    const WsLayout L = ws_layout(w, M);
    const bool tc_ok = w->have_maps && (w->N % 8 == 0) && aligned(Y, 16);
    const bool fused = ad && fuses(w, M, ad->rank, tc_ok, path);
    const AdaptedLayout AL = ad ? adapted_layout(w, M, ad->n_seq, ad->rank, !fused && (ydt != BQ_F32 || w->N % 8 != 0 || !aligned(Y, 16))) : AdaptedLayout{};
    if (!workspace || !aligned(workspace, kWsAlign) || workspace_bytes < (ad ? AL.total : L.total)) return MMD_ERR_WORKSPACE;
    if (!on_device(w)) return BQ_ERR_CUDA;
    if (path >= MMD_PATH_TENSOR && !tc_ok) return MMD_ERR_PATH;
    if (path == MMD_PATH_TENSOR_SOLO && !wants_persistent(w, M)) return MMD_ERR_PATH;
    const bool use_tc = (path >= MMD_PATH_TENSOR) || (path == MMD_PATH_AUTO && tc_ok);
    const bool persistent = use_tc && path != MMD_PATH_TENSOR_TILE && wants_persistent(w, M);
    const bool pairs = persistent && path != MMD_PATH_TENSOR_SOLO && w->have_pair_map;      // the pair kernel's loads need K % 128 == 0
    // a decode step over a layer with fewer tiles than SMs, on request: all tiles' K steps over one CTA per SM.  Not taken by
    // AUTO: as measured, handing partial sums over through global memory costs more than the even shares save.
    const SkPlan sk = (use_tc && !persistent && path == MMD_PATH_TENSOR_STREAMK) ? sk_plan(w, M) : SkPlan{};
    const bool stream_k = sk.ok && workspace_bytes >= L.total + sk.total;
    if (path == MMD_PATH_TENSOR_STREAMK && !stream_k) return sk.ok ? MMD_ERR_WORKSPACE : MMD_ERR_PATH;

    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(workspace);
    int8_t* qx = reinterpret_cast<int8_t*>(ws + L.q);
    float* sx = reinterpret_cast<float*>(ws + L.scale);
    void* sidex = ws + L.side;
    cudaError_t e = rows.gamma
        ? norm_any(w->dtype, X, rows.residual, rows.gamma, M, w->K, rows.eps, w->idx, w->ko, rows.h_out, qx, sx, sidex,
                   ad ? reinterpret_cast<float*>(ws + AL.rms) : nullptr, w->sm_count, stream)
        : rowquant_any(w->dtype, X, M, w->K, w->idx, w->ko, qx, sx, sidex, w->sm_count, stream,
                       stream_k ? reinterpret_cast<int*>(ws + L.total + sk.counters) : nullptr, stream_k ? sk.n_tiles : 0);
    if (e != cudaSuccess) return cuda_fail(e);

    const bool bf = (w->dtype == BQ_BF16), f32out = (ydt == BQ_F32);
    if (stream_k) {
        char* extra = ws + L.total;
        if (bf) e = f32out ? launch_sk<mmdk::kBF16, mmdk::kF32>(w, sk, qx, sidex, sx, Y, M, extra, stream) : launch_sk<mmdk::kBF16, mmdk::kBF16>(w, sk, qx, sidex, sx, Y, M, extra, stream);
        else e = f32out ? launch_sk<mmdk::kF16, mmdk::kF32>(w, sk, qx, sidex, sx, Y, M, extra, stream) : launch_sk<mmdk::kF16, mmdk::kF16>(w, sk, qx, sidex, sx, Y, M, extra, stream);
    } else {
        float* const u = ad ? reinterpret_cast<float*>(ws + AL.u) : nullptr;
        int32_t* const row_id = ad ? reinterpret_cast<int32_t*>(ws + AL.row_id) : nullptr;
        if (ad) {
            const mmda::Input in = {static_cast<const uint16_t*>(rows.gamma && rows.h_out ? rows.h_out : X), static_cast<const uint16_t*>(rows.gamma),
                                    reinterpret_cast<const float*>(ws + AL.rms), M, w->K, w->N};
            e = mmda::launch_shrink(bf, in, *ad, AL.plan, u, row_id, stream);
            if (e != cudaSuccess) return cuda_fail(e);
        }
        if (fused) {
            const mmdk::AdaptArgs args = {ad->b, ad->scale, u, row_id, ad->rank, AL.plan.chunks, size_t(M) * ad->rank};
            e = mmda::launch_fused(w, qx, sx, sidex, Y, M, f32out, args, stream);
        } else {
            // The layer's fp32 rows of a call with adapters lie in the workspace a multiple of eight apart, so that the tensor-core kernels
            // take any N: they see a matrix with up to seven rows more (zeros by the tensor maps; what they read of the scales and side
            // columns behind the last row is the handle's own memory, and the columns are not used).
            const bool far = ad && AL.y32 < AL.total;
            mmd_weights wide;
            const mmd_weights* pw = w;
            Product p = {qx, sx, sidex, far ? ws + AL.y32 : Y, M, use_tc, persistent, pairs};
            if (far && (path == MMD_PATH_AUTO ? w->have_maps : use_tc)) {
                wide = *w;
                wide.N = (w->N + 7) / 8 * 8;
                pw = &wide;
                p.use_tc = true;
                p.persistent = path != MMD_PATH_TENSOR_TILE && wants_persistent(pw, M);
                p.pairs = p.persistent && path != MMD_PATH_TENSOR_SOLO && w->have_pair_map;
            }
            if (bf) e = f32out || ad ? product_as<mmdk::kBF16, mmdk::kF32>(pw, p, stream) : product_as<mmdk::kBF16, mmdk::kBF16>(pw, p, stream);
            else e = f32out || ad ? product_as<mmdk::kF16, mmdk::kF32>(pw, p, stream) : product_as<mmdk::kF16, mmdk::kF16>(pw, p, stream);
            if (e == cudaSuccess && ad)
                e = mmda::launch_expand(bf, M, w->N, *ad, AL.plan, u, row_id, static_cast<const float*>(p.y), pw->N, Y, f32out, stream);
        }
    }
    if (e == cudaErrorNotSupported) return MMD_ERR_PATH;                     // no tensor map for these operands
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

// The adapters of a call, as the kernels see them, after their checks.
int check_adapters(const mmd_weights* w, const mmd_adapters* ad, const int32_t* ids, const int32_t* starts, int n_seq, int M, mmda::Adapters* out) {
    if (!w || !ad) return BQ_ERR_NULL;
    if (ad->count < 1 || ad->rank < 16 || ad->rank > MMD_MAX_RANK || ad->rank % 16 != 0) return BQ_ERR_SIZE;
    if (n_seq < 1 || M < 0 || (!starts && n_seq != M && M > 0)) return BQ_ERR_SIZE;
    if (M == 0) return BQ_OK;
    if (!ad->a || !ad->b || !ad->scale || !ids) return BQ_ERR_NULL;
    if (!aligned(ad->a, 16) || !aligned(ad->b, 16) || !aligned(ad->scale, 4) || !aligned(ids, 4) || !aligned(starts, 4)) return BQ_ERR_SIZE;
    *out = {static_cast<const uint16_t*>(ad->a), static_cast<const uint16_t*>(ad->b), ad->scale, ad->count, ad->rank, ids, starts, n_seq};
    return BQ_OK;
}

}  // namespace

extern "C" {

int mmd_side_columns(int n_features) {
    return n_features <= 0 ? 0 : (n_features + mmdk::kSidePad - 1) / mmdk::kSidePad * mmdk::kSidePad;
}

int mmd_select_features(const float* feature_absmax, int K, float tau, int32_t* idx_out, int* count_out) {
    if (!feature_absmax || !idx_out || !count_out) return BQ_ERR_NULL;
    if (K < 1) return BQ_ERR_SIZE;
    int c = 0;
    for (int k = 0; k < K; ++k)
        if (feature_absmax[k] >= tau) idx_out[c++] = k;
    *count_out = c;
    return BQ_OK;
}

int mmd_rowquant(const void* v, bq_dtype dt, int R, int K, const int32_t* idx, int n_features, int8_t* q_out, float* scale_out,
                 void* side_out, void* cuda_stream) {
    if (!is16(dt)) return BQ_ERR_DTYPE;
    if (R < 0 || K < 16 || K % 16 != 0 || K > kMaxK) return BQ_ERR_SIZE;
    if (n_features < 0 || n_features > kMaxFeatures || n_features >= K) return MMD_ERR_FEATURES;
    if (R == 0) return BQ_OK;
    if (!v || !q_out || !scale_out || (n_features > 0 && (!idx || !side_out))) return BQ_ERR_NULL;
    if (!aligned(v, 16) || !aligned(q_out, 16)) return BQ_ERR_SIZE;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return cuda_fail(e);
    e = rowquant_any(dt, v, R, K, idx, n_features, q_out, scale_out, side_out, sms, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

int mmd_decompose(const void* W, bq_dtype dt, int N, int K, const int32_t* idx_host, int n_features, void* cuda_stream, mmd_weights** out) {
    if (!out) return BQ_ERR_NULL;
    *out = nullptr;
    if (!is16(dt)) return BQ_ERR_DTYPE;
    if (N < 1 || K < 16 || K % 16 != 0 || K > kMaxK) return BQ_ERR_SIZE;
    const int fc = check_features(idx_host, n_features, K);
    if (fc != BQ_OK) return fc;
    if (!W) return BQ_ERR_NULL;
    if (!aligned(W, 16)) return BQ_ERR_SIZE;
    mmd_weights* w = new (std::nothrow) mmd_weights();
    if (!w) return BQ_ERR_CUDA;
    w->N = w->rows = N; w->K = K; w->ko = n_features; w->side_cols = mmd_side_columns(n_features); w->dtype = dt;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = cudaGetDevice(&w->device);
    if (e == cudaSuccess && (w->device < 0 || w->device >= kMaxDevices)) e = cudaErrorInvalidDevice;     // beyond the per-device tables
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&w->sm_count, cudaDevAttrMultiProcessorCount, w->device);
    const size_t o_q = 0;
    const size_t o_scale = round_up(size_t(N) * K, kWsAlign);
    const size_t o_side = o_scale + round_up(size_t(N) * 4, kWsAlign);
    const size_t o_idx = o_side + round_up(size_t(N) * w->side_cols * 2, kWsAlign);
    const size_t o_status = o_idx + round_up(size_t(kMaxFeatures) * 4, kWsAlign);
    const size_t total = o_status + kWsAlign;
    if (e == cudaSuccess) e = cudaMalloc(&w->blob, total);
    if (e != cudaSuccess) { delete w; return cuda_fail(e); }
    char* base = static_cast<char*>(w->blob);
    w->q = reinterpret_cast<int8_t*>(base + o_q);
    w->scale = reinterpret_cast<float*>(base + o_scale);
    w->side = base + o_side;
    w->idx = reinterpret_cast<int32_t*>(base + o_idx);
    w->status = reinterpret_cast<int*>(base + o_status);
    // the feature list is copied from pageable host memory: the copy has left the host buffer when the call returns
    if (e == cudaSuccess && n_features > 0) e = cudaMemcpyAsync(w->idx, idx_host, size_t(n_features) * 4, cudaMemcpyHostToDevice, stream);
    if (e == cudaSuccess) e = rowquant_any(dt, W, N, K, w->idx, n_features, w->q, w->scale, w->side, w->sm_count, stream);
    // Behind the kernel: nothing later starts before this, and so before the kernel's end.  A product may start as soon as the row kernel in front
    // of it has started, which may itself start under this one, and asks for weights at once.
    if (e == cudaSuccess) e = cudaMemsetAsync(w->status, 0, sizeof(int), stream);
    if (e != cudaSuccess) { cudaFree(w->blob); delete w; return cuda_fail(e); }
    w->have_maps = true;
    w->have_pair_map = make_map_kblocks(&w->map_q_pair, w->q, uint64_t(N), uint64_t(K), 128, mmdk::kPairStepBlocks);
    const uint32_t boxes[3] = {256, 128, 64};
    for (int s = 0; s < 3; ++s) {
        w->have_maps = w->have_maps && make_map(&w->map_q[s], w->q, 1, uint64_t(N), uint64_t(K), boxes[s]);
        if (w->side_cols > 0) w->have_maps = w->have_maps && make_map(&w->map_side[s], w->side, 2, uint64_t(N), uint64_t(w->side_cols), boxes[s]);
    }
    *out = w;
    return BQ_OK;
}

int mmd_free(mmd_weights* w) {
    if (!w) return BQ_OK;
    const cudaError_t e = cudaFree(w->blob);
    delete w;
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

int mmd_weights_view(const mmd_weights* w, const int8_t** q, const float** scale, const void** side, const int32_t** idx, int* N, int* K,
                     int* n_features, int* dtype) {
    if (!w) return BQ_ERR_NULL;
    if (q) *q = w->q;
    if (scale) *scale = w->scale;
    if (side) *side = w->side;
    if (idx) *idx = w->idx;
    if (N) *N = w->N;
    if (K) *K = w->K;
    if (n_features) *n_features = w->ko;
    if (dtype) *dtype = w->dtype;
    return BQ_OK;
}

int mmd_workspace_layout(const mmd_weights* w, int M, size_t* offsets3, size_t* total_bytes) {
    if (!w || !total_bytes) return BQ_ERR_NULL;
    if (M < 0) return BQ_ERR_SIZE;
    const WsLayout L = ws_layout(w, M);
    if (offsets3) { offsets3[0] = L.q; offsets3[1] = L.scale; offsets3[2] = L.side; }
    *total_bytes = L.total;
    return BQ_OK;
}

int mmd_workspace_bytes_streamk(const mmd_weights* w, int M, size_t* total_bytes) {
    if (!w || !total_bytes) return BQ_ERR_NULL;
    if (M < 0) return BQ_ERR_SIZE;
    const SkPlan p = sk_plan(w, M);
    *total_bytes = ws_layout(w, M).total + (p.ok ? p.total : 0);
    return BQ_OK;
}

int mmd_linear(const mmd_weights* w, const void* X, int M, void* Y, bq_dtype ydt, void* workspace, size_t workspace_bytes, int path,
               void* cuda_stream) {
    const RowStage rows = {X, nullptr, nullptr, nullptr, 0.0f};
    return linear(w, rows, M, Y, ydt, workspace, workspace_bytes, path, cuda_stream);
}

int mmd_norm_linear(const mmd_weights* w, const void* X, const void* residual, const void* gamma, float eps, int M, void* h_out, void* Y, bq_dtype ydt,
                    void* workspace, size_t workspace_bytes, int path, void* cuda_stream) {
    if (!w) return BQ_ERR_NULL;
    if (path == MMD_PATH_TENSOR_STREAMK) return MMD_ERR_PATH;              // its counters are zeroed by the plain row kernel
    if (M > 0) {
        const int rc = check_norm(X, residual, gamma, h_out, eps, M, w->K);
        if (rc != BQ_OK) return rc;
    }
    const RowStage rows = {X, residual, gamma, h_out, eps};
    return linear(w, rows, M, Y, ydt, workspace, workspace_bytes, path, cuda_stream);
}

int mmd_adapted_workspace(const mmd_weights* w, int M, int n_seq, int rank, int path, size_t* bytes) {
    if (!w || !bytes) return BQ_ERR_NULL;
    if (path < MMD_PATH_AUTO || path > MMD_PATH_TENSOR_SOLO) return MMD_ERR_PATH;
    if (M < 0 || n_seq < 1 || rank < 16 || rank > MMD_MAX_RANK || rank % 16 != 0) return BQ_ERR_SIZE;
    *bytes = adapted_layout(w, M, n_seq, rank, !fuses(w, M, rank, w->have_maps && w->N % 8 == 0, path)).total;
    return BQ_OK;
}

int mmd_linear_adapted(const mmd_weights* w, const mmd_adapters* adapters, const int32_t* ids, const int32_t* starts, int n_seq, const void* X, int M, void* Y,
                       bq_dtype ydt, void* workspace, size_t workspace_bytes, int path, void* cuda_stream) {
    mmda::Adapters ad = {};
    const int rc = check_adapters(w, adapters, ids, starts, n_seq, M, &ad);
    if (rc != BQ_OK) return rc;
    if (path == MMD_PATH_TENSOR_STREAMK) return MMD_ERR_PATH;
    const RowStage rows = {X, nullptr, nullptr, nullptr, 0.0f};
    return linear(w, rows, M, Y, ydt, workspace, workspace_bytes, path, cuda_stream, &ad);
}

int mmd_norm_linear_adapted(const mmd_weights* w, const mmd_adapters* adapters, const int32_t* ids, const int32_t* starts, int n_seq, const void* X,
                            const void* residual, const void* gamma, float eps, int M, void* h_out, void* Y, bq_dtype ydt, void* workspace,
                            size_t workspace_bytes, int path, void* cuda_stream) {
    mmda::Adapters ad = {};
    int rc = check_adapters(w, adapters, ids, starts, n_seq, M, &ad);
    if (rc != BQ_OK) return rc;
    if (path == MMD_PATH_TENSOR_STREAMK) return MMD_ERR_PATH;
    if (M > 0) {
        rc = check_norm(X, residual, gamma, h_out, eps, M, w->K);
        if (rc != BQ_OK) return rc;
    }
    const RowStage rows = {X, residual, gamma, h_out, eps};
    return linear(w, rows, M, Y, ydt, workspace, workspace_bytes, path, cuda_stream, &ad);
}

int mmd_norm_rowquant(const void* x, const void* residual, const void* gamma, float eps, bq_dtype dt, int R, int K, const int32_t* idx, int n_features,
                      void* h_out, int8_t* q_out, float* scale_out, void* side_out, void* cuda_stream) {
    if (!is16(dt)) return BQ_ERR_DTYPE;
    if (R < 0 || K < 16 || K % 16 != 0 || K > kMaxK) return BQ_ERR_SIZE;
    if (n_features < 0 || n_features > kMaxFeatures || n_features >= K) return MMD_ERR_FEATURES;
    if (R == 0) return BQ_OK;
    if (!q_out || !scale_out || (n_features > 0 && (!idx || !side_out))) return BQ_ERR_NULL;
    const int rc = check_norm(x, residual, gamma, h_out, eps, R, K);
    if (rc != BQ_OK) return rc;
    if (!aligned(q_out, 16)) return BQ_ERR_SIZE;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = norm_any(dt, x, residual, gamma, R, K, eps, idx, n_features, h_out, q_out, scale_out, side_out, nullptr, sms, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

int mmd_selftest_bounded_wait(const mmd_weights* w, unsigned limit_us, int* threads_left_out, void* cuda_stream) {
    if (!w || !threads_left_out) return BQ_ERR_NULL;
    if (limit_us < 1 || limit_us > 100000) return BQ_ERR_SIZE;              // 1 us .. 0.1 s: this wait is meant to run out
    if (!on_device(w)) return BQ_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int khz = 0;
    cudaError_t e = cudaDeviceGetAttribute(&khz, cudaDevAttrClockRate, w->device);
    if (e != cudaSuccess) return cuda_fail(e);
    const long long cycles = (long long)limit_us * (khz > 0 ? khz : 1000000) / 1000;
    // the counter lives in the handle's spare status space (the word after the status)
    int* left = w->status + 1;
    e = cudaMemsetAsync(left, 0, sizeof(int), stream);
    if (e != cudaSuccess) return cuda_fail(e);
    mmdk::wait_selftest<<<1, mmdk::kTcThreads, 0, stream>>>(w->status, MMD_SELFTEST_CODE, cycles, left);
    e = cudaGetLastError();
    if (e == cudaSuccess) e = cudaMemcpyAsync(threads_left_out, left, sizeof(int), cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

int mmd_kernel_status(const mmd_weights* w, int* status_out) {
    if (!w || !status_out) return BQ_ERR_NULL;
    if (!on_device(w)) return BQ_ERR_CUDA;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(status_out, w->status, sizeof(int), cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && *status_out != 0) e = cudaMemset(w->status, 0, sizeof(int));
    return e == cudaSuccess ? BQ_OK : cuda_fail(e);
}

}  // extern "C"
