// C entry points of the layer operators (see include/cutoff.h): arguments are checked, a kernel is chosen by sizes, types and alignment,
// work is enqueued.
#include "../../include/cutoff.h"

#include <atomic>
#include <cmath>
#include <type_traits>

#include "launch.cuh"
#include "dropout.cuh"
#include "residual_norm.cuh"
#include "int8_product.cuh"
#include "int8_tc.cuh"

using namespace cutoff;
using namespace cutoff::layers;

namespace {

constexpr int kMostCols = 8192;               // of a norm
constexpr int kMostDevices = 64;

// The result of a call whose CUDA calls all returned success, or not: the thread's last error, which whoever asks next would take for its own, ends here.
int done(bool ok) {
    if (ok) return CUTOFF_OK;
    cudaGetLastError();
    return CUTOFF_ERR_CUDA;
}

int sm_count(int device) {
    static std::atomic<int> sms[kMostDevices] = {};       // the same for every host thread
    if (device >= kMostDevices) return 148;
    int v = sms[device].load(std::memory_order_relaxed);
    if (v > 0) return v;
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || v < 1) return 148;
    sms[device].store(v, std::memory_order_relaxed);
    return v;
}

bool known_type(int32_t type) { return type == CUTOFF_TYPE_FP32 || type == CUTOFF_TYPE_FP16 || type == CUTOFF_TYPE_BF16; }
int type_size(int32_t type) { return type == CUTOFF_TYPE_FP32 ? 4 : 2; }

// f(a value of the element type)
template <typename F>
void with_type(int32_t type, F f) {
    if (type == CUTOFF_TYPE_FP32) f(float{});
    else if (type == CUTOFF_TYPE_FP16) f(__half{});
    else f(__nv_bfloat16{});
}

// Whether every row of a matrix starts on a multiple of `bytes` (a null matrix does).
bool rows_aligned(const void* p, int64_t ld, int size, int bytes) {
    return p == nullptr || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * size % bytes == 0);
}
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
// A matrix that is there with rows that overlap, rows too far apart for 64-bit offsets and tensor maps, or values off their own alignment.
constexpr int64_t kMostApart = int64_t{1} << 38;
bool off(const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % size != 0; }
bool bad_matrix(const void* p, int64_t ld, int64_t cols, int size) { return p != nullptr && (ld < cols || ld > kMostApart || off(p, size)); }
constexpr int kMostProductCols = 1 << 30;     // of dropout, quantised rows and a product's outputs: columns and a tile more fit 32 bits

// ---- dropout ---------------------------------------------------------------------------------------------------------
template <typename T, int V, int LX>
bool launch_dropout(const DropoutArgs& a, int sms, cudaStream_t s) {
    // Rows of a thread on their way: as many as the aligned forms of 32 lanes hold in their 80 registers without spilling.  The forms for odd 16-bit rows
    // spill with as many (of three rows with a residual 322 bytes per thread on 32 lanes, 196 on 8, 170 on 2; without one 28 and 12).
    constexpr int kAdd = sizeof(T) == 2 ? 3 : 2, kPlain = V == 1 ? kAdd : sizeof(T) == 2 ? 5 : 3, kWarps = kDropoutThreads / 32;
    const int unroll = a.residual ? kAdd : kPlain;
    const int64_t row_warps = ceil_div64(a.rows, unroll * (32 / LX));     // warps that find work in a tile of columns
    const int64_t resident = static_cast<int64_t>(sms) * 3 * kWarps;
    int64_t each = resident / a.tiles;
    each = each < 1 ? 1 : each < row_warps ? each : row_warps;
    const unsigned grid = static_cast<unsigned>(ceil_div64(each * a.tiles, kWarps));
    return launch_plain(a.residual ? k_dropout<T, V, LX, kAdd, true> : k_dropout<T, V, LX, kPlain, false>, dim3(grid), dim3(kDropoutThreads), 0, s, a) ==
           cudaSuccess;
}
template <typename T, int V>
bool launch_dropout(DropoutArgs& a, int sms, cudaStream_t s) {
    const int groups = ceil_div(a.cols, 8);
    const auto run = [&](auto lanes) {
        constexpr int LX = decltype(lanes)::value;
        a.tiles = ceil_div(groups, LX);
        return launch_dropout<T, V, LX>(a, sms, s);
    };
    return groups <= 2   ? run(std::integral_constant<int, 2>{})
           : groups <= 8 ? run(std::integral_constant<int, 8>{})
                         : run(std::integral_constant<int, 32>{});
}

// ---- norms -----------------------------------------------------------------------------------------------------------
bool bad_layer(const cutoff_norm_layer* l) {
    if (!l || !known_type(l->type)) return true;
    const int size = type_size(l->type);
    return l->rows < 0 || l->rows > kMostRows || l->cols < 1 || !l->x || bad_matrix(l->x, l->x_ld, l->cols, size) || bad_matrix(l->h, l->h_ld, l->cols, size) ||
           bad_matrix(l->gate, l->gate_ld, l->cols, size) || off(l->scale, 4) || off(l->post_weight, 4) || off(l->post_bias, 4) || off(l->pre_weight, 4) ||
           off(l->pre_bias, 4) || (l->gate && (l->gate_rows < 1 || !l->h)) || l->gate_kind < CUTOFF_GATE_LINEAR ||
           l->gate_kind > CUTOFF_GATE_SILU || l->post < CUTOFF_NORM_NONE || l->post > CUTOFF_NORM_LAYER || l->pre < CUTOFF_NORM_NONE ||
           l->pre > CUTOFF_NORM_LAYER || !(l->eps > 0.f) || !std::isfinite(l->eps) || (!l->h && (l->scale || l->post_weight || l->post_bias));
}

NormArgs norm_args(const cutoff_norm_layer* l) {
    NormArgs a{};
    a.x = l->x; a.h = l->h; a.gate = l->gate;
    a.scale = l->scale; a.post_w = l->post_weight; a.post_b = l->post_bias; a.pre_w = l->pre_weight; a.pre_b = l->pre_bias;
    a.rows = static_cast<int>(l->rows); a.x_ld = l->x_ld; a.h_ld = l->h_ld; a.gate_ld = l->gate_ld;
    a.gate_rows = !l->gate ? 1 : static_cast<int>(l->gate_rows < INT32_MAX ? l->gate_rows : INT32_MAX);
    a.cols = l->cols; a.gate_kind = l->gate_kind; a.post = l->post; a.pre = l->pre;
    a.eps = l->eps; a.inv_cols = 1.f / static_cast<float>(l->cols);
    return a;
}
bool whole_packs(const cutoff_norm_layer* l) {
    const int size = type_size(l->type);
    return l->cols * size % 16 == 0 && rows_aligned(l->x, l->x_ld, size, 16) && rows_aligned(l->h, l->h_ld, size, 16) &&
           rows_aligned(l->gate, l->gate_ld, size, 16) && aligned16(l->scale) && aligned16(l->post_weight) && aligned16(l->post_bias) &&
           aligned16(l->pre_weight) && aligned16(l->pre_bias);
}

// ---- products --------------------------------------------------------------------------------------------------------
// Tensor map over int8 rows: boxes of box_rows rows x 128 bytes, 128-byte swizzle.  The driver entry point is looked up once.
bool make_byte_map(CUtensorMap* map, const int8_t* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
    typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const EncodeFn encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
        return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeFn>(fn) : nullptr;
    }();
    if (!encode) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld)};
    const cuuint32_t box[2] = {kProdK, static_cast<cuuint32_t>(box_rows)};
    const cuuint32_t elem[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles of BN tokens x 128 outputs.
int64_t product_tiles(const ProductArgs& p, int tokens) { return ceil_div64(p.m, tokens) * ceil_div(p.n, kProdM); }

template <typename T, int BN>
bool launch_product_tile(const ProductArgs& p, int device, cudaStream_t s) {
    using Tile = ProductTile<BN>;
    CUtensorMap map_a, map_b;
    if (!make_byte_map(&map_a, p.a, p.m, p.k, p.a_ld, BN) || !make_byte_map(&map_b, p.b, p.n, p.k, p.b_ld, kProdM)) return false;
    if (cudaFuncSetAttribute(k_product_tile<T, BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(Tile::kSmemBytes)) != cudaSuccess) return false;
    const int64_t token_tiles = ceil_div64(p.m, BN), tiles = product_tiles(p, BN);
    // the K blocks of a tile are split until three CTAs for two SMs are there, but no CTA gets less than two blocks
    const int blocks = ceil_div(p.k, kProdK);
    int splits = 1;
    if (Tile::kSplits)
        while (splits < kMostSplits && tiles * splits * 2 < sm_count(device) * 3 && blocks >= 4 * splits) splits *= 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(tiles * splits));
    cfg.blockDim = dim3(Tile::kThreads);
    cfg.dynamicSmemBytes = Tile::kSmemBytes;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = splits;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_product_tile<T, BN>, map_b, map_a, p, static_cast<int>(token_tiles), splits) == cudaSuccess;
}

template <typename T>
bool launch_product_pair(const ProductArgs& p, int device, cudaStream_t s) {
    CUtensorMap map_a, map_b;
    if (!make_byte_map(&map_a, p.a, p.m, p.k, p.a_ld, kPairTokens / 2) || !make_byte_map(&map_b, p.b, p.n, p.k, p.b_ld, kProdM)) return false;
    if (cudaFuncSetAttribute(k_product_pair<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kPairSmem)) != cudaSuccess) return false;
    const int channel_tiles = ceil_div(p.n, 2 * kProdM), token_tiles = static_cast<int>(ceil_div64(p.m, kPairTokens)), pairs = sm_count(device) / 2;
    const int64_t tiles = static_cast<int64_t>(channel_tiles) * token_tiles;
    return launch_dependent(k_product_pair<T>, dim3(static_cast<unsigned>(2 * (tiles < pairs ? tiles : pairs))), dim3(kPairThreads), kPairSmem, s, map_b,
                            map_a, p, channel_tiles, token_tiles) == cudaSuccess;
}

template <typename T>
bool launch_product(const ProductArgs& p, int device, cudaStream_t s) {
    // One token: as its products are few, the vector unit's dot products follow the weights (4096 x 4096 6.1 us, tensor-core tiles 8.5; 8192 x 8192
    // 15.4 and 16.0); with two they do not any more (11.3, 8.5).
    if (p.m == 1) return launch_dependent(k_product_dot<T>, dim3(ceil_div(p.n, kDotWarps)), dim3(kDotWarps * 32), 0, s, p) == cudaSuccess;
    // The fewest tokens per tile that hold them all, or whose tiles, split in four, are resident at a time: the latency of the K blocks bounds a CTA, and
    // what a second tile reads again comes from the L2 (300 x 512 x 8192: 32 tokens 12 us, 64 13, 128 21).  Then whole tiles of 128 tokens, one per
    // SM (512 x 4096 x 4096 16.3 us, pairs of SMs 17.9), then pairs (1000 x 4096 x 4096 18.0 us, tiles of 128 tokens 28.6).
    const int64_t sms = sm_count(device), resident = 2 * sms / kMostSplits;
    if (p.m <= 16 || product_tiles(p, 16) <= resident) return launch_product_tile<T, 16>(p, device, s);
    if (p.m <= 32 || product_tiles(p, 32) <= resident) return launch_product_tile<T, 32>(p, device, s);
    if (p.m <= 64 || product_tiles(p, 64) <= resident) return launch_product_tile<T, 64>(p, device, s);
    if (product_tiles(p, 128) <= sms) return launch_product_tile<T, 128>(p, device, s);
    return launch_product_pair<T>(p, device, s);
}

}  // namespace

extern "C" {

int cutoff_dropout(int device, int32_t type, int64_t rows, int32_t cols, const void* x, int64_t x_ld, const void* residual, int64_t residual_ld,
                   void* y, int64_t y_ld, double p, uint64_t seed, uint32_t step, uint32_t noise_stream, int64_t first_row, void* stream) {
    if (device < 0 || !known_type(type) || rows < 0 || cols < 1 || !x || !y || bad_matrix(x, x_ld, cols, type_size(type)) ||
        bad_matrix(y, y_ld, cols, type_size(type)) || bad_matrix(residual, residual_ld, cols, type_size(type)) || !(p >= 0.0 && p <= 1.0) || first_row < 0 || rows > (int64_t{1} << 32) || first_row > (int64_t{1} << 32) - rows)
        return CUTOFF_ERR_BAD_ARG;
    if (cols > kMostProductCols) return CUTOFF_ERR_TOO_LARGE;
    if (rows == 0) return CUTOFF_OK;
    DeviceGuard guard(device);
    if (guard.err != cudaSuccess) return done(false);
    const uint32_t dropped = static_cast<uint32_t>(std::nearbyint(p * 65536.0));
    DropoutArgs a{};
    a.x = x; a.residual = residual; a.y = y;
    a.rows = rows; a.x_ld = x_ld; a.residual_ld = residual_ld; a.y_ld = y_ld; a.cols = cols;
    a.first_row = static_cast<uint32_t>(first_row); a.stream = noise_stream; a.step = step;
    a.key = NoiseKey{static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32)};
    a.border = dropped < 65536 ? dropped << 16 : 0xffffffffu;
    a.word_mask = dropped < 65536 ? 0xffffffffu : 0u;
    a.scale = dropped < 65536 ? static_cast<float>(65536.0 / (65536 - dropped)) : 0.f;
    const int size = type_size(type);
    const bool packs = cols * static_cast<int64_t>(size) % 16 == 0 && rows_aligned(x, x_ld, size, 16) && rows_aligned(residual, residual_ld, size, 16) &&
                       rows_aligned(y, y_ld, size, 16);
    bool ok = false;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        ok = packs ? launch_dropout<T, kPack<T>>(a, sm_count(device), static_cast<cudaStream_t>(stream))
                   : launch_dropout<T, 1>(a, sm_count(device), static_cast<cudaStream_t>(stream));
    });
    return done(ok);
}

int cutoff_residual_norm(int device, const cutoff_norm_layer* layer, void* residual, int64_t residual_ld, void* norm, int64_t norm_ld, float* norm_scale,
                         void* stream) {
    if (device < 0 || bad_layer(layer) || bad_matrix(residual, residual_ld, layer->cols, type_size(layer->type)) ||
        bad_matrix(norm, norm_ld, layer->cols, norm_scale ? 1 : type_size(layer->type)) || off(norm_scale, 4) || (!residual && !norm) || (!layer->h && residual) || (norm_scale && !norm))
        return CUTOFF_ERR_BAD_ARG;
    if (layer->cols > kMostCols) return CUTOFF_ERR_TOO_LARGE;
    if (layer->rows == 0) return CUTOFF_OK;
    DeviceGuard guard(device);
    if (guard.err != cudaSuccess) return done(false);
    NormArgs a = norm_args(layer);
    a.r = residual; a.n = norm; a.n_scale = norm_scale; a.r_ld = residual_ld; a.n_ld = norm_ld;
    const int size = type_size(layer->type);
    const bool packs = whole_packs(layer) && rows_aligned(residual, residual_ld, size, 16) &&
                       (norm_scale ? rows_aligned(norm, norm_ld, 1, 16 / size) : rows_aligned(norm, norm_ld, size, 16));
    bool ok = false;
    with_type(layer->type, [&](auto t) { ok = run_norm<decltype(t)>(a, packs, sm_count(device), static_cast<cudaStream_t>(stream)); });
    return done(ok);
}

int64_t cutoff_residual_norm_grad_workspace_bytes(int64_t rows, int32_t cols) {
    if (rows < 0 || rows > kMostRows || cols < 1 || cols > kMostCols) return CUTOFF_ERR_BAD_ARG;
    // the largest of what the ways to lay out the teams take
    int64_t most = 0;
    for (const int way : {0, 1, 2}) {
        const GradPlan plan = grad_plan(static_cast<int>(rows), cols, way == 2 ? 4 : 2, way == 1, kMostSms);
        const int64_t floats = 6 * static_cast<int64_t>(plan.ctas) * cols;
        most = floats > most ? floats : most;
    }
    return most * static_cast<int64_t>(sizeof(float)) + 256;
}

int cutoff_residual_norm_grad(int device, const cutoff_norm_layer* layer, const void* d_residual, int64_t d_residual_ld, const void* d_norm,
                              int64_t d_norm_ld, const cutoff_norm_grads* grads, void* workspace, size_t workspace_bytes, void* stream) {
    if (device < 0 || bad_layer(layer) || !grads) return CUTOFF_ERR_BAD_ARG;
    const int size = type_size(layer->type);
    if (bad_matrix(d_residual, d_residual_ld, layer->cols, size) || bad_matrix(d_norm, d_norm_ld, layer->cols, size) || (!d_residual && !d_norm) ||
        bad_matrix(grads->x, grads->x_ld, layer->cols, size) || bad_matrix(grads->h, grads->h_ld, layer->cols, size) ||
        bad_matrix(grads->gate, grads->gate_ld, layer->cols, size) || off(grads->scale, 4) || off(grads->post_weight, 4) || off(grads->post_bias, 4) ||
        off(grads->pre_weight, 4) || off(grads->pre_bias, 4) || (!layer->h && (grads->h || grads->gate)) || (grads->gate && !layer->gate) || !workspace ||
        (grads->scale && !layer->scale) || (grads->post_weight && !layer->post_weight) || (grads->post_bias && !layer->post_bias) ||
        (grads->pre_weight && !layer->pre_weight) || (grads->pre_bias && !layer->pre_bias))
        return CUTOFF_ERR_BAD_ARG;
    if (layer->cols > kMostCols) return CUTOFF_ERR_TOO_LARGE;
    if (static_cast<int64_t>(workspace_bytes) < cutoff_residual_norm_grad_workspace_bytes(layer->rows, layer->cols) || !aligned16(workspace))
        return CUTOFF_ERR_BAD_ARG;
    DeviceGuard guard(device);
    if (guard.err != cudaSuccess) return done(false);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int sms = sm_count(device);
    const bool bias = layer->post_bias || layer->pre_bias, groups = layer->gate && layer->gate_rows > 1;
    const GradPlan plan = grad_plan(static_cast<int>(layer->rows), layer->cols, type_size(layer->type), bias || groups, sms);
    NormFinishArgs q{};
    NormGradArgs& g = q.g;
    g.f = norm_args(layer);
    g.d_r = d_residual; g.d_n = d_norm; g.d_r_ld = d_residual_ld; g.d_n_ld = d_norm_ld;
    g.d_x = grads->x; g.d_h = grads->h; g.d_gate = grads->gate; g.d_x_ld = grads->x_ld; g.d_h_ld = grads->h_ld; g.d_gate_ld = grads->gate_ld;
    g.sums = static_cast<float*>(workspace);
    g.gate_sums = g.sums + 4 * static_cast<int64_t>(plan.ctas) * layer->cols;
    g.teams = plan.teams;
    q.ctas = plan.ctas; q.each = bias ? 4 : 2;
    q.d_scale = grads->scale; q.d_post_w = grads->post_weight; q.d_post_b = grads->post_bias; q.d_pre_w = grads->pre_weight; q.d_pre_b = grads->pre_bias;
    const bool packs = whole_packs(layer) && rows_aligned(d_residual, d_residual_ld, size, 16) && rows_aligned(d_norm, d_norm_ld, size, 16) &&
                       rows_aligned(grads->x, grads->x_ld, size, 16) && rows_aligned(grads->h, grads->h_ld, size, 16) &&
                       rows_aligned(grads->gate, grads->gate_ld, size, 16);
    const bool sums = grads->scale || grads->post_weight || grads->post_bias || grads->pre_weight || grads->pre_bias;
    q.column_blocks = sums ? ceil_div(layer->cols, kFinishColumns) : 0;
    int64_t gate_blocks = 0;
    if (groups && grads->gate && layer->rows > 0) {
        // a slice for every eight CTAs that a group may span
        const int64_t cta_rows = static_cast<int64_t>(g.f.rows / plan.teams) * plan.per_cta, spans = g.f.gate_rows / (cta_rows > 0 ? cta_rows : 1) + 2;
        q.teams_here = plan.per_cta;
        q.groups = ceil_div64(g.f.rows, g.f.gate_rows);
        q.slices = 1;
        while (q.slices < kGateSlices && 8 * q.slices < spans && 8 * q.slices < plan.ctas) q.slices *= 2;
        gate_blocks = static_cast<int64_t>(q.groups < plan.ctas ? q.groups : plan.ctas) * ceil_div(g.f.cols, kGateColumns * (kFinishThreads / q.slices));
    }
    bool ok = false;
    with_type(layer->type, [&](auto t) { ok = run_norm_grad<decltype(t)>(q, plan, packs, bias, groups, q.column_blocks + gate_blocks, s); });
    return done(ok);
}

int cutoff_quantize_rows(int device, int32_t type, int64_t rows, int32_t cols, const void* x, int64_t x_ld, int8_t* q, int64_t q_ld, float* scale,
                         void* stream) {
    if (device < 0 || !known_type(type) || rows < 0 || rows > INT32_MAX || cols < 1 || !x || !q || !scale || bad_matrix(x, x_ld, cols, type_size(type)) ||
        bad_matrix(q, q_ld, cols, 1) || off(scale, 4))
        return CUTOFF_ERR_BAD_ARG;
    if (cols > kMostProductCols) return CUTOFF_ERR_TOO_LARGE;
    if (rows == 0) return CUTOFF_OK;
    DeviceGuard guard(device);
    if (guard.err != cudaSuccess) return done(false);
    const QuantizeArgs a{x, q, scale, rows, x_ld, q_ld, cols};
    const int size = type_size(type);
    bool ok = false;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool packs = cols % kPack<T> == 0 && rows_aligned(x, x_ld, size, 16) && rows_aligned(q, q_ld, 1, kPack<T>);
        const auto run = [&](auto v) {
            constexpr int V = decltype(v)::value;
            const cudaStream_t s = static_cast<cudaStream_t>(stream);
            // rows that a warp holds in registers; otherwise a CTA whose threads hold four packs each, or with few rows (their latency is all there is) one
            if (cols <= 32 * V * kQuantizeKeep && rows > sm_count(device))
                return launch_dependent(k_quantize_rows<T, V, 32>, dim3(static_cast<unsigned>(ceil_div64(rows, kQuantizeWarps))), dim3(kQuantizeWarps * 32), 0, s, a) ==
                       cudaSuccess;
            int threads = ceil_div(ceil_div(cols, rows > 2 * sm_count(device) ? V * kQuantizeKeep : V), 32) * 32;
            threads = threads > 512 ? 512 : threads;
            return launch_dependent(k_quantize_rows<T, V, 0>, dim3(static_cast<unsigned>(rows)), dim3(threads), 0, s, a) == cudaSuccess;
        };
        ok = packs ? run(std::integral_constant<int, kPack<T>>{}) : run(std::integral_constant<int, 1>{});
    });
    return done(ok);
}

int cutoff_quantized_product(int device, int64_t m, int32_t n, int32_t k, const int8_t* a, int64_t a_ld, const float* a_scale, const int8_t* b,
                             int64_t b_ld, const float* b_scale, const float* bias, int32_t type, void* y, int64_t y_ld, void* stream) {
    // a single row has no distance to a next one; tensor maps want one all the same
    if (m == 1 && a_ld >= k && a_ld <= kMostApart) a_ld = (a_ld + 15) / 16 * 16;
    if (n == 1 && b_ld >= k && b_ld <= kMostApart) b_ld = (b_ld + 15) / 16 * 16;
    if (device < 0 || m < 0 || m > kMostRows || n < 1 || k < 1 || !a || !a_scale || !b || !b_scale || !known_type(type) || !y || bad_matrix(a, a_ld, k, 1) ||
        bad_matrix(b, b_ld, k, 1) || bad_matrix(y, y_ld, n, type_size(type)) || off(a_scale, 4) || off(b_scale, 4) || off(bias, 4) || !rows_aligned(a, a_ld, 1, 16) || !rows_aligned(b, b_ld, 1, 16))
        return CUTOFF_ERR_BAD_ARG;
    if (k > CUTOFF_PRODUCT_MAX_K || n > kMostProductCols) return CUTOFF_ERR_TOO_LARGE;
    if (m == 0) return CUTOFF_OK;
    DeviceGuard guard(device);
    if (guard.err != cudaSuccess) return done(false);
    const ProductArgs p{a, b, a_scale, b_scale, bias, y, m, a_ld, b_ld, y_ld, n, k};
    bool ok = false;
    with_type(type, [&](auto t) { ok = launch_product<decltype(t)>(p, device, static_cast<cudaStream_t>(stream)); });
    return done(ok);
}

}  // extern "C"
