// C ABI of the layer calls: argument checks, workspaces, plans, launches. Contracts in include/cfgzip.h.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "cfgzip.h"
#include "cfgzip_layer.cuh"
#include "context.h"
#include "products.h"

using namespace cfgzip;

namespace {

constexpr int kLayerMost = 65536;   // longest row
constexpr int kLayerRows = 1 << 24;

int check_layer_shape(const cfgzip_layer* l) {
    if (!l || l->in <= 0 || l->out <= 0 || l->in % 8 || l->out % 8) return CFGZIP_E_ARG;
    if (l->activation < CFGZIP_ACT_NONE || l->activation > CFGZIP_ACT_SILU) return CFGZIP_E_ARG;
    if (l->bias && l->bias_dtype != CFGZIP_F32 && l->bias_dtype != CFGZIP_BF16) return CFGZIP_E_ARG;
    return l->in > kLayerMost || l->out > kLayerMost ? CFGZIP_E_RANGE : CFGZIP_OK;
}
int check_layer(const cfgzip_layer* l) {
    const int rc = check_layer_shape(l);
    if (rc != CFGZIP_OK) return rc;
    if (!l->weight || l->row_stride < l->in) return CFGZIP_E_ARG;
    return on16(l->weight, l->row_stride * 2) && on16(l->bias, 0) ? CFGZIP_OK : CFGZIP_E_ALIGN;
}
// rows of `n` bf16 numbers
int check_matrix(const void* p, int64_t stride, int n) {
    if (!p || stride < n) return CFGZIP_E_ARG;
    return on16(p, stride * 2) ? CFGZIP_OK : CFGZIP_E_ALIGN;
}

constexpr int kGradientRuns = 64;  // runs of rows that the bias's gradient is summed over, at most
int gradient_run(int32_t rows) { return std::max(64, up(ceil_div(rows, kGradientRuns), 32)); }

// Cuts of the sum over rows in the weights' gradient, where its result has too few tiles to fill the pairs. Each cut is a result in 32 bits
// written and read again, and a launch: not where the last of several rounds could be fuller (8192 rows of 4096 x 4096, whose 256 tiles take 3.5
// rounds: 225 us in two cuts, 205 in one).
int weight_cuts(const cfgzip_layer* l, int32_t rows) {
    const int64_t tiles = int64_t(ceil_div(l->out, kMmaTile)) * ceil_div(l->in, kMmaTile);
    return tiles > kPairs ? 1 : cuts(tiles, ceil_div(rows, kMmaK), int64_t(l->in) * l->out);
}

struct LayerSpace {
    uint16_t* g;
    float *sums, *parts;
    int64_t bytes;
};
// What is taken for `rows` rows is enough for fewer, whose cuts are others.
LayerSpace layer_space(const cfgzip_layer* l, int op, int32_t rows, void* workspace) {
    LayerSpace s{};
    if (op == CFGZIP_LAYER_FORWARD || rows == 0) return s;
    const uintptr_t skip = (256 - reinterpret_cast<uintptr_t>(workspace) % 256) % 256;
    Carve c(workspace ? static_cast<char*>(workspace) + skip : nullptr);
    s.g = c.take<uint16_t>(l->activation == CFGZIP_ACT_NONE ? 0 : int64_t(rows) * l->out);
    s.sums = c.take<float>(int64_t(std::min(kGradientRuns, ceil_div(rows, 64))) * l->out);
    const int64_t tiles = int64_t(ceil_div(l->out, kMmaTile)) * ceil_div(l->in, kMmaTile);
    const int most = tiles > kPairs ? 1 : std::min<int64_t>({kPairs, kCutTiles / tiles, ceil_div(rows, kMmaK) / 16});
    if (most > 1) s.parts = c.take<float>(int64_t(most) * l->in * l->out);
    s.bytes = c.used + 256;
    return s;
}

// A product of the layer's kind, result [rows, features] = A [rows, k] times weights, in whichever way is right for its size.
struct LayerProduct {
    int32_t rows, features, k;
    const void* a;
    int64_t a_stride;
    const void* weight;
    int64_t weight_stride;
    bool turned;  // the weights are [k, features], not [features, k]
    int32_t act;
    const void* bias;
    bool bias_bf16;
    const void* residual;
    int64_t residual_stride;
    void* y;
    int64_t y_stride;
    void* slope;
    int64_t slope_stride;
};

// Tiles of 128 features by `n` rows (at most 256), each over a cluster of `blocks` blocks with `stages` stages each.
struct FewPlan {
    int n, tiles, groups, blocks, stages;
    uint32_t stage_bytes;
    double us;
};
// The rows of a tile and the blocks of a cluster that take the least time: rounds of clusters (not all SMs can be had four or eight at a time)
// times a block's stages and what it takes besides. A stage is bound by its operands' way from the L2, 100 to 130 bytes a ns and SM, which two blocks
// of few stages share where there are more than the SMs. High tiles read the weights fewer times; of low ones there are more, and a block has
// fewer activations to compute at its end (256 rows of 256 x 256: 6.1 us by 128 rows, 4.2 by 32; 128 of 1032 x 2568 8.5 and, by 64, 7.5; 500 of
// 4096 x 4096 37.7 by 64, 21.5 by 128, 18.9 by 256). Over 80 shapes of 1 to 2000 rows the choice of all is 0.5 % slower than the fastest.
FewPlan few_plan(const cfgzip_ctx* ctx, const LayerProduct& p) {
    FewPlan best{};
    best.us = std::numeric_limits<double>::infinity();
    const int tiles = ceil_div(p.features, 128), k_blocks = ceil_div(p.k, kMmaK), all = std::min(256, up(p.rows, 16));
    for (const int n : {all, 192, 128, 96, 64, 48, 32}) {
        const int groups = ceil_div(p.rows, n);
        if (n > all || groups > 65535) continue;
        const uint32_t stage_bytes = kLayerWeights + uint32_t(n) * 128;
        const int most = std::min(kLayerStages, int((200u << 10) / stage_bytes));
        const int least = ceil_div(int64_t(n) * kLayerRow * 4, stage_bytes);  // what the sums take on their way out
        const double clusters = double(tiles) * groups;
        for (int s = 1; s <= kLayerBlocks && (s == 1 || 2 * s <= k_blocks); ++s) {
            const int steps = ceil_div(k_blocks, s), stages = std::max(std::min(most, steps), least);
            const int twice = 2 * (size_t(stages) * stage_bytes + 2560) <= size_t(ctx->smem_optin) ? 2 : 1;
            // (of clusters with a block to an SM; those of 3 and 5 leave SMs over wherever they are placed)
            const int limit = s == 1 ? ctx->sm_count : ctx->cluster_limit[s] - (s == 3 || s == 5 ? 3 : 0);
            if (limit <= 0) continue;
            const double rounds = std::ceil(clusters / (double(limit) * twice)), beside = std::min(double(twice), std::ceil(clusters / limit));
            const double us = 1.0 + rounds * (steps * beside * (0.17 + 0.0008 * n) + (s > 1 ? 3.0 : 2.2) + 0.02 * s + 0.016 * n);
            if (us < best.us) best = FewPlan{n, tiles, groups, s, stages, stage_bytes, us};
        }
    }
    return best;
}

template <bool A_MN, int ACT>
int run_few_as(cfgzip_ctx* ctx, const LayerProduct& p, const FewPlan& f, cudaStream_t st) {
    CUtensorMap map_w, map_x;
    int rc = A_MN ? tensor_map(ctx, &map_w, p.weight, p.k, p.features, p.weight_stride, 64)
                  : tensor_map(ctx, &map_w, p.weight, p.features, p.k, p.weight_stride, 128);
    if (rc != CFGZIP_OK || (rc = tensor_map(ctx, &map_x, p.a, p.rows, p.k, p.a_stride, f.n)) != CFGZIP_OK) return rc;
    LayerArgs a{};
    a.rows = p.rows;
    a.features = p.features;
    a.N = f.n;
    a.k_blocks = ceil_div(p.k, kMmaK);
    a.stage_bytes = f.stage_bytes;
    a.stages = f.stages;
    a.bias = p.bias;
    a.bias_bf16 = p.bias_bf16;
    a.residual = static_cast<const uint16_t*>(p.residual);
    a.residual_stride = p.residual_stride;
    a.y = static_cast<uint16_t*>(p.y);
    a.y_stride = p.y_stride;
    a.slope = static_cast<uint16_t*>(p.slope);
    a.slope_stride = p.slope_stride;
    a.status = ctx->d_status;
    a.expire = ctx->expire_test;
    const size_t smem = size_t(a.stages) * a.stage_bytes + 1024;
    if ((rc = ensure_smem(ctx, k_layer_few<A_MN, ACT>, smem)) != CFGZIP_OK) return rc;
    ctx->cluster_now = f.blocks;
    rc = launch(ctx, k_layer_few<A_MN, ACT>, dim3(unsigned(f.tiles * f.blocks), unsigned(f.groups)), dim3(kLayerThreads), smem, st, a, map_w, map_x);
    ctx->cluster_now = 1;
    return rc;
}

int run_few(cfgzip_ctx* ctx, const LayerProduct& p, const FewPlan& f, cudaStream_t st) {
    if (p.turned) return run_few_as<true, kActNone>(ctx, p, f, st);
    switch (p.act) {
        case CFGZIP_ACT_RELU: return run_few_as<false, kActRelu>(ctx, p, f, st);
        case CFGZIP_ACT_GELU: return run_few_as<false, kActGelu>(ctx, p, f, st);
        case CFGZIP_ACT_GELU_TANH: return run_few_as<false, kActGeluTanh>(ctx, p, f, st);
        case CFGZIP_ACT_SILU: return run_few_as<false, kActSilu>(ctx, p, f, st);
        default: return run_few_as<false, kActNone>(ctx, p, f, st);
    }
}

template <bool B_MN, int ACT>
int run_tall_as(cfgzip_ctx* ctx, MmaArgs& a, const CUtensorMap& map_a, const CUtensorMap& map_b, const CUtensorMap& map_y,
                const CUtensorMap& map_slope, cudaStream_t st) {
    auto kern = k_layer_mma<B_MN, ACT>;
    const size_t smem = size_t(kLayerStagesTall) * 2 * kMmaHalf + 1024 + 8 * 2 * kMmaOut;
    const int rc = ensure_smem(ctx, kern, smem);
    if (rc != CFGZIP_OK) return rc;
    const int64_t tiles = int64_t(a.m_tiles) * a.n_tiles;
    if (tiles >= (int64_t(1) << 30)) return CFGZIP_E_RANGE;
    const unsigned pairs = unsigned(std::min<int64_t>(tiles, ctx->sm_count / 2));
    return launch(ctx, kern, dim3(2 * pairs), dim3(kMmaThreads), smem, st, a, map_a, map_b, map_y, map_slope);
}

int run_tall(cfgzip_ctx* ctx, const LayerProduct& p, cudaStream_t st) {
    MmaArgs a{};
    a.rows = p.rows;
    a.cols = p.features;
    a.width = kMmaTile;
    a.m_tiles = ceil_div(p.rows, kMmaTile);
    a.box = a_box(p.rows);
    a.n_tiles = ceil_div(p.features, kMmaTile);
    a.k_blocks = ceil_div(p.k, kMmaK);
    a.splits = 1;
    a.status = ctx->d_status;
    a.expire = ctx->expire_test;
    a.out = p.y;
    a.ld = p.y_stride;
    a.bias = p.bias;
    a.bias_bf16 = p.bias_bf16;
    a.residual = static_cast<const uint16_t*>(p.residual);
    a.residual_stride = p.residual_stride;
    a.has_slope = p.slope != nullptr;
    CUtensorMap map_a, map_b, map_y, map_slope;
    int rc;
    if ((rc = tensor_map_a(ctx, &map_a, p.a, p.rows, p.k, p.a_stride)) != CFGZIP_OK ||
        (rc = p.turned ? tensor_map(ctx, &map_b, p.weight, p.k, p.features, p.weight_stride, 64)
                       : tensor_map(ctx, &map_b, p.weight, p.features, p.k, p.weight_stride, 128)) != CFGZIP_OK ||
        (rc = tensor_map_out(ctx, &map_y, a, true)) != CFGZIP_OK)
        return rc;
    map_slope = map_y;
    if (p.slope) {
        MmaArgs s = a;
        s.out = p.slope;
        s.ld = p.slope_stride;
        if ((rc = tensor_map_out(ctx, &map_slope, s, true)) != CFGZIP_OK) return rc;
    }
    if (p.turned) return run_tall_as<true, kActNone>(ctx, a, map_a, map_b, map_y, map_slope, st);
    switch (p.act) {
        case CFGZIP_ACT_RELU: return run_tall_as<false, kActRelu>(ctx, a, map_a, map_b, map_y, map_slope, st);
        case CFGZIP_ACT_GELU: return run_tall_as<false, kActGelu>(ctx, a, map_a, map_b, map_y, map_slope, st);
        case CFGZIP_ACT_GELU_TANH: return run_tall_as<false, kActGeluTanh>(ctx, a, map_a, map_b, map_y, map_slope, st);
        case CFGZIP_ACT_SILU: return run_tall_as<false, kActSilu>(ctx, a, map_a, map_b, map_y, map_slope, st);
        default: return run_tall_as<false, kActNone>(ctx, a, map_a, map_b, map_y, map_slope, st);
    }
}

int run_product(cfgzip_ctx* ctx, const LayerProduct& p, cudaStream_t st) {
    const FewPlan f = few_plan(ctx, p);
    // A stage of 64 k of a pair's 256 x 256 takes some 0.3 us, and 8.5 us are not covered by other tiles.
    const int tall_rounds = ceil_div(int64_t(ceil_div(p.rows, kMmaTile)) * ceil_div(p.features, kMmaTile), ctx->sm_count / 2);
    const double tall = tall_rounds * (ceil_div(p.k, kMmaK) * 0.3) + 8.5;
    if (p.rows > 128 && tall < f.us) return run_tall(ctx, p, st);
    return run_few(ctx, p, f, st);
}

}  // namespace

extern "C" {

int cfgzip_layer_workspace(const cfgzip_layer* layer, int op, int32_t rows, int64_t* bytes) {
    if (!bytes || rows < 0 || (op != CFGZIP_LAYER_FORWARD && op != CFGZIP_LAYER_BACKWARD)) return CFGZIP_E_ARG;
    const int rc = check_layer_shape(layer);
    if (rc != CFGZIP_OK) return rc;
    if (rows > kLayerRows) return CFGZIP_E_RANGE;
    *bytes = layer_space(layer, op, rows, nullptr).bytes;
    return CFGZIP_OK;
}

int cfgzip_layer_forward(cfgzip_ctx* ctx, const cfgzip_layer* layer, const void* x, int64_t x_stride, int32_t rows, const void* residual,
                         int64_t residual_stride, void* y, int64_t y_stride, void* slope, int64_t slope_stride, void* workspace,
                         int64_t workspace_bytes, void* stream) {
    int rc = check_layer(layer);
    if (rc != CFGZIP_OK) return rc;
    if (rows < 0) return CFGZIP_E_ARG;
    if (rows > kLayerRows) return CFGZIP_E_RANGE;
    if (rows == 0) return ctx ? CFGZIP_OK : CFGZIP_E_ARG;
    if ((rc = check_matrix(x, x_stride, layer->in)) != CFGZIP_OK || (rc = check_matrix(y, y_stride, layer->out)) != CFGZIP_OK ||
        (residual && (rc = check_matrix(residual, residual_stride, layer->out)) != CFGZIP_OK) ||
        (slope && (rc = check_matrix(slope, slope_stride, layer->out)) != CFGZIP_OK))
        return rc;
    const LayerSpace w = layer_space(layer, CFGZIP_LAYER_FORWARD, rows, workspace);
    if (w.bytes && !workspace) return CFGZIP_E_ARG;
    if (workspace_bytes < w.bytes) return CFGZIP_E_NOMEM;
    // (rows of x are read while others are written; the residual is read where y is written, by the same thread)
    if (y == x || (slope && (slope == x || slope == y || slope == residual))) return CFGZIP_E_ARG;
    if (!ctx) return CFGZIP_E_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    LayerProduct p{};
    p.rows = rows;
    p.features = layer->out;
    p.k = layer->in;
    p.a = x;
    p.a_stride = x_stride;
    p.weight = layer->weight;
    p.weight_stride = layer->row_stride;
    p.act = layer->activation;
    p.bias = layer->bias;
    p.bias_bf16 = layer->bias_dtype == CFGZIP_BF16;
    p.residual = residual;
    p.residual_stride = residual_stride;
    p.y = y;
    p.y_stride = y_stride;
    p.slope = layer->activation != CFGZIP_ACT_NONE ? slope : nullptr;
    p.slope_stride = slope_stride;
    return run_product(ctx, p, static_cast<cudaStream_t>(stream));
}

int cfgzip_layer_backward(cfgzip_ctx* ctx, const cfgzip_layer* layer, const void* x, int64_t x_stride, int32_t rows, const void* slope,
                          int64_t slope_stride, const void* d_y, int64_t d_y_stride, const void* add, int64_t add_stride, void* d_x,
                          int64_t d_x_stride, void* d_weight, int d_weight_dtype, int64_t d_weight_stride, float* d_bias, int accumulate,
                          void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_layer(layer);
    if (rc != CFGZIP_OK) return rc;
    if (rows < 0 || (!d_x && !d_weight && !d_bias)) return CFGZIP_E_ARG;
    if (rows > kLayerRows) return CFGZIP_E_RANGE;
    const bool half = d_weight_dtype == CFGZIP_BF16;
    const size_t size = half ? 2 : 4;
    if (d_weight) {
        if ((!half && d_weight_dtype != CFGZIP_F32) || d_weight_stride < layer->in) return CFGZIP_E_ARG;
        if (!on16(d_weight, d_weight_stride * int64_t(size))) return CFGZIP_E_ALIGN;
    }
    if (d_bias && (reinterpret_cast<uintptr_t>(d_bias) & 3u)) return CFGZIP_E_ALIGN;
    const bool acts = layer->activation != CFGZIP_ACT_NONE;
    if (rows > 0) {
        if ((rc = check_matrix(d_y, d_y_stride, layer->out)) != CFGZIP_OK || (acts && (rc = check_matrix(slope, slope_stride, layer->out)) != CFGZIP_OK) ||
            (d_weight && (rc = check_matrix(x, x_stride, layer->in)) != CFGZIP_OK) || (d_x && (rc = check_matrix(d_x, d_x_stride, layer->in)) != CFGZIP_OK) ||
            (d_x && add && (rc = check_matrix(add, add_stride, layer->in)) != CFGZIP_OK))
            return rc;
        if (!workspace) return CFGZIP_E_ARG;
    }
    const LayerSpace w = layer_space(layer, CFGZIP_LAYER_BACKWARD, rows, workspace);
    if (rows > 0 && workspace_bytes < w.bytes) return CFGZIP_E_NOMEM;
    if (rows > 0 && d_x && (d_x == d_y || d_x == x || (acts && d_x == slope))) return CFGZIP_E_ARG;
    if (!ctx) return CFGZIP_E_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int K = layer->in, O = layer->out;
    if (rows == 0) {  // empty sums
        if (accumulate) return CFGZIP_OK;
        if ((d_weight && cudaMemset2DAsync(d_weight, size_t(d_weight_stride) * size, 0, size_t(K) * size, size_t(O), st) != cudaSuccess) ||
            (d_bias && cudaMemsetAsync(d_bias, 0, size_t(O) * sizeof(float), st) != cudaSuccess)) {
            cudaGetLastError();
            return CFGZIP_E_CUDA;
        }
        return CFGZIP_OK;
    }
    const void* g = d_y;
    int64_t g_stride = d_y_stride;
    if (acts || d_bias) {
        LayerGradientArgs a{};
        a.rows = rows;
        a.features = O;
        a.run = gradient_run(rows);
        a.d_y = static_cast<const uint16_t*>(d_y);
        a.d_y_stride = d_y_stride;
        a.slope = acts ? static_cast<const uint16_t*>(slope) : nullptr;
        a.slope_stride = slope_stride;
        a.g = w.g;
        a.runs = ceil_div(rows, a.run);
        const bool one = a.runs <= kGradientCluster;
        a.sums = d_bias && !one ? w.sums : nullptr;
        a.d_bias = one ? d_bias : nullptr;
        a.accumulate = accumulate;
        ctx->cluster_now = a.d_bias ? a.runs : 1;
        rc = launch(ctx, k_layer_gradient, dim3(unsigned(ceil_div(O, 256) * a.runs)), dim3(256), 0, st, a);
        ctx->cluster_now = 1;
        if (rc != CFGZIP_OK) return rc;
        if (a.sums && (rc = launch(ctx, k_layer_bias, dim3(unsigned(ceil_div(O, 32))), dim3(256), 0, st, (const float*)w.sums, a.runs, O, d_bias,
                                   accumulate)) != CFGZIP_OK)
            return rc;
        if (acts) {
            g = w.g;
            g_stride = O;
        }
    }
    if (d_x) {
        LayerProduct p{};
        p.rows = rows;
        p.features = K;
        p.k = O;
        p.a = g;
        p.a_stride = g_stride;
        p.weight = layer->weight;
        p.weight_stride = layer->row_stride;
        p.turned = true;
        p.act = CFGZIP_ACT_NONE;
        p.residual = add;
        p.residual_stride = add_stride;
        p.y = d_x;
        p.y_stride = d_x_stride;
        if ((rc = run_product(ctx, p, st)) != CFGZIP_OK) return rc;
    }
    if (!d_weight) return CFGZIP_OK;
    CUtensorMap g_mn, x_mn;
    if ((rc = tensor_map(ctx, &g_mn, g, rows, O, g_stride, 64)) != CFGZIP_OK || (rc = tensor_map(ctx, &x_mn, x, rows, K, x_stride, 64)) != CFGZIP_OK)
        return rc;
    MmaArgs b{};
    b.rows = O;
    b.cols = K;
    b.k_blocks = ceil_div(rows, kMmaK);
    b.splits = weight_cuts(layer, rows);
    b.out = b.splits > 1 ? w.parts : d_weight;
    b.ld = b.splits > 1 ? K : d_weight_stride;
    b.split_elems = int64_t(O) * K;
    b.add = b.splits > 1 ? 0 : accumulate;
    rc = half && b.splits == 1 ? run_mma<true, true, kMmaBf16>(ctx, b, g_mn, x_mn, st) : run_mma<true, true, kMmaSum>(ctx, b, g_mn, x_mn, st);
    if (rc != CFGZIP_OK || b.splits == 1) return rc;
    LayerRoundArgs r{};
    r.from = w.parts;
    r.split_elems = b.split_elems;
    r.splits = b.splits;
    r.rows = O;
    r.n = K;
    r.to = d_weight;
    r.to_stride = d_weight_stride;
    r.bf16 = half;
    r.accumulate = accumulate;
    const int64_t blocks = std::min<int64_t>(ceil_div(int64_t(O) * (K / 4), 256), int64_t(ctx->sm_count) * 8);
    return launch(ctx, k_layer_round, dim3(unsigned(blocks)), dim3(256), 0, st, r);
}

}  // extern "C"
