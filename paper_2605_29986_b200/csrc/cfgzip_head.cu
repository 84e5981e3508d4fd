// C ABI of the head calls: argument checks, workspaces, launches. Contracts in include/cfgzip.h.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cfgzip.h"
#include "cfgzip_head_finish.cuh"
#include "cfgzip_head_mma.cuh"
#include "cfgzip_head_step.cuh"
#include "cfgzip_mx.cuh"
#include "context.h"
#include "products.h"

using namespace cfgzip;

namespace {

constexpr int kHeadMost = 65536;      // longest row of a head
constexpr int kHeadTokens = 1 << 30;  // most rows of a head, and of a batch

int check_head_shape(const cfgzip_head* h) {
    if (!h || h->V <= 0 || h->H <= 0 || (h->dtype != CFGZIP_BF16 && h->dtype != CFGZIP_MXFP4) || h->reserved) return CFGZIP_E_ARG;
    if (h->H % (h->dtype == CFGZIP_BF16 ? 8 : kMxBlock)) return CFGZIP_E_ARG;
    return h->H > kHeadMost || h->V > kHeadTokens ? CFGZIP_E_RANGE : CFGZIP_OK;
}

int check_head(const cfgzip_head* h) {
    const int rc = check_head_shape(h);
    if (rc != CFGZIP_OK) return rc;
    if (!h->weight) return CFGZIP_E_ARG;
    if (h->dtype == CFGZIP_BF16) {
        if (h->row_stride < h->H) return CFGZIP_E_ARG;
        return on16(h->weight, h->row_stride * 2) ? CFGZIP_OK : CFGZIP_E_ALIGN;
    }
    if (!h->scales || h->row_stride < h->H / 2 || h->scale_stride < h->H / kMxBlock) return CFGZIP_E_ARG;
    return on16(h->weight, h->row_stride) && on16(h->scales, h->scale_stride) ? CFGZIP_OK : CFGZIP_E_ALIGN;
}

// rows of bf16 of the head's length
int check_rows(const cfgzip_head* h, const void* p, int64_t stride) {
    if (!p || stride < h->H) return CFGZIP_E_ARG;
    return on16(p, stride * 2) ? CFGZIP_OK : CFGZIP_E_ALIGN;
}

constexpr int64_t kPieceBytes = int64_t(256) << 20;  // most of the gradient of the scores that is held at a time
constexpr int kStepBlocks = 148;                     // blocks of a decode step at most

struct HeadSpace {
    // step
    uint16_t* half;
    float* back;
    uint32_t *mask, *any, *bits, *ticket;
    int32_t* counts;
    Partial* states;
    // loss, log probabilities
    float2* part;
    float4* part_entropy;
    float* of_target;
    // gradient
    int32_t piece, splits;  // tokens of a piece, cuts of the sum over them
    uint16_t* g;
    float* sums;
    // ... of log probabilities
    float *rest, *kept;
    int32_t *first_of, *next_of;
    int64_t bytes;
};

// What is taken for `rows` rows is enough for fewer, whose tiles, pieces and cuts are others.
HeadSpace head_space(const cfgzip_head* h, int op, int32_t rows, void* workspace) {
    const uintptr_t skip = (256 - reinterpret_cast<uintptr_t>(workspace) % 256) % 256;
    Carve c(workspace ? static_cast<char*>(workspace) + skip : nullptr);
    HeadSpace s{};
    const int64_t n = rows;
    if (op == CFGZIP_HEAD_STEP) {
        s.mask = c.take<uint32_t>(n * ceil_div(h->V, 32));
        s.any = c.take<uint32_t>(ceil_div(h->V, 32));
        s.bits = c.take<uint32_t>(std::min<int64_t>(up(n, 32), kStepRows) * ceil_div(h->V, 32));
        s.counts = c.take<int32_t>(ceil_div(h->V, 32 * kUnionWords));
        s.ticket = c.take<uint32_t>(1);
        const bool tall = n > kStepRows && h->dtype == CFGZIP_BF16;
        s.states = c.take<Partial>(std::max(std::min<int64_t>(n, kStepRows) * kStepBlocks, tall ? most_states(n, h->V) : 0));
        if (h->dtype == CFGZIP_MXFP4) {
            s.half = c.take<uint16_t>(std::min<int64_t>(n, kStepRowsMx) * up(h->H, 2 * int(kStepAtom)));
            s.back = c.take<float>(kStepRowsMx);
        }
    } else if (op == CFGZIP_HEAD_LOSS) {
        s.part = c.take<float2>(most_states(n, h->V));
        s.of_target = c.take<float>(n);
    } else if (op == CFGZIP_HEAD_LOGPROBS) {
        s.part_entropy = c.take<float4>(most_states(n, h->V));
        s.of_target = c.take<float>(n);
    } else {
        const int64_t all = up(h->V, kMmaTile), room = kPieceBytes / 2, across = ceil_div(h->H, kMmaTile);
        s.piece = int32_t(std::min(all, std::max<int64_t>(room / std::max<int64_t>(n, 1) / kMmaTile * kMmaTile, kMmaTile)));
        s.splits = cuts(ceil_div(n, kMmaTile) * across, s.piece / kMmaK, n * h->H);
        const int64_t most_cuts = std::max<int64_t>(1, std::min({int64_t(kPairs), kCutTiles / across, all / kMmaK / 16}));
        s.g = c.take<uint16_t>(std::max(std::min(n * all, room), n * kMmaTile));
        if (op == CFGZIP_HEAD_LOGPROBS_BACKWARD) {
            s.rest = c.take<float>(n);
            s.next_of = c.take<int32_t>(n);
            s.first_of = c.take<int32_t>(h->V);
            s.kept = c.take<float>(n * h->H);
        }
        s.sums = c.take<float>(std::max(n * h->H, std::min<int64_t>(n * h->H * most_cuts, int64_t(kCutTiles) * kMmaTile * kMmaTile)));
    }
    s.bytes = c.used + 256;
    return s;
}

// Hidden states [rows, stride] (stride a multiple of 256) for tiled copies that bring 256 k of all rows, 64 after 64.
int tensor_map_by_64(cfgzip_ctx* ctx, CUtensorMap* map, const uint16_t* p, int64_t rows, int64_t stride, int box) {
    const cuuint64_t dims[3] = {64, cuuint64_t(rows), cuuint64_t(stride) / 64};
    const cuuint64_t strides[2] = {cuuint64_t(stride) * 2, 128};
    const cuuint32_t boxes[3] = {64, cuuint32_t(box), 4};
    const cuuint32_t steps[3] = {1, 1, 1};
    if (!ctx->encode_tiled ||
        ctx->encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint16_t*>(p), dims, strides, boxes, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return CFGZIP_E_CUDA;
    return CFGZIP_OK;
}

// Threads of a launch that takes a head by vectors of 8 weights (mx_at).
void mx_shape(const cfgzip_head* h, dim3* grid, dim3* block) {
    const int vectors = h->H / 8, y = ceil_div(vectors, 512);
    block->x = unsigned(up(ceil_div(vectors, y), 32));
    block->y = std::max(1u, 256u / block->x);
    grid->x = unsigned(ceil_div(h->V, int64_t(block->y) * kMxRows));
    grid->y = unsigned(y);
}

// Masks of rows that share a partition whose class masks fit a table in shared memory; part null: the vocab masks are there.
struct StepMasks {
    const PartDev* part = nullptr;
    const uint32_t* class_mask = nullptr;
    int64_t class_stride = 0;
    uint32_t* vocab_mask = nullptr;
    int64_t vocab_stride = 0;
};
constexpr int kTableWords = 1280;  // longest class mask for it: 160 KB

// One decode step of up to kStepRows (kStepRowsMx) rows.
int run_step(cfgzip_ctx* ctx, HeadStepArgs& a, const cfgzip_head* head, const uint16_t* hidden, int64_t hidden_stride,
             const HeadSpace& w, const StepMasks& m, cudaStream_t st) {
    const bool mx = head->dtype == CFGZIP_MXFP4;
    CUtensorMap map_x, map_w, map_box;
    int rc;
    a.N = a.B <= 16 ? 16 : up(a.B, 32);
    a.weight = head->weight;
    a.row_bytes = head->row_stride * (mx ? 1 : 2);
    a.bytes = mx ? head->H / 2 : head->H * 2;
    a.row_atoms = ceil_div(a.bytes, kStepAtom);
    a.scales = static_cast<const uint8_t*>(head->scales);
    a.scale_stride = head->scale_stride;
    if (mx) {
        a.hidden = hidden;
        a.hidden_stride = hidden_stride;
        a.half = w.half;
        a.half_stride = up(head->H, 2 * int(kStepAtom));
        a.back = w.back;
    }
    rc = mx ? tensor_map_by_64(ctx, &map_x, w.half, a.B, a.half_stride, a.N)
            : tensor_map(ctx, &map_x, hidden, a.B, head->H, hidden_stride, a.N);
    const int cols = mx ? a.bytes : head->H;
    if (rc != CFGZIP_OK || (rc = tensor_map(ctx, &map_w, head->weight, head->V, cols, head->row_stride, 128, mx)) != CFGZIP_OK ||
        (rc = tensor_map(ctx, &map_box, head->weight, head->V, cols, head->row_stride, kStepBox, mx)) != CFGZIP_OK)
        return rc;
    a.n_counts = ceil_div(a.VW, kUnionWords);
    const dim3 pieces(unsigned(a.n_counts + (mx ? a.B : 0)));
    if (m.part) {
        const size_t table = size_t(m.part->KW) * 128;
        if ((rc = ensure_smem(ctx, k_head_masks, table)) != CFGZIP_OK ||
            (rc = launch(ctx, k_head_masks, pieces, dim3(kUnionThreads), table, st, a, *m.part, m.class_mask, m.class_stride, m.vocab_mask,
                         m.vocab_stride)) != CFGZIP_OK)
            return rc;
    } else if ((rc = launch(ctx, k_head_union, pieces, dim3(kUnionThreads), 0, st, a)) != CFGZIP_OK) {
        return rc;
    }
    if (a.logits) {
        const dim3 grid(unsigned(std::max(1, std::min(ceil_div(a.V, 8192), 64))), unsigned(a.B));
        if ((rc = launch(ctx, a.logits_dtype == CFGZIP_BF16 ? k_head_fill<kBF16> : k_head_fill<kF32>, grid, dim3(256), 0, st, a)) !=
            CFGZIP_OK)
            return rc;
    }
    const unsigned blocks = unsigned(std::min(ctx->sm_count, kStepBlocks));
    a.rounds = ceil_div(ceil_div(a.V, blocks), kStepShare);
    a.smem = 181 << 10;
    a.expire = ctx->expire_test;
    const size_t smem = size_t(a.smem) + 1024 + kStepTile;  // (products read 128 rows, also where fewer are there)
    auto kern = mx ? k_head_step<true> : k_head_step<false>;
    if ((rc = ensure_smem(ctx, kern, smem)) != CFGZIP_OK) return rc;
    return launch(ctx, kern, dim3(blocks), dim3((mx ? kStepWarpsMx : kStepWarps) * 32), smem, st, a, map_x, map_w, map_box);
}

// Do two matrices of `rows` rows of `n` bf16 numbers have memory in common, rows and what is between them taken together?
bool overlap(const void* p, int64_t p_stride, const void* q, int64_t q_stride, int64_t rows, int n) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a < b + uintptr_t((rows - 1) * q_stride + n) * 2 && b < a + uintptr_t((rows - 1) * p_stride + n) * 2;
}

// What a gradient is of: of the loss, or of log probabilities and entropies.
struct GradientOf {
    const int32_t* targets;
    const float *lse, *entropy;
    const float *d_loss, *d_entropy;  // (d_loss: of the log probabilities where `scores` is true)
    bool scores;
};

int head_gradient(cfgzip_ctx* ctx, const cfgzip_head* head, const void* hidden, int64_t hidden_stride, int32_t N, const uint32_t* vocab_mask,
                  int64_t vocab_stride_words, const GradientOf& of, void* d_hidden, int64_t d_hidden_stride, void* d_weight,
                  int d_weight_dtype, int64_t d_weight_stride, int accumulate, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (head->dtype != CFGZIP_BF16 || N < 0 || (!d_hidden && !d_weight)) return CFGZIP_E_ARG;
    if (N > kHeadTokens || (of.scores && int64_t(N) * ceil_div(head->H, kTargetCols) > kHeadTokens)) return CFGZIP_E_RANGE;  // (blocks)
    if (d_weight) {
        if ((d_weight_dtype != CFGZIP_F32 && d_weight_dtype != CFGZIP_BF16) || d_weight_stride < head->H) return CFGZIP_E_ARG;
        if (!on16(d_weight, d_weight_stride * (d_weight_dtype == CFGZIP_BF16 ? 2 : 4))) return CFGZIP_E_ALIGN;
    }
    if (d_hidden && (rc = check_rows(head, d_hidden, d_hidden_stride)) != CFGZIP_OK) return rc;
    if (N > 0) {
        if (of.scores ? !of.d_loss && !of.d_entropy : !of.d_loss) return CFGZIP_E_ARG;
        if (!of.lse || (of.d_loss && !of.targets) || (of.d_entropy && !of.entropy) || (vocab_mask && vocab_stride_words < ceil_div(head->V, 32))) return CFGZIP_E_ARG;
        if ((rc = check_rows(head, hidden, hidden_stride)) != CFGZIP_OK) return rc;
        if (!workspace) return CFGZIP_E_ARG;
    }
    const HeadSpace w = head_space(head, of.scores ? CFGZIP_HEAD_LOGPROBS_BACKWARD : CFGZIP_HEAD_LOSS_BACKWARD, N, workspace);
    if (N > 0 && workspace_bytes < w.bytes) return CFGZIP_E_NOMEM;
    if (!ctx) return CFGZIP_E_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int H = head->H;
    if (N == 0) {  // an empty sum
        if (!d_weight || accumulate) return CFGZIP_OK;
        const size_t es = d_weight_dtype == CFGZIP_BF16 ? 2 : 4;
        if (cudaMemset2DAsync(d_weight, size_t(d_weight_stride) * es, 0, size_t(H) * es, size_t(head->V), st) != cudaSuccess) {
            cudaGetLastError();
            return CFGZIP_E_CUDA;
        }
        return CFGZIP_OK;
    }
    CUtensorMap x_k, x_mn, w_k, w_mn, g_k, g_mn;
    if ((rc = tensor_map_a(ctx, &x_k, hidden, N, H, hidden_stride)) != CFGZIP_OK ||
        (rc = tensor_map(ctx, &x_mn, hidden, N, H, hidden_stride, 64)) != CFGZIP_OK)
        return rc;
    const int32_t* targets = of.d_loss ? of.targets : nullptr;
    if (of.scores && targets && (rc = launch(ctx, k_head_targets, dim3(unsigned(ceil_div(N, 8 * kTargetRows))), dim3(256), 0, st, targets, int(N),
                                                    int(head->V), w.first_of, w.next_of, w.rest)) != CFGZIP_OK)
        return rc;
    for (int32_t t0 = 0; t0 < head->V; t0 += w.piece) {
        const int32_t n = std::min(w.piece, head->V - t0);
        const uint16_t* weights = static_cast<const uint16_t*>(head->weight) + t0 * head->row_stride;
        // (columns of the piece behind the vocabulary are outside the maps: they come as zeros)
        const int width = tile_width(N, n);
        if ((rc = tensor_map(ctx, &w_k, weights, n, H, head->row_stride, width / 2)) != CFGZIP_OK ||
            (rc = tensor_map(ctx, &w_mn, weights, n, H, head->row_stride, 64)) != CFGZIP_OK ||
            (rc = tensor_map_a(ctx, &g_k, w.g, N, n, w.piece)) != CFGZIP_OK ||
            (rc = tensor_map(ctx, &g_mn, w.g, N, n, w.piece, 64)) != CFGZIP_OK)
            return rc;
        MmaArgs a{};
        a.width = width;
        a.rows = N;
        a.cols = n;
        a.k_blocks = ceil_div(H, kMmaK);
        a.m_fast = 1;
        a.t0 = t0;
        a.V = head->V;
        a.mask = vocab_mask;
        a.mask_stride = vocab_stride_words;
        a.targets = of.targets;
        a.lse = of.lse;
        a.d_loss = of.d_loss;
        a.entropy = of.entropy;
        a.d_entropy = of.d_entropy;
        a.rest = w.rest;
        a.out = w.g;
        a.ld = w.piece;
        rc = of.scores ? run_mma<false, false, kMmaGradEntropy>(ctx, a, x_k, w_k, st) : run_mma<false, false, kMmaGrad>(ctx, a, x_k, w_k, st);
        if (rc != CFGZIP_OK) return rc;
        if (d_hidden) {
            MmaArgs b{};
            b.rows = N;
            b.cols = H;
            b.k_blocks = ceil_div(n, kMmaK);
            b.splits = std::min(w.splits, b.k_blocks);
            b.out = w.sums;
            b.ld = H;
            b.split_elems = int64_t(N) * H;
            b.add = t0 > 0;
            if ((rc = run_mma<false, true, kMmaSum>(ctx, b, g_k, w_mn, st)) != CFGZIP_OK) return rc;
        }
        if (d_weight) {
            MmaArgs b{};
            b.rows = n;
            b.cols = H;
            b.k_blocks = ceil_div(N, kMmaK);
            b.ld = d_weight_stride;
            b.add = accumulate;
            const bool half = d_weight_dtype == CFGZIP_BF16;
            b.out = static_cast<char*>(d_weight) + int64_t(t0) * d_weight_stride * (half ? 2 : 4);
            b.t0 = t0;
            b.targets = targets;
            b.text_rows = N;
            b.first_of = w.first_of;
            b.kept = w.kept;
            if (of.scores && targets)
                rc = half ? run_mma<true, true, kMmaBf16Targets>(ctx, b, g_mn, x_mn, st) : run_mma<true, true, kMmaSumTargets>(ctx, b, g_mn, x_mn, st);
            else
                rc = half ? run_mma<true, true, kMmaBf16>(ctx, b, g_mn, x_mn, st) : run_mma<true, true, kMmaSum>(ctx, b, g_mn, x_mn, st);
            if (rc != CFGZIP_OK) return rc;
        }
    }
    const int splits = std::min(w.splits, ceil_div(std::min(w.piece, head->V), kMmaK));
    const int64_t blocks = std::min<int64_t>(ceil_div(int64_t(N) * (H / 4), 256), int64_t(ctx->sm_count) * 8);
    if (of.scores && targets) {
        WeightTargetsArgs t{};
        t.targets = targets;
        t.first_of = w.first_of;
        t.next_of = w.next_of;
        t.rest = w.rest;
        t.kept = w.kept;
        t.hidden = static_cast<const uint16_t*>(hidden);
        t.hidden_stride = hidden_stride;
        t.to = d_weight;
        t.to_stride = d_weight_stride;
        t.N = N;
        t.V = head->V;
        t.H = H;
        t.bf16 = d_weight_dtype == CFGZIP_BF16;
        RoundTargetsArgs r{};
        r.from = w.sums;
        r.split_elems = int64_t(N) * H;
        r.splits = splits;
        r.rows = N;
        r.n = H;
        r.V = head->V;
        r.to = static_cast<uint16_t*>(d_hidden);
        r.to_stride = d_hidden_stride;
        r.targets = targets;
        r.rest = w.rest;
        r.weight = static_cast<const uint16_t*>(head->weight);
        r.weight_stride = head->row_stride;
        const int rows = d_weight ? N : 0, slices = ceil_div(N, kTargetSlice), ahead = d_weight && N > kTargetSteps ? slices * ceil_div(H, kTargetCols) : 0;
        // (in one launch the hidden states would be read while a gradient in their place is written)
        if (rows && d_hidden && overlap(hidden, hidden_stride, d_hidden, d_hidden_stride, N, H)) {
            rc = launch(ctx, k_head_targets_finish, dim3(unsigned(ahead + rows)), dim3(256), 0, st, t, r, ahead, slices, rows);
            return rc != CFGZIP_OK ? rc : launch(ctx, k_head_targets_finish, dim3(unsigned(blocks)), dim3(256), 0, st, t, r, 0, 0, 0);
        }
        return launch(ctx, k_head_targets_finish, dim3(unsigned(ahead + rows + (d_hidden ? blocks : 0))), dim3(256), 0, st, t, r, ahead,
                      slices, rows);
    }
    if (!d_hidden) return CFGZIP_OK;
    return launch(ctx, k_head_round, dim3(unsigned(blocks)), dim3(256), 0, st, (const float*)w.sums, int64_t(N) * H, splits,
                  static_cast<uint16_t*>(d_hidden), d_hidden_stride, int(N), H);
}

}  // namespace

extern "C" {

int cfgzip_head_workspace(const cfgzip_head* head, int op, int32_t rows, int64_t* bytes) {
    const bool known = (op >= CFGZIP_HEAD_STEP && op <= CFGZIP_HEAD_LOSS_BACKWARD) || op == CFGZIP_HEAD_LOGPROBS ||
                       op == CFGZIP_HEAD_LOGPROBS_BACKWARD;
    if (!bytes || rows < 0 || !known) return CFGZIP_E_ARG;
    const int rc = check_head_shape(head);
    if (rc != CFGZIP_OK) return rc;
    if (op != CFGZIP_HEAD_STEP && head->dtype != CFGZIP_BF16) return CFGZIP_E_ARG;
    if (rows > kHeadTokens) return CFGZIP_E_RANGE;
    *bytes = head_space(head, op, rows, nullptr).bytes;
    return CFGZIP_OK;
}

int cfgzip_head_quantize(cfgzip_ctx* ctx, const void* weight, int dtype, int64_t row_stride_elems, const cfgzip_head* head,
                         void* stream) {
    const int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (head->dtype != CFGZIP_MXFP4 || !weight || (dtype != CFGZIP_F32 && dtype != CFGZIP_BF16) || row_stride_elems < head->H) return CFGZIP_E_ARG;
    if (!on16(weight, row_stride_elems * (dtype == CFGZIP_BF16 ? 2 : 4))) return CFGZIP_E_ALIGN;
    if (!ctx) return CFGZIP_E_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    dim3 grid, block;
    mx_shape(head, &grid, &block);
    return launch(ctx, dtype == CFGZIP_BF16 ? k_mx_quantize<kBF16> : k_mx_quantize<kF32>, grid, block, 0,
                  static_cast<cudaStream_t>(stream), weight, row_stride_elems, head->H / 8, int(head->V), static_cast<uint8_t*>(head->weight), head->row_stride,
                  static_cast<uint8_t*>(head->scales), head->scale_stride);
}

int cfgzip_head_dequantize(cfgzip_ctx* ctx, const cfgzip_head* head, void* values, int64_t row_stride_elems, void* stream) {
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (head->dtype != CFGZIP_MXFP4) return CFGZIP_E_ARG;
    if ((rc = check_rows(head, values, row_stride_elems)) != CFGZIP_OK) return rc;
    if (!ctx) return CFGZIP_E_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    dim3 grid, block;
    mx_shape(head, &grid, &block);
    return launch(ctx, k_mx_dequantize, grid, block, 0, static_cast<cudaStream_t>(stream), static_cast<const uint8_t*>(head->weight),
                  head->row_stride, static_cast<const uint8_t*>(head->scales), head->scale_stride, head->H / 8, int(head->V),
                  static_cast<uint16_t*>(values), row_stride_elems);
}

int cfgzip_head_step(cfgzip_ctx* ctx, cfgzip_part_id part0, const int32_t* row_part, const uint32_t* class_mask,
                     int64_t class_stride_words, const cfgzip_head* head, const void* hidden, int64_t hidden_stride, int32_t B,
                     uint32_t* vocab_mask, int64_t vocab_stride_words, void* logits, int logits_dtype, int64_t logits_stride,
                     int32_t* argmax, int32_t* rep, float* logp_argmax, float* lse, void* workspace, int64_t workspace_bytes,
                     void* stream) {
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (B < 0) return CFGZIP_E_ARG;
    if (B > kHeadTokens) return CFGZIP_E_RANGE;
    HeadSpace w{};
    if (B > 0) {
        if (!argmax || !class_mask || class_stride_words <= 0 || (vocab_mask && vocab_stride_words < ceil_div(head->V, 32))) return CFGZIP_E_ARG;
        if (logits && ((logits_dtype != CFGZIP_F32 && logits_dtype != CFGZIP_BF16) || logits_stride < head->V)) return CFGZIP_E_ARG;
        if ((rc = check_rows(head, hidden, hidden_stride)) != CFGZIP_OK) return rc;
        if (!workspace) return CFGZIP_E_ARG;
        w = head_space(head, CFGZIP_HEAD_STEP, B, workspace);
        if (workspace_bytes < w.bytes) return CFGZIP_E_NOMEM;
    }
    if (!ctx) return CFGZIP_E_ARG;
    bool planned;
    const int32_t* rows = row_part;
    if ((rc = resolve_row_part(ctx, part0, &rows, B, &planned)) != CFGZIP_OK) return rc;
    PartSet ps;
    if ((rc = resolve_parts(ctx, part0, rows != nullptr, &ps)) != CFGZIP_OK) return rc;
    if (ps.V != head->V) return CFGZIP_E_RANGE;
    if (B == 0) return CFGZIP_OK;
    if (class_stride_words < ps.maxKW) return CFGZIP_E_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint32_t* mask = vocab_mask ? vocab_mask : w.mask;
    const int64_t mask_stride = vocab_mask ? vocab_stride_words : ps.VW;
    const PartDev& one = ctx->parts[size_t(part0)].dev;
    // More rows than one pass over the weights takes are a product of two tall matrices, over all of the head: what the rows allow
    // together is known on the device alone. (128256 x 4096: 256 rows that allow most of it 236 to 241 us, a pass of 128 rows alone 221, so
    // two of them 442; 256 rows that allow 3 to 21 % of it together would take 177 to 213 in two passes, 129 rows that allow 3 % 112 and
    // not 225. The scores of this product leave in the wrong order to be stored.)
    const bool tall = B > kStepRows && head->dtype == CFGZIP_BF16 && !logits;
    const bool table = !tall && !rows && one.c16 && one.KW <= kTableWords;
    if (!table && (rc = cfgzip_expand_mask(ctx, part0, row_part, class_mask, class_stride_words, mask, mask_stride, B, CFGZIP_DENSE, stream)) !=
        CFGZIP_OK)
        return rc;
    const int32_t most = head->dtype == CFGZIP_MXFP4 ? kStepRowsMx : kStepRows;
    if (tall) {
        CUtensorMap map_x, map_w;
        if ((rc = tensor_map_a(ctx, &map_x, hidden, B, head->H, hidden_stride)) != CFGZIP_OK ||
            (rc = tensor_map(ctx, &map_w, head->weight, head->V, head->H, head->row_stride, tile_width(B, head->V) / 2)) != CFGZIP_OK)
            return rc;
        MmaArgs a{};
        a.width = tile_width(B, head->V);
        a.rows = B;
        a.cols = a.V = head->V;
        a.k_blocks = ceil_div(head->H, kMmaK);
        a.m_fast = 1;
        a.mask = mask;
        a.mask_stride = mask_stride;
        a.states = w.states;
        if ((rc = run_mma<false, false, kMmaStep>(ctx, a, map_x, map_w, st)) != CFGZIP_OK) return rc;
        HeadStepArgs s{};
        s.parts = ctx->d_parts;
        s.part0 = part0;
        s.n_parts = int32_t(ctx->parts.size());
        s.row_part = rows;
        s.B = B;
        s.V = head->V;
        s.part = w.states;
        s.argmax = argmax;
        s.rep = rep;
        s.logp = logp_argmax;
        s.lse = lse;
        s.status = ctx->d_status;
        return launch(ctx, k_head_step_finish, dim3(unsigned(ceil_div(B, 8))), dim3(256), 0, st, s, 2 * a.n_tiles);
    }
    for (int32_t b = 0; b < B; b += most) {
        HeadStepArgs s{};
        StepMasks m;
        if (table) m = StepMasks{&one, class_mask + b * class_stride_words, class_stride_words,
                                 vocab_mask ? vocab_mask + b * vocab_stride_words : nullptr, vocab_stride_words};
        s.parts = ctx->d_parts;
        s.part0 = part0;
        s.n_parts = int32_t(ctx->parts.size());
        s.row_part = rows ? rows + b : nullptr;
        s.mask = mask + b * mask_stride;
        s.mask_stride = mask_stride;
        s.B = std::min(most, B - b);
        s.V = head->V;
        s.VW = ps.VW;
        s.H = head->H;
        s.any = w.any;
        s.bits = w.bits;
        s.counts = w.counts;
        s.ticket = w.ticket;
        s.part = w.states;
        s.logits = logits ? static_cast<char*>(logits) + b * logits_stride * (logits_dtype == CFGZIP_BF16 ? 2 : 4) : nullptr;
        s.logits_dtype = logits_dtype;
        s.logits_stride = logits_stride;
        s.argmax = argmax + b;
        s.rep = rep ? rep + b : nullptr;
        s.logp = logp_argmax ? logp_argmax + b : nullptr;
        s.lse = lse ? lse + b : nullptr;
        s.status = ctx->d_status;
        rc = run_step(ctx, s, head, static_cast<const uint16_t*>(hidden) + b * hidden_stride, hidden_stride, w, m, st);
        if (rc != CFGZIP_OK) return rc;
    }
    return CFGZIP_OK;
}

int cfgzip_head_loss(cfgzip_ctx* ctx, const cfgzip_head* head, const void* hidden, int64_t hidden_stride, int32_t N,
                     const uint32_t* vocab_mask, int64_t vocab_stride_words, const int32_t* targets, float* loss, float* lse,
                     void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (head->dtype != CFGZIP_BF16 || N < 0) return CFGZIP_E_ARG;
    if (N > kHeadTokens) return CFGZIP_E_RANGE;
    if (N == 0) return ctx ? CFGZIP_OK : CFGZIP_E_ARG;
    if (!targets || !loss || (vocab_mask && vocab_stride_words < ceil_div(head->V, 32))) return CFGZIP_E_ARG;
    if ((rc = check_rows(head, hidden, hidden_stride)) != CFGZIP_OK) return rc;
    if (!workspace) return CFGZIP_E_ARG;
    const HeadSpace w = head_space(head, CFGZIP_HEAD_LOSS, N, workspace);
    if (workspace_bytes < w.bytes) return CFGZIP_E_NOMEM;
    if (!ctx) return CFGZIP_E_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    CUtensorMap map_x, map_w;
    if ((rc = tensor_map_a(ctx, &map_x, hidden, N, head->H, hidden_stride)) != CFGZIP_OK ||
        (rc = tensor_map(ctx, &map_w, head->weight, head->V, head->H, head->row_stride, tile_width(N, head->V) / 2)) != CFGZIP_OK)
        return rc;
    MmaArgs a{};
    a.width = tile_width(N, head->V);
    a.rows = N;
    a.cols = a.V = head->V;
    a.k_blocks = ceil_div(head->H, kMmaK);
    a.m_fast = 1;
    a.mask = vocab_mask;
    a.mask_stride = vocab_stride_words;
    a.targets = targets;
    a.part = w.part;
    a.of_target = w.of_target;
    if ((rc = run_mma<false, false, kMmaLoss>(ctx, a, map_x, map_w, st)) != CFGZIP_OK) return rc;
    FinishArgs f{};
    f.part = w.part;
    f.of_target = w.of_target;
    f.tiles = 2 * a.n_tiles;
    f.rows = N;
    f.V = head->V;
    f.mask = vocab_mask;
    f.mask_stride = vocab_stride_words;
    f.targets = targets;
    f.loss = loss;
    f.lse = lse;
    f.status = ctx->d_status;
    return launch(ctx, k_head_loss_finish, dim3(unsigned(ceil_div(N, kFinishRows))), dim3(256), 0, st, f);
}

int cfgzip_head_loss_backward(cfgzip_ctx* ctx, const cfgzip_head* head, const void* hidden, int64_t hidden_stride, int32_t N,
                              const uint32_t* vocab_mask, int64_t vocab_stride_words, const int32_t* targets, const float* lse,
                              const float* d_loss, void* d_hidden, int64_t d_hidden_stride, void* d_weight, int d_weight_dtype,
                              int64_t d_weight_stride, int accumulate, void* workspace, int64_t workspace_bytes, void* stream) {
    const GradientOf of{targets, lse, nullptr, d_loss, nullptr, false};
    return head_gradient(ctx, head, hidden, hidden_stride, N, vocab_mask, vocab_stride_words, of, d_hidden, d_hidden_stride, d_weight,
                         d_weight_dtype, d_weight_stride, accumulate, workspace, workspace_bytes, stream);
}

int cfgzip_head_logprobs(cfgzip_ctx* ctx, const cfgzip_head* head, const void* hidden, int64_t hidden_stride, int32_t N,
                         const uint32_t* vocab_mask, int64_t vocab_stride_words, const int32_t* tokens, float* logp, float* entropy,
                         float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (head->dtype != CFGZIP_BF16 || N < 0) return CFGZIP_E_ARG;
    if (N > kHeadTokens) return CFGZIP_E_RANGE;
    if (N == 0) return ctx ? CFGZIP_OK : CFGZIP_E_ARG;
    if (!tokens || !logp || (vocab_mask && vocab_stride_words < ceil_div(head->V, 32))) return CFGZIP_E_ARG;
    if ((rc = check_rows(head, hidden, hidden_stride)) != CFGZIP_OK) return rc;
    if (!workspace) return CFGZIP_E_ARG;
    const HeadSpace w = head_space(head, CFGZIP_HEAD_LOGPROBS, N, workspace);
    if (workspace_bytes < w.bytes) return CFGZIP_E_NOMEM;
    if (!ctx) return CFGZIP_E_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    CUtensorMap map_x, map_w;
    MmaArgs a{};
    a.width = tile_width(N, head->V);
    if ((rc = tensor_map_a(ctx, &map_x, hidden, N, head->H, hidden_stride)) != CFGZIP_OK ||
        (rc = tensor_map(ctx, &map_w, head->weight, head->V, head->H, head->row_stride, a.width / 2)) != CFGZIP_OK)
        return rc;
    a.rows = N;
    a.cols = a.V = head->V;
    a.k_blocks = ceil_div(head->H, kMmaK);
    a.m_fast = 1;
    a.mask = vocab_mask;
    a.mask_stride = vocab_stride_words;
    a.targets = tokens;
    a.sums = w.part_entropy;
    a.of_target = w.of_target;
    if ((rc = run_mma<false, false, kMmaLogprobs>(ctx, a, map_x, map_w, st)) != CFGZIP_OK) return rc;
    LogprobsFinishArgs f{};
    f.sums = w.part_entropy;
    f.of_target = w.of_target;
    f.tiles = 2 * a.n_tiles;
    f.rows = N;
    f.V = head->V;
    f.mask = vocab_mask;
    f.mask_stride = vocab_stride_words;
    f.tokens = tokens;
    f.logp = logp;
    f.entropy = entropy;
    f.lse = lse;
    f.status = ctx->d_status;
    return launch(ctx, k_head_logprobs_finish, dim3(unsigned(ceil_div(N, kFinishRows))), dim3(256), 0, st, f);
}

int cfgzip_head_logprobs_backward(cfgzip_ctx* ctx, const cfgzip_head* head, const void* hidden, int64_t hidden_stride, int32_t N,
                                  const uint32_t* vocab_mask, int64_t vocab_stride_words, const int32_t* tokens, const float* lse,
                                  const float* entropy, const float* d_logp, const float* d_entropy, void* d_hidden, int64_t d_hidden_stride,
                                  void* d_weight, int d_weight_dtype, int64_t d_weight_stride, int accumulate, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
    const GradientOf of{tokens, lse, entropy, d_logp, d_entropy, true};
    return head_gradient(ctx, head, hidden, hidden_stride, N, vocab_mask, vocab_stride_words, of, d_hidden, d_hidden_stride, d_weight,
                         d_weight_dtype, d_weight_stride, accumulate, workspace, workspace_bytes, stream);
}

}  // extern "C"
