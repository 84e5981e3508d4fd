// C ABI of the head calls: argument checks, workspaces, launches. Contracts in include/cfgzip.h.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cfgzip.h"
#include "cfgzip_head.cuh"
#include "context.h"

using namespace cfgzip;

namespace {

constexpr int kHeadMost = 65536;  // longest row of a head
constexpr int kPiece = 8192;      // tokens whose scores are held at a time

bool on16(const void* p, int64_t stride_bytes) { return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(stride_bytes)) & 15u) == 0; }

int check_head_shape(const cfgzip_head* h) {
    if (!h || h->V <= 0 || h->H <= 0 || (h->dtype != CFGZIP_BF16 && h->dtype != CFGZIP_MXFP4) || h->reserved) return CFGZIP_E_ARG;
    if (h->H % (h->dtype == CFGZIP_BF16 ? 8 : kMxBlock)) return CFGZIP_E_ARG;
    return h->H > kHeadMost ? CFGZIP_E_RANGE : CFGZIP_OK;
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

// A workspace taken apart; with no memory behind it, only counted.
struct Carve {
    char* at;
    int64_t used = 0;
    explicit Carve(void* p) : at(static_cast<char*>(p)) {}
    template <typename T>
    T* take(int64_t n) {
        T* r = at ? reinterpret_cast<T*>(at + used) : nullptr;
        used += (n * int64_t(sizeof(T)) + 255) / 256 * 256;
        return r;
    }
};

struct HeadSpace {
    float* z;
    RowState* state;
    uint16_t *g, *weights;
    float* d_hidden;
    uint32_t* mask;
    int64_t bytes;
};

HeadSpace head_space(const cfgzip_head* h, int op, int32_t rows, void* workspace) {
    const uintptr_t skip = (256 - reinterpret_cast<uintptr_t>(workspace) % 256) % 256;
    Carve c(workspace ? static_cast<char*>(workspace) + skip : nullptr);
    HeadSpace s{};
    s.z = c.take<float>(int64_t(rows) * kPiece);
    if (op != CFGZIP_HEAD_LOSS_BACKWARD) s.state = c.take<RowState>(rows);
    if (op == CFGZIP_HEAD_LOSS_BACKWARD) {
        s.g = c.take<uint16_t>(int64_t(rows) * kPiece);
        s.d_hidden = c.take<float>(int64_t(rows) * h->H);
    }
    if (op == CFGZIP_HEAD_STEP) {
        s.mask = c.take<uint32_t>(int64_t(rows) * ceil_div(h->V, 32));
        if (h->dtype == CFGZIP_MXFP4) s.weights = c.take<uint16_t>(int64_t(kPiece) * h->H);
    }
    s.bytes = c.used + 256;
    return s;
}

int product(cfgzip_ctx* ctx, const ProductArgs& p, cudaStream_t st) {
    return launch(ctx, k_head_product, dim3(unsigned(ceil_div(p.N, 64)), unsigned(ceil_div(p.M, 64))), dim3(256), 0, st, p);
}

int dequantize(cfgzip_ctx* ctx, const cfgzip_head* h, int32_t t0, int32_t n, uint16_t* values, int64_t stride, cudaStream_t st) {
    const int64_t total = int64_t(n) * (h->H / 8);
    return launch(ctx, k_mx_dequantize, dim3(unsigned(ceil_div(total, 256 * kMxUnroll))), dim3(256), 0, st,
                  static_cast<const uint8_t*>(h->weight) + t0 * h->row_stride, h->row_stride,
                  static_cast<const uint8_t*>(h->scales) + t0 * h->scale_stride, h->scale_stride, h->H / 8, total, values, stride);
}

// Scores of a piece of the vocabulary.
int scores(cfgzip_ctx* ctx, const cfgzip_head* h, const HeadSpace& w, const void* hidden, int64_t stride, int32_t rows, int32_t t0,
           int32_t n, cudaStream_t st) {
    const uint16_t* weights = static_cast<const uint16_t*>(h->weight) + t0 * h->row_stride;
    int64_t ld = h->row_stride;
    if (h->dtype == CFGZIP_MXFP4) {
        const int rc = dequantize(ctx, h, t0, n, w.weights, h->H, st);
        if (rc != CFGZIP_OK) return rc;
        weights = w.weights;
        ld = h->H;
    }
    return product(ctx, ProductArgs{static_cast<const uint16_t*>(hidden), weights, stride, 1, ld, 1, w.z, kPiece, rows, n, h->H, 0, 0},
                   st);
}

}  // namespace

extern "C" {

int cfgzip_head_workspace(const cfgzip_head* head, int op, int32_t rows, int64_t* bytes) {
    if (!bytes || rows < 0 || op < CFGZIP_HEAD_STEP || op > CFGZIP_HEAD_LOSS_BACKWARD) return CFGZIP_E_ARG;
    const int rc = check_head_shape(head);
    if (rc != CFGZIP_OK) return rc;
    if (op != CFGZIP_HEAD_STEP && head->dtype != CFGZIP_BF16) return CFGZIP_E_ARG;
    *bytes = head_space(head, op, rows, nullptr).bytes;
    return CFGZIP_OK;
}

int cfgzip_head_quantize(cfgzip_ctx* ctx, const void* weight, int dtype, int64_t row_stride_elems, const cfgzip_head* head,
                         void* stream) {
    if (!ctx || !weight || (dtype != CFGZIP_F32 && dtype != CFGZIP_BF16)) return CFGZIP_E_ARG;
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (head->dtype != CFGZIP_MXFP4 || row_stride_elems < head->H) return CFGZIP_E_ARG;
    if (!on16(weight, row_stride_elems * (dtype == CFGZIP_BF16 ? 2 : 4))) return CFGZIP_E_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    const int64_t total = int64_t(head->V) * (head->H / 8);
    return launch(ctx, dtype == CFGZIP_BF16 ? k_mx_quantize<kBF16> : k_mx_quantize<kF32>,
                  dim3(unsigned(ceil_div(total, 256 * kMxUnroll))), dim3(256), 0, static_cast<cudaStream_t>(stream), weight,
                  row_stride_elems, head->H / 8, total, static_cast<uint8_t*>(head->weight), head->row_stride,
                  static_cast<uint8_t*>(head->scales), head->scale_stride);
}

int cfgzip_head_dequantize(cfgzip_ctx* ctx, const cfgzip_head* head, void* values, int64_t row_stride_elems, void* stream) {
    if (!ctx) return CFGZIP_E_ARG;
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (head->dtype != CFGZIP_MXFP4) return CFGZIP_E_ARG;
    if ((rc = check_rows(head, values, row_stride_elems)) != CFGZIP_OK) return rc;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    return dequantize(ctx, head, 0, head->V, static_cast<uint16_t*>(values), row_stride_elems, static_cast<cudaStream_t>(stream));
}

int cfgzip_head_step(cfgzip_ctx* ctx, cfgzip_part_id part0, const int32_t* row_part, const uint32_t* class_mask,
                     int64_t class_stride_words, const cfgzip_head* head, const void* hidden, int64_t hidden_stride, int32_t B,
                     uint32_t* vocab_mask, int64_t vocab_stride_words, void* logits, int logits_dtype, int64_t logits_stride,
                     int32_t* argmax, int32_t* rep, float* logp_argmax, float* lse, void* workspace, int64_t workspace_bytes,
                     void* stream) {
    if (!ctx || B < 0) return CFGZIP_E_ARG;
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    bool planned;
    const int32_t* rows = row_part;
    if ((rc = resolve_row_part(ctx, part0, &rows, B, &planned)) != CFGZIP_OK) return rc;
    PartSet ps;
    if ((rc = resolve_parts(ctx, part0, rows != nullptr, &ps)) != CFGZIP_OK) return rc;
    if (ps.V != head->V) return CFGZIP_E_RANGE;
    if (B == 0) return CFGZIP_OK;
    if (!argmax || !class_mask || class_stride_words < ps.maxKW || (vocab_mask && vocab_stride_words < ps.VW)) return CFGZIP_E_ARG;
    if (logits && ((logits_dtype != CFGZIP_F32 && logits_dtype != CFGZIP_BF16) || logits_stride < head->V)) return CFGZIP_E_ARG;
    if ((rc = check_rows(head, hidden, hidden_stride)) != CFGZIP_OK) return rc;
    if (!workspace) return CFGZIP_E_ARG;
    const HeadSpace w = head_space(head, CFGZIP_HEAD_STEP, B, workspace);
    if (workspace_bytes < w.bytes) return CFGZIP_E_NOMEM;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint32_t* mask = vocab_mask ? vocab_mask : w.mask;
    const int64_t mask_stride = vocab_mask ? vocab_stride_words : ps.VW;
    if ((rc = cfgzip_expand_mask(ctx, part0, row_part, class_mask, class_stride_words, mask, mask_stride, B, CFGZIP_DENSE, stream)) !=
        CFGZIP_OK)
        return rc;
    RowsArgs a{};
    a.parts = ctx->d_parts;
    a.part0 = part0;
    a.n_parts = int32_t(ctx->parts.size());
    a.row_part = rows;
    a.z = w.z;
    a.ldz = kPiece;
    a.rows = B;
    a.V = head->V;
    a.mask = mask;
    a.mask_stride = mask_stride;
    a.state = w.state;
    a.logits = logits;
    a.logits_dtype = logits_dtype;
    a.logits_stride = logits_stride;
    a.argmax = argmax;
    a.rep = rep;
    a.logp = logp_argmax;
    a.lse = lse;
    a.status = ctx->d_status;
    for (a.t0 = 0; a.t0 < a.V; a.t0 += kPiece) {
        a.n = std::min(kPiece, a.V - a.t0);
        if ((rc = scores(ctx, head, w, hidden, hidden_stride, B, a.t0, a.n, st)) != CFGZIP_OK) return rc;
        if ((rc = launch(ctx, k_head_rows, dim3(unsigned(B)), dim3(256), 0, st, a)) != CFGZIP_OK) return rc;
    }
    return launch(ctx, k_head_finish, dim3(unsigned(ceil_div(B, 256))), dim3(256), 0, st, a);
}

int cfgzip_head_loss(cfgzip_ctx* ctx, const cfgzip_head* head, const void* hidden, int64_t hidden_stride, int32_t N,
                     const uint32_t* vocab_mask, int64_t vocab_stride_words, const int32_t* targets, float* loss, float* lse,
                     void* workspace, int64_t workspace_bytes, void* stream) {
    if (!ctx || N < 0) return CFGZIP_E_ARG;
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (head->dtype != CFGZIP_BF16) return CFGZIP_E_ARG;
    if (N == 0) return CFGZIP_OK;
    if (!targets || !loss || (vocab_mask && vocab_stride_words < ceil_div(head->V, 32))) return CFGZIP_E_ARG;
    if ((rc = check_rows(head, hidden, hidden_stride)) != CFGZIP_OK) return rc;
    if (!workspace) return CFGZIP_E_ARG;
    const HeadSpace w = head_space(head, CFGZIP_HEAD_LOSS, N, workspace);
    if (workspace_bytes < w.bytes) return CFGZIP_E_NOMEM;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    RowsArgs a{};
    a.z = w.z;
    a.ldz = kPiece;
    a.rows = N;
    a.V = head->V;
    a.mask = vocab_mask;
    a.mask_stride = vocab_stride_words;
    a.state = w.state;
    a.targets = targets;
    a.lse = lse;
    a.loss = loss;
    a.status = ctx->d_status;
    for (a.t0 = 0; a.t0 < a.V; a.t0 += kPiece) {
        a.n = std::min(kPiece, a.V - a.t0);
        if ((rc = scores(ctx, head, w, hidden, hidden_stride, N, a.t0, a.n, st)) != CFGZIP_OK) return rc;
        if ((rc = launch(ctx, k_head_rows, dim3(unsigned(N)), dim3(256), 0, st, a)) != CFGZIP_OK) return rc;
    }
    return launch(ctx, k_head_finish, dim3(unsigned(ceil_div(N, 256))), dim3(256), 0, st, a);
}

int cfgzip_head_loss_backward(cfgzip_ctx* ctx, const cfgzip_head* head, const void* hidden, int64_t hidden_stride, int32_t N,
                              const uint32_t* vocab_mask, int64_t vocab_stride_words, const int32_t* targets, const float* lse,
                              const float* d_loss, void* d_hidden, int64_t d_hidden_stride, void* d_weight, int d_weight_dtype,
                              int64_t d_weight_stride, int accumulate, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!ctx || N < 0) return CFGZIP_E_ARG;
    int rc = check_head(head);
    if (rc != CFGZIP_OK) return rc;
    if (head->dtype != CFGZIP_BF16 || (!d_hidden && !d_weight)) return CFGZIP_E_ARG;
    if (d_weight) {
        if ((d_weight_dtype != CFGZIP_F32 && d_weight_dtype != CFGZIP_BF16) || d_weight_stride < head->H) return CFGZIP_E_ARG;
        if (!on16(d_weight, d_weight_stride * (d_weight_dtype == CFGZIP_BF16 ? 2 : 4))) return CFGZIP_E_ALIGN;
    }
    if (d_hidden && (rc = check_rows(head, d_hidden, d_hidden_stride)) != CFGZIP_OK) return rc;
    if (N > 0) {
        if (!targets || !lse || !d_loss || (vocab_mask && vocab_stride_words < ceil_div(head->V, 32))) return CFGZIP_E_ARG;
        if ((rc = check_rows(head, hidden, hidden_stride)) != CFGZIP_OK) return rc;
        if (!workspace) return CFGZIP_E_ARG;
    }
    const HeadSpace w = head_space(head, CFGZIP_HEAD_LOSS_BACKWARD, N, workspace);
    if (N > 0 && workspace_bytes < w.bytes) return CFGZIP_E_NOMEM;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const uint16_t* x = static_cast<const uint16_t*>(hidden);
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
    RowsArgs a{};
    a.z = w.z;
    a.ldz = kPiece;
    a.rows = N;
    a.V = head->V;
    a.mask = vocab_mask;
    a.mask_stride = vocab_stride_words;
    a.targets = targets;
    a.lse_in = lse;
    a.d_loss = d_loss;
    a.g = w.g;
    for (a.t0 = 0; a.t0 < a.V; a.t0 += kPiece) {
        a.n = std::min(kPiece, a.V - a.t0);
        if ((rc = scores(ctx, head, w, hidden, hidden_stride, N, a.t0, a.n, st)) != CFGZIP_OK) return rc;
        if ((rc = launch(ctx, k_head_gradient, dim3(unsigned(N)), dim3(256), 0, st, a)) != CFGZIP_OK) return rc;
        const uint16_t* weights = static_cast<const uint16_t*>(head->weight) + a.t0 * head->row_stride;
        if (d_hidden && (rc = product(ctx, ProductArgs{w.g, weights, kPiece, 1, 1, head->row_stride, w.d_hidden, H, N, H, a.n, 0, a.t0 > 0},
                                      st)) != CFGZIP_OK)
            return rc;
        if (d_weight) {
            const size_t es = d_weight_dtype == CFGZIP_BF16 ? 2 : 4;
            void* out = static_cast<char*>(d_weight) + size_t(a.t0) * size_t(d_weight_stride) * es;
            if ((rc = product(ctx, ProductArgs{w.g, x, 1, kPiece, 1, hidden_stride, out, d_weight_stride, a.n, H, N,
                                               d_weight_dtype == CFGZIP_BF16, accumulate}, st)) != CFGZIP_OK)
                return rc;
        }
    }
    if (!d_hidden) return CFGZIP_OK;
    return launch(ctx, k_head_round, dim3(unsigned(ctx->sm_count) * 8), dim3(256), 0, st, (const float*)w.d_hidden,
                  static_cast<uint16_t*>(d_hidden), d_hidden_stride, int(N), H);
}

}  // extern "C"
