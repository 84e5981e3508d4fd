// C ABI of the log probability calls on logits: argument checks, plans, launches. Contracts in include/cfgzip.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cfgzip.h"
#include "cfgzip_logprobs.cuh"
#include "context.h"

using namespace cfgzip;

namespace {

constexpr int kLogprobsTokens = 1 << 21;  // longest row: a chunk's largest logit each, in the shared memory of a block
constexpr int kLogprobsRows = 1 << 30;

bool on_element(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == CFGZIP_BF16 ? 1u : 3u)) == 0; }

int check_logits(const void* logits, int dtype, int64_t stride, int32_t N, int32_t V, const uint32_t* mask, int64_t mask_stride,
                 float inv_temperature) {
    if (N < 0 || V <= 0 || (dtype != CFGZIP_F32 && dtype != CFGZIP_BF16)) return CFGZIP_E_ARG;
    if (!(inv_temperature > 0.f) || inv_temperature > 1e6f) return CFGZIP_E_ARG;
    if (V > kLogprobsTokens || N > kLogprobsRows) return CFGZIP_E_RANGE;
    if (N == 0) return CFGZIP_OK;
    if (!logits || stride < V || (mask && mask_stride < ceil_div(V, 32))) return CFGZIP_E_ARG;
    return on_element(logits, dtype) ? CFGZIP_OK : CFGZIP_E_ALIGN;
}

// Blocks of a row: as many as there is room for side by side (four to an SM), while a warp keeps a few chunks.
int row_blocks(const cfgzip_ctx* ctx, int32_t N, int32_t V) {
    const int64_t room = int64_t(ctx->sm_count) * 4;
    const int chunks = ceil_div(V, kLogprobsChunk);
    int blocks = 1;
    while (blocks < kClusterMost && int64_t(N) * blocks * 2 <= room && chunks >= blocks * 2 * 8) blocks *= 2;
    return blocks;
}

}  // namespace

extern "C" {

int cfgzip_token_logprobs(cfgzip_ctx* ctx, const void* logits, int dtype, int64_t row_stride_elems, int32_t N, int32_t V,
                          const uint32_t* vocab_mask, int64_t vocab_stride_words, const int32_t* tokens, float inv_temperature, int32_t n_top,
                          float* logp, float* entropy, float* lse, int32_t* top_tokens, float* top_logp, void* stream) {
    int rc = check_logits(logits, dtype, row_stride_elems, N, V, vocab_mask, vocab_stride_words, inv_temperature);
    if (rc != CFGZIP_OK) return rc;
    if (n_top < 0 || n_top > kLogprobsTopMost) return CFGZIP_E_ARG;
    if (N > 0 && ((tokens == nullptr) != (logp == nullptr) || (n_top > 0 && (!top_tokens || !top_logp)))) return CFGZIP_E_ARG;
    if (!ctx) return CFGZIP_E_ARG;
    if (N == 0) return CFGZIP_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    LogprobsArgs a{};
    a.logits = logits;
    a.stride = row_stride_elems;
    a.N = N;
    a.V = V;
    a.mask = vocab_mask;
    a.mask_stride = vocab_stride_words;
    a.tokens = tokens;
    a.inv_temperature = inv_temperature;
    a.n_top = n_top;
    a.logp = logp;
    a.entropy = entropy;
    a.lse = lse;
    a.top_tokens = top_tokens;
    a.top_logp = top_logp;
    a.status = ctx->d_status;
    auto kern = dtype == CFGZIP_BF16 ? (vocab_mask ? k_token_logprobs<kBF16, true> : k_token_logprobs<kBF16, false>)
                                     : (vocab_mask ? k_token_logprobs<kF32, true> : k_token_logprobs<kF32, false>);
    const int blocks = row_blocks(ctx, N, V);
    const size_t smem = n_top ? size_t(ceil_div(V, kLogprobsChunk) + 2) * sizeof(float) : 0;
    if ((rc = ensure_smem(ctx, kern, smem, true)) != CFGZIP_OK) return rc;
    ctx->cluster_now = blocks;
    rc = launch(ctx, kern, dim3(unsigned(N) * unsigned(blocks)), dim3(kLogprobsThreads), smem, static_cast<cudaStream_t>(stream), a, blocks);
    ctx->cluster_now = 1;
    return rc;
}

int cfgzip_token_logprobs_backward(cfgzip_ctx* ctx, const void* logits, int dtype, int64_t row_stride_elems, int32_t N, int32_t V,
                                   const uint32_t* vocab_mask, int64_t vocab_stride_words, const int32_t* tokens, float inv_temperature,
                                   const float* lse, const float* entropy, const float* d_logp, const float* d_entropy, void* d_logits,
                                   int64_t d_stride_elems, void* stream) {
    const int rc = check_logits(logits, dtype, row_stride_elems, N, V, vocab_mask, vocab_stride_words, inv_temperature);
    if (rc != CFGZIP_OK) return rc;
    if (N > 0) {
        if (!lse || !d_logits || d_stride_elems < V || (!d_logp && !d_entropy) || (d_logp && !tokens) || (d_entropy && !entropy)) return CFGZIP_E_ARG;
        if (!on_element(d_logits, dtype)) return CFGZIP_E_ALIGN;
    }
    if (!ctx) return CFGZIP_E_ARG;
    if (N == 0) return CFGZIP_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return CFGZIP_E_CUDA;
    LogprobsBackwardArgs a{};
    a.logits = logits;
    a.stride = row_stride_elems;
    a.N = N;
    a.V = V;
    a.mask = vocab_mask;
    a.mask_stride = vocab_stride_words;
    a.tokens = tokens;
    a.inv_temperature = inv_temperature;
    a.lse = lse;
    a.entropy = entropy;
    a.d_logp = d_logp;
    a.d_entropy = d_entropy;
    a.d_logits = d_logits;
    a.d_stride = d_stride_elems;
    a.pieces = ceil_div(V, 8192);
    if (int64_t(N) * a.pieces >= (int64_t(1) << 31)) return CFGZIP_E_RANGE;
    auto kern = dtype == CFGZIP_BF16 ? (vocab_mask ? k_token_logprobs_backward<kBF16, true> : k_token_logprobs_backward<kBF16, false>)
                                     : (vocab_mask ? k_token_logprobs_backward<kF32, true> : k_token_logprobs_backward<kF32, false>);
    return launch(ctx, kern, dim3(unsigned(N) * unsigned(a.pieces)), dim3(256), 0, static_cast<cudaStream_t>(stream), a);
}

}  // extern "C"
