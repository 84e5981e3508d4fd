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
    if (!(inv_temperature >= 1e-6f) || inv_temperature > 1e6f) return CFGZIP_E_ARG;
    if (V > kLogprobsTokens || N > kLogprobsRows) return CFGZIP_E_RANGE;
    if (N == 0) return CFGZIP_OK;
    if (!logits || stride < V || (mask && mask_stride < ceil_div(V, 32))) return CFGZIP_E_ARG;
    return on_element(logits, dtype) ? CFGZIP_OK : CFGZIP_E_ALIGN;
}

// Blocks of a row: as many as there is room for side by side (two to an SM), while a warp keeps a chunk or two. (32 bf16 rows of 128256 with 20
// alternatives by 1, 2, 4, 8 and 16 blocks: 17.1, 13.2, 11.0, 10.1, 12.3 us; 148 rows 17.6, 15.6, 17.9; one row by 16 8.5.)
int row_blocks(const cfgzip_ctx* ctx, int32_t N, int32_t V) {
    const int64_t room = int64_t(ctx->sm_count) * 2;
    const int chunks = ceil_div(V, kLogprobsChunk);
    int blocks = 1;
    while (blocks < kClusterMost && int64_t(N) * blocks * 2 <= room && chunks >= blocks * 2 * 8) blocks *= 2;
    return blocks;
}

// Warps of a block. What a row costs besides its logits is latency, some 5 us in which its block holds a part of the SM: rows that do not all
// fit side by side by eight warps come by four (4096 bf16 rows of 32000, 5 alternatives: 82 and 69 us, of 128256: 218 and 203), short ones by
// two (of 2000: 38, 24 and 17 us). Not f32 rows with a mask, of which a warp has three chunks in flight (1000 of 100003: 73 and 84 us).
int row_warps(const cfgzip_ctx* ctx, int32_t N, int32_t V, bool f32, bool masked) {
    if (N <= 4 * ctx->sm_count) return 8;
    if (N > 8 * ctx->sm_count && V <= 64 * kLogprobsChunk) return 2;
    return f32 && masked ? 8 : 4;
}

template <int WARPS>
int run_logprobs(cfgzip_ctx* ctx, const LogprobsArgs& a, int dtype, int blocks, cudaStream_t st) {
    auto kern = dtype == CFGZIP_BF16 ? (a.mask ? k_token_logprobs<kBF16, true, WARPS> : k_token_logprobs<kBF16, false, WARPS>)
                                     : (a.mask ? k_token_logprobs<kF32, true, WARPS> : k_token_logprobs<kF32, false, WARPS>);
    const size_t smem = a.n_top ? size_t(ceil_div(a.V, kLogprobsChunk) + 2) * sizeof(float) : 0;
    int rc = ensure_smem(ctx, kern, smem, true);
    if (rc != CFGZIP_OK) return rc;
    ctx->cluster_now = blocks;
    rc = launch(ctx, kern, dim3(unsigned(a.N) * unsigned(blocks)), dim3(WARPS * 32), smem, st, a, blocks);
    ctx->cluster_now = 1;
    return rc;
}

template <int DT>
auto backward_kernel(bool masked, bool together) {
    if (masked) return together ? k_token_logprobs_backward<DT, true, true> : k_token_logprobs_backward<DT, true, false>;
    return together ? k_token_logprobs_backward<DT, false, true> : k_token_logprobs_backward<DT, false, false>;
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
    a.powers.scale = inv_temperature * kLog2e;
    a.powers.far = kFarPowers / a.powers.scale;
    a.powers.slack = kLogprobsSlack / a.powers.scale;
    a.n_top = n_top;
    a.logp = logp;
    a.entropy = entropy;
    a.lse = lse;
    a.top_tokens = top_tokens;
    a.top_logp = top_logp;
    a.status = ctx->d_status;
    const int blocks = row_blocks(ctx, N, V);
    const int warps = row_warps(ctx, N, V, dtype == CFGZIP_F32, vocab_mask != nullptr);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (warps == 2) return run_logprobs<2>(ctx, a, dtype, blocks, st);
    return warps == 4 ? run_logprobs<4>(ctx, a, dtype, blocks, st) : run_logprobs<8>(ctx, a, dtype, blocks, st);
}

int cfgzip_token_logprobs_backward(cfgzip_ctx* ctx, const void* logits, int dtype, int64_t row_stride_elems, int32_t N, int32_t V,
                                   const uint32_t* vocab_mask, int64_t vocab_stride_words, const int32_t* tokens, float inv_temperature,
                                   const float* lse, const float* entropy, const float* d_logp, const float* d_entropy, void* d_logits,
                                   int64_t d_stride_elems, void* stream) {
    const int rc = check_logits(logits, dtype, row_stride_elems, N, V, vocab_mask, vocab_stride_words, inv_temperature);
    if (rc != CFGZIP_OK) return rc;
    if (N > 0) {
        if (!lse || !d_logits || d_stride_elems < V || (!d_logp && !d_entropy) || (d_logp && !tokens) || (d_entropy && !entropy)) return CFGZIP_E_ARG;
        if (d_logits == logits) return CFGZIP_E_ARG;
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
    a.pieces = ceil_div(V, dtype == CFGZIP_BF16 ? kLogprobsPiece<kBF16> : kLogprobsPiece<kF32>);
    if (int64_t(N) * a.pieces >= (int64_t(1) << 31)) return CFGZIP_E_RANGE;
    // do all rows of the gradient start where those of the logits do, relative to 16 bytes?
    const int64_t size = dtype == CFGZIP_BF16 ? 2 : 4;
    const bool together = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(d_logits)) & 15u) == 0 &&
                          (N == 1 || ((row_stride_elems - d_stride_elems) * size & 15) == 0);
    auto kern = dtype == CFGZIP_BF16 ? backward_kernel<kBF16>(vocab_mask != nullptr, together) : backward_kernel<kF32>(vocab_mask != nullptr, together);
    return launch(ctx, kern, dim3(unsigned(N) * unsigned(a.pieces)), dim3(256), 0, static_cast<cudaStream_t>(stream), a);
}

}  // extern "C"
