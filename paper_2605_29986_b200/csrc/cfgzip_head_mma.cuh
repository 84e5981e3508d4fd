// Products of tall matrices for the head: scores of the loss and its gradient, and the two products of the gradient; also the scores of
// decode steps of many rows. Bound by the tensor cores from some 200 rows on: pairs of blocks (cta_group::2) on tiles of 256 x 256, so
// that each SM reads half of either operand from shared memory, six stages of 64 k, sums of two portions in tensor memory so that one
// is read while the next is made. A gradient of 4096 tokens, 128256 x 4096, takes 9.3 to 10.1 ms, 1270 to 1390 TFLOP/s as power allows
// (cuBLAS: 1380 long, 1620 short), the loss of 8192 6.65 to 6.73 ms, 1280 to 1290.
#pragma once

#include <cuda.h>

#include "cfgzip_activation.cuh"
#include "cfgzip_mma.cuh"

namespace cfgzip {

__device__ __forceinline__ float bf16_f32(uint16_t v) { return __uint_as_float(uint32_t(v) << 16); }
constexpr int kMmaThreads = 384;   // a warp for the copies, one for the products, two idle, two sets of four that read the sums
constexpr int kMmaStages = 6;
constexpr int kMmaTile = 256;      // rows and columns of a pair's tile
constexpr int kMmaK = 64;          // k of a stage
// Stages whose sums are left in tensor memory, where every addition is cut off towards zero (-1e-9 of a sum per element of k); scores
// add the portions up in registers, rounded. Those of the gradient too: what counts of them are differences to an lse that was made of
// the loss's (for which a gradient of 4096 tokens of 128256 x 4096 takes 4 % longer, 9.4 -> 9.8 ms in a row).
constexpr int kMmaPortion = 8;
// ... and the sums over tokens of the gradient, which may be over a whole text or vocabulary (in one go 65536 tokens lose 3e-4 of a sum of
// positive terms, 200003 lose 1.3e-3; in portions of 2048 under 8e-6. 4000 tokens of 8000 x 2048: 108 us for d_weight, in one go 104).
constexpr int kMmaOutPortion = 32;
constexpr int kLayerStagesTall = 5;                      // of the layer's products, whose results need twice the room on their way out
constexpr uint32_t kMmaHalf = 128 * kMmaK * 2;           // bytes of one operand of a stage in one block
constexpr size_t kMmaSmem = size_t(kMmaStages) * 2 * kMmaHalf + 1024;
constexpr uint32_t kMmaOut = 32 * 128;                   // bytes a warp has on their way out: 32 rows of 128

// Kinds of products: scores (of the loss, its gradient, a step, log probabilities, their gradient), sums in 32 bits or bf16, the same where the
// sums of some rows are kept, and (kMmaLayer and the activation) a layer.
enum : int { kMmaLoss = 0, kMmaGrad = 1, kMmaSum = 2, kMmaBf16 = 3, kMmaStep = 4, kMmaLogprobs = 5, kMmaGradEntropy = 6, kMmaSumTargets = 7,
             kMmaBf16Targets = 8, kMmaLayer = 16 };
template <int KIND>
constexpr bool kMmaToBf16 = KIND == kMmaBf16 || KIND == kMmaBf16Targets;
template <int KIND>
constexpr bool kMmaOfSums = kMmaToBf16<KIND> || KIND == kMmaSum || KIND == kMmaSumTargets;

struct MmaArgs {
    int32_t rows, cols;        // of the result (tokens x piece of the vocabulary, ...)
    int32_t width;             // columns of a tile
    int32_t m_tiles, n_tiles;
    int32_t box;               // rows of A, where its k is contiguous, that a block fetches at a time
    int32_t k_blocks, splits;  // the k range is cut in `splits`, each with a result of its own
    int32_t m_fast;            // neighbouring tiles go along m
    int32_t* status;
    int32_t expire;            // test hook: the block reports a wait as run out when the first stages are asked for (see cfgzip_set_tuning)
    // scores
    const uint32_t* mask;
    int64_t mask_stride;
    int32_t t0, V;             // the piece starts at token t0
    const int32_t* targets;
    const float *lse, *d_loss;
    const float *entropy, *d_entropy;  // gradient of log probabilities (whose gradient is in d_loss, null where it is 0) and entropies
    float2* part;              // loss: [2 n_tiles, rows] largest score and sum of half a tile
    float4* sums;              // log probabilities: [2 n_tiles, rows] largest score, sum of the others, of exp(d) d, how many are the largest
    float* of_target;          // loss, log probabilities: [rows]
    Partial* states;           // step: [2 n_tiles, rows] the same with the token
    // results
    void* out;
    int64_t ld;                // elements
    int64_t split_elems;
    int32_t add;
    float* rest;               // gradient of log probabilities: [rows] what the targets' g was rounded by
    const int32_t* first_of;   // sums of targets: [V] the first row with this target; anything where there is none
    int32_t text_rows;         // ... of the text, with their targets
    float* kept;               // ... [rows of the text, cols] the sums of its row of the result, in 32 bits
    // layer
    const void* bias;
    const uint16_t* residual;
    int64_t residual_stride;
    int32_t bias_bf16, has_slope;
};

__device__ __forceinline__ void st_global32(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

// The first row of the text with the token for its target, or -1.
__device__ __forceinline__ int first_row(const MmaArgs& a, int token) {
    const int row = ld_after_wait(a.first_of + token);
    return unsigned(row) < unsigned(a.text_rows) && ld_after_wait(a.targets + row) == token ? row : -1;
}

struct MmaTile {
    int m, n, split, k0, k1;
};
__device__ __forceinline__ MmaTile mma_tile(const MmaArgs& a, int i) {
    const int per = a.m_tiles * a.n_tiles, split = i / per, r = i - split * per;
    MmaTile t;
    t.m = a.m_fast ? r % a.m_tiles : r / a.n_tiles;
    t.n = a.m_fast ? r / a.m_tiles : r % a.n_tiles;
    t.split = split;
    t.k0 = int(int64_t(a.k_blocks) * split / a.splits);
    t.k1 = int(int64_t(a.k_blocks) * (split + 1) / a.splits);
    return t;
}

// What a row allows of the tile's tokens from column n0 of the piece on, up to 32 W, 32 to a word.
template <int W>
__device__ __forceinline__ void tile_mask(const MmaArgs& a, const MmaTile& tile, int row, int n0, uint32_t (&bits)[W]) {
    const int t = a.t0 + n0, left = min(a.cols, (tile.n + 1) * a.width) - n0;
    const uint32_t* p = a.mask + (a.mask ? int64_t(row) * a.mask_stride + (t >> 5) : 0);
#pragma unroll
    for (int c = 0; c < W; ++c) {
        const int n = left - 32 * c;
        uint32_t w = 0;
        if (n > 0) w = (a.mask ? ld_after_wait(p + c) : 0xFFFFFFFFu) & (n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u);
        bits[c] = w;
    }
}

// The score of the row's target, where this half tile has it.
__device__ __forceinline__ void store_of_target(const MmaArgs& a, const MmaTile& t, int half, int row, bool valid, const float (&z)[128]) {
    const int n0 = t.n * a.width + 128 * half, mine = min(128, a.width - 128 * half);
    const int asked = valid ? ld_after_wait(a.targets + row) : -1, there = asked < 0 ? -1 : asked - (a.t0 + n0);
    const int target = there < mine ? there : -1;
    if (__any_sync(0xFFFFFFFFu, target >= 0)) {
#pragma unroll
        for (int j = 0; j < 128; ++j)
            if (target == j) a.of_target[row] = z[j];
    }
}

// Largest allowed score and the sum of exponentials, of one row and half a tile's tokens (the first 128 of them, the rest).
__device__ __forceinline__ void loss_epilogue(const MmaArgs& a, const MmaTile& t, int half, int row, bool valid, float (&z)[128],
                                              const uint32_t (&bits)[4]) {
    store_of_target(a, t, half, row, valid, z);
    float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < 128; ++j) {
        z[j] = (bits[j / 32] >> (j & 31)) & 1u ? z[j] : -INFINITY;
        m[j & 3] = fmaxf(m[j & 3], z[j]);
    }
    const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), ref = fmaxf(top, kRefFloor);
    float s[4] = {};
#pragma unroll
    for (int j = 0; j < 128; ++j) s[j & 3] += ex2f((z[j] - ref) * kLog2e);
    if (valid) a.part[int64_t(2 * t.n + half) * a.rows + row] = make_float2(top, (s[0] + s[1]) + (s[2] + s[3]));
}

__device__ __forceinline__ float is_zero(float x) {  // 1 or 0
    float y;
    asm("set.eq.f32.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sum_of(pair2 x) {
    float a, b;
    unpack2(x, a, b);
    return a + b;
}

// The same with the sum of exp(d) d, d = z - largest, which the entropy is made of; the scores that are the largest are counted apart.
__device__ __forceinline__ void logprobs_epilogue(const MmaArgs& a, const MmaTile& t, int half, int row, bool valid, float (&z)[128],
                                                  const uint32_t (&bits)[4]) {
    store_of_target(a, t, half, row, valid, z);
    float m[4] = {kNone, kNone, kNone, kNone};
#pragma unroll
    for (int j = 0; j < 128; ++j) {
        z[j] = (bits[j / 32] >> (j & 31)) & 1u ? z[j] : kNone;
        m[j & 3] = fmaxf(m[j & 3], z[j]);
    }
    const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), ref = fmaxf(top, kFew);
    pair2 s[2] = {}, d[2] = {}, n[2] = {};
#pragma unroll
    for (int j = 0; j < 128; j += 2) {
        float x0, x1;
        unpack2(add2(pack2(z[j], z[j + 1]), both(-ref)), x0, x1);
        const pair2 x = pack2(fmaxf(x0, 2.f * kNone), fmaxf(x1, 2.f * kNone)), e = ex2_pair(mul2(x, both(kLog2e)));
        const pair2 largest = pack2(is_zero(x0), is_zero(x1));
        n[j >> 1 & 1] = add2(n[j >> 1 & 1], largest);
        s[j >> 1 & 1] = add2(s[j >> 1 & 1], fma2(largest, both(-1.f), e));
        d[j >> 1 & 1] = fma2(e, x, d[j >> 1 & 1]);
    }
    if (valid) a.sums[int64_t(2 * t.n + half) * a.rows + row] = make_float4(ref, sum_of(add2(s[0], s[1])), sum_of(add2(d[0], d[1])), sum_of(add2(n[0], n[1])));
}

// Largest allowed score, its lowest token and the sum of exponentials, of one row and half a tile's tokens.
__device__ __forceinline__ void step_epilogue(const MmaArgs& a, const MmaTile& t, int half, int row, bool valid, float (&z)[128],
                                              const uint32_t (&bits)[4]) {
    float m = -INFINITY;
    int at = kNoPos;
#pragma unroll
    for (int c = 3; c >= 0; --c)
        if (bits[c]) at = 32 * c + __ffs(bits[c]) - 1;  // (scores that are all -inf)
#pragma unroll
    for (int j = 0; j < 128; ++j) {
        z[j] = (bits[j / 32] >> (j & 31)) & 1u ? z[j] : -INFINITY;
        at = z[j] > m ? j : at;
        m = fmaxf(m, z[j]);
    }
    const float ref = fmaxf(m, kRefFloor);
    float s[4] = {};
#pragma unroll
    for (int j = 0; j < 128; ++j) s[j & 3] += ex2f((z[j] - ref) * kLog2e);
    if (valid)
        *reinterpret_cast<int4*>(&a.states[int64_t(2 * t.n + half) * a.rows + row]) =
            make_int4(__float_as_int(m), __float_as_int((s[0] + s[1]) + (s[2] + s[3])),
                      at == kNoPos ? kNoPos : a.t0 + t.n * a.width + 128 * half + at, 0);
}

// g = d (exp(z - lse) - [target]) of the allowed tokens, as bf16, of one row and half a tile's tokens. A target that the model is sure of
// has all of its g in the small difference exp(z - lse) - 1: the scores are made as the loss makes them, portion by portion, so that z
// here is the z in lse to the last bit, and the difference is not taken of a rounded exponential. The only token of a row gets 0.
// With entropies (d is minus the gradient of the log probability then): g = p (d + b (x + entropy)) with x = z - lse and b minus the gradient
// of the entropy, on the target d (p - 1) + p b (x + entropy). The entropy has its gradient in rows without a target too. What the target's g,
// as a rule by far the largest of its row, loses in bf16 is kept, and added to the sums of the two products before they are rounded: of few
// rows, whose targets' roundings do not even out, a gradient would be off by up to 2^-8 of itself more.
template <bool ENTROPY>
__device__ __forceinline__ void grad_epilogue(const MmaArgs& a, const MmaTile& t, int half, int row, bool valid, const float (&z)[128],
                                              const uint32_t (&bits)[4]) {
    const int n0 = t.n * a.width + 128 * half, mine = min(128, a.width - 128 * half);
    int target = -1;
    float d = 0.f, lse = 0.f, b = 0.f, entropy = 0.f;
    bool has = false, any = false;
    if (valid) {
        if (!ENTROPY || a.d_loss) target = ld_after_wait(a.targets + row);
        lse = ld_after_wait(a.lse + row);
        has = target >= 0 && target < a.V && lse > -INFINITY;
        if (has && a.mask) has = (ld_after_wait(a.mask + int64_t(row) * a.mask_stride + (target >> 5)) >> (target & 31)) & 1u;
        if (has) d = ld_after_wait(a.d_loss + row);
        target = has ? target - (a.t0 + n0) : -1;
        if (target >= mine) target = -1;
        any = has;
        if (ENTROPY) {
            d = -d;
            any = lse > -INFINITY;
            lse = any ? lse : 0.f;
            if (a.d_entropy && any) {
                b = -ld_after_wait(a.d_entropy + row);
                entropy = ld_after_wait(a.entropy + row);
            }
        }
    }
    const float at_zero = fmaf(b, entropy, d);
    float of_target = 0.f;
    if (__any_sync(0xFFFFFFFFu, target >= 0)) {
#pragma unroll
        for (int j = 0; j < 128; ++j) of_target = target == j ? z[j] : of_target;
        const float x = of_target - lse;
        of_target = d * expm1f(x);
        if (ENTROPY) {
            of_target = fmaf(ex2f(x * kLog2e) * b, x + entropy, of_target);
            if (target >= 0) a.rest[row] = of_target - __uint_as_float(bf16_pair(0.f, of_target) & 0xFFFF0000u);
        }
    }
    uint16_t* p = static_cast<uint16_t*>(a.out) + int64_t(row) * a.ld + n0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        if (16 * c >= mine || n0 + 16 * c >= a.ld) break;
        const uint32_t w = any ? bits[c / 2] >> (16 * (c & 1)) : 0u;
        float g[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            if (ENTROPY) {
                const float x = fmaxf(z[16 * c + j] - lse, -200.f);
                g[j] = (w >> j) & 1u ? ex2f(x * kLog2e) * fmaf(b, x, at_zero) : 0.f;
            } else {
                g[j] = (w >> j) & 1u ? d * ex2f((z[16 * c + j] - lse) * kLog2e) : 0.f;
            }
            g[j] = target == 16 * c + j ? of_target : g[j];
        }
        uint32_t o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = bf16_pair(g[2 * j], g[2 * j + 1]);
        if (valid) st_global32(p + 16 * c, o);
    }
}

__device__ __forceinline__ void tma_store3(const void* tensor_map, int x, int y, int z, uint32_t src_smem) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];\n\tcp.async.bulk.commit_group;" ::"l"(tensor_map),
                 "r"(x), "r"(y), "r"(z), "r"(src_smem)
                 : "memory");
}

// Sums as they are (f32), or rounded to bf16; added to what is there where asked for. Rows start on 16 bytes, columns come in
// multiples of 8. A warp's 32 rows go out 128 bytes at a time by a tiled copy from shared memory, which leaves out what is behind the
// last row or column: sums of few stages wait for nothing but their stores, and stored by lanes, a row each, they took twice as
// long (gradient of 50021 x 1024 for 100 tokens: 50 us).
template <bool BF16>
constexpr int kOutCols = BF16 ? 64 : 32;  // columns in 128 bytes
template <bool BF16, bool TARGETS>
__device__ __forceinline__ void out_columns(const MmaArgs& a, const CUtensorMap& map, const MmaTile& t, int n, int first, int lane, bool add,
                                            int chain, float* f, uint32_t buffer) {
    constexpr int kCols = kOutCols<BF16>;
    if (add) {
        const char* from = static_cast<const char*>(a.out) + (t.split * a.split_elems + int64_t(first + lane) * a.ld + n) * (BF16 ? 2 : 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (n + j * kCols / 8 >= a.cols) break;
            const uint4 b = ld_after_wait(reinterpret_cast<const uint4*>(from + 16 * j));
            const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int k = 0; k < kCols / 8; ++k)
                f[j * kCols / 8 + k] += __uint_as_float(BF16 ? (k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16) : w[k & 3]);
        }
    }
    if (TARGETS && chain >= 0) {  // (a row of some row's target: its sums once more, as they are)
        float* p = a.kept + int64_t(chain) * a.cols + n;
#pragma unroll
        for (int j = 0; j < kCols / 4; ++j)
            if (n + 4 * j < a.cols) *reinterpret_cast<float4*>(p + 4 * j) = make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
    }
    uint32_t o[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) o[j] = BF16 ? bf16_pair(f[2 * j % kCols], f[(2 * j + 1) % kCols]) : __float_as_uint(f[j % kCols]);
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // (the copy before has read the buffer)
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buffer + uint32_t(lane) * 128 + (uint32_t(j ^ (lane & 7)) << 4)),
                     "r"(o[4 * j]), "r"(o[4 * j + 1]), "r"(o[4 * j + 2]), "r"(o[4 * j + 3])
                     : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) tma_store3(&map, n, first, t.split, buffer);
}

// What a warp's next 64 columns need besides the sums, asked for ahead: two biases of a lane, and the residual, a row's 128 bytes by eight lanes
// (by one lane, 16 bytes at a time, the loads of a warp touch 32 lines each).
struct LayerAhead {
    uint32_t bias[2];  // (bf16 ones as they are stored: put in place here, each load would be waited for)
    uint4 residual[8];
    __device__ __forceinline__ void ask_bias(const MmaArgs& a, int n, int end, int lane) {
        if (!a.bias || n >= end) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) bias[h] = n + 32 * h + lane < a.cols ? bias_bits(a.bias, a.bias_bf16, n + 32 * h + lane) : 0u;
    }
    __device__ __forceinline__ void ask_residual(const MmaArgs& a, int first, int n, int end, int lane) {
        if (!a.residual || n >= end) return;
        const int col = n + 8 * (lane & 7);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = first + 4 * j + (lane >> 3);
            residual[j] = make_uint4(0, 0, 0, 0);
            if (row < a.rows && col < a.cols)
                residual[j] = ld_after_wait(reinterpret_cast<const uint4*>(a.residual + int64_t(row) * a.residual_stride + col));
        }
    }
};

// A layer's results, 64 columns of a warp's 32 rows at a time, straight from tensor memory. y and the activation's derivative leave by tiled
// copies from a buffer each; without a derivative y takes the two in turn. The residual comes to its lanes by way of y's place. A bias, the same
// for all lanes, is in 32 floats of shared memory (loaded by all lanes from the L1 it took 10 us of 40).
template <int ACT, bool SLOPE>
__device__ __forceinline__ void layer_columns(const MmaArgs& a, const CUtensorMap& map_y, const CUtensorMap& map_slope, int n, int first,
                                              int lane, uint32_t tmem, uint32_t buffer, float* table, LayerAhead& ahead, int end) {
    const uint32_t row = buffer + uint32_t(lane) * 128, turn = uint32_t(lane & 7);
    // (32 columns at a time: all loads, then all arithmetic, so that its chains run side by side, then all stores)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t v[32], y[16], s[16];
        tmem_ld32(tmem + 32 * h, v);
        if (h == 0) {
            if (lane == 0) {  // (the copies before have read the buffer)
                if (SLOPE)
                    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                else
                    asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            }
            __syncwarp();
            if (a.residual) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t r = uint32_t(4 * j + (lane >> 3));
                    st_shared16(buffer + r * 128 + ((turn ^ (r & 7u)) << 4), ahead.residual[j]);
                }
            }
            ahead.ask_residual(a, first, n + 64, end, lane);
        }
        if (a.bias) table[lane] = __uint_as_float(ahead.bias[h] << (a.bias_bf16 ? 16 : 0));
        if (h == 1) ahead.ask_bias(a, n + 64, end, lane);
        __syncwarp();
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t at = row + ((uint32_t(4 * h + j) ^ turn) << 4);
            pair2 of[4] = {}, bias[4] = {};
            if (a.residual) bf16_pairs(ld_shared16(at), of);
            if (a.bias) {
                const ulonglong2 lo = *reinterpret_cast<const ulonglong2*>(table + 8 * j), hi = *reinterpret_cast<const ulonglong2*>(table + 8 * j + 4);
                bias[0] = lo.x; bias[1] = lo.y; bias[2] = hi.x; bias[3] = hi.y;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                pair2 by;
                const pair2 of_h = activation<ACT>(add2(pack2(__uint_as_float(v[8 * j + 2 * k]), __uint_as_float(v[8 * j + 2 * k + 1])), bias[k]), &by);
                float f0, f1;
                unpack2(add2(of_h, of[k]), f0, f1);
                y[4 * j + k] = bf16_pair(f0, f1);
                if (SLOPE) {
                    unpack2(by, f0, f1);
                    s[4 * j + k] = bf16_pair(f0, f1);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t at = row + ((uint32_t(4 * h + j) ^ turn) << 4);
            st_shared16(at, make_uint4(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]));
            if (SLOPE) st_shared16(at + kMmaOut, make_uint4(s[4 * j], s[4 * j + 1], s[4 * j + 2], s[4 * j + 3]));
        }
        if (h == 0) __syncwarp();  // (the biases have been read)
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        tma_store3(&map_y, n, first, 0, buffer);
        if (SLOPE) tma_store3(&map_slope, n, first, 0, buffer + kMmaOut);
    }
}

// D[rows, cols] = A B^T in tiles of 256 x width by pairs of blocks (each holds 128 rows of A and half of B's, and the sums of its 128
// rows), persistent. Operands K-major (k contiguous) or MN-major, from tensor maps with boxes of 64 x 128 (x width / 2) or 64 x 64;
// an MN-major B and results that go out by tiled copies have a width of 256.
//
// Sums are read portion by portion by both sets of warps, a half of the columns each, and added up in registers. Where no tile's sum
// has more than one portion (LONG false), and what takes the time is the results' way out, the sets take tiles in turn instead, straight
// from tensor memory (100 tokens of 50021 x 1024: 26 us for d_weight against 38).
//
// A layer's sums stay in tensor memory to their end: their results are bf16, and what is cut off (1e-9 of a sum per element of k) is far
// below that. (8192 rows of 4096 -> 4096 with bias, residual and derivative: 180 to 227 us, 1.2 to 1.5 PFLOP/s by the power limit; of
// 512 -> 4096 50 without a derivative, bound by what is done with the sums.)
template <bool A_MN, bool B_MN, int KIND, bool LONG>
__device__ __forceinline__ void mma_products(const MmaArgs& a, const CUtensorMap& map_a, const CUtensorMap& map_b, const CUtensorMap& map_out,
                                             const CUtensorMap& map_slope) {
    constexpr bool kLayer = KIND >= kMmaLayer;
    constexpr int kStages = kLayer ? kLayerStagesTall : kMmaStages;
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages], sums_full[2], sums_empty[2];
    __shared__ __align__(8) uint64_t drained;
    __shared__ __align__(16) float s_bias[kLayer ? 8 : 1][32];
    __shared__ uint32_t s_tmem, s_end[2];  // (of either block: the stages it has asked for, and in the highest bit whether a wait ran out)
    constexpr bool kOut = kMmaOfSums<KIND>, kTargets = KIND == kMmaSumTargets || KIND == kMmaBf16Targets;
    constexpr int kPortion = kLayer ? 1 << 30 : kOut ? kMmaOutPortion : kMmaPortion;
    constexpr bool kTurns = !LONG;
    static_assert(kOut || kLayer || LONG, "scores are summed in portions");
    const uint32_t stages = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int tiles = a.m_tiles * a.n_tiles * a.splits, pairs = gridDim.x / 2, pair = blockIdx.x / 2;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sums_full[i], 1);
            mbar_init(&sums_empty[i], kTurns ? 8 : 16);  // four warps of either block (all eight)
        }
        mbar_init(&drained, 1);
        mbar_init_fence();
        prefetch_tensor_map(&map_a);
        prefetch_tensor_map(&map_b);
    }
    if (warp == 2) tmem_alloc<2>(&s_tmem, 512);
    if (!A_MN && !kLayer && a.rows <= 128) {
        // Rows that no copy brings are zeros: whatever stands there would do, but is multiplied at the expense of the clocks (a second of
        // losses of 16 rows of 128256 x 4096: 250 us each instead of 225). It takes each launch 0.2 us.
        for (int i = 0; i < kStages; ++i)
            for (uint32_t at = (rank == 0 ? uint32_t(a.box) * 128 : 0u) + threadIdx.x * 16; at < kMmaHalf; at += blockDim.x * 16)
                st_shared16(stages + uint32_t(i) * 2 * kMmaHalf + at, make_uint4(0, 0, 0, 0));
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    tmem_fence_before();
    __syncthreads();
    cluster_barrier();
    tmem_fence_after();
    if (kLayer) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t tmem = s_tmem;
    bool ok = warp == 0 || !a.expire;  // (the hook: nothing is done with the first stages asked for)
    uint32_t asked = 0;
    if (warp == 0) {
        if (lane == 0) {
            Ring r;
            for (int i = pair; i < tiles && ok; i += pairs) {
                const MmaTile t = mma_tile(a, i);
                const int m = t.m * kMmaTile + int(rank) * 128, n = t.n * a.width + int(rank) * (a.width / 2);
                const int k1 = a.expire ? min(t.k1, t.k0 + kStages) : t.k1;
                const bool first_only = !A_MN && a.rows <= 128, with_a = !first_only || rank == 0;
                const uint32_t bytes = (A_MN ? 2 * kMmaHalf : uint32_t(a.box) * (first_only ? 1 : 2) * kMmaK * 2) + uint32_t(a.width) * kMmaK * 2;
                for (int k = t.k0; k < k1; ++k) {
                    if (!ring_wait<true>(&empty[r.stage], r.phase ^ 1)) {
                        ok = false;
                        break;
                    }
                    if (rank == 0) mbar_expect_tx(&full[r.stage], bytes);
                    const uint32_t bar = peer_shared(&full[r.stage], 0), at = stages + uint32_t(r.stage) * 2 * kMmaHalf;
                    if (A_MN) {
                        tma_load_pair(at, &map_a, m, k * kMmaK, bar);
                        tma_load_pair(at + kMmaHalf / 2, &map_a, m + 64, k * kMmaK, bar);
                    } else {
                        tma_load_pair_if(with_a, at, &map_a, k * kMmaK, m, bar);
                    }
                    if (B_MN) {
                        tma_load_pair(at + kMmaHalf, &map_b, n, k * kMmaK, bar);
                        tma_load_pair(at + kMmaHalf + kMmaHalf / 2, &map_b, n + 64, k * kMmaK, bar);
                    } else {
                        tma_load_pair(at + kMmaHalf, &map_b, k * kMmaK, n, bar);
                    }
                    ++asked;
                    r.next<kStages>();
                }
                if (a.expire) ok = false;
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t idesc = kMmaBf16Desc<256, 0, A_MN, B_MN> | uint32_t(a.width / 8) << 17;
            Ring r;
            int it = 0;
            for (int i = pair; i < tiles && ok; i += pairs) {
                const MmaTile t = mma_tile(a, i);
                for (int k = t.k0; k < t.k1 && ok; ++it) {
                    const uint32_t d = tmem + (it & 1) * 256;
                    const int first = k, last = min(k + kPortion, t.k1);
                    if (!ring_wait<true>(&sums_empty[it & 1], ((it >> 1) & 1) ^ 1)) {
                        ok = false;
                        break;
                    }
                    tmem_fence_after();
                    for (; k < last; ++k) {
                        if (!ring_wait<true>(&full[r.stage], r.phase)) {
                            ok = false;
                            break;
                        }
                        tmem_fence_after();
                        const uint32_t at = stages + uint32_t(r.stage) * 2 * kMmaHalf;
                        const uint64_t da = mma_desc<A_MN>(at), db = mma_desc<B_MN>(at + kMmaHalf);
                        if (elect_one()) {
#pragma unroll
                            for (int j = 0; j < kMmaK / 16; ++j)
                                mma_f16<2>(d, da + j * kDescStep16<A_MN>, db + j * kDescStep16<B_MN>, idesc, k > first || j > 0);
                            mma_commit<2>(&empty[r.stage]);
                        }
                        __syncwarp();
                        r.next<kStages>();
                    }
                    if (elect_one()) mma_commit<2>(&sums_full[it & 1]);
                    __syncwarp();
                }
            }
        }
    } else if (warp >= 4 && !kTurns) {
        const int half = (warp - 4) >> 2, quad = warp & 3;
        const uint32_t empty_bar[2] = {peer_shared(&sums_empty[0], 0), peer_shared(&sums_empty[1], 0)};
        int it = 0;
        for (int i = pair; i < tiles && ok; i += pairs) {
            const MmaTile t = mma_tile(a, i);
            const int row = t.m * kMmaTile + int(rank) * 128 + quad * 32 + lane;
            const bool valid = row < a.rows;
            uint32_t bits[4];
            if (!kOut) tile_mask(a, t, valid ? row : a.rows - 1, t.n * a.width + 128 * half, bits);
            const int chain = kTargets && valid ? first_row(a, a.t0 + row) : -1;
            float sums[128] = {};
            for (int k = t.k0; k < t.k1; k += kPortion, ++it) {
                if (!ring_wait<true>(&sums_full[it & 1], (it >> 1) & 1)) {
                    ok = false;
                    break;
                }
                tmem_fence_after();
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[32];
                    __syncwarp();
                    tmem_ld32(tmem + (it & 1) * 256 + 128 * half + 32 * c + (uint32_t(quad * 32) << 16), v);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j) sums[32 * c + j] += __uint_as_float(v[j]);
                }
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at_peer(empty_bar[it & 1]);
            }
            if (ok && KIND == kMmaLoss) loss_epilogue(a, t, half, row, valid, sums, bits);
            if (ok && KIND == kMmaStep) step_epilogue(a, t, half, row, valid, sums, bits);
            if (ok && KIND == kMmaLogprobs) logprobs_epilogue(a, t, half, row, valid, sums, bits);
            if (ok && KIND == kMmaGrad) grad_epilogue<false>(a, t, half, row, valid, sums, bits);
            if (ok && KIND == kMmaGradEntropy) grad_epilogue<true>(a, t, half, row, valid, sums, bits);
            if (ok && kOut && row - lane < a.rows) {
                const bool add = a.add && valid;
                constexpr int kCols = kOutCols<kMmaToBf16<KIND>>;
#pragma unroll
                for (int c = 0; c < 128 / kCols; ++c) {
                    const int n = t.n * kMmaTile + 128 * half + kCols * c;
                    if (n >= a.cols) break;
                    out_columns<kMmaToBf16<KIND>, kTargets>(a, map_out, t, n, row - lane, lane, add, chain, sums + kCols * c,
                                                  stages + kStages * 2 * kMmaHalf + uint32_t(warp - 4) * kMmaOut);
                }
            }
        }
        if (kOut && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else if (warp >= 4) {
        const int set = (warp - 4) >> 2, quad = warp & 3;
        const uint32_t empty_bar = peer_shared(&sums_empty[set], 0);
        int it = 0;
        uint32_t turn = 0;
        for (int i = pair; i < tiles && ok; i += pairs, ++it) {
            // (a layer's last tile of a pair is shared: nothing else is left to do meanwhile)
            const bool shared = kLayer && i + pairs >= tiles;
            if ((it & 1) != set && !shared) continue;
            const MmaTile t = mma_tile(a, i);
            const int first = t.m * kMmaTile + int(rank) * 128 + quad * 32;
            const int c0 = shared ? set * 128 : 0, c1 = shared ? c0 + 128 : kMmaTile;
            LayerAhead ahead;
            const int n0 = t.n * kMmaTile + c0, end = min(a.cols, t.n * kMmaTile + c1);
            if constexpr (kLayer) {
                ahead.ask_bias(a, n0, end, lane);
                ahead.ask_residual(a, first, n0, end, lane);
            }
            const int chain = kTargets && first + lane < a.rows ? first_row(a, a.t0 + first + lane) : -1;
            if (!ring_wait<true>(&sums_full[kLayer ? it & 1 : set], (it >> 1) & 1)) {
                ok = false;
                break;
            }
            tmem_fence_after();
            if constexpr (kLayer) {
                constexpr int kAct = KIND - kMmaLayer;
                const uint32_t of_warp = stages + kStages * 2 * kMmaHalf + uint32_t(warp - 4) * (2 * kMmaOut);
#pragma unroll 1
                for (int c = c0, n = n0; n < end && first < a.rows; c += 64, n += 64) {
                    const uint32_t from = tmem + (it & 1) * 256 + c + (uint32_t(quad * 32) << 16);
                    if (kAct != kActNone && a.has_slope) {
                        layer_columns<kAct, true>(a, map_out, map_slope, n, first, lane, from, of_warp, s_bias[warp - 4], ahead, end);
                    } else {
                        layer_columns<kAct, false>(a, map_out, map_slope, n, first, lane, from, of_warp + turn, s_bias[warp - 4], ahead, end);
                        turn ^= kMmaOut;
                    }
                }
            } else {
                const bool add = a.add && first + lane < a.rows;
                constexpr int kCols = kOutCols<kMmaToBf16<KIND>>;
#pragma unroll 1
                for (int n = t.n * kMmaTile, c = 0; c < kMmaTile && n < a.cols && first < a.rows; c += kCols, n += kCols) {
                    float f[kCols];
#pragma unroll
                    for (int h = 0; h < kCols; h += 32) {
                        uint32_t v[32];
                        __syncwarp();
                        tmem_ld32(tmem + set * 256 + c + h + (uint32_t(quad * 32) << 16), v);
                        tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 32; ++j) f[h + j] = __uint_as_float(v[j]);
                    }
                    out_columns<kMmaToBf16<KIND>, kTargets>(a, map_out, t, n, first, lane, add, chain, f, stages + kStages * 2 * kMmaHalf + uint32_t(warp - 4) * kMmaOut);
                }
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0 && !shared) arrive_at_peer(empty_bar);
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    tmem_fence_before();
    const uint32_t failed = __syncthreads_or(!ok) ? 0x80000000u : 0u;
    if (threadIdx.x == 0) {
        s_end[rank] = asked | failed;
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_shared(&s_end[rank], rank ^ 1)), "r"(asked | failed) : "memory");
    }
    __syncwarp();
    cluster_barrier();
    tmem_fence_after();
    if ((s_end[0] | s_end[1]) >> 31) {
        // A wait ran out: the copies that either block has asked for (the first one's barriers count both's) and the products get the same
        // bounded time once more, then the blocks leave without results.
        if (rank == 0 && threadIdx.x == 0) {
            atomicExch(a.status + 3, 1);
            const uint32_t most = max(s_end[0] & 0x7FFFFFFFu, s_end[1] & 0x7FFFFFFFu);
            for (uint32_t i = most - min(most, uint32_t(kStages)); i < most; ++i)
                mbar_wait_cluster(&full[i % kStages], (i / kStages) & 1);
        }
        __syncwarp();
        if (warp == 1) {
            if (rank == 0 && elect_one()) mma_commit<2>(&drained);  // (arrives in both blocks)
            __syncwarp();
            mbar_wait_cluster(&drained, 0);
        }
        __syncwarp();
        __syncthreads();
        cluster_barrier();
    }
    if (warp == 2) tmem_free<2>(tmem, 512);
}

template <bool A_MN, bool B_MN, int KIND, bool LONG>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMmaThreads, 1)
    k_head_mma(const __grid_constant__ MmaArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_out) {
    mma_products<A_MN, B_MN, KIND, LONG>(a, map_a, map_b, map_out, map_out);
}

template <bool B_MN, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMmaThreads, 1)
    k_layer_mma(const __grid_constant__ MmaArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_slope) {
    mma_products<false, B_MN, kMmaLayer + ACT, false>(a, map_a, map_b, map_y, map_slope);
}

}  // namespace cfgzip
