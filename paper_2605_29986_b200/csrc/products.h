// Host side of the tall products: plans, tensor maps, launches, and workspaces taken apart.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cfgzip.h"
#include "cfgzip_head_mma.cuh"
#include "context.h"

namespace cfgzip {

constexpr int kPairs = 74;  // pairs of SMs that plans are made for (a plan is right for any number)

inline bool on16(const void* p, int64_t stride_bytes) { return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(stride_bytes)) & 15u) == 0; }

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

inline int up(int64_t n, int to) { return int((n + to - 1) / to * to); }

// Cuts of a sum over k_blocks stages whose result has `tiles` tiles: more cuts fill the last wave of pairs better, and each is
// one more f32 result written and read. A stage takes a pair about 0.4 us, a result's bytes 1 / 6.5 us per MB. At most kCutTiles
// tiles in all where there are cuts.
constexpr int kCutTiles = 8 * kPairs;
inline int cuts(int64_t tiles, int k_blocks, int64_t result_elems) {
    int best = 1;
    double least = 0;
    for (int s = 1; s <= kPairs && s <= std::max(1, k_blocks / 16) && (s == 1 || s * tiles <= kCutTiles); ++s) {
        const double waves = double((tiles * s + kPairs - 1) / kPairs);
        const double us = waves * ((k_blocks + s - 1) / s) * 0.4 + s * double(result_elems) * 8e-6 / 6.5;
        if (s == 1 || us < least) {
            least = us;
            best = s;
        }
    }
    return best;
}

// Columns of the tiles of scores: 256, or fewer where the last round of pairs would have few tiles (77 rows of 32000: 125 tiles of 256
// take 74 pairs two rounds, and 143 of 224 as well). What a tile costs besides its columns is taken for 32 of them. From 16 rounds on
// there is nothing to gain.
constexpr int kNarrowest = 160, kNarrowTiles = 16 * kPairs;
inline int tile_width(int64_t rows, int64_t cols) {
    const int64_t high = (rows + kMmaTile - 1) / kMmaTile;
    if (high * ((cols + kMmaTile - 1) / kMmaTile) > kNarrowTiles) return kMmaTile;
    int best = kMmaTile;
    int64_t least = 0;
    for (int w = kMmaTile; w >= kNarrowest; w -= 32) {
        const int64_t tiles = high * ((cols + w - 1) / w), cost = (tiles + kPairs - 1) / kPairs * (w + 32);
        if (w == kMmaTile || cost < least) {
            least = cost;
            best = w;
        }
    }
    return best;
}

// The most states, one for each half tile of a row's scores, that any batch of up to `rows` rows comes to.
inline int64_t most_states(int64_t rows, int64_t cols) {
    const int64_t wide = (cols + kMmaTile - 1) / kMmaTile, narrow = (cols + kNarrowest - 1) / kNarrowest;
    return 2 * std::max(rows * wide, std::min<int64_t>(rows, kMmaTile * (kNarrowTiles / wide)) * narrow);
}

// Tiled copies of a matrix of `rows` rows of `cols` bf16 numbers (or bytes), boxes of 128 bytes by `box` rows in the 128-byte swizzle.
// Where rows start off the 128-byte grid a box's row lies in two lines, and reading 256 bytes ahead costs more than it brings (4096 rows of
// a 4984 -> 4096 layer 156 -> 150 us with 128; 1338 TFLOP/s either way at 4992).
inline int tensor_map(cfgzip_ctx* ctx, CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int64_t stride, int box, bool bytes = false) {
    const cuuint64_t dims[2] = {cuuint64_t(cols), cuuint64_t(rows)};
    const cuuint64_t strides[1] = {cuuint64_t(stride) * (bytes ? 1 : 2)};
    const cuuint32_t boxes[2] = {bytes ? 128u : 64u, cuuint32_t(box)};
    const cuuint32_t steps[2] = {1, 1};
    const CUtensorMapL2promotion ahead = strides[0] % 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_256B;
    if (!ctx->encode_tiled ||
        ctx->encode_tiled(map, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, boxes, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, ahead,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return CFGZIP_E_CUDA;
    return CFGZIP_OK;
}

// Results of a product that go out by tiled copies of 128 bytes of 32 rows.
inline int tensor_map_out(cfgzip_ctx* ctx, CUtensorMap* map, const MmaArgs& a, bool bf16) {
    const cuuint64_t es = bf16 ? 2 : 4;
    const cuuint64_t dims[3] = {cuuint64_t(a.cols), cuuint64_t(a.rows), cuuint64_t(a.splits)};
    const cuuint64_t strides[2] = {cuuint64_t(a.ld) * es, cuuint64_t(a.splits > 1 ? a.split_elems : a.ld) * es};
    const cuuint32_t boxes[3] = {cuuint32_t(128 / es), 32, 1};
    const cuuint32_t steps[3] = {1, 1, 1};
    if (!ctx->encode_tiled ||
        ctx->encode_tiled(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, a.out, dims, strides, boxes, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return CFGZIP_E_CUDA;
    return CFGZIP_OK;
}

// Rows of A, where its k is contiguous, in a block's copies: what lies behind the last one is not asked for (rows outside a map cost the
// copies more than they seem: log probabilities of one row of 32000 x 2048 46 -> 31 us, of 128256 x 4096 221 -> 191).
// (MmaArgs::box, and with it the bytes that a stage waits for, and the map are both made from it.)
inline int a_box(int64_t rows) { return int(std::min<int64_t>(128, up(rows, 8))); }
inline int tensor_map_a(cfgzip_ctx* ctx, CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int64_t stride) {
    return tensor_map(ctx, map, p, rows, cols, stride, a_box(rows));
}

template <bool A_MN, bool B_MN, int KIND, bool LONG = true>
int run_mma(cfgzip_ctx* ctx, MmaArgs& a, const CUtensorMap& map_a, const CUtensorMap& map_b, cudaStream_t st) {
    constexpr bool kOut = kMmaOfSums<KIND>;
    a.splits = std::max(1, a.splits);
    if constexpr (kOut && LONG)
        if (ceil_div(a.k_blocks, a.splits) <= kMmaOutPortion) return run_mma<A_MN, B_MN, KIND, false>(ctx, a, map_a, map_b, st);
    if (kOut) a.width = kMmaTile;
    a.m_tiles = ceil_div(a.rows, kMmaTile);
    a.box = a_box(a.rows);
    a.n_tiles = ceil_div(a.cols, a.width);
    a.status = ctx->d_status;
    a.expire = ctx->expire_test;
    auto kern = k_head_mma<A_MN, B_MN, KIND, LONG>;
    const size_t smem = kMmaSmem + (kOut ? 8 * kMmaOut : 0);
    CUtensorMap map_out = map_a;
    int rc = kOut ? tensor_map_out(ctx, &map_out, a, kMmaToBf16<KIND>) : CFGZIP_OK;
    if (rc != CFGZIP_OK || (rc = ensure_smem(ctx, kern, smem)) != CFGZIP_OK) return rc;
    const int64_t tiles = int64_t(a.m_tiles) * a.n_tiles * a.splits;
    if (tiles >= (int64_t(1) << 30)) return CFGZIP_E_RANGE;
    const unsigned pairs = unsigned(std::min<int64_t>(tiles, ctx->sm_count / 2));
    return launch(ctx, kern, dim3(2 * pairs), dim3(kMmaThreads), smem, st, a, map_a, map_b, map_out);
}

}  // namespace cfgzip
