// Products of tall matrices for the head: scores of the loss and its gradient, and the two products of the gradient; also the scores of
// decode steps of many rows. Bound by the tensor cores from some 200 rows on: pairs of blocks (cta_group::2) on tiles of 256 x 256, so
// that each SM reads half of either operand from shared memory, six stages of 64 k, sums of two portions in tensor memory so that one
// is read while the next is made. A gradient of 4096 tokens, 128256 x 4096, takes 9.3 to 10.1 ms, 1270 to 1390 TFLOP/s as power allows
// (cuBLAS: 1380 long, 1620 short), the loss of 8192 6.65 to 6.73 ms, 1280 to 1290.
#pragma once

#include <cuda.h>

#include "cfgzip_mma.cuh"
#include "cfgzip_mx.cuh"

namespace cfgzip {

__device__ __forceinline__ float bf16_f32(uint16_t v) { return __uint_as_float(uint32_t(v) << 16); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {  // nearest, ties to even
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

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
constexpr uint32_t kMmaHalf = 128 * kMmaK * 2;           // bytes of one operand of a stage in one block
constexpr size_t kMmaSmem = size_t(kMmaStages) * 2 * kMmaHalf + 1024;
constexpr uint32_t kMmaOut = 32 * 128;                   // bytes a warp has on their way out: 32 rows of 128

enum : int { kMmaLoss = 0, kMmaGrad = 1, kMmaSum = 2, kMmaBf16 = 3, kMmaStep = 4 };

struct MmaArgs {
    int32_t rows, cols;        // of the result (tokens x piece of the vocabulary, ...)
    int32_t width;             // columns of a tile
    int32_t m_tiles, n_tiles;
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
    float2* part;              // loss: [2 n_tiles, rows] largest score and sum of half a tile
    float* of_target;          // loss: [rows]
    Partial* states;           // step: [2 n_tiles, rows] the same with the token
    // results
    void* out;
    int64_t ld;                // elements
    int64_t split_elems;
    int32_t add;
};

__device__ __forceinline__ void st_global32(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
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

// Largest allowed score and the sum of exponentials, of one row and half a tile's tokens (the first 128 of them, the rest).
__device__ __forceinline__ void loss_epilogue(const MmaArgs& a, const MmaTile& t, int half, int row, bool valid, float (&z)[128],
                                              const uint32_t (&bits)[4]) {
    const int n0 = t.n * a.width + 128 * half, mine = min(128, a.width - 128 * half);
    const int asked = valid ? ld_after_wait(a.targets + row) : -1, there = asked < 0 ? -1 : asked - (a.t0 + n0);
    const int target = there < mine ? there : -1;
    if (__any_sync(0xFFFFFFFFu, target >= 0)) {
#pragma unroll
        for (int j = 0; j < 128; ++j)
            if (target == j) a.of_target[row] = z[j];
    }
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
__device__ __forceinline__ void grad_epilogue(const MmaArgs& a, const MmaTile& t, int half, int row, bool valid, const float (&z)[128],
                                              const uint32_t (&bits)[4]) {
    const int n0 = t.n * a.width + 128 * half, mine = min(128, a.width - 128 * half);
    int target = -1;
    float d = 0.f, lse = 0.f;
    bool has = false;
    if (valid) {
        target = ld_after_wait(a.targets + row);
        lse = ld_after_wait(a.lse + row);
        has = target >= 0 && target < a.V && lse > -INFINITY;
        if (has && a.mask) has = (ld_after_wait(a.mask + int64_t(row) * a.mask_stride + (target >> 5)) >> (target & 31)) & 1u;
        if (has) d = ld_after_wait(a.d_loss + row);
        target = has ? target - (a.t0 + n0) : -1;
        if (target >= mine) target = -1;
    }
    float of_target = 0.f;
    if (__any_sync(0xFFFFFFFFu, target >= 0)) {
#pragma unroll
        for (int j = 0; j < 128; ++j) of_target = target == j ? z[j] : of_target;
        of_target = d * expm1f(of_target - lse);
    }
    uint16_t* p = static_cast<uint16_t*>(a.out) + int64_t(row) * a.ld + n0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        if (16 * c >= mine || n0 + 16 * c >= a.ld) break;
        const uint32_t w = has ? bits[c / 2] >> (16 * (c & 1)) : 0u;
        float g[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            g[j] = (w >> j) & 1u ? d * ex2f((z[16 * c + j] - lse) * kLog2e) : 0.f;
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
template <bool BF16>
__device__ __forceinline__ void out_columns(const MmaArgs& a, const CUtensorMap& map, const MmaTile& t, int n, int first, int lane, bool add,
                                            float* f, uint32_t buffer) {
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

// D[rows, cols] = A B^T in tiles of 256 x width by pairs of blocks (each holds 128 rows of A and half of B's, and the sums of its 128
// rows), persistent. Operands K-major (k contiguous) or MN-major, from tensor maps with boxes of 64 x 128 (x width / 2) or 64 x 64;
// an MN-major B and results that go out by tiled copies have a width of 256.
//
// Sums are read portion by portion by both sets of warps, a half of the columns each, and added up in registers. Where no tile's sum
// has more than one portion (LONG false), and what takes the time is the results' way out, the sets take tiles in turn instead, straight
// from tensor memory (100 tokens of 50021 x 1024: 26 us for d_weight against 38).
template <bool A_MN, bool B_MN, int KIND, bool LONG>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMmaThreads, 1)
    k_head_mma(const __grid_constant__ MmaArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_out) {
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t full[kMmaStages], empty[kMmaStages], sums_full[2], sums_empty[2];
    __shared__ __align__(8) uint64_t drained;
    __shared__ uint32_t s_tmem, s_end[2];  // (of either block: the stages it has asked for, and in the highest bit whether a wait ran out)
    constexpr bool kOut = KIND == kMmaSum || KIND == kMmaBf16;
    constexpr int kPortion = kOut ? kMmaOutPortion : kMmaPortion;
    constexpr bool kTurns = !LONG;
    static_assert(kOut || LONG, "scores are summed in portions");
    const uint32_t stages = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int tiles = a.m_tiles * a.n_tiles * a.splits, pairs = gridDim.x / 2, pair = blockIdx.x / 2;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kMmaStages; ++i) {
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
    tmem_fence_before();
    __syncthreads();
    cluster_barrier();
    tmem_fence_after();
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
                const int k1 = a.expire ? min(t.k1, t.k0 + kMmaStages) : t.k1;
                for (int k = t.k0; k < k1; ++k) {
                    if (!ring_wait<true>(&empty[r.stage], r.phase ^ 1)) {
                        ok = false;
                        break;
                    }
                    if (rank == 0) mbar_expect_tx(&full[r.stage], 2 * kMmaHalf + uint32_t(a.width) * kMmaK * 2);
                    const uint32_t bar = peer_shared(&full[r.stage], 0), at = stages + uint32_t(r.stage) * 2 * kMmaHalf;
                    if (A_MN) {
                        tma_load_pair(at, &map_a, m, k * kMmaK, bar);
                        tma_load_pair(at + kMmaHalf / 2, &map_a, m + 64, k * kMmaK, bar);
                    } else {
                        tma_load_pair(at, &map_a, k * kMmaK, m, bar);
                    }
                    if (B_MN) {
                        tma_load_pair(at + kMmaHalf, &map_b, n, k * kMmaK, bar);
                        tma_load_pair(at + kMmaHalf + kMmaHalf / 2, &map_b, n + 64, k * kMmaK, bar);
                    } else {
                        tma_load_pair(at + kMmaHalf, &map_b, k * kMmaK, n, bar);
                    }
                    ++asked;
                    r.next<kMmaStages>();
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
                        r.next<kMmaStages>();
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
            if (ok && KIND == kMmaGrad) grad_epilogue(a, t, half, row, valid, sums, bits);
            if (ok && kOut && row - lane < a.rows) {
                const bool add = a.add && valid;
                constexpr int kCols = kOutCols<KIND == kMmaBf16>;
#pragma unroll
                for (int c = 0; c < 128 / kCols; ++c) {
                    const int n = t.n * kMmaTile + 128 * half + kCols * c;
                    if (n >= a.cols) break;
                    out_columns<KIND == kMmaBf16>(a, map_out, t, n, row - lane, lane, add, sums + kCols * c,
                                                  stages + kMmaStages * 2 * kMmaHalf + uint32_t(warp - 4) * kMmaOut);
                }
            }
        }
        if (kOut && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else if (warp >= 4) {
        const int set = (warp - 4) >> 2, quad = warp & 3;
        const uint32_t empty_bar = peer_shared(&sums_empty[set], 0);
        int it = 0;
        for (int i = pair; i < tiles && ok; i += pairs, ++it) {
            if ((it & 1) != set) continue;
            const MmaTile t = mma_tile(a, i);
            const int first = t.m * kMmaTile + int(rank) * 128 + quad * 32;
            if (!ring_wait<true>(&sums_full[set], (it >> 1) & 1)) {
                ok = false;
                break;
            }
            tmem_fence_after();
            const bool add = a.add && first + lane < a.rows;
            constexpr int kCols = kOutCols<KIND == kMmaBf16>;
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
                out_columns<KIND == kMmaBf16>(a, map_out, t, n, first, lane, add, f, stages + kMmaStages * 2 * kMmaHalf + uint32_t(warp - 4) * kMmaOut);
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at_peer(empty_bar);
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
            for (uint32_t i = most - min(most, uint32_t(kMmaStages)); i < most; ++i)
                mbar_wait_cluster(&full[i % kMmaStages], (i / kMmaStages) & 1);
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

// Partial states of a row's tiles to its results: four rows by a block, a thread takes every 64th tile of one, five at a time.
constexpr int kFinishRows = 4;
struct FinishArgs {
    const float2* part;
    const float* of_target;
    int32_t tiles, rows, V;
    const uint32_t* mask;
    int64_t mask_stride;
    const int32_t* targets;
    float *loss, *lse;
    int32_t* status;
};
__global__ void __launch_bounds__(256) k_head_loss_finish(const FinishArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x * kFinishRows + (lane & 3);
    float m = -INFINITY, s = 0.f;
    // (what the end needs is asked for before the states: the target's score is there or is not looked at)
    const bool ends = warp == 0 && lane < kFinishRows && row < a.rows;
    const int target = ends ? ld_after_wait(a.targets + row) : -1;
    const float of_target = ends ? ld_after_wait(a.of_target + row) : 0.f;
    if (row < a.rows)
        for (int t = warp * 8 + (lane >> 2); t < a.tiles; t += 320) {
            float2 p[5];
#pragma unroll
            for (int k = 0; k < 5; ++k)
                p[k] = t + 64 * k < a.tiles ? __ldcg(a.part + int64_t(t + 64 * k) * a.rows + row) : make_float2(-INFINITY, 0.f);
            float next = m;
#pragma unroll
            for (int k = 0; k < 5; ++k) next = fmaxf(next, p[k].x);
            const float ref = fmaxf(next, kRefFloor);
            s *= ex2f((fmaxf(m, kRefFloor) - ref) * kLog2e);
#pragma unroll
            for (int k = 0; k < 5; ++k) s += p[k].y * ex2f((fmaxf(p[k].x, kRefFloor) - ref) * kLog2e);
            m = next;
        }
    bool has = target >= 0 && target < a.V;
    if (has && a.mask) has = (ld_after_wait(a.mask + int64_t(row) * a.mask_stride + (target >> 5)) >> (target & 31)) & 1u;
    __shared__ float2 sh[64][kFinishRows];
    sh[warp * 8 + (lane >> 2)][lane & 3] = make_float2(m, s);
    __syncthreads();
    if (warp) return;
    // eight threads a row, eight states each
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 8; ++w) top = fmaxf(top, sh[8 * (lane >> 2) + w][lane & 3].x);
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
    const float ref = fmaxf(top, kRefFloor);
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        const float2 p = sh[8 * (lane >> 2) + w][lane & 3];
        s += p.y * ex2f((fmaxf(p.x, kRefFloor) - ref) * kLog2e);
    }
    s += __shfl_xor_sync(0xFFFFFFFFu, s, 4);
    s += __shfl_xor_sync(0xFFFFFFFFu, s, 8);
    s += __shfl_xor_sync(0xFFFFFFFFu, s, 16);
    if (!ends) return;
    const float log_sum = logf(s);
    if (a.lse) a.lse[row] = s > 0.f ? top + log_sum : -INFINITY;
    if (target >= a.V) atomicAdd(a.status + 1, 1);
    float loss = 0.f;
    if (target >= 0) loss = has && of_target > -INFINITY ? (top - of_target) + log_sum : INFINITY;
    a.loss[row] = loss;
}

// The sums of `splits` cuts, added up and rounded; four to a thread, n a multiple of 8. (Few rows have many cuts: what takes time is
// how many loads a thread waits for, one after the other. 500 x 256 from 37 cuts: 18 us with eight to a thread, four at a time.)
__global__ void __launch_bounds__(256) k_head_round(const float* from, int64_t split_elems, int splits, uint16_t* to, int64_t to_stride,
                                                    int rows, int n) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int vectors = n / 4;
    const int64_t total = int64_t(rows) * vectors;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
        float f[4] = {};
#pragma unroll 8
        for (int s = 0; s < splits; ++s) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(from + s * split_elems + 4 * i));
            f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
        }
        const int64_t row = i / vectors;
        *reinterpret_cast<uint2*>(to + row * to_stride + 4 * (i - row * vectors)) = make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]));
    }
}

}  // namespace cfgzip
