// The layer in front of a head, y = residual + act(x W^T + b): products of few rows, the gradient in front of the activation, and sums over
// rows. Products of many rows are the tall ones (cfgzip_head_mma.cuh).
#pragma once

#include <cuda.h>

#include "cfgzip_activation.cuh"
#include "cfgzip_mma.cuh"

namespace cfgzip {

struct LayerArgs {
    int32_t rows, features;     // of the result
    int32_t N;                  // rows of a tile: a multiple of 16, at most 256
    int32_t k_blocks, stages;
    uint32_t stage_bytes;
    int32_t bias_bf16;
    const void* bias;
    const uint16_t* residual;
    int64_t residual_stride;
    uint16_t* y;
    int64_t y_stride;
    uint16_t* slope;
    int64_t slope_stride;
    int32_t* status;
    int32_t expire;             // test hook (see cfgzip_set_tuning)
};

constexpr int kLayerThreads = 256;
constexpr int kLayerStages = 12;                    // at most
constexpr int kLayerBlocks = 8;                     // blocks of a cluster at most
constexpr uint32_t kLayerWeights = 128 * 64 * 2;    // bytes of weights in a stage

// Where the sums of a row's 128 features lie in shared memory: the first four of every eight side by side, the others behind them, so that 16
// lanes that take eight each read 256 bytes at a time, and 32 that write one each write to all banks.
constexpr int kLayerRow = 144;
__device__ __forceinline__ int layer_place(int feature) { return (feature >> 3) * 4 + (feature & 3) + (feature & 4 ? 80 : 0); }

// Eight features of a row: the sum, by way of the epilogue, to where it goes.
template <int ACT>
__device__ __forceinline__ void layer_finish(const LayerArgs& a, int row, int n, float (&f)[8], const float (&bias)[8], const float (&residual)[8]) {
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        pair2 by;
        const pair2 of_h = activation<ACT>(add2(pack2(f[j], f[j + 1]), pack2(bias[j], bias[j + 1])), &by);
        unpack2(add2(of_h, pack2(residual[j], residual[j + 1])), f[j], f[j + 1]);
        unpack2(by, s[j], s[j + 1]);
    }
    *reinterpret_cast<uint4*>(a.y + int64_t(row) * a.y_stride + n) =
        make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
    if (a.slope)
        *reinterpret_cast<uint4*>(a.slope + int64_t(row) * a.slope_stride + n) =
            make_uint4(bf16_pair(s[0], s[1]), bf16_pair(s[2], s[3]), bf16_pair(s[4], s[5]), bf16_pair(s[6], s[7]));
}

// The results of a thread from its block's share of rows, `first`, `first` + `step` and so on of the tile: eight features of each, features n on
// of the result. The sums of up to BLOCKS blocks are added up, ROWS rows' loads in flight; each block begins with its own sums and goes round
// (all at the same block's, they would get an eighth of its speed each). `next` holds the next rows' residuals, asked for ahead.
constexpr int kLayerAhead = 4;
template <int ACT, int BLOCKS, int ROWS, typename Ask>
__device__ __forceinline__ void layer_rows(const LayerArgs& a, const float* part, int row0, int rows, int first, int step, int n, int blocks,
                                           int rank, const float (&bias)[8], uint4 (&next)[kLayerAhead], const Ask& ask) {
#pragma unroll 1
    for (int at = first; at < rows; at += kLayerAhead * step) {
#pragma unroll
        for (int r0 = 0; r0 < kLayerAhead; r0 += ROWS) {
            if (at + r0 * step >= rows) break;
            uint4 v[ROWS][BLOCKS][2];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int row = min(at + (r0 + r) * step, rows - 1);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
                    if (b < blocks) {
                        const uint32_t from = peer_shared(part + row * kLayerRow, uint32_t(rank + b < blocks ? rank + b : rank + b - blocks));
                        v[r][b][0] = ld_peer_v4(from);
                        v[r][b][1] = ld_peer_v4(from + 80 * sizeof(float));
                    }
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int row = at + (r0 + r) * step;
                if (row >= rows) break;
                float f[8] = {}, residual[8];
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
                    if (b < blocks) {
                        const uint32_t w[8] = {v[r][b][0].x, v[r][b][0].y, v[r][b][0].z, v[r][b][0].w,
                                               v[r][b][1].x, v[r][b][1].y, v[r][b][1].z, v[r][b][1].w};
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] += __uint_as_float(w[j]);
                    }
                bf16_values(next[r0 + r], residual);
                next[r0 + r] = ask(row + kLayerAhead * step);
                layer_finish<ACT>(a, row0 + row, n, f, bias, residual);
            }
        }
    }
}

// Few rows: what counts is reading the weights at the speed of memory, on as many SMs as there are. A cluster of up to 8 blocks shares a
// tile of 128 features and N rows, a part of k each; weights are the long side (operand A, 128 rows to a product), the rows the short one.
// The parts meet in the blocks' shared memory: each block adds up a share of the results over the cluster and finishes it.
//
// Sums stay in tensor memory over all of a block's k: what its additions cut off (1e-9 of the sum per element) is far below the rounding
// of the result to bf16.
//
// Bound by latency (one row of 2048 x 2048: 4.7 us), then by the weights' way from memory (32 rows of 4096 x 4096: 8.4 to 10.5 us, 3.2 to
// 4 TB/s).
template <bool A_MN, int ACT>
__global__ void __launch_bounds__(kLayerThreads, 2)
    k_layer_few(const __grid_constant__ LayerArgs a, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x) {
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t full[kLayerStages], empty[kLayerStages], done, drained;
    __shared__ uint32_t s_tmem;
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    char* const base = smem_raw + (smem - smem_u32(smem_raw));
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const int blocks = int(cluster_blocks()), rank = int(cluster_rank());
    const int n0 = int(blockIdx.x) / blocks * 128, row0 = int(blockIdx.y) * a.N, rows = min(a.N, a.rows - row0);
    const int k0 = int(int64_t(a.k_blocks) * rank / blocks), k1 = int(int64_t(a.k_blocks) * (rank + 1) / blocks);
    const uint32_t columns = a.N <= 32 ? 32u : a.N <= 64 ? 64u : a.N <= 128 ? 128u : 256u;
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(&done, 1);
        mbar_init(&drained, 1);
        mbar_init_fence();
        prefetch_tensor_map(&map_w);
        prefetch_tensor_map(&map_x);
    }
    if (warp == 2) tmem_alloc<1>(&s_tmem, columns);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t tmem = s_tmem;
    bool ok = warp == 0 || !a.expire;  // (the hook: nothing is done with the first stages asked for)
    int asked = 0;

    // This thread's results: eight features each, always the same ones, of every 16 * blocks-th row. What the next ones need besides the sums
    // is asked for ahead.
    const int first = (int(threadIdx.x) >> 4) * blocks + rank, step = blocks * (kLayerThreads / 16);
    const int n = n0 + 8 * (int(threadIdx.x) & 15);
    const bool mine = n < a.features;
    float bias[8] = {};
    uint4 next[kLayerAhead];
    auto ask = [&](int row) {
        return a.residual && mine && row < rows ? ld_after_wait(reinterpret_cast<const uint4*>(a.residual + int64_t(row0 + row) * a.residual_stride + n))
                                                : make_uint4(0, 0, 0, 0);
    };

    if (warp == 0) {
        if (lane == 0) {
            Ring r;
            const int last = a.expire ? min(k1, k0 + a.stages) : k1;
            for (int k = k0; k < last; ++k) {
                if (!ring_wait(&empty[r.stage], r.phase ^ 1)) {
                    ok = false;
                    break;
                }
                char* const to = base + uint32_t(r.stage) * a.stage_bytes;
                mbar_expect_tx(&full[r.stage], kLayerWeights + uint32_t(a.N) * 128u);
                if (A_MN) {
                    tma_g2s_2d(to, &map_w, n0, k * 64, &full[r.stage]);
                    tma_g2s_2d(to + kLayerWeights / 2, &map_w, n0 + 64, k * 64, &full[r.stage]);
                } else {
                    tma_g2s_2d(to, &map_w, k * 64, n0, &full[r.stage]);
                }
                tma_g2s_2d(to + kLayerWeights, &map_x, k * 64, row0, &full[r.stage]);
                ++asked;
                if (++r.stage == a.stages) {
                    r.stage = 0;
                    r.phase ^= 1;
                }
            }
            if (a.expire) ok = false;
        }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t idesc = kMmaBf16Desc<128, 0, A_MN, false> | uint32_t(a.N / 8) << 17;
        Ring r;
        for (int k = k0; k < k1 && ok; ++k) {
            if (!ring_wait(&full[r.stage], r.phase)) {
                ok = false;
                break;
            }
            tmem_fence_after();
            const uint32_t at = smem + uint32_t(r.stage) * a.stage_bytes;
            const uint64_t da = mma_desc<A_MN>(at), db = mma_desc<false>(at + kLayerWeights);
            if (elect_one()) {
#pragma unroll
                for (int j = 0; j < 4; ++j) mma_f16<1>(tmem, da + j * kDescStep16<A_MN>, db + j * kDescStep16<false>, idesc, k > k0 || j > 0);
                mma_commit<1>(&empty[r.stage]);
            }
            __syncwarp();
            if (++r.stage == a.stages) {
                r.stage = 0;
                r.phase ^= 1;
            }
        }
        if (elect_one()) mma_commit<1>(&done);
        __syncwarp();
    }
    if (a.bias && mine && first < rows) bias_values(a.bias, a.bias_bf16, n, bias);
#pragma unroll
    for (int r = 0; r < kLayerAhead; ++r) next[r] = ask(first + r * step);
    if (ok && !ring_wait(&done, 0)) ok = false;
    const bool failed = __syncthreads_or(!ok);
    if (failed) {
        // A wait ran out: the copies asked for and the products get the same bounded time once more; results are undefined.
        if (threadIdx.x == 0) {
            atomicExch(a.status + 3, 1);
            for (int i = asked - min(asked, a.stages); i < asked; ++i) mbar_wait(&full[i % a.stages], uint32_t(i / a.stages) & 1u);
        }
        __syncwarp();
        if (warp == 1) {
            if (elect_one()) mma_commit<1>(&drained);
            __syncwarp();
            mbar_wait(&drained, 0);
        }
        __syncthreads();
    }
    tmem_fence_after();
    // sums to shared memory, a row of features for each of the tile's, over the stages: all copies have landed and all products have read them
    float* const part = reinterpret_cast<float*>(base);
    for (int c = warp >> 2; c * 16 < a.N; c += 2) {
        uint32_t v[16];
        __syncwarp();
        tmem_ld16(tmem + 16 * c + (uint32_t((warp & 3) * 32) << 16), v);
        tmem_wait_ld();
        if (16 * c < rows) {
#pragma unroll
            for (int j = 0; j < 16; ++j) part[(16 * c + j) * kLayerRow + layer_place((warp & 3) * 32 + lane)] = k0 < k1 ? __uint_as_float(v[j]) : 0.f;
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 2) tmem_free<1>(tmem, columns);
    __syncwarp();
    cluster_barrier();
    if (!failed && mine) {
        const float* const mine_of = part + ((n - n0) >> 1);
        if (blocks <= 2) layer_rows<ACT, 2, 4>(a, mine_of, row0, rows, first, step, n, blocks, rank, bias, next, ask);
        else if (blocks <= 4) layer_rows<ACT, 4, 2>(a, mine_of, row0, rows, first, step, n, blocks, rank, bias, next, ask);
        else layer_rows<ACT, kLayerBlocks, 1>(a, mine_of, row0, rows, first, step, n, blocks, rank, bias, next, ask);
    }
    __syncwarp();
    cluster_barrier();  // (no block leaves while others read its sums)
}

// The gradient in front of the activation, g = d_y * slope rounded to bf16 (a factor of two products), and the sums over rows that the
// bias's gradient is made of: a block takes 256 columns of a run of rows, a thread eight columns of every eighth row, and leaves one sum
// per column. Up to eight runs are a cluster, whose first block adds its sums up (500 rows of 2568: a launch less, some 3 us). No slope: g is
// d_y and only the sums are made.
constexpr int kGradientCluster = 8;
struct LayerGradientArgs {
    int32_t rows, features, run, runs;  // rows of a block
    const uint16_t* d_y;
    int64_t d_y_stride;
    const uint16_t* slope;
    int64_t slope_stride;
    uint16_t* g;                        // [rows, features], with a slope
    float* sums;                        // [runs, features] of more than a cluster's runs
    float* d_bias;                      // nullable; of a cluster's runs
    int32_t accumulate;
};
__global__ void __launch_bounds__(256) k_layer_gradient(const LayerGradientArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float sh[8][256 + 8];
    __shared__ float s_total[256];
    const int strip = int(blockIdx.x) / a.runs, part = int(blockIdx.x) - strip * a.runs;
    const int col = strip * 256 + int(threadIdx.x & 31) * 8, warp = threadIdx.x >> 5;
    const int r1 = min(a.rows, (part + 1) * a.run);
    float sum[8] = {};
    if (col < a.features) {
        constexpr int kAhead = 4;
        for (int r = part * a.run + warp; r < r1; r += 8 * kAhead) {
            uint4 d[kAhead], s[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                d[k] = make_uint4(0, 0, 0, 0);
                if (r + 8 * k < r1) d[k] = ld_after_wait(reinterpret_cast<const uint4*>(a.d_y + int64_t(r + 8 * k) * a.d_y_stride + col));
            }
            if (a.slope) {
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (r + 8 * k < r1) s[k] = ld_after_wait(reinterpret_cast<const uint4*>(a.slope + int64_t(r + 8 * k) * a.slope_stride + col));
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (r + 8 * k >= r1) break;
                float f[8];
                bf16_values(d[k], f);
                if (a.slope) {
                    float by[8];
                    bf16_values(s[k], by);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] *= by[j];
                    *reinterpret_cast<uint4*>(a.g + int64_t(r + 8 * k) * a.features + col) =
                        make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += f[j];
            }
        }
    }
    if (!a.sums && !a.d_bias) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sh[warp][int(threadIdx.x & 31) * 8 + j] = sum[j];
    __syncthreads();
    const int c = strip * 256 + int(threadIdx.x);
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) total += sh[w][threadIdx.x];
    if (a.sums) {
        if (c < a.features) a.sums[int64_t(part) * a.features + c] = total;
        return;
    }
    s_total[threadIdx.x] = total;
    __syncwarp();
    cluster_barrier();
    if (part == 0 && c < a.features) {
        float other[kGradientCluster];
#pragma unroll
        for (int r = 1; r < kGradientCluster; ++r) other[r] = r < a.runs ? __uint_as_float(ld_peer_u32(peer_shared(s_total + threadIdx.x, uint32_t(r)))) : 0.f;
#pragma unroll
        for (int r = 1; r < kGradientCluster; ++r) total += other[r];
        a.d_bias[c] = a.accumulate ? a.d_bias[c] + total : total;
    }
    __syncwarp();
    cluster_barrier();  // (no block leaves while its sums are read)
}

// The sums of `parts`, added up; to f32, added to what is there where asked for. A block takes 32 columns, a warp every eighth part.
__global__ void __launch_bounds__(256) k_layer_bias(const float* sums, int parts, int features, float* d_bias, int accumulate) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float sh[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = int(blockIdx.x) * 32 + lane;
    float total = 0.f;
    if (c < features) {
#pragma unroll 8
        for (int p = warp; p < parts; p += 8) total += __ldcg(sums + int64_t(p) * features + c);
    }
    sh[warp][lane] = total;
    __syncthreads();
    if (warp || c >= features) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) total += sh[w][lane];
    d_bias[c] = accumulate ? d_bias[c] + total : total;
}

// The sums of a product's cuts, four columns to a thread; to f32 or bf16, added to what is there where asked for. n a multiple of 8.
struct LayerRoundArgs {
    const float* from;
    int64_t split_elems;
    int32_t splits, rows, n;
    void* to;
    int64_t to_stride;
    int32_t bf16, accumulate;
};
__global__ void __launch_bounds__(256) k_layer_round(const LayerRoundArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int vectors = a.n / 4;
    const int64_t total = int64_t(a.rows) * vectors;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / vectors, at = row * a.to_stride + 4 * (i - row * vectors);
        float f[4] = {};
#pragma unroll 8
        for (int s = 0; s < a.splits; ++s) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(a.from + s * a.split_elems + 4 * i));
            f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
        }
        if (a.bf16) {
            uint2* p = reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.to) + at);
            if (a.accumulate) {
                const uint2 b = *p;
                f[0] += __uint_as_float(b.x << 16); f[1] += __uint_as_float(b.x & 0xFFFF0000u);
                f[2] += __uint_as_float(b.y << 16); f[3] += __uint_as_float(b.y & 0xFFFF0000u);
            }
            *p = make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]));
        } else {
            float4* p = reinterpret_cast<float4*>(static_cast<float*>(a.to) + at);
            if (a.accumulate) {
                const float4 b = *p;
                f[0] += b.x; f[1] += b.y; f[2] += b.z; f[3] += b.w;
            }
            *p = make_float4(f[0], f[1], f[2], f[3]);
        }
    }
}

}  // namespace cfgzip
