// The decode step from hidden states. The scores of a batch are a product with one side short (the rows of the batch), so the
// weights are what takes the time, and only those of tokens that some row allows are read: the union of the rows' masks is
// compacted to a list of tokens, every block takes an equal share of it and gathers those rows of the head by tiled copies.
#pragma once

#include <cuda.h>

#include "cfgzip_mma.cuh"
#include "cfgzip_mx.cuh"

namespace cfgzip {

constexpr int kUnionWords = 32;    // mask words (1024 tokens) counted together
constexpr int kStepRows = 128;     // rows of the batch a launch takes at most
constexpr int kStepShare = 2048;   // tokens a block lists at a time
constexpr int kStepThreads = 384;  // copies of hidden states, products, tensor memory, idle, four warps that read the scores, and
                                   // four that fetch the weights
constexpr int kStepTiles = 2;      // tiles of 128 tokens that share a stage, and with it the hidden states in it
constexpr int kStepStages = 8;     // most stages
constexpr int kStepLag = 3;        // stages whose weights are on their way while the next one is asked for
constexpr uint32_t kStepTileBytes = 128 * 64 * 2;

struct HeadStepArgs {
    const PartDev* parts;
    int32_t part0, n_parts;
    const int32_t* row_part;
    const uint32_t* mask;  // [B, mask_stride] vocab masks
    int64_t mask_stride;
    int32_t B, V, VW, H;
    const void* weight;
    int64_t row_bytes;
    int32_t N;             // columns of a tile: B rounded up to 32
    int32_t stages, k_blocks, rounds;
    uint32_t* any;         // [VW] union of the rows' masks
    int32_t* counts;       // tokens of it in every kUnionWords words
    int32_t n_counts;
    uint32_t* ticket;
    Partial* part;         // [blocks, B]
    void* logits;
    int64_t logits_stride;
    int32_t logits_dtype;
    int32_t *argmax, *rep;
    float *logp, *lse;
    int32_t* status;
};

// Partition of a row, -1 where it has none.
__device__ __forceinline__ int step_row_part(const HeadStepArgs& a, int row) {
    if (!a.row_part) return a.part0;
    const int p = ld_after_wait(a.row_part + row);
    return p >= 0 && p < a.n_parts && a.parts[p].live && a.parts[p].V == a.V ? p : -1;
}

// Union of the rows' masks, 32 words by a block: a warp ORs every eighth row.
__global__ void __launch_bounds__(256) k_head_union(const HeadStepArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, word = blockIdx.x * kUnionWords + lane;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
    uint32_t any = 0;
    if (word < a.VW)
#pragma unroll 4
        for (int row = warp; row < a.B; row += 8)
            if (step_row_part(a, row) >= 0) any |= ld_after_wait(a.mask + row * a.mask_stride + word);
    __shared__ uint32_t sh[8][32];
    sh[warp][lane] = any;
    __syncthreads();
    if (warp) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) any |= sh[w][lane];
    if (word < a.VW) a.any[word] = any;
    const int n = __reduce_add_sync(0xFFFFFFFFu, __popc(any));
    if (lane == 0) a.counts[blockIdx.x] = n;
}

// -inf for every score; the allowed ones are written over it.
template <int DT>
__global__ void __launch_bounds__(256) k_head_fill(const HeadStepArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int ES = DT == kBF16 ? 2 : 4, PER = 16 / ES;
    const int row = blockIdx.y;
    if (step_row_part(a, row) < 0) return;
    char* p = static_cast<char*>(a.logits) + row * a.logits_stride * ES;
    const int head = min(int(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / ES), a.V), vectors = (a.V - head) / PER;
    const uint32_t inf = DT == kBF16 ? 0xFF80FF80u : 0xFF800000u;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < vectors; i += gridDim.x * 256)
        *reinterpret_cast<uint4*>(p + (head + i * PER) * int64_t(ES)) = make_uint4(inf, inf, inf, inf);
    if (blockIdx.x == 0) {
        const int tail = a.V - head - vectors * PER;
        if (int(threadIdx.x) < head) store_neg_inf<DT>(p, threadIdx.x);
        if (int(threadIdx.x) < tail) store_neg_inf<DT>(p, a.V - 1 - int(threadIdx.x));
    }
}

// 16 bytes to shared memory past the L1, zeros where they lie behind the row
__device__ __forceinline__ void copy16(uint32_t dst_smem, const void* src, bool have) {
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst_smem), "l"(src), "r"(have ? 16 : 0) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

struct StepShared {
    uint64_t full[kStepStages], empty[kStepStages], sums_full[2], sums_empty[2];
    uint32_t tmem;
    uint32_t valid[kStepRows / 32];  // rows that have a partition
    int32_t total, entries, is_last;
    int32_t scan[kStepThreads / 32];
    int32_t list[kStepShare];        // the block's tokens, ascending
    alignas(16) int2 entry[kStepShare + 1];      // counted pieces that hold some of them: number, tokens in front of it
};

// The block's share of the union: tokens number lo .. lo + n of it, to sh.list. All threads; ends with a barrier.
__device__ __forceinline__ int step_share(const HeadStepArgs& a, StepShared& sh, int share, int shares) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) sh.total = sh.entries = 0;
    __syncthreads();
    int mine = 0;
    for (int i = tid; i < a.n_counts; i += kStepThreads) mine += __ldcg(a.counts + i);
    mine = __reduce_add_sync(0xFFFFFFFFu, mine);
    if (lane == 0 && mine) atomicAdd(&sh.total, mine);
    __syncthreads();
    const int total = sh.total;
    const int lo = int(int64_t(total) * share / shares), hi = int(int64_t(total) * (share + 1) / shares);
    if (lo < hi) {  // (the same for every thread)
        int front = 0;
        for (int base = 0; base < a.n_counts; base += kStepThreads) {
            const int i = base + tid, n = i < a.n_counts ? __ldcg(a.counts + i) : 0;
            int sum = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xFFFFFFFFu, sum, d);
                if (lane >= d) sum += o;
            }
            if (lane == 31) sh.scan[warp] = sum;
            __syncthreads();
            int before = front + sum - n;
#pragma unroll
            for (int w = 0; w < kStepThreads / 32; ++w) {
                const int o = sh.scan[w];
                if (w < warp) before += o;
                front += o;
            }
            if (n > 0 && before < hi && before + n > lo) sh.entry[atomicAdd(&sh.entries, 1)] = make_int2(i, before);
            __syncthreads();
        }
        for (int e = warp; e < sh.entries; e += kStepThreads / 32) {
            const int2 en = sh.entry[e];
            const int word = en.x * kUnionWords + lane;
            uint32_t w = word < a.VW ? __ldcg(a.any + word) : 0u;
            int n = __popc(w), sum = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xFFFFFFFFu, sum, d);
                if (lane >= d) sum += o;
            }
            for (int at = en.y + sum - n - lo; w; w &= w - 1, ++at)
                if (at >= 0 && at < hi - lo) sh.list[at] = 32 * word + __ffs(w) - 1;
        }
    }
    __syncthreads();
    return hi - lo;
}

// The state of one row from every block's, and the row's results; a warp.
__device__ __forceinline__ void step_finish_row(const HeadStepArgs& a, int row, int blocks, int lane) {
    const int part = step_row_part(a, row);
    if (part < 0) return;
    float top = -INFINITY;
    for (int i = lane; i < blocks; i += 32) top = fmaxf(top, __ldcg(&a.part[i * a.B + row].m));
    top = redux_max(top);
    const float ref = fmaxf(top, kRefFloor);
    float s = 0.f;
    int pos = kNoPos;
    for (int i = lane; i < blocks; i += 32) {
        const int4 v = __ldcg(reinterpret_cast<const int4*>(&a.part[i * a.B + row]));
        const float m = __int_as_float(v.x);
        s += __int_as_float(v.y) * ex2f((fmaxf(m, kRefFloor) - ref) * kLog2e);
        if (m == top) pos = min(pos, v.z);
    }
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    pos = __reduce_min_sync(0xFFFFFFFFu, pos);
    if (lane) return;
    const bool any = pos != kNoPos;
    const float log_sum = logf(s);
    a.argmax[row] = any ? pos : -1;
    if (a.rep) a.rep[row] = any ? a.parts[part].trep[pos] : -1;
    if (a.logp) a.logp[row] = s > 0.f ? -log_sum : -INFINITY;
    if (a.lse) a.lse[row] = s > 0.f ? top + log_sum : -INFINITY;
    if (!any) atomicAdd(a.status, 1);
}

// What the rows allow of one token, a bit a row.
__device__ __forceinline__ void step_bits(const HeadStepArgs& a, const StepShared& sh, int token, bool have, uint32_t (&bits)[kStepRows / 32]) {
    const uint32_t* p = a.mask + (token >> 5);
#pragma unroll
    for (int c = 0; c < kStepRows / 32; ++c) {
        uint32_t w = 0;
        const int n = min(32, a.B - 32 * c);
        if (have)
#pragma unroll 8
            for (int j = 0; j < n; ++j) w |= ((ld_after_wait(p + (32 * c + j) * a.mask_stride) >> (token & 31)) & 1u) << j;
        bits[c] = w & sh.valid[c];
    }
}

// The scores of 128 tokens under the rows of the batch: a lane has a token, a column is a row. Lane j of a warp keeps the state
// of the rows 32 c + j over the warp's tokens.
__device__ __forceinline__ void step_scores(const HeadStepArgs& a, uint32_t tmem, int token, const uint32_t (&bits)[kStepRows / 32],
                                            Partial (&state)[kStepRows / 32], int lane) {
#pragma unroll
    for (int c = 0; c < kStepRows / 32; ++c) {
        if (32 * c >= a.B) break;
        uint32_t v[32];
        tmem_ld32(tmem + 32 * c, v);
        tmem_wait_ld();
        float m = -INFINITY, s = 0.f;
        int pos = kNoPos;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const bool has = (bits[c] >> j) & 1u;
            const uint32_t who = __ballot_sync(0xFFFFFFFFu, has);
            if (!who) continue;
            const float z = has ? __uint_as_float(v[j]) : -INFINITY;
            const float top = redux_max(z);
            float e = has ? ex2f((z - fmaxf(top, kRefFloor)) * kLog2e) : 0.f;
#pragma unroll
            for (int d = 16; d >= 1; d >>= 1) e += __shfl_xor_sync(0xFFFFFFFFu, e, d);
            const int first = __shfl_sync(0xFFFFFFFFu, token, __ffs(__ballot_sync(0xFFFFFFFFu, has && z == top)) - 1);
            if (lane == j) {
                m = top;
                s = e;
                pos = first;
            }
            if (a.logits && has) {
                const int64_t at = (32 * c + j) * a.logits_stride + token;
                if (a.logits_dtype == kBF16) {
                    uint16_t r;
                    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(z));
                    static_cast<uint16_t*>(a.logits)[at] = r;
                } else {
                    static_cast<float*>(a.logits)[at] = z;
                }
            }
        }
        partial_merge(state[c].m, state[c].s, state[c].pos, m, s, pos);
    }
}

__global__ void __launch_bounds__(kStepThreads, 1)
    k_head_step(const __grid_constant__ HeadStepArgs a, const __grid_constant__ CUtensorMap map_x) {
    extern __shared__ char smem_raw[];
    __shared__ __align__(16) StepShared sh;
    const uint32_t stages = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t x_at = kStepTiles * kStepTileBytes, stage_bytes = x_at + uint32_t(a.N) * 128u;
    const uint32_t columns = 2 * kStepTiles * a.N <= 128 ? 128 : 2 * kStepTiles * a.N <= 256 ? 256 : 512;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStepStages; ++i) {
            mbar_init(&sh.full[i], 5);  // hidden states, and the four warps that fetch weights
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.sums_full[i], 1);
            mbar_init(&sh.sums_empty[i], 4);
        }
        mbar_init_fence();
        prefetch_tensor_map(&map_x);
    }
    if (warp == 2) tmem_alloc<1>(&sh.tmem, columns);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (threadIdx.x < kStepRows) {
        const bool v = int(threadIdx.x) < a.B && step_row_part(a, threadIdx.x) >= 0;
        const uint32_t w = __ballot_sync(0xFFFFFFFFu, v);
        if (lane == 0) sh.valid[warp] = w;
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = sh.tmem;
    bool ok = true;
    int stage = 0, group_at = 0;
    uint32_t phase = 0;
    Partial state[kStepRows / 32];
#pragma unroll
    for (int c = 0; c < kStepRows / 32; ++c) state[c] = partial_empty();
    for (int round = 0; round < a.rounds; ++round) {
        const int n = step_share(a, sh, round * gridDim.x + blockIdx.x, a.rounds * gridDim.x);
        const int groups = (n + 128 * kStepTiles - 1) / (128 * kStepTiles);
        if (warp == 0) {
            if (lane == 0)
                for (int i = 0; i < groups * a.k_blocks; ++i) {
                    if (!mbar_wait(&sh.empty[stage], phase ^ 1)) {
                        ok = false;
                        break;
                    }
                    mbar_expect_tx(&sh.full[stage], uint32_t(a.N) * 128u);
                    asm volatile(
                        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], "
                        "[%4];" ::"r"(stages + uint32_t(stage) * stage_bytes + x_at),
                        "l"(&map_x), "r"(i % a.k_blocks * 64), "r"(0), "r"(smem_u32(&sh.full[stage]))
                        : "memory");
                    if (++stage == a.stages) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
        } else if (warp >= 8) {
            // eight lanes bring the 128 bytes of a row, a warp four rows at a time
            const int chunk = lane & 7;
            int issued = 0, done = stage;
            auto arrive = [&] {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.full[done]);
                if (++done == a.stages) done = 0;
            };
            for (int g = 0; g < groups && ok; ++g) {
                const char* from[kStepTiles][8];
#pragma unroll
                for (int t = 0; t < kStepTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int at = (g * kStepTiles + t) * 128 + (warp & 3) * 32 + 4 * i + (lane >> 3);
                        from[t][i] = at < n ? static_cast<const char*>(a.weight) + int64_t(sh.list[at]) * a.row_bytes + chunk * 16 : nullptr;
                    }
                for (int k = 0; k < a.k_blocks; ++k) {
                    if (!mbar_wait(&sh.empty[stage], phase ^ 1)) {
                        ok = false;
                        break;
                    }
                    const bool have = k * 64 + chunk * 8 < a.H;
                    const uint32_t at = stages + uint32_t(stage) * stage_bytes + uint32_t((warp & 3) * 32 + (lane >> 3)) * 128u;
#pragma unroll
                    for (int t = 0; t < kStepTiles; ++t)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (from[t][i])
                                copy16(at + t * kStepTileBytes + i * 512 + uint32_t((chunk ^ ((4 * i + (lane >> 3)) & 7)) << 4),
                                       have ? from[t][i] + k * 128 : from[t][i] - chunk * 16, have);
                    asm volatile("cp.async.commit_group;" ::: "memory");
                    if (++stage == a.stages) {
                        stage = 0;
                        phase ^= 1;
                    }
                    if (++issued > kStepLag) {
                        asm volatile("cp.async.wait_group %0;" ::"n"(kStepLag) : "memory");
                        arrive();
                    }
                }
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            for (int i = 0; i < min(issued, kStepLag); ++i) arrive();
        } else if (warp == 1) {
            if (lane == 0) {
                const uint32_t idesc = kMmaBf16Desc<128, 0, false, false> | uint32_t(a.N / 8) << 17;
                for (int g = 0; g < groups && ok; ++g) {
                    const int it = group_at + g;
                    if (!mbar_wait(&sh.sums_empty[it & 1], ((it >> 1) & 1) ^ 1)) {
                        ok = false;
                        break;
                    }
                    tmem_fence_after();
                    const uint32_t d = tmem + uint32_t(it & 1) * kStepTiles * a.N;
                    for (int k = 0; k < a.k_blocks; ++k) {
                        if (!mbar_wait(&sh.full[stage], phase)) {
                            ok = false;
                            break;
                        }
                        tmem_fence_after();
                        const uint32_t at = stages + uint32_t(stage) * stage_bytes;
                        const uint64_t dx = mma_desc<false>(at + x_at);
#pragma unroll
                        for (int t = 0; t < kStepTiles; ++t) {
                            if ((g * kStepTiles + t) * 128 >= n) break;
                            const uint64_t dw = mma_desc<false>(at + t * kStepTileBytes);
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                mma_f16<1>(d + t * a.N, dw + j * kDescStep16<false>, dx + j * kDescStep16<false>, idesc, k > 0 || j > 0);
                        }
                        mma_commit<1>(&sh.empty[stage]);
                        if (++stage == a.stages) {
                            stage = 0;
                            phase ^= 1;
                        }
                    }
                    mma_commit<1>(&sh.sums_full[it & 1]);
                }
            }
        } else if (warp >= 4) {
            const int quad = warp & 3;
            for (int g = 0; g < groups; ++g) {
                const int it = group_at + g;
                int token[kStepTiles];
                uint32_t bits[kStepTiles][kStepRows / 32];
#pragma unroll
                for (int t = 0; t < kStepTiles; ++t) {
                    const int at = (g * kStepTiles + t) * 128 + quad * 32 + lane;
                    token[t] = at < n ? sh.list[at] : 0;
                    step_bits(a, sh, token[t], at < n, bits[t]);
                }
                if (!mbar_wait(&sh.sums_full[it & 1], (it >> 1) & 1)) {
                    ok = false;
                    break;
                }
                tmem_fence_after();
#pragma unroll
                for (int t = 0; t < kStepTiles; ++t)
                    if ((g * kStepTiles + t) * 128 < n)
                        step_scores(a, tmem + (uint32_t(it & 1) * kStepTiles + t) * a.N + (uint32_t(quad * 32) << 16), token[t], bits[t],
                                    state, lane);
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.sums_empty[it & 1]);
            }
        }
        __syncwarp();
        group_at += groups;
        __syncthreads();
    }
    if (!ok && lane == 0) atomicExch(a.status + 3, 1);
    // the four warps' states to one, out to the others' and, in the last block to come here, to the results
    Partial* mine = reinterpret_cast<Partial*>(sh.entry);
    if (warp >= 4 && warp < 8) {
#pragma unroll
        for (int c = 0; c < kStepRows / 32; ++c) mine[(warp & 3) * kStepRows + 32 * c + lane] = state[c];
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 2) tmem_free<1>(tmem, columns);
    if (int(threadIdx.x) < a.B) {
        Partial p = mine[threadIdx.x];
#pragma unroll
        for (int q = 1; q < 4; ++q) {
            const Partial o = mine[q * kStepRows + threadIdx.x];
            partial_merge(p.m, p.s, p.pos, o.m, o.s, o.pos);
        }
        __stcg(reinterpret_cast<int4*>(&a.part[blockIdx.x * a.B + threadIdx.x]),
               make_int4(__float_as_int(p.m), __float_as_int(p.s), p.pos, 0));
        __threadfence();
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.is_last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!sh.is_last) return;
    __threadfence();
    for (int row = warp; row < a.B; row += kStepThreads / 32) step_finish_row(a, row, gridDim.x, lane);
}

}  // namespace cfgzip
