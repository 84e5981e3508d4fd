// Last steps of the head's tall products: partial states to results, cuts of a sum to bf16.
#pragma once

#include "cfgzip_device.cuh"

namespace cfgzip {

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

// The same for log probabilities and entropies. A state is its largest score, kFew where it has none, the sum of exp(d) without the scores that
// are the largest, the sum of exp(d) d, and how many are the largest: of a row that has one probable token the sum is 1 and little, and the
// little is what its log probability and entropy are. Differences of references are bounded where their exponential is 0: a sum of many times
// one may be infinite, and the sum of exp(d) d with it NaN.
constexpr float kNothing = -4096.f;
__device__ __forceinline__ void add_state(const float4& p, float ref, float& n, float& s, float& d) {
    const float of = fmaxf(p.x - ref, kNothing), f = ex2f(of * kLog2e);
    const bool same = p.x == ref;
    d = fmaf(fmaf(of, p.y + p.w, p.z), f, d);
    n += same ? p.w : 0.f;
    s = fmaf(same ? p.y : p.y + p.w, f, s);
}
struct LogprobsFinishArgs {
    const float4* sums;
    const float* of_target;
    int32_t tiles, rows, V;
    const uint32_t* mask;
    int64_t mask_stride;
    const int32_t* tokens;
    float *logp, *entropy, *lse;
    int32_t* status;
};
__global__ void __launch_bounds__(256) k_head_logprobs_finish(const LogprobsFinishArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x * kFinishRows + (lane & 3);
    const bool ends = warp == 0 && lane < kFinishRows && row < a.rows;
    const int token = ends ? ld_after_wait(a.tokens + row) : -1;
    const float of_token = ends ? ld_after_wait(a.of_target + row) : 0.f;
    float m = kFew, n = 0.f, s = 0.f, d = 0.f;
    if (row < a.rows)
        for (int t = warp * 8 + (lane >> 2); t < a.tiles; t += 320) {
            float4 p[5];
#pragma unroll
            for (int k = 0; k < 5; ++k)
                p[k] = t + 64 * k < a.tiles ? __ldcg(a.sums + int64_t(t + 64 * k) * a.rows + row) : make_float4(kFew, 0.f, 0.f, 0.f);
            float next = m;
#pragma unroll
            for (int k = 0; k < 5; ++k) next = fmaxf(next, p[k].x);
            const float4 before = make_float4(m, s, d, n);
            n = s = d = 0.f;
            add_state(before, next, n, s, d);
#pragma unroll
            for (int k = 0; k < 5; ++k) add_state(p[k], next, n, s, d);
            m = next;
        }
    bool has = token >= 0 && token < a.V;
    if (has && a.mask) has = (ld_after_wait(a.mask + int64_t(row) * a.mask_stride + (token >> 5)) >> (token & 31)) & 1u;
    __shared__ float4 sh[64][kFinishRows];
    sh[warp * 8 + (lane >> 2)][lane & 3] = make_float4(m, s, d, n);
    __syncthreads();
    if (warp) return;
    // eight threads a row, eight states each
    float top = kFew;
#pragma unroll
    for (int w = 0; w < 8; ++w) top = fmaxf(top, sh[8 * (lane >> 2) + w][lane & 3].x);
#pragma unroll
    for (int k = 4; k <= 16; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, k));
    n = s = d = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) add_state(sh[8 * (lane >> 2) + w][lane & 3], top, n, s, d);
#pragma unroll
    for (int k = 4; k <= 16; k <<= 1) {
        n += __shfl_xor_sync(0xFFFFFFFFu, n, k);
        s += __shfl_xor_sync(0xFFFFFFFFu, s, k);
        d += __shfl_xor_sync(0xFFFFFFFFu, d, k);
    }
    if (!ends) return;
    // (n is 0 where nothing is allowed; 1 as a rule, whose logarithm is 0)
    const float log_sum = logf(n) + log1pf(s / n);
    if (a.lse) a.lse[row] = n > 0.f ? top + log_sum : -INFINITY;
    if (a.entropy) a.entropy[row] = n > 0.f ? fmaxf(log_sum - d / (n + s), 0.f) : 0.f;
    if (token >= a.V) atomicAdd(a.status + 1, 1);
    float logp = 0.f;
    if (token >= 0) logp = has && of_token > kFew ? (of_token - top) - log_sum : -INFINITY;
    a.logp[row] = logp;
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

// k_head_round, with what the rows' targets were rounded by.
struct RoundTargetsArgs {
    const float* from;
    int64_t split_elems;
    int32_t splits, rows, n, V;
    uint16_t* to;
    int64_t to_stride;
    const int32_t* targets;
    const float* rest;
    const uint16_t* weight;
    int64_t weight_stride;
};
__device__ __forceinline__ void round_targets(const RoundTargetsArgs& a, int block, int blocks) {
    const int vectors = a.n / 4;
    const int64_t total = int64_t(a.rows) * vectors;
    for (int64_t i = int64_t(block) * 256 + threadIdx.x; i < total; i += int64_t(blocks) * 256) {
        const int64_t row = i / vectors;
        const int col = 4 * int(i - row * vectors);
        const int target = ld_after_wait(a.targets + row);
        const float rest = ld_after_wait(a.rest + row);
        float f[4] = {};
#pragma unroll 8
        for (int s = 0; s < a.splits; ++s) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(a.from + s * a.split_elems + 4 * i));
            f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
        }
        if (target >= 0 && target < a.V && rest != 0.f) {
            const uint2 w = *reinterpret_cast<const uint2*>(a.weight + int64_t(target) * a.weight_stride + col);
            f[0] = fmaf(rest, __uint_as_float(w.x << 16), f[0]);
            f[1] = fmaf(rest, __uint_as_float(w.x & 0xFFFF0000u), f[1]);
            f[2] = fmaf(rest, __uint_as_float(w.y << 16), f[2]);
            f[3] = fmaf(rest, __uint_as_float(w.y & 0xFFFF0000u), f[3]);
        }
        *reinterpret_cast<uint2*>(a.to + row * a.to_stride + col) = make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]));
    }
}

// The rows that have a token for a target as a chain in the order of the rows: the first row of each token that is a target, each row's next
// one. A warp compares its four rows' targets with all others, 32 at a time; no order of arrival plays a part. Tokens that are no target keep
// what the workspace held before: whoever asks for a token's first row looks whether that row has it (first_row), which spares writing, and
// searching for, all of the vocabulary's. Nothing is left of the targets yet (rest 0). (4096 rows: 10 us of a gradient of 9 ms;
// it grows with the square of them.)
constexpr int kTargetRows = 4;
__global__ void __launch_bounds__(256) k_head_targets(const int32_t* targets, int N, int V, int32_t* first_of, int32_t* next_of, float* rest) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = int(threadIdx.x) & 31, r0 = kTargetRows * (int(blockIdx.x) * 8 + int(threadIdx.x >> 5));
    if (r0 >= N) return;
    int mine[kTargetRows], next[kTargetRows];
    bool before[kTargetRows];
#pragma unroll
    for (int j = 0; j < kTargetRows; ++j) {
        mine[j] = r0 + j < N ? ld_after_wait(targets + r0 + j) : -1;
        next[j] = INT_MAX;
        before[j] = false;
    }
    for (int n0 = 0; n0 < N; n0 += 128) {
        int other[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) other[q] = n0 + 32 * q + lane < N ? ld_after_wait(targets + n0 + 32 * q + lane) : -1;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = n0 + 32 * q + lane;
#pragma unroll
            for (int j = 0; j < kTargetRows; ++j) {
                const bool same = other[q] == mine[j];
                before[j] |= same && n < r0 + j;
                if (same && n > r0 + j) next[j] = min(next[j], n);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kTargetRows; ++j) {
        const int found = __reduce_min_sync(0xFFFFFFFFu, next[j]);
        const bool first = !__any_sync(0xFFFFFFFFu, before[j]);
        if (lane == 0 && r0 + j < N) {
            next_of[r0 + j] = found < N ? found : -1;
            rest[r0 + j] = 0.f;
            if (first && mine[j] >= 0 && mine[j] < V) first_of[mine[j]] = r0 + j;
        }
    }
}

// The rows of the head's gradient that are targets, once more: their sums as they were kept, and what their rows' g was rounded by times the
// hidden states. A block a row of the text; the first row of a chain does all of it. Each step along a chain is a load that waits for the one
// before. Answers under a grammar repeat some tokens again and again: chains of more than kTargetSteps rows are listed by looking through the
// targets, and have a block for every kTargetCols columns, in which eight groups of threads add up every eighth row, four loads in flight
// (gradient of 4000 tokens of 2000 x 4096, all the same: 7300 us along the chain, 670 by 512 columns, 440; of twice as many tokens as there are
// in the vocabulary 242, 228 without looking for long chains).
constexpr int kTargetCols = 256, kTargetGroups = 8 * 256 / kTargetCols, kTargetSteps = 8, kTargetList = 1024, kTargetSlice = 8;
struct WeightTargetsArgs {
    const int32_t *targets, *first_of, *next_of;
    const float *rest, *kept;
    const uint16_t* hidden;
    int64_t hidden_stride;
    void* to;
    int64_t to_stride;
    int32_t N, V, H, bf16;
};
__device__ __forceinline__ void store_weight_targets(const WeightTargetsArgs& a, int target, int c, const float4& f) {
    if (a.bf16)
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.to) + target * a.to_stride + c) = make_uint2(bf16_pair(f.x, f.y), bf16_pair(f.z, f.w));
    else
        *reinterpret_cast<float4*>(static_cast<float*>(a.to) + target * a.to_stride + c) = f;
}
__device__ __forceinline__ void weight_targets_of_many(const WeightTargetsArgs& a, int row, int target, int c0) {
    __shared__ int s_row[kTargetList], s_count[32];
    __shared__ float s_rest[kTargetList];
    __shared__ __align__(16) float s_sum[kTargetGroups][kTargetCols];
    const int warp = int(threadIdx.x) >> 5, lane = int(threadIdx.x) & 31, group = int(threadIdx.x) / (kTargetCols / 8), mine = 8 * (int(threadIdx.x) % (kTargetCols / 8));
    const bool some = c0 + mine < a.H;
    float f[8] = {};
    for (int n0 = row; n0 < a.N; n0 += kTargetList) {  // 1024 targets at a time, those that are this one in the rows' order
        uint32_t same[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = n0 + 256 * q + int(threadIdx.x);
            same[q] = __ballot_sync(0xFFFFFFFFu, n < a.N && ld_after_wait(a.targets + n) == target);
            if (lane == 0) s_count[8 * q + warp] = __popc(same[q]);
        }
        __syncthreads();
        const int count = s_count[lane];
        int ahead = count;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int x = __shfl_up_sync(0xFFFFFFFFu, ahead, d);
            ahead += lane >= d ? x : 0;
        }
        const int all = __shfl_sync(0xFFFFFFFFu, ahead, 31);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int at = __shfl_sync(0xFFFFFFFFu, ahead - count, 8 * q + warp) + __popc(same[q] & ((1u << lane) - 1u));
            if ((same[q] >> lane) & 1u) {
                const int n = n0 + 256 * q + int(threadIdx.x);
                s_row[at] = n;
                s_rest[at] = ld_after_wait(a.rest + n);
            }
        }
        __syncthreads();
        if (some) {
#pragma unroll 4
            for (int i = group; i < all; i += kTargetGroups) {
                float x[8];
                bf16_values(ld_after_wait(reinterpret_cast<const uint4*>(a.hidden + int64_t(s_row[i]) * a.hidden_stride + c0 + mine)), x);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = fmaf(s_rest[i], x[j], f[j]);
            }
        }
        __syncthreads();
    }
    if (some) {
        *reinterpret_cast<float4*>(&s_sum[group][mine]) = make_float4(f[0], f[1], f[2], f[3]);
        *reinterpret_cast<float4*>(&s_sum[group][mine + 4]) = make_float4(f[4], f[5], f[6], f[7]);
    }
    __syncthreads();
    const int at = 4 * int(threadIdx.x);
    if (at >= kTargetCols || c0 + at >= a.H) return;
    float4 sum = __ldcg(reinterpret_cast<const float4*>(a.kept + int64_t(row) * a.H + c0 + at));
#pragma unroll
    for (int g = 0; g < kTargetGroups; ++g) {
        const float4 x = *reinterpret_cast<const float4*>(&s_sum[g][at]);
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
    }
    store_weight_targets(a, target, c0 + at, sum);
}
// The first row of a chain: -1 where this row is none, else the row behind it, or kTargetMany behind kTargetSteps rows.
constexpr int kTargetNone = -2, kTargetMany = INT_MAX;
__device__ __forceinline__ int chain_of(const WeightTargetsArgs& a, int row, int target) {
    if (target < 0 || target >= a.V || ld_after_wait(a.first_of + target) != row) return kTargetNone;
    const int next = ld_after_wait(a.next_of + row);
    int m = next;
    for (int n = 1; m >= 0 && n < kTargetSteps; ++n) m = ld_after_wait(a.next_of + m);
    return m >= 0 ? kTargetMany : next;
}
__device__ __forceinline__ void weight_targets(const WeightTargetsArgs& a, int row) {
    const int target = ld_after_wait(a.targets + row), next = chain_of(a, row, target);
    if (next == kTargetNone || next == kTargetMany) return;
    for (int c = 4 * int(threadIdx.x); c < a.H; c += 1024) {
        float4 f = __ldcg(reinterpret_cast<const float4*>(a.kept + int64_t(row) * a.H + c));
        for (int m = row; m >= 0; m = m == row ? next : ld_after_wait(a.next_of + m)) {
            const float rest = ld_after_wait(a.rest + m);
            const uint2 x = *reinterpret_cast<const uint2*>(a.hidden + int64_t(m) * a.hidden_stride + c);
            f.x = fmaf(rest, __uint_as_float(x.x << 16), f.x);
            f.y = fmaf(rest, __uint_as_float(x.x & 0xFFFF0000u), f.y);
            f.z = fmaf(rest, __uint_as_float(x.y << 16), f.z);
            f.w = fmaf(rest, __uint_as_float(x.y & 0xFFFF0000u), f.w);
        }
        store_weight_targets(a, target, c, f);
    }
}
// ... of the chains of many rows that begin in kTargetSlice rows from `first` on, kTargetCols columns from c0 on
__device__ __forceinline__ void weight_targets_of_slice(const WeightTargetsArgs& a, int first, int c0) {
    const int lane = int(threadIdx.x) & 31, mine = first + lane, target = lane < kTargetSlice && mine < a.N ? ld_after_wait(a.targets + mine) : -1;
    uint32_t many = __ballot_sync(0xFFFFFFFFu, chain_of(a, mine, target) == kTargetMany);
    for (; many; many &= many - 1) {
        const int of = __ffs(many) - 1;
        weight_targets_of_many(a, first + of, __shfl_sync(0xFFFFFFFFu, target, of), c0);
        __syncthreads();
    }
}

// Both, one behind the other: the first `ahead` blocks look for chains of many rows, for a number of columns each, `rows` blocks take a row's
// target each.
__global__ void __launch_bounds__(256, 8) k_head_targets_finish(const WeightTargetsArgs w, const RoundTargetsArgs r, int ahead, int slices, int rows) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (int(blockIdx.x) < ahead)
        weight_targets_of_slice(w, int(blockIdx.x) % slices * kTargetSlice, int(blockIdx.x) / slices * kTargetCols);
    else if (int(blockIdx.x) < ahead + rows)
        weight_targets(w, int(blockIdx.x) - ahead);
    else
        round_targets(r, int(blockIdx.x) - ahead - rows, int(gridDim.x) - ahead - rows);
}

}  // namespace cfgzip
