// The product of hidden states with a head, and what is taken from it: normaliser, greedy choice, loss, gradient.
#pragma once

#include "cfgzip_head_mma.cuh"

namespace cfgzip {

__device__ __forceinline__ uint16_t f32_bf16(float v) {  // nearest, ties to even
    uint16_t r;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(v));
    return r;
}

// C[m, n] (+)= sum_k A[m * sam + k * sak] * B[n * sbn + k * sbk], 64 x 64 by a block, 4 x 4 a thread, f32 FMA.
struct ProductArgs {
    const uint16_t *a, *b;
    int64_t sam, sak, sbn, sbk;
    void* c;
    int64_t ldc;
    int M, N, K;
    int bf16_out, accumulate;
};
__global__ void __launch_bounds__(256) k_head_product(const ProductArgs p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float sa[16][65], sb[16][65];
    const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < p.K; k0 += 16) {
        for (int i = threadIdx.x; i < 1024; i += 256) {
            const int r = p.sak == 1 ? i >> 4 : i & 63, k = p.sak == 1 ? i & 15 : i >> 6;
            sa[k][r] = m0 + r < p.M && k0 + k < p.K ? bf16_f32(p.a[(m0 + r) * p.sam + (k0 + k) * p.sak]) : 0.f;
            const int rb = p.sbk == 1 ? i >> 4 : i & 63, kb = p.sbk == 1 ? i & 15 : i >> 6;
            sb[kb][rb] = n0 + rb < p.N && k0 + kb < p.K ? bf16_f32(p.b[(n0 + rb) * p.sbn + (k0 + kb) * p.sbk]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m >= p.M || n >= p.N) continue;
            const int64_t at = m * p.ldc + n;
            if (p.bf16_out) {
                uint16_t* c = static_cast<uint16_t*>(p.c) + at;
                *c = f32_bf16(p.accumulate ? bf16_f32(*c) + acc[i][j] : acc[i][j]);
            } else {
                float* c = static_cast<float*>(p.c) + at;
                *c = p.accumulate ? *c + acc[i][j] : acc[i][j];
            }
        }
}

struct RowState {  // of a row over the pieces of the vocabulary so far
    float m, s;
    int pos;
    float target;  // score of the target
};

struct RowsArgs {
    const PartDev* parts;
    int32_t part0, n_parts;
    const int32_t* row_part;
    const float* z;  // [rows, piece]
    int64_t ldz;
    int32_t rows, V, t0, n;  // the piece is tokens t0 .. t0 + n
    const uint32_t* mask;
    int64_t mask_stride;
    RowState* state;
    void* logits;
    int64_t logits_stride;
    int logits_dtype;
    const int32_t* targets;
    int32_t *argmax, *rep;
    float *logp, *lse, *loss;
    int32_t* status;
    const float *lse_in, *d_loss;
    uint16_t* g;  // [rows, piece]
};

__device__ __forceinline__ bool row_has_part(const RowsArgs& a, int row, int* part) {
    *part = a.part0;
    if (!a.row_part) return true;
    *part = ld_after_wait(a.row_part + row);
    return *part >= 0 && *part < a.n_parts && a.parts[*part].live && a.parts[*part].V == a.V;
}

__device__ __forceinline__ bool allowed(const RowsArgs& a, int row, int t) {
    return !a.mask || ((ld_after_wait(a.mask + row * a.mask_stride + (t >> 5)) >> (t & 31)) & 1u);
}

// One block a row: the piece's scores join the row's state; the masked scores go out where they are wanted.
__global__ void __launch_bounds__(256) k_head_rows(const RowsArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int part;
    if (!row_has_part(a, row, &part)) return;
    const int target = a.targets ? a.targets[row] : -1;
    float m = -INFINITY, s = 0.f, zt = -INFINITY;
    int pos = kNoPos;
    for (int i = threadIdx.x; i < a.n; i += 256) {
        const int t = a.t0 + i;
        const float z = allowed(a, row, t) ? a.z[row * a.ldz + i] : -INFINITY;
        if (allowed(a, row, t)) {
            partial_merge(m, s, pos, z, z > -INFINITY ? ex2f((z - fmaxf(z, kRefFloor)) * kLog2e) : 0.f, t);
            if (t == target) zt = z;
        }
        if (a.logits) {
            const int64_t at = row * a.logits_stride + t;
            if (a.logits_dtype == kBF16) static_cast<uint16_t*>(a.logits)[at] = f32_bf16(z);
            else static_cast<float*>(a.logits)[at] = z;
        }
    }
    partial_warp_allreduce(m, s, pos);
    for (int d = 16; d >= 1; d >>= 1) zt = fmaxf(zt, __shfl_xor_sync(0xFFFFFFFFu, zt, d));
    __shared__ RowState sh[8];
    if (lane == 0) sh[warp] = RowState{m, s, pos, zt};
    __syncthreads();
    if (threadIdx.x) return;
    RowState r = a.t0 ? a.state[row] : RowState{-INFINITY, 0.f, kNoPos, -INFINITY};
    for (int w = 0; w < 8; ++w) {
        partial_merge(r.m, r.s, r.pos, sh[w].m, sh[w].s, sh[w].pos);
        r.target = fmaxf(r.target, sh[w].target);
    }
    a.state[row] = r;
}

__global__ void __launch_bounds__(256) k_head_finish(const RowsArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows) return;
    int part;
    if (!row_has_part(a, row, &part)) return;
    const RowState r = a.state[row];
    const float log_sum = logf(r.s), lse = r.s > 0.f ? r.m + log_sum : -INFINITY;
    if (a.argmax) {
        const bool any = r.pos != kNoPos;
        a.argmax[row] = any ? r.pos : -1;
        if (a.rep) a.rep[row] = any ? a.parts[part].trep[r.pos] : -1;
        if (a.logp) a.logp[row] = r.s > 0.f ? -log_sum : -INFINITY;
        if (!any) atomicAdd(a.status, 1);
    }
    if (a.lse) a.lse[row] = lse;
    if (a.loss) {
        const int t = a.targets[row];
        if (t >= a.V) atomicAdd(a.status + 1, 1);
        a.loss[row] = t < 0 ? 0.f : r.target > -INFINITY ? (r.m - r.target) + log_sum : INFINITY;
    }
}

// The sums of `splits` cuts, added up and rounded; eight to a thread, n a multiple of 8.
__global__ void __launch_bounds__(256) k_head_round(const float* from, int64_t split_elems, int splits, uint16_t* to, int64_t to_stride,
                                                    int rows, int n) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int vectors = n / 8;
    const int64_t total = int64_t(rows) * vectors;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
        float f[8] = {};
        for (int s = 0; s < splits; ++s) {
            const float4* p = reinterpret_cast<const float4*>(from + s * split_elems + 8 * i);
            const float4 x = __ldcg(p), y = __ldcg(p + 1);
            f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
            f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
        }
        const MxAt at = mx_at(i, vectors);
        *reinterpret_cast<uint4*>(to + at.row * to_stride + 8 * at.col) =
            make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
    }
}

}  // namespace cfgzip
