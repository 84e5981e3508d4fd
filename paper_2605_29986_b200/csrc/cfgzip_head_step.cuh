// The decode step from hidden states. The scores of a batch are a product with one side short (the rows of the batch), so the
// weights are what takes the time, and only those of tokens that some row allows are read: the union of the rows' masks is
// compacted to a list of tokens, of which every block takes an equal share. The tokens' rows are the long side of tcgen05 products
// (128 tokens x up to 128 rows), k in stages of shared memory; the scores of a tile go from tensor memory into the rows' running
// maximum, sum and choice. The last block to finish puts the blocks' together.
//
// 32 rows of 128256 x 4096 (bf16, 97 % allowed by some row): 1.05 GB in 173 to 179 us with the masks, 5.9 TB/s; inside the loop the
// copies run at the memory's rate, and some 20 us go to the masks, the list, the first loads and the last scores. From 4 bits: 279 MB
// in 84 to 92 us, one row of 151936 x 2560 in 65. Boxes of 128-byte pieces of 128 rows come at 5.1 to 5.7 TB/s (measured alone), 850
// cycles for 128 tokens x 256 weights, turning those into f16 takes 550 (the loop alone); from 17 rows on the hidden states, which
// every block brings past again for each tile, are as many bytes as the weights (16 rows: 76 us, 32: 84, 64: 113). One row of 32000 x 2048: 20 us, of which the loads need 6; what is left is latency (masks 4, list 3, first loads 2,
// scores and results 3, two launches).
#pragma once

#include <cuda.h>

#include "cfgzip_head_mma.cuh"

namespace cfgzip {

constexpr int kUnionWords = 32;    // mask words (1024 tokens) counted together, by a block
constexpr int kUnionThreads = 512;
constexpr int kUnionEach = kUnionWords / (kUnionThreads / 32);  // words a warp takes
constexpr int kStepRows = 128;     // rows of the batch a launch takes at most
constexpr int kStepRowsMx = 64;    // ... from a 4-bit head: the hidden states are brought past four times as many weights a byte
constexpr int kStepShare = 2048;   // tokens a block lists at a time
constexpr int kStepWarps = 16;     // tiled copies, products, tensor memory, idle, four that read the scores, eight that fetch weights
constexpr int kStepWarpsMx = 24;   // ... and two sets of four that turn 4-bit weights into f16
constexpr int kStepBox = 32;       // rows of weights a small tiled copy brings (a large one: 128)
constexpr int kStepStages = 12;    // most stages
constexpr uint32_t kStepAtom = 128;             // bytes of a weight row in an atom, the width of the swizzle
constexpr uint32_t kStepTile = 128 * kStepAtom; // an atom of 128 tokens

struct HeadStepArgs {
    const PartDev* parts;
    int32_t part0, n_parts;
    const int32_t* row_part;
    const uint32_t* mask;  // [B, mask_stride] vocab masks
    int64_t mask_stride;
    int32_t B, V, VW, H;
    const void* weight;
    int64_t row_bytes;
    const uint8_t* scales;
    int64_t scale_stride;
    int32_t N;             // columns of a tile: B rounded up to 32, or 16
    int32_t row_atoms;     // atoms of a row of weights
    int32_t bytes;         // of a row of weights that count
    int32_t smem;          // shared memory for stages
    int32_t rounds;
    int32_t expire;        // test hook: the block reports a wait as run out when the first stages are asked for (see cfgzip_set_tuning)
    const uint16_t* hidden;  // 4-bit heads: rows brought to at most 2^15 and copied as f16 to `half`
    int64_t hidden_stride;
    uint16_t* half;        // [B, half_stride], zeros behind H
    int32_t half_stride;   // H rounded up to an atom's weights
    float* back;           // [B] what brings a row's products back
    uint32_t* any;         // [VW] union of the rows' masks
    uint32_t* bits;        // [(B + 31) / 32, 32 VW] what 32 rows allow of a token, a bit a row
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

// A row of hidden states as f16, times the power of two that brings its largest to [2^14, 2^15): all of a bf16 number's bits are
// kept down to 2^-29 of the largest, and what is lost below that is 2^-40 of it at most, nothing to a sum in 32 bits.
__device__ __forceinline__ void half_row(const HeadStepArgs& a, int row) {
    __shared__ uint32_t most[kUnionThreads / 32];
    const int vectors = a.H / 8, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint4* x = reinterpret_cast<const uint4*>(a.hidden + row * a.hidden_stride);
    uint32_t top = 0;
    for (int i = threadIdx.x; i < vectors; i += kUnionThreads) {
        const uint4 v = ld_after_wait(x + i);
        top = __vmaxu2(__vmaxu2(top, __vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu)), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
    }
    top = __reduce_max_sync(0xFFFFFFFFu, max(top >> 16, top & 0xFFFFu));
    if (lane == 0) most[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kUnionThreads / 32; ++w) top = max(top, most[w]);
    const int e = min(max(int(top >> 7), 15), 254);  // exponent of the largest, + 127
    const float up = __uint_as_float(uint32_t(268 - e) << 23);  // 2^(14 - (e - 127))
    if (threadIdx.x == 0) a.back[row] = __uint_as_float(uint32_t(max(e - 14, 1)) << 23);
    for (int i = threadIdx.x; i < a.half_stride / 8; i += kUnionThreads) {
        const uint4 v = i < vectors ? ld_after_wait(x + i) : make_uint4(0, 0, 0, 0);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            asm("cvt.rn.f16x2.f32 %0, %1, %2;"
                : "=r"(o[j])
                : "f"(__uint_as_float(w[j] & 0xFFFF0000u) * up), "f"(__uint_as_float(w[j] << 16) * up));
        reinterpret_cast<uint4*>(a.half + int64_t(row) * a.half_stride)[i] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// What 32 words of tokens (kUnionWords) are worth to a batch, from each token's allowing rows: bits to a.bits, count, union; and with
// `masks` the rows' vocab masks. A warp takes kUnionEach words, a lane a token: allow(word, k) gives the bits.
template <typename F>
__device__ __forceinline__ void union_chunk(const HeadStepArgs& a, int c, uint32_t* sh, uint32_t* masks, int64_t mask_stride, F&& allow) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int k = 0; k < kUnionEach; ++k) {
        const int at = blockIdx.x * kUnionWords + kUnionEach * warp + k;
        const uint32_t b = allow(at, k), any = __ballot_sync(0xFFFFFFFFu, b != 0);
        if (at < a.VW) a.bits[(int64_t(c) * a.VW + at) * 32 + lane] = b;
        if (lane == 0 && any) sh[kUnionEach * warp + k] |= any;
        if (masks) {
            const uint32_t w = warp_transpose32(b, lane);
            const int row = 32 * c + lane;
            if (at < a.VW && row < a.B) masks[row * mask_stride + at] = w;
        }
    }
}
__device__ __forceinline__ void union_finish(const HeadStepArgs& a, const uint32_t* sh) {
    __syncthreads();
    if (threadIdx.x >= 32) return;
    const int word = blockIdx.x * kUnionWords + int(threadIdx.x);
    const uint32_t any = sh[threadIdx.x];
    if (word < a.VW) a.any[word] = any;
    const int n = __reduce_add_sync(0xFFFFFFFFu, __popc(any));
    if (threadIdx.x == 0) a.counts[blockIdx.x] = n;
}

// Rows of one partition: class masks turned to a table of 32 rows a class, a token's rows by one lookup. Vocab masks, union and turned
// masks in one launch (expanding and turning by two took 3 to 5 us longer).
__global__ void __launch_bounds__(kUnionThreads) k_head_masks(const HeadStepArgs a, const __grid_constant__ PartDev p, const uint32_t* class_mask,
                                                    int64_t class_stride, uint32_t* masks, int64_t mask_stride) {
    extern __shared__ uint32_t table[];
    __shared__ uint32_t sh[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t cls[kUnionEach];
#pragma unroll
    for (int k = 0; k < kUnionEach; ++k) {
        const int at = blockIdx.x * kUnionWords + kUnionEach * warp + k;
        cls[k] = int(blockIdx.x) < a.n_counts && at < a.VW ? __ldg(p.c16 + int64_t(at) * 32 + lane) : uint32_t(p.K);  // (K: no class)
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
    if (int(blockIdx.x) >= a.n_counts) {
        half_row(a, int(blockIdx.x) - a.n_counts);
        return;
    }
    if (threadIdx.x < 32) sh[threadIdx.x] = 0;
    for (int c = 0; 32 * c < a.B; ++c) {
        const int row = 32 * c + lane;
        const uint32_t* m = class_mask + row * class_stride;
        __syncthreads();
        constexpr int kWarps = kUnionThreads / 32;
        for (int k0 = warp; k0 < p.KW; k0 += 4 * kWarps) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = row < a.B && k0 + kWarps * k < p.KW ? ld_after_wait(m + k0 + kWarps * k) : 0u;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k0 + kWarps * k < p.KW) table[32 * (k0 + kWarps * k) + lane] = warp_transpose32(w[k], lane);
        }
        __syncthreads();
        union_chunk(a, c, sh, masks, mask_stride, [&](int, int k) { return cls[k] < uint32_t(p.K) ? table[cls[k]] : 0u; });
    }
    union_finish(a, sh);
}

// Union of the rows' masks, 32 words by a block, and the masks turned from 32 tokens of a row to 32 rows of a token: a warp takes
// kUnionEach words, a lane a row. Blocks behind those take a row of hidden states.
__global__ void __launch_bounds__(kUnionThreads) k_head_union(const HeadStepArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
    if (int(blockIdx.x) >= a.n_counts) {
        half_row(a, int(blockIdx.x) - a.n_counts);
        return;
    }
    __shared__ uint32_t sh[32];
    if (threadIdx.x < 32) sh[threadIdx.x] = 0;
    __syncthreads();
    for (int c = 0; 32 * c < a.B; ++c) {
        const int row = 32 * c + lane;
        const bool has = row < a.B && step_row_part(a, row) >= 0;
        const uint32_t* p = a.mask + int64_t(row) * a.mask_stride;
        uint32_t w[kUnionEach];
#pragma unroll
        for (int k = 0; k < kUnionEach; ++k) {
            const int at = blockIdx.x * kUnionWords + kUnionEach * warp + k;
            w[k] = has && at < a.VW ? ld_after_wait(p + at) : 0u;
        }
        union_chunk(a, c, sh, nullptr, 0, [&](int, int k) { return warp_transpose32(w[k], lane); });
    }
    union_finish(a, sh);
}

// A union of most of the vocabulary is taken for all of it, in boxes of rows by tiled copies. bf16 weights come one by one at the same
// rate (one row of 128256 x 4096, 95 % allowed: 177 us, all of them 179); 4-bit ones take threads for it that otherwise turn weights
// into f16 (32 rows of the same, 70 %: 79 us, all 83; 58 %: 69 and 83; at 84 % one by one took 10 us longer than all).
__device__ __forceinline__ bool step_takes_all(const HeadStepArgs& a, uint32_t total, bool mx) {
    return int64_t(total) * 16 >= int64_t(a.V) * (mx ? 12 : 15);
}

// -inf for every score; those of allowed tokens are written over it. (Where all tokens are taken, the step writes every score.)
template <int DT>
__global__ void __launch_bounds__(256) k_head_fill(const HeadStepArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ uint32_t total;
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    uint32_t mine = 0;
    for (int i = threadIdx.x; i < a.n_counts; i += 256) mine += uint32_t(__ldcg(a.counts + i));
    mine = __reduce_add_sync(0xFFFFFFFFu, mine);
    if ((threadIdx.x & 31) == 0) atomicAdd(&total, mine);
    __syncthreads();
    if (step_takes_all(a, total, a.half)) return;
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
__device__ __forceinline__ void tma_load(uint32_t dst_smem, const void* tensor_map, int x, int y, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst_smem),
        "l"(tensor_map), "r"(x), "r"(y), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tma_load3(uint32_t dst_smem, const void* tensor_map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst_smem),
        "l"(tensor_map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// Until a counter in shared memory has come to `least` (a count, not a phase: who waits may have let some go by). About half a
// second at most; false: it has not.
__device__ __forceinline__ bool wait_count(const uint32_t* count, uint32_t least) {
    for (int it = 0; it < (1 << 22); ++it) {
        uint32_t v;
        asm volatile("ld.acquire.cta.shared::cta.u32 %0, [%1];" : "=r"(v) : "r"(smem_u32(count)) : "memory");
        if (v >= least) return true;
        if (it > 16) __nanosleep(100);
    }
    return false;
}

struct StepShared {
    uint64_t full[kStepStages], empty[kStepStages], sums_full[2], sums_empty[2], w_full[3], w_empty[3], drained;
    uint32_t tmem;
    uint32_t valid[kStepRows / 32];  // rows that have a partition
    int32_t entries, is_last, stages;
    float back[kStepRowsMx];         // 4-bit heads: what brings a row's products back
    uint32_t largest[2][128];        // ... and the largest scale byte of the rows of a tile's tokens
    uint32_t largest_tiles[4];       // how many tiles' are there, by the quarters of a tile
    int32_t scan[kStepWarpsMx];
    int32_t list[kStepShare];        // the block's tokens, ascending
    union alignas(16) {
        int2 entry[kStepShare + 1];  // counted pieces that hold some of them: number, tokens in front of it
        float turn[4][32 * 33];      // scores on their way from a lane a token to a lane a row
        Partial state[4][kStepRows];
    };
};

// The block's share of the union: its n tokens to sh.list; the longest share of any block to *most, whether all tokens are taken
// to *all. All threads; ends with a barrier.
template <bool MX, int THREADS>
__device__ __forceinline__ int step_share(const HeadStepArgs& a, StepShared& sh, int share, int shares, bool* all, int* most) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) sh.entries = 0;
    const int strip = (a.n_counts + THREADS - 1) / THREADS, c0 = min(tid * strip, a.n_counts), c1 = min(c0 + strip, a.n_counts);
    int mine = 0;
    for (int i = c0; i < c1; ++i) mine += __ldcg(a.counts + i);
    int before = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xFFFFFFFFu, before, d);
        if (lane >= d) before += o;
    }
    if (lane == 31) sh.scan[warp] = before;
    __syncthreads();
    before -= mine;
    uint32_t total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        const int o = sh.scan[w];
        if (w < warp) before += o;
        total += o;
    }
    *all = step_takes_all(a, total, MX);
    if (*all) total = a.V;
    // equal parts, the first `more` of them a token longer
    const uint32_t each = total / uint32_t(shares), more = total - each * uint32_t(shares);
    *most = int(each + (more > 0));
    const int lo = int(each * uint32_t(share) + min(uint32_t(share), more)), hi = lo + int(each + (uint32_t(share) < more));
    if (*all) {
        for (int i = tid; i < hi - lo; i += THREADS) sh.list[i] = lo + i;
    } else if (lo < hi) {  // (the same for every thread)
        for (int i = c0; i < c1; ++i) {
            const int n = strip == 1 ? mine : __ldcg(a.counts + i);
            if (n > 0 && before < hi && before + n > lo) sh.entry[atomicAdd(&sh.entries, 1)] = make_int2(i, before);
            before += n;
        }
        __syncthreads();
        for (int e = warp; e < sh.entries; e += THREADS / 32) {
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

// The state of one row from every block's ([blocks, B] in a.part), and the row's results; a warp.
__device__ __forceinline__ void step_finish_row(const HeadStepArgs& a, int row, int blocks, int lane) {
    const int part = step_row_part(a, row);
    if (part < 0) return;
    const int32_t* reps = a.parts[part].trep;  // (asked for before the states)
    Partial p = partial_empty();
    for (int i = lane; i < blocks; i += 160) {  // (five at a time: what 148 blocks have, in one go)
        int4 v[5];
#pragma unroll
        for (int k = 0; k < 5; ++k)
            v[k] = i + 32 * k < blocks ? __ldcg(reinterpret_cast<const int4*>(&a.part[int64_t(i + 32 * k) * a.B + row]))
                                       : make_int4(__float_as_int(-INFINITY), 0, kNoPos, 0);
#pragma unroll
        for (int k = 0; k < 5; ++k) partial_merge(p.m, p.s, p.pos, __int_as_float(v[k].x), __int_as_float(v[k].y), v[k].z);
    }
    const float top = redux_max(p.m), ref = fmaxf(top, kRefFloor);
    float s = p.s * ex2f((fmaxf(p.m, kRefFloor) - ref) * kLog2e);
    int pos = p.m == top ? p.pos : kNoPos;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    pos = __reduce_min_sync(0xFFFFFFFFu, pos);
    if (lane) return;
    const bool any = uint32_t(pos) < uint32_t(a.V);  // (also where a wait ran out and there are no states)
    const float log_sum = logf(s);
    a.argmax[row] = any ? pos : -1;
    if (a.rep) a.rep[row] = any ? reps[pos] : -1;
    if (a.logp) a.logp[row] = s > 0.f ? -log_sum : -INFINITY;
    if (a.lse) a.lse[row] = s > 0.f ? top + log_sum : -INFINITY;
    if (!any) atomicAdd(a.status, 1);
}

__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}

// Where the sums of a warp's 32 tokens are: `cuts` pieces in tensor memory, cut_step columns apart, and, where they are a later portion
// of a row, what the portions before came to: in tensor memory too, or (4-bit heads, whose weights need the room) in shared memory,
// a lane a word, a column every 512 bytes.
struct StepSums {
    uint32_t at, cut_step, kept;
    float* kept_shared;
    int cuts;
    bool later;
};
// Sixteen columns of them from `column` on.
template <bool MX>
__device__ __forceinline__ void step_sums(const StepSums& p, int column, uint32_t (&v)[16]) {
    __syncwarp();
    tmem_ld16(p.at + column, v);
    tmem_wait_ld();
#pragma unroll 1
    for (int i = MX ? 1 : 1 - int(p.later); i < p.cuts; ++i) {
        uint32_t u[16];
        tmem_ld16(i == 0 ? p.kept + column : p.at + i * p.cut_step + column, u);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + __uint_as_float(u[j]));
    }
    if (MX)  // (not a branch around the loads: with one the kernel takes 80 registers and spills, 86 -> 98 us for 32 rows)
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + (p.later ? p.kept_shared[(column + j) * 128] : 0.f));
}
// A portion that is not a row's last, put with those before it.
template <bool MX>
__device__ __forceinline__ void step_keep(const StepSums& p, int columns) {
#pragma unroll 1
    for (int h = 0; h < columns; h += 16) {
        uint32_t v[16];
        step_sums<MX>(p, h, v);
        if (MX) {
#pragma unroll
            for (int j = 0; j < 16; ++j) p.kept_shared[(h + j) * 128] = __uint_as_float(v[j]);
        } else {
            __syncwarp();
            tmem_st16(p.kept + h, v);
        }
    }
    if (!MX) asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// The scores of a warp's 32 tokens under the rows of the batch: a lane has a token, a column is a row; by way of shared memory a
// lane has a row (32 c + lane) and all of the tokens, and keeps that row's state. The loops stay short: a block comes here four
// times, and straight code cost more in instruction fetches than it saved.
template <bool MX, int W>
__device__ __forceinline__ void step_scores(const HeadStepArgs& a, StepShared& sh, int quad, float back, const int32_t* list, int tokens,
                                            bool all, const StepSums& sums, const uint32_t (&bits)[W], Partial (&state)[W],
                                            int lane) {
    float* turn = sh.turn[quad];
#pragma unroll
    for (int c = 0; c < W; ++c) {
        if (32 * c >= a.B) break;
        const int rows = min(32, a.B - 32 * c);
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            if (32 * c + h >= a.B) break;  // (of rows that are not there nothing is read below)
            uint32_t v[16];
            step_sums<MX>(sums, 32 * c + h, v);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                float z = __uint_as_float(v[j]);
                if (MX) {  // the smaller power first: large hidden states and small weights, or the other way round, meet in the middle
                    const float x = sh.back[32 * c + h + j];
                    z = z * (back < x ? back : x) * (back < x ? x : back);  // (a scale byte of 255 stays NaN)
                }
                turn[(h + j) * 33 + lane] = (bits[c] >> (h + j)) & 1u ? z : -INFINITY;
            }
        }
        const uint32_t has = warp_transpose32(bits[c], lane);
        __syncwarp();
        if (a.logits) {
            const uint32_t write = all ? (lane < tokens ? sh.valid[c] : 0u) : bits[c];
            const int64_t at = 32 * c * a.logits_stride + (lane < tokens ? list[lane] : 0);
            if (a.logits_dtype == kBF16) {
                uint16_t* p = static_cast<uint16_t*>(a.logits) + at;
#pragma unroll 4
                for (int j = 0; j < rows; ++j, p += a.logits_stride)
                    if ((write >> j) & 1u) *p = uint16_t(bf16_pair(turn[j * 33 + lane], 0.f));
            } else {
                float* p = static_cast<float*>(a.logits) + at;
#pragma unroll 4
                for (int j = 0; j < rows; ++j, p += a.logits_stride)
                    if ((write >> j) & 1u) *p = turn[j * 33 + lane];
            }
        }
        const float* mine = turn + lane * 33;
        float m = -INFINITY;
        int at = __ffs(has) - 1;
#pragma unroll 8
        for (int j = 0; j < 32; ++j) {
            const float z = mine[j];
            at = z > m ? j : at;
            m = fmaxf(m, z);
        }
        const float ref = fmaxf(m, kRefFloor);
        float s[4] = {};
#pragma unroll 2
        for (int j = 0; j < 32; j += 4)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] += ex2f((mine[j + k] - ref) * kLog2e);
        if (has) partial_merge(state[c].m, state[c].s, state[c].pos, m, (s[0] + s[1]) + (s[2] + s[3]), list[at]);
        __syncwarp();
    }
}

// 4-bit weights in tensor memory are f16, relative to the largest scale of their row, which becomes 2^13: e2m1 numbers times 2^13 (6 of
// them are below f16's largest number) down to 2^-23 are exact in f16, and of a weight whose scale is below that 6 * 2^-38 of the largest
// scale is lost at most. One conversion and one product for two weights; going to bf16 by shifts, masks and products takes 23
// instructions for eight (32 rows of 128256 x 4096: 163 us, 130).
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ void mx_word(uint32_t w, uint32_t scale, uint32_t* out) {
    uint32_t t[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(t[0]), "=r"(t[1]), "=r"(t[2]), "=r"(t[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = mul_f16x2(t[i], scale);
}
// 2^(byte - largest + kMxTop) twice, as f16; `normal`: none is below 2^-14
constexpr int kMxTop = 13;
__device__ __forceinline__ uint32_t mx_scale_pair(uint32_t byte, uint32_t largest, bool normal) {
    const int e = int(byte) - int(largest) + kMxTop + 15;  // exponent field of a normal number
    if (normal) return uint32_t(e) * 0x04000400u;
    const uint32_t b = e >= 1 ? uint32_t(e) << 10 : e >= -9 ? 1u << (9 + e) : 0u;
    return b | b << 16;
}
// Largest scale byte of a row of n blocks (rows start on 16 bytes).
__device__ __forceinline__ uint32_t mx_largest(const uint8_t* scales, int n) {
    uint32_t top = 0;
#pragma unroll 4
    for (int i = 0; i < n; i += 16) {
        const uint4 v = ld_after_wait(reinterpret_cast<const uint4*>(scales + i));
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int left = n - i - 4 * k;
            top = __vmaxu4(top, left >= 4 ? w[k] : left <= 0 ? 0u : w[k] & ((1u << (8 * left)) - 1u));
        }
    }
    top = __vmaxu4(top, top >> 16);
    return max(top & 255u, (top >> 8) & 255u);
}
__device__ __forceinline__ void mma_f16_from_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
        : "memory");
}

template <bool MX>
constexpr int kStepTiles = MX ? 1 : 2;  // tiles that share a stage at most

// How a block's stages are laid out: for blocks of more than 128 tokens and up to 32 rows two tiles of 128 side by side, which share
// the hidden states; otherwise one (of a 4-bit head they come one by one through tensor memory), of as many rows as there are tokens
// (rounded up to 32) and so many more atoms of them. A product takes 128 rows all the same: what it reads behind the rows that are
// there gives sums that nobody reads.
//
// The products' sums in tensor memory are cut off towards zero at every addition (measured: -1e-9 of the score per element of the
// row, 4e-6 for 4096, ten times what sums that are rounded come to), so that a row's k is cut in `cuts` pieces with sums of their own,
// as many as there is room for, which are added up, and rounded, when they are read. Pieces of more than 1024 elements are not
// taken: a longer row comes in portions of that many pieces, one portion's sums being read while the next one's are made (scores of
// positive products from 4096 to 65536 elements: off by 1.7e-6, 2.2e-6 at most). From 4 bits, whose products have ten bits and lose
// less, 2048 (off by 5e-7, 9e-7 at most; pieces of 1024 leave 1.5e-7, but 64 rows of 128256 x 4096 then take 122 us instead of 113).
template <bool MX>
constexpr int kStepCut = MX ? 2048 / 256 : 1024 / 64;  // atoms
struct StepLayout {
    int tiles, rows, atoms, steps, stages, cuts, cut_atoms;
    int portions, portion_steps, last_cuts;
    uint32_t x_at, bytes, kept;
};
template <bool MX>
__device__ __forceinline__ StepLayout step_layout(const HeadStepArgs& a, int most) {
    constexpr int X = MX ? 4 : 1;  // atoms of hidden states to an atom of weights
    constexpr int kColumns = MX ? 128 : 512, kCut = kStepCut<MX>;
    StepLayout l;
    l.tiles = most > 128 && a.N <= 32 ? kStepTiles<MX> : 1;
    l.rows = most > 128 ? 128 * l.tiles : (max(most, 1) + 31) & ~31;
    const int wide = l.tiles * a.N;
    int room = kColumns / (2 * wide);
    l.cut_atoms = room >= 16 ? (a.row_atoms + 15) >> 4 : room >= 8 ? (a.row_atoms + 7) >> 3 : room >= 4 ? (a.row_atoms + 3) >> 2 : room >= 2 ? (a.row_atoms + 1) >> 1 : a.row_atoms;
    l.atoms = 1;
    int shift = 0;
    while (!MX && shift < 3 && l.atoms < a.row_atoms && 2 * l.atoms * (l.rows + X * a.N) * kStepAtom <= (48u << 10)) {
        l.atoms *= 2;
        ++shift;
    }
    l.steps = (a.row_atoms + l.atoms - 1) >> shift;
    l.x_at = uint32_t(l.atoms) * l.rows * kStepAtom;
    l.bytes = l.x_at + uint32_t(l.atoms) * X * a.N * kStepAtom;
    uint32_t smem = uint32_t(a.smem);
    if (l.cut_atoms <= kCut) {
        l.cuts = l.last_cuts = (a.row_atoms + l.cut_atoms - 1) / l.cut_atoms;
        l.portions = 1;
        l.portion_steps = l.steps;
        l.kept = 0;
    } else {
        // (portions end with a stage: kCut is a multiple of a stage's atoms)
        if (MX) smem -= uint32_t(wide) * 512;
        else room = (kColumns - wide) / (2 * wide);
        l.cut_atoms = kCut;
        l.cuts = room;
        l.portions = (a.row_atoms + room * kCut - 1) / (room * kCut);
        l.portion_steps = (room * kCut) >> shift;
        l.last_cuts = (a.row_atoms - (l.portions - 1) * room * kCut + kCut - 1) / kCut;
        l.kept = MX ? smem : uint32_t(2 * room * wide);
    }
    l.stages = min(kStepStages, int(smem / l.bytes));
    return l;
}

template <bool MX>
__global__ void __launch_bounds__((MX ? kStepWarpsMx : kStepWarps) * 32, 1)
    k_head_step(const __grid_constant__ HeadStepArgs a, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                const __grid_constant__ CUtensorMap map_box) {
    constexpr int kThreads = (MX ? kStepWarpsMx : kStepWarps) * 32, X = MX ? 4 : 1, W = (MX ? kStepRowsMx : kStepRows) / 32;
    constexpr int T = kStepTiles<MX>;
    extern __shared__ char smem_raw[];
    __shared__ __align__(16) StepShared sh;
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStepStages; ++i) mbar_init(&sh.empty[i], MX ? 1 + 4 : 1);  // the products, and the warps that take weights apart
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.sums_full[i], 1);
            mbar_init(&sh.sums_empty[i], 4);
        }
        for (int i = 0; i < 3; ++i) {
            mbar_init(&sh.w_full[i], 4);
            mbar_init(&sh.w_empty[i], 1);
        }
        mbar_init(&sh.drained, 1);
        for (int i = 0; i < 4; ++i) sh.largest_tiles[i] = 0;
        mbar_init_fence();
        prefetch_tensor_map(&map_x);
        prefetch_tensor_map(&map_w);
        prefetch_tensor_map(&map_box);
    }
    if (warp == 2) tmem_alloc<1>(&sh.tmem, 512);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (threadIdx.x < kStepRows) {
        const bool v = int(threadIdx.x) < a.B && step_row_part(a, threadIdx.x) >= 0;
        const uint32_t w = __ballot_sync(0xFFFFFFFFu, v);
        if (lane == 0) sh.valid[warp] = w;
    }
    if (MX && int(threadIdx.x) < a.B) sh.back[threadIdx.x] = ld_after_wait(a.back + threadIdx.x);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = sh.tmem;
    bool ok = true;
    int failed = 0;
    int stage = 0, groups_done = 0;
    uint32_t phase = 0, set_phases = 0;
    Partial state[W];
#pragma unroll
    for (int c = 0; c < W; ++c) state[c] = partial_empty();
    for (int round = 0; round < a.rounds; ++round) {
        const int shares = a.rounds * gridDim.x;
        bool all;
        int most;
        const int n = step_share<MX, kThreads>(a, sh, round * gridDim.x + blockIdx.x, shares, &all, &most);
        const StepLayout l = step_layout<MX>(a, most);  // (the same in every round, as is `all`)
        if (round == 0) {
            if (threadIdx.x == 0) {
                sh.stages = l.stages;
                for (int i = 0; i < kStepStages; ++i) mbar_init(&sh.full[i], all ? 1 : 1 + 256);  // ... and every thread that fetches weights
                mbar_init_fence();
            }
            __syncthreads();
        }
        const int per_group = 128 * l.tiles, groups = (n + per_group - 1) / per_group;
        const int sets = all ? 3 : 2;  // of four warps that take weights apart: with nothing to fetch, there are four more
        int set = 0;
        // the hook: nothing is done with the first stages asked for
        const int asked_steps = a.expire ? min(l.steps, l.stages) : l.steps;
        if (a.expire) ok = warp == 0 || (warp >= 8 && warp < 16 && !all);
        auto next = [&] {
            if (++stage == l.stages) {
                stage = 0;
                phase ^= 1;
            }
        };
        if (warp == 0) {
            for (int g = 0; g < groups && ok; ++g) {
                // Where the tiled copies bring the weights too: whole tiles by one copy each (a copy takes some 130 cycles to go out,
                // whatever it brings up to 4 KB), the rest in small boxes.
                const int rows = all ? min(n - g * per_group, per_group) : 0, token = all ? sh.list[0] + g * per_group : 0;
                int large = rows / 128, small = (rows - 128 * large + kStepBox - 1) / kStepBox;
                if (small == 128 / kStepBox) {
                    ++large;
                    small = 0;
                }
                for (int s = 0; s < asked_steps; ++s) {
                    const int first = s * l.atoms, atoms = min(l.atoms, a.row_atoms - first);
                    if (!ring_wait(&sh.empty[stage], phase ^ 1)) {
                        ok = false;
                        break;
                    }
                    const uint32_t at = smem + uint32_t(stage) * l.bytes;
                    if (elect_one()) {
                        mbar_expect_tx(&sh.full[stage], uint32_t(atoms) * (X * a.N + large * 128 + small * kStepBox) * kStepAtom);
                        for (int p = 0; p < atoms; ++p) {
                            const int x = (first + p) * (MX ? 128 : 64);
                            uint32_t to = at + uint32_t(p * l.rows) * kStepAtom;
                            for (int i = 0; i < large; ++i, to += kStepTile) tma_load(to, &map_w, x, token + 128 * i, &sh.full[stage]);
                            for (int i = 0; i < small; ++i, to += kStepBox * kStepAtom)
                                tma_load(to, &map_box, x, token + 128 * large + i * kStepBox, &sh.full[stage]);
                            to = at + l.x_at + uint32_t(p * X * a.N) * kStepAtom;
                            if (MX) tma_load3(to, &map_x, 0, 0, (first + p) * X, &sh.full[stage]);
                            else tma_load(to, &map_x, x, 0, &sh.full[stage]);
                        }
                    }
                    __syncwarp();
                    next();
                }
                if (a.expire) ok = false;
            }
        } else if (warp == 1) {
            const uint32_t idesc = (MX ? kMmaF16Desc<128, 0, false, false> : kMmaBf16Desc<128, 0, false, false>) | uint32_t(a.N / 8) << 17;
            const uint32_t x_step = uint32_t(a.N) * kStepAtom >> 4, w_step = uint32_t(l.rows) * kStepAtom >> 4;
            for (int g = 0; g < groups && ok; ++g) {
                const int tiles = min(l.tiles, (n - g * per_group + 127) / 128);
                int it = (groups_done + g) * l.portions - 1, left = 0;  // portion, stages left of it
                uint32_t d0 = 0;
                int in_cut = 0;  // atoms of the cut that are through
                for (int s = 0; s < l.steps && ok; ++s) {
                    if (left-- == 0) {
                        if (s > 0) {
                            if (elect_one()) mma_commit<1>(&sh.sums_full[it & 1]);
                            __syncwarp();
                        }
                        ++it;
                        left = l.portion_steps - 1;
                        if (!ring_wait(&sh.sums_empty[it & 1], ((it >> 1) & 1) ^ 1)) {
                            ok = false;
                            break;
                        }
                        tmem_fence_after();
                        d0 = tmem + uint32_t(it & 1) * l.cuts * l.tiles * a.N;
                        in_cut = 0;
                    }
                    if (!ring_wait(&sh.full[stage], phase)) {
                        ok = false;
                        break;
                    }
                    // (weights were written as ordinary shared memory: the products read it another way)
                    if (!all) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    tmem_fence_after();
                    const int atoms = min(l.atoms, a.row_atoms - s * l.atoms);
                    const uint64_t dw = mma_desc<false>(smem + uint32_t(stage) * l.bytes);
                    const uint64_t dx = mma_desc<false>(smem + uint32_t(stage) * l.bytes + l.x_at);
                    if (MX) {
                        if (ok && !ring_wait(&sh.w_full[set], (set_phases >> set) & 1)) ok = false;
                        tmem_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                mma_f16_from_tmem(d0, tmem + 128 * (set + 1) + 8 * j, dx + j / 4 * x_step + (j & 3) * kDescStep16<false>, idesc,
                                                  in_cut > 0 || j > 0);
                            mma_commit<1>(&sh.w_empty[set]);
                        }
                        __syncwarp();
                        set_phases ^= 1u << set;
                        if (++set == sets) set = 0;
                        if (elect_one()) mma_commit<1>(&sh.empty[stage]);
                    } else if (elect_one()) {
                        uint32_t d = d0;
                        int in = in_cut;
                        for (int p = 0; p < atoms; ++p) {
                            for (int t = 0; t < tiles; ++t)
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    mma_f16<1>(d + t * a.N, dw + p * w_step + t * (kStepTile >> 4) + j * kDescStep16<false>,
                                               dx + p * x_step + j * kDescStep16<false>, idesc, in > 0 || j > 0);
                            if (++in == l.cut_atoms) {
                                in = 0;
                                d += l.tiles * a.N;
                            }
                        }
                        mma_commit<1>(&sh.empty[stage]);
                    }
                    __syncwarp();
                    for (in_cut += atoms; in_cut >= l.cut_atoms; in_cut -= l.cut_atoms) d0 += l.tiles * a.N;
                    next();
                }
                if (elect_one()) mma_commit<1>(&sh.sums_full[it & 1]);
                __syncwarp();
            }
        } else if (MX && (warp >= 16 || (all && warp >= 8 && warp < 12))) {
            // a thread a token, a set of warps every second or third atom
            set = warp >= 16 ? (warp - 16) >> 2 : 2;
            const int row = (warp & 3) * 32 + lane, blocks = a.bytes / 16;
            const uint32_t to = tmem + 128 * (set + 1) + (uint32_t((warp & 3) * 32) << 16);
            auto number = [&](int g) { return min(g * 128 + row, n - 1); };
            auto scales_at = [&](int g, int s) {  // of an atom: eight
                return *reinterpret_cast<const uint2*>(a.scales + int64_t(sh.list[number(g)]) * a.scale_stride + 8 * s);
            };
            int g = 0, s = set, at_stage = stage + set, group = -1;
            uint32_t at_phase = phase, largest = 0;
            auto settle = [&] {
                while (s >= l.steps) {
                    s -= l.steps;
                    ++g;
                }
                while (at_stage >= l.stages) {
                    at_stage -= l.stages;
                    at_phase ^= 1;
                }
            };
            settle();
            uint2 scale = g < groups ? scales_at(g, s) : make_uint2(0, 0);
            while (g < groups && ok) {
                const int atom = s, here = at_stage;
                const uint32_t here_phase = at_phase;
                if (g != group) {
                    group = g;
                    const int it = groups_done + g;
                    if (!wait_count(&sh.largest_tiles[warp & 3], uint32_t(it) + 1)) {
                        ok = false;
                        break;
                    }
                    largest = sh.largest[it & 1][row];
                }
                const uint32_t least = (largest > 14 + kMxTop ? largest - (14 + kMxTop) : 0u) * 0x01010101u;
                uint2 eight = scale;
                s += sets;
                at_stage += sets;
                settle();
                if (g < groups) scale = scales_at(g, s);  // (comes while this atom is taken apart)
                const int left = blocks - 8 * atom;  // (behind the row there is no scale, and the weights are zeros)
                if (left < 8) {
                    const uint64_t there = (uint64_t(1) << (8 * left)) - 1, fill = uint64_t(largest) * 0x0101010101010101ull;
                    const uint64_t e = ((uint64_t(eight.y) << 32 | eight.x) & there) | (fill & ~there);
                    eight = make_uint2(uint32_t(e), uint32_t(e >> 32));
                }
                const bool normal = !__any_sync(0xFFFFFFFFu, (__vcmpltu4(eight.x, least) | __vcmpltu4(eight.y, least)) != 0);
                // The products of this set's atom before are through, so all atoms up to that one are: the stage's barrier cannot be a
                // phase behind (there are at least as many stages as sets), and its parity says what it seems to.
                if (!ring_wait(&sh.w_empty[set], (set_phases & 1) ^ 1) || !ring_wait(&sh.full[here], here_phase)) {
                    ok = false;
                    break;
                }
                tmem_fence_after();
                const uint32_t at = smem + uint32_t(here) * l.bytes + uint32_t(min(row, l.rows - 1)) * kStepAtom;
                auto fetch = [&](int k, uint32_t (&w)[4]) {
                    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                                 : "r"(at + (uint32_t(k ^ (row & 7)) << 4)));
                };
                uint32_t w[4];
                fetch(0, w);
#pragma unroll 1
                for (int b = 0; b < 8; ++b) {
                    uint32_t v[16], after[4];
                    fetch((b + 1) & 7, after);
                    const uint32_t sc = mx_scale_pair(eight.x & 255u, largest, normal);
                    eight.x = __funnelshift_r(eight.x, eight.y, 8);
                    eight.y >>= 8;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        mx_word(w[i], sc, v + 4 * i);
                        w[i] = after[i];
                    }
                    __syncwarp();
                    tmem_st16(to + 16 * b, v);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.w_full[set]);
                    mbar_arrive(&sh.empty[here]);
                }
                set_phases ^= 1;
            }
            // (every role goes through all of the round's stages)
            for (int i = 0; i < groups * l.steps; ++i) next();
        } else if (warp >= 8) {
            // eight lanes bring the 128 bytes of a row's atom, the eight warps 32 rows at a time
            const int chunk = lane & 7, row = (warp - 8) * 4 + (lane >> 3);
            for (int g = all ? groups : 0; g < groups && ok; ++g) {  // (tiled copies bring them where all are taken)
                const int rows = min(n - g * per_group, per_group);
                const char* from[4 * T];
#pragma unroll
                for (int i = 0; i < 4 * T; ++i)
                    if (i * 32 < rows)  // (rows behind the last one are filled up with it)
                        from[i] = static_cast<const char*>(a.weight) +
                                  int64_t(sh.list[min(g * per_group + i * 32 + row, n - 1)]) * a.row_bytes + chunk * 16;
                for (int s = 0; s < asked_steps; ++s) {
                    if (!ring_wait(&sh.empty[stage], phase ^ 1)) {
                        ok = false;
                        break;
                    }
                    const int first = s * l.atoms, atoms = min(l.atoms, a.row_atoms - first);
                    uint32_t to = smem + uint32_t(stage) * l.bytes + uint32_t(row) * kStepAtom + uint32_t((chunk ^ (row & 7)) << 4);
                    for (int p = 0; p < atoms; ++p, to += uint32_t(l.rows) * kStepAtom) {
                        const int off = (first + p) * int(kStepAtom);
                        const bool have = off + chunk * 16 < a.bytes;
#pragma unroll
                        for (int i = 0; i < 4 * T; ++i) {
                            if (i * 32 >= rows) break;
                            copy16(to + i * 32 * kStepAtom, have ? from[i] + off : from[i] - chunk * 16, have);
                        }
                    }
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&sh.full[stage])) : "memory");
                    next();
                }
                if (a.expire) ok = false;
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        } else if (warp >= 4) {
            const int quad = warp & 3;
            // 4-bit heads: the largest scales of a tile's rows are looked for a tile ahead
            uint32_t largest = 0, largest_next = 0;
            auto find_largest = [&](int g) {
                if (g >= groups) return;
                const int at = g * 128 + quad * 32 + lane, slot = (groups_done + g) & 1;
                largest_next = mx_largest(a.scales + int64_t(sh.list[min(at, n - 1)]) * a.scale_stride, a.bytes / 16);
                sh.largest[slot][quad * 32 + lane] = largest_next;
                __syncwarp();
                if (lane == 0)
                    asm volatile("st.release.cta.shared::cta.u32 [%0], %1;" ::"r"(smem_u32(&sh.largest_tiles[quad])), "r"(groups_done + g + 1)
                                 : "memory");
            };
            if (MX) find_largest(0);
            for (int g = 0; g < groups && ok; ++g) {
                largest = largest_next;
                if (MX) find_largest(g + 1);
                uint32_t bits[T][W];
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const int at = g * per_group + t * 128 + quad * 32 + lane;
                    const bool have = t < l.tiles && at < n;
                    const int token = have ? sh.list[at] : 0;
#pragma unroll
                    for (int c = 0; c < W; ++c) bits[t][c] = have && 32 * c < a.B ? ld_after_wait(a.bits + int64_t(c) * a.VW * 32 + token) : 0u;
                }
                int it = (groups_done + g) * l.portions;
                auto sums_of = [&](int t, bool last) {
                    const uint32_t lanes = uint32_t(quad * 32) << 16;
                    return StepSums{tmem + uint32_t((it & 1) * l.cuts * l.tiles + t) * a.N + lanes, uint32_t(l.tiles) * a.N,
                                    tmem + l.kept + uint32_t(t) * a.N + lanes,
                                    reinterpret_cast<float*>(smem_raw + (smem - smem_u32(smem_raw)) + l.kept) + quad * 32 + lane,
                                    last ? l.last_cuts : l.cuts, it > (groups_done + g) * l.portions};
                };
                auto wait_sums = [&] {
                    ok = ring_wait(&sh.sums_full[it & 1], (it >> 1) & 1);
                    tmem_fence_after();
                    return ok;
                };
                auto release = [&] {
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.sums_empty[it & 1]);
                };
#pragma unroll 1
                for (int p = 1; p < l.portions && wait_sums(); ++p, ++it) {
#pragma unroll
                    for (int t = 0; t < T; ++t)
                        if (t < l.tiles && g * per_group + t * 128 + quad * 32 < n) step_keep<MX>(sums_of(t, false), a.B);
                    release();
                }
                if (!ok || !wait_sums()) break;
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const int at = g * per_group + t * 128 + quad * 32;
                    if (t < l.tiles && at < n)
                        step_scores<MX>(a, sh, quad, MX ? mx_scale(largest) * (1.f / (1 << kMxTop)) : 1.f, sh.list + at, n - at, all,
                                        sums_of(t, true), bits[t], state, lane);
                }
                release();
            }
        }
        __syncwarp();
        groups_done += groups;
        failed = __syncthreads_or(!ok);
        if (failed) break;
    }
    if (failed) {
        // A wait ran out: the copies in flight and the products get the same bounded time once more (other copies to shared memory have
        // been waited for), then the block leaves with what it has. (In the loop this took the 4-bit kernel 80 registers and spills.)
        if (threadIdx.x == 0) {
            atomicExch(a.status + 3, 1);
            for (int i = 0; i < sh.stages; ++i) mbar_wait(&sh.full[i], i < stage ? phase : phase ^ 1);  // (one never asked for counts as through)
        }
        __syncwarp();
        if (warp == 1) {
            if (elect_one()) mma_commit<1>(&sh.drained);
            __syncwarp();
            mbar_wait(&sh.drained, 0);
        }
        __syncwarp();
    }
    // the four warps' states to one, out to the others' and, in the last block to come here, to the results
    if (warp >= 4 && warp < 8) {
#pragma unroll
        for (int c = 0; c < W; ++c) sh.state[warp & 3][32 * c + lane] = state[c];
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 2) tmem_free<1>(tmem, 512);
    if (int(threadIdx.x) < a.B) {
        Partial p = sh.state[0][threadIdx.x];
#pragma unroll
        for (int q = 1; q < 4; ++q) {
            const Partial o = sh.state[q][threadIdx.x];
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
    for (int row = warp; row < a.B; row += kThreads / 32) step_finish_row(a, row, gridDim.x, lane);
}

// Results of rows whose states are those of `states` pieces of the vocabulary, a warp a row.
__global__ void __launch_bounds__(256) k_head_step_finish(const HeadStepArgs a, int states) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row < a.B) step_finish_row(a, row, states, threadIdx.x & 31);
}

}  // namespace cfgzip
