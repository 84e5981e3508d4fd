// Tensor-core building blocks of the head kernels: tcgen05 products with accumulators in tensor memory, operands brought to
// shared memory by tiled copies in the 128-byte swizzle, and the waits between them. Every wait is bounded (mbar_wait).
#pragma once

#include "cfgzip_device.cuh"

namespace cfgzip {

// ---- descriptors --------------------------------------------------------------------------------------------------------------
// Operand in shared memory, 128-byte swizzle, 16-bit elements. K-major: rows of 64 k (128 bytes), eight of them a 1024-byte
// group, groups 1024 bytes apart. MN-major: rows of 64 m (or n) per k, eight k a group, 64 k a block of 8192 bytes, then the
// next 64 m. Sixteen k further on is 32 bytes (K-major: the swizzle works on address bits) or two groups (MN-major).
template <bool MN>
__device__ __forceinline__ uint64_t mma_desc(uint32_t smem) {
    const uint64_t group = 1024 >> 4, block = MN ? 8192 >> 4 : 1;
    return uint64_t((smem & 0x3FFFFu) >> 4) | block << 16 | group << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
template <bool MN>
constexpr uint32_t kDescStep16 = MN ? 2048 >> 4 : 32 >> 4;

// bf16 x bf16 -> f32, M x N tile
template <int M, int N, bool A_MN, bool B_MN>
constexpr uint32_t kMmaBf16Desc = 1u << 4 | 1u << 7 | 1u << 10 | uint32_t(A_MN) << 15 | uint32_t(B_MN) << 16 | uint32_t(N / 8) << 17 |
                              uint32_t(M / 16) << 24;
// f16 x f16 -> f32
template <int M, int N, bool A_MN, bool B_MN>
constexpr uint32_t kMmaF16Desc = kMmaBf16Desc<M, N, A_MN, B_MN> & ~(1u << 7 | 1u << 10);

// ---- tensor memory ------------------------------------------------------------------------------------------------------------
template <int CTAS>
__device__ __forceinline__ void tmem_alloc(uint32_t* where, uint32_t columns) {  // by one warp (of each block of a pair)
    if (CTAS == 2)
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {
    if (CTAS == 2) {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
    } else {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
    }
}
// 32 columns of the warp's 32 lanes; complete after tmem_wait_ld
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
          "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
          "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(at));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// One lane of the (whole) warp. A loop that all of a warp runs, with only the instructions themselves under this, keeps
// descriptors in uniform registers: issued from a branch of one lane they are moved there every time, 200 cycles a product.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ int uniform_warp() { return __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0); }

// ---- products -----------------------------------------------------------------------------------------------------------------
template <int CTAS>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    if (CTAS == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
            : "memory");
}
// the barrier is arrived at (once) when the products issued so far by this thread are done; pairs: in both blocks
template <int CTAS>
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
    if (CTAS == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                     "h"(uint16_t(3))
                     : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// ---- copies -------------------------------------------------------------------------------------------------------------------
// A box into this block's shared memory, counted on a barrier of the pair's first block (its shared::cluster address).
__device__ __forceinline__ void tma_load_pair(uint32_t dst_smem, const void* tensor_map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            dst_smem),
        "l"(tensor_map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// ... where it is asked for: a branch around it in the loop over stages made all products 1 to 2 % slower (loss of 300 rows of 32000 x 2048 67 and 68 us)
__device__ __forceinline__ void tma_load_pair_if(bool asked, uint32_t dst_smem, const void* tensor_map, int x, int y, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t"
        "@p cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}" ::"r"(
            dst_smem),
        "l"(tensor_map), "r"(x), "r"(y), "r"(bar), "r"(uint32_t(asked))
        : "memory");
}
// An arrival that lets go of sums whose loads from tensor memory are complete (waited for): nothing else has to be seen by who waits, and
// a release would first wait for the warp's stores to global memory (gradient of the scores, 1000 tokens of 50021 x 1024: 96 against 86 us).
__device__ __forceinline__ void arrive_at_peer(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_tensor_map(const void* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// mbar_wait and mbar_wait_cluster for waits that are mostly over when they are asked for, as in a ring of stages: asked without a
// time limit such a wait takes 17 cycles, with one 117. Bounded all the same.
template <bool CLUSTER = false>
__device__ __forceinline__ bool ring_wait(uint64_t* bar, uint32_t parity) {
#pragma unroll 1
    for (int it = 0; it < 32; ++it) {
        uint32_t ok;
        if (CLUSTER)
            asm volatile(
                "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                : "=r"(ok)
                : "r"(smem_u32(bar)), "r"(parity)
                : "memory");
        else
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                         : "=r"(ok)
                         : "r"(smem_u32(bar)), "r"(parity)
                         : "memory");
        if (ok) return true;
    }
    return CLUSTER ? mbar_wait_cluster(bar, parity) : mbar_wait(bar, parity);
}

// Where a kernel stands in a ring of stages.
struct Ring {
    int stage = 0;
    uint32_t phase = 0;
    template <int STAGES>
    __device__ __forceinline__ void next() {
        if (++stage == STAGES) {
            stage = 0;
            phase ^= 1;
        }
    }
};

}  // namespace cfgzip
