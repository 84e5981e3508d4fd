// The context behind the C ABI and what every call does with it: device, launches, partitions, row plans.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <utility>
#include <vector>

#include "cfgzip.h"
#include "cfgzip_device.cuh"

namespace cfgzip {

struct Part {
    bool live = false;
    int32_t V = 0, K = 0, KW = 0, VW = 0;
    void* block = nullptr;  // one device allocation holding every table of the partition
    size_t block_bytes = 0;
    PartDev dev{};
    std::vector<int32_t> sizes;  // host copy of the class sizes (cfgzip_choose_mode)
};

}  // namespace cfgzip

struct cfgzip_ctx {
    int device = 0;
    int sm_count = 0;
    int smem_optin = 0;
    std::vector<cfgzip::Part> parts;
    void* spare_block = nullptr;  // memory of the partition released last, for the next one loaded (given back with the context)
    size_t spare_bytes = 0;
    cfgzip::PartDev* d_parts = nullptr;
    cfgzip::Partial* d_partials = nullptr;
    unsigned int* d_tickets = nullptr;  // reserved_rows entries
    int32_t* d_status = nullptr;        // 4 counters, and 4 that nobody reads (see uncounted)
    bool uncounted = false;             // set around a launch that repeats what another launch of the same call counts
    int32_t* d_group_part = nullptr;
    int32_t* d_group_rows = nullptr;
    int32_t* d_n_groups = nullptr;
    int32_t* d_group_w = nullptr;       // row batches in front of every group
    int32_t* d_row_mode = nullptr;      // automatic mode: which rows the class-list kernel has finished
    int32_t reserved_rows = 0;
    int32_t max_groups = 0;
    // staging for cfgzip_decode_step_host
    void* st_logits = nullptr;
    size_t st_logits_bytes = 0;
    uint32_t* st_cm = nullptr;
    size_t st_cm_bytes = 0;
    uint32_t* st_vm = nullptr;
    size_t st_vm_bytes = 0;
    int32_t* st_small = nullptr;  // row_part, argmax, rep, lse, logp_argmax: 5 arrays of st_rows
    int32_t st_rows = 0;
    int32_t* st_small_host = nullptr;  // pinned mirror of the four result arrays: the kernels write them there, or one copy does
    // pinned host buffers: copies in, the step, copies out run side by side
    cudaStream_t st_in = nullptr, st_out = nullptr;
    cudaEvent_t st_ready = nullptr, st_masks = nullptr, st_expanded = nullptr;
    std::vector<cudaEvent_t> st_chunk_in, st_chunk_done;
    int64_t launches = 0;
    std::vector<std::pair<const void*, size_t>> smem_allowed;  // kernels whose shared-memory limit has been raised, and to what
    // row plan kept by cfgzip_plan_rows (valid until anything overwrites the plan buffers or the partitions change)
    bool plan_valid = false;
    bool plan_in_use = false;  // set for the duration of a call that passed CFGZIP_ROWS_AS_PLANNED
    const int32_t* plan_row_part = nullptr;
    int32_t plan_B = 0, plan_V = 0;
    // tuning
    int32_t ctas_per_sm = 4;
    int32_t token_warps = 0;
    int32_t row_warps = 0;
    int32_t pdl = 1;
    bool pdl_now = true;      // set per call: programmatic dependent launch only pays for short kernels
    int cluster_now = 1;      // set around a launch: blocks per thread-block cluster
    int cluster_limit[cfgzip::kClusterMost + 1] = {};  // clusters of that many blocks that run side by side, a block to an SM
    int prefetch_items = 4;   // work items per warp of the pipelined kernel asked into the L2 before its wait
    int prefetch_min_mbytes = 48;  // ... for steps of at least this many megabytes of logits
    bool prefetch_now = false;     // set per call beside pdl_now
    int rotate = 1;           // the chunk deal of the pipelined kernel starts at another warp slot for every row batch
    // cuTensorMapEncodeTiled, looked up through the runtime (no link against the driver library)
    CUresult (*encode_tiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill) = nullptr;
    int32_t pipeline = 1;     // bulk-copy pipelined dense kernel for aligned logits
    int32_t tensor_map = 1;   // tiled 2-D copies for row batches that are consecutive rows
    int32_t pipe_warps = 16;
    int32_t pipe_depth = 2;
    bool pipe_depth_set = false;  // the knob was set: no automatic third stage
    int32_t waves = 1;        // pipelined kernel: blocks launched per resident block slot
    int32_t spread = 1;       // pad the shared memory of one-block-per-SM launches so that blocks cannot share an SM
    int32_t stage_alias = 0;  // 1: always lay the class-mask staging area over the rings (default: only where it buys warps)
    int32_t lane_octets = 0;  // bf16 pipelined kernel: octets per lane and row (0 = automatic, 1, 2)
    int32_t auto_permille = -1;  // automatic mode: groups that allow under this many thousandths of their tokens go to the
                                 // class lists; -1 = by element type (measured break-even: f32 40, bf16 10)
    int64_t auto_min_bytes = -1;  // automatic mode on device-resident masks: steps of at least this many bytes of logits let the
                                  // GPU choose (one more launch); -1 = never (dense): the choice from host masks costs nothing
    int32_t fold = 0;         // pipelined kernel: the last block of a row group writes the rows' results (one launch per step)
    int32_t one_launch = 1;   // short batches: the whole step in one launch (k_step_cluster); off once a knob shapes the streaming kernel
    int32_t expire_test = 0;  // test hook: the pipelined kernel reports its first completed wait as run out
};

namespace cfgzip {

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev == dev) prev = -1;  // nothing to put back
        else if (cudaSetDevice(dev) != cudaSuccess) ok = false;
    }
    ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

inline int ceil_div(int64_t a, int64_t b) { return int((a + b - 1) / b); }

inline int32_t* status_of(const cfgzip_ctx* ctx) { return ctx->d_status + (ctx->uncounted ? 4 : 0); }

template <typename... KArgs, typename... Args>
int launch(cfgzip_ctx* ctx, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream,
           Args&&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n_attr = 0;
    if (ctx->pdl == 2 || (ctx->pdl && ctx->pdl_now)) {
        attr[n_attr].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n_attr].val.programmaticStreamSerializationAllowed = 1;
        ++n_attr;
    }
    if (ctx->cluster_now > 1) {  // neighbouring blocks along x form a thread-block cluster
        attr[n_attr].id = cudaLaunchAttributeClusterDimension;
        attr[n_attr].val.clusterDim.x = unsigned(ctx->cluster_now);
        attr[n_attr].val.clusterDim.y = 1;
        attr[n_attr].val.clusterDim.z = 1;
        ++n_attr;
    }
    cfg.attrs = attr;
    cfg.numAttrs = unsigned(n_attr);
    if (cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...) != cudaSuccess) {
        cudaGetLastError();
        return CFGZIP_E_CUDA;
    }
    ctx->launches += 1;
    return CFGZIP_OK;
}

// More than 48 KB of dynamic shared memory has to be allowed once per kernel; it is allowed up to the device's limit, so that
// the limit another context may have set is never smaller, and remembered: asking the runtime on every step costs half a
// microsecond of host time. large_clusters: the kernel also comes in clusters of more than eight blocks.
template <typename K>
int ensure_smem(cfgzip_ctx* ctx, K kernel, size_t bytes, bool large_clusters = false) {
    if (bytes <= 48 * 1024 && !large_clusters) return CFGZIP_OK;
    const void* fn = reinterpret_cast<const void*>(kernel);
    for (const auto& k : ctx->smem_allowed)
        if (k.first == fn) return bytes <= k.second ? CFGZIP_OK : CFGZIP_E_CUDA;
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, fn) != cudaSuccess) {
        cudaGetLastError();
        return CFGZIP_E_CUDA;
    }
    const size_t most = size_t(ctx->smem_optin) - std::min(size_t(ctx->smem_optin), attr.sharedSizeBytes);
    if (bytes > most || cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, int(most)) != cudaSuccess ||
        (large_clusters && cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)) {
        cudaGetLastError();
        return CFGZIP_E_CUDA;
    }
    ctx->smem_allowed.emplace_back(fn, most);
    return CFGZIP_OK;
}

// Everything a per-step call needs to know about the partitions it may touch.
struct PartSet {
    int32_t V = 0, VW = 0, maxK = 0, maxKW = 0, n_live_same_v = 0;
    bool all_c16 = true;
    bool all_kw_mult4 = true;
};

inline int resolve_parts(cfgzip_ctx* ctx, cfgzip_part_id part0, bool mixed, PartSet* ps) {
    if (part0 < 0 || size_t(part0) >= ctx->parts.size() || !ctx->parts[size_t(part0)].live) return CFGZIP_E_RANGE;
    const Part& p0 = ctx->parts[size_t(part0)];
    ps->V = p0.V;
    ps->VW = p0.VW;
    if (!mixed) {
        ps->maxK = p0.K;
        ps->maxKW = p0.KW;
        ps->n_live_same_v = 1;
        ps->all_c16 = p0.dev.c16 != nullptr;
        ps->all_kw_mult4 = (p0.KW % 4) == 0;
        return CFGZIP_OK;
    }
    for (const Part& p : ctx->parts) {
        if (!p.live || p.V != p0.V) continue;
        ps->maxK = std::max(ps->maxK, p.K);
        ps->maxKW = std::max(ps->maxKW, p.KW);
        ps->n_live_same_v += 1;
        ps->all_c16 = ps->all_c16 && p.dev.c16 != nullptr;
        ps->all_kw_mult4 = ps->all_kw_mult4 && (p.KW % 4) == 0;
    }
    return CFGZIP_OK;
}

// A call may pass CFGZIP_ROWS_AS_PLANNED for its row -> partition vector: it then means the vector given to the
// last cfgzip_plan_rows, whose grouping is still in the plan buffers.
inline int resolve_row_part(cfgzip_ctx* ctx, cfgzip_part_id part0, const int32_t** row_part, int32_t B, bool* planned) {
    *planned = false;
    if (*row_part != CFGZIP_ROWS_AS_PLANNED) return CFGZIP_OK;
    if (!ctx) return CFGZIP_E_ARG;
    if (!ctx->plan_valid || ctx->plan_B != B || part0 < 0 || size_t(part0) >= ctx->parts.size() ||
        !ctx->parts[size_t(part0)].live || ctx->parts[size_t(part0)].V != ctx->plan_V)
        return CFGZIP_E_ARG;
    *row_part = ctx->plan_row_part;
    *planned = true;
    return CFGZIP_OK;
}

struct PlanUse {  // marks the kept plan as in use for the lifetime of a call
    cfgzip_ctx* ctx;
    PlanUse(cfgzip_ctx* c, bool planned) : ctx(c) { if (ctx) ctx->plan_in_use = planned; }
    ~PlanUse() { if (ctx) ctx->plan_in_use = false; }
};

}  // namespace cfgzip
