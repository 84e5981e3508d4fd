// Log probabilities of given tokens, entropies and top alternatives from logits, and the gradient of the first two.
//
//   zt = z / T over the allowed tokens,  lse = log sum exp zt,  logp = zt[token] - lse,  entropy = lse - sum p zt
//   d_z = (d_logp ([t = token] - p) - d_entropy p (log p + entropy)) / T
//
// Both are one pass over the logits: bound by DRAM from some hundred rows on, by latency below.
#pragma once

#include "cfgzip_device.cuh"

namespace cfgzip {

constexpr int kLogprobsThreads = 256;
constexpr int kLogprobsChunk = 256;      // tokens whose largest logit is kept together: eight to a lane
constexpr int kLogprobsTopMost = 32;     // alternatives at most
constexpr int kLogprobsList = 256;       // candidates that are put in order by counting
constexpr float kLogprobsSlack = 8.f;    // powers of two that a value may be above the reference of its sum

struct LogprobsArgs {
    const void* logits;
    int64_t stride;
    int32_t N, V;
    const uint32_t* mask;  // null: everything is allowed
    int64_t mask_stride;
    const int32_t* tokens;
    float inv_temperature;
    int32_t n_top;
    float *logp, *entropy, *lse;
    int32_t* top_tokens;
    float* top_logp;
    int32_t* status;
};

// A row by vectors of eight from its first 16-byte boundary on: `head` tokens before it, `octets` vectors, `tail` tokens behind.
struct RowShape {
    int head, octets, tail;
};
template <int DT>
__device__ __forceinline__ RowShape row_shape(const void* row, int V) {
    constexpr int kSize = DT == kBF16 ? 2 : 4;
    RowShape s;
    s.head = min(V, int((16u - (uint32_t(reinterpret_cast<uintptr_t>(row)) & 15u)) & 15u) / kSize);
    s.octets = (V - s.head) / 8;
    s.tail = V - s.head - 8 * s.octets;
    return s;
}

// The allow bits of the octet that starts at token head + 8 o.
__device__ __forceinline__ uint32_t octet_bits(const uint8_t* mask, int head, int o) {
    uint32_t b = ld_after_wait(mask + o);
    if (head) b |= ld_after_wait(mask + o + 1) << 8;
    return (b >> head) & 0xFFu;
}

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// Eight logits in registers as they were loaded.
template <int DT>
struct Logits8;
template <>
struct Logits8<kBF16> {
    static constexpr uint32_t kNone2 = 0xF149F149u;  // kNone, rounded
    uint4 v;
    __device__ __forceinline__ void none() { v = make_uint4(kNone2, kNone2, kNone2, kNone2); }
    __device__ __forceinline__ void load(const void* row, int first) {
        v = ld_stream16(static_cast<const uint16_t*>(row) + first);
    }
    // The values, masked ones and what is below kNone as that, and the largest of them.
    __device__ __forceinline__ float values(uint32_t bits, bool masked, float (&f)[8]) {
        if (masked) {
            const uint32_t xl = nibble_to_byte_msbs(bits & 0xFu), xh = nibble_to_byte_msbs(bits >> 4);
            const uint32_t m0 = prmt(xl, 0u, 0x9988), m1 = prmt(xl, 0u, 0xBBAA), m2 = prmt(xh, 0u, 0x9988), m3 = prmt(xh, 0u, 0xBBAA);
            v.x = (v.x & m0) | (kNone2 & ~m0);
            v.y = (v.y & m1) | (kNone2 & ~m1);
            v.z = (v.z & m2) | (kNone2 & ~m2);
            v.w = (v.w & m3) | (kNone2 & ~m3);
        }
        const uint32_t a = max_bf16x2(v.x, kNone2), b = max_bf16x2(v.y, kNone2), c = max_bf16x2(v.z, kNone2), d = max_bf16x2(v.w, kNone2);
        const uint32_t m = max_bf16x2(max_bf16x2(a, b), max_bf16x2(c, d));
        f[0] = __uint_as_float(a << 16); f[1] = __uint_as_float(a & 0xFFFF0000u);
        f[2] = __uint_as_float(b << 16); f[3] = __uint_as_float(b & 0xFFFF0000u);
        f[4] = __uint_as_float(c << 16); f[5] = __uint_as_float(c & 0xFFFF0000u);
        f[6] = __uint_as_float(d << 16); f[7] = __uint_as_float(d & 0xFFFF0000u);
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    }
};
template <>
struct Logits8<kF32> {
    uint4 a, b;
    __device__ __forceinline__ void none() {
        const uint32_t n = __float_as_uint(kNone);
        a = b = make_uint4(n, n, n, n);
    }
    __device__ __forceinline__ void load(const void* row, int first) {
        const float* p = static_cast<const float*>(row) + first;
        a = ld_stream16(p);
        b = ld_stream16(p + 4);
    }
    __device__ __forceinline__ float values(uint32_t bits, bool masked, float (&f)[8]) {
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = fmaxf(__uint_as_float(w[j]), kNone);
            if (masked) f[j] = (bits >> j) & 1u ? f[j] : kNone;
        }
        return fmaxf(fmax3(fmax3(f[0], f[1], f[2]), f[3], f[4]), fmax3(f[5], f[6], f[7]));
    }
};

// Sums of exp((z - ref) / T) and of that times z - ref, the reference a value of the thread's that was its largest up to kLogprobsSlack
// powers of two ago. The differences are taken before anything is multiplied: a row's logits may be far from zero.
struct EntropySums {
    float ref = kFew;
    unsigned long long s = 0, d = 0;  // pairs of partial sums
    __device__ __forceinline__ void add(const float (&f)[8], float top, float scale) {
        if ((top - ref) * scale > kLogprobsSlack) move(top, scale);
        const unsigned long long minus = pack2(-ref, -ref), by = pack2(scale, scale);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const unsigned long long x = add2(pack2(f[j], f[j + 1]), minus);
            float t0, t1;
            unpack2(mul2(x, by), t0, t1);
            const unsigned long long e = pack2(ex2f(t0), ex2f(t1));
            s = add2(s, e);
            d = fma2(e, x, d);
        }
    }
    // to another reference: z - to = (z - ref) + (ref - to)
    __device__ __forceinline__ void move(float to, float scale) {
        const float by = ref - to, e = ex2f(by * scale);
        const unsigned long long e2 = pack2(e, e);
        d = mul2(fma2(pack2(by, by), s, d), e2);
        s = mul2(s, e2);
        ref = to;
    }
    __device__ __forceinline__ float2 total() const {
        float s0, s1, d0, d1;
        unpack2(s, s0, s1);
        unpack2(d, d0, d1);
        return make_float2(s0 + s1, d0 + d1);
    }
};

// Numbers in the order of their values, both zeros alike, and behind it the lower token first.
__device__ __forceinline__ unsigned long long candidate_key(float z, int token) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return (unsigned long long)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | uint32_t(~token);
}
__device__ __forceinline__ float candidate_value(unsigned long long key) {
    const uint32_t b = uint32_t(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7FFFFFFFu : ~b);
}

// A chunk's tokens, up to eight to a lane: chunk 0 the tokens before the row's first vector, then 256 at a time, at last those behind the
// last vector. Returns the first token; the values are kNone where there is none, or none that counts.
template <int DT, bool MASKED>
__device__ __forceinline__ int chunk_values(const LogprobsArgs& a, const void* row, const uint8_t* mask, const RowShape& r, int chunk,
                                            int chunks, int lane, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = kNone;
    if (chunk > 0 && chunk <= chunks) {
        const int o = (chunk - 1) * 32 + lane, first = r.head + 8 * o;
        if (o >= r.octets) return first;
        const uint32_t bits = MASKED ? octet_bits(mask, r.head, o) : 0xFFu;
        Logits8<DT> v;
        v.load(row, first);
        v.values(bits, MASKED, f);
        return first;
    }
    const int token = chunk ? r.head + 8 * r.octets + lane : lane;
    if (lane < (chunk ? r.tail : r.head) && (!MASKED || ((ld_after_wait(mask + (token >> 3)) >> (token & 7)) & 1u)))
        f[0] = fmaxf(load_elem<DT>(row, token), kNone);
    return token;
}

// The first n of `all` largest values by value, then by place, and the last one's value: by one warp, each lane with a run of neighbours
// (of odd length, for the banks). Those taken are struck out. Fewer where no more values count; `places` may be null.
struct Picked {
    int n;
    float bar;
};
__device__ __forceinline__ Picked pick_largest(float* values, int all, int n, int* places, int lane) {
    const int run = ((all + 31) / 32) | 1, lo = min(lane * run, all), hi = min(lo + run, all);
    Picked p{0, kNone};
    float best = kNone;
    int at = lo;
    bool look = true;
    for (;;) {
        if (look) {
            best = kNone;
            for (int i = lo; i < hi; ++i) {
                const float x = values[i];
                if (x > best) {
                    best = x;
                    at = i;
                }
            }
        }
        __syncwarp();
        const float top = redux_max(best);
        if (p.n == n || !(top > kFew)) return p;
        look = lane == __ffs(__ballot_sync(0xFFFFFFFFu, best == top)) - 1;
        if (look) {
            if (places) places[p.n] = at;
            values[at] = kNone;
        }
        p.bar = top;
        ++p.n;
    }
}

// A cluster of blocks (of 1 to 16) a row; a warp takes 256 tokens at a time, four loads of a lane in flight. The blocks' sums meet in the
// first block.
//
// Alternatives: the largest logit of every 256 tokens comes for one warp reduction. In the order (largest logit, then lower place) the
// first n of these chunks hold the first n tokens (n chunks ahead of a token's own hold n tokens ahead of it). One warp picks them, the
// block reads them once more (from the L2, n * 256 tokens), keeps what is not below the n-th chunk's largest, hardly more than n tokens,
// and every one of those counts how many are ahead of it.
template <int DT, bool MASKED>
__global__ void __launch_bounds__(kLogprobsThreads, 4) k_token_logprobs(const LogprobsArgs a, int blocks) {
    extern __shared__ float s_chunk[];  // the first block's: largest logit of every chunk
    __shared__ float s_ref[8], s_sum[8], s_dif[8];
    __shared__ float4 s_block[kClusterMost];
    __shared__ unsigned long long s_list[kLogprobsList];
    __shared__ int s_pick[kLogprobsTopMost], s_picked, s_listed;
    __shared__ float s_bar, s_eight[32 * kLogprobsTopMost];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = blockIdx.x / blocks;
    const int rank = int(blockIdx.x - row * blocks);
    const float scale = a.inv_temperature * kLog2e;
    const char* z = static_cast<const char*>(a.logits) + row * a.stride * (DT == kBF16 ? 2 : 4);
    const uint8_t* mask = MASKED ? reinterpret_cast<const uint8_t*>(a.mask + row * a.mask_stride) : nullptr;
    const RowShape r = row_shape<DT>(z, a.V);
    const int chunks = (r.octets + 31) / 32;
    const int c1 = int(int64_t(chunks) * (rank + 1) / blocks);
    const uint32_t chunk_at = peer_shared(s_chunk, 0);
    if (threadIdx.x == 0) s_listed = 0;
    cluster_barrier();  // (the first block is there to be written to)
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // the given token's logit, asked for ahead
    int token = -1;
    float of_token = -INFINITY;
    if (rank == 0 && threadIdx.x == 0 && a.tokens) {
        token = ld_after_wait(a.tokens + row);
        if (token >= 0 && token < a.V && (!MASKED || ((ld_after_wait(mask + (token >> 3)) >> (token & 7)) & 1u))) of_token = load_elem<DT>(z, token);
    }

    EntropySums sums;
    float most = kNone;
    // tokens beside the vectors
    if (warp == 0 && (rank == 0 || rank == blocks - 1)) {
#pragma unroll 1
        for (int edge = rank == 0 ? 0 : 1; edge < (rank == blocks - 1 ? 2 : 1); ++edge) {
            float f[8];
            chunk_values<DT, MASKED>(a, z, mask, r, edge ? chunks + 1 : 0, chunks, lane, f);
            most = fmaxf(most, f[0]);
            sums.add(f, f[0], scale);
            const float top = redux_max(f[0]);
            if (a.n_top && lane == 0) st_peer_u32(chunk_at + 4u * uint32_t(edge ? chunks + 1 : 0), __float_as_uint(top));
        }
    }
    constexpr int kAhead = 4;
#pragma unroll 1
    for (int c = int(int64_t(chunks) * rank / blocks) + warp; c < c1; c += 8 * kAhead) {
        uint32_t bits[kAhead];
        Logits8<DT> v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int o = (c + 8 * k) * 32 + lane;
            bits[k] = c + 8 * k < c1 && o < r.octets ? (MASKED ? octet_bits(mask, r.head, o) : 0xFFu) : 0u;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {  // (vectors of which nothing is allowed are not read)
            v[k].none();
            if (bits[k]) v[k].load(z, r.head + 8 * ((c + 8 * k) * 32 + lane));
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (c + 8 * k >= c1) break;
            float f[8];
            const float top = v[k].values(bits[k], MASKED, f);
            most = fmaxf(most, top);
            sums.add(f, top, scale);
            if (a.n_top) {
                const float of_chunk = redux_max(top);
                if (lane == 0) st_peer_u32(chunk_at + 4u * uint32_t(c + 8 * k + 1), __float_as_uint(of_chunk));
            }
        }
    }
    // the block's sums
    most = fmaxf(redux_max(most), kFew);
    sums.move(most, scale);
    float2 t = sums.total();
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
        t.x += __shfl_xor_sync(0xFFFFFFFFu, t.x, d);
        t.y += __shfl_xor_sync(0xFFFFFFFFu, t.y, d);
    }
    if (lane == 0) {
        s_ref[warp] = most;
        s_sum[warp] = t.x;
        s_dif[warp] = t.y;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        float m = s_ref[0];
#pragma unroll
        for (int w = 1; w < 8; ++w) m = fmaxf(m, s_ref[w]);
        float s = 0.f, d = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const float by = s_ref[w] - m, e = ex2f(by * scale);
            s = fmaf(s_sum[w], e, s);
            d = fmaf(fmaf(by, s_sum[w], s_dif[w]), e, d);
        }
        const uint32_t at = peer_shared(&s_block[rank], 0);
        st_peer_u32(at, __float_as_uint(m));
        st_peer_u32(at + 4, __float_as_uint(s));
        st_peer_u32(at + 8, __float_as_uint(d));
    }
    __syncwarp();
    cluster_barrier();
    if (rank != 0) return;

    float m = kFew;
    for (int b = 0; b < blocks; ++b) m = fmaxf(m, s_block[b].x);
    float s = 0.f, d = 0.f;
    for (int b = 0; b < blocks; ++b) {
        const float4 p = s_block[b];
        const float by = p.x - m, e = ex2f(by * scale);
        s = fmaf(p.y, e, s);
        d = fmaf(fmaf(by, p.y, p.z), e, d);
    }
    const float log_sum = logf(s);  // (-inf where nothing is allowed)
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[row] = s > 0.f ? fmaf(m, a.inv_temperature, log_sum) : -INFINITY;
        if (a.entropy) a.entropy[row] = s > 0.f ? fmaxf(log_sum - a.inv_temperature * (d / s), 0.f) : 0.f;
        if (a.tokens) {
            float logp = 0.f;
            if (token >= 0) logp = of_token > kFew ? fmaf(of_token - m, a.inv_temperature, -log_sum) : -INFINITY;
            a.logp[row] = logp;
            if (token >= a.V) atomicAdd(a.status + 1, 1);
        }
    }
    if (!a.n_top) return;

    if (warp == 0) {
        const Picked p = pick_largest(s_chunk, chunks + 2, a.n_top, s_pick, lane);
        if (lane == 0) {
            s_picked = p.n;
            s_bar = p.n < a.n_top ? kNone : p.bar;
        }
    }
    __syncthreads();
    const int picked = s_picked;
    if (picked < a.n_top) {
        // Fewer chunks with an allowed token than tokens wanted: the same once more with eight tokens at a time. Where there are fewer of
        // those too, everything they hold fits the list.
        for (int i = warp; i < picked; i += 8) {
            float f[8];
            chunk_values<DT, MASKED>(a, z, mask, r, s_pick[i], chunks, lane, f);
            s_eight[32 * i + lane] = fmax3(fmax3(f[0], f[1], f[2]), fmax3(f[3], f[4], f[5]), fmaxf(f[6], f[7]));
        }
        __syncthreads();
        if (warp == 0) {
            const Picked p = pick_largest(s_eight, 32 * picked, a.n_top, nullptr, lane);
            if (lane == 0 && p.n == a.n_top) s_bar = p.bar;
        }
        __syncthreads();
    }
    const float bar = s_bar;
    for (int i = warp; i < picked; i += 8) {
        float f[8];
        const int first = chunk_values<DT, MASKED>(a, z, mask, r, s_pick[i], chunks, lane, f);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (f[j] >= bar && f[j] > kFew) {
                const int at = atomicAdd(&s_listed, 1);
                if (at < kLogprobsList) s_list[at] = candidate_key(f[j], first + j);
            }
    }
    __syncthreads();
    const int listed = s_listed;
    int32_t* tokens = a.top_tokens + row * a.n_top;
    float* logps = a.top_logp + row * a.n_top;
    if (listed <= kLogprobsList) {
        if (int(threadIdx.x) < listed) {
            const unsigned long long key = s_list[threadIdx.x];
            int ahead = 0;
            for (int i = 0; i < listed; ++i) ahead += s_list[i] > key;
            if (ahead < a.n_top) {
                tokens[ahead] = int(~uint32_t(key));
                logps[ahead] = fmaf(candidate_value(key) - m, a.inv_temperature, -log_sum);
            }
        }
        for (int i = listed + int(threadIdx.x); i < a.n_top; i += kLogprobsThreads) {
            tokens[i] = -1;
            logps[i] = -INFINITY;
        }
        return;
    }
    // More candidates than the list holds (many equal logits): the largest, the largest behind it, and so on, a pass over the chunks each.
    unsigned long long last = ~0ull;
    for (int n = 0; n < a.n_top; ++n) {
        unsigned long long best = 0;
        for (int i = warp; i < picked; i += 8) {
            float f[8];
            const int first = chunk_values<DT, MASKED>(a, z, mask, r, s_pick[i], chunks, lane, f);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (f[j] >= bar && f[j] > kFew) {
                    const unsigned long long key = candidate_key(f[j], first + j);
                    if (key < last && key > best) best = key;
                }
        }
#pragma unroll
        for (int w = 16; w >= 1; w >>= 1) best = max(best, __shfl_xor_sync(0xFFFFFFFFu, best, w));
        __syncthreads();
        if (lane == 0) s_list[warp] = best;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) best = max(best, s_list[w]);
        last = best;
        if (threadIdx.x == 0) {
            tokens[n] = int(~uint32_t(best));
            logps[n] = fmaf(candidate_value(best) - m, a.inv_temperature, -log_sum);
        }
    }
}

struct LogprobsBackwardArgs {
    const void* logits;
    int64_t stride;
    int32_t N, V;
    const uint32_t* mask;
    int64_t mask_stride;
    const int32_t* tokens;
    float inv_temperature;
    const float *lse, *entropy, *d_logp, *d_entropy;
    void* d_logits;
    int64_t d_stride;
    int32_t pieces;  // blocks a row
};

// What of a row's gradient does not depend on the token: g = p (a + b x) with x = zt - lse, and at the given token
// -d expm1(x) + p b (x + entropy), which keeps what is left of d (1 - p) where the model is sure.
struct RowGradient {
    float lse, a, b, d, entropy;
    int token;
    bool any;
    __device__ __forceinline__ float at(float z, float inv_temperature) const {
        const float x = fmaxf(fmaf(z, inv_temperature, -lse), -200.f);
        return ex2f(x * kLog2e) * fmaf(b, x, a);
    }
    __device__ __forceinline__ float at_token(float z, float inv_temperature) const {
        const float x = fmaf(z, inv_temperature, -lse);
        return fmaf(ex2f(x * kLog2e) * b, x + entropy, -d * expm1f(x));
    }
};
template <int DT, bool MASKED>
__device__ __forceinline__ RowGradient row_gradient(const LogprobsBackwardArgs& a, int64_t row, const void* z, const uint8_t* mask) {
    RowGradient g{};
    g.token = -1;
    const float lse = ld_after_wait(a.lse + row);
    if (!(lse > -INFINITY)) return g;
    g.lse = lse;
    if (a.d_logp) {
        const int token = ld_after_wait(a.tokens + row);
        const float d = ld_after_wait(a.d_logp + row);
        if (token >= 0 && token < a.V && (!MASKED || ((ld_after_wait(mask + (token >> 3)) >> (token & 7)) & 1u)) && load_elem<DT>(z, token) > kFew) {
            g.token = token;
            g.d = d * a.inv_temperature;
        }
    }
    if (a.d_entropy) {
        g.entropy = ld_after_wait(a.entropy + row);
        g.b = -ld_after_wait(a.d_entropy + row) * a.inv_temperature;
    }
    g.a = fmaf(g.b, g.entropy, -g.d);
    g.any = g.d != 0.f || g.b != 0.f;
    return g;
}

// An element, an octet at a time from the gradient's own boundaries on. Logits whose rows start at another place relative to 16 bytes are
// read element by element. Rows without a gradient are written without being read.
template <int DT, bool MASKED>
__global__ void __launch_bounds__(256) k_token_logprobs_backward(const LogprobsBackwardArgs a) {
    constexpr int kSize = DT == kBF16 ? 2 : 4;
    const int64_t row = blockIdx.x / a.pieces;
    const int piece = int(blockIdx.x - row * a.pieces);
    const char* z = static_cast<const char*>(a.logits) + row * a.stride * kSize;
    char* to = static_cast<char*>(a.d_logits) + row * a.d_stride * kSize;
    const uint8_t* mask = MASKED ? reinterpret_cast<const uint8_t*>(a.mask + row * a.mask_stride) : nullptr;
    const RowShape r = row_shape<DT>(to, a.V);
    const bool together = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(to)) & 15u) == 0;
    const int o1 = int(int64_t(r.octets) * (piece + 1) / a.pieces);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const RowGradient g = row_gradient<DT, MASKED>(a, row, z, mask);
    const float it = a.inv_temperature;

    if (piece == 0 && threadIdx.x < 16) {  // tokens beside the vectors
        const int i = int(threadIdx.x), token = i < 8 ? i : r.head + 8 * r.octets + i - 8;
        if (i < 8 ? i < r.head : i - 8 < r.tail) {
            float d = 0.f;
            if (g.any && (!MASKED || ((ld_after_wait(mask + (token >> 3)) >> (token & 7)) & 1u))) {
                const float x = load_elem<DT>(z, token);
                d = token == g.token ? g.at_token(x, it) : g.at(x, it);
            }
            if (DT == kBF16)
                reinterpret_cast<uint16_t*>(to)[token] = uint16_t(bf16_pair(d, d));
            else
                reinterpret_cast<float*>(to)[token] = d;
        }
    }
    constexpr int kAhead = 4;
    const bool wide = (reinterpret_cast<uintptr_t>(to + r.head * kSize) & 31u) == 0;
#pragma unroll 1
    for (int o = int(int64_t(r.octets) * piece / a.pieces) + int(threadIdx.x); o < o1; o += 256 * kAhead) {
        uint32_t bits[kAhead];
        Logits8<DT> v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) bits[k] = g.any && o + 256 * k < o1 ? (MASKED ? octet_bits(mask, r.head, o + 256 * k) : 0xFFu) : 0u;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            v[k].none();
            const int first = r.head + 8 * (o + 256 * k);
            if (bits[k]) {
                if (together) {
                    v[k].load(z, first);
                } else {
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        w[j] = DT == kBF16 ? reinterpret_cast<const uint16_t*>(z)[first + j] : reinterpret_cast<const uint32_t*>(z)[first + j];
                    if constexpr (DT == kBF16) {
                        v[k].v = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
                    } else {
                        v[k].a = make_uint4(w[0], w[1], w[2], w[3]);
                        v[k].b = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (o + 256 * k >= o1) break;
            const int first = r.head + 8 * (o + 256 * k);
            float f[8], d[8];
            v[k].values(bits[k], MASKED, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = g.at(f[j], it);
            if (uint32_t(g.token - first) < 8u) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (g.token == first + j) d[j] = g.at_token(f[j], it);
            }
            if constexpr (DT == kBF16) {
                st_stream16(to + int64_t(first) * kSize,
                            make_uint4(bf16_pair(d[0], d[1]), bf16_pair(d[2], d[3]), bf16_pair(d[4], d[5]), bf16_pair(d[6], d[7])));
            } else {
                const uint4 lo = make_uint4(__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3]));
                const uint4 hi = make_uint4(__float_as_uint(d[4]), __float_as_uint(d[5]), __float_as_uint(d[6]), __float_as_uint(d[7]));
                if (wide) {
                    st_stream32(to + int64_t(first) * kSize, lo, hi);
                } else {
                    st_stream16(to + int64_t(first) * kSize, lo);
                    st_stream16(to + int64_t(first) * kSize + 16, hi);
                }
            }
        }
    }
}

}  // namespace cfgzip
