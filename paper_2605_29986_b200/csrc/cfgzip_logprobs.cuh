// Log probabilities of given tokens, entropies and top alternatives from logits, and the gradient of the first two.
//
//   zt = z / T over the allowed tokens,  lse = log sum exp zt,  logp = zt[token] - lse,  entropy = lse - sum p zt
//   d_z = (d_logp ([t = token] - p) - d_entropy p (log p + entropy)) / T
//
// Both are one pass over the logits: bound by DRAM from some hundred rows on, by latency below.
#pragma once

#include "cfgzip_device.cuh"

namespace cfgzip {

constexpr int kLogprobsChunk = 256;      // tokens whose largest logit is kept together: eight to a lane
constexpr int kLogprobsTopMost = 32;     // alternatives at most
constexpr int kLogprobsList = 256;       // candidates that are put in order by counting
constexpr int kLogprobsPicks = 128;      // chunks that are read once more, at most
constexpr int kLogprobsAll = 64;         // ... where all that have an allowed token are
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLogprobsSlack = 4.f;    // powers of two that a logit may be above the reference of its sum (t is rounded the coarser the larger it is)

// Logits in powers of two: `scale` powers to a unit (log2(e) / T); from `far` on the whole number next to a logit's powers would have to be
// rounded itself; `slack` is kLogprobsSlack powers.
struct Powers {
    float scale, far, slack;
};

struct LogprobsArgs {
    const void* logits;
    int64_t stride;
    int32_t N, V;
    const uint32_t* mask;  // null: everything is allowed
    int64_t mask_stride;
    const int32_t* tokens;
    float inv_temperature;
    Powers powers;
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

// The allow bits of the octet that starts at token head + 8 o, alone.
__device__ __forceinline__ uint32_t octet_bits(const uint8_t* mask, int head, int o) {
    uint32_t b = ld_after_wait(mask + o);
    if (head) b |= ld_after_wait(mask + o + 1) << 8;
    return (b >> head) & 0xFFu;
}

// The allow bits of a warp's next chunks (`n` of them, at most 4, `step` apart), eight words of 32 to each: lane l has word l % 8 of chunk
// c + step (l / 8). They are asked for a round ahead of the logits, which wait for them, and put in place when they are used.
struct ChunkBits {
    uint32_t word, after;
    __device__ __forceinline__ void ask(const uint32_t* mask, int head, int V, int c, int c1, int step, int n, int lane) {
        const int chunk = c + step * (lane >> 3), at = 8 * chunk + (lane & 7), words = (V + 31) / 32;
        const bool have = chunk < c1 && lane < 8 * n;
        word = have && at < words ? ld_after_wait(mask + at) : 0u;
        after = have && head && (lane & 7) == 7 && at + 1 < words ? ld_after_wait(mask + at + 1) : 0u;
    }
    __device__ __forceinline__ uint32_t from(int head, int lane) const {  // bits from `head` on: the next word's first ones come in
        const uint32_t next = __shfl_down_sync(0xFFFFFFFFu, word, 1);
        return __funnelshift_r(word, (lane & 7) == 7 ? after : next, head);
    }
};

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
    __device__ __forceinline__ void load_anywhere(const void* row, int first) {
        const uint16_t* p = static_cast<const uint16_t*>(row) + first;
        v = make_uint4(p[0] | uint32_t(p[1]) << 16, p[2] | uint32_t(p[3]) << 16, p[4] | uint32_t(p[5]) << 16, p[6] | uint32_t(p[7]) << 16);
    }
    // Masked ones, and what is below kNone, become that. Returns the largest.
    __device__ __forceinline__ float settle(uint32_t bits, bool masked) {
        if (masked) {
            const uint32_t xl = nibble_to_byte_msbs(bits & 0xFu), xh = nibble_to_byte_msbs(bits >> 4);
            const uint32_t m0 = prmt(xl, 0u, 0x9988), m1 = prmt(xl, 0u, 0xBBAA), m2 = prmt(xh, 0u, 0x9988), m3 = prmt(xh, 0u, 0xBBAA);
            v.x = (v.x & m0) | (kNone2 & ~m0);
            v.y = (v.y & m1) | (kNone2 & ~m1);
            v.z = (v.z & m2) | (kNone2 & ~m2);
            v.w = (v.w & m3) | (kNone2 & ~m3);
        }
        v = make_uint4(max_bf16x2(v.x, kNone2), max_bf16x2(v.y, kNone2), max_bf16x2(v.z, kNone2), max_bf16x2(v.w, kNone2));
        const uint32_t m = max_bf16x2(max_bf16x2(v.x, v.y), max_bf16x2(v.z, v.w));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    }
    // Less `top`, not below kNone (a difference that bf16 does not hold is far beyond what weighs anything: see Reference).
    __device__ __forceinline__ void relative_to(float top) {
        float f[8];
        get(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = fmaxf(f[j] - top, kNone);
        v = make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f[2 * j] = __uint_as_float(w[j] << 16);
            f[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
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
    __device__ __forceinline__ void load_anywhere(const void* row, int first) {
        const uint32_t* p = static_cast<const uint32_t*>(row) + first;
        a = make_uint4(p[0], p[1], p[2], p[3]);
        b = make_uint4(p[4], p[5], p[6], p[7]);
    }
    __device__ __forceinline__ float settle(uint32_t bits, bool masked) {
        uint32_t* const w[8] = {&a.x, &a.y, &a.z, &a.w, &b.x, &b.y, &b.z, &b.w};
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = fmaxf(__uint_as_float(*w[j]), kNone);
            if (masked) f[j] = (bits >> j) & 1u ? f[j] : kNone;
            *w[j] = __float_as_uint(f[j]);
        }
        return fmaxf(fmax3(fmax3(f[0], f[1], f[2]), f[3], f[4]), fmax3(f[5], f[6], f[7]));
    }
    __device__ __forceinline__ void relative_to(float top) {
        uint32_t* const w[8] = {&a.x, &a.y, &a.z, &a.w, &b.x, &b.y, &b.z, &b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) *w[j] = __float_as_uint(fmaxf(__uint_as_float(*w[j]) - top, kNone));
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(w[j]);
    }
};

// What t, the exponent of a logit in powers of two, is relative to: a logit `top`. Near zero that is the whole number of powers next to it, -n:
// t = z scale + n is rounded once, all threads' t are of the same numbers, and a sum goes over to another reference exactly. Far from zero a
// float holds no such n (that of -1e10 would be off by 440 powers): t = (z - top) scale, whose difference is exact wherever it does not come
// to millions of powers. (`top` alone is kept: f32 rows under masks have no register for more, 1000 of 100003 71 and 86 us.)
constexpr float kFarPowers = 4194304.f;
struct Reference {
    float top;
    __device__ __forceinline__ bool far(const Powers& p) const { return fabsf(top) >= p.far; }
    __device__ __forceinline__ float near_n(const Powers& p) const {
        constexpr float kWhole = 12582912.f;  // (its step is 1: nearest whole number)
        return kWhole - fmaf(top, p.scale, kWhole);
    }
    __device__ __forceinline__ float r(const Powers& p) const { return far(p) ? top : 0.f; }
    __device__ __forceinline__ float n(const Powers& p) const { return far(p) ? 0.f : near_n(p); }
    __device__ __forceinline__ float power(float z, const Powers& p) const { return fmaf(z - r(p), p.scale, n(p)); }
    // What has to be added to t to have it relative to a reference that is no lower. (Bounded, so that an empty sum stays 0 and one that is too
    // low to count becomes 0.)
    __device__ __forceinline__ float to(const Reference& other, const Powers& p) const {
        return fminf(fmaxf(fmaf(r(p) - other.r(p), p.scale, other.n(p) - n(p)), -4096.f), 1.f);
    }
};

// Sums of 2^t and 2^t t over a thread's logits. The reference follows the largest logit so far: up to kLogprobsSlack below it.
struct EntropySums {
    Reference at{kFew};
    unsigned long long s = 0, d = 0;  // pairs of partial sums
    __device__ __forceinline__ void follow(float top, const Powers& p) {
        if (top - at.top > p.slack) move(Reference{top}, p);
    }
    // Those of eight logits are added up first (FIRST): of a row that has one probable token the sum is 1 and little, and each addition to the
    // 1 may take half a step of it. Where the reference is far from zero the logits have been made relative to it.
    template <bool FIRST>
    __device__ __forceinline__ void add(const float (&f)[8], float scale, float n) {
        const unsigned long long by = pack2(scale, scale), plus = pack2(n, n);
        unsigned long long of_s = s, of_d = d;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const unsigned long long t = fma2(pack2(f[j], f[j + 1]), by, plus);
            float t0, t1;
            unpack2(t, t0, t1);
            const unsigned long long e = pack2(ex2f(t0), ex2f(t1));
            of_s = j || !FIRST ? add2(of_s, e) : e;
            of_d = j || !FIRST ? fma2(e, t, of_d) : mul2(e, t);
        }
        s = FIRST ? add2(s, of_s) : of_s;
        d = FIRST ? add2(d, of_d) : of_d;
    }
    // ... of eight that a thread has at a time, `top` the largest
    template <bool FIRST>
    __device__ __forceinline__ void take(float (&f)[8], float top, const Powers& p) {
        follow(top, p);
        if (at.far(p) && top > kFew) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = fmaxf(f[j] - at.top, kNone);
        }
        add<FIRST>(f, p.scale, at.n(p));
    }
    __device__ __forceinline__ void move(const Reference& to, const Powers& p) {
        const float by = at.to(to, p), e = ex2f(by);
        const unsigned long long e2 = pack2(e, e);
        d = mul2(fma2(pack2(by, by), s, d), e2);
        s = mul2(s, e2);
        at = to;
    }
    __device__ __forceinline__ double2 total() const {
        float s0, s1, d0, d1;
        unpack2(s, s0, s1);
        unpack2(d, d0, d1);
        return make_double2(double(s0) + double(s1), double(d0) + double(d1));
    }
};

// The sum over `LANES` lanes of sums that each has, relative to a reference that is no lower (in every lane).
template <int LANES>
__device__ __forceinline__ double2 sum_at(const double2& p, const Reference& from, const Reference& to, const Powers& powers) {
    const float by = from.to(to, powers), e = ex2f(by);
    double2 t = make_double2(p.x * double(e), fma(double(by), p.x, p.y) * double(e));
#pragma unroll
    for (int k = LANES / 2; k >= 1; k >>= 1) {
        t.x += __shfl_xor_sync(0xFFFFFFFFu, t.x, k);
        t.y += __shfl_xor_sync(0xFFFFFFFFu, t.y, k);
    }
    return t;
}

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
// last vector. The values are kNone where there is none, or none that counts; `first` is the first value's token. Returns the largest.
template <int DT, bool MASKED>
__device__ __forceinline__ float chunk_values(const LogprobsArgs& a, const void* row, const uint8_t* mask, const RowShape& r, int chunk,
                                              int chunks, int lane, float (&f)[8], int* first) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = kNone;
    if (chunk > 0 && chunk <= chunks) {
        const int o = (chunk - 1) * 32 + lane;
        *first = r.head + 8 * o;
        if (o >= r.octets) return kNone;
        const uint32_t bits = MASKED ? octet_bits(mask, r.head, o) : 0xFFu;
        Logits8<DT> v;
        v.load(row, *first);
        const float top = v.settle(bits, MASKED);
        v.get(f);
        return top;
    }
    const int token = chunk ? r.head + 8 * r.octets + lane : lane;
    *first = token;
    if (lane < (chunk ? r.tail : r.head) && (!MASKED || ((ld_after_wait(mask + (token >> 3)) >> (token & 7)) & 1u)))
        f[0] = fmaxf(load_elem<DT>(row, token), kNone);
    return f[0];
}

// A bar that at least n of the values reach, and hardly more than 1.5 n as long as they come in no order: the n-th largest (n at most 32) of
// the largest values of 64 runs of neighbours, two to a lane of one warp. kNone where fewer than n runs have a value that counts.
__device__ __forceinline__ float bar_of_runs(const float* values, int all, int n, int lane) {
    const int run = ((all + 63) / 64) | 1;  // (odd, for the banks)
    float best[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int lo = min((32 * k + lane) * run, all), hi = min(lo + run, all);
        best[k] = kNone;
        for (int i = lo; i < hi; ++i) best[k] = fmaxf(best[k], values[i]);
    }
    float bar = kNone;
    for (int k = 0; k < n; ++k) {
        const float mine = fmaxf(best[0], best[1]);
        bar = redux_max(mine);
        if (!(bar > kFew)) return kNone;
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, mine == bar);
        if (lane == __ffs(who) - 1) {
            best[1] = best[0] == bar ? best[1] : kNone;
            best[0] = best[0] == bar ? kNone : best[0];
        }
    }
    return bar;
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
// Alternatives: the largest logit of every chunk of 256 tokens comes for one warp reduction. A bar that at least n chunks' largest reach is
// one that at least n tokens reach, and all tokens that reach it are in chunks that do. One warp finds a bar that hardly more than n do
// (bar_of_runs), the block reads those chunks once more from the L2 and lists the tokens, and each of them counts how many are ahead of it.
// Equal logits may put too many chunks above a bar. In the order (largest logit, then place) the first n chunks hold the first n tokens (n
// chunks ahead of a token's own hold n tokens ahead of it), and can be picked one after the other: 0.5 us each.
//
// 4096 bf16 rows of 128256 take 177 to 185 us (5.7 to 5.9 TB/s), with 5 alternatives 192 to 203; 1000 of 100003 under masks 54 to 55, bound by
// instruction issue; 32 of 128256 with 20 alternatives 9 to 10, and one of 32000 5, by latency. What is done in 64 bits, and eight logits added
// up first, are 1.5 % of the large ones, references that hold far from zero 1 % (of short rows, 4096 of 2000, 6).
template <int DT, bool MASKED, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 32 / WARPS) k_token_logprobs(const LogprobsArgs a, int blocks) {
    constexpr int kThreads = WARPS * 32;
    extern __shared__ float s_chunk[];  // the first block's: largest logit of every chunk
    __shared__ float s_ref[WARPS], s_block_ref[kClusterMost];
    __shared__ double2 s_sum[WARPS], s_block[kClusterMost];  // sums of 2^t and 2^t t
    __shared__ unsigned long long s_list[kLogprobsList];
    __shared__ int s_pick[kLogprobsPicks], s_picked, s_listed;
    __shared__ float s_bar, s_most, s_log_sum, s_eight[32 * kLogprobsAll];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = blockIdx.x / blocks;
    const int rank = int(blockIdx.x - row * blocks);
    const char* z = static_cast<const char*>(a.logits) + row * a.stride * (DT == kBF16 ? 2 : 4);
    const uint8_t* mask = MASKED ? reinterpret_cast<const uint8_t*>(a.mask + row * a.mask_stride) : nullptr;
    const RowShape r = row_shape<DT>(z, a.V);
    const int chunks = (r.octets + 31) / 32;
    const int c1 = int(int64_t(chunks) * (rank + 1) / blocks);
    const uint32_t chunk_at = peer_shared(s_chunk, 0);
    if (threadIdx.x == 0) s_listed = s_picked = 0;
    cluster_arrive();
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // the given token's logit, asked for ahead
    int token = -1;
    float of_token = -INFINITY;
    if (rank == 0 && threadIdx.x == 32 && a.tokens) {
        token = ld_after_wait(a.tokens + row);
        if (token >= 0 && token < a.V && (!MASKED || ((ld_after_wait(mask + (token >> 3)) >> (token & 7)) & 1u))) of_token = load_elem<DT>(z, token);
    }

    __syncwarp();
    cluster_wait();  // (the first block is there to be written to)
    // (f32 rows under masks have no registers for it: 1000 of 100003 87 us instead of 70)
    constexpr bool kFirst = !(DT == kF32 && MASKED);
    EntropySums sums;
    float most = kNone;
    // tokens beside the vectors
    if (warp == 0 && (rank == 0 || rank == blocks - 1)) {
#pragma unroll 1
        for (int edge = rank == 0 ? 0 : 1; edge < (rank == blocks - 1 ? 2 : 1); ++edge) {
            float f[8];
            int first;
            const float mine = chunk_values<DT, MASKED>(a, z, mask, r, edge ? chunks + 1 : 0, chunks, lane, f, &first);
            const float top = redux_max(mine);
            most = fmaxf(most, top);
            if (top > kNone) {
                sums.take<kFirst>(f, mine, a.powers);
            }
            if (a.n_top && lane == 0) st_peer_u32(chunk_at + 4u * uint32_t(edge ? chunks + 1 : 0), __float_as_uint(top));
        }
    }
    constexpr int kAhead = DT == kF32 && MASKED ? 3 : 4;  // chunks of a warp at a time (registers)
    int c = int(int64_t(chunks) * rank / blocks) + warp;
    const int whole = min(c1, r.octets / 32);  // (only a row's last chunk may not be)
    const uint32_t* words = MASKED ? a.mask + row * a.mask_stride : nullptr;
    ChunkBits chunk_bits;
    if (MASKED) chunk_bits.ask(words, r.head, a.V, c, c1, WARPS, kAhead, lane);
#pragma unroll 1
    for (; c + WARPS * (kAhead - 1) < whole; c += WARPS * kAhead) {
        Logits8<DT> v[kAhead];
        uint32_t bits[kAhead];
        float top[kAhead];
        const uint32_t of_chunks = MASKED ? chunk_bits.from(r.head, lane) : 0u;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            bits[k] = MASKED ? __shfl_sync(0xFFFFFFFFu, of_chunks, 8 * k + (lane >> 2)) >> (8 * (lane & 3)) & 0xFFu : 0xFFu;
            if (!MASKED || bits[k]) v[k].load(z, r.head + 8 * ((c + WARPS * k) * 32 + lane));  // (what is not read is masked)
        }
        if (MASKED) chunk_bits.ask(words, r.head, a.V, c + WARPS * kAhead, c1, WARPS, kAhead, lane);
        float mine = kNone;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            top[k] = v[k].settle(bits[k], MASKED);
            mine = fmaxf(mine, top[k]);
        }
        most = fmaxf(most, mine);
        sums.follow(mine, a.powers);
        float n = sums.at.near_n(a.powers);
        if (sums.at.far(a.powers)) {
            n = 0.f;
            if (mine > kFew) {  // (masked ones weigh nothing as they are)
#pragma unroll
                for (int k = 0; k < kAhead; ++k) v[k].relative_to(sums.at.top);
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float f[8];
            v[k].get(f);
            sums.add<kFirst>(f, a.powers.scale, n);
        }
        if (a.n_top) {
            float of_chunk = redux_max(top[0]);
#pragma unroll
            for (int k = 1; k < kAhead; ++k) {
                const float x = redux_max(top[k]);
                of_chunk = lane == k ? x : of_chunk;
            }
            if (lane < kAhead) st_peer_u32(chunk_at + 4u * uint32_t(c + WARPS * lane + 1), __float_as_uint(of_chunk));
        }
    }
#pragma unroll 1
    for (; c < c1; c += WARPS) {
        float f[8];
        int first;
        const float mine = chunk_values<DT, MASKED>(a, z, mask, r, c + 1, chunks, lane, f, &first);
        most = fmaxf(most, mine);
        sums.take<kFirst>(f, mine, a.powers);
        if (a.n_top) {
            const float of_chunk = redux_max(mine);
            if (lane == 0) st_peer_u32(chunk_at + 4u * uint32_t(c + 1), __float_as_uint(of_chunk));
        }
    }
    // the block's sums
    most = fmaxf(redux_max(most), kFew);
    sums.move(Reference{most}, a.powers);
    double2 t = sums.total();  // (few additions from here on: in 64 bits)
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
        t.x += __shfl_xor_sync(0xFFFFFFFFu, t.x, d);
        t.y += __shfl_xor_sync(0xFFFFFFFFu, t.y, d);
    }
    if (lane == 0) {
        s_ref[warp] = most;
        s_sum[warp] = t;
    }
    __syncthreads();
    if (warp == 0) {
        const float ref = lane < WARPS ? s_ref[lane] : kFew, m = redux_max(ref);
        t = sum_at<WARPS>(lane < WARPS ? s_sum[lane] : make_double2(0.0, 0.0), Reference{ref}, Reference{m}, a.powers);
        if (lane == 0) {
            st_peer_u32(peer_shared(&s_block_ref[rank], 0), __float_as_uint(m));
            const uint32_t at = peer_shared(&s_block[rank], 0);
            st_peer_u32(at, uint32_t(__double2loint(t.x)));
            st_peer_u32(at + 4, uint32_t(__double2hiint(t.x)));
            st_peer_u32(at + 8, uint32_t(__double2loint(t.y)));
            st_peer_u32(at + 12, uint32_t(__double2hiint(t.y)));
        }
    }
    __syncwarp();
    cluster_barrier();
    if (rank != 0) return;

    if (warp == 1) {  // (the second warp, while the first looks for the alternatives)
        const float ref = lane < blocks ? s_block_ref[lane] : kFew, m = redux_max(ref);
        const Reference to{m};
        t = sum_at<kClusterMost>(lane < blocks ? s_block[lane] : make_double2(0.0, 0.0), Reference{ref}, to, a.powers);
        const double s = t.x, d = t.y;
        // relative to the largest logit itself, whose exponential is taken off and divided out as it was added: a row's only token has log
        // probability 0, and one that is nearly certain keeps what the others have together
        const float of_most = to.power(m, a.powers), e_most = ex2f(of_most);
        const double rest = s - double(e_most);
        const float log_sum = log1pf(float(rest) / e_most);  // (-inf where nothing is allowed)
        if (lane == 0) {
            s_most = m;
            s_log_sum = log_sum;
            if (a.lse) a.lse[row] = s > 0.0 ? fmaf(m, a.inv_temperature, log_sum) : -INFINITY;
            if (a.entropy) a.entropy[row] = s > 0.0 ? fmaxf(log_sum - kLn2 * (float(fma(-double(of_most), rest, d - double(e_most * of_most))) / float(s)), 0.f) : 0.f;
            if (a.tokens) {
                float logp = 0.f;
                if (token >= 0) logp = of_token > kFew ? fmaf(of_token - m, a.inv_temperature, -log_sum) : -INFINITY;
                a.logp[row] = logp;
                if (token >= a.V) atomicAdd(a.status + 1, 1);
            }
        }
    }
    if (!a.n_top) return;
    __syncwarp();

    // the chunks that hold them, by one warp
    if (warp == 0) {
        const float bar = bar_of_runs(s_chunk, chunks + 2, a.n_top, lane);
        if (lane == 0) s_bar = bar;
    }
    __syncthreads();
    const float first_bar = s_bar;
    for (int i = int(threadIdx.x); i < chunks + 2; i += kThreads) {
        const float x = s_chunk[i];
        if (x > kFew && x >= first_bar) {
            const int at = atomicAdd(&s_picked, 1);
            if (at < kLogprobsPicks) s_pick[at] = i;
        }
    }
    __syncthreads();
    int picked = s_picked;
    if (picked > (first_bar > kFew ? kLogprobsPicks : kLogprobsAll)) {  // (many equal ones, or all in a few runs)
        __syncthreads();
        if (warp == 0) {
            const Picked p = pick_largest(s_chunk, chunks + 2, a.n_top, s_pick, lane);
            if (lane == 0) {
                s_picked = p.n;
                s_bar = p.bar;
            }
        }
        __syncthreads();
        picked = s_picked;
    }
    if (!(s_bar > kFew)) {
        // All chunks that have an allowed token, few of them: the same once more with eight tokens at a time. Where fewer of those than
        // tokens wanted have one, everything they hold fits the list.
        for (int i = warp; i < picked; i += WARPS) {
            float f[8];
            int first;
            s_eight[32 * i + lane] = chunk_values<DT, MASKED>(a, z, mask, r, s_pick[i], chunks, lane, f, &first);
        }
        __syncthreads();
        if (warp == 0) {
            float bar = bar_of_runs(s_eight, 32 * picked, a.n_top, lane);
            if (!(bar > kFew)) {
                const Picked p = pick_largest(s_eight, 32 * picked, a.n_top, nullptr, lane);
                if (p.n == a.n_top) bar = p.bar;
            }
            if (lane == 0) s_bar = bar;
        }
        __syncthreads();
    }
    const float bar = s_bar;
    for (int i = warp; i < picked; i += WARPS) {
        float f[8];
        int first;
        if (chunk_values<DT, MASKED>(a, z, mask, r, s_pick[i], chunks, lane, f, &first) >= bar) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (f[j] >= bar && f[j] > kFew) {
                    const int at = atomicAdd(&s_listed, 1);
                    if (at < kLogprobsList) s_list[at] = candidate_key(f[j], first + j);
                }
        }
    }
    __syncthreads();
    const int listed = s_listed;
    const float m = s_most, log_sum = s_log_sum;
    int32_t* tokens = a.top_tokens + row * a.n_top;
    float* logps = a.top_logp + row * a.n_top;
    if (listed <= kLogprobsList) {
        for (int k = int(threadIdx.x); k < listed; k += kThreads) {
            const unsigned long long key = s_list[k];
            int ahead = 0;
            for (int i = 0; i < listed; ++i) ahead += s_list[i] > key;
            if (ahead < a.n_top) {
                tokens[ahead] = int(~uint32_t(key));
                logps[ahead] = fmaf(candidate_value(key) - m, a.inv_temperature, -log_sum);
            }
        }
        for (int i = listed + int(threadIdx.x); i < a.n_top; i += kThreads) {
            tokens[i] = -1;
            logps[i] = -INFINITY;
        }
        return;
    }
    // More candidates than the list holds (many equal logits): the largest, the largest behind it, and so on, a pass over the chunks each.
    unsigned long long last = ~0ull;
    for (int n = 0; n < a.n_top; ++n) {
        unsigned long long best = 0;
        for (int i = warp; i < picked; i += WARPS) {
            float f[8];
            int first;
            chunk_values<DT, MASKED>(a, z, mask, r, s_pick[i], chunks, lane, f, &first);
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
        for (int w = 0; w < WARPS; ++w) best = max(best, s_list[w]);
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
// x above 0 is what lse was rounded by, a half at the most below 2^24; further out lse says nothing of p, which is kept within e.
struct RowGradient {
    float lse, a, b, d, entropy;
    int token;
    static __device__ __forceinline__ float within(float x) { return fminf(fmaxf(x, -200.f), 1.f); }
    __device__ __forceinline__ float at(float z, float inv_temperature) const {
        const float x = within(fmaf(z, inv_temperature, -lse));
        return ex2f(x * kLog2e) * fmaf(b, x, a);
    }
    __device__ __forceinline__ void at_pair(float z0, float z1, float inv_temperature, float* d0, float* d1) const {
        float x0, x1;
        unpack2(fma2(pack2(z0, z1), pack2(inv_temperature, inv_temperature), pack2(-lse, -lse)), x0, x1);
        const unsigned long long x = pack2(within(x0), within(x1));
        unpack2(mul2(x, pack2(kLog2e, kLog2e)), x0, x1);
        unpack2(mul2(pack2(ex2f(x0), ex2f(x1)), fma2(pack2(b, b), x, pack2(a, a))), *d0, *d1);
    }
    __device__ __forceinline__ float at_token(float z, float inv_temperature) const {
        const float x = within(fmaf(z, inv_temperature, -lse));
        return fmaf(ex2f(x * kLog2e) * b, x + entropy, -d * expm1f(x));
    }
};
// ... what is asked for at once, and what depends on it.
struct RowInputs {
    float lse, d_logp, d_entropy, entropy;
    int token;
};
__device__ __forceinline__ RowInputs row_inputs(const LogprobsBackwardArgs& a, int64_t row) {
    RowInputs i;
    i.lse = ld_after_wait(a.lse + row);
    i.token = a.d_logp ? ld_after_wait(a.tokens + row) : -1;
    i.d_logp = a.d_logp ? ld_after_wait(a.d_logp + row) : 0.f;
    i.d_entropy = a.d_entropy ? ld_after_wait(a.d_entropy + row) : 0.f;
    i.entropy = a.d_entropy ? ld_after_wait(a.entropy + row) : 0.f;
    return i;
}
template <int DT, bool MASKED>
__device__ __forceinline__ RowGradient row_gradient(const LogprobsBackwardArgs& a, const RowInputs& i, const void* z, const uint8_t* mask) {
    RowGradient g{};
    g.token = -1;
    if (!(i.lse > -INFINITY)) return g;
    g.lse = i.lse;
    if (i.token >= 0 && i.token < a.V) {
        const float of_token = load_elem<DT>(z, i.token);
        const uint32_t bits = MASKED ? ld_after_wait(mask + (i.token >> 3)) >> (i.token & 7) : 1u;
        if ((bits & 1u) && of_token > kFew) {
            g.token = i.token;
            g.d = i.d_logp * a.inv_temperature;
        }
    }
    g.entropy = i.entropy;
    g.b = -i.d_entropy * a.inv_temperature;
    g.a = fmaf(g.b, g.entropy, -g.d);
    return g;
}

// Octets of a thread of the gradient, and tokens of a block, at most: 32 KB of logits in flight.
template <int DT>
constexpr int kLogprobsOctets = DT == kBF16 ? 8 : 4;
template <int DT>
constexpr int kLogprobsPiece = kLogprobsOctets<DT> * 2048;

// An octet at a time from the gradient's own boundaries on. Logits whose rows start at another place relative to 16 bytes (TOGETHER false) are
// read element by element. Rows without a gradient are written without being read. A block does its tokens in one go: masks and the row's numbers are asked
// for, then the logits, then what the row's constants need of the given token, so that three latencies follow one another, and four or more
// blocks of an SM share them. (4096 bf16 rows of 128256: 305 to 331 us, of which a copy takes 321; 500 f32 rows of 50021 under
// masks 35 to 40, 5.1 to 5.7 TB/s.)
template <int DT, bool MASKED, bool TOGETHER>
__global__ void __launch_bounds__(256, 4) k_token_logprobs_backward(const LogprobsBackwardArgs a) {
    constexpr int kSize = DT == kBF16 ? 2 : 4, kAhead = kLogprobsOctets<DT>;
    const int64_t row = blockIdx.x / a.pieces;
    const int piece = int(blockIdx.x - row * a.pieces);
    const char* z = static_cast<const char*>(a.logits) + row * a.stride * kSize;
    char* to = static_cast<char*>(a.d_logits) + row * a.d_stride * kSize;
    const uint8_t* mask = MASKED ? reinterpret_cast<const uint8_t*>(a.mask + row * a.mask_stride) : nullptr;
    const RowShape r = row_shape<DT>(to, a.V);
    const bool wide = (reinterpret_cast<uintptr_t>(to + r.head * kSize) & 31u) == 0;
    const int o = int(int64_t(r.octets) * piece / a.pieces) + int(threadIdx.x), o1 = int(int64_t(r.octets) * (piece + 1) / a.pieces);
    const float it = a.inv_temperature;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    uint32_t bits[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) bits[k] = o + 256 * k < o1 ? (MASKED ? octet_bits(mask, r.head, o + 256 * k) : 0xFFu) : 0u;
    const RowInputs inputs = row_inputs(a, row);
    const bool any = inputs.lse > -INFINITY && ((inputs.token >= 0 && inputs.d_logp != 0.f) || inputs.d_entropy != 0.f);
    Logits8<DT> v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        if (!MASKED) v[k].none();  // (with a mask, what is not read is masked)
        if (!any) bits[k] = 0u;
        const int first = r.head + 8 * (o + 256 * k);
        if (TOGETHER && bits[k]) v[k].load(z, first);
        if (!TOGETHER && bits[k]) v[k].load_anywhere(z, first);
    }
    const RowGradient g = row_gradient<DT, MASKED>(a, inputs, z, mask);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        if (o + 256 * k >= o1) break;
        const int first = r.head + 8 * (o + 256 * k);
        float f[8], d[8];
        v[k].settle(bits[k], MASKED);
        v[k].get(f);
#pragma unroll
        for (int j = 0; j < 8; j += 2) g.at_pair(f[j], f[j + 1], it, &d[j], &d[j + 1]);
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
    if (piece == 0 && threadIdx.x < 16) {  // tokens beside the vectors
        const int i = int(threadIdx.x), token = i < 8 ? i : r.head + 8 * r.octets + i - 8;
        if (i < 8 ? i < r.head : i - 8 < r.tail) {
            float d = 0.f;
            if (any && (!MASKED || ((ld_after_wait(mask + (token >> 3)) >> (token & 7)) & 1u))) {
                const float x = load_elem<DT>(z, token);
                d = token == g.token ? g.at_token(x, it) : g.at(x, it);
            }
            if (DT == kBF16)
                reinterpret_cast<uint16_t*>(to)[token] = uint16_t(bf16_pair(d, d));
            else
                reinterpret_cast<float*>(to)[token] = d;
        }
    }
}

}  // namespace cfgzip
