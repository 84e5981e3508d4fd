// Activations with their derivatives, and the biases in front of them.
#pragma once

#include "cfgzip_device.cuh"

namespace cfgzip {

enum : int { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4 };

__device__ __forceinline__ float rcpf(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The activation of two numbers, and its derivative. Logistic functions are 1 / (1 + exp), which is 0 or 1 where the exponential leaves the
// numbers; the polynomial of the derivative of the one by way of tanh is taken of arguments within 64, behind which nothing changes any more.
// Without branches, so that the elements of a row are computed side by side, two to an instruction: with an IEEE division the epilogue took as
// long as the product (8192 x 4096 x 4096: 212 against 180 us).
// The normal distribution's Phi is made of the complementary error function as in Abramowitz and Stegun, 7.1.26 (within 1.5e-7), whose
// exponential the derivative needs too. Where Phi itself is small that is 5e-4 of it at -4 and 4e-3 at -6, up to a step of bf16 of a result
// below 1e-4 that has no residual.
using pair2 = unsigned long long;
__device__ __forceinline__ pair2 both(float x) { return pack2(x, x); }
__device__ __forceinline__ pair2 ex2_pair(pair2 x) {
    float a, b;
    unpack2(x, a, b);
    return pack2(ex2f(a), ex2f(b));
}
__device__ __forceinline__ pair2 rcp_pair(pair2 x) {
    float a, b;
    unpack2(x, a, b);
    return pack2(rcpf(a), rcpf(b));
}
__device__ __forceinline__ void bf16_pairs(const uint4& v, pair2 (&p)[4]) {
    float f[8];
    bf16_values(v, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = pack2(f[2 * j], f[2 * j + 1]);
}
template <int ACT>
__device__ __forceinline__ pair2 activation(pair2 h, pair2* slope) {
    float h0, h1;
    unpack2(h, h0, h1);
    if (ACT == kActRelu) {
        *slope = pack2(h0 > 0.f ? 1.f : 0.f, h1 > 0.f ? 1.f : 0.f);
        return pack2(fmaxf(h0, 0.f), fmaxf(h1, 0.f));
    }
    if (ACT == kActGelu) {
        const pair2 e = ex2_pair(mul2(mul2(h, h), both(-0.5f * kLog2e)));
        const pair2 t = rcp_pair(fma2(pack2(fabsf(h0), fabsf(h1)), both(0.3275911f * 0.70710678f), both(1.f)));
        pair2 p = fma2(both(0.5f * 1.061405429f), t, both(0.5f * -1.453152027f));
        p = fma2(p, t, both(0.5f * 1.421413741f));
        p = fma2(p, t, both(0.5f * -0.284496736f));
        p = mul2(mul2(fma2(p, t, both(0.5f * 0.254829592f)), t), e);
        float p0, p1;
        unpack2(p, p0, p1);
        const pair2 phi = pack2(h0 < 0.f ? p0 : 1.f - p0, h1 < 0.f ? p1 : 1.f - p1);
        *slope = fma2(mul2(h, both(0.3989422804f)), e, phi);
        return mul2(h, phi);
    }
    if (ACT == kActGeluTanh) {  // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)), u = k (h + 0.044715 h^3), k = sqrt(2 / pi)
        const pair2 c = pack2(fminf(fmaxf(h0, -64.f), 64.f), fminf(fmaxf(h1, -64.f), 64.f)), square = mul2(c, c);
        constexpr float kTwoK = 1.5957691216f;
        const pair2 u = mul2(c, fma2(both(-kLog2e * kTwoK * 0.044715f), square, both(-kLog2e * kTwoK)));
        const pair2 q = rcp_pair(add2(ex2_pair(u), both(1.f)));
        *slope = fma2(mul2(mul2(c, q), fma2(q, both(-1.f), both(1.f))), fma2(both(kTwoK * 3.f * 0.044715f), square, both(kTwoK)), q);
        return mul2(h, q);
    }
    if (ACT == kActSilu) {
        const pair2 q = rcp_pair(add2(ex2_pair(mul2(h, both(-kLog2e))), both(1.f)));
        *slope = mul2(q, fma2(h, fma2(q, both(-1.f), both(1.f)), both(1.f)));
        return mul2(h, q);
    }
    *slope = both(1.f);
    return h;
}

// One as it is stored, its bits.
__device__ __forceinline__ uint32_t bias_bits(const void* bias, bool bf16, int n) {
    if (!bf16) return ld_after_wait(static_cast<const uint32_t*>(bias) + n);
    uint32_t v;
    asm volatile("ld.global.u16 %0, [%1];" : "=r"(v) : "l"(__cvta_generic_to_global(static_cast<const uint16_t*>(bias) + n)));
    return v;
}
// Eight biases from feature n on (n and their number a multiple of 8).
__device__ __forceinline__ void bias_values(const void* bias, bool bf16, int n, float (&f)[8]) {
    if (bf16) {
        bf16_values(ld_after_wait(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(bias) + n)), f);
    } else {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(bias) + n);
        const uint4 a = ld_after_wait(p), b = ld_after_wait(p + 1);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(w[j]);
    }
}

}  // namespace cfgzip
