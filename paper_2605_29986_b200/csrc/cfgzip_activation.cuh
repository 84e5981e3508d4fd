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

// The activation and its derivative. Logistic functions are 1 / (1 + exp), which is 0 or 1 where the exponential leaves the numbers; the
// polynomials are taken of arguments within 64, behind which nothing changes any more. Without branches, so that the elements of a row are
// computed side by side: with an IEEE division the epilogue took as long as the product (8192 x 4096 x 4096: 212 against 180 us).
// The normal distribution's Phi is made of the complementary error function as in Abramowitz and Stegun, 7.1.26 (within 1.5e-7), whose
// exponential the derivative needs too.
template <int ACT>
__device__ __forceinline__ float activation(float h, float* slope) {
    if (ACT == kActRelu) {
        *slope = h > 0.f ? 1.f : 0.f;
        return fmaxf(h, 0.f);
    }
    if (ACT == kActGelu) {
        const float c = fminf(fmaxf(h, -64.f), 64.f), x = fabsf(c) * 0.70710678f, e = ex2f(c * c * (-0.5f * kLog2e));
        const float t = rcpf(fmaf(0.3275911f, x, 1.f));
        float p = fmaf(1.061405429f, t, -1.453152027f);
        p = fmaf(p, t, 1.421413741f);
        p = fmaf(p, t, -0.284496736f);
        p = fmaf(p, t, 0.254829592f) * t * 0.5f;
        const float phi = h < 0.f ? p * e : fmaf(-p, e, 1.f);
        *slope = fmaf(c * 0.3989422804f, e, phi);
        return h * phi;
    }
    if (ACT == kActGeluTanh) {  // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)), u = k (h + 0.044715 h^3), k = sqrt(2 / pi)
        const float c = fminf(fmaxf(h, -64.f), 64.f), two_k = 1.5957691216f;
        const float q = rcpf(1.f + ex2f(-kLog2e * two_k * c * fmaf(0.044715f, c * c, 1.f)));
        *slope = fmaf(c * q * (1.f - q), two_k * fmaf(3.f * 0.044715f, c * c, 1.f), q);
        return h * q;
    }
    if (ACT == kActSilu) {
        const float q = rcpf(1.f + ex2f(-kLog2e * h));
        *slope = q * fmaf(h, 1.f - q, 1.f);
        return h * q;
    }
    *slope = 1.f;
    return h;
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
