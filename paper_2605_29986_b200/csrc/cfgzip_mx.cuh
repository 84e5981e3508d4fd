// Microscaled 4-bit weights: 32 along a row share a power of two, each is e2m1 (sign, two bits of exponent, one of fraction).
// Both kernels are bound by the memory they move, 2.53 bytes a weight from and to bf16.
#pragma once

#include "cfgzip_device.cuh"

namespace cfgzip {

constexpr int kMxBlock = 32;      // weights per scale
constexpr int kMxUnroll = 4;      // vectors of 8 weights a thread has in flight

// Eight f32 to eight e2m1 codes, ties to even, above 6 to 6; the first in the lowest four bits.
__device__ __forceinline__ uint32_t e2m1_codes(const float (&f)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
    return r;
}

// 2^(scale - 127) as f32; the scale byte 0 is below the normal numbers.
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte ? (byte == 255u ? 0x7FC00000u : byte << 23) : 0x00400000u); }

// Where a vector of 8 weights lies: `vectors` of them to a row, in the order of the memory.
struct MxAt {
    int64_t row;
    int col;  // vector of the row
};
__device__ __forceinline__ MxAt mx_at(int64_t i, int vectors) {
    if (i >> 32) return MxAt{i / vectors, int(i % vectors)};
    const uint32_t r = uint32_t(i) / uint32_t(vectors);
    return MxAt{int64_t(r), int(uint32_t(i) - r * uint32_t(vectors))};
}

// A thread takes a vector of 8 weights, four neighbours a block; the largest goes around by shuffles. A block of threads takes
// kMxUnroll * blockDim consecutive vectors, H is a multiple of 32, so a block of weights never leaves its four lanes.
template <int DT>
__global__ void __launch_bounds__(256) k_mx_quantize(const void* weight, int64_t row_stride, int vectors, int64_t total,
                                                     uint8_t* packed, int64_t packed_stride, uint8_t* scales, int64_t scale_stride) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t first = int64_t(blockIdx.x) * (256 * kMxUnroll) + threadIdx.x;
    uint4 raw[kMxUnroll][DT == kF32 ? 2 : 1];
    MxAt at[kMxUnroll];
#pragma unroll
    for (int u = 0; u < kMxUnroll; ++u) {
        const int64_t i = first + u * 256;
        at[u] = mx_at(i < total ? i : total - 1, vectors);
        const char* p = static_cast<const char*>(weight) + (at[u].row * row_stride + 8 * int64_t(at[u].col)) * (DT == kF32 ? 4 : 2);
        raw[u][0] = ld_stream16(p);
        if (DT == kF32) raw[u][DT == kF32 ? 1 : 0] = ld_stream16(p + 16);
    }
#pragma unroll
    for (int u = 0; u < kMxUnroll; ++u) {
        float f[8];
        const uint32_t* w = &raw[u][0].x;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            f[j] = DT == kF32 ? __uint_as_float(w[j]) : __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
        uint32_t most = 0;  // largest magnitude, as bits: in the order of the values, and NaN above infinity
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(f[j]) & 0x7FFFFFFFu);
        most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
        most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
        const uint32_t e = most >> 23;  // floor(log2) + 127, 0 below the normal numbers
        const uint32_t byte = e == 255u ? 255u : e > 2u ? e - 2u : 0u;
        const float up = __uint_as_float((254u - (byte == 255u ? 0u : byte)) << 23);  // 2^(127 - byte)
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= up;
        const uint32_t codes = byte == 255u ? 0u : e2m1_codes(f);
        if (first + u * 256 < total) {
            *reinterpret_cast<uint32_t*>(packed + at[u].row * packed_stride + 4 * int64_t(at[u].col)) = codes;
            if ((at[u].col & 3) == 0) scales[at[u].row * scale_stride + (at[u].col >> 2)] = uint8_t(byte);
        }
    }
}

// Eight e2m1 codes of a word to bf16 pairs: each times 2^(byte - 127). The product is exact in 32 bits and in bf16.
__device__ __forceinline__ uint4 mx_values(uint32_t codes, uint32_t byte) {
    const float s = mx_scale(byte);
    uint32_t out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t code = codes >> (8 * j + 4 * k);
            // exponent and fraction at the top of the fraction field of a number below the normal ones: 2^126 times too small
            const float m = __uint_as_float((code & 7u) << 22) * 0x1p126f;
            v[k] = (code & 8u ? -m : m) * s;
        }
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(out[j]) : "f"(v[1]), "f"(v[0]));
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

__global__ void __launch_bounds__(256) k_mx_dequantize(const uint8_t* packed, int64_t packed_stride, const uint8_t* scales,
                                                       int64_t scale_stride, int vectors, int64_t total, uint16_t* values,
                                                       int64_t row_stride) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t first = int64_t(blockIdx.x) * (256 * kMxUnroll) + threadIdx.x;
    uint32_t codes[kMxUnroll], byte[kMxUnroll];
    MxAt at[kMxUnroll];
#pragma unroll
    for (int u = 0; u < kMxUnroll; ++u) {
        const int64_t i = first + u * 256;
        at[u] = mx_at(i < total ? i : total - 1, vectors);
        codes[u] = ld_after_wait(reinterpret_cast<const uint32_t*>(packed + at[u].row * packed_stride + 4 * int64_t(at[u].col)));
        byte[u] = ld_after_wait(scales + at[u].row * scale_stride + (at[u].col >> 2));
    }
#pragma unroll
    for (int u = 0; u < kMxUnroll; ++u)
        if (first + u * 256 < total)
            st_stream16(values + at[u].row * row_stride + 8 * int64_t(at[u].col), mx_values(codes[u], byte[u]));
}

}  // namespace cfgzip
