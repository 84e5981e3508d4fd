// Microscaled 4-bit weights: 32 along a row share a power of two, each is e2m1 (sign, two bits of exponent, one of fraction).
// Both kernels are bound by the memory they move, 2.53 bytes a weight from and to bf16.
#pragma once

#include "cfgzip_device.cuh"

namespace cfgzip {

constexpr int kMxBlock = 32;      // weights per scale
constexpr int kMxRows = 4;  // rows a thread has in flight, a vector of 8 weights of each

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

// A thread takes a vector of 8 weights of four neighbouring rows (row0 and on; vectors to a row along x, so that nothing has to be
// divided), four lanes a block of weights, whose largest goes around by shuffles.
struct MxAt {
    int64_t row0;
    int col;  // vector of the rows
    bool have;
};
__device__ __forceinline__ MxAt mx_at(int vectors) {
    const int col = blockIdx.y * blockDim.x + threadIdx.x;
    return MxAt{(int64_t(blockIdx.x) * blockDim.y + threadIdx.y) * kMxRows, min(col, vectors - 1), col < vectors};
}

__device__ __forceinline__ uint32_t mx_byte(uint32_t most) {  // of a block whose largest magnitude has these bits as f32
    const uint32_t e = most >> 23;  // floor(log2) + 127, 0 below the normal numbers
    return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}
// The largest of the four lanes of a block. Magnitudes as bits are in the order of the values, and NaN above infinity.
__device__ __forceinline__ uint32_t mx_block_most(uint32_t most) {
    most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
    return max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
}
// Codes and scale byte of a vector. A weight times 2^(127 - byte) is below 8, and exact or next to nothing, in bf16 as in f32: bf16 weights
// are taken two at a time. One by one, their instructions took longer than the memory (128256 x 4096: 244 us, now 205).
__device__ __forceinline__ uint32_t mx_codes(const uint4 (&raw)[1], uint32_t* byte) {
    uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
    const uint32_t m = __vmaxu2(__vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu), __vmaxu2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
    *byte = mx_byte(mx_block_most(max(m << 16, m & 0xFFFF0000u)));
    const uint32_t up = ((254u - (*byte == 255u ? 0u : *byte)) << 7) * 0x00010001u;  // 2^(127 - byte)
    float f[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(w[j]) : "r"(up));
        f[2 * j] = __uint_as_float(w[j] << 16);
        f[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
    return *byte == 255u ? 0u : e2m1_codes(f);
}
__device__ __forceinline__ uint32_t mx_codes(const uint4 (&raw)[2], uint32_t* byte) {
    const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(w[j]);
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(f[j]) & 0x7FFFFFFFu);
    *byte = mx_byte(mx_block_most(most));
    const float up = __uint_as_float((254u - (*byte == 255u ? 0u : *byte)) << 23);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= up;
    return *byte == 255u ? 0u : e2m1_codes(f);
}

template <int DT>
__global__ void __launch_bounds__(512) k_mx_quantize(const void* weight, int64_t row_stride, int vectors, int rows, uint8_t* packed,
                                                     int64_t packed_stride, uint8_t* scales, int64_t scale_stride) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const MxAt at = mx_at(vectors);
    uint4 raw[kMxRows][DT == kF32 ? 2 : 1];
#pragma unroll
    for (int u = 0; u < kMxRows; ++u) {
        const int64_t row = min(at.row0 + u, int64_t(rows) - 1);
        const char* p = static_cast<const char*>(weight) + (row * row_stride + 8 * int64_t(at.col)) * (DT == kF32 ? 4 : 2);
        raw[u][0] = ld_stream16(p);
        if (DT == kF32) raw[u][DT == kF32 ? 1 : 0] = ld_stream16(p + 16);
    }
#pragma unroll
    for (int u = 0; u < kMxRows; ++u) {
        uint32_t byte;
        const uint32_t codes = mx_codes(raw[u], &byte);
        const int64_t row = at.row0 + u;
        if (at.have && row < rows) {
            *reinterpret_cast<uint32_t*>(packed + row * packed_stride + 4 * int64_t(at.col)) = codes;
            if ((at.col & 3) == 0) scales[row * scale_stride + (at.col >> 2)] = uint8_t(byte);
        }
    }
}

// Eight e2m1 codes of a word as bf16, each times 2^(byte - 127): f16 numbers first, whose bits, with the exponent moved down three
// places, are bf16 numbers 2^112 below the values; the two products that bring them up are exact.
__device__ __forceinline__ uint4 mx_values(uint32_t codes, uint32_t byte) {
    const uint32_t scale = (byte == 255u ? 0x7FC0u : byte ? byte << 7 : 0x0040u) * 0x00010001u;
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t low = (h[j] & 0x80008000u) | ((h[j] & 0x7FFF7FFFu) >> 3);
        asm("{\n\t.reg .b32 t;\n\tmul.rn.bf16x2 t, %1, %2;\n\tmul.rn.bf16x2 %0, t, %3;\n\t}"
            : "=r"(h[j])
            : "r"(low), "r"(0x77807780u), "r"(scale));  // 2^112
    }
    return make_uint4(h[0], h[1], h[2], h[3]);
}

__global__ void __launch_bounds__(512) k_mx_dequantize(const uint8_t* packed, int64_t packed_stride, const uint8_t* scales,
                                                       int64_t scale_stride, int vectors, int rows, uint16_t* values, int64_t row_stride) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const MxAt at = mx_at(vectors);
    uint32_t codes[kMxRows], byte[kMxRows];
#pragma unroll
    for (int u = 0; u < kMxRows; ++u) {
        const int64_t row = min(at.row0 + u, int64_t(rows) - 1);
        codes[u] = ld_after_wait(reinterpret_cast<const uint32_t*>(packed + row * packed_stride + 4 * int64_t(at.col)));
        byte[u] = ld_after_wait(scales + row * scale_stride + (at.col >> 2));
    }
#pragma unroll
    for (int u = 0; u < kMxRows; ++u)
        if (at.have && at.row0 + u < rows) st_stream16(values + (at.row0 + u) * row_stride + 8 * int64_t(at.col), mx_values(codes[u], byte[u]));
}

}  // namespace cfgzip
