// Microscaled 4-bit floating point: elements e2m1 (sign, two bits of exponent, one of mantissa: 0 .5 1 1.5 2 3 4 6), one power of two per 32
// elements of a row, stored as its exponent + 127 (255: the block is NaN).  Rows of codes are 16 bytes per block, element 2i in the low
// nibble of byte i; rows of scales are padded to whole 16 bytes, so that every row of either array starts on a 16-byte boundary.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

namespace llvq {

constexpr int kMxBlock = 32;            // elements per scale
constexpr int kMxBlockBytes = 16;       // codes of a block

__host__ __device__ inline int64_t mx_blocks(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }
__host__ __device__ inline int64_t mx_scale_pitch(int64_t cols) { return (mx_blocks(cols) + 15) / 16 * 16; }
__host__ __device__ inline int64_t mx_code_pitch(int64_t cols) { return mx_blocks(cols) * kMxBlockBytes; }

// The value of a scale byte: 2^(e - 127), which for e = 0 is a subnormal; NaN for 255.
__device__ __forceinline__ float mx_scale_value(uint32_t e)
{
    return __uint_as_float(e == 0u ? 0x00400000u : e == 255u ? 0x7fc00000u : e << 23);
}

// The eight elements of a word of codes, in order.  Every e2m1 value is a binary16 number, and the conversion is one instruction per two.
__device__ __forceinline__ void mx_expand8(uint32_t w, float v[8])
{
    uint32_t h[4];
    asm("{\n .reg .b8 b0, b1, b2, b3;\n mov.b32 {b0, b1, b2, b3}, %4;\n"
        " cvt.rn.f16x2.e2m1x2 %0, b0;\n cvt.rn.f16x2.e2m1x2 %1, b1;\n cvt.rn.f16x2.e2m1x2 %2, b2;\n cvt.rn.f16x2.e2m1x2 %3, b3;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}

// Eight values to e2m1, to nearest with ties to the even code, at most 6 in magnitude.
__device__ __forceinline__ uint32_t mx_pack8(const float v[8])
{
    uint32_t w;
    asm("{\n .reg .b8 b0, b1, b2, b3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n mov.b32 %0, {b0, b1, b2, b3};\n}"
        : "=r"(w) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return w;
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi)
{
    const __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}

}  // namespace llvq
