// Microscaled 4-bit floats: blocks of 32 elements, each a sign, two exponent bits and one mantissa bit (0, 0.5, 1, 1.5, 2, 3,
// 4, 6), under one scale 2^E kept as the byte E + 127.  E is the least (not below -127) that leaves no element above 6, so nothing is
// clamped and the element that makes the scale loses half a step at most.  Byte 255 is a block that held an infinity or a
// NaN: it decodes to NaN throughout.  A scale is a power of two, so x 2^-E and code 2^E
// are exact in fp32 (but for x far below its block's maximum, which is 0 or 0.5 all the same, and for 4 2^126, which is infinite).
#pragma once
#include <cuda_fp16.h>

#include "conef_draw.cuh"

namespace conef {

constexpr int kMx4Block = 32;
constexpr uint32_t kMx4Nan = 255;

// scale byte of a block from the largest |x| in it as bits (as integers NaN > infinity > every finite value)
__device__ __forceinline__ uint32_t mx4_scale(uint32_t abs_bits)
{
    // the exponent, less 2; one more where the significand is above 1.5
    const int b = (int)((abs_bits + 0x003FFFFFu) >> 23) - 2;
    return abs_bits >= 0x7F800000u ? kMx4Nan : (uint32_t)max(b, 0);
}
// 2^-E (for the byte 255: zero)
__device__ __forceinline__ float mx4_inv(uint32_t byte) { return byte == kMx4Nan ? 0.f : __uint_as_float((254u - byte) << 23); }
// 2^E (for the byte 255: NaN)
__device__ __forceinline__ float mx4_pow(uint32_t byte)
{
    return __uint_as_float(byte == 0u ? 0x00400000u : byte == kMx4Nan ? 0x7FFFFFFFu : byte << 23);
}

// codes of two scaled elements, nearest even, lo in the low four bits
__device__ __forceinline__ uint32_t mx4_nearest2(float lo, float hi)
{
    uint32_t r;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Code of one scaled element rounded up where floor(65536 f + 1/2) + u >= 65536, f the part of a step that it lies
// above the code below it and u its number.  From 1 on the codes are the leading bits of the float; below 1 they are evenly spaced
// like those of [1, 2), and 1 is added, rounded towards zero: the comparison is with a multiple of 2^-17 and
// sees no bit that this drops.
__device__ __forceinline__ uint32_t mx4_stochastic(float v, uint32_t u)
{
    const uint32_t bits = __float_as_uint(v), mag = bits & 0x7FFFFFFFu;
    const bool small = mag < 0x3F800000u;
    const uint32_t y = __float_as_uint(__fadd_rz(__uint_as_float(mag), small ? 1.f : 0.f));
    return ((y + (u << 6) + 32u) >> 22) - (small ? 254u : 252u) + ((bits >> 28) & 8u);
}
// values of two codes (low four bits first), still to be scaled
__device__ __forceinline__ float2 mx4_values2(uint32_t byte)
{
    uint32_t h;
    asm("{\n\t.reg .b8 t;\n\tcvt.u8.u32 t, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(h) : "r"(byte));
    return __half22float2(*(const __half2 *)&h);
}
__device__ __forceinline__ float mx4_value(uint32_t code)   // one code
{
    return mx4_values2(code).x;
}

// Where a matrix' form keeps things: a row's codes are 16 bytes per block; scales stand in tiles of 128 rows by 4 blocks, 512 bytes
// each, the order in which the tensor cores' scale operand is loaded, with zeros for rows and blocks that do not exist.
__host__ __device__ __forceinline__ int64_t mx4_blocks(int64_t cols) { return (cols + kMx4Block - 1) / kMx4Block; }
__host__ __device__ __forceinline__ int64_t mx4_scale_tiles(int64_t cols) { return (cols + 127) / 128; }   // along a row
__host__ __device__ __forceinline__ int64_t mx4_scale_at(int64_t row, int64_t block, int64_t tiles)
{
    return ((row >> 7) * tiles + (block >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

}  // namespace conef
