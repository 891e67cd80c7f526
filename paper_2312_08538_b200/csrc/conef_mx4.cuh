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
// codes of eight scaled elements, nearest even, the first in the low four bits
__device__ __forceinline__ uint32_t mx4_nearest8(const float *v)
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// Code of one scaled element rounded up where floor(65536 f + 1/2) + u >= 65536, f the part of a step that it lies
// above the code below it and u its number, given as noise = 256 u + 128.  Times 2^-126 the smallest normal value, 1, becomes fp32's own
// and the evenly spaced codes below it fp32's subnormals, so that the code is the leading bits of the float throughout and f the 22 that follow; rounded
// towards zero, since the comparison is with a multiple of 32 in them and sees no bit that this drops.  Two places up, without the sign, the code is
// the highest byte, and one addition rounds it.  (A zero stays one.)
__device__ __forceinline__ uint32_t mx4_rounded(float v, uint32_t noise) { return __float_as_uint(__fmul_rz(v, 0x1p-126f)) * 4u + noise; }
__device__ __forceinline__ uint32_t mx4_stochastic(float v, uint32_t noise) { return mx4_rounded(v, noise) >> 24 | (__float_as_uint(v) >> 28 & 8u); }
// the noise of the lower and the upper half of a word
__device__ __forceinline__ uint32_t mx4_noise_lo(uint32_t w) { return __byte_perm(w, 0x80u, 0x5104); }
__device__ __forceinline__ uint32_t mx4_noise_hi(uint32_t w) { return __byte_perm(w, 0x80u, 0x5324); }
// codes of eight scaled elements with their noise; the signs are those that rounding to nearest gives
__device__ __forceinline__ uint32_t mx4_stochastic8(const float *v, const uint32_t (&noise)[8])
{
    uint32_t t[8];
#pragma unroll
    for (int q = 0; q < 8; ++q)
        t[q] = mx4_rounded(v[q], noise[q]);
    const uint32_t even = __byte_perm(__byte_perm(t[0], t[2], 0x0073), __byte_perm(t[4], t[6], 0x0073), 0x5410);
    const uint32_t odd = __byte_perm(__byte_perm(t[1], t[3], 0x0073), __byte_perm(t[5], t[7], 0x0073), 0x5410);
    return (mx4_nearest8(v) & 0x88888888u) | (odd * 16u + even);
}
__device__ __forceinline__ uint32_t mx4_stochastic8(const float *v, uint64_t w0, uint64_t w1)
{
    const uint32_t w[4] = {(uint32_t)w0, (uint32_t)(w0 >> 32), (uint32_t)w1, (uint32_t)(w1 >> 32)};
    uint32_t noise[8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        noise[2 * i] = mx4_noise_lo(w[i]), noise[2 * i + 1] = mx4_noise_hi(w[i]);
    return mx4_stochastic8(v, noise);
}
// the largest of the sizes of three, NaN where one is
__device__ __forceinline__ float mx4_absmax3(float a, float b, float c)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float mx4_absmax2(float a, float b) { return mx4_absmax3(a, b, b); }
// ... of n elements, a multiple of 8, in four chains
template <int N>
__device__ __forceinline__ float mx4_absmax(const float *v)
{
    float m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        m[i] = mx4_absmax2(v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int i = 8; i < N; i += 2)
        m[i / 2 % 4] = mx4_absmax3(m[i / 2 % 4], v[i], v[i + 1]);
    return mx4_absmax2(mx4_absmax3(m[0], m[1], m[2]), m[3]);
}
// values of two codes (low four bits first), still to be scaled
__device__ __forceinline__ float2 mx4_values2(uint32_t byte)
{
    uint32_t h;
    asm("{\n\t.reg .b8 t;\n\tcvt.u8.u32 t, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(h) : "r"(byte));
    return __half22float2(*(const __half2 *)&h);
}
// ... of eight codes
__device__ __forceinline__ void mx4_values8(uint32_t w, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*(const __half2 *)&h[i]);
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
}
// Eight codes from element e of a row on, all of them in it, words: its codes
__device__ __forceinline__ uint32_t mx4_codes8(const uint32_t *words, uint32_t e)
{
    const uint32_t w = e >> 3, s = e & 7u;
    return __funnelshift_r(words[w], s ? words[w + 1] : 0u, 4u * s);
}
// ... times their scales, first and last being those of the first and the last of them
__device__ __forceinline__ void mx4_scaled8(uint32_t codes, uint32_t e, uint32_t first, uint32_t last, float (&v)[8])
{
    mx4_values8(codes, v);
    const float a = mx4_pow(first), b = mx4_pow(last);
    const uint32_t border = 32u - (e & 31u);
#pragma unroll
    for (uint32_t q = 0; q < 8; ++q)
        v[q] = __fmul_rn(v[q], q < border ? a : b);
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
