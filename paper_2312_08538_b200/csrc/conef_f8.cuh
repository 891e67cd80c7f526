// 8-bit floats with block scales: elements of CONEF_E4M3 (largest 448) or CONEF_E5M2 (largest 57344), blocks of 128 consecutive elements of a row, or of
// 128 rows by 128 columns, under one scale 2^E kept as the byte E + 127.  E is the least (not below -127) that leaves no element above the
// type's largest, so nothing is clamped.  Byte 255 is a block that held an infinity or a NaN: it decodes to NaN throughout.  A power of two
// as scale loses nothing against the quotient by the maximum but the part of a binade that an 8-bit float's own exponent has to spare, makes x 2^-E and
// code 2^E exact, and is what the tensor cores multiply by themselves.
#pragma once
#include <cuda_fp16.h>

#include "conef_common.cuh"
#include "conef_elem.cuh"

namespace conef {

constexpr int kF8Block = 128;
constexpr uint32_t kF8Nan = 255;
__host__ __device__ inline int64_t f8_blocks(int64_t cols) { return (cols + 127) / 128; }
__host__ __device__ inline int64_t f8_scale_tiles(int64_t cols) { return (cols + 511) / 512; }
// scale byte of a row's block: tiles of 128 rows by 4 blocks, in the order in which the tensor cores take them
__host__ __device__ inline int64_t f8_scale_at(int64_t row, int64_t block, int64_t tiles)
{
    return ((row >> 7) * tiles + (block >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}
// ... by one multiplication
__device__ __forceinline__ uint64_t f8_scale_at32(uint32_t row, uint32_t block, uint32_t tiles)
{
    return (uint64_t)(row >> 7) * (tiles * 512u) + ((block >> 2) * 512u + (row & 31u) * 16u + ((row >> 5) & 3u) * 4u + (block & 3u));
}

__device__ __forceinline__ float absmax4(const float *v) { return absmax3(absmax2(v[0], v[1]), v[2], v[3]); }
// scale byte of a block from the largest |x| in it as bits (as integers NaN > infinity > every finite value)
__device__ __forceinline__ uint32_t f8_scale(uint32_t abs_bits, int kind)
{
    // the exponent, less that of the largest value; one more where the significand is above 1.75, its significand
    const int b = (int)((abs_bits + 0x001FFFFFu) >> 23) - (kind == CONEF_E4M3 ? 8 : 15);
    return abs_bits >= 0x7F800000u ? kF8Nan : (uint32_t)max(b, 0);
}
// 2^-E (for the byte 255: zero)
__device__ __forceinline__ float f8_inv(uint32_t byte) { return byte == kF8Nan ? 0.f : __uint_as_float((254u - byte) << 23); }
// 2^E (for the byte 255: NaN)
__device__ __forceinline__ float f8_pow(uint32_t byte) { return __uint_as_float(byte == 0u ? 0x00400000u : byte == kF8Nan ? 0x7FFFFFFFu : byte << 23); }

// codes of four scaled elements, nearest even, the first in the low byte
__device__ __forceinline__ uint32_t f8_codes4(const float *v, int kind)
{
    uint32_t r;
    if (kind == CONEF_E4M3)
        asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\tmov.b32 %0, {a, b};\n\t}"
            : "=r"(r)
            : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]));
    else
        asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e5m2x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e5m2x2.f32 b, %4, %3;\n\tmov.b32 %0, {a, b};\n\t}"
            : "=r"(r)
            : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]));
    return r;
}
// N elements scaled by 2^-E and rounded; a block that is NaN has codes of zero
template <int N>
__device__ __forceinline__ void f8_encode(const float *v, uint32_t byte, int kind, uint32_t *code)
{
    const float inv = f8_inv(byte);
    const uint64_t both = pair_of(inv, inv);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        float s[4] = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
        mul2(s[0], s[1], both), mul2(s[2], s[3], both);
        const uint32_t c = f8_codes4(s, kind);
        code[i] = byte == kF8Nan ? 0u : c;
    }
}
// values of four codes (before the scale)
__device__ __forceinline__ void f8_values4(uint32_t w, int kind, float *v)
{
    uint32_t lo, hi;
    if (kind == CONEF_E4M3)
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
    else
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e5m2x2 %0, a;\n\tcvt.rn.f16x2.e5m2x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
    const float2 a = __half22float2(*(const __half2 *)&lo), b = __half22float2(*(const __half2 *)&hi);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}
// ------------------------------------------------------------------ rows by warps
// A warp takes 32 N elements of a row at a time, N (8 or 16) to a lane: two or four blocks.  Where rows are aligned (VEC) a lane's are consecutive; else it has every
// 32nd of a block, four of each block, so that single elements come by whole lines.
template <bool VEC, int N>
__device__ __forceinline__ uint32_t lane_col(uint32_t c0, int lane, int q) { return VEC ? c0 + lane * N + q : c0 + (q >> 2) * 128 + (q & 3) * 32 + lane; }

// Bytes 0 to 3 of four neighbouring lanes, turned: lane i has byte i of each.  So codes of every 32nd element of a block leave, and come, as words (8192 x 1601 in bf16
// to codes byte by byte 14.7 us, values of codes 20.8).
__device__ __forceinline__ uint32_t bytes_turned(uint32_t w, int lane)
{
    uint32_t o = __shfl_xor_sync(0xffffffffu, w, 1);
    w = __byte_perm(w, o, lane & 1 ? 0x3715 : 0x6240);
    o = __shfl_xor_sync(0xffffffffu, w, 2);
    return __byte_perm(w, o, lane & 2 ? 0x3276 : 0x5410);
}

// 32 bytes that other kernels may read again
__device__ __forceinline__ void load32_keep(const void *p, uint32_t (&w)[8])
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void store32_keep(void *p, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]),
                 "r"(w[7])
                 : "memory");
}
// N elements of a lane, as they lie in memory (VEC: in sizeof(T) N / 4 words) or one to a word; zero behind the row's end
template <class T, bool VEC, int N = 16>
struct Piece {
    static constexpr int WORDS = VEC ? (int)sizeof(T) * N / 4 : N;
    uint32_t w[WORDS];

    __device__ __forceinline__ void load(const T *row, uint32_t c0, uint32_t cols, int lane, bool aligned32)
    {
        if constexpr (VEC) {
            const uint32_t c = c0 + lane * N;
            if (c + N <= cols) {
                if (WORDS >= 8 && aligned32) {
#pragma unroll
                    for (int i = 0; i + 8 <= WORDS; i += 8)
                        load32_keep((const uint32_t *)(row + c) + i, *(uint32_t(*)[8])(w + i));
                } else {
#pragma unroll
                    for (int i = 0; i < WORDS; i += 4) {
                        const uint4 q = *(const uint4 *)((const uint32_t *)(row + c) + i);
                        w[i] = q.x, w[i + 1] = q.y, w[i + 2] = q.z, w[i + 3] = q.w;
                    }
                }
            } else {
                using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
                const Bits *p = (const Bits *)(row + c);
#pragma unroll
                for (int i = 0; i < WORDS; ++i) {
                    if constexpr (sizeof(T) == 2)
                        w[i] = (c + 2 * i < cols ? (uint32_t)p[2 * i] : 0u) | (c + 2 * i + 1 < cols ? (uint32_t)p[2 * i + 1] << 16 : 0u);
                    else
                        w[i] = c + i < cols ? (uint32_t)p[i] : 0u;
                }
            }
        } else {
            using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const uint32_t c = lane_col<VEC, N>(c0, lane, q);
                w[q] = c < cols ? (uint32_t)((const Bits *)row)[c] : 0u;
            }
        }
    }
    __device__ __forceinline__ void unpack(float *v) const
    {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < WORDS; i += 4)
                Vec16<T>::unpack(make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]), *(float(*)[Vec16<T>::N])(v + i / 4 * Vec16<T>::N));
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                if constexpr (sizeof(T) == 2) {
                    const uint16_t h = (uint16_t)w[q];
                    v[q] = to_f32(*(const T *)&h);
                } else {
                    v[q] = __uint_as_float(w[q]);
                }
            }
        }
    }
    __device__ __forceinline__ void pack(const float *v)
    {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < WORDS; i += 4) {
                const uint4 q = Vec16<T>::pack(*(const float(*)[Vec16<T>::N])(v + i / 4 * Vec16<T>::N));
                w[i] = q.x, w[i + 1] = q.y, w[i + 2] = q.z, w[i + 3] = q.w;
            }
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const T t = from_f32<T>(v[q]);
                if constexpr (sizeof(T) == 2)
                    w[q] = *(const uint16_t *)&t;
                else
                    w[q] = __float_as_uint(t);
            }
        }
    }
    __device__ __forceinline__ void store(T *row, uint32_t c0, uint32_t cols, int lane, bool aligned32) const
    {
        using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
        if constexpr (VEC) {
            const uint32_t c = c0 + lane * N;
            if (c + N <= cols) {
                if (WORDS >= 8 && aligned32) {
#pragma unroll
                    for (int i = 0; i + 8 <= WORDS; i += 8)
                        store32_keep((uint32_t *)(row + c) + i, *(const uint32_t(*)[8])(w + i));
                } else {
#pragma unroll
                    for (int i = 0; i < WORDS; i += 4)
                        *(uint4 *)((uint32_t *)(row + c) + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
                }
            } else {
                Bits *p = (Bits *)(row + c);
#pragma unroll
                for (int q = 0; q < N; ++q)
                    if (c + q < cols)
                        p[q] = sizeof(T) == 2 ? (Bits)(w[q / 2] >> (16 * (q & 1))) : (Bits)w[q % WORDS];
            }
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const uint32_t c = lane_col<VEC, N>(c0, lane, q);
                if (c < cols)
                    ((Bits *)row)[c] = (Bits)w[q];
            }
        }
    }
};

// The codes and scales of a warp's 32 N elements from c0 (a multiple of them) on; scales: where the row's byte of the first block lies.  Blocks that do not exist get the
// byte zero; `there`: the row does.
template <class T, bool VEC, int N = 16>
__device__ __forceinline__ void f8_store_row(const float *v, uint32_t c0, uint32_t blocks, int lane, int kind, bool there, uint8_t *codes_row, uint8_t *scales)
{
    if constexpr (VEC) {
        constexpr int LANES = 128 / N;   // of a block
        uint32_t most = __float_as_uint(absmax<N>(v));
#pragma unroll
        for (int o = 1; o < LANES; o *= 2)
            most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
        const uint32_t byte = f8_scale(most, kind), block = c0 / 128 + lane / LANES;
        uint32_t code[N / 4];
        f8_encode<N>(v, byte, kind, code);
        if (there && block < blocks) {
            if constexpr (N == 16)
                *(uint4 *)(codes_row + c0 + lane * N) = make_uint4(code[0], code[1], code[2], code[3]);
            else
                *(uint2 *)(codes_row + c0 + lane * N) = make_uint2(code[0], code[1]);
        }
        if (lane % LANES == 0)
            scales[lane / LANES] = (uint8_t)(there && block < blocks ? byte : 0u);
    } else {
        uint32_t bytes = 0;
#pragma unroll
        for (int b = 0; b < N / 4; ++b) {
            const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(absmax4(v + 4 * b)));
            const uint32_t byte = f8_scale(most, kind);
            uint32_t code;
            f8_encode<4>(v + 4 * b, byte, kind, &code);
            code = bytes_turned(code, lane);
            if (there && c0 / 128 + b < blocks) {
                bytes |= byte << (8 * b);
                *(uint32_t *)(codes_row + c0 + b * 128 + (lane & 3) * 32 + (lane >> 2) * 4) = code;
            }
        }
        if (lane < N / 4)
            scales[lane] = (uint8_t)(bytes >> (8 * lane));
    }
}

// whether rows of a matrix begin on 16 and on 32 bytes
template <class T>
inline bool rows_on(const void *p, int64_t rows, int64_t ld, uintptr_t bytes) { return (((uintptr_t)p | (rows > 1 ? (uint64_t)ld * sizeof(T) : 0u)) & (bytes - 1)) == 0; }

// A norm's values h r w as a form has them: those of the exact product.  They are rounded to fp32 "to odd": towards zero, with the last bit set where
// something was lost, so that a rounding to fewer bits behind it, and a comparison with a power of two times 1.75, see which side of a tie they lie on.
// (Both products are held as a pair of floats, 48 bits; the pair's lower part, and with it the side of a tie, is lost below 2^-100.)
__device__ __forceinline__ float norm_value(float h, float w, float r)
{
    const float p = __fmul_rn(h, r), pe = __fmaf_rn(h, r, -p), y = __fmul_rn(p, w);   // (h r, unlike h w, is at most the root of the row's length)
    const float e = __fmaf_rn(pe, w, __fmaf_rn(p, w, -y));
    const float s = __fadd_rn(y, e), t = __fsub_rn(e, __fsub_rn(s, y));
    const uint32_t b = __float_as_uint(s);
    const uint32_t to = t == 0.f || (b & 1u) ? b : ((__float_as_uint(t) ^ b) >> 31 ? b - 1u : b + 1u);
    return fabsf(s) < __uint_as_float(0x7F800000u) ? __uint_as_float(to) : s;
}
// ... of N elements.  Ties of the 8-bit types, and 1.75 times powers of two, are multiples of 2^19 units of fp32's last place; two ordinary roundings are off by three
// units at most, so a value further from those than that is on the right side as it is.  One in 2^16 is not, and its thread's are formed exactly.
// All lanes of a warp call; elements that are not `real` become zero.
template <int N>
__device__ __forceinline__ void norm_values(float *v, const float *w, float r, bool real)
{
    static_assert(N % 4 == 0, "");
    float y[N];
    uint32_t near = 0xFFFFFFFFu;   // (shifted, so that what is above the 19 bits falls off)
    const uint64_t root = pair_of(r, r);
#pragma unroll
    for (int q = 0; q < N; q += 2) {
        y[q] = v[q], y[q + 1] = v[q + 1];
        mul2(y[q], y[q + 1], root);
        mul2(y[q], y[q + 1], pair_of(w[q], w[q + 1]));
        near = __vimin3_u32(near, __float_as_uint(y[q]) * 8192u + 4u * 8192u, __float_as_uint(y[q + 1]) * 8192u + 4u * 8192u);
    }
    if (__any_sync(0xffffffffu, real && near <= 8u * 8192u)) {
        bool some = false;   // (zeros, which sums of few bits often are, look the same and are exact)
#pragma unroll
        for (int q = 0; q < N; ++q)
            some = some || (__float_as_uint(y[q]) * 8192u + 4u * 8192u <= 8u * 8192u && v[q] != 0.f);
        if (__any_sync(0xffffffffu, real && some)) {
#pragma unroll
            for (int q = 0; q < N; ++q)
                y[q] = v[q] == 0.f ? y[q] : norm_value(v[q], w[q], r);
        }
    }
#pragma unroll
    for (int q = 0; q < N; ++q)
        v[q] = real ? y[q] : 0.f;
}

// a form that a launch writes, or its transpose's
struct F8Out {
    uint8_t *codes, *scales, *codes_t, *scales_t;
    int kind;
};
// x's columns (and rows, where out.codes is set) to forms; rstd, w: of norm_value(), or NULL.  Blocks of 128 x 128 where square.
cudaError_t f8_tiles(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, const float *rstd, const void *w, bool w32, bool square, const F8Out &out,
                     cudaStream_t s);

}  // namespace conef
