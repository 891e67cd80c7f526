// Element types of the matrix operators (CONEF_F32, CONEF_BF16, CONEF_F16): loads to fp32, stores rounded once to nearest even.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "conef_internal.h"

namespace conef {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// 16 bytes of elements, to fp32 and back
template <class T>
struct Vec16;
template <>
struct Vec16<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&f)[4])
    {
        f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
template <>
struct Vec16<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
    static __device__ __forceinline__ uint32_t pack2(float a, float b)
    {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *(const uint32_t *)&h;
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) { return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])); }
};
template <>
struct Vec16<__half> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 h = __half22float2(*(const __half2 *)&w[i]);
            f[2 * i] = h.x, f[2 * i + 1] = h.y;
        }
    }
    static __device__ __forceinline__ uint32_t pack2(float a, float b)
    {
        const __half2 h = __floats2half2_rn(a, b);
        return *(const uint32_t *)&h;
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) { return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])); }
};

// Division of 32-bit numbers by `by`, above 1, rounding down: high word of x m, corrected for m's 33rd bit (Granlund and Montgomery, "Division by invariant
// integers using multiplication", 1994, the multiplier rounded up)
struct Divider {
    uint32_t by, m, shift;
};
inline Divider divider(uint32_t by)
{
    Divider d;
    d.by = by;
    d.shift = 0;
    while ((1ull << (d.shift + 1)) < by)   // 2^shift < by <= 2^(shift + 1)
        ++d.shift;
    d.m = (uint32_t)((((1ull << (d.shift + 1)) - by) << 32) / by + 1);
    return d;
}
__device__ __forceinline__ uint32_t divide(uint32_t x, const Divider &d)
{
    const uint32_t h = __umulhi(x, d.m);
    return (h + ((x - h) >> 1)) >> d.shift;
}
inline size_t elem_bytes(int dtype) { return dtype == CONEF_F32 ? 4 : 2; }
// calls f with a value of the type; f returns a code
template <class F>
inline int with_elem(int dtype, F f)
{
    return dtype == CONEF_F32 ? f(float()) : dtype == CONEF_BF16 ? f(__nv_bfloat16()) : f(__half());
}

// A matrix argument: rows of `cols` elements, ld elements apart; a side is below 2^31, and so is a row distance
inline int check_matrix(const void *p, int dtype, int64_t rows, int64_t cols, int64_t ld)
{
    if (dtype != CONEF_F32 && dtype != CONEF_BF16 && dtype != CONEF_F16)
        return CONEF_ERR_INVALID_ARG;
    if (rows < 0 || cols < 0 || (rows > 1 && ld < cols) || ld < 0)
        return CONEF_ERR_INVALID_ARG;
    if (rows >= (1ll << 31) || cols >= (1ll << 31) || ld >= (1ll << 31))
        return CONEF_ERR_UNSUPPORTED;
    if (rows && cols && (!p || ((uintptr_t)p & (elem_bytes(dtype) - 1))))
        return CONEF_ERR_INVALID_ARG;
    return CONEF_OK;
}
inline int check_draw(const conef_draw *d) { return !d || d->worker < 0 || d->tensor < 0 || d->step < 0 ? CONEF_ERR_INVALID_ARG : CONEF_OK; }

// 32 bytes, aligned to that
__device__ __forceinline__ void load32(const void *p, uint32_t (&w)[8])
{
    asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8])
{
    asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]),
                 "r"(w[7])
                 : "memory");
}

// the code of a call's launches; what CUDA says is kept for conef_error_string (conef_api.cu)
int launched(cudaError_t e, const char *what);

}  // namespace conef
