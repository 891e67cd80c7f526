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

// the code of a call's launches; what CUDA says is kept for conef_error_string (conef_api.cu)
int launched(cudaError_t e, const char *what);

}  // namespace conef
