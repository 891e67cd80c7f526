// Product of two matrices held in microscaled 4-bit floats: out[i][j] = sum over k of A[i][k] B[j][k], in fp32, rounded
// once to the output's type.
#include "conef_mx4.cuh"
#include "conef_common.cuh"
#include "conef_elem.cuh"

namespace conef {

// 64 x 64 outputs per CTA, 4 x 4 per thread, a block of 32 elements at a time through shared memory
template <class T>
__global__ void __launch_bounds__(256) k_mx4_matmul(const uint8_t *a, const uint8_t *as, int64_t m, const uint8_t *b, const uint8_t *bs, int64_t n,
                                                    int64_t k, T *out, int64_t ld)
{
    __shared__ float sa[32][65], sb[32][65];
    grid_release();
    grid_wait();
    const int64_t i0 = (int64_t)blockIdx.y * 64, j0 = (int64_t)blockIdx.x * 64, blocks = mx4_blocks(k), tiles = mx4_scale_tiles(k);
    const int tid = threadIdx.x, r = tid >> 2, part = tid & 3, tx = tid & 15, ty = tid >> 4;
    float acc[4][4] = {};
    auto bring = [&](float (*dst)[65], const uint8_t *codes, const uint8_t *scales, int64_t row, int64_t rows, int64_t block) {
        const float s = row < rows ? mx4_pow(scales[mx4_scale_at(row, block, tiles)]) : 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float2 v = row < rows ? mx4_values2(codes[(row * blocks + block) * 16 + part * 4 + q]) : make_float2(0.f, 0.f);
            dst[part * 8 + 2 * q][r] = __fmul_rn(v.x, s);
            dst[part * 8 + 2 * q + 1][r] = __fmul_rn(v.y, s);
        }
    };
    for (int64_t block = 0; block < blocks; ++block) {
        bring(sa, a, as, i0 + r, m, block);
        bring(sb, b, bs, j0 + r, n, block);
        __syncthreads();
#pragma unroll 8
        for (int q = 0; q < 32; ++q)
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    acc[y][x] = __fmaf_rn(sa[q][ty + 16 * y], sb[q][tx + 16 * x], acc[y][x]);
        __syncthreads();
    }
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (i0 + ty + 16 * y < m && j0 + tx + 16 * x < n)
                out[(i0 + ty + 16 * y) * ld + j0 + tx + 16 * x] = from_f32<T>(acc[y][x]);
}

}  // namespace conef

using namespace conef;

extern "C" int conef_mx4_matmul(const void *a_codes, const void *a_scales, int64_t m, const void *b_codes, const void *b_scales, int64_t n, int64_t k,
                                void *out, int dtype, int64_t ld, conef_stream stream)
{
    int rc = check_matrix(out, dtype, m, n, ld);
    if (rc != CONEF_OK)
        return rc;
    if (k < 0)
        return CONEF_ERR_INVALID_ARG;
    if (k >= (1ll << 31) || (m + 63) / 64 > 65535)
        return CONEF_ERR_UNSUPPORTED;
    if (m == 0 || n == 0)
        return CONEF_OK;
    if (k && (!a_codes || !a_scales || !b_codes || !b_scales))
        return CONEF_ERR_INVALID_ARG;
    if ((((uintptr_t)a_codes | (uintptr_t)a_scales | (uintptr_t)b_codes | (uintptr_t)b_scales) & 15) != 0)
        return CONEF_ERR_INVALID_ARG;
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        return launched(launch(k_mx4_matmul<T>, dim3((unsigned)((n + 63) / 64), (unsigned)((m + 63) / 64)), 256, 0, (cudaStream_t)stream,
                               (const uint8_t *)a_codes, (const uint8_t *)a_scales, m, (const uint8_t *)b_codes, (const uint8_t *)b_scales, n, k, (T *)out, ld),
                        "conef_mx4_matmul");
    });
}
