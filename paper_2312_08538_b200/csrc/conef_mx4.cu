// Quantisation to microscaled 4-bit floats (conef_mx4.cuh), of a matrix and of its transpose, behind a dropout where one is
// asked for, and the way back.
#include "conef_mx4.cuh"
#include "conef_common.cuh"
#include "conef_elem.cuh"

namespace conef {

// A warp per block, an element per lane; blocks of rows and columns that only the tiles of scales have get their zero.
template <class T, bool TRANSPOSED>
__global__ void __launch_bounds__(256) k_mx4_quantise(const T *x, int64_t rows, int64_t cols, int64_t ld, uint64_t stream, Dropout drop,
                                                      int stochastic, uint8_t *codes, uint8_t *scales)
{
    grid_release();
    grid_wait();
    const int lane = threadIdx.x & 31;
    const int64_t frows = TRANSPOSED ? cols : rows, fcols = TRANSPOSED ? rows : cols;   // of the form
    const int64_t blocks = mx4_blocks(fcols), tiles = mx4_scale_tiles(fcols), padded = (frows + 127) / 128 * 128;
    const uint64_t groups = (uint64_t)(cols + 3) / 4;
    for (int64_t u = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5; u < padded * tiles * 4; u += (int64_t)gridDim.x * 8) {
        const int64_t row = u / (tiles * 4), block = u - row * (tiles * 4), c = block * 32 + lane;
        float v = 0.f;
        uint32_t draw = 0;
        if (row < frows && c < fcols) {
            const int64_t r = TRANSPOSED ? c : row, k = TRANSPOSED ? row : c;
            const uint64_t group = (uint64_t)r * groups + (uint64_t)(k >> 2);
            v = to_f32(x[r * ld + k]);
            if (drop.off)
                v = draw_of(draw_word(stream, group, kDrawDropout), (uint32_t)k) >= drop.off ? __fmul_rn(v, drop.scale) : 0.f;
            if (stochastic)
                draw = draw_of(draw_word(stream, group, kDrawRounding), (uint32_t)k);
        }
        const uint32_t byte = mx4_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7FFFFFFFu));
        v = __fmul_rn(v, mx4_inv(byte));
        uint32_t code = stochastic ? mx4_stochastic(v, draw) : mx4_nearest2(v, 0.f) & 0xFu;
        code = byte == kMx4Nan ? 0u : code;
        code |= __shfl_down_sync(0xffffffffu, code, 1) << 4;
        if (lane == 0)
            scales[mx4_scale_at(row, block, tiles)] = (uint8_t)(row < frows && block < blocks ? byte : 0u);
        if (row < frows && block < blocks && !(lane & 1))
            codes[(row * blocks + block) * 16 + (lane >> 1)] = (uint8_t)code;
    }
}

// two elements per thread
template <class T>
__global__ void __launch_bounds__(256) k_mx4_dequantise(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, T *out,
                                                        int64_t ld)
{
    grid_release();
    grid_wait();
    const int64_t blocks = mx4_blocks(cols), tiles = mx4_scale_tiles(cols);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * blocks * 16; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / (blocks * 16), at = i - row * (blocks * 16), c = at * 2;
        const float2 v = mx4_values2(codes[i]);
        const float s = mx4_pow(scales[mx4_scale_at(row, at >> 4, tiles)]);
        if (c < cols)
            out[row * ld + c] = from_f32<T>(__fmul_rn(v.x, s));
        if (c + 1 < cols)
            out[row * ld + c + 1] = from_f32<T>(__fmul_rn(v.y, s));
    }
}

static dim3 grid_of(int64_t ctas) { return dim3((unsigned)(ctas < 1 ? 1 : ctas < kPlanSMs * 64 ? ctas : kPlanSMs * 64)); }

}  // namespace conef

using namespace conef;

extern "C" {

int conef_mx4_bytes(int64_t rows, int64_t cols, size_t *code_bytes, size_t *scale_bytes)
{
    if (rows < 0 || cols < 0)
        return CONEF_ERR_INVALID_ARG;
    if (rows >= (1ll << 31) || cols >= (1ll << 31))
        return CONEF_ERR_UNSUPPORTED;
    if (code_bytes)
        *code_bytes = (size_t)rows * (size_t)mx4_blocks(cols) * 16;
    if (scale_bytes)
        *scale_bytes = (size_t)((rows + 127) / 128) * (size_t)mx4_scale_tiles(cols) * 512;
    return CONEF_OK;
}

int conef_mx4_quantise(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, double p, int stochastic, const conef_draw *draw,
                       void *codes, void *scales, void *codes_t, void *scales_t, conef_stream stream)
{
    int rc = check_matrix(x, dtype, rows, cols, ld);
    if (rc != CONEF_OK)
        return rc;
    if (!(p >= 0.0 && p <= 1.0) || !codes != !scales || !codes_t != !scales_t || !(codes || codes_t))
        return CONEF_ERR_INVALID_ARG;
    if ((((uintptr_t)codes | (uintptr_t)scales | (uintptr_t)codes_t | (uintptr_t)scales_t) & 15) != 0)
        return CONEF_ERR_INVALID_ARG;
    const Dropout drop = dropout_of(p);
    if ((drop.off || stochastic) && (rc = check_draw(draw)) != CONEF_OK)
        return rc;
    if (rows == 0 || cols == 0)
        return CONEF_OK;
    const uint64_t st = draw ? draw_stream(draw->seed, draw->worker, draw->tensor, draw->step) : 0;
    cudaStream_t s = (cudaStream_t)stream;
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        if (codes)
            rc = launched(launch(k_mx4_quantise<T, false>, grid_of((rows + 127) / 128 * 128 * mx4_scale_tiles(cols) * 4 / 8), 256, 0, s, (const T *)x,
                                 rows, cols, ld, st, drop, stochastic, (uint8_t *)codes, (uint8_t *)scales), "conef_mx4_quantise");
        if (codes_t && rc == CONEF_OK)
            rc = launched(launch(k_mx4_quantise<T, true>, grid_of((cols + 127) / 128 * 128 * mx4_scale_tiles(rows) * 4 / 8), 256, 0, s, (const T *)x,
                                 rows, cols, ld, st, drop, stochastic, (uint8_t *)codes_t, (uint8_t *)scales_t), "conef_mx4_quantise");
        return rc;
    });
}

int conef_mx4_dequantise(const void *codes, const void *scales, int64_t rows, int64_t cols, void *out, int dtype, int64_t ld, conef_stream stream)
{
    int rc = check_matrix(out, dtype, rows, cols, ld);
    if (rc != CONEF_OK || rows == 0 || cols == 0)
        return rc;
    if (!codes || !scales || (((uintptr_t)codes | (uintptr_t)scales) & 15) != 0)
        return CONEF_ERR_INVALID_ARG;
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        return launched(launch(k_mx4_dequantise<T>, grid_of((rows * mx4_blocks(cols) * 16 + 255) / 256), 256, 0, (cudaStream_t)stream, (const uint8_t *)codes,
                               (const uint8_t *)scales, rows, cols, (T *)out, ld), "conef_mx4_dequantise");
    });
}

}  // extern "C"
