// Dropout whose mask is drawn from the counter-based stream in every pass and never stored: y = x 65536 / (65536 - off)
// where the element's number is at least off, else 0; and a residual added in the same pass.
#include "conef_draw.cuh"
#include "conef_common.cuh"
#include "conef_elem.cuh"

namespace conef {

// a group of four columns per thread
template <class T, bool ADD>
__global__ void __launch_bounds__(256) k_dropout(const T *x, const T *add, T *out, int64_t rows, uint32_t cols, int64_t x_ld,
                                                 int64_t add_ld, int64_t out_ld, uint64_t stream, Dropout drop)
{
    grid_release();
    const uint32_t groups = (cols + 3) / 4;
    grid_wait();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * groups; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / groups;
        const uint32_t c0 = (uint32_t)(i - row * groups) * 4u;
        const uint64_t word = draw_word(stream, (uint64_t)i, kDrawDropout);
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
            const uint32_t c = c0 + q;
            if (c < cols) {
                const float r = ADD ? to_f32(add[row * add_ld + c]) : 0.f;
                const float v = __fmaf_rn(to_f32(x[row * x_ld + c]), drop.scale, r);
                out[row * out_ld + c] = from_f32<T>(draw_of(word, q) >= drop.off ? v : r);
            }
        }
    }
}

}  // namespace conef

using namespace conef;

extern "C" int conef_dropout(const void *x, const void *add, void *out, int dtype, int64_t rows, int64_t cols, int64_t x_ld, int64_t add_ld,
                             int64_t out_ld, double p, const conef_draw *draw, conef_stream stream)
{
    int rc = check_matrix(x, dtype, rows, cols, x_ld);
    if (rc == CONEF_OK)
        rc = check_matrix(out, dtype, rows, cols, out_ld);
    if (rc == CONEF_OK && add)
        rc = check_matrix(add, dtype, rows, cols, add_ld);
    if (rc == CONEF_OK && !(p >= 0.0 && p <= 1.0))
        rc = CONEF_ERR_INVALID_ARG;
    if (rc == CONEF_OK)
        rc = check_draw(draw);
    if (rc != CONEF_OK || rows == 0 || cols == 0)
        return rc;
    const uint64_t st = draw_stream(draw->seed, draw->worker, draw->tensor, draw->step);
    const Dropout drop = dropout_of(p);
    const int64_t ctas = (rows * ((cols + 3) / 4) + 255) / 256;
    const dim3 grid((unsigned)(ctas < kPlanSMs * 64 ? ctas : kPlanSMs * 64));
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        const T *xp = (const T *)x, *ap = (const T *)add;
        T *op = (T *)out;
        return launched(add ? launch(k_dropout<T, true>, grid, 256, 0, (cudaStream_t)stream, xp, ap, op, rows, (uint32_t)cols, x_ld, add_ld, out_ld, st, drop)
                            : launch(k_dropout<T, false>, grid, 256, 0, (cudaStream_t)stream, xp, ap, op, rows, (uint32_t)cols, x_ld, add_ld, out_ld, st, drop),
                        "conef_dropout");
    });
}
