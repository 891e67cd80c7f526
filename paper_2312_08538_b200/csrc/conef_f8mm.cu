// Product of two matrices held in 8-bit floats with block scales (conef_f8.cuh), out[i][j] = sum over k of A[i][k] B[j][k], in fp32 on the tensor
// cores' block-scaled path and rounded once to the output's type (the kernel: conef_mm.cuh).
//
// The instruction has a scale per 32 elements; a block of 128 is four of them, that all name the same of the four bytes that a column of scales has.  So
// sums stay in tensor memory from the first product to the last, where scales that are not powers of two would have them out and multiplied for every block.
#include "conef_f8.cuh"
#include "conef_mm.cuh"

namespace conef {

struct F8Format {
    static constexpr uint32_t kStageK = 128, kStepK = 32, kTiles = 1, kTileStages = 4, kScaleColumns = 12;
    static int64_t row_bytes(int64_t k) { return f8_blocks(k) * 128; }
    static int64_t scale_tiles(int64_t k) { return f8_scale_tiles(k); }
    static int per_step(int pair, int width)
    {
        static const int table[2][4] = {{45, 52, 67, 88}, {0, 48, 60, 73}};
        return table[pair][width];
    }
    static int per_tile(int width)
    {
        static const int table[4] = {700, 970, 1240, 2450};
        return table[width];
    }
    template <bool PAIR>
    static __device__ __forceinline__ uint32_t instruction(const MmArgs &P) { return tc::f8_instruction<PAIR>(P.bn, P.kind_a, P.kind_b); }
    // stage ks: its scales to tensor memory, then the products
    template <bool PAIR>
    static __device__ __forceinline__ void issue(const MmArgs &P, uint32_t d, uint32_t a, uint32_t b, uint32_t sc, uint32_t instruction, uint32_t sa, uint32_t sb, uint32_t shift,
                                                 uint32_t scale_rows, uint32_t ks)
    {
        const uint32_t steps = P.k_steps - ks * 4u, number = ks & 3u;
        tc::scales_copy<PAIR>(sa, sc);
        tc::scales_copy<PAIR>(sb, sc + 32);
        if (scale_rows > 1)
            tc::scales_copy<PAIR>(sb + 4, sc + 64);
        instruction |= number << 4 | number << 29;
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t)
            if (t < steps)
                tc::f8_product<PAIR>(d, a + 2 * t, b + 2 * t, instruction, sa, sb + shift, ks + t);
    }
};

// ------------------------------------------------------------------ few rows against many
// Up to 16 rows of one side (tokens) against all of the other's (a weight's), which are read once: 1 x 6400 x 1600 are 10 MB, 1.6 us.  A tile of tcgen05.mma would have
// 128 rows with one used, and a chain of copies and barriers for each (9.5 us); here a warp takes 16 rows of the weight and a share of the blocks along k, eight
// warps a row group, straight from memory to registers, where codes become fp16 (exactly) for mma.m16n8k16.  A lane has 16 bytes of two rows
// and of a token at a time: the instruction's order of k is any that both sides share.  Sums of a block are fp32, times its two scales' power of two, and added in fp32.
constexpr int kFewWarps = 8;
// four codes to two pairs of fp16
__device__ __forceinline__ void few_halves(uint32_t w, uint32_t kind, uint32_t &lo, uint32_t &hi)
{
    if (kind == CONEF_E4M3)
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
    else
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e5m2x2 %0, a;\n\tcvt.rn.f16x2.e5m2x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ void few_product(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2])
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// v 2^(E + F) for scale bytes e and f, in two steps, neither of which leaves the range where the result does not
__device__ __forceinline__ float few_scaled(float v, uint32_t e, uint32_t f)
{
    const int s = (int)(e + f) - 254, half = s >> 1;
    const float x = __fmul_rn(__fmul_rn(v, f8_pow((uint32_t)(half + 127))), f8_pow((uint32_t)(s - half + 127)));
    return e == kF8Nan || f == kF8Nan ? __uint_as_float(0x7FFFFFFFu) : x;
}
struct FewArgs {
    const uint8_t *w, *ws, *t, *ts;   // codes and scales: the weight's, the tokens'
    uint32_t rows, tokens, blocks, tiles;
    uint32_t kind_w, kind_t;
    int64_t row_step, token_step;     // of the output, in elements
};
template <class T, int NT>   // NT: groups of eight tokens
__global__ void __launch_bounds__(kFewWarps * 32) k_f8_few(const __grid_constant__ FewArgs P, T *out)
{
    __shared__ float part[kFewWarps][NT * 8][17];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q = lane & 3, g = lane >> 2;
    const uint64_t pitch = (uint64_t)P.blocks * 128u;
    const uint32_t row0 = blockIdx.x * 16 + g, row1 = row0 + 8;
    const uint8_t *const w0 = P.w + min(row0, P.rows - 1) * pitch + q * 16, *const w1 = P.w + min(row1, P.rows - 1) * pitch + q * 16;   // (what does not exist is not stored)
    const uint8_t *t[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
        t[n] = P.t + min((uint32_t)(n * 8 + g), P.tokens - 1) * pitch + q * 16;
    float sum[NT][4] = {};
    grid_wait();
#pragma unroll 2
    for (uint32_t b = warp; b < P.blocks; b += kFewWarps) {
        uint4 x[2], y[2], z[NT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            x[h] = __ldcs((const uint4 *)(w0 + b * 128ull + h * 64));
            y[h] = __ldcs((const uint4 *)(w1 + b * 128ull + h * 64));
#pragma unroll
            for (int n = 0; n < NT; ++n)
                z[n][h] = *(const uint4 *)(t[n] + b * 128ull + h * 64);
        }
        const uint32_t e0 = P.ws[f8_scale_at32(row0, b, P.tiles)], e1 = P.ws[f8_scale_at32(row1, b, P.tiles)];   // (scales of rows that do not exist do)
        float d[NT][4] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t xw[4] = {x[h].x, x[h].y, x[h].z, x[h].w}, yw[4] = {y[h].x, y[h].y, y[h].z, y[h].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t a[4];
                few_halves(xw[i], P.kind_w, a[0], a[2]);
                few_halves(yw[i], P.kind_w, a[1], a[3]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint32_t zw[4] = {z[n][h].x, z[n][h].y, z[n][h].z, z[n][h].w};
                    uint32_t c[2];
                    few_halves(zw[i], P.kind_t, c[0], c[1]);
                    few_product(d[n], a, c);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t f0 = P.ts[f8_scale_at32(n * 8 + 2 * q, b, P.tiles)], f1 = P.ts[f8_scale_at32(n * 8 + 2 * q + 1, b, P.tiles)];
            sum[n][0] = __fadd_rn(sum[n][0], few_scaled(d[n][0], e0, f0)), sum[n][1] = __fadd_rn(sum[n][1], few_scaled(d[n][1], e0, f1));
            sum[n][2] = __fadd_rn(sum[n][2], few_scaled(d[n][2], e1, f0)), sum[n][3] = __fadd_rn(sum[n][3], few_scaled(d[n][3], e1, f1));
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        part[warp][n * 8 + 2 * q][g] = sum[n][0], part[warp][n * 8 + 2 * q + 1][g] = sum[n][1];
        part[warp][n * 8 + 2 * q][g + 8] = sum[n][2], part[warp][n * 8 + 2 * q + 1][g + 8] = sum[n][3];
    }
    __syncthreads();
    if (threadIdx.x < NT * 128) {
        const uint32_t token = threadIdx.x >> 4, r = threadIdx.x & 15, row = blockIdx.x * 16 + r;
        float s = part[0][token][r];
#pragma unroll
        for (int i = 1; i < kFewWarps; ++i)
            s = __fadd_rn(s, part[i][token][r]);
        if (token < P.tokens && row < P.rows)
            out[token * P.token_step + row * P.row_step] = from_f32<T>(s);
    }
}
template <class T>
static cudaError_t few(const FewArgs &P, T *out, cudaStream_t s)
{
    const dim3 grid((P.rows + 15) / 16);
    return P.tokens <= 8 ? launch(k_f8_few<T, 1>, grid, kFewWarps * 32, 0, s, P, out) : launch(k_f8_few<T, 2>, grid, kFewWarps * 32, 0, s, P, out);
}

}  // namespace conef

using namespace conef;

extern "C" {

int conef_f8_matmul(const void *a_codes, const void *a_scales, int a_kind, int64_t m, const void *b_codes, const void *b_scales, int b_kind, int64_t n, int64_t k, void *out,
                    int dtype, int64_t ld, conef_stream stream)
{
    int rc = check_matrix(out, dtype, m, n, ld);
    if (rc != CONEF_OK)
        return rc;
    if (k < 0 || (a_kind != CONEF_E4M3 && a_kind != CONEF_E5M2) || (b_kind != CONEF_E4M3 && b_kind != CONEF_E5M2))
        return CONEF_ERR_INVALID_ARG;
    if (k >= (1ll << 31))
        return CONEF_ERR_UNSUPPORTED;
    if (m == 0 || n == 0)
        return CONEF_OK;
    if (k && (!a_codes || !a_scales || !b_codes || !b_scales))
        return CONEF_ERR_INVALID_ARG;
    if ((((uintptr_t)a_codes | (uintptr_t)a_scales | (uintptr_t)b_codes | (uintptr_t)b_scales) & 15) != 0)
        return CONEF_ERR_INVALID_ARG;
    if (k == 0)
        return launched(cudaMemset2DAsync(out, (size_t)std::max(ld, n) * elem_bytes(dtype), 0, (size_t)n * elem_bytes(dtype), (size_t)m, (cudaStream_t)stream),
                        "conef_f8_matmul");
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        if (std::min(m, n) <= 16) {
            const bool turned = n < m;   // (the weight's rows are A's)
            FewArgs P = {(const uint8_t *)b_codes, (const uint8_t *)b_scales, (const uint8_t *)a_codes, (const uint8_t *)a_scales, (uint32_t)n, (uint32_t)m, (uint32_t)f8_blocks(k),
                         (uint32_t)f8_scale_tiles(k), (uint32_t)b_kind, (uint32_t)a_kind, 1, ld};
            if (turned)
                P = {(const uint8_t *)a_codes, (const uint8_t *)a_scales, (const uint8_t *)b_codes, (const uint8_t *)b_scales, (uint32_t)m, (uint32_t)n, P.blocks, P.tiles,
                     (uint32_t)a_kind, (uint32_t)b_kind, ld, 1};
            return launched(few(P, (T *)out, (cudaStream_t)stream), "conef_f8_matmul");
        }
        const MmChoice c = mm_choice<F8Format>(m, n, k);
        return (c.pair ? matmul<F8Format, T, true> : matmul<F8Format, T, false>)((const uint8_t *)a_codes, (const uint8_t *)a_scales, m, (const uint8_t *)b_codes,
                                                                                 (const uint8_t *)b_scales, n, k, (T *)out, ld, c.bn, a_kind, b_kind, "conef_f8_matmul",
                                                                                 (cudaStream_t)stream);
    });
}

int conef_f8_timeouts(int64_t *count, conef_stream stream)
{
    if (!count)
        return CONEF_ERR_INVALID_ARG;
    unsigned long long n = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&n, g_mm_ran_out, sizeof n, 0, cudaMemcpyDeviceToHost, (cudaStream_t)stream);
    if (e == cudaSuccess)
        e = cudaStreamSynchronize((cudaStream_t)stream);
    *count = (int64_t)n;
    return launched(e, "conef_f8_timeouts");
}

}  // extern "C"
