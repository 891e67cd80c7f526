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
