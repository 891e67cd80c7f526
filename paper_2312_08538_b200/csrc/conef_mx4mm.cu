// Product of two matrices held in microscaled 4-bit floats, out[i][j] = sum over k of A[i][k] B[j][k], in fp32 on the tensor
// cores' block-scaled path and rounded once to the output's type (the kernel: conef_mm.cuh).
//
// 8192 x 6400 x 1600 in bf16 takes 45.7 us on operands that the launch before left in L2, 50.3 on others (3.7 and 3.3 PFLOP/s).  The products alone would
// take 20 at full rate, the output's 105 MB 16 at the memory's.  Without the loads the kernel takes 33 us, without the stores 33, without either 30, of which
// only the products' 20 are accounted for; with half of the stores 40; with stores that hit the same lines of L2 over and over, by plain coalesced stores
// instead of tiled copies, or with a ring of four instead of five stages 46 to 48.  It is not L2's rate that bounds it: tiles of 256 x 192 move 577 MB in
// and out, 12.6 TB/s, L2's throughput counter reads 50 %, and at k = 4096 (83.5 us) it moves more per second.  A part is rows of codes that do not lie on lines
// of 128 bytes, as those of 800 bytes at k = 1600: 9.0 M requests to L2 where k = 1536 has 6.2 M; k = 1536, 1600, 1664 and 1792 take 42.9, 50.3, 48.6 and 46.2 us.
#include "conef_mx4.cuh"
#include "conef_mm.cuh"

namespace conef {

struct Mx4Format {
    static constexpr uint32_t kStageK = 256, kStepK = 64, kTiles = 2, kTileStages = 1, kScaleColumns = 24;
    static constexpr bool kSplits = false;   // (which would change the order of sums)
    static int64_t row_bytes(int64_t k) { return mx4_blocks(k) * 16; }
    static int64_t scale_tiles(int64_t k) { return mx4_scale_tiles(k); }
    // Nanoseconds per wave of tiles, from 8192 x 6400 by 1600 and by 4096: what a step of 64 along k takes (full rate
    // would be 17, 35, 52, 70), and what does not depend on k (the last where tensor memory has room for one set of sums only).
    // Microseconds, single CTAs and pairs of 64 to 256 columns, the choice marked (for two of them it misses the fastest by a tenth):
    //   8192 x 6400 x 1600   79.3  57.6  51.8  50.8   78.8  51.7  45.4* 51.8        1111 x 2601 x 651   8.7  8.2  7.1* 8.5   11.6  9.6  8.0  8.7
    //   8192 x 1600 x 1600   21.9  17.7  16.1* 18.0   22.9  16.7  14.8  18.7        4000 x 4000 x 300   15.0  12.1  11.9*  11.3   21.7  15.2  13.3  13.5
    //   2048 x 6400 x 1600   22.2  17.8  16.1* 15.4   23.0  16.5  14.8  16.1        300 x 300 x 1600    5.2*  5.9  6.7  8.0   6.0  6.6  7.1  8.2
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
    static __device__ __forceinline__ uint32_t instruction(const MmArgs &P) { return tc::mx4_instruction<PAIR>(P.bn); }
    // stage ks: its scales to tensor memory, then the products
    template <bool PAIR>
    static __device__ __forceinline__ void issue(const MmArgs &P, uint32_t d, uint32_t a, uint32_t b, uint32_t sc, uint32_t instruction, uint32_t sa, uint32_t sb, uint32_t shift,
                                                 uint32_t scale_rows, uint32_t ks, uint32_t ks0)
    {
        const uint32_t steps = P.k_steps - ks * 4u;
#pragma unroll
        for (uint32_t t = 0; t < 2; ++t)
            if (2 * t < steps) {
                tc::scales_copy<PAIR>(sa + 4 * t, sc + 32 * t);
                tc::scales_copy<PAIR>(sb + 8 * t, sc + 64 + 32 * t);
                if (scale_rows > 1)
                    tc::scales_copy<PAIR>(sb + 8 * t + 4, sc + 128 + 32 * t);
            }
#pragma unroll
        for (uint32_t t = 0; t < 2; ++t) {
            if (2 * t < steps)
                tc::mx4_product<PAIR, 0>(d, a + 4 * t, b + 4 * t, instruction, sa + 4 * t, sb + 8 * t + shift, ks - ks0 + t);
            if (2 * t + 1 < steps)
                tc::mx4_product<PAIR, 1>(d, a + 4 * t + 2, b + 4 * t + 2, instruction, sa + 4 * t, sb + 8 * t + shift, 1);
        }
    }
};

}  // namespace conef

using namespace conef;

extern "C" {

int conef_mx4_matmul(const void *a_codes, const void *a_scales, int64_t m, const void *b_codes, const void *b_scales, int64_t n, int64_t k,
                                void *out, int dtype, int64_t ld, conef_stream stream)
{
    int rc = check_matrix(out, dtype, m, n, ld);
    if (rc != CONEF_OK)
        return rc;
    if (k < 0)
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
                        "conef_mx4_matmul");
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        const MmChoice c = mm_choice<Mx4Format>(m, n, k);
        return (c.pair ? matmul<Mx4Format, T, true, false> : matmul<Mx4Format, T, false, false>)((const uint8_t *)a_codes, (const uint8_t *)a_scales, m, (const uint8_t *)b_codes,
                                                             (const uint8_t *)b_scales, n, k, (T *)out, ld, c, 0, 0, "conef_mx4_matmul", (cudaStream_t)stream);
    });
}

int conef_mx4_timeouts(int64_t *count, conef_stream stream)
{
    if (!count)
        return CONEF_ERR_INVALID_ARG;
    unsigned long long n = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&n, g_mm_ran_out, sizeof n, 0, cudaMemcpyDeviceToHost, (cudaStream_t)stream);
    if (e == cudaSuccess)
        e = cudaStreamSynchronize((cudaStream_t)stream);
    *count = (int64_t)n;
    return launched(e, "conef_mx4_timeouts");
}

int conef_mx4_set_waits(int64_t nanoseconds, int64_t loads, int64_t loads_second)
{
    if (nanoseconds < 0 || loads < -1 || loads_second < -1 || loads >= 0xFFFFFFFFll || loads_second >= 0xFFFFFFFFll)
        return CONEF_ERR_INVALID_ARG;
    mm_limit.nanoseconds = nanoseconds ? nanoseconds : 2000000000;
    mm_limit.loads[0] = (uint32_t)loads;           // (-1: 2^32 - 1, more than there are)
    mm_limit.loads[1] = (uint32_t)loads_second;
    return CONEF_OK;
}

}  // extern "C"
