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
    static constexpr bool kSplits = true;
    static int64_t row_bytes(int64_t k) { return f8_blocks(k) * 128; }
    static int64_t scale_tiles(int64_t k) { return f8_scale_tiles(k); }
    // Nanoseconds per wave of tiles, as the 4-bit format has them (conef_mx4mm.cu): a step brings and multiplies the same 32 bytes of a row, and copies, not products, are
    // what a wave waits for.  Microseconds into bf16, single CTAs of 64 to 256 columns and pairs of 128 to 256, the choice marked:
    //   8192 x 6400 x 1600  126.8  84.6  77.1  76.8   79.9  69.8* 75.4        1111 x 2601 x 651   9.7  9.2  7.6*  8.9   11.0   9.3  10.1
    //   8192 x 1600 x 6400  116.9  79.1  71.1  82.5   77.2  63.6* 76.3        4000 x 4000 x 300  19.2 14.9 14.3* 13.3   18.0  15.8  15.9
    //   6400 x 1600 x 8192  121.2  82.3  80.5  85.1   80.6  72.4  75.4*       300 x 300 x 1600    7.1* 7.7  8.6  10.0    8.8   9.3  10.8
    //   8192 x 1600 x 1600   37.0  27.2  24.2  29.0   26.6  23.4* 29.2        1000 x 1600 x 1600  9.8  7.7* 8.2   9.4    8.8   9.0  10.3
    //   2048 x 6400 x 1600   37.4  27.8  25.4  27.1   26.7  23.3* 26.3        128 x 1600 x 6400  13.6 14.5 16.0  19.6   15.9  16.5  20.2 (10.7 by clusters of eight)
    // Where it misses the fastest that costs 4 % (6400 x 1600 x 8192) and 7 % (4000 x 4000 x 300).
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
                                                 uint32_t scale_rows, uint32_t ks, uint32_t ks0)
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
                tc::f8_product<PAIR>(d, a + 2 * t, b + 2 * t, instruction, sa, sb + shift, ks - ks0 + t);
    }
};

// ------------------------------------------------------------------ few rows against many
// Few rows of one side (tokens) against all of the other's (a weight's), which are read once for eight: 1 x 6400 x 1600 are 10 MB, 1.6 us.  A tile of tcgen05.mma would have
// 128 rows with one used, and a chain of copies and barriers for each (16 rows 6.5 us; here one 4.8); here a warp takes eight tokens, 16 rows of the weight and a share
// of the blocks along k, straight from memory to the registers of mma.m16n8k32.  A lane has 16 bytes of two rows and of a
// token at a time: the instruction's order of k is any that both sides share.  Sums of a block are fp32, times its two scales' power of two, and added in fp32.
constexpr int kFewWarps = 8;
constexpr uint32_t kFewAhead = 4, kFewStage = 2048 + 128;
// 16 rows of the weight by eight tokens and 32 of k; KINDS: 0 to 3, the weight's kind and twice the tokens'
template <int KINDS>
__device__ __forceinline__ void few_product(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
#define FEW_PRODUCT(KW, KT)                                                                                                                                              \
    asm("mma.sync.aligned.m16n8k32.row.col.f32." KW "." KT ".f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"                                        \
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])                                                                                                                 \
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1))
    if constexpr (KINDS == 0)
        FEW_PRODUCT("e4m3", "e4m3");
    else if constexpr (KINDS == 1)
        FEW_PRODUCT("e5m2", "e4m3");
    else if constexpr (KINDS == 2)
        FEW_PRODUCT("e4m3", "e5m2");
    else
        FEW_PRODUCT("e5m2", "e5m2");
#undef FEW_PRODUCT
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
    uint32_t groups;                  // of eight tokens: neighbouring CTAs, which find the weight in L2
    uint32_t share;                   // warps that share a row group's blocks: 1, 2, 4 or 8
    int64_t row_step, token_step;     // of the output, in elements
};
template <class T, int KINDS>
__global__ void __launch_bounds__(kFewWarps * 32, 3) k_f8_few(const FewArgs P, T *out)
{
    extern __shared__ __align__(16) uint8_t few_smem[];
    __shared__ float part[kFewWarps][8][17];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q = lane & 3, g = lane >> 2;
    const uint64_t pitch = (uint64_t)P.blocks * 128u;
    const uint32_t at = blockIdx.x / P.groups, token0 = (blockIdx.x - at * P.groups) * 8, tokens = min(8u, P.tokens - token0);
    const uint32_t first = at * (kFewWarps / P.share) * 16, row0 = first + warp / P.share * 16 + g, row1 = row0 + 8;
    const uint32_t have0 = min(row0, P.rows - 1), have1 = min(row1, P.rows - 1);   // (what does not exist is not stored)
    const uint8_t *const w0 = P.w + have0 * pitch + q * 16, *const w1 = P.w + have1 * pitch + q * 16, *const t = P.t + (token0 + min((uint32_t)g, tokens - 1)) * pitch + q * 16;
    // Scales come as words, four blocks of a row: of four lanes one has the weight's row, the next the row eight on, the third a token (one that does not exist is
    // another again: its products with the weight stay normal numbers).
    const uint8_t *const scales = q == 0 ? P.ws + f8_scale_at32(have0, 0, P.tiles) : q == 1 ? P.ws + f8_scale_at32(have1, 0, P.tiles)
                                                                                      : P.ts + f8_scale_at32(token0 + min((uint32_t)g, tokens - 1), 0, P.tiles);
    float sum[4] = {};
    grid_wait();
    // The weight's blocks ahead and scales are copied into shared memory, kFewAhead of 2 KB to a warp, of which a lane reads what it has copied; tokens, which L1 has after a while, come one
    // block ahead in registers (two and three ahead: nothing).  (Tokens by copies that pass L1 by are the same lines of L2 for all SMs: 1 x 50257 x 1600 23 -> 74 us.)
    uint8_t *const ring = few_smem + warp * kFewAhead * kFewStage, *const mine = ring + lane * 16;
    auto copy16 = [](uint8_t *to, const uint8_t *from) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
    };
    auto ask = [&](uint32_t b, uint32_t stage) {
        if (b < P.blocks) {
            uint8_t *const to = mine + stage * kFewStage;
            const uint64_t at = b * 128ull;
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(ring + stage * kFewStage + 2048 + lane * 4)), "l"(scales + (uint64_t)(b >> 2) * 512u)
                         : "memory");
            copy16(to, w0 + at), copy16(to + 512, w0 + at + 64), copy16(to + 1024, w1 + at), copy16(to + 1536, w1 + at + 64);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    uint4 z[2], next[2];
    auto ask_tokens = [&](uint32_t b) {
        if (b < P.blocks)
            next[0] = *(const uint4 *)(t + b * 128ull), next[1] = *(const uint4 *)(t + b * 128ull + 64);
    };
    uint32_t b = warp % P.share, stage = 0;
#pragma unroll
    for (uint32_t i = 0; i < kFewAhead - 1; ++i)
        ask(b + i * P.share, i);
    ask_tokens(b);
    for (; b < P.blocks; b += P.share) {
        ask(b + (kFewAhead - 1) * P.share, (stage + kFewAhead - 1) % kFewAhead);
        z[0] = next[0], z[1] = next[1];
        ask_tokens(b + P.share);
        asm volatile("cp.async.wait_group %0;" ::"n"(kFewAhead - 1) : "memory");
        __syncwarp();
        const uint8_t *const from = mine + stage * kFewStage, *const bytes = ring + stage * kFewStage + 2048 + (b & 3u);
        stage = (stage + 1) % kFewAhead;
        uint4 x[2], y[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            x[h] = *(const uint4 *)(from + h * 512), y[h] = *(const uint4 *)(from + 1024 + h * 512);
        const uint32_t e0 = bytes[g * 16], e1 = bytes[g * 16 + 4], f0 = bytes[q * 32 + 8], f1 = bytes[q * 32 + 24];
        float d[4] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            few_product<KINDS>(d, x[h].x, y[h].x, x[h].y, y[h].y, z[h].x, z[h].y);
            few_product<KINDS>(d, x[h].z, y[h].z, x[h].w, y[h].w, z[h].z, z[h].w);
        }
        // the two scales' product, where it is a normal number (and neither of them NaN: 255 and 127 or more are not)
        const uint32_t least = min(e0, e1) + min(f0, f1), most = max(e0, e1) + max(f0, f1);
        // (... and all lanes have the scales by now, into whose place the next ones go)
        if (__all_sync(0xffffffffu, least > 127u && most < 382u && max(max(e0, e1), max(f0, f1)) < kF8Nan)) {
            sum[0] = __fmaf_rn(d[0], __uint_as_float((e0 + f0 - 127u) << 23), sum[0]), sum[1] = __fmaf_rn(d[1], __uint_as_float((e0 + f1 - 127u) << 23), sum[1]);
            sum[2] = __fmaf_rn(d[2], __uint_as_float((e1 + f0 - 127u) << 23), sum[2]), sum[3] = __fmaf_rn(d[3], __uint_as_float((e1 + f1 - 127u) << 23), sum[3]);
        } else {
            sum[0] = __fadd_rn(sum[0], few_scaled(d[0], e0, f0)), sum[1] = __fadd_rn(sum[1], few_scaled(d[1], e0, f1));
            sum[2] = __fadd_rn(sum[2], few_scaled(d[2], e1, f0)), sum[3] = __fadd_rn(sum[3], few_scaled(d[3], e1, f1));
        }
    }
    part[warp][2 * q][g] = sum[0], part[warp][2 * q + 1][g] = sum[1];
    part[warp][2 * q][g + 8] = sum[2], part[warp][2 * q + 1][g + 8] = sum[3];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < (kFewWarps / P.share) * 128u; i += kFewWarps * 32) {
        const uint32_t group = i >> 7, token = i >> 4 & 7u, r = i & 15u, row = first + group * 16 + r;
        float s = part[group * P.share][token][r];
        for (uint32_t k = 1; k < P.share; ++k)
            s = __fadd_rn(s, part[group * P.share + k][token][r]);
        if (token < tokens && row < P.rows)
            out[(token0 + token) * P.token_step + row * P.row_step] = from_f32<T>(s);
    }
}
// warps that share a row group's blocks: as many as the SMs hold, 24 each, with as many blocks as that leaves (1 x 6400 x 1600 with 12 to an SM 6.4, with 24 5.3 us then)
static uint32_t few_share(int64_t rows, int64_t tokens)
{
    uint32_t share = kFewWarps;
    while (share > 1 && (rows + 15) / 16 * ((tokens + 7) / 8) * share > kPlanSMs * 24)
        share /= 2;
    return share;
}
template <class T>
static cudaError_t few(FewArgs P, int kind_w, int kind_t, T *out, cudaStream_t s)
{
    const int64_t groups = ((int64_t)P.rows + 15) / 16;
    P.groups = (P.tokens + 7) / 8;
    P.share = few_share(P.rows, P.tokens);
    const int64_t per_cta = kFewWarps / P.share;
    static void (*const kernels[4])(FewArgs, T *) = {k_f8_few<T, 0>, k_f8_few<T, 1>, k_f8_few<T, 2>, k_f8_few<T, 3>};
    constexpr size_t smem = kFewWarps * kFewAhead * kFewStage;
    static int done[4][64];
    const int kinds = kind_w + 2 * kind_t;
    const cudaError_t e = opt_in_smem(kernels[kinds], smem, done[kinds]);
    return e != cudaSuccess ? e : launch(kernels[kinds], dim3((unsigned)((groups + per_cta - 1) / per_cta * P.groups)), kFewWarps * 32, smem, s, P, out);
}
// Whether that takes less: up to eight tokens always; then the weight once per eight tokens at 5 TB/s, or 0.4 us for each of a warp's blocks, and 0.7 us less than
// tiles of tcgen05.mma to begin and end with (mm_cost: theirs beside that).  Tiles and this, us: 16 x 6400 x 1600 6.5 and 6.8; 16 x 1600 x 1600 6.1 and 4.1;
// 16 x 4096 x 4096 9 and 8.8, 32 rows 9 and 13.8; 16 x 8192 x 8192 19 and 27; 64 x 64 x 65536 16 and 26.
static bool few_rows(int64_t tokens, int64_t rows, int64_t k, int64_t mm_cost)
{
    if (tokens <= 8 || tokens > 64)
        return tokens <= 8;
    const int64_t share = few_share(rows, tokens), bytes = (tokens + 7) / 8 * rows * f8_blocks(k) * 128, alone = (f8_blocks(k) + share - 1) / share * 400;
    return std::max(bytes / 5000, alone) < mm_cost + 700;
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
        const MmChoice c = mm_choice<F8Format>(m, n, k);
        if (few_rows(std::min(m, n), std::max(m, n), k, c.cost)) {
            const bool turned = n < m;   // (the weight's rows are A's)
            FewArgs P = {(const uint8_t *)b_codes, (const uint8_t *)b_scales, (const uint8_t *)a_codes, (const uint8_t *)a_scales, (uint32_t)n, (uint32_t)m, (uint32_t)f8_blocks(k),
                         (uint32_t)f8_scale_tiles(k), 0, 0, 1, ld};
            if (turned)
                P = {(const uint8_t *)a_codes, (const uint8_t *)a_scales, (const uint8_t *)b_codes, (const uint8_t *)b_scales, (uint32_t)m, (uint32_t)n, P.blocks, P.tiles,
                     0, 0, ld, 1};
            return launched(few(P, turned ? a_kind : b_kind, turned ? b_kind : a_kind, (T *)out, (cudaStream_t)stream), "conef_f8_matmul");
        }
        const auto product = c.pair ? matmul<F8Format, T, true, false> : c.split > 1 ? matmul<F8Format, T, false, true> : matmul<F8Format, T, false, false>;
        return product((const uint8_t *)a_codes, (const uint8_t *)a_scales, m, (const uint8_t *)b_codes, (const uint8_t *)b_scales, n, k, (T *)out, ld, c, a_kind, b_kind,
                       "conef_f8_matmul", (cudaStream_t)stream);
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
