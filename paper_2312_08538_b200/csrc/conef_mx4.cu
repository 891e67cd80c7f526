// Quantisation to microscaled 4-bit floats (conef_mx4.cuh), of a matrix and of its transpose, behind a dropout where one is
// asked for, and the way back.
#include <algorithm>

#include "conef_mx4.cuh"
#include "conef_common.cuh"
#include "conef_elem.cuh"

namespace conef {

constexpr int kQThreads = 256;

// eight elements from p on, of which `have` exist (the rest zero); VEC: p is aligned to their size
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T *p, int have, float (&v)[8])
{
    if (VEC && have >= 8) {
        if constexpr (sizeof(T) == 4) {
            uint32_t w[8];
            load32(p, w);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                v[q] = __uint_as_float(w[q]);
        } else {
            Vec16<T>::unpack(__ldcs((const uint4 *)p), v);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            v[q] = q < have ? to_f32(p[q]) : 0.f;
    }
}
// x behind the dropout, rounded to fp32, of four columns
__device__ __forceinline__ void drop4(float *v, uint64_t word, const Dropout &d)
{
    const uint32_t kept = dropout_kept(word, d);
#pragma unroll
    for (int q = 0; q < 4; ++q)
        v[q] = (kept >> q) & 1u ? __fmul_rn(v[q], d.scale) : 0.f;
}
// max(a, |x|), or NaN where either is one
__device__ __forceinline__ float mx4_absmax(float a, float x)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(x)));
    return r;
}

struct QArgs {
    int64_t rows, cols, ld;
    uint64_t dropout, rounding;   // draw_base() of the two
    Dropout drop;
    uint8_t *codes, *scales, *codes_t, *scales_t;
};

// ------------------------------------------------------------------ rows
// Four lanes per block, eight elements each, U blocks one after the other.  Blocks are counted over the padded tiles of scales, so that the bytes
// of those that do not exist get their zero.
template <class T, bool VEC, bool STOCH, bool DROP, int U>
__global__ void __launch_bounds__(kQThreads) k_mx4_rows(const T *x, const __grid_constant__ QArgs A, const Divider padded, uint32_t units)
{
    grid_release();
    const uint32_t blocks = (uint32_t)mx4_blocks(A.cols), tiles = padded.by / 4, part = threadIdx.x & 3;
    const uint32_t u0 = blockIdx.x * (uint32_t)(kQThreads / 4 * U) + threadIdx.x / 4;
    const uint64_t groups = (uint64_t)(A.cols + 3) / 4;
    grid_wait();
    float v[U][8];
    uint32_t row[U], block[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t u = u0 + i * (kQThreads / 4);
        row[i] = divide(u, padded);
        block[i] = u - row[i] * padded.by;
        const int64_t c = (int64_t)block[i] * 32 + part * 8;
        const int64_t have = u < units && row[i] < A.rows && c < A.cols ? A.cols - c : 0;
        load8<T, VEC>(x + (int64_t)row[i] * A.ld + c, (int)min(have, (int64_t)8), v[i]);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint64_t group = (uint64_t)row[i] * groups + block[i] * 8u + part * 2u;
        if (DROP) {
            drop4(v[i], mix64(A.dropout + kDrawStep * group), A.drop);
            drop4(v[i] + 4, mix64(A.dropout + kDrawStep * (group + 1)), A.drop);
        }
        float most = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q)
            most = mx4_absmax(most, v[i][q]);
        most = mx4_absmax(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = mx4_absmax(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const uint32_t byte = mx4_scale(__float_as_uint(most));
        const float inv = mx4_inv(byte);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            v[i][q] = __fmul_rn(v[i][q], inv);
        uint32_t code = STOCH ? mx4_stochastic8(v[i], mix64(A.rounding + kDrawStep * group), mix64(A.rounding + kDrawStep * (group + 1))) : mx4_nearest8(v[i]);
        code = byte == kMx4Nan ? 0u : code;   // (elements that do not exist are zero, which no number rounds up)
        if (u0 + i * (kQThreads / 4) < units) {
            const bool there = row[i] < A.rows && block[i] < blocks;
            if (part == 0)
                A.scales[mx4_scale_at(row[i], block[i], tiles)] = (uint8_t)(there ? byte : 0u);
            if (there)
                *(uint32_t *)(A.codes + ((uint64_t)row[i] * blocks + block[i]) * 16 + part * 4) = code;
        }
    }
}

// ------------------------------------------------------------------ the transpose, and rows with it
// A warp takes 64 x 64 elements, 32 x 32 at a time: a lane has 32 elements of a row, which is a block of the rows' form, and hands them and
// their numbers through shared memory to the lanes of the columns, of which each has a block of the transpose.  One reading
// of x and one hash per four elements serve both.  Elements of 16 bits lie beside their number in a word.
constexpr int kBothWarps = 4;
template <class T, bool STOCH>
struct alignas(16) BothTile {
    uint32_t v[32][33];
    uint16_t u[sizeof(T) == 4 && STOCH ? 32 : 1][34];
};
template <class T, bool VEC, bool ROWS, bool STOCH, bool DROP>
__global__ void __launch_bounds__(kBothWarps * 32) k_mx4_both(const T *x, const __grid_constant__ QArgs A, uint32_t tiles_c, int64_t n_tiles)
{
    constexpr bool SHORT = sizeof(T) == 2;
    __shared__ BothTile<T, STOCH> S[kBothWarps];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t tile = (int64_t)blockIdx.x * kBothWarps + warp;
    BothTile<T, STOCH> &M = S[warp];
    const int64_t tr = tile / tiles_c, rbase = tr * 64, cbase = (tile - tr * tiles_c) * 64;
    const int64_t blocks = mx4_blocks(A.cols), blocks_t = mx4_blocks(A.rows), scale_tiles = mx4_scale_tiles(A.cols), scale_tiles_t = mx4_scale_tiles(A.rows);
    const uint64_t groups = (uint64_t)(A.cols + 3) / 4;
    grid_wait();
    if (tile >= n_tiles)
        return;
    for (int sc = 0; sc < 2; ++sc)
        for (int sr = 0; sr < 2; ++sr) {
            const int64_t r0 = rbase + sr * 32, c0 = cbase + sc * 32, r = r0 + lane, ct = c0 + lane;
            if (r0 >= A.rows || c0 >= A.cols) {   // scales of blocks that do not exist
                if (ROWS)
                    A.scales[mx4_scale_at(r, c0 >> 5, scale_tiles)] = 0;
                A.scales_t[mx4_scale_at(ct, r0 >> 5, scale_tiles_t)] = 0;
                continue;
            }
            // elements, in fp32 (16 bits: as they are, in M)
            const bool whole = VEC && c0 + 32 <= A.cols;
            float v[32];
            if (whole) {
                const T *p = x + r * A.ld + c0;
                if (r < A.rows) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        load8<T, true>(p + 8 * i, 8, *(float(*)[8])(v + 8 * i));
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        v[i] = 0.f;
                }
            } else {   // a row at a time, and turned
                const T *p = x + r0 * A.ld + ct;
                const int rows = (int)min((int64_t)32, A.rows - r0);
                float t[32];
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    t[i] = i < rows && ct < A.cols ? to_f32(p[i * A.ld]) : 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    M.v[i][lane] = __float_as_uint(t[i]);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    v[i] = __uint_as_float(M.v[lane][i]);
                __syncwarp();
            }
            const uint64_t group = (uint64_t)r * groups + (uint64_t)(c0 >> 2);
            uint64_t word[STOCH ? 8 : 1];
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                if (STOCH)
                    word[g] = mix64(A.rounding + kDrawStep * (group + g));
                uint32_t kept = 0xFu;
                if (DROP)
                    kept = dropout_kept(mix64(A.dropout + kDrawStep * (group + g)), A.drop);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = 4 * g + q;
                    if (DROP)
                        v[i] = (kept >> q) & 1u ? v[i] : 0.f;
                    if (SHORT) {   // (fp32 from 16 bits and back is exact, a NaN stays one)
                        const T s = from_f32<T>(v[i]);
                        M.v[lane][i] = (uint32_t) * (const uint16_t *)&s | (STOCH ? draw_of(word[g], q) << 16 : 0u);
                    }
                    if (DROP)
                        v[i] = __fmul_rn(v[i], A.drop.scale);
                    if (!SHORT) {
                        M.v[lane][i] = __float_as_uint(v[i]);
                        if (STOCH)
                            M.u[lane][i] = (uint16_t)draw_of(word[g], q);
                    }
                }
            }
            if (ROWS) {
                float most = 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    most = mx4_absmax(most, v[i]);
                const uint32_t byte = mx4_scale(__float_as_uint(most));
                const float inv = mx4_inv(byte);
                uint32_t code[4];
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    v[i] = __fmul_rn(v[i], inv);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    code[i] = STOCH ? mx4_stochastic8(v + 8 * i, word[STOCH ? 2 * i : 0], word[STOCH ? 2 * i + 1 : 0]) : mx4_nearest8(v + 8 * i);
                    code[i] = byte == kMx4Nan ? 0u : code[i];
                }
                A.scales[mx4_scale_at(r, c0 >> 5, scale_tiles)] = (uint8_t)(r < A.rows ? byte : 0u);
                if (r < A.rows)
                    *(uint4 *)(A.codes + (r * blocks + (c0 >> 5)) * 16) = make_uint4(code[0], code[1], code[2], code[3]);
            }
            __syncwarp();
            // the columns
            uint32_t n[STOCH ? 32 : 1];
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t w = M.v[i][lane];
                if (SHORT) {
                    const uint16_t h = (uint16_t)w;
                    v[i] = to_f32(*(const T *)&h);
                    if (DROP)
                        v[i] = __fmul_rn(v[i], A.drop.scale);
                    if (STOCH)
                        n[i] = (w >> 10 & 0x3FFFC0u) | 32u;
                } else {
                    v[i] = __uint_as_float(w);
                    if (STOCH)
                        n[i] = M.u[i][lane] * 64u + 32u;
                }
                most = mx4_absmax(most, v[i]);
            }
            const uint32_t byte = mx4_scale(__float_as_uint(most));
            const float inv = mx4_inv(byte);
            uint32_t code[4];
#pragma unroll
            for (int i = 0; i < 32; ++i)
                v[i] = __fmul_rn(v[i], inv);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (STOCH) {
                    code[i] = 0;
#pragma unroll
                    for (int q = 7; q >= 0; --q)
                        code[i] = code[i] * 16u + mx4_stochastic(v[8 * i + q], n[STOCH ? 8 * i + q : 0]);
                } else {
                    code[i] = mx4_nearest8(v + 8 * i);
                }
                code[i] = byte == kMx4Nan ? 0u : code[i];
            }
            A.scales_t[mx4_scale_at(ct, r0 >> 5, scale_tiles_t)] = (uint8_t)(ct < A.cols ? byte : 0u);
            if (ct < A.cols)
                *(uint4 *)(A.codes_t + (ct * blocks_t + (r0 >> 5)) * 16) = make_uint4(code[0], code[1], code[2], code[3]);
            __syncwarp();
        }
}

// ------------------------------------------------------------------ the way back
// Eight elements per thread, U times; rows of the result begin on a boundary of eight elements' size.
template <class T, int U>
__global__ void __launch_bounds__(kQThreads) k_mx4_dequantise(const uint8_t *codes, const uint8_t *scales, const Divider pieces, int64_t rows, int64_t cols,
                                                              T *out, int64_t ld)
{
    grid_release();
    const uint32_t p0 = blockIdx.x * (uint32_t)(kQThreads * U) + threadIdx.x, tiles = (uint32_t)mx4_scale_tiles(cols);
    grid_wait();
    uint32_t w[U], row[U], at[U];
    uint8_t s[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t p = p0 + i * kQThreads;
        row[i] = divide(p, pieces);
        at[i] = p - row[i] * pieces.by;
        if (row[i] < rows) {
            w[i] = __ldcs((const uint32_t *)codes + p);
            s[i] = scales[mx4_scale_at(row[i], at[i] >> 2, tiles)];
        }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int64_t c = (int64_t)at[i] * 8;
        if (row[i] >= rows || c >= cols)
            continue;
        float v[8];
        mx4_values8(w[i], v);
        const float f = mx4_pow(s[i]);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            v[q] = __fmul_rn(v[q], f);
        T *o = out + (int64_t)row[i] * ld + c;
        if (c + 8 <= cols) {
            if constexpr (sizeof(T) == 4) {
                uint32_t b[8];
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    b[q] = __float_as_uint(v[q]);
                store32(o, b);
            } else {
                __stcs((uint4 *)o, Vec16<T>::pack(v));
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (c + q < cols)
                    o[q] = from_f32<T>(v[q]);
        }
    }
}
// ... begin anywhere: a block per warp, an element per lane, U times
template <class T, int U>
__global__ void __launch_bounds__(kQThreads) k_mx4_dequantise_any(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, T *out, int64_t ld)
{
    grid_release();
    const int lane = threadIdx.x & 31;
    const int64_t blocks = mx4_blocks(cols), tiles = mx4_scale_tiles(cols), b0 = ((int64_t)blockIdx.x * (kQThreads / 32) + (threadIdx.x >> 5)) * U;
    grid_wait();
    int64_t row = b0 / blocks, block = b0 - row * blocks;
    uint8_t w[U], s[U];
    T *o[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        o[i] = row < rows && block * 32 + lane < cols ? out + row * ld + block * 32 + lane : nullptr;
        if (row < rows) {
            w[i] = codes[(b0 + i) * 16 + (lane >> 1)];
            s[i] = scales[mx4_scale_at(row, block, tiles)];
        }
        if (++block == blocks)
            block = 0, ++row;
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
        if (o[i])
            *o[i] = from_f32<T>(__fmul_rn(mx4_value(w[i] >> (4 * (lane & 1)) & 0xFu), mx4_pow(s[i])));
}

template <class T>
static cudaError_t quantise(const T *x, QArgs A, bool stochastic, cudaStream_t s)
{
    // eight elements of a row in one or (fp32) one wide load
    const bool vec = (((uintptr_t)x | (A.rows > 1 ? (uint64_t)A.ld * sizeof(T) : 0u)) & (8 * sizeof(T) - 1)) == 0;
    auto by_draws = [&](auto f) {
        using Y = std::true_type;
        using N = std::false_type;
        return stochastic ? (A.drop.off ? f(Y(), Y()) : f(Y(), N())) : (A.drop.off ? f(N(), Y()) : f(N(), N()));
    };
    if (!A.codes_t) {
        // (blocks are counted in 32 bits: as many tiles of 128 rows per launch as that takes)
        const int64_t padded = mx4_scale_tiles(A.cols) * 4, rows = A.rows, most = (1ll << 32) / (padded * 128) * 128 - 128;
        cudaError_t e = cudaSuccess;
        for (int64_t r0 = 0; r0 < rows && e == cudaSuccess; r0 += most) {
            A.rows = std::min(most, rows - r0);
            const int64_t units = (A.rows + 127) / 128 * 128 * padded;
            e = by_draws([&](auto st, auto dr) {
                constexpr bool ST = decltype(st)::value, DR = decltype(dr)::value;
                auto go = [&](auto vc, auto un) {
                    constexpr int U = decltype(un)::value, PER = kQThreads / 4 * U;
                    return launch(k_mx4_rows<T, decltype(vc)::value, ST, DR, U>, dim3((unsigned)((units + PER - 1) / PER)), kQThreads, 0, s, x + r0 * A.ld, A,
                                  divider((uint32_t)padded), (uint32_t)units);
                };
                using One = std::integral_constant<int, 1>;
                using Many = std::integral_constant<int, sizeof(T) == 4 ? 2 : 4>;
                const bool many = units >= (int64_t)kQThreads / 4 * Many::value * kPlanSMs * 8;
                return many ? (vec ? go(std::true_type(), Many()) : go(std::false_type(), Many())) : (vec ? go(std::true_type(), One()) : go(std::false_type(), One()));
            });
            A.codes += most * mx4_blocks(A.cols) * 16;
            A.scales += most / 128 * (padded / 4) * 512;
            A.dropout += kDrawStep * (uint64_t)(most * ((A.cols + 3) / 4));
            A.rounding += kDrawStep * (uint64_t)(most * ((A.cols + 3) / 4));
        }
        return e;
    }
    const int64_t tiles_c = (A.cols + 127) / 128 * 2, n_tiles = (A.rows + 127) / 128 * 2 * tiles_c;
    const dim3 grid((unsigned)((n_tiles + kBothWarps - 1) / kBothWarps));
    return by_draws([&](auto st, auto dr) {
        constexpr bool ST = decltype(st)::value, DR = decltype(dr)::value;
        auto go = [&](auto vc, auto ro) {
            return launch(k_mx4_both<T, decltype(vc)::value, decltype(ro)::value, ST, DR>, grid, kBothWarps * 32, 0, s, x, A, (uint32_t)tiles_c, n_tiles);
        };
        return A.codes ? (vec ? go(std::true_type(), std::true_type()) : go(std::false_type(), std::true_type()))
                       : (vec ? go(std::true_type(), std::false_type()) : go(std::false_type(), std::false_type()));
    });
}

template <class T>
static cudaError_t dequantise(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, T *out, int64_t ld, cudaStream_t s)
{
    const int64_t per_row = mx4_blocks(cols) * 4, pieces = rows * per_row;
    if ((((uintptr_t)out | (rows > 1 ? (uint64_t)ld * sizeof(T) : 0u)) & (8 * sizeof(T) - 1)) == 0 && pieces < (1ll << 32) - 4096) {
        auto go = [&](auto un) {
            constexpr int U = decltype(un)::value, PER = kQThreads * U;
            return launch(k_mx4_dequantise<T, U>, dim3((unsigned)((pieces + PER - 1) / PER)), kQThreads, 0, s, codes, scales, divider((uint32_t)per_row), rows, cols, out, ld);
        };
        return pieces >= (int64_t)kQThreads * 4 * kPlanSMs * 8 ? go(std::integral_constant<int, 4>()) : go(std::integral_constant<int, 1>());
    }
    auto go = [&](auto un) {
        constexpr int U = decltype(un)::value, PER = kQThreads / 32 * U;
        return launch(k_mx4_dequantise_any<T, U>, dim3((unsigned)((rows * mx4_blocks(cols) + PER - 1) / PER)), kQThreads, 0, s, codes, scales, rows, cols, out, ld);
    };
    return rows * mx4_blocks(cols) >= (int64_t)kQThreads / 32 * 8 * kPlanSMs * 8 ? go(std::integral_constant<int, 8>()) : go(std::integral_constant<int, 1>());
}

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
    const QArgs A = {rows, cols, ld, draw_base(st, kDrawDropout), draw_base(st, kDrawRounding), drop, (uint8_t *)codes, (uint8_t *)scales, (uint8_t *)codes_t,
                     (uint8_t *)scales_t};
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        return launched(quantise<T>((const T *)x, A, stochastic != 0, (cudaStream_t)stream), "conef_mx4_quantise");
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
        return launched(dequantise<T>((const uint8_t *)codes, (const uint8_t *)scales, rows, cols, (T *)out, ld, (cudaStream_t)stream), "conef_mx4_dequantise");
    });
}

}  // extern "C"
