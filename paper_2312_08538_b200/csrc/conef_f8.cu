// Quantisation to 8-bit floats with block scales (conef_f8.cuh), of a matrix, of its transpose or of both, and the way back.
#include <algorithm>
#include <type_traits>

#include "conef_f8.cuh"

namespace conef {

constexpr int kF8Threads = 256;

// Warps' pieces of 512 elements are counted in 32 bits: as many rows per launch as that takes
static int64_t rows_per_launch(int64_t tiles) { return std::max<int64_t>(128, ((1ll << 32) - 4096) / tiles / 128 * 128); }
// (a Divider divides by 2 at least)
struct Pieces {
    Divider tiles;
    uint32_t one;
    __device__ __forceinline__ void place(uint32_t u, uint32_t &row, uint32_t &tile) const
    {
        row = one ? u : divide(u, tiles);
        tile = one ? 0u : u - row * tiles.by;
    }
};
static Pieces pieces_of(int64_t tiles) { return {divider((uint32_t)std::max<int64_t>(2, tiles)), tiles == 1 ? 1u : 0u}; }

// ------------------------------------------------------------------ rows
template <class T, bool VEC>
__global__ void __launch_bounds__(kF8Threads) k_f8_rows(const T *x, const Pieces pieces, uint32_t row0, uint32_t units, int64_t rows, int64_t cols, int64_t ld,
                                                        const F8Out out, bool aligned32)
{
    grid_release();
    const int lane = threadIdx.x & 31;
    const uint32_t u = blockIdx.x * (kF8Threads / 32) + (threadIdx.x >> 5);
    if (u >= units)
        return;
    uint32_t at, tile;
    pieces.place(u, at, tile);
    const int64_t row = (int64_t)row0 + at;
    const bool there = row < rows;
    grid_wait();
    Piece<T, VEC> p;
    p.load(x + row * ld, tile * 512u, there ? (uint32_t)cols : 0u, lane, aligned32);
    float v[16];
    p.unpack(v);
    const int64_t blocks = f8_blocks(cols);
    f8_store_row<T, VEC>(v, tile * 512u, (uint32_t)blocks, lane, out.kind, there, out.codes + row * blocks * 128, out.scales + f8_scale_at(row, tile * 4, f8_scale_tiles(cols)));
}

// ------------------------------------------------------------------ the transpose, and rows with it; square blocks
// A CTA takes 128 x 128 elements, which are a block of each of 128 rows and of 128 columns (or one square block): the rows' form from registers, eight lanes to a
// row's block; the columns' from shared memory, where a thread reads 32 rows of two columns.  Elements
// of 16 bits lie there as they came, two to a word; a norm's values, and elements of 32 bits, in a word each, a lane's four pieces of 16 bytes exchanged so that
// its neighbours' go to other banks.  Those take half as many of a thread, 16 rows, whose codes it exchanges with another until each has 32 of one column: 512 threads
// then have the registers of 256, and an SM twice the warps (both forms of 30011 x 1301 in fp32 87 -> 79 us, of 8192 x 6400 in bf16 51 -> 62).
struct TileArgs {
    int64_t rows, cols, ld;
    const float *rstd;
    const void *w;
    F8Out out;
    uint32_t tiles_c;
    bool w32, square, aligned32, whole;   // whole: the transpose's codes begin on 32 bytes
};
template <class T, bool NORM>
__host__ __device__ constexpr int tile_threads() { return NORM || sizeof(T) == 4 ? 512 : 256; }
template <class T, bool VEC, bool NORM>
__global__ void __launch_bounds__((tile_threads<T, NORM>()), NORM || sizeof(T) == 4 ? 2 : 3) k_f8_tiles(const T *x, const __grid_constant__ TileArgs A)
{
    constexpr bool WIDE = NORM || sizeof(T) == 4;
    constexpr int kTileThreads = tile_threads<T, NORM>(), kTileWarps = kTileThreads / 32;
    extern __shared__ __align__(16) uint32_t tile[];   // 128 rows of 128 words (WIDE) or 64
    __shared__ uint32_t col_most[4][128], square_most;
    using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t tr = blockIdx.x / A.tiles_c, r0 = tr * 128, c0 = (int64_t)(blockIdx.x - tr * A.tiles_c) * 128;
    const int64_t blocks = f8_blocks(A.cols), blocks_t = f8_blocks(A.rows), scale_tiles = f8_scale_tiles(A.cols), scale_tiles_t = f8_scale_tiles(A.rows);
    const int kind = A.out.kind;
    if (threadIdx.x == 0)
        square_most = 0;
    grid_wait();
    if (r0 >= A.rows || c0 >= A.cols) {   // scales of blocks that do not exist
        if (threadIdx.x < 128) {
            if (A.out.codes && r0 < A.rows)
                A.out.scales[f8_scale_at(r0 + threadIdx.x, c0 / 128, scale_tiles)] = 0;
            if (A.out.codes_t && c0 < A.cols)
                A.out.scales_t[f8_scale_at(c0 + threadIdx.x, r0 / 128, scale_tiles_t)] = 0;
        }
        return;
    }
    // where (WIDE) column c of a row lies
    auto place = [](uint32_t c) { return (c & ~12u) | ((((c >> 2) ^ (c >> 5)) & 3u) << 2); };
    if constexpr (VEC) {
        const int part = lane & 7, group = threadIdx.x >> 3;
        constexpr int HIGH = kTileThreads / 8, PASSES = 128 / HIGH;
        Piece<T, true> p[PASSES];
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int64_t row = r0 + i * HIGH + group;
            p[i].load(x + row * A.ld, (uint32_t)c0, row < A.rows ? (uint32_t)A.cols : 0u, part, A.aligned32);
        }
        uint32_t all = 0;
        if (A.square) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                float v[16];
                p[i].unpack(v);
                all = max(all, __float_as_uint(absmax<16>(v)));
            }
            all = __reduce_max_sync(0xffffffffu, all);
            if (lane == 0)
                atomicMax(&square_most, all);
            __syncthreads();
            all = square_most;
        }
        float w[NORM ? 16 : 1];
        if constexpr (NORM) {
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int64_t c = c0 + part * 16 + q;
                w[q] = c >= A.cols ? 0.f : A.w32 ? ((const float *)A.w)[c] : to_f32(((const T *)A.w)[c]);
            }
        }
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int64_t row = r0 + i * HIGH + group;
            float v[16];
            p[i].unpack(v);
            if constexpr (NORM) {
                norm_values<16>(v, w, row < A.rows ? A.rstd[row] : 1.f, row < A.rows && c0 + part * 16 < A.cols);
            }
            if (A.out.codes_t) {
                if constexpr (WIDE) {
#pragma unroll
                    for (int q = 0; q < 16; q += 4)
                        *(float4 *)&tile[(i * HIGH + group) * 128 + place(part * 16 + q)] = make_float4(v[q], v[q + 1], v[q + 2], v[q + 3]);
                } else {
#pragma unroll
                    for (int q = 0; q < 8; q += 4)
                        *(uint4 *)&tile[(i * HIGH + group) * 64 + part * 8 + q] = make_uint4(p[i].w[q], p[i].w[q + 1], p[i].w[q + 2], p[i].w[q + 3]);
                }
            }
            if (A.out.codes) {
                uint32_t most = all;
                if (!A.square) {
                    most = __float_as_uint(absmax<16>(v));
#pragma unroll
                    for (int o = 1; o < 8; o *= 2)
                        most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
                }
                const uint32_t byte = f8_scale(most, kind);
                uint32_t code[4];
                f8_encode<16>(v, byte, kind, code);
                if (row < A.rows)
                    *(uint4 *)(A.out.codes + (row * blocks + c0 / 128) * 128 + part * 16) = make_uint4(code[0], code[1], code[2], code[3]);
                if (part == 0)
                    A.out.scales[f8_scale_at(row, c0 / 128, scale_tiles)] = (uint8_t)(row < A.rows ? byte : 0u);
            }
        }
    } else {
        // a row of the tile per warp, every 32nd element to a lane
        uint32_t all = 0;
        float w[4];
        if constexpr (NORM) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t c = c0 + q * 32 + lane;
                w[q] = c >= A.cols ? 0.f : A.w32 ? ((const float *)A.w)[c] : to_f32(((const T *)A.w)[c]);
            }
        }
        auto codes = [&](const float *v, int64_t row, uint32_t most) {
            const uint32_t byte = f8_scale(most, kind);
            uint32_t code;
            f8_encode<4>(v, byte, kind, &code);
            code = bytes_turned(code, lane);
            if (row < A.rows)
                *(uint32_t *)(A.out.codes + (row * blocks + c0 / 128) * 128 + (lane & 3) * 32 + (lane >> 2) * 4) = code;
            if (lane == 0)
                A.out.scales[f8_scale_at(row, c0 / 128, scale_tiles)] = (uint8_t)(row < A.rows ? byte : 0u);
        };
#pragma unroll
        for (int half = 0; half < 128 / (4 * kTileWarps); ++half) {
            Bits b[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t row = r0 + (half * 4 + i) * kTileWarps + warp;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t c = c0 + q * 32 + lane;
                    b[i][q] = row < A.rows && c < A.cols ? ((const Bits *)x)[row * A.ld + c] : (Bits)0;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = (half * 4 + i) * kTileWarps + warp;
                const int64_t row = r0 + at;
                float v[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    v[q] = to_f32(*(const T *)&b[i][q]);
                if constexpr (NORM)
                    norm_values<4>(v, w, row < A.rows ? A.rstd[row] : 1.f, row < A.rows && c0 + lane < A.cols);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (WIDE)
                        tile[at * 128 + place(q * 32 + lane)] = __float_as_uint(v[q]);
                    else
                        ((uint16_t *)tile)[at * 128 + q * 32 + lane] = b[i][q];
                }
                const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(absmax4(v)));
                if (A.square)
                    all = max(all, most);
                else if (A.out.codes)
                    codes(v, row, most);
            }
        }
        if (A.square) {
            __syncthreads();
            if (lane == 0)
                atomicMax(&square_most, all);
            __syncthreads();
            if (A.out.codes)
                for (int at = warp; at < 128; at += kTileWarps) {
                    float v[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if constexpr (WIDE) {
                            v[q] = __uint_as_float(tile[at * 128 + place(q * 32 + lane)]);
                        } else {
                            const uint16_t h = ((const uint16_t *)tile)[at * 128 + q * 32 + lane];
                            v[q] = to_f32(*(const T *)&h);
                        }
                    }
                    codes(v, r0 + at, square_most);
                }
        }
    }
    if (!A.out.codes_t)
        return;
    __syncthreads();
    // ROWS rows of two columns
    constexpr int ROWS = WIDE ? 16 : 32;
    const int quarter = WIDE ? warp >> 2 : threadIdx.x >> 6, half = WIDE ? lane >> 4 : 0, pair = WIDE ? (warp & 3) * 16 + (lane & 15) : threadIdx.x & 63;
    const int row = quarter * 32 + half * 16;
    const int64_t c = c0 + 2 * pair;
    float v[2][ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if constexpr (WIDE) {
            const float2 f = *(const float2 *)&tile[(row + i) * 128 + place(2 * pair)];
            v[0][i] = f.x, v[1][i] = f.y;
        } else {
            const uint32_t word = tile[(row + i) * 64 + pair];
            const uint16_t lo = (uint16_t)word, hi = (uint16_t)(word >> 16);
            v[0][i] = to_f32(*(const T *)&lo), v[1][i] = to_f32(*(const T *)&hi);
        }
    }
    uint32_t most[2];
    if (!A.square) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            most[h] = __float_as_uint(absmax<ROWS>(v[h]));
            if (WIDE)
                most[h] = max(most[h], __shfl_xor_sync(0xffffffffu, most[h], 16));
        }
        if (half == 0)
            *(uint2 *)&col_most[quarter][2 * pair] = make_uint2(most[0], most[1]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint2 o = *(const uint2 *)&col_most[i][2 * pair];
            most[0] = max(most[0], o.x), most[1] = max(most[1], o.y);
        }
    } else {
        most[0] = most[1] = square_most;
    }
    auto store = [&](int64_t column, uint32_t byte, const uint32_t *code) {
        if (column < A.cols) {
            uint4 *const to = (uint4 *)(A.out.codes_t + (column * blocks_t + r0 / 128) * 128 + quarter * 32);
            if (A.whole) {   // (a sector at once)
                store32_keep(to, *(const uint32_t(*)[8])code);
            } else {
                to[0] = make_uint4(code[0], code[1], code[2], code[3]);
                to[1] = make_uint4(code[4], code[5], code[6], code[7]);
            }
        }
        if (quarter == 0)
            A.out.scales_t[f8_scale_at(column, r0 / 128, scale_tiles_t)] = (uint8_t)(column < A.cols ? byte : 0u);
    };
    uint32_t byte[2], code[2][ROWS / 4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        byte[h] = f8_scale(most[h], kind);
        f8_encode<ROWS>(v[h], byte[h], kind, code[h]);
        if (!WIDE)
            store(c + h, byte[h], code[h]);
    }
    if constexpr (WIDE) {   // the lower half of a warp takes the first column's 32 rows, the upper one the second's
        uint32_t mine[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, half ? code[0][i] : code[1][i], 16);
            mine[i] = half ? other : code[0][i], mine[4 + i] = half ? code[1][i] : other;
        }
        store(c + half, half ? byte[1] : byte[0], mine);
    }
}

// ------------------------------------------------------------------ the way back
template <class T, bool VEC>
__global__ void __launch_bounds__(kF8Threads) k_f8_dequantise(const uint8_t *codes, const uint8_t *scales, int kind, const Pieces pieces, uint32_t row0, uint32_t units,
                                                              int64_t cols, T *out, int64_t ld, bool aligned32)
{
    grid_release();
    const int lane = threadIdx.x & 31;
    const uint32_t u = blockIdx.x * (kF8Threads / 32) + (threadIdx.x >> 5);
    if (u >= units)
        return;
    uint32_t at, tile;
    pieces.place(u, at, tile);
    const int64_t row = (int64_t)row0 + at, blocks = f8_blocks(cols);
    const uint8_t *const from = codes + row * blocks * 128, *const s = scales + f8_scale_at(row, tile * 4, f8_scale_tiles(cols));
    const uint32_t c0 = tile * 512u;
    grid_wait();
    float v[16];
    if constexpr (VEC) {
        const uint32_t c = c0 + lane * 16;
        if (c >= cols)
            return;
        const uint4 w = __ldcs((const uint4 *)(from + c));
        const float f = f8_pow(s[lane >> 3]);
        f8_values4(w.x, kind, v), f8_values4(w.y, kind, v + 4), f8_values4(w.z, kind, v + 8), f8_values4(w.w, kind, v + 12);
#pragma unroll
        for (int q = 0; q < 16; ++q)
            v[q] = __fmul_rn(v[q], f);
    } else {
        const uint32_t bytes = *(const uint32_t *)s;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const uint32_t c = c0 + b * 128 + (lane & 3) * 32 + (lane >> 2) * 4;   // (rows are padded to blocks)
            f8_values4(bytes_turned(c0 / 128 + b < blocks ? *(const uint32_t *)(from + c) : 0u, lane), kind, v + 4 * b);
            const float f = f8_pow(bytes >> (8 * b) & 255u);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[4 * b + q] = __fmul_rn(v[4 * b + q], f);
        }
    }
    Piece<T, VEC> p;
    p.pack(v);
    p.store(out + row * ld, c0, (uint32_t)cols, lane, aligned32);
}

template <class T>
static cudaError_t rows_form(const T *x, int64_t rows, int64_t cols, int64_t ld, const F8Out &out, cudaStream_t s)
{
    const bool vec = rows_on<T>(x, rows, ld, 16), aligned32 = rows_on<T>(x, rows, ld, 32);
    const int64_t tiles = f8_scale_tiles(cols), padded = (rows + 127) / 128 * 128, most = rows_per_launch(tiles);
    cudaError_t e = cudaSuccess;
    for (int64_t r0 = 0; r0 < padded && e == cudaSuccess; r0 += most) {
        const int64_t units = std::min(most, padded - r0) * tiles;
        const dim3 grid((unsigned)((units + kF8Threads / 32 - 1) / (kF8Threads / 32)));
        e = vec ? launch(k_f8_rows<T, true>, grid, kF8Threads, 0, s, x, pieces_of(tiles), (uint32_t)r0, (uint32_t)units, rows, cols, ld, out, aligned32)
                : launch(k_f8_rows<T, false>, grid, kF8Threads, 0, s, x, pieces_of(tiles), (uint32_t)r0, (uint32_t)units, rows, cols, ld, out, aligned32);
    }
    return e;
}

template <class T, bool NORM>
static cudaError_t tiles_form(const T *x, const TileArgs &A, int64_t n_tiles, cudaStream_t s)
{
    const size_t smem = (NORM || sizeof(T) == 4 ? 128 : 64) * 128 * 4;
    static int done[2][64];
    const bool vec = rows_on<T>(x, A.rows, A.ld, 16);
    cudaError_t e = vec ? opt_in_smem(k_f8_tiles<T, true, NORM>, smem, done[1]) : opt_in_smem(k_f8_tiles<T, false, NORM>, smem, done[0]);
    if (e == cudaSuccess)
        e = vec ? launch(k_f8_tiles<T, true, NORM>, dim3((unsigned)n_tiles), tile_threads<T, NORM>(), smem, s, x, A)
                : launch(k_f8_tiles<T, false, NORM>, dim3((unsigned)n_tiles), tile_threads<T, NORM>(), smem, s, x, A);
    return e;
}

cudaError_t f8_tiles(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, const float *rstd, const void *w, bool w32, bool square, const F8Out &out,
                     cudaStream_t s)
{
    TileArgs A = {rows, cols, ld, rstd, w, out, (uint32_t)(f8_scale_tiles(cols) * 4), w32, square, false, ((uintptr_t)out.codes_t & 31) == 0};
    const int64_t tiles_r = out.codes_t ? f8_scale_tiles(rows) * 4 : (rows + 127) / 128;
    cudaError_t e = cudaErrorInvalidValue;
    with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        A.aligned32 = rows_on<T>(x, rows, ld, 32);
        e = rstd ? tiles_form<T, true>((const T *)x, A, tiles_r * A.tiles_c, s) : tiles_form<T, false>((const T *)x, A, tiles_r * A.tiles_c, s);
        return 0;
    });
    return e;
}

template <class T>
static cudaError_t dequantise(const uint8_t *codes, const uint8_t *scales, int kind, int64_t rows, int64_t cols, T *out, int64_t ld, cudaStream_t s)
{
    const bool vec = rows_on<T>(out, rows, ld, 16), aligned32 = rows_on<T>(out, rows, ld, 32);
    const int64_t tiles = f8_scale_tiles(cols), most = rows_per_launch(tiles);
    cudaError_t e = cudaSuccess;
    for (int64_t r0 = 0; r0 < rows && e == cudaSuccess; r0 += most) {
        const int64_t units = std::min(most, rows - r0) * tiles;
        const dim3 grid((unsigned)((units + kF8Threads / 32 - 1) / (kF8Threads / 32)));
        e = vec ? launch(k_f8_dequantise<T, true>, grid, kF8Threads, 0, s, codes, scales, kind, pieces_of(tiles), (uint32_t)r0, (uint32_t)units, cols, out, ld, aligned32)
                : launch(k_f8_dequantise<T, false>, grid, kF8Threads, 0, s, codes, scales, kind, pieces_of(tiles), (uint32_t)r0, (uint32_t)units, cols, out, ld, aligned32);
    }
    return e;
}

}  // namespace conef

using namespace conef;

extern "C" {

int conef_f8_bytes(int64_t rows, int64_t cols, size_t *code_bytes, size_t *scale_bytes)
{
    if (rows < 0 || cols < 0)
        return CONEF_ERR_INVALID_ARG;
    if (rows >= (1ll << 31) || cols >= (1ll << 31))
        return CONEF_ERR_UNSUPPORTED;
    if (code_bytes)
        *code_bytes = (size_t)rows * (size_t)f8_blocks(cols) * 128;
    if (scale_bytes)
        *scale_bytes = (size_t)((rows + 127) / 128) * (size_t)f8_scale_tiles(cols) * 512;
    return CONEF_OK;
}

int conef_f8_quantise(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int kind, int square, void *codes, void *scales, void *codes_t, void *scales_t,
                      conef_stream stream)
{
    int rc = check_matrix(x, dtype, rows, cols, ld);
    if (rc != CONEF_OK)
        return rc;
    if ((kind != CONEF_E4M3 && kind != CONEF_E5M2) || !codes != !scales || !codes_t != !scales_t || !(codes || codes_t))
        return CONEF_ERR_INVALID_ARG;
    if ((((uintptr_t)codes | (uintptr_t)scales | (uintptr_t)codes_t | (uintptr_t)scales_t) & 15) != 0)
        return CONEF_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0)
        return CONEF_OK;
    const F8Out out = {(uint8_t *)codes, (uint8_t *)scales, (uint8_t *)codes_t, (uint8_t *)scales_t, kind};
    if (!codes_t && !square)
        return with_elem(dtype, [&](auto t) {
            using T = decltype(t);
            return launched(rows_form<T>((const T *)x, rows, cols, ld, out, (cudaStream_t)stream), "conef_f8_quantise");
        });
    if (f8_scale_tiles(rows) * 4 * (f8_scale_tiles(cols) * 4) >= (1ll << 31))
        return CONEF_ERR_UNSUPPORTED;
    return launched(f8_tiles(x, dtype, rows, cols, ld, nullptr, nullptr, false, square != 0, out, (cudaStream_t)stream), "conef_f8_quantise");
}

int conef_f8_dequantise(const void *codes, const void *scales, int64_t rows, int64_t cols, int kind, void *out, int dtype, int64_t ld, conef_stream stream)
{
    int rc = check_matrix(out, dtype, rows, cols, ld);
    if (rc != CONEF_OK)
        return rc;
    if (kind != CONEF_E4M3 && kind != CONEF_E5M2)
        return CONEF_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0)
        return CONEF_OK;
    if (!codes || !scales || (((uintptr_t)codes | (uintptr_t)scales) & 15) != 0)
        return CONEF_ERR_INVALID_ARG;
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        return launched(dequantise<T>((const uint8_t *)codes, (const uint8_t *)scales, kind, rows, cols, (T *)out, ld, (cudaStream_t)stream), "conef_f8_dequantise");
    });
}

}  // extern "C"
