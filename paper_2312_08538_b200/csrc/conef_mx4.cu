// Quantisation to microscaled 4-bit floats (conef_mx4.cuh), of a matrix and of its transpose, behind a dropout where one is
// asked for, and the way back.
#include <algorithm>

#include "conef_mx4.cuh"
#include "conef_common.cuh"
#include "conef_elem.cuh"

namespace conef {

constexpr int kQThreads = 256;

// eight elements from p on, which is aligned to their size
template <class T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
        uint32_t w[8];
        load32(p, w);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            v[q] = __uint_as_float(w[q]);
    } else {
        Vec16<T>::unpack(__ldcs((const uint4 *)p), v);
    }
}
// x behind the dropout, rounded to fp32, of four columns
__device__ __forceinline__ void drop4(float *v, uint64_t word, const Dropout &d)
{
    const uint32_t lo = (uint32_t)word, hi = (uint32_t)(word >> 32);
    v[0] = (lo << 16) > d.limit ? __fmul_rn(v[0], d.scale) : 0.f;
    v[1] = lo > d.limit ? __fmul_rn(v[1], d.scale) : 0.f;
    v[2] = (hi << 16) > d.limit ? __fmul_rn(v[2], d.scale) : 0.f;
    v[3] = hi > d.limit ? __fmul_rn(v[3], d.scale) : 0.f;
}

struct QArgs {
    int64_t rows, cols, ld;
    uint64_t dropout, rounding;   // draw_base() of the two
    Dropout drop;
    uint8_t *codes, *scales, *codes_t, *scales_t;
};

// ------------------------------------------------------------------ rows
// LANES lanes per block.  Blocks are counted over the padded tiles of scales, so that the bytes of those that do not exist get their zero.  Four lanes
// load side by side, but what does not depend on the number of elements is then done for eight of them: 8192 x 6400 in bf16 took 34 us, with a lane per
// block 18 (7.2 TB/s), with two 22; with stochastic rounding 52, 34, 41.  In fp32 a lane's 128 bytes are four requests to 32 lines each, and rounding to
// nearest does less for them: 50257 x 1600 with four, two and one lane 58, 52, 62 us, stochastic 84, 70, 63.  So one, or two in fp32 without draws;
// four where rows are not aligned, and where there are too few blocks for all SMs.
template <class T, bool VEC, bool STOCH, bool DROP, int LANES>
__global__ void __launch_bounds__(kQThreads) k_mx4_rows(const T *x, const __grid_constant__ QArgs A, const Divider padded, uint32_t row0, uint32_t units)
{
    constexpr int E = 32 / LANES, W = E / 8;   // elements and words of codes per lane
    grid_release();
    const uint32_t blocks = (uint32_t)mx4_blocks(A.cols), tiles = padded.by / 4, part = threadIdx.x % LANES;
    const uint32_t u = blockIdx.x * (uint32_t)(kQThreads / LANES) + threadIdx.x / LANES;
    const uint32_t groups = (uint32_t)(A.cols + 3) / 4, at = divide(u, padded), row = row0 + at, block = u - at * padded.by, c = block * 32u + part * E;
    const T *p = x + (int64_t)row * A.ld + c;
    const uint32_t have = u < units && row < A.rows && c < A.cols ? (uint32_t)A.cols - c : 0u;
    grid_wait();
    float v[E];
    if (VEC && have >= (uint32_t)E) {
#pragma unroll
        for (int w = 0; w < W; ++w)
            load8<T>(p + 8 * w, *(float(*)[8])(v + 8 * w));
    } else {
#pragma unroll
        for (int q = 0; q < E; ++q)
            v[q] = (uint32_t)q < have ? to_f32(p[q]) : 0.f;
    }
    const uint64_t group = (uint64_t)row * groups + block * 8u + part * (E / 4);
    if (DROP) {
        const uint64_t z = A.dropout + kDrawStep * group;
#pragma unroll
        for (int g = 0; g < E / 4; ++g)
            drop4(v + 4 * g, mix64(z + kDrawStep * g), A.drop);
    }
    float most = absmax<E>(v);
#pragma unroll
    for (int o = 1; o < LANES; o *= 2)
        most = absmax2(most, __shfl_xor_sync(0xffffffffu, most, o));
    const uint32_t byte = mx4_scale(__float_as_uint(most));
    const float inv = mx4_inv(byte);
#pragma unroll
    for (int q = 0; q < E; ++q)
        v[q] = __fmul_rn(v[q], inv);
    uint32_t code[W];
    const uint64_t z = A.rounding + kDrawStep * group;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        code[w] = STOCH ? mx4_stochastic8(v + 8 * w, mix64(z + kDrawStep * (2 * w)), mix64(z + kDrawStep * (2 * w + 1))) : mx4_nearest8(v + 8 * w);
        code[w] = byte == kMx4Nan ? 0u : code[w];   // (elements that do not exist are zero, which no number rounds up)
    }
    if (u < units) {
        const bool there = row < A.rows && block < blocks;
        if (part == 0)
            A.scales[mx4_scale_at(row, block, tiles)] = (uint8_t)(there ? byte : 0u);
        if (there) {
            uint8_t *o = A.codes + ((uint64_t)row * blocks + block) * 16 + part * (E / 2);
            if constexpr (W == 4)
                *(uint4 *)o = make_uint4(code[0], code[1], code[2], code[3]);
            else if constexpr (W == 2)
                *(uint2 *)o = make_uint2(code[0], code[1]);
            else
                *(uint32_t *)o = code[0];
        }
    }
}

// ------------------------------------------------------------------ the transpose, and rows with it
// A warp takes 64 x 64 elements, 32 x 32 at a time: a lane has 32 elements of a row, which is a block of the rows' form, and hands them and
// their numbers through shared memory to the lanes of the columns, of which each has a block of the transpose.  One reading
// of x and one hash per four elements serve both.
//
// Words of a tile are exchanged within a row, 16 bytes at a time, so that a lane stores four at once and a column's are read without bank conflicts.
// Rows come in lines of 128 bytes by eight lanes each, and are turned to a row per lane in shared memory, or (LINES and PAIRS false) straight to
// the lane that has the row, 32 bytes per request.  8192 x 6400 in fp32, lines and lanes: to nearest 55 and 75 us, stochastic behind a dropout 86 and 87.
// Elements of 16 bits (PAIRS) stay in shared memory as they came, 32 rows of 64, their numbers in as many words again, and a lane
// reads two columns at a time: to nearest it writes and reads half as much there, which was what it spent its time on; stochastic it need not put
// elements and numbers together.  bf16 to nearest both forms 38 us, the columns alone 27; a word per element in lines 48 and 38, by lanes 58 and 44;
// stochastic 56, a word per element 63.  Behind a dropout, which has a second hash per four elements, it was no faster
// (77; a word per element, by lanes, 75: ALU pipe 78 %).
constexpr int kBothWarps = 4;
template <class T, bool STOCH, bool DROP>
struct alignas(128) BothTile {
    uint32_t v[32 * 32];   // 32 x 32 elements, a word each (16 bits: with their numbers above), or 32 x 64 of 16 bits, two to a word
    uint32_t n[sizeof(T) == 2 && STOCH && !DROP ? 32 * 32 : 4];   // ... their numbers
    uint16_t u[sizeof(T) == 4 && STOCH ? 32 : 1][34];
};
__device__ __forceinline__ uint32_t both_piece(uint32_t row, uint32_t piece) { return row * 32u + ((piece ^ (row & 7u)) << 2); }   // words
__device__ __forceinline__ uint32_t both_word(uint32_t row, uint32_t col) { return both_piece(row, col >> 2) + (col & 3u); }
// four elements of 16 bits, two to a word: what their numbers keep (their scale comes later)
__device__ __forceinline__ void drop_pairs(uint32_t &a, uint32_t &b, uint64_t d, const Dropout &drop)
{
    const uint32_t lo = (uint32_t)d, hi = (uint32_t)(d >> 32);
    a &= ((lo << 16) > drop.limit ? 0xFFFFu : 0u) | (lo > drop.limit ? 0xFFFF0000u : 0u);
    b &= ((hi << 16) > drop.limit ? 0xFFFFu : 0u) | (hi > drop.limit ? 0xFFFF0000u : 0u);
}
template <class T, bool VEC, bool ROWS, bool STOCH, bool DROP>
__global__ void __launch_bounds__(kBothWarps * 32, STOCH ? 4 : 5) k_mx4_both(const T *x, const __grid_constant__ QArgs A, uint32_t tiles_c, int64_t n_tiles)
{
    constexpr bool SHORT = sizeof(T) == 2, LINES = VEC && !SHORT, PAIRS = VEC && SHORT && !(STOCH && DROP);
    __shared__ BothTile<T, STOCH, DROP> S[kBothWarps];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t tile = (int64_t)blockIdx.x * kBothWarps + warp;
    BothTile<T, STOCH, DROP> &M = S[warp];
    const int64_t tr = tile / tiles_c, rbase = tr * 64, cbase = (tile - tr * tiles_c) * 64;
    const int64_t blocks = mx4_blocks(A.cols), blocks_t = mx4_blocks(A.rows), scale_tiles = mx4_scale_tiles(A.cols), scale_tiles_t = mx4_scale_tiles(A.rows);
    const uint64_t groups = (uint64_t)(A.cols + 3) / 4;
    const bool aligned32 = (((uintptr_t)x | (uint64_t)A.ld * sizeof(T)) & 31) == 0;
    grid_wait();
    if (tile >= n_tiles)
        return;
    float v[32];
    // scales 32 elements; the scale
    auto scaled = [&](float (&v)[32]) {
        float most = absmax<32>(v);
        if (SHORT && DROP)   // (the largest product is that of the largest element)
            most = __fmul_rn(most, A.drop.scale);
        const uint32_t byte = mx4_scale(__float_as_uint(most));
        float inv = mx4_inv(byte);
        if (SHORT && DROP) {
            // Times the dropout's scale, rounded, and times a power of two: one product by both is the same where neither step leaves the
            // normal range.  From 2^-95 on (the byte 32) a product below it is 0 either way.
            if (byte >= 32u) {
                inv = __fmul_rn(inv, A.drop.scale);
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    v[i] = __fmul_rn(v[i], A.drop.scale);
            }
        }
#pragma unroll
        for (int i = 0; i < 32; ++i)
            v[i] = __fmul_rn(v[i], inv);
        return byte;
    };
    // 32 elements' codes; their scale
    auto encode = [&](auto &&codes_of, uint32_t (&code)[4]) {
        const uint32_t byte = scaled(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            code[i] = codes_of(i);
            code[i] = byte == kMx4Nan ? 0u : code[i];   // (elements that do not exist are zero, which no number rounds up)
        }
        return byte;
    };
    for (int sr = 0; sr < 2; ++sr) {
        if constexpr (PAIRS) if (rbase + sr * 32 < A.rows && cbase + 64 <= A.cols) {
            const int64_t r0 = rbase + sr * 32, r = r0 + lane;
            uint32_t code[4];
            uint4 w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t row = r0 + 4 * k + (lane >> 3);
                w[k] = row < A.rows ? __ldcs((const uint4 *)(x + row * A.ld + cbase) + (lane & 7)) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                *(uint4 *)&M.v[both_piece(4 * k + (lane >> 3), lane & 7)] = w[k];
            __syncwarp();
            if (ROWS || DROP || STOCH) {
                uint32_t bytes = 0;
#pragma unroll
                for (int sc = 0; sc < 2; ++sc) {
                    const uint64_t group = (uint64_t)r * groups + (uint64_t)((cbase >> 2) + sc * 8), zd = A.dropout + kDrawStep * group,
                                   zr = A.rounding + kDrawStep * group;
                    uint64_t word[STOCH ? 8 : 1];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t at = both_piece(lane, sc * 4 + i);
                        uint4 q = *(const uint4 *)&M.v[at];
                        if (DROP) {
                            drop_pairs(q.x, q.y, mix64(zd + kDrawStep * (2 * i)), A.drop);
                            drop_pairs(q.z, q.w, mix64(zd + kDrawStep * (2 * i + 1)), A.drop);
                            *(uint4 *)&M.v[at] = q;
                        }
                        if constexpr (STOCH) {
                            const uint64_t a = mix64(zr + kDrawStep * (2 * i)), b = mix64(zr + kDrawStep * (2 * i + 1));
                            *(uint4 *)&M.n[at] = make_uint4((uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32));
                            word[2 * i] = a, word[2 * i + 1] = b;
                        }
                        Vec16<T>::unpack(q, *(float(*)[8])(v + 8 * i));
                    }
                    if (ROWS) {
                        bytes |= encode([&](int i) { return STOCH ? mx4_stochastic8(v + 8 * i, word[STOCH ? 2 * i : 0], word[STOCH ? 2 * i + 1 : 0]) : mx4_nearest8(v + 8 * i); }, code) << (8 * sc);
                        if (r < A.rows)
                            *(uint4 *)(A.codes + (r * blocks + (cbase >> 5) + sc) * 16) = make_uint4(code[0], code[1], code[2], code[3]);
                    }
                }
                if (ROWS)
                    *(uint16_t *)&A.scales[mx4_scale_at(r, cbase >> 5, scale_tiles)] = (uint16_t)(r < A.rows ? bytes : 0u);
                if (DROP || STOCH)
                    __syncwarp();   // (lanes wrote to their own rows)
            }
            // two columns to a lane
            const int64_t ct = cbase + 2 * lane;
            float v1[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t w = M.v[both_word(i, lane)];
                const uint16_t lo = (uint16_t)w, hi = (uint16_t)(w >> 16);
                v[i] = to_f32(*(const T *)&lo), v1[i] = to_f32(*(const T *)&hi);
            }
            const uint32_t byte = scaled(v), byte1 = scaled(v1);
            uint32_t code1[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (STOCH) {
                    uint32_t lo[8], hi[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const uint32_t w = M.n[both_word(8 * i + q, lane)];
                        lo[q] = mx4_noise_lo(w), hi[q] = mx4_noise_hi(w);
                    }
                    code[i] = mx4_stochastic8(v + 8 * i, lo), code1[i] = mx4_stochastic8(v1 + 8 * i, hi);
                } else {
                    code[i] = mx4_nearest8(v + 8 * i), code1[i] = mx4_nearest8(v1 + 8 * i);
                }
                code[i] = byte == kMx4Nan ? 0u : code[i], code1[i] = byte1 == kMx4Nan ? 0u : code1[i];
            }
            A.scales_t[mx4_scale_at(ct, r0 >> 5, scale_tiles_t)] = (uint8_t)byte, A.scales_t[mx4_scale_at(ct + 1, r0 >> 5, scale_tiles_t)] = (uint8_t)byte1;
            uint8_t *const to = A.codes_t + (ct * blocks_t + (r0 >> 5)) * 16;
            *(uint4 *)to = make_uint4(code[0], code[1], code[2], code[3]), *(uint4 *)(to + blocks_t * 16) = make_uint4(code1[0], code1[1], code1[2], code1[3]);
            __syncwarp();
            continue;
        }
        for (int sc = 0; sc < 2; ++sc) {
            const int64_t r0 = rbase + sr * 32, c0 = cbase + sc * 32, r = r0 + lane, ct = c0 + lane;
            if (r0 >= A.rows || c0 >= A.cols) {   // scales of blocks that do not exist
                if (ROWS)
                    A.scales[mx4_scale_at(r, c0 >> 5, scale_tiles)] = 0;
                A.scales_t[mx4_scale_at(ct, r0 >> 5, scale_tiles_t)] = 0;
                continue;
            }
            // a lane's row: 16 bits as they are, two to a word, or fp32
            constexpr int RAW = SHORT ? 16 : 32;
            uint32_t raw[RAW];
            const bool lines = LINES && c0 + 32 <= A.cols;
            if (lines) {
                // eight lanes per 128-byte line, four lines at a time, turned to a row per lane in shared memory
                uint4 w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int64_t row = r0 + 4 * k + (lane >> 3);
                    w[k] = row < A.rows ? __ldcs((const uint4 *)(x + row * A.ld + c0) + (lane & 7)) : make_uint4(0u, 0u, 0u, 0u);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    *(uint4 *)&M.v[both_piece(4 * k + (lane >> 3), lane & 7)] = w[k];
                __syncwarp();
#pragma unroll
                for (int i = 0; i < RAW; i += 4) {
                    const uint4 q = *(const uint4 *)&M.v[both_piece(lane, i / 4)];
                    raw[i] = q.x, raw[i + 1] = q.y, raw[i + 2] = q.z, raw[i + 3] = q.w;
                }
            } else if (VEC && c0 + 32 <= A.cols) {
                const T *p = x + r * A.ld + c0;
#pragma unroll
                for (int i = 0; i < RAW; i += 8) {
                    if (r < A.rows) {
                        if (!SHORT || aligned32) {
                            load32((const uint32_t *)p + i, *(uint32_t(*)[8])(raw + i));
                        } else {
                            const uint4 a = __ldcs((const uint4 *)((const uint32_t *)p + i)), b = __ldcs((const uint4 *)((const uint32_t *)p + i + 4));
                            raw[i] = a.x, raw[i + 1] = a.y, raw[i + 2] = a.z, raw[i + 3] = a.w, raw[i + 4] = b.x, raw[i + 5] = b.y, raw[i + 6] = b.z, raw[i + 7] = b.w;
                        }
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            raw[i + q] = 0u;
                    }
                }
            } else {   // a row at a time, and turned
                const T *p = x + r0 * A.ld + ct;
                const int rows = (int)min((int64_t)32, A.rows - r0);
                using Bits = std::conditional_t<SHORT, uint16_t, uint32_t>;
                uint32_t t[32];
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    t[i] = i < rows && ct < A.cols ? (uint32_t)((const Bits *)p)[i * A.ld] : 0u;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    M.v[both_word(i, lane)] = t[i];
                __syncwarp();
#pragma unroll
                for (int g = 0; g < 8; ++g) {
                    const uint4 w = *(const uint4 *)&M.v[both_piece(lane, g)];
                    if constexpr (SHORT)
                        raw[2 * g] = w.x | w.y << 16, raw[2 * g + 1] = w.z | w.w << 16;
                    else
                        raw[4 * g] = w.x, raw[4 * g + 1] = w.y, raw[4 * g + 2] = w.z, raw[4 * g + 3] = w.w;
                }
                __syncwarp();
            }
            const uint64_t group = (uint64_t)r * groups + (uint64_t)(c0 >> 2);
            uint64_t word[STOCH ? 8 : 1];
            if (STOCH) {
                const uint64_t z = A.rounding + kDrawStep * group;
#pragma unroll
                for (int g = 0; g < 8; ++g)
                    word[STOCH ? g : 0] = mix64(z + kDrawStep * g);
            }
            if (DROP) {
                const uint64_t z = A.dropout + kDrawStep * group;
#pragma unroll
                for (int g = 0; g < 8; ++g) {
                    const uint64_t d = mix64(z + kDrawStep * g);
                    if constexpr (SHORT)
                        drop_pairs(raw[2 * g], raw[2 * g + 1], d, A.drop);
                    else
                        drop4((float *)raw + 4 * g, d, A.drop);
                }
            }
            // for the columns: an element (16 bits: with its number above)
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                uint32_t w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t n = STOCH ? (uint32_t)(word[STOCH ? g : 0] >> (q & 2 ? 32 : 0)) : 0u;   // its number is one half of this
                    if (SHORT) {
                        const uint32_t pair = raw[(2 * g + q / 2) % RAW];
                        w[q] = STOCH ? __byte_perm(pair, n, q & 1 ? 0x7632 : 0x5410) : q & 1 ? pair >> 16 : pair;
                    } else {
                        w[q] = raw[(4 * g + q) % RAW];
                        if (STOCH)
                            M.u[lane][4 * g + q] = (uint16_t)(q & 1 ? n >> 16 : n);
                    }
                }
                if (SHORT || DROP || !lines)   // (else they are there)
                    *(uint4 *)&M.v[both_piece(lane, g)] = make_uint4(w[0], w[1], w[2], w[3]);
            }
            uint32_t code[4];
            if (ROWS) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (SHORT) {
                        const uint4 q = make_uint4(raw[4 * i], raw[4 * i + 1], raw[4 * i + 2], raw[4 * i + 3]);
                        Vec16<T>::unpack(q, *(float(*)[8])(v + 8 * i));
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            v[8 * i + q] = __uint_as_float(raw[(8 * i + q) % RAW]);
                    }
                }
                const uint32_t byte = encode([&](int i) { return STOCH ? mx4_stochastic8(v + 8 * i, word[STOCH ? 2 * i : 0], word[STOCH ? 2 * i + 1 : 0]) : mx4_nearest8(v + 8 * i); }, code);
                A.scales[mx4_scale_at(r, c0 >> 5, scale_tiles)] = (uint8_t)(r < A.rows ? byte : 0u);
                if (r < A.rows)
                    *(uint4 *)(A.codes + (r * blocks + (c0 >> 5)) * 16) = make_uint4(code[0], code[1], code[2], code[3]);
            }
            __syncwarp();
            // the columns
            uint32_t noise[STOCH ? 32 : 8];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t w = M.v[both_word(i, lane)];
                if constexpr (SHORT) {
                    const uint16_t h = (uint16_t)w;
                    v[i] = to_f32(*(const T *)&h);
                    if (STOCH)
                        noise[STOCH ? i : 0] = mx4_noise_hi(w);
                } else {
                    v[i] = __uint_as_float(w);
                    if (STOCH)
                        noise[STOCH ? i : 0] = mx4_noise_lo(M.u[i][lane]);
                }
            }
            const uint32_t byte = encode([&](int i) { return STOCH ? mx4_stochastic8(v + 8 * i, *(uint32_t(*)[8])(noise + (STOCH ? 8 * i : 0))) : mx4_nearest8(v + 8 * i); }, code);
            A.scales_t[mx4_scale_at(ct, r0 >> 5, scale_tiles_t)] = (uint8_t)(ct < A.cols ? byte : 0u);
            if (ct < A.cols)
                *(uint4 *)(A.codes_t + (ct * blocks_t + (r0 >> 5)) * 16) = make_uint4(code[0], code[1], code[2], code[3]);
            __syncwarp();
        }
    }
}

// ------------------------------------------------------------------ the way back
// Eight elements per thread, U times; rows of the result begin on a boundary of eight elements' size.
template <class T, int U>
__global__ void __launch_bounds__(kQThreads) k_mx4_dequantise(const uint8_t *codes, const uint8_t *scales, const Divider pieces, uint32_t row0, int64_t rows,
                                                              int64_t cols, T *out, int64_t ld)
{
    grid_release();
    const uint32_t p0 = blockIdx.x * (uint32_t)(kQThreads * U) + threadIdx.x, tiles = (uint32_t)mx4_scale_tiles(cols);
    grid_wait();
    uint32_t w[U], row[U], at[U];
    uint8_t s[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t p = p0 + i * kQThreads;
        const uint32_t r = divide(p, pieces);
        row[i] = row0 + r;
        at[i] = p - r * pieces.by;
        if (row[i] < rows) {
            w[i] = __ldcs((const uint32_t *)codes + (uint64_t)row0 * pieces.by + p);
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
// ... begin anywhere: a thread takes those eight elements that fill an aligned piece of the result (`pieces` of them to a row at most), whose codes it cuts out
// of two words and whose scales are those of two blocks at most; pieces over a row's ends are stored element by element.  8192 x 1601 to
// fp32: a block per warp and an element per lane took 44 us, this takes 13.5 (4.4 TB/s); 8192 x 6400 to fp32 and bf16 58 and 41 (on aligned rows 38 and 22).
template <class T, int U>
__global__ void __launch_bounds__(kQThreads) k_mx4_dequantise_any(const uint8_t *codes, const uint8_t *scales, const Divider pieces, uint32_t row0, int64_t rows, int64_t cols,
                                                                  T *out, int64_t ld)
{
    grid_release();
    const uint32_t p0 = blockIdx.x * (uint32_t)(kQThreads * U) + threadIdx.x, tiles = (uint32_t)mx4_scale_tiles(cols), words = (uint32_t)mx4_blocks(cols) * 4;
    grid_wait();
    uint32_t w[U], a[U], b[U], row[U] = {};
    int64_t e[U] = {};
    auto full = [&](int i) { return row[i] < rows && e[i] >= 0 && e[i] + 8 <= cols; };
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t p = p0 + i * kQThreads;
        const uint32_t r = divide(p, pieces);
        row[i] = row0 + r;
        const uint32_t shift = (uint32_t)((uintptr_t)(out + (int64_t)row[i] * ld) / sizeof(T)) & 7u;
        e[i] = (int64_t)(p - r * pieces.by) * 8 - shift;
        if (full(i)) {
            w[i] = mx4_codes8((const uint32_t *)codes + (uint64_t)row[i] * words, (uint32_t)e[i]);
            a[i] = scales[mx4_scale_at(row[i], e[i] >> 5, tiles)];
            b[i] = scales[mx4_scale_at(row[i], (e[i] + 7) >> 5, tiles)];
        }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        T *o = out + (int64_t)row[i] * ld;
        if (full(i)) {
            float v[8];
            mx4_scaled8(w[i], (uint32_t)e[i], a[i], b[i], v);
            if constexpr (sizeof(T) == 4)
                store32(o + e[i], *(const uint32_t(*)[8])v);
            else
                __stcs((uint4 *)(o + e[i]), Vec16<T>::pack(v));
        } else if (row[i] < rows) {
            for (int64_t j = e[i] < 0 ? 0 : e[i]; j < e[i] + 8 && j < cols; ++j)
                o[j] = from_f32<T>(__fmul_rn(mx4_value(((const uint32_t *)codes)[(uint64_t)row[i] * words + (j >> 3)] >> (4 * (j & 7)) & 0xFu),
                                             mx4_pow(scales[mx4_scale_at(row[i], j >> 5, tiles)])));
        }
    }
}

template <class T>
static cudaError_t quantise(const T *x, const QArgs &A, bool stochastic, cudaStream_t s)
{
    // eight elements of a row in one or (fp32) one wide load
    const bool vec = (((uintptr_t)x | (A.rows > 1 ? (uint64_t)A.ld * sizeof(T) : 0u)) & (8 * sizeof(T) - 1)) == 0;
    auto by_draws = [&](auto f) {
        using Y = std::true_type;
        using N = std::false_type;
        return stochastic ? (A.drop.off ? f(Y(), Y()) : f(Y(), N())) : (A.drop.off ? f(N(), Y()) : f(N(), N()));
    };
    if (!A.codes_t) {
        // (blocks are counted in 32 bits: as many rows per launch as that takes)
        const int64_t padded = mx4_scale_tiles(A.cols) * 4, rows = (A.rows + 127) / 128 * 128, most = ((1ll << 32) - 4096) / padded;
        cudaError_t e = cudaSuccess;
        for (int64_t r0 = 0; r0 < rows && e == cudaSuccess; r0 += most) {
            const int64_t units = std::min(most, rows - r0) * padded;
            e = by_draws([&](auto st, auto dr) {
                constexpr bool ST = decltype(st)::value, DR = decltype(dr)::value;
                auto go = [&](auto vc, auto ln) {
                    constexpr int LANES = decltype(ln)::value, PER = kQThreads / LANES;
                    return launch(k_mx4_rows<T, decltype(vc)::value, ST, DR, LANES>, dim3((unsigned)((units + PER - 1) / PER)), kQThreads, 0, s, x, A,
                                  divider((uint32_t)padded), (uint32_t)r0, (uint32_t)units);
                };
                using Few = std::integral_constant<int, 4>;
                using Many = std::integral_constant<int, sizeof(T) == 4 && !ST && !DR ? 2 : 1>;
                if (!vec)
                    return go(std::false_type(), Few());
                return units < (int64_t)kQThreads / 4 * kPlanSMs * 16 ? go(std::true_type(), Few()) : go(std::true_type(), Many());
            });
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
    const bool vec = (((uintptr_t)out | (rows > 1 ? (uint64_t)ld * sizeof(T) : 0u)) & (8 * sizeof(T) - 1)) == 0;
    // (pieces are counted in 32 bits: as many rows per launch as that takes)
    const int64_t per_row = vec ? mx4_blocks(cols) * 4 : std::max<int64_t>(2, (cols + 14) / 8), most = ((1ll << 32) - 4096) / per_row;
    cudaError_t e = cudaSuccess;
    for (int64_t r0 = 0; r0 < rows && e == cudaSuccess; r0 += most) {
        const int64_t end = std::min(rows, r0 + most), pieces = (end - r0) * per_row;
        auto go = [&](auto un) {
            constexpr int U = decltype(un)::value, PER = kQThreads * U;
            return launch(vec ? k_mx4_dequantise<T, U> : k_mx4_dequantise_any<T, U>, dim3((unsigned)((pieces + PER - 1) / PER)), kQThreads, 0, s, codes, scales,
                          divider((uint32_t)per_row), (uint32_t)r0, end, cols, out, ld);
        };
        e = pieces >= (int64_t)kQThreads * 4 * kPlanSMs * 8 ? go(std::integral_constant<int, 4>()) : go(std::integral_constant<int, 1>());
    }
    return e;
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
