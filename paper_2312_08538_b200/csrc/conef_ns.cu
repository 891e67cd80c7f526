// A matrix brought near the orthogonal one next to it by Newton-Schulz products (as the Muon optimiser does with its updates): X0 = G / |G|, the
// Frobenius norm, then so many times X <- (a + b A + c A^2) X with A = X X^T, X having no more rows than columns (else it is G's transpose).
// For X0 = U S V^T that is U f(f(..S)) V^T with f(s) = a s + b s^3 + c s^5.
//
// Each time f raises small singular values by a (3.4 times; five times over 480), and with them what a rounding put next to them.  With operands of 16
// bits an update whose spectrum falls off by two decades is off by 1e-2 to 5e-2 (bf16) or 1e-3 to 6e-3 (fp16) of its size, where rounding the result
// to bf16 loses 1.7e-3.  So:
//  - X is kept as two fp16, hi + lo, under a power of two that keeps it below fp16's largest (bounds of X, A and C follow from the coefficients on the
//    host), which is 22 bits; a X is added in fp32 and only C X, C = b A + c A^2, is a product: its share of a rounding's noise in the directions
//    of small singular values is as small as A has them.
//  - A and C are kept likewise, and a product is the sum of hi hi, hi lo and lo hi in one set of fp32 sums on the tensor cores: as exact as 32-bit
//    arithmetic at three times 16-bit's cost, not at the 20 times that 32-bit units take.  (hi hi alone in products of the first steps leaves an error of 1e-3 in five
//    steps, 4e-3 in twenty, ahead of the rounding, whose own is 1.7e-3 in bf16 and 2e-4 in fp16: no product does so.  It would take 257 us for 1600 x 1600 in place of 350, and
//    764 for 2 x 6400 x 1600 in place of 1436.)
//
// Per step three launches: A (symmetric: tiles on and above the diagonal, stored twice), C (likewise, A added on the way out), C X (a X added).
#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "conef_common.cuh"
#include "conef_f8.cuh"
#include "conef_mm.cuh"

namespace conef {

// A stack of n x m matrices kept as hi + lo, rows `pitch` elements apart
struct Split {
    __half *hi, *lo;
    int64_t rows, cols, pitch;
};
__device__ __forceinline__ void split(float v, __half &hi, __half &lo)
{
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}

// ------------------------------------------------------------------ the norm and X0
constexpr int kNsParts = 512;   // partial sums per matrix at most
struct NsIn {
    const void *x;
    int64_t rows, cols, ld, stride;   // as the caller has it
    double *parts;                    // kNsParts per matrix
    uint32_t n_parts;
};
// Sums of squares of a matrix's rows, part by part, in 64 bits (VEC: 16 bytes of a row at a time)
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_ns_squares(const __grid_constant__ NsIn A)
{
    constexpr int N = VEC ? Vec16<T>::N : 1;
    __shared__ double part[8];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const T *const x = (const T *)A.x + blockIdx.y * A.stride;
    grid_wait();
    double sum = 0;
    auto add = [&](const float *v) {
#pragma unroll
        for (int q = 0; q < N; ++q)
            sum = __fma_rn((double)v[q], (double)v[q], sum);
    };
    // N elements of a row's, or fewer at its end
    auto piece = [&](const T *p, int64_t have) {
        float v[N];
        if (VEC && have >= N) {
            if constexpr (VEC)
                Vec16<T>::unpack(*(const uint4 *)p, v);
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q)
                v[q] = q < have ? to_f32(p[q]) : 0.f;
        }
        add(v);
    };
    if (VEC && A.ld == A.cols) {   // one array: four pieces of each thread's on their way
        const int64_t all = A.rows * A.cols, step = (int64_t)A.n_parts * 256 * N;
        int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N;
        for (; at + 3 * step + N <= all; at += 4 * step) {
            uint4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = *(const uint4 *)(x + at + i * step);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[N];
                if constexpr (VEC)
                    Vec16<T>::unpack(w[i], v);
                add(v);
            }
        }
        for (; at < all; at += step)
            piece(x + at, all - at);
    } else {
        for (int64_t row = (int64_t)blockIdx.x * 8 + warp; row < A.rows; row += (int64_t)A.n_parts * 8)
#pragma unroll 4
            for (int64_t c = (int64_t)lane * N; c < A.cols; c += 32 * N)
                piece(x + row * A.ld + c, A.cols - c);
    }
#pragma unroll
    for (int o = 16; o; o /= 2)
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0)
        part[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i)
            sum += part[i];
        A.parts[blockIdx.y * kNsParts + blockIdx.x] = sum;
    }
}
// X0 times a power of two, in tiles of 64 x 64 (FLIP: X is the transpose).  VEC: a thread reads 16 bytes.
template <class T, bool FLIP, bool VEC>
__global__ void __launch_bounds__(256) k_ns_start(const __grid_constant__ NsIn A, const Split X, uint32_t tiles_c, double scale)
{
    __shared__ float tile[FLIP ? 64 : 1][65];
    __shared__ double part[8];
    __shared__ float factor[2];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    const int64_t r0 = (int64_t)tr * 64, c0 = (int64_t)tc * 64, batch = blockIdx.y;
    const T *const x = (const T *)A.x + batch * A.stride;
    __half *const hi = X.hi + batch * X.rows * X.pitch, *const lo = X.lo + batch * X.rows * X.pitch;
    grid_wait();
    // a thread's elements: 16 of a row
    const int r = threadIdx.x >> 2, c = (threadIdx.x & 3) * 16;
    const bool there = r0 + r < A.rows;
    const T *const from = x + (r0 + r) * A.ld + c0 + c;
    float v[16];
    if (VEC && there && c0 + c + 16 <= A.cols) {
#pragma unroll
        for (int q = 0; q < 16; q += Vec16<T>::N)
            Vec16<T>::unpack(*(const uint4 *)(from + q), *(float(*)[Vec16<T>::N])(v + q));
    } else {
#pragma unroll
        for (int q = 0; q < 16; ++q)
            v[q] = there && c0 + c + q < A.cols ? to_f32(from[q]) : 0.f;
    }
    double sum = 0;
    for (uint32_t i = threadIdx.x; i < A.n_parts; i += 256)
        sum += A.parts[batch * kNsParts + i];
#pragma unroll
    for (int o = 16; o; o /= 2)
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0)
        part[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i)
            sum += part[i];
        const double by = sum == 0 ? 0 : scale / sqrt(sum);   // (a matrix of zeros stays one)
        // (in two factors, the first a power of two: either alone, times elements of any size, stays in range)
        const double first = sum == 0 || !(by > 0) ? 1.0 : ldexp(1.0, ilogb(by) / 2);
        factor[0] = (float)first, factor[1] = (float)(by / first);
    }
    __syncthreads();
    const float f0 = factor[0], f1 = factor[1];
#pragma unroll
    for (int q = 0; q < 16; ++q)
        v[q] = __fmul_rn(__fmul_rn(v[q], f0), f1);
    if constexpr (FLIP) {
#pragma unroll
        for (int q = 0; q < 16; ++q)
            tile[r][c + q] = v[q];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 16; ++q)
            v[q] = tile[c + q][r];   // (a row of X)
    }
    const int64_t row = (FLIP ? c0 : r0) + r, col = (FLIP ? r0 : c0) + c;
    if (row < X.rows && col < X.cols) {   // (rows are padded to 64 elements, which nothing reads)
        __half h[16], l[16];
#pragma unroll
        for (int q = 0; q < 16; ++q)
            split(v[q], h[q], l[q]);
        store32_keep(hi + row * X.pitch + col, *(const uint32_t(*)[8])h);
        store32_keep(lo + row * X.pitch + col, *(const uint32_t(*)[8])l);
    }
}

// ------------------------------------------------------------------ products
// D = f_sum (L R) + f_add E for stacks of matrices; R along k like L (A = X X^T, A A), or (CROSS) as it is multiplied, along D's columns (C X).
// The kernel is that of conef_mm.cuh with another ring and another way out.  A stage has 64 elements of k of L and R, their hi parts or their lo parts; two in a row
// are three products.  What leaves is split again, or rounded to the result; it goes through shared memory
// and tiled copies, and so does E: a row to a lane, straight to memory, 16 accesses to 32 lines each made 12000 cycles of a tile of 256 x 256, whose
// products hi hi take 13000 at k = 1600.
struct NsArgs {
    void *result;                // the last product's, instead of the outputs
    int64_t result_ld, result_stride;
    float f_sum, f_add;
    uint32_t n, m, k;            // of D = n x m
    uint32_t k_steps, stages_k, per_matrix, tiles_m, n_tiles;
    uint32_t tiles_wide;            // (symmetric) tiles are 256 x 128
    uint32_t symmetric, flip, dtype;
    uint32_t bn, stage_bytes, stages;   // columns of a tile; the ring
    uint32_t add;                   // E
    uint32_t wide;                  // the result goes by tiled copies
    uint64_t limit, sums_limit;
    uint32_t loads[2];
    uint32_t split, split_stages;   // CTAs of a cluster that share a tile's k, and stages of each (an even number; the last one's may be fewer)
    __half *hi, *lo;                // ... which store their outputs themselves
    int64_t out_pitch, out_stride;
};
struct NsMaps {
    CUtensorMap lh, ll, rh, rl;     // tiles of 64 elements by 128 rows (CROSS, R: 64)
    CUtensorMap eh, el, oh, ol;     // of 64 by 32: E, outputs or (oh) the result
    CUtensorMap th, tl;             // of 32 by 64: the outputs' or the result's transpose
};
constexpr uint32_t kNsLeft = 128 * 128, kNsStaging = 4096;   // bytes: 128 rows of L; a warp's 32 x 64 elements of what leaves
// ... of R: 128 per row, or (CROSS) for each of k's 64, columns of 64 elements
__host__ __device__ inline uint32_t ns_right(uint32_t bn, bool pair, bool cross)
{
    const uint32_t rows = pair ? bn / 2 : bn;
    return cross ? (rows + 63) / 64 * 8192 : rows * 128;
}
struct NsShared {
    MmShared mm;
    uint64_t added[kMmEpilogue];
};
struct NsTile {
    uint32_t batch, i, j;
};
__device__ __forceinline__ NsTile ns_tile(const NsArgs &P, uint32_t tile)
{
    NsTile t;
    t.batch = tile / P.per_matrix;
    uint32_t in = tile - t.batch * P.per_matrix;
    if (P.symmetric && P.tiles_wide) {   // tiles twice as high as wide on and above the diagonal: columns 2 p and 2 p + 1 have p + 1 each
        uint32_t p = (uint32_t)((sqrtf(4.f * (float)in + 1.f) - 1.f) * 0.5f);
        while (p * (p + 1) > in)
            --p;
        while ((p + 1) * (p + 2) <= in)
            ++p;
        in -= p * (p + 1);
        const uint32_t second = in > p ? 1u : 0u;
        t.j = 2 * p + second, t.i = in - second * (p + 1);
    } else if (P.symmetric) {   // columns of a triangle
        uint32_t j = (uint32_t)((sqrtf(8.f * (float)in + 1.f) - 1.f) * 0.5f);
        while (j * (j + 1) / 2 > in)
            --j;
        while ((j + 1) * (j + 2) / 2 <= in)
            ++j;
        t.j = j, t.i = in - j * (j + 1) / 2;
    } else {
        t.j = in / P.tiles_m, t.i = in - t.j * P.tiles_m;
    }
    return t;
}
// a lane's row of 64 elements (32 words) in a warp's staging memory, 16-byte pieces exchanged as tiled copies do
__device__ __forceinline__ void staging_read(uint32_t staging, int lane, uint32_t (&w)[32])
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                     : "r"(staging + lane * 128 + ((i ^ (lane & 7)) << 4))
                     : "memory");
}
// Tiles of it to memory, as they are and (mirror) transposed: 64 rows of 32 elements.  `again`: an earlier store reads that memory, perhaps still.
template <bool TURNED>
__device__ __forceinline__ void staging_store(uint32_t staging, bool again, int lane, const uint32_t (&w)[32], const void *map, uint32_t x, uint32_t y, uint32_t z)
{
    if (again) {
        if (lane == 0)
            tc::store_wait_read();
        __syncwarp();
    }
    if constexpr (TURNED) {
        // two rows of a column to a lane: even lanes take even columns, odd ones odd columns, of both rows
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, w[i], 1), c = 2 * i + (lane & 1);
            const uint32_t both = lane & 1 ? __byte_perm(other, w[i], 0x7632) : __byte_perm(w[i], other, 0x5410);
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(staging + c * 64 + (lane & ~1) * 2), "r"(both) : "memory");
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(staging + lane * 128 + ((i ^ (lane & 7)) << 4)), "r"(w[4 * i]), "r"(w[4 * i + 1]), "r"(w[4 * i + 2]),
                         "r"(w[4 * i + 3])
                         : "memory");
    }
    tc::store_fence();
    __syncwarp();
    if (lane == 0)
        tc::tile_store3(map, staging, x, y, z);
}
// 64 columns of a lane's row of the result, two to a word, element by element
__device__ __forceinline__ void ns_result(const NsArgs &P, uint32_t batch, uint32_t row, uint32_t col, const uint32_t (&w)[32])
{
    if (row >= P.n)
        return;
    uint16_t *const out = (uint16_t *)P.result + (int64_t)batch * P.result_stride;
#pragma unroll
    for (int i = 0; i < 64; ++i)
        if (col + i < P.m)
            out[P.flip ? (int64_t)(col + i) * P.result_ld + row : (int64_t)row * P.result_ld + col + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
}

// The sums of a tile whose k the CTAs of a cluster share (conef_mm.cuh): each CTA adds up its columns, four to a thread, in the CTAs' order, and stores them, twice off the diagonal
template <int SPLIT>
__device__ __forceinline__ void ns_join(const NsArgs &P, const float *sums, const int &dead, const NsTile &t, uint32_t part)
{
    constexpr uint32_t width = 128 / SPLIT, quads = width / 4;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < SPLIT; ++i)
        any |= tc::load_at(tc::address_in(&dead, i));
    __half *const hi = P.hi + (int64_t)t.batch * P.out_stride, *const lo = P.lo + (int64_t)t.batch * P.out_stride;
    for (uint32_t e = threadIdx.x; e < 128 * quads; e += kMmThreads) {
        const uint32_t r = e / quads, c = part * width + e % quads * 4, row = t.i * 128 + r, col = t.j * 128 + c;
        if (row >= P.n || col >= P.m)
            continue;
        float4 v[SPLIT];
#pragma unroll
        for (int i = 0; i < SPLIT; ++i)
            v[i] = tc::load_at4(tc::address_in(sums + r * 132 + c, i));
        float f[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
        for (int i = 1; i < SPLIT; ++i)
            f[0] = __fadd_rn(f[0], v[i].x), f[1] = __fadd_rn(f[1], v[i].y), f[2] = __fadd_rn(f[2], v[i].z), f[3] = __fadd_rn(f[3], v[i].w);
        __half h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            split(any ? __uint_as_float(0x7FFFFFFFu) : __fmul_rn(f[i], P.f_sum), h[i], l[i]);
        const int64_t at = (int64_t)row * P.out_pitch + col;   // (rows are padded to 64 elements)
        *(uint2 *)(hi + at) = *(const uint2 *)h;
        *(uint2 *)(lo + at) = *(const uint2 *)l;
        if (t.i != t.j)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (col + i < P.m) {
                    const int64_t turned = (int64_t)(col + i) * P.out_pitch + row;
                    hi[turned] = h[i];
                    lo[turned] = l[i];
                }
    }
}

// A tile is 128 x 128, or of a pair of CTAs 256 by 128, 192 (not symmetric) or 256: with 128 x 128 a product reads as many bytes of shared memory per cycle as there
// are, so that the copies into it have to wait; a pair's CTA has half of R for as many rows of L.
template <bool PAIR, bool CROSS, bool SPLIT>
__global__ void __launch_bounds__(kMmThreads, 1) k_ns_product(const __grid_constant__ NsMaps maps, const __grid_constant__ NsArgs P)
{
    constexpr uint32_t BM = PAIR ? 256 : 128;
    const uint32_t BN = P.bn, right = ns_right(BN, PAIR, CROSS);
    extern __shared__ __align__(1024) uint8_t mm_smem[];
    __shared__ NsShared N;
    MmShared &S = N.mm;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? blockIdx.x & 1u : 0u, first = PAIR ? blockIdx.x / 2 : SPLIT ? blockIdx.x / P.split : blockIdx.x, step = PAIR ? gridDim.x / 2 : gridDim.x;
    const uint32_t part = SPLIT ? blockIdx.x - first * P.split : 0u, ks0 = SPLIT ? part * P.split_stages : 0u, ks1 = SPLIT ? min(ks0 + P.split_stages, P.stages_k) : P.stages_k;
    uint8_t *const ring = mm_smem + ((1024u - (tc::saddr(mm_smem) & 1023u)) & 1023u);
    const tc::Waits waits = {&S.dead, PAIR ? tc::address_in(&S.dead, rank ^ 1u) : 0u, &g_mm_ran_out};
    if (warp == 1 && lane < (int)(sizeof maps / sizeof maps.lh))
        tc::prefetch_map(&maps.lh + lane);
    if (warp == 0) {
        tc::tmem_alloc<PAIR>(&S.tmem, kMmColumns);
        if (lane == 0) {
            for (int i = 0; i < kMmMaxStages; ++i) {
                tc::bar_init(&S.full[i], 1);
                tc::bar_init(&S.empty[i], 1);
            }
            for (int i = 0; i < 2; ++i) {
                tc::bar_init(&S.sums[i], 1);
                tc::bar_init(&S.taken[i], BN / 16 * (PAIR ? 2 : 1));
            }
            for (int i = 0; i < kMmEpilogue; ++i)
                tc::bar_init(&N.added[i], 1);
            tc::bar_init(&S.drain, 1);
            S.dead = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        tc::fence_before();
    }
    __syncthreads();
    if (PAIR)
        tc::cluster_sync();
    tc::fence_after();
    grid_release();
    grid_wait();
    asm volatile("fence.proxy.async;" ::: "memory");   // (what the launch before stored, ordinary stores, is read by copies)

    auto load = [&](uint32_t s, uint32_t ks, const NsTile &t) {
        const uint32_t st = tc::saddr(ring) + s * P.stage_bytes, k0 = ks / 2 * 64, i0 = t.i * BM + rank * 128, j0 = t.j * BN + rank * (BN / 2);
        const bool low = ks & 1;
        const void *const l = low ? &maps.ll : &maps.lh, *const r = low ? &maps.rl : &maps.rh;
        auto part = [&](uint32_t dst, const void *map, uint32_t x, uint32_t y) {
            if constexpr (PAIR)
                tc::tile_load3_pair(dst, map, x, y, t.batch, tc::leaders(&S.full[s]));
            else
                tc::tile_load3(dst, map, x, y, t.batch, &S.full[s]);
        };
        if (rank == 0)
            tc::bar_expect(&S.full[s], (PAIR ? 2 : 1) * (kNsLeft + right));
        part(st, l, k0, i0);
        if constexpr (CROSS) {
            part(st + kNsLeft, r, j0, k0);
            if (right > 8192)
                part(st + kNsLeft + 8192, r, j0 + 64, k0);
        } else {
            part(st + kNsLeft, r, k0, j0);
        }
    };
    uint32_t armed = 0;
    if (warp == kMmEpilogue) {
        uint32_t s = 0, phase = 0;
        bool ok = true;
        for (uint32_t tile = first; ok && tile < P.n_tiles; tile += step) {
            const NsTile t = ns_tile(P, tile);
            for (uint32_t ks = ks0; ks < ks1; ++ks) {
                if (!(ok = armed < P.loads[rank] && tc::bar_wait(&S.empty[s], phase ^ 1u, waits, P.limit)))
                    break;
                if (tc::elect())
                    load(s, ks, t);
                ++armed;
                if (++s == P.stages)
                    s = 0, phase ^= 1u;
            }
        }
        if (lane == 0)
            S.armed = armed;
        __syncwarp();
    } else if (warp == kMmEpilogue + 1) {
        const uint32_t instruction = tc::f16_instruction<PAIR, CROSS>(BN);
        constexpr uint32_t k_step = CROSS ? 128 : 2;   // (16 of k: 32 bytes of a row, or two groups of eight rows)
        const uint32_t a0 = tc::desc_low(ring), b0 = CROSS ? tc::desc_low_across(tc::saddr(ring) + kNsLeft, 8192) : a0 + kNsLeft / 16, step16 = P.stage_bytes / 16;
        uint32_t s = 0, phase = 0, set = 0, turn = 0;
        bool ok = true;
        for (uint32_t tile = rank ? P.n_tiles : first; ok && tile < P.n_tiles; tile += step) {
            const uint32_t d = set * BN;
            if (!(ok = tc::bar_wait(&S.taken[set], turn ^ 1u, waits, P.limit)))
                break;
            tc::fence_after();
            uint32_t high = 0;   // the stage before, where that has the hi parts
            for (uint32_t ks = ks0; ks < ks1; ++ks) {
                if (!(ok = tc::bar_wait(&S.full[s], phase, waits, P.limit)))
                    break;
                tc::fence_after();
                if (tc::elect()) {
                    const uint32_t a = a0 + s * step16, b = b0 + s * step16;
                    const uint32_t steps = P.k_steps - ks / 2 * 4u;
                    if (!(ks & 1)) {
#pragma unroll
                        for (uint32_t t = 0; t < 4; ++t)
                            if (t < steps)
                                tc::f16_product<PAIR>(d, a + 2 * t, b + k_step * t, instruction, ks - ks0 + t);
                    } else {
                        const uint32_t ah = a0 + high * step16, bh = b0 + high * step16;
#pragma unroll
                        for (uint32_t t = 0; t < 4; ++t)
                            if (t < steps) {
                                tc::f16_product<PAIR>(d, ah + 2 * t, b + k_step * t, instruction, 1);
                                tc::f16_product<PAIR>(d, a + 2 * t, bh + k_step * t, instruction, 1);
                            }
                        tc::commit<PAIR>(&S.empty[high]);
                        tc::commit<PAIR>(&S.empty[s]);
                    }
                }
                high = s;
                if (++s == P.stages)
                    s = 0, phase ^= 1u;
            }
            if (ok && tc::elect())
                tc::commit<PAIR>(&S.sums[set]);
            if (++set == 2)
                set = 0, turn ^= 1u;
        }
        __syncwarp();
    } else if (SPLIT) {
        const uint32_t c0 = (uint32_t)(warp >> 2) * 64;
        if (c0 < BN && tc::bar_wait(&S.sums[0], 0, waits, P.sums_limit)) {   // (where the wait runs out, `dead` tells all CTAs)
            tc::fence_after();
            uint4 *const to = (uint4 *)ring + (((warp & 3) * 32 + lane) * 132 + c0) / 4;
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                uint32_t v[16];
                tc::tmem_load16(((uint32_t)(warp & 3) << 21) + c0 + q * 16, v);
                tc::tmem_load_wait();
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    to[q * 4 + i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
        }
        __syncwarp();
    } else {
        // Sums of 32 rows (a lane each) and 64 columns.  E comes while they are formed.
        uint32_t set = 0, turn = 0, asked = 0;
        bool ok = true;
        const uint32_t c0 = (uint32_t)(warp >> 2) * 64, staging = tc::saddr(ring) + P.stages * P.stage_bytes + warp * kNsStaging;
        for (uint32_t tile = c0 < BN ? first : P.n_tiles; tile < P.n_tiles; tile += step) {
            const NsTile t = ns_tile(P, tile);
            const uint32_t row0 = t.i * BM + rank * 128 + (warp & 3) * 32, row = row0 + lane, col = t.j * BN + c0;
            const bool there = row0 < P.n && col < P.m;
            uint32_t h[32] = {}, l[32] = {};
            auto fetch = [&](const void *map, uint32_t (&w)[32]) {
                if (lane == 0) {
                    tc::store_wait_read();
                    tc::bar_expect(&N.added[warp], kNsStaging);
                    tc::tile_load3(staging, map, col, row0, t.batch, &N.added[warp]);
                }
                __syncwarp();
                if (!tc::bar_wait(&N.added[warp], asked & 1u, waits, P.limit)) {   // (it comes all the same, and before this block ends)
                    ok = false;
                    tc::bar_drain(&N.added[warp], asked & 1u, tc::nanoseconds());
                }
                ++asked;
                staging_read(staging, lane, w);
                tc::store_fence();   // (the reads come before the next copy into that memory, however long the queue of other warps' accesses)
                __syncwarp();
            };
            if (P.add && there) {
                fetch(&maps.eh, h);
                fetch(&maps.el, l);
            }
            ok = ok && tc::bar_wait(&S.sums[set], turn, waits, P.sums_limit);
            if (ok)
                tc::fence_after();
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                uint32_t v[16];
                if (ok) {
                    tc::tmem_load16(((uint32_t)(warp & 3) << 21) + set * BN + c0 + q * 16, v);
                    tc::tmem_load_wait();
                } else {   // a wait ran out: what was not computed is NaN
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        v[i] = 0x7FFFFFFFu;
                }
                float f[16];
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    f[i] = __fmul_rn(__uint_as_float(v[i]), P.f_sum);
                if (P.add) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float2 a = __half22float2(*(const __half2 *)&h[8 * q + i]);
                        const float2 b = __half22float2(*(const __half2 *)&l[8 * q + i]);
                        a.x = __fadd_rn(a.x, b.x), a.y = __fadd_rn(a.y, b.y);
                        f[2 * i] = __fmaf_rn(a.x, P.f_add, f[2 * i]), f[2 * i + 1] = __fmaf_rn(a.y, P.f_add, f[2 * i + 1]);
                    }
                }
                if (P.result && P.dtype == CONEF_BF16) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        h[8 * q + i] = Vec16<__nv_bfloat16>::pack2(f[2 * i], f[2 * i + 1]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        h[8 * q + i] = Vec16<__half>::pack2(f[2 * i], f[2 * i + 1]);
                    if (!P.result) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float2 r = __half22float2(*(const __half2 *)&h[8 * q + i]);
                            l[8 * q + i] = Vec16<__half>::pack2(__fsub_rn(f[2 * i], r.x), __fsub_rn(f[2 * i + 1], r.y));
                        }
                    }
                }
            }
            if (ok) {
                tc::fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR)
                        tc::bar_arrive_at(tc::leaders(&S.taken[set]));
                    else
                        tc::bar_arrive(&S.taken[set]);
                }
            }
            if (++set == 2)
                set = 0, turn ^= 1u;
            if (!there)
                continue;
            if (P.result) {
                if (!P.wide)
                    ns_result(P, t.batch, row, col, h);
                else if (P.flip)
                    staging_store<true>(staging, true, lane, h, &maps.th, row0, col, t.batch);
                else
                    staging_store<false>(staging, true, lane, h, &maps.oh, col, row0, t.batch);
                continue;
            }
            // Up to four stores.  Behind the last tile's sums the ring is free, and they need not wait for one another.
            const uint32_t more = ok && tile + step >= P.n_tiles ? min(3u, P.stages * P.stage_bytes / (BN / 16 * kNsStaging)) : 0u;
            const bool mirror = P.symmetric && t.i != (P.tiles_wide ? t.j / 2 : t.j);
            auto place = [&](uint32_t n) { return n && n <= more ? tc::saddr(ring) + (warp * more + n - 1) * kNsStaging : staging; };
            auto again = [&](uint32_t n) { return n == 0 || n > more; };
            staging_store<false>(staging, true, lane, h, &maps.oh, col, row0, t.batch);
            staging_store<false>(place(1), again(1), lane, l, &maps.ol, col, row0, t.batch);
            if (mirror) {
                staging_store<true>(place(2), again(2), lane, h, &maps.th, row0, col, t.batch);
                staging_store<true>(place(3), again(3), lane, l, &maps.tl, row0, col, t.batch);
            }
        }
        if (lane == 0)
            tc::store_wait_read();   // (what the launch behind waits for is the whole grid's end)
        __syncwarp();
    }
    tc::fence_before();
    __syncthreads();
    if (PAIR || SPLIT)
        tc::cluster_sync();   // neither CTA tells a barrier of one that has ended
    tc::fence_after();
    if constexpr (SPLIT) {
        const NsTile t = ns_tile(P, first);
        if (P.split == 2)
            ns_join<2>(P, (const float *)ring, S.dead, t, part);
        else if (P.split == 4)
            ns_join<4>(P, (const float *)ring, S.dead, t, part);
        else
            ns_join<8>(P, (const float *)ring, S.dead, t, part);
        __syncthreads();
        tc::cluster_sync();   // (all have read)
    }
    if (*waits.dead) {   // as in conef_mm.cuh: what is in flight ends before shared and tensor memory are given back
        const uint64_t t0 = tc::nanoseconds();
        if (warp == kMmEpilogue) {
            const uint32_t all = PAIR ? max(armed, tc::load_at(tc::address_in(&S.armed, rank ^ 1u))) : armed;
            for (; armed < all; ++armed) {
                const uint32_t nth = armed / P.stages_k;
                const NsTile t = ns_tile(P, first + nth * step);
                if (tc::elect())
                    load(armed % P.stages, armed - nth * P.stages_k, t);
                __syncwarp();
            }
            if (rank == 0)
                for (uint32_t i = 0; i < P.stages && i < all; ++i)
                    tc::bar_drain(&S.full[(all - 1 - i) % P.stages], ((all - 1 - i) / P.stages) & 1u, t0);
        } else if (warp == kMmEpilogue + 1 && rank == 0) {
            if (tc::elect())
                tc::commit<PAIR>(&S.drain);
            __syncwarp();
            tc::bar_drain(&S.drain, 0, t0);
        }
        __syncthreads();
        if (PAIR)
            tc::cluster_sync();
        tc::fence_after();
    }
    if (warp == 0)
        tc::tmem_free<PAIR>(0, kMmColumns);
}

// ------------------------------------------------------------------ host

// tiles of `width` elements (64, or 32 unpermuted) by `box` rows of a stack of matrices of 16-bit elements, `ld` and `stride` apart
static bool encode_stack(CUtensorMap *map, const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t stride, int64_t batch, uint32_t width, uint32_t box)
{
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)batch}, strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)stride * 2};
    const cuuint32_t tile[3] = {width, box, 1}, steps[3] = {1, 1, 1};
    return encode_tiled() && encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, (void *)p, dims, strides, tile, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                            width == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
static bool encode_split(CUtensorMap *map, const __half *p, const Split &s, int64_t batch, uint32_t width, uint32_t box)
{
    return encode_stack(map, p, s.rows, s.cols, s.pitch, s.pitch * s.rows, batch, width, box);
}

// The tile whose waves over the SMs take least.  Nanoseconds per wave: of 64 elements along k, and of what does not depend on k, from 1600 x 1600 and
// 2 x 1600 x 6400.  At full rate the first would be 400, 400, 600, 800.  All of five steps, us, with the choice, which is made for each of a step's three products, and with tiles
// of one kind throughout (X X^T and A A by pairs of 128 columns in place of 192):
//   256 x 512            140   146   145   152   197        1024 x 4096       384   442   389   435   585        1600 x 6400       761   887   762   803  1093
//   512 x 512            174   178   178   191   257        1600 x 1600       350   409   365   351   495        2 x 6400 x 1600  1435  1623  1507  1518  1435
//   768 x 768            199   212   209   222   312        2048 x 2048       449   508   447   518   627        4 x 1600 x 1600   933  1015   935   964  1014
//   12 x 768 x 768       404   416   387   387   419        3 x 700 x 2500    425   441   403   415   582
// (Where it misses the fastest, in stacks of small matrices, that costs 4 and 5 %.)
struct NsTiles {
    bool pair;
    uint32_t bn;
    int step, fixed;
    uint32_t split;   // CTAs that share a tile along k
};
static NsTiles ns_tiles(int64_t n, int64_t m, int64_t k, int64_t batch, bool symmetric, bool splits)
{
    static const NsTiles kinds[] = {{false, 128, 740, 4500, 1}, {true, 128, 600, 5500, 1}, {true, 192, 880, 6000, 1}, {true, 256, 980, 7000, 1}};
    NsTiles best = {};
    int64_t least = -1;
    for (const NsTiles &c : kinds) {
        if (symmetric && c.bn == 192)
            continue;
        const int64_t high = c.pair ? 256 : 128, ti = (n + high - 1) / high, tj = (m + c.bn - 1) / c.bn, sets = c.pair ? kPlanSMs / 2 : kPlanSMs;
        int64_t tiles = ti * tj;
        if (symmetric)
            tiles = c.bn == high ? ti * (ti + 1) / 2 : tj / 2 * (tj / 2 + 1) + (tj & 1 ? tj / 2 + 1 : 0);
        // (what a tile leaves goes out while the next one's sums are formed)
        const int64_t waves = (tiles * batch + sets - 1) / sets, cost = waves * ((k + 63) / 64) * c.step + c.fixed;
        if (least < 0 || cost < least)
            best = c, least = cost;
    }
    // A of X with few rows: clusters, as many as run at once (conef_mm.cuh), which take 3.5 us more to begin, to join and to end.  All of five steps without and with: 64 x 4096
    // 240 and 115 us, 100 x 1000 151 and 122.
    for (uint32_t split = 2; splits && split <= 8; split *= 2) {
        const int64_t ti = (n + 127) / 128, tiles = ti * (ti + 1) / 2 * batch, stages = (k + 63) / 64, each = (stages + split - 1) / split;
        const int64_t cost = each * kinds[0].step + kinds[0].fixed + 3500;
        if (tiles <= (split == 2 ? 72 : split == 4 ? 32 : 14) && each * (split - 1) < stages && cost < least)
            best = kinds[0], best.split = split, least = cost;
    }
    return best;
}

// E, out: NULL without; P has the factors, the parts and the result
template <bool CROSS>
static cudaError_t ns_product(const Split &L, const Split &R, const Split *E, const Split *out, int64_t batch, NsArgs P, cudaStream_t s)
{
    P.n = (uint32_t)L.rows;
    P.m = (uint32_t)(CROSS ? R.cols : R.rows);
    P.k = (uint32_t)L.cols;
    P.k_steps = (P.k + 15) / 16;
    P.stages_k = (P.k + 63) / 64 * 2;
    const NsTiles kind = ns_tiles(P.n, P.m, P.k, batch, P.symmetric, !CROSS && !E);
    const bool pair = kind.pair;
    const uint32_t high = pair ? 256 : 128;
    P.bn = kind.bn;
    P.tiles_wide = pair && P.bn == 128;
    P.tiles_m = (P.n + high - 1) / high;
    P.add = E != nullptr;
    const int64_t tj = (P.m + P.bn - 1) / P.bn;
    const int64_t per = !P.symmetric ? P.tiles_m * tj : P.tiles_wide ? tj / 2 * (tj / 2 + 1) + (tj & 1 ? tj / 2 + 1 : 0) : (int64_t)P.tiles_m * (P.tiles_m + 1) / 2;
    const uint32_t staging = P.bn / 16 * kNsStaging;
    P.stage_bytes = kNsLeft + ns_right(P.bn, pair, CROSS);
    P.stages = std::min<uint32_t>(kMmMaxStages, (kMmSmem - 1024 - staging) / P.stage_bytes);
    if (per * batch >= (1ll << 31))
        return cudaErrorInvalidValue;
    P.per_matrix = (uint32_t)per;
    P.n_tiles = (uint32_t)(per * batch);
    P.limit = (uint64_t)mm_limit.nanoseconds.load();
    P.sums_limit = P.limit + 4096ull * P.stages_k;
    P.loads[0] = mm_limit.loads[0].load();
    P.loads[1] = mm_limit.loads[1].load();
    P.split = kind.split;
    const uint32_t stages = (P.k + 63) / 64;
    P.split_stages = (stages + P.split - 1) / P.split * 2;
    if (P.split > 1)
        P.hi = out->hi, P.lo = out->lo, P.out_pitch = out->pitch, P.out_stride = out->pitch * out->rows;
    NsMaps maps = {};
    const uint32_t r_box = CROSS ? 64 : pair ? P.bn / 2 : P.bn;
    bool ok = encode_split(&maps.lh, L.hi, L, batch, 64, 128) && encode_split(&maps.ll, L.lo, L, batch, 64, 128) && encode_split(&maps.rh, R.hi, R, batch, 64, r_box) &&
              encode_split(&maps.rl, R.lo, R, batch, 64, r_box);
    if (E)
        ok = ok && encode_split(&maps.eh, E->hi, *E, batch, 64, 32) && encode_split(&maps.el, E->lo, *E, batch, 64, 32);
    if (out)
        ok = ok && encode_split(&maps.oh, out->hi, *out, batch, 64, 32) && encode_split(&maps.ol, out->lo, *out, batch, 64, 32) &&
             (!P.symmetric || (encode_split(&maps.th, out->hi, *out, batch, 32, 64) && encode_split(&maps.tl, out->lo, *out, batch, 32, 64)));
    if (P.result && P.wide) {
        // (a matrix alone: any distance to the next)
        const int64_t stride = batch > 1 ? P.result_stride : 8;
        ok = ok && (P.flip ? encode_stack(&maps.th, P.result, P.m, P.n, P.result_ld, stride, batch, 32, 64)
                           : encode_stack(&maps.oh, P.result, P.n, P.m, P.result_ld, stride, batch, 64, 32));
    }
    if (!ok)
        return cudaErrorInvalidValue;
    static int done[3][64];
    const size_t smem = 1024 + (size_t)P.stages * P.stage_bytes + staging;
    if constexpr (!CROSS)
        if (P.split > 1) {
            const cudaError_t e = opt_in_smem(k_ns_product<false, false, true>, kMmSmem, done[2]);
            return e != cudaSuccess ? e : launch_cluster(k_ns_product<false, false, true>, (int)P.n_tiles, (int)P.split, kMmThreads, s, smem, maps, P);
        }
    const cudaError_t e = pair ? opt_in_smem(k_ns_product<true, CROSS, false>, kMmSmem, done[1]) : opt_in_smem(k_ns_product<false, CROSS, false>, kMmSmem, done[0]);
    if (e != cudaSuccess)
        return e;
    // (a pair leaves no shared memory on its SMs: conef_mm.cuh)
    return pair ? launch_cluster(k_ns_product<true, CROSS, false>, (int)std::min<uint32_t>(P.n_tiles, kPlanSMs / 2), 2, kMmThreads, s, (size_t)kMmSmem, maps, P)
                : launch(k_ns_product<false, CROSS, false>, dim3(std::min<uint32_t>(P.n_tiles, kPlanSMs)), kMmThreads, smem, s, maps, P);
}

// the largest |b t + c t^2| for 0 <= t <= top, and the largest |s (a + b s^2 + c s^4)| for 0 <= s <= top
static double largest_factor(double b, double c, double top)
{
    double most = std::fabs(b * top + c * top * top);
    const double t = c != 0 ? -b / (2 * c) : -1;
    if (t > 0 && t < top)
        most = std::max(most, std::fabs(b * t + c * t * t));
    return most;
}
static double largest_value(double a, double b, double c, double top)
{
    auto f = [&](double s) { return std::fabs(s * (a + b * s * s + c * s * s * s * s)); };
    double most = f(top);
    const double root = 9 * b * b - 20 * a * c;   // f' = a + 3 b t + 5 c t^2, t = s^2
    auto at = [&](double t) {
        if (t > 0 && t < top * top)
            most = std::max(most, f(std::sqrt(t)));
    };
    if (c != 0 && root >= 0) {
        at((-3 * b + std::sqrt(root)) / (10 * c));
        at((-3 * b - std::sqrt(root)) / (10 * c));
    } else if (c == 0 && b != 0) {
        at(-a / (3 * b));
    }
    return most;
}
// a power of two that brings `bound` below 2^15, half of fp16's range
static double fp16_scale(double bound) { return std::ldexp(1.0, 14 - std::ilogb(std::max(bound, 1e-30))); }

// whether no two matrices of a stack share an element: one behind the other, or row by row among one another's rows
static bool ns_apart(int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride)
{
    return stride >= (rows - 1) * ld + cols || (stride >= cols && stride <= ld && (batch - 1) * stride + cols <= ld);
}

struct NsSizes {
    int64_t n, m, pitch_x, pitch_a;   // rows <= columns
    bool flip;
};
static NsSizes ns_sizes(int64_t rows, int64_t cols)
{
    NsSizes z;
    z.flip = rows > cols;
    z.n = std::min(rows, cols), z.m = std::max(rows, cols);
    z.pitch_x = (z.m + 63) / 64 * 64, z.pitch_a = (z.n + 63) / 64 * 64;
    return z;
}

}  // namespace conef

using namespace conef;

extern "C" {

int conef_orthogonalise_bytes(int64_t batch, int64_t rows, int64_t cols, size_t *bytes)
{
    if (batch < 0 || rows < 0 || cols < 0 || !bytes)
        return CONEF_ERR_INVALID_ARG;
    if (rows >= (1ll << 31) || cols >= (1ll << 31) || batch >= (1ll << 16))
        return CONEF_ERR_UNSUPPORTED;
    const NsSizes z = ns_sizes(rows, cols);
    // X twice, A and C, hi and lo each, and the norms' parts
    *bytes = batch && rows && cols ? ((size_t)batch * z.n * (2 * z.pitch_x + 2 * z.pitch_a) * 2 * sizeof(__half) + (size_t)batch * kNsParts * sizeof(double)) : 0;
    return CONEF_OK;
}

int conef_orthogonalise(const void *x, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride, int steps, const double *coefficients, double scale,
                        void *out, int out_dtype, int64_t out_ld, int64_t out_stride, void *workspace, size_t workspace_bytes, conef_stream stream)
{
    int rc = check_matrix(x, dtype, batch ? rows : 0, cols, ld);
    if (rc == CONEF_OK)
        rc = check_matrix(out, out_dtype, batch ? rows : 0, cols, out_ld);
    if (rc != CONEF_OK)
        return rc;
    if (batch < 0 || out_dtype == CONEF_F32 || steps < 1 || steps > 32 || !coefficients || !std::isfinite(scale) || std::fabs(scale) > 1e30)
        return CONEF_ERR_INVALID_ARG;
    if (batch > 1 && rows && cols && !(ns_apart(batch, rows, cols, ld, stride) && ns_apart(batch, rows, cols, out_ld, out_stride)))
        return CONEF_ERR_INVALID_ARG;
    // bounds of X before each step: a power of two each that keeps them within fp16
    double top[33];
    const double a = coefficients[0], b = coefficients[1], c = coefficients[2];
    top[0] = 1.0;
    for (int t = 0; t < steps; ++t) {
        top[t + 1] = largest_value(a, b, c, top[t]);
        if (!(top[t + 1] <= 1e4))
            return CONEF_ERR_INVALID_ARG;   // (the polynomial does not keep singular values bounded)
    }
    size_t need = 0;
    if ((rc = conef_orthogonalise_bytes(batch, rows, cols, &need)) != CONEF_OK)
        return rc;
    if (!need)
        return CONEF_OK;
    if (!workspace || workspace_bytes < need)
        return CONEF_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace & 127)
        return CONEF_ERR_INVALID_ARG;
    const NsSizes z = ns_sizes(rows, cols);
    cudaStream_t s = (cudaStream_t)stream;
    __half *at = (__half *)workspace;
    auto take = [&](int64_t columns, int64_t pitch) {
        Split m = {at, at + batch * z.n * pitch, z.n, columns, pitch};
        at += 2 * batch * z.n * pitch;
        return m;
    };
    Split X = take(z.m, z.pitch_x), Y = take(z.m, z.pitch_x), A = take(z.n, z.pitch_a), C = take(z.n, z.pitch_a);
    NsIn in = {x, rows, cols, ld, stride, (double *)at, (uint32_t)std::min<int64_t>(kNsParts, (rows * cols + 8191) / 8192)};
    double sx = fp16_scale(top[0]);
    cudaError_t e = cudaErrorInvalidValue;
    const int64_t tiles_c = (cols + 63) / 64, tiles = (rows + 63) / 64 * tiles_c;
    if (tiles >= (1ll << 31))
        return CONEF_ERR_UNSUPPORTED;
    with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        const bool vec = rows_on<T>(x, rows, ld, 16) && (batch == 1 || stride * (int64_t)sizeof(T) % 16 == 0);
        e = launch(vec ? k_ns_squares<T, true> : k_ns_squares<T, false>, dim3(in.n_parts, (unsigned)batch), 256, 0, s, in);
        if (e == cudaSuccess)
            e = launch(z.flip ? (vec ? k_ns_start<T, true, true> : k_ns_start<T, true, false>) : (vec ? k_ns_start<T, false, true> : k_ns_start<T, false, false>),
                       dim3((unsigned)tiles, (unsigned)batch), 256, 0, s, in, X, (uint32_t)tiles_c, sx);
        return 0;
    });
    for (int t = 0; t < steps && e == cudaSuccess; ++t) {
        const double sa = fp16_scale(top[t] * top[t]), sc = fp16_scale(largest_factor(b, c, top[t] * top[t])), sy = fp16_scale(top[t + 1]);
        const bool last = t + 1 == steps;
        NsArgs P = {};
        P.symmetric = 1;
        P.f_sum = (float)(sa / (sx * sx));
        e = ns_product<false>(X, X, nullptr, &A, batch, P, s);
        if (e != cudaSuccess)
            break;
        P.f_sum = (float)(c * sc / (sa * sa));
        P.f_add = (float)(b * sc / sa);
        e = ns_product<false>(A, A, &A, &C, batch, P, s);
        if (e != cudaSuccess)
            break;
        const double to = last ? scale : sy;
        NsArgs U = {};
        U.f_sum = (float)(to / (sc * sx));
        U.f_add = (float)(a * to / sx);
        if (last) {
            U.result = out;
            U.result_ld = rows > 1 ? out_ld : cols;
            U.result_stride = batch > 1 ? out_stride : 0;
            U.flip = z.flip;
            U.dtype = (uint32_t)out_dtype;
            // (a tiled copy writes a row's last 16 bytes whole, whatever the map says of its end; a map's matrices follow one another)
            U.wide = (((uintptr_t)out | (uint64_t)(U.result_ld | U.result_stride | cols) * 2) & 15) == 0 && (batch == 1 || out_stride >= out_ld);
        }
        e = ns_product<true>(C, X, &X, last ? nullptr : &Y, batch, U, s);
        std::swap(X, Y);
        sx = sy;
    }
    return launched(e, "conef_orthogonalise");
}

int conef_orthogonalise_timeouts(int64_t *count, conef_stream stream)
{
    if (!count)
        return CONEF_ERR_INVALID_ARG;
    unsigned long long n = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&n, g_mm_ran_out, sizeof n, 0, cudaMemcpyDeviceToHost, (cudaStream_t)stream);
    if (e == cudaSuccess)
        e = cudaStreamSynchronize((cudaStream_t)stream);
    *count = (int64_t)n;
    return launched(e, "conef_orthogonalise_timeouts");
}

}  // extern "C"
