// Product of two matrices held in few bits with block scales, out[i][j] = sum over k of A[i][k] B[j][k], in fp32 on the tensor cores' block-scaled
// path and rounded once to the output's type: the kernel and its launch, for the formats of conef_mx4mm.cu and conef_f8mm.cu.
//
// A CTA per SM, or a pair of CTAs on two SMs that share the rows of B, walks over tiles of 128 (256) x BN outputs, BN 64 to 256.  18 warps with a
// part each: one brings 128 bytes of each row at a time into a ring of stages (codes by tiled copies; scales, which lie in memory as the
// tensor cores take them, by plain bulk ones), one issues the products, and sixteen move the sums of a tile from tensor memory through registers and shared
// memory to the output while the next tile's are formed in a second set.
#pragma once
#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "conef_common.cuh"
#include "conef_elem.cuh"
#include "conef_tc.cuh"

namespace conef {

constexpr int kMmM = 128;                                // rows of A per tile
constexpr int kMmEpilogue = 16, kMmThreads = (kMmEpilogue + 2) * 32;   // (four warps per 64 columns)
constexpr int kMmMaxStages = 6;
constexpr uint32_t kMmSmem = 226 * 1024;                 // of a CTA's 227 KB, beside the barriers
constexpr uint32_t kMmAlone = 116 * 1024;                // more than half of an SM's 228 KB
constexpr uint32_t kMmColumns = 512;                     // tensor memory, all of it, so from column 0 on: the sums, then the scales of each stage

// A format F says how its elements lie in a stage, which is 128 bytes of a row in every format, four instructions' worth:
//   kStageK, kStepK    elements of k in a stage and in an instruction
//   kTiles             tiles of scales that a stage brings, of 4 (A) and up to 8 columns (B) each
//   kTileStages        stages that one tile serves (one after the other)
//   row_bytes(k), scale_tiles(k)
//   instruction<PAIR>(n, P), issue<PAIR>(...)
//   kSplits            whether few tiles may be shared along k

struct MmArgs {
    const uint8_t *as, *bs;      // scales (a single CTA's)
    int64_t m, n, ld;
    uint32_t k_steps, stages_k;  // instructions and stages along k
    uint32_t tiles;              // tiles of scales along k
    uint32_t b_rows;             // ... of 128 rows of B
    uint32_t bn;
    Divider band, low;           // tiles of a whole band, rows of tiles in the last one (2 at least)
    uint32_t last_band, last_rows;
    uint32_t n_tiles, stages;
    uint32_t tiled;              // outputs go by tiled copies
    uint32_t sums, scale_column; // sets of sums in tensor memory, and the first column of scales
    uint64_t limit, sums_limit;  // nanoseconds that a wait takes at most, and the one for a tile's sums, which lasts for all of k
    uint32_t loads[2];           // stages that the CTA(s) of a pair bring at most (tests)
    uint32_t copied;             // bytes of codes that fill a stage (a single CTA's)
    uint32_t kind_a, kind_b;     // types of elements, where the format has several
    uint32_t split, split_stages;   // CTAs of a cluster that share a tile's k, and stages of each (the last one's may be fewer)
};
// CTAs in which a wait has run out, since the library was loaded (a count per format, whose file includes this)
static __device__ unsigned long long g_mm_ran_out;
struct MmMaps {
    CUtensorMap a, b, out;       // (out: where it is `tiled`)
    CUtensorMap as, bs;          // of scales, for pairs, whose copies have to tell the leader's barrier
};

// stage: A 128 x 128 bytes, B bn x 128 bytes (of a pair: half), then 1024 bytes per 128 rows, for one or two tiles of scales along k
__host__ __device__ inline uint32_t mm_scale_rows(uint32_t bn) { return bn > 128 ? 2 : 1; }
__host__ __device__ inline uint32_t mm_stage_bytes(uint32_t bn, bool pair) { return kMmM * 128 + bn * (pair ? 64 : 128) + 1024 * (1 + mm_scale_rows(bn)); }
inline uint32_t mm_staging(uint32_t bn) { return bn / 16 * 4096; }   // per storing warp 32 rows of 128 bytes, where outputs are turned from a row per lane

// Tiles are taken in bands of kMmBand along m, so that what runs at a time is about as high as wide (8192 x 6400 x 1600, pairs of 256 columns: in bands
// of 8 and of 4 53 us, of one 59, in one band of all 55.6; with 192 columns 47.6 to 48.8, by an earlier form).  No division: a tile's place is
// on the way of the products from one tile to the next.
constexpr uint32_t kMmBand = 8;
struct MmTile {
    uint32_t m, n;
};
__device__ __forceinline__ MmTile mm_tile(const MmArgs &P, uint32_t tile)
{
    const uint32_t band = divide(tile, P.band), in = tile - band * P.band.by;
    uint32_t n = in / kMmBand, rows = kMmBand;
    if (band == P.last_band) {
        rows = P.last_rows;
        n = rows == 1 ? in : divide(in, P.low);
    }
    return {band * kMmBand + in - n * rows, n};
}

struct MmShared {
    uint64_t full[kMmMaxStages], empty[kMmMaxStages], sums[2], taken[2], drain;
    uint32_t tmem, armed;        // (armed: stages brought)
    int dead;
};

// 16 bytes of outputs from the sums of a row
template <class T>
__device__ __forceinline__ uint4 pack16(const uint32_t *v);
template <>
__device__ __forceinline__ uint4 pack16<float>(const uint32_t *v)
{
    return make_uint4(v[0], v[1], v[2], v[3]);
}
template <class F>
__device__ __forceinline__ uint4 pack16_short(const uint32_t *v, F pack)
{
    uint4 w;
    w.x = pack(__uint_as_float(v[0]), __uint_as_float(v[1]));
    w.y = pack(__uint_as_float(v[2]), __uint_as_float(v[3]));
    w.z = pack(__uint_as_float(v[4]), __uint_as_float(v[5]));
    w.w = pack(__uint_as_float(v[6]), __uint_as_float(v[7]));
    return w;
}
template <>
__device__ __forceinline__ uint4 pack16<__nv_bfloat16>(const uint32_t *v)
{
    return pack16_short(v, [](float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *(const uint32_t *)&h;
    });
}
template <>
__device__ __forceinline__ uint4 pack16<__half>(const uint32_t *v)
{
    return pack16_short(v, [](float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *(const uint32_t *)&h;
    });
}

// The sums of a tile whose k the CTAs of a cluster share: each CTA adds up its columns, of all, in the CTAs' order, four columns to a thread
template <int SPLIT, class T>
__device__ __forceinline__ void mm_join(const MmArgs &P, const float *sums, const int &dead, const MmTile &at, uint32_t part, T *out)
{
    const uint32_t width = P.bn / SPLIT, quads = width / 4, shift = 31 - __clz(quads);   // (a power of two)
    const int64_t row0 = (int64_t)at.m * kMmM, col0 = (int64_t)at.n * P.bn;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < SPLIT; ++i)
        any |= tc::load_at(tc::address_in(&dead, i));
    const uint32_t all = (uint32_t)min((int64_t)kMmM, P.m - row0) << shift;
    for (uint32_t e = threadIdx.x; e < all; e += kMmThreads) {
        const uint32_t r = e >> shift, c = part * width + (e & (quads - 1)) * 4;
        const int64_t col = col0 + c;
        if (col >= P.n)
            continue;
        const float *const mine = sums + r * (P.bn + 4) + c;
        float4 v[SPLIT];
#pragma unroll
        for (int i = 0; i < SPLIT; ++i)
            v[i] = tc::load_at4(tc::address_in(mine, i));
        float f[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
        for (int i = 1; i < SPLIT; ++i)
            f[0] = __fadd_rn(f[0], v[i].x), f[1] = __fadd_rn(f[1], v[i].y), f[2] = __fadd_rn(f[2], v[i].z), f[3] = __fadd_rn(f[3], v[i].w);
        T *const to = out + (row0 + r) * P.ld + col;
        T o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] = from_f32<T>(any ? __uint_as_float(0x7FFFFFFFu) : f[i]);   // (a wait ran out: what was not computed is NaN)
        if (P.tiled && col + 4 <= P.n) {
            if constexpr (sizeof(T) == 4)
                *(uint4 *)to = *(const uint4 *)o;
            else
                *(uint2 *)to = *(const uint2 *)o;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < P.n)
                    to[i] = o[i];
        }
    }
}

// SPLIT: the CTAs of a cluster have one tile, and each a part of k.  What they have summed goes to their own shared memory, where all stages have been used, and each
// adds up a share of the columns, in the CTAs' order.
template <class F, class T, bool PAIR, bool SPLIT>
__global__ void __launch_bounds__(kMmThreads, 1) k_matmul(const __grid_constant__ MmMaps maps, const __grid_constant__ MmArgs P, T *out)
{
    extern __shared__ __align__(1024) uint8_t mm_smem[];
    __shared__ MmShared S;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;   // (known to be the same in all lanes)
    const uint32_t stage_bytes = mm_stage_bytes(P.bn, PAIR), scale_rows = mm_scale_rows(P.bn), b_bytes = P.bn * (PAIR ? 64u : 128u);
    const uint32_t rank = PAIR ? blockIdx.x & 1u : 0u, first = PAIR ? blockIdx.x / 2 : SPLIT ? blockIdx.x / P.split : blockIdx.x;
    const uint32_t step = PAIR ? gridDim.x / 2 : gridDim.x;   // (SPLIT: beyond the tiles)
    const uint32_t part = SPLIT ? blockIdx.x - first * P.split : 0u, ks0 = SPLIT ? part * P.split_stages : 0u, ks1 = SPLIT ? min(ks0 + P.split_stages, P.stages_k) : P.stages_k;
    uint8_t *const ring = mm_smem + ((1024u - (tc::saddr(mm_smem) & 1023u)) & 1023u);
    const tc::Waits waits = {&S.dead, PAIR ? tc::address_in(&S.dead, rank ^ 1u) : 0u, &g_mm_ran_out};
    if (warp == 1 && lane < (int)(sizeof maps / sizeof maps.a))
        tc::prefetch_map(&maps.a + lane);
    if (warp == 0) {
        tc::tmem_alloc<PAIR>(&S.tmem, kMmColumns);
        if (lane == 0) {
            for (int i = 0; i < kMmMaxStages; ++i) {
                tc::bar_init(&S.full[i], 1);
                tc::bar_init(&S.empty[i], 1);
            }
            for (int i = 0; i < 2; ++i) {
                tc::bar_init(&S.sums[i], 1);
                tc::bar_init(&S.taken[i], P.bn / 16 * (PAIR ? 2 : 1));
            }
            tc::bar_init(&S.drain, 1);
            S.dead = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        tc::fence_before();
    }
    __syncthreads();
    if (PAIR)
        tc::cluster_sync();   // the other CTA's barriers exist
    tc::fence_after();
    grid_release();
    grid_wait();
    asm volatile("fence.proxy.async;" ::: "memory");   // (what the launch before stored, ordinary stores, is read by copies)

    // step ks of a tile into stage s: row tm of scales of A (128 rows of codes), columns from n0 on
    auto load = [&](uint32_t s, uint32_t ks, uint32_t tm, uint32_t n0) {
        const uint32_t st = tc::saddr(ring) + s * stage_bytes, sc = st + kMmM * 128 + b_bytes;
        if constexpr (PAIR) {
            // (what does not exist of rows and tiles of scales is filled with zeros)
            const uint32_t bar = tc::leaders(&S.full[s]);
            if (rank == 0)
                tc::bar_expect(&S.full[s], 2 * (kMmM * 128 + b_bytes + F::kTiles * 512 * (1 + scale_rows)));
            tc::tile_load_pair(st, &maps.a, ks * 128, tm * kMmM, bar);
            tc::tile_load_pair(st + kMmM * 128, &maps.b, ks * 128, n0 + rank * (P.bn / 2), bar);
            tc::tile_load_pair(sc, &maps.as, ks / F::kTileStages * (F::kTiles * 128), tm, bar);
            tc::tile_load_pair(sc + F::kTiles * 512, &maps.bs, ks / F::kTileStages * (F::kTiles * 128), n0 / 128, bar);
        } else {
            const uint32_t tile = ks / F::kTileStages * F::kTiles, scale_bytes = min(P.tiles - tile, (uint32_t)F::kTiles) * 512u;
            tc::bar_expect(&S.full[s], P.copied + scale_bytes * (1 + scale_rows));
            tc::tile_load(st, &maps.a, ks * 128, tm * kMmM, &S.full[s]);
            tc::tile_load(st + kMmM * 128, &maps.b, ks * 128, n0, &S.full[s]);
            tc::bulk_load(sc, P.as + ((size_t)tm * P.tiles + tile) * 512, scale_bytes, &S.full[s]);
            for (uint32_t r = 0; r < scale_rows; ++r)   // (rows past the last tile, whose products nobody stores: the last one's)
                tc::bulk_load(sc + F::kTiles * 512 * (1 + r), P.bs + ((size_t)min(n0 / 128 + r, P.b_rows - 1) * P.tiles + tile) * 512, scale_bytes, &S.full[s]);
        }
    };
    uint32_t armed = 0;   // (the loading warp's)
    if (warp == kMmEpilogue) {
        uint32_t s = 0, phase = 0;
        bool ok = true;
        for (uint32_t tile = first; ok && tile < P.n_tiles; tile += step) {
            const MmTile at = mm_tile(P, tile);
            const uint32_t tm = at.m * (PAIR ? 2 : 1) + rank, n0 = at.n * P.bn;   // (tm in 128 rows)
            for (uint32_t ks = ks0; ks < ks1; ++ks) {
                if (!(ok = armed < P.loads[rank] && tc::bar_wait(&S.empty[s], phase ^ 1u, waits, P.limit)))
                    break;
                if (tc::elect())
                    load(s, ks, tm, n0);
                ++armed;
                if (++s == P.stages)
                    s = 0, phase ^= 1u;
            }
        }
        if (lane == 0)
            S.armed = armed;
        __syncwarp();
    } else if (warp == kMmEpilogue + 1) {
        const uint32_t instruction = F::template instruction<PAIR>(P);
        const uint32_t a0 = tc::desc_low(ring), b0 = a0 + kMmM * 8, sc0 = b0 + b_bytes / 16, step16 = stage_bytes >> 4;
        uint32_t s = 0, phase = 0, set = 0, turn = 0;
        bool ok = true;
        for (uint32_t tile = rank ? P.n_tiles : first; ok && tile < P.n_tiles; tile += step) {
            const uint32_t n0 = mm_tile(P, tile).n * P.bn, d = set * P.bn;
            const uint32_t shift = (n0 & 127u) >> 5;   // columns of the first tile of scales ahead of row n0
            if (!(ok = tc::bar_wait(&S.taken[set], turn ^ 1u, waits, P.limit)))
                break;
            tc::fence_after();
            for (uint32_t ks = ks0; ks < ks1; ++ks) {
                if (!(ok = tc::bar_wait(&S.full[s], phase, waits, P.limit)))
                    break;
                tc::fence_after();
                if (tc::elect()) {
                    const uint32_t sa = P.scale_column + s * F::kScaleColumns, sb = sa + F::kTiles * 4;
                    F::template issue<PAIR>(P, d, a0 + s * step16, b0 + s * step16, sc0 + s * step16, instruction, sa, sb, shift, scale_rows, ks, ks0);
                    tc::commit<PAIR>(&S.empty[s]);
                }
                if (++s == P.stages)
                    s = 0, phase ^= 1u;
            }
            if (ok && tc::elect())
                tc::commit<PAIR>(&S.sums[set]);
            if (++set == P.sums)
                set = 0, turn ^= 1u;
        }
        __syncwarp();
    } else if (SPLIT) {
        const uint32_t c0 = (uint32_t)(warp >> 2) * 64;
        if (c0 < P.bn && tc::bar_wait(&S.sums[0], 0, waits, P.sums_limit)) {   // (where the wait runs out, `dead` tells all CTAs)
            tc::fence_after();
            uint4 *const to = (uint4 *)ring + (((warp & 3) * 32 + lane) * (P.bn + 4) + c0) / 4;   // (rows 16 bytes apart: eight lanes' go to all banks)
#pragma unroll
            for (uint32_t q = 0; q < 64; q += 32) {
                uint32_t v[32];
                tc::tmem_load32(((uint32_t)(warp & 3) << 21) + c0 + q, v);
                tc::tmem_load_wait();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    to[q / 4 + i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
        }
        __syncwarp();
    } else {
        // sums of 32 rows (a lane each) and 64 columns
        constexpr int PER = 16 / sizeof(T), PASS = 128 / sizeof(T);   // outputs in 16 and in 128 bytes
        uint32_t set = 0, turn = 0;
        bool ok = true;
        const uint32_t c0 = (uint32_t)(warp >> 2) * 64;
        const uint32_t staging = tc::saddr(ring) + P.stages * stage_bytes + warp * 4096;
        float *const turned = (float *)(ring + P.stages * stage_bytes + warp * 4096);
        for (uint32_t tile = c0 < P.bn ? first : P.n_tiles; tile < P.n_tiles; tile += step) {
            const MmTile at = mm_tile(P, tile);
            const int64_t row0 = ((int64_t)at.m * (PAIR ? 2 : 1) + rank) * kMmM + (warp & 3) * 32, col0 = (int64_t)at.n * P.bn + c0;
            ok = ok && tc::bar_wait(&S.sums[set], turn, waits, P.sums_limit);
            uint32_t v[64];
            if (ok) {
                tc::fence_after();
                const uint32_t sums = ((uint32_t)(warp & 3) << 21) + set * P.bn + c0;
                tc::tmem_load32(sums, *(uint32_t(*)[32])v);
                tc::tmem_load32(sums + 32, *(uint32_t(*)[32])(v + 32));
                tc::tmem_load_wait();
                tc::fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR)
                        tc::bar_arrive_at(tc::leaders(&S.taken[set]));
                    else
                        tc::bar_arrive(&S.taken[set]);
                }
            } else {   // a wait ran out: what was not computed is NaN
#pragma unroll
                for (int i = 0; i < 64; ++i)
                    v[i] = 0x7FFFFFFFu;
            }
            if (row0 < P.m && P.tiled) {
#pragma unroll
                for (int c = 0; c < 64; c += PASS) {
                    if (lane == 0)
                        tc::store_wait_read();
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint4 w = pack16<T>(v + c + i * PER);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(staging + lane * 128 + ((i ^ (lane & 7)) << 4)), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
                    }
                    tc::store_fence();
                    __syncwarp();
                    if (lane == 0 && col0 + c < P.n)
                        tc::tile_store(&maps.out, staging, (uint32_t)(col0 + c), (uint32_t)row0);
                }
            } else if (row0 < P.m) {
                // a warp stores 32 outputs of a row
                const int rows = (int)min((int64_t)32, P.m - row0);
#pragma unroll
                for (int c = 0; c < 64; c += 32) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        turned[lane * 32 + (i ^ lane)] = __uint_as_float(v[c + i]);
                    __syncwarp();
                    if (col0 + c + lane < P.n)
                        for (int r = 0; r < rows; ++r)
                            out[(row0 + r) * P.ld + col0 + c + lane] = from_f32<T>(turned[r * 32 + (lane ^ r)]);
                    __syncwarp();
                }
            }
            if (++set == P.sums)
                set = 0, turn ^= 1u;
        }
        if (lane == 0)
            tc::store_wait();
        __syncwarp();
    }
    tc::fence_before();
    __syncthreads();
    if (PAIR || SPLIT)
        tc::cluster_sync();   // neither CTA tells a barrier of one that has ended
    tc::fence_after();
    if constexpr (SPLIT) {
        if (P.split == 2)
            mm_join<2>(P, (const float *)ring, S.dead, mm_tile(P, first), part, out);
        else if (P.split == 4)
            mm_join<4>(P, (const float *)ring, S.dead, mm_tile(P, first), part, out);
        else
            mm_join<8>(P, (const float *)ring, S.dead, mm_tile(P, first), part, out);
        __syncthreads();
        tc::cluster_sync();   // (all have read)
    }
    if (*waits.dead) {
        // A wait has run out (in a pair both know by now).  What is in flight ends before shared and tensor memory are given back: the copies, for whose
        // barriers to be told of all their bytes each CTA of a pair brings what the other has, and the products.
        const uint64_t t0 = tc::nanoseconds();
        if (warp == kMmEpilogue) {
            const uint32_t all = PAIR ? max(armed, tc::load_at(tc::address_in(&S.armed, rank ^ 1u))) : armed;
            for (; armed < all; ++armed) {
                const uint32_t nth = armed / P.stages_k;
                const MmTile at = mm_tile(P, first + nth * step);
                if (tc::elect())
                    load(armed % P.stages, armed - nth * P.stages_k, at.m * (PAIR ? 2 : 1) + rank, at.n * P.bn);
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

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled()
{
    static EncodeTiled f = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (EncodeTiled)p;
    }();
    return f;
}
// Rows of `row_bytes` bytes, `ld` apart, as elements of `type`, copied in tiles of `width` elements by `box` rows; what lies past either end is read as
// zero and not written
static bool encode(CUtensorMap *map, CUtensorMapDataType type, int elem, const void *p, int64_t rows, int64_t row_bytes, int64_t ld, uint32_t width, uint32_t box)
{
    const cuuint64_t dims[2] = {(cuuint64_t)(row_bytes / elem), (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
    const cuuint32_t tile[2] = {width, box}, steps[2] = {1, 1};
    return encode_tiled() && encode_tiled()(map, type, 2, (void *)p, dims, strides, tile, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                            width * elem == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Columns per tile, and whether pairs of CTAs take tiles of 256 rows: the choice whose waves of tiles over the SMs take least.  F::per_step() and F::per_tile() have
// what a wave takes in nanoseconds, by columns (64, 128, 192, 256), per instruction's step along k (single CTAs, pairs) and beside that; a launch of pairs takes a
// microsecond more.  Pairs of 64 columns are left out: they take as many waves as single CTAs at least, none of them shorter.
struct MmChoice {
    uint32_t bn;
    bool pair;
    uint32_t split;
    int64_t cost;
};
template <class F>
static MmChoice mm_choice(int64_t m, int64_t n, int64_t k)
{
    const int64_t k_steps = (k + F::kStepK - 1) / F::kStepK;
    MmChoice best = {0, false, 1, 0};
    for (int pair = 0; pair < 2; ++pair)
        for (uint32_t bn = pair ? 128 : 64; bn <= 256; bn += 64) {
            const int64_t rows = pair ? 2 * kMmM : kMmM, sets = pair ? kPlanSMs / 2 : kPlanSMs;
            const int64_t waves = ((m + rows - 1) / rows * ((n + bn - 1) / bn) + sets - 1) / sets;
            const int64_t cost = waves * (k_steps * F::per_step(pair, bn / 64 - 1) + F::per_tile(bn / 64 - 1)) + pair * 1000;
            if (!best.bn || cost < best.cost)
                best = {bn, pair != 0, 1, cost};
        }
    if constexpr (F::kSplits) {
        // Clusters that share tiles along k, as many as run at once (74, 33 or 15 with a CTA to an SM, which lie in groups of 16 to 20: a second wave of one takes
        // as long as the first; 256 x 512 x 8192 by 16 clusters 16 us, 448 columns by 14 9.2); to begin, to join the sums and to end they take 2 us more.
        // Without and with: 64 x 1600 x 6400 13.4 and 8.7 us, 64 x 4096 x 4096 10.6 and 8.7, 768 x 768 x 8192 17 and 13, 256 x 256 x 32768 53 and 14.
        const int64_t stages = (k + F::kStageK - 1) / F::kStageK;
        for (uint32_t bn = 64; bn <= 128; bn += 64)
            for (uint32_t split = 2; split <= 8; split *= 2) {
                const int64_t tiles = (m + kMmM - 1) / kMmM * ((n + bn - 1) / bn), each = (stages + split - 1) / split;
                const int64_t cost = each * (F::kStageK / F::kStepK) * F::per_step(0, bn / 64 - 1) + F::per_tile(bn / 64 - 1) + 2000;
                if (tiles <= (split == 2 ? 72 : split == 4 ? 32 : 14) && each >= 4 && each * (split - 1) < stages && cost < best.cost)
                    best = {bn, false, split, cost};
            }
    }
    return best;
}

struct MmLimit {
    std::atomic<int64_t> nanoseconds{2000000000};
    std::atomic<uint32_t> loads[2] = {{0xFFFFFFFFu}, {0xFFFFFFFFu}};
};
inline MmLimit mm_limit;   // (of all formats)

template <class F, class T, bool PAIR, bool SPLIT>
static int matmul(const uint8_t *a, const uint8_t *as, int64_t m, const uint8_t *b, const uint8_t *bs, int64_t n, int64_t k, T *out, int64_t ld, const MmChoice &choice,
                  int kind_a, int kind_b, const char *what, cudaStream_t s)
{
    constexpr int64_t kRows = PAIR ? 2 * kMmM : kMmM;
    const uint32_t bn = choice.bn;
    MmArgs P;
    P.as = as;
    P.bs = bs;
    P.m = m;
    P.n = n;
    P.ld = ld;
    P.k_steps = (uint32_t)((k + F::kStepK - 1) / F::kStepK);
    P.stages_k = (uint32_t)((k + F::kStageK - 1) / F::kStageK);
    P.kind_a = (uint32_t)kind_a;
    P.kind_b = (uint32_t)kind_b;
    P.split = SPLIT ? choice.split : 1;
    P.split_stages = (P.stages_k + P.split - 1) / P.split;
    P.limit = (uint64_t)mm_limit.nanoseconds.load();
    // (a stage takes 0.4 us at most where nothing else runs)
    P.sums_limit = P.limit + 4096ull * P.stages_k;
    P.loads[0] = mm_limit.loads[0].load();
    P.loads[1] = mm_limit.loads[1].load();
    // Rows that a copy brings: of a matrix with fewer than a tile's, in eights; behind them a product has whatever the stage held, in sums that nobody stores.  (Filled with
    // zeros to a tile's 128, matrices of less than 128 KB took up to twice as long: 9 x 8192 x 8192 32 us, 16 rows 19.)
    const uint32_t a_box = PAIR ? kMmM : (uint32_t)std::min<int64_t>(kMmM, (m + 7) / 8 * 8), b_box = PAIR ? bn / 2 : (uint32_t)std::min<int64_t>(bn, (n + 7) / 8 * 8);
    P.copied = (a_box + b_box) * 128;
    P.tiles = (uint32_t)F::scale_tiles(k);
    P.b_rows = (uint32_t)((n + 127) / 128);
    P.bn = bn;
    const int64_t tiles_m = (m + kRows - 1) / kRows, tiles_n = (n + bn - 1) / bn, tiles = tiles_m * tiles_n;
    if (tiles >= (1ll << 32) - kPlanSMs || tiles_n >= (1ll << 28))
        return CONEF_ERR_UNSUPPORTED;
    P.n_tiles = (uint32_t)tiles;
    P.band = divider((uint32_t)(tiles_n * kMmBand));
    P.last_band = (uint32_t)((tiles_m - 1) / kMmBand);
    P.last_rows = (uint32_t)(tiles_m - (int64_t)P.last_band * kMmBand);
    P.low = divider(std::max(2u, P.last_rows));
    // tensor memory: two sets of sums where that leaves room for the scales
    P.sums = bn <= 192 ? 2 : 1;
    P.scale_column = P.sums * bn > 256 ? 384 : 256;
    const uint32_t stage_bytes = mm_stage_bytes(bn, PAIR);
    const uint32_t room = kMmSmem - 1024 - mm_staging(bn);
    P.stages = std::min<uint32_t>({(uint32_t)kMmMaxStages, (kMmColumns - P.scale_column) / F::kScaleColumns, room / stage_bytes, std::max(2u, P.split_stages)});   // (SPLIT: a tile's sums fit two)
    // (a tiled copy writes a row's last 16 bytes whole, whatever the map says of its end)
    P.tiled = (((uint64_t)ld * sizeof(T)) | ((uint64_t)n * sizeof(T)) | (uintptr_t)out) % 16 == 0;
    MmMaps maps = {};
    const int64_t row_bytes = F::row_bytes(k), scale_bytes = (int64_t)P.tiles * 512;
    bool ok = encode(&maps.a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a, m, row_bytes, row_bytes, 128, a_box) &&
              encode(&maps.b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b, n, row_bytes, row_bytes, 128, b_box);
    if (P.tiled)
        ok = ok && encode(&maps.out, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, sizeof(T), out, m, n * (int64_t)sizeof(T),
                          (m > 1 ? ld : n) * (int64_t)sizeof(T), 128 / sizeof(T), 32);
    if (PAIR)
        ok = ok && encode(&maps.as, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, as, (m + 127) / 128, scale_bytes, scale_bytes, F::kTiles * 128, 1) &&
             encode(&maps.bs, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, bs, P.b_rows, scale_bytes, scale_bytes, F::kTiles * 128, mm_scale_rows(bn));
    if (!ok)
        return launched(cudaErrorInvalidValue, what);
    // Never two CTAs on an SM, of two products at once either: each takes all of tensor memory, and of two pairs on the same SMs
    // each could hold one half.  A pair leaves no shared memory at all, since the other one could be any kernel's.
    const size_t smem = PAIR ? kMmSmem : std::max<size_t>(1024 + (size_t)P.stages * stage_bytes + mm_staging(bn), kMmAlone);
    static int done[64];
    cudaError_t e = opt_in_smem(k_matmul<F, T, PAIR, SPLIT>, kMmSmem, done);
    if (e == cudaSuccess) {
        if (PAIR)
            e = launch_cluster(k_matmul<F, T, PAIR, SPLIT>, (int)std::min<uint32_t>(P.n_tiles, kPlanSMs / 2), 2, kMmThreads, s, smem, maps, P, out);
        else if (SPLIT)
            e = launch_cluster(k_matmul<F, T, PAIR, SPLIT>, (int)P.n_tiles, (int)P.split, kMmThreads, s, smem, maps, P, out);
        else
            e = launch(k_matmul<F, T, PAIR, SPLIT>, dim3(std::min<uint32_t>(P.n_tiles, kPlanSMs)), kMmThreads, smem, s, maps, P, out);
    }
    return launched(e, what);
}

}  // namespace conef
