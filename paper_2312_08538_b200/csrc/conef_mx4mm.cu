// Product of two matrices held in microscaled 4-bit floats, out[i][j] = sum over k of A[i][k] B[j][k], in fp32 on the tensor
// cores' block-scaled path and rounded once to the output's type.
//
// A CTA per SM walks over tiles of 128 x BN outputs (BN 64 to 256), ten warps with a part each: one brings 256 elements of k at a time
// into a ring of stages (codes by tiled copies, scales, which lie in memory as the tensor cores take them, by plain bulk ones), one
// issues the products, and eight move the sums from tensor memory to registers, let the next tile begin, and store.
#include <cuda.h>

#include <algorithm>

#include "conef_mx4.cuh"
#include "conef_common.cuh"
#include "conef_elem.cuh"
#include "conef_tc.cuh"

namespace conef {

constexpr int kMmM = 128, kMmK = 256;                    // rows of A per tile, elements of k per stage
constexpr int kMmEpilogue = 8, kMmThreads = (kMmEpilogue + 2) * 32;
constexpr int kMmMaxStages = 6;
// tensor memory, all of it, so from column 0 on: the sums, then 32 columns of scales per stage (24 used)
constexpr uint32_t kMmColumns = 512, kMmScaleColumn = 256;

struct MmArgs {
    const uint8_t *as, *bs;      // scales
    int64_t m, n, ld;
    uint32_t k64, stages_k;      // steps of 64 and of kMmK elements along k
    uint32_t tiles;              // tiles of scales along k
    uint32_t b_rows;             // ... of 128 rows of B
    uint32_t bn, tiles_m;
    uint32_t n_tiles, stages;
};

// stage: A 128 x 128 bytes, B bn x 128 bytes, then 1024 bytes of scales per 128 rows (two tiles along k)
__host__ __device__ inline uint32_t mm_scale_rows(uint32_t bn) { return bn > 128 ? 2 : 1; }
__host__ __device__ inline uint32_t mm_stage_bytes(uint32_t bn) { return kMmM * 128 + bn * 128 + 1024 * (1 + mm_scale_rows(bn)); }
constexpr uint32_t kMmStaging = kMmEpilogue * 32 * 33 * 4;   // per warp 32 x 32 outputs where rows are stored piece by piece

struct MmShared {
    uint64_t full[kMmMaxStages], empty[kMmMaxStages], sums, taken, drain;
    uint32_t tmem;
    int dead;
};

template <class T>
__device__ __forceinline__ void store32(T *out, const uint32_t (&v)[32]);   // 32 outputs of a row, 32-byte aligned
__device__ __forceinline__ void store_v8(void *p, const uint32_t *w)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]),
                 "r"(w[7])
                 : "memory");
}
template <>
__device__ __forceinline__ void store32<float>(float *out, const uint32_t (&v)[32])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        store_v8(out + 8 * i, v + 8 * i);
}
template <class H2, class F>
__device__ __forceinline__ void store32_short(void *out, const uint32_t (&v)[32], F pack)
{
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const H2 h = pack(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
        w[i] = *(const uint32_t *)&h;
    }
    store_v8(out, w);
    store_v8((uint8_t *)out + 32, w + 8);
}
template <>
__device__ __forceinline__ void store32<__nv_bfloat16>(__nv_bfloat16 *out, const uint32_t (&v)[32])
{
    store32_short<__nv_bfloat162>(out, v, [](float a, float b) { return __floats2bfloat162_rn(a, b); });
}
template <>
__device__ __forceinline__ void store32<__half>(__half *out, const uint32_t (&v)[32])
{
    store32_short<__half2>(out, v, [](float a, float b) { return __floats2half2_rn(a, b); });
}

template <class T>
__global__ void __launch_bounds__(kMmThreads, 1) k_mx4_matmul(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                              const __grid_constant__ MmArgs P, T *out)
{
    extern __shared__ __align__(1024) uint8_t mm_smem[];
    __shared__ MmShared S;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t stage_bytes = mm_stage_bytes(P.bn), scale_rows = mm_scale_rows(P.bn);
    uint8_t *const ring = mm_smem + ((1024u - (tc::saddr(mm_smem) & 1023u)) & 1023u);
    volatile int *const dead = &S.dead;
    if (warp == 0) {
        tc::tmem_alloc(&S.tmem, kMmColumns);
        if (lane == 0) {
            for (int i = 0; i < kMmMaxStages; ++i) {
                tc::bar_init(&S.full[i], 1);
                tc::bar_init(&S.empty[i], 1);
            }
            tc::bar_init(&S.sums, 1);
            tc::bar_init(&S.taken, kMmEpilogue);
            tc::bar_init(&S.drain, 1);
            S.dead = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        tc::fence_before();
    }
    __syncthreads();
    tc::fence_after();
    grid_release();
    grid_wait();
    if (warp == kMmEpilogue) {
        if (lane == 0) {
            uint32_t s = 0, phase = 0, armed = 0;
            bool ok = true;
            for (uint32_t tile = blockIdx.x; ok && tile < P.n_tiles; tile += gridDim.x) {
                const uint32_t tm = tile % P.tiles_m, tn = tile / P.tiles_m;
                const uint32_t n0 = tn * P.bn;
                const uint8_t *as = P.as + (size_t)tm * P.tiles * 512;
                for (uint32_t ks = 0; ks < P.stages_k; ++ks) {
                    if (!(ok = tc::bar_wait(&S.empty[s], phase ^ 1u, dead)))
                        break;
                    uint8_t *st = ring + s * stage_bytes;
                    const uint32_t scale_bytes = min(P.tiles - ks * 2u, 2u) * 512u;
                    tc::bar_expect(&S.full[s], kMmM * 128 + P.bn * 128 + scale_bytes * (1 + scale_rows));
                    tc::tile_load(st, &map_a, ks * 128, tm * kMmM, &S.full[s]);
                    tc::tile_load(st + kMmM * 128, &map_b, ks * 128, n0, &S.full[s]);
                    uint8_t *sc = st + kMmM * 128 + P.bn * 128;
                    tc::bulk_load(sc, as + ks * 1024u, scale_bytes, &S.full[s]);
                    for (uint32_t r = 0; r < scale_rows; ++r)   // (rows past the last tile, whose products nobody stores: the last one's)
                        tc::bulk_load(sc + 1024 * (1 + r), P.bs + ((size_t)min(n0 / 128 + r, P.b_rows - 1) * P.tiles + ks * 2) * 512, scale_bytes, &S.full[s]);
                    ++armed;
                    if (++s == P.stages)
                        s = 0, phase ^= 1u;
                }
            }
            if (!ok)   // copies in flight end before the CTA does
                for (uint32_t i = 0; i < P.stages && i < armed; ++i) {
                    const uint32_t at = (armed - 1 - i) % P.stages;
                    tc::bar_drain(&S.full[at], ((armed - 1 - i) / P.stages) & 1u);
                }
        }
        __syncwarp();
    } else if (warp == kMmEpilogue + 1) {
        const uint32_t e = tc::elect(), instruction = tc::mx4_instruction(P.bn);
        const uint32_t a0 = tc::desc_low(ring), b0 = a0 + kMmM * 8, sc0 = b0 + P.bn * 8, step16 = stage_bytes >> 4;
        uint32_t s = 0, phase = 0, turn = 0;
        bool ok = true;
        for (uint32_t tile = blockIdx.x; ok && tile < P.n_tiles; tile += gridDim.x, turn ^= 1u) {
            const uint32_t n0 = tile / P.tiles_m * P.bn;
            const uint32_t shift = (n0 & 127u) >> 5;   // columns of the first tile of scales ahead of row n0
            if (!(ok = tc::bar_wait(&S.taken, turn ^ 1u, dead)))
                break;
            tc::fence_after();
            for (uint32_t ks = 0; ks < P.stages_k; ++ks) {
                if (!(ok = tc::bar_wait(&S.full[s], phase, dead)))
                    break;
                tc::fence_after();
                const uint32_t steps = P.k64 - ks * 4u, sa = kMmScaleColumn + s * 32u, sb = sa + 8u;
                const uint32_t a = a0 + s * step16, b = b0 + s * step16, sc = sc0 + s * step16;
#pragma unroll
                for (uint32_t t = 0; t < 2; ++t)
                    if (2 * t < steps) {
                        tc::scales_copy(e, sa + 4 * t, sc + 32 * t);
                        tc::scales_copy(e, sb + 8 * t, sc + 64 + 32 * t);
                        if (scale_rows > 1)
                            tc::scales_copy(e, sb + 8 * t + 4, sc + 128 + 32 * t);
                    }
#pragma unroll
                for (uint32_t t = 0; t < 2; ++t) {
                    if (2 * t < steps)
                        tc::mx4_product<0>(e, 0, a + 4 * t, b + 4 * t, instruction, sa + 4 * t, sb + 8 * t + shift, ks + t);
                    if (2 * t + 1 < steps)
                        tc::mx4_product<1>(e, 0, a + 4 * t + 2, b + 4 * t + 2, instruction, sa + 4 * t, sb + 8 * t + shift, 1);
                }
                tc::commit(e, &S.empty[s]);
                if (++s == P.stages)
                    s = 0, phase ^= 1u;
            }
            if (ok)
                tc::commit(e, &S.sums);
        }
        if (!ok) {   // products in flight end before tensor memory is given back
            tc::commit(e, &S.drain);
            tc::bar_drain(&S.drain, 0);
        }
        __syncwarp();
    } else {
        uint32_t turn = 0;
        bool ok = true;
        const uint32_t half = P.bn / 2, c0 = (warp >> 2) * half, groups = half / 32;
        const bool wide = ((P.ld * sizeof(T)) | (uintptr_t)out) % 32 == 0;
        float(*stage)[33] = (float(*)[33])(ring + P.stages * stage_bytes) + warp * 32;
        for (uint32_t tile = blockIdx.x; tile < P.n_tiles; tile += gridDim.x, turn ^= 1u) {
            const int64_t row0 = (int64_t)(tile % P.tiles_m) * kMmM + (warp & 3) * 32, col0 = (int64_t)(tile / P.tiles_m) * P.bn + c0;
            ok = ok && tc::bar_wait(&S.sums, turn, dead);
            ok = __all_sync(0xffffffffu, ok);
            if (ok)
                tc::fence_after();
            // 64 columns at a time: with all 128 of a warp in registers the kernel spilled
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                uint32_t v[2][32];
                if (ok) {
#pragma unroll
                    for (uint32_t g = 0; g < 2; ++g)
                        if (2 * h + g < groups)
                            tc::tmem_load32(((uint32_t)(warp & 3) << 21) + c0 + (2 * h + g) * 32, v[g]);
                    tc::tmem_load_wait();
                    if (h == 1) {
                        tc::fence_before();
                        __syncwarp();
                        if (lane == 0)
                            tc::bar_arrive(&S.taken);
                    }
                } else {   // a wait ran out: what was not computed is NaN
#pragma unroll
                    for (uint32_t g = 0; g < 2; ++g)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            v[g][i] = 0x7FFFFFFFu;
                }
#pragma unroll
                for (uint32_t g = 0; g < 2; ++g) {
                    const int64_t col = col0 + (2 * h + g) * 32;
                    if (2 * h + g < groups && col < P.n) {
                        if (wide && col + 32 <= P.n) {
                            if (row0 + lane < P.m)
                                store32<T>(out + (row0 + lane) * P.ld + col, v[g]);
                        } else {
                            // lanes hold rows: turned in shared memory, so that a warp stores 32 outputs of a row
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                stage[lane][i] = __uint_as_float(v[g][i]);
                            __syncwarp();
                            const int rows = (int)max((int64_t)0, min((int64_t)32, P.m - row0));
                            if (col + lane < P.n)
                                for (int r = 0; r < rows; ++r)
                                    out[(row0 + r) * P.ld + col + lane] = from_f32<T>(stage[r][lane]);
                            __syncwarp();
                        }
                    }
                }
            }
        }
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == 0)
        tc::tmem_free(0, kMmColumns);
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
// `rows` rows of codes, copied in tiles of 128 bytes by `box` rows; what lies past either end is zero
static bool codes_map(CUtensorMap *map, const void *codes, int64_t rows, int64_t row_bytes, uint32_t box)
{
    const cuuint64_t dims[2] = {(cuuint64_t)row_bytes, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)row_bytes};
    const cuuint32_t tile[2] = {128, box}, steps[2] = {1, 1};
    return encode_tiled() && encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void *)codes, dims, strides, tile, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Columns per tile: the width whose waves of tiles over the SMs cost least, a tile's cost taken as its width and 64 columns
// more for what does not depend on it
static uint32_t mm_columns(int64_t m, int64_t n)
{
    const int64_t tiles_m = (m + kMmM - 1) / kMmM;
    int64_t least = 0;
    uint32_t best = 0;
    for (uint32_t bn = 256; bn >= 64; bn -= 64) {
        const int64_t cost = (tiles_m * ((n + bn - 1) / bn) + kPlanSMs - 1) / kPlanSMs * (bn + 64);
        if (!best || cost < least)
            best = bn, least = cost;
    }
    return best;
}

template <class T>
static int matmul(const uint8_t *a, const uint8_t *as, int64_t m, const uint8_t *b, const uint8_t *bs, int64_t n, int64_t k, T *out, int64_t ld, cudaStream_t s)
{
    MmArgs P;
    P.as = as;
    P.bs = bs;
    P.m = m;
    P.n = n;
    P.ld = ld;
    P.k64 = (uint32_t)((k + 63) / 64);
    P.stages_k = (uint32_t)((k + kMmK - 1) / kMmK);
    P.tiles = (uint32_t)mx4_scale_tiles(k);
    P.b_rows = (uint32_t)((n + 127) / 128);
    P.bn = mm_columns(m, n);
    P.tiles_m = (uint32_t)((m + kMmM - 1) / kMmM);
    const int64_t tiles = (int64_t)P.tiles_m * ((n + P.bn - 1) / P.bn);
    if (tiles >= (1ll << 32) - kPlanSMs)
        return CONEF_ERR_UNSUPPORTED;
    P.n_tiles = (uint32_t)tiles;
    // (the staging is left out where no store needs it)
    const bool wide = n % 32 == 0 && ((ld * sizeof(T)) | (uintptr_t)out) % 32 == 0;
    const uint32_t room = 224 * 1024 - 1024 - (wide ? 0 : kMmStaging);
    P.stages = std::min<uint32_t>({(uint32_t)kMmMaxStages, room / mm_stage_bytes(P.bn), std::max(2u, P.stages_k)});
    CUtensorMap map_a, map_b;
    const int64_t row_bytes = mx4_blocks(k) * 16;
    if (!codes_map(&map_a, a, m, row_bytes, kMmM) || !codes_map(&map_b, b, n, row_bytes, P.bn))
        return launched(cudaErrorInvalidValue, "conef_mx4_matmul: tensor map");
    const size_t smem = 1024 + (size_t)P.stages * mm_stage_bytes(P.bn) + (wide ? 0 : kMmStaging);
    static int done[64];
    cudaError_t e = opt_in_smem(k_mx4_matmul<T>, 224 * 1024, done);
    if (e == cudaSuccess)
        e = launch(k_mx4_matmul<T>, dim3(std::min<uint32_t>(P.n_tiles, kPlanSMs)), kMmThreads, smem, s, map_a, map_b, P, out);
    return launched(e, "conef_mx4_matmul");
}

}  // namespace conef

using namespace conef;

extern "C" int conef_mx4_matmul(const void *a_codes, const void *a_scales, int64_t m, const void *b_codes, const void *b_scales, int64_t n, int64_t k,
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
        return matmul<T>((const uint8_t *)a_codes, (const uint8_t *)a_scales, m, (const uint8_t *)b_codes, (const uint8_t *)b_scales, n, k, (T *)out, ld,
                         (cudaStream_t)stream);
    });
}
