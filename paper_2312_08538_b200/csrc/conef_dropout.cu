// Dropout whose mask is drawn from the counter-based stream in every pass and never stored: y = x 65536 / (65536 - off)
// where the element's number is at least off, else 0; and a residual added in the same pass.
//
// HBM-bound: 2 or 3 values per element (8192 x 6400 in bf16 35 us, 6.0 TB/s, launches on one output; as a call whose output is allocated 5.5).  A hash (two 64-bit multiplies, about 22 instructions) serves four elements, so a thread works on 16
// bytes at a time and hashes once for four or twice for eight of them.
#include <algorithm>

#include "conef_draw.cuh"
#include "conef_common.cuh"
#include "conef_elem.cuh"

namespace conef {

constexpr int kDropThreads = 256;

template <class T, bool ADD>
__device__ __forceinline__ uint4 dropped(const uint4 &x, const uint4 &add, uint32_t kept, float scale)
{
    constexpr int N = Vec16<T>::N;
    float v[N], r[N];
    Vec16<T>::unpack(x, v);
    if (ADD)
        Vec16<T>::unpack(add, r);
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const float base = ADD ? r[q] : 0.f, y = ADD ? __fmaf_rn(v[q], scale, r[q]) : __fmul_rn(v[q], scale);
        v[q] = (kept >> q) & 1u ? y : base;
    }
    return Vec16<T>::pack(v);
}
template <class T, bool ADD>
__device__ __forceinline__ void dropped_one(const T *x, const T *add, T *out, bool kept, float scale)
{
    // (without a residual a product, as in dropped(): -0 is added, which leaves a zero its sign)
    const float base = ADD ? to_f32(*add) : 0.f;
    *out = from_f32<T>(kept ? __fmaf_rn(to_f32(*x), scale, ADD ? base : -0.f) : base);
}

// ------------------------------------------------------------------ rows that are one array
// With rows one behind the other and whole groups of four columns in each (or one row), the group of an element is its
// place in the array over four, whatever row that is.  16 bytes per thread, U times.
template <class T, bool ADD, int U>
__global__ void __launch_bounds__(kDropThreads) k_dropout_flat(const T *x, const T *add, T *out, int64_t n, uint64_t base, const Dropout drop)
{
    constexpr int N = Vec16<T>::N;
    grid_release();
    const int64_t c0 = (int64_t)blockIdx.x * (kDropThreads * U) + threadIdx.x, whole = n / N;
    grid_wait();
    uint4 v[U], r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t c = c0 + u * kDropThreads;
        if (c < whole) {
            v[u] = __ldcs((const uint4 *)x + c);
            if (ADD)
                r[u] = __ldcs((const uint4 *)add + c);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t c = c0 + u * kDropThreads;
        const uint64_t z = base + kDrawStep * (uint64_t)(c * (N / 4));
        uint32_t kept = dropout_kept(mix64(z), drop);
        if (N == 8)
            kept |= dropout_kept(mix64(z + kDrawStep), drop) << 4;
        kept |= drop.all;
        if (c < whole) {
            ((uint4 *)out)[c] = dropped<T, ADD>(v[u], r[u], kept, drop.scale);
        } else if (c == whole) {
            for (int q = 0; q < (int)(n - whole * N); ++q)
                dropped_one<T, ADD>(x + c * N + q, add + c * N + q, out + c * N + q, (kept >> q) & 1u, drop.scale);
        }
    }
}

// ------------------------------------------------------------------ rows that are one array of any width
// A thread's 16 bytes begin anywhere in a row: of the groups that they lie in it hashes all but the last, whose mask the next lane has (the last
// lane's is that of a warp's next step).  Where a row ends among them, it hashes all that it needs.  `shift` is the number of elements by which the array begins behind a 16-byte boundary.
// 60000 x 1301 in fp32: a warp per row, edges element by element, 134 us; this 100 (6.2 TB/s), without the last lanes' exchange 118.  In bf16, which
// is bound by the hashes' instructions, 88 and 76 us.
template <class T, bool ADD, int U>
__global__ void __launch_bounds__(kDropThreads) k_dropout_array(const T *x, const T *add, T *out, uint32_t n, uint32_t shift, const Divider width, uint64_t base,
                                                                const Dropout drop)
{
    constexpr int N = Vec16<T>::N;
    grid_release();
    const uint32_t lane = threadIdx.x & 31, c0 = (blockIdx.x * kDropThreads + (threadIdx.x & ~31u)) * U + lane, cols = width.by, groups = (cols + 3) / 4;
    const uint64_t end = (uint64_t)n + shift;
    x -= shift, add -= shift, out -= shift;
    grid_wait();
    uint4 v[U], r[U];
    uint32_t row[U], col[U], mask[U];
    auto mask_of = [&](uint32_t row, uint32_t group, int words) {
        const uint64_t z = base + kDrawStep * (uint64_t)(row * groups + group);   // (no more groups than elements)
        uint32_t m = dropout_kept(mix64(z), drop);
        if (words > 1)
            m |= dropout_kept(mix64(z + kDrawStep), drop) << 4;
        if (words > 2)
            m |= dropout_kept(mix64(z + 2 * kDrawStep), drop) << 8;
        return m;
    };
    auto full = [&](int u) {
        const uint64_t at = (uint64_t)(c0 + u * 32) * N;
        return at >= shift && at + N <= end;
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t c = c0 + u * 32;
        if (full(u)) {
            v[u] = __ldcs((const uint4 *)x + c);
            if (ADD)
                r[u] = __ldcs((const uint4 *)add + c);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t at = (uint64_t)(c0 + u * 32) * N;   // counted from the boundary ahead of the array
        const uint32_t first = (uint32_t)min(at < shift ? (uint64_t)0 : at - shift, (uint64_t)n - 1u);
        row[u] = divide(first, width);
        col[u] = first - row[u] * cols;
        mask[u] = mask_of(row[u], col[u] >> 2, N / 4);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t at = (uint64_t)(c0 + u * 32) * N;
        const uint32_t lead = at < shift ? shift - (uint32_t)at : 0u, s = col[u] & 3u;
        // the group behind: the first one of the next lane, whose piece continues this row
        uint32_t next = __shfl_sync(0xffffffffu, lane == 0 && u + 1 < U ? mask[u + 1 < U ? u + 1 : u] : mask[u], (lane + 1) & 31);
        uint32_t kept;
        if (s == 0 ? cols - col[u] >= N : cols - col[u] > N) {
            if (u + 1 == U && lane == 31 && s)
                next = mask_of(row[u], (col[u] >> 2) + N / 4, 1);
            kept = ((mask[u] | next << N) >> s) << lead;
        } else {   // a row ends here: what is left of it, and the first groups of the next, while there are any
            uint32_t rr = row[u], have = cols - col[u];
            if (have + s > N)
                next = mask_of(rr, (col[u] >> 2) + N / 4, 1);
            kept = ((mask[u] | next << N) >> s & ((1u << have) - 1u)) << lead;
            for (have += lead; have < N; have += cols)
                kept |= (mask_of(++rr, 0, N / 4) & (cols < N ? (1u << cols) - 1u : (1u << N) - 1u)) << have;
        }
        kept |= drop.all;
        if (full(u)) {
            ((uint4 *)out)[at / N] = dropped<T, ADD>(v[u], r[u], kept, drop.scale);
        } else {
            for (uint32_t q = lead; q < N && at + q < end; ++q)
                dropped_one<T, ADD>(x + at + q, add + at + q, out + at + q, (kept >> q) & 1u, drop.scale);
        }
    }
}

// ------------------------------------------------------------------ rows that begin anywhere
// A row is cut at 16-byte boundaries; `lanes` lanes (a power of two) walk along it, or along kDropRun steps of it.  The columns of a lane's 16
// bytes begin s columns before a group of its own hash, s the same in the whole row, so it takes the upper bits of its own mask and the
// lower ones of that of the lane before; the last lane hands its mask on to the next step.  Rows of x, add and out begin
// equally far from a boundary.
constexpr int kDropRun = 16;   // steps of a warp along a row
template <class T, bool ADD>
__global__ void __launch_bounds__(kDropThreads) k_dropout_rows(const T *x, const T *add, T *out, int64_t rows, int64_t cols, int64_t x_ld, int64_t add_ld,
                                                               int64_t out_ld, int64_t runs, int lanes, uint64_t base, const Dropout drop)
{
    constexpr int N = Vec16<T>::N;
    grid_release();
    const int lane = threadIdx.x & 31, sub = lane & (lanes - 1), before = (lane & ~(lanes - 1)) | ((lane - 1) & (lanes - 1));
    const int64_t unit = ((int64_t)blockIdx.x * kDropThreads + threadIdx.x) / lanes;
    int64_t row = unit / runs;
    const int64_t run = unit - row * runs;
    const bool there = row < rows;
    row = there ? row : 0;
    const T *xr = x + row * x_ld;
    const uint32_t s = (uint32_t)((uintptr_t)xr / sizeof(T)) % N;
    xr -= s;
    const T *ar = ADD ? add + row * add_ld - s : nullptr;
    T *yr = out + row * out_ld - s;
    const int64_t steps = there ? (cols + s + N - 1) / N : 0;   // pieces of 16 bytes
    const int64_t end = min(steps, (run + 1) * kDropRun * lanes);
    const uint64_t row_base = base + kDrawStep * (uint64_t)(row * ((cols + 3) / 4));
    auto mask_of = [&](int64_t c) {
        const uint64_t z = row_base + kDrawStep * (uint64_t)(c * (N / 4));
        uint32_t m = dropout_kept(mix64(z), drop);
        if (N == 8)
            m |= dropout_kept(mix64(z + kDrawStep), drop) << 4;
        return m;
    };
    int64_t c = run * kDropRun * lanes + sub;
    uint32_t last = run > 0 ? mask_of(run * kDropRun * lanes - 1) : 0u;   // (used of the last lane)
    grid_wait();
    // (all lanes of a warp take the same number of steps: the shuffles are theirs together)
    const int64_t left = end - run * kDropRun * lanes;   // at most kDropRun * lanes
    const uint32_t most = __reduce_max_sync(0xffffffffu, left > 0 ? (uint32_t)(left + lanes - 1) / (uint32_t)lanes : 0u);
    for (uint32_t i = 0; i < most; ++i, c += lanes) {
        const int64_t col = c * N - s;
        const bool mine = c < end, full = mine && col >= 0 && col + N <= cols;
        uint4 v, r;
        if (full) {
            v = __ldcs((const uint4 *)(xr + c * N));
            if (ADD)
                r = __ldcs((const uint4 *)(ar + c * N));
        }
        const uint32_t mask = mask_of(c);
        const uint32_t prev = __shfl_sync(0xffffffffu, sub == lanes - 1 ? last : mask, before);
        last = mask;
        const uint32_t kept = ((prev | mask << N) >> (N - s)) | drop.all;
        if (full) {
            *(uint4 *)(yr + c * N) = dropped<T, ADD>(v, r, kept, drop.scale);
        } else if (mine) {
#pragma unroll
            for (int q = 0; q < N; ++q)
                if (col + q >= 0 && col + q < cols)
                    dropped_one<T, ADD>(xr + c * N + q, ar + c * N + q, yr + c * N + q, (kept >> q) & 1u, drop.scale);
        }
    }
}

// ------------------------------------------------------------------ rows that begin differently: a group of four columns per thread
// Element by element, since no 16 bytes of one lie on 16 of the other: 8192 x 6400 in bf16 83 us (2.5 TB/s; rows that begin alike 35).
template <class T, bool ADD>
__global__ void __launch_bounds__(kDropThreads) k_dropout(const T *x, const T *add, T *out, int64_t rows, uint32_t cols, int64_t x_ld, int64_t add_ld,
                                                          int64_t out_ld, uint64_t stream, const Dropout drop)
{
    grid_release();
    const uint32_t groups = (cols + 3) / 4;
    grid_wait();
    for (int64_t i = (int64_t)blockIdx.x * kDropThreads + threadIdx.x; i < rows * groups; i += (int64_t)gridDim.x * kDropThreads) {
        const int64_t row = i / groups;
        const uint32_t c0 = (uint32_t)(i - row * groups) * 4u;
        const uint32_t kept = dropout_kept(draw_word(stream, (uint64_t)i, kDrawDropout), drop) | drop.all;
        const T *xr = x + row * x_ld + c0, *ar = add + row * add_ld + c0;
        T *yr = out + row * out_ld + c0;
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
            if (c0 + q < cols)
                dropped_one<T, ADD>(xr + q, ar + q, yr + q, (kept >> q) & 1u, drop.scale);
    }
}

template <class T, bool ADD>
static cudaError_t dropout(const T *x, const T *add, T *out, int64_t rows, int64_t cols, int64_t x_ld, int64_t add_ld, int64_t out_ld, uint64_t stream,
                           const Dropout &drop, cudaStream_t s)
{
    constexpr int N = Vec16<T>::N;
    const uint64_t base = draw_base(stream, kDrawDropout);
    const uintptr_t off = ((uintptr_t)x | (uintptr_t)out | (uintptr_t)add) & 15;
    const bool one = rows == 1 || (x_ld == cols && out_ld == cols && (!ADD || add_ld == cols));
    if (one && off == 0 && (cols % 4 == 0 || rows == 1)) {
        const int64_t n = rows * cols, pieces = (n + N - 1) / N;
        // two per thread where that still makes some CTAs per SM
        if (pieces >= (int64_t)kDropThreads * 2 * kPlanSMs * 4)
            return launch(k_dropout_flat<T, ADD, 2>, dim3((unsigned)((pieces + 2 * kDropThreads - 1) / (2 * kDropThreads))), kDropThreads, 0, s, x, add, out, n, base, drop);
        return launch(k_dropout_flat<T, ADD, 1>, dim3((unsigned)((pieces + kDropThreads - 1) / kDropThreads)), kDropThreads, 0, s, x, add, out, n, base, drop);
    }
    const bool same = (((uintptr_t)x ^ (uintptr_t)out) & 15) == 0 && (!ADD || (((uintptr_t)x ^ (uintptr_t)add) & 15) == 0);
    if (one && same && cols > 1 && rows * cols < (1ll << 32) - 16) {
        const uint32_t n = (uint32_t)(rows * cols), shift = (uint32_t)(((uintptr_t)x & 15) / sizeof(T));
        const int64_t pieces = ((int64_t)n + shift + N - 1) / N;
        constexpr int U = ADD ? 2 : 4;
        if (pieces >= (int64_t)kDropThreads * U * kPlanSMs * 4)
            return launch(k_dropout_array<T, ADD, U>, dim3((unsigned)((pieces + U * kDropThreads - 1) / (U * kDropThreads))), kDropThreads, 0, s, x, add, out, n, shift,
                          divider((uint32_t)cols), base, drop);
        return launch(k_dropout_array<T, ADD, 1>, dim3((unsigned)((pieces + kDropThreads - 1) / kDropThreads)), kDropThreads, 0, s, x, add, out, n, shift,
                      divider((uint32_t)cols), base, drop);
    }
    auto alike = [&](const T *p, int64_t ld) { return (((uintptr_t)p - (uintptr_t)x) & 15) == 0 && (rows == 1 || ((ld - x_ld) * (int64_t)sizeof(T)) % 16 == 0); };
    if (alike(out, out_ld) && (!ADD || alike(add, add_ld))) {
        const int64_t pieces = (cols + 2 * N - 2) / N;   // of a row, wherever it begins
        int lanes = 1;
        while (lanes < 32 && lanes < pieces)
            lanes *= 2;
        const int64_t runs = (pieces + (int64_t)kDropRun * lanes - 1) / ((int64_t)kDropRun * lanes), ctas = (rows * runs * lanes + kDropThreads - 1) / kDropThreads;
        if (ctas < (1ll << 31))
            return launch(k_dropout_rows<T, ADD>, dim3((unsigned)ctas), kDropThreads, 0, s, x, add, out, rows, cols, x_ld, add_ld, out_ld, runs, lanes, base, drop);
    }
    const int64_t ctas = (rows * ((cols + 3) / 4) + kDropThreads - 1) / kDropThreads;
    return launch(k_dropout<T, ADD>, dim3((unsigned)std::min<int64_t>(ctas, kPlanSMs * 64)), kDropThreads, 0, s, x, add, out, rows, (uint32_t)cols, x_ld, add_ld, out_ld,
                  stream, drop);
}

}  // namespace conef

using namespace conef;

extern "C" int conef_dropout(const void *x, const void *add, void *out, int dtype, int64_t rows, int64_t cols, int64_t x_ld, int64_t add_ld,
                             int64_t out_ld, double p, const conef_draw *draw, conef_stream stream)
{
    int rc = check_matrix(x, dtype, rows, cols, x_ld);
    if (rc == CONEF_OK)
        rc = check_matrix(out, dtype, rows, cols, out_ld);
    if (rc == CONEF_OK && add)
        rc = check_matrix(add, dtype, rows, cols, add_ld);
    if (rc == CONEF_OK && !(p >= 0.0 && p <= 1.0))
        rc = CONEF_ERR_INVALID_ARG;
    if (rc == CONEF_OK)
        rc = check_draw(draw);
    if (rc != CONEF_OK || rows == 0 || cols == 0)
        return rc;
    const uint64_t st = draw_stream(draw->seed, draw->worker, draw->tensor, draw->step);
    const Dropout drop = dropout_of(p);
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        return launched((add ? dropout<T, true> : dropout<T, false>)((const T *)x, (const T *)add, (T *)out, rows, cols, x_ld, add_ld, out_ld, st, drop, (cudaStream_t)stream),
                        "conef_dropout");
    });
}
