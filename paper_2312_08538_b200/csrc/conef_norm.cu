// Root-mean-square norm of rows with the residual's addition, into the rows' type or into 8-bit floats with block scales (conef_f8.cuh), and its gradient.
#include <algorithm>

#include "conef_f8.cuh"

namespace conef {

struct NormArgs {
    const void *x, *add, *w;
    void *h, *y;
    uint8_t *codes, *scales;
    float *rstd;
    int64_t rows, cols;
    uint32_t x_ld, add_ld, h_ld, y_ld;
    double eps, share;   // share: of a column in the mean
    int kind;
    bool w32, aligned32, aligned_w;
};

// ------------------------------------------------------------------ rows by blocks
// A lane has 8 elements of a row and a block all of it, 256 elements to a warp (rows of up to 256: a warp has all of it); blocks stay and take rows a grid apart.  So
// little to a lane leaves room for 32 warps on an SM, which hide what is done once per row: sums across lanes and warps, a barrier, the root.  The rows ahead
// are copied into shared memory meanwhile, DEPTH of them, each lane what it will read: 6.5 TB/s are 44 KB on their way to each SM at a latency of a microsecond.
// Rows on odd addresses, which copies would take four bytes at a time or not at all, are read when they are wanted, by the norm one row ahead (30011 x 1301
// in fp32 and its gradient by copies of four bytes 73 and 111 us, as they are wanted 71 and 85, ahead in registers 61 and 129).
// 8192 x 1600 in bf16 with a residual, and the gradient: 16 elements to a lane 37 and 39 us, 32 elements 35 and 51, 8 with one row ahead in registers 27 and 32.
constexpr int kNormPer = 8, kNormWarp = 32 * kNormPer;   // elements of a lane and of a warp
constexpr int64_t kNormWidest = 32 * kNormWarp;
template <class T, bool VEC>
using NormPiece = Piece<T, VEC, kNormPer>;

template <class T, bool VEC, int ARRAYS>
struct Ahead {
    static constexpr bool ON = VEC;
    static constexpr int CHUNK = 16, PER = CHUNK / (int)sizeof(T), CHUNKS = kNormPer / PER;   // bytes and elements of a copy; copies per array
    static constexpr int STAGE = ARRAYS * kNormWarp * (int)sizeof(T), FIT = 6144 / STAGE, DEPTH = !ON ? 1 : FIT < 4 ? FIT : 4;   // (6 KB to each of 32 warps)
    static constexpr int BYTES = ON ? STAGE * DEPTH : 0;                                                               // of a warp

    uint8_t *at;   // the lane's place
    uint32_t c0, cols;
    int lane, now, next;

    __device__ __forceinline__ Ahead(uint8_t *smem, int warp, int lane, uint32_t c0, uint32_t cols)
        : at(smem + warp * BYTES + lane * CHUNK), c0(c0), cols(cols), lane(lane), now(0), next(0)
    {
    }
    __device__ __forceinline__ uint32_t first(int i) const { return c0 + lane * kNormPer + i * PER; }
    // asks for a row's elements; then close(), once for all arrays (also where there is no row any more)
    __device__ __forceinline__ void ask(int array, const T *row) const
    {
        if constexpr (ON) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const uint32_t c = first(i), to = (uint32_t)__cvta_generic_to_shared(at + next * STAGE + (array * CHUNKS + i) * (32 * CHUNK));
                if (c < cols)   // (zeros behind the row's end)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(row + c), "r"(min((cols - c) * (uint32_t)sizeof(T), 16u)) : "memory");
            }
        }
    }
    __device__ __forceinline__ void close()
    {
        if constexpr (ON) {
            asm volatile("cp.async.commit_group;" ::: "memory");
            next = next + 1 == DEPTH ? 0 : next + 1;
        }
    }
    // waits for the oldest row asked for, DEPTH being; take()s of its arrays follow, then done()
    static __device__ __forceinline__ void wait()
    {
        if constexpr (ON)
            asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
    }
    __device__ __forceinline__ void take(int array, const T *row, NormPiece<T, VEC> &p) const
    {
        if constexpr (ON) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const uint8_t *const from = at + now * STAGE + (array * CHUNKS + i) * (32 * CHUNK);
                const uint4 w = first(i) < cols ? *(const uint4 *)from : make_uint4(0u, 0u, 0u, 0u);
                p.w[4 * i] = w.x, p.w[4 * i + 1] = w.y, p.w[4 * i + 2] = w.z, p.w[4 * i + 3] = w.w;
            }
        } else {
            p.load(row, c0, cols, lane, false);
        }
    }
    __device__ __forceinline__ void done()
    {
        if constexpr (ON)
            now = now + 1 == DEPTH ? 0 : now + 1;
    }
};

// the weights of a lane's columns (aligned: 16 bytes of them are)
template <class T, bool VEC>
__device__ __forceinline__ void load_weights(const void *w, bool w32, bool aligned, uint32_t c0, uint32_t cols, int lane, float *v)
{
    constexpr int N = kNormPer;
    const uint32_t c = c0 + lane * N;
    if (VEC && aligned && c + N <= cols) {
        if (w32) {
#pragma unroll
            for (int q = 0; q < N; q += 4)
                Vec16<float>::unpack(*(const uint4 *)((const float *)w + c + q), *(float(*)[4])(v + q));
        } else {
#pragma unroll
            for (int q = 0; q < N; q += Vec16<T>::N)
                Vec16<T>::unpack(*(const uint4 *)((const T *)w + c + q), *(float(*)[Vec16<T>::N])(v + q));
        }
        return;
    }
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const uint32_t i = lane_col<VEC, N>(c0, lane, q);
        v[q] = i >= cols ? 0.f : w32 ? ((const float *)w)[i] : to_f32(((const T *)w)[i]);
    }
}

// 1 / sqrt(m) to 64 bits' precision: two steps of Newton's iteration from fp32's estimate, whose relative error of 2^-22 each squares (times 3/2).  (Divided and
// rooted by the 64-bit functions, which are long, a row took a microsecond more.)
__device__ __forceinline__ double root_of(double m)
{
    if (!(m > 1e-30 && m < 1e30))
        return 1.0 / sqrt(m);
    double r = (double)rsqrtf((float)m);
    const double half = 0.5 * m;
    r = r * __fma_rn(-half * r, r, 1.5);
    return r * __fma_rn(-half * r, r, 1.5);
}
// what a lane's elements become behind the norm
template <class T, bool VEC>
__device__ __forceinline__ void norm_finish(const NormArgs &A, const NormPiece<T, VEC> &p, const float *w, float root, uint32_t c0, int lane, uint32_t row)
{
    constexpr int N = kNormPer;
    float v[N];
    p.unpack(v);
    if (A.codes) {
        const uint32_t blocks = ((uint32_t)A.cols + 127u) / 128u;
        uint8_t *const scales = A.scales + f8_scale_at32(row, c0 / 128u, ((uint32_t)A.cols + 511u) / 512u);
        norm_values<N>(v, w, root, lane_col<VEC, N>(c0, lane, 0) < (uint32_t)A.cols);
        f8_store_row<T, VEC, N>(v, c0, blocks, lane, A.kind, true, A.codes + (uint64_t)row * (blocks * 128u), scales);
        if (c0 % 512 == 0 && c0 + kNormWarp >= (uint32_t)A.cols && lane < 2)   // (the last tile's second half)
            scales[2 + lane] = 0;
    } else {
#pragma unroll
        for (int q = 0; q < N; ++q)
            v[q] = __fmul_rn(__fmul_rn(v[q], root), w[q]);
        NormPiece<T, VEC> o;
        o.pack(v);
        o.store((T *)A.y + (uint64_t)row * A.y_ld, c0, (uint32_t)A.cols, lane, A.aligned32);
    }
}
// h, rounded to its type
template <class T, bool VEC>
__device__ __forceinline__ void norm_join(NormPiece<T, VEC> &p, const NormPiece<T, VEC> &o)
{
    float a[kNormPer], b[kNormPer];
    p.unpack(a), o.unpack(b);
#pragma unroll
    for (int q = 0; q < kNormPer; ++q)
        a[q] = __fadd_rn(a[q], b[q]);
    p.pack(a);
}
// Squares are summed in 64 bits, which fp32's rounding of the root then does not show: a row's values, and so the codes, do not depend on how it is cut.
template <class T, bool VEC>
__device__ __forceinline__ double norm_squares(const NormPiece<T, VEC> &p)
{
    float v[kNormPer];
    p.unpack(v);
    double a = 0, b = 0;
#pragma unroll
    for (int q = 0; q < kNormPer; q += 2) {
        a = __fma_rn((double)v[q], (double)v[q], a);
        b = __fma_rn((double)v[q + 1], (double)v[q + 1], b);
    }
    return a + b;
}
template <class V>
__device__ __forceinline__ V warp_sum(V v)
{
#pragma unroll
    for (int o = 16; o; o /= 2)
        v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// scales of rows that do not exist, from `row` on
__device__ __forceinline__ void norm_no_rows(const NormArgs &A, int64_t row, int64_t step, uint32_t thread, uint32_t threads)
{
    const int64_t tiles = f8_scale_tiles(A.cols);
    for (; row < (A.rows + 127) / 128 * 128; row += step)
        for (uint32_t t = thread; t < (uint32_t)tiles; t += threads)
            *(uint32_t *)(A.scales + f8_scale_at(row, t * 4, tiles)) = 0u;
}
// ALONE: a warp has a row
template <class T, bool VEC, bool ALONE>
__global__ void __launch_bounds__(ALONE ? 256 : 1024, ALONE ? 4 : 1) k_rms_norm(const __grid_constant__ NormArgs A)
{
    extern __shared__ __align__(16) uint8_t norm_smem[];
    __shared__ double part[2][32];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const uint32_t cols = (uint32_t)A.cols, c0 = ALONE ? 0u : warp * kNormWarp;
    uint32_t row = ALONE ? blockIdx.x * 8 + warp : blockIdx.x;   // (rows are fewer than 2^31)
    const uint32_t step = ALONE ? gridDim.x * 8 : gridDim.x;
    grid_wait();
    float w[kNormPer];
    load_weights<T, VEC>(A.w, A.w32, A.aligned_w, c0, cols, lane, w);
    Ahead<T, VEC, 2> rows(norm_smem, warp, lane, c0, cols);
    const T *const x = (const T *)A.x, *const add = (const T *)A.add;
    NormPiece<T, VEC> x_next, a_next;   // (where copies are not ON)
    auto ask = [&](uint32_t row) {
        if (row < (uint32_t)A.rows) {
            if constexpr (rows.ON) {
                rows.ask(0, x + (uint64_t)row * A.x_ld);
                if (add)
                    rows.ask(1, add + (uint64_t)row * A.add_ld);
            } else {
                x_next.load(x + (uint64_t)row * A.x_ld, c0, cols, lane, false);
                if (add)
                    a_next.load(add + (uint64_t)row * A.add_ld, c0, cols, lane, false);
            }
        }
        rows.close();
    };
    if constexpr (!rows.ON)
        ask(row);
#pragma unroll
    for (int d = 0; d < rows.DEPTH - 1; ++d)
        ask(row + d * step);
    for (int turn = 0; row < (uint32_t)A.rows; row += step, turn ^= 1) {
        NormPiece<T, VEC> p = x_next, a = a_next;
        ask(row + (rows.ON ? rows.DEPTH - 1 : 1) * step);
        rows.wait();
        if constexpr (rows.ON)
            rows.take(0, x + (uint64_t)row * A.x_ld, p);
        if (add) {
            if constexpr (rows.ON)
                rows.take(1, add + (uint64_t)row * A.add_ld, a);
            norm_join(p, a);
            p.store((T *)A.h + (uint64_t)row * A.h_ld, c0, cols, lane, A.aligned32);
        }
        rows.done();
        double sum = warp_sum(norm_squares(p));
        if constexpr (!ALONE) {
            if (lane == 0)
                part[turn][warp] = sum;
            __syncthreads();
            sum = warp_sum(lane < warps ? part[turn][lane] : 0.0);
        }
        const float root = (float)root_of(__fma_rn(sum, A.share, A.eps));
        if ((ALONE || warp == 0) && lane == 0)
            A.rstd[row] = root;
        if (A.y || A.codes)
            norm_finish<T, VEC>(A, p, w, root, c0, lane, row);
    }
    if (A.codes)
        norm_no_rows(A, row, step, ALONE ? lane : threadIdx.x, ALONE ? 32 : blockDim.x);
}
// ... of any length, a row per block: the second reading is from h or x (a lane reads what it wrote)
template <class T, bool VEC>
__global__ void __launch_bounds__(1024) k_rms_norm_long(const __grid_constant__ NormArgs A)
{
    __shared__ double part[32];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t row = blockIdx.x;
    const uint32_t cols = (uint32_t)A.cols, step = 32 * kNormWarp;
    const T *const x = (const T *)A.x + (uint64_t)row * A.x_ld;
    T *const h = (T *)A.h + (uint64_t)row * A.h_ld;
    grid_wait();
    if (row >= (uint32_t)A.rows) {
        norm_no_rows(A, row, 1ll << 40, threadIdx.x, 1024);
        return;
    }
    double sum = 0;
    NormPiece<T, VEC> p, o;
#pragma unroll 2
    for (uint32_t c0 = warp * kNormWarp; c0 < cols; c0 += step) {
        p.load(x, c0, cols, lane, A.aligned32);
        if (A.add) {
            o.load((const T *)A.add + (uint64_t)row * A.add_ld, c0, cols, lane, A.aligned32);
            norm_join(p, o);
            p.store(h, c0, cols, lane, A.aligned32);
        }
        sum += norm_squares(p);
    }
    sum = warp_sum(sum);
    if (lane == 0)
        part[warp] = sum;
    __syncthreads();
    sum = warp_sum(part[lane]);
    const float root = (float)root_of(__fma_rn(sum, A.share, A.eps));
    if (threadIdx.x == 0)
        A.rstd[row] = root;
    if (!A.y && !A.codes)
        return;
#pragma unroll 2
    for (uint32_t c0 = warp * kNormWarp; c0 < cols; c0 += step) {
        float w[kNormPer];
        load_weights<T, VEC>(A.w, A.w32, A.aligned_w, c0, cols, lane, w);
        p.load(A.add ? h : x, c0, cols, lane, A.aligned32);
        norm_finish<T, VEC>(A, p, w, root, c0, lane, row);
    }
}

// ------------------------------------------------------------------ the gradient
// With n = h r and g = dy w: dx = r (g - n mean(g n)) + add, dw = the sum over rows of dy n.  The columns' sums stay in registers, in 32 bits for kNormChain rows at
// most, and are written once per block and so many rows, to be added in 64 bits and in their order by k_norm_columns: results do not depend on which block is done first.
// (One chain for all rows of a block loses up to 2^-24 with each: 4 columns of 20 million rows, 4223 to a warp, 6e-5.)
constexpr uint32_t kNormChain = 256;
struct NormGradArgs {
    const void *dy, *h, *w, *add;
    void *dx;
    const float *rstd;
    const float *means;     // per row, where a row has more columns than a group
    float *partial;         // per segment, block and column, or NULL
    uint32_t segments;      // of kNormChain rows of a block's (a warp's)
    int64_t rows, cols;
    uint32_t dy_ld, h_ld, add_ld, dx_ld;
    float share;
    bool w32, aligned32, aligned_w;
};
// GIVEN: the means are; a block has 8192 columns (the grid's first dimension, of which there may be more than 65535) of its rows (the second)
template <class T, bool VEC, bool ALONE, bool GIVEN>
__global__ void __launch_bounds__(ALONE ? 256 : 1024, ALONE ? 4 : 1) k_norm_grad(const __grid_constant__ NormGradArgs A)
{
    constexpr int N = kNormPer;
    extern __shared__ __align__(16) uint8_t norm_smem[];
    __shared__ float part[2][32];
    __shared__ float other[ALONE ? 8 * kNormWarp : 1];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const uint32_t cols = (uint32_t)A.cols, c0 = ALONE ? 0u : ((GIVEN ? blockIdx.x * 32 : 0u) + warp) * kNormWarp, block = GIVEN ? blockIdx.y : blockIdx.x, blocks = GIVEN ? gridDim.y : gridDim.x;
    uint32_t row = ALONE ? block * 8 + warp : block;   // (rows are fewer than 2^31)
    const uint32_t step = ALONE ? blocks * 8 : blocks;
    grid_wait();
    float w[N], sums[N];
    load_weights<T, VEC>(A.w, A.w32, A.aligned_w, c0, cols, lane, w);
#pragma unroll
    for (int q = 0; q < N; ++q)
        sums[q] = 0.f;
    Ahead<T, VEC, 3> rows(norm_smem, warp, lane, c0, cols);
    const T *const dy = (const T *)A.dy, *const h = (const T *)A.h, *const add = (const T *)A.add;
    auto ask = [&](uint32_t row) {
        if (row < (uint32_t)A.rows) {
            rows.ask(0, dy + (uint64_t)row * A.dy_ld);
            rows.ask(1, h + (uint64_t)row * A.h_ld);
            if (add)
                rows.ask(2, add + (uint64_t)row * A.add_ld);
        }
        rows.close();
    };
#pragma unroll
    for (int k = 0; k < rows.DEPTH - 1; ++k)
        ask(row + k * step);
    float r = row < (uint32_t)A.rows ? A.rstd[row] : 0.f;
    int turn = 0;
    auto take = [&] {
        ask(row + (rows.DEPTH - 1) * step);
        const float root = r;
        r = row + step < (uint32_t)A.rows ? A.rstd[row + step] : 0.f;
        float m = GIVEN ? A.means[row] : 0.f;
        rows.wait();
        float d[N], n[N];
        NormPiece<T, VEC> a;
        rows.take(0, dy + (uint64_t)row * A.dy_ld, a);
        a.unpack(d);
        rows.take(1, h + (uint64_t)row * A.h_ld, a);
        a.unpack(n);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            n[q] = __fmul_rn(n[q], root);
            sums[q] = __fmaf_rn(d[q], n[q], sums[q]);
            d[q] = __fmul_rn(d[q], w[q]);
            if (!GIVEN)
                m = __fmaf_rn(d[q], n[q], m);
        }
        if constexpr (!GIVEN) {
            m = warp_sum(m);
            if constexpr (!ALONE) {
                if (lane == 0)
                    part[turn][warp] = m;
                __syncthreads();
                m = warp_sum(lane < warps ? part[turn][lane] : 0.f);
            }
            m *= A.share;
        }
#pragma unroll
        for (int q = 0; q < N; ++q)
            d[q] = __fmul_rn(__fmaf_rn(-n[q], m, d[q]), root);
        if (add) {
            rows.take(2, add + (uint64_t)row * A.add_ld, a);
            a.unpack(n);
#pragma unroll
            for (int q = 0; q < N; ++q)
                d[q] = __fadd_rn(d[q], n[q]);
        }
        rows.done();
        a.pack(d);
        a.store((T *)A.dx + (uint64_t)row * A.dx_ld, c0, cols, lane, A.aligned32);
    };
    for (uint32_t segment = 0; segment < A.segments; ++segment) {
        for (uint32_t i = 0; i < kNormChain && row < (uint32_t)A.rows; ++i, row += step, turn ^= 1)
            take();
        if (!A.partial)
            continue;
        if constexpr (ALONE) {   // a block's warps one after the other
#pragma unroll
            for (int q = 0; q < N; ++q)
                other[(warp * N + q) * 32 + lane] = sums[q];
            __syncthreads();
            if (warp == 0)
                for (int i = 1; i < 8; ++i)
#pragma unroll
                    for (int q = 0; q < N; ++q)
                        sums[q] += other[(i * N + q) * 32 + lane];
            __syncthreads();
        }
        float *const partial = A.partial + ((uint64_t)segment * blocks + block) * cols;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const uint32_t c = lane_col<VEC, N>(c0, lane, q);
            if (c < cols && (!ALONE || warp == 0))
                partial[c] = sums[q];
            sums[q] = 0.f;
        }
    }
}
// ... the rows' means alone, a block each
template <class T, bool VEC>
__global__ void __launch_bounds__(1024) k_norm_means(const __grid_constant__ NormGradArgs A, float *means)
{
    __shared__ double part[32];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = blockIdx.x;
    grid_wait();
    const float root = A.rstd[row];
    double m = 0;   // (of up to 2^21 lanes' parts)
#pragma unroll 2
    for (uint32_t c0 = warp * kNormWarp; c0 < (uint32_t)A.cols; c0 += 32 * kNormWarp) {
        NormPiece<T, VEC> a, b;
        a.load((const T *)A.dy + (uint64_t)row * A.dy_ld, c0, (uint32_t)A.cols, lane, A.aligned32);
        b.load((const T *)A.h + (uint64_t)row * A.h_ld, c0, (uint32_t)A.cols, lane, A.aligned32);
        float d[kNormPer], n[kNormPer], w[kNormPer], s = 0.f;
        a.unpack(d), b.unpack(n);
        load_weights<T, VEC>(A.w, A.w32, A.aligned_w, c0, (uint32_t)A.cols, lane, w);
#pragma unroll
        for (int q = 0; q < kNormPer; ++q)
            s = __fmaf_rn(__fmul_rn(d[q], w[q]), __fmul_rn(n[q], root), s);
        m += (double)s;
    }
    m = warp_sum(m);
    if (lane == 0)
        part[warp] = m;
    __syncthreads();
    m = warp_sum(part[lane]);
    if (threadIdx.x == 0)
        means[row] = (float)m * A.share;
}
// the blocks' sums of 32 columns
__global__ void __launch_bounds__(1024) k_norm_columns(const float *partial, uint32_t groups, int64_t cols, float *dw)
{
    __shared__ double part[32][33];
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    grid_wait();
    double sum = 0;
    if (c < cols) {
        const float *const p = fresh(partial) + c;
#pragma unroll 8
        for (uint32_t g = warp; g < groups; g += 32)
            sum += (double)load_global(p + (int64_t)g * cols);
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < cols) {
        for (int i = 1; i < 32; ++i)
            sum += part[i][lane];
        dw[c] = (float)sum;
    }
}

// ------------------------------------------------------------------ host

// warps of a block: one with a row of its own each, or as many as a row has (beyond the widest: with as many of its columns)
static int norm_warps(int64_t cols) { return cols <= kNormWarp ? 8 : (int)((std::min(cols, kNormWidest) + kNormWarp - 1) / kNormWarp); }
// blocks that share the rows: 32 warps to an SM
static uint32_t norm_blocks(int64_t rows, int64_t cols)
{
    return (uint32_t)std::min<int64_t>((int64_t)kPlanSMs * (32 / norm_warps(cols)), cols <= kNormWarp ? (rows + 7) / 8 : rows);
}

// how often a block of the gradient writes its columns' sums
static uint32_t norm_segments(int64_t rows, int64_t cols)
{
    const int64_t chains = (int64_t)norm_blocks(rows, cols) * (cols <= kNormWarp ? 8 : 1);
    return (uint32_t)(((rows + chains - 1) / chains + kNormChain - 1) / kNormChain);
}
static size_t norm_partials(int64_t rows, int64_t cols) { return (size_t)norm_blocks(rows, cols) * norm_segments(rows, cols) * (size_t)cols; }

template <auto KERNEL, int BYTES, class A>   // BYTES: of a warp
static cudaError_t launch_norm(dim3 grid, int warps, cudaStream_t s, const A &args)
{
    static int done[64];
    const size_t smem = (size_t)warps * BYTES;
    const cudaError_t e = opt_in_smem(KERNEL, smem + 10240, done);   // (48 KB hold what the kernel declares, too)
    return e != cudaSuccess ? e : launch(KERNEL, grid, warps * 32, smem, s, args);
}

template <class T, bool VEC>
static cudaError_t norm(const NormArgs &A, cudaStream_t s)
{
    const int64_t rows = A.codes ? (A.rows + 127) / 128 * 128 : A.rows;   // (scales of rows that do not exist are zero)
    if (A.cols > kNormWidest)
        return launch(k_rms_norm_long<T, VEC>, dim3((unsigned)rows), 1024, 0, s, A);
    constexpr int bytes = Ahead<T, VEC, 2>::BYTES;
    const dim3 grid(norm_blocks(rows, A.cols));
    return A.cols <= kNormWarp ? launch_norm<k_rms_norm<T, VEC, true>, bytes>(grid, norm_warps(A.cols), s, A)
                               : launch_norm<k_rms_norm<T, VEC, false>, bytes>(grid, norm_warps(A.cols), s, A);
}

template <class T, bool VEC>
static cudaError_t norm_grad(NormGradArgs A, float *means, float *dw, cudaStream_t s)
{
    const unsigned blocks = norm_blocks(A.rows, A.cols);
    const int warps = norm_warps(A.cols);
    constexpr int bytes = Ahead<T, VEC, 3>::BYTES;
    cudaError_t e;
    if (A.cols > kNormWidest) {
        e = launch(k_norm_means<T, VEC>, dim3((unsigned)A.rows), 1024, 0, s, A, means);
        A.means = means;
        if (e == cudaSuccess)
            e = launch_norm<k_norm_grad<T, VEC, false, true>, bytes>(dim3((unsigned)((A.cols + kNormWidest - 1) / kNormWidest), blocks), warps, s, A);
    } else {
        e = A.cols <= kNormWarp ? launch_norm<k_norm_grad<T, VEC, true, false>, bytes>(dim3(blocks), warps, s, A)
                                : launch_norm<k_norm_grad<T, VEC, false, false>, bytes>(dim3(blocks), warps, s, A);
    }
    if (e == cudaSuccess && dw)
        e = launch(k_norm_columns, dim3((unsigned)((A.cols + 31) / 32)), 1024, 0, s, (const float *)A.partial, (uint32_t)blocks * A.segments, A.cols, dw);
    return e;
}

static int check_weight(const void *w, int dtype, int w_dtype, int64_t cols)
{
    if (w_dtype != dtype && w_dtype != CONEF_F32)
        return CONEF_ERR_INVALID_ARG;
    return cols && (!w || ((uintptr_t)w & (elem_bytes(w_dtype) - 1))) ? CONEF_ERR_INVALID_ARG : CONEF_OK;
}

}  // namespace conef

using namespace conef;

extern "C" {

int conef_rms_norm(const void *x, const void *add, const void *weight, int dtype, int weight_dtype, int64_t rows, int64_t cols, int64_t x_ld, int64_t add_ld, double eps,
                   void *h, int64_t h_ld, float *rstd, void *y, int64_t y_ld, int kind, void *codes, void *scales, void *codes_t, void *scales_t, conef_stream stream)
{
    int rc = check_matrix(x, dtype, rows, cols, x_ld);
    if (rc == CONEF_OK && add && (rc = check_matrix(add, dtype, rows, cols, add_ld)) == CONEF_OK)
        rc = check_matrix(h, dtype, rows, cols, h_ld);
    if (rc == CONEF_OK && y)
        rc = check_matrix(y, dtype, rows, cols, y_ld);
    if (rc == CONEF_OK)
        rc = check_weight(weight, dtype, weight_dtype, cols);
    if (rc != CONEF_OK)
        return rc;
    if (!(eps >= 0.0) || eps > 1e300 || (!add && h) || !codes != !scales || !codes_t != !scales_t || (y && (codes || codes_t)) ||
        ((codes || codes_t) && kind != CONEF_E4M3 && kind != CONEF_E5M2))
        return CONEF_ERR_INVALID_ARG;
    if ((((uintptr_t)codes | (uintptr_t)scales | (uintptr_t)codes_t | (uintptr_t)scales_t) & 15) != 0)
        return CONEF_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0)
        return CONEF_OK;
    if (!rstd || ((uintptr_t)rstd & 3))
        return CONEF_ERR_INVALID_ARG;
    if (codes_t && f8_scale_tiles(rows) * 4 * (f8_scale_tiles(cols) * 4) >= (1ll << 31))
        return CONEF_ERR_UNSUPPORTED;
    // (with the transpose's form both are made by the second kernel, which needs the rows' roots first)
    const bool second = codes_t != nullptr;
    NormArgs A = {x, add, weight, h, y, second ? nullptr : (uint8_t *)codes, second ? nullptr : (uint8_t *)scales, rstd, rows, cols, (uint32_t)x_ld, (uint32_t)add_ld, (uint32_t)h_ld, (uint32_t)y_ld, eps, 1.0 / (double)cols,
                  kind, weight_dtype == CONEF_F32, false, ((uintptr_t)weight & 15) == 0};
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        auto on = [&](uintptr_t bytes) {
            return rows_on<T>(x, rows, x_ld, bytes) && (!add || (rows_on<T>(add, rows, add_ld, bytes) && rows_on<T>(h, rows, h_ld, bytes))) && (!y || rows_on<T>(y, rows, y_ld, bytes));
        };
        A.aligned32 = on(32);
        cudaError_t e = on(16) ? norm<T, true>(A, (cudaStream_t)stream) : norm<T, false>(A, (cudaStream_t)stream);
        if (e == cudaSuccess && second) {
            const F8Out out = {(uint8_t *)codes, (uint8_t *)scales, (uint8_t *)codes_t, (uint8_t *)scales_t, kind};
            e = f8_tiles(add ? h : x, dtype, rows, cols, add ? h_ld : x_ld, rstd, weight, A.w32, false, out, (cudaStream_t)stream);
        }
        return launched(e, "conef_rms_norm");
    });
}

int conef_rms_norm_grad_bytes(int64_t rows, int64_t cols, size_t *bytes)
{
    if (rows < 0 || cols < 0 || !bytes)
        return CONEF_ERR_INVALID_ARG;
    if (rows >= (1ll << 31) || cols >= (1ll << 31))
        return CONEF_ERR_UNSUPPORTED;
    *bytes = rows && cols ? (norm_partials(rows, cols) + (cols > kNormWidest ? (size_t)rows : 0)) * sizeof(float) : 0;
    return CONEF_OK;
}

int conef_rms_norm_grad(const void *dy, const void *h, const void *weight, const float *rstd, const void *add, int dtype, int weight_dtype, int64_t rows, int64_t cols,
                        int64_t dy_ld, int64_t h_ld, int64_t add_ld, void *dx, int64_t dx_ld, float *dweight, void *workspace, size_t workspace_bytes,
                        conef_stream stream)
{
    int rc = check_matrix(dy, dtype, rows, cols, dy_ld);
    if (rc == CONEF_OK)
        rc = check_matrix(h, dtype, rows, cols, h_ld);
    if (rc == CONEF_OK && add)
        rc = check_matrix(add, dtype, rows, cols, add_ld);
    if (rc == CONEF_OK)
        rc = check_matrix(dx, dtype, rows, cols, dx_ld);
    if (rc == CONEF_OK)
        rc = check_weight(weight, dtype, weight_dtype, cols);
    if (rc != CONEF_OK)
        return rc;
    if (((uintptr_t)rstd | (uintptr_t)dweight | (uintptr_t)workspace) & 3)
        return CONEF_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0)
        return dweight && cols ? launched(cudaMemsetAsync(dweight, 0, (size_t)cols * sizeof(float), (cudaStream_t)stream), "conef_rms_norm_grad") : CONEF_OK;
    if (!rstd)
        return CONEF_ERR_INVALID_ARG;
    size_t need = 0;
    conef_rms_norm_grad_bytes(rows, cols, &need);
    if (!workspace || workspace_bytes < need)
        return CONEF_ERR_WORKSPACE_TOO_SMALL;
    float *const partial = (float *)workspace;
    NormGradArgs A = {dy, h, weight, add, dx, rstd, nullptr, dweight ? partial : nullptr, norm_segments(rows, cols), rows, cols, (uint32_t)dy_ld, (uint32_t)h_ld, (uint32_t)add_ld, (uint32_t)dx_ld, 1.f / (float)cols,
                      weight_dtype == CONEF_F32, false, ((uintptr_t)weight & 15) == 0};
    float *const means = partial + norm_partials(rows, cols);
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        auto on = [&](uintptr_t bytes) {
            return rows_on<T>(dy, rows, dy_ld, bytes) && rows_on<T>(h, rows, h_ld, bytes) && (!add || rows_on<T>(add, rows, add_ld, bytes)) && rows_on<T>(dx, rows, dx_ld, bytes);
        };
        A.aligned32 = on(32);
        return launched(on(16) ? norm_grad<T, true>(A, means, dweight, (cudaStream_t)stream) : norm_grad<T, false>(A, means, dweight, (cudaStream_t)stream),
                        "conef_rms_norm_grad");
    });
}

}  // extern "C"
