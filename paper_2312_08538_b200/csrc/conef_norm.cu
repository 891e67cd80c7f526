// Root-mean-square norm of rows with the residual's addition, into the rows' type or into 8-bit floats with block scales (conef_f8.cuh), and its gradient.
#include <algorithm>

#include "conef_f8.cuh"

namespace conef {

struct NormArgs {
    const void *x, *add, *w;
    void *h, *y;
    uint8_t *codes, *scales;
    float *rstd;
    int64_t rows, cols, x_ld, add_ld, h_ld, y_ld;
    double eps;
    int kind;
    uint32_t groups;
    bool w32, aligned32, aligned_w;
};

// the weights of a lane's 16 columns (aligned: 16 of them are)
template <class T, bool VEC>
__device__ __forceinline__ void load_weights(const void *w, bool w32, bool aligned, uint32_t c0, uint32_t cols, int lane, float *v)
{
    const uint32_t c = c0 + lane * 16;
    if (VEC && aligned && c + 16 <= cols) {
        if (w32) {
#pragma unroll
            for (int q = 0; q < 16; q += 4)
                Vec16<float>::unpack(*(const uint4 *)((const float *)w + c + q), *(float(*)[4])(v + q));
        } else {
#pragma unroll
            for (int q = 0; q < 16; q += Vec16<T>::N)
                Vec16<T>::unpack(*(const uint4 *)((const T *)w + c + q), *(float(*)[Vec16<T>::N])(v + q));
        }
        return;
    }
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        const uint32_t i = lane_col<T, VEC>(c0, lane, q);
        v[q] = i >= cols ? 0.f : w32 ? ((const float *)w)[i] : to_f32(((const T *)w)[i]);
    }
}

// ------------------------------------------------------------------ rows on their way
// Groups of W warps walk over rows, a piece of 512 elements to a warp, and have those ahead copied into shared memory meanwhile, each lane what it will read: DEPTH rows
// of ARRAYS matrices.  (A row at a time without that waits for memory once per row: norm-and-gradient of 8192 x 1600 in bf16 with two rows in registers 30 + 30 us.)
// Elements of 16 bits on odd addresses, which no copy takes, are read when they are wanted.
template <class T, bool VEC, int ARRAYS>
struct Rows {
    static constexpr bool AHEAD = VEC || sizeof(T) == 4;
    static constexpr int CHUNK = VEC ? 16 : 4, PER = CHUNK / (int)sizeof(T), CHUNKS = 16 / PER;   // bytes and elements of a copy; copies per piece
    static constexpr int STAGE = ARRAYS * (int)sizeof(T) * 512, DEPTH = sizeof(T) == 2 ? 4 : 2, BYTES = AHEAD ? STAGE * DEPTH : 16;   // of a warp

    uint32_t at;   // the warp's shared memory, and the lane's place in it
    uint32_t c0, cols;
    int lane;

    __device__ __forceinline__ Rows(const uint8_t *smem, uint32_t c0, uint32_t cols, int lane) : c0(c0), cols(cols), lane(lane)
    {
        at = (uint32_t)__cvta_generic_to_shared(smem) + lane * CHUNK;
    }
    __device__ __forceinline__ uint32_t first(int i) const { return VEC ? c0 + lane * 16 + i * PER : lane_col<T, VEC>(c0, lane, i); }
    __device__ __forceinline__ uint32_t slot(int stage, int array, int i) const { return at + stage * STAGE + (array * CHUNKS + i) * (32 * CHUNK); }
    __device__ __forceinline__ void ask(int stage, int array, const T *row) const
    {
        if constexpr (AHEAD) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const uint32_t c = first(i);
                if (c >= cols)
                    continue;
                if constexpr (VEC) {
                    const uint32_t bytes = min((cols - c) * (uint32_t)sizeof(T), 16u);   // (zeros behind the row's end)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(slot(stage, array, i)), "l"(row + c), "r"(bytes) : "memory");
                } else {
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(slot(stage, array, i)), "l"(row + c) : "memory");
                }
            }
        }
    }
    static __device__ __forceinline__ void close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory"); }   // (for the oldest of DEPTH)
    __device__ __forceinline__ void take(int stage, int array, const T *row, Piece<T, VEC> &p) const
    {
        if constexpr (!AHEAD) {
            p.load(row, c0, cols, lane, false);
        } else {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const bool there = first(i) < cols;
                if constexpr (VEC) {
                    uint32_t x = 0, y = 0, z = 0, w = 0;
                    if (there)
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x), "=r"(y), "=r"(z), "=r"(w) : "r"(slot(stage, array, i)) : "memory");
                    p.w[4 * i] = x, p.w[4 * i + 1] = y, p.w[4 * i + 2] = z, p.w[4 * i + 3] = w;
                } else {
                    uint32_t x = 0;
                    if (there)
                        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(slot(stage, array, i)) : "memory");
                    p.w[i] = x;
                }
            }
        }
    }
};
template <int W>
__device__ __forceinline__ void group_sync(int group)   // the W warps of a group
{
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(W * 32) : "memory");
}
__host__ __device__ constexpr int norm_threads(int w) { return w > 4 ? w * 32 : 128; }
__host__ __device__ constexpr int norm_groups(int w) { return w > 4 ? 1 : 4 / w; }   // of a block

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
template <class T, bool VEC>
__device__ __forceinline__ void norm_finish(const NormArgs &A, const Piece<T, VEC> &p, const float *w, float root, uint32_t c0, int lane, int64_t row)
{
    float v[16];
    p.unpack(v);
    if (A.codes) {
        const uint32_t blocks = (uint32_t)f8_blocks(A.cols);
        norm_values<16>(v, w, root);
        f8_store_row<T, VEC>(v, c0, blocks, lane, A.kind, true, A.codes + row * blocks * 128, A.scales + f8_scale_at(row, c0 / 128, f8_scale_tiles(A.cols)));
    } else {
#pragma unroll
        for (int q = 0; q < 16; ++q)
            v[q] = __fmul_rn(__fmul_rn(v[q], root), w[q]);
        Piece<T, VEC> o;
        o.pack(v);
        o.store((T *)A.y + row * A.y_ld, c0, (uint32_t)A.cols, lane, A.aligned32);
    }
}
// h, rounded to its type
template <class T, bool VEC>
__device__ __forceinline__ void norm_join(Piece<T, VEC> &p, const Piece<T, VEC> &o)
{
    float a[16], b[16];
    p.unpack(a), o.unpack(b);
#pragma unroll
    for (int q = 0; q < 16; ++q)
        a[q] = __fadd_rn(a[q], b[q]);
    p.pack(a);
}
// Squares are summed in 64 bits, which fp32's rounding of the root then does not show: a row's values, and so the codes, do not depend on how it is cut.
template <class T, bool VEC>
__device__ __forceinline__ double norm_squares(const Piece<T, VEC> &p)
{
    float v[16];
    p.unpack(v);
    double a = 0, b = 0;
#pragma unroll
    for (int q = 0; q < 16; q += 2) {
        a = __fma_rn((double)v[q], (double)v[q], a);
        b = __fma_rn((double)v[q + 1], (double)v[q + 1], b);
    }
    return a + b;
}
template <class T, bool VEC, int W>
__global__ void __launch_bounds__(norm_threads(W)) k_rms_norm(const __grid_constant__ NormArgs A)
{
    using R = Rows<T, VEC, 2>;
    constexpr int G = norm_groups(W);
    extern __shared__ __align__(16) uint8_t norm_smem[];
    __shared__ double part[2][G][W];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = warp / W, wq = warp % W;
    const uint32_t c0 = wq * 512u;
    const R rows(norm_smem + warp * R::BYTES, c0, (uint32_t)A.cols, lane);
    const int64_t first = (int64_t)blockIdx.x * G + g, step = A.groups;
    const T *const x = (const T *)A.x, *const add = (const T *)A.add;
    grid_wait();
    float w[16];
    load_weights<T, VEC>(A.w, A.w32, A.aligned_w, c0, (uint32_t)A.cols, lane, w);
    auto ask = [&](int stage, int64_t row) {
        if (row < A.rows) {
            rows.ask(stage, 0, x + row * A.x_ld);
            if (add)
                rows.ask(stage, 1, add + row * A.add_ld);
        }
        R::close();
    };
#pragma unroll
    for (int d = 0; d < R::DEPTH - 1; ++d)
        ask(d, first + d * step);
    int stage = 0, turn = 0;
    int64_t row = first;
    for (; row < A.rows; row += step) {
        ask((stage + R::DEPTH - 1) % R::DEPTH, row + (R::DEPTH - 1) * step);
        R::wait();
        Piece<T, VEC> p;
        rows.take(stage, 0, x + row * A.x_ld, p);
        if (add) {
            Piece<T, VEC> o;
            rows.take(stage, 1, add + row * A.add_ld, o);
            norm_join(p, o);
            p.store((T *)A.h + row * A.h_ld, c0, (uint32_t)A.cols, lane, A.aligned32);
        }
        double sum = norm_squares(p);
#pragma unroll
        for (int o = 16; o; o /= 2)
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if constexpr (W > 1) {
            if (lane == 0)
                part[turn][g][wq] = sum;
            group_sync<W>(g);
            sum = 0;
#pragma unroll
            for (int i = 0; i < W; ++i)
                sum += part[turn][g][i];
            turn ^= 1;
        }
        const float root = (float)root_of(sum / (double)A.cols + A.eps);
        if (wq == 0 && lane == 0)
            A.rstd[row] = root;
        if ((A.y || A.codes) && c0 < (uint32_t)A.cols)
            norm_finish<T, VEC>(A, p, w, root, c0, lane, row);
        stage = (stage + 1) % R::DEPTH;
    }
    if (A.codes && c0 < (uint32_t)A.cols && lane == 0)   // scales of rows that do not exist
        for (; row < (A.rows + 127) / 128 * 128; row += step)
            *(uint32_t *)(A.scales + f8_scale_at(row, c0 / 128, f8_scale_tiles(A.cols))) = 0u;
}
// ... of any length: a CTA per row, the second reading from h or x (a lane reads what it wrote)
template <class T, bool VEC>
__global__ void __launch_bounds__(512) k_rms_norm_long(const __grid_constant__ NormArgs A)
{
    constexpr int W = 16;
    __shared__ double part[W];
    grid_release();
    const int wq = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = blockIdx.x;
    const uint32_t cols = (uint32_t)A.cols;
    const T *const x = (const T *)A.x + row * A.x_ld;
    T *const h = (T *)A.h + row * A.h_ld;
    grid_wait();
    if (row >= A.rows) {   // scales of rows that do not exist
        for (uint32_t t = threadIdx.x; t < (uint32_t)f8_scale_tiles(A.cols); t += 512)
            *(uint32_t *)(A.scales + f8_scale_at(row, t * 4, f8_scale_tiles(A.cols))) = 0u;
        return;
    }
    double sum = 0;
    Piece<T, VEC> p, o;
    for (uint32_t c0 = wq * 512u; c0 < cols; c0 += W * 512u) {
        p.load(x, c0, cols, lane, A.aligned32);
        if (A.add) {
            o.load((const T *)A.add + row * A.add_ld, c0, cols, lane, A.aligned32);
            norm_join(p, o);
            p.store(h, c0, cols, lane, A.aligned32);
        }
        sum += norm_squares(p);
    }
#pragma unroll
    for (int o = 16; o; o /= 2)
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0)
        part[wq] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int i = 0; i < W; ++i)
        sum += part[i];
    const float root = (float)root_of(sum / (double)A.cols + A.eps);
    if (threadIdx.x == 0)
        A.rstd[row] = root;
    if (!A.y && !A.codes)
        return;
    for (uint32_t c0 = wq * 512u; c0 < cols; c0 += W * 512u) {
        float w[16];
        load_weights<T, VEC>(A.w, A.w32, A.aligned_w, c0, cols, lane, w);
        p.load(A.add ? h : x, c0, cols, lane, A.aligned32);
        norm_finish<T, VEC>(A, p, w, root, c0, lane, row);
    }
}

// ------------------------------------------------------------------ the gradient
// With n = h r and g = dy w: dx = r (g - n mean(g n)) + add, dw = the sum over rows of dy n.  The columns' sums stay in registers (in 32 bits: rows of a group are
// few) and are written once per group, to be added in 64 bits and in their order by k_norm_columns: results do not depend on which group is done first.
struct NormGradArgs {
    const void *dy, *h, *w, *add;
    void *dx;
    const float *rstd;
    const float *means;     // per row, where a row has more columns than a group
    float *partial;         // per group and column, or NULL
    int64_t rows, cols, dy_ld, h_ld, add_ld, dx_ld;
    uint32_t groups;
    bool w32, aligned32, aligned_w;
};
template <class T, bool VEC, int W, bool GIVEN>
__global__ void __launch_bounds__(norm_threads(W)) k_norm_grad(const __grid_constant__ NormGradArgs A)
{
    using R = Rows<T, VEC, 3>;
    constexpr int G = norm_groups(W);
    extern __shared__ __align__(16) uint8_t norm_smem[];
    __shared__ float part[2][G][W];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = warp / W, wq = warp % W;
    const uint32_t c0 = (blockIdx.y * W + wq) * 512u, group = blockIdx.x * G + g;
    const R rows(norm_smem + warp * R::BYTES, c0, (uint32_t)A.cols, lane);
    const T *const dy = (const T *)A.dy, *const h = (const T *)A.h, *const add = (const T *)A.add;
    grid_wait();
    float w[16], sums[16];
    load_weights<T, VEC>(A.w, A.w32, A.aligned_w, c0, (uint32_t)A.cols, lane, w);
#pragma unroll
    for (int q = 0; q < 16; ++q)
        sums[q] = 0.f;
    auto ask = [&](int stage, int64_t row) {
        if (row < A.rows) {
            rows.ask(stage, 0, dy + row * A.dy_ld);
            rows.ask(stage, 1, h + row * A.h_ld);
            if (add)
                rows.ask(stage, 2, add + row * A.add_ld);
        }
        R::close();
    };
#pragma unroll
    for (int d = 0; d < R::DEPTH - 1; ++d)
        ask(d, group + (int64_t)d * A.groups);
    const float share = 1.f / (float)A.cols;
    int stage = 0, turn = 0;
    for (int64_t row = group; row < A.rows; row += A.groups) {
        ask((stage + R::DEPTH - 1) % R::DEPTH, row + (int64_t)(R::DEPTH - 1) * A.groups);
        const float root = A.rstd[row];
        R::wait();
        float d[16], n[16];
        Piece<T, VEC> p;
        rows.take(stage, 0, dy + row * A.dy_ld, p);
        p.unpack(d);
        rows.take(stage, 1, h + row * A.h_ld, p);
        p.unpack(n);
        float m = 0.f;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            n[q] = __fmul_rn(n[q], root);
            sums[q] = __fmaf_rn(d[q], n[q], sums[q]);
            d[q] = __fmul_rn(d[q], w[q]);
            m = __fmaf_rn(d[q], n[q], m);
        }
        if constexpr (GIVEN) {
            m = A.means[row];
        } else {
#pragma unroll
            for (int s = 16; s; s /= 2)
                m += __shfl_xor_sync(0xffffffffu, m, s);
            if constexpr (W > 1) {
                if (lane == 0)
                    part[turn][g][wq] = m;
                group_sync<W>(g);
                m = 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i)
                    m += part[turn][g][i];
                turn ^= 1;
            }
            m *= share;
        }
#pragma unroll
        for (int q = 0; q < 16; ++q)
            d[q] = __fmul_rn(__fmaf_rn(-n[q], m, d[q]), root);
        if (add) {
            rows.take(stage, 2, add + row * A.add_ld, p);
            p.unpack(n);
#pragma unroll
            for (int q = 0; q < 16; ++q)
                d[q] = __fadd_rn(d[q], n[q]);
        }
        p.pack(d);
        p.store((T *)A.dx + row * A.dx_ld, c0, (uint32_t)A.cols, lane, A.aligned32);
        stage = (stage + 1) % R::DEPTH;
    }
    if (A.partial) {
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const uint32_t c = lane_col<T, VEC>(c0, lane, q);
            if (c < (uint32_t)A.cols)
                A.partial[(int64_t)group * A.cols + c] = sums[q];
        }
    }
}
// ... the rows' means alone, a CTA each
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_norm_means(const __grid_constant__ NormGradArgs A, float *means)
{
    __shared__ float part[8];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = blockIdx.x;
    grid_wait();
    const float root = A.rstd[row];
    float m = 0.f;
    for (uint32_t c0 = warp * 512u; c0 < (uint32_t)A.cols; c0 += 8 * 512u) {
        Piece<T, VEC> a, b;
        a.load((const T *)A.dy + row * A.dy_ld, c0, (uint32_t)A.cols, lane, A.aligned32);
        b.load((const T *)A.h + row * A.h_ld, c0, (uint32_t)A.cols, lane, A.aligned32);
        float dy[16], n[16], w[16], s = 0.f;
        a.unpack(dy), b.unpack(n);
        load_weights<T, VEC>(A.w, A.w32, A.aligned_w, c0, (uint32_t)A.cols, lane, w);
#pragma unroll
        for (int q = 0; q < 16; ++q)
            s = __fmaf_rn(__fmul_rn(dy[q], w[q]), __fmul_rn(n[q], root), s);
        m += s;
    }
#pragma unroll
    for (int s = 16; s; s /= 2)
        m += __shfl_xor_sync(0xffffffffu, m, s);
    if (lane == 0)
        part[warp] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        m = 0.f;
        for (int i = 0; i < 8; ++i)
            m += part[i];
        means[row] = m / (float)A.cols;
    }
}
// the groups' sums of 32 columns
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

// warps per row, and the groups that share the rows: as many as there are warps for, `per_sm` to an SM
static int norm_warps(int64_t cols) { return cols <= 512 ? 1 : cols <= 1024 ? 2 : cols <= 2048 ? 4 : cols <= 4096 ? 8 : 16; }
constexpr int64_t kNormWidest = 16 * 512;
static uint32_t row_groups(int64_t rows, int64_t cols, int per_sm)
{
    const int w = norm_warps(cols), g = norm_groups(w);
    return (uint32_t)std::min<int64_t>(kPlanSMs * per_sm / w, (rows + g - 1) / g * g);
}
static uint32_t grad_groups(int64_t rows, int64_t cols) { return row_groups(rows, cols, 16); }
// f by the warps that a row takes
template <class F>
static cudaError_t by_warps(int64_t cols, F f)
{
    switch (norm_warps(cols)) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    }
    return f(std::integral_constant<int, 16>());
}

template <class T, bool VEC>
static cudaError_t norm(NormArgs A, cudaStream_t s)
{
    if (A.cols > kNormWidest)
        return launch(k_rms_norm_long<T, VEC>, dim3((unsigned)(A.codes ? (A.rows + 127) / 128 * 128 : A.rows)), 512, 0, s, A);
    A.groups = row_groups(A.codes ? (A.rows + 127) / 128 * 128 : A.rows, A.cols, 24);   // (scales of rows that do not exist are zero)
    return by_warps(A.cols, [&](auto w) {
        constexpr int W = decltype(w)::value;
        constexpr size_t smem = (size_t)Rows<T, VEC, 2>::BYTES * norm_threads(W) / 32;
        static int done[64];
        const cudaError_t e = opt_in_smem(k_rms_norm<T, VEC, W>, smem + 1024, done);
        return e != cudaSuccess ? e : launch(k_rms_norm<T, VEC, W>, dim3(A.groups / norm_groups(W)), norm_threads(W), smem, s, A);
    });
}

template <class T, bool VEC>
static cudaError_t norm_grad(NormGradArgs A, float *means, float *dw, cudaStream_t s)
{
    auto go = [&](auto w, auto given) {
        constexpr int W = decltype(w)::value;
        constexpr bool GIVEN = decltype(given)::value;
        constexpr size_t smem = (size_t)Rows<T, VEC, 3>::BYTES * norm_threads(W) / 32;
        static int done[64];
        const cudaError_t e = opt_in_smem(k_norm_grad<T, VEC, W, GIVEN>, smem + 1024, done);   // (48 KB hold what the kernel declares, too)
        const dim3 grid(A.groups / norm_groups(W), (unsigned)((A.cols + W * 512 - 1) / (W * 512)));
        return e != cudaSuccess ? e : launch(k_norm_grad<T, VEC, W, GIVEN>, grid, norm_threads(W), smem, s, A);
    };
    cudaError_t e;
    if (A.cols > kNormWidest) {
        e = launch(k_norm_means<T, VEC>, dim3((unsigned)A.rows), 256, 0, s, A, means);
        A.means = means;
        if (e == cudaSuccess)
            e = go(std::integral_constant<int, 16>(), std::true_type());
    } else {
        e = by_warps(A.cols, [&](auto w) { return go(w, std::false_type()); });
    }
    if (e == cudaSuccess && dw)
        e = launch(k_norm_columns, dim3((unsigned)((A.cols + 31) / 32)), 1024, 0, s, (const float *)A.partial, A.groups, A.cols, dw);
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
    NormArgs A = {x, add, weight, h, y, second ? nullptr : (uint8_t *)codes, second ? nullptr : (uint8_t *)scales, rstd, rows, cols, x_ld, add_ld, h_ld, y_ld, eps,
                  kind, 0, weight_dtype == CONEF_F32, false, ((uintptr_t)weight & 15) == 0};
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
    *bytes = rows && cols ? ((size_t)grad_groups(rows, cols) * (size_t)cols + (cols > kNormWidest ? (size_t)rows : 0)) * sizeof(float) : 0;
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
    NormGradArgs A = {dy, h, weight, add, dx, rstd, nullptr, dweight ? partial : nullptr, rows, cols, dy_ld, h_ld, add_ld, dx_ld, grad_groups(rows, cols),
                      weight_dtype == CONEF_F32, false, ((uintptr_t)weight & 15) == 0};
    float *const means = partial + (size_t)A.groups * cols;
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
