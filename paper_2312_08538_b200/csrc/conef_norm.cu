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
    bool w32, aligned32;
};

// the weights of a lane's 16 columns
template <class T, bool VEC>
__device__ __forceinline__ void load_weights(const void *w, bool w32, uint32_t c0, uint32_t cols, int lane, float *v)
{
    // (a weight begins anywhere; 16 elements of it come from L1)
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        const uint32_t c = lane_col<T, VEC>(c0, lane, q);
        v[q] = c >= cols ? 0.f : w32 ? ((const float *)w)[c] : to_f32(((const T *)w)[c]);
    }
}

// W warps to a row, NIT pieces of 512 elements to a warp, which stay in registers (0: any number; the second reading is from h or x).
// Squares are summed in 64 bits, which fp32's rounding of the root then does not show: a row's values, and so the codes, do not depend on how it is cut.
template <class T, bool VEC, int W, int NIT>
__global__ void __launch_bounds__(W >= 8 ? W * 32 : 256) k_rms_norm(const __grid_constant__ NormArgs A)
{
    constexpr int ROWS = W >= 8 ? 1 : 8 / W;
    __shared__ double part[ROWS][W];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = warp / W, wq = warp % W;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    const bool there = row < A.rows;
    const uint32_t cols = there ? (uint32_t)A.cols : 0u;
    const T *const x = (const T *)A.x + row * A.x_ld, *const add = (const T *)A.add + row * A.add_ld;
    T *const h = (T *)A.h + row * A.h_ld, *const y = (T *)A.y + row * A.y_ld;
    grid_wait();
    double sum = 0;
    auto join = [&](Piece<T, VEC> &p, const Piece<T, VEC> &o, uint32_t c0) {   // h, which rounds to its type
        float a[16], b[16];
        p.unpack(a), o.unpack(b);
#pragma unroll
        for (int q = 0; q < 16; ++q)
            a[q] = __fadd_rn(a[q], b[q]);
        p.pack(a);
        p.store(h, c0, cols, lane, A.aligned32);
    };
    auto squares = [&](const Piece<T, VEC> &p) {
        float v[16];
        p.unpack(v);
#pragma unroll
        for (int q = 0; q < 16; ++q)
            sum = __fma_rn((double)v[q], (double)v[q], sum);
    };
    Piece<T, VEC> keep[NIT ? NIT : 1];
    if constexpr (NIT > 0) {
#pragma unroll
        for (int it = 0; it < NIT; ++it)
            keep[it].load(x, (it * W + wq) * 512u, cols, lane, A.aligned32);
        if (A.add) {
            Piece<T, VEC> o[NIT];
#pragma unroll
            for (int it = 0; it < NIT; ++it)
                o[it].load(add, (it * W + wq) * 512u, cols, lane, A.aligned32);
#pragma unroll
            for (int it = 0; it < NIT; ++it)
                join(keep[it], o[it], (it * W + wq) * 512u);
        }
#pragma unroll
        for (int it = 0; it < NIT; ++it)
            squares(keep[it]);
    } else {
        for (uint32_t c0 = wq * 512u; c0 < cols; c0 += W * 512u) {
            keep[0].load(x, c0, cols, lane, A.aligned32);
            if (A.add) {
                Piece<T, VEC> o;
                o.load(add, c0, cols, lane, A.aligned32);
                join(keep[0], o, c0);
            }
            squares(keep[0]);
        }
    }
#pragma unroll
    for (int o = 16; o; o /= 2)
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if constexpr (W > 1) {
        if (lane == 0)
            part[r][wq] = sum;
        __syncthreads();
        sum = 0;
#pragma unroll
        for (int i = 0; i < W; ++i)
            sum += part[r][i];
    }
    const float root = (float)(1.0 / sqrt(sum / (double)A.cols + A.eps));
    if (there && wq == 0 && lane == 0)
        A.rstd[row] = root;
    if (!A.y && !A.codes)
        return;
    const uint32_t blocks = (uint32_t)f8_blocks(A.cols), tiles = (uint32_t)f8_scale_tiles(A.cols);
    auto finish = [&](const Piece<T, VEC> &p, uint32_t c0) {
        float v[16], w[16];
        p.unpack(v);
        load_weights<T, VEC>(A.w, A.w32, c0, cols, lane, w);
        if (A.codes) {
#pragma unroll
            for (int q = 0; q < 16; ++q)
                v[q] = norm_value(v[q], w[q], root);
            f8_store_row<T, VEC>(v, c0, blocks, lane, A.kind, there, A.codes + row * blocks * 128, A.scales + f8_scale_at(row, c0 / 128, tiles));
        } else {
#pragma unroll
            for (int q = 0; q < 16; ++q)
                v[q] = __fmul_rn(__fmul_rn(v[q], root), w[q]);
            Piece<T, VEC> o;
            o.pack(v);
            o.store(y, c0, cols, lane, A.aligned32);
        }
    };
    if constexpr (NIT > 0) {
#pragma unroll
        for (int it = 0; it < NIT; ++it)
            if ((it * W + wq) * 512u < (uint32_t)A.cols)
                finish(keep[it], (it * W + wq) * 512u);
    } else {
        for (uint32_t c0 = wq * 512u; c0 < (uint32_t)A.cols; c0 += W * 512u) {   // (a lane reads what it wrote)
            if (A.add)
                keep[0].load(h, c0, cols, lane, A.aligned32);
            else
                keep[0].load(x, c0, cols, lane, A.aligned32);
            finish(keep[0], c0);
        }
    }
}

// ------------------------------------------------------------------ the gradient
// With n = h r and g = dy w: dx = r (g - n mean(g n)) + add, dw = the sum over rows of dy n.  W warps have a row's columns, a piece of 512 each, and take R
// rows at a time, so that one barrier serves R means; the columns' sums stay in registers (in 32 bits: rows of a group are few) and are written once per
// group, to be added in 64 bits and in their order by k_norm_columns: results do not depend on which group is done first.
struct NormGradArgs {
    const void *dy, *h, *w, *add;
    void *dx;
    const float *rstd;
    const float *means;     // per row, where a row has more columns than a group
    float *partial;         // per group and column, or NULL
    int64_t rows, cols, dy_ld, h_ld, add_ld, dx_ld;
    uint32_t groups;
    bool w32, aligned32;
};
template <class T, bool VEC, int W, bool GIVEN>
__global__ void __launch_bounds__(W > 4 ? W * 32 : 128, W > 4 ? 16 / W : 4) k_norm_grad(const __grid_constant__ NormGradArgs A)
{
    constexpr int G = W > 4 ? 1 : 4 / W, R = 2;
    __shared__ float part[2][G][R][W];
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = warp / W, wq = warp % W;
    const uint32_t c0 = (blockIdx.y * W + wq) * 512u, group = blockIdx.x * G + g;
    float w[16], sums[16];
    grid_wait();
    load_weights<T, VEC>(A.w, A.w32, c0, (uint32_t)A.cols, lane, w);
#pragma unroll
    for (int q = 0; q < 16; ++q)
        sums[q] = 0.f;
    const float share = 1.f / (float)A.cols;
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * G * R; first < A.rows; first += (int64_t)A.groups * R, turn ^= 1) {   // (the same number of turns for a block's groups)
        const int64_t row0 = first + g * R;
        Piece<T, VEC> a[R], b[R], o[R];
        float root[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = row0 + i;
            const uint32_t cols = row < A.rows ? (uint32_t)A.cols : 0u;
            a[i].load((const T *)A.dy + row * A.dy_ld, c0, cols, lane, A.aligned32);
            b[i].load((const T *)A.h + row * A.h_ld, c0, cols, lane, A.aligned32);
            if (A.add)
                o[i].load((const T *)A.add + row * A.add_ld, c0, cols, lane, A.aligned32);
            root[i] = row < A.rows ? A.rstd[row] : 0.f;
        }
        float mean[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float dy[16], n[16];
            a[i].unpack(dy), b[i].unpack(n);
            float m = 0.f;
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                n[q] = __fmul_rn(n[q], root[i]);
                m = __fmaf_rn(__fmul_rn(dy[q], w[q]), n[q], m);
                sums[q] = __fmaf_rn(dy[q], n[q], sums[q]);
            }
            if constexpr (!GIVEN) {
#pragma unroll
                for (int s = 16; s; s /= 2)
                    m += __shfl_xor_sync(0xffffffffu, m, s);
                if (W > 1 && lane == 0)
                    part[turn][g][i][wq] = m;
                mean[i] = m;
            }
        }
        if constexpr (GIVEN) {
#pragma unroll
            for (int i = 0; i < R; ++i)
                mean[i] = row0 + i < A.rows ? A.means[row0 + i] : 0.f;
        } else {
            if constexpr (W > 1) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    mean[i] = 0.f;
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        mean[i] += part[turn][g][i][j];
                }
            }
#pragma unroll
            for (int i = 0; i < R; ++i)
                mean[i] *= share;
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = row0 + i;
            float dy[16], n[16];
            a[i].unpack(dy), b[i].unpack(n);
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const float d = __fmaf_rn(-__fmul_rn(n[q], root[i]), mean[i], __fmul_rn(dy[q], w[q]));
                dy[q] = __fmul_rn(d, root[i]);
            }
            if (A.add) {
                o[i].unpack(n);
#pragma unroll
                for (int q = 0; q < 16; ++q)
                    dy[q] = __fadd_rn(dy[q], n[q]);
            }
            Piece<T, VEC> d;
            d.pack(dy);
            d.store((T *)A.dx + row * A.dx_ld, c0, row < A.rows ? (uint32_t)A.cols : 0u, lane, A.aligned32);
        }
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
        load_weights<T, VEC>(A.w, A.w32, c0, (uint32_t)A.cols, lane, w);
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
__global__ void __launch_bounds__(256) k_norm_columns(const float *partial, uint32_t groups, int64_t cols, float *dw)
{
    __shared__ double part[8][32];
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    grid_wait();
    double sum = 0;
    if (c < cols) {
        const float *const p = fresh(partial) + c;
#pragma unroll 8
        for (uint32_t g = warp; g < groups; g += 8)
            sum += (double)load_global(p + (int64_t)g * cols);
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < cols) {
        for (int i = 1; i < 8; ++i)
            sum += part[i][lane];
        dw[c] = (float)sum;
    }
}

// ------------------------------------------------------------------ host

// warps per row of the gradient, and the groups that share the rows (as many as there are warps for, 16 to an SM)
static int grad_warps(int64_t cols) { return cols <= 512 ? 1 : cols <= 1024 ? 2 : cols <= 2048 ? 4 : cols <= 4096 ? 8 : 16; }
constexpr int64_t kGradWidest = 16 * 512;
static uint32_t grad_groups(int64_t rows, int64_t cols)
{
    const int w = grad_warps(cols), per_block = w > 4 ? 1 : 4 / w;
    const int64_t most = kPlanSMs * 16 / w, blocks = (rows + 2 * per_block - 1) / (2 * per_block);
    return (uint32_t)std::min<int64_t>(most, blocks * per_block);
}

template <class T, bool VEC>
static cudaError_t norm(const NormArgs &A, cudaStream_t s)
{
    const int64_t rows = A.codes ? (A.rows + 127) / 128 * 128 : A.rows;   // (scales of rows that do not exist are zero)
    auto go = [&](auto w, auto n) {
        constexpr int W = decltype(w)::value, NIT = decltype(n)::value, ROWS = W >= 8 ? 1 : 8 / W;
        return launch(k_rms_norm<T, VEC, W, NIT>, dim3((unsigned)((rows + ROWS - 1) / ROWS)), W >= 8 ? W * 32 : 256, 0, s, A);
    };
    using I1 = std::integral_constant<int, 1>;
    using I4 = std::integral_constant<int, 4>;
    if (A.cols <= 512)
        return go(I1(), I1());
    if (A.cols <= 2048)
        return A.rows >= 2 * kPlanSMs ? go(I1(), I4()) : go(I4(), I1());
    if (A.cols <= 8192)
        return go(I4(), I4());
    return go(std::integral_constant<int, 16>(), std::integral_constant<int, 0>());
}

template <class T, bool VEC>
static cudaError_t norm_grad(NormGradArgs A, float *means, float *dw, cudaStream_t s)
{
    auto go = [&](auto w, auto given) {
        constexpr int W = decltype(w)::value, G = W > 4 ? 1 : 4 / W;
        const dim3 grid(A.groups / G, (unsigned)((A.cols + W * 512 - 1) / (W * 512)));
        return launch(k_norm_grad<T, VEC, W, decltype(given)::value>, grid, W > 4 ? W * 32 : 128, 0, s, A);
    };
    using N = std::false_type;
    cudaError_t e;
    if (A.cols > kGradWidest) {
        e = launch(k_norm_means<T, VEC>, dim3((unsigned)A.rows), 256, 0, s, A, means);
        A.means = means;
        if (e == cudaSuccess)
            e = go(std::integral_constant<int, 16>(), std::true_type());
    } else {
        switch (grad_warps(A.cols)) {
        case 1: e = go(std::integral_constant<int, 1>(), N()); break;
        case 2: e = go(std::integral_constant<int, 2>(), N()); break;
        case 4: e = go(std::integral_constant<int, 4>(), N()); break;
        case 8: e = go(std::integral_constant<int, 8>(), N()); break;
        default: e = go(std::integral_constant<int, 16>(), N()); break;
        }
    }
    if (e == cudaSuccess && dw)
        e = launch(k_norm_columns, dim3((unsigned)((A.cols + 31) / 32)), 256, 0, s, (const float *)A.partial, A.groups, A.cols, dw);
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
                  kind, weight_dtype == CONEF_F32, false};
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
    *bytes = rows && cols ? ((size_t)grad_groups(rows, cols) * (size_t)cols + (cols > kGradWidest ? (size_t)rows : 0)) * sizeof(float) : 0;
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
                      weight_dtype == CONEF_F32, false};
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
