// Layer normalization of the rows of a matrix in fp32, bf16 or fp16, forward and backward: the
// dense vectors of section 3.5 (layernorm.hip has the pooled ones).
//
// Bound by HBM: the forward pass reads x and writes y, the backward pass reads dy and x and writes
// dx.  A group of lanes owns a row and keeps it in registers, so that every element is read once;
// the statistics come from the registers in two passes (the mean, then the centred squares).
// Groups are as narrow as the row allows, from one lane to the 1024 of a workgroup; wider rows
// are read again for each pass, from the caches.  The backward pass gives each workgroup
// rows a grid apart and sums their products column by column in registers; one partial row per
// workgroup goes to memory, and a second kernel adds those in order.
#include "elem_io.h"
#include "ss_common.h"

namespace ss {
namespace {

// Elements per 16-byte access.
template <int DT> constexpr int per_access() { return DT == SS_F32 ? 4 : 8; }

template <int LANES> constexpr int wg_size() { return LANES > kWG ? LANES : kWG; }

// Sum over the group of lanes that owns a row; in all of them.  Groups of several wavefronts are
// the whole workgroup; `s` then has a float per wavefront and is not used by the sum before.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float *s)
{
    constexpr int W = LANES < 64 ? LANES : 64;
#pragma unroll
    for (int off = W / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, W);
    if constexpr (LANES > 64) {
        if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) v += s[w];
    }
    return v;
}

// A lane's share of a row: P vectors of N elements, LANES vectors apart; zeros past the row.
template <int DT, int LANES, int P, int N>
__device__ __forceinline__ void load_share(const void *base, int64_t row, int c, int dim,
                                           Raw<DT, N> (&r)[P])
{
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int col = (i * LANES + c) * N;
        if (col + N <= dim) r[i] = load_raw<DT, N>(base, row + col);
        else r[i] = load_raw_part<DT, N>(base, row + col, dim - col);
    }
}
template <int DT, int N>
__device__ __forceinline__ void store_some(void *base, int64_t row, int col, int dim,
                                           const float (&f)[N])
{
    const Raw<DT, N> r = from_float<DT, N>(f);
    if (col + N <= dim) store_raw<DT, N>(base, row + col, r);
    else store_raw_part<DT, N>(base, row + col, r, dim - col);
}
// The parameters of a lane's columns; `absent` where there are none.
template <int WT, int LANES, int P, int N>
__device__ __forceinline__ void load_params(const void *p, int c, int dim, float absent,
                                            float (&f)[P][N])
{
    if (p) {
        Raw<WT, N> r[P];
        load_share<WT, LANES, P, N>(p, 0, c, dim, r);
#pragma unroll
        for (int i = 0; i < P; ++i) to_float(r[i], f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) f[i][k] = absent;
    }
}

template <int DT, int WT, int LANES, int P>
__global__ __launch_bounds__(wg_size<LANES>()) void rows_forward_kernel(
    const void *x, int64_t x_stride, int rows, const int32_t *__restrict__ n_valid,
    const void *gamma, const void *beta, float eps, void *y, int64_t y_stride,
    float *__restrict__ mean, float *__restrict__ rstd, int dim)
{
    constexpr int N = per_access<DT>(), NG = wg_size<LANES>() / LANES;
    __shared__ float s[2][LANES > 64 ? LANES / 64 : 1];
    const int n = clamp_valid(n_valid, rows);
    const int g = threadIdx.x / LANES, c = threadIdx.x % LANES;
    const float inv = 1.0f / (float)dim;
    float gam[P][N], bet[P][N];
    load_params<WT, LANES, P, N>(gamma, c, dim, 1.0f, gam);
    load_params<WT, LANES, P, N>(beta, c, dim, 0.0f, bet);
    for (int64_t r = (int64_t)blockIdx.x * NG + g; r < n; r += (int64_t)gridDim.x * NG) {
        Raw<DT, N> raw[P];
        load_share<DT, LANES, P, N>(x, r * x_stride, c, dim, raw);
        float v[P][N], sum = 0.0f, q = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            to_float(raw[i], v[i]);
#pragma unroll
            for (int k = 0; k < N; ++k) sum += v[i][k];
        }
        const float mu = row_sum<LANES>(sum, s[0]) * inv;
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[i][k] = (i * LANES + c) * N + k < dim ? v[i][k] - mu : 0.0f;
                q = fmaf(v[i][k], v[i][k], q);
            }
        const float rs = 1.0f / sqrtf(fmaf(row_sum<LANES>(q, s[1]), inv, eps));
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float o[N];
#pragma unroll
            for (int k = 0; k < N; ++k) o[k] = fmaf(v[i][k] * rs, gam[i][k], bet[i][k]);
            store_some<DT, N>(y, r * y_stride, (i * LANES + c) * N, dim, o);
        }
        if (c == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
    }
}

// part: [2][gridDim.x][dim], the products' sums and the gradients' sums; may be null.
template <int DT, int WT, int LANES, int P>
__global__ __launch_bounds__(wg_size<LANES>()) void rows_backward_kernel(
    const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int rows,
    const int32_t *__restrict__ n_valid, const void *gamma, const float *__restrict__ mean,
    const float *__restrict__ rstd, void *dx, int64_t dx_stride, int dim,
    float *__restrict__ part)
{
    constexpr int N = per_access<DT>(), NG = wg_size<LANES>() / LANES;
    __shared__ float s[4][LANES > 64 ? LANES / 64 : 1];
    __shared__ float s_col[NG > 1 ? kWG * N : 1];
    const int n = clamp_valid(n_valid, rows);
    const int g = threadIdx.x / LANES, c = threadIdx.x % LANES;
    const float inv = 1.0f / (float)dim;
    float gam[P][N], acc_g[P][N], acc_b[P][N];
    load_params<WT, LANES, P, N>(gamma, c, dim, 1.0f, gam);
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) acc_g[i][k] = acc_b[i][k] = 0.0f;
    int turn = 0;
    for (int64_t r = (int64_t)blockIdx.x * NG + g; r < n; r += (int64_t)gridDim.x * NG, turn ^= 2) {
        Raw<DT, N> xr[P], dr[P];
        load_share<DT, LANES, P, N>(x, r * x_stride, c, dim, xr);
        load_share<DT, LANES, P, N>(dy, r * dy_stride, c, dim, dr);
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float xf[N], df[N];
            to_float(xr[i], xf);
            to_float(dr[i], df);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float xh = (xf[k] - mu) * rs, gd = gam[i][k] * df[k];
                s1 += gd;                                // df is 0 past the row
                s2 = fmaf(gd, xh, s2);
                acc_g[i][k] = fmaf(df[k], xh, acc_g[i][k]);
                acc_b[i][k] += df[k];
            }
        }
        const float m1 = row_sum<LANES>(s1, s[turn]) * inv;
        const float m2 = row_sum<LANES>(s2, s[turn + 1]) * inv;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float xf[N], df[N], o[N];
            to_float(xr[i], xf);
            to_float(dr[i], df);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float xh = (xf[k] - mu) * rs;
                o[k] = fmaf(-xh, m2, fmaf(gam[i][k], df[k], -m1)) * rs;
            }
            store_some<DT, N>(dx, r * dx_stride, (i * LANES + c) * N, dim, o);
        }
    }
    if (!part) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *out = part + ((int64_t)which * gridDim.x + blockIdx.x) * dim;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float t[N];
#pragma unroll
            for (int k = 0; k < N; ++k) t[k] = which ? acc_b[i][k] : acc_g[i][k];
            if constexpr (NG > 1) {                      // the groups' sums, in their order
                __syncthreads();
#pragma unroll
                for (int k = 0; k < N; ++k) s_col[k * kWG + threadIdx.x] = t[k];
                __syncthreads();
                if (g != 0) continue;
                for (int o = 1; o < NG; ++o)
#pragma unroll
                    for (int k = 0; k < N; ++k) t[k] += s_col[k * kWG + o * LANES + c];
            }
            store_some<SS_F32, N>(out, 0, (i * LANES + c) * N, dim, t);
        }
    }
}

// ---- rows wider than a workgroup's registers ------------------------------------------------
constexpr int kWideThreads = 1024;

template <int DT, int WT>
__global__ __launch_bounds__(kWideThreads) void wide_forward_kernel(
    const void *x, int64_t x_stride, int rows, const int32_t *__restrict__ n_valid,
    const void *gamma, const void *beta, float eps, void *y, int64_t y_stride,
    float *__restrict__ mean, float *__restrict__ rstd, int dim)
{
    constexpr int N = per_access<DT>(), T = kWideThreads;
    __shared__ float s[2][T / 64];
    const int n = clamp_valid(n_valid, rows);
    const float inv = 1.0f / (float)dim;
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        float sum = 0.0f, q = 0.0f;
        for (int col = threadIdx.x * N; col < dim; col += T * N) {
            Raw<DT, N> raw[1];
            float f[N];
            load_share<DT, 1, 1, N>(x, r * x_stride + col, 0, dim - col, raw);
            to_float(raw[0], f);
#pragma unroll
            for (int k = 0; k < N; ++k) sum += f[k];
        }
        const float mu = row_sum<T>(sum, s[0]) * inv;
        for (int col = threadIdx.x * N; col < dim; col += T * N) {
            Raw<DT, N> raw[1];
            float f[N];
            load_share<DT, 1, 1, N>(x, r * x_stride + col, 0, dim - col, raw);
            to_float(raw[0], f);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float d = col + k < dim ? f[k] - mu : 0.0f;
                q = fmaf(d, d, q);
            }
        }
        const float rs = 1.0f / sqrtf(fmaf(row_sum<T>(q, s[1]), inv, eps));
        for (int col = threadIdx.x * N; col < dim; col += T * N) {
            Raw<DT, N> raw[1];
            float f[N], gam[1][N], bet[1][N];
            load_share<DT, 1, 1, N>(x, r * x_stride + col, 0, dim - col, raw);
            const auto at = [&](const void *p) -> const void * {
                return p ? static_cast<const typename ElemOf<WT>::type *>(p) + col : nullptr;
            };
            load_params<WT, 1, 1, N>(at(gamma), 0, dim - col, 1.0f, gam);
            load_params<WT, 1, 1, N>(at(beta), 0, dim - col, 0.0f, bet);
            to_float(raw[0], f);
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = fmaf((f[k] - mu) * rs, gam[0][k], bet[0][k]);
            store_some<DT, N>(y, r * y_stride, col, dim, f);
        }
        if (threadIdx.x == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
    }
}

template <int DT, int WT>
__global__ __launch_bounds__(kWideThreads) void wide_backward_kernel(
    const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int rows,
    const int32_t *__restrict__ n_valid, const void *gamma, const float *__restrict__ mean,
    const float *__restrict__ rstd, void *dx, int64_t dx_stride, int dim)
{
    constexpr int N = per_access<DT>(), T = kWideThreads;
    __shared__ float s[4][T / 64];
    const int n = clamp_valid(n_valid, rows);
    const float inv = 1.0f / (float)dim;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x, turn ^= 2) {
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.0f, s2 = 0.0f, m1 = 0.0f, m2 = 0.0f;
        for (int pass = 0; pass < 2; ++pass) {
            for (int col = threadIdx.x * N; col < dim; col += T * N) {
                Raw<DT, N> xr[1], dr[1];
                float xf[N], df[N], gam[1][N];
                load_share<DT, 1, 1, N>(x, r * x_stride + col, 0, dim - col, xr);
                load_share<DT, 1, 1, N>(dy, r * dy_stride + col, 0, dim - col, dr);
                load_params<WT, 1, 1, N>(
                    gamma ? static_cast<const typename ElemOf<WT>::type *>(gamma) + col : nullptr, 0,
                    dim - col, 1.0f, gam);
                to_float(xr[0], xf);
                to_float(dr[0], df);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float xh = (xf[k] - mu) * rs, gd = gam[0][k] * df[k];
                    s1 += gd;
                    s2 = fmaf(gd, xh, s2);
                    df[k] = fmaf(-xh, m2, fmaf(gam[0][k], df[k], -m1)) * rs;
                }
                if (pass) store_some<DT, N>(dx, r * dx_stride, col, dim, df);
            }
            if (pass == 0) {
                m1 = row_sum<T>(s1, s[turn]) * inv;
                m2 = row_sum<T>(s2, s[turn + 1]) * inv;
            }
        }
    }
}

// Column sums of wide rows: workgroup (b, w) takes a block of columns of every gridDim.y-th row.
template <int DT>
__global__ __launch_bounds__(kWG) void wide_columns_kernel(
    const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int rows,
    const int32_t *__restrict__ n_valid, const float *__restrict__ mean,
    const float *__restrict__ rstd, int dim, float *__restrict__ part)
{
    constexpr int N = per_access<DT>();
    const int n = clamp_valid(n_valid, rows);
    const int64_t col = ((int64_t)blockIdx.x * kWG + threadIdx.x) * N;
    if (col >= dim) return;
    float acc_g[N], acc_b[N];
#pragma unroll
    for (int k = 0; k < N; ++k) acc_g[k] = acc_b[k] = 0.0f;
#pragma unroll 2
    for (int64_t r = blockIdx.y; r < n; r += gridDim.y) {
        Raw<DT, N> xr[1], dr[1];
        float xf[N], df[N];
        load_share<DT, 1, 1, N>(x, r * x_stride + col, 0, dim - (int)col, xr);
        load_share<DT, 1, 1, N>(dy, r * dy_stride + col, 0, dim - (int)col, dr);
        const float mu = mean[r], rs = rstd[r];
        to_float(xr[0], xf);
        to_float(dr[0], df);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            acc_g[k] = fmaf(df[k], (xf[k] - mu) * rs, acc_g[k]);
            acc_b[k] += df[k];
        }
    }
    store_some<SS_F32, N>(part + (int64_t)blockIdx.y * dim, 0, (int)col, dim, acc_g);
    store_some<SS_F32, N>(part + ((int64_t)gridDim.y + blockIdx.y) * dim, 0, (int)col, dim, acc_b);
}

// out[col] = sum of the column's partial sums: thread (p, col) adds every kParts-th row from p on,
// then the kParts sums are added in order.
constexpr int kRedCols = 64, kParts = 16;

template <int WT>
__global__ __launch_bounds__(kRedCols * kParts) void columns_reduce_kernel(
    const float *__restrict__ part, int n_part, int dim, void *dgamma, void *dbeta)
{
    __shared__ float s[kParts][kRedCols];
    const int c = threadIdx.x % kRedCols, p = threadIdx.x / kRedCols;
    const int col = blockIdx.x * kRedCols + c;
    void *out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    const float *__restrict__ in = part + (int64_t)blockIdx.y * n_part * dim;
    float sum = 0.0f;
    if (col < dim) {
#pragma unroll 8
        for (int w = p; w < n_part; w += kParts) sum += in[(int64_t)w * dim + col];
    }
    s[p][c] = sum;
    __syncthreads();
    if (p == 0 && col < dim) {
        for (int q = 1; q < kParts; ++q) sum += s[q][c];
        static_cast<typename ElemOf<WT>::type *>(out)[col] = (typename ElemOf<WT>::type)sum;
    }
}

// ---- which kernel takes a row ---------------------------------------------------------------
// Lanes of a row and vectors per lane: the narrowest group whose lanes hold the row in one vector
// each, up to a wavefront; then two and four vectors per lane, then several wavefronts.
struct Shape {
    int lanes, vectors;        // lanes == 0: too wide for registers
};

Shape shape_of(int dim, int per, int most_vectors)
{
    const int64_t v = ((int64_t)dim + per - 1) / per;
    int lanes = 1;
    while (lanes < v && lanes < 64) lanes *= 2;
    if (v <= 64) return {lanes, 1};
    if (v <= 64 * 2) return {64, 2};
    if (v <= 64 * 4) return {64, 4};
    if (v <= 256 * 2) return {256, 2};
    if (v <= 256 * 4) return {256, 4};
    if (v <= 1024 * 2) return {1024, 2};
    if (v <= 1024 * 4 && most_vectors >= 4) return {1024, 4};
    return {0, 0};
}

#define SS_ROWS_TYPES(dt, wt, ...)                                                            \
    if ((dt) == SS_F32) { constexpr int DT = SS_F32, WT = SS_F32; __VA_ARGS__; }              \
    else if ((dt) == SS_BF16 && (wt) == SS_BF16) { constexpr int DT = SS_BF16, WT = SS_BF16; __VA_ARGS__; } \
    else if ((dt) == SS_BF16) { constexpr int DT = SS_BF16, WT = SS_F32; __VA_ARGS__; }       \
    else if ((wt) == SS_F16) { constexpr int DT = SS_F16, WT = SS_F16; __VA_ARGS__; }         \
    else { constexpr int DT = SS_F16, WT = SS_F32; __VA_ARGS__; }

#define SS_ROWS_CASE(l, p, ...)                                                               \
    if (sh.lanes == l && sh.vectors == p) { constexpr int LANES = l, P = p; __VA_ARGS__; }
#define SS_ROWS_SHAPES(...)                                                                   \
    SS_ROWS_CASE(1, 1, __VA_ARGS__) else SS_ROWS_CASE(2, 1, __VA_ARGS__)                      \
    else SS_ROWS_CASE(4, 1, __VA_ARGS__) else SS_ROWS_CASE(8, 1, __VA_ARGS__)                 \
    else SS_ROWS_CASE(16, 1, __VA_ARGS__) else SS_ROWS_CASE(32, 1, __VA_ARGS__)               \
    else SS_ROWS_CASE(64, 1, __VA_ARGS__) else SS_ROWS_CASE(64, 2, __VA_ARGS__)               \
    else SS_ROWS_CASE(64, 4, __VA_ARGS__) else SS_ROWS_CASE(256, 2, __VA_ARGS__)              \
    else SS_ROWS_CASE(256, 4, __VA_ARGS__) else SS_ROWS_CASE(1024, 2, __VA_ARGS__)

// Partial rows that the column sums are split into: a workgroup each.  At most kMostParts, and
// kPartFloats in all (but kLeastParts where a row is that wide).
constexpr int kMostParts = 1024, kLeastParts = 16;
constexpr int64_t kPartFloats = 4 << 20;

int most_parts(int rows, int dim)
{
    int64_t w = kPartFloats / dim;
    w = w > kMostParts ? kMostParts : w < kLeastParts ? kLeastParts : w;
    return (int)(w < rows ? w : rows);
}

// What they take at most: as most_parts without the rounding down, so that it falls in neither
// argument.
int64_t part_floats(int rows, int dim)
{
    int64_t n = (int64_t)kMostParts * dim;
    n = n > kPartFloats ? kPartFloats : n;
    n = n < (int64_t)kLeastParts * dim ? (int64_t)kLeastParts * dim : n;
    const int64_t all = (int64_t)(rows > 0 ? rows : 1) * dim;
    return n < all ? n : all;
}

constexpr int kForwardWgs = 2048;

int32_t check_rows(const char *who, int32_t dtype, int32_t param_dtype, int32_t rows, int32_t dim)
{
    if (dtype < SS_F32 || dtype > SS_F16)
        return fail(SS_ERR_INVALID_ARG, "%s: dtype = %d", who, dtype);
    if (param_dtype != dtype && param_dtype != SS_F32)
        return fail(SS_ERR_INVALID_ARG, "%s: param_dtype = %d (need dtype or SS_F32)", who,
                    param_dtype);
    if (rows < 0) return fail(SS_ERR_INVALID_ARG, "%s: rows = %d", who, rows);
    if (dim < 1 || dim > 1 << 20)
        return fail(SS_ERR_INVALID_ARG, "%s: dim = %d (need 1 to %d)", who, dim, 1 << 20);
    return SS_OK;
}

int32_t check_matrix(const char *who, const char *name, const void *p, int64_t stride, int32_t rows,
                     int32_t dim, int32_t dtype)
{
    if (rows > 0 && !p) return fail(SS_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
    if (stride < dim || stride > 1LL << 40)
        return fail(SS_ERR_INVALID_ARG, "%s: %s: rows are %lld elements apart (dim is %d)", who,
                    name, (long long)stride, dim);
    if (reinterpret_cast<uintptr_t>(p) % (dtype == SS_F32 ? 4 : 2) != 0)
        return fail(SS_ERR_INVALID_ARG, "%s: %s is not aligned to its type", who, name);
    return SS_OK;
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" {

int32_t ss_layernorm_rows_forward(int32_t dtype, int32_t param_dtype, int32_t rows, int32_t dim,
                                  const void *x, int64_t x_stride, const int32_t *n_valid,
                                  const void *gamma, const void *beta, float eps, void *y,
                                  int64_t y_stride, float *mean, float *rstd, void *stream)
{
    const char *who = "ss_layernorm_rows_forward";
    int32_t rc = check_rows(who, dtype, param_dtype, rows, dim);
    if (!rc) rc = check_matrix(who, "x", x, x_stride, rows, dim, dtype);
    if (!rc) rc = check_matrix(who, "y", y, y_stride, rows, dim, dtype);
    if (!rc) rc = check_matrix(who, "gamma", gamma, dim, 0, dim, param_dtype);
    if (!rc) rc = check_matrix(who, "beta", beta, dim, 0, dim, param_dtype);
    if (rc) return rc;
    if (rows > 0 && (!mean || !rstd))
        return fail(SS_ERR_INVALID_ARG, "%s: mean or rstd is NULL", who);
    if (!(eps >= 0.0f)) return fail(SS_ERR_INVALID_ARG, "%s: eps = %g", who, (double)eps);
    if (y == x && y_stride != x_stride && rows > 1)
        return fail(SS_ERR_INVALID_ARG, "%s: y is x with another stride", who);
    if (rows == 0) return SS_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const Shape sh = shape_of(dim, dtype == SS_F32 ? 4 : 8, 4);
    ProfScope prof("rows_forward_kernel", st);
#define SS_ROWS_FWD                                                                           \
    const int64_t groups = wg_size<LANES>() / LANES, need = (rows + groups - 1) / groups;     \
    launch(rows_forward_kernel<DT, WT, LANES, P>,                                             \
           dim3((unsigned)(need < kForwardWgs ? need : kForwardWgs)), dim3(wg_size<LANES>()), \
           st, x, x_stride, rows, n_valid, gamma, beta, eps, y, y_stride, mean, rstd, dim)
    SS_ROWS_TYPES(dtype, param_dtype,
                  SS_ROWS_SHAPES(SS_ROWS_FWD) else SS_ROWS_CASE(1024, 4, SS_ROWS_FWD) else launch(
                      wide_forward_kernel<DT, WT>, dim3(rows < kForwardWgs ? rows : kForwardWgs),
                      dim3(kWideThreads), st, x, x_stride, rows, n_valid, gamma, beta, eps, y,
                      y_stride, mean, rstd, dim))
#undef SS_ROWS_FWD
    return check_launch(who);
}

size_t ss_layernorm_rows_workspace_bytes(int32_t rows, int32_t dim)
{
    if (rows < 0 || dim < 1 || dim > 1 << 20) return 0;
    return align_up((size_t)2 * part_floats(rows, dim) * sizeof(float), 256);
}

int32_t ss_layernorm_rows_backward(int32_t dtype, int32_t param_dtype, int32_t rows, int32_t dim,
                                   const void *dy, int64_t dy_stride, const void *x,
                                   int64_t x_stride, const int32_t *n_valid, const void *gamma,
                                   const float *mean, const float *rstd, void *dx,
                                   int64_t dx_stride, void *dgamma, void *dbeta, void *ws,
                                   size_t ws_bytes, void *stream)
{
    const char *who = "ss_layernorm_rows_backward";
    int32_t rc = check_rows(who, dtype, param_dtype, rows, dim);
    if (!rc) rc = check_matrix(who, "dy", dy, dy_stride, rows, dim, dtype);
    if (!rc) rc = check_matrix(who, "x", x, x_stride, rows, dim, dtype);
    if (!rc) rc = check_matrix(who, "dx", dx, dx_stride, rows, dim, dtype);
    if (!rc) rc = check_matrix(who, "gamma", gamma, dim, 0, dim, param_dtype);
    if (!rc) rc = check_matrix(who, "dgamma", dgamma, dim, 0, dim, param_dtype);
    if (!rc) rc = check_matrix(who, "dbeta", dbeta, dim, 0, dim, param_dtype);
    if (rc) return rc;
    if (rows > 0 && (!mean || !rstd))
        return fail(SS_ERR_INVALID_ARG, "%s: mean or rstd is NULL", who);
    if (rows > 1 && ((dx == dy && dx_stride != dy_stride) || (dx == x && dx_stride != x_stride)))
        return fail(SS_ERR_INVALID_ARG, "%s: dx is dy or x with another stride", who);
    const bool params = dgamma || dbeta;
    if (params && (!ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0 ||
                   ws_bytes < ss_layernorm_rows_workspace_bytes(rows, dim)))
        return fail(SS_ERR_WORKSPACE, "%s: workspace missing, misaligned or under %zu bytes", who,
                    ss_layernorm_rows_workspace_bytes(rows, dim));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int per = dtype == SS_F32 ? 4 : 8;
    const Shape sh = shape_of(dim, per, 2);
    float *part = params ? static_cast<float *>(ws) : nullptr;
    int n_part = 0;
    if (rows > 0) {
        const int most = most_parts(rows, dim);
#define SS_ROWS_BWD                                                                           \
    const int64_t groups = wg_size<LANES>() / LANES, need = (rows + groups - 1) / groups;     \
    n_part = (int)(need < most ? need : most);                                                \
    ProfScope prof("rows_backward_kernel", st);                                               \
    launch(rows_backward_kernel<DT, WT, LANES, P>, dim3(n_part), dim3(wg_size<LANES>()), st,  \
           dy, dy_stride, x, x_stride, rows, n_valid, gamma, mean, rstd, dx, dx_stride, dim,  \
           part)
#define SS_ROWS_WIDE                                                                          \
    if (params) {                    /* first: dx may be dy or x */                           \
        n_part = most;                                                                        \
        ProfScope prof("wide_columns_kernel", st);                                            \
        launch(wide_columns_kernel<DT>, dim3((dim + kWG * per - 1) / (kWG * per), n_part),    \
               dim3(kWG), st, dy, dy_stride, x, x_stride, rows, n_valid, mean, rstd, dim,     \
               part);                                                                         \
    }                                                                                         \
    ProfScope prof("rows_backward_kernel", st);                                               \
    launch(wide_backward_kernel<DT, WT>, dim3(rows < kForwardWgs ? rows : kForwardWgs),       \
           dim3(kWideThreads), st, dy, dy_stride, x, x_stride, rows, n_valid, gamma, mean,    \
           rstd, dx, dx_stride, dim)
        SS_ROWS_TYPES(dtype, param_dtype, SS_ROWS_SHAPES(SS_ROWS_BWD) else { SS_ROWS_WIDE; })
#undef SS_ROWS_BWD
#undef SS_ROWS_WIDE
    }
    if (params) {
        ProfScope prof("columns_reduce_kernel", st);
        const dim3 grid((dim + kRedCols - 1) / kRedCols, 2);
        SS_ROWS_TYPES(param_dtype, param_dtype,
                      launch(columns_reduce_kernel<WT>, grid, dim3(kRedCols * kParts), st,
                             (const float *)part, n_part, dim, dgamma, dbeta));
    }
    return check_launch(who);
}

}  // extern "C"
