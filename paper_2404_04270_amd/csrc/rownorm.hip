// Layer normalization of the rows of a matrix in fp32, bf16 or fp16, forward and backward: the
// dense vectors of section 3.5 (layernorm.hip has the pooled ones).
//
// Bound by HBM: the forward pass reads x and writes y, the backward pass reads dy and x and writes
// dx.  A group of lanes owns a row and keeps it in registers, so that every element is read once; the
// statistics come from the registers in two passes (the mean, then the centred squares: a row whose
// mean is large against its spread keeps its digits).  Groups are as narrow as the row allows, from
// one lane to a workgroup of 512; wider rows are read again for each pass, from the caches as long as
// the rows under way fit them (below).  While a group works on a row its next one is being loaded.
// The backward pass gives a workgroup rows that are a grid apart and sums their products column by
// column in registers; one partial row per workgroup goes to memory, and a second kernel adds those
// in order.
//
// us, and TB/s of x, y, dy and dx (a device-wide addition of a constant reaches 6.2): forward
// 16384 x 8192 bf16 89 (6.1), 65536 x 512 fp16 22.7 (5.9), 10007 x 1001 fp32 13.3 (6.0, partly from the
// last-level cache); backward 32768 x 4096 bf16 139 (5.8), 16384 x 4096 fp32 139 (5.8),
// 16384 x 1024 bf16 22.2 (4.5), 10007 x 1001 fp16 18 (3.4), each with about 4 us for the second
// kernel.  Widths just above a border leave lanes without elements: 16384 x 1025 bf16 21.6 forward and
// 33.7 backward (1024: 13.0 and 22.5), x 4097 67.7 and 109 (4096: 48.4 and 75.3), 7000 x 9001 fp16 73
// and 105 (3.4 and 3.6).  Wide rows: 4096 x 20000 bf16 90 and 200 (3.6 and 2.5), 256 x 262144 110 and
// 221, 64 x 1048576 294 and 581 (0.9 and 0.7: 64 workgroups, and more rows under way than the caches
// hold).
#include "elem_io.h"
#include "ss_common.h"

namespace ss {
namespace {

constexpr int kStreamOut = 1, kStreamIn = 2;       // past the caches

// Elements per 16-byte access.
template <int DT> constexpr int per_access() { return DT == SS_F32 ? 4 : 8; }

// Threads of a workgroup: forward few, so that several share a compute unit; backward 512, since
// every workgroup ends in a partial row of the parameters' gradients.  (With 1024 each of them has
// 128 registers and spills: 32768 x 4096 bf16 backward 159 us, 150 with 512.)
template <int LANES> constexpr int fwd_threads() { return LANES > kWG ? LANES : kWG; }
constexpr int kBwdThreads = 512;

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Sum over W lanes (a power of two, at most a wavefront) that start at a multiple of W; in all of
// them.  Exchanges inside a row of 16 lanes are part of the addition, the two beyond are swaps of rows
// and of halves: nothing goes through LDS.
template <int W> __device__ __forceinline__ float lane_sum(float v)
{
    if constexpr (W >= 2) v += dpp<0xB1>(v);           // quad_perm 1 0 3 2
    if constexpr (W >= 4) v += dpp<0x4E>(v);           // quad_perm 2 3 0 1
    if constexpr (W >= 8) v += dpp<0x141>(v);          // row_half_mirror
    if constexpr (W >= 16) v += dpp<0x140>(v);         // row_mirror
    if constexpr (W >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                        false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if constexpr (W >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                        false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return v;
}

// Sums of K values over the group of lanes that owns a row; in all of them.  A group of several
// wavefronts passes through `s` (a float per wavefront of the workgroup and value), which is free
// again behind the next barrier.
template <int LANES, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float *s)
{
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lane_sum<(LANES < 64 ? LANES : 64)>(v[k]);
    if constexpr (LANES > 64) {
        constexpr int WAVES = LANES / 64;
        const int wave = threadIdx.x / 64;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) s[wave * K + k] = v[k];
        __syncthreads();
        const float *mine = s + wave / WAVES * WAVES * K;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[k] += mine[w * K + k];
        }
    }
}
template <int LANES> __device__ __forceinline__ float row_sum(float v, float *s)
{
    float one[1] = {v};
    row_sums<LANES, 1>(one, s);
    return one[0];
}

// Columns [col, col + count) of a row belong to a lane's vector of N (count <= 0: none).
template <int LANES, int N> struct Columns {
    int col, count;
    __device__ __forceinline__ Columns(int i, int c, int dim)
        : col((i * LANES + c) * N), count(dim - col < N ? dim - col : N)
    {
    }
};

// Between the two sides of a branch that differ in nothing but the cache policy of an access: the
// compiler would make one access of them, and take the policy of neither.
__device__ __forceinline__ void apart() { asm volatile(""); }

// Zeros past the row.  The last vector of a row that is no multiple of N is read where it ends with the
// row (there is room for that: a row of several lanes is longer than N) and shifted down: one load
// for a lane where elements taken one by one would cost its whole wavefront N.  The shift is a step
// of its own, so that asking for a row does not wait for it.
template <int DT, int LANES, int N>
__device__ __forceinline__ Raw<DT, N> ask_columns(const void *base, int64_t row,
                                                  const Columns<LANES, N> &at,
                                                  bool stream = false)
{
    if constexpr (LANES == 1) {
        if (at.count < N) return load_raw_part<DT, N>(base, row + at.col, at.count);
        return load_raw<DT, N>(base, row + at.col);
    }
    Raw<DT, N> r;
    r.v = 0.0f;
    if (at.count > 0) {
        const int64_t from = row + at.col + at.count - N;
        if (stream) {
            apart();
            r = load_raw<DT, N, true>(base, from);
            apart();
        } else {
            r = load_raw<DT, N>(base, from);
        }
    }
    return r;
}
template <int DT, int LANES, int N>
__device__ __forceinline__ void settle(Raw<DT, N> &r, const Columns<LANES, N> &at)
{
    if (LANES == 1 || at.count == N || at.count <= 0) return;
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(Raw<DT, N>) / 4)));
    constexpr int W = sizeof(words) / 4, kSize = sizeof(typename Raw<DT, N>::E);
    words w = __builtin_bit_cast(words, r.v);
    const int bytes = (N - at.count) * kSize;
    if constexpr (W >= 8)
        if (bytes & 16)
#pragma unroll
            for (int j = 0; j < W; ++j) w[j] = j + 4 < W ? w[j + 4] : 0u;
    if (bytes & 8)
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = j + 2 < W ? w[j + 2] : 0u;
    if (bytes & 4)
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = j + 1 < W ? w[j + 1] : 0u;
    if (kSize == 2 && (bytes & 2))
#pragma unroll
        for (int j = 0; j < W; ++j)
            w[j] = __builtin_amdgcn_alignbyte(j + 1 < W ? w[j + 1] : 0u, w[j], 2);
    r.v = __builtin_bit_cast(typename Raw<DT, N>::V, w);
}
// The first n of four, n < 4.
template <int DT>
__device__ __forceinline__ void store_rest(void *base, int64_t at, int n, const Raw<DT, 4> &r)
{
    Raw<DT, 2> two;
    two.v = __builtin_shufflevector(r.v, r.v, 0, 1);
    if (n & 2) store_raw<DT, 2>(base, at, two);
    Raw<DT, 1> one;
    one.v = n & 2 ? r.v[2] : r.v[0];
    if (n & 1) store_raw<DT, 1>(base, at + (n & 2), one);
}
// A row's rest of fewer than N columns: in up to log2(N) stores.
template <int DT, int LANES, int N>
__device__ __forceinline__ void store_columns(void *base, int64_t row, const Columns<LANES, N> &at,
                                              const float (&f)[N], bool stream = false)
{
    const Raw<DT, N> r = from_float<DT, N>(f);
    if (at.count == N) {
        if (stream) {
            apart();
            store_raw<DT, N, true>(base, row + at.col, r);
            apart();
        } else {
            store_raw<DT, N>(base, row + at.col, r);
        }
    } else if (at.count > 0) {
        if constexpr (N == 8) {
            Raw<DT, 4> four;
            four.v = __builtin_shufflevector(r.v, r.v, 0, 1, 2, 3);
            const bool low = (at.count & 4) != 0;
            if (low) store_raw<DT, 4>(base, row + at.col, four);
            four.v = low ? __builtin_shufflevector(r.v, r.v, 4, 5, 6, 7) : four.v;
            store_rest<DT>(base, row + at.col + (at.count & 4), at.count & 3, four);
        } else {
            store_rest<DT>(base, row + at.col, at.count, r);
        }
    }
}
// The parameters of a lane's columns; `absent` where there are none.
template <int WT, int LANES, int N>
__device__ __forceinline__ void load_params(const void *p, const Columns<LANES, N> &at, float absent,
                                            float (&f)[N])
{
    if (p) {
        Raw<WT, N> r = ask_columns<WT>(p, 0, at);
        settle(r, at);
        to_float(r, f);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = absent;
    }
}
// The same bits, which the compiler takes for others: what was worked out of them is worked out again
// instead of being kept.
template <int DT, int N> __device__ __forceinline__ void forget(Raw<DT, N> &r)
{
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(r.v) / 4)));
    words w = __builtin_bit_cast(words, r.v);
    asm("" : "+v"(w));
    r.v = __builtin_bit_cast(typename Raw<DT, N>::V, w);
}

// Which of the workgroup's groups of lanes this is: a scalar where wavefronts are not shared, and
// with it everything that goes by the row.
template <int LANES> __device__ __forceinline__ uint32_t group_of_lanes()
{
    const int g = threadIdx.x / LANES;
    return LANES >= 64 ? __builtin_amdgcn_readfirstlane(g) : g;
}

template <int DT, int WT, int LANES, int P>
__global__ __launch_bounds__(fwd_threads<LANES>()) void rows_forward_kernel(
    const void *x, int64_t x_stride, int rows, const int32_t *__restrict__ n_valid,
    const void *gamma, const void *beta, float eps, void *y, int64_t y_stride,
    float *__restrict__ mean, float *__restrict__ rstd, int dim, int flow)
{
    constexpr int N = per_access<DT>(), T = fwd_threads<LANES>(), NG = T / LANES;
    __shared__ float s[2][LANES > 64 ? T / 64 : 1];
    const uint32_t n = clamp_valid(n_valid, rows), step = gridDim.x * NG;
    const int c = threadIdx.x % LANES;
    const float inv = 1.0f / (float)dim;
    uint32_t r = blockIdx.x * NG + group_of_lanes<LANES>();
    int64_t x_at = r * x_stride, y_at = r * y_stride;
    Raw<DT, N> raw[P];
    const auto ask = [&] {
#pragma unroll
        for (int i = 0; i < P; ++i)
            raw[i] = ask_columns<DT>(x, x_at, Columns<LANES, N>(i, c, dim), flow & kStreamIn);
    };
    if (r < n) ask();
    float gam[P][N], bet[P][N];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        load_params<WT>(gamma, Columns<LANES, N>(i, c, dim), 1.0f, gam[i]);
        load_params<WT>(beta, Columns<LANES, N>(i, c, dim), 0.0f, bet[i]);
    }
    for (; r < n; r += step, y_at += step * y_stride) {
        float v[P][N], sum = 0.0f, q = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            settle(raw[i], Columns<LANES, N>(i, c, dim));
            to_float(raw[i], v[i]);
        }
        x_at += step * x_stride;
        if (r + step < n) ask();           // the next row is under way while this one is worked on
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) sum += v[i][e];
        const float mu = row_sum<LANES>(sum, s[0]) * inv;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int count = Columns<LANES, N>(i, c, dim).count;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                v[i][e] = e < count ? v[i][e] - mu : 0.0f;
                q = fmaf(v[i][e], v[i][e], q);
            }
        }
        const float rs = 1.0f / sqrtf(fmaf(row_sum<LANES>(q, s[1]), inv, eps));
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float o[N];
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = fmaf(v[i][e] * rs, gam[i][e], bet[i][e]);
            store_columns<DT>(y, y_at, Columns<LANES, N>(i, c, dim), o, flow & kStreamOut);
        }
        if (c == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
    }
}

// Whether vector i lies past the row for all lanes of this wavefront.
template <int LANES, int N> __device__ __forceinline__ bool past(int i, int dim)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x % LANES / 64);
    return (i * LANES + wave * 64) * N >= dim;
}

// part: [2][gridDim.x][dim], the products' sums and the gradients' sums.  A workgroup that is alone
// writes dgamma and dbeta itself and needs no part.
template <int DT, int WT, int LANES, int P>
__global__ __launch_bounds__(kBwdThreads) void rows_backward_kernel(
    const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int rows,
    const int32_t *__restrict__ n_valid, const void *gamma, const float *__restrict__ mean,
    const float *__restrict__ rstd, void *dx, int64_t dx_stride, int dim, int flow,
    float *__restrict__ part, void *dgamma, void *dbeta)
{
    constexpr int N = per_access<DT>(), T = kBwdThreads, NG = T / LANES;
    // A lane with 32 elements has its column sums in LDS (128 KB of it; no other lane reads them) and
    // gamma as it came: the registers are for the next row.  4096 x 16384 bf16 84 us, with the sums
    // in registers and no row ahead 114; 4096 x 10000 fp32 97 and 124, 7000 x 9000 fp16 91 and 150.
    // Its wavefronts leave out the vectors past the row (7000 x 9000 fp16 102 us without; where a row
    // of fewer elements has several vectors per lane it costs as much as it saves).
    constexpr bool kLds = P * N > 16;
    typedef float quad __attribute__((ext_vector_type(4)));
    __shared__ quad s_acc[kLds ? 2 * P * N / 4 : 1][kLds ? T : 1];
    __shared__ float s[2][LANES > 64 ? T / 64 * 2 : 1];
    __shared__ float s_col[NG > 1 ? T * N : 1];
    const uint32_t n = clamp_valid(n_valid, rows), step = gridDim.x * NG;
    int c = threadIdx.x % LANES;
    const float inv = 1.0f / (float)dim;
    uint32_t r = blockIdx.x * NG + group_of_lanes<LANES>();
    int64_t x_at = r * x_stride, dy_at = r * dy_stride, dx_at = r * dx_stride;
    Raw<DT, N> xn[P], dn[P];               // the next row's
    float mu_n = 0.0f, rs_n = 0.0f;
    const auto ask = [&](uint32_t row) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const Columns<LANES, N> at(i, c, dim);
            xn[i] = ask_columns<DT>(x, x_at, at, flow & kStreamIn);
            dn[i] = ask_columns<DT>(dy, dy_at, at, flow & kStreamIn);
        }
        mu_n = mean[row];
        rs_n = rstd[row];
    };
    if (r < n) ask(r);
    Raw<kLds ? WT : SS_F32, N> gam[P];
    float acc_g[P][N], acc_b[P][N];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float g[N];
        load_params<WT>(gamma, Columns<LANES, N>(i, c, dim), 1.0f, g);
        gam[i] = from_float<kLds ? WT : SS_F32, N>(g);
        if constexpr (kLds) {
#pragma unroll
            for (int e = 0; e < 2 * N / 4; ++e) s_acc[i * 2 * N / 4 + e][threadIdx.x] = 0.0f;
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) acc_g[i][e] = acc_b[i][e] = 0.0f;
        }
    }
    // groups of several wavefronts meet at barriers: all take the turns that the first one has
    uint32_t lead = blockIdx.x * NG;
    for (int turn = 0; (LANES > 64 ? lead : r) < n; turn ^= 1) {
        const bool here = LANES <= 64 || r < n;
        Raw<DT, N> xr[P], dr[P];
        float sums[2] = {0.0f, 0.0f};
        const float mu = mu_n, rs = rs_n;
        // the columns are worked out again for each row: kept, they and what is asked of them spill
        // (4096 x 16384 fp32 192 us, 156 without)
        if (kLds) asm volatile("" : "+v"(c));
#pragma unroll
        for (int i = 0; i < P; ++i) xr[i] = xn[i], dr[i] = dn[i];
        lead += step;
        r += step;
        x_at += step * x_stride;
        dy_at += step * dy_stride;
        if (r < n) ask(r);       // the next row is under way while this one is worked on
        if (here) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if (kLds && past<LANES, N>(i, dim)) break;
                float xf[N], df[N];
                settle(xr[i], Columns<LANES, N>(i, c, dim));
                settle(dr[i], Columns<LANES, N>(i, c, dim));
                to_float(xr[i], xf);
                to_float(dr[i], df);
                float gm[N];
                to_float(gam[i], gm);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    xf[e] = (xf[e] - mu) * rs;
                    if constexpr (!kLds) {
                        acc_g[i][e] = fmaf(df[e], xf[e], acc_g[i][e]);
                        acc_b[i][e] += df[e];
                    }
                }
                if constexpr (kLds) {
#pragma unroll
                    for (int e = 0; e < N; e += 4) {
                        quad &g = s_acc[(i * N + e) / 2][threadIdx.x];
                        quad &b = s_acc[(i * N + e) / 2 + 1][threadIdx.x];
                        quad tg = g, tb = b;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            tg[k] = fmaf(df[e + k], xf[e + k], tg[k]);
                            tb[k] += df[e + k];
                        }
                        g = tg;
                        b = tb;
                    }
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    df[e] *= gm[e];                  // 0 past the row
                    sums[0] += df[e];
                    sums[1] = fmaf(df[e], xf[e], sums[1]);
                }
                if (kLds) __builtin_amdgcn_sched_barrier(0);
            }
        }
        row_sums<LANES, 2>(sums, s[turn]);
        const float m1 = sums[0] * inv, m2 = sums[1] * inv;
        if (here) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if (kLds && past<LANES, N>(i, dim)) break;
                float xf[N], df[N], o[N];
                forget(xr[i]);
                forget(dr[i]);
                to_float(xr[i], xf);
                to_float(dr[i], df);
                float gm[N];
                to_float(gam[i], gm);
#pragma unroll
                for (int e = 0; e < N; ++e)
                    o[e] = fmaf((mu - xf[e]) * rs, m2, fmaf(df[e], gm[e], -m1)) * rs;
                store_columns<DT>(dx, dx_at, Columns<LANES, N>(i, c, dim), o, flow & kStreamOut);
                if (kLds) __builtin_amdgcn_sched_barrier(0);
            }
        }
        dx_at += step * dx_stride;
    }
    if (!dgamma && !dbeta) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        void *const own = which ? dbeta : dgamma;
        if (!own) continue;
        float *out = part + ((int64_t)which * gridDim.x + blockIdx.x) * dim;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const Columns<LANES, N> at(i, c, dim);
            float t[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if constexpr (kLds) t[e] = s_acc[(i * N + e) / 4 * 2 + which][threadIdx.x][e % 4];
                else t[e] = which ? acc_b[i][e] : acc_g[i][e];
            }
            if constexpr (NG > 1) {                      // the groups' sums, in their order
                __syncthreads();
#pragma unroll
                for (int e = 0; e < N; ++e) s_col[e * T + threadIdx.x] = t[e];
                __syncthreads();
                // column j of this vector belongs to element j % N of lane j / N of each group
                for (int j = threadIdx.x; j < LANES * N; j += T) {
                    const int col = i * LANES * N + j;
                    if (col >= dim) break;
                    float sum = 0.0f;
                    for (int o = 0; o < NG; ++o) sum += s_col[j % N * T + o * LANES + j / N];
                    typedef typename ElemOf<WT>::type W;
                    if (gridDim.x == 1) static_cast<W *>(own)[col] = (W)sum;
                    else out[col] = sum;
                }
            } else if (gridDim.x == 1) {
                store_columns<WT>(own, 0, at, t);
            } else {
                store_columns<SS_F32>(out, 0, at, t);
            }
        }
    }
}

// ---- rows wider than a workgroup's registers ------------------------------------------------
constexpr int kWideThreads = 1024;

template <int DT, int N>
__device__ __forceinline__ Raw<DT, N> load_some(const void *base, int64_t row, int col, int dim)
{
    if (col + N <= dim) return load_raw<DT, N>(base, row + col);
    return load_raw_part<DT, N>(base, row + col, dim - col);
}
template <int DT, int N>
__device__ __forceinline__ void store_some(void *base, int64_t row, int col, int dim,
                                           const float (&f)[N])
{
    const Raw<DT, N> r = from_float<DT, N>(f);
    if (col + N <= dim) store_raw<DT, N>(base, row + col, r);
    else store_raw_part<DT, N>(base, row + col, r, dim - col);
}
template <int WT, int N>
__device__ __forceinline__ void some_params(const void *p, int col, int dim, float absent,
                                            float (&f)[N])
{
    if (p) {
        to_float(load_some<WT, N>(p, 0, col, dim), f);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = absent;
    }
}

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
            const Raw<DT, N> raw = load_some<DT, N>(x, r * x_stride, col, dim);
            float f[N];
            to_float(raw, f);
#pragma unroll
            for (int k = 0; k < N; ++k) sum += f[k];
        }
        const float mu = row_sum<T>(sum, s[0]) * inv;
        for (int col = threadIdx.x * N; col < dim; col += T * N) {
            const Raw<DT, N> raw = load_some<DT, N>(x, r * x_stride, col, dim);
            float f[N];
            to_float(raw, f);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float d = col + k < dim ? f[k] - mu : 0.0f;
                q = fmaf(d, d, q);
            }
        }
        const float rs = 1.0f / sqrtf(fmaf(row_sum<T>(q, s[1]), inv, eps));
        for (int col = threadIdx.x * N; col < dim; col += T * N) {
            const Raw<DT, N> raw = load_some<DT, N>(x, r * x_stride, col, dim);
            float f[N], gam[N], bet[N];
            some_params<WT, N>(gamma, col, dim, 1.0f, gam);
            some_params<WT, N>(beta, col, dim, 0.0f, bet);
            to_float(raw, f);
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = fmaf((f[k] - mu) * rs, gam[k], bet[k]);
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
                const Raw<DT, N> xr = load_some<DT, N>(x, r * x_stride, col, dim);
                const Raw<DT, N> dr = load_some<DT, N>(dy, r * dy_stride, col, dim);
                float xf[N], df[N], gam[N];
                some_params<WT, N>(gamma, col, dim, 1.0f, gam);
                to_float(xr, xf);
                to_float(dr, df);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float xh = (xf[k] - mu) * rs, gd = gam[k] * df[k];
                    s1 += gd;
                    s2 = fmaf(gd, xh, s2);
                    df[k] = fmaf(-xh, m2, fmaf(gam[k], df[k], -m1)) * rs;
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
        const Raw<DT, N> xr = load_some<DT, N>(x, r * x_stride, (int)col, dim);
        const Raw<DT, N> dr = load_some<DT, N>(dy, r * dy_stride, (int)col, dim);
        float xf[N], df[N];
        const float mu = mean[r], rs = rstd[r];
        to_float(xr, xf);
        to_float(dr, df);
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
constexpr int kRedCols = 32, kParts = 32;

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
        for (int w0 = p; w0 < n_part; w0 += kParts * 8) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int w = w0 + k * kParts;
                v[k] = w < n_part ? in[(int64_t)w * dim + col] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[k];
        }
    }
    s[p][c] = sum;
    __syncthreads();
    if (p == 0 && col < dim) {
#pragma unroll
        for (int q = 1; q < kParts; ++q) sum += s[q][c];
        static_cast<typename ElemOf<WT>::type *>(out)[col] = (typename ElemOf<WT>::type)sum;
    }
}

// ---- which kernel takes a row ---------------------------------------------------------------
// The narrowest group whose lanes hold the row in one vector each, up to a wavefront (sums then stay
// within rows of lanes); then up to 16 elements per lane, of one, four and eight wavefronts, which a
// barrier joins; then 32 per lane.  (8192 to 16384 elements as 16 per lane of 1024 threads spill
// backward: 4096 x 16384 bf16 126 to 149 us.)
struct Shape {
    int lanes, vectors;        // lanes == 0: too wide for registers
};

Shape shape_of(int dim, int per)
{
    const int v = (dim + per - 1) / per, most = 16 / per;       // vectors of a row; a lane's at most
    int lanes = 1;
    while (lanes < v && lanes < 64) lanes *= 2;
    for (; lanes <= 512; lanes *= lanes == 64 ? 4 : 2)
        for (int p = 1; p <= most; p *= 2)
            if (v <= lanes * p && (lanes <= 256 || p == most)) return {lanes, p};
    if (v <= 512 * 2 * most) return {512, 2 * most};
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
    else SS_ROWS_FULL(64, __VA_ARGS__) else SS_ROWS_CASE(256, 1, __VA_ARGS__)                 \
    else SS_ROWS_CASE(256, 2, __VA_ARGS__) else SS_ROWS_FULL(256, __VA_ARGS__)                \
    else SS_ROWS_FULL(512, __VA_ARGS__) else SS_ROWS_TWICE(__VA_ARGS__)
#define SS_ROWS_TWICE(...)                                                                    \
    if (sh.lanes == 512 && sh.vectors == 32 / per_access<DT>()) { constexpr int LANES = 512, P = 32 / per_access<DT>(); __VA_ARGS__; }
// 16 elements a lane
#define SS_ROWS_FULL(l, ...)                                                                  \
    if (sh.lanes == l && sh.vectors == 16 / per_access<DT>()) { constexpr int LANES = l, P = 16 / per_access<DT>(); __VA_ARGS__; }

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

// Threads of a forward launch: four wavefronts per SIMD.  With half / twice as many 16384 x 2048 bf16
// takes 34.2 / 26.9 us instead of 26.6, 16384 x 1024 14.5 / 14.5 instead of 13.2.
constexpr int kForwardThreads = 256 * 1024;
constexpr int kWideWgs = 1024;
// Workgroups of a backward launch: one per compute unit.  Two where a lane has one vector of a row,
// and so half as much under way: 16384 x 2048 bf16 44 us with two and 55 with one, 300000 x 100
// fp32 71 and 81.  Elsewhere the second adds partial rows and nothing else: 32768 x 4096 bf16 157 and
// 150, 2048 x 4096 19.6 and 17.2, 16384 x 1024 29.3 and 24.4.  The same without column sums: with up to
// 1024 workgroups 10007 x 1001 fp16 takes 17.1 instead of 12.8 us, 16384 x 1024 bf16 20.4 and 17.2,
// 300000 x 100 fp32 71 and 65, 7000 x 9001 fp16 96 and 91, 4096 x 16384 bf16 80 and 71 (32768 x 4096
// bf16 132 and 136, 8192 x 8192 67 and 69).
constexpr int kBackwardWgs = 256;
// Up to so many rows per group of lanes and elements in all one workgroup takes them, if there are
// column sums, and has no second launch: from call to call 128 x 64 fp32 8.7 instead of 11.9 us,
// 32 x 1024 bf16 9.6 and 12.2, 4 x 8192 fp32 9.1 and 12.0, 3 x 9000 bf16 10.3 and 11.9.  Of rows of 32
// elements per lane each takes 2 to 4 us: 2 x 16384 bf16 / fp32 10.4 / 12.2 and 12.1 / 11.8, 4 x 9000
// bf16 12.6 and 11.9, 4 x 16384 bf16 / fp32 17.6 / 21.2 and 12.0 / 12.1 (without column sums 16.5 / 19.7
// and 7.3).
constexpr int kAloneRows = 4;
constexpr int64_t kAloneElems = 32768;

// What goes past the caches.  Results do from 32 MB on, where none of them would stay in the L2s (below,
// whoever reads them next would lose), if their rows start at even places: 65536 x 512 fp16 forward
// 26.1 -> 22.7 us, 16384 x 2048 bf16 26.2 -> 22.9, 32768 x 4096 bf16 backward 150 -> 146 (odd places:
// 10007 x 1001 fp32 forward 13.3 -> 14.9).  What is read does from 256 MB in all on, which is more
// than the last-level cache: 32768 x 4096 bf16 backward 146 -> 140, 16384 x 4096 fp32 152 -> 140, 16384 x
// 8192 bf16 forward 94 -> 92 (16384 x 2048 forward, 134 MB, 22.9 -> 25.7).
int flow_of(int rows, int dim, int dtype, const void *out, int64_t out_stride, int arrays)
{
    const int size = dtype == SS_F32 ? 4 : 2;
    const int64_t bytes = (int64_t)rows * dim * size;
    const bool even = ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(out_stride * size)) & 15) == 0;
    return (bytes >= 32 << 20 && even ? kStreamOut : 0) |
           (bytes * arrays >= 256 << 20 ? kStreamIn : 0);
}

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
    const Shape sh = shape_of(dim, dtype == SS_F32 ? 4 : 8);
    const int flow = flow_of(rows, dim, dtype, y, y_stride, 2);
    ProfScope prof("rows_forward_kernel", st);
#define SS_ROWS_FWD                                                                           \
    const int threads = fwd_threads<LANES>();                                                 \
    const int64_t groups = threads / LANES, need = (rows + groups - 1) / groups;              \
    const int64_t most = kForwardThreads / threads;                                           \
    launch(rows_forward_kernel<DT, WT, LANES, P>, dim3((unsigned)(need < most ? need : most)),\
           dim3(threads), st, x, x_stride, rows, n_valid, gamma, beta, eps, y, y_stride, mean,\
           rstd, dim, flow)
    SS_ROWS_TYPES(dtype, param_dtype,
                  SS_ROWS_SHAPES(SS_ROWS_FWD) else launch(
                      wide_forward_kernel<DT, WT>, dim3(rows < kWideWgs ? rows : kWideWgs),
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
    const Shape sh = shape_of(dim, per);
    const int flow = flow_of(rows, dim, dtype, dx, dx_stride, 3);
    float *part = params ? static_cast<float *>(ws) : nullptr;
    int n_part = 0;
    if (rows > 0) {
        const int most = most_parts(rows, dim);
        const bool few = params && (int64_t)rows * dim <= kAloneElems;
#define SS_ROWS_BWD                                                                           \
    const int threads = kBwdThreads;                                                          \
    const int64_t groups = threads / LANES, need = (rows + groups - 1) / groups;              \
    n_part = (int)(need < most ? need : most);                                                \
    const int wgs = P > 1 ? kBackwardWgs : 2 * kBackwardWgs;                                  \
    n_part = few && need <= kAloneRows ? 1 : n_part < wgs ? n_part : wgs;                     \
    ProfScope prof("rows_backward_kernel", st);                                               \
    launch(rows_backward_kernel<DT, WT, LANES, P>, dim3(n_part), dim3(threads), st, dy,       \
           dy_stride, x, x_stride, rows, n_valid, gamma, mean, rstd, dx, dx_stride, dim,      \
           flow, part, dgamma, dbeta)
#define SS_ROWS_WIDE                                                                          \
    if (params) {                    /* first: dx may be dy or x */                           \
        n_part = most;                                                                        \
        ProfScope prof("wide_columns_kernel", st);                                            \
        launch(wide_columns_kernel<DT>, dim3((dim + kWG * per - 1) / (kWG * per), n_part),    \
               dim3(kWG), st, dy, dy_stride, x, x_stride, rows, n_valid, mean, rstd, dim,     \
               part);                                                                         \
    }                                                                                         \
    ProfScope prof("rows_backward_kernel", st);                                               \
    launch(wide_backward_kernel<DT, WT>, dim3(rows < kWideWgs ? rows : kWideWgs),             \
           dim3(kWideThreads), st, dy, dy_stride, x, x_stride, rows, n_valid, gamma, mean,    \
           rstd, dx, dx_stride, dim)
        SS_ROWS_TYPES(dtype, param_dtype, SS_ROWS_SHAPES(SS_ROWS_BWD) else { SS_ROWS_WIDE; })
#undef SS_ROWS_BWD
#undef SS_ROWS_WIDE
    }
    if (params && !(sh.lanes > 0 && n_part == 1)) {
        ProfScope prof("columns_reduce_kernel", st);
        const dim3 grid((dim + kRedCols - 1) / kRedCols, 2);
        SS_ROWS_TYPES(param_dtype, param_dtype,
                      launch(columns_reduce_kernel<WT>, grid, dim3(kRedCols * kParts), st,
                             (const float *)part, n_part, dim, dgamma, dbeta));
    }
    return check_launch(who);
}

}  // extern "C"
