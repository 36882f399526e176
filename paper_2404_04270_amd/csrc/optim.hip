// The optimizer of the parameters that are no tables: AdamW over the tensors of a list in one
// launch, with moments in 32 or in 8 bits, and the norm of all their gradients.
//
// All of it is bound by HBM.  A step in fp32 reads p, g, m and v and writes p, m and v, 28 bytes per
// element; with 8-bit moments and 16-bit parameters it is 10.  The work table cuts the tensors into
// chunks, a workgroup takes a chunk, and every access of a lane is as wide as its elements allow
// (8 or 16 bytes).  A chunk names its tensor, so that tensors of all sizes and types share a launch.
#include <math.h>

#include "elem_io.h"
#include "ss_common.h"

namespace ss {
namespace {

// An entry of the work table: elements [first, first + count) of a tensor, whose moments start
// at `state`.
struct Chunk {
    int64_t state, first;
    int32_t tensor, count;
    int32_t kind;              // dtype | grad_dtype << 2 | no_decay << 4
    int32_t reserved;
};
static_assert(sizeof(Chunk) == SS_CHUNK_BYTES, "the header says how large an entry is");

constexpr int kPass = 2048;                // elements that a workgroup takes at a time
constexpr int kChunk = 4 * kPass;

__device__ __forceinline__ Chunk load_chunk(const void *chunks, int64_t c)
{
    return static_cast<const Chunk *>(chunks)[c];
}

// ---- gradient norm ------------------------------------------------------------------------
constexpr int kNormWgs = 2048;             // eight workgroups per compute unit
constexpr int kFinalThreads = 1024;

template <int G>
__device__ __forceinline__ double chunk_squares(const void *g, const Chunk &c)
{
    constexpr int N = G == SS_F32 ? 4 : 8, U = G == SS_F32 ? 4 : 2;
    double sum = 0.0;
    for (int e0 = threadIdx.x * N; e0 < c.count; e0 += kWG * N * U) {
        Raw<G, N> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = e0 + u * kWG * N;
            if (e + N <= c.count) r[u] = load_raw<G, N>(g, c.first + e);
            else r[u] = load_raw_part<G, N>(g, c.first + e, c.count - e);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[N];
            to_float(r[u], f);
#pragma unroll
            for (int k = 0; k < N; ++k) sum = fma((double)f[k], (double)f[k], sum);
        }
    }
    return sum;
}

// The sum of a workgroup's values, in thread order; valid in thread 0.
template <int THREADS>
__device__ __forceinline__ double wg_sum(double v)
{
    __shared__ double s[THREADS / 64];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < THREADS / 64; ++w) v += s[w];
    return v;
}

__global__ __launch_bounds__(kWG) void norm_partial_kernel(const void *chunks, int num_chunks,
                                                           const void *const *grads,
                                                           double *__restrict__ part)
{
    double sum = 0.0;
    for (int64_t i = blockIdx.x; i < num_chunks; i += gridDim.x) {
        const Chunk c = load_chunk(chunks, i);
        const void *g = grads[c.tensor];
        switch (c.kind >> 2 & 3) {
        case SS_F32: sum += chunk_squares<SS_F32>(g, c); break;
        case SS_BF16: sum += chunk_squares<SS_BF16>(g, c); break;
        default: sum += chunk_squares<SS_F16>(g, c); break;
        }
    }
    sum = wg_sum<kWG>(sum);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kFinalThreads) void norm_final_kernel(const double *__restrict__ part,
                                                                   int n, double max_norm,
                                                                   double grad_scale,
                                                                   float *__restrict__ clip)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += kFinalThreads) sum += part[i];
    sum = wg_sum<kFinalThreads>(sum);
    if (threadIdx.x == 0) {
        const double norm = fabs(grad_scale) * sqrt(sum);
        const bool finite = norm < INFINITY;
        const double ratio = max_norm / (norm + 1e-6);
        clip[0] = (float)norm;
        clip[1] = finite ? (float)(grad_scale * (ratio < 1.0 ? ratio : 1.0)) : 0.0f;
        clip[2] = finite ? 1.0f : 0.0f;
        clip[3] = 0.0f;
    }
}

// ---- AdamW --------------------------------------------------------------------------------
// What a step needs apart from its tensors, in the caller's 64 bytes of counters.
struct Scalars {
    int64_t steps, left_out;
    float size;                // lr / (1 - beta1^t)
    float keep;                // 1 - lr * weight_decay
    float root;                // 1 / sqrt(1 - beta2^t)
    float factor;              // of the gradients
    uint32_t dither;           // of element 0
    int32_t apply;
    int32_t reserved[6];
};
static_assert(sizeof(Scalars) == 64, "the header says how large the counters are");

constexpr uint32_t kDitherElement = 0x6A09E667u;   // the fraction of sqrt(2)
constexpr uint32_t kDitherStep = 0x9E3779B9u;      // the golden ratio

// The step's part of the dither.  It has to change as if drawn: with t * kDitherStep alone an
// element's steps up come at even distances, which its value then follows (v 2 % too large under
// steady gradients).
__device__ __forceinline__ uint32_t mixed(uint32_t t)
{
    uint32_t h = t * kDitherStep;
    h = (h ^ h >> 15) * kDitherElement;
    h = (h ^ h >> 13) * kDitherStep;
    return h ^ h >> 16;
}

__global__ __launch_bounds__(64) void adamw_begin_kernel(Scalars *__restrict__ s,
                                                         const float *__restrict__ clip,
                                                         const float *__restrict__ lr_device,
                                                         double lr, double beta1, double beta2,
                                                         double weight_decay)
{
    if (threadIdx.x != 0) return;
    if (lr_device) lr = *lr_device;
    const bool apply = !clip || clip[2] != 0.0f;
    const int64_t t = s->steps + (apply ? 1 : 0);
    s->steps = t;
    if (!apply) s->left_out += 1;
    s->apply = apply;
    s->factor = clip ? clip[1] : 1.0f;
    // 1 - beta^t without the cancellation of a beta next to 1; log(0) gives 1
    s->size = (float)(lr / -expm1((double)t * log(beta1)));
    s->keep = (float)(1.0 - lr * weight_decay);
    s->root = (float)(1.0 / sqrt(-expm1((double)t * log(beta2))));
    s->dither = mixed((uint32_t)t);
}

struct Betas {
    float b1, c1, b2, c2, eps;     // c = 1 - b, rounded from the difference in fp64
};

// The new moments.  No product becomes part of an FMA: packed moments are rounded by comparison, and
// then a last bit decides between two codes.
__device__ __forceinline__ void moments(float g, float &m, float &v, const Betas &k)
{
#pragma clang fp contract(off)
    m = k.b1 * m + k.c1 * g;
    v = k.b2 * v + k.c2 * (g * g);
}

__device__ __forceinline__ float stepped(float p, float m, float v, const Betas &k,
                                         const Scalars &s, float keep)
{
    return p * keep - s.size * (m / (sqrtf(v) * s.root + k.eps));
}

// The stored copy of a parameter is what its 16-bit value is rounded from: without this the last FMA
// of a step and the conversion to fp16 become one instruction that rounds once.
template <int N> __device__ __forceinline__ void as_stored(float (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm("" : "+v"(f[i]));
}

// Elements [e, e + N) of a chunk, n of them there.
template <int P, int G, bool MASTER, bool WHOLE>
__device__ __forceinline__ void step_four(const Chunk &c, int e, int n, void *p, const void *g,
                                          float *m, float *v, float *master, const Betas &k,
                                          const Scalars &s, float keep)
{
    constexpr int N = 4;
    const int64_t at = c.first + e, st = c.state + e;
    Raw<P, N> pr;
    Raw<G, N> gr;
    if (WHOLE) {
        if (!MASTER) pr = load_raw<P, N>(p, at);
        gr = load_raw<G, N>(g, at);
    } else {
        if (!MASTER) pr = load_raw_part<P, N>(p, at, n);
        gr = load_raw_part<G, N>(g, at, n);
    }
    const f4 m4 = *(gptr<const f4>)(m + st), v4 = *(gptr<const f4>)(v + st);
    float pf[N], gf[N], mf[N], vf[N];
    if (MASTER) {
        const f4 p4 = *(gptr<const f4>)(master + st);
#pragma unroll
        for (int i = 0; i < N; ++i) pf[i] = p4[i];
    } else {
        to_float(pr, pf);
    }
    to_float(gr, gf);
    f4 mo, vo, po;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        mf[i] = m4[i];
        vf[i] = v4[i];
        if (!WHOLE && i >= n) gf[i] = mf[i] = vf[i] = pf[i] = 0.0f;
        moments(gf[i] * s.factor, mf[i], vf[i], k);
        pf[i] = stepped(pf[i], mf[i], vf[i], k, s, keep);
        mo[i] = mf[i];
        vo[i] = vf[i];
        po[i] = pf[i];
    }
    *(gptr<f4>)(m + st) = mo;
    *(gptr<f4>)(v + st) = vo;
    if (MASTER) *(gptr<f4>)(master + st) = po;
    if (MASTER) as_stored(pf);
    const Raw<P, N> pw = from_float<P, N>(pf);
    if (WHOLE) store_raw<P, N>(p, at, pw);
    else store_raw_part<P, N>(p, at, pw, n);
}

template <int P, int G, bool MASTER>
__device__ __forceinline__ void step_chunk(const Chunk &c, void *p, const void *g, float *m,
                                           float *v, float *master, const Betas &k,
                                           const Scalars &s, float keep)
{
    constexpr int N = 4;
    for (int e = threadIdx.x * N; e < c.count; e += kWG * N) {
        if (e + N <= c.count)
            step_four<P, G, MASTER, true>(c, e, N, p, g, m, v, master, k, s, keep);
        else
            step_four<P, G, MASTER, false>(c, e, c.count - e, p, g, m, v, master, k, s, keep);
    }
}

#define SS_DISPATCH_KIND(kind, with_master, ...)                                              \
    switch ((kind) & 15) {                                                                    \
    case SS_F32 | SS_F32 << 2: { constexpr int P = SS_F32, G = SS_F32; constexpr bool MASTER = false; __VA_ARGS__; } break; \
    case SS_BF16 | SS_BF16 << 2: { constexpr int P = SS_BF16, G = SS_BF16; SS_WITH_MASTER(with_master, __VA_ARGS__) } break; \
    case SS_BF16 | SS_F32 << 2: { constexpr int P = SS_BF16, G = SS_F32; SS_WITH_MASTER(with_master, __VA_ARGS__) } break; \
    case SS_F16 | SS_F16 << 2: { constexpr int P = SS_F16, G = SS_F16; SS_WITH_MASTER(with_master, __VA_ARGS__) } break; \
    default: { constexpr int P = SS_F16, G = SS_F32; SS_WITH_MASTER(with_master, __VA_ARGS__) } break; \
    }
#define SS_WITH_MASTER(with_master, ...)                                                      \
    if (with_master) { constexpr bool MASTER = true; __VA_ARGS__; }                           \
    else { constexpr bool MASTER = false; __VA_ARGS__; }

__global__ __launch_bounds__(kWG) void adamw_kernel(const void *chunks, void *const *params,
                                                    const void *const *grads, float *m, float *v,
                                                    float *master,
                                                    const Scalars *__restrict__ scalars, Betas k)
{
    const Scalars s = *scalars;
    if (!s.apply) return;
    const Chunk c = load_chunk(chunks, blockIdx.x);
    void *p = params[c.tensor];
    const void *g = grads[c.tensor];
    const float keep = c.kind & 16 ? 1.0f : s.keep;
    SS_DISPATCH_KIND(c.kind, master != nullptr,
                     step_chunk<P, G, MASTER>(c, p, g, m, v, master, k, s, keep));
}

// ---- AdamW with moments in 8 bits -----------------------------------------------------------
// A block of 128 elements belongs to 16 lanes of 8, so that its largest values are found with four
// exchanges inside a row of 16 lanes.
constexpr int kLane8 = 8;
typedef uint32_t w2 __attribute__((ext_vector_type(2)));
constexpr int kTopM = 14, kTopV = 30;      // exponent fields of a block's largest codes
constexpr uint32_t kInfBits = 0x7F800000u;

template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x)
{
    const uint32_t y = __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true);
    return x > y ? x : y;
}
// Largest of 16 lanes that lie in a row; in all of them.
__device__ __forceinline__ uint32_t row_max(uint32_t x)
{
    x = max_dpp<0xB1>(x);          // quad_perm 1 0 3 2
    x = max_dpp<0x4E>(x);          // quad_perm 2 3 0 1
    x = max_dpp<0x141>(x);         // row_half_mirror
    return max_dpp<0x140>(x);      // row_mirror
}

__device__ __forceinline__ float unpack_m(uint32_t word, int k, int shift)
{
    const uint32_t b = (uint32_t)((int32_t)(word << (24 - 8 * k)) >> 4) & 0x87F00000u;
    return ldexpf(__uint_as_float(b), shift);
}
__device__ __forceinline__ float unpack_v(uint32_t word, int k, int shift)
{
    const uint32_t b = (word >> (8 * k) & 255u) << 20;
    return ldexpf(__uint_as_float(b), shift);
}

__device__ __forceinline__ int field_of(uint32_t bits, int least)
{
    const int b = (int)(bits >> 23);
    return b > least ? b : least;
}

template <int P, int G, bool MASTER>
__device__ __forceinline__ void step_chunk8(const Chunk &c, void *p, const void *g, uint8_t *mc,
                                            uint8_t *vc, uint8_t *exps, float *master,
                                            const Betas &k, const Scalars &s, float keep)
{
    constexpr int N = kLane8;
    // whole blocks: the lanes of one stay together
    for (int e = threadIdx.x * N; e / SS_MOMENT_BLOCK * SS_MOMENT_BLOCK < c.count; e += kWG * N) {
        const int64_t at = c.first + e, st = c.state + e;
        const int n = c.count - e;         // elements there; may be 0 or less
        Raw<P, N> pr;
        Raw<G, N> gr;
        if (n >= N) {
            if (!MASTER) pr = load_raw<P, N>(p, at);
            gr = load_raw<G, N>(g, at);
        } else {
            if (!MASTER) pr = load_raw_part<P, N>(p, at, n);
            gr = load_raw_part<G, N>(g, at, n);
        }
        const w2 mw = *(gptr<const w2>)(mc + st), vw = *(gptr<const w2>)(vc + st);
        const uint32_t ex = *(gptr<const uint16_t>)(exps + st / SS_MOMENT_BLOCK * 2);
        float pf[N], gf[N], m[N], v[N];
        if (MASTER) {
            const f4 a = *(gptr<const f4>)(master + st), b = *(gptr<const f4>)(master + st + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) pf[i] = a[i], pf[4 + i] = b[i];
        } else {
            to_float(pr, pf);
        }
        to_float(gr, gf);
        const int sm = (int)(ex & 255u) - kTopM, sv = (int)(ex >> 8) - kTopV;
        uint32_t top_m = 0, top_v = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            m[i] = unpack_m(mw[i / 4], i % 4, sm);
            v[i] = unpack_v(vw[i / 4], i % 4, sv);
            if (i >= n) m[i] = v[i] = 0.0f;
            moments(gf[i] * s.factor, m[i], v[i], k);
            pf[i] = stepped(pf[i], m[i], v[i], k, s, keep);
            const uint32_t bm = __float_as_uint(m[i]) & 0x7FFFFFFFu, bv = __float_as_uint(v[i]);
            top_m = bm > top_m ? bm : top_m;
            top_v = bv > top_v ? bv : top_v;
        }
        uint32_t lost = 0;                 // elements whose v is not finite
        if (__any(top_v >= kInfBits)) {
            top_m = top_v = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (__float_as_uint(v[i]) >= kInfBits) {
                    lost |= 1u << i;
                    m[i] = v[i] = 0.0f;
                }
                const uint32_t bm = __float_as_uint(m[i]) & 0x7FFFFFFFu, bv = __float_as_uint(v[i]);
                top_m = bm > top_m ? bm : top_m;
                top_v = bv > top_v ? bv : top_v;
            }
        }
        const int b_m = field_of(row_max(top_m), kTopM), b_v = field_of(row_max(top_v), kTopV);
        w2 mo = {0, 0}, vo = {0, 0};
        const uint32_t u0 = s.dither + (uint32_t)st * kDitherElement;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t um = (u0 + i * kDitherElement) >> 12, uv = um ^ 0x80000u;
            const uint32_t bm = __float_as_uint(ldexpf(fabsf(m[i]), kTopM - b_m));
            const uint32_t bv = __float_as_uint(ldexpf(v[i], kTopV - b_v));
            const uint32_t cm = ((bm + um) >> 20) | (__float_as_uint(m[i]) >> 24 & 0x80u);
            uint32_t cv = (bv + uv) >> 20;
            cv = cv == 0 && v[i] > 0.0f ? 1u : cv;
            if (lost >> i & 1) cv = 255u;
            mo[i / 4] |= cm << (8 * (i % 4));
            vo[i / 4] |= cv << (8 * (i % 4));
        }
        *(gptr<w2>)(mc + st) = mo;
        *(gptr<w2>)(vc + st) = vo;
        if (threadIdx.x % 16 == 0)
            *(gptr<uint16_t>)(exps + st / SS_MOMENT_BLOCK * 2) = (uint16_t)(b_m | b_v << 8);
        if (MASTER) {
#pragma unroll
            for (int i = 0; i < N; ++i) pf[i] = i < n ? pf[i] : 0.0f;
            *(gptr<f4>)(master + st) = f4{pf[0], pf[1], pf[2], pf[3]};
            *(gptr<f4>)(master + st + 4) = f4{pf[4], pf[5], pf[6], pf[7]};
        }
        if (MASTER) as_stored(pf);
        const Raw<P, N> pw = from_float<P, N>(pf);
        if (n >= N) store_raw<P, N>(p, at, pw);
        else store_raw_part<P, N>(p, at, pw, n);
    }
}

__global__ __launch_bounds__(kWG) void adamw_packed_kernel(const void *chunks, void *const *params,
                                                           const void *const *grads, uint8_t *m,
                                                           uint8_t *v, uint8_t *exps,
                                                           float *master,
                                                           const Scalars *__restrict__ scalars,
                                                           Betas k)
{
    const Scalars s = *scalars;
    if (!s.apply) return;
    const Chunk c = load_chunk(chunks, blockIdx.x);
    void *p = params[c.tensor];
    const void *g = grads[c.tensor];
    const float keep = c.kind & 16 ? 1.0f : s.keep;
    SS_DISPATCH_KIND(c.kind, master != nullptr,
                     step_chunk8<P, G, MASTER>(c, p, g, m, v, exps, master, k, s, keep));
}

// The values that packed moments stand for: 8 elements per lane.
__global__ __launch_bounds__(kWG) void moments_kernel(const uint8_t *__restrict__ mc,
                                                      const uint8_t *__restrict__ vc,
                                                      const uint8_t *__restrict__ exps, int64_t n,
                                                      void *m_out, void *v_out)
{
    constexpr int N = kLane8;
    const int64_t step = (int64_t)gridDim.x * kWG * N;
    for (int64_t st = ((int64_t)blockIdx.x * kWG + threadIdx.x) * N; st < n; st += step) {
        const w2 mw = *(gptr<const w2>)(mc + st), vw = *(gptr<const w2>)(vc + st);
        const uint32_t ex = *(gptr<const uint16_t>)(exps + st / SS_MOMENT_BLOCK * 2);
        const int sm = (int)(ex & 255u) - kTopM, sv = (int)(ex >> 8) - kTopV;
        float m[N], v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            m[i] = unpack_m(mw[i / 4], i % 4, sm);
            v[i] = unpack_v(vw[i / 4], i % 4, sv);
        }
        if (m_out) store_raw<SS_BF16, N>(m_out, st, from_float<SS_BF16, N>(m));
        if (v_out) store_raw<SS_BF16, N>(v_out, st, from_float<SS_BF16, N>(v));
    }
}

int32_t check_list(const char *who, const ss_tensor_list *list)
{
    if (!list) return fail(SS_ERR_INVALID_ARG, "%s: list is NULL", who);
    if (list->num_tensors < 0 || list->num_chunks < 0 || list->state_elems < 0)
        return fail(SS_ERR_INVALID_ARG, "%s: list was not planned", who);
    if (list->num_chunks > 0 && !list->chunks)
        return fail(SS_ERR_INVALID_ARG, "%s: list->chunks is NULL", who);
    if (reinterpret_cast<uintptr_t>(list->chunks) % 8 != 0)
        return fail(SS_ERR_INVALID_ARG, "%s: list->chunks is not 8-byte aligned", who);
    return SS_OK;
}

int32_t check_state(const char *who, const ss_tensor_list *list, const ss_adamw_state *state)
{
    if (!state) return fail(SS_ERR_INVALID_ARG, "%s: state is NULL", who);
    if (state->bits != 32 && state->bits != 8)
        return fail(SS_ERR_INVALID_ARG, "%s: bits = %d (need 32 or 8)", who, state->bits);
    if (list->state_elems > 0 &&
        (!state->m || !state->v || (state->bits == 8 && !state->exps)))
        return fail(SS_ERR_INVALID_ARG, "%s: state->m, v or exps is NULL", who);
    const void *const ptrs[] = {state->m, state->v, state->exps, state->master};
    const char *const names[] = {"m", "v", "exps", "master"};
    for (int i = 0; i < 4; ++i)
        if (reinterpret_cast<uintptr_t>(ptrs[i]) % 16 != 0)
            return fail(SS_ERR_INVALID_ARG, "%s: state->%s is not 16-byte aligned", who, names[i]);
    return SS_OK;
}

int norm_wgs(const ss_tensor_list *list)
{
    return list->num_chunks < kNormWgs ? list->num_chunks : kNormWgs;
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" {

int32_t ss_tensor_list_plan(const ss_tensor *tensors, int32_t n, ss_tensor_list *list,
                            void *chunks, size_t chunks_bytes)
{
    const char *who = "ss_tensor_list_plan";
    if (n < 0) return fail(SS_ERR_INVALID_ARG, "%s: n = %d", who, n);
    if (!list || (n > 0 && !tensors))
        return fail(SS_ERR_INVALID_ARG, "%s: tensors or list is NULL", who);
    int64_t num = 0, elems = 0;
    for (int32_t k = 0; k < n; ++k) {
        const ss_tensor &t = tensors[k];
        if (t.numel < 0 || t.numel > (1LL << 46))
            return fail(SS_ERR_INVALID_ARG, "%s: tensors[%d].numel = %lld", who, k,
                        (long long)t.numel);
        if (t.dtype < SS_F32 || t.dtype > SS_F16)
            return fail(SS_ERR_INVALID_ARG, "%s: tensors[%d].dtype = %d", who, k, t.dtype);
        if (t.grad_dtype != t.dtype && t.grad_dtype != SS_F32)
            return fail(SS_ERR_INVALID_ARG,
                        "%s: tensors[%d].grad_dtype = %d (need dtype or SS_F32)", who, k,
                        t.grad_dtype);
        if (t.reserved != 0 || t.no_decay < 0 || t.no_decay > 1)
            return fail(SS_ERR_INVALID_ARG, "%s: tensors[%d].no_decay or reserved", who, k);
        num += (t.numel + kChunk - 1) / kChunk;
        elems += (t.numel + SS_MOMENT_BLOCK - 1) / SS_MOMENT_BLOCK * SS_MOMENT_BLOCK;
        if (num > 0x7fffffffLL) return fail(SS_ERR_UNSUPPORTED, "%s: list too long", who);
    }
    if (chunks) {
        if (chunks_bytes < (size_t)num * sizeof(Chunk))
            return fail(SS_ERR_WORKSPACE, "%s: chunks has %zu bytes, needs %zu", who, chunks_bytes,
                        (size_t)num * sizeof(Chunk));
        Chunk *out = static_cast<Chunk *>(chunks);
        int64_t state = 0;
        for (int32_t k = 0; k < n; ++k) {
            const ss_tensor &t = tensors[k];
            for (int64_t at = 0; at < t.numel; at += kChunk) {
                const int64_t left = t.numel - at;
                *out++ = Chunk{state + at, at, k, (int32_t)(left < kChunk ? left : kChunk),
                               t.dtype | t.grad_dtype << 2 | t.no_decay << 4, 0};
            }
            state += (t.numel + SS_MOMENT_BLOCK - 1) / SS_MOMENT_BLOCK * SS_MOMENT_BLOCK;
        }
    }
    list->num_tensors = n;
    list->num_chunks = (int32_t)num;
    list->state_elems = elems;
    return SS_OK;
}

size_t ss_grad_norm_workspace_bytes(const ss_tensor_list *list)
{
    if (!list || list->num_chunks < 0) return 0;
    return align_up((size_t)(norm_wgs(list) + 1) * sizeof(double), 256);
}

int32_t ss_grad_norm(const ss_tensor_list *list, const void *const *grads, double max_norm,
                     double grad_scale, float *clip, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ss_grad_norm";
    int32_t rc = check_list(who, list);
    if (rc) return rc;
    if ((list->num_chunks > 0 && !grads) || !clip)
        return fail(SS_ERR_INVALID_ARG, "%s: grads or clip is NULL", who);
    if (reinterpret_cast<uintptr_t>(clip) % 16 != 0)
        return fail(SS_ERR_INVALID_ARG, "%s: clip is not 16-byte aligned", who);
    if (!(max_norm > 0.0)) return fail(SS_ERR_INVALID_ARG, "%s: max_norm = %g", who, max_norm);
    if (!isfinite(grad_scale))
        return fail(SS_ERR_INVALID_ARG, "%s: grad_scale = %g", who, grad_scale);
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0 ||
        ws_bytes < ss_grad_norm_workspace_bytes(list))
        return fail(SS_ERR_WORKSPACE, "%s: workspace missing, misaligned or under %zu bytes", who,
                    ss_grad_norm_workspace_bytes(list));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int wgs = norm_wgs(list);
    double *part = static_cast<double *>(ws);
    if (wgs > 0) {
        ProfScope prof("norm_partial_kernel", s);
        launch(norm_partial_kernel, dim3(wgs), dim3(kWG), s, list->chunks, list->num_chunks, grads,
               part);
    }
    ProfScope prof("norm_final_kernel", s);
    launch(norm_final_kernel, dim3(1), dim3(kFinalThreads), s, (const double *)part, wgs, max_norm,
           grad_scale, clip);
    return check_launch(who);
}

int32_t ss_adamw_step(const ss_tensor_list *list, void *const *params, const void *const *grads,
                      const ss_adamw_state *state, const ss_adamw_hyper *hyper, const float *clip,
                      void *stream)
{
    const char *who = "ss_adamw_step";
    int32_t rc = check_list(who, list);
    if (rc) return rc;
    if (list->num_chunks > 0 && (!params || !grads))
        return fail(SS_ERR_INVALID_ARG, "%s: params or grads is NULL", who);
    rc = check_state(who, list, state);
    if (rc) return rc;
    if (!state->counters || reinterpret_cast<uintptr_t>(state->counters) % 64 != 0)
        return fail(SS_ERR_INVALID_ARG, "%s: state->counters is NULL or not 64-byte aligned", who);
    if (reinterpret_cast<uintptr_t>(clip) % 16 != 0)
        return fail(SS_ERR_INVALID_ARG, "%s: clip is not 16-byte aligned", who);
    if (!hyper) return fail(SS_ERR_INVALID_ARG, "%s: hyper is NULL", who);
    const ss_adamw_hyper h = *hyper;
    if (!isfinite(h.lr) || !isfinite(h.weight_decay) || h.lr < 0.0 || h.weight_decay < 0.0)
        return fail(SS_ERR_INVALID_ARG, "%s: lr = %g, weight_decay = %g", who, h.lr,
                    h.weight_decay);
    if (!(h.beta1 >= 0.0 && h.beta1 < 1.0 && h.beta2 >= 0.0 && h.beta2 < 1.0))
        return fail(SS_ERR_INVALID_ARG, "%s: beta1 = %g, beta2 = %g (need [0, 1))", who, h.beta1,
                    h.beta2);
    if (!(h.eps >= 1e-30 && h.eps <= 1e30))
        return fail(SS_ERR_INVALID_ARG, "%s: eps = %g (need 1e-30 to 1e30)", who, h.eps);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    Scalars *scalars = static_cast<Scalars *>(state->counters);
    const Betas k{(float)h.beta1, (float)(1.0 - h.beta1), (float)h.beta2, (float)(1.0 - h.beta2),
                  (float)h.eps};
    {
        ProfScope prof("adamw_begin_kernel", s);
        launch(adamw_begin_kernel, dim3(1), dim3(64), s, scalars, clip, h.lr_device, h.lr, h.beta1,
               h.beta2, h.weight_decay);
    }
    if (list->num_chunks > 0) {
        const dim3 grid((unsigned)list->num_chunks);
        if (state->bits == 32) {
            ProfScope prof("adamw_kernel", s);
            launch(adamw_kernel, grid, dim3(kWG), s, list->chunks, params, grads,
                   static_cast<float *>(state->m), static_cast<float *>(state->v), state->master,
                   (const Scalars *)scalars, k);
        } else {
            ProfScope prof("adamw_packed_kernel", s);
            launch(adamw_packed_kernel, grid, dim3(kWG), s, list->chunks, params, grads,
                   static_cast<uint8_t *>(state->m), static_cast<uint8_t *>(state->v), state->exps,
                   state->master, (const Scalars *)scalars, k);
        }
    }
    return check_launch(who);
}

int32_t ss_adamw_moments(const ss_tensor_list *list, const ss_adamw_state *state, void *m_bf,
                         void *v_bf, void *stream)
{
    const char *who = "ss_adamw_moments";
    int32_t rc = check_list(who, list);
    if (rc) return rc;
    rc = check_state(who, list, state);
    if (rc) return rc;
    if (state->bits != 8)
        return fail(SS_ERR_INVALID_ARG, "%s: the moments are in %d bits", who, state->bits);
    if (reinterpret_cast<uintptr_t>(m_bf) % 16 != 0 || reinterpret_cast<uintptr_t>(v_bf) % 16 != 0)
        return fail(SS_ERR_INVALID_ARG, "%s: an output is not 16-byte aligned", who);
    if (list->state_elems == 0 || (!m_bf && !v_bf)) return SS_OK;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t wgs = (list->state_elems + kPass - 1) / kPass;
    ProfScope prof("moments_kernel", s);
    launch(moments_kernel, dim3((unsigned)(wgs < 1 << 20 ? wgs : 1 << 20)), dim3(kWG), s,
           static_cast<const uint8_t *>(state->m), static_cast<const uint8_t *>(state->v),
           (const uint8_t *)state->exps, list->state_elems, m_bf, v_bf);
    return check_launch(who);
}

}  // extern "C"
