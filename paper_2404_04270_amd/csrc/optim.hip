// The optimizer of the parameters that are no tables: AdamW over the tensors of a list in one
// launch, with moments in 32 or in 8 bits, and the norm of all their gradients.
//
// All of it is bound by HBM.  A step in fp32 reads p, g, m and v and writes p, m and v, 28 bytes per
// element; with 8-bit moments and 16-bit parameters it is 10.  The work table cuts the tensors into
// chunks, a workgroup takes a chunk, and every access of a lane is as wide as its elements allow
// (8 or 16 bytes).  A chunk names its tensor, so that tensors of all sizes and types share a launch.
//
// us, and TB/s of what a step cannot do without (a device-wide addition of a constant reaches 6.2):
// 2^28 fp32 elements 1300 to 1360 (5.5 to 5.8), 2^28 bf16 with master copies 1280 to 1350 (5.6 to
// 5.9); packed moments: 2^28 bf16 505 (5.3), 2^28 fp32 747 (5.8).  A bf16 step with packed moments
// is at the end of what its arithmetic allows, too: about 60 instructions per element.
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

// Elements that a workgroup takes: one round trip to memory with all of its loads in flight.  With
// 4096 elements in two rounds a step over 2^28 fp32 elements takes 1394 instead of 1341 us, in one
// round of twice the loads 1334 instead of 1296.
constexpr int kChunk = 2048;
constexpr int64_t kMostChunks = 0xFFFFFFFFLL / kWG;    // threads of a launch are counted in 32 bits
// Workgroups run on the eight XCDs in turn.  Eight chunks next to each other go to the same XCD,
// which then works on pieces of 64 KB: 1296 instead of 1341 us.
constexpr int kRun = 8;

__device__ __forceinline__ int64_t chunk_of_block()
{
    const unsigned b = blockIdx.x, group = b / (8 * kRun), w = b % (8 * kRun);
    if ((group + 1) * (8 * kRun) > gridDim.x) return b;
    return group * (8 * kRun) + w % 8 * kRun + w / 8;
}

__device__ __forceinline__ Chunk load_chunk(const void *chunks, int64_t c)
{
    return static_cast<const Chunk *>(chunks)[c];
}

// ---- gradient norm ------------------------------------------------------------------------
// Four workgroups per compute unit, and past the caches: 2^29 bf16 elements 170 us, 2^28 fp32 161 (6.3
// and 6.7 TB/s); with twice as many 196 to 229, with half as many 174 and 180, through the caches 177
// and 177.
constexpr int kNormWgs = 1024;
constexpr int kFinalThreads = 1024;
// Up to so many chunks go to one workgroup and one launch: 7.2 instead of 10.1 us from call to call
// with 1 to 48 chunks, 8.6 and 10.2 with 64 of fp32.
constexpr int kAloneChunks = 64;

template <int G, int N>
__device__ __forceinline__ void add_squares(const Raw<G, N> &r, double &sum)
{
    float f[N];
    to_float(r, f);
#pragma unroll
    for (int k = 0; k < N; ++k) sum = fma((double)f[k], (double)f[k], sum);
}

// Sum of the squares of a wavefront's chunk, a lane's part.
template <int G>
__device__ __forceinline__ double chunk_squares(const void *g, const Chunk &c)
{
    constexpr int N = G == SS_F32 ? 4 : 8, U = kChunk / (64 * N);
    const int lane = threadIdx.x % 64;
    double sum = 0.0;
    if (c.count == kChunk) {
        Raw<G, N> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = load_raw<G, N, true>(g, c.first + (u * 64 + lane) * N);
#pragma unroll
        for (int u = 0; u < U; ++u) add_squares(r[u], sum);
        return sum;
    }
    for (int e = lane * N; e < c.count; e += 64 * N) {
        if (e + N <= c.count) add_squares(load_raw<G, N>(g, c.first + e), sum);
        else add_squares(load_raw_part<G, N>(g, c.first + e, c.count - e), sum);
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

// A wavefront takes a chunk at a time; the entry of its next one is fetched meanwhile.
template <int THREADS>
__device__ __forceinline__ double chunks_squares(const void *chunks, int num_chunks,
                                                 const void *const *grads)
{
    constexpr int kWaves = THREADS / 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t step = (int64_t)gridDim.x * kWaves;
    int64_t i = (int64_t)blockIdx.x * kWaves + wave;
    double sum = 0.0;
    Chunk next{};
    const void *g_next = nullptr;
    if (i < num_chunks) {
        next = load_chunk(chunks, i);
        g_next = grads[next.tensor];
    }
    for (; i < num_chunks; i += step) {
        const Chunk c = next;
        const void *g = g_next;
        if (i + step < num_chunks) {
            next = load_chunk(chunks, i + step);
            g_next = grads[next.tensor];
        }
        switch (c.kind >> 2 & 3) {
        case SS_F32: sum += chunk_squares<SS_F32>(g, c); break;
        case SS_BF16: sum += chunk_squares<SS_BF16>(g, c); break;
        default: sum += chunk_squares<SS_F16>(g, c); break;
        }
    }
    return wg_sum<THREADS>(sum);
}

__device__ __forceinline__ void write_clip(double sum, double max_norm, double grad_scale,
                                           float *__restrict__ clip)
{
    const double norm = fabs(grad_scale) * sqrt(sum);
    const bool finite = norm < INFINITY;
    const double ratio = max_norm / (norm + 1e-6);
    clip[0] = (float)norm;
    clip[1] = finite ? (float)(grad_scale * (ratio < 1.0 ? ratio : 1.0)) : 0.0f;
    clip[2] = finite ? 1.0f : 0.0f;
    clip[3] = 0.0f;
}

__global__ __launch_bounds__(kWG) void norm_partial_kernel(const void *chunks, int num_chunks,
                                                           const void *const *grads,
                                                           double *__restrict__ part)
{
    const double sum = chunks_squares<kWG>(chunks, num_chunks, grads);
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
    if (threadIdx.x == 0) write_clip(sum, max_norm, grad_scale, clip);
}

__global__ __launch_bounds__(kFinalThreads) void norm_alone_kernel(const void *chunks,
                                                                   int num_chunks,
                                                                   const void *const *grads,
                                                                   double max_norm,
                                                                   double grad_scale,
                                                                   float *__restrict__ clip)
{
    const double sum = chunks_squares<kFinalThreads>(chunks, num_chunks, grads);
    if (threadIdx.x == 0) write_clip(sum, max_norm, grad_scale, clip);
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
    uint32_t lines_ended;      // lines below whose workgroups have all ended
    int32_t reserved[5];
};
// A cache line for every kEndLines-th workgroup of a step that tells its own end (below).
constexpr int kEndLines = 32;
struct Counters {
    Scalars scalars;
    struct {
        uint32_t ended, reserved[15];
    } line[kEndLines];
};
static_assert(sizeof(Counters) == SS_ADAMW_COUNTER_BYTES, "the header says how large they are");

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

struct Begin {
    double lr, log1, log2, weight_decay;       // log1, log2: of the betas
    const float *lr_device, *clip;
};

// The scalars of the step that follows what *old counts.
__device__ __forceinline__ Scalars begin_step(const Scalars *__restrict__ old, const Begin &b)
{
    Scalars s;
    const double lr = b.lr_device ? (double)*b.lr_device : b.lr;
    s.apply = !b.clip || b.clip[2] != 0.0f;
    s.factor = b.clip ? b.clip[1] : 1.0f;
    s.steps = old->steps + s.apply;
    s.left_out = old->left_out + !s.apply;
    // 1 - beta^t without the cancellation of a beta next to 1; a beta of 0 (log -inf) gives 1
    s.size = (float)(lr / -expm1((double)s.steps * b.log1));
    s.keep = (float)(1.0 - lr * b.weight_decay);
    s.root = (float)(1.0 / sqrt(-expm1((double)s.steps * b.log2)));
    s.dither = mixed((uint32_t)s.steps);
    return s;
}

__global__ __launch_bounds__(64) void adamw_begin_kernel(Scalars *scalars, Begin b)
{
    if (threadIdx.x != 0) return;
    Scalars s = begin_step(scalars, b);
    s.lines_ended = 0;
    *scalars = s;
}

// A step of few workgroups has one launch: each works out the scalars for itself, and the last to end
// counts the step (nobody waits: all have read the count by then).  A workgroup's turn at a counter
// takes about 16 ns, so they count themselves on kEndLines counters first, and the last of each there
// on one.  us per fp32 step of 60 / 260 / 380 / 500 / 1000 / 2000 chunks in one launch and in two 5.6 /
// 5.5 / 6.4 / 7.8 / 11.1 / 19.2 and 9.0 / 8.0 / 7.9 / 8.6 / 11.9 / 20.1 (on a single counter 5.2 / 6.9 /
// 9.0 / 11.5 / 19.5 / 32.1); packed moments 5.3 / 5.6 / - / 6.1 / 8.0 / 12.7 and 7.5 / 7.9 / - / 7.9 /
// 8.7 / 12.3.
constexpr int kSoloChunks = 1024;

__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform(float x) { return __int_as_float(uniform(__float_as_int(x))); }

// The scalars of a solo step, from the first wavefront (it is the arithmetic in fp64 that takes time).
__device__ __forceinline__ Scalars begin_solo(const Scalars *scalars, const Begin &b)
{
    __shared__ Scalars shared;
    if (threadIdx.x < 64) {
        const Scalars s = begin_step(scalars, b);
        if (threadIdx.x == 0) shared = s;
    }
    __syncthreads();
    Scalars s = shared;
    s.size = uniform(s.size);
    s.keep = uniform(s.keep);
    s.root = uniform(s.root);
    s.factor = uniform(s.factor);
    s.dither = (uint32_t)uniform((int32_t)s.dither);
    s.apply = uniform(s.apply);
    return s;
}

__device__ __forceinline__ bool last_of(uint32_t *counter, uint32_t n)
{
    const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED,
                                                   __HIP_MEMORY_SCOPE_AGENT);
    if (before + 1 != n) return false;
    *counter = 0;              // for the next step
    return true;
}

__device__ __forceinline__ void end_solo(Counters *c, const Scalars &s)
{
    __syncthreads();           // every wavefront has used the count it read
    if (threadIdx.x != 0) return;
    const uint32_t line = blockIdx.x % kEndLines, n = gridDim.x;
    if (!last_of(&c->line[line].ended, (n - line - 1) / kEndLines + 1)) return;
    if (!last_of(&c->scalars.lines_ended, n < kEndLines ? n : kEndLines)) return;
    c->scalars.steps = s.steps;
    c->scalars.left_out = s.left_out;
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

// Four elements of a chunk on their way: what a lane has asked for.
template <int P, int G, bool MASTER> struct Four {
    Raw<P, 4> p;
    Raw<G, 4> g;
    f4 m, v, w;                // w: the master copy
};

// How a chunk is read and written: through the caches, past them, or past them but for parameters
// and gradients (whose narrow accesses share cache lines where a tensor starts at an odd place).
enum Flow { kCached, kStream, kStreamMoments };

template <Flow F> __device__ __forceinline__ f4 load_moments(const float *p)
{
    if constexpr (F != kCached) return __builtin_nontemporal_load((gptr<const f4>)p);
    return *(gptr<const f4>)p;
}
template <Flow F> __device__ __forceinline__ void store_moments(float *p, f4 v)
{
    if constexpr (F != kCached) __builtin_nontemporal_store(v, (gptr<f4>)p);
    else *(gptr<f4>)p = v;
}

// Tensors and moments of a chunk; element e of it is p[first + e] and m[state + e].
struct Places {
    void *p;
    const void *g;
    float *m, *v, *master;
    int64_t first, state;
};

template <Flow F, int P, int G, bool MASTER, bool WHOLE>
__device__ __forceinline__ void ask_four(const Places &at, int e, int n, Four<P, G, MASTER> &q)
{
    if (WHOLE) {
        if (!MASTER) q.p = load_raw<P, 4, F == kStream>(at.p, at.first + e);
        q.g = load_raw<G, 4, F == kStream>(at.g, at.first + e);
    } else {
        if (!MASTER) q.p = load_raw_part<P, 4>(at.p, at.first + e, n);
        q.g = load_raw_part<G, 4>(at.g, at.first + e, n);
    }
    q.m = load_moments<F>(at.m + at.state + e);
    q.v = load_moments<F>(at.v + at.state + e);
    if (MASTER) q.w = load_moments<F>(at.master + at.state + e);
}

template <Flow F, int P, int G, bool MASTER, bool WHOLE>
__device__ __forceinline__ void step_four(const Places &at, int e, int n,
                                          const Four<P, G, MASTER> &q, const Betas &k,
                                          const Scalars &s, float keep)
{
    float p[4], g[4], m[4], v[4];
    if (!MASTER) to_float(q.p, p);
    to_float(q.g, g);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (MASTER) p[i] = q.w[i];
        m[i] = q.m[i];
        v[i] = q.v[i];
        if (!WHOLE && i >= n) g[i] = m[i] = v[i] = p[i] = 0.0f;      // padding becomes 0
        moments(g[i] * s.factor, m[i], v[i], k);
        p[i] = stepped(p[i], m[i], v[i], k, s, keep);
    }
    if (MASTER) as_stored(p);
    store_moments<F>(at.m + at.state + e, f4{m[0], m[1], m[2], m[3]});
    store_moments<F>(at.v + at.state + e, f4{v[0], v[1], v[2], v[3]});
    if (MASTER) store_moments<F>(at.master + at.state + e, f4{p[0], p[1], p[2], p[3]});
    const Raw<P, 4> out = from_float<P, 4>(p);
    if (WHOLE) store_raw<P, 4, F == kStream>(at.p, at.first + e, out);
    else store_raw_part<P, 4>(at.p, at.first + e, out, n);
}

template <Flow F, int P, int G, bool MASTER>
__device__ __forceinline__ void step_chunk(const Places &at, int count, const Betas &k,
                                           const Scalars &s, float keep)
{
    constexpr int U = kChunk / (kWG * 4), kStep = kWG * 4;
    int e = threadIdx.x * 4;
    if (count == kChunk) {
        Four<P, G, MASTER> q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) ask_four<F, P, G, MASTER, true>(at, e + u * kStep, 4, q[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            step_four<F, P, G, MASTER, true>(at, e + u * kStep, 4, q[u], k, s, keep);
        return;
    }
    for (; e < count; e += kStep) {
        Four<P, G, MASTER> q;
        if (e + 4 <= count) {
            ask_four<F, P, G, MASTER, true>(at, e, 4, q);
            step_four<F, P, G, MASTER, true>(at, e, 4, q, k, s, keep);
        } else {
            ask_four<F, P, G, MASTER, false>(at, e, count - e, q);
            step_four<F, P, G, MASTER, false>(at, e, count - e, q, k, s, keep);
        }
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

// From this many elements on a step goes past the caches: parameters, gradients and moments have
// been replaced there before the next step reads them.  us per step over 2 / 4 / 8 / 16 / 32 M fp32
// elements, streamed and not, three models in turn: 13.3 / 22.4 / 40.3 / 75.7 / 147 and 12.0 / 20.0 /
// 45.4 / 86.5 / 167; one model with nothing else between its steps: 12.0 / 20.8 / 39.4 / 75.5 / 146
// and 10.0 / 19.9 / 35.5 / 69.8 / 170.
constexpr int64_t kStreamElems = 8 << 20;

template <bool STREAM, bool SOLO>
__global__ __launch_bounds__(kWG) void adamw_kernel(const void *chunks, void *const *params,
                                                    const void *const *grads, float *m, float *v,
                                                    float *master, Counters *counters, Betas k,
                                                    Begin b)
{
    const Chunk c = load_chunk(chunks, chunk_of_block());
    const Scalars s = SOLO ? begin_solo(&counters->scalars, b) : counters->scalars;
    const Places at{params[c.tensor], grads[c.tensor], m, v, master, c.first, c.state};
    const float keep = c.kind & 16 ? 1.0f : s.keep;
    if (!s.apply) {
        if (SOLO) end_solo(counters, s);
        return;
    }
    // 16 bits at odd places: 20 M bf16 elements with master copies 92 instead of 103 us; fp32 does not
    // mind them (2^28 elements at odd places 1333 past the caches, 1338 to 1354 otherwise)
    const bool even = ((reinterpret_cast<uintptr_t>(at.p) | reinterpret_cast<uintptr_t>(at.g)) &
                       15) == 0 || (c.kind & 15) == (SS_F32 | SS_F32 << 2);
    if (!STREAM) {
        SS_DISPATCH_KIND(c.kind, master != nullptr,
                         step_chunk<kCached, P, G, MASTER>(at, c.count, k, s, keep));
    } else if (even) {
        SS_DISPATCH_KIND(c.kind, master != nullptr,
                         step_chunk<kStream, P, G, MASTER>(at, c.count, k, s, keep));
    } else {
        SS_DISPATCH_KIND(c.kind, master != nullptr,
                         step_chunk<kStreamMoments, P, G, MASTER>(at, c.count, k, s, keep));
    }
    if (SOLO) end_solo(counters, s);
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

// stepped() with the hardware's root and reciprocal, each within a step of fp32 of its value: a
// packed step has so little to read that the exact ones show (2^28 bf16 elements 568 instead of 493
// us).  The root takes v below 2^-126 for 0: against eps >= 1e-12 that is nothing, smaller ones go the
// exact way.
constexpr double kLeastFastEps = 1e-12;

__device__ __forceinline__ float stepped_fast(float p, float m, float v, const Betas &k,
                                              const Scalars &s, float keep)
{
    const float den = __builtin_amdgcn_sqrtf(v) * s.root + k.eps;
    return p * keep - s.size * (m * __builtin_amdgcn_rcpf(den));
}

// Packed moments and master copies go past the caches in lists of any size: 16 M fp32 elements 47 us
// a step, 51 through the caches, 4 M bf16 elements 12.3 and 12.6, 2^28 fp32 747 and 772.
template <typename T> __device__ __forceinline__ T past_caches(const void *p)
{
    return __builtin_nontemporal_load((gptr<const T>)p);
}

template <bool EXACT, int P, int G, bool MASTER>
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
        const w2 mw = past_caches<w2>(mc + st), vw = past_caches<w2>(vc + st);
        const uint32_t ex = *(gptr<const uint16_t>)(exps + st / SS_MOMENT_BLOCK * 2);
        float pf[N], gf[N], m[N], v[N];
        if (MASTER) {
            const f4 a = past_caches<f4>(master + st), b = past_caches<f4>(master + st + 4);
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
            const uint32_t bm = __float_as_uint(m[i]) & 0x7FFFFFFFu, bv = __float_as_uint(v[i]);
            top_m = bm > top_m ? bm : top_m;
            top_v = bv > top_v ? bv : top_v;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            pf[i] = EXACT ? stepped(pf[i], m[i], v[i], k, s, keep)
                          : stepped_fast(pf[i], m[i], v[i], k, s, keep);
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
        __builtin_nontemporal_store(mo, (gptr<w2>)(mc + st));
        __builtin_nontemporal_store(vo, (gptr<w2>)(vc + st));
        if (threadIdx.x % 16 == 0)
            *(gptr<uint16_t>)(exps + st / SS_MOMENT_BLOCK * 2) = (uint16_t)(b_m | b_v << 8);
        if (MASTER) {
#pragma unroll
            for (int i = 0; i < N; ++i) pf[i] = i < n ? pf[i] : 0.0f;
            __builtin_nontemporal_store(f4{pf[0], pf[1], pf[2], pf[3]}, (gptr<f4>)(master + st));
            __builtin_nontemporal_store(f4{pf[4], pf[5], pf[6], pf[7]}, (gptr<f4>)(master + st + 4));
        }
        if (MASTER) as_stored(pf);
        const Raw<P, N> pw = from_float<P, N>(pf);
        if (n >= N) store_raw<P, N>(p, at, pw);
        else store_raw_part<P, N>(p, at, pw, n);
    }
}

template <bool SOLO, bool EXACT>
__global__ __launch_bounds__(kWG) void adamw_packed_kernel(const void *chunks, void *const *params,
                                                           const void *const *grads, uint8_t *m,
                                                           uint8_t *v, uint8_t *exps,
                                                           float *master, Counters *counters,
                                                           Betas k, Begin b)
{
    const Chunk c = load_chunk(chunks, chunk_of_block());
    const Scalars s = SOLO ? begin_solo(&counters->scalars, b) : counters->scalars;
    void *p = params[c.tensor];
    const void *g = grads[c.tensor];
    const float keep = c.kind & 16 ? 1.0f : s.keep;
    if (s.apply) {
        SS_DISPATCH_KIND(c.kind, master != nullptr,
                         step_chunk8<EXACT, P, G, MASTER>(c, p, g, m, v, exps, master, k, s, keep));
    }
    if (SOLO) end_solo(counters, s);
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
    if (list->num_tensors < 0 || list->num_chunks < 0 || list->num_chunks > kMostChunks ||
        list->state_elems < 0)
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
    const int64_t wgs = ((int64_t)list->num_chunks + kWG / 64 - 1) / (kWG / 64);
    return (int)(wgs < kNormWgs ? wgs : kNormWgs);
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
        if (num > kMostChunks) return fail(SS_ERR_UNSUPPORTED, "%s: list too long", who);
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
    if (list->num_chunks <= kAloneChunks) {
        ProfScope prof("norm_alone_kernel", s);
        launch(norm_alone_kernel, dim3(1), dim3(kFinalThreads), s, list->chunks, list->num_chunks,
               grads, max_norm, grad_scale, clip);
        return check_launch(who);
    }
    const int wgs = norm_wgs(list);
    double *part = static_cast<double *>(ws);
    {
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
                      const ss_adamw_state *state, double lr, const float *lr_device, double beta1,
                      double beta2, double eps, double weight_decay, const float *clip,
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
    if (!isfinite(lr) || !isfinite(weight_decay) || lr < 0.0 || weight_decay < 0.0)
        return fail(SS_ERR_INVALID_ARG, "%s: lr = %g, weight_decay = %g", who, lr, weight_decay);
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0))
        return fail(SS_ERR_INVALID_ARG, "%s: beta1 = %g, beta2 = %g (need [0, 1))", who, beta1,
                    beta2);
    if (!(eps >= 1e-30 && eps <= 1e30))
        return fail(SS_ERR_INVALID_ARG, "%s: eps = %g (need 1e-30 to 1e30)", who, eps);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    Counters *counters = static_cast<Counters *>(state->counters);
    const Betas k{(float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2),
                  (float)eps};
    const Begin b{lr, log(beta1), log(beta2), weight_decay, lr_device, clip};
    const dim3 grid((unsigned)list->num_chunks);
    const bool solo = list->num_chunks > 0 && list->num_chunks <= kSoloChunks;
    if (!solo) {
        ProfScope prof("adamw_begin_kernel", s);
        launch(adamw_begin_kernel, dim3(1), dim3(64), s, &counters->scalars, b);
    }
    if (list->num_chunks > 0 && state->bits == 32) {
        ProfScope prof("adamw_kernel", s);
        launch(solo ? adamw_kernel<false, true>
                    : list->state_elems >= kStreamElems ? adamw_kernel<true, false>
                                                        : adamw_kernel<false, false>,
               grid, dim3(kWG), s, list->chunks, params, grads, static_cast<float *>(state->m),
               static_cast<float *>(state->v), state->master, counters, k, b);
    } else if (list->num_chunks > 0) {
        ProfScope prof("adamw_packed_kernel", s);
        const bool exact = eps < kLeastFastEps;
        launch(exact ? solo ? adamw_packed_kernel<true, true> : adamw_packed_kernel<false, true>
               : solo ? adamw_packed_kernel<true, false> : adamw_packed_kernel<false, false>,
               grid, dim3(kWG), s, list->chunks, params, grads,
               static_cast<uint8_t *>(state->m), static_cast<uint8_t *>(state->v), state->exps,
               state->master, counters, k, b);
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
    const int64_t wgs = (list->state_elems + kWG * kLane8 - 1) / (kWG * kLane8);
    ProfScope prof("moments_kernel", s);
    launch(moments_kernel, dim3((unsigned)(wgs < 1 << 20 ? wgs : 1 << 20)), dim3(kWG), s,
           static_cast<const uint8_t *>(state->m), static_cast<const uint8_t *>(state->v),
           (const uint8_t *)state->exps, list->state_elems, m_bf, v_bf);
    return check_launch(who);
}

}  // extern "C"
