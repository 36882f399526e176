// Elements of 32 and 16 bits in vectors, at any alignment their type allows: a tensor of a flat
// buffer starts where the one before it ends, and rows of odd length begin at odd places.  The
// hardware takes a 16-byte access at any address, so there is one path for all of them.
#pragma once
#include "ss_common.h"

namespace ss {

template <int DT> struct ElemOf;
template <> struct ElemOf<SS_F32> { typedef float type; };
template <> struct ElemOf<SS_BF16> { typedef __bf16 type; };
template <> struct ElemOf<SS_F16> { typedef _Float16 type; };

// N consecutive elements as they lie in memory, aligned to the element only.
template <int DT, int N> struct Raw {
    typedef typename ElemOf<DT>::type E;
    typedef E V __attribute__((ext_vector_type(N)));
    typedef V VU __attribute__((aligned(sizeof(E))));
    V v;
};

// STREAM: past the caches, for data that nobody reads again before they have been replaced.
template <int DT, int N, bool STREAM = false>
__device__ __forceinline__ Raw<DT, N> load_raw(const void *base, int64_t i)
{
    typedef Raw<DT, N> R;
    R r;
    const auto p = (gptr<const typename R::VU>)((gptr<const typename R::E>)base + i);
    if constexpr (STREAM) r.v = __builtin_nontemporal_load(p);
    else r.v = *p;
    return r;
}

// The first n of them; zeros behind.
template <int DT, int N>
__device__ __forceinline__ Raw<DT, N> load_raw_part(const void *base, int64_t i, int n)
{
    typedef Raw<DT, N> R;
    R r;
    const auto p = (gptr<const typename R::E>)base + i;
#pragma unroll
    for (int k = 0; k < N; ++k) r.v[k] = k < n ? p[k] : (typename R::E)0.0f;
    return r;
}

template <int DT, int N>
__device__ __forceinline__ void to_float(const Raw<DT, N> &r, float (&f)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = (float)r.v[k];
}

// Rounded to the nearest, ties to even.
template <int DT, int N>
__device__ __forceinline__ Raw<DT, N> from_float(const float (&f)[N])
{
    Raw<DT, N> r;
#pragma unroll
    for (int k = 0; k < N; ++k) r.v[k] = (typename Raw<DT, N>::E)f[k];
    return r;
}

template <int DT, int N, bool STREAM = false>
__device__ __forceinline__ void store_raw(void *base, int64_t i, const Raw<DT, N> &r)
{
    typedef Raw<DT, N> R;
    const auto p = (gptr<typename R::VU>)((gptr<typename R::E>)base + i);
    if constexpr (STREAM) __builtin_nontemporal_store(r.v, p);
    else *p = r.v;
}

template <int DT, int N>
__device__ __forceinline__ void store_raw_part(void *base, int64_t i, const Raw<DT, N> &r, int n)
{
    typedef Raw<DT, N> R;
    const auto p = (gptr<typename R::E>)base + i;
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (k < n) p[k] = r.v[k];
}

}  // namespace ss
