// layer_common.cuh - device helpers of the operators over tokens: activations, vectors of channels, packed sequences.
#pragma once

#include <string.h>

#include "vmb.h"
#include "vmb_common.cuh"

namespace vmb {

// ------------------------------------------------------------ activations

// 1 / (1 + e^-z): e^-z overflows to infinity, whose reciprocal is the limit.
__device__ __forceinline__ float logistic(float z) { return rcp(1.0f + ex2(-z * kLog2e)); }

template <int ACT> __device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == VMB_ACT_SILU) return z * logistic(z);
    // z Phi(z) through the complement, which keeps its digits where Phi is small
    if constexpr (ACT == VMB_ACT_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);
    return z;
}
template <int ACT> __device__ __forceinline__ float activate_slope(float z) {
    if constexpr (ACT == VMB_ACT_SILU) {
        const float s = logistic(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    if constexpr (ACT == VMB_ACT_GELU)
        return fmaf(z * 0.39894228040143268f, ex2(-0.5f * kLog2e * z * z), 0.5f * erfcf(-0.70710678118654752f * z));
    return 1.0f;
}

// ------------------------------------------------------------ vectors of channels

template <typename T, int V> struct alignas(sizeof(T) * V) Vec { T v[V]; };

template <typename T, int V> __device__ __forceinline__ void load_vec(float (&out)[V], const T* p) {
    const Vec<T, V> a = *reinterpret_cast<const Vec<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = io<T>::cvt(a.v[i]);
}
template <typename T, int V> __device__ __forceinline__ void store_vec(T* p, const float (&in)[V]) {
    Vec<T, V> a;
#pragma unroll
    for (int i = 0; i < V; ++i) a.v[i] = io<T>::to(in[i]);
    *reinterpret_cast<Vec<T, V>*>(p) = a;
}

// ------------------------------------------------------------ packed sequences

// The largest b in [0, n] with place(b) <= t, or -1, for a non-decreasing place; by one warp, 32 places a round.  A place that
// decreases gives some b of that range.
template <typename F> __device__ __forceinline__ int last_at_most(int n, long long t, F place) {
    int lo = -1, hi = n + 1;
    const int lane = threadIdx.x & 31;
    while (hi - lo > 1) {
        const int step = (hi - lo - 1 + 31) / 32, at = lo + 1 + lane * step;
        const unsigned found = __ballot_sync(0xffffffffu, at < hi && place(at) <= t);
        const int c = __popc(found);
        const int nlo = c ? lo + 1 + (c - 1) * step : lo, nhi = lo + 1 + c * step;
        if (nhi < hi && c < 32) hi = nhi;
        lo = nlo;
    }
    return lo;
}

// offsets[b] and offsets[b + 1] cut to [0, total], the end not before the start; *bad is set when that changed them.
__device__ __forceinline__ void sequence_span(const int* offsets, int b, long long total, long long* start, long long* end, bool* bad) {
    const long long s = offsets[b], e = offsets[b + 1];
    const long long s1 = s < 0 ? 0 : s > total ? total : s, e1 = e < s1 ? s1 : e > total ? total : e;
    *bad = s1 != s || e1 != e;
    *start = s1, *end = e1;
}

}  // namespace vmb
