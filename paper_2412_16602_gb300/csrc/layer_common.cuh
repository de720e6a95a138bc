// layer_common.cuh - device helpers of the operators over tokens: activations, vectors of channels, packed sequences.
#pragma once

#include <string.h>

#include "vmb.h"
#include "vmb_common.cuh"

namespace vmb {

// ------------------------------------------------------------ activations

// 1 / (1 + e^-z): e^-z overflows to infinity, whose reciprocal is the limit.
__device__ __forceinline__ float logistic(float z) { return rcp(1.0f + ex2(-z * kLog2e)); }

// The normal distribution's tail: Phi(-a) = e^(-a^2 / 2) m(a) for a >= 0, m(a) = t (p0 + p1 t + .. + p4 t^4) with t = 1 / (1 + 0.38 a),
// the p by linear programming for the least relative error over [0, 14]: 3.6e-5, and it keeps that where Phi is small (beyond 14
// e^(-a^2 / 2) is below the smallest float).
// For outputs in bf16.
constexpr float kTailC = 0.38f, kTail0 = 0.15122510492801666f, kTail1 = 0.15782970190048218f, kTail2 = 0.09197915345430374f,
                kTail3 = 0.18887709081172943f, kTail4 = -0.08992857486009598f, kGaussLog2 = -0.5f * kLog2e;
__device__ __forceinline__ float normal_tail(float a, float e) {
    const float t = rcp(fmaf(kTailC, a, 1.0f));
    return e * (t * fmaf(fmaf(fmaf(fmaf(kTail4, t, kTail3), t, kTail2), t, kTail1), t, kTail0));
}

template <int ACT> __device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == VMB_ACT_SILU) return z * logistic(z);
    // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
    if constexpr (ACT == VMB_ACT_GELU) return fmaf(-fabsf(z), normal_tail(fabsf(z), ex2(kGaussLog2 * z * z)), fmaxf(z, 0.0f));
    return z;
}
template <int ACT> __device__ __forceinline__ float activate_slope(float z) {
    if constexpr (ACT == VMB_ACT_SILU) {
        const float s = logistic(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    // Phi(z) + z phi(z): its terms cancel for z < 0, and sums of it are kept in fp32
    if constexpr (ACT == VMB_ACT_GELU) return fmaf(z * 0.39894228040143268f, ex2(kGaussLog2 * z * z), 0.5f * erfcf(-0.70710678118654752f * z));
    return 1.0f;
}
// Two values at once, in packed arithmetic.
template <int ACT> __device__ __forceinline__ float2 activate2(float2 z) {
    const auto all = [](float v) { return make_float2(v, v); };
    if constexpr (ACT == VMB_ACT_SILU) {
        const float2 q = __fmul2_rn(z, all(-kLog2e)), d = __fadd2_rn(make_float2(ex2(q.x), ex2(q.y)), all(1.0f));
        return __fmul2_rn(z, make_float2(rcp(d.x), rcp(d.y)));
    }
    if constexpr (ACT == VMB_ACT_GELU) {
        const float2 a = make_float2(fabsf(z.x), fabsf(z.y)), d = __ffma2_rn(a, all(kTailC), all(1.0f)), t = make_float2(rcp(d.x), rcp(d.y));
        const float2 q = __fmul2_rn(__fmul2_rn(z, all(kGaussLog2)), z);
        float2 p = __ffma2_rn(t, all(kTail4), all(kTail3));
        p = __ffma2_rn(p, t, all(kTail2));
        p = __ffma2_rn(p, t, all(kTail1));
        p = __ffma2_rn(p, t, all(kTail0));
        p = __fmul2_rn(__fmul2_rn(p, t), make_float2(ex2(q.x), ex2(q.y)));
        return __ffma2_rn(__fmul2_rn(p, all(-1.0f)), a, make_float2(fmaxf(z.x, 0.0f), fmaxf(z.y, 0.0f)));
    }
    return z;
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
