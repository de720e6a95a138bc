// layer_common.cuh - device helpers of the operators over tokens: activations, vectors of channels, packed sequences.
#pragma once

#include <string.h>

#include "vmb.h"
#include "vmb_common.cuh"

namespace vmb {

// ------------------------------------------------------------ activations

// 1 / (1 + e^-z): e^-z overflows to infinity, whose reciprocal is the limit.
__device__ __forceinline__ float logistic(float z) { return rcp(1.0f + ex2(-z * kLog2e)); }

// The normal distribution's tail as a power of two: log2 Phi(b) for b in [-13.2, 0] is a polynomial of degree eight in b, by linear programming
// for the least error, 1.8e-4 of its power (with the coefficients and sums in fp32 1.5e-4): Phi keeps 12 bits also where it is small.  Below
// -13.2 it is less than the smallest float.  For outputs in bf16; one exponential, where a quotient of polynomials takes a reciprocal too.
constexpr float kTailEnd = -13.2f, kTail0 = -1.0001838207244873f, kTail1 = 1.1490356922149658f, kTail2 = -0.4627901613712311f, kTail3 = 0.05079496651887894f,
                kTail4 = 0.00741631118580699f, kTail5 = 0.0007434896542690694f, kTail6 = 4.7549950977554545e-05f, kTail7 = 1.7312547697656555e-06f, kTail8 = 2.716298652671867e-08f;
__device__ __forceinline__ float relu(float z) {  // NaN stays
    float y;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(z));
    return y;
}

template <int ACT> __device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == VMB_ACT_SILU) return z * logistic(z);
    // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
    if constexpr (ACT == VMB_ACT_GELU) {
        const float b = fmaxf(-fabsf(z), kTailEnd);
        float p = fmaf(kTail8, b, kTail7);
        p = fmaf(fmaf(fmaf(fmaf(p, b, kTail6), b, kTail5), b, kTail4), b, kTail3);
        return fmaf(ex2(fmaf(fmaf(fmaf(p, b, kTail2), b, kTail1), b, kTail0)), b, relu(z));
    }
    return z;
}
template <int ACT> __device__ __forceinline__ float activate_slope(float z) {
    if constexpr (ACT == VMB_ACT_SILU) {
        const float s = logistic(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    // Phi(z) + z phi(z): its terms cancel for z < 0, and sums of it are kept in fp32
    if constexpr (ACT == VMB_ACT_GELU) return fmaf(z * 0.39894228040143268f, ex2(-0.5f * kLog2e * z * z), 0.5f * erfcf(-0.70710678118654752f * z));
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
        const float2 b = make_float2(fmaxf(-fabsf(z.x), kTailEnd), fmaxf(-fabsf(z.y), kTailEnd));
        float2 p = __ffma2_rn(b, all(kTail8), all(kTail7));
        p = __ffma2_rn(p, b, all(kTail6));
        p = __ffma2_rn(p, b, all(kTail5));
        p = __ffma2_rn(p, b, all(kTail4));
        p = __ffma2_rn(p, b, all(kTail3));
        p = __ffma2_rn(p, b, all(kTail2));
        p = __ffma2_rn(p, b, all(kTail1));
        p = __ffma2_rn(p, b, all(kTail0));
        return __ffma2_rn(make_float2(ex2(p.x), ex2(p.y)), b, make_float2(relu(z.x), relu(z.y)));
    }
    return z;
}

// ------------------------------------------------------------ vectors of channels

// (no more than 16 bytes: what the checks of pointers ask for, though the device has loads of 32 bytes that need more)
template <typename T, int V> struct alignas(sizeof(T) * V < 16 ? sizeof(T) * V : 16) Vec { T v[V]; };

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

// offsets[b] and offsets[b + 1] cut to [0, total], the end not before the start.
__device__ __forceinline__ void sequence_span(const int* offsets, int b, long long total, long long* start, long long* end) {
    const long long s = offsets[b], e = offsets[b + 1];
    *start = s < 0 ? 0 : s > total ? total : s;
    *end = e < *start ? *start : e > total ? total : e;
}

}  // namespace vmb
