// group_norm.cu - group norm with an activation, channels last: forward and gradients.
//
//   n = (x - mean) / sqrt(var + eps) over the pixels and the C / G channels of a group, y = act(w n + b).
//   dz = dy act'(w n + b);  dweight = sum dz n, dbias = sum dz (over batch and pixels);
//   dx = rstd (w dz - mean(w dz) - n mean(w dz n)), the means over the group.
//
// What bounds both is memory: x (and dy) read, y (dx) written, once each where the pixels of a few groups fit the
// shared memory of a cluster of CTAs: every CTA holds a run of pixels, the cluster exchanges its sums through
// distributed shared memory, and the results are formed from the tile (norm_cluster_kernel, norm_cluster_grad_kernel).
// Larger samples take two passes over the same tiles (a run of pixels of one sample, all channels): the first leaves a
// tile's sums per channel, and the last tile of a sample to finish joins them; the second applies them.  It finds x in
// the L2 cache, because a launch covers only as many samples as its share of the cache holds.
// With one to three CTAs on an SM the phases of a cluster (load, sum, exchange, store) overlap only in part: DRAM works at 36 to
// 38% in fp32, 15 to 22% in bf16, where half the bytes meet the same instructions (8 x 128 x 128 x 192 in bf16: 41 us forward;
// 32 x 56 x 56 x 192 in fp32, forward and gradients: 108 us).
//
// Variances are formed from sums of differences to a value of the tile (two passes: a thread's first pixel; clusters: the
// mean of eight values of the group) and joined as (mean, M2) pairs
// (Chan, Golub & LeVeque 1979), so a mean far from zero costs no digits.  All sums are fp32 in a fixed order.
#include <cooperative_groups.h>

#include <initializer_list>

#include "delta_internal.h"
#include "mixer_internal.h"
#include "vmb_common.cuh"
#include "vmb_internal.h"

namespace vmb {

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormMostChannels = 16384;  // of the C ABI
constexpr size_t kNormL2 = 40u << 20;  // bytes of x (and dy) per launch pair
// Counters at a fixed place, so that calls of any sizes find them at zero: one per sample of a launch, and the
// last for the samples of all launches of a call.
constexpr int kNormCounters = 16384;

template <typename T, int V> struct alignas(sizeof(T) * V) NPack { T v[V]; };

struct NormPlan {
    int rows;    // pixels per tile
    int tiles;   // tiles per sample
    int group;   // samples per launch pair
    size_t partial, means, chan, total;
};

NormPlan plan_norm(int B, long long L, int C, int G, vmb_dtype dtype, bool grads, int sms) {
    NormPlan p{};
    const size_t es = dtype == VMB_BF16 ? 2 : 4;
    const size_t sample = (size_t)L * C * es * (grads ? 2 : 1);
    long long group = sample ? (long long)(kNormL2 / sample) : B;
    if (group > kNormCounters - 1) group = kNormCounters - 1;
    p.group = (int)(group < 1 ? 1 : group > B ? B : group);
    // tiles: about four CTAs per SM over a launch, at least 8 pixels each
    long long tiles = (4LL * sms + p.group - 1) / p.group;
    const long long most = (L + 7) / 8;
    if (tiles > most) tiles = most;
    if (tiles < 1) tiles = 1;
    p.rows = (int)((L + tiles - 1) / tiles);
    p.tiles = (int)((L + p.rows - 1) / p.rows);
    size_t at = kNormCounters * 4;
    p.partial = at;  // forward [group][tiles][G][2], gradients [group][tiles][C][2]
    at += align_up((size_t)p.group * p.tiles * (grads ? C : G) * 8, 256);
    p.means = at;    // [B][G][2]: forward mean and rstd, gradients the two means
    at += align_up((size_t)B * G * 8, 256);
    p.chan = at;     // gradients: [B][C][2] sums of a sample
    if (grads) at += align_up((size_t)B * C * 8, 256);
    p.total = at;
    return p;
}

struct NormLaunch {
    NormArgs a;
    NormPlan p;
    int first;  // first sample of the launch
};

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
// The logistic function of two values, 1 / (1 + e^-z), to a few 2^-22 of itself: where z is far below zero the results are
// small and keep their digits (half of 1 + tanh(z / 2), one operation of the MUFU pipe instead of two, does not: 2^-12 of one).
__device__ __forceinline__ float2 sigmoid2(float2 z) {
    const float2 e = __fmul2_rn(z, both(-kLog2e));
    const float2 d = __fadd2_rn(make_float2(ex2(e.x), ex2(e.y)), both(1.0f));
    return make_float2(rcp(d.x), rcp(d.y));
}
// Of two values the normal distribution's tail, Phi(-|z|) = e^(-z^2 / 2) M(|z|), and that exponential.  M (Mills' ratio over
// sqrt(2 pi)) is t times a polynomial in t = 1 / (1 + 0.28 |z|), fitted here to the smallest largest relative error over all
// |z|: 1.7e-7, 4.8e-7 in fp32.  The tail keeps its digits, which (1 + erf) / 2 loses below -3.  The square's rounding
// error enters the exponent beside it; beyond 16 everything is zero.
__device__ __forceinline__ float2 normal_tail(float2 z, float2& e) {
    const float2 y = make_float2(fminf(fabsf(z.x), 16.0f), fminf(fabsf(z.y), 16.0f));
    const float2 d = __ffma2_rn(y, both(0.28f), both(1.0f)), t = make_float2(rcp(d.x), rcp(d.y));
    const float2 h = __fmul2_rn(y, y), l = __ffma2_rn(y, y, make_float2(-h.x, -h.y));
    const float2 x = __ffma2_rn(h, both(-0.5f * kLog2e), __fmul2_rn(l, both(-0.5f * kLog2e)));
    e = make_float2(ex2(x.x), ex2(x.y));
    constexpr float k[] = {0.0247199844f, -0.0935931646f, 0.0924281759f, -0.00644922176f, 0.0727750275f, 0.0836307883f, 0.103084665f, 0.111699803f, 0.111703858f};
    float2 m = both(k[0]);
#pragma unroll
    for (int i = 1; i < 9; ++i) m = __ffma2_rn(m, t, both(k[i]));
    return __fmul2_rn(__fmul2_rn(m, t), e);
}
__device__ __forceinline__ float2 normal_cdf(float2 z, float2 tail) { return make_float2(z.x < 0.0f ? tail.x : 1.0f - tail.x, z.y < 0.0f ? tail.y : 1.0f - tail.y); }
template <int ACT> __device__ __forceinline__ float2 act_value(float2 z) {
    if constexpr (ACT == VMB_ACT_SILU) return __fmul2_rn(z, sigmoid2(z));
    if constexpr (ACT == VMB_ACT_GELU) {
        float2 e;
        return __fmul2_rn(z, normal_cdf(z, normal_tail(z, e)));
    }
    return z;
}
template <int ACT> __device__ __forceinline__ float2 act_slope(float2 z) {
    if constexpr (ACT == VMB_ACT_SILU) {  // s (1 + z (1 - s)) = s + (z s) (1 - s)
        const float2 s = sigmoid2(z), r = __ffma2_rn(s, both(-1.0f), both(1.0f));
        return __ffma2_rn(__fmul2_rn(z, s), r, s);
    }
    if constexpr (ACT == VMB_ACT_GELU) {  // Phi(z) + z e^(-z^2 / 2) / sqrt(2 pi)
        float2 e;
        const float2 p = normal_cdf(z, normal_tail(z, e));
        return __ffma2_rn(__fmul2_rn(z, both(0.39894228040143268f)), e, p);
    }
    return both(1.0f);
}

// A thread's vector of V channels as pairs (V = 1: the pair's second value is not used).
template <typename T, int V> struct Vec {
    static constexpr int P = (V + 1) / 2;
    float2 v[P];
};
template <typename T, int V> __device__ __forceinline__ Vec<T, V> load_vec(const T* p) {
    const NPack<T, V> f = *reinterpret_cast<const NPack<T, V>*>(p);
    Vec<T, V> r;
#pragma unroll
    for (int i = 0; i < Vec<T, V>::P; ++i) r.v[i] = make_float2(io<T>::cvt(f.v[2 * i]), V > 1 ? io<T>::cvt(f.v[(2 * i + 1) % V]) : 0.0f);
    return r;
}
template <typename T, int V> __device__ __forceinline__ void store_vec(T* p, const Vec<T, V>& r) {
    NPack<T, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.v[i] = io<T>::to(i & 1 ? r.v[i / 2].y : r.v[i / 2].x);
    *reinterpret_cast<NPack<T, V>*>(p) = o;
}
template <int V, typename F> __device__ __forceinline__ void fill(float2 (&v)[(V + 1) / 2], F f) {  // v = f(channel of the vector)
#pragma unroll
    for (int i = 0; i < (V + 1) / 2; ++i) v[i] = make_float2(f(2 * i), V > 1 ? f(2 * i + 1) : 0.0f);
}

// y = act(a x + c) over a thread's pixels, a = weight rstd and c = bias - mean a of its channels.
template <typename T, int V, int ACT>
__device__ __forceinline__ void apply_rows(const T* x, long long x_step, T* y, long long y_step, int first, int rows, int lanes,
                                           const float2 (&a)[(V + 1) / 2], const float2 (&c)[(V + 1) / 2]) {
#pragma unroll 4
    for (int r = first; r < rows; r += lanes) {
        Vec<T, V> f = load_vec<T, V>(x + r * x_step);
#pragma unroll
        for (int i = 0; i < Vec<T, V>::P; ++i) f.v[i] = act_value<ACT>(__ffma2_rn(f.v[i], a[i], c[i]));
        store_vec<T, V>(y + r * y_step, f);
    }
}
// The sums of dz and of dz (x - mean) over a thread's pixels.
template <typename T, int V, int ACT>
__device__ __forceinline__ void slope_sums(const T* x, const T* dy, long long step, int first, int rows, int lanes, const float2 (&a)[(V + 1) / 2],
                                           const float2 (&c)[(V + 1) / 2], const float2 (&mean)[(V + 1) / 2], float2 (&s1)[(V + 1) / 2],
                                           float2 (&s2)[(V + 1) / 2]) {
#pragma unroll 2
    for (int r = first; r < rows; r += lanes) {
        const Vec<T, V> f = load_vec<T, V>(x + r * step), d = load_vec<T, V>(dy + r * step);
#pragma unroll
        for (int i = 0; i < Vec<T, V>::P; ++i) {
            const float2 dz = __fmul2_rn(d.v[i], act_slope<ACT>(__ffma2_rn(f.v[i], a[i], c[i])));
            s1[i] = __fadd2_rn(s1[i], dz);
            s2[i] = __ffma2_rn(dz, __ffma2_rn(mean[i], both(-1.0f), f.v[i]), s2[i]);
        }
    }
}
// dx = rstd (w dz - m1) - rstd^2 m2 (x - mean) = a dz - k1 - k2 (x - mean)
template <typename T, int V, int ACT>
__device__ __forceinline__ void dx_rows(const T* x, const T* dy, long long step, T* dx, long long dx_step, int first, int rows, int lanes,
                                        const float2 (&a)[(V + 1) / 2], const float2 (&c)[(V + 1) / 2], const float2 (&mean)[(V + 1) / 2],
                                        const float2 (&k1)[(V + 1) / 2], const float2 (&k2)[(V + 1) / 2]) {
#pragma unroll 2
    for (int r = first; r < rows; r += lanes) {
        Vec<T, V> f = load_vec<T, V>(x + r * step);
        const Vec<T, V> d = load_vec<T, V>(dy + r * step);
#pragma unroll
        for (int i = 0; i < Vec<T, V>::P; ++i) {
            const float2 dz = __fmul2_rn(d.v[i], act_slope<ACT>(__ffma2_rn(f.v[i], a[i], c[i])));
            const float2 t = __ffma2_rn(__ffma2_rn(mean[i], both(-1.0f), f.v[i]), k2[i], k1[i]);
            f.v[i] = __ffma2_rn(t, both(-1.0f), __fmul2_rn(a[i], dz));
        }
        store_vec<T, V>(dx + r * dx_step, f);
    }
}
// Differences to a pivot and their squares, summed over a thread's pixels.
template <typename T, int V>
__device__ __forceinline__ void pivot_sums(const T* x, long long step, int first, int rows, int lanes, const float2 (&pivot)[(V + 1) / 2],
                                           float2 (&s1)[(V + 1) / 2], float2 (&s2)[(V + 1) / 2]) {
#pragma unroll 4
    for (int r = first; r < rows; r += lanes) {
        const Vec<T, V> f = load_vec<T, V>(x + r * step);
#pragma unroll
        for (int i = 0; i < Vec<T, V>::P; ++i) {
            const float2 d = __ffma2_rn(pivot[i], both(-1.0f), f.v[i]);
            s1[i] = __fadd2_rn(s1[i], d);
            s2[i] = __ffma2_rn(d, d, s2[i]);
        }
    }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// True in every thread of the sample's last tile; the counter is left at zero.
__device__ __forceinline__ bool last_tile(unsigned* counter, int tiles, unsigned* flag) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned old = atomicAdd(counter, 1u);
        *flag = old == (unsigned)tiles - 1;
        if (*flag) *counter = 0;
    }
    __syncthreads();
    const bool last = *flag != 0;
    if (last) __threadfence();
    return last;
}

// First pass, forward: (mean, M2) of every group of a tile, joined over the sample's tiles by the last one.
// A thread takes one vector of V channels and every RL-th pixel.
template <typename T, int V>
__global__ void __launch_bounds__(kNormThreads) norm_stats_kernel(NormLaunch c) {
    extern __shared__ float sm[];
    __shared__ unsigned flag;
    const NormArgs& a = c.a;
    const int C = a.C, Cv = C / V, tid = threadIdx.x;
    float *cm = sm, *c2 = sm + C, *scratch = sm + 2 * C;  // per channel mean and M2; [threads][V][2]
    pdl_launch_dependents();
    pdl_wait();
    const int local = blockIdx.x / c.p.tiles, tile = blockIdx.x % c.p.tiles, b = c.first + local;
    const long long r0 = (long long)tile * c.p.rows;
    const int rows = (int)min((long long)c.p.rows, a.L - r0);
    const T* x = (const T*)a.x + (b * a.L + r0) * C;
    for (int col0 = 0; col0 < Cv; col0 += kNormThreads) {
        const int cols = min(Cv - col0, kNormThreads), lanes = kNormThreads / cols;
        const int col = tid % cols, rl = tid / cols;
        if (rl < lanes && rl < rows) {
            const T* p = x + (long long)(col0 + col) * V;
            const Vec<T, V> f = load_vec<T, V>(p + (long long)rl * C);
            float2 s1[Vec<T, V>::P] = {}, s2[Vec<T, V>::P] = {};
            pivot_sums<T, V>(p, C, rl, rows, lanes, f.v, s1, s2);
            const float inv = 1.0f / (float)((rows - rl + lanes - 1) / lanes);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float t1 = i & 1 ? s1[i / 2].y : s1[i / 2].x, t2 = i & 1 ? s2[i / 2].y : s2[i / 2].x;
                const float m = t1 * inv;
                scratch[(tid * V + i) * 2] = (i & 1 ? f.v[i / 2].y : f.v[i / 2].x) + m;
                scratch[(tid * V + i) * 2 + 1] = fmaf(-m, t1, t2);
            }
        }
        __syncthreads();
        for (int ch = tid; ch < cols * V; ch += kNormThreads) {
            float mean = 0.0f, m2 = 0.0f;
            for (int l = 0; l < lanes && l < rows; ++l)
                mean += (float)((rows - l + lanes - 1) / lanes) * scratch[((l * cols + ch / V) * V + ch % V) * 2];
            mean /= rows;
            for (int l = 0; l < lanes && l < rows; ++l) {
                const float* q = scratch + ((l * cols + ch / V) * V + ch % V) * 2;
                const float d = q[0] - mean;
                m2 += q[1] + (float)((rows - l + lanes - 1) / lanes) * d * d;
            }
            cm[col0 * V + ch] = mean;
            c2[col0 * V + ch] = m2;
        }
        __syncthreads();
    }
    const int m = C / a.G, w = tid >> 5, lane = tid & 31;
    float2* part = reinterpret_cast<float2*>((char*)a.ws + c.p.partial) + (long long)local * c.p.tiles * a.G;
    for (int g = w; g < a.G; g += kNormThreads / 32) {
        float s = 0.0f, q = 0.0f;
        for (int i = lane; i < m; i += 32) s += cm[g * m + i];
        const float mean = warp_sum(s) / m;
        for (int i = lane; i < m; i += 32) {
            const float d = cm[g * m + i] - mean;
            q += fmaf(d * d, (float)rows, c2[g * m + i]);
        }
        q = warp_sum(q);
        if (lane == 0) part[(long long)tile * a.G + g] = make_float2(mean, q);
    }
    if (!last_tile(reinterpret_cast<unsigned*>(a.ws) + local, c.p.tiles, &flag)) return;
    float2* out = reinterpret_cast<float2*>((char*)a.ws + c.p.means) + (long long)b * a.G;
    for (int g = w; g < a.G; g += kNormThreads / 32) {
        float s = 0.0f, q = 0.0f;
        for (int i = lane; i < c.p.tiles; i += 32)
            s += (float)min((long long)c.p.rows, a.L - (long long)i * c.p.rows) * __ldcg(&part[(long long)i * a.G + g]).x;
        const float mean = warp_sum(s) / (float)a.L;
        for (int i = lane; i < c.p.tiles; i += 32) {
            const float2 v = __ldcg(&part[(long long)i * a.G + g]);
            const float d = v.x - mean;
            q += fmaf(d * d, (float)min((long long)c.p.rows, a.L - (long long)i * c.p.rows) * m, v.y);
        }
        q = warp_sum(q);
        if (lane == 0) {
            const float2 v = make_float2(mean, 1.0f / sqrtf(q / ((float)a.L * m) + a.eps));
            out[g] = v;
            if (a.stats) reinterpret_cast<float2*>(a.stats)[(long long)b * a.G + g] = v;
        }
    }
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_apply_kernel(NormLaunch c) {
    const NormArgs& a = c.a;
    const int C = a.C, Cv = C / V, tid = threadIdx.x, m = C / a.G;
    pdl_launch_dependents();
    pdl_wait();
    const int tile = blockIdx.x % c.p.tiles, b = c.first + blockIdx.x / c.p.tiles;
    const long long r0 = (long long)tile * c.p.rows;
    const int rows = (int)min((long long)c.p.rows, a.L - r0);
    const T* x = (const T*)a.x + (b * a.L + r0) * C;
    T* y = (T*)a.y + (b * a.L + r0) * C;
    const float2* st = reinterpret_cast<const float2*>((const char*)a.ws + c.p.means) + (long long)b * a.G;
    for (int col0 = 0; col0 < Cv; col0 += kNormThreads) {
        const int cols = min(Cv - col0, kNormThreads), lanes = kNormThreads / cols;
        const int ch = (col0 + tid % cols) * V, rl = tid / cols;
        if (rl >= lanes) continue;
        float2 ca[Vec<T, V>::P], cc[Vec<T, V>::P];
        fill<V>(ca, [&](int i) { return __ldcg(&st[(ch + i) / m]).y * (a.weight ? a.weight[ch + i] : 1.0f); });
        fill<V>(cc, [&](int i) {
            const float v = i & 1 ? ca[i / 2].y : ca[i / 2].x;
            return fmaf(-__ldcg(&st[(ch + i) / m]).x, v, a.bias ? a.bias[ch + i] : 0.0f);
        });
        apply_rows<T, V, ACT>(x + ch, C, y + ch, C, rl, rows, lanes, ca, cc);
    }
}

// Of a thread's channels: a = weight rstd, c = bias - mean a, mean.
template <typename T, int V>
__device__ __forceinline__ void channel_values(const NormArgs& n, const float2* st, int ch, int m, float2 (&a)[(V + 1) / 2], float2 (&c)[(V + 1) / 2],
                                               float2 (&mean)[(V + 1) / 2]) {
    fill<V>(mean, [&](int i) { return st[(ch + i) / m].x; });
    fill<V>(a, [&](int i) { return st[(ch + i) / m].y * (n.weight ? n.weight[ch + i] : 1.0f); });
    fill<V>(c, [&](int i) {
        return fmaf(-(i & 1 ? mean[i / 2].y : mean[i / 2].x), i & 1 ? a[i / 2].y : a[i / 2].x, n.bias ? n.bias[ch + i] : 0.0f);
    });
}

// First pass of the gradients: per channel sums of dz and dz n over a tile; the sample's last tile joins them,
// forms the two means of every group and, as the last sample of all, dweight and dbias.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_sums_kernel(NormLaunch c) {
    __shared__ float scratch[kNormThreads * V * 2];
    __shared__ unsigned flag;
    const NormArgs& a = c.a;
    const int C = a.C, Cv = C / V, tid = threadIdx.x, m = C / a.G;
    pdl_launch_dependents();
    pdl_wait();
    const int local = blockIdx.x / c.p.tiles, tile = blockIdx.x % c.p.tiles, b = c.first + local;
    const long long r0 = (long long)tile * c.p.rows;
    const int rows = (int)min((long long)c.p.rows, a.L - r0);
    const T *x = (const T*)a.x + (b * a.L + r0) * C, *dy = (const T*)a.dy + (b * a.L + r0) * C;
    const float2* st = reinterpret_cast<const float2*>(a.stats) + (long long)b * a.G;
    float2* part = reinterpret_cast<float2*>((char*)a.ws + c.p.partial) + (long long)local * c.p.tiles * C;
    for (int col0 = 0; col0 < Cv; col0 += kNormThreads) {
        const int cols = min(Cv - col0, kNormThreads), lanes = kNormThreads / cols;
        const int ch = (col0 + tid % cols) * V, rl = tid / cols;
        float2 s1[Vec<T, V>::P] = {}, s2[Vec<T, V>::P] = {};
        if (rl < lanes) {
            float2 ca[Vec<T, V>::P], cc[Vec<T, V>::P], mu[Vec<T, V>::P];
            channel_values<T, V>(a, st, ch, m, ca, cc, mu);
            slope_sums<T, V, ACT>(x + ch, dy + ch, C, rl, rows, lanes, ca, cc, mu, s1, s2);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            scratch[(tid * V + i) * 2] = i & 1 ? s1[i / 2].y : s1[i / 2].x;
            scratch[(tid * V + i) * 2 + 1] = (rl < lanes ? st[(ch + i) / m].y : 0.0f) * (i & 1 ? s2[i / 2].y : s2[i / 2].x);
        }
        __syncthreads();
        for (int k = tid; k < cols * V; k += kNormThreads) {
            float t1 = 0.0f, t2 = 0.0f;
            for (int l = 0; l < lanes; ++l) {
                t1 += scratch[((l * cols + k / V) * V + k % V) * 2];
                t2 += scratch[((l * cols + k / V) * V + k % V) * 2 + 1];
            }
            part[(long long)tile * C + col0 * V + k] = make_float2(t1, t2);
        }
        __syncthreads();
    }
    unsigned* counters = reinterpret_cast<unsigned*>(a.ws);
    if (!last_tile(counters + local, c.p.tiles, &flag)) return;
    float2* chan = reinterpret_cast<float2*>((char*)a.ws + c.p.chan) + (long long)b * C;
    for (int k = tid; k < C; k += kNormThreads) {
        float t1 = 0.0f, t2 = 0.0f;
#pragma unroll 16
        for (int i = 0; i < c.p.tiles; ++i) {
            const float2 v = __ldcg(&part[(long long)i * C + k]);
            t1 += v.x;
            t2 += v.y;
        }
        chan[k] = make_float2(t1, t2);
    }
    __syncthreads();
    const int w = tid >> 5, lane = tid & 31;
    float2* means = reinterpret_cast<float2*>((char*)a.ws + c.p.means) + (long long)b * a.G;
    for (int g = w; g < a.G; g += kNormThreads / 32) {
        float t1 = 0.0f, t2 = 0.0f;
        for (int i = lane; i < m; i += 32) {
            const float2 v = chan[g * m + i];
            const float wt = a.weight ? a.weight[g * m + i] : 1.0f;
            t1 = fmaf(wt, v.x, t1);
            t2 = fmaf(wt, v.y, t2);
        }
        t1 = warp_sum(t1);
        t2 = warp_sum(t2);
        if (lane == 0) means[g] = make_float2(t1 / ((float)a.L * m), t2 / ((float)a.L * m));
    }
    if (!last_tile(counters + kNormCounters - 1, a.B, &flag)) return;
    const float2* all = reinterpret_cast<const float2*>((const char*)a.ws + c.p.chan);
    for (int k = tid; k < C; k += kNormThreads) {
        float t1 = 0.0f, t2 = 0.0f;
#pragma unroll 16
        for (int i = 0; i < a.B; ++i) {
            const float2 v = __ldcg(&all[(long long)i * C + k]);
            t1 += v.x;
            t2 += v.y;
        }
        if (a.dbias) a.dbias[k] = t1;
        if (a.dweight) a.dweight[k] = t2;
    }
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_dx_kernel(NormLaunch c) {
    const NormArgs& a = c.a;
    const int C = a.C, Cv = C / V, tid = threadIdx.x, m = C / a.G;
    pdl_launch_dependents();
    pdl_wait();
    const int tile = blockIdx.x % c.p.tiles, b = c.first + blockIdx.x / c.p.tiles;
    const long long r0 = (long long)tile * c.p.rows, at = (b * a.L + r0) * C;
    const int rows = (int)min((long long)c.p.rows, a.L - r0);
    const T *x = (const T*)a.x + at, *dy = (const T*)a.dy + at;
    T* dx = (T*)a.dx + at;
    const float2 *st = reinterpret_cast<const float2*>(a.stats) + (long long)b * a.G,
                 *mn = reinterpret_cast<const float2*>((const char*)a.ws + c.p.means) + (long long)b * a.G;
    for (int col0 = 0; col0 < Cv; col0 += kNormThreads) {
        const int cols = min(Cv - col0, kNormThreads), lanes = kNormThreads / cols;
        const int ch = (col0 + tid % cols) * V, rl = tid / cols;
        if (rl >= lanes) continue;
        float2 ca[Vec<T, V>::P], cc[Vec<T, V>::P], mu[Vec<T, V>::P], k1[Vec<T, V>::P], k2[Vec<T, V>::P];
        channel_values<T, V>(a, st, ch, m, ca, cc, mu);
        fill<V>(k1, [&](int i) { return st[(ch + i) / m].y * __ldcg(&mn[(ch + i) / m]).x; });
        fill<V>(k2, [&](int i) { return st[(ch + i) / m].y * (st[(ch + i) / m].y * __ldcg(&mn[(ch + i) / m]).y); });
        dx_rows<T, V, ACT>(x + ch, dy + ch, C, dx + ch, C, rl, rows, lanes, ca, cc, mu, k1, k2);
    }
}

// ------------------------------------------------------------------ samples that fit a cluster

// A slab: the pixels of one sample and `width` neighbouring channels (whole groups), cut into `ctas` runs of `rows`
// pixels, one per CTA of a cluster.
struct NormSlab {
    int width, slabs, ctas, rows;
};
// Several CTAs per SM, so that some load or store while others compute; a cluster of eight is the portable limit (16 CTAs
// of half the size were slower: 66 against 44 us for 8 x 128 x 128 x 192 in bf16).
constexpr int kSlabCluster = 8, kSlabThreads = 256;
constexpr size_t kSlabSmem = 113 * 1024, kSlabSmall = 57 * 1024;  // two CTAs per SM, three or four
// The tile, a sum per thread and channel of its vector, two partial sums per thread, and what the cluster's CTAs send:
// forward one pair per group, gradients one per channel.
inline size_t slab_smem(long long rows, int width, int groups, int ctas, size_t es, bool grads) {
    return (((size_t)rows * width * es * (grads ? 2 : 1) + 15) & ~(size_t)15) + kSlabThreads * (16 / es) * 4 + (size_t)(width > kSlabThreads ? width : kSlabThreads) * 8 +
           (size_t)ctas * (grads ? width : groups) * 8 + (size_t)groups * 8;
}

// Channels per slab: as many groups as a cluster holds, at least 32 bytes of every pixel (a sector of memory), fewer as
// long as that gives every SM two CTAs and a pixel still 64 bytes.  CTAs per slab: as few as hold it, more where the
// SMs would not have two each and the runs stay at 16 pixels or more.  Forward with small tiles where they fit (32 x 56 x
// 56 x 192 in fp32: 36 us in six CTAs of 50 KB, 42 in eight of 75 KB); the gradients hold x and dy, and their CTAs use
// more registers (73 us in six CTAs of 100 KB, 79 in clusters of 12 channels of 60 KB).
bool norm_slab(int B, long long L, int C, int G, vmb_dtype dtype, bool grads, int sms, NormSlab* out) {
    const size_t es = dtype == VMB_BF16 ? 2 : 4;
    const int m = C / G, v = (int)(16 / es);
    if (C % v || L > 1 << 24) return false;
    for (const size_t limit : {kSlabSmall, kSlabSmem}) {
        if (grads && limit == kSlabSmall) continue;
        int best = 0;
        for (int g = 1; g <= G; ++g) {
            if (G % g || (g * m) % v || g * m / v > kSlabThreads || g * m > 2048) continue;
            if (slab_smem((L + kSlabCluster - 1) / kSlabCluster, g * m, g, kSlabCluster, es, grads) > limit) break;
            const long long ctas = (long long)B * (G / g) * kSlabCluster;
            if (best && (size_t)best * es >= 64 && ctas < 2LL * sms) break;
            best = g * m;
        }
        if (!best || (size_t)best * es < 32) continue;
        out->width = best;
        out->slabs = C / best;
        int n = 1;
        while (n < kSlabCluster && (slab_smem((L + n - 1) / n, best, best / m, n, es, grads) > limit ||
                                    ((long long)B * out->slabs * n < 2LL * sms && L / (n + 1) >= 16)))
            ++n;
        out->ctas = n;
        out->rows = (int)((L + n - 1) / n);
        return true;
    }
    return false;
}

struct SlabLaunch {
    NormArgs a;
    NormSlab s;
    float2* chan;        // gradients: [B][C] sums of a sample
    unsigned* counter;
};

// A CTA's shared memory is written to by the others only once it has started: every CTA says so and, before it sends,
// waits for the others.  Nothing but the start itself is passed on, so that the arrival orders no memory.
__device__ __forceinline__ void cluster_started() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_cluster_started() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }

// A thread's sums of its V channels, two each, summed over the threads of a column in two steps, in order: afterwards
// part[k width + ch], k < parts, holds the partial sums of channel ch.  ch0, k0: the thread's number as k0 width + ch0.
template <typename T, int V>
__device__ __forceinline__ void column_parts(const float2 (&s1)[(V + 1) / 2], const float2 (&s2)[(V + 1) / 2], float* scratch, float2* part, int width,
                                            int cols, int lanes, int ch0, int k0, int parts) {
    const int tid = threadIdx.x;
#pragma unroll
    for (int round = 0; round < 2; ++round) {
        const float2(&v)[(V + 1) / 2] = round ? s2 : s1;
#pragma unroll
        for (int i = 0; i < V; ++i) scratch[tid * V + i] = i & 1 ? v[i / 2].y : v[i / 2].x;
        __syncthreads();
        for (int i = tid, ch = ch0, k = k0; i < parts * width; i += kSlabThreads, ch += kSlabThreads) {
            if (ch >= width) ch -= width, ++k;  // (more than one turn only where parts = 1)
            float s = 0.0f;
#pragma unroll 4
            for (int l = k; l < lanes; l += parts) s += scratch[l * cols * V + ch];
            (round ? part[i].y : part[i].x) = s;
        }
        __syncthreads();
    }
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kSlabThreads, 3) norm_cluster_kernel(SlabLaunch c) {
    namespace cg = cooperative_groups;
    extern __shared__ __align__(16) unsigned char shm[];
    const NormArgs& a = c.a;
    const cg::cluster_group cl = cg::this_cluster();
    const int ctas = c.s.ctas, rank = (int)cl.block_rank(), width = c.s.width, tid = threadIdx.x;
    const int m = a.C / a.G, groups = width / m, cols = width / V, lanes = kSlabThreads / cols;
    T* tile = reinterpret_cast<T*>(shm);
    float* scratch = reinterpret_cast<float*>(shm + (((size_t)c.s.rows * width * sizeof(T) + 15) & ~(size_t)15));
    float2 *part = reinterpret_cast<float2*>(scratch + kSlabThreads * V), *sent = part + max(width, kSlabThreads);  // sent: [ctas][groups] mean and M2
    float2* all = sent + ctas * groups;
    cluster_started();
    pdl_launch_dependents();
    pdl_wait();
    const long long slab = blockIdx.x / ctas;
    const int b = (int)(slab / c.s.slabs), ch0 = (int)(slab % c.s.slabs) * width;
    const long long r0 = (long long)rank * c.s.rows;
    const int rows = (int)max(0LL, min((long long)c.s.rows, a.L - r0));
    const T* x = (const T*)a.x + (b * a.L + r0) * a.C + ch0;
    const int col = tid % cols, rl = tid / cols;
    const bool on = rl < lanes;
    if (on)
        for (int r = rl; r < rows; r += lanes) cp_async16(tile + (long long)r * width + col * V, x + (long long)r * a.C + col * V, 16);
    cp_async_commit();
    const int parts = width < kSlabThreads ? min(kSlabThreads / width, lanes) : 1, ch1 = tid % width, k1 = tid / width;
    const int w = tid >> 5, lane = tid & 31;
    const int left = (int)a.L - (tid & 7) * c.s.rows, run = max(0, min(c.s.rows, left));  // pixels of CTA tid % 8
    cp_async_wait<0>();
    __syncthreads();
    // a pivot for every group, the mean of eight of its values: their sum's square then takes little from the squares' sum
    float* pivots = reinterpret_cast<float*>(all);
    for (int g = tid; g < groups; g += kSlabThreads) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += rows > 0 ? io<T>::cvt(tile[(long long)(i * rows / 8) * width + g * m + (i & 1) * (m - 1)]) : 0.0f;
        pivots[g] = 0.125f * s;
    }
    __syncthreads();
    {
        // sums of the differences to the pivot of each group, and of their squares
        float2 s1[Vec<T, V>::P] = {}, s2[Vec<T, V>::P] = {}, pivot[Vec<T, V>::P];
        if (on && rows > 0) {
            fill<V>(pivot, [&](int i) { return pivots[(col * V + i) / m]; });
            pivot_sums<T, V>(tile + col * V, width, rl, rows, lanes, pivot, s1, s2);
        }
        column_parts<T, V>(s1, s2, scratch, part, width, cols, lanes, ch1, k1, parts);
        wait_cluster_started();
        const float inv = 1.0f / ((float)max(rows, 1) * m);
        for (int g = w; g < groups; g += kSlabThreads / 32) {
            float t1 = 0.0f, t2 = 0.0f;
            for (int ch = g * m + lane; ch < g * m + m; ch += 32) {
#pragma unroll 4
                for (int k = 0; k < parts; ++k) {
                    const float2 v = part[k * width + ch];
                    t1 += v.x;
                    t2 += v.y;
                }
            }
            t1 = warp_sum(t1);
            t2 = warp_sum(t2);
            const float2 v = make_float2(pivots[g] + t1 * inv, fmaf(-t1 * inv, t1, t2));
            if (lane < ctas) *cl.map_shared_rank(sent + rank * groups + g, lane) = v;  // to every CTA of the cluster
        }
    }
    cl.sync();
    // every CTA joins the cluster's means and M2 for itself: eight threads per group, one for each CTA
    static_assert(kSlabCluster == 8, "threads per group");
    for (int g0 = 0; g0 < groups; g0 += kSlabThreads / 8) {
        const int g = g0 + (tid >> 3), r = tid & 7;
        const bool mine = g < groups && r < ctas;
        const float2 v = mine ? sent[r * groups + g] : make_float2(0.0f, 0.0f);
        const float n = mine ? (float)run : 0.0f;
        float mu = n * v.x;
        mu += __shfl_xor_sync(0xffffffffu, mu, 1);
        mu += __shfl_xor_sync(0xffffffffu, mu, 2);
        mu += __shfl_xor_sync(0xffffffffu, mu, 4);
        mu /= (float)a.L;
        const float d = v.x - mu;
        float q = mine ? fmaf(d * d, n * m, v.y) : 0.0f;
        q += __shfl_xor_sync(0xffffffffu, q, 1);
        q += __shfl_xor_sync(0xffffffffu, q, 2);
        q += __shfl_xor_sync(0xffffffffu, q, 4);
        if (mine && r == 0) {
            const float2 out = make_float2(mu, 1.0f / sqrtf(q / ((float)a.L * m) + a.eps));
            all[g] = out;
            if (a.stats && rank == 0) reinterpret_cast<float2*>(a.stats)[(long long)b * a.G + ch0 / m + g] = out;
        }
    }
    __syncthreads();
    if (!on) return;
    float2 ca[Vec<T, V>::P], cc[Vec<T, V>::P];
    const int ch = ch0 + col * V;
    fill<V>(ca, [&](int i) { return all[(col * V + i) / m].y * (a.weight ? a.weight[ch + i] : 1.0f); });
    fill<V>(cc, [&](int i) {
        return fmaf(-all[(col * V + i) / m].x, i & 1 ? ca[i / 2].y : ca[i / 2].x, a.bias ? a.bias[ch + i] : 0.0f);
    });
    apply_rows<T, V, ACT>(tile + col * V, width, (T*)a.y + (b * a.L + r0) * a.C + ch, a.C, rl, rows, lanes, ca, cc);
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kSlabThreads, 2) norm_cluster_grad_kernel(SlabLaunch c) {
    namespace cg = cooperative_groups;
    extern __shared__ __align__(16) unsigned char shm[];
    __shared__ unsigned flag;
    const NormArgs& a = c.a;
    const cg::cluster_group cl = cg::this_cluster();
    const int ctas = c.s.ctas, rank = (int)cl.block_rank(), width = c.s.width, tid = threadIdx.x;
    const int m = a.C / a.G, groups = width / m, cols = width / V, lanes = kSlabThreads / cols;
    T *tx = reinterpret_cast<T*>(shm), *td = tx + (size_t)c.s.rows * width;
    float* scratch = reinterpret_cast<float*>(shm + (((size_t)2 * c.s.rows * width * sizeof(T) + 15) & ~(size_t)15));
    float2 *part = reinterpret_cast<float2*>(scratch + kSlabThreads * V), *sent = part + max(width, kSlabThreads);  // sent: [ctas][width] sums of dz, dz n
    float2* mine = sent + ctas * width;
    cluster_started();
    pdl_launch_dependents();
    pdl_wait();
    const long long slab = blockIdx.x / ctas;
    const int b = (int)(slab / c.s.slabs), ch0 = (int)(slab % c.s.slabs) * width;
    const long long r0 = (long long)rank * c.s.rows, at = (b * a.L + r0) * a.C + ch0;
    const int rows = (int)max(0LL, min((long long)c.s.rows, a.L - r0));
    const int col = tid % cols, rl = tid / cols;
    const bool on = rl < lanes;
    if (on) {
        const T *x = (const T*)a.x + at + col * V, *dy = (const T*)a.dy + at + col * V;
        for (int r = rl; r < rows; r += lanes) {
            cp_async16(tx + (long long)r * width + col * V, x + (long long)r * a.C, 16);
            cp_async16(td + (long long)r * width + col * V, dy + (long long)r * a.C, 16);
        }
    }
    cp_async_commit();
    float2 ca[Vec<T, V>::P], cc[Vec<T, V>::P], mu[Vec<T, V>::P];
    const float2* st = reinterpret_cast<const float2*>(a.stats) + (long long)b * a.G;
    const int mych = ch0 + (on ? col * V : 0);
    const int parts = width < kSlabThreads ? min(kSlabThreads / width, lanes) : 1, ch1 = tid % width, k1 = tid / width;
    channel_values<T, V>(a, st, mych, m, ca, cc, mu);
    cp_async_wait<0>();  // (a thread reads back what it copied itself)
    {
        float2 s1[Vec<T, V>::P] = {}, s2[Vec<T, V>::P] = {};
        if (on) slope_sums<T, V, ACT>(tx + col * V, td + col * V, width, rl, rows, lanes, ca, cc, mu, s1, s2);
        column_parts<T, V>(s1, s2, scratch, part, width, cols, lanes, ch1, k1, parts);
        wait_cluster_started();
        for (int ch = tid; ch < width; ch += kSlabThreads) {  // to every CTA of the cluster
            float2 s = make_float2(0.0f, 0.0f);
#pragma unroll 4
            for (int k = 0; k < parts; ++k) s = __fadd2_rn(s, part[k * width + ch]);
            s.y *= st[(ch0 + ch) / m].y;
            for (int r = 0; r < ctas; ++r) *cl.map_shared_rank(sent + rank * width + ch, r) = s;
        }
    }
    cl.sync();
    {
        const int w = tid >> 5, lane = tid & 31;
        for (int g = w; g < groups; g += kSlabThreads / 32) {
            float t1 = 0.0f, t2 = 0.0f;
            for (int i = lane; i < m; i += 32) {
                float2 u = make_float2(0.0f, 0.0f);
#pragma unroll 8
                for (int k = 0; k < ctas; ++k) u = __fadd2_rn(u, sent[k * width + g * m + i]);
                const float wv = a.weight ? a.weight[ch0 + g * m + i] : 1.0f;
                t1 = fmaf(wv, u.x, t1);
                t2 = fmaf(wv, u.y, t2);
                if (rank == 0) c.chan[(long long)b * a.C + ch0 + g * m + i] = u;
            }
            t1 = warp_sum(t1);
            t2 = warp_sum(t2);
            if (lane == 0) mine[g] = make_float2(t1 / ((float)a.L * m), t2 / ((float)a.L * m));
        }
    }
    __syncthreads();
    if (on) {
        float2 f1[Vec<T, V>::P], f2[Vec<T, V>::P];
        fill<V>(f1, [&](int i) { return st[(mych + i) / m].y * mine[(col * V + i) / m].x; });
        fill<V>(f2, [&](int i) { return st[(mych + i) / m].y * (st[(mych + i) / m].y * mine[(col * V + i) / m].y); });
        dx_rows<T, V, ACT>(tx + col * V, td + col * V, width, (T*)a.dx + at + col * V, a.C, rl, rows, lanes, ca, cc, mu, f1, f2);
    }
    if (rank != 0 || (!a.dweight && !a.dbias)) return;
    if (!last_tile(c.counter, a.B * c.s.slabs, &flag)) return;  // the last slab of all: the sums over the batch
    for (int k = tid; k < a.C; k += kSlabThreads) {
        float t1 = 0.0f, t2 = 0.0f;
#pragma unroll 16
        for (int i = 0; i < a.B; ++i) {
            const float2 v = __ldcg(&c.chan[(long long)i * a.C + k]);
            t1 += v.x;
            t2 += v.y;
        }
        if (a.dbias) a.dbias[k] = t1;
        if (a.dweight) a.dweight[k] = t2;
    }
}

template <typename T, int V, int ACT>
vmb_status run_slabs(const NormArgs& a, const NormSlab& s, bool grads, size_t chan_off, cudaStream_t stream) {
    SlabLaunch c{a, s, reinterpret_cast<float2*>((char*)a.ws + chan_off), reinterpret_cast<unsigned*>(a.ws) + kNormCounters - 1};
    const void* fn = grads ? (const void*)norm_cluster_grad_kernel<T, V, ACT> : (const void*)norm_cluster_kernel<T, V, ACT>;
    const size_t smem = slab_smem(s.rows, s.width, s.width / (a.C / a.G), s.ctas, sizeof(T), grads);
    if (!allow_smem(fn, kSlabSmem)) return VMB_ERR_CUDA;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((long long)a.B * s.slabs * s.ctas));
    cfg.blockDim = dim3(kSlabThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)s.ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    void* args[] = {&c};
    return cudaLaunchKernelExC(&cfg, fn, args) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

template <typename T, int V, int ACT>
vmb_status run_norm(const NormArgs& a, bool grads, cudaStream_t stream) {
    NormLaunch c{a, plan_norm(a.B, a.L, a.C, a.G, a.dtype, grads, device_sm_count()), 0};
    if (a.ws_bytes < c.p.total) return VMB_ERR_WORKSPACE;
    NormSlab slab;
    if constexpr (V * sizeof(T) == 16)
        if (norm_slab(a.B, a.L, a.C, a.G, a.dtype, grads, device_sm_count(), &slab) &&
            (long long)a.B * slab.slabs * slab.ctas <= 2147483647LL && (long long)a.B * slab.slabs <= 2147483647LL)
            return run_slabs<T, V, ACT>(a, slab, grads, c.p.chan, stream);
    const void* one = grads ? (const void*)norm_sums_kernel<T, V, ACT> : (const void*)norm_stats_kernel<T, V>;
    const void* two = grads ? (const void*)norm_dx_kernel<T, V, ACT> : (const void*)norm_apply_kernel<T, V, ACT>;
    const size_t smem = grads ? 0 : (size_t)a.C * 8 + kNormThreads * V * 8;
    // (a kernel's limit is set once, to what the widest map needs: another thread may be between its own and its launch)
    if (smem > 48 * 1024 && !allow_smem(one, kNormMostChannels * 8 + kNormThreads * V * 8)) return VMB_ERR_CUDA;
    void* args[] = {&c};
    for (int b = 0; b < a.B; b += c.p.group) {
        c.first = b;
        const int n = a.B - b < c.p.group ? a.B - b : c.p.group;
        const dim3 grid((unsigned)((long long)n * c.p.tiles));
        if (launch_kernel(one, grid, dim3(kNormThreads), smem, args, stream) != cudaSuccess) return VMB_ERR_CUDA;
        if (launch_kernel(two, grid, dim3(kNormThreads), 0, args, stream) != cudaSuccess) return VMB_ERR_CUDA;
    }
    return VMB_OK;
}
template <typename T, int V>
vmb_status run_act(const NormArgs& a, bool grads, cudaStream_t stream) {
    if (a.act == VMB_ACT_SILU) return run_norm<T, V, VMB_ACT_SILU>(a, grads, stream);
    if (a.act == VMB_ACT_GELU) return run_norm<T, V, VMB_ACT_GELU>(a, grads, stream);
    return run_norm<T, V, VMB_ACT_NONE>(a, grads, stream);
}
vmb_status run_type(const NormArgs& a, bool grads, cudaStream_t stream) {
    const unsigned es = a.dtype == VMB_BF16 ? 2 : 4;
    const uintptr_t bits = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.dy) |
                           reinterpret_cast<uintptr_t>(a.dx) | (uintptr_t)a.C * es;
    const bool vec = bits % 16 == 0;
    if (a.dtype == VMB_BF16) return vec ? run_act<__nv_bfloat16, 8>(a, grads, stream) : run_act<__nv_bfloat16, 1>(a, grads, stream);
    return vec ? run_act<float, 4>(a, grads, stream) : run_act<float, 1>(a, grads, stream);
}

}  // namespace

size_t norm_workspace_bytes(int B, long long L, int C, int G, vmb_dtype dtype, bool grads) {
    return plan_norm(B, L, C, G, dtype, grads, device_sm_count()).total;
}
vmb_status launch_norm_fwd(const NormArgs& a, cudaStream_t stream) { return run_type(a, false, stream); }
vmb_status launch_norm_bwd(const NormArgs& a, cudaStream_t stream) { return run_type(a, true, stream); }

}  // namespace vmb
