// rotary.cu - rotary positions with several axes.
//
// Pair i of a head's first 2P channels is turned by the angle p f_i, p the token's position on the axis
// that pair i belongs to:  (x, y) -> (x cos - y sin, y cos + x sin).  The gradient is the turn by the
// opposite angle.  Bound by the bytes of q and k, read and written once: the sines of a token are
// computed once into shared memory and serve all of its heads.  (32 x 784 tokens of 6 heads of 64 in fp32: 24.4 us, 93% of
// the copy rate.  4 videos of 12544 tokens, 12 + 6 heads of 96 in bf16 and three axes: 88.6 us, 58%: the 28 warps of an SM
// have too few loads in flight, and a token's 36 sines serve half the bytes per value.)
//
// The error of an angle does not grow with the position (the product p f alone is off by 2^-24 p f: 2e-4 at
// position 4096): up to 1024 radians the product's rounding error, lo = p f - hi, is turned by to first order
// (lo^2 / 2 < 2^-31); larger angles, and positions that a float may not hold (from 2^24 on), which few tokens have, are
// brought into [-pi, pi] in 64 bits, again with the product's rounding error.
#include <string.h>

#include "mixer_internal.h"
#include "vmb_common.cuh"
#include "vmb_internal.h"

namespace vmb {

namespace {

constexpr int kRotThreads = 256;

template <typename T, int V, bool kLoose> struct alignas(kLoose ? sizeof(T) : sizeof(T) * V) Pack { T v[V]; };

// cos and sin of p f
__device__ __forceinline__ float2 turn(int p, float f) {
    const float ph = (float)p;
    float hi = ph * f, lo = fmaf(ph, f, -hi);
    if (!(fabsf(hi) <= 1024.0f && fabsf(ph) < 16777216.0f)) {
        const double a = (double)p * (double)f, n = rint(a * 0.15915494309189535), low = fma((double)p, (double)f, -a);  // turns
        hi = (float)(fma(-n, 2.4492935982947064e-16, fma(-n, 6.283185307179586, a)) + low), lo = 0.0f;  // 2 pi in two parts
    }
    float s, c;
    sincosf(hi, &s, &c);
    return make_float2(fmaf(-lo, s, c), fmaf(lo, c, s));
}
// one pair turned: (u cos - v sin, v cos + u sin), the same operations on every path
__device__ __forceinline__ float2 turned(float u, float v, float2 w) {
    return make_float2(fmaf(u, w.x, -__fmul_rn(v, w.y)), fmaf(v, w.x, __fmul_rn(u, w.y)));
}

// Two bf16 values of a word, and back.
__device__ __forceinline__ float2 unpack2(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// A head's items: half: vectors of V pairs (V channels from each half); interleaved: vectors of V channels (V / 2 pairs);
// then the vectors of V channels that stay as they are (kLoose, for pairs in rows of no alignment: single channels).
// A thread keeps its items of a token, of q and k alike, and goes from token to token, so that nothing is divided in
// the loop; kBatch tokens' values are read before the first is written, the first batch before the sines are computed.
constexpr int kBatch = 4;
template <typename T, int V, bool kInter, bool kLoose> struct Turner {
    const T *s0, *s1;
    T *d0, *d1;
    const float2* cs;
    long long src_t, dst_t;
    int first, lanes;  // tokens first, first + lanes, ...
    bool turns, two;
    Pack<T, V, kLoose> a[kBatch], b[kBatch];

    __device__ __forceinline__ void set(const T* src, T* dst, const float2* table, long long st, int H, int D, int P, int e, int items, int n) {
        const int h = e / items, j = e - h * items;
        turns = j < n;
        two = !kInter && turns;
        const long long at = (long long)h * D + (turns ? j * V : 2 * P + (j - n) * (kLoose ? 1 : V));
        s0 = src + at, s1 = s0 + P;
        d0 = dst + at, d1 = d0 + P;
        cs = table + j * (kInter ? V / 2 : V);
        src_t = st, dst_t = (long long)H * D;
    }
    __device__ __forceinline__ void read(int t0, int tokens) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int t = t0 + u * lanes;
            if (t >= tokens) break;
            if (kLoose && !turns) {
                a[u].v[0] = s0[t * src_t];
                continue;
            }
            a[u] = *reinterpret_cast<const Pack<T, V, kLoose>*>(s0 + t * src_t);
            if (two) b[u] = *reinterpret_cast<const Pack<T, V, kLoose>*>(s1 + t * src_t);
        }
    }
    __device__ __forceinline__ void write(int t0, int tokens, int P) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int t = t0 + u * lanes;
            if (t >= tokens) break;
            if (kLoose && !turns) {
                d0[t * dst_t] = a[u].v[0];
                continue;
            }
            if (turns) {
                const float2* w = cs + t * P;
                if constexpr (sizeof(T) == 2 && V >= 2 && !kLoose) {  // a word, two channels, at a time
                    uint32_t wa[V / 2], wb[V / 2];
                    memcpy(wa, &a[u], sizeof(wa));
                    if constexpr (!kInter) memcpy(wb, &b[u], sizeof(wb));
#pragma unroll
                    for (int x = 0; x < V / 2; ++x) {
                        const float2 p = unpack2(wa[x]);
                        if constexpr (kInter) {
                            const float2 o = turned(p.x, p.y, w[x]);
                            wa[x] = pack2(o.x, o.y);
                        } else {
                            const float2 q = unpack2(wb[x]), o0 = turned(p.x, q.x, w[2 * x]), o1 = turned(p.y, q.y, w[2 * x + 1]);
                            wa[x] = pack2(o0.x, o1.x);
                            wb[x] = pack2(o0.y, o1.y);
                        }
                    }
                    memcpy(&a[u], wa, sizeof(wa));
                    if constexpr (!kInter) {
                        memcpy(&b[u], wb, sizeof(wb));
                        *reinterpret_cast<Pack<T, V, kLoose>*>(d1 + t * dst_t) = b[u];
                    }
                } else if constexpr (kInter) {
#pragma unroll
                    for (int x = 0; x < V / 2; ++x) {
                        const float2 o = turned(io<T>::cvt(a[u].v[2 * x]), io<T>::cvt(a[u].v[2 * x + 1]), w[x]);
                        a[u].v[2 * x] = io<T>::to(o.x);
                        a[u].v[2 * x + 1] = io<T>::to(o.y);
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < V; ++x) {
                        const float2 o = turned(io<T>::cvt(a[u].v[x]), io<T>::cvt(b[u].v[x]), w[x]);
                        a[u].v[x] = io<T>::to(o.x);
                        b[u].v[x] = io<T>::to(o.y);
                    }
                    *reinterpret_cast<Pack<T, V, kLoose>*>(d1 + t * dst_t) = b[u];
                }
            }
            *reinterpret_cast<Pack<T, V, kLoose>*>(d0 + t * dst_t) = a[u];
        }
    }
};

template <typename T, int V, bool kInter, bool kLoose>
__global__ void __launch_bounds__(kRotThreads, 4) rotary_kernel(RotaryArgs a, int per_block, int blocks_per_row) {
    extern __shared__ float2 table[];
    const int P = a.pair_end[a.axes - 1];
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x / blocks_per_row, t0 = (blockIdx.x % blocks_per_row) * per_block;
    const int n = min(per_block, a.T - t0);
    const int turns = kInter ? 2 * P / V : P / V, items = turns + (a.D - 2 * P) / (kLoose ? 1 : V);
    const int per_q = a.Hq * items, per = per_q + a.Hk * items;
    Turner<T, V, kInter, kLoose> w;
    w.lanes = per < kRotThreads ? kRotThreads / per : 1;
    int e0 = threadIdx.x;
    auto set = [&]() {
        w.first = w.lanes > 1 ? e0 / per : 0;
        const int e = w.lanes > 1 ? e0 - w.first * per : e0;
        if (e < per_q)
            w.set((const T*)a.q + b * a.q_b + t0 * a.q_t, (T*)a.q_out + ((long long)b * a.T + t0) * a.Hq * a.D, table, a.q_t, a.Hq, a.D, P, e,
                  items, turns);
        else
            w.set((const T*)a.k + b * a.k_b + t0 * a.k_t, (T*)a.k_out + ((long long)b * a.T + t0) * a.Hk * a.D, table, a.k_t, a.Hk, a.D, P,
                  e - per_q, items, turns);
    };
    const bool on = e0 < per * w.lanes;
    if (on) {
        set();
        w.read(w.first, n);
    }
    for (int i = threadIdx.x; i < n * P; i += kRotThreads) {
        const int tok = t0 + i / P, j = i % P;
        int axis = 0;
        while (axis < a.axes - 1 && j >= a.pair_end[axis]) ++axis;
        int p;
        if (a.positions) {
            p = a.positions[((long long)axis * a.B + b) * a.T + tok];
        } else {
            int rest = tok;
            for (int x = a.axes - 1; x > axis; --x) rest /= a.grid[x];
            p = rest % a.grid[axis];
        }
        const float2 cs = turn(p, a.freq[j]);
        table[i] = make_float2(cs.x, a.inverse ? -cs.y : cs.y);
    }
    __syncthreads();
    if (!on) return;
    for (;;) {
        for (int t = w.first;;) {
            w.write(t, n, P);
            t += kBatch * w.lanes;
            if (t >= n) break;
            w.read(t, n);
        }
        e0 += kRotThreads;
        if (e0 >= per * w.lanes) return;
        set();
        w.read(w.first, n);
    }
}

template <typename T, int V, bool kLoose = false>
vmb_status launch_v(const RotaryArgs& a, cudaStream_t stream) {
    const int P = a.pair_end[a.axes - 1];
    // tokens per block: one batch per thread (two in bf16, whose vectors hold twice the channels, so that a token's sines
    // are spread over enough of them: 24.3 and 25.0 us in fp32, 102 and 93 us in bf16), within 32 KB of sines, and enough
    // blocks for every SM
    constexpr int kBatches = sizeof(T) == 2 ? 2 : 1;
    const long long per_token = (long long)(a.Hq + a.Hk) * ((a.interleaved ? 2 * P / V : P / V) + (a.D - 2 * P) / V);
    long long per = per_token <= kRotThreads ? kBatches * kBatch * (kRotThreads / per_token) : kBatches * kBatch;
    const long long most = 32 * 1024 / (8 * (long long)P), spread = ((long long)a.B * a.T + 2 * device_sm_count() - 1) / (2 * device_sm_count());
    per = per < most ? per : most;
    per = per < spread ? per : spread;
    if (per < 1) per = 1;
    if (per > a.T) per = a.T;
    int per_block = (int)per, blocks = (int)((a.T + per - 1) / per);
    if ((long long)blocks * a.B > 2147483647LL) return VMB_ERR_UNSUPPORTED;
    const void* fn;
    if constexpr (V == 1)
        fn = (const void*)rotary_kernel<T, V, false, false>;
    else if constexpr (kLoose)
        fn = (const void*)rotary_kernel<T, V, true, true>;
    else
        fn = a.interleaved ? (const void*)rotary_kernel<T, V, true, false> : (const void*)rotary_kernel<T, V, false, false>;
    RotaryArgs arg = a;
    void* args[] = {&arg, &per_block, &blocks};
    return launch_kernel(fn, dim3((unsigned)(blocks * (long long)a.B)), dim3(kRotThreads), (size_t)per_block * P * 8, args, stream) == cudaSuccess
               ? VMB_OK : VMB_ERR_CUDA;
}

}  // namespace

// The widest vectors (up to 16 bytes) that divide the turned channels (each half of them, unless pairs are
// neighbours), the rows and the addresses.
vmb_status launch_rotary(const RotaryArgs& a, cudaStream_t stream) {
    const int P = a.pair_end[a.axes - 1];
    const unsigned es = a.dtype == VMB_BF16 ? 2 : 4;
    const unsigned long long bytes = (reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.q_out) | reinterpret_cast<uintptr_t>(a.k) |
                                      reinterpret_cast<uintptr_t>(a.k_out)) |
                                     (unsigned long long)es * ((unsigned long long)(a.interleaved ? 2 * P : P) | (unsigned)a.D | (unsigned long long)a.q_b |
                                                              (unsigned long long)a.q_t | (unsigned long long)(a.k ? a.k_b | a.k_t : 0));
    const unsigned v = (bytes % 16 == 0 ? 16 : bytes % 8 == 0 ? 8 : bytes % 4 == 0 ? 4 : 2) / es;
    if (a.interleaved && v == 1)  // rows of no alignment: pairs of single loads
        return a.dtype == VMB_BF16 ? launch_v<__nv_bfloat16, 2, true>(a, stream) : launch_v<float, 2, true>(a, stream);
    if (a.dtype == VMB_BF16)
        return v == 8 ? launch_v<__nv_bfloat16, 8>(a, stream) : v == 4 ? launch_v<__nv_bfloat16, 4>(a, stream)
             : v == 2 ? launch_v<__nv_bfloat16, 2>(a, stream) : launch_v<__nv_bfloat16, 1>(a, stream);
    return v == 4 ? launch_v<float, 4>(a, stream) : v == 2 ? launch_v<float, 2>(a, stream) : launch_v<float, 1>(a, stream);
}

}  // namespace vmb
