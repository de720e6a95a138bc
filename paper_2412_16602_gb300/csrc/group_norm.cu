// group_norm.cu - group norm with an activation, channels last: forward and gradients.
//
//   n = (x - mean) / sqrt(var + eps) over the pixels and the C / G channels of a group, y = act(w n + b).
//   dz = dy act'(w n + b);  dweight = sum dz n, dbias = sum dz (over batch and pixels);
//   dx = rstd (w dz - mean(w dz) - n mean(w dz n)), the means over the group.
//
// Two passes each way, both in the same tiles (a run of pixels of one sample, all channels): the first leaves a
// tile's sums per channel, and the last tile of a sample to finish joins them; the second applies them.  What
// bounds both is memory: x (and dy) read, y (dx) written.  The second pass finds x in the L2 cache, because a
// launch covers only as many samples as its share of the cache holds.
//
// Variances are formed from sums of differences to the tile's first pixel and joined as (mean, M2) pairs
// (Chan, Golub & LeVeque 1979), so a mean far from zero costs no digits.  All sums are fp32 in a fixed order.
#include "mixer_internal.h"
#include "vmb_common.cuh"
#include "vmb_internal.h"

namespace vmb {

namespace {

constexpr int kNormThreads = 256;
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

template <int ACT> __device__ __forceinline__ float act_value(float z) {
    if (ACT == VMB_ACT_SILU) return z * rcp(1.0f + ex2(-z * kLog2e));
    if (ACT == VMB_ACT_GELU) return z * 0.5f * (1.0f + erff(z * 0.70710678118654752f));
    return z;
}
template <int ACT> __device__ __forceinline__ float act_slope(float z) {
    if (ACT == VMB_ACT_SILU) {
        const float s = rcp(1.0f + ex2(-z * kLog2e));
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    if (ACT == VMB_ACT_GELU)
        return fmaf(z * 0.39894228040143268f, expf(-0.5f * z * z), 0.5f * (1.0f + erff(z * 0.70710678118654752f)));
    return 1.0f;
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
        float s1[V] = {}, s2[V] = {}, pivot[V];
        int n = 0;
        if (rl < lanes && rl < rows) {
            const T* p = x + (long long)(col0 + col) * V;
            const NPack<T, V> f = *reinterpret_cast<const NPack<T, V>*>(p + (long long)rl * C);
#pragma unroll
            for (int i = 0; i < V; ++i) pivot[i] = io<T>::cvt(f.v[i]);
            n = (rows - rl + lanes - 1) / lanes;
#pragma unroll 4
            for (int r = rl; r < rows; r += lanes) {
                const NPack<T, V> f = *reinterpret_cast<const NPack<T, V>*>(p + (long long)r * C);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = io<T>::cvt(f.v[i]) - pivot[i];
                    s1[i] += d;
                    s2[i] = fmaf(d, d, s2[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float m = s1[i] / n;
                scratch[(tid * V + i) * 2] = pivot[i] + m;
                scratch[(tid * V + i) * 2 + 1] = fmaf(-m, s1[i], s2[i]);
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
        float mean[V], rstd[V], wt[V], bs[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float2 s = __ldcg(&st[(ch + i) / m]);
            mean[i] = s.x;
            rstd[i] = s.y;
            wt[i] = a.weight ? a.weight[ch + i] : 1.0f;
            bs[i] = a.bias ? a.bias[ch + i] : 0.0f;
        }
#pragma unroll 4
        for (int r = rl; r < rows; r += lanes) {
            const NPack<T, V> f = *reinterpret_cast<const NPack<T, V>*>(x + (long long)r * C + ch);
            NPack<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i)
                o.v[i] = io<T>::to(act_value<ACT>(fmaf((io<T>::cvt(f.v[i]) - mean[i]) * rstd[i], wt[i], bs[i])));
            *reinterpret_cast<NPack<T, V>*>(y + (long long)r * C + ch) = o;
        }
    }
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
        float s1[V] = {}, s2[V] = {};
        if (rl < lanes) {
            float mean[V], rstd[V], wt[V], bs[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 s = st[(ch + i) / m];
                mean[i] = s.x;
                rstd[i] = s.y;
                wt[i] = a.weight ? a.weight[ch + i] : 1.0f;
                bs[i] = a.bias ? a.bias[ch + i] : 0.0f;
            }
#pragma unroll 2
            for (int r = rl; r < rows; r += lanes) {
                const NPack<T, V> f = *reinterpret_cast<const NPack<T, V>*>(x + (long long)r * C + ch);
                const NPack<T, V> d = *reinterpret_cast<const NPack<T, V>*>(dy + (long long)r * C + ch);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float n = (io<T>::cvt(f.v[i]) - mean[i]) * rstd[i];
                    const float dz = io<T>::cvt(d.v[i]) * act_slope<ACT>(fmaf(n, wt[i], bs[i]));
                    s1[i] += dz;
                    s2[i] = fmaf(dz, n, s2[i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) scratch[(tid * V + i) * 2] = s1[i], scratch[(tid * V + i) * 2 + 1] = s2[i];
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
#pragma unroll 4
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
#pragma unroll 4
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
        float mean[V], rstd[V], wt[V], bs[V], m1[V], m2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float2 s = st[(ch + i) / m], q = __ldcg(&mn[(ch + i) / m]);
            mean[i] = s.x;
            rstd[i] = s.y;
            m1[i] = q.x;
            m2[i] = q.y;
            wt[i] = a.weight ? a.weight[ch + i] : 1.0f;
            bs[i] = a.bias ? a.bias[ch + i] : 0.0f;
        }
#pragma unroll 2
        for (int r = rl; r < rows; r += lanes) {
            const NPack<T, V> f = *reinterpret_cast<const NPack<T, V>*>(x + (long long)r * C + ch);
            const NPack<T, V> d = *reinterpret_cast<const NPack<T, V>*>(dy + (long long)r * C + ch);
            NPack<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float n = (io<T>::cvt(f.v[i]) - mean[i]) * rstd[i];
                const float dz = io<T>::cvt(d.v[i]) * act_slope<ACT>(fmaf(n, wt[i], bs[i]));
                o.v[i] = io<T>::to(rstd[i] * (fmaf(wt[i], dz, -m1[i]) - n * m2[i]));
            }
            *reinterpret_cast<NPack<T, V>*>(dx + (long long)r * C + ch) = o;
        }
    }
}

template <typename T, int V, int ACT>
vmb_status run_norm(const NormArgs& a, bool grads, cudaStream_t stream) {
    NormLaunch c{a, plan_norm(a.B, a.L, a.C, a.G, a.dtype, grads, device_sm_count()), 0};
    if (a.ws_bytes < c.p.total) return VMB_ERR_WORKSPACE;
    const void* one = grads ? (const void*)norm_sums_kernel<T, V, ACT> : (const void*)norm_stats_kernel<T, V>;
    const void* two = grads ? (const void*)norm_dx_kernel<T, V, ACT> : (const void*)norm_apply_kernel<T, V, ACT>;
    const size_t smem = grads ? 0 : (size_t)a.C * 8 + kNormThreads * V * 8;
    if (smem > 48 * 1024 && cudaFuncSetAttribute(one, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
        return VMB_ERR_CUDA;
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
