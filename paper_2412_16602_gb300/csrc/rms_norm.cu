// rms_norm.cu - root-mean-square norm of rows of channels with the residual's addition, an output in the storage type or in 8
// bits with a scale for each row, and its gradients.
//
//   s = x + residual (rounded to the storage type: the residual stream that goes on),  r = 1 / sqrt(mean(s^2) + eps),
//   y = s r w;   in 8 bits: y / scale with scale = max |y| / 448 of the row (448: the largest e4m3 value).
//   dx = r (w dy - n mean(w dy n)) + dsum, n = s r (the residual's gradient is the same),  dw = sum over rows of dy n.
//
// Bound by memory: each value is read once and held in registers between the sums and the output.  In the forward a row
// belongs to one warp where 32 values a thread hold it, so that its sums need no barrier (16384 x 1536 in bf16 with the residual's addition: 31 us in two warps
// of 24 values a thread, in one of 48 36 us); in the gradients, which hold six values for each and the next row's, to as many threads as hold it in
// two or three vectors (16384 x 1536: 82 us in bf16, 27% of the copy rate: few rows are on their way; 74 in fp32).  8 bits, residual added, with 64 registers a thread:
// 42 us in bf16 (63% of the copy rate), 12288 x 2048 50, 6144 x 4096 50, 3000 x 8192 51; without that limit 43, 50, 50 and 61.  In fp32 the limit costs
// spills where a thread holds eight vectors: 49, 59, 59 and 60 us, without it 49, 49, 49 and 50.
#include <cuda_fp8.h>

#include <initializer_list>

#include "layer_common.cuh"
#include "layer_internal.h"
#include "vmb_internal.h"

namespace vmb {

namespace {

constexpr int kRmsBlock = 128;
constexpr float kLeastScale = 7.888609052210118e-31f;  // 2^-100: rows of zeros keep a scale that can be divided by


struct RmsKernel {
    RmsArgs a;
    int lanes, rows_per;  // threads of a row, rows of a block
    float* partial;       // gradients: [blocks x rows_per][C]
};

// The sum (or maximum) over the threads of a row, the same in all of them.
template <bool kMax> __device__ __forceinline__ float row_join(float v, int lanes, float* scratch) {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const float o = __shfl_xor_sync(0xffffffffu, v, d);
        v = kMax ? fmaxf(v, o) : v + o;
    }
    if (lanes > 32) {
        const int w = threadIdx.x >> 5, n = lanes >> 5, first = w / n * n;
        __syncthreads();  // the scratch of an earlier sum has been read
        if ((threadIdx.x & 31) == 0) scratch[w] = v;
        __syncthreads();
        v = scratch[first];
        for (int i = 1; i < n; ++i) v = kMax ? fmaxf(v, scratch[first + i]) : v + scratch[first + i];
    }
    return v;
}

// v / d with inv = 1 / d rounded: the product with inv, corrected by the remainder, which is the quotient rounded once (a product alone is off by
// up to two roundings, and one value in 6 million got the other of two neighbouring 8-bit values).  For an infinite d both d and inv are 0.
__device__ __forceinline__ float quotient(float v, float d, float inv) {
    const float q = v * inv;
    return fmaf(fmaf(-q, d, v), inv, q);
}

// 8-bit values of V floats, rounded to nearest even, beyond 448 (by a rounding of the division) to 448.
template <int V> __device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = (uint8_t)__nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
    } else {
        Vec<uint16_t, V / 2> o;
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
            o.v[i] = (uint16_t)__nv_cvt_float2_to_fp8x2(make_float2(v[2 * i], v[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        *reinterpret_cast<Vec<uint16_t, V / 2>*>(p) = o;
    }
}

template <typename T, int V, int NV, bool kBits8> __global__ void __launch_bounds__(512, kBits8 ? 2 : 1) rms_fwd_kernel(RmsKernel k) {
    __shared__ float scratch[32];
    const RmsArgs& a = k.a;
    pdl_wait();
    pdl_launch_dependents();
    const int lx = threadIdx.x % k.lanes;
    const long long row = (long long)blockIdx.x * k.rows_per + threadIdx.x / k.lanes;
    const bool live = row < a.rows;
    const T *x = (const T*)a.x + row * a.C, *res = (const T*)a.residual + row * a.C;
    float s[NV][V];
    float ss = 0.0f;
    Vec<T, V> rx[NV], rr[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (lx + j * k.lanes) * V;
        rx[j] = rr[j] = Vec<T, V>{};
        if (live && c < a.C) {
            rx[j] = *reinterpret_cast<const Vec<T, V>*>(x + c);
            if (a.residual) rr[j] = *reinterpret_cast<const Vec<T, V>*>(res + c);
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[j][i] = io<T>::cvt(rx[j].v[i]);
            if (a.residual) s[j][i] = io<T>::cvt(io<T>::to(s[j][i] + io<T>::cvt(rr[j].v[i])));
        }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (lx + j * k.lanes) * V;
        if (a.residual && live && c < a.C) store_vec<T, V>((T*)a.sum + row * a.C + c, s[j]);
#pragma unroll
        for (int i = 0; i < V; ++i) ss = fmaf(s[j][i], s[j][i], ss);
    }
    ss = row_join<false>(ss, k.lanes, scratch);
    const float rstd = 1.0f / sqrtf(ss / (float)a.C + a.eps);
    if (a.rstd && live && lx == 0) a.rstd[row] = rstd;
    float most = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (lx + j * k.lanes) * V;
        if (!live || c >= a.C) continue;
        float w[V];
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = 1.0f;
        if (a.weight) load_vec<float, V>(w, a.weight + c);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[j][i] = s[j][i] * rstd * w[i];
            most = fmaxf(most, fabsf(s[j][i]));
        }
        if constexpr (!kBits8) store_vec<T, V>((T*)a.y + row * a.C + c, s[j]);
    }
    if constexpr (kBits8) {
        most = row_join<true>(most, k.lanes, scratch);
        const float scale = fmaxf(most / 448.0f, kLeastScale), inv = 1.0f / scale, over = inv > 0.0f ? scale : 0.0f;
        if (live && lx == 0) a.scale[row] = scale;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (lx + j * k.lanes) * V;
            if (!live || c >= a.C) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] = quotient(s[j][i], over, inv);
            store_e4m3<V>((uint8_t*)a.y + row * a.C + c, s[j]);
        }
    }
}

// Gradients: a block takes rows in turn and keeps its sums of dw in registers, one row of partial sums at its end.
template <typename T, int V, int NV> __global__ void __launch_bounds__(512) rms_bwd_kernel(RmsKernel k) {
    __shared__ float scratch[32];
    const RmsArgs& a = k.a;
    pdl_wait();
    pdl_launch_dependents();
    const int lx = threadIdx.x % k.lanes, ly = threadIdx.x / k.lanes;
    float dw[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) dw[j][i] = 0.0f;
    const long long step = (long long)gridDim.x * k.rows_per;
    Vec<T, V> rx[NV], rd[NV], rg[NV];
    float next = 0.0f;  // rstd of the row under way
    auto load = [&](long long row) {
        const bool live = row < a.rows;
        next = live ? a.rstd[row] : 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (lx + j * k.lanes) * V;
            rx[j] = rd[j] = rg[j] = Vec<T, V>{};
            if (live && c < a.C) {
                rx[j] = *reinterpret_cast<const Vec<T, V>*>((const T*)a.x + row * a.C + c);
                rd[j] = *reinterpret_cast<const Vec<T, V>*>((const T*)a.dy + row * a.C + c);
                if (a.dsum) rg[j] = *reinterpret_cast<const Vec<T, V>*>((const T*)a.dsum + row * a.C + c);
            }
        }
    };
    load((long long)blockIdx.x * k.rows_per + ly);
    for (long long r0 = (long long)blockIdx.x * k.rows_per; r0 < a.rows; r0 += step) {
        const long long row = r0 + ly;
        const bool live = row < a.rows;
        const float rstd = next;
        float n[NV][V], d[NV][V], dot = 0.0f;
        Vec<T, V> more[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (lx + j * k.lanes) * V;
            more[j] = rg[j];
            float w[V];
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = 1.0f;
            if (a.weight && c < a.C) load_vec<float, V>(w, a.weight + c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                n[j][i] = io<T>::cvt(rx[j].v[i]) * rstd;
                d[j][i] = io<T>::cvt(rd[j].v[i]);
                dw[j][i] = fmaf(d[j][i], n[j][i], dw[j][i]);
                d[j][i] *= w[i];
                dot = fmaf(d[j][i], n[j][i], dot);
            }
        }
        load(row + step);  // under way while this row's sum is joined
        dot = row_join<false>(dot, k.lanes, scratch) / (float)a.C;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (lx + j * k.lanes) * V;
            if (!live || c >= a.C) continue;
            float g[V];
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = fmaf(rstd, fmaf(-n[j][i], dot, d[j][i]), io<T>::cvt(more[j].v[i]));
            store_vec<T, V>((T*)a.dx + row * a.C + c, g);
        }
    }
    if (!k.partial) return;
    float* p = k.partial + ((long long)blockIdx.x * k.rows_per + ly) * a.C;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (lx + j * k.lanes) * V;
        if (c >= a.C) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) p[c + i] = dw[j][i];
    }
}

// Vectors that a thread may hold of a row, and the threads of a row: a power of two of warps.
// (8192 channels in 512 threads are two vectors of eight, four of four or sixteen single channels each.)
constexpr int kFwdMost = 4;
int rms_most(int V, bool grads) { return V == 1 ? 16 : !grads ? (V == 8 ? kFwdMost : 8) : V == 8 ? 2 : 3; }
int rms_lanes(int C, int V, bool grads) {
    int lanes = 32;
    while (lanes < 512 && lanes * V * rms_most(V, grads) < C) lanes *= 2;
    return lanes;
}
// Vectors that a thread does hold: of these a kernel is made for each of a few numbers.
int rms_vecs(int C, int V, int lanes) { return ((C + V - 1) / V + lanes - 1) / lanes; }
template <typename T, int V, bool kBits8> const void* rms_fwd_fn(int nv) {
    if constexpr (V == 1) return (const void*)rms_fwd_kernel<T, 1, 16, kBits8>;
    else if constexpr (V == 8)  // (no more than kFwdMost)
        return nv <= 1   ? (const void*)rms_fwd_kernel<T, V, 1, kBits8>
               : nv <= 2 ? (const void*)rms_fwd_kernel<T, V, 2, kBits8>
               : nv <= 3 ? (const void*)rms_fwd_kernel<T, V, 3, kBits8>
                         : (const void*)rms_fwd_kernel<T, V, 4, kBits8>;
    else
        return nv <= 1   ? (const void*)rms_fwd_kernel<T, V, 1, kBits8>
               : nv <= 2 ? (const void*)rms_fwd_kernel<T, V, 2, kBits8>
               : nv <= 3 ? (const void*)rms_fwd_kernel<T, V, 3, kBits8>
               : nv <= 4 ? (const void*)rms_fwd_kernel<T, V, 4, kBits8>
               : nv <= 6 ? (const void*)rms_fwd_kernel<T, V, 6, kBits8>
                         : (const void*)rms_fwd_kernel<T, V, 8, kBits8>;
}
template <typename T, int V> const void* rms_bwd_fn(int nv) {
    if constexpr (V == 1) return (const void*)rms_bwd_kernel<T, 1, 16>;
    else if constexpr (V == 8) return nv <= 1 ? (const void*)rms_bwd_kernel<T, V, 1> : (const void*)rms_bwd_kernel<T, V, 2>;
    else
        return nv <= 1   ? (const void*)rms_bwd_kernel<T, V, 1>
               : nv <= 2 ? (const void*)rms_bwd_kernel<T, V, 2>
               : nv <= 3 ? (const void*)rms_bwd_kernel<T, V, 3>
                         : (const void*)rms_bwd_kernel<T, V, 4>;
}
int rms_width(vmb_dtype dt) { return dt == VMB_BF16 ? 8 : 4; }

bool rms_vectors(const RmsArgs& a) {
    if (a.C % rms_width(a.dtype)) return false;
    for (const void* p : {a.x, a.residual, (const void*)a.y, (const void*)a.sum, a.dy, a.dsum, (const void*)a.dx, (const void*)a.weight})
        if (reinterpret_cast<uintptr_t>(p) & (p == a.weight && p ? 15 : p == a.y && a.bits8 ? 7 : 15)) return false;
    return true;
}

constexpr int kRmsBlocksPerSm = 6;
long long rms_bwd_blocks(long long rows, int rows_per, int block) {
    long long most = (long long)device_sm_count() * (kRmsBlocksPerSm * kRmsBlock / block > 1 ? kRmsBlocksPerSm * kRmsBlock / block : 1);
    const long long want = (rows + rows_per - 1) / rows_per;
    return want < most ? want : most;
}

void rms_shape(RmsKernel& k, int V, bool grads, int* block) {
    k.lanes = rms_lanes(k.a.C, V, grads);
    *block = k.lanes > kRmsBlock ? k.lanes : kRmsBlock;
    k.rows_per = *block / k.lanes;
}

}  // namespace

size_t rms_workspace_bytes(long long rows, int C, vmb_dtype dtype) {
    size_t most = 0;
    for (int V : {1, rms_width(dtype)}) {
        const int lanes = rms_lanes(C, V, true), block = lanes > kRmsBlock ? lanes : kRmsBlock;
        const size_t n = (size_t)rms_bwd_blocks(rows, block / lanes, block) * (block / lanes) * C * 4;
        if (n > most) most = n;
    }
    return align_up(most, 256) + 256;
}

vmb_status launch_rms_fwd(const RmsArgs& a, cudaStream_t stream) {
    RmsKernel k{a};
    const bool vec = rms_vectors(a);
    const int V = vec ? rms_width(a.dtype) : 1;
    int block;
    rms_shape(k, V, false, &block);
    const int nv = rms_vecs(a.C, V, k.lanes);
    const void* fn;
    if (a.dtype == VMB_BF16)
        fn = a.bits8 ? (vec ? rms_fwd_fn<__nv_bfloat16, 8, true>(nv) : rms_fwd_fn<__nv_bfloat16, 1, true>(nv))
                     : (vec ? rms_fwd_fn<__nv_bfloat16, 8, false>(nv) : rms_fwd_fn<__nv_bfloat16, 1, false>(nv));
    else
        fn = a.bits8 ? (vec ? rms_fwd_fn<float, 4, true>(nv) : rms_fwd_fn<float, 1, true>(nv)) : (vec ? rms_fwd_fn<float, 4, false>(nv) : rms_fwd_fn<float, 1, false>(nv));
    void* args[] = {&k};
    return launch_kernel(fn, dim3((unsigned)((a.rows + k.rows_per - 1) / k.rows_per)), dim3(block), 0, args, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

vmb_status launch_rms_bwd(const RmsArgs& a, cudaStream_t stream) {
    RmsKernel k{a};
    const bool vec = rms_vectors(a);
    const int V = vec ? rms_width(a.dtype) : 1;
    int block;
    rms_shape(k, V, true, &block);
    const int nv = rms_vecs(a.C, V, k.lanes);
    const long long blocks = rms_bwd_blocks(a.rows, k.rows_per, block);
    const long long parts = blocks * k.rows_per;
    k.partial = nullptr;
    if (a.dweight) {
        if (a.ws_bytes < (size_t)parts * a.C * 4 + 256) return VMB_ERR_WORKSPACE;
        k.partial = (float*)((char*)a.ws + 256);
    }
    const void* fn = a.dtype == VMB_BF16 ? (vec ? rms_bwd_fn<__nv_bfloat16, 8>(nv) : rms_bwd_fn<__nv_bfloat16, 1>(nv))
                                         : (vec ? rms_bwd_fn<float, 4>(nv) : rms_bwd_fn<float, 1>(nv));
    void* args[] = {&k};
    if (launch_kernel(fn, dim3((unsigned)blocks), dim3(block), 0, args, stream) != cudaSuccess) return VMB_ERR_CUDA;
    return a.dweight ? launch_column_sums(k.partial, (int)parts, a.C, a.C, 1, a.dweight, nullptr, 0, nullptr, stream) : VMB_OK;
}

}  // namespace vmb
