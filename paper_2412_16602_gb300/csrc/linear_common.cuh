// linear_common.cuh - what the kernels of the matrix product share: operands with any strides, and the epilogue.
#pragma once

#include "layer_common.cuh"
#include "layer_internal.h"
#include "vmb_internal.h"

namespace vmb {

// What a product out [M][N] = A [M][K] B [N][K]^T does with its sums:
//   z = sum row_scale[m] col_scale[n] + bias[n],  pre = z,  out = act(z) + residual.
struct GemmEpilogue {
    const float *row_scale, *col_scale, *bias;  // null: 1, 1, 0
    const __nv_bfloat16* residual;              // null: 0; rows of N
    __nv_bfloat16 *out, *pre;                   // rows of N; pre may be null
    int act;
};

struct GemmProblem {
    const void *A, *B;
    long long M;
    int N;
    long long K;
    long long a_r, a_c, b_r, b_c;  // elements between rows and between the contraction's steps of A and of B
    GemmEpilogue e;
};

__device__ __forceinline__ float act_of(float z, int act) {
    return act == VMB_ACT_SILU ? activate<VMB_ACT_SILU>(z) : act == VMB_ACT_GELU ? activate<VMB_ACT_GELU>(z) : z;
}
__device__ __forceinline__ float slope_of(float z, int act) {
    return act == VMB_ACT_SILU ? activate_slope<VMB_ACT_SILU>(z) : act == VMB_ACT_GELU ? activate_slope<VMB_ACT_GELU>(z) : 1.0f;
}
// The factors and the bias of V columns from n on.
template <int V> struct ColumnTerms {
    float scale[V], bias[V];
    __device__ __forceinline__ void load(const GemmEpilogue& e, int n) {
        const auto take = [n](float (&v)[V], const float* p, float other) {
            if (p && V == 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
                const float4 a = *reinterpret_cast<const float4*>(p + n), b = *reinterpret_cast<const float4*>(p + n + V / 2);
                const float all[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = all[i];
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = p ? p[n + i] : other;
            }
        };
        take(scale, e.col_scale, 1.0f);
        take(bias, e.bias, 0.0f);
    }
};

template <int ACT> __device__ __forceinline__ void activate_all(float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const float2 y = activate2<ACT>(make_float2(v[i], v[i + 1]));
        v[i] = y.x, v[i + 1] = y.y;
    }
}
template <int ACT> __device__ __forceinline__ void activate_all(float (&v)[1]) { v[0] = activate<ACT>(v[0]); }

// The sums of V columns of a row (8: in range, 16-byte aligned): the output is at `at`; `residual` holds the residual's values there.
template <int V>
__device__ __forceinline__ void finish(const GemmEpilogue& e, float (&v)[V], const ColumnTerms<V>& t, float row_scale, const Vec<__nv_bfloat16, V>& residual, long long at) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = e.row_scale ? fmaf(v[i], row_scale * t.scale[i], t.bias[i]) : v[i] + t.bias[i];
    if (e.pre) store_vec<__nv_bfloat16, V>(e.pre + at, v);
    if (e.act == VMB_ACT_SILU) activate_all<VMB_ACT_SILU>(v);
    else if (e.act == VMB_ACT_GELU) activate_all<VMB_ACT_GELU>(v);
    if (e.residual) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += __bfloat162float(residual.v[i]);
    }
    store_vec<__nv_bfloat16, V>(e.out + at, v);
}
template <int V> __device__ __forceinline__ Vec<__nv_bfloat16, V> residual_at(const GemmEpilogue& e, long long at) {
    return e.residual ? *reinterpret_cast<const Vec<__nv_bfloat16, V>*>(e.residual + at) : Vec<__nv_bfloat16, V>{};
}
// Rows of vectors of eight bf16: out, pre and residual may be read and written in 16 bytes.
inline bool epilogue_vectors(const GemmProblem& p) {
    return p.N % 8 == 0 &&
           ((reinterpret_cast<uintptr_t>(p.e.out) | reinterpret_cast<uintptr_t>(p.e.pre) | reinterpret_cast<uintptr_t>(p.e.residual)) & 15) == 0;
}

// bf16 operands, or e4m3.  Any strides and sizes (linear.cu):
vmb_status launch_gemm_any(const GemmProblem& p, bool bits8, cudaStream_t stream);
// Operands that tensor copies can read: one stride is 1, the other a multiple of 16 bytes, as is the base (linear_tc.cu).  *taken is false where
// they are not, and nothing was launched.  `partial`: what gemm_partial_bytes says, of this problem.
vmb_status launch_gemm_tc(const GemmProblem& p, bool bits8, float* partial, unsigned* err, cudaStream_t stream, bool* taken);
// Up to 32 rows of A, contractions dense in whole vectors of 16 bytes (linear_few.cu); *taken as above.
vmb_status launch_gemm_few(const GemmProblem& p, bool bits8, cudaStream_t stream, bool* taken);
size_t gemm_partial_bytes(long long M, int N, long long K, bool bits8);

}  // namespace vmb
