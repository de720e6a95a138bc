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
template <int ACT, int V> __device__ __forceinline__ void activate_all(float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = activate<ACT>(v[i]);
}

// V sums of row m from column n on, all in range and 16-byte aligned (V 8) or one.
template <int V> __device__ __forceinline__ void finish(const GemmEpilogue& e, float (&v)[V], const float (&scale)[V], const float (&bias)[V], float row_scale,
                                                        long long at) {
    if (e.row_scale) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = v[i] * (row_scale * scale[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += bias[i];
    if (e.pre) store_vec<__nv_bfloat16, V>(e.pre + at, v);
    if (e.act == VMB_ACT_SILU) activate_all<VMB_ACT_SILU, V>(v);
    else if (e.act == VMB_ACT_GELU) activate_all<VMB_ACT_GELU, V>(v);
    if (e.residual) {
        float r[V];
        load_vec<__nv_bfloat16, V>(r, e.residual + at);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += r[i];
    }
    store_vec<__nv_bfloat16, V>(e.out + at, v);
}
template <int V> __device__ __forceinline__ void column_terms(const GemmEpilogue& e, int n, float (&scale)[V], float (&bias)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        scale[i] = e.col_scale ? e.col_scale[n + i] : 1.0f;
        bias[i] = e.bias ? e.bias[n + i] : 0.0f;
    }
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
size_t gemm_partial_bytes(long long M, int N, long long K, bool bits8);

}  // namespace vmb
