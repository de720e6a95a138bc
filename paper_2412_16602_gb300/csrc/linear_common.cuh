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

// bf16 operands, or e4m3.  Any strides and sizes (linear.cu); rows that tensor copies can read (linear_tc.cu).
vmb_status launch_gemm_any(const GemmProblem& p, bool bits8, cudaStream_t stream);

}  // namespace vmb
