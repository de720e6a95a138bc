// linear_few.cu - the matrix product of a few rows (up to 32), where every weight is read once and that is what bounds it.
//
// A CTA takes 16 columns and cuts the contraction among its eight warps.  A lane reads 16 bytes of a row of the weights and 16 of a row of x, both
// at the same place in the contraction: which of its values meet in which product of a step is free as long as both sides agree,
// so the fragments of mma.sync are whole vectors from global memory and nothing passes through shared memory but the warps' sums,
// which are joined in order.  e4m3 values are widened to f16, which holds them exactly.
// 1 x 2048 x 4096 in bf16, 16.8 MB: 6.8 us (through tiles of 128 rows on the tensor cores 10.3), 32 rows 9.3; eight steps ahead instead of four 7.2.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "linear_common.cuh"

namespace vmb {

namespace {

constexpr int kFewWarps = 8, kFewCols = 16;

template <bool kHalf> __device__ __forceinline__ void few_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (kHalf)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes as pairs of 16-bit values: of bf16 as they are, of e4m3 widened.
template <bool kBits8> __device__ __forceinline__ void few_pairs(uint32_t (&out)[kBits8 ? 8 : 4], const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kBits8) {
            const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i] & 0xffff), __NV_E4M3);
            const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i] >> 16), __NV_E4M3);
            out[2 * i] = lo.x | (uint32_t)lo.y << 16;
            out[2 * i + 1] = hi.x | (uint32_t)hi.y << 16;
        } else {
            out[i] = w[i];
        }
    }
}

// MT: tiles of 16 rows of x.
template <bool kBits8, int MT> __global__ void __launch_bounds__(32 * kFewWarps) gemm_few_kernel(GemmProblem p) {
    constexpr int kElem = kBits8 ? 1 : 2, kStep = 64 / kElem, kPairs = kBits8 ? 8 : 4, kAhead = 4;  // a step: four lanes' 16 bytes of the contraction
    __shared__ float sums[kFewWarps][MT * 16][kFewCols + 1];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, n0 = blockIdx.x * kFewCols;
    const int steps = (int)((p.K + kStep - 1) / kStep), per = (steps + kFewWarps - 1) / kFewWarps, s0 = w * per, s1 = min(steps, s0 + per);
    const char *A = (const char*)p.A, *B = (const char*)p.B;
    float acc[MT][2][4] = {};
    for (int s = s0; s < s1; s += kAhead) {
        uint4 a[kAhead][MT][2], b[kAhead][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const long long k = (long long)(s + i) * kStep + t * (16 / kElem);
            const bool in = s + i < s1 && k < p.K;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                b[i][c] = make_uint4(0, 0, 0, 0);
                if (in && n0 + c * 8 + g < p.N) b[i][c] = *reinterpret_cast<const uint4*>(B + ((n0 + c * 8 + g) * p.b_r + k) * kElem);
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    a[i][m][r] = make_uint4(0, 0, 0, 0);
                    if (in && m * 16 + r * 8 + g < p.M) a[i][m][r] = *reinterpret_cast<const uint4*>(A + ((m * 16 + r * 8 + g) * p.a_r + k) * kElem);
                }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            uint32_t pb[2][kPairs];
            few_pairs<kBits8>(pb[0], b[i][0]);
            few_pairs<kBits8>(pb[1], b[i][1]);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                uint32_t pa[2][kPairs];
                few_pairs<kBits8>(pa[0], a[i][m][0]);
                few_pairs<kBits8>(pa[1], a[i][m][1]);
#pragma unroll
                for (int q = 0; q < kPairs; q += 2)
#pragma unroll
                    for (int c = 0; c < 2; ++c) few_mma<kBits8>(acc[m][c], pa[0][q], pa[1][q], pa[0][q + 1], pa[1][q + 1], pb[c][q], pb[c][q + 1]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[w][m * 16 + g + (i >> 1) * 8][c * 8 + t * 2 + (i & 1)] = acc[m][c][i];
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int row = m * 16 + (threadIdx.x >> 4), col = threadIdx.x & 15, n = n0 + col;
        if (row >= p.M || n >= p.N) continue;
        float v[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < kFewWarps; ++i) v[0] += sums[i][row][col];
        ColumnTerms<1> terms;
        terms.load(p.e, n);
        const long long at = (long long)row * p.N + n;
        finish<1>(p.e, v, terms, p.e.row_scale ? p.e.row_scale[row] : 1.0f, residual_at<1>(p.e, at), at);
    }
}

}  // namespace

vmb_status launch_gemm_few(const GemmProblem& p0, bool bits8, cudaStream_t stream, bool* taken) {
    GemmProblem p = p0;
    const long long es = bits8 ? 1 : 2;
    *taken = p.M <= 32 && p.K > 0 && p.a_c == 1 && p.b_c == 1 && p.K * es % 16 == 0 && p.a_r * es % 16 == 0 && p.b_r * es % 16 == 0 &&
             ((reinterpret_cast<uintptr_t>(p.A) | reinterpret_cast<uintptr_t>(p.B)) & 15) == 0;
    if (!*taken) return VMB_OK;
    void* args[] = {&p};
    const void* fn = p.M <= 16 ? (bits8 ? (const void*)gemm_few_kernel<true, 1> : (const void*)gemm_few_kernel<false, 1>)
                               : (bits8 ? (const void*)gemm_few_kernel<true, 2> : (const void*)gemm_few_kernel<false, 2>);
    return launch_kernel(fn, dim3((unsigned)((p.N + kFewCols - 1) / kFewCols)), dim3(32 * kFewWarps), 0, args, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

}  // namespace vmb
