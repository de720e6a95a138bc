// linear.cu - the matrix product of a projection with bias, activation and residual in its epilogue, and its gradients.
//
//   z = x W^T + bias, y = act(z) + residual;   dZ = dy act'(z) (bf16),  dx = dZ W,  dW = dZ^T x,  dbias = sum over rows of dZ.
//
// linear_tc.cu has the products of many rows, linear_few.cu those of few; here are dZ with the sums of its columns (bound by memory; 8192 x 4096
// with SiLU 32 us; with GELU 66, by erfcf in its slope) and, for what tensor copies cannot read:
// gemm_any_kernel takes operands of any strides: those that tensor copies cannot read (rows that do not start on 16 bytes), element by element
// through shared memory, which bounds it: 4096 x 1023 x 4096 952 us (36 TFLOP/s), 16 x 1001 x 1024 152 us.
#include <cuda_fp8.h>

#include "linear_common.cuh"

namespace vmb {

namespace {

constexpr int kAnyTile = 64, kAnyK = 32, kAnyThreads = 128, kAnyPitch = kAnyK + 8;

__device__ __forceinline__ __nv_bfloat16 operand(const __nv_bfloat16* p) { return *p; }
// (e4m3 values are exact in bf16)
__device__ __forceinline__ __nv_bfloat16 operand(const __nv_fp8_e4m3* p) { return __float2bfloat16_rn((float)*p); }

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// A CTA takes 64 x 64 outputs, a warp 32 x 32 of them; operands pass element by element through shared memory.
template <typename T> __global__ void __launch_bounds__(kAnyThreads) gemm_any_kernel(GemmProblem p, int tiles_n) {
    __shared__ __align__(16) __nv_bfloat16 sa[kAnyTile * kAnyPitch], sb[kAnyTile * kAnyPitch];
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, wm = (w >> 1) * 32, wn = (w & 1) * 32;
    const long long m0 = (long long)(blockIdx.x / tiles_n) * kAnyTile;
    const int n0 = (int)(blockIdx.x % tiles_n) * kAnyTile;
    const T *A = (const T*)p.A, *B = (const T*)p.B;
    float acc[2][4][4] = {};
    for (long long k0 = 0; k0 < p.K; k0 += kAnyK) {
        for (int i = tid; i < kAnyTile * kAnyK; i += kAnyThreads) {
            // neighbouring threads along whichever axis is dense
            const int ar = p.a_c == 1 ? i / kAnyK : i % kAnyTile, ac = p.a_c == 1 ? i % kAnyK : i / kAnyTile;
            const int br = p.b_c == 1 ? i / kAnyK : i % kAnyTile, bc = p.b_c == 1 ? i % kAnyK : i / kAnyTile;
            sa[ar * kAnyPitch + ac] = m0 + ar < p.M && k0 + ac < p.K ? operand(A + (m0 + ar) * p.a_r + (k0 + ac) * p.a_c) : __nv_bfloat16(0.0f);
            sb[br * kAnyPitch + bc] = n0 + br < p.N && k0 + bc < p.K ? operand(B + (n0 + br) * p.b_r + (k0 + bc) * p.b_c) : __nv_bfloat16(0.0f);
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kAnyK; kk += 16) {
            uint32_t a[2][4], b[4][2];
            const int g = lane >> 2, t = (lane & 3) * 2;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    a[i][q] = *reinterpret_cast<const uint32_t*>(sa + (wm + i * 16 + g + (q & 1) * 8) * kAnyPitch + kk + t + (q >> 1) * 8);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int q = 0; q < 2; ++q) b[j][q] = *reinterpret_cast<const uint32_t*>(sb + (wn + j * 8 + g) * kAnyPitch + kk + t + q * 8);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) mma_bf16(acc[i][j], a[i], b[j]);
        }
        __syncthreads();
    }
    const GemmEpilogue& e = p.e;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const long long m = m0 + wm + i * 16 + (lane >> 2) + (q >> 1) * 8;
                const int n = n0 + wn + j * 8 + (lane & 3) * 2 + (q & 1);
                if (m >= p.M || n >= p.N) continue;
                float z = acc[i][j][q];
                if (e.row_scale) z = z * e.row_scale[m] * e.col_scale[n];
                if (e.bias) z += e.bias[n];
                const long long at = m * p.N + n;
                if (e.pre) e.pre[at] = __float2bfloat16_rn(z);
                z = act_of(z, e.act);
                if (e.residual) z += __bfloat162float(e.residual[at]);
                e.out[at] = __float2bfloat16_rn(z);
            }
}

// dZ = dy act'(pre) and, per block row, the sums of its columns before the rounding.  Vectors of V columns a thread, the rows of a
// block in turn over eight warps.
constexpr int kDzRows = 8;
template <int V> __global__ void __launch_bounds__(32 * kDzRows) linear_dz_kernel(const __nv_bfloat16* dy, const __nv_bfloat16* pre, __nv_bfloat16* dz,
                                                                                  float* partial, long long M, int N, int act) {
    __shared__ float part[kDzRows][32 * V + 1];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * V;
    const bool on = c < N;
    float sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.0f;
    if (on)
        for (long long r = (long long)blockIdx.y * kDzRows + w; r < M; r += (long long)gridDim.y * kDzRows) {
            float g[V], z[V];
            load_vec<__nv_bfloat16, V>(g, dy + r * N + c);
            if (act != VMB_ACT_NONE) {
                load_vec<__nv_bfloat16, V>(z, pre + r * N + c);
#pragma unroll
                for (int i = 0; i < V; ++i) g[i] *= slope_of(z[i], act);
                store_vec<__nv_bfloat16, V>(dz + r * N + c, g);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += g[i];
        }
    if (!partial) return;
#pragma unroll
    for (int i = 0; i < V; ++i) part[w][lane * V + i] = sum[i];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * V; i += 32 * kDzRows) {
        const int col = blockIdx.x * 32 * V + i;
        if (col >= N) continue;
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < kDzRows; ++j) s += part[j][i];
        partial[(long long)blockIdx.y * N + col] = s;
    }
}

struct DzGrid {
    unsigned x, y;
};
DzGrid dz_grid(long long M, int N, int V) {
    DzGrid g;
    g.x = (unsigned)((N + 32 * V - 1) / (32 * V));
    const long long fill = 8LL * device_sm_count() / g.x, rows = (M + 4 * kDzRows - 1) / (4 * kDzRows);
    const long long y = fill < rows ? fill : rows;
    g.y = (unsigned)(y < 1 ? 1 : y);
    return g;
}

struct LinearLayout {
    size_t dz, sums, parts, bytes;  // dZ; partial sums of its columns; parts of split contractions
};
LinearLayout linear_layout(long long M, int K, int N, bool grads) {
    LinearLayout l{256, 256, 256, 256};
    size_t parts;
    if (grads) {
        l.sums = l.dz + align_up((size_t)M * N * 2, 256);
        const size_t rows = dz_grid(M, N, 1).y > dz_grid(M, N, 8).y ? dz_grid(M, N, 1).y : dz_grid(M, N, 8).y;
        l.parts = l.sums + align_up(rows * N * 4, 256);
        const size_t a = K ? gemm_partial_bytes(M, K, N, false) : 0, b = K ? gemm_partial_bytes(N, K, M, false) : 0;
        parts = a > b ? a : b;
    } else {
        const size_t a = gemm_partial_bytes(M, N, K, false), b = gemm_partial_bytes(M, N, K, true);
        parts = a > b ? a : b;
    }
    l.bytes = l.parts + parts;
    return l;
}

vmb_status launch_gemm(const GemmProblem& p, bool bits8, const LinearArgs& a, const LinearLayout& l, cudaStream_t stream) {
    bool taken = false;
    const vmb_status s = launch_gemm_tc(p, bits8, (float*)((char*)a.ws + l.parts), &((WsHeader*)a.ws)->err, stream, &taken);
    return s != VMB_OK || taken ? s : launch_gemm_any(p, bits8, stream);
}

}  // namespace

vmb_status launch_gemm_any(const GemmProblem& p0, bool bits8, cudaStream_t stream) {
    GemmProblem p = p0;
    int tiles_n = (p.N + kAnyTile - 1) / kAnyTile;
    const long long grid = (p.M + kAnyTile - 1) / kAnyTile * tiles_n;
    if (grid > 0x7fffffffLL) return VMB_ERR_UNSUPPORTED;
    if (grid == 0) return VMB_OK;
    void* args[] = {&p, &tiles_n};
    const void* fn = bits8 ? (const void*)gemm_any_kernel<__nv_fp8_e4m3> : (const void*)gemm_any_kernel<__nv_bfloat16>;
    return launch_kernel(fn, dim3((unsigned)grid), dim3(kAnyThreads), 0, args, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

size_t linear_workspace_bytes(long long M, int K, int N, bool grads) { return linear_layout(M, K, N, grads).bytes; }

vmb_status launch_linear_fwd(const LinearArgs& a, cudaStream_t stream) {
    if (a.ws_bytes < 256) return VMB_ERR_WORKSPACE;
    const GemmProblem p{a.x, a.weight, a.M, a.N, a.K, a.x_t, 1, a.K, 1,
                        {a.x_scale, a.weight_scale, a.bias, (const __nv_bfloat16*)a.residual, (__nv_bfloat16*)a.y, (__nv_bfloat16*)a.pre, a.act}};
    bool taken = false;
    const vmb_status s = launch_gemm_few(p, a.x_scale != nullptr, stream, &taken);
    if (s != VMB_OK || taken) return s;
    const LinearLayout l = linear_layout(a.M, a.K, a.N, false);
    return a.ws_bytes < l.bytes ? VMB_ERR_WORKSPACE : launch_gemm(p, a.x_scale != nullptr, a, l, stream);
}

vmb_status launch_linear_bwd(const LinearArgs& a, cudaStream_t stream) {
    const LinearLayout l = linear_layout(a.M, a.K, a.N, true);
    if (a.ws_bytes < l.bytes) return VMB_ERR_WORKSPACE;
    const __nv_bfloat16 *dy = (const __nv_bfloat16*)a.dy, *pre = (const __nv_bfloat16*)a.pre, *dz = dy;
    long long M = a.M;
    int N = a.N, act = a.act;
    if (act != VMB_ACT_NONE || a.dbias) {
        const bool vec = N % 8 == 0 && ((reinterpret_cast<uintptr_t>(dy) | reinterpret_cast<uintptr_t>(pre)) & 15) == 0;
        const DzGrid g = dz_grid(M, N, vec ? 8 : 1);
        __nv_bfloat16* out = (__nv_bfloat16*)((char*)a.ws + l.dz);
        float* partial = a.dbias ? (float*)((char*)a.ws + l.sums) : nullptr;
        void* args[] = {&dy, &pre, &out, &partial, &M, &N, &act};
        const void* fn = vec ? (const void*)linear_dz_kernel<8> : (const void*)linear_dz_kernel<1>;
        if (launch_kernel(fn, dim3(g.x, g.y), dim3(32 * kDzRows), 0, args, stream) != cudaSuccess) return VMB_ERR_CUDA;
        if (partial) {
            const vmb_status s = launch_column_sums(partial, (int)g.y, N, N, 1, a.dbias, nullptr, 0, nullptr, stream);
            if (s != VMB_OK) return s;
        }
        if (act != VMB_ACT_NONE) dz = out;
    }
    if (a.dx && a.K > 0) {
        const GemmProblem p{dz, a.weight, M, a.K, N, N, 1, 1, a.K, {nullptr, nullptr, nullptr, nullptr, (__nv_bfloat16*)a.dx, nullptr, VMB_ACT_NONE}};
        const vmb_status s = launch_gemm(p, false, a, l, stream);
        if (s != VMB_OK) return s;
    }
    if (a.dweight && a.K > 0) {
        const GemmProblem p{dz, a.x, N, a.K, M, 1, N, 1, a.x_t, {nullptr, nullptr, nullptr, nullptr, (__nv_bfloat16*)a.dweight, nullptr, VMB_ACT_NONE}};
        return launch_gemm(p, false, a, l, stream);
    }
    return VMB_OK;
}

}  // namespace vmb
