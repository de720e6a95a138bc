// layer_internal.h - the operators of a layer around the scan over tokens (short causal convolution, selective scan,
// root-mean-square norm, matrix product) between the C ABI (vmb_abi_layer.cu) and their kernels.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "vmb.h"

namespace vmb {

// B sequences: dense (offsets null), T tokens each, or packed rows of `total` tokens.
struct ConvArgs {
    const void* x;
    const float *weight, *bias;  // [C][W], [C] or null
    const void* initial;         // [B][W - 1][C] or null
    const int* offsets;          // [B + 1] or null
    void* y;
    void* final;  // [B][W - 1][C] or null
    int B, T;
    long long total;
    int C, W;
    long long x_b, x_t;  // elements between batch rows and between tokens
    vmb_act act;
    vmb_dtype dtype;
    // gradients
    const void *dy = nullptr, *dfinal = nullptr;
    void *dx = nullptr, *dinitial = nullptr;
    float *dweight = nullptr, *dbias = nullptr;
    void* ws = nullptr;
    size_t ws_bytes = 0;
    // steps
    void* state = nullptr;  // [pool][W - 1][C]
    const int* slots = nullptr;
    int pool = 0;
};
size_t conv_workspace_bytes(int B, int T, long long total, bool packed, int C, int W, vmb_dtype dtype);
vmb_status launch_conv_fwd(const ConvArgs& a, cudaStream_t stream);
vmb_status launch_conv_bwd(const ConvArgs& a, cudaStream_t stream);
vmb_status launch_conv_step(const ConvArgs& a, cudaStream_t stream);

struct TokenScanArgs {
    const void *x, *delta, *Bm, *Cm, *z;  // z may be null
    const float *A, *skip, *bias;         // [D][N]; [D] or null
    const float* initial;                 // [B][D][N] or null
    const int* offsets;
    void* y;
    float* final;
    float* saved;  // [slots of 16 tokens][D][N] or null: the state before each
    int B, T;
    long long total;
    int D, N;
    long long x_b, x_t, d_b, d_t, B_b, B_t, C_b, C_t, z_b, z_t;
    int softplus;
    vmb_dtype dtype;
    void* ws = nullptr;
    size_t ws_bytes = 0;
    // gradients
    const void* dy = nullptr;
    const float* dfinal = nullptr;
    void *dx = nullptr, *ddelta = nullptr, *dB = nullptr, *dC = nullptr, *dz = nullptr;
    float *dA = nullptr, *dskip = nullptr, *dbias = nullptr, *dinitial = nullptr;
    // steps
    float* state = nullptr;  // [pool][D][N]
    const int* slots = nullptr;
    int pool = 0;
};
constexpr int kScanChunk = 64;  // segments are of whole chunks of so many tokens
constexpr int kScanSaved = 16;  // tokens between two saved states
size_t token_scan_workspace_bytes(int B, int T, long long total, bool packed, int D, int N, bool grads, vmb_dtype dtype);
// Chunks of `chunk` tokens that B sequences of up to T tokens (packed: of `total` tokens) have at most: the chunks of packed
// sequence b start at place offsets[b] / chunk + b.
inline long long scan_slots(int B, int T, long long total, bool packed, int chunk) {
    return packed ? total / chunk + (B > 0 ? B : 1) : (long long)B * (T > 0 ? ((long long)T + chunk - 1) / chunk : 1);
}
vmb_status launch_token_scan_fwd(const TokenScanArgs& a, cudaStream_t stream);
vmb_status launch_token_scan_bwd(const TokenScanArgs& a, cudaStream_t stream);
vmb_status launch_token_scan_step(const TokenScanArgs& a, cudaStream_t stream);

struct RmsArgs {
    const void *x, *residual;  // residual may be null
    const float* weight;       // [C] or null
    void *y, *sum;             // y in the storage type, or e4m3 with `scale`
    float *scale, *rstd;       // [rows] or null
    long long rows;
    int C;
    float eps;
    bool bits8;
    vmb_dtype dtype;
    // gradients (x is the normalised sum)
    const void *dy = nullptr, *dsum = nullptr;
    void* dx = nullptr;
    float* dweight = nullptr;
    void* ws = nullptr;
    size_t ws_bytes = 0;
};
size_t rms_workspace_bytes(long long rows, int C, vmb_dtype dtype);
vmb_status launch_rms_fwd(const RmsArgs& a, cudaStream_t stream);
vmb_status launch_rms_bwd(const RmsArgs& a, cudaStream_t stream);

struct LinearArgs {
    const void *x, *weight;
    const float *x_scale, *weight_scale;  // both null: bf16; else e4m3 operands
    const float* bias;                    // [N] or null
    const void* residual;                 // [M][N] or null
    void *y, *pre;                        // pre may be null
    long long M;
    int K, N;
    long long x_t;  // elements between rows of x
    vmb_act act;
    // gradients (pre: the forward's)
    const void* dy = nullptr;
    void *dx = nullptr, *dweight = nullptr;
    float* dbias = nullptr;
    void* ws = nullptr;
    size_t ws_bytes = 0;
};
size_t linear_workspace_bytes(long long M, int K, int N, bool grads);
vmb_status launch_linear_fwd(const LinearArgs& a, cudaStream_t stream);
vmb_status launch_linear_bwd(const LinearArgs& a, cudaStream_t stream);

// Sums of the columns of p [rows][cols] fp32 in a fixed order: of the first taps * C columns, column j C + c goes to out[c taps + j], of
// the others the first n_rest to rest, those behind them to more.  Outputs may be null.
vmb_status launch_column_sums(const float* p, int rows, long long cols, int C, int taps, float* out, float* rest, int n_rest, float* more,
                              cudaStream_t stream);

}  // namespace vmb
