// mixer_internal.h - rotary positions and group norm between the C ABI (vmb_abi_mixer.cu) and their kernels.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "vmb.h"

namespace vmb {

struct RotaryArgs {
    const void *q, *k;  // k may be null
    const float* freq;
    const int* positions;  // [axes][B][T], or null: grid
    void *q_out, *k_out;
    int B, T, Hq, Hk, D, axes;
    int pair_end[4];  // pairs of axes 0 .. i together
    int grid[4];
    long long q_b, q_t, k_b, k_t;  // elements between batch rows and between tokens
    int interleaved, inverse;
    vmb_dtype dtype;
};
vmb_status launch_rotary(const RotaryArgs& a, cudaStream_t stream);

struct NormArgs {
    const void* x;
    const float *weight, *bias;  // [C] or null
    void* y;
    float* stats;  // [B][G][2]: mean, 1 / sqrt(var + eps)
    int B;
    long long L;
    int C, G;
    float eps;
    vmb_act act;
    vmb_dtype dtype;
    // gradients
    const void* dy = nullptr;
    void* dx = nullptr;
    float *dweight = nullptr, *dbias = nullptr;
    void* ws;
    size_t ws_bytes;
};
size_t norm_workspace_bytes(int B, long long L, int C, int G, vmb_dtype dtype, bool grads);
vmb_status launch_norm_fwd(const NormArgs& a, cudaStream_t stream);
vmb_status launch_norm_bwd(const NormArgs& a, cudaStream_t stream);

}  // namespace vmb
