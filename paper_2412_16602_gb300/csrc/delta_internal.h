// delta_internal.h - the gated delta rule between the C ABI (vmb_abi_mixer.cu) and its kernels.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "vmb.h"

namespace vmb {

// One problem as the ABI received it.  B sequences: dense (offsets null), T tokens each, or packed
// rows of `total` tokens, none longer than T.
struct DeltaArgs {
    const void *q = nullptr, *k = nullptr, *v = nullptr, *g = nullptr, *beta = nullptr;
    const float* initial = nullptr;  // [B][Hv][Dk][Dv]
    const int* offsets = nullptr;    // [B + 1]
    void* o = nullptr;               // [tokens][Hv][Dv]
    float* final = nullptr;          // [B][Hv][Dk][Dv]
    void* saved = nullptr;           // [slots][Hv][Dv][Dk], storage type: the state before each chunk, and
    void* saved_r = nullptr;         // [tokens][Hv][Dv]: the residuals r
    // gradients
    const void* dout = nullptr;      // [tokens][Hv][Dv]
    const float* dfinal = nullptr;   // [B][Hv][Dk][Dv]
    void *dq = nullptr, *dk = nullptr, *dv = nullptr, *dg = nullptr, *dbeta = nullptr;
    float* dinitial = nullptr;
    int B, T, Hk, Hv, Dk, Dv;
    long long total;
    long long q_b, q_t, k_b, k_t, v_b = 0, v_t = 0;  // elements between batch rows and between tokens
    float scale;
    vmb_dtype dtype;
    void* ws = nullptr;
    size_t ws_bytes = 0;
};

// How the chains (sequence, value head) are cut: `segs` segments of `seg_chunks` chunks, the
// segments of one chain joined through their state maps when there is more than one.
struct DeltaPlan {
    int chunks;      // chunks of the longest sequence
    int segs, seg_chunks;
    bool wide;       // 128 rows of the state per CTA instead of 64
    long long slots; // chunk states kept
    size_t maps_off, sums_off;        // segment maps [chain][seg][dk][dk] and sums [chain][seg][Dv][dk], fp32, dk = 64 or 128
    size_t ds_off, dx_off, part_off;  // gradients: chunk-end dS, dX, per-value-head dq and dk
    size_t bytes;
};
DeltaPlan plan_delta(const DeltaArgs& a, bool grads, int sms);
long long delta_slots(int B, int T, long long total, bool packed);

// What a launch of the chain kernels does.
struct DeltaChain {
    DeltaArgs a;
    int segs, seg_chunks, slices;
    bool wide;
    int summary;       // 1: write the sums (and, forward, the maps) of every segment and nothing else
    int maps_only;     // forward summary: the maps alone, for the reverse
    float* maps;       // [chain][seg][dk][dk], dk = 64 or 128 (maps_only: transposed)
    float* sums;       // [chain][seg][Dv][dk]: the sums, then the state at each segment's start (end in reverse)
    void* ds;          // reverse: [slots][Hv][Dv][Dk] dS at each chunk's end
    void* dx;          // reverse: [tokens][Hv][Dv]
    unsigned* err;
};
struct DeltaGrad {
    DeltaArgs a;
    const void* ds;
    const void* dx;
    float* part;       // per-value-head dq, dk [tokens][Hv][2][Dk] fp32 when heads are shared
    unsigned* err;
};
struct DeltaStep {
    const void *q, *k, *v, *g, *beta;
    float* state;      // [pool][Hv][Dk][Dv]
    const int* slots;  // [B] or null
    void* o;
    int B, T, Hk, Hv, Dk, Dv;
    long long q_b, q_t, k_b, k_t, v_b, v_t;
    int pool;
    float scale;
    vmb_dtype dtype;
};

// Allow a kernel `bytes` of dynamic shared memory (always the same for one kernel) on the current device.
bool allow_smem(const void* fn, int bytes);

vmb_status launch_delta_fwd(const DeltaArgs& a, cudaStream_t stream);
vmb_status launch_delta_bwd(const DeltaArgs& a, cudaStream_t stream);
vmb_status launch_delta_step(const DeltaStep& a, cudaStream_t stream);
// per storage type (delta_f32.cu, delta_bf16.cu); reverse = the gradients' chain
vmb_status launch_chain_f32(const DeltaChain& c, bool reverse, cudaStream_t stream);
vmb_status launch_chain_bf16(const DeltaChain& c, bool reverse, cudaStream_t stream);
vmb_status launch_grad_f32(const DeltaGrad& c, cudaStream_t stream);
vmb_status launch_grad_bf16(const DeltaGrad& c, cudaStream_t stream);

}  // namespace vmb
