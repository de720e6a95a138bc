// delta_bf16.cu - the gated delta rule's kernels for bf16 storage.
#include "delta_chain.cuh"
#include "delta_grad.cuh"

namespace vmb {
vmb_status launch_chain_bf16(const DeltaChain& c, bool reverse, cudaStream_t stream) { return launch_chain<__nv_bfloat16>(c, reverse, stream); }
vmb_status launch_grad_bf16(const DeltaGrad& c, cudaStream_t stream) { return launch_grad<__nv_bfloat16>(c, stream); }
}  // namespace vmb
