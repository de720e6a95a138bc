// delta_f32.cu - the gated delta rule's kernels for fp32 storage.
#include "delta_chain.cuh"
#include "delta_grad.cuh"

namespace vmb {
vmb_status launch_chain_f32(const DeltaChain& c, bool reverse, cudaStream_t stream) { return launch_chain<float>(c, reverse, stream); }
vmb_status launch_grad_f32(const DeltaGrad& c, cudaStream_t stream) { return launch_grad<float>(c, stream); }
}  // namespace vmb
