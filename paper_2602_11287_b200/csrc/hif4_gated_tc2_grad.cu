// Gradient instances of the CTA-pair linear kernel, gated: dG and dU as BF16 parts and the bias gradients' column sums.
#include "hif4_linear_tc2_launch.cuh"

namespace hif4 {

hif4_status launch_gated_tc2_grad(const LinearCall& c, void* workspace, cudaStream_t st) {
  return c.dt == HIF4_BF16 ? launch_linear<true, true, __nv_bfloat16>(c, workspace, st) : launch_linear<true, true, __half>(c, workspace, st);
}

}  // namespace hif4
