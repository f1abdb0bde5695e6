// Gradient instances of the CTA-pair linear kernel, one projection: dZ as BF16 parts and the bias gradient's column sums.
#include "hif4_linear_tc2_launch.cuh"

namespace hif4 {

hif4_status launch_linear_tc2_grad(const LinearCall& c, void* workspace, cudaStream_t st) {
  if (c.gated) return launch_gated_tc2_grad(c, workspace, st);
  return c.dt == HIF4_BF16 ? launch_linear<false, true, __nv_bfloat16>(c, workspace, st) : launch_linear<false, true, __half>(c, workspace, st);
}

}  // namespace hif4
