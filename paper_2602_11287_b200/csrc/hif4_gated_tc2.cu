// Forward instances of the CTA-pair linear kernel, gated.
#include "hif4_linear_tc2_launch.cuh"

namespace hif4 {

hif4_status launch_gated_tc2(const LinearCall& c, void* workspace, cudaStream_t st) {
  if (c.dt == HIF4_BF16) return launch_linear<true, false, __nv_bfloat16>(c, workspace, st);
  if (c.dt == HIF4_FP16) return launch_linear<true, false, __half>(c, workspace, st);
  return launch_linear<true, false, float>(c, workspace, st);
}

}  // namespace hif4
