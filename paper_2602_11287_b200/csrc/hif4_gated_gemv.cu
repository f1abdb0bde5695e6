// Weight-streaming instances of the gated feed-forward (M <= 32).
#include "hif4_gemv_kernel.cuh"

namespace hif4 {

hif4_status launch_gated_gemv(const LinearCall& c, const void* x, int dt_x, int64_t ld_x, void* workspace, cudaStream_t st) {
  if (!x) return gemv_from_units<kEpiGated>(c.A, c.B, nullptr, c.M, c.N, c.K, 0, workspace, &c, st);
  return gemv_from_rows<kEpiGated>(x, static_cast<hif4_dtype>(dt_x), ld_x, c.rha, c.B, nullptr, c.M, c.N, c.K, 0, workspace, &c, st);
}

}  // namespace hif4
