// Weight-streaming instances of the linear layer with its epilogue (M <= 32).
#include "hif4_gemv_kernel.cuh"

namespace hif4 {

hif4_status launch_gated_gemv(const LinearCall& c, const void* x, int dt_x, int64_t ld_x, void* workspace, cudaStream_t st);

hif4_status launch_linear_gemv(const LinearCall& c, const void* x, int dt_x, int64_t ld_x, void* workspace, cudaStream_t st) {
  if (c.gated) return launch_gated_gemv(c, x, dt_x, ld_x, workspace, st);
  if (!x) return gemv_from_units<kEpiLinear>(c.A, c.B, nullptr, c.M, c.N, c.K, 0, workspace, &c, st);
  return gemv_from_rows<kEpiLinear>(x, static_cast<hif4_dtype>(dt_x), ld_x, c.rha, c.B, nullptr, c.M, c.N, c.K, 0, workspace, &c, st);
}

}  // namespace hif4
