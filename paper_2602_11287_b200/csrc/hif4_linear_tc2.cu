// Forward instances of the CTA-pair linear kernel, one projection; sizes of all of them.
#include "hif4_linear_tc2_launch.cuh"

namespace hif4 {

size_t linear_tc2_workspace(bool gated, int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || N <= 0) return 0;
  const Tc2Plan pl = linear_plan(M, N, K, gated ? kPairN / 2 : kPairN);
  return pl.slices > 1 ? pl.flag_bytes + partial_tiles(pl) * kPartialTileBytes : 0;
}

hif4_status linear_tc2_clear(bool gated, int64_t M, int64_t N, int64_t K, void* workspace, cudaStream_t st) {
  const Tc2Plan pl = linear_plan(M, N, K, gated ? kPairN / 2 : kPairN);
  return pl.slices > 1 && cudaMemsetAsync(workspace, 0, pl.flag_bytes, st) != cudaSuccess ? HIF4_ERR_CUDA : HIF4_OK;
}

bool linear_tc2_supported(bool gated, int64_t M, int64_t N, int64_t K) {
  return M < (1ll << 31) - kPairM && N < (1ll << 31) - kPairN && K < (1ll << 31) &&
         ceil_div64(M, kPairM) * ceil_div64(N, gated ? kPairN / 2 : kPairN) <= 0x7FFFFFFFll;
}

hif4_status launch_linear_tc2(const LinearCall& c, void* workspace, cudaStream_t st) {
  if (c.gated) return launch_gated_tc2(c, workspace, st);
  if (c.dt == HIF4_BF16) return launch_linear<false, false, __nv_bfloat16>(c, workspace, st);
  if (c.dt == HIF4_FP16) return launch_linear<false, false, __half>(c, workspace, st);
  return launch_linear<false, false, float>(c, workspace, st);
}

}  // namespace hif4
