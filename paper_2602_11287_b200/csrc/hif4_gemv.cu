// hif4_gemm and hif4_linear for M <= 32 tokens: entry points of the weight-streaming kernel (hif4_gemv_kernel.cuh).
#include "hif4_gemv_kernel.cuh"

namespace hif4 {

constexpr int kResidentMaxBytes = 128 * 1024;         // resident tokens: K / 256 chunks of (n-tiles x 8 words x rows x 64) bytes
// At most two n-tiles of tokens and few enough token elements: the streaming kernel builds them itself, in shared
// memory.  Returns the token rows kept per n-tile (the next power of two >= M, eight for two tiles), 0 when the
// two-launch form is the faster one.  Every CTA repeats the build before its main loop, so it pays only while it costs
// less than the launch it saves: measured break-even (rows kept x K) about 57 000 elements when the tokens are decoded
// from packed units and about 16 000 when they are first converted from BF16 with Algorithm 1.
constexpr int64_t kResidentMaxElemsUnits = 49152, kResidentMaxElemsBf16 = 16384;
int gemv_resident_rows(int64_t M, int num_kc, bool from_bf16) {
  if (M > 16) return 0;
  const int64_t max_elems = from_bf16 ? kResidentMaxElemsBf16 : kResidentMaxElemsUnits;
  const int tiles = M <= 8 ? 1 : 2;
  const int rows = M <= 1 ? 1 : M <= 2 ? 2 : M <= 4 ? 4 : 8;
  const int64_t elems = static_cast<int64_t>(num_kc) * 256 * tiles * rows;
  return elems <= max_elems && elems * 2 <= kResidentMaxBytes ? rows : 0;
}

bool gemv_supported(const void* A, const void* B, int64_t M, int64_t N, int64_t K) {
  return M >= 1 && M <= kGemvMaxM && gemm_tc_supported(B, B, N, N, N, K) && (reinterpret_cast<uintptr_t>(A) & 3u) == 0;
}

size_t gemv_workspace_bytes(int64_t M, int64_t K) {
  if (M < 1 || M > kGemvMaxM || K <= 0 || K % 256 != 0) return 0;
  return static_cast<size_t>(gemv_m_pad(M) * K * 2);
}

hif4_status launch_gemv(const void* A, const void* B, float* C, int64_t M, int64_t N, int64_t K, int64_t ldc,
                        void* workspace, cudaStream_t st) {
  return gemv_from_units<kEpiNone>(A, B, C, M, N, K, ldc, workspace, nullptr, st);
}

bool gemv_linear_supported(const void* X, hif4_dtype dt, int64_t ld_x, const void* B, int64_t M, int64_t N, int64_t K) {
  const int64_t esz = dt == HIF4_FP32 ? 4 : 2;
  return M >= 1 && M <= kGemvMaxM && gemm_tc_supported(B, B, N, N, N, K) && (reinterpret_cast<uintptr_t>(X) & 15u) == 0 &&
         ld_x >= K && (ld_x * esz) % 16 == 0;
}

hif4_status launch_gemv_linear(const void* X, hif4_dtype dt, int64_t ld_x, int rha, const void* B, float* C, int64_t M,
                               int64_t N, int64_t K, int64_t ldc, void* workspace, cudaStream_t st) {
  return gemv_from_rows<kEpiNone>(X, dt, ld_x, rha, B, C, M, N, K, ldc, workspace, nullptr, st);
}

}  // namespace hif4
