// Internal launchers behind hif4_linear_act / hif4_gated_linear and their backward passes (arguments already validated).
#pragma once
#include <cuda_bf16.h>

#include "hif4_common.cuh"
#include "hif4_tc_common.cuh"

namespace hif4 {

// One product with what follows it.  Forward: side = residual, y.  Gradient: side = dY, dz and colsum.
struct LinearCall {
  bool gated, grad;
  int64_t M, N, K;
  const void *A, *B, *B2;           // units
  int dt;                           // type of bias, side and y
  const void *bias, *bias_up;
  int act;
  const void* side;
  int64_t ld_side;
  float res_scale;
  void* y;
  int64_t ld_y;
  int units, rha;
  __nv_bfloat16* dz;                // planes of [M, ld_dz]: the BF16 parts of dZ (dG, then those of dU), or NULL
  int64_t ld_dz, dz_plane;
  int parts;                        // of an element of dZ: 1 or 2 (FP16: 2)
  float* colsum;                    // [1 or 2][ceil(M / 32)][N], or NULL
};

namespace {
struct LinearParams {
  int64_t M, N;
  int num_kc, n_tiles, full_rounds, tail_tiles, slices, sk_tiles, sk_tile0;      // schedule (hif4_tc2_dense.cuh)
  unsigned int* flags;              // [shared tiles][slices][8]: 16-column steps of this slice's sums that are there, per 32 rows
  float* partial;                   // [shared tiles][slices - 1][2 ranks][4 warps][16 x 16 columns][4][32 rows][4]
  unsigned int* error_word;
  DecodeMul mul;
  int tma;                          // 1: units come through TMA, 0: copied word by word
  const uint8_t *A, *B, *B2;
  int64_t pitch;                    // bytes of a row of units
  int upr;                          // units of a row
  const void *bias, *bias_up;
  const void* side;
  int64_t ld_side;
  int side_vec, side_tma;
  float res_scale;
  void* y;
  int64_t ld_y;
  int tma_store, units, rha;
  __nv_bfloat16* dz;
  int64_t ld_dz, dz_plane;
  float* colsum;
  int64_t colsum_plane;
};
}  // namespace

// Weight-streaming form for M <= kGemvMaxM tokens (same requirements and workspace as launch_gemv / launch_gemv_linear);
// A holds units (x = nullptr), or x the activations, row stride ld_x.
hif4_status launch_linear_gemv(const LinearCall& c, const void* x, int dt_x, int64_t ld_x, void* workspace, cudaStream_t st);

size_t linear_tc2_workspace(bool gated, int64_t M, int64_t N, int64_t K);
// Zeroes the workspace's counts of finished steps; before the launch of the activations' conversion, so that the product's
// kernel follows that one directly and can overlap it.
hif4_status linear_tc2_clear(bool gated, int64_t M, int64_t N, int64_t K, void* workspace, cudaStream_t st);
bool linear_tc2_supported(bool gated, int64_t M, int64_t N, int64_t K);
hif4_status launch_linear_tc2(const LinearCall& c, void* workspace, cudaStream_t st);
hif4_status launch_gated_tc2(const LinearCall& c, void* workspace, cudaStream_t st);
hif4_status launch_linear_tc2_grad(const LinearCall& c, void* workspace, cudaStream_t st);
hif4_status launch_gated_tc2_grad(const LinearCall& c, void* workspace, cudaStream_t st);

// dX = sum over phases dZ W: `parts` BF16 planes of [M, ld_dz] per weight matrix (rows 16-byte aligned, plane after
// plane), one or two weight matrices.  The tensor core takes BF16, so an element of dZ is one BF16 number or the sum of two.  One
// has the eight bits that dY and dX have, and is what a chain of BF16 layers keeps of dZ anyway; two hold 16 bits, FP16's eleven
// among them, and multiply twice.  BF16, one and two: 2048 x 4096 x 4096 178 and 247 us, error of dX against 64 bits 2.2e-3 and
// 1.7e-3 (the rounding of dX alone); gated 1024 x 14336 x 4096 469 and 799 us, 2.3e-3 and 1.7e-3.
struct InputGradCall {
  int64_t M, N, K;
  const void* dz;
  int64_t ld_dz;
  int parts;
  const void *B, *B2;
  int dt;                           // BF16 or FP16
  void* dx;
  int64_t ld_dx;
};
size_t input_grad_tc2_workspace(int64_t M, int64_t N, int64_t K, int phases);
hif4_status input_grad_tc2_clear(int64_t M, int64_t N, int64_t K, int phases, void* workspace, cudaStream_t st);
bool input_grad_tc2_supported(int64_t M, int64_t N, int64_t K, int phases);
hif4_status launch_input_grad_tc2(const InputGradCall& c, void* workspace, cudaStream_t st);

}  // namespace hif4
