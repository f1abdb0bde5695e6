// hif4_linear_act, hif4_gated_linear and their backward passes: argument checks, then the products and what follows them.
#include "hif4_common.cuh"
#include "hif4_gemm_internal.cuh"
#include "hif4_linear_internal.cuh"
#include "hif4_vec8.cuh"

namespace hif4 {
namespace {

// A gradient that needs no activation: dZ = dY.  BF16 parts of dY (when the product cannot read dY itself) and the sums
// of 32 rows at a time; one thread per column of a row block, so that the lanes of a warp read neighbouring elements.  The row
// blocks go round the grid's second dimension, which ends at 65535.
template <typename T>
__global__ void __launch_bounds__(256)
split_rows_kernel(const T* dy, int64_t ld_dy, int64_t M, int64_t N, __nv_bfloat16* dz, int64_t ld_dz, int parts, float* colsum) {
  const int64_t col = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (col >= N) return;
  for (int64_t block = blockIdx.y; block * 32 < M; block += gridDim.y) {
    const int64_t r0 = block * 32, r1 = r0 + 32 < M ? r0 + 32 : M;
    float s = 0.0f;
#pragma unroll 8
    for (int64_t r = r0; r < r1; ++r) {
      float v = to_f32(dy[r * ld_dy + col]);
      s += v;
      if (!dz) continue;
      for (int part = 0; part < parts; ++part) {
        const __nv_bfloat16 b = __float2bfloat16_rn(v);
        dz[(part * M + r) * ld_dz + col] = b;
        v = rest_of(v, __bfloat162float(b));
      }
    }
    if (colsum) colsum[block * N + col] = s;
  }
}

// out[col] = sum of the row blocks' sums: 32 columns per block, 32 ways over the row blocks, joined in a fixed order.
__global__ void __launch_bounds__(1024) column_finish_kernel(const float* colsum, int64_t blocks, int64_t N, float* out, float* out_up) {
  __shared__ float part[32][33];
  const int lane = threadIdx.x & 31, way = threadIdx.x >> 5;
  const int64_t col = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  const float* src = colsum + blockIdx.y * blocks * N;
  float* dst = blockIdx.y ? out_up : out;
  if (!dst) return;
  float s = 0.0f;
  if (col < N)
    for (int64_t b = way; b < blocks; b += 32) s += src[b * N + col];
  part[way][lane] = s;
  __syncthreads();
  if (way == 0 && col < N) {
#pragma unroll
    for (int w = 1; w < 32; ++w) s += part[w][lane];
    dst[col] = s;
  }
}

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }
bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t esize(int dt) { return dt == HIF4_FP32 ? 4 : 2; }
bool is_type(int dt) { return dt == HIF4_BF16 || dt == HIF4_FP32 || dt == HIF4_FP16; }

// Up to 32 tokens stream the weights (K % 256 == 0, 16-byte aligned units); more of them, or other weights, take the pair kernel.
bool streams(const hif4_linear_act_args* a, bool gated) {
  return gemv_supported(a->X, a->W_units, a->M, a->N, a->K) && (!gated || is_aligned(a->W_up_units, 16)) &&
         (a->x_units || gemv_linear_supported(a->X, a->dt_x, a->ld_x, a->W_units, a->M, a->N, a->K));
}

// Forward workspace: packed activations, the pair kernel's shared tiles, and for units the rows before their conversion where
// the kernel cannot convert them itself (the streaming kernel's blocks do not hold whole units; 64 FP32 columns of a
// row do not fit the pair kernel's staging buffer).  The size does not depend on the addresses.
struct ForwardScratch {
  size_t x, pair, y, total;
  bool rows_first, stream;          // stream: the weight-streaming kernel (its tokens take the place of x and pair)
};
hif4_status forward_plan(const hif4_linear_act_args* a, bool gated, ForwardScratch& s) {
  s = ForwardScratch{};
  if (a->M < 0 || a->N < 0 || a->K < 0 || a->K % kUnitElems != 0) return HIF4_ERR_SHAPE;
  if (a->M == 0 || a->N == 0) return HIF4_OK;
  if (!linear_tc2_supported(gated, a->M, a->N, a->K)) return HIF4_ERR_SHAPE;
  s.stream = streams(a, gated);
  s.rows_first = a->y_units && (a->dt == HIF4_FP32 || s.stream);
  s.pair = a->x_units ? 0 : pad256(hif4_packed_bytes(a->M, a->K));
  s.y = s.pair + pad256(linear_tc2_workspace(gated, a->M, a->N, a->K));
  const size_t tokens = pad256(gemv_workspace_bytes(a->M, a->K));
  if (tokens > s.y) s.y = tokens;
  s.total = s.y + (a->y_units ? pad256(static_cast<size_t>(a->M) * a->N * esize(a->dt)) : 0);
  return HIF4_OK;
}

// Backward workspace: packed activations, the recomputed product's shared tiles, the BF16 planes of dZ, column sums, the
// last product's shared tiles.
struct BackwardScratch {
  size_t x, pair, dz, colsum, last, total;
  int parts, phases;
  bool recompute, direct;           // direct: the last product reads dY itself
  int64_t ld_dz;
};
hif4_status backward_plan(const hif4_linear_act_backward_args* a, bool gated, BackwardScratch& s) {
  s = BackwardScratch{};
  if (a->M < 0 || a->N < 0 || a->K < 0 || a->K % kUnitElems != 0) return HIF4_ERR_SHAPE;
  if (a->M == 0 || a->N == 0) return HIF4_OK;
  s.recompute = gated || a->act != HIF4_ACT_NONE;
  s.parts = a->dt == HIF4_FP16 || (a->precise && s.recompute) ? 2 : 1;      // (dZ = dY of BF16 is one BF16 number)
  s.phases = s.parts * (gated ? 2 : 1);
  s.ld_dz = (a->N + 7) / 8 * 8;
  if (!linear_tc2_supported(gated, a->M, a->N, a->K) || !input_grad_tc2_supported(a->M, a->N, a->K, s.phases)) return HIF4_ERR_SHAPE;
  s.pair = s.recompute && !a->x_units ? pad256(hif4_packed_bytes(a->M, a->K)) : 0;
  s.dz = s.pair + (s.recompute ? pad256(linear_tc2_workspace(gated, a->M, a->N, a->K)) : 0);
  s.colsum = s.dz + pad256(static_cast<size_t>(s.phases) * a->M * s.ld_dz * 2);
  s.last = s.colsum + pad256(static_cast<size_t>(gated ? 2 : 1) * ceil_div64(a->M, 32) * a->N * 4);
  s.total = s.last + pad256(input_grad_tc2_workspace(a->M, a->N, a->K, s.phases));
  s.direct = !s.recompute && s.parts == 1 && is_aligned(a->dY, 16) && a->ld_dy % 8 == 0;
  return HIF4_OK;
}

// Checks that both directions share.  `reads_x`: X and the products take part.
template <typename Args>
hif4_status check_operands(const Args* a, bool gated, bool reads_x) {
  if (!is_type(a->dt) || !is_type(a->dt_x) || (a->mode != HIF4_RNE && a->mode != HIF4_RHA) || a->act < HIF4_ACT_NONE || a->act > HIF4_ACT_GELU_TANH)
    return HIF4_ERR_DTYPE;
  if (a->M < 0 || a->N < 0 || a->K < 0 || a->K % kUnitElems != 0 || (reads_x && !a->x_units && a->ld_x < a->K)) return HIF4_ERR_SHAPE;
  if (a->M == 0 || a->N == 0) return HIF4_OK;
  if (a->K > 0 && ((reads_x && !a->X) || !a->W_units || (gated && !a->W_up_units))) return HIF4_ERR_NULL;
  if (reads_x && a->K > 0 && (a->x_units ? !is_aligned(a->X, 4) : !is_aligned(a->X, 16) || (a->M > 1 && a->ld_x * esize(a->dt_x) % 16 != 0)))
    return HIF4_ERR_ALIGN;
  if (!is_aligned(a->W_units, 4) || (gated && !is_aligned(a->W_up_units, 4))) return HIF4_ERR_ALIGN;
  const size_t e = esize(a->dt);
  if (!is_aligned(a->bias, e) || (gated && !is_aligned(a->bias_up, e))) return HIF4_ERR_ALIGN;
  return HIF4_OK;
}

// The arguments with the row stride of a single row of activations set to its length: no row follows it, so no kernel's or
// conversion's rule on strides applies.
template <typename Args>
Args single_row_stride(const Args& a) {
  Args c = a;
  if (c.M == 1 && !c.x_units && c.ld_x > c.K) c.ld_x = c.K;
  return c;
}

hif4_status forward(const hif4_linear_act_args* args, bool gated, void* workspace, size_t workspace_bytes, void* stream) {
  if (!args) return HIF4_ERR_NULL;
  const hif4_linear_act_args one = single_row_stride(*args), *a = &one;
  const hif4_status chk = check_operands(a, gated, true);
  if (chk != HIF4_OK) return chk;
  if ((a->y_units && a->N % kUnitElems != 0) || (!a->y_units && a->ld_y < a->N) || (a->residual && a->ld_residual < a->N)) return HIF4_ERR_SHAPE;
  if (a->M == 0 || a->N == 0) return HIF4_OK;
  if (!a->Y) return HIF4_ERR_NULL;
  const size_t e = esize(a->dt);
  if (!is_aligned(a->Y, a->y_units ? 4 : e) || !is_aligned(a->residual, e)) return HIF4_ERR_ALIGN;
  ForwardScratch s;
  const hif4_status ps = forward_plan(a, gated, s);
  if (ps != HIF4_OK) return ps;
  if (s.total > 0 && (!workspace || workspace_bytes < s.total)) return HIF4_ERR_WORKSPACE;
  if (!is_aligned(workspace, 256)) return HIF4_ERR_ALIGN;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  LinearCall c{};
  c.gated = gated;
  c.M = a->M; c.N = a->N; c.K = a->K;
  c.A = a->X; c.B = a->W_units; c.B2 = a->W_up_units;
  c.dt = a->dt; c.bias = a->bias; c.bias_up = gated ? a->bias_up : nullptr; c.act = a->act;
  c.side = a->residual; c.ld_side = a->ld_residual; c.res_scale = a->res_scale;
  c.y = a->Y; c.ld_y = a->ld_y; c.units = a->y_units ? 1 : 0; c.rha = a->mode == HIF4_RHA;
  if (s.rows_first) { c.y = ws + s.y; c.ld_y = a->N; c.units = 0; }
  hif4_status pr;
  if (s.stream) {
    pr = launch_linear_gemv(c, a->x_units ? nullptr : a->X, a->dt_x, a->ld_x, ws, st);
  } else {
    pr = linear_tc2_clear(gated, a->M, a->N, a->K, ws + s.pair, st);
    if (pr != HIF4_OK) return pr;
    if (!a->x_units) {
      const hif4_status q = hif4_quantize(a->X, a->dt_x, a->M, a->K, a->ld_x, ws + s.x, a->mode, stream);
      if (q != HIF4_OK) return q;
      c.A = ws + s.x;
    }
    pr = launch_linear_tc2(c, ws + s.pair, st);
  }
  if (!s.rows_first) return pr;
  return pr != HIF4_OK ? pr : hif4_quantize(ws + s.y, a->dt, a->M, a->N, a->N, a->Y, a->mode, stream);
}

hif4_status backward(const hif4_linear_act_backward_args* args, bool gated, void* workspace, size_t workspace_bytes, void* stream) {
  if (!args) return HIF4_ERR_NULL;
  const hif4_linear_act_backward_args one = single_row_stride(*args), *a = &one;
  if (a->dt == HIF4_FP32) return HIF4_ERR_DTYPE;
  const bool reads_x = gated || a->act != HIF4_ACT_NONE;
  const hif4_status chk = check_operands(a, gated, reads_x);
  if (chk != HIF4_OK) return chk;
  if (a->ld_dy < a->N || (a->dX && a->ld_dx < a->K)) return HIF4_ERR_SHAPE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->M == 0 || a->N == 0) {                              // sums over nothing
    if (a->dX && a->M > 0 && a->K > 0 && cudaMemset2DAsync(a->dX, a->ld_dx * 2, 0, a->K * 2, a->M, st) != cudaSuccess) return HIF4_ERR_CUDA;
    for (float* v : {a->dbias, gated ? a->dbias_up : nullptr})
      if (v && a->N > 0 && cudaMemsetAsync(v, 0, a->N * 4, st) != cudaSuccess) return HIF4_ERR_CUDA;
    return HIF4_OK;
  }
  if (!a->dY) return HIF4_ERR_NULL;
  if (!is_aligned(a->dY, 2) || !is_aligned(a->dX, 2) || !is_aligned(a->dbias, 4) || (gated && !is_aligned(a->dbias_up, 4))) return HIF4_ERR_ALIGN;
  BackwardScratch s;
  const hif4_status ps = backward_plan(a, gated, s);
  if (ps != HIF4_OK) return ps;
  if (!workspace || workspace_bytes < s.total) return HIF4_ERR_WORKSPACE;
  if (!is_aligned(workspace, 256)) return HIF4_ERR_ALIGN;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const bool wants_dx = a->dX && a->K > 0, wants_db = a->dbias || (gated && a->dbias_up);
  if (!wants_dx && !wants_db) return HIF4_OK;
  float* colsum = wants_db ? reinterpret_cast<float*>(ws + s.colsum) : nullptr;
  __nv_bfloat16* dz = wants_dx && !s.direct ? reinterpret_cast<__nv_bfloat16*>(ws + s.dz) : nullptr;
  if (wants_dx) {
    const hif4_status z = input_grad_tc2_clear(a->M, a->N, a->K, s.phases, ws + s.last, st);
    if (z != HIF4_OK) return z;
  }
  if (s.recompute) {
    const hif4_status z = linear_tc2_clear(gated, a->M, a->N, a->K, ws + s.pair, st);
    if (z != HIF4_OK) return z;
    LinearCall c{};
    c.gated = gated; c.grad = true;
    c.M = a->M; c.N = a->N; c.K = a->K;
    c.A = a->X; c.B = a->W_units; c.B2 = a->W_up_units;
    if (!a->x_units) {
      const hif4_status q = hif4_quantize(a->X, a->dt_x, a->M, a->K, a->ld_x, ws + s.x, a->mode, stream);
      if (q != HIF4_OK) return q;
      c.A = ws + s.x;
    }
    c.dt = a->dt; c.bias = a->bias; c.bias_up = gated ? a->bias_up : nullptr; c.act = a->act;
    c.side = a->dY; c.ld_side = a->ld_dy;
    c.dz = dz; c.ld_dz = s.ld_dz; c.dz_plane = a->M * s.ld_dz; c.parts = s.parts;
    c.colsum = colsum;
    const hif4_status pr = launch_linear_tc2_grad(c, ws + s.pair, st);
    if (pr != HIF4_OK) return pr;
  } else if (dz || colsum) {
    const int64_t row_blocks = ceil_div64(a->M, 32);
    const dim3 grid(static_cast<unsigned>(ceil_div64(a->N, 256)), static_cast<unsigned>(row_blocks < 65535 ? row_blocks : 65535));
    if (a->dt == HIF4_BF16)
      split_rows_kernel<<<grid, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(a->dY), a->ld_dy, a->M, a->N, dz, s.ld_dz, s.parts, colsum);
    else
      split_rows_kernel<<<grid, 256, 0, st>>>(static_cast<const __half*>(a->dY), a->ld_dy, a->M, a->N, dz, s.ld_dz, s.parts, colsum);
    note_launch();
    if (cudaGetLastError() != cudaSuccess) return HIF4_ERR_CUDA;
  }
  if (wants_dx) {
  InputGradCall g{};
  g.M = a->M; g.N = a->N; g.K = a->K;
  g.dz = s.direct ? a->dY : dz;
  g.ld_dz = s.direct ? a->ld_dy : s.ld_dz;
  g.parts = s.parts;
  g.B = a->W_units; g.B2 = gated ? a->W_up_units : nullptr;
  g.dt = a->dt; g.dx = a->dX; g.ld_dx = a->ld_dx;
  const hif4_status last = launch_input_grad_tc2(g, ws + s.last, st);
  if (last != HIF4_OK) return last;
  }
  if (wants_db) {
    const dim3 grid(static_cast<unsigned>(ceil_div64(a->N, 32)), gated ? 2u : 1u);
    column_finish_kernel<<<grid, 1024, 0, st>>>(colsum, ceil_div64(a->M, 32), a->N, a->dbias, gated ? a->dbias_up : nullptr);
    note_launch();
    if (cudaGetLastError() != cudaSuccess) return HIF4_ERR_CUDA;
  }
  return HIF4_OK;
}

hif4_status forward_workspace(const hif4_linear_act_args* a, bool gated, size_t* bytes) {
  if (!a || !bytes) return HIF4_ERR_NULL;
  ForwardScratch s;
  const hif4_status st = forward_plan(a, gated, s);
  if (st == HIF4_OK) *bytes = s.total;
  return st;
}
hif4_status backward_workspace(const hif4_linear_act_backward_args* a, bool gated, size_t* bytes) {
  if (!a || !bytes) return HIF4_ERR_NULL;
  BackwardScratch s;
  const hif4_status st = backward_plan(a, gated, s);
  if (st == HIF4_OK) *bytes = s.total;
  return st;
}

}  // namespace
}  // namespace hif4

using namespace hif4;

extern "C" hif4_status hif4_linear_act_workspace(const hif4_linear_act_args* args, size_t* bytes) { return forward_workspace(args, false, bytes); }
extern "C" hif4_status hif4_gated_linear_workspace(const hif4_linear_act_args* args, size_t* bytes) { return forward_workspace(args, true, bytes); }
extern "C" hif4_status hif4_linear_act_backward_workspace(const hif4_linear_act_backward_args* args, size_t* bytes) {
  return backward_workspace(args, false, bytes);
}
extern "C" hif4_status hif4_gated_linear_backward_workspace(const hif4_linear_act_backward_args* args, size_t* bytes) {
  return backward_workspace(args, true, bytes);
}
extern "C" hif4_status hif4_linear_act(const hif4_linear_act_args* args, void* workspace, size_t workspace_bytes, void* stream) {
  return forward(args, false, workspace, workspace_bytes, stream);
}
extern "C" hif4_status hif4_gated_linear(const hif4_linear_act_args* args, void* workspace, size_t workspace_bytes, void* stream) {
  return forward(args, true, workspace, workspace_bytes, stream);
}
extern "C" hif4_status hif4_linear_act_backward(const hif4_linear_act_backward_args* args, void* workspace, size_t workspace_bytes,
                                                void* stream) {
  return backward(args, false, workspace, workspace_bytes, stream);
}
extern "C" hif4_status hif4_gated_linear_backward(const hif4_linear_act_backward_args* args, void* workspace, size_t workspace_bytes,
                                                  void* stream) {
  return backward(args, true, workspace, workspace_bytes, stream);
}
