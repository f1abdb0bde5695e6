// hif4_linear_act, hif4_gated_linear and their backward passes: argument checks, then the products and what follows them.
#include "hif4_activation.cuh"
#include "hif4_common.cuh"
#include "hif4_gemm_internal.cuh"
#include "hif4_linear_internal.cuh"
#include "hif4_vec8.cuh"

namespace hif4 {
namespace {

struct EpilogueGradParams {
  float *z, *u;                     // FP32 products [M, N], overwritten by their gradients
  int64_t M, N;
  const void *bias, *bias_up;
  int act;
  const void* dy;
  int64_t ld_dy;
};
template <typename T>
__global__ void __launch_bounds__(256) epilogue_grad_kernel(const EpilogueGradParams p) {
  const int64_t idx = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (idx >= p.M * p.N) return;
  const int64_t row = idx / p.N, col = idx - row * p.N;
  const float dy = to_f32(static_cast<const T*>(p.dy)[row * p.ld_dy + col]);
  float z = p.act != HIF4_ACT_NONE || p.u ? p.z[idx] : 0.0f, a, slope;
  if (p.bias) z += to_f32(static_cast<const T*>(p.bias)[col]);
  activate_slope(z, p.act, a, slope);
  if (p.u) {
    float u = p.u[idx];
    if (p.bias_up) u += to_f32(static_cast<const T*>(p.bias_up)[col]);
    p.u[idx] = dy * a;
    p.z[idx] = dy * u * slope;
  } else {
    p.z[idx] = dy * slope;
  }
}
__global__ void __launch_bounds__(256) column_sum_kernel(const float* z, int64_t M, int64_t N, float* out) {
  const int64_t col = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (col >= N) return;
  float s = 0.0f;
  for (int64_t m = 0; m < M; ++m) s += z[m * N + col];
  out[col] = s;
}
// dX[M, K] (+)= dZ[M, N] W[N, K]: 32 rows x 64 columns (one unit) per block.
template <typename T>
__global__ void __launch_bounds__(256)
input_grad_kernel(const float* dz, const float* du, const uint32_t* w, const uint32_t* wu, int64_t M, int64_t N, int64_t upr, T* dx,
                  int64_t ld_dx) {
  __shared__ float zs[32][33], ws[32][65];
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * 32, unit = blockIdx.x;
  const int row = threadIdx.x >> 3, g = threadIdx.x & 7;
  float acc[8] = {};
  for (int pass = 0; pass < (du ? 2 : 1); ++pass) {
    const float* z = pass ? du : dz;
    const uint32_t* units = pass ? wu : w;
    for (int64_t n0 = 0; n0 < N; n0 += 32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = g * 4 + i;
        zs[row][c] = m0 + row < M && n0 + c < N ? z[(m0 + row) * N + n0 + c] : 0.0f;
      }
      const bool in = n0 + row < N;
      const uint32_t* u = units + ((n0 + row) * upr + unit) * kUnitWords;
      const uint32_t meta = in ? u[0] : 0u, code = in ? u[1 + g] : 0u, byte = meta & 0xFFu;
      const float s1 = byte == 0xFFu ? __uint_as_float(0x7FC00000u) : __uint_as_float((byte + 316u) << 21);   // E6M2 re-biased to FP32
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t nib = (code >> (4 * e)) & 15u;
        const uint32_t sh = ((meta >> (8 + g)) & 1u) + ((meta >> (16 + 2 * g + (e >> 2))) & 1u);
        const float v = static_cast<float>((nib & 7u) << sh) * 0.25f * s1;
        ws[row][8 * g + e] = nib & 8u ? -v : v;
      }
      __syncthreads();
      for (int n = 0; n < 32; ++n) {
        const float a = zs[row][n];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(a, ws[n][8 * g + e], acc[e]);
      }
      __syncthreads();
    }
  }
  if (m0 + row < M) {
#pragma unroll
    for (int e = 0; e < 8; ++e) dx[(m0 + row) * ld_dx + unit * 64 + 8 * g + e] = from_f32<T>(acc[e]);
  }
}

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }
bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t esize(int dt) { return dt == HIF4_FP32 ? 4 : 2; }
bool is_type(int dt) { return dt == HIF4_BF16 || dt == HIF4_FP32 || dt == HIF4_FP16; }

struct Scratch {
  size_t x, z, u, gemm, total;      // offsets
};
hif4_status plan(int64_t M, int64_t N, int64_t K, bool gated, Scratch& s) {
  if (M < 0 || N < 0 || K < 0 || K % kUnitElems != 0) return HIF4_ERR_SHAPE;
  s = Scratch{};
  if (M == 0 || N == 0) return HIF4_OK;
  size_t g = 0;
  const hif4_status st = hif4_gemm_workspace(M, N, K, &g);
  if (st != HIF4_OK) return st;
  s.z = s.x + pad256(hif4_packed_bytes(M, K));
  s.u = s.z + pad256(static_cast<size_t>(M) * N * 4);
  s.gemm = s.u + (gated ? pad256(static_cast<size_t>(M) * N * 4) : 0);
  s.total = s.gemm + pad256(g);
  return HIF4_OK;
}

// Forward workspace: packed activations, the pair kernel's shared tiles, and for FP32 units the rows before their
// conversion (64 FP32 columns of a row do not fit a thread's registers or the kernel's staging buffer).
struct ForwardScratch {
  size_t x, pair, y, total;
  bool rows_first;
};
hif4_status forward_plan(const hif4_linear_act_args* a, bool gated, ForwardScratch& s) {
  s = ForwardScratch{};
  if (a->M < 0 || a->N < 0 || a->K < 0 || a->K % kUnitElems != 0) return HIF4_ERR_SHAPE;
  if (a->M == 0 || a->N == 0) return HIF4_OK;
  if (!linear_tc2_supported(gated, a->M, a->N, a->K)) return HIF4_ERR_SHAPE;
  s.rows_first = a->y_units && a->dt == HIF4_FP32;
  s.pair = a->x_units ? 0 : pad256(hif4_packed_bytes(a->M, a->K));
  s.y = s.pair + pad256(linear_tc2_workspace(gated, a->M, a->N, a->K));
  s.total = s.y + (s.rows_first ? static_cast<size_t>(a->M) * a->N * 4 : 0);
  return HIF4_OK;
}

// The products of X with W (and W_up) as FP32 matrices in the workspace.
template <typename Args>
hif4_status products(const Args* a, bool gated, uint8_t* ws, const Scratch& s, void* stream) {
  const void* x = a->X;
  if (!a->x_units) {
    const hif4_status q = hif4_quantize(a->X, a->dt_x, a->M, a->K, a->ld_x, ws + s.x, a->mode, stream);
    if (q != HIF4_OK) return q;
    x = ws + s.x;
  }
  hif4_status st = hif4_gemm(x, a->W_units, reinterpret_cast<float*>(ws + s.z), a->M, a->N, a->K, a->N, ws + s.gemm, s.total - s.gemm, stream);
  if (st == HIF4_OK && gated)
    st = hif4_gemm(x, a->W_up_units, reinterpret_cast<float*>(ws + s.u), a->M, a->N, a->K, a->N, ws + s.gemm, s.total - s.gemm, stream);
  return st;
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

hif4_status forward(const hif4_linear_act_args* a, bool gated, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a) return HIF4_ERR_NULL;
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
  if (!a->x_units) {
    const hif4_status q = hif4_quantize(a->X, a->dt_x, a->M, a->K, a->ld_x, ws + s.x, a->mode, stream);
    if (q != HIF4_OK) return q;
    c.A = ws + s.x;
  }
  c.dt = a->dt; c.bias = a->bias; c.bias_up = gated ? a->bias_up : nullptr; c.act = a->act;
  c.side = a->residual; c.ld_side = a->ld_residual; c.res_scale = a->res_scale;
  c.y = a->Y; c.ld_y = a->ld_y; c.units = a->y_units ? 1 : 0; c.rha = a->mode == HIF4_RHA;
  if (!s.rows_first) return launch_linear_tc2(c, ws + s.pair, st);
  c.y = ws + s.y; c.ld_y = a->N; c.units = 0;
  const hif4_status pr = launch_linear_tc2(c, ws + s.pair, st);
  return pr != HIF4_OK ? pr : hif4_quantize(ws + s.y, a->dt, a->M, a->N, a->N, a->Y, a->mode, stream);
}

template <typename T>
hif4_status backward_t(const hif4_linear_act_backward_args* a, bool gated, uint8_t* ws, const Scratch& s, cudaStream_t st) {
  EpilogueGradParams p{};
  p.z = reinterpret_cast<float*>(ws + s.z);
  p.u = gated ? reinterpret_cast<float*>(ws + s.u) : nullptr;
  p.M = a->M; p.N = a->N; p.bias = a->bias; p.bias_up = a->bias_up; p.act = a->act; p.dy = a->dY; p.ld_dy = a->ld_dy;
  const int64_t blocks = ceil_div64(a->M * a->N, 256);
  if (blocks > 0x7FFFFFFFll || ceil_div64(a->M, 32) > 65535) return HIF4_ERR_SHAPE;
  epilogue_grad_kernel<T><<<static_cast<unsigned>(blocks), 256, 0, st>>>(p);
  note_launch();
  const unsigned cols = static_cast<unsigned>(ceil_div64(a->N, 256));
  if (a->dbias) { column_sum_kernel<<<cols, 256, 0, st>>>(p.z, a->M, a->N, a->dbias); note_launch(); }
  if (gated && a->dbias_up) { column_sum_kernel<<<cols, 256, 0, st>>>(p.u, a->M, a->N, a->dbias_up); note_launch(); }
  if (a->dX && a->K > 0) {
    const dim3 grid(static_cast<unsigned>(a->K / 64), static_cast<unsigned>(ceil_div64(a->M, 32)));
    input_grad_kernel<T><<<grid, 256, 0, st>>>(p.z, p.u, static_cast<const uint32_t*>(a->W_units), static_cast<const uint32_t*>(a->W_up_units),
                                               a->M, a->N, a->K / 64, static_cast<T*>(a->dX), a->ld_dx);
    note_launch();
  }
  return launch_status();
}

hif4_status backward(const hif4_linear_act_backward_args* a, bool gated, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a) return HIF4_ERR_NULL;
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
  Scratch s;
  const hif4_status ps = plan(a->M, a->N, a->K, gated, s);
  if (ps != HIF4_OK) return ps;
  if (!workspace || workspace_bytes < s.total) return HIF4_ERR_WORKSPACE;
  if (!is_aligned(workspace, 256)) return HIF4_ERR_ALIGN;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (reads_x) {
    const hif4_status pr = products(a, gated, ws, s, stream);
    if (pr != HIF4_OK) return pr;
  }
  return a->dt == HIF4_BF16 ? backward_t<__nv_bfloat16>(a, gated, ws, s, st) : backward_t<__half>(a, gated, ws, s, st);
}

template <typename Args>
hif4_status workspace_size(const Args* a, bool gated, size_t* bytes) {
  if (!a || !bytes) return HIF4_ERR_NULL;
  Scratch s;
  const hif4_status st = plan(a->M, a->N, a->K, gated, s);
  if (st == HIF4_OK) *bytes = s.total;
  return st;
}

}  // namespace
}  // namespace hif4

using namespace hif4;

namespace {
hif4_status forward_workspace(const hif4_linear_act_args* a, bool gated, size_t* bytes) {
  if (!a || !bytes) return HIF4_ERR_NULL;
  ForwardScratch s;
  const hif4_status st = forward_plan(a, gated, s);
  if (st == HIF4_OK) *bytes = s.total;
  return st;
}
}  // namespace
extern "C" hif4_status hif4_linear_act_workspace(const hif4_linear_act_args* args, size_t* bytes) { return forward_workspace(args, false, bytes); }
extern "C" hif4_status hif4_gated_linear_workspace(const hif4_linear_act_args* args, size_t* bytes) { return forward_workspace(args, true, bytes); }
extern "C" hif4_status hif4_linear_act_backward_workspace(const hif4_linear_act_backward_args* args, size_t* bytes) {
  return workspace_size(args, false, bytes);
}
extern "C" hif4_status hif4_gated_linear_backward_workspace(const hif4_linear_act_backward_args* args, size_t* bytes) {
  return workspace_size(args, true, bytes);
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
