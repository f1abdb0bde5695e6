// hif4_block_norm / hif4_block_norm_backward -- the norms after and before a block with gate, residual and residual
// scale, and their gradients.  One pass over the matrices: a row lives in the registers of one thread block from its
// loads to its stores, the row statistics are block-wide FP32 sums, and the result can leave as HiF4 units without the
// 16-bit matrix being written.  Bound by HBM traffic (forward 6.6 - 8 bytes an element in 16 bits, backward 12).
//
// A thread owns groups of eight columns (16-byte accesses when the matrices allow them).  Blocks take contiguous runs
// of rows and keep the next row's loads in flight while they reduce the current one; weights and gates are re-read
// per row, from L1 after a block's first row.
#include "hif4_common.cuh"
#include "hif4_vec8.cuh"

namespace hif4 {
namespace {

constexpr int64_t kNormMaxCols = 32768;

struct NormParams {
  int64_t rows;
  int cols;
  int kind_pre, kind_post;
  int dt_w;
  const void *x, *residual, *gate, *post_weight, *pre_weight, *pre_bias;
  int64_t ld_x, ld_residual, ld_gate, rows_per_gate;
  float res_scale, eps;
  void *h, *y;
  int64_t ld_h, ld_y;
  int units, rha;
  int strided;              // element-wise access: element j of a group is column base + j * blockDim.x
};

struct NormGradParams {
  int64_t rows;
  int cols;
  int kind_pre, kind_post;
  int dt_w;
  const void *dy, *dh, *h, *x, *gate, *post_weight, *pre_weight;
  int64_t ld_dy, ld_dh, ld_h, ld_x, ld_gate, rows_per_gate;
  float res_scale, eps;
  void *dx, *dresidual, *dgate;
  int64_t ld_dx, ld_dresidual;
  float *dpre_weight, *dpre_bias, *dpost_weight;
  float* partial;           // [5][grid][cols]: dpre_weight, dpre_bias, dpost_weight, first and last group of gates of each block
  int grid;
  int strided;
};

// Columns of a thread's group i: eight consecutive ones, or (element-wise access of rows that are not cut into groups
// of eight) one in every blockDim.x, so that the lanes of a warp still touch neighbouring elements.
struct Cols {
  int base, step;
  __device__ __forceinline__ Cols(int i, int strided) {
    const int t = i * static_cast<int>(blockDim.x);
    base = strided ? 8 * t + static_cast<int>(threadIdx.x) : 8 * (t + static_cast<int>(threadIdx.x));
    step = strided ? static_cast<int>(blockDim.x) : 1;
  }
};

template <bool kVec, typename T>
__device__ __forceinline__ Raw8<T> load_group(const T* row, const Cols& c, int cols) {
  Raw8<T> r;
  zero8(r);
  if (kVec) {
    if (c.base < cols) r = load8(row + c.base);
  } else {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = c.base + j * c.step;
      v[j] = e < cols ? to_f32(row[e]) : 0.0f;
    }
    r = pack8<T>(v);                                     // exact: the values come from T
  }
  return r;
}
template <bool kVec, typename T>
__device__ __forceinline__ void store_group(T* row, const Cols& c, int cols, const Raw8<T>& r) {
  if (kVec) {
    if (c.base < cols) store8(row + c.base, r);
  } else {
    float v[8];
    unpack8(r, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = c.base + j * c.step;
      if (e < cols) row[e] = from_f32<T>(v[j]);
    }
  }
}
// Weights of any type as FP32; `fill` where there is no weight vector.
template <bool kVec>
__device__ __forceinline__ void load_weights(const void* w, int dt_w, const Cols& c, int cols, float fill, float (&v)[8]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = fill;
    return;
  }
  if (dt_w == HIF4_BF16) unpack8(load_group<kVec>(static_cast<const __nv_bfloat16*>(w), c, cols), v);
  else if (dt_w == HIF4_FP16) unpack8(load_group<kVec>(static_cast<const __half*>(w), c, cols), v);
  else unpack8(load_group<kVec>(static_cast<const float*>(w), c, cols), v);
}

// Sums of kN values over the block.  `slot` alternates between calls, so that one barrier per call is enough: a warp
// can only be one call ahead of another, and then it writes the other half.
template <int kN>
__device__ __forceinline__ void block_sums(float (&v)[kN], float (*red)[4][32], uint32_t& slot) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int n = 0; n < kN; ++n)
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) v[n] += __shfl_xor_sync(0xFFFFFFFFu, v[n], s);
  if (warps == 1) return;
  if (lane == 0) {
#pragma unroll
    for (int n = 0; n < kN; ++n) red[slot & 1u][n][warp] = v[n];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    v[n] = lane < warps ? red[slot & 1u][n][lane] : 0.0f;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) v[n] += __shfl_xor_sync(0xFFFFFFFFu, v[n], s);
  }
  ++slot;
}

// Mean (LAYER only, else 0) and 1 / sqrt(mean of squares around it + eps) of a row held as v[kVpt][8].  Columns past
// the row's end hold zeros; the LAYER form keeps them out of the centred sum.
template <int kVpt>
__device__ __forceinline__ void row_stats(const float (&v)[kVpt][8], int kind, const NormParams& p, float (*red)[4][32],
                                          uint32_t& slot, float& mean, float& rstd) {
  mean = 0.0f;
  if (kind == HIF4_NORM_LAYER) {
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < kVpt; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[0] += v[i][j];
    block_sums(s, red, slot);
    mean = s[0] / static_cast<float>(p.cols);
  }
  float s[1] = {0.0f};
#pragma unroll
  for (int i = 0; i < kVpt; ++i) {
    const Cols c(i, p.strided);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = c.base + j * c.step < p.cols ? v[i][j] - mean : 0.0f;
      s[0] = fmaf(d, d, s[0]);
    }
  }
  block_sums(s, red, slot);
  rstd = 1.0f / sqrtf(s[0] / static_cast<float>(p.cols) + p.eps);
}

template <typename T, int kVpt, bool kVec>
__global__ void __launch_bounds__(kVpt == 4 ? 1024 : 512)
block_norm_kernel(const NormParams p) {
  __shared__ float red[2][4][32];
  uint32_t slot = 0;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows / gridDim.x;
  const int64_t row1 = (static_cast<int64_t>(blockIdx.x) + 1) * p.rows / gridDim.x;
  const T* x = static_cast<const T*>(p.x);
  const T* res = static_cast<const T*>(p.residual);
  Raw8<T> xr[kVpt], rr[kVpt];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i, p.strided);
      xr[i] = load_group<kVec>(x + row * p.ld_x, c, p.cols);
      if (res) rr[i] = load_group<kVec>(res + row * p.ld_residual, c, p.cols);
      else zero8(rr[i]);
    }
  };
  if (row0 < row1) fetch(row0);
  for (int64_t row = row0; row < row1; ++row) {
    float v[kVpt][8], r[kVpt][8];
#pragma unroll
    for (int i = 0; i < kVpt; ++i) { unpack8(xr[i], v[i]); unpack8(rr[i], r[i]); }
    if (row + 1 < row1) fetch(row + 1);
    if (p.kind_post != HIF4_NORM_NONE) {
      float mean, rstd;
      row_stats<kVpt>(v, p.kind_post, p, red, slot, mean, rstd);
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        float w[8];
        load_weights<kVec>(p.post_weight, p.dt_w, Cols(i, p.strided), p.cols, 1.0f, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - mean) * rstd * w[j];
      }
    }
    if (p.gate) {
      const T* gate = static_cast<const T*>(p.gate) + (row / p.rows_per_gate) * p.ld_gate;
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        float g[8];
        unpack8(load_group<kVec>(gate, Cols(i, p.strided), p.cols), g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
      }
    }
    if (res) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = fmaf(p.res_scale, r[i][j], v[i][j]);
    }
    if (p.h) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
        store_group<kVec>(static_cast<T*>(p.h) + row * p.ld_h, Cols(i, p.strided), p.cols, pack8<T>(v[i]));
    }
    if (!p.y) continue;
    float mean, rstd;
    row_stats<kVpt>(v, p.kind_pre, p, red, slot, mean, rstd);
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i, p.strided);
      float w[8], b[8];
      load_weights<kVec>(p.pre_weight, p.dt_w, c, p.cols, 1.0f, w);
      load_weights<kVec>(p.pre_bias, p.dt_w, c, p.cols, 0.0f, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = fmaf((v[i][j] - mean) * rstd, w[j], b[j]);
      const Raw8<T> out = pack8<T>(v[i]);
      if (!p.units) {
        store_group<kVec>(static_cast<T*>(p.y) + row * p.ld_y, c, p.cols, out);
      } else {
        // eight consecutive lanes hold a unit (cols % 64 == 0, so a unit is inside the row or outside as a whole)
        const int group = c.base >> 3, g = group & 7;
        uint32_t meta;
        const uint32_t code = p.rha ? encode_unit_octet<true>(out, g, meta) : encode_unit_octet<false>(out, g, meta);
        if (c.base < p.cols) {
          uint32_t* dst = static_cast<uint32_t*>(p.y) + (row * (p.cols >> 6) + (group >> 3)) * kUnitWords;
          dst[1 + g] = code;
          if (g == 0) dst[0] = meta;
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------------- backward
// Column sums (weights, biases, gates) are kept in registers over a block's run of rows.  The weights' sums go to
// `partial` once per block.  A group of gates that lies inside one block's run is finished there; at most two groups
// of a block reach into a neighbour's run, and their parts go to `partial` as well.  norm_grad_finish_kernel adds the
// parts in block order, so the result does not depend on scheduling.
// kPath: the gradient also passes a gate or a post norm, i.e. x takes part.
template <typename T, int kVpt, bool kVec, bool kPath>
__global__ void __launch_bounds__(kVpt == 4 ? 1024 : 512)
block_norm_backward_kernel(const NormGradParams p) {
  __shared__ float red[2][4][32];
  uint32_t slot = 0;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows / gridDim.x;
  const int64_t row1 = (static_cast<int64_t>(blockIdx.x) + 1) * p.rows / gridDim.x;
  const float inv_cols = 1.0f / static_cast<float>(p.cols);
  const bool pre_layer = p.kind_pre == HIF4_NORM_LAYER, post_layer = p.kind_post == HIF4_NORM_LAYER;
  const bool post = kPath && p.kind_post != HIF4_NORM_NONE;
  float dw[kVpt][8], db[kVpt][8], dwp[kPath ? kVpt : 1][8], dg[kPath ? kVpt : 1][8];
#pragma unroll
  for (int i = 0; i < kVpt; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dw[i][j] = db[i][j] = 0.0f;
      if (kPath) dwp[i][j] = dg[i][j] = 0.0f;
    }
  int64_t group = kPath && p.gate ? row0 / p.rows_per_gate : 0;
  for (int64_t row = row0; row < row1; ++row) {
    float a[kVpt][8], t[kVpt][8], x[kPath ? kVpt : 1][8], dyv[kVpt][8];      // h, gradient of h, x, dy
    float s1[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i, p.strided);
      Raw8<T> z;
      zero8(z);
      unpack8(p.dy ? load_group<kVec>(static_cast<const T*>(p.h) + row * p.ld_h, c, p.cols) : z, a[i]);
      unpack8(p.dy ? load_group<kVec>(static_cast<const T*>(p.dy) + row * p.ld_dy, c, p.cols) : z, dyv[i]);
      unpack8(p.dh ? load_group<kVec>(static_cast<const T*>(p.dh) + row * p.ld_dh, c, p.cols) : z, t[i]);
      if (kPath) unpack8(p.x ? load_group<kVec>(static_cast<const T*>(p.x) + row * p.ld_x, c, p.cols) : z, x[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) { s1[0] += a[i][j]; if (kPath) s1[1] += x[i][j]; }
    }
    float mean = 0.0f, mean_x = 0.0f;
    if (pre_layer || post_layer) {
      block_sums(s1, red, slot);
      if (pre_layer) mean = s1[0] * inv_cols;
      if (post_layer) mean_x = s1[1] * inv_cols;
    }
    // sums over the row: (h - mean)^2, dn (h - mean), dn, (x - mean_x)^2; columns past the end hold zero gradients
    float s2[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i, p.strided);
      float w[8];
      load_weights<kVec>(p.pre_weight, p.dt_w, c, p.cols, 1.0f, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = c.base + j * c.step < p.cols;
        a[i][j] = in ? a[i][j] - mean : 0.0f;
        const float dn = dyv[i][j] * w[j];
        s2[0] = fmaf(a[i][j], a[i][j], s2[0]);
        s2[1] = fmaf(dn, a[i][j], s2[1]);
        s2[2] += dn;
        if (kPath) {
          x[i][j] = in ? x[i][j] - mean_x : 0.0f;
          s2[3] = fmaf(x[i][j], x[i][j], s2[3]);
        }
      }
    }
    block_sums(s2, red, slot);
    const float rstd = 1.0f / sqrtf(s2[0] * inv_cols + p.eps);
    const float m1 = s2[1] * rstd * inv_cols, m0 = pre_layer ? s2[2] * inv_cols : 0.0f;
    const float rstd_x = post ? 1.0f / sqrtf(s2[3] * inv_cols + p.eps) : 1.0f;
    const T* gate = kPath && p.gate ? static_cast<const T*>(p.gate) + (row / p.rows_per_gate) * p.ld_gate : nullptr;
    float s3[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i, p.strided);
      float w[8], o[8];
      if (p.dy) {
        load_weights<kVec>(p.pre_weight, p.dt_w, c, p.cols, 1.0f, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float n = a[i][j] * rstd, d = dyv[i][j];
          dw[i][j] = fmaf(d, n, dw[i][j]);
          db[i][j] += d;
          t[i][j] = fmaf(rstd, fmaf(-n, m1, d * w[j] - m0), t[i][j]);
        }
      }
      if (p.dresidual) {
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = p.res_scale * t[i][j];
        store_group<kVec>(static_cast<T*>(p.dresidual) + row * p.ld_dresidual, c, p.cols, pack8<T>(o));
      }
      if (kPath) {
        float g[8], wp[8];
        if (gate) unpack8(load_group<kVec>(gate, c, p.cols), g);
        else {
#pragma unroll
          for (int j = 0; j < 8; ++j) g[j] = 1.0f;
        }
        load_weights<kVec>(post ? p.post_weight : nullptr, p.dt_w, c, p.cols, 1.0f, wp);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float xn = x[i][j] * rstd_x;                     // x itself without a post norm
          const float dp = t[i][j] * g[j];
          dg[i][j] = fmaf(t[i][j], xn * wp[j], dg[i][j]);
          dwp[i][j] = fmaf(dp, xn, dwp[i][j]);
          x[i][j] = xn;
          const bool in = c.base + j * c.step < p.cols;
          t[i][j] = in ? dp * wp[j] : 0.0f;
          s3[0] = fmaf(t[i][j], xn, s3[0]);
          s3[1] += t[i][j];
        }
      }
    }
    if (post && p.dx) {
      block_sums(s3, red, slot);
      const float q1 = s3[0] * inv_cols, q0 = post_layer ? s3[1] * inv_cols : 0.0f;
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) t[i][j] = rstd_x * (fmaf(-x[i][j], q1, t[i][j]) - q0);
    }
    if (p.dx) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
        store_group<kVec>(static_cast<T*>(p.dx) + row * p.ld_dx, Cols(i, p.strided), p.cols, pack8<T>(t[i]));
    }
    if (kPath && p.dgate) {
      const int64_t end = (group + 1) * p.rows_per_gate < p.rows ? (group + 1) * p.rows_per_gate : p.rows;
      if (row + 1 == end || row + 1 == row1) {
        const bool starts_here = group * p.rows_per_gate >= row0, ends_here = row + 1 == end;
#pragma unroll
        for (int i = 0; i < kVpt; ++i) {
          const Cols c(i, p.strided);
          if (starts_here && ends_here) {
            store_group<kVec>(static_cast<T*>(p.dgate) + group * p.cols, c, p.cols, pack8<T>(dg[i]));
          } else {
            float* part = p.partial + (static_cast<int64_t>(starts_here ? 4 : 3) * gridDim.x + blockIdx.x) * p.cols;
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (c.base + j * c.step < p.cols) part[c.base + j * c.step] = dg[i][j];
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) dg[i][j] = 0.0f;
        }
        ++group;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kVpt; ++i) {
    const Cols c(i, p.strided);
    float* part = p.partial + static_cast<int64_t>(blockIdx.x) * p.cols;
    const int64_t plane = static_cast<int64_t>(gridDim.x) * p.cols;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = c.base + j * c.step;
      if (e >= p.cols) continue;
      if (p.dpre_weight) part[e] = dw[i][j];
      if (p.dpre_bias) part[plane + e] = db[i][j];
      if (kPath && p.dpost_weight) part[2 * plane + e] = dwp[i][j];
    }
  }
}

// blockIdx.y 0..2: one of the weight gradients, summed over the blocks of the pass above.  blockIdx.y = 3 + b, b >= 1: the
// group of gates that runs over the boundary between blocks b - 1 and b, if that is the first boundary it crosses.
constexpr int kFinishCols = 32, kFinishWays = 32;
template <typename T>
__global__ void __launch_bounds__(kFinishCols * kFinishWays)
norm_grad_finish_kernel(const NormGradParams p) {
  __shared__ float part[kFinishWays][kFinishCols + 1];
  const int col = blockIdx.x * kFinishCols + (threadIdx.x & (kFinishCols - 1)), way = threadIdx.x / kFinishCols;
  const int64_t plane = static_cast<int64_t>(p.grid) * p.cols;
  if (blockIdx.y < 3) {
    float* out = blockIdx.y == 0 ? p.dpre_weight : blockIdx.y == 1 ? p.dpre_bias : p.dpost_weight;
    if (!out) return;
    float s = 0.0f;
    if (col < p.cols)
      for (int b = way; b < p.grid; b += kFinishWays) s += p.partial[blockIdx.y * plane + static_cast<int64_t>(b) * p.cols + col];
    part[way][threadIdx.x & (kFinishCols - 1)] = s;
    __syncthreads();
    if (way == 0 && col < p.cols) {
#pragma unroll
      for (int w = 1; w < kFinishWays; ++w) s += part[w][threadIdx.x];
      out[col] = s;
    }
    return;
  }
  const int b = static_cast<int>(blockIdx.y) - 3 + 1;
  const int64_t start = static_cast<int64_t>(b) * p.rows / p.grid;                       // first row of block b
  const int64_t group = start / p.rows_per_gate, g0 = group * p.rows_per_gate;
  if (g0 == start || g0 < static_cast<int64_t>(b - 1) * p.rows / p.grid) return;         // does not cross, or crossed before
  const int64_t g1 = g0 + p.rows_per_gate < p.rows ? g0 + p.rows_per_gate : p.rows;
  if (way != 0 || col >= p.cols) return;
  float s = p.partial[4 * plane + static_cast<int64_t>(b - 1) * p.cols + col];
  for (int k = b; k < p.grid && static_cast<int64_t>(k) * p.rows / p.grid < g1; ++k)
    s += p.partial[3 * plane + static_cast<int64_t>(k) * p.cols + col];
  static_cast<T*>(p.dgate)[group * p.cols + col] = from_f32<T>(s);
}

// ------------------------------------------------------------------------------------------------------- host side
int device_sms() {
  static int cache[64] = {};
  int dev = 0, v = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 148;
  if (dev >= 0 && dev < 64 && cache[dev] > 0) return cache[dev];
  if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v <= 0) return 148;
  if (dev >= 0 && dev < 64) cache[dev] = v;
  return v;
}

// Groups of eight columns per thread: one up to 4096 columns, then two, then four (and up to 1024 threads).
int groups_per_thread(int64_t cols) { return cols <= 4096 ? 1 : cols <= 8192 ? 2 : 4; }
int threads_for(int64_t cols, int vpt) {
  const int64_t t = ceil_div64(ceil_div64(cols, 8), vpt);
  return static_cast<int>(ceil_div64(t, 32) * 32);
}
// Blocks that one SM holds: about 1024 threads keep enough loads in flight, and no block may be alone with its barriers.
int grid_for(int64_t rows, int threads, int per_sm_threads) {
  const int per_sm = per_sm_threads / threads < 1 ? 1 : per_sm_threads / threads > 16 ? 16 : per_sm_threads / threads;
  const int64_t g = static_cast<int64_t>(device_sms()) * per_sm;
  return static_cast<int>(rows < g ? rows : g);
}
constexpr int kForwardThreadsPerSm = 1024, kBackwardThreadsPerSm = 512;

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t type_size(int dt) { return dt == HIF4_FP32 ? 4 : 2; }
bool known_type(int dt) { return dt == HIF4_BF16 || dt == HIF4_FP32 || dt == HIF4_FP16; }
bool known_kind(int k) { return k == HIF4_NORM_NONE || k == HIF4_NORM_RMS || k == HIF4_NORM_LAYER; }

// One matrix or vector argument: NULL is fine here; the stride must hold a row and the address an element.
struct Operand {
  const void* p;
  int64_t ld;
  int dt;
};
hif4_status check_operands(const Operand* o, int n, int64_t rows, int64_t cols, bool& vec) {
  vec = cols % 8 == 0;
  for (int i = 0; i < n; ++i) {
    if (!o[i].p) continue;
    if (o[i].ld < cols) return HIF4_ERR_SHAPE;
    const size_t e = type_size(o[i].dt);
    if (!aligned_to(o[i].p, e)) return HIF4_ERR_ALIGN;
    vec = vec && aligned_to(o[i].p, 16) && (rows <= 1 || o[i].ld * e % 16 == 0);
  }
  return HIF4_OK;
}

template <typename T, int kVpt>
hif4_status launch_norm(const NormParams& p, bool vec, cudaStream_t st) {
  const int threads = threads_for(p.cols, kVpt), grid = grid_for(p.rows, threads, kForwardThreadsPerSm);
  if (vec) block_norm_kernel<T, kVpt, true><<<grid, threads, 0, st>>>(p);
  else block_norm_kernel<T, kVpt, false><<<grid, threads, 0, st>>>(p);
  note_launch();
  return launch_status();
}
template <typename T>
hif4_status launch_norm_t(const NormParams& p, bool vec, cudaStream_t st) {
  switch (groups_per_thread(p.cols)) {
    case 1: return launch_norm<T, 1>(p, vec, st);
    case 2: return launch_norm<T, 2>(p, vec, st);
    default: return launch_norm<T, 4>(p, vec, st);
  }
}

template <typename T, int kVpt>
void launch_norm_grad(const NormGradParams& p, bool vec, bool path, int threads, cudaStream_t st) {
  if (path) {
    if (vec) block_norm_backward_kernel<T, kVpt, true, true><<<p.grid, threads, 0, st>>>(p);
    else block_norm_backward_kernel<T, kVpt, false, true><<<p.grid, threads, 0, st>>>(p);
  } else {
    if (vec) block_norm_backward_kernel<T, kVpt, true, false><<<p.grid, threads, 0, st>>>(p);
    else block_norm_backward_kernel<T, kVpt, false, false><<<p.grid, threads, 0, st>>>(p);
  }
}
template <typename T>
hif4_status launch_norm_grad_t(NormGradParams p, bool vec, cudaStream_t st) {
  const int vpt = groups_per_thread(p.cols), threads = threads_for(p.cols, vpt);
  const bool path = p.kind_post != HIF4_NORM_NONE || p.gate != nullptr;
  if (vpt == 1) launch_norm_grad<T, 1>(p, vec, path, threads, st);
  else if (vpt == 2) launch_norm_grad<T, 2>(p, vec, path, threads, st);
  else launch_norm_grad<T, 4>(p, vec, path, threads, st);
  note_launch();
  if (cudaGetLastError() != cudaSuccess) return HIF4_ERR_CUDA;
  const int planes = p.dgate ? 3 + p.grid - 1 : (p.dpre_weight || p.dpre_bias || p.dpost_weight) ? 3 : 0;
  if (planes == 0) return HIF4_OK;
  const dim3 grid(static_cast<unsigned>(ceil_div64(p.cols, kFinishCols)), static_cast<unsigned>(planes));
  norm_grad_finish_kernel<T><<<grid, kFinishCols * kFinishWays, 0, st>>>(p);
  note_launch();
  return launch_status();
}

int backward_grid(int64_t rows, int64_t cols) {
  return grid_for(rows, threads_for(cols, groups_per_thread(cols)), kBackwardThreadsPerSm);
}

}  // namespace
}  // namespace hif4

using namespace hif4;

extern "C" hif4_status hif4_block_norm(const hif4_block_norm_args* a, void* stream) {
  if (!a) return HIF4_ERR_NULL;
  if (!known_type(a->dt) || !known_type(a->dt_w) || !known_kind(a->pre) || !known_kind(a->post) ||
      (a->mode != HIF4_RNE && a->mode != HIF4_RHA))
    return HIF4_ERR_DTYPE;
  if (a->rows < 0 || a->cols < 0 || a->cols > kNormMaxCols || (a->gate && a->rows_per_gate < 1) || !(a->eps >= 0.0f) ||
      (a->y && a->pre == HIF4_NORM_NONE) || (a->pre_bias && a->pre != HIF4_NORM_LAYER) || (a->y_units && a->cols % kUnitElems != 0))
    return HIF4_ERR_SHAPE;
  if (a->rows == 0 || a->cols == 0) return HIF4_OK;
  if (!a->x || (!a->h && !a->y)) return HIF4_ERR_NULL;
  const Operand ops[] = {{a->x, a->ld_x, a->dt}, {a->residual, a->ld_residual, a->dt}, {a->gate, a->ld_gate, a->dt},
                         {a->h, a->ld_h, a->dt}, {a->y_units ? nullptr : a->y, a->ld_y, a->dt},
                         {a->post_weight, a->cols, a->dt_w}, {a->pre_weight, a->cols, a->dt_w}, {a->pre_bias, a->cols, a->dt_w}};
  bool vec;
  const hif4_status chk = check_operands(ops, 5, a->rows, a->cols, vec);
  if (chk != HIF4_OK) return chk;
  bool vec_w;
  const hif4_status chk_w = check_operands(ops + 5, 3, 1, a->cols, vec_w);
  if (chk_w != HIF4_OK) return chk_w;
  if (a->y_units && a->y && !aligned_to(a->y, 4)) return HIF4_ERR_ALIGN;
  NormParams p{};
  p.rows = a->rows; p.cols = static_cast<int>(a->cols);
  p.kind_pre = a->pre; p.kind_post = a->post; p.dt_w = a->dt_w;
  p.x = a->x; p.residual = a->residual; p.gate = a->gate;
  p.post_weight = a->post_weight; p.pre_weight = a->pre_weight; p.pre_bias = a->pre_bias;
  p.ld_x = a->ld_x; p.ld_residual = a->ld_residual; p.ld_gate = a->ld_gate; p.rows_per_gate = a->rows_per_gate;
  p.res_scale = a->res_scale; p.eps = a->eps;
  p.h = a->h; p.y = a->y; p.ld_h = a->ld_h; p.ld_y = a->ld_y;
  p.units = a->y_units ? 1 : 0; p.rha = a->mode == HIF4_RHA;
  vec = vec && vec_w;
  p.strided = vec || p.units ? 0 : 1;                    // units: eight consecutive columns per lane, whatever the access
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dt == HIF4_BF16) return launch_norm_t<__nv_bfloat16>(p, vec, st);
  if (a->dt == HIF4_FP16) return launch_norm_t<__half>(p, vec, st);
  return launch_norm_t<float>(p, vec, st);
}

extern "C" hif4_status hif4_block_norm_backward_workspace(int64_t rows, int64_t cols, size_t* bytes) {
  if (!bytes) return HIF4_ERR_NULL;
  if (rows < 0 || cols < 0 || cols > kNormMaxCols) return HIF4_ERR_SHAPE;
  *bytes = rows == 0 || cols == 0 ? 0 : static_cast<size_t>(5) * backward_grid(rows, cols) * cols * sizeof(float);
  return HIF4_OK;
}

extern "C" hif4_status hif4_block_norm_backward(const hif4_block_norm_backward_args* a, void* workspace, size_t workspace_bytes,
                                                void* stream) {
  if (!a) return HIF4_ERR_NULL;
  if (!known_type(a->dt) || !known_type(a->dt_w) || !known_kind(a->pre) || !known_kind(a->post)) return HIF4_ERR_DTYPE;
  size_t need = 0;
  const hif4_status ws = hif4_block_norm_backward_workspace(a->rows, a->cols, &need);
  if (ws != HIF4_OK) return ws;
  if ((a->gate && a->rows_per_gate < 1) || !(a->eps >= 0.0f) || (a->dy && a->pre == HIF4_NORM_NONE) ||
      (a->dpost_weight && a->post == HIF4_NORM_NONE))
    return HIF4_ERR_SHAPE;
  const bool wants_x = a->post != HIF4_NORM_NONE || a->dgate;
  const size_t vec_bytes = static_cast<size_t>(a->cols) * sizeof(float);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->rows == 0 || a->cols == 0) {                    // sums over no rows
    for (float* v : {a->dpre_weight, a->dpre_bias, a->dpost_weight})
      if (v && vec_bytes && cudaMemsetAsync(v, 0, vec_bytes, st) != cudaSuccess) return HIF4_ERR_CUDA;
    return HIF4_OK;
  }
  if ((!a->dy && !a->dh) || (a->dy && !a->h) || (wants_x && !a->x) || (a->dgate && !a->gate)) return HIF4_ERR_NULL;
  if (a->dx && a->dx == a->dresidual) return HIF4_ERR_ALIGN;
  const Operand ops[] = {{a->dy, a->ld_dy, a->dt}, {a->dh, a->ld_dh, a->dt}, {a->dy ? a->h : nullptr, a->ld_h, a->dt},
                         {wants_x ? a->x : nullptr, a->ld_x, a->dt}, {a->gate, a->ld_gate, a->dt}, {a->dx, a->ld_dx, a->dt},
                         {a->dresidual, a->ld_dresidual, a->dt}, {a->dgate, a->cols, a->dt},
                         {a->post_weight, a->cols, a->dt_w}, {a->pre_weight, a->cols, a->dt_w},
                         {a->dpre_weight, a->cols, HIF4_FP32}, {a->dpre_bias, a->cols, HIF4_FP32}, {a->dpost_weight, a->cols, HIF4_FP32}};
  bool vec, vec_w;
  const hif4_status chk = check_operands(ops, 8, a->rows, a->cols, vec);
  if (chk != HIF4_OK) return chk;
  const hif4_status chk_w = check_operands(ops + 8, 5, 1, a->cols, vec_w);
  if (chk_w != HIF4_OK) return chk_w;
  if (!workspace || workspace_bytes < need) return HIF4_ERR_WORKSPACE;
  if (!aligned_to(workspace, 256)) return HIF4_ERR_ALIGN;
  vec = vec && vec_w;
  NormGradParams p{};
  p.rows = a->rows; p.cols = static_cast<int>(a->cols);
  p.kind_pre = a->pre; p.kind_post = a->post; p.dt_w = a->dt_w;
  p.dy = a->dy; p.dh = a->dh; p.h = a->h; p.x = wants_x ? a->x : nullptr; p.gate = a->gate;
  p.post_weight = a->post_weight; p.pre_weight = a->pre_weight;
  p.ld_dy = a->ld_dy; p.ld_dh = a->ld_dh; p.ld_h = a->ld_h; p.ld_x = a->ld_x; p.ld_gate = a->ld_gate;
  p.rows_per_gate = a->gate ? a->rows_per_gate : 1;
  p.res_scale = a->res_scale; p.eps = a->eps;
  p.dx = a->dx; p.dresidual = a->dresidual; p.dgate = a->dgate; p.ld_dx = a->ld_dx; p.ld_dresidual = a->ld_dresidual;
  p.dpre_weight = a->dpre_weight; p.dpre_bias = a->dpre_bias; p.dpost_weight = a->dpost_weight;
  p.partial = static_cast<float*>(workspace);
  p.grid = backward_grid(a->rows, a->cols);
  p.strided = vec ? 0 : 1;
  if (a->dt == HIF4_BF16) return launch_norm_grad_t<__nv_bfloat16>(p, vec, st);
  if (a->dt == HIF4_FP16) return launch_norm_grad_t<__half>(p, vec, st);
  return launch_norm_grad_t<float>(p, vec, st);
}
