// hif4_block_norm / hif4_block_norm_backward -- the norms after and before a block with gate, residual and residual
// scale, and their gradients.  One pass over the matrices: a row lives in the registers of one thread block from its
// loads to its stores, the row statistics are block-wide FP32 sums, and the result can leave as HiF4 units without the
// 16-bit matrix being written.  Bound by HBM traffic (forward 6.6 - 8 bytes an element in 16 bits, backward 12).
//
// Behind the loads comes the latency of a block's instruction stream, broken at every block-wide sum, so the arithmetic runs in packed
// FP32 pairs.
// A thread owns groups of eight columns (16-byte accesses when the matrices allow them; rows at odd addresses are read in
// 16-byte words and shifted).  Blocks take contiguous runs
// of rows and keep the next row's loads in flight while they reduce the current one; weights and gates are re-read
// per row, from L1 after a block's first row.
#include "hif4_common.cuh"
#include "hif4_tc_common.cuh"
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
  int stages;               // ring depth of the bulk form
  unsigned int* error_word;
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
  int grid, light;
  int stages;
  unsigned int* error_word;
};

// Columns of a thread's group i: base .. base + 7.
struct Cols {
  int base;
  __device__ __forceinline__ explicit Cols(int i) { base = 8 * (i * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)); }
};

// Eight 16-bit elements from two neighbouring 16-byte words of which they take bytes o .. o + 15 (o even, the same for all
// threads of a row).
__device__ __forceinline__ uint4 take16(const uint4& a, const uint4& b, uint32_t o) {
  uint32_t w[5];
  switch (o >> 2) {
    case 0: w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; break;
    case 1: w[0] = a.y; w[1] = a.z; w[2] = a.w; w[3] = b.x; w[4] = b.y; break;
    case 2: w[0] = a.z; w[1] = a.w; w[2] = b.x; w[3] = b.y; w[4] = b.z; break;
    default: w[0] = a.w; w[1] = b.x; w[2] = b.y; w[3] = b.z; w[4] = b.w; break;
  }
  const uint32_t s = (o & 2u) * 8u;
  return make_uint4(__funnelshift_r(w[0], w[1], s), __funnelshift_r(w[1], w[2], s), __funnelshift_r(w[2], w[3], s), __funnelshift_r(w[3], w[4], s));
}
// A group of a row of any alignment: 16-byte loads, one or two of them, wherever those stay inside the row.
template <bool kVec, typename T>
__device__ __forceinline__ Raw8<T> load_group(const T* row, const Cols& c, int cols) {
  Raw8<T> r;
  zero8(r);
  if (kVec) {
    if (c.base < cols) r = load8(row + c.base);
    return r;
  }
  const uint32_t o = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row)) & 15u;
  if (o == 0u && c.base + 8 <= cols) return load8(row + c.base);
  if constexpr (sizeof(T) == 2) {
    if (c.base >= 8 && c.base + 16 <= cols) {
      const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row + c.base) - o);
      r.a = take16(p[0], p[1], o);
      return r;
    }
  }
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = c.base + j < cols ? to_f32(row[c.base + j]) : 0.0f;
  return pack8<T>(v);                                      // exact: the values come from T
}
// The same for stores: 16-byte ones where the row allows them, else 4-byte ones with single elements at the odd ends.
template <bool kVec, typename T>
__device__ __forceinline__ void store_group(T* row, const Cols& c, int cols, const Raw8<T>& r) {
  if (kVec) {
    if (c.base < cols) store8(row + c.base, r);
    return;
  }
  const uint32_t o = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row)) & 15u;
  if (c.base + 8 <= cols) {
    if (o == 0u) {
      store8(row + c.base, r);
      return;
    }
    if constexpr (sizeof(T) == 2) {
      const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
      uint16_t* d = reinterpret_cast<uint16_t*>(row + c.base);
      if ((o & 2u) == 0u) {
#pragma unroll
        for (int k = 0; k < 4; ++k) reinterpret_cast<uint32_t*>(d)[k] = w[k];
      } else {
        d[0] = static_cast<uint16_t>(w[0]);
#pragma unroll
        for (int k = 0; k < 3; ++k) reinterpret_cast<uint32_t*>(d + 1)[k] = __funnelshift_r(w[k], w[k + 1], 16);
        d[7] = static_cast<uint16_t>(w[3] >> 16);
      }
      return;
    }
  }
  float v[8];
  unpack8(r, v);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (c.base + j < cols) row[c.base + j] = from_f32<T>(v[j]);
}
// Column sums of a group to an FP32 row of the workspace (16-byte aligned where the columns come in groups).
template <bool kVec>
__device__ __forceinline__ void store_sums(float* row, const Cols& c, int cols, const Pairs& g) {
  store_group<kVec>(row, c, cols, raw_of<float>(g));
}
// Weights of any type as FP32; `fill` where there is no weight vector.
template <bool kVec>
__device__ __forceinline__ Pairs load_weights(const void* w, int dt_w, const Cols& c, int cols, float fill) {
  if (!w) return pairs_filled(fill);
  if (dt_w == HIF4_BF16) return pairs_of(load_group<kVec>(static_cast<const __nv_bfloat16*>(w), c, cols));
  if (dt_w == HIF4_FP16) return pairs_of(load_group<kVec>(static_cast<const __half*>(w), c, cols));
  return pairs_of(load_group<kVec>(static_cast<const float*>(w), c, cols));
}
// Sums of kN (1, 2 or 4) values over the block.  A lane halves the values it still carries at every exchange until it
// holds one, so kN values cost 5 + log2 kN exchanges per level instead of 5 kN.  `slot` alternates between calls, so
// that one barrier per call is enough: a warp can only be one call ahead of another, and then it writes the other half.
template <int kN, bool kAlwaysSync = false>
__device__ __forceinline__ void block_sums(float (&v)[kN], float (*red)[4][32], uint32_t& slot) {
  constexpr int kLanes = 32 / kN;                        // lanes that carry one value
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if constexpr (kN == 4) {
    const bool up = lane & 16;
    const float s0 = up ? v[0] : v[2], s1 = up ? v[1] : v[3];
    v[0] = (up ? v[2] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, s0, 16);
    v[1] = (up ? v[3] : v[1]) + __shfl_xor_sync(0xFFFFFFFFu, s1, 16);
  }
  if constexpr (kN >= 2) {
    const bool up = lane & kLanes;
    const float s0 = up ? v[0] : v[1];
    v[0] = (up ? v[1] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, s0, kLanes);
  }
#pragma unroll
  for (int s = kLanes / 2; s > 0; s >>= 1) v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], s);
  float total = v[0];
  if (kAlwaysSync || warps > 1) {
    const int n = lane / kLanes, k = lane % kLanes;      // value and place of this lane
    if (k == 0) red[slot & 1u][n][warp] = v[0];
    __syncthreads();
    total = 0.0f;
    for (int w = k; w < warps; w += kLanes) total += red[slot & 1u][n][w];
#pragma unroll
    for (int s = kLanes / 2; s > 0; s >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, s);
    ++slot;
  }
#pragma unroll
  for (int n = 0; n < kN; ++n) v[n] = kN == 1 ? total : __shfl_sync(0xFFFFFFFFu, total, n * kLanes);
}

// ... with a block barrier even where one warp needs none.
template <int kN>
__device__ __forceinline__ void block_sums_synced(float (&v)[kN], float (*red)[4][32], uint32_t& slot) { block_sums<kN, true>(v, red, slot); }

// What is taken from the elements of a group to centre them: the mean, but zero past the row's end, where the elements
// are zeros and have to stay that.
template <bool kVec>
__device__ __forceinline__ Pairs centre(float mean, const Cols& c, int cols) {
  if (kVec || c.base + 8 <= cols || c.base >= cols) return pairs_filled(c.base < cols ? mean : 0.0f);
  Pairs m;
#pragma unroll
  for (int j = 0; j < 4; ++j) m.p[j] = make_float2(c.base + 2 * j < cols ? mean : 0.0f, c.base + 2 * j + 1 < cols ? mean : 0.0f);
  return m;
}
template <bool kVec>
__device__ __forceinline__ void subtract_mean(Pairs& g, float mean, const Cols& c, int cols) {
  const Pairs m = centre<kVec>(-mean, c, cols);
#pragma unroll
  for (int j = 0; j < 4; ++j) g.p[j] = add2(g.p[j], m.p[j]);
}
template <int kVpt>
__device__ __forceinline__ float sum_of(const Pairs (&v)[kVpt]) {
  float2 s = both(0.0f);
#pragma unroll
  for (int i = 0; i < kVpt; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s = add2(s, v[i].p[j]);
  return s.x + s.y;
}
template <int kVpt>
__device__ __forceinline__ float dot_of(const Pairs (&a)[kVpt], const Pairs (&b)[kVpt]) {
  float2 s = both(0.0f);
#pragma unroll
  for (int i = 0; i < kVpt; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s = fma2(a[i].p[j], b[i].p[j], s);
  return s.x + s.y;
}
// Centres a row held as v (LAYER only) and returns 1 / sqrt(mean of squares + eps).
template <bool kVec, int kVpt>
__device__ __forceinline__ float normalise(Pairs (&v)[kVpt], int kind, const NormParams& p, float inv_cols, float (*red)[4][32], uint32_t& slot) {
  if (kind == HIF4_NORM_LAYER) {
    float s[1] = {sum_of(v)};
    block_sums(s, red, slot);
#pragma unroll
    for (int i = 0; i < kVpt; ++i) subtract_mean<kVec>(v[i], s[0] * inv_cols, Cols(i), p.cols);
  }
  float s[1] = {dot_of(v, v)};
  block_sums(s, red, slot);
  return rsqrtf(fmaf(s[0], inv_cols, p.eps));
}

template <typename T, int kVpt, bool kVec>
__global__ void __launch_bounds__(kVpt <= 2 ? 320 : 512)
block_norm_kernel(const NormParams p) {
  __shared__ float red[2][4][32];
  uint32_t slot = 0;
  grid_launch_next();
  grid_wait();
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows / gridDim.x;
  const int64_t row1 = (static_cast<int64_t>(blockIdx.x) + 1) * p.rows / gridDim.x;
  const T* x = static_cast<const T*>(p.x);
  const T* res = static_cast<const T*>(p.residual);
  Raw8<T> xr[kVpt], rr[kVpt];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i);
      xr[i] = load_group<kVec>(x + row * p.ld_x, c, p.cols);
      if (res) rr[i] = load_group<kVec>(res + row * p.ld_residual, c, p.cols);
      else zero8(rr[i]);
    }
  };
  const float inv_cols = 1.0f / static_cast<float>(p.cols);
  if (row0 < row1) fetch(row0);
  // gates: one row of them serves rows_per_gate rows
  Raw8<T> gr[kVpt];
  int64_t gate_row = p.gate ? row0 / p.rows_per_gate : 0, gate_end = row0;
  for (int64_t row = row0; row < row1; ++row) {
    if (p.gate && row == gate_end) {
      if (row != row0) ++gate_row;
      gate_end = (gate_row + 1) * p.rows_per_gate;
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
        gr[i] = load_group<kVec>(static_cast<const T*>(p.gate) + gate_row * p.ld_gate, Cols(i), p.cols);
    }
    Pairs v[kVpt], r[kVpt];
#pragma unroll
    for (int i = 0; i < kVpt; ++i) { v[i] = pairs_of(xr[i]); r[i] = pairs_of(rr[i]); }
    if (row + 1 < row1) fetch(row + 1);
    if (p.kind_post != HIF4_NORM_NONE) {
      const float2 rstd = both(normalise<kVec>(v, p.kind_post, p, inv_cols, red, slot));
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        const Cols c(i);
        const Pairs w = load_weights<kVec>(p.post_weight, p.dt_w, c, p.cols, 1.0f);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(mul2(v[i].p[j], rstd), w.p[j]);
      }
    }
    if (p.gate) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        const Pairs g = pairs_of(gr[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], g.p[j]);
      }
    }
    if (res) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].p[j] = fma2(both(p.res_scale), r[i].p[j], v[i].p[j]);
    }
    if (p.h) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
        store_group<kVec>(static_cast<T*>(p.h) + row * p.ld_h, Cols(i), p.cols, raw_of<T>(v[i]));
    }
    if (!p.y) continue;
    const float2 rstd = both(normalise<kVec>(v, p.kind_pre, p, inv_cols, red, slot));
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i);
      Pairs w = load_weights<kVec>(p.pre_weight, p.dt_w, c, p.cols, 1.0f);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(mul2(v[i].p[j], rstd), w.p[j]);
      if (p.pre_bias) {
        w = load_weights<kVec>(p.pre_bias, p.dt_w, c, p.cols, 0.0f);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].p[j] = add2(v[i].p[j], w.p[j]);
      }
      const Raw8<T> out = raw_of<T>(v[i]);
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
  grid_launch_next();
  grid_wait();
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows / gridDim.x;
  const int64_t row1 = (static_cast<int64_t>(blockIdx.x) + 1) * p.rows / gridDim.x;
  const float inv_cols = 1.0f / static_cast<float>(p.cols);
  const bool pre_layer = p.kind_pre == HIF4_NORM_LAYER, post_layer = p.kind_post == HIF4_NORM_LAYER;
  const bool post = kPath && p.kind_post != HIF4_NORM_NONE;
  Pairs dw[kVpt], db[kVpt], dwp[kPath ? kVpt : 1], dg[kPath ? kVpt : 1];
#pragma unroll
  for (int i = 0; i < kVpt; ++i) {
    dw[i] = db[i] = pairs_filled(0.0f);
    if (kPath) dwp[i] = dg[i] = pairs_filled(0.0f);
  }
  int64_t group = kPath && p.gate ? row0 / p.rows_per_gate : 0;
  const T* m_dy = static_cast<const T*>(p.dy);
  const T* m_dh = static_cast<const T*>(p.dh);
  const T* m_h = p.dy ? static_cast<const T*>(p.h) : nullptr;
  const T* m_x = kPath ? static_cast<const T*>(p.x) : nullptr;
  Raw8<T> gr[kPath ? kVpt : 1];
  int64_t gate_row = group, gate_end = row0;
  for (int64_t row = row0; row < row1; ++row) {
    if (kPath && p.gate && row == gate_end) {
      if (row != row0) ++gate_row;
      gate_end = (gate_row + 1) * p.rows_per_gate;
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
        gr[i] = load_group<kVec>(static_cast<const T*>(p.gate) + gate_row * p.ld_gate, Cols(i), p.cols);
    }
    Pairs a[kVpt], t[kVpt], x[kPath ? kVpt : 1], dy[kVpt];      // h, gradient of h, x, dy
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i);
      Raw8<T> z;
      zero8(z);
      a[i] = pairs_of(m_h ? load_group<kVec>(m_h + row * p.ld_h, c, p.cols) : z);
      dy[i] = pairs_of(m_dy ? load_group<kVec>(m_dy + row * p.ld_dy, c, p.cols) : z);
      t[i] = pairs_of(m_dh ? load_group<kVec>(m_dh + row * p.ld_dh, c, p.cols) : z);
      if (kPath) x[i] = pairs_of(m_x ? load_group<kVec>(m_x + row * p.ld_x, c, p.cols) : z);
    }
    if (pre_layer || post_layer) {
      float s1[2] = {sum_of(a), 0.0f};
      if constexpr (kPath) s1[1] = sum_of(x);
      block_sums(s1, red, slot);
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        const Cols c(i);
        if (pre_layer) subtract_mean<kVec>(a[i], s1[0] * inv_cols, c, p.cols);
        if (kPath && post_layer) subtract_mean<kVec>(x[i], s1[1] * inv_cols, c, p.cols);
      }
    }
    // sums over the row: (h - mean)^2, dn (h - mean), (x - mean_x)^2, dn; columns past the end hold zero gradients
    float s2[4] = {dot_of(a, a), 0.0f, 0.0f, 0.0f};
    if constexpr (kPath) s2[2] = dot_of(x, x);
    Pairs dn[kVpt];
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i);
      const Pairs w = load_weights<kVec>(p.pre_weight, p.dt_w, c, p.cols, 1.0f);
#pragma unroll
      for (int j = 0; j < 4; ++j) dn[i].p[j] = mul2(dy[i].p[j], w.p[j]);
    }
    s2[1] = dot_of(dn, a);
    if (pre_layer) s2[3] = sum_of(dn);
    if (kPath || pre_layer) {
      block_sums(s2, red, slot);
    } else {
      float s[2] = {s2[0], s2[1]};
      block_sums(s, red, slot);
      s2[0] = s[0]; s2[1] = s[1];
    }
    const float rstd = rsqrtf(fmaf(s2[0], inv_cols, p.eps));
    const float m1 = -s2[1] * rstd * inv_cols, m0 = -s2[3] * inv_cols;
    const float rstd_x = post ? rsqrtf(fmaf(s2[2], inv_cols, p.eps)) : 1.0f;
    float2 s3a = both(0.0f), s3b = both(0.0f);
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Cols c(i);
      if (p.dy) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 n = mul2(a[i].p[j], both(rstd));
          dw[i].p[j] = fma2(dy[i].p[j], n, dw[i].p[j]);
          float2 d = fma2(n, both(m1), dn[i].p[j]);
          if (pre_layer) {
            db[i].p[j] = add2(db[i].p[j], dy[i].p[j]);
            d = add2(d, both(m0));
          }
          t[i].p[j] = fma2(both(rstd), d, t[i].p[j]);
        }
      }
      if (p.dresidual) {
        Pairs o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o.p[j] = mul2(both(p.res_scale), t[i].p[j]);
        store_group<kVec>(static_cast<T*>(p.dresidual) + row * p.ld_dresidual, c, p.cols, raw_of<T>(o));
      }
      if (kPath) {
        if (pre_layer) {                                 // the shift by mean(dn) reached the columns past the end
          const Pairs in = centre<kVec>(1.0f, c, p.cols);
#pragma unroll
          for (int j = 0; j < 4; ++j) t[i].p[j] = mul2(t[i].p[j], in.p[j]);
        }
        const Pairs g = p.gate ? pairs_of(gr[i]) : pairs_filled(1.0f);
        Pairs wp = pairs_filled(1.0f);
        if (post) {
          wp = load_weights<kVec>(p.post_weight, p.dt_w, c, p.cols, 1.0f);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 xn = mul2(x[i].p[j], both(rstd_x));         // x itself without a post norm
          const float2 dp = mul2(t[i].p[j], g.p[j]);
          dg[i].p[j] = fma2(t[i].p[j], mul2(xn, wp.p[j]), dg[i].p[j]);
          dwp[i].p[j] = fma2(dp, xn, dwp[i].p[j]);
          x[i].p[j] = xn;
          t[i].p[j] = mul2(dp, wp.p[j]);
          s3a = fma2(t[i].p[j], xn, s3a);
          s3b = add2(s3b, t[i].p[j]);
        }
      }
    }
    if (post && p.dx) {
      float s3[2] = {s3a.x + s3a.y, s3b.x + s3b.y};
      block_sums(s3, red, slot);
      const float2 q1 = both(-s3[0] * inv_cols), q0 = both(post_layer ? -s3[1] * inv_cols : 0.0f);
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) t[i].p[j] = mul2(both(rstd_x), add2(fma2(x[i].p[j], q1, t[i].p[j]), q0));
    }
    if (p.dx) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
        store_group<kVec>(static_cast<T*>(p.dx) + row * p.ld_dx, Cols(i), p.cols, raw_of<T>(t[i]));
    }
    if (kPath && p.dgate) {
      const int64_t end = (group + 1) * p.rows_per_gate < p.rows ? (group + 1) * p.rows_per_gate : p.rows;
      if (row + 1 == end || row + 1 == row1) {
        const bool starts_here = group * p.rows_per_gate >= row0, ends_here = row + 1 == end;
#pragma unroll
        for (int i = 0; i < kVpt; ++i) {
          const Cols c(i);
          if (starts_here && ends_here) {
            store_group<kVec>(static_cast<T*>(p.dgate) + group * p.cols, c, p.cols, raw_of<T>(dg[i]));
          } else {
            float* part = p.partial + (static_cast<int64_t>(starts_here ? 4 : 3) * gridDim.x + blockIdx.x) * p.cols;
            store_sums<kVec>(part, c, p.cols, dg[i]);
          }
          dg[i] = pairs_filled(0.0f);
        }
        ++group;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kVpt; ++i) {
    const Cols c(i);
    float* part = p.partial + static_cast<int64_t>(blockIdx.x) * p.cols;
    const int64_t plane = static_cast<int64_t>(gridDim.x) * p.cols;
    if (p.dpre_weight) store_sums<kVec>(part, c, p.cols, dw[i]);
    if (p.dpre_bias) store_sums<kVec>(part + plane, c, p.cols, db[i]);
    if (kPath && p.dpost_weight) store_sums<kVec>(part + 2 * plane, c, p.cols, dwp[i]);
  }
}

#include "hif4_block_norm_bulk.cuh"

// blockIdx.y 0..2: one of the weight gradients, summed over the blocks of the pass above.  From 3 on: the groups of gates
// that run over a boundary between two blocks, found from the group or from the boundary, whichever there are fewer of.
constexpr int kFinishCols = 32, kFinishWays = 16;
template <typename T>
__global__ void __launch_bounds__(kFinishCols * kFinishWays)
norm_grad_finish_kernel(const NormGradParams p, int by_group) {
  __shared__ float part[kFinishWays][kFinishCols + 1];
  const int lane = threadIdx.x & (kFinishCols - 1), col = blockIdx.x * kFinishCols + lane, way = threadIdx.x / kFinishCols;
  const int64_t plane = static_cast<int64_t>(p.grid) * p.cols;
  const float* src;                                      // parts first .. last of a plane, and one more in front
  int first = 0, last = p.grid;
  const float* front = nullptr;
  int64_t group = 0;
  if (blockIdx.y < 3) {
    if (!(blockIdx.y == 0 ? p.dpre_weight : blockIdx.y == 1 ? p.dpre_bias : p.dpost_weight)) return;
    src = p.partial + blockIdx.y * plane;
  } else {
    const int k = static_cast<int>(blockIdx.y) - 3;
    group = by_group ? k : static_cast<int64_t>(k + 1) * p.rows / p.grid / p.rows_per_gate;
    const int64_t g0 = group * p.rows_per_gate, g1 = g0 + p.rows_per_gate < p.rows ? g0 + p.rows_per_gate : p.rows;
    const int b0 = static_cast<int>(((g0 + 1) * p.grid - 1) / p.rows), b1 = static_cast<int>((g1 * p.grid - 1) / p.rows);   // blocks of its ends
    if (b0 == b1 || (!by_group && b0 != k)) return;      // inside one block, or another boundary's
    src = p.partial + 3 * plane;
    front = p.partial + 4 * plane + static_cast<int64_t>(b0) * p.cols;
    first = b0 + 1; last = b1 + 1;
  }
  float s = 0.0f;
  if (col < p.cols) {
    if (front && way == 0) s = front[col];
    for (int b = first + way; b < last; b += kFinishWays) s += src[static_cast<int64_t>(b) * p.cols + col];
  }
  part[way][lane] = s;
  __syncthreads();
  if (way != 0 || col >= p.cols) return;
#pragma unroll
  for (int w = 1; w < kFinishWays; ++w) s += part[w][lane];
  if (front) static_cast<T*>(p.dgate)[group * p.cols + col] = from_f32<T>(s);
  else (blockIdx.y == 0 ? p.dpre_weight : blockIdx.y == 1 ? p.dpre_bias : p.dpost_weight)[col] = s;
}

// ------------------------------------------------------------------------------------------------------- host side
// Groups of eight columns per thread.  Forward: two while 320 threads reach the row's end (8192 x 5120, two blocks an SM:
// 63 us; one group 78 us, four 68 us), more beyond.  Backward: the column sums take 32 registers a group, so one while
// 512 threads reach (4000 x 4096 with post norm and gates: 69 us, two groups 70 us and more spills beyond).
int groups_forward(int64_t cols) { return cols <= 1024 ? 1 : cols <= 5120 ? 2 : cols <= 16384 ? 4 : 8; }
int groups_backward(int64_t cols) { return cols <= 4096 ? 1 : cols <= 8192 ? 2 : 4; }
int threads_for(int64_t cols, int vpt) {
  const int64_t t = ceil_div64(ceil_div64(cols, 8), vpt);
  return static_cast<int>(ceil_div64(t, 32) * 32);
}
// Shared memory that the rings of an SM's blocks share, and the most stages of one.
constexpr int kRingBytes = 200 * 1024, kMaxRing = 8;
// Blocks per SM from the thread count alone: the sums of the backward pass run block by block, and their order must depend
// on nothing but the sizes.  The forward pass also asks how many blocks the registers admit (launch_norm).
int blocks_per_sm(int threads, int threads_per_sm) {
  const int b = threads_per_sm / threads;
  return b < 1 ? 1 : b > 16 ? 16 : b;
}
int grid_for(int64_t rows, int threads, int threads_per_sm) {
  const int64_t g = static_cast<int64_t>(sm_count()) * blocks_per_sm(threads, threads_per_sm);
  return static_cast<int>(rows < g ? rows : g);
}
constexpr int kForwardThreadsPerSm = 768, kBackwardThreadsPerSm = 512;

// Stages of the ring beside `weights` bytes of weights, or 0: rows too short, too few of them per block, or too wide for two stages.
int ring_stages(int64_t rows, int grid, int per_sm, size_t stage_bytes, size_t weights) {
  if (stage_bytes < 4096 || rows < 2 * static_cast<int64_t>(grid) || weights + 2 * stage_bytes > kRingBytes / static_cast<size_t>(per_sm)) return 0;
  const size_t n = (kRingBytes / per_sm - weights) / stage_bytes;
  return n < 2 ? 0 : n > kMaxRing ? kMaxRing : static_cast<int>(n);
}

size_t type_size(int dt) { return dt == HIF4_FP32 ? 4 : 2; }
bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
template <typename T> int type_of() { return HIF4_BF16; }
template <> int type_of<__half>() { return HIF4_FP16; }
template <> int type_of<float>() { return HIF4_FP32; }
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

template <typename T, typename W, int kVpt>
hif4_status launch_norm_bulk(const NormParams& p, int grid, int threads, size_t smem, cudaStream_t st) {
  static uint64_t smem_opt_in = 0;
  if (!ensure_dynamic_smem(block_norm_bulk_kernel<T, W, kVpt>, kRingBytes + 128, smem_opt_in)) return HIF4_ERR_CUDA;
  return launch_overlapped(block_norm_bulk_kernel<T, W, kVpt>, grid, threads, smem, st, p);
}
template <typename T, int kVpt>
hif4_status launch_norm(NormParams p, bool vec, cudaStream_t st) {
  const int threads = threads_for(p.cols, kVpt);
  const bool wide = p.dt_w == HIF4_FP32;
  const size_t stage = static_cast<size_t>(p.cols) * sizeof(T) * (p.residual ? 2 : 1);
  const size_t weights = static_cast<size_t>(p.cols) * type_size(p.dt_w) * ((p.y ? 1 : 0) + (p.kind_post != HIF4_NORM_NONE ? 1 : 0) + (p.pre_bias ? 1 : 0));
  if (vec && (wide || p.dt_w == type_of<T>())) {
    // blocks that the registers let run side by side: a block that had to wait for another's end would double the time
    int fits = 1;
    const cudaError_t e = wide ? cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fits, block_norm_bulk_kernel<T, float, kVpt>, threads, 0)
                               : cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fits, block_norm_bulk_kernel<T, T, kVpt>, threads, 0);
    if (e != cudaSuccess) return HIF4_ERR_CUDA;
    const int want = blocks_per_sm(threads, kForwardThreadsPerSm), per_sm = fits < 1 ? 1 : fits < want ? fits : want;
    const int64_t all = static_cast<int64_t>(sm_count()) * per_sm;
    const int grid = static_cast<int>(p.rows < all ? p.rows : all);
    p.stages = ring_stages(p.rows, grid, per_sm, stage, weights);
    if (p.stages > 0) {
      p.error_word = device_error_word();
      if (!p.error_word) return HIF4_ERR_CUDA;
      const size_t smem = 128 + weights + p.stages * stage;
      return wide ? launch_norm_bulk<T, float, kVpt>(p, grid, threads, smem, st) : launch_norm_bulk<T, T, kVpt>(p, grid, threads, smem, st);
    }
  }
  const int grid = grid_for(p.rows, threads, kForwardThreadsPerSm);
  if (vec) return launch_overlapped(block_norm_kernel<T, kVpt, true>, grid, threads, 0, st, p);
  return launch_overlapped(block_norm_kernel<T, kVpt, false>, grid, threads, 0, st, p);
}
template <typename T>
hif4_status launch_norm_t(const NormParams& p, bool vec, cudaStream_t st) {
  switch (groups_forward(p.cols)) {
    case 1: return launch_norm<T, 1>(p, vec, st);
    case 2: return launch_norm<T, 2>(p, vec, st);
    case 4: return launch_norm<T, 4>(p, vec, st);
    default: return launch_norm<T, 8>(p, vec, st);
  }
}

template <typename T, typename W, int kVpt, bool kPath, bool kLayer>
hif4_status launch_norm_grad_bulk(const NormGradParams& p, int threads, size_t smem, cudaStream_t st) {
  static uint64_t smem_opt_in = 0;
  if (!ensure_dynamic_smem(block_norm_backward_bulk_kernel<T, W, kVpt, kPath, kLayer>, kRingBytes + 128, smem_opt_in)) return HIF4_ERR_CUDA;
  return launch_overlapped(block_norm_backward_bulk_kernel<T, W, kVpt, kPath, kLayer>, p.grid, threads, smem, st, p);
}
template <typename T, int kVpt, bool kPath>
hif4_status launch_norm_grad(NormGradParams p, bool vec, int threads, cudaStream_t st) {
  const bool wide = p.dt_w == HIF4_FP32;
  const int mats = (p.dy ? 2 : 0) + (p.dh ? 1 : 0) + (kPath && p.x ? 1 : 0);
  const size_t stage = static_cast<size_t>(p.cols) * sizeof(T) * mats;
  const size_t weights = static_cast<size_t>(p.cols) * (type_size(p.dt_w) * ((p.dy ? 1 : 0) + (p.kind_post != HIF4_NORM_NONE ? 1 : 0)) +
                                                        (p.gate && p.kind_post != HIF4_NORM_NONE ? 4 : 0));      // and the post weight's sums
  p.stages = vec && (wide || p.dt_w == type_of<T>()) ? ring_stages(p.rows, p.grid, blocks_per_sm(threads, p.light && kVpt == 1 ? 2 * kBackwardThreadsPerSm : kBackwardThreadsPerSm), stage, weights) : 0;
  if (p.stages > 0) {
    p.error_word = device_error_word();
    if (!p.error_word) return HIF4_ERR_CUDA;
    const size_t smem = 128 + weights + p.stages * stage;
    // (dbias of an RMS norm is refused, so only a LAYER norm has one)
    const bool layer = p.kind_pre == HIF4_NORM_LAYER || p.kind_post == HIF4_NORM_LAYER;
    if (layer) return wide ? launch_norm_grad_bulk<T, float, kVpt, kPath, true>(p, threads, smem, st) : launch_norm_grad_bulk<T, T, kVpt, kPath, true>(p, threads, smem, st);
    return wide ? launch_norm_grad_bulk<T, float, kVpt, kPath, false>(p, threads, smem, st) : launch_norm_grad_bulk<T, T, kVpt, kPath, false>(p, threads, smem, st);
  }
  if (vec) return launch_overlapped(block_norm_backward_kernel<T, kVpt, true, kPath>, p.grid, threads, 0, st, p);
  return launch_overlapped(block_norm_backward_kernel<T, kVpt, false, kPath>, p.grid, threads, 0, st, p);
}
template <typename T, int kVpt>
hif4_status launch_norm_grad(const NormGradParams& p, bool vec, int threads, cudaStream_t st) {
  if (p.kind_post != HIF4_NORM_NONE || p.gate) return launch_norm_grad<T, kVpt, true>(p, vec, threads, st);
  return launch_norm_grad<T, kVpt, false>(p, vec, threads, st);
}
template <typename T>
hif4_status launch_norm_grad_t(const NormGradParams& p, bool vec, cudaStream_t st) {
  const int vpt = groups_backward(p.cols), threads = threads_for(p.cols, vpt);
  const hif4_status s = vpt == 1   ? launch_norm_grad<T, 1>(p, vec, threads, st)
                        : vpt == 2 ? launch_norm_grad<T, 2>(p, vec, threads, st) : launch_norm_grad<T, 4>(p, vec, threads, st);
  if (s != HIF4_OK) return s;
  int planes = p.dpre_weight || p.dpre_bias || p.dpost_weight ? 3 : 0, by_group = 0;
  if (p.dgate) {
    const int64_t groups = ceil_div64(p.rows, p.rows_per_gate);
    by_group = groups < p.grid - 1;
    planes = 3 + (by_group ? static_cast<int>(groups) : p.grid - 1);
  }
  if (planes == 0) return HIF4_OK;
  const dim3 grid(static_cast<unsigned>(ceil_div64(p.cols, kFinishCols)), static_cast<unsigned>(planes));
  norm_grad_finish_kernel<T><<<grid, kFinishCols * kFinishWays, 0, st>>>(p, by_group);
  note_launch();
  return launch_status();
}

// Blocks of the backward pass.  `light`: RMS norm alone, whose 61 registers a thread (one group) let twice the threads run
// (8192 x 4096: 76 us with one block an SM).
int backward_grid(int64_t rows, int64_t cols, bool light) {
  const int vpt = groups_backward(cols);
  return grid_for(rows, threads_for(cols, vpt), light && vpt == 1 ? 2 * kBackwardThreadsPerSm : kBackwardThreadsPerSm);
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
  p.ld_x = a->ld_x; p.ld_residual = a->ld_residual; p.ld_gate = a->ld_gate;
  p.rows_per_gate = a->rows_per_gate < a->rows ? a->rows_per_gate : a->rows;      // (no product with it overflows)
  p.res_scale = a->res_scale; p.eps = a->eps;
  p.h = a->h; p.y = a->y; p.ld_h = a->ld_h; p.ld_y = a->ld_y;
  p.units = a->y_units ? 1 : 0; p.rha = a->mode == HIF4_RHA;
  vec = vec && vec_w;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dt == HIF4_BF16) return launch_norm_t<__nv_bfloat16>(p, vec, st);
  if (a->dt == HIF4_FP16) return launch_norm_t<__half>(p, vec, st);
  return launch_norm_t<float>(p, vec, st);
}

extern "C" hif4_status hif4_block_norm_backward_workspace(int64_t rows, int64_t cols, size_t* bytes) {
  if (!bytes) return HIF4_ERR_NULL;
  if (rows < 0 || cols < 0 || cols > kNormMaxCols) return HIF4_ERR_SHAPE;
  *bytes = rows == 0 || cols == 0 ? 0 : static_cast<size_t>(5) * backward_grid(rows, cols, true) * cols * sizeof(float);
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
      (a->dpost_weight && a->post == HIF4_NORM_NONE) || (a->dpre_bias && a->pre != HIF4_NORM_LAYER))
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
  if (!a->dx && !a->dresidual && !a->dgate && !a->dpre_weight && !a->dpre_bias && !a->dpost_weight) return HIF4_OK;
  vec = vec && vec_w;
  NormGradParams p{};
  p.rows = a->rows; p.cols = static_cast<int>(a->cols);
  p.kind_pre = a->pre; p.kind_post = a->post; p.dt_w = a->dt_w;
  p.dy = a->dy; p.dh = a->dh; p.h = a->h; p.x = wants_x ? a->x : nullptr; p.gate = a->gate;
  p.post_weight = a->post_weight; p.pre_weight = a->pre_weight;
  p.ld_dy = a->ld_dy; p.ld_dh = a->ld_dh; p.ld_h = a->ld_h; p.ld_x = a->ld_x; p.ld_gate = a->ld_gate;
  p.rows_per_gate = !a->gate ? 1 : a->rows_per_gate < a->rows ? a->rows_per_gate : a->rows;      // (no product with it overflows)
  p.res_scale = a->res_scale; p.eps = a->eps;
  p.dx = a->dx; p.dresidual = a->dresidual; p.dgate = a->dgate; p.ld_dx = a->ld_dx; p.ld_dresidual = a->ld_dresidual;
  p.dpre_weight = a->dpre_weight; p.dpre_bias = a->dpre_bias; p.dpost_weight = a->dpost_weight;
  p.partial = static_cast<float*>(workspace);
  p.light = a->post == HIF4_NORM_NONE && !a->gate && a->pre != HIF4_NORM_LAYER;
  p.grid = backward_grid(a->rows, a->cols, p.light);
  if (a->dt == HIF4_BF16) return launch_norm_grad_t<__nv_bfloat16>(p, vec, st);
  if (a->dt == HIF4_FP16) return launch_norm_grad_t<__half>(p, vec, st);
  return launch_norm_grad_t<float>(p, vec, st);
}
