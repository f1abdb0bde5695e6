// The linear layer with its epilogue on CTA pairs: 256 x 256 accumulator tile per pair of SMs (tcgen05.mma
// cta_group::2), operands decoded from packed units as in the FP32 GEMM of hif4_gemm_tc2.cu, whose stages, barriers and
// schedule this kernel shares.  What differs:
//   - B rows.  Gated: rank 0 decodes 128 rows of W, rank 1 the same 128 rows of W_up, so that a row of the tile has the
//     gate products in columns 0..127 and the up products of the same outputs in columns 128..255 of one TMEM lane, and
//     the thread that reads both finishes the output.
//   - Loads.  TMA needs K % 256 == 0 and 16-byte aligned units; otherwise the producer warp copies the 144-byte row
//     chunks word by word (cp.async, zeros past the last unit), which costs it 288 instructions per K = 256 chunk
//     beside the decode warps' 6000.
//   - Rows past M and columns past N are not decoded: their accumulators are garbage that no one reads (a row of the
//     product depends on its own row of A only), and few rows leave the decode warps to the weights.
//   - Epilogue.  Bias, activation, product, residual in FP32 on 16 columns of a row at a time; one rounding; 64-byte
//     rows staged in shared memory and written with TMA stores, or 64-column rows converted to units there by eight
//     lanes each.  The gradient form writes dZ (dG, dU) as BF16 parts for the product that follows, and FP32 column
//     sums per 32 rows for the bias gradients.
//   - Tiles shared along K pass FP32 partial sums through the workspace (the epilogue is not linear, so nothing can be
//     added in place): slice s adds its part to what slice s - 1 left and the last slice finishes the tile, always in
//     this order.
#pragma once
#include "hif4_activation.cuh"
#include "hif4_gemm_internal.cuh"
#include "hif4_linear_internal.cuh"
#include "hif4_tc2_dense.cuh"
#include "hif4_vec8.cuh"

namespace hif4 {
namespace {

constexpr int kSlabBytes = 32 * 64;                   // 32 rows of one epilogue warp x 64 bytes
constexpr int kStageOutBytes = 4 * 2 * kSlabBytes;    // 4 warps x 2 buffers (or one buffer of 32 x 128 bytes for units)
constexpr int kLinSmemBytes = 1024 /*alignment slack*/ + kDecStages * kDecStageBytes + kRawStages * kRawStageBytes + kStageOutBytes +
                              256 /*barriers*/ + 1024 /*spread table*/;
constexpr uint32_t kLinInstrDesc = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(kPairN >> 3) << 17) |
                                   (static_cast<uint32_t>(kPairM >> 4) << 24);

// Sixteen consecutive elements of a row as FP32; `vec`: 16-byte accesses are aligned and inside the row.
template <typename T>
__device__ __forceinline__ void load16(const T* p, bool vec, int valid, float (&v)[16]) {
  if (vec) {
    float a[8], b[8];
    unpack8(load8(p), a);
    unpack8(load8(p + 8), b);
#pragma unroll
    for (int e = 0; e < 8; ++e) { v[e] = a[e]; v[8 + e] = b[e]; }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = e < valid ? to_f32(p[e]) : 0.0f;
  }
}
__device__ __forceinline__ void activate16(float (&v)[16], int act) {
  switch (act) {
#define HIF4_ACT_CASE(kind) \
  case kind:                \
    _Pragma("unroll") for (int e = 0; e < 16; ++e) v[e] = activate(v[e], kind); \
    break;
    HIF4_ACT_CASE(HIF4_ACT_RELU)
    HIF4_ACT_CASE(HIF4_ACT_SILU)
    HIF4_ACT_CASE(HIF4_ACT_GELU)
    HIF4_ACT_CASE(HIF4_ACT_GELU_TANH)
#undef HIF4_ACT_CASE
    default: break;
  }
}
// a = act(z), z = act'(z)
__device__ __forceinline__ void activate_slope16(float (&z)[16], float (&a)[16], int act) {
  switch (act) {
#define HIF4_ACT_CASE(kind) \
  case kind:                \
    _Pragma("unroll") for (int e = 0; e < 16; ++e) { float s; activate_slope(z[e], kind, a[e], s); z[e] = s; } \
    break;
    HIF4_ACT_CASE(HIF4_ACT_RELU)
    HIF4_ACT_CASE(HIF4_ACT_SILU)
    HIF4_ACT_CASE(HIF4_ACT_GELU)
    HIF4_ACT_CASE(HIF4_ACT_GELU_TANH)
#undef HIF4_ACT_CASE
    default:
#pragma unroll
      for (int e = 0; e < 16; ++e) { a[e] = z[e]; z[e] = 1.0f; }
  }
}
// Sums of the 16 columns over the 32 rows of a warp (lane = row), halving the columns a lane still owns at every step:
// lane l ends with column (l >> 1) & 15 ... of the order below, both lanes of a pair with the same sum.
__device__ __forceinline__ float column_sum16(const float (&v)[16], int lane) {
  float t[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) t[e] = v[e];
#pragma unroll
  for (int w = 16; w > 1; w >>= 1) {                     // columns owned before the step; partner lane ^ w
    const bool up = (lane & w) != 0;
#pragma unroll
    for (int e = 0; e < w / 2; ++e) {
      const float send = up ? t[e] : t[e + w / 2];
      const float keep = up ? t[e + w / 2] : t[e];
      t[e] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, w);
    }
  }
  return t[0] + __shfl_xor_sync(0xFFFFFFFFu, t[0], 1);
}
// The column whose sum column_sum16 leaves in `lane`: bit w of the lane number chose the upper half at width w.
__device__ __forceinline__ int column_of_lane(int lane) { return (lane & 16 ? 8 : 0) + (lane & 8 ? 4 : 0) + (lane & 4 ? 2 : 0) + (lane & 2 ? 1 : 0); }

// BF16 parts of 16 values: part 0 holds the leading 8 bits, part 1 what is left of them.
template <int kParts>
__device__ __forceinline__ void store_parts(const float (&v)[16], __nv_bfloat16* dst, int64_t plane, int64_t room) {
  float rest[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) rest[e] = v[e];
#pragma unroll
  for (int part = 0; part < kParts; ++part) {
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = pack2(rest[2 * e], rest[2 * e + 1], __nv_bfloat16());
      if (part + 1 < kParts) {
        rest[2 * e] -= __uint_as_float(w[e] << 16);
        rest[2 * e + 1] -= __uint_as_float(w[e] & 0xFFFF0000u);
      }
    }
    uint4* q = reinterpret_cast<uint4*>(dst + part * plane);
    if (room > 0) q[0] = make_uint4(w[0], w[1], w[2], w[3]);       // the row pitch is a multiple of eight elements
    if (room > 8) q[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// kGated: two projections.  kGrad: the gradient form.  T: type of bias, residual, Y and dY.
template <bool kGated, bool kGrad, typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_tc2_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                  const __grid_constant__ CUtensorMap tmB2, const __grid_constant__ CUtensorMap tmY, const LinearParams p) {
  constexpr int kOutCols = kGated ? kPairN / 2 : kPairN;             // outputs per tile row
  constexpr int kSlabCols = 64 / sizeof(T);                          // outputs per staged 64-byte row
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t dec_base = smem_base;
  const uint32_t raw_base = dec_base + kDecStages * kDecStageBytes;
  const uint32_t out_base = raw_base + kRawStages * kRawStageBytes;
  const uint32_t bar_base = out_base + kStageOutBytes;
  const uint32_t raw_full = bar_base, raw_empty = bar_base + 16, dec_full = bar_base + 32, dec_empty = bar_base + 64,
                 tmem_full = bar_base + 96, tmem_empty = bar_base + 112;
  uint8_t* gen_base = smem_raw + (smem_base - smem_u32(smem_raw));
  volatile uint32_t* tmem_ptr_smem = reinterpret_cast<volatile uint32_t*>(gen_base + (bar_base - smem_base) + 128);
  volatile uint32_t* abort_flag = tmem_ptr_smem + 1;
  const uint32_t lut = bar_base + 256;
  if (threadIdx.x < 256)
    reinterpret_cast<uint32_t*>(gen_base + (lut - smem_base))[threadIdx.x] = spread_e8_entry(threadIdx.x);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const int n_items = num_work_items(p, pair, num_pairs);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kRawStages; ++s) {
      mbar_init(raw_full + 8 * s, p.tma ? 1 : 32);
      mbar_init(raw_empty + 8 * s, kDecodeThreads);
    }
    for (int s = 0; s < kDecStages; ++s) {
      mbar_init(dec_full + 8 * s, kDecodeThreads / 32);   // 8 warps of each CTA per stage (used on rank 0)
      mbar_init(dec_empty + 8 * s, 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(tmem_full + 8 * s, 1);
      mbar_init(tmem_empty + 8 * s, 8);               // 4 epilogue warps of each CTA (used on rank 0)
    }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(bar_base + 128), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();            // the peer's barriers are initialised before anyone arrives on them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_ptr_smem;

  if (warp == 0) {
    // ---------------------------------------------------------------- producer
    if (p.tma) {
      if (lane == 0) {
        const CUtensorMap* mapB = kGated && rank ? &tmB2 : &tmB;
        uint32_t n = 0;
        bool ok = true;
        for (int i = 0; i < n_items && ok; ++i) {
          const WorkItem w = work_item<kOutCols>(p, pair, num_pairs, i);
          const int b_row = w.n0 + (kGated ? 0 : static_cast<int>(rank) * kRows);
          for (int kc = w.kc0; kc < w.kc1; ++kc, ++n) {
            const uint32_t s = n & 1u, ph = (n >> 1) & 1u;
            if (!(ok = mbar_wait(raw_empty + 8 * s, ph ^ 1u, abort_flag, 128))) break;
            mbar_expect_tx(raw_full + 8 * s, kRawStageBytes);
            const uint32_t dst = raw_base + s * kRawStageBytes;
            tma_load_2d(dst, &tmA, kc * kRawRowBytes, w.m0 + static_cast<int>(rank) * kRows, raw_full + 8 * s);
            tma_load_2d(dst + kRawHalfBytes, mapB, kc * kRawRowBytes, b_row, raw_full + 8 * s);
          }
        }
      }
    } else {
      uint32_t n = 0;
      bool ok = true;
      for (int i = 0; i < n_items && ok; ++i) {
        const WorkItem w = work_item<kOutCols>(p, pair, num_pairs, i);
        for (int kc = w.kc0; kc < w.kc1; ++kc, ++n) {
          const uint32_t s = n & 1u, ph = (n >> 1) & 1u;
          if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(raw_empty + 8 * s, ph ^ 1u, abort_flag, 32)))) break;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint8_t* base = half == 0 ? p.A : kGated && rank ? p.B2 : p.B;
            const int64_t rows = half == 0 ? p.M : p.N;
            const int64_t row0 = half == 0 ? static_cast<int64_t>(w.m0) + rank * kRows : static_cast<int64_t>(w.n0) + (kGated ? 0 : rank * kRows);
            const uint32_t dst = raw_base + s * kRawStageBytes + half * kRawHalfBytes;
            const int units = p.upr - kc * kRawUnits;                  // units of this chunk that exist (may exceed 4)
            int row = 0, off = lane;                                   // word `off` of the 36 of row chunk `row`
            for (int j = lane; j < kRows * 36; j += 32) {
              const int unit = (off >= 9) + (off >= 18) + (off >= 27);
              const bool in = row0 + row < rows && unit < units;
              const uint8_t* src = in ? base + (row0 + row) * p.pitch + static_cast<int64_t>(kc) * kRawRowBytes + 4 * off : base;
              asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 4 * j), "l"(src), "r"(in ? 4 : 0) : "memory");
              off += 32;
              if (off >= 36) { off -= 36; ++row; }
            }
          }
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(raw_full + 8 * s) : "memory");
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer (rank 0 only)
    if (rank == 0 && lane == 0) {
      uint32_t n = 0, tcount = 0;
      bool ok = true;
      for (int it = 0; it < n_items && ok; ++it, ++tcount) {
        const WorkItem w = work_item<kOutCols>(p, pair, num_pairs, it);
        const uint32_t acc = tcount & 1u, aph = (tcount >> 1) & 1u;
        if (!(ok = mbar_wait_cluster(tmem_empty + 8 * acc, aph ^ 1u, abort_flag))) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + acc * kPairN;
        for (int kc = w.kc0; kc < w.kc1 && ok; ++kc, ++n) {
          // stages 0 and 2 are ready first: the K blocks of a chunk are consumed in the order 0, 2, 1, 3
#pragma unroll
          for (int i = 0; i < kDecStages; ++i) {
            const int u = ((i & 1) << 1) | (i >> 1);
            if (!(ok = mbar_wait_cluster(dec_full + 8 * u, n & 1u, abort_flag))) break;
            tc_fence_after();
            const uint64_t adesc = make_desc(dec_base + u * kDecStageBytes);
            const uint64_t bdesc = make_desc(dec_base + u * kDecStageBytes + kDecHalfBytes);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              tc2_mma(d_tmem, adesc + 2 * kk, bdesc + 2 * kk, kLinInstrDesc, ((kc - w.kc0) | i | kk) != 0 ? 1u : 0u);
            tc2_commit_both(dec_empty + 8 * u);       // both CTAs may overwrite the stage once these MMAs have read it
          }
        }
        if (!ok) break;
        tc2_commit_both(tmem_full + 8 * acc);         // accumulator complete, in both CTAs
      }
    }
  } else if (warp < kDecodeWarp0) {
    // ---------------------------------------------------------------- epilogue
    const int q = warp & 3;                      // TMEM lane quadrant this warp may read
    const uint32_t tmem_empty_leader = mapa(tmem_empty, 0);
    const uint32_t stage = out_base + static_cast<uint32_t>(q) * (2 * kSlabBytes);
    const T* bias = static_cast<const T*>(p.bias);
    const T* bias2 = static_cast<const T*>(p.bias_up);
    const T* side = static_cast<const T*>(p.side);        // residual, or dY in the gradient form
    const bool bias_vec = (reinterpret_cast<uintptr_t>(bias) & 15u) == 0 && (reinterpret_cast<uintptr_t>(bias2) & 15u) == 0;
    uint32_t tcount = 0, slabs = 0;
    for (int it = 0; it < n_items; ++it, ++tcount) {
      const WorkItem w = work_item<kOutCols>(p, pair, num_pairs, it);
      const uint32_t acc = tcount & 1u, aph = (tcount >> 1) & 1u;
      if (!__all_sync(0xFFFFFFFFu, mbar_wait(tmem_full + 8 * acc, aph, abort_flag, 256))) break;
      tc_fence_after();
      const bool shared_tile = w.tail >= 0 && p.slices > 1;
      const bool adds = shared_tile && w.slice > 0, leaves = shared_tile && w.slice + 1 < p.slices;
      unsigned int* my_flag = shared_tile ? p.flags + (static_cast<size_t>(w.tail) * p.slices + w.slice) * 8 + rank * 4 + q : nullptr;
      if (adds && !__all_sync(0xFFFFFFFFu, wait_count(my_flag - 8, 1u, abort_flag))) break;
      // this thread's row of the partial sums, column after column
      float* part = shared_tile ? p.partial + (static_cast<size_t>(w.tail) * 2 + rank) * (kRows * kPairN) + q * 32 + lane : nullptr;
      const int64_t row0 = static_cast<int64_t>(w.m0) + rank * kRows + q * 32, row = row0 + lane;
      const bool row_ok = row < p.M;
      const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * kPairN;
#pragma unroll 1
      for (int slab = 0; slab < kOutCols / kSlabCols; ++slab) {
        const int64_t col0 = static_cast<int64_t>(w.n0) + slab * kSlabCols;
        const bool inside = row0 < p.M && col0 < p.N;                    // same for the whole warp
        uint32_t words[16];
#pragma unroll
        for (int h = 0; h < kSlabCols / 16; ++h) {
          const int c = slab * kSlabCols + h * 16;                       // tile column
          float z[16], u[16];
          if (inside) {
            uint32_t r[16];
            tc_ld16(t_row + c, r);
            if (kGated) {
              uint32_t r2[16];
              tc_ld16(t_row + kOutCols + c, r2);
              tc_wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) u[e] = __uint_as_float(r2[e]);
            } else {
              tc_wait_ld();
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) z[e] = __uint_as_float(r[e]);
          }
          if (slab == kOutCols / kSlabCols - 1 && h == kSlabCols / 16 - 1) {   // accumulator fully read: hand it back before the rest
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + 8 * acc);
          }
          if (!inside) continue;
          if (adds) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              z[e] += __ldcg(part + (c + e) * kRows);
              if (kGated) u[e] += __ldcg(part + (kOutCols + c + e) * kRows);
            }
          }
          if (leaves) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              __stcg(part + (c + e) * kRows, z[e]);
              if (kGated) __stcg(part + (kOutCols + c + e) * kRows, u[e]);
            }
            continue;
          }
          const int64_t col = col0 + h * 16;
          const int valid = p.N - col < 16 ? static_cast<int>(p.N - col) : 16;      // may be <= 0 in the second half of a slab
          if (bias) {
            float b[16];
            load16(bias + col, bias_vec && valid == 16, valid, b);
#pragma unroll
            for (int e = 0; e < 16; ++e) z[e] += b[e];
          }
          if (kGated && bias2) {
            float b[16];
            load16(bias2 + col, bias_vec && valid == 16, valid, b);
#pragma unroll
            for (int e = 0; e < 16; ++e) u[e] += b[e];
          }
          if (!kGrad) {
            activate16(z, p.act);
            if (kGated) {
#pragma unroll
              for (int e = 0; e < 16; ++e) z[e] *= u[e];
            }
            if (side && row_ok) {
              float s[16];
              load16(side + row * p.ld_side + col, p.side_vec && valid == 16, valid, s);
#pragma unroll
              for (int e = 0; e < 16; ++e) z[e] = fmaf(p.res_scale, s[e], z[e]);
            }
            if (sizeof(T) == 2) {
#pragma unroll
              for (int e = 0; e < 8; ++e) words[(8 * h + e) & 15] = pack2(z[2 * e], z[2 * e + 1], T16<T>());
            } else {
#pragma unroll
              for (int e = 0; e < 16; ++e) words[e] = __float_as_uint(z[e]);
            }
          } else {
            float d[16], a[16];
            load16(side + (row_ok ? row : row0) * p.ld_side + col, p.side_vec && valid == 16, valid, d);
            activate_slope16(z, a, p.act);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const bool in = row_ok && e < valid;
              z[e] = in ? d[e] * z[e] * (kGated ? u[e] : 1.0f) : 0.0f;
              if (kGated) u[e] = in ? d[e] * a[e] : 0.0f;
            }
            constexpr int kParts = sizeof(T16<T>) == 2 && IsHalf<T>::value ? 2 : 1;
            if (p.dz && row_ok) {
              __nv_bfloat16* dst = p.dz + row * p.ld_dz + col;
              store_parts<kParts>(z, dst, p.dz_plane, p.ld_dz - col);
              if (kGated) store_parts<kParts>(u, dst + kParts * p.dz_plane, p.dz_plane, p.ld_dz - col);
            }
            if (p.colsum) {
              const float sz = column_sum16(z, lane);
              const int cl = column_of_lane(lane);
              float* sums = p.colsum + (row0 >> 5) * p.N + col;
              if ((lane & 1) == 0 && cl < valid) sums[cl] = sz;
              if (kGated) {
                const float su = column_sum16(u, lane);
                if ((lane & 1) == 0 && cl < valid) sums[p.colsum_plane + cl] = su;
              }
            }
          }
        }
        if (kGrad || !inside || leaves) continue;
        if (p.units) {
          // 64 columns of 32 rows as 128-byte rows, 16-byte chunk c of row r at c ^ (r & 7); then eight lanes per unit
          if (sizeof(T) == 2) {
            const uint32_t my = stage + static_cast<uint32_t>(lane) * 128u;
#pragma unroll
            for (int v = 0; v < 4; ++v)
              sts128(my + (((static_cast<uint32_t>(slab & 1) * 4u + v) ^ (static_cast<uint32_t>(lane) & 7u)) << 4), words[4 * v], words[4 * v + 1],
                     words[4 * v + 2], words[4 * v + 3]);
            if (slab & 1) {
              __syncwarp();
#pragma unroll 1
              for (int pass = 0; pass < 8; ++pass) {
                const int r = pass * 4 + (lane >> 3), g = lane & 7;
                Raw8<T16<T>> x;
                x.a = lds128(stage + static_cast<uint32_t>(r) * 128u + ((static_cast<uint32_t>(g) ^ (static_cast<uint32_t>(r) & 7u)) << 4));
                uint32_t meta;
                const uint32_t code = p.rha ? encode_unit_octet<true>(x, g, meta) : encode_unit_octet<false>(x, g, meta);
                if (row0 + r < p.M) {
                  uint32_t* dst = static_cast<uint32_t*>(p.y) + ((row0 + r) * (p.N >> 6) + (col0 >> 6)) * kUnitWords;
                  dst[1 + g] = code;
                  if (g == 0) dst[0] = meta;
                }
              }
              __syncwarp();
            }
          }
        } else if (p.tma_store) {
          const uint32_t buf = stage + (slabs & 1u) * kSlabBytes;
          const uint32_t my = buf + static_cast<uint32_t>(lane) * 64u, sw = (static_cast<uint32_t>(lane) >> 1) & 3u;    // SWIZZLE_64B
          if (lane == 0) bulk_wait_read<1>();        // the store that used this buffer two slabs ago has read it
          __syncwarp();
#pragma unroll
          for (int v = 0; v < 4; ++v)
            sts128(my + ((static_cast<uint32_t>(v) ^ sw) << 4), words[4 * v], words[4 * v + 1], words[4 * v + 2], words[4 * v + 3]);
          fence_proxy_async_smem();                  // generic-proxy writes -> visible to the TMA store
          __syncwarp();
          if (lane == 0) {
            tma_store_2d(&tmY, static_cast<int>(col0), static_cast<int>(row0), buf);
            bulk_commit();
          }
          ++slabs;
        } else if (row_ok) {
          T* dst = static_cast<T*>(p.y) + row * p.ld_y + col0;
          if (p.y_vec && col0 + kSlabCols <= p.N) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
              reinterpret_cast<uint4*>(dst)[v] = make_uint4(words[4 * v], words[4 * v + 1], words[4 * v + 2], words[4 * v + 3]);
          } else {
            const int64_t left = p.N - col0;
#pragma unroll
            for (int e = 0; e < kSlabCols; ++e) {
              if (e >= left) continue;
              if (sizeof(T) == 2) reinterpret_cast<uint16_t*>(dst)[e] = static_cast<uint16_t>(words[(e >> 1) & 15] >> (16 * (e & 1)));
              else reinterpret_cast<uint32_t*>(dst)[e] = words[e & 15];
            }
          }
        }
      }
      if (leaves) {                                  // this warp's rows of the partial sums are there for the next slice
        __syncwarp();
        if (lane == 0) {
          __threadfence();
          asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(my_flag), "r"(1u) : "memory");
        }
      }
    }
    if (lane == 0) bulk_wait_all();                  // shared memory stays valid until the last store has read it
  } else {
    // ---------------------------------------------------------------- decode
    const int d = threadIdx.x - kDecodeWarp0 * 32;            // 0..511
    const int h = d >> 8;                                     // which unit pair of the raw chunk
    const int row = d & 255;                                  // 0..127 A rows, 128..255 B rows
    const uint32_t r7 = static_cast<uint32_t>(row) & 7u;
    const uint32_t raw_row = static_cast<uint32_t>(row) * kRawRowBytes + static_cast<uint32_t>(h) * 64u;
    const uint32_t dec_row = dec_base + static_cast<uint32_t>(2 * h) * kDecStageBytes + static_cast<uint32_t>(row) * 128u;
    uint32_t chunk_addr[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) chunk_addr[j] = dec_row + ((static_cast<uint32_t>(j) ^ r7) << 4);
    const uint32_t dec_empty0 = dec_empty + 16 * h;
    const uint32_t dec_full0_leader = mapa(dec_full, 0) + 16 * h;
    uint32_t n = 0;
    bool ok = true;
    for (int i = 0; i < n_items && ok; ++i) {
      const WorkItem w = work_item<kOutCols>(p, pair, num_pairs, i);
      // the first of this warp's 32 rows exists (whole warps of rows past the edge are left out)
      const int warp_row = row & ~31;
      const bool live = warp_row < kRows ? static_cast<int64_t>(w.m0) + rank * kRows + warp_row < p.M
                                         : static_cast<int64_t>(w.n0) + (kGated ? 0 : rank * kRows) + (warp_row - kRows) < p.N;
      for (int kc = w.kc0; kc < w.kc1 && ok; ++kc, ++n) {
        const uint32_t s = n & 1u, ph = (n >> 1) & 1u;
        if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(raw_full + 8 * s, ph, abort_flag)))) break;
        uint32_t W[18];
        if (live) {
          uint32_t L[20];
          const uint32_t src = raw_base + s * kRawStageBytes + raw_row;
#pragma unroll
          for (int i = 0; i < 5; ++i) {
            const uint4 v = lds128(src + 16 * i);
            L[4 * i] = v.x; L[4 * i + 1] = v.y; L[4 * i + 2] = v.z; L[4 * i + 3] = v.w;
          }
          fence_proxy_async_smem();                  // these reads before the async proxy refills the stage
#pragma unroll
          for (int i = 0; i < 18; ++i) W[i] = h ? L[i + 2] : L[i];
        }
        mbar_arrive(raw_empty + 8 * s);
        ok = decode_two_units(W, chunk_addr, lut, p.mul, dec_empty0, dec_full0_leader, (n & 1u) ^ 1u, abort_flag, live);
      }
    }
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  if (*abort_flag) {
    // Some wait gave up: give copies and MMAs that are still in flight time to land before the
    // shared and tensor memory they target is released.
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 2000000ull) {}
    if (threadIdx.x == 0) atomicExch(p.error_word, 1u);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();            // neither CTA leaves while the other may still read its shared memory or arrive on its barriers
  if (warp == 1) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

}  // namespace
}  // namespace hif4
