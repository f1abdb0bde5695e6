// The linear layer with its epilogue on CTA pairs: 256 x 256 accumulator tile per pair of SMs (tcgen05.mma
// cta_group::2), operands decoded from packed units as in the FP32 GEMM of hif4_gemm_tc2.cu, whose stages, barriers and
// schedule this kernel shares.  What differs:
//   - B rows.  Gated: rank 0 decodes 128 rows of W, rank 1 the same 128 rows of W_up, so that a row of the tile has the
//     gate products in columns 0..127 and the up products of the same outputs in columns 128..255 of one TMEM lane, and
//     the thread that reads both finishes the output.
//   - Loads.  TMA needs K % 256 == 0 and 16-byte aligned units; otherwise the producer warp copies the 144-byte row
//     chunks word by word (cp.async, zeros past the last unit): 288 copies per K = 256 chunk, each with its address and bounds,
//     by one warp that the other warps then wait for (2048 x 4096 x 4160 444 us, x 4096 through TMA 74 us).
//   - Rows past M and columns past N are not decoded: their accumulators are garbage that no one reads (a row of the
//     product depends on its own row of A only), and few rows leave the decode warps to the weights.
//   - Epilogue.  Bias, activation, product, residual in FP32 on 16 columns of a row at a time; one rounding; 64-byte
//     rows staged in shared memory and written with TMA stores, or 64-column rows converted to units there by eight
//     lanes each.  The gradient form writes dZ (dG, dU) as BF16 parts for the product that follows, and FP32 column
//     sums per 32 rows for the bias gradients.
//   - The last tile of a CTA is finished by all of its warps: the decode warps, out of work, take four fifths of the
//     columns (staged in the operand stages, which are free by then).  With few tiles this tail is most of the call.
//   - Tiles shared along K pass FP32 partial sums through the workspace (the epilogue is not linear, so nothing can be added
//     in place): every slice but the last leaves its part, the last adds them to its own in slice order and finishes the
//     tile.  It waits for slices of lower index only, so a grid that is partly resident cannot wait for itself.
// What bounds it: long products, what bounds the FP32 product (decode and tensor core take 3080 and 2350 clocks per K = 256
// chunk by themselves and share issue slots and the shared-memory port); short ones, set-up, pipeline fill and the last
// tile's epilogue.  From units, one call after another on the same inputs: 4096 x 14336 x 4096 gated 814 us (1.18 PFLOP/s, 0.71 of
// the measured burst rate, 0.84 of the sustained one), 4096 x 4096 x 14336 with residual 418 us; from rows that change from call to
// call 871 and 463 us, the conversion among them.  64 x 4096 x 4096 27 to 32 us on different machines.
#pragma once
#include "hif4_activation.cuh"
#include "hif4_gemm_internal.cuh"
#include "hif4_linear_internal.cuh"
#include "hif4_tc2_dense.cuh"
#include "hif4_vec8.cuh"

namespace hif4 {
namespace {

constexpr int kSlabBytes = 32 * 64;                   // 32 rows of one epilogue warp x 64 bytes
constexpr int kStageBufs = 3;
constexpr int kStageOutBytes = 4 * kStageBufs * kSlabBytes;    // 4 warps x 3 buffers (units: two of them as one of 32 x 128 bytes)
constexpr int kEpiGroups = 5;                         // warps per TMEM quadrant that finish a CTA's last tile: its epilogue warp and four decode warps
constexpr int kLinBarBytes = 640;                     // mbarriers: 144 bytes, then kStageBufs per warp that may take part in an epilogue (20)
constexpr int kLinSmemBytes = 1024 /*alignment slack*/ + kDecStages * kDecStageBytes + kRawStages * kRawStageBytes + kStageOutBytes +
                              kLinBarBytes + 1024 /*spread table*/;
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
// Partial sums of 16 columns of a row: four 16-byte words, each beside those of the warp's other rows.  The `others` parts of
// a tile lie one after another and are added in that order.
constexpr size_t kPartialTileWords = static_cast<size_t>(kPairM) * kPairN / 4;
__device__ __forceinline__ void add_partial16(float (&v)[16], const float4* part, int others) {
#pragma unroll 2
  for (int s = 0; s < others; ++s, part += kPartialTileWords) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 f = __ldcg(part + k * 32);
      v[4 * k] += f.x; v[4 * k + 1] += f.y; v[4 * k + 2] += f.z; v[4 * k + 3] += f.w;
    }
  }
}
__device__ __forceinline__ void leave_partial16(const float (&v)[16], float4* part) {
#pragma unroll
  for (int k = 0; k < 4; ++k) __stcg(part + k * 32, make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]));
}
// A warp's corner of a part of a shared tile: 256 columns x 32 rows, 16 columns (2 KB) after 16 columns.
__device__ __forceinline__ float4* partial_of(float* partial, int part, uint32_t rank, int q, int lane) {
  return reinterpret_cast<float4*>(partial) + static_cast<size_t>(part) * kPartialTileWords + (rank * 4 + q) * (32 * kPairN / 4) + lane;
}
// Waits until the parts before the last have all `steps` counted in this quadrant.
__device__ __forceinline__ bool wait_parts(const unsigned int* flags, int others, unsigned int steps, volatile uint32_t* abort_flag) {
  for (int s = 0; s < others; ++s)
    if (!__all_sync(0xFFFFFFFFu, wait_count(flags + 8 * s, steps, abort_flag))) return false;
  return true;
}
template <int kAct>
__device__ __forceinline__ void activate16(float (&v)[16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = activate(v[e], kAct);
}
// a = act(z), z = act'(z)
template <int kAct>
__device__ __forceinline__ void activate_slope16(float (&z)[16], float (&a)[16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float s;
    activate_slope(z[e], kAct, a[e], s);
    z[e] = s;
  }
}
template <bool kValue> struct Flag { static constexpr bool value = kValue; };

// z += 16 elements of a bias vector (16-byte aligned, inside the row).
template <typename T>
__device__ __forceinline__ void add16(float (&z)[16], const Raw8<T>& lo, const Raw8<T>& hi) {
  float a[8], b[8];
  unpack8(lo, a);
  unpack8(hi, b);
#pragma unroll
  for (int e = 0; e < 8; ++e) { z[e] += a[e]; z[8 + e] += b[e]; }
}
// 16 elements of a staged 64-byte row (32 or 16 elements; `h`: which half of a 16-bit row).
template <typename T>
__device__ __forceinline__ void read_staged16(float (&v)[16], uint32_t row_at, uint32_t sw, int h) {
  Raw8<T> lo, hi;
  if constexpr (sizeof(T) == 2) {
    lo.a = lds128(row_at + (((2u * h) ^ sw) << 4));
    hi.a = lds128(row_at + (((2u * h + 1u) ^ sw) << 4));
  } else {
    lo.a = lds128(row_at + ((0u ^ sw) << 4));
    lo.b = lds128(row_at + ((1u ^ sw) << 4));
    hi.a = lds128(row_at + ((2u ^ sw) << 4));
    hi.b = lds128(row_at + ((3u ^ sw) << 4));
  }
  float a[8], b[8];
  unpack8(lo, a);
  unpack8(hi, b);
#pragma unroll
  for (int e = 0; e < 8; ++e) { v[e] = a[e]; v[8 + e] = b[e]; }
}
// The same place written with 16 results, rounded to T.
template <typename T>
__device__ __forceinline__ void pack16(uint4 (&out)[sizeof(T)], const float (&z)[16]) {
  const float a[8] = {z[0], z[1], z[2], z[3], z[4], z[5], z[6], z[7]};
  const float b[8] = {z[8], z[9], z[10], z[11], z[12], z[13], z[14], z[15]};
  const Raw8<T> lo = pack8<T>(a), hi = pack8<T>(b);
  if constexpr (sizeof(T) == 2) {
    out[0] = lo.a; out[1] = hi.a;
  } else {
    out[0] = lo.a; out[1] = lo.b; out[2] = hi.a; out[3] = hi.b;
  }
}
// A slab (32 rows of 64 bytes) between a matrix of any alignment and the staging buffer, neighbouring lanes on neighbouring
// elements; rows past `rows` and columns past `cols` are left out (read as zeros).
template <typename T, bool kStore>
__device__ __forceinline__ void copy_slab(T* matrix, int64_t ld, uint32_t buf, int lane, int64_t rows, int64_t cols) {
  constexpr int kCols = 64 / sizeof(T), kRowsAtOnce = 32 / kCols;
  const int c = lane & (kCols - 1), r0 = lane / kCols;
  const uint32_t byte = static_cast<uint32_t>(c) * sizeof(T);
#pragma unroll 8
  for (int r = r0; r < 32; r += kRowsAtOnce) {
    const uint32_t at = buf + static_cast<uint32_t>(r) * 64u + (((byte >> 4) ^ ((static_cast<uint32_t>(r) >> 1) & 3u)) << 4) + (byte & 15u);
    const bool in = r < rows && c < cols;
    if constexpr (sizeof(T) == 2) {
      uint16_t v = 0;
      if constexpr (kStore) {
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
        if (in) reinterpret_cast<uint16_t*>(matrix)[r * ld + c] = v;
      } else {
        if (in) v = reinterpret_cast<const uint16_t*>(matrix)[r * ld + c];
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(v) : "memory");
      }
    } else {
      uint32_t v = 0;
      if constexpr (kStore) {
        v = lds32(at);
        if (in) reinterpret_cast<uint32_t*>(matrix)[r * ld + c] = v;
      } else {
        if (in) v = reinterpret_cast<const uint32_t*>(matrix)[r * ld + c];
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
      }
    }
  }
}
// Waits for a tcgen05.ld into r; the registers pass through, so that nothing reads them before.
__device__ __forceinline__ void tc_wait_ld16(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
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

// BF16 parts of 16 values: part 0 holds the leading 8 bits, part 1 what is left of them (nothing of an infinity: the
// difference would be NaN).
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
        rest[2 * e] = rest_of(rest[2 * e], __uint_as_float(w[e] << 16));
        rest[2 * e + 1] = rest_of(rest[2 * e + 1], __uint_as_float(w[e] & 0xFFFF0000u));
      }
    }
    uint4* q = reinterpret_cast<uint4*>(dst + part * plane);
    if (room > 0) q[0] = make_uint4(w[0], w[1], w[2], w[3]);       // the row pitch is a multiple of eight elements
    if (room > 8) q[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// kGated: two projections.  kGrad: the gradient form.  T: type of bias, residual, Y and dY.  kAct: the activation (one kernel
// each: five activations side by side cost the epilogue spills and instruction-cache misses).  kParts: BF16 numbers per element of
// dZ (gradient form; see InputGradCall).
template <bool kGated, bool kGrad, typename T, int kAct, int kParts>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_tc2_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                  const __grid_constant__ CUtensorMap tmB2, const __grid_constant__ CUtensorMap tmY,
                  const __grid_constant__ CUtensorMap tmSide, const LinearParams p) {
  constexpr int kOutCols = kGated ? kPairN / 2 : kPairN;             // outputs per tile row
  constexpr int kSlabCols = 64 / sizeof(T);                          // outputs per staged 64-byte row
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t dec_base = smem_base;
  const uint32_t raw_base = dec_base + kDecStages * kDecStageBytes;
  const uint32_t out_base = raw_base + kRawStages * kRawStageBytes;
  const uint32_t bar_base = out_base + kStageOutBytes;
  const uint32_t raw_full = bar_base, raw_empty = bar_base + 16, dec_full = bar_base + 32, dec_empty = bar_base + 64,
                 tmem_full = bar_base + 96, tmem_empty = bar_base + 112, last_full = bar_base + 136,
                 side_full = bar_base + 144;      // [20 warps][kStageBufs]
  uint8_t* gen_base = smem_raw + (smem_base - smem_u32(smem_raw));
  volatile uint32_t* tmem_ptr_smem = reinterpret_cast<volatile uint32_t*>(gen_base + (bar_base - smem_base) + 128);
  volatile uint32_t* abort_flag = tmem_ptr_smem + 1;
  const uint32_t lut = bar_base + kLinBarBytes;
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
    for (int s = 0; s < 4 * kEpiGroups * kStageBufs; ++s) mbar_init(side_full + 8 * s, 1);
    mbar_init(last_full, 1);
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
  grid_launch_next();
  grid_wait();                   // everything above overlaps the preceding kernel; nothing before this line reads or writes global memory

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
        if (it == n_items - 1) tc2_commit_both(last_full);        // the same, for the helpers of the last epilogue
      }
    }
  } else {
    // ---------------------------------------------------------------- decode, then its warps join the epilogue of the last tile
    bool ok = true;
    if (warp >= kDecodeWarp0) {
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

    // ---------------------------------------------------------------- epilogue
    // Warps 2-5 finish every tile; the CTA's last one, which no product hides, is shared with the decode warps, which have
    // nothing left to decode: the slabs of a quadrant go round five warps.
    const bool helper = warp >= kDecodeWarp0;
    const int q = warp & 3;                      // TMEM lane quadrant this warp may read
    const int group = helper ? 1 + (warp - kDecodeWarp0) / 4 : 0;
    const uint32_t tmem_empty_leader = mapa(tmem_empty, 0);
    // helpers stage in the operand stages, which the last tile's products no longer need once they are complete
    const uint32_t stage = helper ? dec_base + static_cast<uint32_t>(warp - kDecodeWarp0) * (kStageBufs * kSlabBytes)
                                  : out_base + static_cast<uint32_t>(q) * (kStageBufs * kSlabBytes);
    const uint32_t my_side_full = side_full + static_cast<uint32_t>(group * 4 + q) * (8 * kStageBufs);
    const uint32_t sw = (static_cast<uint32_t>(lane) >> 1) & 3u;          // SWIZZLE_64B: 16-byte chunk c of row r at c ^ ((r >> 1) & 3)
    const T* bias = static_cast<const T*>(p.bias);
    const T* bias2 = static_cast<const T*>(p.bias_up);
    const T* side = static_cast<const T*>(p.side);        // residual, or dY in the gradient form
    const bool bias_vec = (reinterpret_cast<uintptr_t>(bias) & 15u) == 0 && (reinterpret_cast<uintptr_t>(bias2) & 15u) == 0;
    constexpr int kSlabParts = kSlabCols / 16;
    uint32_t buf = 0, buf_phase = 0;                      // staging buffer in turn, parity of its side barrier
    const int first = helper && n_items > 0 ? n_items - 1 : 0;
    uint32_t tcount = static_cast<uint32_t>(first);
    for (int it = first; it < n_items && ok; ++it, ++tcount) {
      const WorkItem w = work_item<kOutCols>(p, pair, num_pairs, it);
      const uint32_t acc = tcount & 1u, aph = (tcount >> 1) & 1u;
      const int64_t row0 = static_cast<int64_t>(w.m0) + rank * kRows + q * 32, row = row0 + lane;
      const bool row_ok = row < p.M;
      const bool shared_tile = w.tail >= 0 && p.slices > 1;
      const bool leaves = shared_tile && w.slice + 1 < p.slices, adds = shared_tile && !leaves;
      const int others = p.slices - 1;                   // parts that the last slice adds to its own
      const int groups = it == n_items - 1 ? kEpiGroups : 1;
      // columns that hold outputs, in whole slabs
      const int64_t cols_left = p.N - w.n0;
      const int cols = row0 >= p.M ? 0 : cols_left >= kOutCols ? kOutCols : static_cast<int>((cols_left + kSlabCols - 1) / kSlabCols) * kSlabCols;
      // Residual or dY through the staging buffers: two slabs are requested ahead, the first two while the product still runs
      // (by a helper once it is complete).
      const bool side_staged = p.side_tma && !leaves;
      auto request_side = [&](int column, uint32_t b) {
        mbar_expect_tx(my_side_full + 8 * b, kSlabBytes);
        tma_load_2d(stage + b * kSlabBytes, &tmSide, w.n0 + column, static_cast<int>(row0), my_side_full + 8 * b);
      };
      auto request_first = [&]() {
        if (!side_staged || lane != 0) return;
        bulk_wait_read<1>();                             // the two buffers' last stores have read them
        for (int i = 0; i < 2; ++i) {
          const int column = (group + i * groups) * kSlabCols;
          if (column < cols) request_side(column, (buf + i) % kStageBufs);
        }
      };
      if (!helper) request_first();
      // A helper has not followed the phases of tmem_full, and with short items several may still be to come: the parity would
      // not tell it which one it sees.  Its own barrier completes once.
      if (!__all_sync(0xFFFFFFFFu, helper ? mbar_wait(last_full, 0u, abort_flag, 32) : mbar_wait(tmem_full + 8 * acc, aph, abort_flag, 256))) break;
      tc_fence_after();
      if (helper) request_first();
      // sixteen-column steps that the other slices' warps have left in this quadrant: all of the tile's
      unsigned int* flags = shared_tile ? p.flags + static_cast<size_t>(w.tail) * p.slices * 8 + rank * 4 + q : nullptr;
      if (adds && cols > 0 && !wait_parts(flags, others, static_cast<unsigned int>(cols / 16), abort_flag)) break;
      float4* part_sums = shared_tile ? partial_of(p.partial, w.tail * others + (leaves ? w.slice : 0), rank, q, lane) : nullptr;
      const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * kPairN;
      // Eight lanes convert one unit of a staged 32 x 64 block (16-bit types), four rows at a time; `col`: a column of the block.
      auto convert_units = [&](int64_t col) {
        if constexpr (sizeof(T) == 2) {
          __syncwarp();
          uint32_t* dst = static_cast<uint32_t*>(p.y) + ((row0 + (lane >> 3)) * (p.N >> 6) + (col >> 6)) * kUnitWords;
          const int g = lane & 7;
#pragma unroll 1
          for (int rr = lane >> 3; rr < 32; rr += 4) {
            Raw8<T> x;
            x.a = lds128(stage + static_cast<uint32_t>(rr) * 128u + ((static_cast<uint32_t>(g) ^ (static_cast<uint32_t>(rr) & 7u)) << 4));
            uint32_t meta;
            const uint32_t code = p.rha ? encode_unit_octet<true>(x, g, meta) : encode_unit_octet<false>(x, g, meta);
            if (row0 + rr < p.M) {
              dst[1 + g] = code;
              if (g == 0) dst[0] = meta;
            }
            dst += 4 * (p.N >> 6) * kUnitWords;
          }
          __syncwarp();
        }
      };
      // Asks for this warp's slab after next in the buffer that was stored, or read, a slab ago; steps on.
      auto next_buffer = [&](bool request, int column) {
        if (request && column < cols && lane == 0) {
          bulk_wait_read<1>();
          request_side(column, buf >= 1 ? buf - 1 : kStageBufs - 1);       // (buf + 2) mod 3
        }
        if (++buf == kStageBufs) { buf = 0; buf_phase ^= 1u; }
      };
      // Whole, unshared tiles: the steps of a slab in one straight run of instructions per combination of bias and side
      // matrix.  A warp alone on its scheduler's instruction stream pays for every jump over code that it does not run
      // (8192 x 8192 x 256, SiLU: 190 us in the general loop below).
      auto whole_tile = [&](auto has_bias, auto has_side, auto to_units) {
        constexpr int kStep = to_units.value ? 64 : kSlabCols;          // columns taken at a time
        const T* b1 = bias + w.n0;
        const T* b2 = bias2 + w.n0;
#pragma unroll 1
        for (int at = group * kStep; at < kOutCols; at += groups * kStep)
#pragma unroll 1
        for (int c0 = at; c0 < at + kStep; c0 += kSlabCols) {
          const uint32_t my = stage + buf * kSlabBytes + static_cast<uint32_t>(lane) * 64u;
          uint32_t r[kSlabParts][16];
          if (!kGated) {
#pragma unroll
            for (int h = 0; h < kSlabParts; ++h) tc_ld16(t_row + c0 + 16 * h, r[h]);
          }
          if constexpr (has_side.value) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(my_side_full + 8 * buf, buf_phase, abort_flag)) && ok;
          } else if constexpr (!to_units.value && !kGrad) {
            if (lane == 0) bulk_wait_read<kStageBufs - 1>();        // the store that used this buffer has read it
            __syncwarp();
          }
#pragma unroll
          for (int h = 0; h < kSlabParts; ++h) {
            const int c = c0 + 16 * h;
            float z[16], u[16];
            Raw8<T> bz0, bz1, bu0, bu1;
            if constexpr (has_bias.value) {
              bz0 = load8(b1 + c); bz1 = load8(b1 + c + 8);
              if constexpr (kGated) { bu0 = load8(b2 + c); bu1 = load8(b2 + c + 8); }
            }
            if constexpr (kGated) {
              uint32_t r2[16];
              tc_ld16(t_row + c, r[0]);
              tc_ld16(t_row + kOutCols + c, r2);
              tc_wait_ld16(r[0]);
              tc_wait_ld16(r2);
#pragma unroll
              for (int e = 0; e < 16; ++e) { z[e] = __uint_as_float(r[0][e]); u[e] = __uint_as_float(r2[e]); }
            } else {
              tc_wait_ld16(r[h]);
#pragma unroll
              for (int e = 0; e < 16; ++e) z[e] = __uint_as_float(r[h][e]);
            }
            if constexpr (has_bias.value) {
              add16<T>(z, bz0, bz1);
              if constexpr (kGated) add16<T>(u, bu0, bu1);
            }
            float s[16];
            if constexpr (has_side.value) read_staged16<T>(s, my, sw, h);
            if constexpr (!kGrad) {
              activate16<kAct>(z);
              if constexpr (kGated) {
#pragma unroll
                for (int e = 0; e < 16; ++e) z[e] *= u[e];
              }
              if constexpr (has_side.value) {
#pragma unroll
                for (int e = 0; e < 16; ++e) z[e] = fmaf(p.res_scale, s[e], z[e]);
              }
              uint4 out[sizeof(T)];
              pack16<T>(out, z);
              if constexpr (to_units.value) {
                const uint32_t mine = stage + static_cast<uint32_t>(lane) * 128u, k = (static_cast<uint32_t>(c) & 63u) >> 3, r7 = static_cast<uint32_t>(lane) & 7u;
                sts128(mine + ((k ^ r7) << 4), out[0].x, out[0].y, out[0].z, out[0].w);
                sts128(mine + (((k + 1u) ^ r7) << 4), out[1].x, out[1].y, out[1].z, out[1].w);
              } else {
#pragma unroll
                for (int v = 0; v < static_cast<int>(sizeof(T)); ++v)
                  sts128(my + (((static_cast<uint32_t>(sizeof(T)) * h + v) ^ sw) << 4), out[v].x, out[v].y, out[v].z, out[v].w);
              }
            } else {
              float a[16];
              activate_slope16<kAct>(z, a);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                z[e] = row_ok ? s[e] * z[e] * (kGated ? u[e] : 1.0f) : 0.0f;
                if (kGated) u[e] = row_ok ? s[e] * a[e] : 0.0f;
              }
              const int64_t col = static_cast<int64_t>(w.n0) + c;
              if (p.dz && row_ok) {
                __nv_bfloat16* dst = p.dz + row * p.ld_dz + col;
                store_parts<kParts>(z, dst, p.dz_plane, 16);
                if (kGated) store_parts<kParts>(u, dst + kParts * p.dz_plane, p.dz_plane, 16);
              }
              if (p.colsum) {
                float* sums = p.colsum + (row0 >> 5) * p.N + col + column_of_lane(lane);
                const float sz = column_sum16(z, lane);
                if ((lane & 1) == 0) *sums = sz;
                if (kGated) {
                  const float su = column_sum16(u, lane);
                  if ((lane & 1) == 0) sums[p.colsum_plane] = su;
                }
              }
            }
          }
          if constexpr (to_units.value) {
            if (c0 & 32) convert_units(static_cast<int64_t>(w.n0) + c0);
          } else {
            fence_proxy_async_smem();                  // generic-proxy writes (reads) before the async proxy reads (writes) the buffer
            __syncwarp();
            if (!kGrad && lane == 0) {
              tma_store_2d(&tmY, w.n0 + c0, static_cast<int>(row0), stage + buf * kSlabBytes);
              bulk_commit();
            }
            next_buffer(has_side.value, c0 + 2 * groups * kSlabCols);
          }
        }
      };
      const bool whole = !shared_tile && cols == kOutCols && cols_left >= kOutCols && ((!bias && !bias2) || (bias_vec && bias && (!kGated || bias2))) &&
                         (kGrad ? side_staged : p.units ? !side : p.tma_store && (!side || side_staged));
      if (whole) {
        if constexpr (kGrad) {
          if (bias) whole_tile(Flag<true>{}, Flag<true>{}, Flag<false>{});
          else whole_tile(Flag<false>{}, Flag<true>{}, Flag<false>{});
        } else {
          if (p.units) {
            if constexpr (sizeof(T) == 2) {
              if (bias) whole_tile(Flag<true>{}, Flag<false>{}, Flag<true>{});
              else whole_tile(Flag<false>{}, Flag<false>{}, Flag<true>{});
            }
          } else if (side) {
            if (bias) whole_tile(Flag<true>{}, Flag<true>{}, Flag<false>{});
            else whole_tile(Flag<false>{}, Flag<true>{}, Flag<false>{});
          } else {
            if (bias) whole_tile(Flag<true>{}, Flag<false>{}, Flag<false>{});
            else whole_tile(Flag<false>{}, Flag<false>{}, Flag<false>{});
          }
        }
      } else if (leaves) {
        // a part of the contraction: FP32 sums for the last slice, which adds them all (16 columns are 128 words of 16 bytes)
        unsigned int left = 0;
#pragma unroll 1
        for (int c = group * 16; c < cols; c += groups * 16, ++left) {
          uint32_t r[16];
          float z[16];
#pragma unroll
          for (int half = 0; half < (kGated ? 2 : 1); ++half) {
            const int cc = c + half * kOutCols;
            tc_ld16(t_row + cc, r);
            tc_wait_ld16(r);
#pragma unroll
            for (int e = 0; e < 16; ++e) z[e] = __uint_as_float(r[e]);
            leave_partial16(z, part_sums + cc * 8);
          }
        }
        __syncwarp();
        if (lane == 0 && left > 0) {
          __threadfence();
          asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(flags + 8 * w.slice), "r"(left) : "memory");
        }
      } else {
        const int step = !kGrad && p.units ? 64 : kSlabCols;
#pragma unroll 1
        for (int at = group * step; at < cols; at += groups * step)
#pragma unroll 1
        for (int c0 = at; c0 < at + step; c0 += kSlabCols) {
          const uint32_t slab = stage + buf * kSlabBytes, my = slab + static_cast<uint32_t>(lane) * 64u;
          const int64_t col0 = static_cast<int64_t>(w.n0) + c0, rows_here = p.M - row0, cols_here = p.N - col0;
          // (with units the staging buffers hold them: the residual comes straight from its matrix)
          const bool side_copied = side && !side_staged && (kGrad || !p.units);
          if (side_staged) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(my_side_full + 8 * buf, buf_phase, abort_flag)) && ok;
          } else if (kGrad || !p.units) {
            if (lane == 0) bulk_wait_read<kStageBufs - 1>();          // the store that used this buffer has read it
            __syncwarp();
            if (side_copied) {
              copy_slab<T, false>(const_cast<T*>(side) + row0 * p.ld_side + col0, p.ld_side, slab, lane, rows_here, cols_here);
              __syncwarp();
            }
          }
#pragma unroll 1
          for (int h = 0; h < kSlabParts; ++h) {
            const int c = c0 + 16 * h;
            const int64_t col = static_cast<int64_t>(w.n0) + c;
            float z[16], u[16];
            {
              uint32_t r[16];
              tc_ld16(t_row + c, r);
              tc_wait_ld16(r);
#pragma unroll
              for (int e = 0; e < 16; ++e) z[e] = __uint_as_float(r[e]);
              if (kGated) {
                tc_ld16(t_row + kOutCols + c, r);
                tc_wait_ld16(r);
#pragma unroll
                for (int e = 0; e < 16; ++e) u[e] = __uint_as_float(r[e]);
              }
            }
            if (adds) {
              add_partial16(z, part_sums + c * 8, others);
              if (kGated) add_partial16(u, part_sums + (kOutCols + c) * 8, others);
            }
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
            float s[16];
            if (side_staged || side_copied) read_staged16<T>(s, my, sw, h);
            else if (side) load16(side + (row_ok ? row : row0) * p.ld_side + col, p.side_vec && valid == 16, valid, s);
            if constexpr (!kGrad) {
              activate16<kAct>(z);
              if (kGated) {
#pragma unroll
                for (int e = 0; e < 16; ++e) z[e] *= u[e];
              }
              if (side) {
#pragma unroll
                for (int e = 0; e < 16; ++e) z[e] = fmaf(p.res_scale, s[e], z[e]);
              }
              uint4 out[sizeof(T)];
              pack16<T>(out, z);
              if (p.units) {
                // 64 columns of 32 rows as 128-byte rows, 16-byte chunk c of row r at c ^ (r & 7); then eight lanes per unit
                if constexpr (sizeof(T) == 2) {
                  const uint32_t mine = stage + static_cast<uint32_t>(lane) * 128u, k = (static_cast<uint32_t>(c) & 63u) >> 3, r7 = static_cast<uint32_t>(lane) & 7u;
                  sts128(mine + ((k ^ r7) << 4), out[0].x, out[0].y, out[0].z, out[0].w);
                  sts128(mine + (((k + 1u) ^ r7) << 4), out[1].x, out[1].y, out[1].z, out[1].w);
                }
              } else {
#pragma unroll
                for (int v = 0; v < static_cast<int>(sizeof(T)); ++v)
                  sts128(my + (((static_cast<uint32_t>(sizeof(T)) * h + v) ^ sw) << 4), out[v].x, out[v].y, out[v].z, out[v].w);
              }
            } else {
              float a[16];
              activate_slope16<kAct>(z, a);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const bool in = row_ok && e < valid;
                z[e] = in ? s[e] * z[e] * (kGated ? u[e] : 1.0f) : 0.0f;
                if (kGated) u[e] = in ? s[e] * a[e] : 0.0f;
              }
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
          if (!kGrad && p.units) {
            if (c0 & 32) convert_units(col0);
            continue;
          }
          fence_proxy_async_smem();                  // generic-proxy writes (reads) before the async proxy reads (writes) the buffer
          __syncwarp();
          if (!kGrad) {
            if (p.tma_store) {
              if (lane == 0) {
                tma_store_2d(&tmY, static_cast<int>(col0), static_cast<int>(row0), slab);
                bulk_commit();
              }
            } else {
              copy_slab<T, true>(static_cast<T*>(p.y) + row0 * p.ld_y + col0, p.ld_y, slab, lane, rows_here, cols_here);
              if (side_staged) {
                fence_proxy_async_smem();
                __syncwarp();
              }
            }
          }
          next_buffer(side_staged, c0 + 2 * groups * kSlabCols);
        }
      }
      if (!helper) {
        tc_fence_before();                           // accumulator fully read: hand it back
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + 8 * acc);
      }
    }
    if (lane == 0) bulk_wait_all();                  // shared memory stays valid until the last store has read it
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
