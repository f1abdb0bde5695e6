// CTA-pair form of the block-scaled product for prompts: a cluster of two CTAs on 256 tokens x 256 rows of B
// (tcgen05.mma.cta_group::2), persistent over its tiles.  Each CTA holds its 128 tokens and 128 of the rows of B, so an SM reads
// 8 KB from L2 for a K = 64 step of 128 x 256 outputs; it needs the scales of all 256 rows of B, though.
//
// Per CTA: a TMA warp (5 stages of K = 256: 32 KB codes, 6 KB scales), four warps that move the scales of a stage to tensor memory
// (48 columns a stage beside the 256 accumulator columns) and say so to the leader's MMA thread, eight epilogue warps.  The
// accumulator is single: 16-bit outputs are read into registers as pairs and the accumulator handed back before any of them is
// stored, so that the next tile's first MMAs wait for tensor-memory reads only.
#include "hif4_bfp4_gemm.cuh"

namespace hif4 {
namespace {

constexpr int kThreads = 512;                // warps: TMA, MMA, TMEM allocation, idle, 4 x scales, 8 x epilogue
constexpr int kTile = 256, kHalf = 128;
constexpr int kStages = 5;
constexpr int kCodeBytes = 2 * kHalf * kRowBytes;
constexpr int kSfBytes = (kHalf + kTile) * 16;
constexpr int kBars = kStages * (kCodeBytes + kSfBytes);
constexpr int kSmem = 1024 + kBars + 256;
constexpr int kSfCols = 48;                  // of a stage: 16 for the tokens, 32 for B
constexpr int kTmemCols = 512;
constexpr int kBand = 16;                    // token tiles that are walked together (their codes stay in L2)
static_assert(kTile + kStages * kSfCols <= kTmemCols, "TMEM");
static_assert(kSmem <= 227 * 1024, "shared memory");

// Scale words of 256 rows -> 32 columns: column 8 k + c holds step k of rows 32 c .. 32 c + 31.
template <bool kNv>
__device__ __forceinline__ void move_scales_256(uint32_t smem, uint32_t taddr, int lane, int half) {
  uint32_t lo[16], hi[16];
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const uint4 v = lds128(smem + (c * 32 + lane) * 16);
    if (kNv) {
      lo[c] = v.x; lo[8 + c] = v.y; hi[c] = v.z; hi[8 + c] = v.w;
    } else {
      lo[c] = half ? v.z : v.x; lo[8 + c] = half ? v.w : v.y;
    }
  }
  tmem_st16(taddr, lo);
  if (kNv) tmem_st16(taddr + 16, hi);
}

struct PairTile { int m0, n0; };
__device__ __forceinline__ PairTile pair_tile(const Bfp4Params& p, int t) {
  const int band_tiles = kBand * p.n_tiles, band = t / band_tiles, in = t - band * band_tiles;
  const int rows = min(kBand, p.m_tiles - band * kBand);
  const int nt = in / rows, mt = band * kBand + in - nt * rows;
  return {mt * kTile, nt * kTile};
}

__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
               "r"(w[6]), "r"(w[7]) : "memory");
}

template <bool kNv>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
bfp4_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ Bfp4Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sf = smem + kStages * kCodeBytes, bars = smem + kBars;
  const uint32_t full = bars, ready = bars + 8 * kStages, empty = bars + 16 * kStages, acc_full = bars + 24 * kStages, acc_empty = acc_full + 8,
                 slot = acc_full + 16;
  uint8_t* gen = smem_raw + (smem - smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + (slot - smem));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1, tiles = p.m_tiles * p.n_tiles;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(ready + 8 * s, 8);                       // four warps of each CTA (used on rank 0)
      mbar_init(empty + 8 * s, 1);
    }
    mbar_init(acc_full, 1);
    mbar_init(acc_empty, 16);                            // eight warps of each CTA (used on rank 0)
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, sf_cols = tmem + kTile;

  if (warp == 0) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 1u;
      bool ok = true;
      for (int t = pair; t < tiles && ok; t += pairs) {
        const PairTile w = pair_tile(p, t);
        const int m0 = w.m0 + static_cast<int>(rank) * kHalf, n0 = w.n0 + static_cast<int>(rank) * kHalf;
        const uint32_t sf_a = static_cast<uint32_t>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(kHalf), p.M - m0))) * 16u;
        const uint32_t sf_b = static_cast<uint32_t>(min(static_cast<int64_t>(kTile), p.N - w.n0)) * 16u;
        const uint8_t *a_sf = p.a_scales + static_cast<int64_t>(m0) * 16, *b_sf = p.b_scales + static_cast<int64_t>(w.n0) * 16;
        for (int k = 0; k < p.chunks; ++k) {
          if (!(ok = mbar_wait(empty + 8 * s, ph, abort_flag))) break;
          const uint32_t bar = full + 8 * s, at = smem + s * kCodeBytes, sfs = sf + s * kSfBytes;
          mbar_expect_tx(bar, kCodeBytes + sf_a + sf_b);
          tma_load_2d(at, &tmA, k * kRowBytes, m0, bar);
          tma_load_2d(at + kHalf * kRowBytes, &tmB, k * kRowBytes, n0, bar);
          const int64_t word = kNv ? k : k >> 1;
          if (sf_a) bulk_load(sfs, a_sf + word * p.M * 16, sf_a, bar);
          bulk_load(sfs + kHalf * 16, b_sf + word * p.N * 16, sf_b, bar);
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && lane == 0) {
      constexpr uint32_t kDesc = instr_desc<kNv, kTile, kTile>();
      int s = 0;
      uint32_t ph = 0u, aph = 1u;
      bool ok = true;
      for (int t = pair; t < tiles && ok; t += pairs) {
        if (!(ok = mbar_wait_cluster(acc_empty, aph, abort_flag))) break;
        aph ^= 1u;
        tc_fence_after();
        for (int k = 0; k < p.chunks; ++k) {
          if (!(ok = mbar_wait_cluster(ready + 8 * s, ph, abort_flag))) break;
          tc_fence_after();
          const uint64_t ad = make_desc(smem + s * kCodeBytes), bd = make_desc(smem + s * kCodeBytes + kHalf * kRowBytes);
          const uint32_t sfa = sf_cols + s * kSfCols, sfb = sfa + 16;
          const int steps = k == p.chunks - 1 ? p.last_steps : 4;
          for (int j = 0; j < steps; ++j) {
            const uint32_t word = kNv ? j : j >> 1;
            const uint32_t desc = kDesc | (kNv ? 0u : (static_cast<uint32_t>(j & 1) * 2u) * ((1u << 4) | (1u << 29)));
            mma_scaled<kNv, 2>(tmem, ad + 2 * j, bd + 2 * j, desc, sfa + 4 * word, sfb + 8 * word, (k | j) != 0);
          }
          tc2_commit_both(empty + 8 * s);
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
        if (ok) tc2_commit_both(acc_full);
      }
    }
  } else if (warp >= 4 && warp < 8) {
    const int q = warp & 3;
    const uint32_t ready_leader = mapa(ready, 0);
    int s = 0;
    uint32_t ph = 0u;
    bool ok = true;
    for (int t = pair; t < tiles && ok; t += pairs) {
      for (int k = 0; k < p.chunks; ++k) {
        if (!(ok = mbar_wait(full + 8 * s, ph, abort_flag))) break;
        tc_fence_after();
        const uint32_t src = sf + s * kSfBytes, dst = sf_cols + s * kSfCols + (static_cast<uint32_t>(q * 32) << 16);
        move_scales<kNv, 4>(src, dst, lane, k & 1);
        move_scales_256<kNv>(src + kHalf * 16, dst + 16, lane, k & 1);
        tmem_wait_st();
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(ready_leader + 8 * s);
        if (++s == kStages) { s = 0; ph ^= 1u; }
      }
    }
  } else if (warp >= 8) {
    const int q = warp & 3, c0 = (warp >= 12 ? kHalf : 0);
    const uint32_t acc = tmem + (static_cast<uint32_t>(q * 32) << 16) + c0, empty_leader = mapa(acc_empty, 0);
    const float alpha = p.alpha ? *p.alpha : 1.0f;
    const int size = p.dt == HIF4_FP32 ? 4 : 2;
    uint32_t ph = 0u;
    for (int t = pair; t < tiles; t += pairs) {
      const PairTile w = pair_tile(p, t);
      if (!__all_sync(0xFFFFFFFFu, mbar_wait(acc_full, ph, abort_flag, 64))) break;
      ph ^= 1u;
      tc_fence_after();
      const int64_t m = w.m0 + static_cast<int64_t>(rank) * kHalf + q * 32 + lane, n = w.n0 + c0;
      const bool whole = p.wide && n + kHalf <= p.N;
      uint8_t* row = static_cast<uint8_t*>(p.y) + (m * p.ld_y + n) * size;
      if (whole && size == 2) {
        uint32_t packed[64];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t r[32];
          tc_ld32(acc + 32 * c, r);
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float lo = alpha * __uint_as_float(r[2 * i]), hi = alpha * __uint_as_float(r[2 * i + 1]);
            packed[16 * c + i] = p.dt == HIF4_BF16 ? pack2(lo, hi, __nv_bfloat16()) : pack2(lo, hi, __half());
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(empty_leader);
        if (m < p.M) {
#pragma unroll
          for (int i = 0; i < 8; ++i) store32(row + 32 * i, packed + 8 * i);
        }
      } else {
        for (int c = 0; c < 4; ++c) {
          uint32_t r[32];
          tc_ld32(acc + 32 * c, r);
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(alpha * __uint_as_float(r[i]));
          if (m < p.M) {
            if (whole) {
#pragma unroll
              for (int i = 0; i < 4; ++i) store32(row + 128 * c + 32 * i, r + 8 * i);
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (n + 32 * c + i < p.N) store_y(p, m, n + 32 * c + i, __uint_as_float(r[i]));
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(empty_leader);
      }
    }
  }

  __syncwarp();
  if (*abort_flag) {
    // a wait gave up: let copies and MMAs in flight land before their memory is released
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 2000000ull) {}
    if (threadIdx.x == 0) atomicExch(p.error_word, 1u);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();            // neither CTA leaves while the other may still read its shared memory or arrive on its barriers
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

template <bool kNv>
hif4_status launch_pairs(const hif4_bfp4_gemm_args& a, Bfp4Params p, cudaStream_t st) {
  static uint64_t ready = 0;
  if (!ensure_dynamic_smem(bfp4_pair_kernel<kNv>, kSmem, ready)) return HIF4_ERR_CUDA;
  CUtensorMap tmA, tmB;
  if (!make_code_map(&tmA, a.A_codes, a.M, a.K, kHalf) || !make_code_map(&tmB, a.B_codes, a.N, a.K, kHalf)) return HIF4_ERR_CUDA;
  const int64_t m_tiles = ceil_div64(a.M, kTile), n_tiles = ceil_div64(a.N, kTile);
  if (m_tiles * n_tiles > 0x7FFFFFFFll - 1024 || n_tiles > 0x7FFFFFFFll / kBand) return HIF4_ERR_SHAPE;
  p.m_tiles = static_cast<int>(m_tiles);
  p.n_tiles = static_cast<int>(n_tiles);
  const int most = sm_count() / 2, tiles = p.m_tiles * p.n_tiles;
  bfp4_pair_kernel<kNv><<<2 * (tiles < most ? tiles : most), kThreads, kSmem, st>>>(tmA, tmB, p);
  note_launch();
  return launch_status();
}

}  // namespace

hif4_status launch_bfp4_pairs(const hif4_bfp4_gemm_args& a, Bfp4Params p, cudaStream_t st) {
  return a.fmt == HIF4_FMT_NVFP4 ? launch_pairs<true>(a, p, st) : launch_pairs<false>(a, p, st);
}

}  // namespace hif4
