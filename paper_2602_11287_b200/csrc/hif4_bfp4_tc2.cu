// CTA-pair form of the block-scaled product for prompts and large groups: a cluster of two CTAs on 256 tokens x 256 rows of B
// (tcgen05.mma.cta_group::2), persistent over its tiles.  Each CTA holds its 128 tokens and 128 of the rows of B, so an SM reads
// 8 KB from L2 for a K = 64 step of 128 x 256 outputs; it needs the scales of all 256 rows of B, though.
//
// Codes and scales have rings of their own (5 stages of 32 KB, 5 of 6 KB), so that the scales' way to tensor memory does not add to
// the codes' latency: four warps read a chunk's scales ahead of time, store them (48 columns beside the 256 accumulator columns)
// as soon as the MMAs that used these columns are done, and tell the leader's MMA thread; one more thread tells it that a CTA's codes
// are there.  Eight epilogue warps.  The accumulator is single: 16-bit outputs are read into registers as pairs and the accumulator
// handed back before any of them is stored, so that the next tile's first MMAs wait for tensor-memory reads only; Y leaves
// through swizzled slabs and TMA stores (32-byte stores from registers: 108 us against 97).
//
// 4096 x 14336 x 4096 NVFP4 on a warm device 97 us, 5.0 PFLOP/s; K = 14336 5.7; tensor pipe 69 % active.  MMAs alone run at 7.7
// PFLOP/s, the loads alone would feed 8.0, both together 6.0: they share the shared-memory port and the ring holds 160 KB of 1.3 us
// of latency.  The rest: Y's 117 MB, 13 rounds for 12.1 rounds of tiles, and a drained accumulator between tiles (0.3 us each).
#include "hif4_bfp4_gemm.cuh"

namespace hif4 {
namespace {

constexpr int kThreads = 512;                // warps: codes, MMA, TMEM allocation and arrival of codes, scales, 4 x scales to TMEM, 8 x epilogue
constexpr int kTile = 256, kHalf = 128;
constexpr int kStages = 5, kSfStages = 5;
constexpr int kCodeBytes = 2 * kHalf * kRowBytes;
constexpr int kSfBytes = (kHalf + kTile) * 16;
constexpr int kSlabBytes = 32 * 128;         // 32 rows x 128 bytes of Y, one per epilogue warp, in SWIZZLE_128B order
constexpr int kSlabs = kStages * kCodeBytes;
constexpr int kSf = kSlabs + 8 * kSlabBytes;
constexpr int kTable = kSf + kSfStages * kSfBytes;
constexpr int kBars = kTable + kGroupTableBytes;
constexpr int kSmem = 1024 + kBars + 512;
constexpr int kSfCols = 48;                  // of a stage: 16 for the tokens, 32 for B
constexpr int kTmemCols = 512;
constexpr int kBand = 16;                    // token tiles that are walked together (their codes stay in L2)
static_assert(kTile + kStages * kSfCols <= kTmemCols, "TMEM");
static_assert(kSmem <= 227 * 1024, "shared memory");

// Tile t of a dense product (bands of token tiles, within a band the token tiles of the same rows of B) or of a grouped one.
struct PairTile { int group, m0, m_end, n0; };
template <bool kGrouped>
__device__ __forceinline__ PairTile pair_tile(const GroupTable& table, const Bfp4Params& p, int t) {
  if (kGrouped) {
    const GroupTile w = group_tile(table, p, t, kTile);
    return {w.group, w.m0, w.m_end, w.nt * kTile};
  }
  const int band_tiles = kBand * p.n_tiles, band = t / band_tiles, in = t - band * band_tiles;
  const int rows = min(kBand, p.m_tiles - band * kBand);
  const int nt = in / rows, mt = band * kBand + in - nt * rows;
  return {0, mt * kTile, static_cast<int>(p.M), nt * kTile};
}

// Y is written once and larger than what the codes leave of L2: its lines are the first to go.
__device__ __forceinline__ uint64_t evict_first_policy() {
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ void tma_store_hinted(const CUtensorMap* map, int x, int y, uint32_t src, uint64_t policy) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group.L2::cache_hint [%0, {%1, %2}], [%3], %4;" ::"l"(map), "r"(x), "r"(y), "r"(src),
               "l"(policy) : "memory");
}
// A warp's 32 words per lane (128 bytes of its lane's row) -> its slab, once the copy before has read it.
__device__ __forceinline__ void fill_slab(uint32_t slab, const uint32_t* w, int lane) {
  if (lane == 0) bulk_wait_read<0>();
  __syncwarp();
  const uint32_t row = slab + lane * 128u, r7 = static_cast<uint32_t>(lane) & 7u;
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) sts128(row + ((i ^ r7) << 4), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}
__device__ __forceinline__ void store_slab(const CUtensorMap* map, int x, int y, uint32_t slab, const uint32_t* w, int lane, uint64_t policy) {
  fill_slab(slab, w, lane);
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) {
    tma_store_hinted(map, x, y, slab, policy);
    bulk_commit();
  }
}
// The same without a box, for rows at any address and the last rows of a group: a row after the other, the lanes along it (four bytes
// a lane where Y allows, so that a row's 128 bytes are one store).  From the registers, a row a lane, 3798 x 2836 x 1024 took 125 us.
template <typename Word>
__device__ __forceinline__ void copy_slab(Word* y, int64_t ld, int rows, int cols, uint32_t slab, int lane) {
  constexpr int kOfRow = 128 / static_cast<int>(sizeof(Word));
  for (int r = 0; r < rows; ++r) {
#pragma unroll
    for (int e0 = 0; e0 < kOfRow; e0 += 32) {
      const uint32_t e = static_cast<uint32_t>(e0 + lane), at = e * sizeof(Word), src = slab + r * 128u + (((at >> 4) ^ (r & 7u)) << 4) + (at & 15u);
      if (static_cast<int>(e) < cols) {
        if constexpr (sizeof(Word) == 4) {
          y[r * ld + e] = lds32(src);
        } else {
          uint16_t v;
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(src));
          y[r * ld + e] = v;
        }
      }
    }
  }
}
__device__ __forceinline__ void store_rows(const Bfp4Params& p, int n, int m, int m_end, uint32_t slab, const uint32_t* w, int lane) {
  fill_slab(slab, w, lane);
  __syncwarp();
  const int rows = min(32, m_end - m);
  const int64_t at = static_cast<int64_t>(m) * p.ld_y + n;
  const int64_t cols = p.N - n;
  if (p.dt == HIF4_FP32) copy_slab(static_cast<uint32_t*>(p.y) + at, p.ld_y, rows, static_cast<int>(min(cols, static_cast<int64_t>(32))), slab, lane);
  else if (p.pair_words) copy_slab(static_cast<uint32_t*>(p.y) + at / 2, p.ld_y / 2, rows, static_cast<int>(min(cols, static_cast<int64_t>(64)) / 2), slab, lane);
  else copy_slab(static_cast<uint16_t*>(p.y) + at, p.ld_y, rows, static_cast<int>(min(cols, static_cast<int64_t>(64))), slab, lane);
  __syncwarp();
}

template <bool kNv, bool kGrouped>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
bfp4_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmY,
                 const __grid_constant__ Bfp4Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sf = smem + kSf, bars = smem + kBars;
  // full: this CTA's codes; empty: codes and scale columns are free; sf_full, sf_empty: ring of scales; ready (on rank 0): codes and
  // scale columns of both CTAs
  const uint32_t full = bars, empty = full + 8 * kStages, ready = empty + 8 * kStages, sf_full = ready + 8 * kStages,
                 sf_empty = sf_full + 8 * kSfStages, acc_full = sf_empty + 8 * kSfStages, acc_empty = acc_full + 8, slot = acc_full + 16;
  uint8_t* gen = smem_raw + (smem - smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + (slot - smem));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  GroupTable& table = *reinterpret_cast<GroupTable*>(gen + kTable);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
      mbar_init(ready + 8 * s, 10);                      // of each CTA: four warps for the scales, one thread for the codes
    }
    for (int s = 0; s < kSfStages; ++s) {
      mbar_init(sf_full + 8 * s, 1);
      mbar_init(sf_empty + 8 * s, 4);
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
  grid_wait();
  grid_launch_next();
  if (kGrouped && warp == 3) build_group_table(table, p, kTile, lane);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, sf_cols = tmem + kTile;
  const int tiles = (kGrouped ? table.tiles[p.num_groups] : p.m_tiles) * p.n_tiles;

  if (warp == 0) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 1u;
      bool ok = true;
      for (int t = pair; t < tiles && ok; t += pairs) {
        const PairTile w = pair_tile<kGrouped>(table, p, t);
        const int m0 = w.m0 + static_cast<int>(rank) * kHalf, n0 = static_cast<int>(w.group * p.N + w.n0) + static_cast<int>(rank) * kHalf;
        for (int k = 0; k < p.chunks; ++k) {
          if (!(ok = mbar_wait(empty + 8 * s, ph, abort_flag))) break;
          const uint32_t bar = full + 8 * s, at = smem + s * kCodeBytes;
          mbar_expect_tx(bar, kCodeBytes);
          tma_load_2d(at, &tmA, k * kRowBytes, m0, bar);
          tma_load_2d(at + kHalf * kRowBytes, &tmB, k * kRowBytes, n0, bar);
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 3) {
    if (lane == 0) {
      int z = 0;
      uint32_t ph = 1u;
      bool ok = true;
      for (int t = pair; t < tiles && ok; t += pairs) {
        const PairTile w = pair_tile<kGrouped>(table, p, t);
        const int m0 = w.m0 + static_cast<int>(rank) * kHalf;
        const uint32_t sf_a = static_cast<uint32_t>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(kHalf), p.M - m0))) * 16u;
        const uint32_t sf_b = static_cast<uint32_t>(min(static_cast<int64_t>(kTile), p.N - w.n0)) * 16u;
        const uint8_t *a_sf = p.a_scales + static_cast<int64_t>(m0) * 16, *b_sf = p.b_scales + w.group * p.b_scale_group + static_cast<int64_t>(w.n0) * 16;
        for (int k = 0; k < p.chunks; ++k) {
          if (!(ok = mbar_wait(sf_empty + 8 * z, ph, abort_flag))) break;
          const uint32_t bar = sf_full + 8 * z, sfs = sf + z * kSfBytes;
          mbar_expect_tx(bar, sf_a + sf_b);
          const int64_t word = kNv ? k : k >> 1;
          if (sf_a) bulk_load(sfs, a_sf + word * p.M * 16, sf_a, bar);
          bulk_load(sfs + kHalf * 16, b_sf + word * p.N * 16, sf_b, bar);
          if (++z == kSfStages) { z = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 2) {
    if (lane == 0) {
      const uint32_t ready_leader = mapa(ready, 0);
      int s = 0;
      uint32_t ph = 0u;
      bool ok = true;
      for (int t = pair; t < tiles && ok; t += pairs) {
        for (int k = 0; k < p.chunks; ++k) {
          if (!(ok = mbar_wait(full + 8 * s, ph, abort_flag))) break;
          mbar_arrive_cluster(ready_leader + 8 * s);
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      constexpr uint32_t kDesc = instr_desc<kNv, kTile, kTile>();
      const uint64_t ad0 = make_desc(smem), bd0 = make_desc(smem + kHalf * kRowBytes);
      const bool issuer = elect_one();
      int s = 0;
      uint32_t ph = 0u, aph = 1u;
      bool ok = true;
      for (int t = pair; t < tiles && ok; t += pairs) {
        if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(acc_empty, aph, abort_flag)))) break;
        aph ^= 1u;
        tc_fence_after();
        for (int k = 0; k < p.chunks; ++k) {
          if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(ready + 8 * s, ph, abort_flag)))) break;
          tc_fence_after();
          const uint64_t off = static_cast<uint64_t>(s * (kCodeBytes >> 4));
          const uint32_t sfa = sf_cols + s * kSfCols;
          if (issuer) {
            mma_stage<kNv, 2, 4, 8>(tmem, ad0 + off, bd0 + off, kDesc, sfa, sfa + 16, k == p.chunks - 1 ? p.last_steps : 4, k == 0);
            tc2_commit_both(empty + 8 * s);
          }
          __syncwarp();
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
        if (ok && issuer) tc2_commit_both(acc_full);
        __syncwarp();
      }
    }
  } else if (warp >= 4 && warp < 8) {
    const int q = warp & 3;
    const uint32_t ready_leader = mapa(ready, 0);
    int s = 0, z = 0;
    uint32_t ph = 1u, sph = 0u;
    bool ok = true;
    for (int t = pair; t < tiles && ok; t += pairs) {
      for (int k = 0; k < p.chunks; ++k) {
        if (!(ok = mbar_wait(sf_full + 8 * z, sph, abort_flag))) break;
        uint32_t wa[16], wb[32];
        read_scales<kNv, 4>(sf + z * kSfBytes, lane, k & 1, wa);
        read_scales<kNv, 8>(sf + z * kSfBytes + kHalf * 16, lane, k & 1, wb);
        if (!(ok = mbar_wait(empty + 8 * s, ph, abort_flag))) break;
        tc_fence_after();
        const uint32_t dst = sf_cols + s * kSfCols + (static_cast<uint32_t>(q * 32) << 16);
        tmem_st16(dst, wa);
        tmem_st16(dst + 16, *reinterpret_cast<const uint32_t(*)[16]>(wb));
        if (kNv) tmem_st16(dst + 32, *reinterpret_cast<const uint32_t(*)[16]>(wb + 16));
        tmem_wait_st();                                  // the words have been read, so the ring's stage may be filled again
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive_cluster(ready_leader + 8 * s);
          mbar_arrive(sf_empty + 8 * z);
        }
        if (++s == kStages) { s = 0; ph ^= 1u; }
        if (++z == kSfStages) { z = 0; sph ^= 1u; }
      }
    }
  } else if (warp >= 8) {
    const int q = warp & 3, c0 = (warp >= 12 ? kHalf : 0);
    const uint32_t acc = tmem + (static_cast<uint32_t>(q * 32) << 16) + c0, empty_leader = mapa(acc_empty, 0);
    const uint32_t slab = smem + kSlabs + (warp - 8) * kSlabBytes;
    const uint64_t policy = evict_first_policy();
    uint32_t ph = 0u;
    for (int t = pair; t < tiles; t += pairs) {
      const PairTile w = pair_tile<kGrouped>(table, p, t);
      if (!__all_sync(0xFFFFFFFFu, mbar_wait(acc_full, ph, abort_flag, 64))) break;
      ph ^= 1u;
      tc_fence_after();
      const int m = w.m0 + static_cast<int>(rank) * kHalf + q * 32, n = w.n0 + c0;       // the warp's first row and column
      const bool inside = m < w.m_end && n < p.N, boxes = p.tma_store && (!kGrouped || m + 32 <= w.m_end);      // (a box would reach into the next group)
      const float alpha = p.alpha ? p.alpha[w.group] : 1.0f;
      if (p.dt != HIF4_FP32) {
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
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          if (!inside || n + 64 * c >= p.N) continue;
          if (boxes) store_slab(&tmY, n + 64 * c, m, slab, packed + 32 * c, lane, policy);
          else store_rows(p, n + 64 * c, m, w.m_end, slab, packed + 32 * c, lane);
        }
      } else {
        for (int c = 0; c < 4; ++c) {
          uint32_t r[32];
          tc_ld32(acc + 32 * c, r);
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(alpha * __uint_as_float(r[i]));
          if (!inside || n + 32 * c >= p.N) continue;
          if (boxes) store_slab(&tmY, n + 32 * c, m, slab, r, lane, policy);
          else store_rows(p, n + 32 * c, m, w.m_end, slab, r, lane);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(empty_leader);
      }
    }
    if (lane == 0) bulk_wait_all();
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

template <bool kNv, bool kGrouped>
hif4_status launch_pairs(const hif4_bfp4_gemm_args& a, Bfp4Params p, cudaStream_t st) {
  static uint64_t ready = 0;
  if (!ensure_dynamic_smem(bfp4_pair_kernel<kNv, kGrouped>, kSmem, ready)) return HIF4_ERR_CUDA;
  CUtensorMap tmA, tmB, tmY;
  if (!make_code_map(&tmA, a.A_codes, a.M, a.K, kHalf) || !make_code_map(&tmB, a.B_codes, a.N * (kGrouped ? a.num_groups : 1), a.K, kHalf)) return HIF4_ERR_CUDA;
  // (a TMA store clips the innermost dimension in 16-byte pieces, so a row's length has to be whole ones)
  const int64_t size = a.dt == HIF4_FP32 ? 4 : 2;
  p.tma_store = (reinterpret_cast<uintptr_t>(a.Y) & 15u) == 0 && a.ld_y * size % 16 == 0 && a.N * size % 16 == 0 && make_y_map(&tmY, a, static_cast<int>(128 / size), 32, CU_TENSOR_MAP_SWIZZLE_128B);
  if (!p.tma_store) tmY = tmA;                           // not used
  p.pair_words = size == 2 && ((reinterpret_cast<uintptr_t>(a.Y) | static_cast<uintptr_t>(2 * (a.ld_y | a.N))) & 3u) == 0;
  const int64_t m_tiles = ceil_div64(a.M, kTile) + (kGrouped ? a.num_groups : 0), n_tiles = ceil_div64(a.N, kTile);
  if (m_tiles * n_tiles > 0x7FFFFFFFll - 1024 || n_tiles > 0x7FFFFFFFll / kBand) return HIF4_ERR_SHAPE;
  p.m_tiles = static_cast<int>(m_tiles);
  p.n_tiles = static_cast<int>(n_tiles);
  const int most = sm_count() / 2, tiles = p.m_tiles * p.n_tiles;
  return launch_overlapped(bfp4_pair_kernel<kNv, kGrouped>, static_cast<unsigned>(2 * (tiles < most ? tiles : most)), kThreads, kSmem, st, tmA, tmB, tmY, p);
}

}  // namespace

hif4_status launch_bfp4_pairs(const hif4_bfp4_gemm_args& a, Bfp4Params p, cudaStream_t st) {
  const bool nv = a.fmt == HIF4_FMT_NVFP4;
  if (a.num_groups > 0) return nv ? launch_pairs<true, true>(a, p, st) : launch_pairs<false, true>(a, p, st);
  return nv ? launch_pairs<true, false>(a, p, st) : launch_pairs<false, false>(a, p, st);
}

}  // namespace hif4
