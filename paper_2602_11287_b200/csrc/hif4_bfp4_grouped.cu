// Persistent form of the block-scaled product for groups of few rows (experts of a small batch): a CTA an SM walks tiles of 128
// rows of B times T tokens (the MMA's N side), so that a group of few rows costs few columns.  Bound by the stream of B's codes:
// the tiles of a group that share rows of B follow one another, so that B comes from HBM once.
//
// Warps: codes and scales (TMA, one ring), MMA, table of the groups, two teams of four that move scales to tensor memory (even and
// odd stages: a stage's way through shared memory, registers and tensor memory takes longer than its MMAs), eight epilogue warps on two
// accumulators.  A lane is a column of Y: a tile goes through shared memory and leaves as one copy per token's row.  (Stored from
// the registers, 32 elements a warp and instruction, Y took longer than all else: 119 us against 64 without stores, 32 experts,
// 4096 rows, 2048 -> 7168.)
#include "hif4_bfp4_gemm.cuh"

namespace hif4 {
namespace {

constexpr int kThreads = 640;
constexpr int BW = 128;
constexpr int kTmemCols = 512;

template <int T> struct Shape {
  static constexpr int kStages = T == 128 ? 4 : T == 64 ? 6 : 8;      // even: a stage always has the same team
  static constexpr int kCodeBytes = (BW + T) * kRowBytes;
  static constexpr int kSfBytes = (BW + T) * 16;
  static constexpr int kRows = kStages * (kCodeBytes + kSfBytes);       // T rows of 128 elements of Y
  static constexpr int kTable = kRows + T * BW * 4;
  static constexpr int kBars = kTable + kGroupTableBytes;
  static constexpr int kSmem = 1024 + kBars + 512;
  static_assert(2 * T + kStages * 32 <= kTmemCols && kSmem <= 227 * 1024 && T >= 32, "TMEM, shared memory");
};

// Barrier of an epilogue team's 128 threads.
__device__ __forceinline__ void team_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }
// The same, and whether any of them says so.
__device__ __forceinline__ bool team_any(int id, bool mine) {
  uint32_t any;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.or.pred q, %1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(any) : "r"(id), "r"(static_cast<uint32_t>(mine)) : "memory");
  return any != 0u;
}
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}

template <int T, bool kNv>
__global__ void __launch_bounds__(kThreads, 1)
bfp4_grouped_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ Bfp4Params p) {
  using S = Shape<T>;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sf = smem + kStages * S::kCodeBytes, bars = smem + S::kBars;
  const uint32_t full = bars, ready = full + 8 * kStages, empty = ready + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 16,
                 slot = acc_empty + 16;
  uint8_t* gen = smem_raw + (smem - smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + (slot - smem));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  GroupTable& table = *reinterpret_cast<GroupTable*>(gen + S::kTable);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(ready + 8 * s, 4);
      mbar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(acc_full + 8 * b, 1);
      mbar_init(acc_empty + 8 * b, 2);
    }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_wait();
  grid_launch_next();
  if (warp == 3) build_group_table(table, p, T, lane);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, sf_cols = tmem + 2 * T;
  const int tiles = table.tiles[p.num_groups] * p.n_tiles;

  if (warp == 0) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 1u;
      bool ok = true;
      for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
        const GroupTile w = group_tile(table, p, t, T);
        const int64_t n0 = static_cast<int64_t>(w.nt) * BW;
        const int b_row = static_cast<int>(w.group * p.N + n0);
        const uint32_t rows_b = static_cast<uint32_t>(min(static_cast<int64_t>(BW), p.N - n0)) * 16u;
        const uint32_t rows_a = static_cast<uint32_t>(min(static_cast<int64_t>(T), p.M - w.m0)) * 16u;
        const uint8_t *b_sf = p.b_scales + w.group * p.b_scale_group + n0 * 16, *a_sf = p.a_scales + static_cast<int64_t>(w.m0) * 16;
        for (int k = 0; k < p.chunks; ++k) {
          if (!(ok = mbar_wait(empty + 8 * s, ph, abort_flag))) break;
          const uint32_t bar = full + 8 * s, at = smem + s * S::kCodeBytes, sfs = sf + s * S::kSfBytes;
          mbar_expect_tx(bar, S::kCodeBytes + rows_a + rows_b);
          const int64_t word = kNv ? k : k >> 1;
          bulk_load(sfs, b_sf + word * p.N * 16, rows_b, bar);
          bulk_load(sfs + BW * 16, a_sf + word * p.M * 16, rows_a, bar);
          tma_load_2d(at, &tmB, k * kRowBytes, b_row, bar);
          tma_load_2d(at + BW * kRowBytes, &tmA, k * kRowBytes, w.m0, bar);
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    constexpr uint32_t kDesc = instr_desc<kNv, BW, T>();
    const uint64_t bd0 = make_desc(smem), ad0 = make_desc(smem + BW * kRowBytes);
    const bool issuer = elect_one();
    int s = 0, b = 0;
    uint32_t ph = 0u, aph = 1u;
    bool ok = true;
    for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
      if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(acc_empty + 8 * b, aph, abort_flag)))) break;
      tc_fence_after();
      for (int k = 0; k < p.chunks; ++k) {
        if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(full + 8 * s, ph, abort_flag) && mbar_wait(ready + 8 * s, ph, abort_flag)))) break;
        tc_fence_after();
        const uint64_t off = static_cast<uint64_t>(s * (S::kCodeBytes >> 4));
        const uint32_t sfb = sf_cols + s * 32;
        if (issuer) {
          mma_stage<kNv, 1, 4, 4>(tmem + b * T, bd0 + off, ad0 + off, kDesc, sfb, sfb + 16, k == p.chunks - 1 ? p.last_steps : 4, k == 0);
          tc_commit(empty + 8 * s);
        }
        __syncwarp();
        if (++s == kStages) { s = 0; ph ^= 1u; }
      }
      if (ok && issuer) tc_commit(acc_full + 8 * b);
      __syncwarp();
      b ^= 1;
      if (b == 0) aph ^= 1u;
    }
  } else if (warp >= 4 && warp < 12) {
    const int q = warp & 3, team = (warp >> 2) - 1;
    int s = 0;
    uint32_t ph = 0u;
    bool ok = true;
    for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
      for (int k = 0; k < p.chunks; ++k) {
        if ((s & 1) == team) {
          if (!(ok = mbar_wait(full + 8 * s, ph, abort_flag))) break;
          tc_fence_after();
          const uint32_t src = sf + s * S::kSfBytes, dst = sf_cols + s * 32 + (static_cast<uint32_t>(q * 32) << 16);
          move_scales<kNv, 4>(src, dst, lane, k & 1);
          move_scales<kNv, T / 32>(src + BW * 16, dst + 16, lane, k & 1);
          tmem_wait_st();                                // the words have been read: the stage may be filled again after its MMAs
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(ready + 8 * s);
        }
        if (++s == kStages) { s = 0; ph ^= 1u; }
      }
    }
  } else if (warp >= 12) {
    // two teams of four warps, half of the tokens each
    const int q = warp & 3, team = warp >= 16 ? 1 : 0, c0 = team * (T / 2), thread = threadIdx.x & 127;
    const int size = p.dt == HIF4_FP32 ? 4 : 2;
    uint8_t* rows = gen + S::kRows + c0 * BW * 4;
    int b = 0;
    uint32_t ph = 0u;
    for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
      const GroupTile w = group_tile(table, p, t, T);
      const float alpha = p.alpha ? p.alpha[w.group] : 1.0f;
      const int64_t n0 = static_cast<int64_t>(w.nt) * BW, n = n0 + q * 32 + lane;
      const int m = w.m0 + c0, count = w.m_end - m;       // (may be none or negative)
      const bool ok = mbar_wait(acc_full + 8 * b, ph, abort_flag, 32);
      if (p.row_copies) bulk_wait_read<0>();              // the copies before have read the rows
      if (team_any(1 + team, !ok)) break;                 // one answer for the whole team: it leaves together or not at all
      tc_fence_after();
      const uint32_t acc = tmem + b * T + c0 + (static_cast<uint32_t>(q * 32) << 16);
#pragma unroll
      for (int c = 0; c < T / 2; c += 16) {
        uint32_t r[16];
        tc_ld16(acc + c, r);
        tc_wait_ld();
        if (!p.row_copies) {
          if (n < p.N) store_tokens(p, m + c, count - c, n, alpha, r);
        } else if (p.dt == HIF4_FP32) {
          store_tokens_as(reinterpret_cast<float*>(rows) + c * BW + q * 32 + lane, BW, 16, alpha, r);
        } else if (p.dt == HIF4_BF16) {
          store_tokens_as(reinterpret_cast<__nv_bfloat16*>(rows) + c * BW + q * 32 + lane, BW, 16, alpha, r);
        } else {
          store_tokens_as(reinterpret_cast<__half*>(rows) + c * BW + q * 32 + lane, BW, 16, alpha, r);
        }
      }
      tc_fence_before();
      fence_proxy_async_smem();
      team_sync(1 + team);
      if (thread == 0) mbar_arrive(acc_empty + 8 * b);
      if (p.row_copies && thread < T / 2 && thread < count) {
        const uint32_t bytes = static_cast<uint32_t>(min(static_cast<int64_t>(BW), p.N - n0)) * size;
        bulk_store(static_cast<uint8_t*>(p.y) + ((static_cast<int64_t>(m) + thread) * p.ld_y + n0) * size, smem_u32(rows) + thread * BW * size, bytes);
        bulk_commit();
      }
      b ^= 1;
      if (b == 0) ph ^= 1u;
    }
    bulk_wait_all();
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
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

template <int T, bool kNv>
hif4_status launch(const hif4_bfp4_gemm_args& a, Bfp4Params p, cudaStream_t st) {
  const auto kernel = bfp4_grouped_kernel<T, kNv>;
  static uint64_t ready = 0;
  if (!ensure_dynamic_smem(kernel, Shape<T>::kSmem, ready)) return HIF4_ERR_CUDA;
  CUtensorMap tmA, tmB;
  if (!make_code_map(&tmA, a.A_codes, a.M, a.K, T) || !make_code_map(&tmB, a.B_codes, a.N * a.num_groups, a.K, BW)) return HIF4_ERR_CUDA;
  const int64_t size = a.dt == HIF4_FP32 ? 4 : 2;
  p.row_copies = ((reinterpret_cast<uintptr_t>(a.Y) | static_cast<uintptr_t>(a.ld_y * size) | static_cast<uintptr_t>(a.N * size)) & 15u) == 0;
  const int64_t most = (ceil_div64(a.M, T) + a.num_groups) * p.n_tiles;
  if (most > 0x7FFFFFFFll - 1024) return HIF4_ERR_SHAPE;
  return launch_overlapped(kernel, static_cast<unsigned>(most < sm_count() ? most : sm_count()), kThreads, Shape<T>::kSmem, st, tmA, tmB, p);
}

}  // namespace

hif4_status launch_bfp4_grouped(const hif4_bfp4_gemm_args& a, Bfp4Params p, cudaStream_t st) {
  const bool nv = a.fmt == HIF4_FMT_NVFP4;
  const int64_t mean = ceil_div64(a.M, a.num_groups);
  if (mean <= 32) return nv ? launch<32, true>(a, p, st) : launch<32, false>(a, p, st);
  if (mean <= 64) return nv ? launch<64, true>(a, p, st) : launch<64, false>(a, p, st);
  return nv ? launch<128, true>(a, p, st) : launch<128, false>(a, p, st);
}

}  // namespace hif4
