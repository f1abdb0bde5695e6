// Persistent form of the block-scaled product for groups of few rows (experts of a small batch): a CTA an SM walks tiles of 128
// rows of B times T tokens (the MMA's N side), so that a group of few rows costs few columns.  Bound by the stream of B's codes:
// the tiles of a group that share rows of B follow one another, so that B comes from HBM once.
//
// Warps: codes, MMA, scales and table of the groups, two teams of four that move scales to tensor memory, eight epilogue warps on two
// accumulators.  Codes and scales have rings of their own, so that a stage of codes waits for its bytes and its MMAs only.  A
// lane is a column of Y: 8 KB at a time go through shared memory and leave as one copy, or as one copy per token's row where the
// group ends.
//
// 32 experts, 4096 rows, 2048 -> 7168, MXFP4: 65 us BF16, 70 us FP32 (floor 51 and 57: 249 MB of codes and scales, Y), 60 without Y.
// Before: one ring of four stages for both 74 and 78 us; Y stored from the registers, 32 elements a warp and instruction, 130 and 119.
// 256 experts, 7168 -> 4096, 2048 rows: 620 us for 4.1 GB of weights (6.6 TB/s).
#include "hif4_bfp4_gemm.cuh"

namespace hif4 {
namespace {

constexpr int kThreads = 640;
constexpr int BW = 128;
constexpr int kTmemCols = 512;

constexpr int kRowBufBytes = 8192;           // 16 tokens in FP32, 32 in 16 bits

template <int T> struct Shape {
  static constexpr int kStages = T == 128 ? 5 : T == 64 ? 6 : 8;         // codes
  static constexpr int kSfStages = 6;                                   // scales; even: a stage always has the same team
  static constexpr int kCodeBytes = (BW + T) * kRowBytes;
  static constexpr int kSfBytes = (BW + T) * 16;
  static constexpr int kSf = kStages * kCodeBytes;
  static constexpr int kRows = kSf + kSfStages * kSfBytes;               // rows of 128 elements of Y: two buffers for each team
  static constexpr int kTable = kRows + 4 * kRowBufBytes;
  static constexpr int kBars = kTable + kGroupTableBytes;
  static constexpr int kSmem = 1024 + kBars + 512;
  static_assert(2 * T + kSfStages * 32 <= kTmemCols && kSmem <= 227 * 1024 && T >= 32, "TMEM, shared memory");
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
bfp4_grouped_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmY,
                    const __grid_constant__ Bfp4Params p) {
  using S = Shape<T>;
  constexpr int kStages = S::kStages, kSfStages = S::kSfStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sf = smem + S::kSf, bars = smem + S::kBars;
  // codes: full, empty; scales: sf_full, sf_empty in shared memory, ready, free in tensor memory
  const uint32_t full = bars, empty = full + 8 * kStages, sf_full = empty + 8 * kStages, sf_empty = sf_full + 8 * kSfStages, ready = sf_empty + 8 * kSfStages,
                 free = ready + 8 * kSfStages, acc_full = free + 8 * kSfStages, acc_empty = acc_full + 16, slot = acc_empty + 16;
  uint8_t* gen = smem_raw + (smem - smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + (slot - smem));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  GroupTable& table = *reinterpret_cast<GroupTable*>(gen + S::kTable);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int z = 0; z < kSfStages; ++z) {
      mbar_init(sf_full + 8 * z, 1);
      mbar_init(sf_empty + 8 * z, 4);
      mbar_init(ready + 8 * z, 4);
      mbar_init(free + 8 * z, 1);
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
        const int b_row = static_cast<int>(w.group * p.N + static_cast<int64_t>(w.nt) * BW);
        for (int k = 0; k < p.chunks; ++k) {
          if (!(ok = mbar_wait(empty + 8 * s, ph, abort_flag))) break;
          const uint32_t bar = full + 8 * s, at = smem + s * S::kCodeBytes;
          mbar_expect_tx(bar, S::kCodeBytes);
          tma_load_2d(at, &tmB, k * kRowBytes, b_row, bar);
          tma_load_2d(at + BW * kRowBytes, &tmA, k * kRowBytes, w.m0, bar);
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 3) {
    if (lane == 0) {
      int z = 0;
      uint32_t ph = 1u;
      bool ok = true;
      for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
        const GroupTile w = group_tile(table, p, t, T);
        const int64_t n0 = static_cast<int64_t>(w.nt) * BW;
        const uint32_t rows_b = static_cast<uint32_t>(min(static_cast<int64_t>(BW), p.N - n0)) * 16u;
        const uint32_t rows_a = static_cast<uint32_t>(min(static_cast<int64_t>(T), p.M - w.m0)) * 16u;
        const uint8_t *b_sf = p.b_scales + w.group * p.b_scale_group + n0 * 16, *a_sf = p.a_scales + static_cast<int64_t>(w.m0) * 16;
        for (int k = 0; k < p.chunks; ++k) {
          if (!(ok = mbar_wait(sf_empty + 8 * z, ph, abort_flag))) break;
          const uint32_t bar = sf_full + 8 * z, at = sf + z * S::kSfBytes;
          const int64_t word = kNv ? k : k >> 1;
          mbar_expect_tx(bar, rows_a + rows_b);
          bulk_load(at, b_sf + word * p.N * 16, rows_b, bar);
          bulk_load(at + BW * 16, a_sf + word * p.M * 16, rows_a, bar);
          if (++z == kSfStages) { z = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    constexpr uint32_t kDesc = instr_desc<kNv, BW, T>();
    const uint64_t bd0 = make_desc(smem), ad0 = make_desc(smem + BW * kRowBytes);
    const bool issuer = elect_one();
    int s = 0, z = 0, b = 0;
    uint32_t ph = 0u, zph = 0u, aph = 1u;
    bool ok = true;
    for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
      if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(acc_empty + 8 * b, aph, abort_flag)))) break;
      tc_fence_after();
      for (int k = 0; k < p.chunks; ++k) {
        if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(ready + 8 * z, zph, abort_flag) && mbar_wait(full + 8 * s, ph, abort_flag)))) break;
        tc_fence_after();
        const uint64_t off = static_cast<uint64_t>(s * (S::kCodeBytes >> 4));
        const uint32_t sfb = sf_cols + z * 32;
        if (issuer) {
          mma_stage<kNv, 1, 4, 4>(tmem + b * T, bd0 + off, ad0 + off, kDesc, sfb, sfb + 16, k == p.chunks - 1 ? p.last_steps : 4, k == 0);
          tc_commit(empty + 8 * s);
          tc_commit(free + 8 * z);
        }
        __syncwarp();
        if (++s == kStages) { s = 0; ph ^= 1u; }
        if (++z == kSfStages) { z = 0; zph ^= 1u; }
      }
      if (ok && issuer) tc_commit(acc_full + 8 * b);
      __syncwarp();
      b ^= 1;
      if (b == 0) aph ^= 1u;
    }
  } else if (warp >= 4 && warp < 12) {
    const int q = warp & 3, team = (warp >> 2) - 1;
    int z = 0;
    uint32_t ph = 0u;
    bool ok = true;
    for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
      for (int k = 0; k < p.chunks; ++k) {
        if ((z & 1) == team) {
          if (!(ok = mbar_wait(sf_full + 8 * z, ph, abort_flag))) break;
          uint32_t wb[16], wa[16];
          read_scales<kNv, 4>(sf + z * S::kSfBytes, lane, k & 1, wb);
          read_scales_128<kNv, T / 32>(sf + z * S::kSfBytes + BW * 16, lane, k & 1, wa);
          if (!(ok = mbar_wait(free + 8 * z, ph ^ 1u, abort_flag))) break;
          tc_fence_after();
          const uint32_t dst = sf_cols + z * 32 + (static_cast<uint32_t>(q * 32) << 16);
          tmem_st16(dst, wb);
          tmem_st16(dst + 16, wa);
          tmem_wait_st();                                // the words have been read: the ring's stage may be filled again
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(ready + 8 * z);
            mbar_arrive(sf_empty + 8 * z);
          }
        }
        if (++z == kSfStages) { z = 0; ph ^= 1u; }
      }
    }
  } else if (warp >= 12) {
    // two teams of four warps, half of the tokens each
    const int q = warp & 3, team = warp >= 16 ? 1 : 0, c0 = team * (T / 2), thread = threadIdx.x & 127;
    const int size = p.dt == HIF4_FP32 ? 4 : 2;
    const int pass = min(T / 2, kRowBufBytes / (BW * size));              // tokens a buffer
    uint8_t* rows0 = gen + S::kRows + team * 2 * kRowBufBytes;
    int b = 0, buf = 0;
    uint32_t ph = 0u;
    bool ok = true;
    for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
      const GroupTile w = group_tile(table, p, t, T);
      const float alpha = p.alpha ? p.alpha[w.group] : 1.0f;
      const int64_t n0 = static_cast<int64_t>(w.nt) * BW, n = n0 + q * 32 + lane;
      ok = mbar_wait(acc_full + 8 * b, ph, abort_flag, 32);
      for (int c1 = 0; c1 < T / 2; c1 += pass) {
        const int m = w.m0 + c0 + c1, count = w.m_end - m;    // (may be none or negative)
        uint8_t* rows = rows0 + buf * kRowBufBytes;
        buf ^= 1;
        if (p.row_copies) bulk_wait_read<1>();            // the copies before the last have read this buffer
        ok = !team_any(1 + team, !ok);                    // one answer for the whole team: it leaves together or not at all
        if (!ok) break;
        tc_fence_after();
        const uint32_t acc = tmem + b * T + c0 + c1 + (static_cast<uint32_t>(q * 32) << 16);
        for (int c = 0; c < pass; c += 16) {
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
        if (c1 + pass == T / 2 && thread == 0) mbar_arrive(acc_empty + 8 * b);
        if (p.row_copies) {
          // every thread closes a group a pass, so that its count of groups is that of the buffers
          if (count >= pass) {
            if (thread == 0) tma_store_2d(&tmY, static_cast<int>(n0), m, smem_u32(rows));
          } else if (thread < count) {
            bulk_store(static_cast<uint8_t*>(p.y) + ((static_cast<int64_t>(m) + thread) * p.ld_y + n0) * size, smem_u32(rows) + thread * BW * size,
                       static_cast<uint32_t>(min(static_cast<int64_t>(BW), p.N - n0)) * size);
          }
          bulk_commit();
        }
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
  CUtensorMap tmA, tmB, tmY;
  if (!make_code_map(&tmA, a.A_codes, a.M, a.K, T) || !make_code_map(&tmB, a.B_codes, a.N * a.num_groups, a.K, BW)) return HIF4_ERR_CUDA;
  const int64_t size = a.dt == HIF4_FP32 ? 4 : 2;
  const int pass = static_cast<int>(T / 2 < kRowBufBytes / (BW * size) ? T / 2 : kRowBufBytes / (BW * size));
  // (a TMA store clips the innermost dimension in 16-byte pieces, so a row's length has to be whole ones)
  p.row_copies = ((reinterpret_cast<uintptr_t>(a.Y) | static_cast<uintptr_t>(a.ld_y * size) | static_cast<uintptr_t>(a.N * size)) & 15u) == 0 &&
                 make_y_map(&tmY, a, BW, pass, CU_TENSOR_MAP_SWIZZLE_NONE);
  if (!p.row_copies) tmY = tmA;                           // not used
  const int64_t most = (ceil_div64(a.M, T) + a.num_groups) * p.n_tiles;
  if (most > 0x7FFFFFFFll - 1024) return HIF4_ERR_SHAPE;
  return launch_overlapped(kernel, static_cast<unsigned>(most < sm_count() ? most : sm_count()), kThreads, Shape<T>::kSmem, st, tmA, tmB, tmY, p);
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
