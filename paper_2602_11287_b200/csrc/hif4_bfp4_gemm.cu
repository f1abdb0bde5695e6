// hif4_bfp4_gemm, hif4_bfp4_grouped_gemm -- Y = alpha A B^T for operands in MXFP4 or NVFP4, on the tensor core's block-scaled
// instructions: codes go from HBM through shared memory into the MMA as they are, nothing is decoded.
//
// A CTA computes 128 rows of B (the MMA's M side: TMEM lanes) times T tokens (rows of A: accumulator columns), so that few
// tokens cost few columns.  Per K = 256 a stage holds 128-byte code rows of both operands (TMA, SWIZZLE_128B) and their
// scales (one 16-byte word per row, the words of consecutive rows consecutive: a single bulk copy).  The MMA wants
// a scale word of row r in TMEM lane r % 32 (the same in all four lane quarters) and column r / 32, for each K = 64; four
// warps read the rows' words, which are just the four K = 64 steps of a row, and store them to their lane quarter.
// Few tiles: the K chunks of a tile are dealt to the CTAs of a cluster, whose FP32 sums are added through distributed
// shared memory in rank order (no atomics, no workspace).
//
// One token, 14336 x 4096 NVFP4: 8.3 us in a graph, 9.3 us over weights that come from HBM (33 MB: 5.1 us); 4096 x 4096 5.8 us.  What is
// left is start-up (barriers, tensor memory, tensor maps: 2 us), the cluster's two barriers and the launch.
#include "hif4_bfp4_gemm.cuh"

namespace hif4 {
namespace {

constexpr int kThreads = 256;               // warps: producer, MMA, tile lookup and TMEM, idle, 4 x scales and epilogue
constexpr int BW = 128;                     // rows of B a tile

template <int T> struct Shape {
  // CTAs an SM: four of two stages for few tokens (a tile's chunks are dealt to many CTAs, all of whose loads start at once),
  // two for more
  static constexpr int kCtas = T <= 32 ? 4 : 2;
  static constexpr int kStages = T <= 32 ? 2 : T == 128 ? 3 : 4;
  static constexpr int kTmemCols = 512 / kCtas;
  static constexpr int kCodeBytes = (BW + T) * kRowBytes;
  static constexpr int kSfRows = T < 32 ? 32 : T;
  static constexpr int kSfBytes = (BW + kSfRows) * 16;
  static constexpr int kBars = kStages * (kCodeBytes + kSfBytes);
  static constexpr int kSmem = 1024 + kBars + 256;
  static constexpr int kAccCols = T < 32 ? 32 : T;
  static_assert(kAccCols + kStages * 32 <= kTmemCols, "TMEM");
  static_assert(T * BW * 4 <= kStages * kCodeBytes, "sums of a cluster");
};

__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

template <int T, bool kNv>
__global__ void __launch_bounds__(kThreads, Shape<T>::kCtas)
bfp4_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const Bfp4Params p) {
  using S = Shape<T>;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t codes = smem, sf = codes + kStages * S::kCodeBytes, bars = smem + S::kBars;
  const uint32_t full = bars, ready = bars + 8 * kStages, empty = bars + 16 * kStages, done = bars + 24 * kStages;
  uint8_t* gen = smem_raw + (smem - smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + S::kBars + 24 * kStages + 8);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  volatile int* where = reinterpret_cast<volatile int*>(const_cast<uint32_t*>(tmem_slot) + 2);       // m0, m_end, group
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t rank = 0u, ranks = 1u;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const int tile = static_cast<int>(blockIdx.x / ranks);
  const int mt = tile / p.n_tiles, nt = tile - mt * p.n_tiles;
  const int64_t n0 = static_cast<int64_t>(nt) * BW;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(ready + 8 * s, 4);
      mbar_init(empty + 8 * s, 1);
    }
    mbar_init(done, 1);
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(bars + 24 * kStages + 8), "r"(S::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_wait();
  grid_launch_next();
  if (warp == 3) {
    // the tile's rows: dense ones follow from the index, grouped ones from the offsets (tiles of a group, added up)
    int64_t m0 = static_cast<int64_t>(mt) * T, m_end = p.M;
    int group = 0;
    if (p.num_groups) {
      group = -1;
      int64_t before = 0;
      for (int g0 = 0; g0 < p.num_groups && group < 0; g0 += 32) {
        const int g = g0 + lane;
        int64_t lo = 0, hi = 0;
        if (g < p.num_groups) {
          lo = max(static_cast<int64_t>(0), min(p.M, p.offsets[g]));
          hi = max(lo, min(p.M, p.offsets[g + 1]));
        }
        const int64_t tiles = (hi - lo + T - 1) / T;
        int64_t incl = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int64_t v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
          if (lane >= o) incl += v;
        }
        const bool hit = mt >= before + incl - tiles && mt < before + incl;
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, hit);
        if (who) {
          const int l = __ffs(who) - 1;
          m0 = __shfl_sync(0xFFFFFFFFu, lo + (mt - before - incl + tiles) * T, l);
          m_end = __shfl_sync(0xFFFFFFFFu, hi, l);
          group = g0 + l;
        }
        before += __shfl_sync(0xFFFFFFFFu, incl, 31);
      }
    }
    if (lane == 0) {
      where[0] = static_cast<int>(m0);
      where[1] = static_cast<int>(m_end);
      where[2] = group;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int m0 = where[0], m_end = where[1], group = where[2];
  // this CTA's share of the chunks (none for a tile that no group has)
  const int k_first = group < 0 ? 0 : static_cast<int>(static_cast<int64_t>(p.chunks) * rank / ranks);
  const int k_last = group < 0 ? 0 : static_cast<int>(static_cast<int64_t>(p.chunks) * (rank + 1) / ranks);
  const uint32_t sf_cols = tmem + S::kAccCols;

  if (warp == 0) {
    if (lane == 0) {
      const int b_row = static_cast<int>(group * p.N + n0);
      const uint32_t rows_b = static_cast<uint32_t>(min(static_cast<int64_t>(BW), p.N - n0)) * 16u;
      const uint32_t rows_a = static_cast<uint32_t>(min(static_cast<int64_t>(T), p.M - m0)) * 16u;
      const uint8_t* b_sf = p.b_scales + group * p.b_scale_group + n0 * 16;
      const uint8_t* a_sf = p.a_scales + static_cast<int64_t>(m0) * 16;
      for (int k = k_first, i = 0; k < k_last; ++k, ++i) {
        const int s = i % kStages;
        if (!mbar_wait(empty + 8 * s, ((i / kStages) & 1) ^ 1, abort_flag)) break;
        const uint32_t bar = full + 8 * s, at = codes + s * S::kCodeBytes, sfs = sf + s * S::kSfBytes;
        mbar_expect_tx(bar, S::kCodeBytes + rows_a + rows_b);
        tma_load_2d(at, &tmB, k * kRowBytes, b_row, bar);
        tma_load_2d(at + BW * kRowBytes, &tmA, k * kRowBytes, m0, bar);
        const int64_t word = kNv ? k : k >> 1;
        bulk_load(sfs, b_sf + word * p.N * 16, rows_b, bar);
        bulk_load(sfs + BW * 16, a_sf + word * p.M * 16, rows_a, bar);
      }
    }
  } else if (warp == 1) {
    constexpr uint32_t kDesc = instr_desc<kNv, BW, T>();
    const uint64_t bd0 = make_desc(codes), ad0 = make_desc(codes + BW * kRowBytes);
    const bool issuer = elect_one();
    bool ok = true;
    int s = 0;
    uint32_t ph = 0u;
    for (int k = k_first; k < k_last; ++k) {
      if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(full + 8 * s, ph, abort_flag) && mbar_wait(ready + 8 * s, ph, abort_flag)))) break;
      tc_fence_after();
      const uint64_t off = static_cast<uint64_t>(s * (S::kCodeBytes >> 4));
      const uint32_t sfb = sf_cols + s * 32;
      if (issuer) {
        mma_stage<kNv, 1, 4, 4>(tmem, bd0 + off, ad0 + off, kDesc, sfb, sfb + 16, k == p.chunks - 1 ? p.last_steps : 4, k == k_first);
        tc_commit(empty + 8 * s);
      }
      __syncwarp();
      if (++s == kStages) { s = 0; ph ^= 1u; }
    }
    if (ok && issuer && k_last > k_first) tc_commit(done);
    __syncwarp();
  } else if (warp >= 4) {
    const int q = warp & 3;
    bool ok = true;
    for (int k = k_first, i = 0; k < k_last; ++k, ++i) {
      const int s = i % kStages;
      if (!(ok = mbar_wait(full + 8 * s, (i / kStages) & 1, abort_flag))) break;
      tc_fence_after();
      const uint32_t src = sf + s * S::kSfBytes, dst = sf_cols + s * 32 + (static_cast<uint32_t>(q * 32) << 16);
      uint32_t wb[16], wa[16];
      read_scales<kNv, 4>(src, lane, k & 1, wb);
      read_scales_128<kNv, S::kSfRows / 32>(src + BW * 16, lane, k & 1, wa);
      tmem_st16(dst, wb);
      tmem_st16(dst + 16, wa);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(ready + 8 * s);
    }
    if (ok && k_last > k_first) ok = mbar_wait(done, 0, abort_flag);
    if (ok && k_last > k_first) {
      tc_fence_after();
      const uint32_t acc = tmem + (static_cast<uint32_t>(q * 32) << 16);
      const float alpha = p.alpha ? p.alpha[p.num_groups ? group : 0] : 1.0f;
      const int64_t n = n0 + q * 32 + lane;
      for (int c = 0; c < T; c += 16) {
        uint32_t r[16];
        tc_ld16(acc + c, r);
        tc_wait_ld();
        if (ranks == 1) {
          if (n < p.N) store_tokens(p, m0 + c, m_end - m0 - c, n, alpha, r);
        } else {
          float* sums = reinterpret_cast<float*>(gen) + q * 32 + lane;
#pragma unroll
          for (int j = 0; j < 16; ++j) sums[(c + j) * BW] = __uint_as_float(r[j]);
        }
      }
    }
    tc_fence_before();
  }
  __syncwarp();
  if (ranks > 1) {
    cluster_sync_all();
    if (group >= 0) {
      const float alpha = p.alpha ? p.alpha[p.num_groups ? group : 0] : 1.0f;
      // four columns of Y a thread: all CTAs' sums are on their way before the first is added
      const int c0 = static_cast<int>(T * rank / ranks), c1 = static_cast<int>(T * (rank + 1) / ranks), at = (threadIdx.x & 31) * 4;
      const int64_t n = n0 + at;
      for (int c = c0 + warp; c < c1 && m0 + c < m_end; c += kThreads / 32) {
        float4 part[8];
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r)
          if (r < ranks) part[r] = ld_cluster_f32x4(mapa(smem + (c * BW + at) * 4, r));
        float4 v = part[0];
#pragma unroll
        for (uint32_t r = 1; r < 8; ++r)
          if (r < ranks) { v.x += part[r].x; v.y += part[r].y; v.z += part[r].z; v.w += part[r].w; }
        const float out[4] = {alpha * v.x, alpha * v.y, alpha * v.z, alpha * v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < p.N) store_y(p, m0 + c, n + i, out[i]);
      }
    }
    cluster_sync_all();
  }
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
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols) : "memory");
  }
}

// ------------------------------------------------------------------------------------ host side
template <int T, bool kNv>
hif4_status launch_tiles(const hif4_bfp4_gemm_args& a, Bfp4Params p, int64_t m_tiles, cudaStream_t st) {
  const auto kernel = bfp4_gemm_kernel<T, kNv>;
  static uint64_t ready = 0;
  if (!ensure_dynamic_smem(kernel, Shape<T>::kSmem, ready)) return HIF4_ERR_CUDA;
  CUtensorMap tmA, tmB;
  const int64_t b_rows = a.N * (a.num_groups > 0 ? a.num_groups : 1);
  if (!make_code_map(&tmA, a.A_codes, a.M, a.K, T) || !make_code_map(&tmB, a.B_codes, b_rows, a.K, BW)) return HIF4_ERR_CUDA;
  const int64_t tiles = m_tiles * p.n_tiles;
  if (tiles > 0x7FFFFFFFll / 8) return HIF4_ERR_SHAPE;
  // a cluster splits K while CTAs are missing and every one keeps two chunks
  int ranks = 1;
  while (ranks < 8 && tiles * ranks * 2 <= Shape<T>::kCtas * sm_count() && p.chunks >= 4 * ranks) ranks *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * ranks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Shape<T>::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {static_cast<unsigned>(ranks), 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, kernel, tmA, tmB, p) != cudaSuccess) {
    (void)cudaGetLastError();
    return HIF4_ERR_CUDA;
  }
  note_launch();
  return HIF4_OK;
}

hif4_status product(const hif4_bfp4_gemm_args& a, bool grouped, void* stream) {
  if (a.M < 0 || a.N < 0 || a.K < 1 || a.K % kUnitElems != 0 || a.ld_y < a.N || (grouped && a.num_groups < 0)) return HIF4_ERR_SHAPE;
  if ((a.fmt != HIF4_FMT_MXFP4 && a.fmt != HIF4_FMT_NVFP4) || (a.dt != HIF4_BF16 && a.dt != HIF4_FP16 && a.dt != HIF4_FP32)) return HIF4_ERR_DTYPE;
  if (a.M == 0 || a.N == 0 || (grouped && a.num_groups == 0)) return HIF4_OK;
  constexpr int64_t kMost = (1ll << 31) - 512;                 // rows and bytes of a row are 32-bit TMA coordinates
  if (a.M >= kMost || a.K >= kMost || a.N >= kMost / (grouped ? a.num_groups : 1)) return HIF4_ERR_SHAPE;
  if (!a.Y || !a.A_codes || !a.A_scales || !a.B_codes || !a.B_scales || (grouped && !a.group_offsets)) return HIF4_ERR_NULL;
  const int64_t size = a.dt == HIF4_FP32 ? 4 : 2;
  const auto off = [](const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; };
  if (off(a.A_codes, 16) || off(a.A_scales, 16) || off(a.B_codes, 16) || off(a.B_scales, 16) || off(a.alpha, 4) ||
      off(a.Y, static_cast<uintptr_t>(size)) || off(a.group_offsets, 8))
    return HIF4_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool nv = a.fmt == HIF4_FMT_NVFP4;
  Bfp4Params p{};
  p.M = a.M; p.N = a.N;
  p.chunks = static_cast<int>(ceil_div64(a.K, kChunk));
  p.last_steps = static_cast<int>(a.K / 64 - 4 * (static_cast<int64_t>(p.chunks) - 1));
  p.n_tiles = static_cast<int>(ceil_div64(a.N, BW));
  p.a_scales = static_cast<const uint8_t*>(a.A_scales);
  p.b_scales = static_cast<const uint8_t*>(a.B_scales);
  p.b_scale_group = grouped ? scale_words(a.K, nv) * a.N * 16 : 0;
  p.alpha = a.alpha;
  p.y = a.Y; p.ld_y = a.ld_y; p.dt = a.dt;
  p.num_groups = grouped ? a.num_groups : 0;
  p.offsets = a.group_offsets;
  hif4_bfp4_gemm_args b = a;
  b.num_groups = grouped ? a.num_groups : 0;
  p.error_word = device_error_word();
  if (!p.error_word) return HIF4_ERR_CUDA;
  // More than 64 tokens: 256 x 256 tiles on CTA pairs, unless few tiles have many chunks, which a cluster shares out here and one pair
  // has to walk alone, or so few that its longer start is not made up.  Pairs / clusters, us: 512 x 4096 x 4096 10.9 / 12.4,
  // 128 x 14336 x 4096 11.4 / 12.5, 256 x 4096 x 14336 22.1 / 16.4, 512 x 4096 x 14336 22.8 / 22.9, 2048 x 512 x 512 6.5 / 5.4;
  // 64 x 4096 x 4096 9.9 / 8.4.  The rule for K <= 512 looks at none but small Ys, where it is right (BF16 Y: 2048 x 512 x 512 6.5 / 5.2,
  // 512 x 4096 x 512 6.5 / 5.2); of larger ones it takes the slower side (512 x 14336 x 512 8.3 / 12.0, 8192 x 4096 x 256 15.9 / 37.5,
  // 4096 x 14336 x 512 28 / 69, 4096 x 32768 x 512 56 / 148).
  if (!grouped && a.M > 64 && p.chunks > 2 && (p.chunks <= 16 || ceil_div64(a.M, 256) * ceil_div64(a.N, 256) * 4 >= sm_count()))
    return launch_bfp4_pairs(b, p, st);
  // Groups (this kernel takes any number of them): pairs where a mean group fills more than half of their 256 rows.  Pairs / one CTA, us,
  // 32 groups of 2048 -> 7168: 4096 rows 69.5 / 66.0, 6144 79.8 / 83.6, 8192 92 / 108, 16384 153 / 183.
  if (grouped && a.num_groups <= kMaxTableGroups)
    return ceil_div64(a.M, a.num_groups) > 128 ? launch_bfp4_pairs(b, p, st) : launch_bfp4_grouped(b, p, st);
  // tokens of a tile: the fewest that hold the rows of a (mean) group, at most 128
  const int64_t mean = grouped ? ceil_div64(a.M, a.num_groups) : a.M;
  const int T = mean <= 16 ? 16 : mean <= 32 ? 32 : mean <= 64 ? 64 : 128;
  const int64_t m_tiles = ceil_div64(a.M, T) + (grouped ? a.num_groups : 0);
  switch (T) {
    case 16: return nv ? launch_tiles<16, true>(b, p, m_tiles, st) : launch_tiles<16, false>(b, p, m_tiles, st);
    case 32: return nv ? launch_tiles<32, true>(b, p, m_tiles, st) : launch_tiles<32, false>(b, p, m_tiles, st);
    case 64: return nv ? launch_tiles<64, true>(b, p, m_tiles, st) : launch_tiles<64, false>(b, p, m_tiles, st);
    default: return nv ? launch_tiles<128, true>(b, p, m_tiles, st) : launch_tiles<128, false>(b, p, m_tiles, st);
  }
}

}  // namespace
}  // namespace hif4

extern "C" hif4_status hif4_bfp4_gemm(const hif4_bfp4_gemm_args* args, void* stream) {
  return args ? hif4::product(*args, false, stream) : HIF4_ERR_NULL;
}
extern "C" hif4_status hif4_bfp4_grouped_gemm(const hif4_bfp4_gemm_args* args, void* stream) {
  return args ? hif4::product(*args, true, stream) : HIF4_ERR_NULL;
}
