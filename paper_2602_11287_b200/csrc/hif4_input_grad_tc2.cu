// Gradient of a linear layer's activations on CTA pairs: dX[M, K] = sum over phases of dZ[M, N] W[N, K], BF16 times
// decoded HiF4 units, FP32 accumulators in tensor memory, 256 x 256 tile per pair of SMs.
//
// The weights are the units of the forward pass (cut along K), contracted along N: a unit is 64 neighbouring columns
// of the product for one step of the contraction.  Decoded, it is one 128-byte row of an MN-major SWIZZLE_128B operand
// (64 columns x 8 contraction steps per swizzle atom), so the decoder of the forward kernels writes it unchanged; the order
// in which it leaves the eight elements of a level-2 group (0 4 1 5 2 6 3 7) is undone by the epilogue, whose registers
// hold whole groups.  dZ arrives as BF16 through TMA, already in operand form: per K = 64 step a CTA decodes 128 units
// where the forward kernel decodes 256, and the tensor pipe is the tighter bound.
//   warp 0      raw units: 64 rows x 80 bytes (the CTA's two units of a 144-byte chunk, and eight bytes beside) per step,
//               eight stages ahead, by TMA or word by word as in the forward kernel
//   warp 22     dZ: 128 rows x 64 columns per step into the operand stage that the MMA has released
//   warps 6-21  decode, four teams of four warps on steps in turn: thread = one unit; a warp reports a step once its units
//               are written and the step's dZ has landed.  (A unit is 200 dependent instructions of one warp: two teams
//               took as long over a step as the tensor core.)
//   warp 1      rank 0: MMA issue;   warps 2-5  epilogue, TMA stores of 64-byte rows (the last tile with the decode warps)
// Phases: the BF16 parts of dZ (one for BF16 gradients, two for FP16), for both projections of a gated layer.
// Tiles shared along the contraction pass FP32 partial sums as in the forward kernel.
// What bounds it: a K = 64 step takes 816 clocks as the issuing thread sees them (590 in the forward kernel, 512 by its operations;
// waits for operands are 105 on top).  The MN-major operand is read, dZ and the decoded units are written through the same
// shared-memory port in that time; which of them costs the difference has not been measured apart.  2048 x 4096 x 4096 72 to 77 us
// on different machines (0.89 to 0.95 PFLOP/s), 4096 x 4096 x 14336 421 to 428 us (1.13), 64 x 4096 x 4096 29 to 33 us.
#include "hif4_linear_tc2_launch.cuh"

namespace hif4 {
namespace {

constexpr int kStepRows = 64;                          // contraction per step
constexpr int kSteps = 4;                              // steps per scheduled chunk (256)
constexpr int kWinBytes = 80;                          // raw window of a row
constexpr int kRawStepBytes = kStepRows * kWinBytes;   // 5120
constexpr int kRawRing = 8;
constexpr int kOpHalfBytes = kRows * 128;              // dZ: 128 rows x 64 BF16; W: 2 x 64 columns x 64 steps
constexpr int kOpStageBytes = 2 * kOpHalfBytes;
constexpr int kOpRing = 5;
constexpr int kTeamThreads = 128;
constexpr int kTeams = 4;
constexpr int kGradDecodeWarp0 = 6, kGradZWarp = kGradDecodeWarp0 + kTeams * kTeamThreads / 32;
constexpr int kGradThreads = (kGradZWarp + 1) * 32;
constexpr int kGradSmemBytes = 1024 + kOpRing * kOpStageBytes + kRawRing * kRawStepBytes + kStageOutBytes + 512 /*barriers*/ + 1024 /*table*/;
constexpr uint32_t kGradInstrDesc = kLinInstrDesc | (1u << 16);      // B is MN-major

struct InputGradParams {
  int64_t M, N, K;
  int num_kc, n_tiles, full_rounds, tail_tiles, slices, sk_tiles, sk_tile0;      // schedule; a chunk is 256 rows of one phase
  int chunks_per_phase, parts;      // phase / parts chooses the weights
  unsigned int* flags;
  float* partial;
  unsigned int* error_word;
  DecodeMul mul;
  int tma;
  const uint8_t *B, *B2;
  int64_t pitch;
  int upr;
  void* dx;
  int64_t ld_dx;
  int dx_vec, tma_store;
};

// MN-major SWIZZLE_128B operand descriptor: eight contraction steps (128-byte rows) are 1024 bytes, the next 64 columns
// start kStepRows rows further on.
__device__ __forceinline__ uint64_t make_desc_mn(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>((kStepRows * 128) >> 4) << 16) |
         (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

struct StepRange {            // the steps of chunk kc that hold rows of the contraction
  int phase, n0, steps;
};
__device__ __forceinline__ StepRange chunk_steps(const InputGradParams& p, int kc) {
  StepRange r;
  r.phase = kc / p.chunks_per_phase;
  r.n0 = (kc - r.phase * p.chunks_per_phase) * (kSteps * kStepRows);
  const int64_t left = (p.N - r.n0 + kStepRows - 1) / kStepRows;
  r.steps = left < kSteps ? static_cast<int>(left) : kSteps;
  return r;
}
struct Ring {                 // position in a ring of `n` stages
  uint32_t s = 0, ph = 0;
  __device__ __forceinline__ void next(uint32_t n) { if (++s == n) { s = 0; ph ^= 1u; } }
};

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGradThreads, 1)
input_grad_tc2_kernel(const __grid_constant__ CUtensorMap tmZ, const __grid_constant__ CUtensorMap tmB,
                      const __grid_constant__ CUtensorMap tmB2, const __grid_constant__ CUtensorMap tmX, const InputGradParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t op_base = smem_base;
  const uint32_t out_base = op_base + kOpRing * kOpStageBytes;
  const uint32_t raw_base = out_base + kStageOutBytes;
  const uint32_t bar_base = raw_base + kRawRing * kRawStepBytes;
  const uint32_t raw_full = bar_base, raw_empty = raw_full + 8 * kRawRing, z_full = raw_empty + 8 * kRawRing, op_full = z_full + 8 * kOpRing,
                 op_empty = op_full + 8 * kOpRing, tmem_full = op_empty + 8 * kOpRing, tmem_empty = tmem_full + 16,
                 last_full = tmem_empty + 16, tmem_slot = last_full + 8;
  uint8_t* gen_base = smem_raw + (smem_base - smem_u32(smem_raw));
  volatile uint32_t* tmem_ptr_smem = reinterpret_cast<volatile uint32_t*>(gen_base + (tmem_slot - smem_base));
  volatile uint32_t* abort_flag = tmem_ptr_smem + 1;
  const uint32_t lut = bar_base + 512;
  if (threadIdx.x < 256)
    reinterpret_cast<uint32_t*>(gen_base + (lut - smem_base))[threadIdx.x] = spread_e8_entry(threadIdx.x);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const int n_items = num_work_items(p, pair, num_pairs);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kRawRing; ++s) {
      mbar_init(raw_full + 8 * s, p.tma ? 1 : 32);
      mbar_init(raw_empty + 8 * s, kTeamThreads);
    }
    for (int s = 0; s < kOpRing; ++s) {
      mbar_init(z_full + 8 * s, 1);
      mbar_init(op_full + 8 * s, 2 * kTeamThreads / 32);  // a team's warps in each CTA (used on rank 0)
      mbar_init(op_empty + 8 * s, 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(tmem_full + 8 * s, 1);
      mbar_init(tmem_empty + 8 * s, 8);               // 4 epilogue warps of each CTA (used on rank 0)
    }
    mbar_init(last_full, 1);
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();            // the peer's barriers are initialised before anyone arrives on them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_ptr_smem;
  grid_launch_next();
  grid_wait();                   // (as in the forward kernel)

  if (warp == 0) {
    // ---------------------------------------------------------------- raw units
    if (p.tma && lane != 0) {
    } else {
      Ring ring;
      bool ok = true;
      for (int i = 0; i < n_items && ok; ++i) {
        const WorkItem w = work_item<kPairN>(p, pair, num_pairs, i);
        const int unit0 = w.n0 / kUnitElems;                             // first of the tile's four units
        for (int kc = w.kc0; kc < w.kc1 && ok; ++kc) {
          const StepRange c = chunk_steps(p, kc);
          const bool second = c.phase >= p.parts;
          for (int step = 0; step < c.steps; ++step, ring.next(kRawRing)) {
            const uint32_t full = raw_full + 8 * ring.s, dst = raw_base + ring.s * kRawStepBytes;
            const int row0 = c.n0 + step * kStepRows;
            ok = mbar_wait(raw_empty + 8 * ring.s, ring.ph ^ 1u, abort_flag, 64);
            if (!p.tma) ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            if (p.tma) {
              mbar_expect_tx(full, kRawStepBytes);
              tma_load_2d(dst, second ? &tmB2 : &tmB, unit0 * kUnitBytes + static_cast<int>(rank) * 64, row0, full);
            } else {
              const uint8_t* base = second ? p.B2 : p.B;
              int row = lane / 20, off = lane % 20;                      // word `off` of the window of row `row`
              for (int j = lane; j < kStepRows * 20; j += 32) {
                const int word = static_cast<int>(rank) * 16 + off;
                const int unit = unit0 + (word >= 9) + (word >= 18) + (word >= 27);
                const bool in = row0 + row < p.N && unit < p.upr;
                const uint8_t* src = in ? base + static_cast<int64_t>(row0 + row) * p.pitch + static_cast<int64_t>(unit0) * kUnitBytes + 4 * word : base;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 4 * j), "l"(src), "r"(in ? 4 : 0) : "memory");
                off += 12; ++row;
                if (off >= 20) { off -= 20; ++row; }
              }
              asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full) : "memory");
            }
          }
        }
      }
      if (!p.tma) asm volatile("cp.async.wait_all;" ::: "memory");
    }
  } else if (warp == kGradZWarp) {
    // ---------------------------------------------------------------- dZ
    if (lane == 0) {
      Ring ring;
      bool ok = true;
      for (int i = 0; i < n_items && ok; ++i) {
        const WorkItem w = work_item<kPairN>(p, pair, num_pairs, i);
        for (int kc = w.kc0; kc < w.kc1 && ok; ++kc) {
          const StepRange c = chunk_steps(p, kc);
          const int row0 = static_cast<int>(c.phase * p.M) + w.m0 + static_cast<int>(rank) * kRows;      // planes of M rows
          for (int step = 0; step < c.steps; ++step, ring.next(kOpRing)) {
            if (!(ok = mbar_wait(op_empty + 8 * ring.s, ring.ph ^ 1u, abort_flag, 32))) break;
            mbar_expect_tx(z_full + 8 * ring.s, kOpHalfBytes);
            tma_load_2d(op_base + ring.s * kOpStageBytes, &tmZ, c.n0 + step * kStepRows, row0, z_full + 8 * ring.s);
          }
        }
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer (rank 0 only)
    if (rank == 0 && lane == 0) {
      Ring ring;
      uint32_t tcount = 0;
      bool ok = true;
      for (int i = 0; i < n_items && ok; ++i, ++tcount) {
        const WorkItem w = work_item<kPairN>(p, pair, num_pairs, i);
        const uint32_t acc = tcount & 1u, aph = (tcount >> 1) & 1u;
        if (!(ok = mbar_wait_cluster(tmem_empty + 8 * acc, aph ^ 1u, abort_flag))) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + acc * kPairN;
        uint32_t accumulate = 0;
        for (int kc = w.kc0; kc < w.kc1 && ok; ++kc) {
          const StepRange c = chunk_steps(p, kc);
          for (int step = 0; step < c.steps; ++step, ring.next(kOpRing)) {
            if (!(ok = mbar_wait_cluster(op_full + 8 * ring.s, ring.ph, abort_flag))) break;
            tc_fence_after();
            const uint32_t stage = op_base + ring.s * kOpStageBytes;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {            // 16 contraction steps: 32 bytes of dZ's rows, 16 rows of the weights
              tc2_mma(d_tmem, make_desc(stage) + 2 * kk, make_desc_mn(stage + kOpHalfBytes + kk * 2048), kGradInstrDesc, accumulate);
              accumulate = 1u;
            }
            tc2_commit_both(op_empty + 8 * ring.s);
          }
        }
        if (!ok) break;
        tc2_commit_both(tmem_full + 8 * acc);
        if (i == n_items - 1) tc2_commit_both(last_full);         // the same, for the helpers of the last epilogue
      }
    }
  } else {
    // ---------------------------------------------------------------- decode, then its warps join the epilogue of the last tile
    bool ok = true;
    if (warp >= kGradDecodeWarp0) {
      const int d = threadIdx.x - kGradDecodeWarp0 * 32;
      const uint32_t team = static_cast<uint32_t>(d) / kTeamThreads;
      const int t = d & (kTeamThreads - 1), row = t & (kStepRows - 1), block = t >> 6;      // contraction row, 64-column block
      // The unit's nine words within the row's five 16-byte words: 2 rank + 9 block words from its start.  Three 16-byte
      // loads (a row pitch of 80 bytes spreads eight of them over all banks; single words would meet four at a bank) from
      // the 16-byte word it starts in, or the one before, then a shift by 0 to 3 words.
      const uint32_t src0 = raw_base + static_cast<uint32_t>(row) * kWinBytes + static_cast<uint32_t>(block) * 32u;
      const bool shift1 = block != 0, shift2 = rank != 0;
      const uint32_t op_row = op_base + kOpHalfBytes + static_cast<uint32_t>(block) * (kStepRows * 128) + static_cast<uint32_t>(row) * 128u;
      uint32_t chunk_addr[8];
  #pragma unroll
      for (int j = 0; j < 8; ++j) chunk_addr[j] = op_row + ((static_cast<uint32_t>(j) ^ (static_cast<uint32_t>(row) & 7u)) << 4);
      const uint32_t op_full_leader = mapa(op_full, 0);
      Ring raw, op;
      uint32_t n = 0;
      for (int i = 0; i < n_items && ok; ++i) {
        const WorkItem w = work_item<kPairN>(p, pair, num_pairs, i);
        for (int kc = w.kc0; kc < w.kc1 && ok; ++kc) {
          const StepRange c = chunk_steps(p, kc);
          for (int step = 0; step < c.steps; ++step, ++n, raw.next(kRawRing), op.next(kOpRing)) {
            if (n % kTeams != team) continue;
            if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(raw_full + 8 * raw.s, raw.ph, abort_flag)))) break;
            uint32_t L[12], W[9];
  #pragma unroll
            for (int k = 0; k < 3; ++k) {
              const uint4 v = lds128(src0 + raw.s * kRawStepBytes + 16 * k);
              L[4 * k] = v.x; L[4 * k + 1] = v.y; L[4 * k + 2] = v.z; L[4 * k + 3] = v.w;
            }
  #pragma unroll
            for (int k = 0; k < 11; ++k) L[k] = shift1 ? L[k + 1] : L[k];
  #pragma unroll
            for (int k = 0; k < 9; ++k) W[k] = shift2 ? L[k + 2] : L[k];
            fence_proxy_async_smem();                  // these reads before the async proxy refills the stage
            mbar_arrive(raw_empty + 8 * raw.s);
            if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(op_empty + 8 * op.s, op.ph ^ 1u, abort_flag)))) break;
            decode_unit_balanced(W[0], &W[1], chunk_addr, op.s * kOpStageBytes, lut, p.mul);
            fence_proxy_async_smem();                  // generic-proxy writes -> visible to the tensor core
            if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(z_full + 8 * op.s, op.ph, abort_flag)))) break;
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(op_full_leader + 8 * op.s);
          }
        }
      }
    }

    // ---------------------------------------------------------------- epilogue (as in the forward kernel)
    const bool helper = warp >= kGradDecodeWarp0;
    const int q = warp & 3;
    const int group = helper ? 1 + (warp - kGradDecodeWarp0) / 4 : 0;
    const uint32_t tmem_empty_leader = mapa(tmem_empty, 0);
    const uint32_t stage = helper ? op_base + static_cast<uint32_t>(warp - kGradDecodeWarp0) * (2 * kSlabBytes)
                                  : out_base + static_cast<uint32_t>(q) * (2 * kSlabBytes);
    uint32_t slabs = 0;
    const int first = helper && n_items > 0 ? n_items - 1 : 0;
    uint32_t tcount = static_cast<uint32_t>(first);
    for (int it = first; it < n_items && ok; ++it, ++tcount) {
      const WorkItem w = work_item<kPairN>(p, pair, num_pairs, it);
      const uint32_t acc = tcount & 1u, aph = (tcount >> 1) & 1u;
      // A helper has not followed the phases of tmem_full, and with short items several may still be to come: the parity would
      // not tell it which one it sees.  Its own barrier completes once.
      if (!__all_sync(0xFFFFFFFFu, helper ? mbar_wait(last_full, 0u, abort_flag, 32) : mbar_wait(tmem_full + 8 * acc, aph, abort_flag, 256))) break;
      tc_fence_after();
      const bool shared_tile = w.tail >= 0 && p.slices > 1;
      const bool leaves = shared_tile && w.slice + 1 < p.slices, adds = shared_tile && !leaves;
      const int others = p.slices - 1;
      const int groups = it == n_items - 1 ? kEpiGroups : 1;
      const int64_t row0 = static_cast<int64_t>(w.m0) + rank * kRows + q * 32, row = row0 + lane;
      const int64_t cols_left = p.K - w.n0;              // K is a multiple of 64: a slab is inside or outside as a whole
      const int cols = row0 >= p.M ? 0 : cols_left < kPairN ? static_cast<int>(cols_left) : kPairN;
      unsigned int* flags = shared_tile ? p.flags + static_cast<size_t>(w.tail) * p.slices * 8 + rank * 4 + q : nullptr;
      if (adds && cols > 0 && !wait_parts(flags, others, static_cast<unsigned int>(cols / 32), abort_flag)) break;
      float4* part = shared_tile ? partial_of(p.partial, w.tail * others + (leaves ? w.slice : 0), rank, q, lane) : nullptr;
      const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * kPairN;
      unsigned int left = 0;
#pragma unroll 1
      for (int c0 = group * 32; c0 < cols; c0 += groups * 32) {
        const int64_t col0 = static_cast<int64_t>(w.n0) + c0;
        uint32_t r[2][16], words[16];
        tc_ld16(t_row + c0, r[0]);
        tc_ld16(t_row + c0 + 16, r[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float z[16];
          tc_wait_ld16(r[h]);
#pragma unroll
          for (int e = 0; e < 16; ++e) z[e] = __uint_as_float(r[h][e]);
          if (adds) add_partial16(z, part + (c0 + 16 * h) * 8, others);
          if (leaves) leave_partial16(z, part + (c0 + 16 * h) * 8);
#pragma unroll
          for (int g = 0; g < 2; ++g) {                 // group of eight columns, held in the order 0 4 1 5 2 6 3 7
            const float* v = z + 8 * g;
            uint32_t* o = words + 8 * h + 4 * g;
            o[0] = pack2(v[0], v[2], T());
            o[1] = pack2(v[4], v[6], T());
            o[2] = pack2(v[1], v[3], T());
            o[3] = pack2(v[5], v[7], T());
          }
        }
        if (leaves) {
          ++left;
          continue;
        }
        if (p.tma_store) {
          const uint32_t buf = stage + (slabs & 1u) * kSlabBytes;
          const uint32_t my = buf + static_cast<uint32_t>(lane) * 64u, sw = (static_cast<uint32_t>(lane) >> 1) & 3u;    // SWIZZLE_64B
          if (lane == 0) bulk_wait_read<1>();
          __syncwarp();
#pragma unroll
          for (int v = 0; v < 4; ++v)
            sts128(my + ((static_cast<uint32_t>(v) ^ sw) << 4), words[4 * v], words[4 * v + 1], words[4 * v + 2], words[4 * v + 3]);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            tma_store_2d(&tmX, static_cast<int>(col0), static_cast<int>(row0), buf);
            bulk_commit();
          }
          ++slabs;
        } else if (row < p.M) {
          T* dst = static_cast<T*>(p.dx) + row * p.ld_dx + col0;
          if (p.dx_vec) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
              reinterpret_cast<uint4*>(dst)[v] = make_uint4(words[4 * v], words[4 * v + 1], words[4 * v + 2], words[4 * v + 3]);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) reinterpret_cast<uint16_t*>(dst)[e] = static_cast<uint16_t>(words[e >> 1] >> (16 * (e & 1)));
          }
        }
      }
      if (leaves) {
        __syncwarp();
        if (lane == 0 && left > 0) {
          __threadfence();
          asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(flags + 8 * w.slice), "r"(left) : "memory");
        }
      }
      if (!helper) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + 8 * acc);
      }
    }
    if (lane == 0) bulk_wait_all();
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  if (*abort_flag) {
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 2000000ull) {}        // let copies and MMAs that are still in flight land
    if (threadIdx.x == 0) atomicExch(p.error_word, 1u);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

// dZ planes as one matrix of `rows` rows: boxes of 64 columns x 128 rows, SWIZZLE_128B; columns past N read as zeros.
bool make_z_map(CUtensorMap* map, const void* z, int64_t rows, int64_t N, int64_t ld) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(N), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * 2};
  const cuuint32_t box[2] = {64, kRows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(z), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Raw units: windows of 80 bytes x 64 rows.
bool make_window_map(CUtensorMap* map, const void* base, int64_t rows, int64_t upr) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(upr * kUnitBytes), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(upr * kUnitBytes)};
  const cuuint32_t box[2] = {kWinBytes, kStepRows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

Tc2Plan grad_plan(int64_t M, int64_t N, int64_t K, int phases) { return linear_plan(M, K, ceil_div64(N, 256) * 256 * phases, kPairN); }

template <typename T>
hif4_status launch_input_grad_t(const InputGradCall& c, void* workspace, cudaStream_t st) {
  static uint64_t smem_opt_in = 0;
  if (!ensure_dynamic_smem(input_grad_tc2_kernel<T>, kGradSmemBytes, smem_opt_in)) return HIF4_ERR_CUDA;
  InputGradParams p{};
  p.M = c.M; p.N = c.N; p.K = c.K;
  p.error_word = device_error_word();
  if (!p.error_word) return HIF4_ERR_CUDA;
  p.chunks_per_phase = static_cast<int>(ceil_div64(c.N, 256));
  p.parts = c.parts;
  const int phases = c.parts * (c.B2 ? 2 : 1);
  p.num_kc = p.chunks_per_phase * phases;
  p.n_tiles = static_cast<int>(ceil_div64(c.K, kPairN));
  const Tc2Plan pl = grad_plan(c.M, c.N, c.K, phases);
  p.full_rounds = pl.full_rounds; p.tail_tiles = pl.tail_tiles; p.slices = pl.slices;
  p.sk_tiles = pl.sk_tiles; p.sk_tile0 = pl.sk_tile0;
  p.mul = make_decode_mul();
  const int64_t upr = c.K / kUnitElems;
  p.B = static_cast<const uint8_t*>(c.B);
  p.B2 = static_cast<const uint8_t*>(c.B2);
  p.pitch = upr * kUnitBytes;
  p.upr = static_cast<int>(upr);
  CUtensorMap tmZ{}, tmB{}, tmB2{}, tmX{};
  if (!make_z_map(&tmZ, c.dz, c.M * phases, c.N, c.ld_dz)) return HIF4_ERR_CUDA;
  p.tma = c.K % (kRawUnits * kUnitElems) == 0 && at16(c.B) && at16(c.B2);
  if (p.tma) {
    if (!make_window_map(&tmB, c.B, c.N, upr) || (c.B2 && !make_window_map(&tmB2, c.B2, c.N, upr))) return HIF4_ERR_CUDA;
  }
  p.dx = c.dx; p.ld_dx = c.ld_dx;
  p.dx_vec = at16(c.dx) && (c.M == 1 || c.ld_dx * 2 % 16 == 0);
  p.tma_store = p.dx_vec && c.ld_dx * 2 % 16 == 0 && make_y_map<T>(&tmX, c.dx, c.M, c.K, c.ld_dx);
  if (p.slices > 1) {
    p.flags = static_cast<unsigned int*>(workspace);
    p.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + pl.flag_bytes);
  }
  const int pairs = p.full_rounds == 0 && p.sk_tiles == 0 ? p.tail_tiles * p.slices : pl.pairs;
  return launch_overlapped(input_grad_tc2_kernel<T>, 2 * pairs, kGradThreads, kGradSmemBytes, st, tmZ, tmB, tmB2, tmX, p);
}

}  // namespace

size_t input_grad_tc2_workspace(int64_t M, int64_t N, int64_t K, int phases) {
  if (M <= 0 || N <= 0 || K <= 0) return 0;
  const Tc2Plan pl = grad_plan(M, N, K, phases);
  return pl.slices > 1 ? pl.flag_bytes + partial_tiles(pl) * kPartialTileBytes : 0;
}
hif4_status input_grad_tc2_clear(int64_t M, int64_t N, int64_t K, int phases, void* workspace, cudaStream_t st) {
  const Tc2Plan pl = grad_plan(M, N, K, phases);
  return pl.slices > 1 && cudaMemsetAsync(workspace, 0, pl.flag_bytes, st) != cudaSuccess ? HIF4_ERR_CUDA : HIF4_OK;
}
bool input_grad_tc2_supported(int64_t M, int64_t N, int64_t K, int phases) {
  return M * phases < (1ll << 31) - kPairM && N < (1ll << 29) && K < (1ll << 31) - kPairN &&
         ceil_div64(M, kPairM) * ceil_div64(K, kPairN) <= 0x7FFFFFFFll;
}
hif4_status launch_input_grad_tc2(const InputGradCall& c, void* workspace, cudaStream_t st) {
  return c.dt == HIF4_BF16 ? launch_input_grad_t<__nv_bfloat16>(c, workspace, st) : launch_input_grad_t<__half>(c, workspace, st);
}

}  // namespace hif4
