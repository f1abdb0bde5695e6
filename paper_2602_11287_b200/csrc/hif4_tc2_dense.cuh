// What the dense CTA-pair kernels share: tile and stage sizes, the schedule that deals tiles and K ranges out to the
// pairs, the wait on a neighbour's part of a tile, and the decode step of a thread.
//
// A kernel's parameters carry the schedule in fields of these names: num_kc (K = 256 chunks), n_tiles, full_rounds,
// tail_tiles, slices, sk_tiles, sk_tile0.
#pragma once
#include "hif4_tc2_common.cuh"

namespace hif4 {
namespace {

constexpr int kPairM = 256, kPairN = 256;             // output tile of a CTA pair
constexpr int kRows = 128;                            // A rows and B rows per CTA
constexpr int kRawHalfBytes = kRows * kRawRowBytes;   // 18432
constexpr int kRawStageBytes = 2 * kRawHalfBytes;     // A rows then B rows
constexpr int kDecHalfBytes = kRows * 128;            // 128 rows x 64 BF16
constexpr int kDecStageBytes = 2 * kDecHalfBytes;
constexpr int kRawStages = 2;
constexpr int kDecStages = 4;                         // one per unit of a raw chunk
constexpr int kTmemCols = 512;                        // two 256-column accumulators

constexpr int kDecodeWarp0 = 6;
constexpr int kDecodeThreads = 4 * kRows;             // 512: (A rows + B rows) x 2 unit pairs
constexpr int kThreads = kDecodeWarp0 * 32 + kDecodeThreads;   // 704

constexpr int kMaxSlices = 4;

struct WorkItem {
  int m0, n0;           // tile origin
  int kc0, kc1;         // K = 256 chunks [kc0, kc1)
  int tail;             // index among the tail tiles, -1 for a whole tile
  int slice;            // K slice of a tail tile
};
// First and last chunk (exclusive) of a pair's run in the balanced rounds, in chunks of the sk_tiles tiles laid end to
// end.  The runs go to the pairs in descending order (`run` = num_pairs - 1 - pair), so that the pair that waits
// for its neighbour's part of a shared tile has the higher index: CTAs are handed out in index order, and a
// grid that is only partly resident still cannot wait for a CTA that has not started.
template <typename Params>
__device__ __forceinline__ int balanced_run(const Params& p, int pair, int num_pairs, int64_t& c0, int64_t& c1) {
  const int64_t total = static_cast<int64_t>(p.sk_tiles) * p.num_kc;
  const int run = num_pairs - 1 - pair;
  c0 = total * run / num_pairs;
  c1 = total * (run + 1) / num_pairs;
  return run;
}
template <typename Params>
__device__ __forceinline__ int num_work_items(const Params& p, int pair, int num_pairs) {
  if (p.sk_tiles > 0) {
    int64_t c0, c1;
    balanced_run(p, pair, num_pairs, c0, c1);
    return p.full_rounds + static_cast<int>((c1 - 1) / p.num_kc - c0 / p.num_kc) + 1;
  }
  return p.full_rounds + (pair < p.tail_tiles * p.slices ? 1 : 0);
}
template <int kTileN, typename Params>
__device__ __forceinline__ WorkItem work_item(const Params& p, int pair, int num_pairs, int i) {
  WorkItem w;
  int t;
  if (i < p.full_rounds) {
    t = i * num_pairs + pair;
    w.kc0 = 0; w.kc1 = p.num_kc; w.tail = -1; w.slice = 0;
  } else if (p.sk_tiles > 0) {
    int64_t c0, c1;
    const int run = balanced_run(p, pair, num_pairs, c0, c1);
    const int64_t tr = c0 / p.num_kc + (i - p.full_rounds);
    const int64_t first = tr * p.num_kc;
    w.kc0 = c0 > first ? static_cast<int>(c0 - first) : 0;
    w.kc1 = c1 < first + p.num_kc ? static_cast<int>(c1 - first) : p.num_kc;
    t = p.sk_tile0 + static_cast<int>(tr);
    if (w.kc0 > 0) { w.tail = run; w.slice = 0; }                        // end of a tile: computed first, stored
    else if (w.kc1 < p.num_kc) { w.tail = run + 1; w.slice = 1; }        // beginning of a tile: computed last, added
    else { w.tail = -1; w.slice = 0; }
  } else {
    w.tail = pair % p.tail_tiles;
    w.slice = pair / p.tail_tiles;
    t = p.full_rounds * num_pairs + w.tail;
    w.kc0 = static_cast<int>(static_cast<int64_t>(w.slice) * p.num_kc / p.slices);
    w.kc1 = static_cast<int>(static_cast<int64_t>(w.slice + 1) * p.num_kc / p.slices);
  }
  const int mt = t / p.n_tiles;
  w.m0 = mt * kPairM;
  w.n0 = (t - mt * p.n_tiles) * kTileN;
  return w;
}

// Bounded wait until a word in global memory, written by another CTA after a __threadfence(), has reached
// `want`.  Returns false when the budget ran out or another thread has already given up.
__device__ __noinline__ bool wait_count(const unsigned int* counter, unsigned int want, volatile uint32_t* abort_flag) {
  const uint64_t t0 = global_ns();
  for (uint32_t it = 1;; ++it) {
    unsigned int v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
    if (v >= want) return true;
    __nanosleep(128);
    if ((it & 63u) == 0u) {
      if (*abort_flag) return false;
      if (global_ns() - t0 > kWaitBudgetNs) {
        *abort_flag = 1u;
        return false;
      }
    }
  }
}

// Decodes the two units held in raw words W[0..8] and W[9..17] into decoded stages 2h and 2h+1 (not `live`: the
// rows are past the matrix, only the barriers are served).  Returns false when a wait gave up.
__device__ __forceinline__ bool decode_two_units(const uint32_t (&W)[18], const uint32_t (&chunk_addr)[8], uint32_t lut,
                                                 const DecodeMul& mul, uint32_t dec_empty0, uint32_t dec_full0_leader,
                                                 uint32_t parity_free, volatile uint32_t* abort_flag, bool live = true) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    // warp-uniform outcome, so that the warp barrier below is never reached by a part of the warp
    if (!__all_sync(0xFFFFFFFFu, mbar_wait(dec_empty0 + 8 * u, parity_free, abort_flag))) return false;
    if (live) decode_unit_balanced(W[9 * u], &W[9 * u + 1], chunk_addr, u * kDecStageBytes, lut, mul);
    fence_proxy_async_smem();                  // generic-proxy writes -> visible to the tensor core
    // One remote arrive per warp; the warp barrier orders the other lanes' writes and proxy fences
    // before it.
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive_cluster(dec_full0_leader + 8 * u);
  }
  return true;
}

// Tile schedule of a dense pair kernel for this shape on this device (see the fields of the kernels' parameters).
struct Tc2Plan {
  int pairs, full_rounds, tail_tiles, slices, sk_tiles, sk_tile0;
  size_t flag_bytes, bytes;          // workspace: the slices' completion words
};
inline Tc2Plan tc2_plan(int64_t M, int64_t N, int64_t K, int tile_n = kPairN) {
  Tc2Plan pl{};
  const int64_t tiles = ceil_div64(M, kPairM) * ceil_div64(N, tile_n);
  const int64_t max_pairs = sm_count() / 2;
  pl.pairs = static_cast<int>(tiles < max_pairs ? tiles : max_pairs);
  pl.slices = 1;
  if (pl.pairs <= 0 || tiles > 0x7FFFFFFFll) return pl;
  pl.full_rounds = static_cast<int>(tiles / pl.pairs);
  pl.tail_tiles = static_cast<int>(tiles % pl.pairs);
  if (tiles < max_pairs) {            // a single, partial round: all its tiles are "tail" tiles
    pl.full_rounds = 0;
    pl.tail_tiles = static_cast<int>(tiles);
  }
  if (pl.tail_tiles > 0) {
    // Slice s starts its epilogue when slice s - 1 has finished its own, which adds about the time of
    // 3.5 K = 256 chunks per extra slice (measured): take the slice count with the shortest critical path.
    int64_t s_max = max_pairs / pl.tail_tiles;
    if (s_max > kMaxSlices) s_max = kMaxSlices;
    const int64_t chunks = ceil_div64(K, 256);
    int64_t best = 1, best_cost = 2 * chunks;
    for (int64_t s = 2; s <= s_max; ++s) {
      const int64_t cost = 2 * ceil_div64(chunks, s) + 7 * (s - 1);       // in half chunks
      if (cost < best_cost) { best = s; best_cost = cost; }
    }
    pl.slices = static_cast<int>(best);
  }
  if (pl.full_rounds >= 1 && pl.tail_tiles > 0) {
    // Several rounds and a partial one: the last whole round and the partial one are balanced chunk by chunk
    // instead (every pair then works tail_tiles / pairs of a tile longer than the whole rounds take, which is never
    // more than the K slices of the partial round alone would cost).
    pl.full_rounds -= 1;
    pl.sk_tile0 = pl.full_rounds * pl.pairs;
    pl.sk_tiles = pl.pairs + pl.tail_tiles;
    pl.tail_tiles = 0;
    pl.slices = 2;
    pl.flag_bytes = (static_cast<size_t>(pl.pairs + 1) * 2 * 8 * sizeof(unsigned int) + 255) / 256 * 256;
    pl.bytes = pl.flag_bytes;
  } else if (pl.slices > 1) {
    pl.flag_bytes = (static_cast<size_t>(pl.tail_tiles) * pl.slices * 8 * sizeof(unsigned int) + 255) / 256 * 256;
    pl.bytes = pl.flag_bytes;
  }
  return pl;
}

}  // namespace
}  // namespace hif4
