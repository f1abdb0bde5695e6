// hif4_expert_plan, hif4_dispatch, hif4_combine, hif4_combine_backward -- the experts' rows of a mixture-of-experts
// layer: their order, the rows themselves, the weighted sum of what comes back, and its gradient.  All but the plan are
// bound by HBM traffic: a token's row is read (and converted) once, the experts' rows are read or written once.
//
// 4096 tokens, 8 of 256 experts, 7168 columns, BF16: rows as they are 86 us (6.1 TB/s), HiF4 units 44 us (4.3), MXFP4 33 us (5.5),
// NVFP4 37 us (5.2); FP32 rows back to tokens with a residual 155 us (6.8 TB/s).  Its gradient, 2047 x 6 x 2056 BF16: 21 us (5.2 TB/s).
// The plan of 32768 assignments: 8 us in two launches, of 64: 2.3 us in one.
#include <type_traits>

#include "hif4_bfp4_device.cuh"
#include "hif4_tc_common.cuh"

namespace hif4 {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kAll = 0xFFFFFFFFu;

// ----------------------------------------------------------------------------- order of the rows
// A stable counting sort by expert.  A warp owns a run of consecutive assignments: it counts them per expert, the counts are
// summed over warps (and blocks) in their order, and the warp then goes through its run again, 32 assignments a step, giving
// each the next row of its expert: match_any finds the lanes with the same expert, their order is the lanes'.  A block's ids are
// loaded at once; many assignments are counted by one launch and placed by a second, few take one launch.
constexpr int kPlanWarps = 16, kPlanSteps = 4;
constexpr int kPlanItems = kPlanWarps * kPlanSteps * 32;     // assignments that a block holds in registers
constexpr int kPlanBlocks = 256;                             // at most; beyond, blocks go through several times kPlanItems

__global__ void __launch_bounds__(kPlanWarps * 32)
plan_count_kernel(const int32_t* __restrict__ ids, int64_t n, int64_t per_block, int experts, int32_t* __restrict__ counts) {
  extern __shared__ int32_t hist[];
  grid_wait();
  grid_launch_next();
  for (int e = threadIdx.x; e < experts; e += blockDim.x) hist[e] = 0;
  __syncthreads();
  const int64_t first = static_cast<int64_t>(blockIdx.x) * per_block, last = min(n, first + per_block);
  for (int64_t i0 = first; i0 < last; i0 += kPlanItems) {
    int id[kPlanSteps];
#pragma unroll
    for (int j = 0; j < kPlanSteps; ++j) {
      const int64_t i = i0 + j * (kPlanWarps * 32) + threadIdx.x;
      id[j] = i < last ? ids[i] : -1;
    }
#pragma unroll
    for (int j = 0; j < kPlanSteps; ++j)
      if (id[j] >= 0 && id[j] < experts) atomicAdd(&hist[id[j]], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < experts; e += blockDim.x) counts[static_cast<int64_t>(blockIdx.x) * experts + e] = hist[e];
}

// `runs` warps own assignments (the others only help with the sums).
__global__ void __launch_bounds__(kPlanWarps * 32)
plan_place_kernel(const int32_t* __restrict__ ids, int64_t n, int64_t per_block, int runs, int experts, const int32_t* __restrict__ counts, int blocks,
                  int64_t* __restrict__ offsets, int32_t* __restrict__ row_of) {
  extern __shared__ int32_t hist[];                     // [runs][experts]
  __shared__ int32_t warp_total[kPlanWarps + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  grid_wait();
  grid_launch_next();
  const int64_t block_first = static_cast<int64_t>(blockIdx.x) * per_block, block_last = min(n, block_first + per_block);
  const int passes = static_cast<int>((per_block + kPlanItems - 1) / kPlanItems);
  const int64_t run = static_cast<int64_t>(passes) * kPlanSteps * 32;
  const int64_t first = min(block_last, block_first + warp * run), last = warp < runs ? min(block_last, first + run) : first;
  int id[kPlanSteps];
  const auto load = [&](int pass) {
#pragma unroll
    for (int j = 0; j < kPlanSteps; ++j) {
      const int64_t i = first + (static_cast<int64_t>(pass) * kPlanSteps + j) * 32 + lane;
      id[j] = i < last ? ids[i] : -1;
      if (id[j] >= experts) id[j] = -1;
    }
  };
  load(0);
  for (int e = threadIdx.x; e < experts * runs; e += blockDim.x) hist[e] = 0;
  __syncthreads();
  int32_t* mine = hist + warp * experts;
  for (int pass = 0; pass < passes; ++pass) {
    if (passes > 1) load(pass);
#pragma unroll
    for (int j = 0; j < kPlanSteps; ++j)
      if (id[j] >= 0) atomicAdd(&mine[id[j]], 1);
  }
  __syncthreads();
  int past = 0;                                         // rows of the experts before these
  for (int e0 = 0; e0 < experts; e0 += blockDim.x) {
    const int e = e0 + threadIdx.x;
    int before = 0, total = 0;                          // of expert e: before this block, in all blocks
    int of_run[kPlanWarps];                             // (registers, so that the loads do not wait for the stores below)
    if (e < experts) {
#pragma unroll
      for (int w = 0; w < kPlanWarps; ++w) of_run[w] = w < runs ? hist[w * experts + e] : 0;
      if (blocks == 1) {
#pragma unroll
        for (int w = 0; w < kPlanWarps; ++w) total += of_run[w];
      } else {
#pragma unroll 8
        for (int b = 0; b < blocks; ++b) {
          const int c = counts[static_cast<int64_t>(b) * experts + e];
          before += b < static_cast<int>(blockIdx.x) ? c : 0;
          total += c;
        }
      }
    }
    int incl = total;                                   // scan over these experts
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(kAll, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) warp_total[warp] = incl;
    __syncthreads();
    int ahead = past, all = 0;
    for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) {
      ahead += w < warp ? warp_total[w] : 0;
      all += warp_total[w];
    }
    __syncthreads();
    past += all;
    if (e < experts) {
      const int end = ahead + incl;
      int at = end - total + before;
#pragma unroll
      for (int w = 0; w < kPlanWarps; ++w) {            // the warps' first places
        if (w < runs) hist[w * experts + e] = at;
        at += of_run[w];
      }
      if (blockIdx.x == 0) {
        if (e == 0) offsets[0] = 0;
        offsets[e + 1] = end;
      }
    }
  }
  __syncthreads();
  if (warp >= runs) return;
  for (int pass = 0; pass < passes; ++pass) {
    if (passes > 1) load(pass);
#pragma unroll
    for (int j = 0; j < kPlanSteps; ++j) {
      const int64_t i = first + (static_cast<int64_t>(pass) * kPlanSteps + j) * 32 + lane;
      if (i - lane >= last) break;
      const uint32_t same = __match_any_sync(kAll, id[j]);
      const int rank = __popc(same & ((1u << lane) - 1u));
      int row = -1;
      if (id[j] >= 0) row = mine[id[j]] + rank;
      __syncwarp();
      if (id[j] >= 0 && rank == 0) mine[id[j]] += __popc(same);
      __syncwarp();
      if (i < last) row_of[i] = row;
    }
  }
}

// ----------------------------------------------------------------------------- rows of the experts
struct Gather {
  int64_t rows, cols;
  int top_k, segments;                                  // blocks of a token
  const int32_t* row_of;
};
__device__ __forceinline__ bool has_row(int row, int64_t rows) { return row >= 0 && row < rows; }

// Rows that are no multiples of 16 bytes move in words of 4 or 2 bytes, kNarrow of them a thread, so that as many bytes are under way
// (2048 tokens x 6 of 4097 BF16 elements, with one word a thread -> with four: rows 59 -> 33 us, their sum 90 -> 49, its gradient
// 74 -> 68; of 4098 35 -> 29, 55 -> 43, 74 -> 54).
constexpr int kNarrow = 4;
// Word: as many bytes as addresses, row strides and the row's length allow.
template <typename Word, int kAcross>
__global__ void __launch_bounds__(kThreads)
dispatch_plain_kernel(Gather g, const Word* __restrict__ x, int64_t ld_x, Word* __restrict__ out, int64_t ld_out, int64_t words) {
  grid_wait();
  grid_launch_next();
  const int64_t t = blockIdx.x / g.segments;
  const int seg = static_cast<int>(blockIdx.x - t * g.segments);
  const int32_t* row_of = g.row_of + t * g.top_k;
  const int64_t w0 = static_cast<int64_t>(seg) * kThreads * kAcross + threadIdx.x;
  Word v[kAcross];
#pragma unroll
  for (int i = 0; i < kAcross; ++i)
    if (w0 + i * kThreads < words) v[i] = x[t * ld_x + w0 + i * kThreads];
  for (int j = 0; j < g.top_k; ++j) {
    const int row = row_of[j];
    if (!has_row(row, g.rows)) continue;
#pragma unroll
    for (int i = 0; i < kAcross; ++i)
      if (w0 + i * kThreads < words) out[row * ld_out + w0 + i * kThreads] = v[i];
  }
}

// Eight lanes convert a unit.  A block's units are collected in shared memory and copied to every row in 16-byte words (4-byte ones
// where rows of units are not multiples of 16 bytes): stored by the lanes that made them, 4 bytes a lane, 4096 x 7168 tokens for
// eight experts each took 51 us.
constexpr int kBlockUnits = 128;
template <typename T, bool kRHA>
__global__ void __launch_bounds__(kThreads)
dispatch_hif4_kernel(Gather g, const T* __restrict__ x, int64_t ld_x, uint32_t* __restrict__ out, int block_units, int wide) {
  __shared__ __align__(16) uint32_t units[kBlockUnits * kUnitWords];
  grid_wait();
  grid_launch_next();
  const int64_t t = blockIdx.x / g.segments;
  const int seg = static_cast<int>(blockIdx.x - t * g.segments);
  const int32_t* row_of = g.row_of + t * g.top_k;
  const int part = threadIdx.x & 7;
  const int64_t upr = g.cols / kUnitElems, first = static_cast<int64_t>(seg) * block_units;
  const int count = static_cast<int>(min(static_cast<int64_t>(block_units), upr - first));
  for (int u0 = 0; u0 < count; u0 += kThreads / 8) {
    const int mine = u0 + (threadIdx.x >> 3), u = min(mine, count - 1);
    uint32_t meta;
    const uint32_t code = encode_unit_octet<kRHA>(load8(x + t * ld_x + (first + u) * kUnitElems + 8 * part), part, meta);
    if (mine < count) {
      units[mine * kUnitWords + 1 + part] = code;
      if (part == 0) units[mine * kUnitWords] = meta;
    }
  }
  __syncthreads();
  for (int j = 0; j < g.top_k; ++j) {
    const int row = row_of[j];
    if (!has_row(row, g.rows)) continue;
    uint32_t* dst = out + (row * upr + first) * kUnitWords;
    if (wide) {
      for (int i = threadIdx.x; i < count * kUnitWords / 4; i += kThreads) reinterpret_cast<uint4*>(dst)[i] = reinterpret_cast<const uint4*>(units)[i];
    } else {
      for (int i = threadIdx.x; i < count * kUnitWords; i += kThreads) dst[i] = units[i];
    }
  }
}

// A thread converts 32 elements.
template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
dispatch_bfp4_kernel(Gather g, const T* __restrict__ x, int64_t ld_x, const float* __restrict__ gain, uint4* __restrict__ codes,
                     uint8_t* __restrict__ scales) {
  grid_wait();
  grid_launch_next();
  const int64_t t = blockIdx.x / g.segments;
  const int seg = static_cast<int>(blockIdx.x - t * g.segments);
  const int32_t* row_of = g.row_of + t * g.top_k;
  const int64_t n32 = g.cols / 32, c = static_cast<int64_t>(seg) * blockDim.x + threadIdx.x;
  constexpr int kOfWord = kNv ? 8 : 16;                  // threads of a scale word
  const int64_t padded = scale_words(g.cols, kNv) * kOfWord;
  if (c >= padded) return;
  uint4 code = make_uint4(0u, 0u, 0u, 0u);
  uint32_t sa = 0u, sb = 0u;                             // (0 past the last block)
  const float f = gain ? *gain : 1.0f;
  if (c < n32) {
    const Raw16<T> ra = load_raw16(x + t * ld_x + 32 * c, false), rb = load_raw16(x + t * ld_x + 32 * c + 16, false);
    Sixteen a = sixteen_of(ra), b = sixteen_of(rb);
    uint32_t pa = peak16(ra), pb = peak16(rb);
    if (!kNv) pa = pb = max(pa, pb);
    if (gain) apply_gain<kNv>(a, b, pa, pb, f);
    const uint2 ca = encode16<kNv>(a, pa, sa), cb = encode16<kNv>(b, pb, sb);
    code = make_uint4(ca.x, ca.y, cb.x, cb.y);
  }
  const int64_t word = c / kOfWord;
  const int at = static_cast<int>(c - word * kOfWord);
#pragma unroll 4
  for (int j = 0; j < g.top_k; ++j) {
    const int row = row_of[j];
    if (!has_row(row, g.rows)) continue;
    if (c < n32) codes[row * n32 + c] = code;
    uint8_t* scale = scales + (word * g.rows + row) * 16;
    if (kNv) reinterpret_cast<uint16_t*>(scale)[at] = static_cast<uint16_t>(sa | (sb << 8));
    else scale[at] = static_cast<uint8_t>(sa);
  }
}

// ----------------------------------------------------------------------------- sums over a token's experts
// kVec elements a thread: eight, or where rows are not 16-byte aligned two of 16 bits each, or one.
template <typename T, int kVec>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[kVec]) {
  if constexpr (kVec == 8) {
    unpack8(load8(p), v);
  } else if constexpr (kVec == 2) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(p);              // 16-bit elements only
    v[0] = to_f32(reinterpret_cast<const T*>(&w)[0]);
    v[1] = to_f32(reinterpret_cast<const T*>(&w)[1]);
  } else {
    v[0] = to_f32(*p);
  }
}
template <typename T, int kVec>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[kVec]) {
  if constexpr (kVec == 8) store8(p, pack8<T>(v));
  else if constexpr (kVec == 2) *reinterpret_cast<uint32_t*>(p) = pack2(v[0], v[1], T());
  else *p = from_f32<T>(v[0]);
}

template <typename TI, typename TO, int kVec, int kAcross>
__global__ void __launch_bounds__(kThreads)
combine_kernel(Gather g, const TI* __restrict__ in, int64_t ld_in, const float* __restrict__ weights, const TO* residual, int64_t ld_r,
               float res_scale, TO* y, int64_t ld_y) {
  grid_wait();
  grid_launch_next();
  const int64_t t = blockIdx.x / g.segments;
  const int seg = static_cast<int>(blockIdx.x - t * g.segments);
  const int32_t* row_of = g.row_of + t * g.top_k;
  const int64_t c0 = (static_cast<int64_t>(seg) * kThreads * kAcross + threadIdx.x) * kVec;
  constexpr int kStep = kThreads * kVec;
  if (c0 >= g.cols) return;
  float acc[kAcross][kVec], v[kAcross][kVec];
#pragma unroll
  for (int u = 0; u < kAcross; ++u)
#pragma unroll
    for (int i = 0; i < kVec; ++i) acc[u][i] = 0.0f;
  const auto add = [&](const auto* from, float w) {
#pragma unroll
    for (int u = 0; u < kAcross; ++u)
      if (c0 + u * kStep < g.cols) load_vec(from + c0 + u * kStep, v[u]);
#pragma unroll
    for (int u = 0; u < kAcross; ++u)
      if (c0 + u * kStep < g.cols) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc[u][i] = fmaf(w, v[u][i], acc[u][i]);
      }
  };
#pragma unroll 4
  for (int j = 0; j < g.top_k; ++j) {
    const int row = row_of[j];
    const float w = weights ? weights[t * g.top_k + j] : 1.0f;
    if (has_row(row, g.rows)) add(in + row * ld_in, w);
  }
  if (residual) add(residual + t * ld_r, res_scale);
#pragma unroll
  for (int u = 0; u < kAcross; ++u)
    if (c0 + u * kStep < g.cols) store_vec(y + t * ld_y + c0 + u * kStep, acc[u]);
}

// A block goes over a token's row, eight assignments at a time, whose rows are loaded together.
constexpr int kTogether = 8;
template <typename TD, typename TI, int kVec>
__global__ void __launch_bounds__(kThreads, 3)
combine_backward_kernel(Gather g, const TD* __restrict__ dy, int64_t ld_dy, const float* __restrict__ weights, const TI* __restrict__ in,
                        int64_t ld_in, TI* __restrict__ din, int64_t ld_din, float* __restrict__ dweights) {
  __shared__ float sums[kThreads / 32][kTogether];
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  grid_wait();
  grid_launch_next();
  for (int j0 = 0; j0 < g.top_k; j0 += kTogether) {
    int row[kTogether];
    float w[kTogether], acc[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const bool there = j0 + j < g.top_k;
      row[j] = there ? g.row_of[t * g.top_k + j0 + j] : -1;
      if (!has_row(row[j], g.rows)) row[j] = -1;
      w[j] = there && weights ? weights[t * g.top_k + j0 + j] : 1.0f;
      acc[j] = 0.0f;
    }
    constexpr int kAcross = kVec == 8 ? 1 : kNarrow;
    for (int64_t c = static_cast<int64_t>(threadIdx.x) * kVec; c < g.cols; c += blockDim.x * kVec * kAcross) {
      if constexpr (kVec == 8) {
        const Raw8<TD> raw_d = load8(dy + t * ld_dy + c);
        Raw8<TI> raw[kTogether];
        if (dweights) {
#pragma unroll
          for (int j = 0; j < kTogether; ++j)
            if (row[j] >= 0) raw[j] = load8(in + row[j] * ld_in + c);
        }
        const Pairs d = pairs_of(raw_d);
        if (dweights) {
#pragma unroll
          for (int j = 0; j < kTogether; ++j) {
            if (row[j] < 0) continue;
            const Pairs v = pairs_of(raw[j]);
            float2 part = mul2(d.p[0], v.p[0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) part = fma2(d.p[i], v.p[i], part);
            acc[j] += part.x + part.y;
          }
        }
        if (din) {
#pragma unroll
          for (int j = 0; j < kTogether; ++j) {
            if (row[j] < 0) continue;
            Pairs v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v.p[i] = mul2(both(w[j]), d.p[i]);
            store8(din + row[j] * ld_din + c, raw_of<TI>(v));
          }
        }
      } else {
        TD d[kAcross];
        TI v[kTogether][kAcross];
        int64_t at[kAcross];                            // past the row: its last element, loaded and not used
#pragma unroll
        for (int u = 0; u < kAcross; ++u) at[u] = min(c + u * static_cast<int>(blockDim.x), g.cols - 1);
#pragma unroll
        for (int u = 0; u < kAcross; ++u) d[u] = dy[t * ld_dy + at[u]];
        if (dweights) {
#pragma unroll
          for (int j = 0; j < kTogether; ++j)
            if (row[j] >= 0) {
#pragma unroll
              for (int u = 0; u < kAcross; ++u) v[j][u] = in[row[j] * ld_in + at[u]];
            }
        }
#pragma unroll
        for (int j = 0; j < kTogether; ++j) {
          if (row[j] < 0) continue;
#pragma unroll
          for (int u = 0; u < kAcross; ++u) {
            if (c + u * static_cast<int>(blockDim.x) >= g.cols) continue;
            if (dweights) acc[j] = fmaf(to_f32(d[u]), to_f32(v[j][u]), acc[j]);
            if (din) din[row[j] * ld_din + at[u]] = from_f32<TI>(__fmul_rn(w[j], to_f32(d[u])));
          }
        }
      }
    }
    if (dweights) {
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc[j] += __shfl_xor_sync(kAll, acc[j], o);
        if (lane == 0) sums[warp][j] = acc[j];
      }
      __syncthreads();
      if (threadIdx.x < kTogether && j0 + static_cast<int>(threadIdx.x) < g.top_k) {
        float s = 0.0f;
        for (int i = 0; i < static_cast<int>(blockDim.x >> 5); ++i) s += sums[i][threadIdx.x];
        dweights[t * g.top_k + j0 + threadIdx.x] = s;
      }
      __syncthreads();
    }
  }
}

// A warp goes over the row of one assignment, `kAtOnce` loads of both operands at a time: no barrier, and the warps of a token read
// its gradient from L1 after the first.
constexpr int kAtOnce = 4;
template <typename TD, typename TI, int kVec>
__global__ void __launch_bounds__(kThreads)
combine_backward_rows_kernel(Gather g, int64_t assignments, const TD* __restrict__ dy, int64_t ld_dy, const float* __restrict__ weights,
                             const TI* __restrict__ in, int64_t ld_in, TI* __restrict__ din, int64_t ld_din, float* __restrict__ dweights) {
  const int lane = threadIdx.x & 31;
  const int64_t a = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  grid_wait();
  grid_launch_next();
  if (a >= assignments) return;
  const int row = g.row_of[a];
  float acc = 0.0f;
  if (has_row(row, g.rows)) {
    const float w = weights ? weights[a] : 1.0f;
    const TD* d_row = dy + (a / g.top_k) * ld_dy;
    const TI* in_row = in + row * ld_in;
    TI* out = din + row * ld_din;
    constexpr int kStep = 32 * kVec;
    for (int64_t c0 = lane * kVec; c0 < g.cols; c0 += (kVec == 8 ? kAtOnce : 2 * kAtOnce) * kStep) {
      if constexpr (kVec == 8) {
        Raw8<TD> rd[kAtOnce];
        Raw8<TI> rv[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int64_t c = c0 + u * kStep;
          if (c < g.cols) {
            rd[u] = load8(d_row + c);
            if (dweights) rv[u] = load8(in_row + c);
          }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int64_t c = c0 + u * kStep;
          if (c >= g.cols) continue;
          const Pairs d = pairs_of(rd[u]);
          if (dweights) {
            const Pairs v = pairs_of(rv[u]);
            float2 part = mul2(d.p[0], v.p[0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) part = fma2(d.p[i], v.p[i], part);
            acc += part.x + part.y;
          }
          if (din) {
            Pairs v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v.p[i] = mul2(both(w), d.p[i]);
            store8(out + c, raw_of<TI>(v));
          }
        }
      } else {
        constexpr int kMany = 2 * kAtOnce;
        const auto some = [&](auto whole) {
          constexpr bool kWhole = decltype(whole)::value;
          float d[kMany][kVec], v[kMany][kVec];
#pragma unroll
          for (int u = 0; u < kMany; ++u) {
            if (!kWhole && c0 + u * kStep >= g.cols) break;
            load_vec(d_row + c0 + u * kStep, d[u]);
            if (dweights) load_vec(in_row + c0 + u * kStep, v[u]);
          }
#pragma unroll
          for (int u = 0; u < kMany; ++u) {
            if (!kWhole && c0 + u * kStep >= g.cols) break;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
              if (dweights) acc = fmaf(d[u][i], v[u][i], acc);
              d[u][i] = __fmul_rn(w, d[u][i]);
            }
            if (din) store_vec(out + c0 + u * kStep, d[u]);
          }
        };
        if (c0 + (kMany - 1) * kStep < g.cols) some(std::true_type());
        else some(std::false_type());
      }
    }
  }
  if (dweights) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(kAll, acc, o);
    if (lane == 0) dweights[a] = acc;
  }
}

// ----------------------------------------------------------------------------- arguments
bool type_ok(int dt) { return dt == HIF4_BF16 || dt == HIF4_FP16 || dt == HIF4_FP32; }
int64_t type_size(int dt) { return dt == HIF4_FP32 ? 4 : 2; }
uintptr_t bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }
bool aligned(const void* p, int64_t to) { return bits(p) % static_cast<uintptr_t>(to) == 0; }
// Row r of a matrix starts at a multiple of 16 bytes, for every r.
bool rows_aligned(const void* p, int64_t ld, int dt) { return aligned(p, 16) && ld * type_size(dt) % 16 == 0; }
// Rows of 16-bit elements go in whole 4-byte words.
bool words_aligned(const void* p, int64_t ld, int64_t cols) { return aligned(p, 4) && (ld | cols) % 2 == 0; }

int64_t plan_per_block(int64_t n) { return kPlanItems * ceil_div64(n > 0 ? n : 1, static_cast<int64_t>(kPlanItems) * kPlanBlocks); }
int64_t plan_blocks(int64_t n) { return n > 0 ? ceil_div64(n, plan_per_block(n)) : 1; }

hif4_status check_sizes(int64_t tokens, int64_t cols, int64_t top_k, int64_t rows) {
  if (tokens < 0 || cols < 0 || top_k < 1 || rows < 0) return HIF4_ERR_SHAPE;
  if (top_k > 0x7FFFFFFFll || rows > 0x7FFFFFFFll || cols > (1ll << 40) || tokens > 0x7FFFFFFFll / top_k) return HIF4_ERR_SHAPE;
  return HIF4_OK;
}
// Blocks of a token: enough that few tokens fill the GPU, no more than there is work for `per_block` elements each.
hif4_status make_gather(Gather& g, int64_t tokens, int64_t cols, int64_t top_k, int64_t rows, const int32_t* row_of, int64_t per_block,
                        int64_t* blocks) {
  g.rows = rows; g.cols = cols; g.top_k = static_cast<int>(top_k); g.row_of = row_of;
  const int64_t segments = ceil_div64(cols, per_block);
  if (segments > 0x7FFFFFFFll / (tokens > 0 ? tokens : 1)) return HIF4_ERR_SHAPE;
  g.segments = static_cast<int>(segments);
  *blocks = tokens * segments;
  return HIF4_OK;
}

template <typename Word, int kAcross>
hif4_status launch_plain(const hif4_dispatch_args& a, cudaStream_t st) {
  const int64_t n = static_cast<int64_t>(sizeof(Word)) / type_size(a.dt);
  Gather g;
  int64_t blocks = 0;
  const hif4_status s = make_gather(g, a.tokens, a.cols, a.top_k, a.rows, a.row_of, kThreads * kAcross * n, &blocks);
  if (s != HIF4_OK) return s;
  return launch_overlapped(dispatch_plain_kernel<Word, kAcross>, static_cast<unsigned>(blocks), kThreads, 0, st, g, static_cast<const Word*>(a.x), a.ld_x / n,
                           static_cast<Word*>(a.out), a.ld_out / n, a.cols / n);
}
template <typename T>
hif4_status launch_converted(const hif4_dispatch_args& a, cudaStream_t st) {
  const T* x = static_cast<const T*>(a.x);
  Gather g;
  int64_t blocks = 0;
  if (a.kind == HIF4_ROWS_HIF4) {
    // a whole row a block where tokens fill the GPU, else as many blocks as there are rounds of 32 units
    const int64_t upr = a.cols / kUnitElems, per_round = kThreads / 8;
    const int block_units = a.tokens * ceil_div64(upr, kBlockUnits) >= 4ll * sm_count() ? kBlockUnits : static_cast<int>(per_round);
    const hif4_status s = make_gather(g, a.tokens, a.cols, a.top_k, a.rows, a.row_of, static_cast<int64_t>(block_units) * kUnitElems, &blocks);
    if (s != HIF4_OK) return s;
    const int wide = upr % 4 == 0 && aligned(a.out, 16);
    return launch_overlapped(a.mode == HIF4_RHA ? dispatch_hif4_kernel<T, true> : dispatch_hif4_kernel<T, false>, static_cast<unsigned>(blocks), kThreads, 0,
                             st, g, x, a.ld_x, static_cast<uint32_t*>(a.out), block_units, wide);
  }
  // a thread per 32 elements of the scale words' span, in blocks that share a row's evenly
  const bool nv = a.kind == HIF4_ROWS_NVFP4;
  const int64_t span = scale_words(a.cols, nv) * (nv ? 8 : 16), rounds = ceil_div64(span, kThreads);
  const unsigned threads = static_cast<unsigned>(ceil_div64(ceil_div64(span, rounds), 32) * 32);
  const hif4_status s = make_gather(g, a.tokens, span, a.top_k, a.rows, a.row_of, threads, &blocks);
  if (s != HIF4_OK) return s;
  g.cols = a.cols;
  return launch_overlapped(nv ? dispatch_bfp4_kernel<T, true> : dispatch_bfp4_kernel<T, false>, static_cast<unsigned>(blocks), threads, 0, st, g, x, a.ld_x,
                           a.gain, static_cast<uint4*>(a.out), static_cast<uint8_t*>(a.out_scales));
}

template <typename TI, typename TO>
hif4_status launch_combine(const hif4_combine_args& a, cudaStream_t st) {
  const bool vec = a.cols % 8 == 0 && rows_aligned(a.in, a.ld_in, a.dt_in) && rows_aligned(a.residual, a.residual ? a.ld_residual : 8, a.dt) &&
                   rows_aligned(a.y, a.ld_y, a.dt);
  const bool pairs = !vec && sizeof(TI) == 2 && sizeof(TO) == 2 && words_aligned(a.in, a.ld_in, a.cols) && words_aligned(a.y, a.ld_y, a.cols) &&
                     (!a.residual || words_aligned(a.residual, a.ld_residual, a.cols));
  Gather g;
  int64_t blocks = 0;
  const hif4_status s = make_gather(g, a.tokens, a.cols, a.top_k, a.rows, a.row_of, kThreads * (vec ? 8 : kNarrow * (pairs ? 2 : 1)), &blocks);
  if (s != HIF4_OK) return s;
  auto kernel = vec ? combine_kernel<TI, TO, 8, 1> : combine_kernel<TI, TO, 1, kNarrow>;
  if constexpr (sizeof(TI) == 2 && sizeof(TO) == 2)
    if (pairs) kernel = combine_kernel<TI, TO, 2, kNarrow>;
  return launch_overlapped(kernel, static_cast<unsigned>(blocks), kThreads, 0, st, g,
                           static_cast<const TI*>(a.in), a.ld_in, a.weights, static_cast<const TO*>(a.residual), a.ld_residual, a.res_scale,
                           static_cast<TO*>(a.y), a.ld_y);
}
template <typename TI, typename TD>
hif4_status launch_combine_backward(const hif4_combine_backward_args& a, cudaStream_t st) {
  const bool vec = a.cols % 8 == 0 && rows_aligned(a.dy, a.ld_dy, a.dt) && (!a.dweights || rows_aligned(a.in, a.ld_in, a.dt_in)) &&
                   (!a.din || rows_aligned(a.din, a.ld_din, a.dt_in));
  Gather g;
  int64_t blocks = 0;
  const hif4_status s = make_gather(g, a.tokens, a.cols, a.top_k, a.rows, a.row_of, a.cols > 0 ? a.cols : 1, &blocks);
  if (s != HIF4_OK) return s;
  // a warp a row where there are enough of them for all SMs, else a block a token
  const int64_t assignments = a.tokens * a.top_k;
  if (assignments >= 8ll * sm_count()) {
    auto kernel = vec ? combine_backward_rows_kernel<TD, TI, 8> : combine_backward_rows_kernel<TD, TI, 1>;
    if constexpr (sizeof(TI) == 2 && sizeof(TD) == 2)
      if (!vec && words_aligned(a.dy, a.ld_dy, a.cols) && (!a.dweights || words_aligned(a.in, a.ld_in, a.cols)) && (!a.din || words_aligned(a.din, a.ld_din, a.cols)))
        kernel = combine_backward_rows_kernel<TD, TI, 2>;
    return launch_overlapped(kernel, static_cast<unsigned>(ceil_div64(assignments, kThreads / 32)), kThreads, 0, st, g, assignments, static_cast<const TD*>(a.dy),
                             a.ld_dy, a.weights, static_cast<const TI*>(a.in), a.ld_in, static_cast<TI*>(a.din), a.ld_din, a.dweights);
  }
  // as many threads as go over the row in equal rounds
  const int64_t words = ceil_div64(a.cols > 0 ? a.cols : 1, vec ? 8 : 1), rounds = ceil_div64(words, kThreads);
  const unsigned threads = static_cast<unsigned>(ceil_div64(ceil_div64(words, rounds), 32) * 32);
  return launch_overlapped(vec ? combine_backward_kernel<TD, TI, 8> : combine_backward_kernel<TD, TI, 1>, static_cast<unsigned>(a.tokens), threads, 0, st,
                           g, static_cast<const TD*>(a.dy), a.ld_dy, a.weights, static_cast<const TI*>(a.in), a.ld_in, static_cast<TI*>(a.din), a.ld_din,
                           a.dweights);
}

}  // namespace
}  // namespace hif4

using namespace hif4;

// f<type of the experts' rows, type of the tokens' rows>(a, st)
#define HIF4_BY_TYPES(f, dt_in, dt, a, st)                                                                                       \
  (dt_in == HIF4_BF16 ? (dt == HIF4_BF16 ? f<__nv_bfloat16, __nv_bfloat16>(a, st) : dt == HIF4_FP16 ? f<__nv_bfloat16, __half>(a, st) \
                                                                                                    : f<__nv_bfloat16, float>(a, st)) \
   : dt_in == HIF4_FP16 ? (dt == HIF4_BF16 ? f<__half, __nv_bfloat16>(a, st) : dt == HIF4_FP16 ? f<__half, __half>(a, st)         \
                                                                                               : f<__half, float>(a, st))         \
                        : (dt == HIF4_BF16 ? f<float, __nv_bfloat16>(a, st) : dt == HIF4_FP16 ? f<float, __half>(a, st) : f<float, float>(a, st)))

extern "C" hif4_status hif4_expert_plan_workspace(int64_t tokens, int64_t top_k, int64_t experts, size_t* bytes) {
  if (!bytes) return HIF4_ERR_NULL;
  const hif4_status s = check_sizes(tokens, 0, top_k, 0);
  if (s != HIF4_OK) return s;
  if (experts < 1) return HIF4_ERR_SHAPE;
  if (experts > HIF4_ROUTE_MAX_EXPERTS) return HIF4_ERR_UNSUPPORTED;
  const int64_t blocks = plan_blocks(tokens * top_k);
  *bytes = blocks > 1 ? (static_cast<size_t>(blocks) * experts * sizeof(int32_t) + 255) / 256 * 256 : 0;
  return HIF4_OK;
}

extern "C" hif4_status hif4_expert_plan(const int32_t* ids, int64_t tokens, int64_t top_k, int64_t experts, int64_t* offsets, int32_t* row_of,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  const hif4_status s = hif4_expert_plan_workspace(tokens, top_k, experts, &need);
  if (s != HIF4_OK) return s;
  const int64_t n = tokens * top_k;
  if (!offsets || (n > 0 && (!ids || !row_of)) || (need > 0 && !workspace)) return HIF4_ERR_NULL;
  if (!aligned(ids, 4) || !aligned(row_of, 4) || !aligned(offsets, 8) || (need > 0 && !aligned(workspace, 256))) return HIF4_ERR_ALIGN;
  if (workspace_bytes < need) return HIF4_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int64_t blocks = plan_blocks(n), per_block = plan_per_block(n);
  const int64_t block_items = blocks > 1 ? kPlanItems : n;
  const int runs = n == 0 ? 1 : static_cast<int>(ceil_div64(block_items, kPlanSteps * 32)), of_experts = static_cast<int>(ceil_div64(experts, 32));
  const int warps = runs > of_experts ? runs : of_experts < kPlanWarps ? of_experts : kPlanWarps;
  const int smem = static_cast<int>(experts) * runs * 4;
  static uint64_t ready = 0;                             // (a launch that has not asked gets 48 KB, the kernel's own arrays included)
  if (!ensure_dynamic_smem(plan_place_kernel, HIF4_ROUTE_MAX_EXPERTS * kPlanWarps * 4, ready)) return HIF4_ERR_CUDA;
  int32_t* counts = static_cast<int32_t*>(workspace);
  if (blocks > 1) {
    const hif4_status c = launch_overlapped(plan_count_kernel, static_cast<unsigned>(blocks), kPlanWarps * 32, static_cast<size_t>(experts) * 4, st, ids, n,
                                            per_block, static_cast<int>(experts), counts);
    if (c != HIF4_OK) return c;
  }
  return launch_overlapped(plan_place_kernel, static_cast<unsigned>(blocks), static_cast<unsigned>(warps) * 32, static_cast<size_t>(smem), st, ids, n,
                           per_block, runs, static_cast<int>(experts), static_cast<const int32_t*>(counts), static_cast<int>(blocks), offsets, row_of);
}

extern "C" hif4_status hif4_dispatch(const hif4_dispatch_args* args, void* stream) {
  if (!args) return HIF4_ERR_NULL;
  const hif4_dispatch_args& a = *args;
  const hif4_status s = check_sizes(a.tokens, a.cols, a.top_k, a.rows);
  if (s != HIF4_OK) return s;
  if (!type_ok(a.dt) || a.kind < HIF4_ROWS_PLAIN || a.kind > HIF4_ROWS_NVFP4 || (a.kind == HIF4_ROWS_HIF4 && a.mode != HIF4_RNE && a.mode != HIF4_RHA))
    return HIF4_ERR_DTYPE;
  const bool plain = a.kind == HIF4_ROWS_PLAIN, scaled = a.kind == HIF4_ROWS_MXFP4 || a.kind == HIF4_ROWS_NVFP4;
  if (a.ld_x < a.cols || (plain && a.ld_out < a.cols) || (!plain && a.cols % kUnitElems != 0)) return HIF4_ERR_SHAPE;
  if (a.tokens == 0 || a.cols == 0 || a.rows == 0) return HIF4_OK;
  if (!a.x || !a.row_of || !a.out || (scaled && !a.out_scales)) return HIF4_ERR_NULL;
  if (!aligned(a.row_of, 4) || !aligned(a.x, type_size(a.dt)) || (plain && !aligned(a.out, type_size(a.dt))) ||
      (!plain && !rows_aligned(a.x, a.tokens > 1 ? a.ld_x : 0, a.dt)) || (a.kind == HIF4_ROWS_HIF4 && !aligned(a.out, 4)) ||
      (scaled && (!aligned(a.out, 16) || !aligned(a.out_scales, 16) || !aligned(a.gain, 4))))
    return HIF4_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!plain)
    return a.dt == HIF4_BF16   ? launch_converted<__nv_bfloat16>(a, st)
           : a.dt == HIF4_FP16 ? launch_converted<__half>(a, st)
                               : launch_converted<float>(a, st);
  const int64_t e = type_size(a.dt);
  const uintptr_t all = bits(a.x) | bits(a.out) | static_cast<uintptr_t>(a.cols * e) | static_cast<uintptr_t>(a.tokens > 1 ? a.ld_x * e : 0) |
                        static_cast<uintptr_t>(a.rows > 1 ? a.ld_out * e : 0);
  const int64_t word = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 2;
  return word == 16 ? launch_plain<uint4, 1>(a, st) : word == 4 ? launch_plain<uint32_t, kNarrow>(a, st) : launch_plain<uint16_t, kNarrow>(a, st);
}

extern "C" hif4_status hif4_combine(const hif4_combine_args* args, void* stream) {
  if (!args) return HIF4_ERR_NULL;
  const hif4_combine_args& a = *args;
  const hif4_status s = check_sizes(a.tokens, a.cols, a.top_k, a.rows);
  if (s != HIF4_OK) return s;
  if (!type_ok(a.dt) || !type_ok(a.dt_in)) return HIF4_ERR_DTYPE;
  if (a.ld_in < a.cols || a.ld_y < a.cols || (a.residual && a.ld_residual < a.cols)) return HIF4_ERR_SHAPE;
  if (a.tokens == 0 || a.cols == 0) return HIF4_OK;
  if ((!a.in && a.rows > 0) || !a.row_of || !a.y) return HIF4_ERR_NULL;
  if (!aligned(a.in, type_size(a.dt_in)) || !aligned(a.row_of, 4) || !aligned(a.weights, 4) || !aligned(a.residual, type_size(a.dt)) ||
      !aligned(a.y, type_size(a.dt)))
    return HIF4_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return HIF4_BY_TYPES(launch_combine, a.dt_in, a.dt, a, st);
}

extern "C" hif4_status hif4_combine_backward(const hif4_combine_backward_args* args, void* stream) {
  if (!args) return HIF4_ERR_NULL;
  const hif4_combine_backward_args& a = *args;
  const hif4_status s = check_sizes(a.tokens, a.cols, a.top_k, a.rows);
  if (s != HIF4_OK) return s;
  if (!type_ok(a.dt) || !type_ok(a.dt_in)) return HIF4_ERR_DTYPE;
  if (a.ld_dy < a.cols || (a.din && a.ld_din < a.cols) || (a.dweights && a.ld_in < a.cols)) return HIF4_ERR_SHAPE;
  if (a.tokens == 0 || (!a.din && !a.dweights)) return HIF4_OK;
  if ((!a.dy && a.cols > 0) || !a.row_of || (a.dweights && !a.in && a.rows > 0 && a.cols > 0)) return HIF4_ERR_NULL;
  if (!aligned(a.dy, type_size(a.dt)) || !aligned(a.row_of, 4) || !aligned(a.weights, 4) || !aligned(a.in, type_size(a.dt_in)) ||
      !aligned(a.din, type_size(a.dt_in)) || !aligned(a.dweights, 4))
    return HIF4_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return HIF4_BY_TYPES(launch_combine_backward, a.dt_in, a.dt, a, st);
}
