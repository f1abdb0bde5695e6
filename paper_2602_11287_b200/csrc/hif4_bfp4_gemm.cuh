// What the block-scaled products share: parameters, the MMA and its descriptor, the scales' way into tensor memory, the tensor map of
// packed codes.
//
// The MMA wants a scale word of row r in TMEM lane r % 32 (the same in all four lane quarters) and column r / 32, for
// each K = 64.  A row's scales of a K = 256 chunk are one 16-byte word in memory, which is just its four words; a warp of each
// lane quarter reads the rows' words and stores them.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hif4_bfp4_device.cuh"
#include "hif4_tc2_common.cuh"

namespace hif4 {

struct Bfp4Params {
  int64_t M, N;
  int chunks, last_steps;                   // K chunks of 256; K = 64 steps of the last one
  int n_tiles, m_tiles;
  const uint8_t *a_scales, *b_scales;
  int64_t b_scale_group;                    // bytes of a group's scales of B
  const float* alpha;
  void* y;
  int64_t ld_y;
  int dt, tma_store, row_copies, pair_words;  // how Y leaves shared memory: boxes, whole rows, two 16-bit elements at a time
  int num_groups;                           // 0: dense
  const int64_t* offsets;
  unsigned int* error_word;
};
// The CTA-pair kernel (256 x 256 tiles) and the persistent kernel for groups of few rows; grouped: up to kMaxTableGroups groups.
constexpr int kMaxTableGroups = 256;
hif4_status launch_bfp4_pairs(const hif4_bfp4_gemm_args& a, Bfp4Params p, cudaStream_t st);
hif4_status launch_bfp4_grouped(const hif4_bfp4_gemm_args& a, Bfp4Params p, cudaStream_t st);

namespace {

constexpr int kChunk = 256;                 // elements of K a stage
constexpr int kRowBytes = kChunk / 2;

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// kNv: four scales a K = 64 step (E4M3); else two (E8M0), of which the instruction descriptor names the half word.
template <bool kNv, int kCtas>
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
#define HIF4_MMA_SCALED(form)                                                                         \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\ttcgen05.mma." form " [%0], %1, %2, %3, [%4], [%5], p;\n\t}" \
               ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory")
  if (kNv && kCtas == 1) HIF4_MMA_SCALED("cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X");
  else if (kNv) HIF4_MMA_SCALED("cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X");
  else if (kCtas == 1) HIF4_MMA_SCALED("cta_group::1.kind::mxf4.block_scale.scale_vec::2X");
  else HIF4_MMA_SCALED("cta_group::2.kind::mxf4.block_scale.scale_vec::2X");
#undef HIF4_MMA_SCALED
}
// One lane of the warp (all lanes call).  The loops around MMAs are run by whole warps with only the MMAs under this condition: their
// descriptors are then uniform values for the compiler, where a loop run by one lane moves every operand to uniform registers
// before each MMA (218 clocks an MMA, waits included, that takes 128: 4096 x 14336 x 4096 152 -> 128 us).
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0u;
}
// The MMAs of one stage (`steps` of K = 64) and their descriptors' half words; kA, kB: columns of a step's scales.
template <bool kNv, int kCtas, int kA, int kB>
__device__ __forceinline__ void mma_stage(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, int steps, bool first) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (j < steps) {
      const int word = kNv ? j : j >> 1;
      const uint32_t half = kNv ? 0u : (static_cast<uint32_t>(j & 1) * 2u) * ((1u << 4) | (1u << 29));
      mma_scaled<kNv, kCtas>(d, adesc + 2 * j, bdesc + 2 * j, idesc | half, sfa + kA * word, sfb + kB * word, !first || j > 0);
    }
  }
}
// E2M1 operands, scale type, sizes; the scales' half word is added where it is used (bits 4 and 29).
template <bool kNv, int kM, int kN>
__host__ __device__ constexpr uint32_t instr_desc() {
  return (1u << 7) | (1u << 10) | (static_cast<uint32_t>(kN >> 3) << 17) | (kNv ? 0u : 1u << 23) | (static_cast<uint32_t>(kM >> 4) << 24);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Scale words of the lane's rows, as the columns want them: of 128 rows column 4 k + c holds step k of rows 32 c .. 32 c + 31, of 256
// rows column 8 k + c.
template <bool kNv, int kRuns>
__device__ __forceinline__ void read_scales(uint32_t smem, int lane, int half, uint32_t (&w)[kRuns * 4]) {
#pragma unroll
  for (int c = 0; c < kRuns; ++c) {
    const uint4 v = lds128(smem + (c * 32 + lane) * 16);
    if (kNv) {
      w[c] = v.x; w[kRuns + c] = v.y; w[2 * kRuns + c] = v.z; w[3 * kRuns + c] = v.w;
    } else {
      w[c] = half ? v.z : v.x; w[kRuns + c] = half ? v.w : v.y; w[2 * kRuns + c] = w[3 * kRuns + c] = 0u;
    }
  }
}

// The same of 32 kRuns <= 128 rows in the columns of 128 (zeros for rows that are not there).
template <bool kNv, int kRuns>
__device__ __forceinline__ void read_scales_128(uint32_t smem, int lane, int half, uint32_t (&w)[16]) {
  uint32_t v[kRuns * 4];
  read_scales<kNv, kRuns>(smem, lane, half, v);
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = (i & 3) < kRuns ? v[(i >> 2) * kRuns + (i & 3)] : 0u;
}

__device__ __forceinline__ void store_y(const Bfp4Params& p, int64_t m, int64_t n, float v) {
  const int64_t at = m * p.ld_y + n;
  if (p.dt == HIF4_FP32) static_cast<float*>(p.y)[at] = v;
  else if (p.dt == HIF4_BF16) static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p.y)[at] = __float2half_rn(v);
}
// A lane's column of Y: tokens m .. m + kCount - 1, of which `count` are there.
template <typename TO, int kCount>
__device__ __forceinline__ void store_tokens_as(TO* y, int64_t ld, int count, float alpha, const uint32_t (&r)[kCount]) {
#pragma unroll
  for (int j = 0; j < kCount; ++j, y += ld)
    if (j < count) *y = from_f32<TO>(alpha * __uint_as_float(r[j]));
}
template <int kCount>
__device__ __forceinline__ void store_tokens(const Bfp4Params& p, int64_t m, int count, int64_t n, float alpha, const uint32_t (&r)[kCount]) {
  const int64_t at = m * p.ld_y + n;
  if (p.dt == HIF4_FP32) store_tokens_as(static_cast<float*>(p.y) + at, p.ld_y, count, alpha, r);
  else if (p.dt == HIF4_BF16) store_tokens_as(static_cast<__nv_bfloat16*>(p.y) + at, p.ld_y, count, alpha, r);
  else store_tokens_as(static_cast<__half*>(p.y) + at, p.ld_y, count, alpha, r);
}

// ------------------------------------------------------------------------------------ tiles of a grouped product
// First rows, ends and running number of row tiles of the groups, in shared memory.
struct GroupTable { int tiles[kMaxTableGroups + 1], first[kMaxTableGroups], end[kMaxTableGroups]; };
constexpr int kGroupTableBytes = (static_cast<int>(sizeof(GroupTable)) + 15) / 16 * 16;
// One warp, from the offsets (clamped to 0 .. M; a group that ends before it begins is empty).
__device__ __forceinline__ void build_group_table(GroupTable& table, const Bfp4Params& p, int tile_rows, int lane) {
  int before = 0;
  for (int g0 = 0; g0 < p.num_groups; g0 += 32) {
    const int g = g0 + lane;
    int64_t lo = 0, hi = 0;
    if (g < p.num_groups) {
      lo = max(static_cast<int64_t>(0), min(p.M, p.offsets[g]));
      hi = max(lo, min(p.M, p.offsets[g + 1]));
    }
    int tiles = static_cast<int>((hi - lo + tile_rows - 1) / tile_rows);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, tiles, o);
      if (lane >= o) tiles += v;
    }
    if (g < p.num_groups) {
      table.tiles[g + 1] = before + tiles;
      table.first[g] = static_cast<int>(lo);
      table.end[g] = static_cast<int>(hi);
    }
    before += __shfl_sync(0xFFFFFFFFu, tiles, 31);
  }
  if (lane == 0) table.tiles[0] = 0;
}
// Tile t: groups one after the other, within a group the row tiles of the same rows of B.
struct GroupTile { int group, m0, m_end, nt; };
__device__ __forceinline__ GroupTile group_tile(const GroupTable& table, const Bfp4Params& p, int t, int tile_rows) {
  const int rows_before = t / p.n_tiles;                 // groups with table.tiles <= this end before the tile
  int lo = 0, hi = p.num_groups - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (table.tiles[mid + 1] <= rows_before) lo = mid + 1;
    else hi = mid;
  }
  const int mt = table.tiles[lo + 1] - table.tiles[lo], in = t - table.tiles[lo] * p.n_tiles;
  const int nt = in / mt;
  return {lo, table.first[lo] + (in - nt * mt) * tile_rows, table.end[lo], nt};
}

// Codes of a matrix: [rows, K / 2] bytes, box = 128 bytes x box_rows; what lies outside reads as zeros.
bool make_code_map(CUtensorMap* map, const void* base, int64_t rows, int64_t K, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(K / 2), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(K / 2)};
  const cuuint32_t box[2] = {kRowBytes, static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Y for an epilogue's copies.
bool make_y_map(CUtensorMap* map, const hif4_bfp4_gemm_args& a, int box_cols, int box_rows, CUtensorMapSwizzle swizzle) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const int size = a.dt == HIF4_FP32 ? 4 : 2;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(a.N), static_cast<cuuint64_t>(a.M)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(a.ld_y) * size};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, a.dt == HIF4_FP32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : a.dt == HIF4_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
            2, a.Y, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace hif4
