// Host side of the CTA-pair linear kernel: tensor maps, schedule, launch.
#pragma once
#include "hif4_linear_tc2.cuh"

namespace hif4 {
namespace {

inline bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// View of Y for the TMA stores: boxes of 64 bytes x 32 rows, SWIZZLE_64B.
template <typename T>
bool make_y_map(CUtensorMap* map, void* y, int64_t M, int64_t N, int64_t ld) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const CUtensorMapDataType type = sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(N), static_cast<cuuint64_t>(M)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * sizeof(T)};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(64 / sizeof(T)), 32};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, type, 2, y, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The schedule of the FP32 product, but for a single round of tiles its own number of K slices: here the parts are left side
// by side and one slice adds them all, where the FP32 product chains them.  A chunk (K = 256) is about 1.8 us; leaving and
// meeting the parts costs about 2.5 us once, and adding one about 1.1 us for 256 columns (64 x 1024 x 14336: eight slices,
// 35 us; the FP32 product with its chain of four 45 us).
constexpr int kMaxLinearSlices = 32;
inline Tc2Plan linear_plan(int64_t M, int64_t N, int64_t K, int tile_n) {
  Tc2Plan pl = tc2_plan(M, N, K, tile_n);
  if (pl.full_rounds > 0 || pl.sk_tiles > 0 || pl.tail_tiles <= 0) return pl;
  const int64_t chunks = ceil_div64(K, 256), columns = N < tile_n ? N : tile_n;
  int64_t s_max = sm_count() / 2 / pl.tail_tiles;
  if (s_max > kMaxLinearSlices) s_max = kMaxLinearSlices;
  if (s_max > chunks) s_max = chunks;
  int64_t best = 1, best_cost = 18 * chunks;                                     // in tenths of a microsecond
  for (int64_t s = 2; s <= s_max; ++s) {
    const int64_t cost = 18 * ceil_div64(chunks, s) + 25 + 11 * (s - 1) * columns / tile_n;
    if (cost < best_cost) { best = s; best_cost = cost; }
  }
  pl.slices = static_cast<int>(best);
  pl.flag_bytes = best > 1 ? (static_cast<size_t>(pl.tail_tiles) * best * 8 * sizeof(unsigned int) + 255) / 256 * 256 : 0;
  pl.bytes = pl.flag_bytes;
  return pl;
}
inline size_t partial_tiles(const Tc2Plan& pl) {
  return pl.sk_tiles > 0 ? static_cast<size_t>(pl.pairs) + 1 : pl.slices > 1 ? static_cast<size_t>(pl.tail_tiles) * (pl.slices - 1) : 0;
}
constexpr size_t kPartialTileBytes = static_cast<size_t>(kPairM) * kPairN * sizeof(float);

template <bool kGated, bool kGrad, typename T, int kAct, int kParts>
hif4_status launch_linear_parts(const LinearCall& c, void* workspace, cudaStream_t st) {
  constexpr int kTileN = kGated ? kPairN / 2 : kPairN;
  static uint64_t smem_opt_in = 0;
  if (!ensure_dynamic_smem(linear_tc2_kernel<kGated, kGrad, T, kAct, kParts>, kLinSmemBytes, smem_opt_in)) return HIF4_ERR_CUDA;
  LinearParams p{};
  p.M = c.M; p.N = c.N;
  p.error_word = device_error_word();
  if (!p.error_word) return HIF4_ERR_CUDA;
  const int64_t upr = c.K / kUnitElems;
  p.num_kc = c.K > 0 ? static_cast<int>(ceil_div64(upr, kRawUnits)) : 1;       // K = 0: one chunk of zeros
  p.n_tiles = static_cast<int>(ceil_div64(c.N, kTileN));
  const Tc2Plan pl = linear_plan(c.M, c.N, c.K, kTileN);
  p.full_rounds = pl.full_rounds; p.tail_tiles = pl.tail_tiles; p.slices = pl.slices;
  p.sk_tiles = pl.sk_tiles; p.sk_tile0 = pl.sk_tile0;
  p.mul = make_decode_mul();
  // no operand byte is read for K = 0, but the copy loop wants an address
  p.A = static_cast<const uint8_t*>(c.K > 0 ? c.A : p.error_word);
  p.B = static_cast<const uint8_t*>(c.K > 0 ? c.B : p.error_word);
  p.B2 = static_cast<const uint8_t*>(c.K > 0 ? c.B2 : p.error_word);
  p.pitch = upr * kUnitBytes;
  p.upr = static_cast<int>(upr);
  CUtensorMap tmA{}, tmB{}, tmB2{}, tmY{}, tmSide{};
  p.tma = c.K > 0 && c.K % (kRawUnits * kUnitElems) == 0 && at16(c.A) && at16(c.B) && (!kGated || at16(c.B2));
  if (p.tma) {
    if (!make_unit_map(&tmA, c.A, c.M, upr, kRows) || !make_unit_map(&tmB, c.B, c.N, upr, kRows)) return HIF4_ERR_CUDA;
    if (kGated && !make_unit_map(&tmB2, c.B2, c.N, upr, kRows)) return HIF4_ERR_CUDA;
  }
  p.bias = c.bias; p.bias_up = c.bias_up;
  p.side = c.side; p.ld_side = c.ld_side; p.res_scale = c.res_scale;
  p.side_vec = at16(c.side) && (c.M == 1 || c.ld_side * sizeof(T) % 16 == 0);
  // through the staging buffers where they are not taken by units (a load clips columns past N element by element)
  p.side_tma = c.side && p.side_vec && c.ld_side * sizeof(T) % 16 == 0 && !c.units && make_y_map<T>(&tmSide, const_cast<void*>(c.side), c.M, c.N, c.ld_side);
  p.y = c.y; p.ld_y = c.ld_y; p.units = c.units; p.rha = c.rha;
  if (!kGrad && !c.units) {
    // (a TMA store clips the innermost dimension in 16-byte pieces: other widths are copied from the staging buffers)
    p.tma_store = at16(c.y) && c.ld_y * sizeof(T) % 16 == 0 && c.N * sizeof(T) % 16 == 0 && make_y_map<T>(&tmY, c.y, c.M, c.N, c.ld_y);
  }
  p.dz = c.dz; p.ld_dz = c.ld_dz; p.dz_plane = c.dz_plane;
  p.colsum = c.colsum; p.colsum_plane = ceil_div64(c.M, 32) * c.N;
  if (p.slices > 1) {
    p.flags = static_cast<unsigned int*>(workspace);
    p.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + pl.flag_bytes);
  }
  const int pairs = p.full_rounds == 0 && p.sk_tiles == 0 ? p.tail_tiles * p.slices : pl.pairs;      // a single round: one pair per slice
  return launch_overlapped(linear_tc2_kernel<kGated, kGrad, T, kAct, kParts>, 2 * pairs, kThreads, kLinSmemBytes, st, tmA, tmB, tmB2, tmY, tmSide, p);
}

template <bool kGated, bool kGrad, typename T, int kAct>
hif4_status launch_linear_act(const LinearCall& c, void* workspace, cudaStream_t st) {
  if constexpr (kGrad && IsHalf<T>::value) return launch_linear_parts<kGated, kGrad, T, kAct, 2>(c, workspace, st);
  if constexpr (kGrad && !IsHalf<T>::value) {
    if (c.parts == 2) return launch_linear_parts<kGated, kGrad, T, kAct, 2>(c, workspace, st);
  }
  return launch_linear_parts<kGated, kGrad, T, kAct, 1>(c, workspace, st);
}

template <bool kGated, bool kGrad, typename T>
hif4_status launch_linear(const LinearCall& c, void* workspace, cudaStream_t st) {
  switch (c.act) {
    case HIF4_ACT_RELU: return launch_linear_act<kGated, kGrad, T, HIF4_ACT_RELU>(c, workspace, st);
    case HIF4_ACT_SILU: return launch_linear_act<kGated, kGrad, T, HIF4_ACT_SILU>(c, workspace, st);
    case HIF4_ACT_GELU: return launch_linear_act<kGated, kGrad, T, HIF4_ACT_GELU>(c, workspace, st);
    case HIF4_ACT_GELU_TANH: return launch_linear_act<kGated, kGrad, T, HIF4_ACT_GELU_TANH>(c, workspace, st);
    default: break;
  }
  if constexpr (kGrad && !kGated) return HIF4_ERR_UNSUPPORTED;          // dZ = dY needs no product
  else return launch_linear_act<kGated, kGrad, T, HIF4_ACT_NONE>(c, workspace, st);
}

}  // namespace
}  // namespace hif4
