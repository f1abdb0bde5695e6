// hif4_bfp4_quantize, hif4_bfp4_quantize_transposed, hif4_bfp4_dequantize -- MXFP4 and NVFP4 operands from BF16, FP16
// and FP32 matrices and back.  HBM bound: 2 (4) bytes read and 0.53 (MXFP4) or 0.5625 (NVFP4) written per element.
#include "hif4_bfp4_device.cuh"
#include "hif4_vec8.cuh"

namespace hif4 {
namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ void load16(const T* p, float (&v)[16]) {
  float a[8];
  unpack8(load8(p), a);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = a[i];
  unpack8(load8(p + 8), a);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[8 + i] = a[i];
}

// A thread converts sixteen elements: a block of NVFP4, half a block of MXFP4 (its neighbour has the other half).
template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
bfp4_quantize_kernel(const T* __restrict__ src, int64_t rows, int64_t n16, int64_t ld, const float* __restrict__ gain,
                     uint2* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const bool in = i < rows * n16;
  const int64_t row = in ? i / n16 : 0, c = in ? i - row * n16 : 0;
  float v[16];
  load16(src + row * ld + 16 * c, v);
  if (gain) {
    const float g = *gain;
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = __fmul_rn(v[k], g);
  }
  uint32_t peak = peak16(v), byte;
  if (!kNv) peak = max(peak, __shfl_xor_sync(0xFFFFFFFFu, peak, 1));
  const uint2 code = encode16<kNv>(v, peak, byte);
  if (!in) return;
  codes[i] = code;
  const int64_t block = kNv ? c : c >> 1;
  if (kNv || !(c & 1)) scales[scale_at(row, block, rows)] = static_cast<uint8_t>(byte);
  if (c == n16 - 1)
    for (int64_t b = block + 1; b & 15; ++b) scales[scale_at(row, b, rows)] = 0;
}

// Tile of 256 rows x 32 columns in shared memory; a thread converts 32 rows of one column.
constexpr int kTileRows = 256, kTileCols = 32;
template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
bfp4_quantize_transposed_kernel(const T* __restrict__ src, int64_t rows, int64_t cols, int64_t ld, const float* __restrict__ gain,
                                uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int64_t row_tiles) {
  __shared__ __align__(16) T tile[kTileRows * kTileCols];
  const int64_t ct = blockIdx.x / row_tiles, r0 = (blockIdx.x - ct * row_tiles) * kTileRows, c0 = ct * kTileCols;
  constexpr int kPer = 16 / sizeof(T), kChunks = kTileCols / kPer;      // elements of a 16-byte chunk, chunks of a tile row
  for (int n = threadIdx.x; n < kTileRows * kChunks; n += kThreads) {
    const int r = n / kChunks, ch = n - r * kChunks;
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (r0 + r < rows && c0 + ch * kPer < cols) w = *reinterpret_cast<const uint4*>(src + (r0 + r) * ld + c0 + ch * kPer);
    *reinterpret_cast<uint4*>(tile + r * kTileCols + ch * kPer) = w;
  }
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const int64_t c = c0 + lane, r = r0 + (threadIdx.x >> 5) * 32;
  if (c >= cols || r >= rows) return;
  const T* mine = tile + (threadIdx.x >> 5) * 32 * kTileCols + lane;
  const float g = gain ? *gain : 1.0f;
  float a[16], b[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    a[k] = to_f32(mine[k * kTileCols]);
    b[k] = to_f32(mine[(16 + k) * kTileCols]);
    if (gain) { a[k] = __fmul_rn(a[k], g); b[k] = __fmul_rn(b[k], g); }
  }
  uint32_t pa = peak16(a), pb = peak16(b), sa, sb;
  if (!kNv) pa = pb = max(pa, pb);
  const uint2 ca = encode16<kNv>(a, pa, sa), cb = encode16<kNv>(b, pb, sb);
  *reinterpret_cast<uint4*>(codes + c * (rows / 2) + r / 2) = make_uint4(ca.x, ca.y, cb.x, cb.y);
  int64_t block = r / (kNv ? 16 : 32);
  scales[scale_at(c, block, cols)] = static_cast<uint8_t>(sa);
  if (kNv) scales[scale_at(c, ++block, cols)] = static_cast<uint8_t>(sb);
  if (r + 32 == rows)
    for (++block; block & 15; ++block) scales[scale_at(c, block, cols)] = 0;
}

template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
bfp4_dequantize_kernel(const uint2* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, int64_t n16,
                       const float* __restrict__ gain, T* __restrict__ dst, int64_t ld) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= rows * n16) return;
  const int64_t row = i / n16, c = i - row * n16;
  const uint2 code = codes[i];
  const float s = scale_value<kNv>(scales[scale_at(row, kNv ? c : c >> 1, rows)]);
  float v[16];
  e2m1_to8(code.x, v);
  e2m1_to8(code.y, v + 8);
  const float g = gain ? *gain : 1.0f;
  float lo[8], hi[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    lo[k] = __fmul_rn(v[k], s);
    hi[k] = __fmul_rn(v[8 + k], s);
    if (gain) { lo[k] = __fdiv_rn(lo[k], g); hi[k] = __fdiv_rn(hi[k], g); }
  }
  T* p = dst + row * ld + 16 * c;
  store8(p, pack8<T>(lo));
  store8(p + 8, pack8<T>(hi));
}

bool format_ok(int fmt) { return fmt == HIF4_FMT_MXFP4 || fmt == HIF4_FMT_NVFP4; }
size_t type_size(int dt) { return dt == HIF4_FP32 ? 4 : 2; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace hif4

using namespace hif4;

extern "C" size_t hif4_bfp4_scale_bytes(int64_t rows, int64_t cols, hif4_bfp4_format fmt) {
  if (rows < 0 || cols < 0 || cols % kUnitElems != 0 || !format_ok(fmt)) return 0;
  return static_cast<size_t>(rows) * static_cast<size_t>(scale_words(cols, fmt == HIF4_FMT_NVFP4)) * 16;
}

#define HIF4_BFP4_LAUNCH(kernel, ...)                                                                       \
  do {                                                                                                      \
    const bool nv = fmt == HIF4_FMT_NVFP4;                                                                  \
    if (dt == HIF4_BF16) nv ? kernel<__nv_bfloat16, true>(__VA_ARGS__) : kernel<__nv_bfloat16, false>(__VA_ARGS__); \
    else if (dt == HIF4_FP16) nv ? kernel<__half, true>(__VA_ARGS__) : kernel<__half, false>(__VA_ARGS__);  \
    else nv ? kernel<float, true>(__VA_ARGS__) : kernel<float, false>(__VA_ARGS__);                         \
  } while (0)

namespace {
template <typename T, bool kNv>
void quantize_rows(const void* src, int64_t rows, int64_t cols, int64_t ld, const float* gain, void* codes, void* scales, cudaStream_t st) {
  const int64_t blocks = ceil_div64(rows * (cols / 16), kThreads);
  bfp4_quantize_kernel<T, kNv><<<static_cast<unsigned>(blocks), kThreads, 0, st>>>(static_cast<const T*>(src), rows, cols / 16, ld, gain,
                                                                                    static_cast<uint2*>(codes), static_cast<uint8_t*>(scales));
}
template <typename T, bool kNv>
void quantize_columns(const void* src, int64_t rows, int64_t cols, int64_t ld, const float* gain, void* codes, void* scales, cudaStream_t st) {
  const int64_t row_tiles = ceil_div64(rows, kTileRows), blocks = row_tiles * ceil_div64(cols, kTileCols);
  bfp4_quantize_transposed_kernel<T, kNv><<<static_cast<unsigned>(blocks), kThreads, 0, st>>>(
      static_cast<const T*>(src), rows, cols, ld, gain, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), row_tiles);
}
template <typename T, bool kNv>
void dequantize_rows(const void* codes, const void* scales, int64_t rows, int64_t cols, const float* gain, void* dst, int64_t ld, cudaStream_t st) {
  const int64_t blocks = ceil_div64(rows * (cols / 16), kThreads);
  bfp4_dequantize_kernel<T, kNv><<<static_cast<unsigned>(blocks), kThreads, 0, st>>>(
      static_cast<const uint2*>(codes), static_cast<const uint8_t*>(scales), rows, cols / 16, gain, static_cast<T*>(dst), ld);
}
hif4_status check(const void* src, hif4_dtype dt, int64_t rows, int64_t cols, int64_t ld, hif4_bfp4_format fmt, const float* gain,
                  const void* codes, const void* scales) {
  if (rows < 0 || cols < 0 || ld < cols) return HIF4_ERR_SHAPE;
  if ((dt != HIF4_BF16 && dt != HIF4_FP16 && dt != HIF4_FP32) || !format_ok(fmt)) return HIF4_ERR_DTYPE;
  if (rows == 0 || cols == 0) return HIF4_OK;
  if (cols / 16 + 1 > 0x7FFFFFFFll / (rows / 16 + 1)) return HIF4_ERR_SHAPE;      // more blocks than a grid has
  if (!src || !codes || !scales) return HIF4_ERR_NULL;
  if (!aligned16(src) || (static_cast<size_t>(ld) * type_size(dt)) % 16 != 0 || !aligned16(codes) || !aligned16(scales) ||
      (reinterpret_cast<uintptr_t>(gain) & 3u))
    return HIF4_ERR_ALIGN;
  return HIF4_OK;
}
}  // namespace

extern "C" hif4_status hif4_bfp4_quantize(const void* src, hif4_dtype dt, int64_t rows, int64_t cols, int64_t ld_src, hif4_bfp4_format fmt,
                                          const float* gain, void* codes, void* scales, void* stream) {
  if (cols % kUnitElems != 0) return HIF4_ERR_SHAPE;
  const hif4_status s = check(src, dt, rows, cols, ld_src, fmt, gain, codes, scales);
  if (s != HIF4_OK || rows == 0 || cols == 0) return s;
  HIF4_BFP4_LAUNCH(quantize_rows, src, rows, cols, ld_src, gain, codes, scales, static_cast<cudaStream_t>(stream));
  note_launch();
  return launch_status();
}

extern "C" hif4_status hif4_bfp4_quantize_transposed(const void* src, hif4_dtype dt, int64_t rows, int64_t cols, int64_t ld_src,
                                                     hif4_bfp4_format fmt, const float* gain, void* codes, void* scales, void* stream) {
  if (rows % kUnitElems != 0 || cols % 8 != 0) return HIF4_ERR_SHAPE;
  const hif4_status s = check(src, dt, rows, cols, ld_src, fmt, gain, codes, scales);
  if (s != HIF4_OK || rows == 0 || cols == 0) return s;
  HIF4_BFP4_LAUNCH(quantize_columns, src, rows, cols, ld_src, gain, codes, scales, static_cast<cudaStream_t>(stream));
  note_launch();
  return launch_status();
}

extern "C" hif4_status hif4_bfp4_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, hif4_bfp4_format fmt,
                                            const float* gain, void* dst, hif4_dtype dt, int64_t ld_dst, void* stream) {
  if (cols % kUnitElems != 0) return HIF4_ERR_SHAPE;
  if (dt != HIF4_BF16 && dt != HIF4_FP32) return HIF4_ERR_DTYPE;
  const hif4_status s = check(dst, dt, rows, cols, ld_dst, fmt, gain, codes, scales);
  if (s != HIF4_OK || rows == 0 || cols == 0) return s;
  const bool nv = fmt == HIF4_FMT_NVFP4;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dt == HIF4_BF16)
    nv ? dequantize_rows<__nv_bfloat16, true>(codes, scales, rows, cols, gain, dst, ld_dst, st)
       : dequantize_rows<__nv_bfloat16, false>(codes, scales, rows, cols, gain, dst, ld_dst, st);
  else
    nv ? dequantize_rows<float, true>(codes, scales, rows, cols, gain, dst, ld_dst, st)
       : dequantize_rows<float, false>(codes, scales, rows, cols, gain, dst, ld_dst, st);
  note_launch();
  return launch_status();
}
