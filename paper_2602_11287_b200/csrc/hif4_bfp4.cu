// hif4_bfp4_quantize, hif4_bfp4_quantize_transposed, hif4_bfp4_dequantize -- MXFP4 and NVFP4 operands from BF16, FP16
// and FP32 matrices and back.  HBM bound: 2 (4) bytes read and 0.53 (MXFP4) or 0.5625 (NVFP4) written per element.
#include "hif4_bfp4_device.cuh"
#include "hif4_tc_common.cuh"

namespace hif4 {
namespace {

constexpr int kThreads = 256;

// A thread converts sixteen elements: a block of NVFP4, half a block of MXFP4 (its neighbour has the other half).
template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
bfp4_quantize_kernel(const T* __restrict__ src, int64_t rows, int64_t items, Divider n16, int64_t ld, int wide, const float* __restrict__ gain,
                     uint2* __restrict__ codes, uint8_t* __restrict__ scales) {
  grid_wait();
  grid_launch_next();
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * kThreads; first < items; first += static_cast<int64_t>(gridDim.x) * kThreads) {
    const int64_t i = first + threadIdx.x;
    const bool in = i < items;
    const int64_t at = in ? i : 0;
    const int64_t row = items <= 0x7FFFFFFF ? n16.quotient(static_cast<uint32_t>(at)) : at / n16.d;
    const uint32_t c = static_cast<uint32_t>(at - row * n16.d);
    Sixteen v = sixteen_of(load_raw16(src + row * ld + 16 * static_cast<int64_t>(c), wide));
    if (gain) scale16(v, *gain);
    uint32_t peak = peak16(v), byte;
    if (!kNv) peak = max(peak, __shfl_xor_sync(0xFFFFFFFFu, peak, 1));
    const uint2 code = encode16<kNv>(v, peak, byte);
    if (!in) continue;
    codes[i] = code;
    const uint32_t block = kNv ? c : c >> 1;
    if (kNv || !(c & 1)) scales[scale_at(row, block, rows)] = static_cast<uint8_t>(byte);
    if (c == n16.d - 1)
      for (uint32_t b = block + 1; b & 15; ++b) scales[scale_at(row, b, rows)] = 0;
  }
}

// Tile of 256 rows x 32 columns in shared memory; a thread converts 32 rows of one column.
constexpr int kTileRows = 256, kTileCols = 32;
template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
bfp4_quantize_transposed_kernel(const T* __restrict__ src, int64_t rows, int64_t cols, int64_t ld, const float* __restrict__ gain,
                                uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int64_t row_tiles) {
  __shared__ __align__(16) T tile[kTileRows * kTileCols];
  grid_wait();
  grid_launch_next();
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
  Sixteen a, b;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    a.p[k] = make_float2(to_f32(mine[2 * k * kTileCols]), to_f32(mine[(2 * k + 1) * kTileCols]));
    b.p[k] = make_float2(to_f32(mine[(16 + 2 * k) * kTileCols]), to_f32(mine[(17 + 2 * k) * kTileCols]));
  }
  if (gain) {
    scale16(a, *gain);
    scale16(b, *gain);
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

// Sixteen values m s (m an E2M1 number), or m s / g.  Only 1 and 1.5 times a power of two occur among the m, so two divisions make
// all quotients of a block, the rest are exact products with powers of two; where those might leave FP32's range each
// element is divided.
template <typename T, bool kNv>
__device__ __forceinline__ void decode16(uint2 code, uint32_t byte, const float* gain, float (&v)[16]) {
  const float s = scale_value<kNv>(byte);
  e2m1_to8(code.x, v);
  e2m1_to8(code.y, v + 8);
  if (!gain) {
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] *= s;
    return;
  }
  const float g = *gain, d1 = __fdiv_rn(s, g), d3 = __fdiv_rn(1.5f * s, g), size = fabsf(d1);
  if (size > 0x1p-100f && size < 0x1p100f && s > 0x1p-120f) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const uint32_t m = __float_as_uint(v[k]);
      v[k] = __uint_as_float(m & 0xFF800000u) * ((m & 0x00400000u) ? d3 : d1);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = __fdiv_rn(__fmul_rn(v[k], s), g);
  }
}

__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
               "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void store_row16(__nv_bfloat16* p, const float (&v)[16], bool wide) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1], __nv_bfloat16());
  if (wide) {
    store32(p, w);
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
__device__ __forceinline__ void store_row16(float* p, const float (&v)[16], bool wide) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[8 * h + i]);
    if (wide) {
      store32(p + 8 * h, w);
    } else {
      reinterpret_cast<uint4*>(p + 8 * h)[0] = make_uint4(w[0], w[1], w[2], w[3]);
      reinterpret_cast<uint4*>(p + 8 * h)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
}

template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
bfp4_dequantize_kernel(const uint2* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, int64_t items, Divider n16,
                       const float* __restrict__ gain, T* __restrict__ dst, int64_t ld, int wide) {
  grid_wait();
  grid_launch_next();
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < items; i += static_cast<int64_t>(gridDim.x) * kThreads) {
    const int64_t row = items <= 0x7FFFFFFF ? n16.quotient(static_cast<uint32_t>(i)) : i / n16.d;
    const uint32_t c = static_cast<uint32_t>(i - row * n16.d);
    float v[16];
    decode16<T, kNv>(codes[i], scales[scale_at(row, kNv ? c : c >> 1, rows)], gain, v);
    store_row16(dst + row * ld + 16 * static_cast<int64_t>(c), v, wide);
  }
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

#define HIF4_BFP4_LAUNCH(f, nv, ...)                                                                                    \
  (dt == HIF4_BF16 ? (nv ? f<__nv_bfloat16, true>(__VA_ARGS__) : f<__nv_bfloat16, false>(__VA_ARGS__))                   \
   : dt == HIF4_FP16 ? (nv ? f<__half, true>(__VA_ARGS__) : f<__half, false>(__VA_ARGS__))                               \
                     : (nv ? f<float, true>(__VA_ARGS__) : f<float, false>(__VA_ARGS__)))

namespace {
unsigned blocks_for(int64_t items) {
  const int64_t blocks = ceil_div64(items, kThreads);
  return static_cast<unsigned>(blocks < 0x7FFFFFFFll ? blocks : 0x7FFFFFFFll);
}
int rows_wide(const void* p, int64_t ld, size_t size) { return (reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld) * size) % 32 == 0; }
template <typename T, bool kNv>
hif4_status quantize_rows(const void* src, int64_t rows, int64_t cols, int64_t ld, const float* gain, void* codes, void* scales, cudaStream_t st) {
  const int64_t items = rows * (cols / 16);
  return launch_overlapped(bfp4_quantize_kernel<T, kNv>, blocks_for(items), kThreads, 0, st, static_cast<const T*>(src), rows, items,
                           make_divider(static_cast<uint32_t>(cols / 16)), ld, rows_wide(src, ld, sizeof(T)), gain, static_cast<uint2*>(codes),
                           static_cast<uint8_t*>(scales));
}
template <typename T, bool kNv>
hif4_status quantize_columns(const void* src, int64_t rows, int64_t cols, int64_t ld, const float* gain, void* codes, void* scales, cudaStream_t st) {
  const int64_t row_tiles = ceil_div64(rows, kTileRows), blocks = row_tiles * ceil_div64(cols, kTileCols);
  return launch_overlapped(bfp4_quantize_transposed_kernel<T, kNv>, static_cast<unsigned>(blocks), kThreads, 0, st,
      static_cast<const T*>(src), rows, cols, ld, gain, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), row_tiles);
}
template <typename T, bool kNv>
hif4_status dequantize_rows(const void* codes, const void* scales, int64_t rows, int64_t cols, const float* gain, void* dst, int64_t ld, cudaStream_t st) {
  const int64_t items = rows * (cols / 16);
  return launch_overlapped(bfp4_dequantize_kernel<T, kNv>, blocks_for(items), kThreads, 0, st,
      static_cast<const uint2*>(codes), static_cast<const uint8_t*>(scales), rows, items, make_divider(static_cast<uint32_t>(cols / 16)), gain,
      static_cast<T*>(dst), ld, rows_wide(dst, ld, sizeof(T)));
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
  return HIF4_BFP4_LAUNCH(quantize_rows, fmt == HIF4_FMT_NVFP4, src, rows, cols, ld_src, gain, codes, scales, static_cast<cudaStream_t>(stream));
}

extern "C" hif4_status hif4_bfp4_quantize_transposed(const void* src, hif4_dtype dt, int64_t rows, int64_t cols, int64_t ld_src,
                                                     hif4_bfp4_format fmt, const float* gain, void* codes, void* scales, void* stream) {
  if (rows % kUnitElems != 0 || cols % 8 != 0) return HIF4_ERR_SHAPE;
  const hif4_status s = check(src, dt, rows, cols, ld_src, fmt, gain, codes, scales);
  if (s != HIF4_OK || rows == 0 || cols == 0) return s;
  return HIF4_BFP4_LAUNCH(quantize_columns, fmt == HIF4_FMT_NVFP4, src, rows, cols, ld_src, gain, codes, scales, static_cast<cudaStream_t>(stream));
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
    return nv ? dequantize_rows<__nv_bfloat16, true>(codes, scales, rows, cols, gain, dst, ld_dst, st)
              : dequantize_rows<__nv_bfloat16, false>(codes, scales, rows, cols, gain, dst, ld_dst, st);
  return nv ? dequantize_rows<float, true>(codes, scales, rows, cols, gain, dst, ld_dst, st)
            : dequantize_rows<float, false>(codes, scales, rows, cols, gain, dst, ld_dst, st);
}
