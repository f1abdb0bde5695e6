// hif4_bfp4_quantize, hif4_bfp4_quantize_transposed, hif4_bfp4_dequantize -- MXFP4 and NVFP4 operands from BF16, FP16
// and FP32 matrices and back.  HBM bound: 2 (4) bytes read and 0.53 (MXFP4) or 0.5625 (NVFP4) written per element.
// 8192 x 5120 BF16: 16.7 us to MXFP4 (6.4 TB/s), 18.8 us to NVFP4 (5.7), 17.7 and 18.7 us back; FP32 33 us; down the columns 29 and 32 us,
// FP32 33 us.  With a gain MXFP4 17.4 us, NVFP4 19.4; back from NVFP4 21 us, the integer pipe 44 % (there) and 73 % (back) busy.
#include "hif4_bfp4_device.cuh"
#include "hif4_tc_common.cuh"

namespace hif4 {
namespace {

constexpr int kThreads = 256;

// A thread takes 32 elements: two blocks of NVFP4, one of MXFP4.  A warp takes the scale words of one place in four rows (NVFP4, eight lanes a
// word) or two (MXFP4, sixteen lanes): the words of neighbouring rows are neighbours in memory.  Warps go along the rows first.
// (Sixteen elements a thread: half as long again, addresses and scales cost as much as the elements.)
struct WordTask { int64_t row; uint32_t word, c; };           // c: the lane's 32 elements within the row
template <bool kNv>
__device__ __forceinline__ WordTask word_task(uint32_t warp, const Divider& words, int lane) {
  const uint32_t line = words.quotient(warp), word = warp - line * words.d;
  if (kNv) return {static_cast<int64_t>(line) * 4 + (lane >> 3), word, word * 8 + (lane & 7)};
  return {static_cast<int64_t>(line) * 2 + (lane >> 4), word, word * 16 + (lane & 15)};
}
// Where the lane's scale bytes are.
template <bool kNv>
__device__ __forceinline__ int64_t scale_offset(const WordTask& t, int64_t rows, int lane) {
  return (t.word * rows + t.row) * 16 + (kNv ? 2 * (lane & 7) : lane & 15);
}

template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
bfp4_quantize_kernel(const T* __restrict__ src, int64_t rows, uint32_t n32, uint32_t tasks, Divider words, int64_t ld, int wide,
                     const float* __restrict__ gain, uint4* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int lane = threadIdx.x & 31;
  const uint32_t warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  grid_wait();
  grid_launch_next();
  if (warp >= tasks) return;
  const WordTask t = word_task<kNv>(warp, words, lane);
  if (t.row >= rows) return;
  uint32_t sa = 0u, sb = 0u;                                              // (0 past the last block)
  const float g = gain ? *gain : 1.0f;
  if (t.c < n32) {
    const T* p = src + t.row * ld + 32 * static_cast<int64_t>(t.c);
    const Raw16<T> ra = load_raw16(p, wide), rb = load_raw16(p + 16, wide);
    Sixteen a = sixteen_of(ra), b = sixteen_of(rb);
    uint32_t pa = peak16(ra), pb = peak16(rb);
    if (!kNv) pa = pb = max(pa, pb);
    if (gain) apply_gain<kNv>(a, b, pa, pb, g);
    const uint2 ca = encode16<kNv>(a, pa, sa), cb = encode16<kNv>(b, pb, sb);
    codes[t.row * n32 + t.c] = make_uint4(ca.x, ca.y, cb.x, cb.y);
  }
  uint8_t* scale = scales + scale_offset<kNv>(t, rows, lane);
  if (kNv) *reinterpret_cast<uint16_t*>(scale) = static_cast<uint16_t>(sa | (sb << 8));
  else *scale = static_cast<uint8_t>(sa);
}

// Tile of 256 rows x 128 bytes in shared memory; a thread converts 32 rows of a column.  Codes and scales are collected in shared
// memory and leave as 128 bytes and one word (half a word) per column: stored by the threads that made them, 16 and 1 bytes to
// another line each, they bounded the kernel (8192 x 5120 BF16 to MXFP4 38 us, NVFP4 46 us).
constexpr int kTileRows = 256;
template <typename T> constexpr int kTileCols = 128 / static_cast<int>(sizeof(T));
constexpr int kCodePitch = kTileRows / 2 + 16;           // bytes of a column's codes; an odd number of 16-byte words: no bank conflicts
template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
bfp4_quantize_transposed_kernel(const T* __restrict__ src, int64_t rows, int64_t cols, int64_t ld, const float* __restrict__ gain,
                                uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int64_t row_tiles) {
  constexpr int kCols = kTileCols<T>, kPer = 16 / sizeof(T);                // elements of a 16-byte chunk; eight chunks a tile row
  constexpr int kLoads = kTileRows * 8 / kThreads;
  __shared__ __align__(16) T tile[kTileRows * kCols];
  __shared__ __align__(16) uint8_t code_tile[kCols * kCodePitch];
  __shared__ __align__(16) uint8_t scale_tile[kCols * 16];
  grid_wait();
  grid_launch_next();
  const int64_t ct = blockIdx.x / row_tiles, r0 = (blockIdx.x - ct * row_tiles) * kTileRows, c0 = ct * kCols;
  uint4 w[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int n = i * kThreads + threadIdx.x, r = n >> 3, ch = n & 7;
    w[i] = make_uint4(0u, 0u, 0u, 0u);
    if (r0 + r < rows && c0 + ch * kPer < cols) w[i] = __ldg(reinterpret_cast<const uint4*>(src + (r0 + r) * ld + c0 + ch * kPer));
  }
#pragma unroll
  for (int i = 0; i < kLoads; ++i) reinterpret_cast<uint4*>(tile)[i * kThreads + threadIdx.x] = w[i];
  for (int i = threadIdx.x; i < kCols * 4; i += kThreads) reinterpret_cast<uint32_t*>(scale_tile)[i] = 0u;
  __syncthreads();
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;              // rows 32 part .. 32 part + 31 of the tile
  if (r0 + part * 32 < rows) {
    const float g = gain ? *gain : 1.0f;
#pragma unroll
    for (int col = lane; col < kCols; col += 32) {
      const T* mine = tile + part * 32 * kCols + col;
      Sixteen a, b;
      uint32_t pa, pb, sa, sb;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        a.p[k] = make_float2(to_f32(mine[2 * k * kCols]), to_f32(mine[(2 * k + 1) * kCols]));
        b.p[k] = make_float2(to_f32(mine[(16 + 2 * k) * kCols]), to_f32(mine[(17 + 2 * k) * kCols]));
      }
      if (gain) {
        scale16(a, g);
        scale16(b, g);
      }
      pa = peak_of(a);
      pb = peak_of(b);
      if (!kNv) pa = pb = max(pa, pb);
      const uint2 ca = encode16<kNv>(a, pa, sa), cb = encode16<kNv>(b, pb, sb);
      *reinterpret_cast<uint4*>(code_tile + col * kCodePitch + part * 16) = make_uint4(ca.x, ca.y, cb.x, cb.y);
      if (kNv) *reinterpret_cast<uint16_t*>(scale_tile + col * 16 + 2 * part) = static_cast<uint16_t>(sa | (sb << 8));
      else scale_tile[col * 16 + part] = static_cast<uint8_t>(sa);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kCols * 8; i += kThreads) {
    const int col = i >> 3, ch = i & 7;
    if (c0 + col < cols && r0 + ch * 32 < rows)
      *reinterpret_cast<uint4*>(codes + (c0 + col) * (rows / 2) + r0 / 2 + ch * 16) = *reinterpret_cast<const uint4*>(code_tile + col * kCodePitch + ch * 16);
  }
  if (threadIdx.x < kCols && c0 + threadIdx.x < cols) {
    const uint4 word = reinterpret_cast<const uint4*>(scale_tile)[threadIdx.x];
    // a tile is the sixteen blocks of an NVFP4 word, or eight of an MXFP4 word's; the last tile also writes what is past the last block
    const int64_t tile_row = r0 / kTileRows;
    uint8_t* out = scales + ((kNv ? tile_row : tile_row >> 1) * cols + c0 + threadIdx.x) * 16;
    if (kNv || (!(tile_row & 1) && r0 + kTileRows >= rows)) *reinterpret_cast<uint4*>(out) = word;
    else *reinterpret_cast<uint2*>(out + 8 * (tile_row & 1)) = make_uint2(word.x, word.y);
  }
}

// Values m s of E2M1 numbers m, or m s / g, FP32.
template <bool kNv>
__device__ __forceinline__ void decode16(uint2 code, float s, bool scaled, float gain, float (&v)[16]) {
  e2m1_to8(code.x, v);
  e2m1_to8(code.y, v + 8);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    v[k] = __fmul_rn(v[k], s);
    if (scaled) v[k] = __fdiv_rn(v[k], gain);
  }
}

// The eight BF16 magnitudes of a block, as tables of low and high bytes.  Only 1 and 1.5 times a power of two occur among the E2M1
// numbers, so the quotients s / g and 1.5 s / g and steps of their exponents make all of them.
struct Bf16Table { uint32_t low0, low1, high0, high1; };
// The gain with its reciprocal, rounded once: then a quotient within an ulp and one correction from the exact remainder is the
// quotient rounded once (Markstein 1990, theorem on division with a correctly rounded reciprocal).  The first correction here
// makes it that near; `fine`: far enough from both ends of FP32's range that nothing on the way leaves it.
struct Gain { float g, y; bool given, fine; };
__device__ __forceinline__ Gain load_gain(const float* p) {
  Gain k{1.0f, 1.0f, p != nullptr, true};
  if (p) {
    k.g = *p;
    k.y = __frcp_rn(k.g);
    k.fine = fabsf(k.g) > 0x1p-60f && fabsf(k.g) < 0x1p60f;
  }
  return k;
}
__device__ __forceinline__ float quotient(float a, const Gain& k) {
  if (!k.fine || a > 0x1p60f || a < 0x1p-60f) return __fdiv_rn(a, k.g);
  float q = a * k.y;
  q = fmaf(fmaf(-q, k.g, a), k.y, q);
  return fmaf(fmaf(-q, k.g, a), k.y, q);
}
__device__ __forceinline__ bool make_table(float s, const Gain& gain, Bf16Table& t) {
  float d1 = s, d3 = 1.5f * s;
  if (gain.given) {
    if (s > 0x1p125f) return false;                                      // the values leave FP32's range before the division
    d1 = quotient(d1, gain);
    d3 = quotient(d3, gain);
  }
  const uint32_t pair = pack2(d1, d3, __nv_bfloat16());                   // 1 and 1.5
  const uint32_t exponent = (pair >> 7) & 0xFFu, sign = pair & 0x8000u;
  uint32_t w0, w1 = pair, w2, w3;                                        // (0, 0.5), (1, 1.5), (2, 3), (4, 6)
  if (s == 0.0f && d1 == 0.0f) {
    w0 = w1 = w2 = w3 = sign * 0x10001u;
  } else if (d1 != d1) {
    w0 = w1 = w2 = w3 = 0x7FC07FC0u;
  } else {
    if (exponent < 2u || exponent > 250u) return false;                 // steps of the exponent might leave BF16's normal numbers
    w0 = ((pair - 0x80u) << 16) | sign;
    w2 = pair + 0x00800080u;
    w3 = pair + 0x01000100u;
  }
  t.low0 = prmt(w0, w1, 0x6420u); t.low1 = prmt(w2, w3, 0x6420u);
  t.high0 = prmt(w0, w1, 0x7531u); t.high1 = prmt(w2, w3, 0x7531u);
  return true;
}
// Eight codes -> four pairs.
__device__ __forceinline__ void look_up8(uint32_t codes, const Bf16Table& t, uint32_t* out) {
  const uint32_t magnitude = codes & 0x77777777u, sign = (codes >> 3) & 0x11111111u;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t low = prmt(t.low0, t.low1, magnitude >> (16 * h));
    const uint32_t high = prmt(t.high0, t.high1, magnitude >> (16 * h)) ^ prmt(0x00008000u, 0u, sign >> (16 * h));
    out[2 * h] = prmt(low, high, 0x5140u);
    out[2 * h + 1] = prmt(low, high, 0x7362u);
  }
}

__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
               "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void store_words8(void* p, const uint32_t* w, bool wide) {
  if (wide) {
    store32(p, w);
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    static_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// Sixteen codes of a block -> the row.
template <typename T, bool kNv>
__device__ __forceinline__ void store_decoded(T* p, uint2 code, uint32_t byte, const Gain& gain, bool wide) {
  const float s = scale_value<kNv>(byte);
  uint32_t w[16];
  if (sizeof(T) == 2) {
    Bf16Table table;
    if (make_table(s, gain, table)) {
      look_up8(code.x, table, w);
      look_up8(code.y, table, w + 4);
    } else {
      float v[16];
      decode16<kNv>(code, s, gain.given, gain.g, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1], __nv_bfloat16());
    }
    store_words8(p, w, wide);
  } else {
    float v[16];
    decode16<kNv>(code, s, gain.given, gain.g, v);
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(v[i]);
    store_words8(p, w, wide);
    store_words8(p + 8, w + 8, wide);
  }
}

template <typename T, bool kNv>
__global__ void __launch_bounds__(kThreads)
bfp4_dequantize_kernel(const uint4* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, uint32_t n32, uint32_t tasks, Divider words,
                       const float* __restrict__ gain, T* __restrict__ dst, int64_t ld, int wide) {
  const int lane = threadIdx.x & 31;
  const uint32_t warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  grid_wait();
  grid_launch_next();
  if (warp >= tasks) return;
  const WordTask t = word_task<kNv>(warp, words, lane);
  if (t.row >= rows || t.c >= n32) return;
  const uint4 code = codes[t.row * n32 + t.c];
  const uint8_t* scale = scales + scale_offset<kNv>(t, rows, lane);
  const uint32_t bytes = kNv ? *reinterpret_cast<const uint16_t*>(scale) : *scale * 0x101u;
  const Gain k = load_gain(gain);
  T* p = dst + t.row * ld + 32 * static_cast<int64_t>(t.c);
  store_decoded<T, kNv>(p, make_uint2(code.x, code.y), bytes & 0xFFu, k, wide);
  store_decoded<T, kNv>(p + 16, make_uint2(code.z, code.w), bytes >> 8, k, wide);
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
// Warps' tasks of a matrix (HIF4_ERR_SHAPE where they are more than 2^31).
struct Tasks { bool ok; uint32_t n32, count, blocks; Divider words; };
Tasks word_tasks(int64_t rows, int64_t cols, bool nv) {
  const int64_t words = scale_words(cols, nv), lines = ceil_div64(rows, nv ? 4 : 2);
  if (words > 0x7FFFFFFFll / lines) return {false, 0, 0, 0, {}};
  const int64_t count = words * lines;
  return {true, static_cast<uint32_t>(cols / 32), static_cast<uint32_t>(count), static_cast<uint32_t>(ceil_div64(count, kThreads / 32)),
          make_divider(static_cast<uint32_t>(words))};
}
int rows_wide(const void* p, int64_t ld, size_t size) { return (reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld) * size) % 32 == 0; }
template <typename T, bool kNv>
hif4_status quantize_rows(const void* src, int64_t rows, int64_t cols, int64_t ld, const float* gain, void* codes, void* scales, cudaStream_t st) {
  const Tasks t = word_tasks(rows, cols, kNv);
  if (!t.ok) return HIF4_ERR_SHAPE;
  return launch_overlapped(bfp4_quantize_kernel<T, kNv>, t.blocks, kThreads, 0, st, static_cast<const T*>(src), rows, t.n32, t.count, t.words, ld, rows_wide(src, ld, sizeof(T)), gain, static_cast<uint4*>(codes),
                           static_cast<uint8_t*>(scales));
}
template <typename T, bool kNv>
hif4_status quantize_columns(const void* src, int64_t rows, int64_t cols, int64_t ld, const float* gain, void* codes, void* scales, cudaStream_t st) {
  const int64_t row_tiles = ceil_div64(rows, kTileRows), blocks = row_tiles * ceil_div64(cols, kTileCols<T>);
  return launch_overlapped(bfp4_quantize_transposed_kernel<T, kNv>, static_cast<unsigned>(blocks), kThreads, 0, st,
      static_cast<const T*>(src), rows, cols, ld, gain, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), row_tiles);
}
template <typename T, bool kNv>
hif4_status dequantize_rows(const void* codes, const void* scales, int64_t rows, int64_t cols, const float* gain, void* dst, int64_t ld, cudaStream_t st) {
  const Tasks t = word_tasks(rows, cols, kNv);
  if (!t.ok) return HIF4_ERR_SHAPE;
  return launch_overlapped(bfp4_dequantize_kernel<T, kNv>, t.blocks, kThreads, 0, st, static_cast<const uint4*>(codes),
                           static_cast<const uint8_t*>(scales), rows, t.n32, t.count, t.words, gain, static_cast<T*>(dst), ld, rows_wide(dst, ld, sizeof(T)));
}
hif4_status check(const void* src, hif4_dtype dt, int64_t rows, int64_t cols, int64_t ld, hif4_bfp4_format fmt, const float* gain,
                  const void* codes, const void* scales) {
  if (rows < 0 || cols < 0 || ld < cols) return HIF4_ERR_SHAPE;
  if ((dt != HIF4_BF16 && dt != HIF4_FP16 && dt != HIF4_FP32) || !format_ok(fmt)) return HIF4_ERR_DTYPE;
  if (rows == 0 || cols == 0) return HIF4_OK;
  if (cols / 16 + 1 > 0x7FFFFFFFll / (rows / 16 + 1)) return HIF4_ERR_SHAPE;      // more blocks than a grid has
  if (!src || !codes || !scales) return HIF4_ERR_NULL;
  if (!aligned16(src) || (rows > 1 && (static_cast<size_t>(ld) * type_size(dt)) % 16 != 0) || !aligned16(codes) || !aligned16(scales) ||
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
