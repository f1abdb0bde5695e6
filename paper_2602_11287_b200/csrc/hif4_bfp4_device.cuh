// MXFP4 and NVFP4 on the device: one block of elements to codes and scale byte, and back.  The steps are those of the
// quantization-error study: FP32, one rounding each.
//   MXFP4  blocks of 32, scale 2^(floor(log2 peak) - 2) as E8M0, elements E2M1 of v / scale
//   NVFP4  blocks of 16, scale E4M3(peak / 6), elements E2M1 of v / scale
// E2M1 rounds to nearest, ties to the even code, saturating at 6; so does the conversion instruction.
#pragma once
#include <cuda_fp16.h>

#include "hif4_common.cuh"

namespace hif4 {
namespace {

// Eight values -> eight E2M1 codes, element i in bits 4i .. 4i + 3.
__device__ __forceinline__ uint32_t e2m1_of8(const float* v) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// Eight E2M1 codes -> values.
__device__ __forceinline__ void e2m1_to8(uint32_t codes, float* v) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint32_t e4m3_of(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(v));
  return r & 0xFFu;
}
// Value of a scale byte that is not NaN.
__device__ __forceinline__ float e4m3_value(uint32_t byte) {           // the bits as an FP32 number 2^120 too small, subnormals too
  return __uint_as_float(byte << 20) * __uint_as_float(247u << 23);
}
__device__ __forceinline__ float e8m0_value(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }
template <bool kNv> __device__ __forceinline__ float scale_value(uint32_t byte) {
  if (byte == (kNv ? 0x7Fu : 0xFFu)) return __int_as_float(0x7FC00000);
  return kNv ? e4m3_value(byte) : e8m0_value(byte);
}

// Largest |v| of sixteen values as a bit pattern (a NaN sorts above infinity).
__device__ __forceinline__ uint32_t peak16(const float (&v)[16]) {
  uint32_t p = 0u;
#pragma unroll
  for (int i = 0; i < 16; ++i) p = max(p, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return p;
}
// Sixteen values of a block whose peak is given -> codes (element i in nibble i) and the block's scale byte.
template <bool kNv>
__device__ __forceinline__ uint2 encode16(const float (&v)[16], uint32_t peak, uint32_t& byte) {
  if (peak > 0x7F800000u) {
    byte = kNv ? 0x7Fu : 0xFFu;
    return make_uint2(0u, 0u);
  }
  float q[16];
  if (kNv) {
    byte = e4m3_of(__fdiv_rn(__uint_as_float(peak), 6.0f));
    const float s = e4m3_value(byte);
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = byte ? __fdiv_rn(v[i], s) : __uint_as_float(__float_as_uint(v[i]) & 0x80000000u);
  } else {
    const int e = max(static_cast<int>(peak >> 23) - 127 - 2, -127);     // floor(log2 peak) - 2; infinity: 126
    byte = peak ? static_cast<uint32_t>(e + 127) : 0u;
    const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);      // the division by a power of two is exact
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = __fmul_rn(v[i], inv);
  }
  return make_uint2(e2m1_of8(q), e2m1_of8(q + 8));
}

// Scales of a matrix: [words][rows][16 bytes].
template <bool kNv> constexpr int kScaleSpan = kNv ? 256 : 512;          // elements of a row that a 16-byte word covers
__host__ __device__ inline int64_t scale_words(int64_t cols, bool nv) { return ceil_div64(cols, nv ? 256 : 512); }
__device__ __forceinline__ int64_t scale_at(int64_t row, int64_t block, int64_t rows) {
  return ((block >> 4) * rows + row) * 16 + (block & 15);
}

}  // namespace
}  // namespace hif4
