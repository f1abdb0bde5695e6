// MXFP4 and NVFP4 on the device: one block of elements to codes and scale byte, and back.  The steps are those of the
// quantization-error study: FP32, one rounding each.
//   MXFP4  blocks of 32, scale 2^(floor(log2 peak) - 2) as E8M0, elements E2M1 of v / scale
//   NVFP4  blocks of 16, scale E4M3(peak / 6), elements E2M1 of v / scale
// E2M1 rounds to nearest, ties to the even code, saturating at 6; so does the conversion instruction.
#pragma once
#include <cuda_fp16.h>

#include "hif4_vec8.cuh"

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

// Sixteen elements of a matrix row, as pairs.
struct Sixteen { float2 p[8]; };
template <typename T> struct Raw16 { uint32_t w[8 * sizeof(T) / 2]; };
// One 32-byte instruction per lane (two for FP32): a warp's lanes lie side by side, so every sector is touched once.
__device__ __forceinline__ void load32(const void* p, uint32_t* w) {
  asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
__device__ __forceinline__ void load16b(const void* p, uint32_t* w) {
  const uint4 v = __ldg(static_cast<const uint4*>(p));
  w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}
// `wide`: the address is a multiple of 32 bytes.
template <typename T>
__device__ __forceinline__ Raw16<T> load_raw16(const T* p, bool wide) {
  Raw16<T> r;
  constexpr int kParts = static_cast<int>(sizeof(T)) / 2;
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    if (wide) load32(reinterpret_cast<const char*>(p) + 32 * i, r.w + 8 * i);
    else {
      load16b(reinterpret_cast<const char*>(p) + 32 * i, r.w + 8 * i);
      load16b(reinterpret_cast<const char*>(p) + 32 * i + 16, r.w + 8 * i + 4);
    }
  }
  return r;
}
__device__ __forceinline__ Sixteen sixteen_of(const Raw16<__nv_bfloat16>& r) {
  Sixteen v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v.p[i] = make_float2(__uint_as_float(r.w[i] << 16), __uint_as_float(r.w[i] & 0xFFFF0000u));
  return v;
}
__device__ __forceinline__ Sixteen sixteen_of(const Raw16<__half>& r) {
  Sixteen v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v.p[i] = __half22float2(*reinterpret_cast<const __half2*>(&r.w[i]));
  return v;
}
__device__ __forceinline__ Sixteen sixteen_of(const Raw16<float>& r) {
  Sixteen v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v.p[i] = make_float2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1]));
  return v;
}
__device__ __forceinline__ void scale16(Sixteen& v, float gain) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v.p[i] = mul2(v.p[i], both(gain));
}

// Largest magnitude of sixteen elements as FP32 bits (a NaN sorts above infinity): the largest pattern without its sign, and
// patterns order like values.
__device__ __forceinline__ uint32_t peak_of_words(const uint32_t (&w)[8]) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
  return max(m & 0xFFFFu, m >> 16);
}
__device__ __forceinline__ uint32_t peak16(const Raw16<__nv_bfloat16>& r) { return peak_of_words(r.w) << 16; }
__device__ __forceinline__ uint32_t peak16(const Raw16<__half>& r) {
  return __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(peak_of_words(r.w)))));
}
__device__ __forceinline__ uint32_t peak16(const Raw16<float>& r) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = max(m, r.w[i] & 0x7FFFFFFFu);
  return m;
}
__device__ __forceinline__ uint32_t peak_of(const Sixteen& v) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, max(__float_as_uint(v.p[i].x) & 0x7FFFFFFFu, __float_as_uint(v.p[i].y) & 0x7FFFFFFFu));
  return m;
}

constexpr uint32_t kInfBits = 0x7F800000u, kMostBits = 0x7F7FFFFFu;
// A gain multiplied into two runs of sixteen elements with these peaks.  The peak of the products with a finite gain is the product with the
// peak: rounding keeps the order.  An infinite gain makes zeros NaN, which only the products show.
template <bool kNv>
__device__ __forceinline__ void apply_gain(Sixteen& a, Sixteen& b, uint32_t& pa, uint32_t& pb, float gain) {
  scale16(a, gain);
  scale16(b, gain);
  const auto scaled = [gain](uint32_t peak) { return __float_as_uint(fabsf(__fmul_rn(__uint_as_float(peak), gain))); };
  if ((__float_as_uint(gain) & 0x7FFFFFFFu) == kInfBits) {
    pa = peak_of(a);
    pb = peak_of(b);
    if (!kNv) pa = pb = max(pa, pb);
  } else {
    pa = scaled(pa);
    pb = kNv ? scaled(pb) : pa;
  }
}
// a / b by the reciprocal y of b (within 2^-23 of its value) and one correction from the exact remainder: q0 = a y, q = q0 + (a - q0 b) y.
// Before its last rounding q is off by 2^-45 of its value at most.  For b of up to four significant bits (an E4M3 scale, 6) and a of 24 no
// quotient lies that near to the middle between two FP32 numbers: a = m b with an odd 25-bit m would need 26 bits.  So q is a / b
// rounded once, like __fdiv_rn, at a quarter of its instructions.
// The remainder is exact in every rounding; rounded down, a remainder of zero is -0, which leaves the sign of q0 = -0 alone.
__device__ __forceinline__ float2 divide2(float2 a, float2 minus_b, float2 y) {
  const float2 q0 = mul2(a, y);
  float2 r;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rm.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(q0.x), "f"(q0.y), "f"(minus_b.x), "f"(minus_b.y), "f"(a.x), "f"(a.y));
  return fma2(r, y, q0);
}

// Sixteen values of a block whose peak is given -> codes (element i in nibble i) and the block's scale byte.
template <bool kNv>
__device__ __forceinline__ uint2 encode16(Sixteen v, uint32_t peak, uint32_t& byte) {
  if (peak > kInfBits) {
    byte = kNv ? 0x7Fu : 0xFFu;
    return make_uint2(0u, 0u);
  }
  float q[16];
  if (kNv) {
    if (peak == kInfBits) {                              // saturates as the largest number does
      peak = kMostBits;
      const float most = __uint_as_float(kMostBits);
#pragma unroll
      for (int i = 0; i < 8; ++i) v.p[i] = make_float2(fminf(fmaxf(v.p[i].x, -most), most), fminf(fmaxf(v.p[i].y, -most), most));
    }
    const float p = __uint_as_float(peak), p6 = p * (1.0f / 6.0f);
    byte = e4m3_of(fmaf(fmaf(p6, -6.0f, p), 1.0f / 6.0f, p6));
    const float s = e4m3_value(byte);
    float rcp;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rcp) : "f"(s));
    const float2 y = both(byte ? rcp : 0.0f), minus_s = both(-s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 d = divide2(v.p[i], minus_s, y);
      q[2 * i] = d.x;
      q[2 * i + 1] = d.y;
    }
  } else {
    const int e = max(static_cast<int>(peak >> 23) - 127 - 2, -127);     // floor(log2 peak) - 2; infinity: 126
    byte = peak ? static_cast<uint32_t>(e + 127) : 0u;
    const float2 inv = both(__uint_as_float(static_cast<uint32_t>(127 - e) << 23));      // the division by a power of two is exact
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 d = mul2(v.p[i], inv);
      q[2 * i] = d.x;
      q[2 * i + 1] = d.y;
    }
  }
  return make_uint2(e2m1_of8(q), e2m1_of8(q + 8));
}

// Item and block numbers as row and column: division by a number known at launch (Granlund and Montgomery's multiplication by a
// rounded-up reciprocal; exact for dividends below 2^31).
struct Divider {
  uint32_t d, mul, shift;
  __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return d == 1u ? n : __umulhi(n, mul) >> shift; }
};
inline Divider make_divider(uint32_t d) {
  Divider r{d, 0u, 0u};
  if (d <= 1u) return r;
  uint32_t log = 0;
  while ((1ull << log) < d) ++log;
  r.shift = log - 1;
  r.mul = static_cast<uint32_t>(((1ull << (31 + log)) + d - 1) / d);
  return r;
}

// Scales of a matrix: [words][rows][16 bytes].
__host__ __device__ inline int64_t scale_words(int64_t cols, bool nv) { return ceil_div64(cols, nv ? 256 : 512); }
}  // namespace
}  // namespace hif4
