// Groups of eight consecutive elements of a BF16, FP16 or FP32 matrix as FP32 registers: the unit in which the
// element-wise kernels load, compute and store (one level-2 group of a HiF4 unit), and the conversion of eight
// neighbouring lanes' groups to one HiF4 unit.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hif4_common.cuh"
#include "hif4_quantize_device.cuh"

namespace hif4 {
namespace {

template <typename T> struct Raw8 { uint4 a; };              // eight 16-bit elements as loaded
template <> struct Raw8<float> { uint4 a, b; };

template <typename T> struct IsHalf { static constexpr bool value = false; };
template <> struct IsHalf<__half> { static constexpr bool value = true; };

__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(float v) { return v; }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }

// What a rounded part leaves of v: zero where the part is infinite or NaN, which it then stands for by itself.
__device__ __forceinline__ float rest_of(float v, float part) { return fabsf(part) < __int_as_float(0x7F800000) ? v - part : 0.0f; }

__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16>& r, float (&v)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack8(const Raw8<__half>& r, float (&v)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    v[2 * i] = f.x; v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&v)[8]) {
  v[0] = __uint_as_float(r.a.x); v[1] = __uint_as_float(r.a.y); v[2] = __uint_as_float(r.a.z); v[3] = __uint_as_float(r.a.w);
  v[4] = __uint_as_float(r.b.x); v[5] = __uint_as_float(r.b.y); v[6] = __uint_as_float(r.b.z); v[7] = __uint_as_float(r.b.w);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half) {
  const __half2 p = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}
template <typename T>
__device__ __forceinline__ Raw8<T> pack8(const float (&v)[8]) {
  Raw8<T> r;
  r.a = make_uint4(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()), pack2(v[4], v[5], T()), pack2(v[6], v[7], T()));
  return r;
}
template <>
__device__ __forceinline__ Raw8<float> pack8<float>(const float (&v)[8]) {
  Raw8<float> r;
  r.a = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  r.b = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
  return r;
}
template <typename T>
__device__ __forceinline__ void zero8(Raw8<T>& r) { r.a = make_uint4(0u, 0u, 0u, 0u); }
__device__ __forceinline__ void zero8(Raw8<float>& r) { r.a = r.b = make_uint4(0u, 0u, 0u, 0u); }

template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
  Raw8<T> r;
  r.a = *reinterpret_cast<const uint4*>(p);
  return r;
}
__device__ __forceinline__ Raw8<float> load8(const float* p) {
  Raw8<float> r;
  r.a = *reinterpret_cast<const uint4*>(p);
  r.b = *reinterpret_cast<const uint4*>(p + 4);
  return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const Raw8<T>& r) { *reinterpret_cast<uint4*>(p) = r.a; }
__device__ __forceinline__ void store8(float* p, const Raw8<float>& r) {
  *reinterpret_cast<uint4*>(p) = r.a;
  *reinterpret_cast<uint4*>(p + 4) = r.b;
}

// Two FP32 operations in one instruction (sm_100 issues packed FP32 arithmetic at the rate of scalar instructions).
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// A group as four pairs.
struct Pairs { float2 p[4]; };
template <typename T>
__device__ __forceinline__ Pairs pairs_of(const Raw8<T>& r) {
  float v[8];
  unpack8(r, v);
  Pairs g;
#pragma unroll
  for (int i = 0; i < 4; ++i) g.p[i] = make_float2(v[2 * i], v[2 * i + 1]);
  return g;
}
template <typename T>
__device__ __forceinline__ Raw8<T> raw_of(const Pairs& g) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = g.p[i].x; v[2 * i + 1] = g.p[i].y; }
  return pack8<T>(v);
}
__device__ __forceinline__ Pairs pairs_filled(float v) {
  Pairs g;
#pragma unroll
  for (int i = 0; i < 4; ++i) g.p[i] = both(v);
  return g;
}

// Eight consecutive lanes (lane & 7 = level-2 group g of the unit) hold one unit: Algorithm 1 in BF16 arithmetic for
// BF16 groups, in FP32 arithmetic for FP16 and FP32 groups, i.e. the bits that hif4_quantize writes for a matrix of
// that type.  Returns the lane's code word; `meta` is the unit's metadata word in all eight lanes.  All 32 lanes call.
template <bool kRHA>
__device__ __forceinline__ uint32_t encode_unit_octet(const Raw8<__nv_bfloat16>& r, int g, uint32_t& meta) {
  constexpr uint32_t kAbs = 0x7FFF7FFFu;
  uint32_t vm = hmax_halves(umax2(umax2(r.a.x & kAbs, r.a.y & kAbs), umax2(r.a.z & kAbs, r.a.w & kAbs)));
#pragma unroll
  for (int s = 1; s < 8; s <<= 1) vm = max(vm, __shfl_xor_sync(0xFFFFFFFFu, vm, s));
  const uint32_t sf = mul_bf16x2(vm, 0x3E12u) & 0xFFFFu;             // Vmax * (1/7)_BF16
  const uint32_t byte = e6m2_from_bits<7, kRHA>(sf);
  const uint32_t lut = prmt(0x122B4D80u, 0u, (byte & 3u) | 0x4440u);
  const uint32_t rec2 = (lut + 0x5700u - ((byte & 0xFCu) << 5)) * 0x10001u;
  uint32_t e8, e16a, e16b;
  const uint32_t code = encode_group_bf16<kRHA>(r.a.x, r.a.y, r.a.z, r.a.w, rec2, e8, e16a, e16b);
  uint32_t m = (e8 << (8 + g)) | ((e16a + 2u * e16b) << (16 + 2 * g));
#pragma unroll
  for (int s = 1; s < 8; s <<= 1) m |= __shfl_xor_sync(0xFFFFFFFFu, m, s);
  const bool unit_nan = vm > 0x7F80u;
  meta = unit_nan ? 0xFFu : m | byte;
  return unit_nan ? 0u : code;
}
template <bool kRHA>
__device__ __forceinline__ uint32_t encode_unit_octet_fp32(const float (&v)[8], int g, uint32_t& meta) {
  uint32_t xb[8], vm = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) { xb[e] = __float_as_uint(v[e]); vm = max(vm, xb[e] & 0x7FFFFFFFu); }
#pragma unroll
  for (int s = 1; s < 8; s <<= 1) vm = max(vm, __shfl_xor_sync(0xFFFFFFFFu, vm, s));
  const float sf = __fmul_rn(__uint_as_float(vm), __uint_as_float(0x3E124925u));   // (1/7)_FP32
  const uint32_t byte = e6m2_from_bits<23, kRHA>(__float_as_uint(sf));
  const uint32_t M = byte & 3u;
  const uint32_t lut = M == 0 ? 0x3F800000u : M == 1 ? 0x3F4CCCCDu : M == 2 ? 0x3F2AAAABu : 0x3F124925u;   // 1, 0.8, 2/3, 4/7
  const float rec = __uint_as_float(lut + (48u << 23) - ((byte >> 2) << 23));
  const uint32_t xa[4] = {xb[0], xb[1], xb[2], xb[3]}, xc[4] = {xb[4], xb[5], xb[6], xb[7]};
  float ta[4], tb[4];
  uint32_t pa = 0u, pb = 0u;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    ta[e] = __fmul_rn(fabsf(v[e]), rec);
    tb[e] = __fmul_rn(fabsf(v[4 + e]), rec);
    pa = max(pa, __float_as_uint(ta[e]));
    pb = max(pb, __float_as_uint(tb[e]));
  }
  const uint32_t e8 = max(pa, pb) >= 0x40800000u;                      // >= 4.0
  uint32_t e16a, e16b;
  const uint32_t lo = encode_group_fp32<kRHA>(xa, ta, pa, e8, e16a), hi = encode_group_fp32<kRHA>(xc, tb, pb, e8, e16b);
  uint32_t m = (e8 << (8 + g)) | ((e16a + 2u * e16b) << (16 + 2 * g));
#pragma unroll
  for (int s = 1; s < 8; s <<= 1) m |= __shfl_xor_sync(0xFFFFFFFFu, m, s);
  const bool unit_nan = vm > 0x7F800000u;
  meta = unit_nan ? 0xFFu : m | byte;
  return unit_nan ? 0u : (lo | (hi << 16));
}
template <bool kRHA>
__device__ __forceinline__ uint32_t encode_unit_octet(const Raw8<__half>& r, int g, uint32_t& meta) {
  float v[8];
  unpack8(r, v);
  return encode_unit_octet_fp32<kRHA>(v, g, meta);
}
template <bool kRHA>
__device__ __forceinline__ uint32_t encode_unit_octet(const Raw8<float>& r, int g, uint32_t& meta) {
  float v[8];
  unpack8(r, v);
  return encode_unit_octet_fp32<kRHA>(v, g, meta);
}

}  // namespace
}  // namespace hif4
