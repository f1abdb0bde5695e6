// Activations of the linear layers' epilogues and their derivatives, FP32.  An activation is within (8 + 2 |e|) 2^-22 of its
// value, e the exponent in its formula (-z for SiLU, z^2 / 2 for GELU, twice the argument of tanh for its tanh form): the
// rounding of the exponent, which grows with it, and a few units in the last place.  A sigmoid below 2^-126 is zero.
#pragma once
#include "hif4_common.cuh"

namespace hif4 {
namespace {

constexpr float kLog2E = 1.44269504088896341f;               // log2(e)
constexpr float kInvSqrt2Pi = 0.39894228040143268f;          // 1 / sqrt(2 pi)
constexpr float kGeluTanh2 = 1.5957691216057308f;            // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;

// 2^x and 1/x to about two units in the last place (results below 2^-126 are zero).
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 1 / (1 + e^-z): 1 for large z, 0 for small ones (e^-z overflows to infinity there).
__device__ __forceinline__ float sigmoid(float z) { return rcp_fast(1.0f + exp2_fast(-kLog2E * z)); }

// The normal distribution function and its density's exponential e^(-z^2/2).  With a = |z|, Phi(-a) = e^(-a^2/2) R(a) where
// R falls from 1/2 like 1 / (a sqrt(2 pi)), so R / t with t = 1 / (1 + 39/128 a) stays between 0.22 and 0.5 and is a smooth
// function of s = 1 - 2 t.  The polynomial is its minimax fit of degree 7 for a <= 14 (where the exponential is zero), 9.1e-8 of
// the value; every coefficient's size falls, so Horner's rule loses nothing.  The error of Phi is therefore relative in both tails: an
// approximation with an absolute bound (1.5e-7, four terms fewer) left GELU 5e-4 of its value off at z = -4 and 2 % at -10.
__device__ __forceinline__ float normal_cdf(float z, float& density) {
  const float t = rcp_fast(fmaf(0.3046875f, fabsf(z), 1.0f)), s = fmaf(-2.0f, t, 1.0f);
  density = exp2_fast(-0.5f * kLog2E * z * z);
  float y = fmaf(-2.8711059e-4f, s, -3.9197330e-4f);
  y = fmaf(y, s, 2.5145807e-3f);
  y = fmaf(y, s, 8.8245666e-4f);
  y = fmaf(y, s, -2.6012365e-2f);
  y = fmaf(y, s, 8.5283898e-2f);
  y = fmaf(y, s, -1.6545852e-1f);
  y = fmaf(y, s, 2.2498225e-1f);
  y *= t * density;
  return z < 0.0f ? y : 1.0f - y;
}

// act(z).  The tanh form of GELU is z * sigmoid(2 u), because (1 + tanh u) / 2 = sigmoid(2 u).
__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case HIF4_ACT_RELU: return z < 0.0f ? 0.0f : z;                       // NaN passes
    case HIF4_ACT_SILU: return z * sigmoid(z);
    case HIF4_ACT_GELU: {
      float density;
      return z * normal_cdf(z, density);
    }
    case HIF4_ACT_GELU_TANH: return z * sigmoid(kGeluTanh2 * fmaf(kGeluCubic * z * z, z, z));
    default: return z;
  }
}
// act(z) and act'(z).  (The cap keeps 0 * infinity out of the tanh form where the sigmoid is already 0 or 1.)
__device__ __forceinline__ void activate_slope(float z, int act, float& a, float& slope) {
  switch (act) {
    case HIF4_ACT_RELU:
      a = z < 0.0f ? 0.0f : z;
      slope = z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;                      // NaN passes
      return;
    case HIF4_ACT_SILU: {
      const float s = sigmoid(z);
      a = z * s;
      slope = fmaf(a, 1.0f - s, s);
      return;
    }
    case HIF4_ACT_GELU: {
      float density;
      const float phi = normal_cdf(z, density);
      a = z * phi;
      slope = fmaf(z * kInvSqrt2Pi, density, phi);
      return;
    }
    case HIF4_ACT_GELU_TANH: {
      const float z2 = fminf(z * z, 1e8f), s = sigmoid(kGeluTanh2 * fmaf(kGeluCubic * z2, z, z));
      a = z * s;
      slope = fmaf(a * (1.0f - s), kGeluTanh2 * fmaf(3.0f * kGeluCubic, z2, 1.0f), s);
      return;
    }
    default: a = z; slope = 1.0f;
  }
}

}  // namespace
}  // namespace hif4
