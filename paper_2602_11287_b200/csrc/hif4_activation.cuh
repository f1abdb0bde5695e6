// Activations of the linear layers' epilogues and their derivatives, FP32.
#pragma once
#include "hif4_common.cuh"

namespace hif4 {
namespace {

constexpr float kLog2E = 1.44269504088896341f;               // log2(e)
constexpr float kSqrtHalf = 0.70710678118654752f;            // sqrt(1/2)
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

// The normal distribution function and its density's exponential e^(-z^2/2).  Abramowitz and Stegun, Handbook of
// Mathematical Functions, 7.1.26: erfc(x) = (a1 t + ... + a5 t^5) e^(-x^2) with t = 1 / (1 + p x), x >= 0, within 1.5e-7
// (half of that here); a third of the instructions of erfcf, which an epilogue of 256 columns feels.
__device__ __forceinline__ float normal_cdf(float z, float& density) {
  const float x = fabsf(z) * kSqrtHalf;
  const float t = rcp_fast(fmaf(0.3275911f, x, 1.0f));
  density = exp2_fast(-0.5f * kLog2E * z * z);
  float y = fmaf(1.061405429f, t, -1.453152027f);
  y = fmaf(y, t, 1.421413741f);
  y = fmaf(y, t, -0.284496736f);
  y = fmaf(y, t, 0.254829592f);
  y *= 0.5f * t * density;
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
