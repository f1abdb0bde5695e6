// Activations of the linear layers' epilogues and their derivatives, FP32.
#pragma once
#include "hif4_common.cuh"

namespace hif4 {
namespace {

constexpr float kSqrtHalf = 0.70710678118654752f;            // sqrt(1/2)
constexpr float kInvSqrt2Pi = 0.39894228040143268f;          // 1 / sqrt(2 pi)
constexpr float kGeluTanh2 = 1.5957691216057308f;            // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;

// 1 / (1 + e^-z): 1 for large z, 0 for small ones (e^-z overflows to infinity there).
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

// act(z).  The tanh form of GELU is z * sigmoid(2 u), because (1 + tanh u) / 2 = sigmoid(2 u).
__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case HIF4_ACT_RELU: return z < 0.0f ? 0.0f : z;                       // NaN passes
    case HIF4_ACT_SILU: return z * sigmoid(z);
    case HIF4_ACT_GELU: return 0.5f * z * erfcf(-z * kSqrtHalf);
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
      const float phi = 0.5f * erfcf(-z * kSqrtHalf);
      a = z * phi;
      slope = fmaf(z * kInvSqrt2Pi, __expf(-0.5f * z * z), phi);
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
