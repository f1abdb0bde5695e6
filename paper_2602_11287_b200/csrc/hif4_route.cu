// hif4_route / hif4_route_backward -- which experts a token goes to, with which weights, and the weights' gradient.
//
// A warp holds the scores of one token: lane l has the experts l, l + 32, ...  The choice is an order, so it is made in
// 64 bits: two experts whose choices differ by less than FP32 holds would otherwise change places from one
// implementation to the next.  Weights and gradients are FP32.
#include "hif4_common.cuh"
#include "hif4_vec8.cuh"

namespace hif4 {
namespace {

constexpr int kRouteWarps = 4;
constexpr uint32_t kAll = 0xFFFFFFFFu;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
// Largest value of the warp and its place; of equal ones the lowest place.
__device__ __forceinline__ void warp_best(double& v, int& at) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const double w = __shfl_xor_sync(kAll, v, o);
    const int b = __shfl_xor_sync(kAll, at, o);
    if (w > v || (w == v && b < at)) { v = w; at = b; }
  }
}

// Sigmoid of x times e^-m, m = min(0, largest x of the sum): a common factor of all terms of a ratio, so that no ratio of very
// small sigmoids loses its terms.
__device__ __forceinline__ float sigmoid_scaled(float x, float m) {
  return x > 0.0f ? 1.0f / (1.0f + expf(-x)) : expf(x - m) / (1.0f + expf(x));
}

// V: experts a lane holds (experts <= 32 V).
template <typename T, int V>
__global__ void __launch_bounds__(kRouteWarps * 32)
route_kernel(const T* __restrict__ logits, int64_t ld, int64_t tokens, int experts, int top_k, const float* __restrict__ bias,
             int sigmoid, int groups, int top_groups, int group_best, int renormalize, float scale, int32_t* __restrict__ ids,
             float* __restrict__ weights) {
  extern __shared__ double choices[];                   // [warps][groups][experts / groups + 1], with more than one group
  const double kNone = -__longlong_as_double(0x7FF0000000000000ll);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kRouteWarps + warp;
  if (t >= tokens) return;
  const T* row = logits + t * ld;
  const float kInf = __int_as_float(0x7F800000);
  float x[V];
  float top = -kInf;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = i * 32 + lane;
    x[i] = e < experts ? to_f32(row[e]) : -kInf;
    bad |= x[i] != x[i];
    top = fmaxf(top, x[i]);
  }
  top = warp_max(top);
  bad = __any_sync(kAll, bad) || (!sigmoid && top == kInf);

  // choices in 64 bits
  const bool by_logit = !bias && (groups == 1 || group_best == 1);
  double c[V];
  if (by_logit) {
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = x[i] != x[i] ? kNone : static_cast<double>(x[i]);
  } else {
    double total = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (sigmoid) {
        c[i] = 1.0 / (1.0 + exp(-static_cast<double>(x[i])));
      } else {
        c[i] = x[i] == top ? 1.0 : x[i] != x[i] ? 0.0 : exp(static_cast<double>(x[i]) - static_cast<double>(top));
        if (top == -kInf) c[i] = 0.0;
        total += c[i];
      }
    }
    if (!sigmoid) total = warp_sum(total);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = i * 32 + lane;
      if (!sigmoid && total > 0.0) c[i] /= total;
      if (bias && e < experts) c[i] += static_cast<double>(bias[e]);
      if (e >= experts || x[i] == -kInf || !(c[i] >= kNone) || x[i] != x[i]) c[i] = kNone;
    }
  }

  if (groups > 1) {
    const int per = experts / groups;
    double* mine = choices + static_cast<size_t>(warp) * groups * (per + 1);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = i * 32 + lane;
      if (e < experts) mine[e + e / per] = c[i];
    }
    __syncwarp();
    double value = kNone;
    if (lane < groups) {
      double first = kNone, second = kNone;
      for (int e = 0; e < per; ++e) {
        const double v = mine[lane * (per + 1) + e];
        if (v > first) { second = first; first = v; }
        else if (v > second) second = v;
      }
      value = group_best == 2 ? first + second : first;
      if (!(value >= kNone)) value = kNone;
    }
    uint32_t open = 0u;
    for (int n = 0; n < top_groups; ++n) {
      double v = value;
      int at = lane < groups && !((open >> lane) & 1u) ? lane : 64;
      if (at == 64) v = kNone;
      warp_best(v, at);
      open |= 1u << (at & 31);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = i * 32 + lane;
      if (e < experts && !((open >> (e / per)) & 1u)) c[i] = kNone;
    }
  }

  int id = -1;                                          // lane j: the j-th choice and its logit
  float xc = -kInf;
  for (int j = 0; j < top_k; ++j) {
    double v = kNone;
    int at = 1 << 30;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (c[i] > v) { v = c[i]; at = i * 32 + lane; }
    warp_best(v, at);
    if (v == kNone) break;
    float xv = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (at == i * 32 + lane) { c[i] = kNone; xv = x[i]; }
    xv = __shfl_sync(kAll, xv, at & 31);
    if (lane == j) { id = at; xc = xv; }
  }

  float w = 0.0f;
  const float high = warp_max(xc);                      // of the chosen
  if (sigmoid) {
    const float m = renormalize ? fminf(0.0f, high) : 0.0f;
    w = id >= 0 ? sigmoid_scaled(xc, m) : 0.0f;
    if (renormalize) {
      const float sum = warp_sum(w);
      w = sum > 0.0f ? w / sum : 0.0f;
    }
  } else if (renormalize) {
    w = id >= 0 ? expf(xc - high) : 0.0f;
    const float sum = warp_sum(w);
    w = sum > 0.0f ? w / sum : 0.0f;
  } else {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) sum += expf(x[i] - top);
    sum = warp_sum(sum);
    w = id >= 0 ? expf(xc - top) / sum : 0.0f;
  }
  if (lane < top_k) {
    ids[t * top_k + lane] = id;
    weights[t * top_k + lane] = bad ? __int_as_float(0x7FC00000) : scale * w;
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kRouteWarps * 32)
route_backward_kernel(const T* __restrict__ logits, int64_t ld, int64_t tokens, int experts, int top_k, const int32_t* __restrict__ ids,
                      const float* __restrict__ dweights, int sigmoid, int renormalize, float scale, T* __restrict__ dlogits, int64_t ld_d) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kRouteWarps + warp;
  if (t >= tokens) return;
  const float kInf = __int_as_float(0x7F800000);
  const T* row = logits + t * ld;
  int id = -1;
  float g = 0.0f, xc = -kInf;
  if (lane < top_k) {
    id = ids[t * top_k + lane];
    if (id < 0 || id >= experts) id = -1;
    if (id >= 0) { g = scale * dweights[t * top_k + lane]; xc = to_f32(row[id]); }
  }
  float d[V];                                           // first ds (or, where only the chosen matter, the result), per expert
#pragma unroll
  for (int i = 0; i < V; ++i) d[i] = 0.0f;
  float mine;                                           // lane j: what assignment j gives to its expert
  const float high = warp_max(xc);
  if (renormalize) {
    // shares v of the chosen: dx = v (g - sum g v), times 1 - s for a sigmoid
    float v = id < 0 ? 0.0f : sigmoid ? sigmoid_scaled(xc, fminf(0.0f, high)) : expf(xc - high);
    const float sum = warp_sum(v);
    v = sum > 0.0f ? v / sum : 0.0f;
    mine = v * (g - warp_sum(id < 0 ? 0.0f : g * v));
    if (sigmoid) mine *= 1.0f / (1.0f + expf(xc));
  } else if (sigmoid) {
    mine = g * sigmoid_scaled(xc, 0.0f) * (1.0f / (1.0f + expf(xc)));
  } else {
    mine = g;
  }
  for (int j = 0; j < top_k; ++j) {
    const int at = __shfl_sync(kAll, id, j);
    const float v = __shfl_sync(kAll, mine, j);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (at == i * 32 + lane) d[i] += v;
  }
  if (!renormalize && !sigmoid) {
    float x[V];
    float top = -kInf;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = i * 32 + lane;
      x[i] = e < experts ? to_f32(row[e]) : -kInf;
      top = fmaxf(top, x[i]);
    }
    top = warp_max(top);
    float sum = 0.0f, dot = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[i] = top == -kInf ? 0.0f : expf(x[i] - top);
      sum += x[i];
      dot += x[i] * d[i];
    }
    sum = warp_sum(sum);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    dot = warp_sum(dot) * inv;
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = x[i] * inv * (d[i] - dot);
  }
  T* out = dlogits + t * ld_d;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = i * 32 + lane;
    if (e < experts) out[e] = from_f32<T>(d[i]);
  }
}

template <typename T, int V>
hif4_status launch_route(const hif4_route_args& a, cudaStream_t st) {
  const int64_t blocks = ceil_div64(a.tokens, kRouteWarps);
  const int groups = static_cast<int>(a.groups), experts = static_cast<int>(a.experts);
  const size_t smem = groups > 1 ? sizeof(double) * kRouteWarps * (experts + groups) : 0;
  route_kernel<T, V><<<static_cast<unsigned>(blocks), kRouteWarps * 32, smem, st>>>(
      static_cast<const T*>(a.logits), a.ld_logits, a.tokens, experts, static_cast<int>(a.top_k), a.bias, a.score == HIF4_SCORE_SIGMOID,
      groups, static_cast<int>(a.top_groups), static_cast<int>(a.group_best), a.renormalize != 0, a.scale, a.ids, a.weights);
  note_launch();
  return launch_status();
}
template <typename T, int V>
hif4_status launch_route_backward(const hif4_route_backward_args& a, cudaStream_t st) {
  const int64_t blocks = ceil_div64(a.tokens, kRouteWarps);
  route_backward_kernel<T, V><<<static_cast<unsigned>(blocks), kRouteWarps * 32, 0, st>>>(
      static_cast<const T*>(a.logits), a.ld_logits, a.tokens, static_cast<int>(a.experts), static_cast<int>(a.top_k), a.ids, a.dweights,
      a.score == HIF4_SCORE_SIGMOID, a.renormalize != 0, a.scale, static_cast<T*>(a.dlogits), a.ld_dlogits);
  note_launch();
  return launch_status();
}

#define HIF4_ROUTE_BY_WIDTH(launch, T, a, st)                                                                            \
  (a.experts <= 32 ? launch<T, 1>(a, st) : a.experts <= 64 ? launch<T, 2>(a, st) : a.experts <= 128 ? launch<T, 4>(a, st) \
   : a.experts <= 256 ? launch<T, 8>(a, st) : a.experts <= 512 ? launch<T, 16>(a, st) : launch<T, 32>(a, st))
#define HIF4_ROUTE_BY_TYPE(launch, a, st)                                                                                   \
  (a.dt == HIF4_BF16 ? HIF4_ROUTE_BY_WIDTH(launch, __nv_bfloat16, a, st) : a.dt == HIF4_FP16 ? HIF4_ROUTE_BY_WIDTH(launch, __half, a, st) \
                                                                               : HIF4_ROUTE_BY_WIDTH(launch, float, a, st))

bool type_ok(int dt) { return dt == HIF4_BF16 || dt == HIF4_FP16 || dt == HIF4_FP32; }
size_t type_size(int dt) { return dt == HIF4_FP32 ? 4 : 2; }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// What both directions ask of their sizes and types.
hif4_status check_router(int64_t tokens, int64_t experts, int64_t top_k, int64_t ld, int dt, int score) {
  if (tokens < 0 || experts < 1 || top_k < 1 || top_k > experts || ld < experts) return HIF4_ERR_SHAPE;
  if (!type_ok(dt) || (score != HIF4_SCORE_SOFTMAX && score != HIF4_SCORE_SIGMOID)) return HIF4_ERR_DTYPE;
  if (experts > HIF4_ROUTE_MAX_EXPERTS || top_k > HIF4_ROUTE_MAX_TOP_K) return HIF4_ERR_UNSUPPORTED;
  if (ceil_div64(tokens, kRouteWarps) > 0x7FFFFFFFll) return HIF4_ERR_SHAPE;
  return HIF4_OK;
}

}  // namespace
}  // namespace hif4

using namespace hif4;

extern "C" hif4_status hif4_route(const hif4_route_args* args, void* stream) {
  if (!args) return HIF4_ERR_NULL;
  const hif4_route_args& a = *args;
  const hif4_status s = check_router(a.tokens, a.experts, a.top_k, a.ld_logits, a.dt, a.score);
  if (s != HIF4_OK) return s;
  if (a.groups < 1 || a.experts % a.groups != 0 || a.top_groups < 1 || a.top_groups > a.groups || a.group_best < 1 || a.group_best > 2 ||
      a.group_best > a.experts / a.groups || a.top_k > a.top_groups * (a.experts / a.groups))
    return HIF4_ERR_SHAPE;
  if (a.groups > HIF4_ROUTE_MAX_GROUPS) return HIF4_ERR_UNSUPPORTED;
  if (a.tokens == 0) return HIF4_OK;
  if (!a.logits || !a.ids || !a.weights) return HIF4_ERR_NULL;
  if (!aligned(a.logits, type_size(a.dt)) || !aligned(a.bias, 4) || !aligned(a.ids, 4) || !aligned(a.weights, 4)) return HIF4_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return HIF4_ROUTE_BY_TYPE(launch_route, a, st);
}

extern "C" hif4_status hif4_route_backward(const hif4_route_backward_args* args, void* stream) {
  if (!args) return HIF4_ERR_NULL;
  const hif4_route_backward_args& a = *args;
  const hif4_status s = check_router(a.tokens, a.experts, a.top_k, a.ld_logits, a.dt, a.score);
  if (s != HIF4_OK) return s;
  if (a.ld_dlogits < a.experts) return HIF4_ERR_SHAPE;
  if (a.tokens == 0) return HIF4_OK;
  if (!a.logits || !a.ids || !a.dweights || !a.dlogits) return HIF4_ERR_NULL;
  if (!aligned(a.logits, type_size(a.dt)) || !aligned(a.ids, 4) || !aligned(a.dweights, 4) || !aligned(a.dlogits, type_size(a.dt)))
    return HIF4_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return HIF4_ROUTE_BY_TYPE(launch_route_backward, a, st);
}
