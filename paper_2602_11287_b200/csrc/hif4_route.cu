// hif4_route / hif4_route_backward -- which experts a token goes to, with which weights, and the weights' gradient.
//
// A warp routes a token: lane l holds V consecutive experts, so that the lowest lane holds the lowest index and a group of
// experts is a run of lanes.  The best of the warp is one redux over keys (the bits of a choice, made to order like whole
// numbers) and one ballot; only the lane it came from looks through its experts again.
//
// The order is that of the choices in 64 bits: two experts whose choices differ by less than FP32 holds would change
// places from one implementation to the next.  Choices are made in FP32 first, whose error is bounded (below); only where two
// that are neighbours in the order, or a group kept and one left, are nearer than that, the warp starts again in
// 64 bits.  16384 tokens x 256 experts in 8 groups, top 8, FP32: 25 to 27 us (74 us with every choice in 64 bits, 64-bit shuffles and a lane
// per group); 15 us without groups and bias.  Bound by instruction issue, 71 % busy with 1050 warp instructions a token, of which
// 430 stay with one expert chosen; the 16.8 MB of logits would take 2.6 us.  More or fewer tokens a warp change nothing.
#include "hif4_tc_common.cuh"
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

// Numbers as whole numbers of the same order (no NaN; -0 below +0, which no choice is by itself).
template <bool kWide> struct Keys;
template <> struct Keys<false> {
  using Real = float;
  using Key = int;
  static __device__ __forceinline__ Key of(float v) { const int b = __float_as_int(v + 0.0f); return b ^ ((b >> 31) & 0x7FFFFFFF); }
  static __device__ __forceinline__ float value(Key k) { return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)); }
  static __device__ __forceinline__ Key warp_max(Key k) { return __reduce_max_sync(kAll, k); }
};
template <> struct Keys<true> {
  using Real = double;
  using Key = long long;
  static __device__ __forceinline__ Key of(double v) { const long long b = __double_as_longlong(v + 0.0); return b ^ ((b >> 63) & 0x7FFFFFFFFFFFFFFFll); }
  static __device__ __forceinline__ double value(Key k) { return __longlong_as_double(k ^ ((k >> 63) & 0x7FFFFFFFFFFFFFFFll)); }
  static __device__ __forceinline__ Key warp_max(Key k) {
    const int high = __reduce_max_sync(kAll, static_cast<int>(k >> 32));
    const unsigned low = __reduce_max_sync(kAll, static_cast<int>(k >> 32) == high ? static_cast<unsigned>(k) : 0u);
    return (static_cast<long long>(high) << 32) | low;
  }
};

__device__ __forceinline__ float fast_rcp(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float fast_exp2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f;

// Sigmoid of x times e^-m, m = min(0, largest x of the sum): a common factor of all terms of a ratio, so that no ratio of very
// small sigmoids loses its terms.  The reciprocal is off by an ulp at most, half an ulp more than a division, and less than the
// exponential.
__device__ __forceinline__ float sigmoid_scaled(float x, float m) {
  const float t = expf(-fabsf(x));
  return (x > 0.0f ? 1.0f : m == 0.0f ? t : expf(x - m)) * fast_rcp(1.0f + t);
}

struct RouteParams {
  int64_t tokens, ld;
  int experts, top_k, sigmoid, by_logit, groups, per, top_groups, group_best, renormalize, vec;
  float scale;
  const float* bias;
};

// A lane's logits (-inf past the last expert) and biases (-inf for a NaN).
template <typename T, int V>
__device__ __forceinline__ void load_logits(const T* row, const RouteParams& p, int lane, float (&x)[V]) {
  row += lane * V;
  if (p.vec && (lane + 1) * V <= p.experts) {            // 16-byte loads
    constexpr int kWords = static_cast<int>(V * sizeof(T) / 4);
    if constexpr (kWords >= 4 && kWords % 4 == 0) {
      uint32_t w[kWords];
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(row) + i / 4);
        w[i] = q.x; w[i + 1] = q.y; w[i + 2] = q.z; w[i + 3] = q.w;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = to_f32(reinterpret_cast<const T*>(w)[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = lane * V + i < p.experts ? to_f32(row[i]) : -__int_as_float(0x7F800000);
  }
}
template <int V>
__device__ __forceinline__ void load_bias(const RouteParams& p, int lane, float (&b)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float v = p.bias && lane * V + i < p.experts ? p.bias[lane * V + i] : 0.0f;
    b[i] = v == v ? v : -__int_as_float(0x7F800000);
  }
}
template <int V>
__device__ __forceinline__ float largest(const float (&x)[V]) {
  float top = -__int_as_float(0x7F800000);
#pragma unroll
  for (int i = 0; i < V; ++i) top = fmaxf(top, x[i]);
  return Keys<false>::value(Keys<false>::warp_max(Keys<false>::of(top)));
}

// The two largest keys of a lane that `used` (a bit per expert) does not hold, and where they are.
template <typename Key, int V>
__device__ __forceinline__ void best_two(const Key (&c)[V], uint32_t used, Key none, Key& first, int& at, Key& second, int& at2) {
  first = second = none;
  at = at2 = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const Key v = (used >> i) & 1u ? none : c[i];
    if (v > first) { second = first; at2 = at; first = v; at = i; }
    else if (v > second) { second = v; at2 = i; }
  }
}

// The choice of one token from the lane's logits x and biases b; top is the largest logit that is a number.  Lane j gets the j-th
// expert (or -1).  Sets `contested` where neighbours were too near to tell apart.
//
// Errors in FP32: a sigmoid 1 / (1 + e) with e = exp2(-x log2 e): 2^-22 from exp2 and 1.5 |x| 2^-24 from its argument reach the
// result through e / (1 + e)^2 <= 1/4 (and |x| e / (1 + e)^2 < 0.23), 1 + e and the reciprocal add 2^-24 + 2^-23: together below
// 1.1 2^-22, two of them below 2^-20.  A softmax: terms, relative to the largest, 1.21 2^-22, two of them 2.4 2^-22.  Their sum over
// at most 1024 experts: 3.5 2^-22 from the terms (their mean distance from the largest logit, weighted by them, is below 4.5),
// (V + 4) 2^-24 from the additions; it and quotient and products (0.8 2^-22) move the distance of two scores by that part of it: together
// below (32 + V) 2^-24 of the largest.  The bias's addition: 2^-24 of the choice, two of them 2^-23.
// A group's value is off by its terms' errors, however small a sum they leave (one large and positive, one large and negative), and by
// 2^-24 of itself: half the sum of two by 2^-24 of the terms' magnitudes (twice that with the rounding of its bounds) and half of
// `near`, which is two scores' error.  So groups are told apart by bounds of their own, the lowest of those kept against the highest of
// those left.
//
// Neighbours with the same logit and bias are equal in any arithmetic, and in their places by index: BF16 logits have such in
// most rows (16384 tokens x 256 experts in 8 groups without bias: 47 us where they are chosen again, 28 us as here; 264 tokens 10.6, 5.1).
template <bool kWide, typename T, int V>
__device__ __forceinline__ int choose(const T* row, const float (&x)[V], const float (&b)[V], float top, const RouteParams& p, long long* scratch, long long* notes, int lane, bool& contested) {
  using K = Keys<kWide>;
  using Real = typename K::Real;
  using Key = typename K::Key;
  const float kInf = __int_as_float(0x7F800000);
  const Key none = K::of(static_cast<Real>(-kInf));
  Key c[V];
  Real near = 0;                                        // how near two choices may be and still be told apart
  if (p.by_logit) {
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = x[i] > -kInf ? K::of(static_cast<Real>(x[i])) : none;
  } else {
    Real v[V];
    if (p.sigmoid) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        v[i] = kWide ? static_cast<Real>(1.0 / (1.0 + exp(-static_cast<double>(x[i])))) : static_cast<Real>(fast_rcp(1.0f + fast_exp2(-kLog2e * x[i])));
      near = static_cast<Real>(0x1p-20);
    } else {
      Real total = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[i] = x[i] == top ? Real(1) : kWide ? static_cast<Real>(exp(static_cast<double>(x[i]) - static_cast<double>(top))) : static_cast<Real>(fast_exp2(kLog2e * (x[i] - top)));
        if (!(x[i] > -kInf)) v[i] = 0;
        total += v[i];
      }
      total = warp_sum(total);
      const Real inv = total > 0 ? Real(1) / total : Real(0);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = kWide ? (total > 0 ? v[i] / total : v[i]) : v[i] * inv;
      near = static_cast<Real>((32 + V) * 0x1p-24) * inv;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = x[i] > -kInf ? K::of(v[i] + static_cast<Real>(b[i])) : none;
  }
  const auto told_apart = [&](Key high, Key low) {      // (a key of none is far from all others)
    if (p.by_logit || kWide || low == none) return true;
    const Real h = K::value(high), l = K::value(low);
    return h - l > near + static_cast<Real>(0x1p-21) * fmaxf(fabsf(h), fabsf(l));
  };
  // half of the sum of two, whose order is the same: a sum of two finite choices may be none that FP32 holds
  const auto half_sum = [&](Key first, Key second) {
    return p.group_best == 1 ? first : first == none || second == none ? none : K::of(Real(0.5) * K::value(first) + Real(0.5) * K::value(second));
  };
  contested = false;

  // span: lanes of a group, where groups are whole lanes; else as many as there are for each, which share its experts
  const bool grouped = p.top_groups < p.groups, whole = p.per % V == 0 && (p.per / V & (p.per / V - 1)) == 0;
  const int span = whole ? p.per / V : 1 << (__clz(p.groups - 1) - 27);
  Key first, second;
  int at, at2;
  if (!grouped || whole) best_two(c, 0u, none, first, at, second, at2);
  if (grouped) {
    const int own = lane / span;                        // this lane's group
    Key f = none, s = none;
    if (whole) {
      f = first;
      s = second;
    } else {
      Key* mine = reinterpret_cast<Key*>(scratch);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (lane * V + i < p.experts) mine[lane * V + i] = c[i];
      __syncwarp();
      if (own < p.groups) {
        for (int e = lane % span; e < p.per; e += span) {
          const Key v = mine[own * p.per + e];
          s = max(s, min(f, v));
          f = max(f, v);
        }
      }
      __syncwarp();
    }
    for (int o = 1; o < span; o <<= 1) {
      const Key f2 = __shfl_xor_sync(kAll, f, o), s2 = __shfl_xor_sync(kAll, s, o);
      s = max(min(f, f2), max(s, s2));
      f = max(f, f2);
    }
    Key value = half_sum(f, s);
    bool free = own < p.groups;
    if (!free) value = none;
    uint32_t open = 0u;
    for (int n = 0; n < p.top_groups; ++n) {
      const Key best = K::warp_max(free ? value : none);
      const int g = __shfl_sync(kAll, own, __ffs(__ballot_sync(kAll, free && value == best)) - 1);
      open |= 1u << g;
      if (own == g) free = false;
    }
    if constexpr (!kWide) {
      if (!p.by_logit) {                                // (an infinite value is exact, and so is that of a group that has none)
        const bool there = value != none, kept = own < p.groups && !free;
        const float v = K::value(value), terms = 0x1p-23f * fabsf(K::value(f)) + 0x1p-23f * fabsf(K::value(p.group_best == 2 ? s : f));
        const float off = v == kInf ? 0.0f : 0.5f * near + terms;
        const Key highest = K::warp_max(free && there ? K::of(v + off) : none);
        const Key lowest = ~K::warp_max(~K::of(kept && there ? v - off : kInf));
        contested = highest != none && !(lowest > highest);
      }
    }
    if (whole) {
      if (own >= p.groups || !((open >> own) & 1u)) first = second = none;
    } else {
      int g = lane * V / p.per, left = p.per - (lane * V - g * p.per);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!((open >> (g & 31)) & 1u)) c[i] = none;
        if (--left == 0) { ++g; left = p.per; }
      }
      best_two(c, 0u, none, first, at, second, at2);
    }
  }

  // the lane that holds the best notes it as the j-th choice (the lowest lane of equal ones, the lowest index of a lane)
  struct Chosen { Key key; int id; };
  Chosen* chosen = reinterpret_cast<Chosen*>(notes);
  const uint32_t lower = (1u << lane) - 1u;
  Key most = none;
  uint32_t used = 0u;
  bool known = true;                                    // whether `second` is the best that is left besides `first`
  int found = 0;
  for (;; ++found) {                                    // the last round only looks at who would be next
    most = K::warp_max(first);
    if (most == none || found == p.top_k) break;
    const uint32_t holders = __ballot_sync(kAll, first == most);
    if (first == most && !(holders & lower)) {
      chosen[found] = {most, lane * V + at};
      used |= 1u << at;
      if (known) {
        first = second;
        at = at2;
        known = false;
      } else {
        best_two(c, used, none, first, at, second, at2);
        known = true;
      }
    }
    __syncwarp();
  }
  const bool here = lane < found;
  Key mine = none, next = most;
  int id = -1;
  if (here) {
    mine = chosen[lane].key;
    id = chosen[lane].id;
    if (lane + 1 < found) next = chosen[lane + 1].key;
  }
  __syncwarp();
  if (kWide || contested) return id;
  bool doubt = here && !told_apart(mine, next);
  if (__any_sync(kAll, doubt)) {
    const float xs = here ? to_f32(row[id]) : 0.0f, bs = here && p.bias ? p.bias[id] : 0.0f;
    const float xn = __shfl_down_sync(kAll, xs, 1), bn = __shfl_down_sync(kAll, bs, 1);
    const float xl = __shfl_sync(kAll, xs, found - 1), bl = __shfl_sync(kAll, bs, found - 1);
    const Key end = __shfl_sync(kAll, mine, found - 1);
    doubt = doubt && lane + 1 < found && !(xs == xn && bs == bn);
    if (first != none) {                                // of those left, all that are as near to the last have to be its equals
      float again[V];                                   // (held until here, the logits' registers would cost the common path)
      load_logits(row, p, lane, again);
#pragma unroll
      for (int i = 0; i < V; ++i)
        doubt |= !((used >> i) & 1u) && c[i] != none && !(again[i] == xl && b[i] == bl) && !told_apart(end, c[i]);
    }
    contested = __any_sync(kAll, doubt);
  }
  return id;
}

// The choice in 64 bits.  A call of its own: it is rare, and its registers are not the common path's.
template <typename T, int V>
__device__ __noinline__ int choose_wide(const T* row, const RouteParams* p, long long* scratch, long long* notes) {
  const int lane = threadIdx.x & 31;
  float x[V], b[V];
  load_logits(row, *p, lane, x);
  load_bias(*p, lane, b);
  bool contested;
  return choose<true>(row, x, b, largest(x), *p, scratch, notes, lane, contested);
}

// V: experts a lane holds (experts <= 32 V).
template <typename T, int V>
__global__ void __launch_bounds__(kRouteWarps * 32, V <= 8 ? 8 : V == 16 ? 5 : 3)
route_kernel(const T* __restrict__ logits, const __grid_constant__ RouteParams p, int32_t* __restrict__ ids, float* __restrict__ weights) {
  extern __shared__ long long scratch[];                // [warps][experts], where groups are not whole lanes
  __shared__ long long notes[kRouteWarps][2 * HIF4_ROUTE_MAX_TOP_K];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float kInf = __int_as_float(0x7F800000);
  grid_wait();
  grid_launch_next();
  float b[V];
  load_bias(p, lane, b);
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kRouteWarps + warp; t < p.tokens; t += static_cast<int64_t>(gridDim.x) * kRouteWarps) {
    const T* row = logits + t * p.ld;
    float x[V];
    load_logits(row, p, lane, x);
    const float top = p.sigmoid ? 0.0f : largest(x);
    float probe = 0.0f;                                 // NaN where one of the logits is
#pragma unroll
    for (int i = 0; i < V; ++i) probe = max_nan(probe, x[i]);
    const bool bad = __any_sync(kAll, probe != probe) || (!p.sigmoid && top == kInf);

    long long* mine = scratch + static_cast<size_t>(warp) * p.experts;
    bool contested;
    int id = choose<false>(row, x, b, top, p, mine, notes[warp], lane, contested);      // lane j: the j-th choice
    if (contested) id = choose_wide<T, V>(row, &p, mine, notes[warp]);
    const float xc = id >= 0 ? to_f32(row[id]) : -kInf;

    float w = 0.0f;
    const float high = Keys<false>::value(Keys<false>::warp_max(Keys<false>::of(xc)));       // of the chosen
    if (p.sigmoid) {
      const float m = p.renormalize ? fminf(0.0f, high) : 0.0f;
      w = id >= 0 ? sigmoid_scaled(xc, m) : 0.0f;
      if (p.renormalize) {
        const float sum = warp_sum(w);
        w = sum > 0.0f ? w / sum : 0.0f;
      }
    } else if (p.renormalize) {
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
    if (lane < p.top_k) {
      ids[t * p.top_k + lane] = id;
      weights[t * p.top_k + lane] = bad ? __int_as_float(0x7FC00000) : p.scale * w;
    }
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kRouteWarps * 32)
route_backward_kernel(const T* __restrict__ logits, int64_t ld, int64_t tokens, int experts, int top_k, const int32_t* __restrict__ ids,
                      const float* __restrict__ dweights, int sigmoid, int renormalize, float scale, T* __restrict__ dlogits, int64_t ld_d) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kRouteWarps + warp;
  grid_wait();
  grid_launch_next();
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

bool type_ok(int dt) { return dt == HIF4_BF16 || dt == HIF4_FP16 || dt == HIF4_FP32; }
size_t type_size(int dt) { return dt == HIF4_FP32 ? 4 : 2; }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <typename T, int V>
hif4_status launch_route(const hif4_route_args& a, cudaStream_t st) {
  RouteParams p{};
  p.tokens = a.tokens; p.ld = a.ld_logits;
  p.experts = static_cast<int>(a.experts); p.top_k = static_cast<int>(a.top_k);
  p.sigmoid = a.score == HIF4_SCORE_SIGMOID;
  p.groups = static_cast<int>(a.groups); p.per = p.experts / p.groups;
  p.top_groups = static_cast<int>(a.top_groups); p.group_best = static_cast<int>(a.group_best);
  p.by_logit = !a.bias && (p.groups == 1 || p.group_best == 1);
  p.renormalize = a.renormalize != 0;
  p.vec = aligned(a.logits, 16) && a.ld_logits * type_size(a.dt) % 16 == 0 && V * sizeof(T) % 16 == 0;
  p.scale = a.scale;
  p.bias = a.bias;
  const int span = p.per / V;
  const bool scratch = p.top_groups < p.groups && (p.per % V != 0 || (span & (span - 1)) != 0);
  const size_t smem = scratch ? sizeof(long long) * kRouteWarps * p.experts : 0;
  // every warp keeps the biases of its experts over the tokens it routes
  const int64_t most = static_cast<int64_t>(sm_count()) * 16, blocks = ceil_div64(a.tokens, kRouteWarps);
  return launch_overlapped(route_kernel<T, V>, static_cast<unsigned>(blocks < most ? blocks : most), kRouteWarps * 32, smem, st,
                           static_cast<const T*>(a.logits), p, a.ids, a.weights);
}
template <typename T, int V>
hif4_status launch_route_backward(const hif4_route_backward_args& a, cudaStream_t st) {
  const int64_t blocks = ceil_div64(a.tokens, kRouteWarps);
  return launch_overlapped(route_backward_kernel<T, V>, static_cast<unsigned>(blocks), kRouteWarps * 32, 0, st, static_cast<const T*>(a.logits),
                           a.ld_logits, a.tokens, static_cast<int>(a.experts), static_cast<int>(a.top_k), a.ids, a.dweights,
                           static_cast<int>(a.score == HIF4_SCORE_SIGMOID), static_cast<int>(a.renormalize != 0), a.scale,
                           static_cast<T*>(a.dlogits), a.ld_dlogits);
}

#define HIF4_ROUTE_BY_WIDTH(launch, T, a, st)                                                                            \
  (a.experts <= 32 ? launch<T, 1>(a, st) : a.experts <= 64 ? launch<T, 2>(a, st) : a.experts <= 128 ? launch<T, 4>(a, st) \
   : a.experts <= 256 ? launch<T, 8>(a, st) : a.experts <= 512 ? launch<T, 16>(a, st) : launch<T, 32>(a, st))
#define HIF4_ROUTE_BY_TYPE(launch, a, st)                                                                                   \
  (a.dt == HIF4_BF16 ? HIF4_ROUTE_BY_WIDTH(launch, __nv_bfloat16, a, st) : a.dt == HIF4_FP16 ? HIF4_ROUTE_BY_WIDTH(launch, __half, a, st) \
                                                                               : HIF4_ROUTE_BY_WIDTH(launch, float, a, st))


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
