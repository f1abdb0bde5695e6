// The block norms for many long rows whose matrices are 16-byte aligned: a ring of shared-memory stages that one thread
// fills rows ahead with bulk copies, weights staged in shared memory once per block, and row loops without per-group
// conditions.  (Included by hif4_block_norm.cu inside its namespace.)
//
// What bounds these kernels besides the traffic is the latency of a warp's instruction stream, about six cycles an instruction at the
// 16 to 32 warps that registers allow, and of the block-wide sums in it (two or three a row one after another: the gradient with post
// norm and gates issues in 41 % of the cycles, the forward pass in 57 %).  So threads past the row's end compute on column 0 and are kept out of sums and
// stores only, absent weights are staged as ones, the stage is refilled behind the first sum's barrier, and pointers
// advance by rows.  W: type of the weights, T or FP32.

__device__ __forceinline__ void bulk_row(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// Ring of stages of `kMats` rows each (absent matrices take no room); one mbarrier per stage, since a block barrier
// separates the reads of a stage from its refill by thread 0.
template <typename T, int kMats>
struct RowRing {
  const T* mat[kMats];
  int64_t ld[kMats];
  uint32_t bars, base, row_bytes, stage_bytes, offset[kMats], cur, phase;
  int stages, stage;
  int64_t next, row1;                      // next row to fetch (thread 0)
  __device__ __forceinline__ void start(uint32_t smem, int n_stages, int cols, int64_t row0, int64_t end) {
    row_bytes = static_cast<uint32_t>(cols) * sizeof(T);
    uint32_t mats = 0;
#pragma unroll
    for (int m = 0; m < kMats; ++m) {
      offset[m] = mats * row_bytes;
      mats += mat[m] != nullptr;
    }
    stages = n_stages;
    stage_bytes = mats * row_bytes;
    bars = smem;
    base = cur = smem + 128;
    stage = 0;
    phase = 0;
    next = row0;
    row1 = end;
#pragma unroll
    for (int m = 0; m < kMats; ++m)
      if (mat[m]) mat[m] += row0 * ld[m];
    if (threadIdx.x == 0) {
      for (int s = 0; s < stages; ++s) mbar_init(bars + 8 * s, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (threadIdx.x == 0)
      for (int s = 0; s < stages && next < row1; ++s) fill(s);
  }
  __device__ __forceinline__ void fill(int s) {
    mbar_expect_tx(bars + 8 * s, stage_bytes);
#pragma unroll
    for (int m = 0; m < kMats; ++m)
      if (mat[m]) {
        bulk_row(base + s * stage_bytes + offset[m], mat[m], row_bytes, bars + 8 * s);
        mat[m] += ld[m];
      }
    ++next;
  }
  // Waits for the current stage.  A wait that runs out raises the abort word: nothing is refilled from then on, later waits
  // give up at once, and the block runs through its remaining rows without meaning (finish() reports it).
  __device__ __forceinline__ void wait(volatile uint32_t* abort_word) const { mbar_wait(bars + 8 * stage, phase, abort_word); }
  __device__ __forceinline__ uint32_t at(int m) const { return cur + offset[m]; }
  // Behind a block barrier after the stage was read (each thread having fenced its reads): refill it and step on.
  __device__ __forceinline__ void refill(const volatile uint32_t* abort_word) {
    if (threadIdx.x == 0 && next < row1 && !*abort_word) fill(stage);
    cur += stage_bytes;
    if (++stage == stages) {
      stage = 0;
      cur = base;
      phase ^= 1u;
    }
  }
  __device__ __forceinline__ void finish(const volatile uint32_t* abort_word, unsigned int* error_word) const {
    if (!*abort_word) return;
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 2000000ull) {}           // let copies that are still in flight land
    if (threadIdx.x == 0) atomicExch(error_word, 1u);
  }
};

template <typename T>
__device__ __forceinline__ Raw8<T> lds_group(uint32_t at) {
  Raw8<T> r;
  r.a = lds128(at);
  if constexpr (sizeof(T) == 4) r.b = lds128(at + 16);
  return r;
}
// A weight vector in shared memory; ones (`fill`) where there is none.
template <typename W>
__device__ __forceinline__ void stage_vector(const void* w, uint32_t at, int cols, float fill) {
  Raw8<W> ones;
  ones = raw_of<W>(pairs_filled(fill));
  for (int c = threadIdx.x * 8; c < cols; c += blockDim.x * 8) {
    const Raw8<W> r = w ? load8(static_cast<const W*>(w) + c) : ones;
    sts128(at + c * sizeof(W), r.a.x, r.a.y, r.a.z, r.a.w);
    if constexpr (sizeof(W) == 4) sts128(at + c * sizeof(W) + 16, r.b.x, r.b.y, r.b.z, r.b.w);
  }
}

// A thread's groups: column, the column it reads (0 past the row's end), and 1 or 0 for its part in sums.
template <int kVpt>
struct Groups {
  int col[kVpt];
  bool in[kVpt];
  __device__ __forceinline__ explicit Groups(int cols) {
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const int c = 8 * (i * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x));
      in[i] = c < cols;
      col[i] = in[i] ? c : 0;
    }
  }
  template <typename F>
  __device__ __forceinline__ float sum(F&& term) const {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      float2 t = both(0.0f);
#pragma unroll
      for (int j = 0; j < 4; ++j) t = term(i, j, t);
      s += in[i] ? t.x + t.y : 0.0f;
    }
    return s;
  }
};

template <typename T, typename W, int kVpt>
__global__ void __launch_bounds__(kVpt <= 2 ? 320 : 512)
block_norm_bulk_kernel(const NormParams p) {
  __shared__ float red[2][4][32];
  __shared__ uint32_t abort_word;
  extern __shared__ __align__(128) uint8_t ring_smem[];
  uint32_t slot = 0;
  grid_launch_next();
  grid_wait();
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows / gridDim.x;
  const int64_t row1 = (static_cast<int64_t>(blockIdx.x) + 1) * p.rows / gridDim.x;
  const float inv_cols = 1.0f / static_cast<float>(p.cols);
  const Groups<kVpt> g(p.cols);
  const bool post = p.kind_post != HIF4_NORM_NONE, has_res = p.residual != nullptr, has_bias = p.pre_bias != nullptr;
  const uint32_t wb = static_cast<uint32_t>(p.cols) * sizeof(W);
  const uint32_t sm_pre = smem_u32(ring_smem), sm_post = sm_pre + (p.y ? wb : 0u), sm_bias = sm_post + (post ? wb : 0u);
  if (p.y) stage_vector<W>(p.pre_weight, sm_pre, p.cols, 1.0f);
  if (post) stage_vector<W>(p.post_weight, sm_post, p.cols, 1.0f);
  if (has_bias) stage_vector<W>(p.pre_bias, sm_bias, p.cols, 0.0f);
  if (threadIdx.x == 0) abort_word = 0u;
  RowRing<T, 2> ring{{static_cast<const T*>(p.x), static_cast<const T*>(p.residual)}, {p.ld_x, p.ld_residual}};
  ring.start(sm_bias + (has_bias ? wb : 0u), p.stages, p.cols, row0, row1);
  T* h = p.h ? static_cast<T*>(p.h) + row0 * p.ld_h : nullptr;
  T* y = p.y && !p.units ? static_cast<T*>(p.y) + row0 * p.ld_y : nullptr;
  uint32_t* u = p.y && p.units ? static_cast<uint32_t*>(p.y) + row0 * (p.cols >> 6) * kUnitWords : nullptr;
  Raw8<T> gr[kVpt];
  int64_t gate_row = p.gate ? row0 / p.rows_per_gate : 0, gate_end = row0;
  for (int64_t row = row0; row < row1; ++row) {
    if (p.gate && row == gate_end) {
      if (row != row0) ++gate_row;
      gate_end = (gate_row + 1) * p.rows_per_gate;
#pragma unroll
      for (int i = 0; i < kVpt; ++i) gr[i] = load8(static_cast<const T*>(p.gate) + gate_row * p.ld_gate + g.col[i]);
    }
    ring.wait(&abort_word);
    Pairs v[kVpt];
    Raw8<T> rr[kVpt];
#pragma unroll
    for (int i = 0; i < kVpt; ++i) v[i] = pairs_of(lds_group<T>(ring.at(0) + g.col[i] * sizeof(T)));
    if (has_res) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i) rr[i] = lds_group<T>(ring.at(1) + g.col[i] * sizeof(T));
    }
    fence_proxy_async_smem();              // these reads before the async proxy writes the stage again
    bool refilled = false;
    // centres v (LAYER) and returns the factor of the norm; the first barrier on the way frees the stage
    auto normalise = [&](int kind) {
      if (kind == HIF4_NORM_LAYER) {
        float s[1] = {g.sum([&](int i, int j, float2 t) { return add2(t, v[i].p[j]); })};
        block_sums_synced(s, red, slot);
        if (!refilled) { ring.refill(&abort_word); refilled = true; }
        const float2 m = both(-s[0] * inv_cols);
#pragma unroll
        for (int i = 0; i < kVpt; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) v[i].p[j] = add2(v[i].p[j], m);
      }
      float s[1] = {g.sum([&](int i, int j, float2 t) { return fma2(v[i].p[j], v[i].p[j], t); })};
      block_sums_synced(s, red, slot);
      if (!refilled) { ring.refill(&abort_word); refilled = true; }
      return both(rsqrtf(fmaf(s[0], inv_cols, p.eps)));
    };
    if (post) {
      const float2 rstd = normalise(p.kind_post);
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        const Pairs w = pairs_of(lds_group<W>(sm_post + g.col[i] * sizeof(W)));
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(mul2(v[i].p[j], rstd), w.p[j]);
      }
    }
    if (p.gate) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        const Pairs w = pairs_of(gr[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], w.p[j]);
      }
    }
    if (has_res) {
      const float2 scale = both(p.res_scale);
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        const Pairs r = pairs_of(rr[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].p[j] = fma2(scale, r.p[j], v[i].p[j]);
      }
    }
    if (h) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
        if (g.in[i]) store8(h + g.col[i], raw_of<T>(v[i]));
      h += p.ld_h;
    }
    if (!p.y) {
      __syncthreads();
      if (!refilled) ring.refill(&abort_word);
      continue;
    }
    const float2 rstd = normalise(p.kind_pre);
#pragma unroll
    for (int i = 0; i < kVpt; ++i) {
      const Pairs w = pairs_of(lds_group<W>(sm_pre + g.col[i] * sizeof(W)));
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(mul2(v[i].p[j], rstd), w.p[j]);
    }
    if (has_bias) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        const Pairs b = pairs_of(lds_group<W>(sm_bias + g.col[i] * sizeof(W)));
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].p[j] = add2(v[i].p[j], b.p[j]);
      }
    }
    if (y) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
        if (g.in[i]) store8(y + g.col[i], raw_of<T>(v[i]));
      y += p.ld_y;
    } else {
      // eight consecutive lanes hold a unit (cols % 64 == 0, so a unit is inside the row or outside as a whole)
      const int k = threadIdx.x & 7;
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        const Raw8<T> out = raw_of<T>(v[i]);
        uint32_t meta;
        const uint32_t code = p.rha ? encode_unit_octet<true>(out, k, meta) : encode_unit_octet<false>(out, k, meta);
        if (g.in[i]) {
          uint32_t* dst = u + (g.col[i] >> 6) * kUnitWords;
          dst[1 + k] = code;
          if (k == 0) dst[0] = meta;
        }
      }
      u += (p.cols >> 6) * kUnitWords;
    }
  }
  ring.finish(&abort_word, p.error_word);
}

// Gradients.  One sum over the rows, S = sum dt xhat(x) within a row of gates, gives both gradients that the path to x has:
// dgate = S wp and dwp = sum over the rows of gates gate S; the latter is kept in shared memory, since it only changes where the
// gates do.  kLayer: one of the norms is a LAYER norm (the RMS form has no means, no bias and fewer registers to carry).
template <typename T, typename W, int kVpt, bool kPath, bool kLayer>
__global__ void __launch_bounds__(kVpt == 4 ? 1024 : 512)
block_norm_backward_bulk_kernel(const NormGradParams p) {
  __shared__ float red[2][4][32];
  __shared__ uint32_t abort_word;
  extern __shared__ __align__(128) uint8_t ring_smem[];
  uint32_t slot = 0;
  grid_launch_next();
  grid_wait();
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows / gridDim.x;
  const int64_t row1 = (static_cast<int64_t>(blockIdx.x) + 1) * p.rows / gridDim.x;
  const float inv_cols = 1.0f / static_cast<float>(p.cols);
  const bool pre_layer = kLayer && p.kind_pre == HIF4_NORM_LAYER, post_layer = kLayer && p.kind_post == HIF4_NORM_LAYER;
  const bool post = kPath && p.kind_post != HIF4_NORM_NONE, has_dy = p.dy != nullptr, has_dh = p.dh != nullptr, has_x = kPath && p.x;
  const bool has_gate = kPath && p.gate, sums_dwp = post && has_gate;
  const Groups<kVpt> g(p.cols);
  constexpr int kPathVpt = kPath ? kVpt : 1, kLayerVpt = kLayer ? kVpt : 1;
  Pairs dw[kVpt], db[kLayerVpt], S[kPathVpt];
#pragma unroll
  for (int i = 0; i < kVpt; ++i) {
    dw[i] = pairs_filled(0.0f);
    if (kLayer) db[i] = pairs_filled(0.0f);
    if (kPath) S[i] = pairs_filled(0.0f);
  }
  const uint32_t wb = static_cast<uint32_t>(p.cols) * sizeof(W);
  const uint32_t sm_pre = smem_u32(ring_smem), sm_post = sm_pre + (has_dy ? wb : 0u), sm_dwp = sm_post + (post ? wb : 0u);
  if (has_dy) stage_vector<W>(p.pre_weight, sm_pre, p.cols, 1.0f);
  if (post) stage_vector<W>(p.post_weight, sm_post, p.cols, 1.0f);
  if (sums_dwp) stage_vector<float>(nullptr, sm_dwp, p.cols, 0.0f);
  if (threadIdx.x == 0) abort_word = 0u;
  RowRing<T, 4> ring{{has_dy ? static_cast<const T*>(p.h) : nullptr, static_cast<const T*>(p.dy), static_cast<const T*>(p.dh),
                      has_x ? static_cast<const T*>(p.x) : nullptr},
                     {p.ld_h, p.ld_dy, p.ld_dh, p.ld_x}};
  ring.start(sm_dwp + (sums_dwp ? static_cast<uint32_t>(p.cols) * 4u : 0u), p.stages, p.cols, row0, row1);
  T* dx = p.dx ? static_cast<T*>(p.dx) + row0 * p.ld_dx : nullptr;
  T* dres = p.dresidual ? static_cast<T*>(p.dresidual) + row0 * p.ld_dresidual : nullptr;
  Raw8<T> gr[kPathVpt];
  int64_t group = has_gate ? row0 / p.rows_per_gate : 0;
  int64_t gate_end = has_gate ? group * p.rows_per_gate : row1 + 1;      // first row of the next gates; the first row loads its own
  for (int64_t row = row0; row < row1; ++row) {
    if (kPath && has_gate && (row >= gate_end || row == row0)) {
      if (row != row0) ++group;
      gate_end = (group + 1) * p.rows_per_gate;
      if (gate_end > p.rows) gate_end = p.rows;
#pragma unroll
      for (int i = 0; i < kVpt; ++i) gr[i] = load8(static_cast<const T*>(p.gate) + group * p.ld_gate + g.col[i]);
    }
    ring.wait(&abort_word);
    Pairs a[kVpt], t[kVpt], x[kPathVpt], dn[kVpt];      // h, gradient of h, x, gradient of the normalised row
    Raw8<T> dy[kVpt];
    if (has_dy) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        a[i] = pairs_of(lds_group<T>(ring.at(0) + g.col[i] * sizeof(T)));
        dy[i] = lds_group<T>(ring.at(1) + g.col[i] * sizeof(T));
        const Pairs w = pairs_of(lds_group<W>(sm_pre + g.col[i] * sizeof(W))), d = pairs_of(dy[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) dn[i].p[j] = mul2(d.p[j], w.p[j]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        a[i] = dn[i] = pairs_filled(0.0f);
        zero8(dy[i]);
      }
    }
    if (has_dh) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i) t[i] = pairs_of(lds_group<T>(ring.at(2) + g.col[i] * sizeof(T)));
    } else {
#pragma unroll
      for (int i = 0; i < kVpt; ++i) t[i] = pairs_filled(0.0f);
    }
    if constexpr (kPath) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i) x[i] = has_x ? pairs_of(lds_group<T>(ring.at(3) + g.col[i] * sizeof(T))) : pairs_filled(0.0f);
    }
    fence_proxy_async_smem();              // these reads before the async proxy writes the stage again
    if constexpr (kLayer) {
      float s[2] = {g.sum([&](int i, int j, float2 c) { return add2(c, a[i].p[j]); }), 0.0f};
      if constexpr (kPath) s[1] = g.sum([&](int i, int j, float2 c) { return add2(c, x[i].p[j]); });
      block_sums_synced(s, red, slot);
      ring.refill(&abort_word);
      const float2 m = both(pre_layer ? -s[0] * inv_cols : 0.0f), mx = both(post_layer ? -s[1] * inv_cols : 0.0f);
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          a[i].p[j] = add2(a[i].p[j], m);
          if constexpr (kPath) x[i].p[j] = add2(x[i].p[j], mx);
        }
    }
    // sums over the row: (h - mean)^2, dn (h - mean), (x - mean_x)^2, dn
    float s2[4];
    s2[0] = g.sum([&](int i, int j, float2 c) { return fma2(a[i].p[j], a[i].p[j], c); });
    s2[1] = g.sum([&](int i, int j, float2 c) { return fma2(dn[i].p[j], a[i].p[j], c); });
    s2[2] = s2[3] = 0.0f;
    if constexpr (kPath) {
      if (post) s2[2] = g.sum([&](int i, int j, float2 c) { return fma2(x[i].p[j], x[i].p[j], c); });
    }
    if constexpr (kLayer) s2[3] = g.sum([&](int i, int j, float2 c) { return add2(c, dn[i].p[j]); });
    if constexpr (kPath || kLayer) {
      block_sums_synced(s2, red, slot);
    } else {
      float s[2] = {s2[0], s2[1]};
      block_sums_synced(s, red, slot);
      s2[0] = s[0]; s2[1] = s[1];
    }
    if constexpr (!kLayer) ring.refill(&abort_word);
    const float rstd = rsqrtf(fmaf(s2[0], inv_cols, p.eps));
    if (has_dy) {
      const float2 r2 = both(rstd), m1 = both(-s2[1] * rstd * inv_cols);
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        const Pairs d = pairs_of(dy[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 n = mul2(a[i].p[j], r2);
          dw[i].p[j] = fma2(d.p[j], n, dw[i].p[j]);
          t[i].p[j] = fma2(r2, fma2(n, m1, dn[i].p[j]), t[i].p[j]);
        }
        if constexpr (kLayer) {
          const float2 shift = both(pre_layer ? -rstd * s2[3] * inv_cols : 0.0f);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            db[i].p[j] = add2(db[i].p[j], d.p[j]);
            t[i].p[j] = add2(t[i].p[j], shift);
          }
        }
      }
    }
    if (dres) {
      const float2 scale = both(p.res_scale);
#pragma unroll
      for (int i = 0; i < kVpt; ++i) {
        Pairs o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o.p[j] = mul2(scale, t[i].p[j]);
        if (g.in[i]) store8(dres + g.col[i], raw_of<T>(o));
      }
      dres += p.ld_dresidual;
    }
    if constexpr (kPath) {
      if (post) {
        const float2 rx = both(rsqrtf(fmaf(s2[2], inv_cols, p.eps)));
#pragma unroll
        for (int i = 0; i < kVpt; ++i) {
          const Pairs wp = pairs_of(lds_group<W>(sm_post + g.col[i] * sizeof(W)));
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 xn = mul2(x[i].p[j], rx);
            S[i].p[j] = fma2(t[i].p[j], xn, S[i].p[j]);
            x[i].p[j] = xn;
            t[i].p[j] = mul2(t[i].p[j], wp.p[j]);
          }
          if (has_gate) {
            const Pairs gate = pairs_of(gr[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) t[i].p[j] = mul2(t[i].p[j], gate.p[j]);
          }
        }
        if (dx) {
          float s3[2] = {g.sum([&](int i, int j, float2 c) { return fma2(t[i].p[j], x[i].p[j], c); }), 0.0f};
          if constexpr (kLayer) {
            s3[1] = g.sum([&](int i, int j, float2 c) { return add2(c, t[i].p[j]); });
            block_sums_synced(s3, red, slot);
          } else {
            float s1[1] = {s3[0]};
            block_sums_synced(s1, red, slot);
            s3[0] = s1[0];
          }
          const float2 q1 = both(-s3[0] * inv_cols), q0 = both(post_layer ? -s3[1] * inv_cols : 0.0f);
#pragma unroll
          for (int i = 0; i < kVpt; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float2 d = fma2(x[i].p[j], q1, t[i].p[j]);
              if constexpr (kLayer) d = add2(d, q0);
              t[i].p[j] = mul2(rx, d);
            }
        }
      } else {                             // a gate without a norm
#pragma unroll
        for (int i = 0; i < kVpt; ++i) {
          const Pairs gate = pairs_of(gr[i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            S[i].p[j] = fma2(t[i].p[j], x[i].p[j], S[i].p[j]);
            t[i].p[j] = mul2(t[i].p[j], gate.p[j]);
          }
        }
      }
    }
    if (dx) {
#pragma unroll
      for (int i = 0; i < kVpt; ++i)
        if (g.in[i]) store8(dx + g.col[i], raw_of<T>(t[i]));
      dx += p.ld_dx;
    }
    if constexpr (kPath) {
      if (has_gate && (row + 1 == gate_end || row + 1 == row1)) {      // these gates' rows, or the block's, end here
        const bool starts_here = group * p.rows_per_gate >= row0, ends_here = row + 1 == gate_end;
        float* part = p.partial + (static_cast<int64_t>(starts_here ? 4 : 3) * gridDim.x + blockIdx.x) * p.cols;
#pragma unroll
        for (int i = 0; i < kVpt; ++i) {
          if (g.in[i]) {
            if (p.dgate) {
              Pairs d = S[i];
              if (post) {
                const Pairs wp = pairs_of(lds_group<W>(sm_post + g.col[i] * sizeof(W)));
#pragma unroll
                for (int j = 0; j < 4; ++j) d.p[j] = mul2(d.p[j], wp.p[j]);
              }
              if (starts_here && ends_here) store8(static_cast<T*>(p.dgate) + group * p.cols + g.col[i], raw_of<T>(d));
              else store8(part + g.col[i], raw_of<float>(d));
            }
            if (sums_dwp) {
              const uint32_t at = sm_dwp + g.col[i] * 4u;
              const Pairs gate = pairs_of(gr[i]), old = pairs_of(lds_group<float>(at));
              Pairs now;
#pragma unroll
              for (int j = 0; j < 4; ++j) now.p[j] = fma2(gate.p[j], S[i].p[j], old.p[j]);
              const Raw8<float> r = raw_of<float>(now);
              sts128(at, r.a.x, r.a.y, r.a.z, r.a.w);
              sts128(at + 16, r.b.x, r.b.y, r.b.z, r.b.w);
            }
          }
          S[i] = pairs_filled(0.0f);
        }
      }
    }
  }
  const int64_t plane = static_cast<int64_t>(gridDim.x) * p.cols;
  float* part = p.partial + static_cast<int64_t>(blockIdx.x) * p.cols;
#pragma unroll
  for (int i = 0; i < kVpt; ++i) {
    if (!g.in[i]) continue;
    if (p.dpre_weight) store8(part + g.col[i], raw_of<float>(dw[i]));
    if (p.dpre_bias) store8(part + plane + g.col[i], kLayer ? raw_of<float>(db[kLayer ? i : 0]) : raw_of<float>(pairs_filled(0.0f)));
    if constexpr (kPath) {
      if (p.dpost_weight) store8(part + 2 * plane + g.col[i], sums_dwp ? lds_group<float>(sm_dwp + g.col[i] * 4u) : raw_of<float>(S[i]));
    }
  }
  ring.finish(&abort_word, p.error_word);
}

