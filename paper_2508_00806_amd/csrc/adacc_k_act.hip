// Activations (GELU, its tanh form, SiLU) and gated activations, y = act(a) or act(a) * up, and their gradients from the inputs as they were or from their 8-bit rows.
// One pass over the data either way; binary32 in registers, rounded once.
//
// What bounds them is memory.  Sixteen lanes hold a group of 128, eight values a lane, so that its largest magnitude takes four exchanges in the vector unit; a lane has a place in four groups, whose loads
// are all under way before the first is used; data pass with the streaming hint.  bfloat16, with codes: GELU of [8192, 16384] 110 us forward and 111 backward (6.1 TB/s both; two products fewer in its
// tail, 107 and 108), SiLU 101 and 97; SiLU gated [16384, 11008] 226 and 238 (6.4 and 6.1); a copy runs at 6.3.  binary32, [8192, 8192]: GELU 118 and 109 (5.2, 5.6), SiLU gated 176 and 166 (5.4, 5.7).
// Rows whose length is no multiple of eight: [1999, 4093] 12.0 and 11.6 us; [8191, 8191] 69 and 66 (4.9, 5.1).
#include "adacc_layers.hpp"

namespace adacc {

__device__ __forceinline__ uint32_t left_of(uint32_t cols, uint32_t col) { return col < cols ? cols - col : 0u; }

template <uint32_t TYPE, uint32_t KIND, bool GATED, bool CODES, bool EVEN>
__global__ __launch_bounds__(kThreads) void act_forward_kernel(ActArgs p) {
  constexpr bool kFine = TYPE == kTypeF32;
  const uint32_t groups = (p.cols + kR8Group - 1u) / kR8Group;
  const uint64_t unit = (uint64_t)blockIdx.x * (kThreads / kR8Lanes * kR8Units) + threadIdx.x / kR8Lanes;
  uint32_t row = (uint32_t)(unit / groups), group = (uint32_t)(unit % groups);
  const uint32_t in = threadIdx.x % kR8Lanes * 8u;
  Octet<TYPE> a[kR8Units], up[GATED ? kR8Units : 1u];
  uint32_t rows[kR8Units], cols[kR8Units], left[kR8Units];
#pragma unroll
  for (uint32_t u = 0; u < kR8Units; ++u) {
    rows[u] = row;
    cols[u] = group * kR8Group + in;
    left[u] = row < p.rows ? left_of(p.cols, cols[u]) : 0u;
    row += p.step_rows;
    group += p.step_groups;
    if (group >= groups) {
      group -= groups;
      ++row;
    }
  }
  if constexpr (EVEN) {
#pragma unroll
    for (uint32_t u = 0; u < kR8Units; ++u) {
      a[u].template load_even<true>(p.a.at, (uint64_t)rows[u] * p.a.stride + cols[u], left[u]);
      if constexpr (GATED) up[u].template load_even<true>(p.up.at, (uint64_t)rows[u] * p.up.stride + cols[u], left[u]);
    }
  } else {
#pragma unroll
    for (uint32_t u = 0; u < kR8Units; ++u) {
      a[u].load(p.a.at, (uint64_t)rows[u] * p.a.stride, cols[u], left[u]);
      if constexpr (GATED) up[u].load(p.up.at, (uint64_t)rows[u] * p.up.stride, cols[u], left[u]);
    }
  }
#pragma unroll
  for (uint32_t u = 0; u < kR8Units; ++u) {
    float v[8], w[8], r[8], none;
    a[u].get(v);
    if constexpr (GATED) up[u].get(w);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
      activate<KIND, kFine, false>(v[i], &r[i], &none);
      if constexpr (GATED) r[i] *= w[i];
    }
    Octet<TYPE> o;
    o.set(r);
    if constexpr (EVEN) o.template store_even<true>(p.y.at, (uint64_t)rows[u] * p.y.stride + cols[u], left[u]);
    else o.store(p.y.at, (uint64_t)rows[u] * p.y.stride + cols[u], left[u]);
    if constexpr (CODES) {
      write_group(p.a8, rows[u], cols[u], v, left[u] != 0u);
      if constexpr (GATED) write_group(p.up8, rows[u], cols[u], w, left[u] != 0u);
    }
  }
}

// what is kept of an input, as it is in memory
template <uint32_t TYPE, bool CODES>
struct Kept {
  Octet<TYPE> x;
  uint2 code;
  float scale;
  __device__ __forceinline__ void load(const Strided& m, const Rows8& b, bool even, uint32_t row, uint32_t col, uint32_t left) {
    if constexpr (CODES) {
      code = left ? *reinterpret_cast<const uint2*>(b.codes + (uint64_t)row * b.pitch + col) : make_uint2(0u, 0u);
      scale = left ? b.scales[(uint64_t)row * b.groups + col / kR8Group] : 0.0f;
    } else {
      if (even) x.template load_even<true>(m.at, (uint64_t)row * m.stride + col, left);
      else x.load(m.at, (uint64_t)row * m.stride, col, left);
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    if constexpr (CODES) restore8(code, scale, v);
    else x.get(v);
  }
};

template <uint32_t TYPE, uint32_t KIND, bool GATED, bool CODES, bool EVEN>
__global__ __launch_bounds__(kThreads) void act_backward_kernel(ActArgs p) {
  constexpr bool kFine = TYPE == kTypeF32;
  const uint32_t groups = (p.cols + kR8Group - 1u) / kR8Group;
  const uint64_t unit = (uint64_t)blockIdx.x * (kThreads / kR8Lanes * kR8Units) + threadIdx.x / kR8Lanes;
  uint32_t row = (uint32_t)(unit / groups), group = (uint32_t)(unit % groups);
  const uint32_t in = threadIdx.x % kR8Lanes * 8u;
  Octet<TYPE> dy[kR8Units];
  Kept<TYPE, CODES> a[kR8Units], up[GATED ? kR8Units : 1u];
  uint32_t rows[kR8Units], cols[kR8Units], left[kR8Units];
#pragma unroll
  for (uint32_t u = 0; u < kR8Units; ++u) {
    rows[u] = row;
    cols[u] = group * kR8Group + in;
    left[u] = row < p.rows ? left_of(p.cols, cols[u]) : 0u;
    row += p.step_rows;
    group += p.step_groups;
    if (group >= groups) {
      group -= groups;
      ++row;
    }
  }
  if constexpr (EVEN) {
#pragma unroll
    for (uint32_t u = 0; u < kR8Units; ++u) {
      dy[u].template load_even<true>(p.y.at, (uint64_t)rows[u] * p.y.stride + cols[u], left[u]);
      a[u].load(p.a, p.a8, true, rows[u], cols[u], left[u]);
      if constexpr (GATED) up[u].load(p.up, p.up8, true, rows[u], cols[u], left[u]);
    }
  } else {
#pragma unroll
    for (uint32_t u = 0; u < kR8Units; ++u) {
      dy[u].load(p.y.at, (uint64_t)rows[u] * p.y.stride, cols[u], left[u]);
      a[u].load(p.a, p.a8, false, rows[u], cols[u], left[u]);
      if constexpr (GATED) up[u].load(p.up, p.up8, false, rows[u], cols[u], left[u]);
    }
  }
#pragma unroll
  for (uint32_t u = 0; u < kR8Units; ++u) {
    float g[8], v[8], w[8], value[8];
    dy[u].get(g);
    a[u].get(v);
    if constexpr (GATED) up[u].get(w);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
      float slope;
      activate<KIND, kFine, true>(v[i], &value[i], &slope);
      value[i] *= g[i];
      v[i] = slope * (GATED ? g[i] * w[i] : g[i]);
    }
    Octet<TYPE> o;
    if (!GATED || p.da.at) {
      o.set(v);
      if constexpr (EVEN) o.template store_even<true>(p.da.at, (uint64_t)rows[u] * p.da.stride + cols[u], left[u]);
      else o.store(p.da.at, (uint64_t)rows[u] * p.da.stride + cols[u], left[u]);
    }
    if constexpr (GATED) {
      if (p.dup.at) {
        o.set(value);
        if constexpr (EVEN) o.template store_even<true>(p.dup.at, (uint64_t)rows[u] * p.dup.stride + cols[u], left[u]);
        else o.store(p.dup.at, (uint64_t)rows[u] * p.dup.stride + cols[u], left[u]);
      }
    }
  }
}

// The same for an activation within a product, with the sums of the gradient's columns (the bias's gradient): a workgroup takes a strip of `wide` groups of 128
// columns and 16 / wide rows at a time of every P-th bunch.  kActNone: the sums of dy alone.  The gradient goes to memory in 16 bits, as the matrix instructions of the two products behind it take it (the
// plain form's 32 would double what they read and halve their rate); the sums are taken before that.  [8192, 8192] of codes, GELU 70 us (4.8 TB/s), SiLU 67, the sums of dy alone 31; half
// or a quarter as many workgroups: 78 and 103.
template <uint32_t TYPE, uint32_t KIND, bool CODES>
__global__ __launch_bounds__(kThreads) void act_columns_kernel(ActArgs p) {
  __shared__ float sums[kThreads / kR8Lanes][kR8Group + 4];
  const uint32_t wide = p.step_groups, bunch = 16u / wide;
  const uint32_t strips = ((p.cols + kR8Group - 1u) / kR8Group + wide - 1u) / wide;
  const uint32_t part = blockIdx.x / strips, unit = threadIdx.x / kR8Lanes;
  const uint32_t col = ((blockIdx.x % strips) * wide + unit % wide) * kR8Group + threadIdx.x % kR8Lanes * 8u;
  const uint32_t left = left_of(p.cols, col);
  float sum[8];
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) sum[i] = 0.0f;
  constexpr uint32_t kAhead = 4u;  // rows at once
  const bool even = p.cols % 8u == 0u;
  const uint64_t step = (uint64_t)p.partials * bunch;
  for (uint64_t first = (uint64_t)part * bunch + unit / wide; first < p.rows; first += kAhead * step) {
    Octet<TYPE> dy[kAhead];
    Kept<TYPE, CODES> a[kAhead];
    if (even) {
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) {
        const uint64_t row = first + k * step;
        const uint32_t have = row < p.rows ? left : 0u;
        dy[k].template load_even<true>(p.y.at, row * p.y.stride + col, have);
        if constexpr (KIND != kActNone) a[k].load(p.a, p.a8, true, (uint32_t)row, col, have);
      }
    } else {
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) {
        const uint64_t row = first + k * step;
        const uint32_t have = row < p.rows ? left : 0u;
        dy[k].load(p.y.at, row * p.y.stride, col, have);
        if constexpr (KIND != kActNone) a[k].load(p.a, p.a8, false, (uint32_t)row, col, have);
      }
    }
#pragma unroll
    for (uint32_t k = 0; k < kAhead; ++k) {
      const uint64_t row = first + k * step;
      float g[8];
      dy[k].get(g);
      if constexpr (KIND != kActNone) {
        float v[8], none;
        a[k].get(v);
        const bool have = row < p.rows;
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
          float slope;
          activate<KIND, false, true>(v[i], &none, &slope);
          g[i] *= slope;
          if (have) sum[i] += g[i];
        }
        Octet<TYPE> o;
        o.set(g);
        if (even) o.template store_even<true>(p.da.at, row * p.da.stride + col, have ? left : 0u);
        else o.store(p.da.at, row * p.da.stride + col, have ? left : 0u);
      } else {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) sum[i] += g[i];
      }
    }
  }
  if (!p.partial) return;
  // [unit][128]: the rows of a bunch are added up
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) sums[unit][threadIdx.x % kR8Lanes * 8u + i] = sum[i];
  __syncthreads();
  for (uint32_t t = threadIdx.x; t < wide * kR8Group; t += kThreads) {
    const uint32_t at = (blockIdx.x % strips) * wide * kR8Group + t;
    if (at >= p.cols) continue;
    float v = 0.0f;
    for (uint32_t k = 0; k < bunch; ++k) v += sums[k * wide + t / kR8Group][t % kR8Group];
    p.partial[(uint64_t)part * p.cols + at] = v;
  }
}

template <uint32_t TYPE, uint32_t KIND, bool EVEN>
static ActFn act_of(bool backward, bool gated, bool codes) {
  if (backward) {
    if (gated) return codes ? act_backward_kernel<TYPE, KIND, true, true, EVEN> : act_backward_kernel<TYPE, KIND, true, false, EVEN>;
    return codes ? act_backward_kernel<TYPE, KIND, false, true, EVEN> : act_backward_kernel<TYPE, KIND, false, false, EVEN>;
  }
  if (gated) return codes ? act_forward_kernel<TYPE, KIND, true, true, EVEN> : act_forward_kernel<TYPE, KIND, true, false, EVEN>;
  return codes ? act_forward_kernel<TYPE, KIND, false, true, EVEN> : act_forward_kernel<TYPE, KIND, false, false, EVEN>;
}
template <uint32_t TYPE, bool EVEN>
static ActFn act_by_kind(uint32_t kind, bool backward, bool gated, bool codes) {
  return kind == kActGelu ? act_of<TYPE, kActGelu, EVEN>(backward, gated, codes)
         : kind == kActGeluTanh ? act_of<TYPE, kActGeluTanh, EVEN>(backward, gated, codes) : act_of<TYPE, kActSilu, EVEN>(backward, gated, codes);
}
template <bool EVEN>
static ActFn act_by_type(uint32_t type, uint32_t kind, bool backward, bool gated, bool codes) {
  return type == kTypeF32 ? act_by_kind<kTypeF32, EVEN>(kind, backward, gated, codes)
         : type == kTypeF16 ? act_by_kind<kTypeF16, EVEN>(kind, backward, gated, codes) : act_by_kind<kTypeBf16, EVEN>(kind, backward, gated, codes);
}
static ActFn act_fn(uint32_t type, uint32_t kind, bool backward, bool gated, bool codes, bool even) {
  return even ? act_by_type<true>(type, kind, backward, gated, codes) : act_by_type<false>(type, kind, backward, gated, codes);
}
ActFn act_forward_fn(uint32_t type, uint32_t kind, bool gated, bool codes, bool even) { return act_fn(type, kind, false, gated, codes, even); }
ActFn act_backward_fn(uint32_t type, uint32_t kind, bool gated, bool codes, bool even) { return act_fn(type, kind, true, gated, codes, even); }

template <uint32_t TYPE>
static ActFn columns_by_kind(uint32_t kind, bool codes) {
  if (kind == kActNone) return act_columns_kernel<TYPE, kActNone, false>;
  if (kind == kActGelu) return codes ? act_columns_kernel<TYPE, kActGelu, true> : act_columns_kernel<TYPE, kActGelu, false>;
  if (kind == kActGeluTanh) return codes ? act_columns_kernel<TYPE, kActGeluTanh, true> : act_columns_kernel<TYPE, kActGeluTanh, false>;
  return codes ? act_columns_kernel<TYPE, kActSilu, true> : act_columns_kernel<TYPE, kActSilu, false>;
}
ActFn act_columns_fn(uint32_t type, uint32_t kind, bool codes) {
  return type == kTypeF16 ? columns_by_kind<kTypeF16>(kind, codes) : columns_by_kind<kTypeBf16>(kind, codes);  // (a product's types)
}

}  // namespace adacc
