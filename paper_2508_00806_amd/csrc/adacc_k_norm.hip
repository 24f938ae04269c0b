// Layer norm: y = (x - mean) / sigma * w + b, and its gradients, the input being read as it was or from its 8-bit rows.
//
//   forward   mean, 1 / sigma (kept for the backward pass), y, and the codes of x: one reading of x
//   backward  xh = (x~ - mean) / sigma, g = dy * w:  dx = (g - avg(g) - xh * avg(g * xh)) / sigma;  dw = sum over the rows of dy * xh, db = sum of dy
//
// A row is held in the registers of 16, 32 or 64 lanes, or of a workgroup of up to 512, up to 32 values each: the variance is taken about the mean, not as a difference of
// sums.  Wider rows are read in pieces, once for each of those steps.  Sums are binary32, in an order that depends on rows and cols alone.
//
// A workgroup of the backward pass takes every P-th row (or bunch of rows), so that a lane's columns stay the same, and adds the parameters' gradients up in its
// registers; the P sums go to memory and are added in turn by reduce_kernel.
//
// What bounds both is memory.  Forward and backward pass in turn, with the parameters' gradients: bfloat16 [32768, 2048] 124 us from the input as it was (5.4 TB/s), 137 from codes (4.9), [8192, 8192] 120 (5.6),
// binary16 [8191, 11008] 170 (5.3); a copy runs at 6.3.  Results go to memory with the streaming hint: without it a forward pass that follows a backward pass takes 90 us for [8191, 11008] instead of 64.
// Rows of 1999 x 4093 binary32: 17 and 28.  Two rows ahead, or half and twice as many workgroups, were slower.
//   Fewer rows are further from that: bfloat16 [8191, 2048] forward with codes 17 us (4.8 TB/s), backward 36 (2.4), of which joining the parameters' sums is 7; rows that eight does not divide add to the forward
// pass, [8191, 2047] 21 and 37.  More than 16384 columns, read in pieces three times: [4096, 20480] served 105 us (3.2 TB/s of one reading), forward with codes 123, backward from codes 183, from the input 209;
// [4096, 20479] 139, 157, 232, 304; [4096, 16384], in registers, 42, 56, 80, 94.
#include "adacc_layers.hpp"

namespace adacc {

// Over the lanes of a row; N sums at once.  LANES = 0: over the workgroup's wavefronts, by LDS (two halves in turn, so that one barrier a sum is enough)
template <uint32_t LANES, uint32_t N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* lds, uint32_t* turn) {
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) v[i] = lane_sum<LANES ? LANES : (uint32_t)kWave>(v[i]);
  if constexpr (LANES == 0) {
    const uint32_t waves = blockDim.x / kWave, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    float* at = lds + *turn * 32u;
    *turn ^= 1u;
    if (lane < N) {
      float mine = v[0];
#pragma unroll
      for (uint32_t i = 1; i < N; ++i) mine = lane == i ? v[i] : mine;
      at[lane * 16u + wave] = mine;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) v[i] = lane_sum<16>(lane % 16u < waves ? at[i * 16u + lane % 16u] : 0.0f);
  }
}

template <uint32_t TYPE>
__device__ __forceinline__ void load_params(const void* p, bool even, uint32_t col, uint32_t left, float (&v)[8]) {
  Octet<TYPE> o;
  if (even) o.template load_even<false>(p, col, left);
  else o.load(p, 0u, col, left);
  o.get(v);
}
template <uint32_t TYPE>
__device__ __forceinline__ void load_params(uint32_t type, const void* p, bool even, uint32_t col, uint32_t left, float other, float (&v)[8]) {
  if (p == nullptr) {
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) v[i] = other;
  } else if (type == kTypeF32) {
    load_params<kTypeF32>(p, even, col, left, v);
  } else {
    load_params<TYPE == kTypeF16 ? kTypeF16 : kTypeBf16>(p, even, col, left, v);
  }
}
__device__ __forceinline__ uint32_t left_of(uint32_t cols, uint32_t col) { return col < cols ? cols - col : 0u; }

// ------------------------------------------------------------------ forward
// Workgroups take every P-th row, or bunch of rows: the parameters stay in registers, and the next row is on its way while this one is summed up.
template <uint32_t TYPE, uint32_t LANES, uint32_t C, bool CODES, bool EVEN>
__global__ __launch_bounds__(LANES ? (uint32_t)kThreads : kNormThreads) void norm_forward_kernel(NormArgs p) {
  __shared__ float lds[64];
  uint32_t turn = 0;
  const uint32_t lanes = LANES ? LANES : blockDim.x, lane = LANES ? threadIdx.x % LANES : threadIdx.x;
  constexpr uint32_t kBunch = LANES ? kThreads / (LANES ? LANES : 1u) : 1u;
  uint32_t col[C], left[C];
  float w[C][8], b[C][8];
#pragma unroll
  for (uint32_t c = 0; c < C; ++c) {
    col[c] = (c * lanes + lane) * 8u;
    left[c] = left_of(p.cols, col[c]);
    load_params<TYPE>(p.wtype, p.weight, EVEN, col[c], left[c], 1.0f, w[c]);
    load_params<TYPE>(p.wtype, p.bias, EVEN, col[c], left[c], 0.0f, b[c]);
  }
  Octet<TYPE> next[C];
  const auto fetch = [&](uint32_t r) {
    if constexpr (EVEN) {
#pragma unroll
      for (uint32_t c = 0; c < C; ++c) next[c].template load_even<false>(p.x.at, (uint64_t)r * p.x.stride + col[c], r < p.rows ? left[c] : 0u);
    } else {
#pragma unroll
      for (uint32_t c = 0; c < C; ++c) next[c].load(p.x.at, (uint64_t)r * p.x.stride, col[c], r < p.rows ? left[c] : 0u);
    }
  };
  const uint32_t step = gridDim.x * kBunch;
  uint32_t row = blockIdx.x * kBunch + (LANES ? threadIdx.x / lanes : 0u);
  fetch(row);
  const float per = (float)p.cols;
  // (all lanes of a workgroup go round as often: its last rows may be none)
  for (uint32_t first = blockIdx.x * kBunch; first < p.rows; first += step, row += step) {
    const bool live = row < p.rows;
    float v[C][8], sum[1] = {0.0f};
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) {
      next[c].hold();
      next[c].get(v[c]);
    }
    if (first + step < p.rows) fetch(row + step);
#pragma unroll
    for (uint32_t c = 0; c < C; ++c)
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) sum[0] += v[c][i];
    row_sums<LANES, 1>(sum, lds, &turn);
    const float mean = sum[0] / per;
    float square[1] = {0.0f};
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) {
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) {
        const float d = i < left[c] ? v[c][i] - mean : 0.0f;
        square[0] = fmaf(d, d, square[0]);
      }
    }
    row_sums<LANES, 1>(square, lds, &turn);
    const float rstd = 1.0f / sqrtf(square[0] / per + p.eps);
    if (live && lane == 0u && p.stats) p.stats[row] = make_float2(mean, rstd);
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) {
      const uint32_t have = live ? left[c] : 0u;
      if constexpr (CODES) write_group(p.blob, row, col[c], v[c], have != 0u);
      float r[8];
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) r[i] = fmaf((v[c][i] - mean) * rstd, w[c][i], b[c][i]);
      Octet<TYPE> out;
      out.set(r);
      if constexpr (EVEN) out.template store_even<true>(p.y.at, (uint64_t)row * p.y.stride + col[c], have);
      else out.store(p.y.at, (uint64_t)row * p.y.stride + col[c], have);
    }
  }
}

// rows of any length
template <uint32_t TYPE, bool CODES>
__global__ __launch_bounds__(1024) void norm_forward_pieces_kernel(NormArgs p) {
  __shared__ float lds[64];
  uint32_t turn = 0;
  const uint32_t row = blockIdx.x;
  const uint64_t x_at = (uint64_t)row * p.x.stride, y_at = (uint64_t)row * p.y.stride;
  const uint32_t whole = (p.cols + 8191u) / 8192u * 8192u;  // (every lane takes part in a group's largest magnitude)
  float sum[1] = {0.0f}, square[1] = {0.0f};
  for (uint32_t col = threadIdx.x * 8u; col < p.cols; col += 8192u) {
    Octet<TYPE> o;
    float v[8];
    o.load(p.x.at, x_at, col, p.cols - col);
    o.get(v);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) sum[0] += v[i];
  }
  row_sums<0, 1>(sum, lds, &turn);
  const float mean = sum[0] / (float)p.cols;
  for (uint32_t col = threadIdx.x * 8u; col < p.cols; col += 8192u) {
    Octet<TYPE> o;
    float v[8];
    o.load(p.x.at, x_at, col, p.cols - col);
    o.get(v);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
      const float d = i < p.cols - col ? v[i] - mean : 0.0f;
      square[0] = fmaf(d, d, square[0]);
    }
  }
  row_sums<0, 1>(square, lds, &turn);
  const float rstd = 1.0f / sqrtf(square[0] / (float)p.cols + p.eps);
  if (threadIdx.x == 0u && p.stats) p.stats[row] = make_float2(mean, rstd);
  for (uint32_t col = threadIdx.x * 8u; col < whole; col += 8192u) {
    const uint32_t left = left_of(p.cols, col);
    Octet<TYPE> o;
    float v[8], w[8], b[8];
    o.load(p.x.at, x_at, col, left);
    o.get(v);
    if constexpr (CODES) write_group(p.blob, row, col, v, left != 0u);
    load_params<TYPE>(p.wtype, p.weight, false, col, left, 1.0f, w);
    load_params<TYPE>(p.wtype, p.bias, false, col, left, 0.0f, b);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) v[i] = fmaf((v[i] - mean) * rstd, w[i], b[i]);
    o.set(v);
    o.store(p.y.at, y_at + col, left);
  }
}

// ------------------------------------------------------------------ backward
// An octet of the kept input and of dy, as they are in memory
template <uint32_t TYPE, bool CODES>
struct NormIn {
  Octet<TYPE> dy, x;
  uint2 code;
  float scale;
  __device__ __forceinline__ void load(const NormArgs& p, bool even, uint32_t row, uint32_t col, uint32_t left) {
    if (even) dy.template load_even<true>(p.dy.at, (uint64_t)row * p.dy.stride + col, left);
    else dy.load(p.dy.at, (uint64_t)row * p.dy.stride, col, left);
    if constexpr (CODES) {
      code = left ? *reinterpret_cast<const uint2*>(p.blob.codes + (uint64_t)row * p.blob.pitch + col) : make_uint2(0u, 0u);
      scale = left ? p.blob.scales[(uint64_t)row * p.blob.groups + col / kR8Group] : 0.0f;
    } else {
      if (even) x.template load_even<true>(p.x.at, (uint64_t)row * p.x.stride + col, left);
      else x.load(p.x.at, (uint64_t)row * p.x.stride, col, left);
    }
  }
  __device__ __forceinline__ void get(float (&g)[8], float (&v)[8]) {
    dy.hold();
    if constexpr (!CODES) x.hold();
    dy.get(g);
    if constexpr (CODES) restore8(code, scale, v);
    else x.get(v);
  }
};

template <uint32_t TYPE, uint32_t LANES, uint32_t C, bool CODES, bool EVEN>
__global__ __launch_bounds__(LANES ? (uint32_t)kThreads : kNormThreads) void norm_backward_kernel(NormArgs p) {
  extern __shared__ float sums[];  // LANES != 0: the parameters' gradients of the workgroup's lanes; C == 4: the weight
  __shared__ float lds[64];
  uint32_t turn = 0;
  const uint32_t lanes = LANES ? LANES : blockDim.x, lane = LANES ? threadIdx.x % LANES : threadIdx.x;
  constexpr uint32_t kBunch = LANES ? kThreads / (LANES ? LANES : 1u) : 1u;  // rows at a time
  // Four octets a lane leave no registers for the weight, which is kept in LDS, and of binary32 none for the next row either
  const bool even = CODES ? p.cols % 8u == 0u : EVEN;  // (from codes one kernel for both: 32768 x 2048 forward and backward 137 us, with one for even rows alone 146)
  constexpr bool kKeep = C < 4u, kAhead = C < 4u || TYPE != kTypeF32;
  float4* const weights = reinterpret_cast<float4*>(sums) + lane;  // [2 * C][lanes]
  uint32_t col[C], left[C];
  float w[kKeep ? C : 1u][8], dw[C][8], db[C][8];
#pragma unroll
  for (uint32_t c = 0; c < C; ++c) {
    col[c] = (c * lanes + lane) * 8u;
    left[c] = left_of(p.cols, col[c]);
    load_params<TYPE>(p.wtype, p.weight, even, col[c], left[c], 1.0f, w[kKeep ? c : 0u]);
    if constexpr (!kKeep) {  // (a lane reads what it has written)
      weights[2u * c * lanes] = make_float4(w[0][0], w[0][1], w[0][2], w[0][3]);
      weights[(2u * c + 1u) * lanes] = make_float4(w[0][4], w[0][5], w[0][6], w[0][7]);
    }
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) dw[c][i] = db[c][i] = 0.0f;
  }
  const float per = 1.0f / (float)p.cols;
  NormIn<TYPE, CODES> next[C];
  float2 next_stats;
  const uint32_t step = gridDim.x * kBunch;
  uint32_t row = blockIdx.x * kBunch + (LANES ? threadIdx.x / lanes : 0u);
  const auto fetch = [&](uint32_t r) {
    if (even) {
#pragma unroll
      for (uint32_t c = 0; c < C; ++c) next[c].load(p, true, r, col[c], r < p.rows ? left[c] : 0u);
    } else {
#pragma unroll
      for (uint32_t c = 0; c < C; ++c) next[c].load(p, false, r, col[c], r < p.rows ? left[c] : 0u);
    }
    next_stats = r < p.rows ? p.stats[r] : make_float2(0.0f, 0.0f);
  };
  if constexpr (kAhead) fetch(row);
  // (all lanes of a workgroup go round as often: its last rows may be none)
  for (uint32_t first = blockIdx.x * kBunch; first < p.rows; first += step, row += step) {
    if constexpr (!kAhead) fetch(row);
    float g[C][8], xh[C][8];
    const float mean = next_stats.x, rstd = next_stats.y;
    const bool live = row < p.rows;
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) next[c].get(g[c], xh[c]);
    if constexpr (kAhead) {
      if (first + step < p.rows) fetch(row + step);
    }
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) {
      const uint32_t at = kKeep ? c : 0u;
      if constexpr (!kKeep) {
        const float4 lo = weights[2u * c * lanes], hi = weights[(2u * c + 1u) * lanes];
        w[0][0] = lo.x; w[0][1] = lo.y; w[0][2] = lo.z; w[0][3] = lo.w;
        w[0][4] = hi.x; w[0][5] = hi.y; w[0][6] = hi.z; w[0][7] = hi.w;
      }
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) {
        const float dy = g[c][i];
        xh[c][i] = (xh[c][i] - mean) * rstd;  // (columns that are not there: dy is 0, and nothing of theirs is kept)
        dw[c][i] = fmaf(dy, xh[c][i], dw[c][i]);
        db[c][i] += dy;
        g[c][i] = dy * w[at][i];
        s[0] += g[c][i];
        s[1] = fmaf(g[c][i], xh[c][i], s[1]);
      }
    }
    row_sums<LANES, 2>(s, lds, &turn);
    const float a = s[0] * per, b = s[1] * per;
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) {
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) g[c][i] = (g[c][i] - fmaf(xh[c][i], b, a)) * rstd;
      Octet<TYPE> o;
      o.set(g[c]);
      if (p.dx.at) {
        if (even) o.template store_even<true>(p.dx.at, (uint64_t)row * p.dx.stride + col[c], live ? left[c] : 0u);
        else o.store(p.dx.at, (uint64_t)row * p.dx.stride + col[c], live ? left[c] : 0u);
      }
    }
  }
  if (!p.partial) return;
  float* out = p.partial + (uint64_t)blockIdx.x * 2u * p.cols;
  if constexpr (LANES == 0) {
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) {
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) {
        if (i < left[c]) {
          out[col[c] + i] = dw[c][i];
          out[p.cols + col[c] + i] = db[c][i];
        }
      }
    }
  } else {
    // [which][bunch][LANES * C * 8]
    static_assert(kKeep, "");  // (the weight would be where the sums go)
    constexpr uint32_t kWide = (LANES ? LANES : 1u) * C * 8u;
    const uint32_t slot = threadIdx.x / lanes;
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) {
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) {
        sums[slot * kWide + col[c] + i] = dw[c][i];
        sums[(kBunch + slot) * kWide + col[c] + i] = db[c][i];
      }
    }
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < 2u * kWide; t += kThreads) {
      const uint32_t which = t / kWide, at = t % kWide;
      if (at >= p.cols) continue;
      float v = 0.0f;
      for (uint32_t k = 0; k < kBunch; ++k) v += sums[(which * kBunch + k) * kWide + at];
      out[which * p.cols + at] = v;
    }
  }
}

// rows of any length: dx
template <uint32_t TYPE, bool CODES>
__global__ __launch_bounds__(1024) void norm_backward_pieces_kernel(NormArgs p) {
  __shared__ float lds[64];
  uint32_t turn = 0;
  const uint32_t row = blockIdx.x;
  const float2 stats = p.stats[row];
  const float per = 1.0f / (float)p.cols;
  float s[2] = {0.0f, 0.0f};
  for (uint32_t col = threadIdx.x * 8u; col < p.cols; col += 8192u) {
    NormIn<TYPE, CODES> in;
    float g[8], v[8], w[8];
    in.load(p, false, row, col, p.cols - col);
    in.get(g, v);
    load_params<TYPE>(p.wtype, p.weight, false, col, p.cols - col, 1.0f, w);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
      g[i] *= w[i];
      s[0] += g[i];
      s[1] = fmaf(g[i], (v[i] - stats.x) * stats.y, s[1]);
    }
  }
  row_sums<0, 2>(s, lds, &turn);
  for (uint32_t col = threadIdx.x * 8u; col < p.cols; col += 8192u) {
    NormIn<TYPE, CODES> in;
    float g[8], v[8], w[8];
    in.load(p, false, row, col, p.cols - col);
    in.get(g, v);
    load_params<TYPE>(p.wtype, p.weight, false, col, p.cols - col, 1.0f, w);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) g[i] = (g[i] * w[i] - fmaf((v[i] - stats.x) * stats.y, s[1] * per, s[0] * per)) * stats.y;
    Octet<TYPE> o;
    o.set(g);
    o.store(p.dx.at, (uint64_t)row * p.dx.stride + col, p.cols - col);
  }
}
// ... and the parameters' gradients: a workgroup takes 2048 columns of every P-th row
template <uint32_t TYPE, bool CODES>
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(NormArgs p) {
  const uint32_t strips = (p.cols + 2047u) / 2048u;
  const uint32_t part = blockIdx.x / strips, col = (blockIdx.x % strips) * 2048u + threadIdx.x * 8u;
  if (col >= p.cols) return;
  const uint32_t left = p.cols - col;
  float dw[8], db[8];
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) dw[i] = db[i] = 0.0f;
  for (uint32_t row = part; row < p.rows; row += p.partials) {
    NormIn<TYPE, CODES> in;
    float g[8], v[8];
    in.load(p, false, row, col, left);
    in.get(g, v);
    const float2 stats = p.stats[row];
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
      dw[i] = fmaf(g[i], (v[i] - stats.x) * stats.y, dw[i]);
      db[i] += g[i];
    }
  }
  float* out = p.partial + (uint64_t)part * 2u * p.cols + col;
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) {
    if (i < left) {
      out[i] = dw[i];
      out[p.cols + i] = db[i];
    }
  }
}

// ------------------------------------------------------------------ sums of the workgroups' sums
// 64 columns at a time, sixteen wavefronts that take every sixteenth of the partial sums each.  Workgroups go round where a launch does not take one for every 64 columns.
__global__ __launch_bounds__(1024) void reduce_kernel(ReduceArgs p) {
  __shared__ float sums[16][kReduceCols];
  const uint32_t lane = threadIdx.x % kReduceCols, wave = threadIdx.x / kReduceCols;
  const uint32_t tiles = (p.cols + kReduceCols - 1u) / kReduceCols;
  for (uint32_t at = blockIdx.x; at < tiles * p.parts; at += gridDim.x) {
    const uint32_t which = at / tiles, col = (at % tiles) * kReduceCols + lane;
    if (p.out[which] == nullptr) continue;
    if (at != blockIdx.x) __syncthreads();  // (the sums of the round before have been read)
    float v = 0.0f;
    if (col < p.cols) {
      const float* from = p.partial + (uint64_t)which * p.cols + col;
      const uint64_t apart = (uint64_t)p.parts * p.cols;
      uint32_t k = wave;
      for (; k + 48u < p.partials; k += 64u) {
        const float a = from[k * apart], b = from[(k + 16u) * apart], c = from[(k + 32u) * apart], d = from[(k + 48u) * apart];
        v += (a + b) + (c + d);
      }
      for (; k < p.partials; k += 16u) v += from[k * apart];
    }
    sums[wave][lane] = v;
    __syncthreads();
    if (wave == 0u && col < p.cols) {
#pragma unroll
      for (uint32_t k = 1; k < 16u; ++k) v += sums[k][lane];
      store1(p.type, p.out[which], col, v);
    }
  }
}
ReduceFn reduce_fn() { return reduce_kernel; }

// ------------------------------------------------------------------ 8-bit rows by themselves
// Sixteen lanes a group of 128 values, four groups one after the other
template <uint32_t TYPE, bool RESTORE>
__global__ __launch_bounds__(kThreads) void rows8_kernel(Rows8Args p) {
  const uint64_t unit = (uint64_t)blockIdx.x * (kThreads / kR8Lanes * kR8Units) + threadIdx.x / kR8Lanes;
  uint32_t row = (uint32_t)(unit / p.blob.groups), group = (uint32_t)(unit % p.blob.groups);
  const uint32_t in = threadIdx.x % kR8Lanes * 8u;
  const bool even = p.cols % 8u == 0u;
#pragma unroll
  for (uint32_t u = 0; u < kR8Units; ++u) {
    const uint32_t col = group * kR8Group + in, left = row < p.rows ? left_of(p.cols, col) : 0u;
    Octet<TYPE> o;
    float v[8];
    if constexpr (RESTORE) {
      if (left) {
        restore8(*reinterpret_cast<const uint2*>(p.blob.codes + (uint64_t)row * p.blob.pitch + col), p.blob.scales[(uint64_t)row * p.blob.groups + group], v);
        o.set(v);
        o.store(p.m.at, (uint64_t)row * p.m.stride + col, left);
      }
    } else {
      if (even) o.template load_even<true>(p.m.at, (uint64_t)row * p.m.stride + col, left);
      else o.load(p.m.at, (uint64_t)row * p.m.stride, col, left);
      o.get(v);
      write_group(p.blob, row, col, v, left != 0u);
    }
    row += p.step_rows;
    group += p.step_groups;
    if (group >= p.blob.groups) {
      group -= p.blob.groups;
      ++row;
    }
  }
}
Rows8Fn rows8_compress_fn(uint32_t type) {
  return type == kTypeF32 ? rows8_kernel<kTypeF32, false> : type == kTypeF16 ? rows8_kernel<kTypeF16, false> : rows8_kernel<kTypeBf16, false>;
}
Rows8Fn rows8_restore_fn(uint32_t type) {
  return type == kTypeF32 ? rows8_kernel<kTypeF32, true> : type == kTypeF16 ? rows8_kernel<kTypeF16, true> : rows8_kernel<kTypeBf16, true>;
}

template <uint32_t TYPE, bool CODES, bool EVEN>
static NormFn forward_of(NormShape s) {
  if (s.octets == 0) return norm_forward_pieces_kernel<TYPE, CODES>;
  if (s.lanes == 16) return norm_forward_kernel<TYPE, 16, 1, CODES, EVEN>;
  if (s.lanes == 32) return norm_forward_kernel<TYPE, 32, 1, CODES, EVEN>;
  if (s.lanes == 64) return s.octets == 1 ? norm_forward_kernel<TYPE, 64, 1, CODES, EVEN> : norm_forward_kernel<TYPE, 64, 2, CODES, EVEN>;
  return s.octets == 1 ? norm_forward_kernel<TYPE, 0, 1, CODES, EVEN> : s.octets == 2 ? norm_forward_kernel<TYPE, 0, 2, CODES, EVEN> : norm_forward_kernel<TYPE, 0, 4, CODES, EVEN>;
}
template <uint32_t TYPE>
static NormFn forward_by(NormShape s, bool codes, bool even) {
  if (codes) return even ? forward_of<TYPE, true, true>(s) : forward_of<TYPE, true, false>(s);
  return even ? forward_of<TYPE, false, true>(s) : forward_of<TYPE, false, false>(s);
}
NormFn norm_forward_fn(uint32_t type, NormShape s, bool codes, bool even) {
  return type == kTypeF32 ? forward_by<kTypeF32>(s, codes, even) : type == kTypeF16 ? forward_by<kTypeF16>(s, codes, even) : forward_by<kTypeBf16>(s, codes, even);
}
template <uint32_t TYPE, bool CODES, bool EVEN>
static NormFn backward_of(NormShape s) {
  if (s.octets == 0) return norm_backward_pieces_kernel<TYPE, CODES>;
  if (s.lanes == 16) return norm_backward_kernel<TYPE, 16, 1, CODES, EVEN>;
  if (s.lanes == 32) return norm_backward_kernel<TYPE, 32, 1, CODES, EVEN>;
  if (s.lanes == 64) return s.octets == 1 ? norm_backward_kernel<TYPE, 64, 1, CODES, EVEN> : norm_backward_kernel<TYPE, 64, 2, CODES, EVEN>;
  return s.octets == 1 ? norm_backward_kernel<TYPE, 0, 1, CODES, EVEN> : s.octets == 2 ? norm_backward_kernel<TYPE, 0, 2, CODES, EVEN> : norm_backward_kernel<TYPE, 0, 4, CODES, EVEN>;
}
template <uint32_t TYPE>
static NormFn backward_by(NormShape s, bool codes, bool even) {
  if (codes) return backward_of<TYPE, true, true>(s);
  return even ? backward_of<TYPE, false, true>(s) : backward_of<TYPE, false, false>(s);
}
NormFn norm_backward_fn(uint32_t type, NormShape s, bool codes, bool even) {
  return type == kTypeF32 ? backward_by<kTypeF32>(s, codes, even) : type == kTypeF16 ? backward_by<kTypeF16>(s, codes, even) : backward_by<kTypeBf16>(s, codes, even);
}
NormFn norm_columns_fn(uint32_t type, bool codes) {
  if (type == kTypeF32) return codes ? norm_columns_kernel<kTypeF32, true> : norm_columns_kernel<kTypeF32, false>;
  if (type == kTypeF16) return codes ? norm_columns_kernel<kTypeF16, true> : norm_columns_kernel<kTypeF16, false>;
  return codes ? norm_columns_kernel<kTypeBf16, true> : norm_columns_kernel<kTypeBf16, false>;
}

}  // namespace adacc
