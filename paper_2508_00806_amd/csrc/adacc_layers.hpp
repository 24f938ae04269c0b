// The layers whose saved activations are compressed: what the kernels of layer norm, activations and products share with the host code.
//
// 8-bit rows: a row is cut into groups of 128 values from its start, the last one may be short.  M = max|x| of a group (binary32), inv = 127 / M held at the
// largest finite number, code = nearest integer of binary32(x * inv), ties to even, in [-127, 127], S = M / 127, or, for an M next to binary32's largest, the largest number
// whose 127-fold is finite.  Restored value = binary32(S * code).  M = 0: codes 0, S = 0.  An Inf or NaN in the group: S = NaN, whatever the codes.  (Eq. 2 with the full range of codes, as
// ADACC_SCALE_FULLRANGE has it: nothing is cut off, every value is within half a step but in groups below 2^-119, whose values are within M; the scale is one division and so is the inverse.)
#pragma once

#include "adacc_common.hpp"

namespace adacc {

constexpr uint32_t kR8Group = 128;  // values per scale: 16 lanes of 8
constexpr uint32_t kR8Lanes = 16;

enum : uint32_t { kTypeBf16 = 0, kTypeF16 = 1, kTypeF32 = 2 };
enum : uint32_t { kActNone = 0, kActGelu = 1, kActGeluTanh = 2, kActSilu = 3 };

// 8-bit rows in memory: the code of column c at c + row * pitch, pitch a multiple of 16; scales [rows][groups].  codes == nullptr: none
struct Rows8 {
  uint8_t* codes;
  float* scales;
  uint64_t pitch;
  uint32_t groups;  // of a row
};

// A matrix whose rows lie in one piece each, at any element's address
struct Strided {
  void* at;
  uint64_t stride;  // elements
};

struct Rows8Args {
  uint32_t rows, cols;
  uint32_t step_rows, step_groups;  // 16 groups further on, in rows and groups
  Strided m;
  Rows8 blob;
};

struct NormArgs {
  uint32_t rows, cols;
  uint32_t wtype;     // of weight, bias and their gradients
  uint32_t partials;  // workgroups of the backward pass
  float eps;
  Strided x, y;       // y: forward
  Strided dy, dx;     // backward
  Rows8 blob;
  const void* weight;
  const void* bias;
  float2* stats;      // mean, 1 / sigma of the rows
  float* partial;     // [partials][2][cols]: sums over a workgroup's rows of dy * xh, and of dy
};

struct ActArgs {
  uint32_t rows, cols;
  uint32_t step_rows, step_groups;
  uint32_t partials;
  Strided a, up;          // up.at == nullptr: not gated
  Strided y;              // forward: the result; backward: its gradient
  Strided da, dup;        // backward
  Rows8 a8, up8;          // forward: written; backward: read in the place of a and up
  float* partial;         // [partials][cols]: sums of da over a workgroup's rows
};

struct ReduceArgs {
  uint32_t cols, partials;
  uint32_t type;       // of the results
  uint32_t parts;      // partial[partials][parts][cols], a result for each
  const float* partial;
  void* out[2];        // nullptr: not wanted
};

typedef void (*Rows8Fn)(Rows8Args);
typedef void (*NormFn)(NormArgs);
typedef void (*ActFn)(ActArgs);
typedef void (*ReduceFn)(ReduceArgs);

Rows8Fn rows8_compress_fn(uint32_t type);
Rows8Fn rows8_restore_fn(uint32_t type);
constexpr uint32_t kR8Units = 4;  // groups of 128 that a lane takes part in, one after the other (a workgroup: 16 * 4)

// how a row of layer norm is shared out
struct NormShape {
  uint32_t lanes;  // of a row: 16, 32 or 64 of a wavefront, or those of a whole workgroup
  uint32_t octets; // a lane's: 1, 2 or 4; 0: rows of any length, in pieces
};
constexpr uint32_t kNormThreads = 512;
constexpr uint32_t kNormWidest = kNormThreads * 32;  // columns that a workgroup holds in registers, four octets a lane
// even: rows are multiples of eight values long, so that a lane's eight are there or not.  Kernels of their own: with both ways in one, 32768 x 2048 takes 146 us forward and backward instead of 124, the GELU of
// 8192 x 16384 239 instead of 222 (what the ends of other rows need stays in the way of the loads).  The norm's backward pass from codes is one kernel for both, which is faster there.
NormFn norm_forward_fn(uint32_t type, NormShape shape, bool codes, bool even);
NormFn norm_backward_fn(uint32_t type, NormShape shape, bool codes, bool even);
NormFn norm_columns_fn(uint32_t type, bool codes);  // the parameters' gradients of rows of any length
ReduceFn reduce_fn();
constexpr uint32_t kReduceCols = 64;

ActFn act_forward_fn(uint32_t type, uint32_t kind, bool gated, bool codes, bool even);
ActFn act_backward_fn(uint32_t type, uint32_t kind, bool gated, bool codes, bool even);
ActFn act_columns_fn(uint32_t type, uint32_t kind, bool codes);  // not gated, with the sums of its columns; kActNone: the sums alone

// ---- products: out[i][j] = sum over c of A(i, c) * B(j, c)
// How an operand lies in memory: kAlong [i][c], the contraction along the rows; kAcross [c][i], the rows along the contraction; kAcross8 the same as 8-bit rows
enum : uint32_t { kAlong = 0, kAcross = 1, kAcross8 = 2 };

struct Epilogue {
  uint32_t m, n;         // of the result
  uint32_t act;
  uint32_t btype;
  const void* bias;      // nullptr: none
  Strided residual;      // at == nullptr: none
  Strided out;
  Strided pre;           // what the activation was given; at == nullptr: not wanted
  Rows8 pre8;            // the same in 8 bits
};
struct ProductArgs {
  Epilogue e;
  Strided a, b;
  Rows8 b8;
  uint32_t k;                  // length of the contraction
  uint32_t m_tiles, n_tiles;
  uint32_t splits, split_steps;  // the contraction in parts of so many steps of 64
  float* partial;              // splits > 1: [splits][m][n]
};
struct JoinArgs {
  Epilogue e;
  const float* partial;
  uint32_t splits;
};
typedef void (*ProductFn)(ProductArgs);
typedef void (*JoinFn)(JoinArgs);
typedef void (*PadFn)(const uint16_t* src, uint64_t stride, uint32_t rows, uint32_t cols, uint4* dst);
PadFn pad_fn();
constexpr uint32_t kLinShort = 8;  // rows of fewer values are copied to rows of eight
constexpr uint32_t kLinStep = 64;
ProductFn product_fn(uint32_t type, uint32_t a_mode, uint32_t b_mode, uint32_t tile);
uint32_t product_lds(uint32_t tile);
JoinFn join_fn(uint32_t type);
ProductFn linear_few_fn(uint32_t type, uint32_t ms, uint32_t ns);  // 16 * ms rows by 16 * ns columns a workgroup: (1, 1), (2, 1), (2, 4)

#if defined(__HIPCC__)
// ------------------------------------------------------------------ device
typedef uint32_t u4_any __attribute__((ext_vector_type(4), aligned(1)));  // loads and stores at any address
typedef uint32_t u2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef __bf16 lay_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 lay_f16x2 __attribute__((ext_vector_type(2)));
typedef float lay_f32x2 __attribute__((ext_vector_type(2)));

template <uint32_t TYPE>
constexpr uint32_t kSizeOf = TYPE == kTypeF32 ? 4u : 2u;

template <uint32_t TYPE>
__device__ __forceinline__ uint32_t narrow2(float lo, float hi) {  // round to nearest even
  const lay_f32x2 v = {lo, hi};
  if constexpr (TYPE == kTypeBf16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, lay_bf16x2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, lay_f16x2));
}
template <uint32_t TYPE>
__device__ __forceinline__ float widen_lo(uint32_t w) {
  if constexpr (TYPE == kTypeBf16) return __uint_as_float(w << 16);
  else return (float)__builtin_bit_cast(_Float16, (uint16_t)w);
}
template <uint32_t TYPE>
__device__ __forceinline__ float widen_hi(uint32_t w) {
  if constexpr (TYPE == kTypeBf16) return __uint_as_float(w & 0xFFFF0000u);
  else return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16));
}
template <uint32_t TYPE>
__device__ __forceinline__ float load1(const void* p, uint64_t at) {
  if constexpr (TYPE == kTypeF32) return static_cast<const float*>(p)[at];
  else return widen_lo<TYPE>(static_cast<const uint16_t*>(p)[at]);
}
template <uint32_t TYPE>
__device__ __forceinline__ void store1(void* p, uint64_t at, float v) {
  if constexpr (TYPE == kTypeF32) static_cast<float*>(p)[at] = v;
  else static_cast<uint16_t*>(p)[at] = (uint16_t)narrow2<TYPE>(v, v);
}
// What an activation is given, as it is kept in 16 bits: finite values beyond the type's range at its end, where every slope is what it is further out.  (As an infinity, which has no
// slope, a finite result would have NaN for its gradient.)
template <uint32_t TYPE>
__device__ __forceinline__ float held(float v) {
  constexpr float kMost = TYPE == kTypeF16 ? 65504.0f : 0x1.FEp127f;
  return __builtin_isfinite(v) ? __builtin_amdgcn_fmed3f(v, -kMost, kMost) : v;
}
__device__ __forceinline__ float load1(uint32_t type, const void* p, uint64_t at) {
  return type == kTypeF32 ? load1<kTypeF32>(p, at) : type == kTypeF16 ? load1<kTypeF16>(p, at) : load1<kTypeBf16>(p, at);
}
__device__ __forceinline__ void store1(uint32_t type, void* p, uint64_t at, float v) {
  if (type == kTypeF32) store1<kTypeF32>(p, at, v);
  else if (type == kTypeF16) store1<kTypeF16>(p, at, v);
  else store1<kTypeBf16>(p, at, v);
}

// Exchanges within 16 lanes, in the vector unit (a shuffle through LDS takes a hundred cycles, and four follow each other).  Each joins halves that are uniform by then, so that all
// lanes come to the same sum: lanes i and i ^ 1, i ^ 2, then 7 - i in eight, 15 - i in sixteen.
constexpr int kSwapPairs = 0xB1, kSwapTwos = 0x4E, kMirrorEight = 0x141, kMirrorSixteen = 0x140;
template <int HOW>
__device__ __forceinline__ uint32_t cross(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, HOW, 0xF, 0xF, true);
}
template <int HOW>
__device__ __forceinline__ float cross(float v) {
  return __uint_as_float(cross<HOW>(__float_as_uint(v)));
}
// sum over LANES (16, 32 or 64) adjacent lanes, the same in all of them
template <uint32_t LANES>
__device__ __forceinline__ float lane_sum(float v) {
  v += cross<kSwapPairs>(v);
  v += cross<kSwapTwos>(v);
  v += cross<kMirrorEight>(v);
  v += cross<kMirrorSixteen>(v);
  if constexpr (LANES >= 32u) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (LANES >= 64u) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// Eight adjacent values of a row, as they are in memory.  `left` of them exist; the others are zeros, and nothing of their places is read or written.
template <uint32_t TYPE>
struct Octet {
  u4_any w[TYPE == kTypeF32 ? 2 : 1];
  // values col to col + 7 of the row that begins at `at`.  At a row's end eight values that are there are read, and moved
  __device__ __forceinline__ void load(const void* p, uint64_t at, uint32_t col, uint32_t left) {
    const uint8_t* from = static_cast<const uint8_t*>(p) + (at + col) * kSizeOf<TYPE>;
    asm volatile("" : "+v"(left));  // (what follows of it is worked out here, not kept in registers over a kernel's loop)
    const uint32_t back = left < 8u ? 8u - left : 0u;
    constexpr uint32_t kWords = TYPE == kTypeF32 ? 8u : 4u;
    uint32_t t[kWords];
    load_even<false>(from - back * kSizeOf<TYPE>, 0u, col >= 8u || back == 0u ? left : 0u);
    if (back == 0u) return;
#pragma unroll
    for (uint32_t i = 0; i < kWords; ++i) t[i] = w[i / 4u][i % 4u];
    if (col >= 8u) {
      const uint32_t words = TYPE == kTypeF32 ? back : back / 2u;
#pragma unroll
      for (uint32_t by = 1u; by <= kWords; by *= 2u)
#pragma unroll
        for (uint32_t i = 0; i < kWords; ++i) t[i] = words & by ? (i + by < kWords ? t[i + by] : 0u) : t[i];
      if constexpr (TYPE != kTypeF32) {
#pragma unroll
        for (uint32_t i = 0; i < kWords; ++i) t[i] = back % 2u ? t[i] >> 16 | (i + 1u < kWords ? t[i + 1u] << 16 : 0u) : t[i];
      }
    } else {  // a row of fewer than eight: value by value, from the last one on (a loop, as this is seldom and would be most of the code)
#pragma unroll 1
      for (uint32_t i = left; i-- > 0u;) {
        if constexpr (TYPE == kTypeF32) {
#pragma unroll
          for (uint32_t k = kWords - 1u; k > 0u; --k) t[k] = t[k - 1u];
          t[0] = reinterpret_cast<const uint32_t*>(from)[i];
        } else {
#pragma unroll
          for (uint32_t k = kWords - 1u; k > 0u; --k) t[k] = t[k] << 16 | t[k - 1u] >> 16;
          t[0] = t[0] << 16 | reinterpret_cast<const uint16_t*>(from)[i];
        }
      }
    }
    w[0] = u4_any{t[0], t[1], t[2], t[3]};
    if constexpr (TYPE == kTypeF32) w[1] = u4_any{t[4], t[5], t[6], t[7]};
  }
  __device__ __forceinline__ void store(void* p, uint64_t at, uint32_t left) const {
    uint8_t* to = static_cast<uint8_t*>(p) + at * kSizeOf<TYPE>;
    if (left >= 8u) {
      *reinterpret_cast<u4_any*>(to) = w[0];
      if constexpr (TYPE == kTypeF32) *reinterpret_cast<u4_any*>(to + 16) = w[1];
      return;
    }
    constexpr uint32_t kWords = TYPE == kTypeF32 ? 8u : 4u;
    uint32_t t[kWords];
#pragma unroll
    for (uint32_t i = 0; i < kWords; ++i) t[i] = w[i / 4u][i % 4u];
#pragma unroll 1
    for (uint32_t i = 0; i < left; ++i) {
      if constexpr (TYPE == kTypeF32) {
        reinterpret_cast<uint32_t*>(to)[i] = t[0];
#pragma unroll
        for (uint32_t k = 0; k + 1u < kWords; ++k) t[k] = t[k + 1u];
      } else {
        reinterpret_cast<uint16_t*>(to)[i] = (uint16_t)t[0];
#pragma unroll
        for (uint32_t k = 0; k + 1u < kWords; ++k) t[k] = t[k] >> 16 | t[k + 1u] << 16;
        t[kWords - 1u] >>= 16;
      }
    }
  }
  // Where the rows are multiples of eight values long: all are there, or none.  (The loop above would part the loads of several octets.)  STREAM: with the streaming hint, for what is read
  // or written once
  template <bool STREAM>
  __device__ __forceinline__ void load_even(const void* p, uint64_t at, uint32_t left) {
    const u4_any* from = reinterpret_cast<const u4_any*>(static_cast<const uint8_t*>(p) + at * kSizeOf<TYPE>);
    w[0] = u4_any{0u, 0u, 0u, 0u};
    if constexpr (TYPE == kTypeF32) w[1] = w[0];
    if (left) {
      w[0] = STREAM ? __builtin_nontemporal_load(from) : *from;
      if constexpr (TYPE == kTypeF32) w[1] = STREAM ? __builtin_nontemporal_load(from + 1) : from[1];
    }
  }
  template <bool STREAM>
  __device__ __forceinline__ void store_even(void* p, uint64_t at, uint32_t left) const {
    u4_any* to = reinterpret_cast<u4_any*>(static_cast<uint8_t*>(p) + at * kSizeOf<TYPE>);
    if (left) {
      if constexpr (STREAM) {
        __builtin_nontemporal_store(w[0], to);
        if constexpr (TYPE == kTypeF32) __builtin_nontemporal_store(w[1], to + 1);
      } else {
        to[0] = w[0];
        if constexpr (TYPE == kTypeF32) to[1] = w[1];
      }
    }
  }
  // Keeps the compiler from widening the values where they are loaded, which takes twice the registers and waits for the load
  __device__ __forceinline__ void hold() {
#pragma unroll
    for (uint32_t i = 0; i < (TYPE == kTypeF32 ? 8u : 4u); ++i) {
      uint32_t t = w[i / 4u][i % 4u];
      asm volatile("" : "+v"(t));
      w[i / 4u][i % 4u] = t;
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    if constexpr (TYPE == kTypeF32) {
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) v[i] = __uint_as_float(w[i / 4u][i % 4u]);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 4u; ++i) {
        v[2 * i] = widen_lo<TYPE>(w[0][i]);
        v[2 * i + 1] = widen_hi<TYPE>(w[0][i]);
      }
    }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    if constexpr (TYPE == kTypeF32) {
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) w[i / 4u][i % 4u] = __float_as_uint(v[i]);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 4u; ++i) w[0][i] = narrow2<TYPE>(v[2 * i], v[2 * i + 1]);
    }
  }
};

// The scale of a group and the factor to its codes, from the group's largest magnitude as a bit pattern
struct Scale8 {
  float scale, inverse;
};
constexpr float kScaleMost = 0x1.0204060000000p+121f;  // the largest whose 127-fold is finite
__device__ __forceinline__ Scale8 scale8(uint32_t most) {
  Scale8 s;
  if (most >= 0x7F800000u) {
    s.scale = __uint_as_float(0x7FC00000u);
    s.inverse = 0.0f;
  } else if (most == 0u) {
    s.scale = s.inverse = 0.0f;
  } else {
    const float m = __uint_as_float(most);
    s.scale = fminf(m / 127.0f, kScaleMost);
    s.inverse = fminf(127.0f / m, 3.402823466e38f);
  }
  return s;
}
__device__ __forceinline__ uint32_t most_of(const float (&v)[8]) {
  uint32_t m = 0u;
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return m;
}
// over the 16 lanes of a group
__device__ __forceinline__ uint32_t most_of_group(uint32_t m) {
  m = max(m, cross<kSwapPairs>(m));
  m = max(m, cross<kSwapTwos>(m));
  m = max(m, cross<kMirrorEight>(m));
  return max(m, cross<kMirrorSixteen>(m));
}
// Codes of four values.  x * inv + 1.5 * 2^23 has the nearest integer in its low bits; the product is rounded on its own (no contraction).
constexpr float kCodeMagic = 12582912.0f;
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inverse) {
  const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b * inverse + kCodeMagic), __float_as_uint(a * inverse + kCodeMagic), 0x0C0C0400u);
  const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d * inverse + kCodeMagic), __float_as_uint(c * inverse + kCodeMagic), 0x04000C0Cu);
  return lo | hi;
}
__device__ __forceinline__ uint2 codes8(const float (&v)[8], const Scale8& s) {
  return make_uint2(codes4(v[0], v[1], v[2], v[3], s.inverse), codes4(v[4], v[5], v[6], v[7], s.inverse));
}
__device__ __forceinline__ void restore8(uint2 c, float scale, float (&v)[8]) {
#pragma unroll
  for (uint32_t i = 0; i < 4u; ++i) {
    v[i] = (float)(int8_t)(c.x >> (8u * i)) * scale;
    v[4 + i] = (float)(int8_t)(c.y >> (8u * i)) * scale;
  }
}

// One lane's part of writing a group of 8-bit rows: eight codes, and the scale by the group's first lane
__device__ __forceinline__ void write_group(const Rows8& b, uint32_t row, uint32_t col, const float (&v)[8], bool live) {
  const Scale8 s = scale8(most_of_group(most_of(v)));
  if (live) {
    *reinterpret_cast<uint2*>(b.codes + (uint64_t)row * b.pitch + col) = codes8(v, s);
    if (col % kR8Group == 0u) b.scales[(uint64_t)row * b.groups + col / kR8Group] = s.scale;
  }
}

// ------------------------------------------------------------------ activations
// Phi(-|x|), the normal distribution's tail, as a power of two:  2^-P(|x|), P = -log2 Phi(-|x|), which is smooth, as a polynomial fitted on [0, 14] for the tail's relative error, which is below
// 1.9e-5 up to |x| = 6 and below 1.5e-4 beyond, as binary32 evaluates it: a thirteenth of half a step of bfloat16 there, which has such results down to |x| = 13, a twenty-fifth of binary16's,
// whose results end at 5.7.  (Eight coefficients for [0, 10] gave those of bfloat16 in steps too many: 9 % at -10, 63 % at -12.)  It grows from there on.  Ten products and one exponential: 16 cycles
// of the vector unit's quarter-rate part where exp(-x^2 / 2) R(1 / (1 + c |x|)) has 32, and a product's results wait for nothing else.
__device__ __forceinline__ float gelu_tail(float x) {
  const float u = fabsf(x);
  float p = 2.0191617267073525e-09f;
  p = fmaf(p, u, -1.4789505087264843e-07f);
  p = fmaf(p, u, 4.734183221444255e-06f);
  p = fmaf(p, u, -8.773975423537195e-05f);
  p = fmaf(p, u, 0.0010561312083154917f);
  p = fmaf(p, u, -0.008840742520987988f);
  p = fmaf(p, u, 0.05443132296204567f);
  p = fmaf(p, u, 0.4581434428691864f);
  p = fmaf(p, u, 1.1513323783874512f);
  p = fmaf(p, u, 0.9999920129776001f);
  return __builtin_amdgcn_exp2f(-p);
}
// For binary32: exp(-x^2 / 2) R(t), t = 1 / (1 + c |x|), R = erfcx(|x| / sqrt 2) / 2 as a polynomial without constant term, fitted for the least largest relative error on [0, 40]: 3.9e-7 as
// binary32 evaluates it.  e: that exponential, whose argument's roundings add x^2 2^-23 at most (2.4e-6 of the tail at 4.5, 2e-5 at 13)
__device__ __forceinline__ float gelu_tail_fine(float x, float e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.277f, fabsf(x), 1.0f));
  float r = 0.02679574303328991f;
  r = fmaf(r, t, -0.10612984746694565f);
  r = fmaf(r, t, 0.1184319406747818f);
  r = fmaf(r, t, -0.02626964822411537f);
  r = fmaf(r, t, 0.0830615684390068f);
  r = fmaf(r, t, 0.08055075258016586f);
  r = fmaf(r, t, 0.10257980972528458f);
  r = fmaf(r, t, 0.11047180742025375f);
  r = fmaf(r, t, 0.11050789803266525f);
  return e * (r * t);
}
constexpr float kLog2E = 1.44269504089f;
constexpr float kTanhTwice = 1.59576912161f;  // 2 sqrt(2 / pi)
constexpr float kTanhCube = 0.044715f;

// value = x * share, slope = d value / dx.  A share below 2^-126 is 0: the exponential and the reciprocal have no results below that.
template <uint32_t KIND, bool FINE, bool SLOPE>
__device__ __forceinline__ void activate(float x, float* value, float* slope) {
  if constexpr (KIND == kActNone) {
    *value = x;
    if constexpr (SLOPE) *slope = 1.0f;
  } else if constexpr (KIND == kActGelu) {
    float e = 0.0f;
    if constexpr (FINE || SLOPE) e = __builtin_amdgcn_exp2f(x * x * (-0.5f * kLog2E));
    const float tail = FINE ? gelu_tail_fine(x, e) : gelu_tail(x);
    const float share = x < 0.0f ? tail : 1.0f - tail;  // (NaN stays: the tail is NaN)
    *value = x * share;
    if constexpr (SLOPE) *slope = fmaf(x * 0.3989422804f, e, share);
  } else {
    // beyond 64 the share is 0 or 1; the cube may overflow, of which the slope would become NaN
    const float u = SLOPE && KIND == kActGeluTanh && fabsf(x) > 64.0f ? copysignf(64.0f, x) : x;
    const float z = KIND == kActSilu ? u : u * kTanhTwice * fmaf(kTanhCube * u, u, 1.0f);
    const float share = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -kLog2E));
    *value = x * share;
    if constexpr (SLOPE) {
      const float dz = KIND == kActSilu ? u : u * kTanhTwice * fmaf(3.0f * kTanhCube * u, u, 1.0f);  // x * dz/dx
      *slope = share * fmaf(dz, 1.0f - share, 1.0f);
    }
  }
}
// ------------------------------------------------------------------ what follows a product
// The bias of eight columns; zeros where there is none
template <uint32_t TYPE>
__device__ __forceinline__ void load_bias(const Epilogue& e, uint32_t col, uint32_t left, float (&b)[8]) {
  if (!e.bias) {
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) b[i] = 0.0f;
  } else if (e.btype == kTypeF32) {
    Octet<kTypeF32> o;
    o.load(e.bias, 0u, col, left);
    o.get(b);
  } else {
    Octet<TYPE> o;
    o.load(e.bias, 0u, col, left);
    o.get(b);
  }
}
template <uint32_t TYPE, uint32_t KIND, uint32_t N>
__device__ __forceinline__ void activate_octets(float (&v)[N][8]) {
  float none;
#pragma unroll
  for (uint32_t n = 0; n < N; ++n)
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) activate<KIND, false, false>(v[n][i], &v[n][i], &none);
}
// N times eight sums to results, in rows row[n], the same eight columns of each, `left[n]` of which are there.  Sixteen lanes hold 128 adjacent columns (where the activation's input is
// kept in 8 bits, all of them take part).
template <uint32_t TYPE, uint32_t N>
__device__ __forceinline__ void finish(const Epilogue& e, const uint32_t (&row)[N], uint32_t col, const uint32_t (&left)[N], const float (&bias)[8], float (&v)[N][8]) {
  Octet<TYPE> r[N];
  if (e.residual.at) {
#pragma unroll
    for (uint32_t n = 0; n < N; ++n) r[n].load(e.residual.at, (uint64_t)row[n] * e.residual.stride, col, left[n]);
  }
#pragma unroll
  for (uint32_t n = 0; n < N; ++n)
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) v[n][i] += bias[i];
  if (e.act != kActNone) {
    if (e.pre8.codes) {
#pragma unroll
      for (uint32_t n = 0; n < N; ++n) {
        if (left[n] < 8u) {  // columns that are not there: sums of whatever the tile held
#pragma unroll
          for (uint32_t i = 0; i < 8u; ++i) v[n][i] = i < left[n] ? v[n][i] : 0.0f;
        }
        write_group(e.pre8, row[n], col, v[n], left[n] != 0u);
      }
    } else if (e.pre.at) {
#pragma unroll
      for (uint32_t n = 0; n < N; ++n) {
        float w[8];
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) w[i] = held<TYPE>(v[n][i]);
        Octet<TYPE> o;
        o.set(w);
        o.store(e.pre.at, (uint64_t)row[n] * e.pre.stride + col, left[n]);
      }
    }
    if (e.act == kActGelu) activate_octets<TYPE, kActGelu>(v);
    else if (e.act == kActGeluTanh) activate_octets<TYPE, kActGeluTanh>(v);
    else activate_octets<TYPE, kActSilu>(v);
  }
#pragma unroll
  for (uint32_t n = 0; n < N; ++n) {
    if (e.residual.at) {
      float w[8];
      r[n].get(w);
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i) v[n][i] += w[i];
    }
    Octet<TYPE> o;
    o.set(v[n]);
    o.store(e.out.at, (uint64_t)row[n] * e.out.stride + col, left[n]);
  }
}
#endif

}  // namespace adacc
