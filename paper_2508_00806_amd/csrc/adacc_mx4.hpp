// Microscaled 4-bit floating point: what its kernels and the host code share.
//
// A matrix is cut into blocks of 32 consecutive values along its rows.  A block has one power of two 2^e, kept as the byte
// e + 127, and a 4-bit code per value: sign, and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  Value = code * 2^e.  (The element and
// scale formats of the OCP Microscaling specification 1.0, MXFP4: E2M1 and E8M0.)
//
// Blob: codes [steps][rows][64 bytes], a step being 128 columns (what two halves of the matrix instructions take), element 2j in the low
// nibble of byte j, zeros behind the row's end; scales [4 * steps][pitch], one byte for a block, the bytes of a block column
// next to each other.
//   Step by step, because a product's workgroup reads 64 bytes of each of its rows at a time: row by row those are halves of
// cache lines, and the loads of a tile of 256 x 256 take 1200 cycles a step; adjacent, 745 (1024 are the matrix instructions').
//   Block by block, so that the 32-bit word that a lane hands to the scaled matrix instruction holds the scales of four adjacent rows,
// one for each of the four tiles that the lane's operand registers belong to (the instruction picks a byte).  pitch is the number of
// rows, rounded up to 16; the bytes behind the last row are not read as scales of anything that is kept.
#pragma once

#include "adacc_common.hpp"

namespace adacc {

constexpr uint32_t kMxBlock = 32;        // values per scale
constexpr uint32_t kMxStep = 128;        // columns per step: codes of 64 bytes, 4 scales
constexpr uint32_t kMxStepBytes = 64;
constexpr uint32_t kMxTileRows = 128;    // rows of a workgroup of the compression, and what an expert's tokens are padded to across
constexpr uint32_t kMxWaveRows = 8;      // rows of a wavefront of the compression along the rows, and of the restoration
constexpr uint32_t kMxMaxGroups = 4096;
constexpr uint32_t kMxNanByte = 255;
// wavefronts of a workgroup of the product of few rows, at most: sixteen leave a lane 128 registers, eight 256
constexpr uint32_t mx4_few_waves(uint32_t ms) { return ms == 1 ? 16u : 8u; }

enum : uint32_t { kMxBf16 = 0, kMxF16 = 1, kMxF32 = 2, kMxReady = 3 };  // kMxReady: a left operand that is compressed already

// One compressed matrix
struct MxMatrix {
  uint8_t* codes;
  uint8_t* scales;
  uint64_t step_bytes;  // 64 * rows
  uint64_t pitch;
  uint32_t rows;
  uint32_t steps;
};

// Rows sorted by group: group g has the rows [offsets[g], offsets[g + 1]); offsets[0] counts as 0 and what lies behind
// offsets[groups] belongs to nothing.  The offsets are device data, which the host does not see: the kernels hold every one
// between 0 and the number of rows, so that none leads outside of a buffer.
struct MxGroups {
  const int32_t* offsets;  // nullptr: one group of all rows
  uint32_t groups;
  uint32_t rows;
};

struct MxCompressArgs {
  uint32_t first;  // workgroup of the call that the launch begins with
  const void* src;
  uint64_t row_stride, mat_stride;  // elements
  uint32_t mats, rows, cols;        // of one matrix; blob rows = mats * rows
  uint32_t fullrange;
  uint32_t row_tiles, col_tiles;
  MxGroups g;
  MxMatrix along;   // [mats * rows][cols]
  MxMatrix across;  // [mats * cols][rows], or [cols][padded positions] with groups
};

struct MxDecompressArgs {
  uint32_t first;  // as above
  MxMatrix m;
  uint32_t cols;
  void* dst;
  uint64_t row_stride;
  uint32_t col_tiles;
};

struct MxProductArgs {
  MxMatrix a;        // [rows of the output][contraction]
  MxMatrix b;        // [columns of the output, group after group][contraction]
  void* out;
  uint64_t out_stride;   // elements
  uint64_t out_group;    // gradient: elements between the matrices of two groups
  uint32_t out_type;
  uint32_t m, n;         // rows (of all groups) and columns of the output
  uint32_t m_tiles, n_tiles;
  MxGroups g;
  // few rows: the left operand as it is
  const void* x;
  uint64_t x_stride;
  uint32_t k;
  uint32_t fullrange;
};

typedef void (*MxCompressFn)(MxCompressArgs);
typedef void (*MxDecompressFn)(MxDecompressArgs);
typedef void (*MxProductFn)(MxProductArgs);
MxCompressFn mx4_compress_fn(uint32_t type, bool along, bool across, bool narrow);  // narrow: rows that a lane's load does not fit in; not for both at once
MxDecompressFn mx4_decompress_fn(uint32_t type);
MxProductFn mx4_product_fn(uint32_t tile, bool gradient);  // tile: 256, 128 or 64 rows and columns a workgroup
uint32_t mx4_product_lds(uint32_t tile);
MxProductFn mx4_few_fn(uint32_t ms, uint32_t ns, uint32_t src);  // 16 * ms rows by 16 * ns columns a workgroup; src: kMx* or kMxReady

#if defined(__HIPCC__)
// ------------------------------------------------------------------ device
__device__ __forceinline__ uint32_t mx_offset(const MxGroups& g, uint32_t i) {
  if (i == 0) return 0u;
  const int32_t o = g.offsets[i];
  return o < 0 ? 0u : ((uint32_t)o > g.rows ? g.rows : (uint32_t)o);
}

// The group that holds unit `unit`, where group i has ceil(rows_i / per) units (at least one if `least`, and the rows start at a
// multiple of 4 if `lower`).  Every lane of the wavefront takes part, 64 groups at a time.
struct MxPlace {
  uint32_t group;   // g.groups: behind the last one
  uint32_t unit;    // within the group
  uint32_t first;   // rows [first, last) of the group
  uint32_t last;
  uint32_t before;  // units of the groups before it
};
template <bool LOWER>
__device__ __forceinline__ MxPlace mx_place(const MxGroups& g, uint32_t unit, uint32_t per) {
  MxPlace p;
  if (g.offsets == nullptr) {
    const uint32_t n = (g.rows + per - 1u) / per;
    p.group = unit < n ? 0u : 1u;
    p.unit = unit; p.first = 0u; p.last = g.rows; p.before = 0u;
    return p;
  }
  const uint32_t lane = threadIdx.x % kWave;
  uint32_t base = 0u, tail = 0u;
  for (uint32_t g0 = 0; g0 < g.groups; g0 += kWave) {
    const uint32_t i = g0 + lane;
    uint32_t first = 0u, last = 0u;
    if (i < g.groups) { first = mx_offset(g, i); last = mx_offset(g, i + 1u); }
    if (last < first) last = first;
    const uint32_t from = LOWER ? first & ~3u : first;
    const uint32_t mine = last > first ? (last - from + per - 1u) / per : 0u;
    uint32_t sum = mine;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const uint32_t o = __shfl_up(sum, d);
      if (lane >= (uint32_t)d) sum += o;
    }
    const uint64_t hit = __ballot(base + sum > unit);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      p.group = g0 + (uint32_t)l;
      p.before = base + __shfl(sum - mine, l);
      p.unit = unit - p.before;
      p.first = __shfl(first, l);
      p.last = __shfl(last, l);
      p.group = __builtin_amdgcn_readfirstlane(p.group);
      p.before = __builtin_amdgcn_readfirstlane(p.before);
      p.unit = __builtin_amdgcn_readfirstlane(p.unit);
      p.first = __builtin_amdgcn_readfirstlane(p.first);
      p.last = __builtin_amdgcn_readfirstlane(p.last);
      return p;
    }
    base += __shfl(sum, kWave - 1);
    tail = mx_offset(g, g0 + kWave < g.groups ? g0 + kWave : g.groups);
  }
  p.group = g.groups;
  p.before = __builtin_amdgcn_readfirstlane(base);
  p.unit = unit - p.before;
  p.first = __builtin_amdgcn_readfirstlane(tail);
  p.last = g.rows;
  return p;
}

// How many units there are, those of the rows behind the last group included
template <bool LOWER>
__device__ __forceinline__ uint32_t mx_units(const MxGroups& g, uint32_t per) {
  const MxPlace p = mx_place<LOWER>(g, 0xFFFFFFFFu, per);
  if (g.offsets == nullptr) return (g.rows + per - 1u) / per;
  const uint32_t from = LOWER ? p.first & ~3u : p.first;
  return p.before + (p.last > p.first ? (p.last - from + per - 1u) / per : 0u);
}

typedef uint32_t mx_u4u __attribute__((ext_vector_type(4), aligned(1)));  // loads and stores at any address
typedef uint32_t mx_u2u __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t mx_u1u __attribute__((aligned(1)));
typedef uint16_t mx_h1u __attribute__((aligned(1)));

// The scale byte of a block whose largest magnitude has the binary32 pattern `most`.  floor: 2^e = a quarter of the largest power of
// two that does not exceed it (magnitudes beyond 6 * 2^e are held at 6).  fullrange: the smallest power of two with most <= 6 * 2^e.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t most, uint32_t fullrange) {
  if (most >= 0x7F800000u) return kMxNanByte;
  const uint32_t e = (most + (fullrange ? 0x003FFFFFu : 0u)) >> 23;
  return e > 2u ? e - 2u : 0u;
}
// 2^(byte - 127) as the conversion instructions take it (they look at the exponent alone; 0 would be 0, so that 2^-127 is given as
// the subnormal that it is)
__device__ __forceinline__ float mx_scale_value(uint32_t byte) {
  return __uint_as_float(byte ? byte << 23 : 0x00400000u);
}
#endif

}  // namespace adacc
