// Compression of matrices to microscaled 4-bit floating point, along the rows, across them or both from one reading, and their
// restoration (adacc_mx4.hpp describes the format).  Every kernel is a stream: what bounds it is the reading of the tensor and the
// writing of codes, or the other way round.
#include "adacc_mx4.hpp"

namespace adacc {

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 mx_f16x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t mx_u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t mx_pk_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(mx_u16x2, a), __builtin_bit_cast(mx_u16x2, b)));
}

// A lane holds W words of a row: V values.  The wavefront covers a strip of 64 * V columns, kMxBlock / V lanes share a block.
template <uint32_t TYPE, uint32_t W>
struct MxElem {
  static constexpr uint32_t kBytes = TYPE == kMxF32 ? 4u : 2u;
  static constexpr uint32_t V = 4u * W / kBytes;
  static constexpr uint32_t kLanes = kMxBlock / V;  // per block
  static constexpr uint32_t kStrip = kWave * V;
  // the binary32 pattern of a magnitude
  __device__ static __forceinline__ uint32_t bits32(uint32_t mag) {
    if constexpr (TYPE == kMxBf16) return mag << 16;
    else if constexpr (TYPE == kMxF16) return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)mag));
    else return mag;
  }
};
template <uint32_t W>
struct MxWords {
  uint32_t w[W];
};

template <uint32_t SEL, uint32_t TYPE>
__device__ __forceinline__ uint32_t mx_encode2(uint32_t into, uint32_t w, float scale) {
  if constexpr (TYPE == kMxBf16) return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(into, __builtin_bit_cast(mx_bf16x2, w), scale, SEL);
  else return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(into, __builtin_bit_cast(mx_f16x2, w), scale, SEL);
}
template <uint32_t SEL>
__device__ __forceinline__ uint32_t mx_encode2f(uint32_t into, uint32_t a, uint32_t b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(into, __uint_as_float(a), __uint_as_float(b), scale, SEL);
}

// 8 * EIGHTS rows of the strip, `rows` of which exist (at least one); `row` points to the start of the first.  All loads are in flight at once
// and at any address: a row behind the last reads the last one, a lane behind the row's end reads its start, and both are dropped; the lane that
// the end cuts reads the row's last 4 * W bytes and moves them down.  NARROW: rows of fewer bytes than that, value by value.
template <uint32_t TYPE, uint32_t W, uint32_t EIGHTS, bool NARROW>
__device__ __forceinline__ void mx_load_rows(MxWords<W> (&raw)[EIGHTS][8], const uint8_t* row, uint64_t stride_bytes, uint32_t col, uint32_t cols, uint32_t rows) {
  using E = MxElem<TYPE, W>;
  constexpr uint32_t N = 8u * EIGHTS;
  if constexpr (NARROW) {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      const uint8_t* p = row + (uint64_t)min(i, rows - 1u) * stride_bytes;
#pragma unroll
      for (uint32_t k = 0; k < W; ++k) raw[i / 8u][i % 8u].w[k] = 0u;
#pragma unroll
      for (uint32_t e = 0; e < E::V - 1u; ++e) {  // (col is 0, or behind the end)
        const bool there = col + e < cols && i < rows;
        const uint32_t at = min(e, cols - 1u);
        if constexpr (TYPE == kMxF32) { const uint32_t v = reinterpret_cast<const uint32_t*>(p)[at]; raw[i / 8u][i % 8u].w[e] = there ? v : 0u; }
        else { const uint32_t v = reinterpret_cast<const uint16_t*>(p)[at]; raw[i / 8u][i % 8u].w[e / 2u] |= there ? v << (16u * (e % 2u)) : 0u; }
      }
    }
  } else {
    const bool there = col < cols;
    const uint32_t from = there ? min(col, cols - E::V) : 0u;
    const uint8_t* p = row + (uint64_t)from * E::kBytes;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      const uint8_t* q = p + (uint64_t)min(i, rows - 1u) * stride_bytes;
      if constexpr (W == 4) {
        const mx_u4u v = __builtin_nontemporal_load(reinterpret_cast<const mx_u4u*>(q));
        raw[i / 8u][i % 8u].w[0] = v.x; raw[i / 8u][i % 8u].w[1] = v.y; raw[i / 8u][i % 8u].w[2] = v.z; raw[i / 8u][i % 8u].w[3] = v.w;
      } else {
        const mx_u2u v = __builtin_nontemporal_load(reinterpret_cast<const mx_u2u*>(q));
        raw[i / 8u][i % 8u].w[0] = v.x; raw[i / 8u][i % 8u].w[1] = v.y;
      }
    }
    const uint32_t all = there ? ~0u : 0u;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      const uint32_t keep = i < rows ? all : 0u;
#pragma unroll
      for (uint32_t k = 0; k < W; ++k) raw[i / 8u][i % 8u].w[k] &= keep;
    }
    if (cols % E::V) {
      const uint32_t gone = there ? (col - from) * E::kBytes : 0u;  // bytes that belong to the lane before
      const bool by8 = gone & 8u, by4 = gone & 4u;
      const uint32_t bits = (gone & 3u) * 8u;
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        MxWords<W>& v = raw[i / 8u][i % 8u];
        if constexpr (W == 4) {
          const uint32_t x = by8 ? v.w[2] : v.w[0], y = by8 ? v.w[3] : v.w[1], z = by8 ? 0u : v.w[2], u = by8 ? 0u : v.w[3];
          const uint32_t x4 = by4 ? y : x, y4 = by4 ? z : y, z4 = by4 ? u : z, u4 = by4 ? 0u : u;
          v.w[0] = __builtin_amdgcn_alignbit(y4, x4, bits);
          v.w[1] = __builtin_amdgcn_alignbit(z4, y4, bits);
          v.w[2] = __builtin_amdgcn_alignbit(u4, z4, bits);
          v.w[3] = u4 >> bits;
        } else {
          const uint32_t x = by4 ? v.w[1] : v.w[0], y = by4 ? 0u : v.w[1];
          v.w[0] = __builtin_amdgcn_alignbit(y, x, bits);
          v.w[1] = y >> bits;
        }
      }
    }
  }
}

// the largest magnitude of a lane's values, as a pattern of its own type
template <uint32_t TYPE, uint32_t W>
__device__ __forceinline__ uint32_t mx_lane_max(const MxWords<W>& v) {
  uint32_t most = 0u;
#pragma unroll
  for (uint32_t k = 0; k < W; ++k) {
    if constexpr (TYPE == kMxF32) most = max(most, v.w[k] & 0x7FFFFFFFu);
    else most = mx_pk_max(most, v.w[k] & 0x7FFF7FFFu);
  }
  return TYPE == kMxF32 ? most : max(most & 0xFFFFu, most >> 16);
}

// the maximum over the lanes of a block, in all of them
template <uint32_t LANES>
__device__ __forceinline__ uint32_t mx_block_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));  // lanes 1 0 3 2
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));  // lanes 2 3 0 1
  if constexpr (LANES == 8u) v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));  // mirrored within eight
  return v;
}

// a lane's codes of one row: 4 bytes (V = 8) or 2 (V = 4)
template <uint32_t TYPE, uint32_t W>
__device__ __forceinline__ uint32_t mx_row_codes(const MxWords<W>& v, uint32_t byte) {
  const float s = mx_scale_value(byte);
  uint32_t c = 0u;
  if constexpr (TYPE == kMxF32) {
    c = mx_encode2f<0>(c, v.w[0], v.w[1], s);
    c = mx_encode2f<1>(c, v.w[2], v.w[3], s);
  } else {
    c = mx_encode2<0, TYPE>(c, v.w[0], s);
    c = mx_encode2<1, TYPE>(c, v.w[1], s);
    if constexpr (W == 4) {
      c = mx_encode2<2, TYPE>(c, v.w[2], s);
      c = mx_encode2<3, TYPE>(c, v.w[3], s);
    }
  }
  return byte == kMxNanByte ? 0u : c;
}

// `count` (at most 8) rows of the strip along the rows: codes stored, the scale bytes returned.  (A wavefront's row is two or four pieces
// of 64 bytes, adjacent rows' lie next to each other: plain stores, which the cache puts together, are 5 % faster than streaming ones.)
template <uint32_t TYPE, uint32_t W>
__device__ __forceinline__ uint64_t mx_rows8(const MxWords<W> (&raw)[8], const MxMatrix& m, uint64_t row0, uint32_t count, uint32_t col, bool inside,
                                             uint32_t fullrange) {
  using E = MxElem<TYPE, W>;
  uint64_t bytes = 0;
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) {
    const uint32_t most = mx_block_max<E::kLanes>(mx_lane_max<TYPE, W>(raw[i]));
    const uint32_t byte = mx_scale_byte(E::bits32(most), fullrange);
    bytes |= (uint64_t)byte << (8u * i);
    const uint32_t c = mx_row_codes<TYPE, W>(raw[i], byte);
    if (inside && i < count) {
      uint8_t* p = m.codes + (uint64_t)(col / kMxStep) * m.step_bytes + (row0 + i) * kMxStepBytes + col % kMxStep / 2u;
      if constexpr (E::V == 8u) *reinterpret_cast<uint32_t*>(p) = c;
      else *reinterpret_cast<uint16_t*>(p) = (uint16_t)c;
    }
  }
  return bytes;
}

// the scale bytes of rows [row, row + 8), of which `count` exist
__device__ __forceinline__ void mx_store_scales8(uint8_t* p, uint64_t bytes, int32_t count) {
  if (count >= 8) {
    const mx_u2u v = {(uint32_t)bytes, (uint32_t)(bytes >> 32)};
    *reinterpret_cast<mx_u2u*>(p) = v;
  } else {
    for (int32_t i = 0; i < count; ++i) p[i] = (uint8_t)(bytes >> (8 * i));
  }
}

// ------------------------------------------------------------------ along the rows
// A wavefront takes kMxWaveRows = 8 rows of a strip, eight loads in flight a lane.  Every lane of a block knows the block's byte of all rows; the
// first one stores them.  ([32768, 2048] bf16 28 us, 6.0 TB/s; two or four times eight rows one after the other: as long, and 1 to 4 us more for
// tensors that leave a compute unit few wavefronts.)
template <uint32_t TYPE, bool NARROW>
__global__ __launch_bounds__(kThreads) void mx4_along_kernel(MxCompressArgs a) {
  using E = MxElem<TYPE, 4>;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const uint32_t block = a.first + blockIdx.x;
  const uint32_t ct = block % a.col_tiles;
  const uint32_t rt = block / a.col_tiles;
  const uint32_t mat = rt / a.row_tiles;
  const uint32_t row0 = ((rt - mat * a.row_tiles) * kWavesPerWg + wave) * kMxWaveRows;
  if (row0 >= a.rows) return;
  const uint32_t col = ct * E::kStrip + lane * E::V;
  const bool inside = col < a.along.steps * kMxStep;
  const uint8_t* src = static_cast<const uint8_t*>(a.src) + ((uint64_t)mat * a.mat_stride + (uint64_t)row0 * a.row_stride) * E::kBytes;
  const uint64_t brow = (uint64_t)mat * a.rows + row0;
  const uint32_t rows = min(a.rows - row0, kMxWaveRows);
  MxWords<4> raw[1][8];
  mx_load_rows<TYPE, 4, 1, NARROW>(raw, src, a.row_stride * E::kBytes, col, a.cols, rows);
  const uint64_t bytes = mx_rows8<TYPE, 4>(raw[0], a.along, brow, rows, col, inside, a.fullrange);
  if (inside && lane % E::kLanes == 0u)
    mx_store_scales8(a.along.scales + (uint64_t)(col / kMxBlock) * a.along.pitch + brow, bytes, (int32_t)rows);
}

// ------------------------------------------------------------------ across the rows, and both
// A workgroup takes 128 rows of a strip, a wavefront 32 of them: all 32 values of a column's block lie in one lane, whose maximum
// and codes need no other lane.  The codes of the strip's columns, 64 bytes each, are turned over in LDS.
// (A lane's V columns are 64 * V bytes of LDS and 16 more, so that sixteen lanes write to different banks.  8 bytes of a row a lane, where 16 would
// be as wide a load: 64 registers of values instead of 128, four wavefronts a SIMD instead of two; both directions of [32768, 2048] bf16 37 us instead of
// 41, 205 MB.)
template <uint32_t TYPE, bool ALONG, bool NARROW>
__global__ __launch_bounds__(kThreads, TYPE == kMxF32 ? 2 : 4) void mx4_across_kernel(MxCompressArgs a) {
  constexpr uint32_t W = TYPE == kMxF32 ? 4u : 2u;
  using E = MxElem<TYPE, W>;
  constexpr uint32_t V = E::V;
  constexpr uint32_t kLaneRoom = V * kMxStepBytes + 16u;
  __shared__ __attribute__((aligned(16))) uint8_t turn[kWave * kLaneRoom];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const uint32_t block = a.first + blockIdx.x;
  const uint32_t ct = block % a.col_tiles;
  const uint32_t rt = block / a.col_tiles;
  uint32_t mat = 0u, row0, last, step;
  bool across;
  if (a.g.offsets != nullptr) {
    const MxPlace p = mx_place<false>(a.g, rt, kMxTileRows);
    if ((uint64_t)p.unit * kMxTileRows >= (uint64_t)(p.last - p.first)) return;
    row0 = p.first + p.unit * kMxTileRows;
    last = p.last;
    step = p.before + p.unit;
    across = p.group < a.g.groups && step < a.across.steps;
    if (!ALONG && !across) return;
  } else {
    mat = rt / a.row_tiles;
    step = rt - mat * a.row_tiles;
    row0 = step * kMxTileRows;
    last = a.rows;
    across = true;
  }
  row0 += wave * kMxBlock;
  const uint32_t rows = row0 >= last ? 0u : min(last - row0, kMxBlock);
  const uint32_t col = ct * E::kStrip + lane * V;
  const int64_t left = (int64_t)a.cols - (int64_t)col;
  const uint8_t* src = static_cast<const uint8_t*>(a.src) + ((uint64_t)mat * a.mat_stride + (uint64_t)row0 * a.row_stride) * E::kBytes;
  MxWords<W> raw[4][8];
  if (rows) {
    mx_load_rows<TYPE, W, 4, NARROW>(raw, src, a.row_stride * E::kBytes, col, a.cols, rows);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kMxBlock; ++i)
#pragma unroll
      for (uint32_t k = 0; k < W; ++k) raw[i / 8u][i % 8u].w[k] = 0u;
  }
  if constexpr (ALONG) {
    const bool inside = col < a.along.steps * kMxStep;
    const uint64_t brow = (uint64_t)mat * a.rows + row0;
    const uint32_t q = lane % E::kLanes;
    uint64_t mine = 0;
#pragma unroll
    for (uint32_t b = 0; b < 4u; ++b) {
      const uint64_t bytes = mx_rows8<TYPE, W>(raw[b], a.along, brow + 8u * b, rows > 8u * b ? rows - 8u * b : 0u, col, inside, a.fullrange);
      if (q == b) mine = bytes;
    }
    if (inside && q < 4u && q * 8u < rows)
      mx_store_scales8(a.along.scales + (uint64_t)(col / kMxBlock) * a.along.pitch + brow + q * 8u, mine, (int32_t)(rows - q * 8u));
  }
  if (!across) return;  // (the whole workgroup)
  // the columns' blocks
  uint32_t byte[V];
  {
    uint32_t most[W];
#pragma unroll
    for (uint32_t k = 0; k < W; ++k) most[k] = 0u;
#pragma unroll
    for (uint32_t i = 0; i < kMxBlock; ++i) {
#pragma unroll
      for (uint32_t k = 0; k < W; ++k) {
        if constexpr (TYPE == kMxF32) most[k] = max(most[k], raw[i / 8u][i % 8u].w[k] & 0x7FFFFFFFu);
        else most[k] = mx_pk_max(most[k], raw[i / 8u][i % 8u].w[k] & 0x7FFF7FFFu);
      }
    }
#pragma unroll
    for (uint32_t c = 0; c < V; ++c) {
      const uint32_t mag = TYPE == kMxF32 ? most[c % W] : (most[c / 2u % W] >> (16u * (c % 2u))) & 0xFFFFu;
      byte[c] = mx_scale_byte(E::bits32(mag), a.fullrange);
    }
  }
  uint8_t* mine = turn + lane * kLaneRoom + wave * 16u;
#pragma unroll
  for (uint32_t c = 0; c < V; ++c) {
    const float s = mx_scale_value(byte[c]);
    uint32_t o[4];
#pragma unroll
    for (uint32_t k = 0; k < 4u; ++k) {
      uint32_t w = 0u;
#define ADACC_MX_PAIR(P)                                                                                          \
  {                                                                                                               \
    const MxWords<W>&lo = raw[k][2 * P], &hi = raw[k][2 * P + 1];                                                 \
    if constexpr (TYPE == kMxF32) w = mx_encode2f<P>(w, lo.w[c % W], hi.w[c % W], s);                             \
    else w = mx_encode2<P, TYPE>(w, __builtin_amdgcn_perm(hi.w[c / 2u % W], lo.w[c / 2u % W], c % 2u ? 0x07060302u : 0x05040100u), s); \
  }
      ADACC_MX_PAIR(0) ADACC_MX_PAIR(1) ADACC_MX_PAIR(2) ADACC_MX_PAIR(3)
#undef ADACC_MX_PAIR
      o[k] = byte[c] == kMxNanByte ? 0u : w;
    }
    *reinterpret_cast<uint4*>(mine + c * kMxStepBytes) = make_uint4(o[0], o[1], o[2], o[3]);
  }
  const uint64_t trow = (uint64_t)mat * a.cols;  // the matrix's first row of the result across
  {
    uint8_t* p = a.across.scales + (uint64_t)(4u * step + wave) * a.across.pitch + trow + col;
    if (left >= (int64_t)V) {
      static_assert(V == 4u, "four bytes");
      *reinterpret_cast<mx_u1u*>(p) = byte[0] | byte[1] << 8 | byte[2] << 16 | byte[3] << 24;
    } else {
#pragma unroll
      for (uint32_t c = 0; c < V; ++c) if ((int64_t)c < left) p[c] = (uint8_t)byte[c];
    }
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < V; ++i) {  // four threads a column, 64 columns a turn
    const uint32_t c = i * (kThreads / 4u) + threadIdx.x / 4u;
    const uint64_t column = (uint64_t)ct * E::kStrip + c;
    if (column >= a.cols) break;
    const uint4 v = *reinterpret_cast<const uint4*>(turn + (c / V) * kLaneRoom + (c % V) * kMxStepBytes + (threadIdx.x % 4u) * 16u);
    store_stream16(a.across.codes + (uint64_t)step * a.across.step_bytes + (trow + column) * kMxStepBytes + (threadIdx.x % 4u) * 16u, v);
  }
}

// ------------------------------------------------------------------ restoration
// A wavefront takes 8 rows of a strip; the eight scale bytes of a block column are one load.  ([32768, 2048] to bf16 32 us; codes read by plain
// loads 35; sixteen rows, eight after eight, 37.)
template <uint32_t TYPE>
__global__ __launch_bounds__(kThreads) void mx4_restore_kernel(MxDecompressArgs a) {
  using E = MxElem<TYPE, 4>;
  constexpr uint32_t V = E::V;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const uint32_t block = a.first + blockIdx.x;
  const uint32_t ct = block % a.col_tiles;
  const uint32_t row0 = ((block / a.col_tiles) * kWavesPerWg + wave) * kMxWaveRows;
  const uint32_t col = ct * E::kStrip + lane * V;
  if (row0 >= a.m.rows || col >= a.cols) return;
  const uint32_t rows = min(a.m.rows - row0, kMxWaveRows);
  const uint32_t left = a.cols - col;
  const uint8_t* codes = a.m.codes + (uint64_t)(col / kMxStep) * a.m.step_bytes + (uint64_t)row0 * kMxStepBytes + col % kMxStep / 2u;
  const uint8_t* scales = a.m.scales + (uint64_t)(col / kMxBlock) * a.m.pitch + row0;
  uint8_t* dst = static_cast<uint8_t*>(a.dst) + ((uint64_t)row0 * a.row_stride + col) * E::kBytes;
  const uint2 s8 = *reinterpret_cast<const uint2*>(scales);  // (row0 is a multiple of 8, and so is the pitch)
  uint32_t c[8];
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) {
    const uint32_t at = min(i, rows - 1u);
    if constexpr (V == 8u) c[i] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(codes + (uint64_t)at * kMxStepBytes));
    else c[i] = __builtin_nontemporal_load(reinterpret_cast<const uint16_t*>(codes + (uint64_t)at * kMxStepBytes));
  }
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) {
    if (i >= rows) break;
    const float s = mx_scale_value(((i < 4u ? s8.x : s8.y) >> (8u * (i % 4u))) & 0xFFu);
    uint32_t w[4];
    if constexpr (TYPE == kMxF32) {
      const mx_f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 1);
      w[0] = __float_as_uint(lo.x); w[1] = __float_as_uint(lo.y); w[2] = __float_as_uint(hi.x); w[3] = __float_as_uint(hi.y);
    } else if constexpr (TYPE == kMxBf16) {
      w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 0));
      w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 1));
      w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 2));
      w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 3));
    } else {
      w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[i], s, 0));
      w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[i], s, 1));
      w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[i], s, 2));
      w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[i], s, 3));
    }
    uint8_t* p = dst + (uint64_t)i * a.row_stride * E::kBytes;
    if (left >= V) {
      const mx_u4u v = {w[0], w[1], w[2], w[3]};
      __builtin_nontemporal_store(v, reinterpret_cast<mx_u4u*>(p));
    } else {
#pragma unroll
      for (uint32_t e = 0; e < V; ++e) {
        if (e < left) {
          if constexpr (TYPE == kMxF32) reinterpret_cast<uint32_t*>(p)[e] = w[e % 4u];
          else reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(w[(e / 2u) % 4u] >> (16u * (e % 2u)));
        }
      }
    }
  }
}

template <uint32_t TYPE, bool NARROW>
static MxCompressFn compress_of(bool along, bool across) {
  if (!across) return mx4_along_kernel<TYPE, NARROW>;
  if constexpr (!NARROW)
    if (along) return mx4_across_kernel<TYPE, true, NARROW>;
  return mx4_across_kernel<TYPE, false, NARROW>;
}
MxCompressFn mx4_compress_fn(uint32_t type, bool along, bool across, bool narrow) {
  switch (type) {
    case kMxBf16: return narrow ? compress_of<kMxBf16, true>(along, across) : compress_of<kMxBf16, false>(along, across);
    case kMxF16: return narrow ? compress_of<kMxF16, true>(along, across) : compress_of<kMxF16, false>(along, across);
    default: return narrow ? compress_of<kMxF32, true>(along, across) : compress_of<kMxF32, false>(along, across);
  }
}
MxDecompressFn mx4_decompress_fn(uint32_t type) {
  return type == kMxBf16 ? mx4_restore_kernel<kMxBf16> : type == kMxF16 ? mx4_restore_kernel<kMxF16> : mx4_restore_kernel<kMxF32>;
}

}  // namespace adacc
