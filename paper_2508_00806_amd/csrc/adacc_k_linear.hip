// Products of 16-bit matrices on the matrix cores, with bias, activation and residual in the epilogue, and their gradients:
//
//   y = act(x w^T + b) + r        both operands along the contraction
//   dx = dpre w                   w across it
//   dw = dpre^T x~                both across it, x~ in 16 bits or as 8-bit rows, which are restored on the way
//
// One kernel for all: what differs is how a tile of an operand comes to LDS, where it always lies along the contraction.
#include <type_traits>
#include <utility>

#include "adacc_layers.hpp"

namespace adacc {

typedef float lin_f16v __attribute__((ext_vector_type(16)));
typedef float lin_f4v __attribute__((ext_vector_type(4)));
typedef __bf16 lin_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 lin_f16x8 __attribute__((ext_vector_type(8)));

template <uint32_t TYPE>
__device__ __forceinline__ lin_f16v mfma32(uint4 a, uint4 b, lin_f16v c) {
  if constexpr (TYPE == kTypeBf16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(lin_bf16x8, a), __builtin_bit_cast(lin_bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(lin_f16x8, a), __builtin_bit_cast(lin_f16x8, b), c, 0, 0, 0);
}
template <uint32_t TYPE>
__device__ __forceinline__ lin_f4v mfma16(uint4 a, uint4 b, lin_f4v c) {
  if constexpr (TYPE == kTypeBf16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(lin_bf16x8, a), __builtin_bit_cast(lin_bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(lin_f16x8, a), __builtin_bit_cast(lin_f16x8, b), c, 0, 0, 0);
}

template <uint32_t N, typename F, uint32_t... I>
__device__ __forceinline__ void each(F&& f, std::integer_sequence<uint32_t, I...>) {
  (f(std::integral_constant<uint32_t, I>{}), ...);
}
template <uint32_t N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each<N>(f, std::make_integer_sequence<uint32_t, N>{});
}
// those of f(0) ... f(N - 1) that belong to slot SLOT, where they are spread evenly over slots FROM to TO - 1
constexpr uint32_t spread(uint32_t n, uint32_t from, uint32_t to, uint32_t slot) { return slot <= from ? 0u : slot >= to ? n : (n * (slot - from) + (to - from) - 1u) / (to - from); }
template <uint32_t N, uint32_t FROM, uint32_t TO, uint32_t SLOT, typename F>
__device__ __forceinline__ void in_slot(F&& f) {
  constexpr uint32_t kFirst = spread(N, FROM, TO, SLOT), kLast = spread(N, FROM, TO, SLOT + 1u);
  each<kLast - kFirst>([&](auto i) __attribute__((always_inline)) { f(std::integral_constant<uint32_t, kFirst + decltype(i)::value>{}); });
}

// ------------------------------------------------------------------ an operand's way to LDS
// A step is 64 of the contraction: 128 bytes of each of the tile's rows, in eight pieces of 16 bytes.
//   Rows lie in the order in which a wavefront's lanes read them: with S = TILE / 64, row j of the tile is number (j % S) * 32 + (j % 32 S) / S of its half (32 S rows).  Two numbers
// share 256 bytes, the 64 banks; the odd one lies behind the even one, or ahead of it where bit 4 of the number is set.  Piece p of number q lies at place p ^ (q / 2 % 8) of its 128 bytes.  So
// sixteen lanes meet all banks that read one piece of adjacent numbers, that write the pieces of two of them, or one piece of every second one.  (In the order of the rows, where such lanes
// met half of the banks and the loads of a step came in one run, 8192^3 took 1.03 ms; so it takes 0.86.)
template <uint32_t TILE>
__device__ __forceinline__ uint32_t lin_number(uint32_t row) {
  constexpr uint32_t S = TILE / 64u, kHalf = 32u * S;
  return row / kHalf * kHalf + row % S * 32u + row % kHalf / S;
}
template <uint32_t TILE>
__device__ __forceinline__ uint32_t lin_row(uint32_t number) {
  constexpr uint32_t S = TILE / 64u, kHalf = 32u * S;
  return number / kHalf * kHalf + number % 32u * S + number % kHalf / 32u;
}
__device__ __forceinline__ uint32_t lin_slot(uint32_t number) { return number ^ (number >> 4 & 1u); }  // (its own inverse)
__device__ __forceinline__ uint32_t lin_place(uint32_t number, uint32_t piece) { return lin_slot(number) * 128u + ((piece ^ (number / 2u & 7u)) * 16u); }

// a pointer to global memory that is the same in all lanes, known to be so
typedef const __attribute__((address_space(1))) uint8_t* lin_global;
__device__ __forceinline__ lin_global lin_uniform(const void* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (lin_global)((uint64_t)hi << 32 | lo);
}
template <typename V>
__device__ __forceinline__ V lin_fetch(lin_global p) {
  return *(const __attribute__((address_space(1))) V*)p;
}

// 128 bits, `by` (0 to 128) bits down
__device__ __forceinline__ uint4 lin_move_down(uint4 v, uint32_t by) {
  const uint64_t lo = (uint64_t)v.y << 32 | v.x, hi = (uint64_t)v.w << 32 | v.z;
  const uint64_t low = by == 0u ? lo : by < 64u ? lo >> by | hi << (64u - by) : by < 128u ? hi >> (by - 64u) : 0u;
  const uint64_t high = by < 64u ? hi >> by : 0u;
  return make_uint4((uint32_t)low, (uint32_t)(low >> 32), (uint32_t)high, (uint32_t)(high >> 32));
}

// TILE rows (of the result) by a step, through the registers of a thread: kLoads loads and kStores stores
//   aim(...)    the tile's rows from row0 on, `rows` of which there are in all, at least 8 to a row of the memory
//   turn(...)   the step that is loaded next; nothing behind the contraction's end is read: the last step's loads are moved back to what is there ...
//   mend(...)   ... and put right before they are stored: `have` of its 64 values are there, the others are zeros
// Rows of the result behind the last have values of others: they are not kept.
template <uint32_t TYPE, uint32_t MODE, uint32_t TILE>
struct Loader;

template <uint32_t TYPE, uint32_t TILE>
struct Loader<TYPE, kAlong, TILE> {
  static constexpr uint32_t kLoads = TILE / 32u, kStores = kLoads;
  uint4 r[kLoads];
  lin_global base, now;
  uint32_t off[kLoads], back;
  __device__ __forceinline__ void aim(const Strided& m, const Rows8&, uint32_t row0, uint32_t rows) {
    // (offsets count from eight values ahead of the row's first, so that none becomes negative when it is moved back)
    base = lin_uniform(static_cast<const uint8_t*>(m.at) + (uint64_t)row0 * m.stride * 2u - 16u);
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
      const uint32_t row = min(lin_row<TILE>(i * 32u + threadIdx.x / 8u), rows - row0 - 1u);
      off[i] = (row * (uint32_t)m.stride + threadIdx.x % 8u * 8u) * 2u + 16u;
    }
  }
  __device__ __forceinline__ void turn(uint32_t step, uint32_t k) {
    now = base + (uint64_t)step * (2u * kLinStep);
    const uint32_t end = threadIdx.x % 8u * 8u + 8u, have = k - step * kLinStep;
    back = (max(end, have) - have) * 2u;
  }
  template <uint32_t I>
  __device__ __forceinline__ void load() {
    const u4_any t = lin_fetch<u4_any>(now + (off[I] - back));
    r[I] = make_uint4(t.x, t.y, t.z, t.w);
  }
  __device__ __forceinline__ void mend(uint32_t have) {
    const uint32_t first = threadIdx.x % 8u * 8u, left = have > first ? have - first : 0u;
    if (left >= 8u) return;
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) r[i] = lin_move_down(r[i], 16u * (8u - left));
  }
  template <uint32_t I>
  __device__ __forceinline__ void store(uint8_t* lds) const {
    *reinterpret_cast<uint4*>(lds + lin_place(I * 32u + threadIdx.x / 8u, threadIdx.x % 8u)) = r[I];
  }
};

// A thread takes eight of the contraction (piece threadIdx.x / 32) by Q columns of the memory's rows.  Columns that are not all there are moved back to where they are:
// some of the rows in LDS are then written twice, with the same values.
template <uint32_t TILE>
struct AcrossPlace {
  static constexpr uint32_t Q = TILE / 32u;  // 8 or 4
  uint32_t col, to[Q];                       // col: from the first of the tile's columns on, or from that many ahead of it (aim's result)
  __device__ __forceinline__ uint32_t aim(uint32_t there) {  // columns from the tile's first on
    const uint32_t ahead = there < Q ? Q - there : 0u;      // a tile of fewer than Q: what is ahead of it goes to a row that is not kept
    col = min(threadIdx.x % 32u * Q, there + ahead - Q);
#pragma unroll
    for (uint32_t i = 0; i < Q; ++i) to[i] = lin_place(lin_number<TILE>(col + i >= ahead ? col + i - ahead : TILE - 1u), threadIdx.x / 32u);
    return ahead;
  }
};
template <uint32_t TYPE, uint32_t TILE>
struct Loader<TYPE, kAcross, TILE> {
  static constexpr uint32_t Q = TILE / 32u;
  static constexpr uint32_t kLoads = 8u, kStores = Q;
  AcrossPlace<TILE> place;
  uint32_t r[8][Q / 2u];
  lin_global base, now;
  uint32_t off, down, most;  // bytes
  __device__ __forceinline__ void aim(const Strided& m, const Rows8&, uint32_t row0, uint32_t rows) {
    const uint32_t ahead = place.aim(rows - row0);
    base = lin_uniform(static_cast<const uint8_t*>(m.at) + (uint64_t)(row0 - ahead) * 2u);
    down = (uint32_t)m.stride * 2u;
    off = threadIdx.x / 32u * 8u * down + place.col * 2u;
  }
  __device__ __forceinline__ void turn(uint32_t step, uint32_t k) {
    now = base + (uint64_t)step * kLinStep * down;
    most = min(k - 1u - step * kLinStep, kLinStep - 1u) * down + place.col * 2u;
  }
  template <uint32_t I>
  __device__ __forceinline__ void load() {
    const lin_global from = now + min(off + I * down, most);
    if constexpr (Q == 8u) {
      const u4_any t = lin_fetch<u4_any>(from);
      r[I][0] = t.x; r[I][1] = t.y; r[I][2] = t.z; r[I][3] = t.w;
    } else {
      const u2_any t = lin_fetch<u2_any>(from);
      r[I][0] = t.x; r[I][1] = t.y;
    }
  }
  __device__ __forceinline__ void mend(uint32_t have) {
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i)
#pragma unroll
      for (uint32_t j = 0; j < Q / 2u; ++j) r[i][j] = threadIdx.x / 32u * 8u + i < have ? r[i][j] : 0u;
  }
  template <uint32_t I>
  __device__ __forceinline__ void store(uint8_t* lds) const {
    uint32_t w[4];
#pragma unroll
    for (uint32_t d = 0; d < 4u; ++d)  // halves I % 2 of two rows
      w[d] = __builtin_amdgcn_perm(r[2 * d + 1][I / 2u], r[2 * d][I / 2u], I % 2u ? 0x07060302u : 0x05040100u);
    *reinterpret_cast<uint4*>(lds + place.to[I]) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// The same of 8-bit rows: codes and a scale for every row, restored when they are stored.  A row of codes is as long as its pitch.
template <uint32_t TYPE, uint32_t TILE>
struct Loader<TYPE, kAcross8, TILE> {
  static constexpr uint32_t Q = TILE / 32u;
  static constexpr uint32_t kLoads = 8u, kStores = Q;
  AcrossPlace<TILE> place;
  uint32_t r[8][Q / 4u];
  float s[8];
  lin_global base, now, scales, scales_now;
  uint32_t off, down, most, scale_off, scale_down, scale_most, group;
  __device__ __forceinline__ void aim(const Strided&, const Rows8& b, uint32_t row0, uint32_t) {
    base = lin_uniform(b.codes + row0);
    scales = lin_uniform(b.scales + row0 / kR8Group);
    place.aim((uint32_t)b.pitch - row0);
    down = (uint32_t)b.pitch;
    scale_down = b.groups * 4u;
    group = min(place.col / kR8Group, b.groups - 1u - row0 / kR8Group) * 4u;
    off = threadIdx.x / 32u * 8u * down + place.col;
    scale_off = threadIdx.x / 32u * 8u * scale_down + group;
  }
  __device__ __forceinline__ void turn(uint32_t step, uint32_t k) {
    const uint32_t last = min(k - 1u - step * kLinStep, kLinStep - 1u);
    now = base + (uint64_t)step * kLinStep * down;
    scales_now = scales + (uint64_t)step * kLinStep * scale_down;
    most = last * down + place.col;
    scale_most = last * scale_down + group;
  }
  template <uint32_t I>
  __device__ __forceinline__ void load() {
    const lin_global from = now + min(off + I * down, most);
    if constexpr (Q == 8u) {
      const u32x2_t t = lin_fetch<u32x2_t>(from);
      r[I][0] = t.x; r[I][1] = t.y;
    } else {
      r[I][0] = lin_fetch<uint32_t>(from);
    }
    s[I] = lin_fetch<float>(scales_now + min(scale_off + I * scale_down, scale_most));
  }
  __device__ __forceinline__ void mend(uint32_t have) {  // (by zero; a scale may be NaN, a code is none)
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) s[i] = threadIdx.x / 32u * 8u + i < have ? s[i] : 0.0f;
  }
  template <uint32_t I>
  __device__ __forceinline__ void store(uint8_t* lds) const {
    uint32_t w[4];
#pragma unroll
    for (uint32_t d = 0; d < 4u; ++d) {
      const float lo = (float)(int8_t)(r[2 * d][I / 4u] >> (8u * (I % 4u))) * s[2 * d];
      const float hi = (float)(int8_t)(r[2 * d + 1][I / 4u] >> (8u * (I % 4u))) * s[2 * d + 1];
      w[d] = narrow2<TYPE>(lo, hi);
    }
    *reinterpret_cast<uint4*>(lds + place.to[I]) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

__device__ __forceinline__ void lin_meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// The eight dies have a second-level cache each and take workgroups in turn: numbered so that a die's are neighbours, tiles go in bands of 8 tile rows, column by
// column, so that what runs at the same time on a die shares both operands.
__device__ __forceinline__ uint32_t lin_by_die(uint32_t id, uint32_t total) {
  constexpr uint32_t kDies = 8u;
  const uint32_t die = id % kDies, turn = id / kDies, each = total / kDies, more = total % kDies;
  return die * each + min(die, more) + turn;
}
__device__ __forceinline__ void lin_band(uint32_t id, uint32_t m_tiles, uint32_t n_tiles, uint32_t* mt, uint32_t* nt) {
  constexpr uint32_t kBand = 8u;
  const uint32_t band = id / (kBand * n_tiles), in = id - band * kBand * n_tiles;
  const uint32_t high = min(kBand, m_tiles - band * kBand);
  *nt = in / high;
  *mt = band * kBand + in - *nt * high;
}

// ------------------------------------------------------------------ tiles
// Four wavefronts, two by two, each S x S tiles of 32 x 32 (S = 4, or 2).  Row S * r + i of a wavefront's rows is row r of its tile i, so that a lane's S columns of
// the results lie side by side.
//   What bounds the tile of 256 (32 x 32 x 16 products, a step of 64 in 2048 cycles of the matrix unit, one workgroup a compute unit, 496 registers a lane): the one wavefront of a SIMD, and
// power.  8192^3 of N(0, 1) 0.82 ms, 1.33 PFLOP/s (the library's product 0.67, 1.65), of zeros, where power is no limit, 0.60, 1.83 PFLOP/s (0.49, 2.27): random data cost both a quarter, and on both this
// kernel is a fifth behind.  Whatever the wavefront issues beside its products it issues between them, and a load or store that has to wait stops them.  bfloat16, us: 16384 x 11008 x 4096 1168
// to 1215 (library 1085 to 1166), with SiLU 1223, with GELU and its codes 1350; 8192 x 8192 x 2048 245 (189 to 194), with GELU 281, with GELU and codes, or its input kept, 319: there the results and a
// tile's first loads are a seventh of the time, and nothing else runs under them.  Gradients: dx 220 (library 203 to 256), dw 220 (247 to 291), from codes 245.
//   Tried: loads that pass the registers by (no faster: the same addresses are taken at the same rate), two register sets for the step's loads (the sums no longer fit), results through LDS for
// this tile as for that of 128 (260 instead of 239).
template <uint32_t TILE>
struct LinTile {
  static constexpr uint32_t S = TILE / 64u;
  static constexpr uint32_t kOperand = TILE * 128u;  // bytes of a step
  static constexpr uint32_t kStage = 2u * kOperand;
  static constexpr uint32_t kPassRows = 8u * S;      // rows of a wavefront's results that go through LDS at a time: a quarter
  static constexpr uint32_t kLds = 2u * kStage;
};

// ------------------------------------------------------------------ results of tiles of 256
// Straight from the registers: lane (r, h) of a wavefront holds rows 4 * (8 * (e / 4) + 4 * h + e % 4) + i and columns 4 r to 4 r + 3, so that 32 lanes hold the 128 columns of a
// group of 8-bit rows, and a store of a wavefront is 256 bytes of two rows.  Sixteen rows of each half at a time.
struct LinResults {
  uint32_t row, rows_left;  // this half wavefront's first row; of it and those behind it, how many there are
  uint32_t col, have;       // this lane's first column; how many of its four there are
};
template <uint32_t TYPE>
__device__ __forceinline__ void store_four(const Strided& m, uint32_t row, const LinResults& at, const float (&v)[4]) {
  uint16_t* const to = static_cast<uint16_t*>(m.at) + (uint64_t)row * m.stride + at.col;
  const u2_any w = {narrow2<TYPE>(v[0], v[1]), narrow2<TYPE>(v[2], v[3])};
  if (at.have >= 4u) {
    *reinterpret_cast<u2_any*>(to) = w;
  } else {
    if (at.have >= 1u) to[0] = (uint16_t)w.x;
    if (at.have >= 2u) to[1] = (uint16_t)(w.x >> 16);
    if (at.have >= 3u) to[2] = (uint16_t)w.y;
  }
}
// 8-bit rows of sixteen rows.  A row's largest magnitude comes to the lanes of the row's number, so that the divisions are done once for all sixteen, and the inverse goes back.
__device__ __forceinline__ void keep_codes(const Rows8& b, const LinResults& at, uint32_t first, const float (&v)[16][4]) {
  const uint32_t lane = threadIdx.x % 32u;
  uint32_t most = 0u, sign_off[4];  // (columns that are not there have no part)
#pragma unroll
  for (uint32_t j = 0; j < 4u; ++j) sign_off[j] = j < at.have ? 0x7FFFFFFFu : 0u;
#pragma unroll
  for (uint32_t k = 0; k < 16u; ++k) {
    uint32_t m = 0u;
#pragma unroll
    for (uint32_t j = 0; j < 4u; ++j) m = max(m, __float_as_uint(v[k][j]) & sign_off[j]);
    m = most_of_group(m);
    const auto other = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max((uint32_t)other[0], (uint32_t)other[1]);
    most = lane % 16u == k ? m : most;
  }
  const Scale8 mine = scale8(most);
  if (lane < 16u && lane + first < at.rows_left && at.col - 4u * lane < (uint32_t)b.pitch) {
    // (of the group that begins at the half wavefront's first column)
    b.scales[(uint64_t)(at.row + first + lane) * b.groups + (at.col - 4u * lane) / kR8Group] = mine.scale;
  }
#pragma unroll
  for (uint32_t k = 0; k < 16u; ++k) {
    const float inverse = __shfl(mine.inverse, (int)k, 32);
    if (first + k < at.rows_left && at.have)
      *reinterpret_cast<uint32_t*>(b.codes + (uint64_t)(at.row + first + k) * b.pitch + at.col) = codes4(v[k][0], v[k][1], v[k][2], v[k][3], inverse);
  }
}
template <uint32_t TYPE, uint32_t KIND, bool WHOLE_EPILOGUE>
__device__ __forceinline__ void results_of(const Epilogue& e, const LinResults& at, const lin_f16v (&acc)[4][4], const float (&bias)[4]) {
  each<4>([&](auto pass) __attribute__((always_inline)) {
    constexpr uint32_t P = decltype(pass)::value;
    float v[16][4];
    u2_any r[16];
    if constexpr (WHOLE_EPILOGUE) {
      if (e.residual.at) {
#pragma unroll
        for (uint32_t k = 0; k < 16u; ++k) {
          r[k] = u2_any{0u, 0u};
          if (32u * P + k < at.rows_left) {
            const uint16_t* from = static_cast<const uint16_t*>(e.residual.at) + (uint64_t)(at.row + 32u * P + k) * e.residual.stride + at.col;
            if (at.have >= 4u) {
              r[k] = *reinterpret_cast<const u2_any*>(from);
            } else {
              if (at.have >= 1u) r[k].x = from[0];
              if (at.have >= 2u) r[k].x |= (uint32_t)from[1] << 16;
              if (at.have >= 3u) r[k].y = from[2];
            }
          }
        }
      }
    }
#pragma unroll
    for (uint32_t k = 0; k < 16u; ++k)
#pragma unroll
      for (uint32_t j = 0; j < 4u; ++j) {
        v[k][j] = acc[k % 4u][j][4u * P + k / 4u];
        if constexpr (WHOLE_EPILOGUE) {
          asm volatile("" : "+v"(v[k][j]));  // (or the compiler adds the bias to all sums ahead of the branch by activation)
          v[k][j] += bias[j];
        }
      }
    if constexpr (KIND != kActNone) {
      if (e.pre8.codes) {
        keep_codes(e.pre8, at, 32u * P, v);
      } else if (e.pre.at) {
#pragma unroll
        for (uint32_t k = 0; k < 16u; ++k) {
          const float w[4] = {held<TYPE>(v[k][0]), held<TYPE>(v[k][1]), held<TYPE>(v[k][2]), held<TYPE>(v[k][3])};
          if (32u * P + k < at.rows_left) store_four<TYPE>(e.pre, at.row + 32u * P + k, at, w);
        }
      }
    }
#pragma unroll
    for (uint32_t k = 0; k < 16u; ++k) {
      float none;
#pragma unroll
      for (uint32_t j = 0; j < 4u; ++j) activate<KIND, false, false>(v[k][j], &v[k][j], &none);
      if constexpr (WHOLE_EPILOGUE) {
        if (e.residual.at) {
          v[k][0] += widen_lo<TYPE>(r[k].x);
          v[k][1] += widen_hi<TYPE>(r[k].x);
          v[k][2] += widen_lo<TYPE>(r[k].y);
          v[k][3] += widen_hi<TYPE>(r[k].y);
        }
      }
      if (32u * P + k < at.rows_left) store_four<TYPE>(e.out, at.row + 32u * P + k, at, v[k]);
    }
  });
}

template <uint32_t TYPE, uint32_t A_MODE, uint32_t B_MODE, uint32_t TILE>
__global__ __launch_bounds__(kThreads, TILE == 256 ? 1 : 2) void lin_product_kernel(ProductArgs p) {
  using T = LinTile<TILE>;
  constexpr uint32_t S = T::S;
  extern __shared__ __attribute__((aligned(16))) uint8_t lin_lds[];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const uint32_t wm = wave / 2u, wn = wave % 2u, r = lane % 32u, h = lane / 32u;
  const uint32_t per = p.m_tiles * p.n_tiles, total = per * p.splits;
  const uint32_t all_steps = (p.k + kLinStep - 1u) / kLinStep, whole_steps = p.k / kLinStep;

  Loader<TYPE, A_MODE, TILE> la;
  Loader<TYPE, B_MODE, TILE> lb;
  using LA = Loader<TYPE, A_MODE, TILE>;
  using LB = Loader<TYPE, B_MODE, TILE>;

  uint32_t a_at[4], b_at[4];  // this lane's row of tile 0, by quarter of a step; of tile i: 32 numbers further on
#pragma unroll
  for (uint32_t i = 0; i < 4u; ++i) {
    a_at[i] = lin_place(wm * 32u * S + r, 2u * i + h);
    b_at[i] = lin_place(wn * 32u * S + r, 2u * i + h) + T::kOperand;
  }
  uint4 a[2][S], b[2][S];
  const auto read = [&](auto k, const uint8_t* from, auto sub) {  // read K of a quarter of a step
    constexpr uint32_t K = decltype(k)::value, SUB = decltype(sub)::value;
    if constexpr (K < S) b[SUB % 2u][K] = *reinterpret_cast<const uint4*>(from + b_at[SUB] + K * 4096u);
    else a[SUB % 2u][K - S] = *reinterpret_cast<const uint4*>(from + a_at[SUB] + (K - S) * 4096u);
  };
  lin_f16v acc[S][S];
  // S x S products of a quarter, with what f(slot) does after each
  const auto multiply = [&](auto sub, auto&& f) __attribute__((always_inline)) {
    constexpr uint32_t SUB = decltype(sub)::value;
    each<S * S>([&](auto q) __attribute__((always_inline)) {
      constexpr uint32_t Q = decltype(q)::value, I = Q / S, J = Q % S;
      acc[I][J] = mfma32<TYPE>(a[SUB % 2u][I], b[SUB % 2u][J], acc[I][J]);
      f(std::integral_constant<uint32_t, SUB * S * S + Q>{});
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  uint32_t id = blockIdx.x;
  uint32_t row0 = 0, col0 = 0, split = 0, step0 = 0, steps = 0;
  const auto take = [&]() __attribute__((always_inline)) {  // the next tile
    // (a division is done in the vector unit; what comes of it goes back to scalar registers here, not ahead of every load)
    split = __builtin_amdgcn_readfirstlane(id / per);
    uint32_t mt, nt;
    lin_band(lin_by_die(id - split * per, per), p.m_tiles, p.n_tiles, &mt, &nt);
    row0 = __builtin_amdgcn_readfirstlane(mt) * TILE;
    col0 = __builtin_amdgcn_readfirstlane(nt) * TILE;
    step0 = split * p.split_steps;
    steps = min(all_steps - min(step0, all_steps), p.split_steps);
    // (rows of the memory that were shorter than eight values are eight long here)
    la.aim(p.a, p.b8, row0, A_MODE == kAcross ? max(p.e.m, kLinShort) : p.e.m);
    lb.aim(p.b, p.b8, col0, B_MODE == kAcross ? max(p.e.n, kLinShort) : p.e.n);
  };
  constexpr uint32_t kReads = 2u * S;
  const uint32_t a_k = A_MODE == kAlong ? max(p.k, kLinShort) : p.k, b_k = B_MODE == kAlong ? max(p.k, kLinShort) : p.k;
  const auto turn = [&](uint32_t step) __attribute__((always_inline)) {
    la.turn(step, a_k);
    lb.turn(step, b_k);
  };
  const auto load_step = [&](uint32_t step) __attribute__((always_inline)) {
    turn(step);
    each<LA::kLoads>([&](auto i) __attribute__((always_inline)) { la.template load<decltype(i)::value>(); });
    each<LB::kLoads>([&](auto i) __attribute__((always_inline)) { lb.template load<decltype(i)::value>(); });
  };
  const auto mend = [&](uint32_t step) __attribute__((always_inline)) {
    if (step == whole_steps) {  // (uniform)
      la.mend(a_k - step * kLinStep);
      lb.mend(b_k - step * kLinStep);
    }
  };

  if (id >= total) return;
  take();
  if (steps) load_step(step0);
  for (;;) {
#pragma unroll
    for (uint32_t i = 0; i < S; ++i)
#pragma unroll
      for (uint32_t j = 0; j < S; ++j)
#pragma unroll
        for (uint32_t e = 0; e < 16u; ++e) acc[i][j][e] = 0.0f;
    if (steps) {  // (uniform)
      const uint32_t last = step0 + steps - 1u;
      mend(step0);
      each<LA::kStores>([&](auto i) { la.template store<decltype(i)::value>(lin_lds); });
      each<LB::kStores>([&](auto i) { lb.template store<decltype(i)::value>(lin_lds + T::kOperand); });
      load_step(min(step0 + 1u, last));
      lin_meet();
      each<kReads>([&](auto k) { read(k, lin_lds, std::integral_constant<uint32_t, 0>{}); });
      // A step's operands are read from one half of LDS, a quarter ahead of their products, while the next step's go from registers to the other, and those of the step behind that from memory
      // to the registers.  (Behind the last step it is loaded and stored again: one way through the loop for all of them.  A branch would part the loop's matrix instructions, and the
      // compiler moves the sums about between the parts.)
      //   The loads are spread over most of a step: the compute unit takes 64 bytes of them a cycle, 1024 cycles' worth of the 2048 that a step's matrix instructions take, and a wavefront
      // whose load is not taken issues nothing else either.
#pragma unroll 1
      for (uint32_t t = step0; t <= last; ++t) {
        uint8_t* const from = lin_lds + ((t - step0) % 2u) * T::kStage;
        uint8_t* const to = lin_lds + (1u - (t - step0) % 2u) * T::kStage;
        mend(min(t + 1u, last));
        turn(min(t + 2u, last));
        constexpr uint32_t P = S * S;  // slots of a quarter
        const auto task = [&](auto slot) __attribute__((always_inline)) {
          constexpr uint32_t SLOT = decltype(slot)::value, SUB = SLOT / P;
          in_slot<kReads, SUB * P, SUB * P + P / 2u, SLOT>([&](auto k) __attribute__((always_inline)) {
            read(k, SUB < 3u ? from : to, std::integral_constant<uint32_t, (SUB + 1u) % 4u>{});
          });
          in_slot<LA::kStores, P / 2u, P, SLOT>([&](auto k) __attribute__((always_inline)) { la.template store<decltype(k)::value>(to); });
          in_slot<LB::kStores, P + P / 2u, 2u * P, SLOT>([&](auto k) __attribute__((always_inline)) { lb.template store<decltype(k)::value>(to + T::kOperand); });
          in_slot<LA::kLoads, P, 5u * P / 2u, SLOT>([&](auto k) __attribute__((always_inline)) { la.template load<decltype(k)::value>(); });
          in_slot<LB::kLoads, 5u * P / 2u, 4u * P, SLOT>([&](auto k) __attribute__((always_inline)) { lb.template load<decltype(k)::value>(); });
        };
        multiply(std::integral_constant<uint32_t, 0>{}, task);
        multiply(std::integral_constant<uint32_t, 1>{}, task);
        multiply(std::integral_constant<uint32_t, 2>{}, task);
        lin_meet();  // the next step is there, and this one has been read
        multiply(std::integral_constant<uint32_t, 3>{}, task);
      }
    }
    const uint32_t out_row0 = row0, out_col0 = col0, out_split = split;
    id += gridDim.x;
    const bool more = id < total;
    if (more) {
      take();
      if (steps) load_step(step0);
    }
    if constexpr (TILE == 256u) {
      constexpr bool kWhole = A_MODE == kAlong && B_MODE == kAlong;  // (a gradient has nothing behind its product)
      LinResults at;
      const uint32_t first = out_row0 + wm * 128u + 16u * h;
      at.row = first;
      at.rows_left = first < p.e.m ? p.e.m - first : 0u;
      at.col = out_col0 + wn * 128u + 4u * r;
      at.have = at.col < p.e.n ? min(p.e.n - at.col, 4u) : 0u;
      if (at.have == 0u) at.rows_left = kWhole && p.e.pre8.codes ? at.rows_left : 0u;  // (all lanes take part in a group's scale)
      if constexpr (kWhole) {
        float bias[4];
#pragma unroll
        for (uint32_t j = 0; j < 4u; ++j) bias[j] = p.e.bias && j < at.have ? load1(p.e.btype, p.e.bias, at.col + j) : 0.0f;
        if (p.e.act == kActNone) results_of<TYPE, kActNone, true>(p.e, at, acc, bias);
        else if (p.e.act == kActGelu) results_of<TYPE, kActGelu, true>(p.e, at, acc, bias);
        else if (p.e.act == kActGeluTanh) results_of<TYPE, kActGeluTanh, true>(p.e, at, acc, bias);
        else results_of<TYPE, kActSilu, true>(p.e, at, acc, bias);
      } else {
        const float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        results_of<TYPE, kActNone, false>(p.e, at, acc, none);
      }
    } else {
      // Results by way of LDS, a quarter at a time: lane (r, h) holds rows 8 * (e / 4) + 4 * h + e % 4 and column r of a tile.  A thread then has the same eight columns of several rows.
      float* const room = reinterpret_cast<float*>(lin_lds);
      constexpr uint32_t kWide = TILE, kHalf = T::kPassRows, kOctets = kWide / 8u, kRows = 2u * kHalf, kDown = kThreads / kOctets, kAtOnce = 2u;
      static_assert(kRows % (kDown * kAtOnce) == 0u && kRows * kWide * 4u <= T::kStage, "");
      const uint32_t at = threadIdx.x % kOctets * 8u, col = out_col0 + at;
      const uint32_t wide = col < p.e.n ? p.e.n - col : 0u;
      float bias[8];
      load_bias<TYPE>(p.e, col, p.splits > 1u ? 0u : wide, bias);
      each<4>([&](auto pass) {
        constexpr uint32_t P = decltype(pass)::value;
        lin_meet();
#pragma unroll
        for (uint32_t e = 0; e < 4u; ++e) {
#pragma unroll
          for (uint32_t i = 0; i < S; ++i) {
            float* to = room + (wm * kHalf + S * (4u * h + e) + i) * kWide + wn * 32u * S + S * r;
            if constexpr (S == 4u) *reinterpret_cast<float4*>(to) = make_float4(acc[i][0][4 * P + e], acc[i][1][4 * P + e], acc[i][2][4 * P + e], acc[i][3][4 * P + e]);
            else *reinterpret_cast<float2*>(to) = make_float2(acc[i][0][4 * P + e], acc[i][1][4 * P + e]);
          }
        }
        lin_meet();
        // row `down` of half wm of the pass is row 32 * S * wm + kHalf * P + down
#pragma unroll 1
        for (uint32_t first = threadIdx.x / kOctets; first < kRows; first += kDown * kAtOnce) {
          float v[kAtOnce][8];
          uint32_t row[kAtOnce], left[kAtOnce];
#pragma unroll
          for (uint32_t n = 0; n < kAtOnce; ++n) {
            const uint32_t in = first + n * kDown, half = in / kHalf, down = in % kHalf;
            row[n] = out_row0 + half * 32u * S + kHalf * P + down;
            left[n] = row[n] < p.e.m ? wide : 0u;
            const float* from = room + in * kWide + at;
            const float4 lo = *reinterpret_cast<const float4*>(from), hi = *reinterpret_cast<const float4*>(from + 4);
            v[n][0] = lo.x; v[n][1] = lo.y; v[n][2] = lo.z; v[n][3] = lo.w;
            v[n][4] = hi.x; v[n][5] = hi.y; v[n][6] = hi.z; v[n][7] = hi.w;
          }
          if (p.splits > 1u) {
#pragma unroll
            for (uint32_t n = 0; n < kAtOnce; ++n) {
              Octet<kTypeF32> o;
              o.set(v[n]);
              o.store(p.partial, ((uint64_t)out_split * p.e.m + row[n]) * p.e.n + col, left[n]);
            }
          } else {
            finish<TYPE, kAtOnce>(p.e, row, col, left, bias, v);
          }
        }
      });
    }
    if (!more) return;
    lin_meet();
  }
}

// The parts of a contraction that was cut, added up in their order
template <uint32_t TYPE>
__global__ __launch_bounds__(kThreads) void lin_join_kernel(JoinArgs p) {
  const uint32_t groups = (p.e.n + kR8Group - 1u) / kR8Group;
  const uint64_t unit = (uint64_t)blockIdx.x * (kThreads / kR8Lanes) + threadIdx.x / kR8Lanes;
  const uint32_t row = (uint32_t)(unit / groups), col = (uint32_t)(unit % groups) * kR8Group + threadIdx.x % kR8Lanes * 8u;
  const uint32_t left[1] = {row < p.e.m && col < p.e.n ? p.e.n - col : 0u}, rows[1] = {row};
  float v[1][8], bias[8];
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) v[0][i] = 0.0f;
  for (uint32_t s = 0; s < p.splits; ++s) {
    Octet<kTypeF32> o;
    float w[8];
    o.load(p.partial, ((uint64_t)s * p.e.m + row) * p.e.n, col, left[0]);
    o.get(w);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) v[0][i] += w[i];
  }
  load_bias<TYPE>(p.e, col, left[0], bias);
  finish<TYPE, 1>(p.e, rows, col, left, bias, v);
}
JoinFn join_fn(uint32_t type) { return type == kTypeF16 ? lin_join_kernel<kTypeF16> : lin_join_kernel<kTypeBf16>; }

// ------------------------------------------------------------------ few rows
// Where nothing is kept of what an activation is given.  A workgroup takes 16 * NS rows of w and up to 16 * MS rows of x; its wavefronts share the contraction, U steps of 32 at a time in turn,
// and add their sums up in LDS, in the wavefronts' order.  Values go from memory to the operand registers: lane (r, q) = (lane % 16, lane / 16) reads values 8 q to 8 q + 7 of the step of its row.  A turn's loads
// are under way while the turn before is multiplied.
//   What bounds it is reading w once, from many compute units at a time: one row by 11008 x 4096 18 us (5.0 TB/s), by 4096 x 4096 8.5; 16 rows by 4096 x 11008 22 to 26 (4.1 to 3.4), of which 6 are x,
// which every workgroup reads; 17 rows by 11008 x 4096 23, 32 rows 26 (3.9 and 3.5), by 4096 x 4096 11 and 14, 32 by 4096 x 11008 32: x again, twice as much of it.  Tried for the first two: 12 and 16 wavefronts (19.8 and 21.2; 26.2 and 26.3); 32 and 64 columns a workgroup (25.0 and 24.5; 33.9 and 52.4); each workgroup
// beginning elsewhere in the contraction (20.4; 24.9).
template <uint32_t MS, uint32_t NS>
struct FewTurn {
  static constexpr uint32_t U = NS + MS <= 3u ? 4u : 2u;  // two turns in the registers of a lane
  uint4 b[U][NS];
  uint4 a[U][MS];
};

// Rows' ends are loaded piece after piece: all of them at once would not fit in the registers
__device__ __forceinline__ void in_turn() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <uint32_t TYPE, uint32_t MS, uint32_t NS>
__global__ __launch_bounds__(8 * kWave) void lin_few_kernel(ProductArgs p) {
  using F = FewTurn<MS, NS>;
  constexpr uint32_t U = F::U;
  extern __shared__ __attribute__((aligned(16))) uint8_t lin_lds[];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, waves = blockDim.x / kWave;
  const uint32_t r = lane % 16u, q = lane / 16u;
  const uint32_t row0 = blockIdx.x / p.n_tiles * 16u * MS, col0 = blockIdx.x % p.n_tiles * 16u * NS;
  const uint32_t rows = min(p.e.m - row0, 16u * MS), cols = min(p.e.n - col0, 16u * NS);
  const uint32_t steps = (p.k + 31u) / 32u;

  lin_f4v acc[MS][NS];
#pragma unroll
  for (uint32_t i = 0; i < MS; ++i)
#pragma unroll
    for (uint32_t j = 0; j < NS; ++j) acc[i][j] = lin_f4v{0.0f, 0.0f, 0.0f, 0.0f};
  // rows behind the last read the last one: results that are not kept
  const uint16_t* b_row[NS];
  const uint16_t* a_row[MS];
#pragma unroll
  for (uint32_t j = 0; j < NS; ++j) b_row[j] = static_cast<const uint16_t*>(p.b.at) + (uint64_t)(col0 + min(NS * r + j, cols - 1u)) * p.b.stride + 8u * q;
#pragma unroll
  for (uint32_t i = 0; i < MS; ++i) a_row[i] = static_cast<const uint16_t*>(p.a.at) + (uint64_t)(row0 + min(16u * i + r, rows - 1u)) * p.a.stride + 8u * q;

  const auto one = [&](const uint16_t* row, uint32_t c) {  // values c + 8 q ... of a row, zeros behind its end: read where there are eight, and moved
    const uint32_t at = c + 8u * q, left = at < p.k ? min(p.k - at, 8u) : 0u;
    const u4_any w = *reinterpret_cast<const u4_any*>(row + (int32_t)(min(at, p.k - 8u) - 8u * q));
    return lin_move_down(make_uint4(w.x, w.y, w.z, w.w), 16u * (8u - left));
  };
  const auto load = [&](F& t, uint32_t s0) {
    if ((s0 + U) * 32u <= p.k) {
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
#pragma unroll
        for (uint32_t j = 0; j < NS; ++j) {
          const u4_any w = *reinterpret_cast<const u4_any*>(b_row[j] + (s0 + u) * 32u);
          t.b[u][j] = make_uint4(w.x, w.y, w.z, w.w);
        }
      }
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
#pragma unroll
        for (uint32_t i = 0; i < MS; ++i) {
          const u4_any w = *reinterpret_cast<const u4_any*>(a_row[i] + (s0 + u) * 32u);
          t.a[u][i] = make_uint4(w.x, w.y, w.z, w.w);
        }
      }
    } else {
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
#pragma unroll
        for (uint32_t j = 0; j < NS; ++j) {
          t.b[u][j] = one(b_row[j], (s0 + u) * 32u);
          in_turn();
        }
#pragma unroll
        for (uint32_t i = 0; i < MS; ++i) {
          t.a[u][i] = one(a_row[i], (s0 + u) * 32u);
          in_turn();
        }
      }
    }
  };
  const auto multiply = [&](F& t) {  // (what is behind the contraction's end is zeros)
#pragma unroll
    for (uint32_t u = 0; u < U; ++u)
#pragma unroll
      for (uint32_t i = 0; i < MS; ++i)
#pragma unroll
        for (uint32_t j = 0; j < NS; ++j) acc[i][j] = mfma16<TYPE>(t.a[u][i], t.b[u][j], acc[i][j]);
  };
  const uint32_t apart = U * waves;
  uint32_t s0 = U * wave;
  F first, second;
  if (s0 < steps) {  // (uniform in the wavefront)
    load(first, s0);
    for (;;) {
      if (s0 + apart < steps) load(second, s0 + apart);
      multiply(first);
      s0 += apart;
      if (s0 >= steps) break;
      if (s0 + apart < steps) load(first, s0 + apart);
      multiply(second);
      s0 += apart;
      if (s0 >= steps) break;
    }
  }
  // lane (r, q) holds rows 4 * q + e and column r of a tile; [wave][row][column] in LDS
  float* sums = reinterpret_cast<float*>(lin_lds);
  constexpr uint32_t kCols = 16u * NS, kRows = 16u * MS;
#pragma unroll
  for (uint32_t i = 0; i < MS; ++i)
#pragma unroll
    for (uint32_t e = 0; e < 4u; ++e)
#pragma unroll
      for (uint32_t j = 0; j < NS; ++j) sums[(wave * kRows + 16u * i + 4u * q + e) * kCols + NS * r + j] = acc[i][j][e];
  __syncthreads();
  for (uint32_t t = threadIdx.x; t < rows * kCols; t += blockDim.x) {
    const uint32_t row = t / kCols, in = t % kCols;
    if (in >= cols) continue;
    float v = 0.0f, none;
    for (uint32_t u = 0; u < waves; ++u) v += sums[(u * kRows + row) * kCols + in];
    const uint32_t col = col0 + in;
    if (p.e.bias) v += load1(p.e.btype, p.e.bias, col);
    if (p.e.act == kActGelu) activate<kActGelu, false, false>(v, &v, &none);
    else if (p.e.act == kActGeluTanh) activate<kActGeluTanh, false, false>(v, &v, &none);
    else if (p.e.act == kActSilu) activate<kActSilu, false, false>(v, &v, &none);
    if (p.e.residual.at) v += load1<TYPE>(p.e.residual.at, (uint64_t)(row0 + row) * p.e.residual.stride + col);
    store1<TYPE>(p.e.out.at, (uint64_t)(row0 + row) * p.e.out.stride + col, v);
  }
}

// Rows of fewer than eight values to rows of eight, zeros behind them
__global__ __launch_bounds__(kThreads) void lin_pad_kernel(const uint16_t* src, uint64_t stride, uint32_t rows, uint32_t cols, uint4* dst) {
  const uint32_t row = blockIdx.x * kThreads + threadIdx.x;
  if (row >= rows) return;
  Octet<kTypeBf16> o;
  o.load(src, (uint64_t)row * stride, 0u, cols);
  dst[row] = make_uint4(o.w[0].x, o.w[0].y, o.w[0].z, o.w[0].w);
}
PadFn pad_fn() { return lin_pad_kernel; }

template <uint32_t TYPE>
static ProductFn few_of(uint32_t ms, uint32_t ns) {
  return ms == 1 ? lin_few_kernel<TYPE, 1, 1> : ns == 1 ? lin_few_kernel<TYPE, 2, 1> : lin_few_kernel<TYPE, 2, 4>;
}
ProductFn linear_few_fn(uint32_t type, uint32_t ms, uint32_t ns) { return type == kTypeF16 ? few_of<kTypeF16>(ms, ns) : few_of<kTypeBf16>(ms, ns); }

template <uint32_t TYPE, uint32_t TILE>
static ProductFn product_of(uint32_t a_mode, uint32_t b_mode) {
  if (a_mode == kAlong) return b_mode == kAlong ? lin_product_kernel<TYPE, kAlong, kAlong, TILE> : lin_product_kernel<TYPE, kAlong, kAcross, TILE>;
  return b_mode == kAcross ? lin_product_kernel<TYPE, kAcross, kAcross, TILE> : lin_product_kernel<TYPE, kAcross, kAcross8, TILE>;
}
ProductFn product_fn(uint32_t type, uint32_t a_mode, uint32_t b_mode, uint32_t tile) {
  if (type == kTypeF16) return tile == 256 ? product_of<kTypeF16, 256>(a_mode, b_mode) : product_of<kTypeF16, 128>(a_mode, b_mode);
  return tile == 256 ? product_of<kTypeBf16, 256>(a_mode, b_mode) : product_of<kTypeBf16, 128>(a_mode, b_mode);
}
uint32_t product_lds(uint32_t tile) { return tile == 256 ? LinTile<256>::kLds : LinTile<128>::kLds; }

}  // namespace adacc
