// Products of matrices in microscaled 4-bit floating point: out[m][n] = sum over k of a[m][k] * b[n][k], both operands' blocks along the
// contraction.  Dense; with the rows of a sorted by group and a matrix b for each group (experts); and the gradient of such matrices, where
// the groups cut the contraction.
//
// The scaled matrix instructions multiply 32 x 64 by 64 x 32 codes (or 16 x 128 by 128 x 16): a lane gives 16 bytes of codes, one block
// of a row, and that block's scale byte.  The products of two codes are exact, sums are kept in binary32.
#include <type_traits>
#include <utility>

#include "adacc_mx4.hpp"

namespace adacc {

typedef int mx_i8v __attribute__((ext_vector_type(8)));
typedef float mx_f16v __attribute__((ext_vector_type(16)));
typedef float mx_f4v __attribute__((ext_vector_type(4)));
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 mx_f16x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t mx_u16x2 __attribute__((ext_vector_type(2)));

constexpr int kMxFp4 = 4;  // the matrix instructions' code for E2M1

__device__ __forceinline__ mx_i8v mx_operand(uint4 c) {
  const mx_i8v v = {(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};  // (4-bit codes fill the first four registers)
  return v;
}

// two values in a 16-bit format, round to nearest even
__device__ __forceinline__ uint32_t mx_narrow2(uint32_t type, float lo, float hi) {
  const mx_f32x2 v = {lo, hi};
  return type == kMxBf16 ? __builtin_bit_cast(uint32_t, __builtin_convertvector(v, mx_bf16x2))
                         : __builtin_bit_cast(uint32_t, __builtin_convertvector(v, mx_f16x2));
}
__device__ __forceinline__ void mx_store1(void* out, uint32_t type, uint64_t at, float v) {
  if (type == kMxF32) static_cast<float*>(out)[at] = v;
  else static_cast<uint16_t*>(out)[at] = (uint16_t)mx_narrow2(type, v, v);
}
// N (1, 2 or 4) adjacent values, at any element's address (rows of an odd number of values are not aligned)
template <uint32_t N>
__device__ __forceinline__ void mx_store(uint8_t* p, uint32_t type, const float (&v)[N]) {
  if constexpr (N == 1) {
    mx_store1(p, type, 0, v[0]);
  } else if (type == kMxF32) {
    if constexpr (N == 4) *reinterpret_cast<mx_u4u*>(p) = mx_u4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    else *reinterpret_cast<mx_u2u*>(p) = mx_u2u{__float_as_uint(v[0]), __float_as_uint(v[1])};
  } else {
    if constexpr (N == 4) *reinterpret_cast<mx_u2u*>(p) = mx_u2u{mx_narrow2(type, v[0], v[1]), mx_narrow2(type, v[2], v[3])};
    else *reinterpret_cast<mx_u1u*>(p) = mx_narrow2(type, v[0], v[1]);
  }
}

// ------------------------------------------------------------------ tiles
// A workgroup of four wavefronts, two by two, takes a tile of BM x BN results, a wavefront SM x SN tiles of 32 x 32 of it.  Codes and scales
// of a step (128 columns) go to LDS by loads that pass the registers by, DEPTH steps in a ring.
//
// What bounds it is power: a step of a tile of 256 takes 1110 to 1180 cycles, 1024 of which are matrix instructions, but on random codes the clock is 1.5 GHz
// meanwhile (2.4 on zeros).  8192 x 2048 x 8192 takes 63 us, 4.3 PFLOP/s, 16384 x 11008 x 4096 335 to 350, 4.2 to 4.4: the matrix unit is busy 70 and 57 % of the cycles, but as
// often a second in both, the clock being 1.4 and 1.7 GHz.  Beside the steps a round of tiles has its ring's start and its results (33 MB in 16 bits, within 6 us; all 361 MB of
// the second product 77 us, by a contraction of length zero).
//
// Row SM * r + i of a wavefront's rows is row r of its tile i: the SM scale bytes that a lane needs lie side by side, and so do, on the
// right-hand side, the SN columns of the results that it holds.
//
// A load of a wavefront brings 16 adjacent rows' 64 bytes of a step, one KiB of memory and of LDS, in four pieces of 16 bytes a row.  Within it LDS holds
// the rows tile by tile (Q = 16 / SM of each), and piece c of a tile's row r at place c ^ (r / 4 % 4), so that sixteen lanes that read one
// piece of adjacent rows of a tile meet all banks.
template <uint32_t BM, uint32_t BN, uint32_t DEPTH>
struct MxTile {
  static constexpr uint32_t SM = BM / 64u, SN = BN / 64u;
  static constexpr uint32_t QM = 16u / SM, QN = 16u / SN;
  static constexpr uint32_t kA = BM * kMxStepBytes, kB = BN * kMxStepBytes;
  static constexpr uint32_t kScaleA = kA + kB, kScaleB = kScaleA + 4u * BM;
  static constexpr uint32_t kStage = kScaleB + 4u * BN;
  static constexpr uint32_t kLds = kStage * DEPTH;
  static constexpr uint32_t kCodeLoads = (BM + BN) / 16u / kWavesPerWg;  // of 1 KiB, by each wavefront
  static constexpr uint32_t kScaleWords = (BM + BN) / 64u;               // loads of 256 bytes by all of them
  static constexpr uint32_t kScaleLoads = kScaleWords < kWavesPerWg ? 1u : kScaleWords / kWavesPerWg;
  static constexpr uint32_t kLoads = kCodeLoads + kScaleLoads;
};

// 16 (or 4) bytes a lane from base + voff to LDS at `lds` and, lane after lane, behind it.  The counter of vector loads counts it; nothing waits for it
// but mx_wait_loads (the compiler would wait for all such loads before any read of LDS).
// m0 holds the address in LDS; it is an operand, so that the compiler knows of it, and the block waits one state between its write and the load.  A vector
// load may read an SGPR that a vector instruction has written (readfirstlane, or readlane of a spilled one) five wait states later; the compiler does not look into
// the block, so tests/test_mx4_instructions.py looks at what it puts ahead of it.  (Five states in the block: 1 % of a product's time.)
__device__ __forceinline__ void mx_to_lds16(uint32_t lds, const uint8_t* base, uint32_t voff) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "{m0}"(lds), "v"(voff), "s"(base) : "memory");
}
__device__ __forceinline__ void mx_to_lds4(uint32_t lds, const uint8_t* base, uint32_t voff) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, %2" : : "{m0}"(lds), "v"(voff), "s"(base) : "memory");
}
// a pointer that is the same in all lanes, known to be so
__device__ __forceinline__ const uint8_t* mx_uniform(const uint8_t* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const uint8_t*>((uint64_t)hi << 32 | lo);
}
template <uint32_t N>
__device__ __forceinline__ void mx_wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
// every wavefront's reads of LDS before it have returned, its loads are where mx_wait_loads has left them
__device__ __forceinline__ void mx_meet() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

__device__ __forceinline__ uint32_t mx_lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

template <uint32_t S>
__device__ __forceinline__ uint32_t mx_scales_of(const uint8_t* p) {
  if constexpr (S == 4) return *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (S == 2) return *reinterpret_cast<const uint16_t*>(p);
  else return *p;
}

template <uint32_t I, uint32_t J>
__device__ __forceinline__ mx_f16v mx_mfma32(uint4 a, uint4 b, mx_f16v c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_operand(a), mx_operand(b), c, kMxFp4, kMxFp4, I, (int)sa, J, (int)sb);
}
constexpr uint32_t mx_least(uint32_t a, uint32_t b) { return a < b ? a : b; }

// f(0), f(1), ... f(N - 1), with constants
template <uint32_t N, typename F, uint32_t... I>
__device__ __forceinline__ void mx_each(F&& f, std::integer_sequence<uint32_t, I...>) {
  (f(std::integral_constant<uint32_t, I>{}), ...);
}
template <uint32_t N, typename F>
__device__ __forceinline__ void mx_each(F&& f) {
  mx_each<N>(f, std::make_integer_sequence<uint32_t, N>{});
}
// The SM x SN tiles of a half step, with TASKS tasks spread over them: a wavefront issues in order, and the 32 cycles that a matrix
// instruction takes are the time for everything else.  (All other instructions ahead of the matrix instructions, as the compiler puts
// them: 4.1k cycles a step in tiles of 256, of which 1k are matrix instructions.)
template <uint32_t TASKS, uint32_t SM, uint32_t SN, typename F>
__device__ __forceinline__ void mx_multiply(mx_f16v (&acc)[SM][SN], const uint4 (&a)[SM], const uint4 (&b)[SN], uint32_t sa, uint32_t sb, F&& task) {
  mx_each<SM * SN>([&](auto q) {
    constexpr uint32_t Q = decltype(q)::value, I = Q / SN, J = Q % SN;
    acc[I][J] = mx_mfma32<I, J>(a[I], b[J], acc[I][J], sa, sb);
    constexpr uint32_t kEach = (TASKS + SM * SN - 1u) / (SM * SN);  // tasks come early: what they read has the rest of the half step to arrive
    constexpr uint32_t kFrom = Q * kEach < TASKS ? Q * kEach : TASKS, kTo = (Q + 1u) * kEach < TASKS ? (Q + 1u) * kEach : TASKS;
    mx_each<kTo - kFrom>([&](auto k) { task(std::integral_constant<uint32_t, kFrom + decltype(k)::value>{}); });
    __builtin_amdgcn_sched_barrier(0);
  });
}

// What a workgroup computes: rows [a_row0, ..) of a by rows [b_row0, ..) of b over steps [step0, step0 + steps)
struct MxWork {
  uint32_t a_row0, b_row0;   // multiples of 4
  uint32_t step0, steps;
  uint32_t a_first, a_last;  // rows of a that are kept
  uint32_t b_first, b_last;
  void* out;                 // the result of (a_first, b_first) ...
  uint64_t stride;
};

// The workgroup's tiles, one after the other: next(&work) gives the next one, or false.  The first loads of a tile are on their way while the
// results of the one before are written.
template <uint32_t BM, uint32_t BN, uint32_t DEPTH, typename Next>
__device__ __forceinline__ void mx_tiles(const MxProductArgs& p, uint8_t* lds, Next&& next_work) {
  using T = MxTile<BM, BN, DEPTH>;
  constexpr uint32_t SM = T::SM, SN = T::SN;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const uint32_t wm = wave / 2u, wn = wave % 2u;
  const uint32_t r = lane % 32u, h = lane / 32u;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(mx_lds_address(lds));

  // ---- what this wavefront loads of every step
  constexpr uint32_t kALoads = BM / 16u / kWavesPerWg;  // of 1 KiB, by a wavefront
  constexpr uint32_t kAWords = BM / 64u;                // of 256 bytes, by all of them
  const uint8_t* a_mem;  // of the next step to be loaded
  const uint8_t* b_mem;
  const uint8_t* scale_mem[T::kScaleLoads];
  uint64_t scale_step[T::kScaleLoads];
  uint32_t code_off[T::kCodeLoads], scale_off[T::kScaleLoads];
  // Rows behind the matrix's last read the last one: the results are not kept.
  const auto aim = [&](const MxWork& w) {
    a_mem = mx_uniform(p.a.codes + (uint64_t)w.step0 * p.a.step_bytes + (uint64_t)w.a_row0 * kMxStepBytes);
    b_mem = mx_uniform(p.b.codes + (uint64_t)w.step0 * p.b.step_bytes + (uint64_t)w.b_row0 * kMxStepBytes);
#pragma unroll
    for (uint32_t i = 0; i < T::kCodeLoads; ++i) {
      const bool is_a = i < kALoads;
      const uint32_t block = (is_a ? i : i - kALoads) * kWavesPerWg + wave, slot = lane / 4u;
      const uint32_t s = is_a ? SM : SN, q = 16u / s;
      const uint32_t row = block * 16u + s * (slot % q) + slot / q;
      const uint32_t most = (is_a ? p.a.rows - w.a_row0 : p.b.rows - w.b_row0) - 1u;
      const uint32_t piece = (lane % 4u) ^ ((block * q + slot % q) / 4u % 4u);  // (a tile's rows are counted by 32, a multiple of 16)
      code_off[i] = min(row, most) * kMxStepBytes + piece * 16u;
    }
#pragma unroll
    for (uint32_t i = 0; i < T::kScaleLoads; ++i) {
      const uint32_t load = (i * kWavesPerWg + wave) % T::kScaleWords;
      const bool is_a = load < kAWords;
      const uint32_t rows = is_a ? BM : BN;
      const uint32_t at = (is_a ? load : load - kAWords) * 256u + lane * 4u;
      const uint64_t pitch = is_a ? p.a.pitch : p.b.pitch;
      const uint32_t row0 = is_a ? w.a_row0 : w.b_row0;
      scale_off[i] = (uint32_t)((at / rows) * pitch) + min(at % rows, (uint32_t)pitch - row0 - 4u);
      scale_mem[i] = mx_uniform((is_a ? p.a.scales : p.b.scales) + (uint64_t)(4u * w.step0) * pitch + row0);
      scale_step[i] = 4u * pitch;
    }
  };
  // load I of the next step, to `stage`; the last of a matrix moves on
  const auto load = [&](auto i, uint32_t stage) {
    constexpr uint32_t I = decltype(i)::value;
    const uint32_t to = lds0 + stage * T::kStage;
    if constexpr (I < T::kCodeLoads) {
      mx_to_lds16(to + (I * kWavesPerWg + wave) * 1024u, I < kALoads ? a_mem : b_mem, code_off[I]);
      if constexpr (I == kALoads - 1u) a_mem += p.a.step_bytes;
      if constexpr (I == T::kCodeLoads - 1u) b_mem += p.b.step_bytes;
    } else {
      constexpr uint32_t S = I - T::kCodeLoads;
      const uint32_t word = (S * kWavesPerWg + wave) % T::kScaleWords;
      mx_to_lds4(to + T::kScaleA + word * 256u, scale_mem[S], scale_off[S]);
      scale_mem[S] += scale_step[S];
    }
  };
  // A step's loads go out in two parts, one in either half of the step before last, so that every half has as many tasks
  constexpr uint32_t kEarly = T::kLoads / 2u;
  const auto load_early = [&](uint32_t to) { mx_each<kEarly>([&](auto i) { load(i, to); }); };
  const auto load_rest = [&](uint32_t to) { mx_each<T::kLoads - kEarly>([&](auto i) { load(std::integral_constant<uint32_t, kEarly + decltype(i)::value>{}, to); }); };
  const auto load_first = [&](uint32_t steps) {
    for (uint32_t d = 0; d + 1u < DEPTH && d < steps; ++d) {
      load_early(d);
      load_rest(d);
    }
    if (steps >= DEPTH) load_early(DEPTH - 1u);
  };

  // ---- where this lane reads its row of tile 0 (of the others: QM resp. QN rows further on)
  uint32_t a_at[2], b_at[2];  // by half of the step
#pragma unroll
  for (uint32_t s = 0; s < 2u; ++s) {
    const uint32_t place = ((2u * s + h) ^ (r / 4u % 4u)) * 16u;
    a_at[s] = wm * 32u * SM * kMxStepBytes + (r / T::QM) * 1024u + r % T::QM * kMxStepBytes + place;
    b_at[s] = T::kA + wn * 32u * SN * kMxStepBytes + (r / T::QN) * 1024u + r % T::QN * kMxStepBytes + place;
  }
  const uint32_t as_at = T::kScaleA + h * BM + wm * 32u * SM + SM * r;
  const uint32_t bs_at = T::kScaleB + h * BN + wn * 32u * SN + SN * r;
  uint4 a[2][SM], b[2][SN];
  uint32_t sa[2], sb[2];
  constexpr uint32_t kReads = SM + SN + 2u;
  const auto read = [&](auto k, const uint8_t* from, uint32_t s) {  // read K of half a step
    constexpr uint32_t K = decltype(k)::value;
    if constexpr (K == 0) sa[s] = mx_scales_of<SM>(from + as_at + 2u * s * BM);
    else if constexpr (K == 1) sb[s] = mx_scales_of<SN>(from + bs_at + 2u * s * BN);
    else if constexpr (K < 2u + SN) b[s][K - 2u] = *reinterpret_cast<const uint4*>(from + b_at[s] + (K - 2u) * T::QN * kMxStepBytes);
    else a[s][K - 2u - SN] = *reinterpret_cast<const uint4*>(from + a_at[s] + (K - 2u - SN) * T::QM * kMxStepBytes);
  };

  mx_f16v acc[SM][SN];
  MxWork w;
  if (!next_work(w)) return;
  aim(w);
  load_first(w.steps);
  // Stores count as loads do, in order: the kStores of the tile before went out behind this tile's first loads, and what waits for one of those
  // need not wait for them.  (Where a tile of results was not stored in one piece, their number is not known, and they are waited for.)
  constexpr uint32_t kStores = 16u * SM;
  bool behind = false;
  for (;;) {
    MxWork following;
    const bool more = next_work(following);
#pragma unroll
    for (uint32_t i = 0; i < SM; ++i)
#pragma unroll
      for (uint32_t j = 0; j < SN; ++j)
#pragma unroll
        for (uint32_t e = 0; e < 16u; ++e) acc[i][j][e] = 0.0f;

    if (w.steps) {  // (uniform in the workgroup)
      if (w.steps >= DEPTH) {
        if (behind) mx_wait_loads<mx_least(T::kLoads * (DEPTH - 2u) + kEarly + kStores, 63u)>();
        else mx_wait_loads<T::kLoads * (DEPTH - 2u) + kEarly>();
      } else {
        mx_wait_loads<0>();
        behind = false;
      }
      mx_meet();
      mx_each<kReads>([&](auto k) { read(k, lds, 0u); });
      uint32_t stage = 0, t = 0;
      // One step, but the last: its first half is in registers; the second half of the step is read under the first half's products, the
      // first half of the next step under the second's.  REST: the step DEPTH - 1 further on exists, its second part is loaded to where the
      // step before was; EARLY: so does the one behind it, whose first part is loaded to this step's place.
      const auto step = [&](auto rest, auto early) {
        constexpr uint32_t kRest = decltype(rest)::value ? T::kLoads - kEarly : 0u, kFirst = decltype(early)::value ? kEarly : 0u;
        const uint8_t* from = lds + stage * T::kStage;
        const uint32_t next = stage + 1u == DEPTH ? 0u : stage + 1u, before = stage == 0u ? DEPTH - 1u : stage - 1u;
        mx_multiply<kReads + kRest>(acc, a[0], b[0], sa[0], sb[0], [&](auto k) {
          constexpr uint32_t K = decltype(k)::value;
          if constexpr (K < kReads) read(k, from, 1u);
          else load(std::integral_constant<uint32_t, kEarly + K - kReads>{}, before);
        });
        // the next step has landed (of those behind it DEPTH - 2 are on their way), this one has been read: for every wavefront
        if constexpr (kRest) {
          if (behind && t + 2u < DEPTH) mx_wait_loads<mx_least(T::kLoads * (DEPTH - 2u) + kStores, 63u)>();
          else mx_wait_loads<T::kLoads * (DEPTH - 2u)>();
        } else {
          mx_wait_loads<0>();
        }
        mx_meet();
        const uint8_t* from_next = lds + next * T::kStage;
        mx_multiply<kReads + kFirst>(acc, a[1], b[1], sa[1], sb[1], [&](auto k) {
          constexpr uint32_t K = decltype(k)::value;
          if constexpr (K < kReads) read(k, from_next, 0u);
          else load(std::integral_constant<uint32_t, K - kReads>{}, stage);
        });
        stage = next;
        ++t;
      };
      while (t + DEPTH < w.steps) step(std::true_type{}, std::true_type{});
      if (t + DEPTH == w.steps) step(std::true_type{}, std::false_type{});
      while (t + 1u < w.steps) step(std::false_type{}, std::false_type{});
      const uint8_t* from = lds + stage * T::kStage;
      mx_multiply<kReads>(acc, a[0], b[0], sa[0], sb[0], [&](auto k) { read(k, from, 1u); });
      mx_multiply<0>(acc, a[1], b[1], sa[1], sb[1], [](auto) {});
    }
    if (more) {
      mx_meet();  // every wavefront has read its last step
      aim(following);
      load_first(following.steps);
    }

    // results: lane (r, h) holds rows 8 * (e / 4) + 4 * h + e % 4 and column r of a tile
    const uint32_t row0 = w.a_row0 + wm * 32u * SM, col0 = w.b_row0 + wn * 32u * SN;  // of the wavefront
    const uint32_t size = p.out_type == kMxF32 ? 4u : 2u;
    const uint32_t high = w.a_last - w.a_first, wide = w.b_last - w.b_first;
    const uint32_t from_row = row0 - w.a_first, from_col = col0 - w.b_first;  // (beyond the ends, or "negative", at a group's edges)
    behind = w.stride < (1u << 24) && from_row < high && 32u * SM <= high - from_row && from_col < wide && 32u * SN <= wide - from_col;  // (uniform)
    const uint64_t down = w.stride * size;
    if (behind) {
      uint8_t* out = static_cast<uint8_t*>(w.out) + (uint64_t)from_row * down + (uint64_t)from_col * size;
      const uint32_t lane_off = (SM * 4u * h * (uint32_t)w.stride + SN * r) * size;  // (below 2^32: uniform addresses and an offset a lane)
      const auto store_all = [&](auto type) {
        constexpr uint32_t kType = decltype(type)::value;
#pragma unroll
        for (uint32_t e = 0; e < 16u; ++e) {
#pragma unroll
          for (uint32_t i = 0; i < SM; ++i) {
            float v[SN];
#pragma unroll
            for (uint32_t j = 0; j < SN; ++j) v[j] = acc[i][j][e];
            mx_store<SN>(out + (uint64_t)(SM * (8u * (e / 4u) + e % 4u) + i) * down + lane_off, kType, v);
          }
        }
      };
      if (p.out_type == kMxBf16) store_all(std::integral_constant<uint32_t, kMxBf16>{});
      else if (p.out_type == kMxF16) store_all(std::integral_constant<uint32_t, kMxF16>{});
      else store_all(std::integral_constant<uint32_t, kMxF32>{});
    } else {
      // at the edges: rows are looked at one by one, and the columns of a lane that has some inside and some outside
      const uint32_t lane_col = from_col + SN * r;
      const bool whole = lane_col < wide && SN <= wide - lane_col;
      const auto store_some = [&](auto type) {
        constexpr uint32_t kType = decltype(type)::value;
        uint32_t row = from_row + SM * 4u * h;
        uint8_t* at = static_cast<uint8_t*>(w.out) + (int64_t)(int32_t)row * (int64_t)down + (int64_t)(int32_t)lane_col * size;
#pragma unroll
        for (uint32_t e = 0; e < 16u; ++e) {
#pragma unroll
          for (uint32_t i = 0; i < SM; ++i) {
            if (row < high) {
              float v[SN];
#pragma unroll
              for (uint32_t j = 0; j < SN; ++j) {
                v[j] = acc[i][j][e];
                asm volatile("" : "+v"(v[j]));  // (or the compiler rounds all values ahead of the branch, for all ways at once)
              }
              if (whole) {
                mx_store<SN>(at, kType, v);
              } else if constexpr (SN < 4u) {  // (tiles of 256 are only asked for where a lane's columns are all inside or all outside)
#pragma unroll
                for (uint32_t j = 0; j < SN; ++j)
                  if (lane_col + j < wide) mx_store1(at, kType, j, v[j]);
              }
            }
            const uint32_t by = e % 4u == 3u && i == SM - 1u ? 4u * SM + 1u : 1u;
            row += by;
            at += by * down;
            // (row after row: 64 addresses at once would not fit in the registers.  Of a pointer that has gone through here the compiler does not know that it is
            // global: the stores are flat, and waited for with the next tile's first reads of LDS.  Global ones, by a distance: 16384 rows of 16 groups by 4096 x 2048, 98 us, take 1 us more)
            asm volatile("" : "+v"(row), "+v"(at));
          }
        }
      };
      if (p.out_type == kMxBf16) store_some(std::integral_constant<uint32_t, kMxBf16>{});
      else if (p.out_type == kMxF16) store_some(std::integral_constant<uint32_t, kMxF16>{});
      else store_some(std::integral_constant<uint32_t, kMxF32>{});
    }
    if (!more) return;
    w = following;
  }
}

__device__ __forceinline__ void* mx_out_at(const MxProductArgs& p, uint64_t elems) {
  return static_cast<uint8_t*>(p.out) + elems * (p.out_type == kMxF32 ? 4u : 2u);
}

// The eight dies have a second-level cache each and take workgroups in turn: numbered so that a die's are neighbours, tiles go in
// bands of 8 tile rows, column by column, so that what runs at the same time on a die shares both operands.
__device__ __forceinline__ uint32_t mx_by_die(uint32_t id, uint32_t total) {
  constexpr uint32_t kDies = 8u;
  const uint32_t die = id % kDies, turn = id / kDies, each = total / kDies, more = total % kDies;
  return die * each + min(die, more) + turn;
}
__device__ __forceinline__ void mx_band(uint32_t id, uint32_t m_tiles, uint32_t n_tiles, uint32_t* mt, uint32_t* nt) {
  constexpr uint32_t kBand = 8u;
  const uint32_t band = id / (kBand * n_tiles), in = id - band * kBand * n_tiles;
  const uint32_t high = min(kBand, m_tiles - band * kBand);
  *nt = in / high;
  *mt = band * kBand + in - *nt * high;
}

// Workgroups take tiles blockIdx.x, blockIdx.x + gridDim.x, ... (the host launches as many as run at the same time)
// ---- rows by groups (or one group): a tile row lies within a group
template <uint32_t BM, uint32_t BN, uint32_t DEPTH>
__global__ __launch_bounds__(kThreads, BM == 256 ? 1 : 2) void mx4_product_kernel(MxProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t mx_lds[];
  // p.m_tiles is what there may be at most; numbered by it, the last die would have next to nothing to do
  const uint32_t m_tiles = min(p.m_tiles, mx_units<true>(p.g, BM)), total = m_tiles * p.n_tiles;
  uint32_t id = blockIdx.x;
  mx_tiles<BM, BN, DEPTH>(p, mx_lds, [&](MxWork& w) {
    for (; id < total; id += gridDim.x) {
      uint32_t mt, nt;
      mx_band(mx_by_die(id, total), m_tiles, p.n_tiles, &mt, &nt);
      const MxPlace at = mx_place<true>(p.g, mt, BM);
      const uint32_t a_low = at.first & ~3u;
      if (at.last <= at.first || (uint64_t)at.unit * BM >= (uint64_t)(at.last - a_low)) continue;
      const bool nobody = at.group >= p.g.groups && p.g.offsets != nullptr;  // rows behind the last group: zeros
      w.b_first = nobody ? 0u : at.group * p.n;
      w.b_last = w.b_first + p.n;
      w.b_row0 = (w.b_first & ~3u) + nt * BN;
      if (w.b_row0 >= w.b_last) continue;
      w.a_row0 = a_low + at.unit * BM;
      w.a_first = at.first;
      w.a_last = at.last;
      w.step0 = 0;
      w.steps = nobody ? 0u : p.a.steps;
      w.out = mx_out_at(p, (uint64_t)at.first * p.out_stride);
      w.stride = p.out_stride;
      id += gridDim.x;
      return true;
    }
    return false;
  });
}

// ---- the contraction by groups: out[g] = sum over the group's padded positions
template <uint32_t BM, uint32_t BN, uint32_t DEPTH>
__global__ __launch_bounds__(kThreads, BM == 256 ? 1 : 2) void mx4_gradient_kernel(MxProductArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t mx_lds[];
  const uint32_t per = p.m_tiles * p.n_tiles, total = per * p.g.groups;
  uint32_t id = blockIdx.x;
  mx_tiles<BM, BN, DEPTH>(p, mx_lds, [&](MxWork& w) {
    if (id >= total) return false;
    // group by group, every die with a part of each: groups differ in how much there is to do
    const uint32_t group = id / per;
    uint32_t mt, nt;
    mx_band(mx_by_die(id - group * per, per), p.m_tiles, p.n_tiles, &mt, &nt);
    id += gridDim.x;
    // steps of the groups before this one, and its own
    const uint32_t lane = threadIdx.x % kWave;
    uint32_t before = 0;
    for (uint32_t g0 = 0; g0 < group; g0 += kWave) {
      const uint32_t i = g0 + lane;
      uint32_t steps = 0;
      if (i < group) {
        const uint32_t first = mx_offset(p.g, i), last = mx_offset(p.g, i + 1u);
        steps = last > first ? (last - first + kMxStep - 1u) / kMxStep : 0u;
      }
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) steps += __shfl_xor(steps, d);
      before += steps;
    }
    const uint32_t first = mx_offset(p.g, group), last = mx_offset(p.g, group + 1u);
    w.step0 = __builtin_amdgcn_readfirstlane(min(before, p.a.steps));
    w.steps = __builtin_amdgcn_readfirstlane(last > first ? min((last - first + kMxStep - 1u) / kMxStep, p.a.steps - w.step0) : 0u);
    w.a_row0 = mt * BM;
    w.a_first = 0;
    w.a_last = p.m;
    w.b_row0 = nt * BN;
    w.b_first = 0;
    w.b_last = p.n;
    w.out = mx_out_at(p, (uint64_t)group * p.out_group);
    w.stride = p.out_stride;
    return true;
  });
}

// ------------------------------------------------------------------ few rows
// What bounds a product of few rows is the reading of b (one row by 11008 x 4096: 24 MB in 7.3 us, 3.3 TB/s; 64 rows in 32 groups by 2048 x 2048:
// 72 MB in 14, 5.1).  A workgroup takes 16 * NS rows of b and up to 16 * MS rows of a; its wavefronts
// share the contraction, U steps at a time in turn, and add their sums up in LDS, in the wavefronts' order.  Codes go from memory to the
// operand registers: lane (r, q) = (lane % 16, lane / 16) reads block q of the step of its row.  Row NS * r + j of b is row r of
// tile j, as above.  A turn's loads are under way while the turn before is multiplied, and nothing is loaded under a condition: what is not
// there is read from a place that is, and its codes are dropped.  (Plain loads: a tile's rows are every NS-th, and a load takes half of each cache line, the other
// half of which is the next load's; with the streaming hint 11008 x 4096 takes 8.6 us instead of 7.3.)
// SRC: a is compressed on the way (kMxBf16 ... kMxF32), by every workgroup for itself: a thread takes a block of 32 values, whose codes and
// scale byte go to LDS.  kMxReady: a is compressed.
template <uint32_t MS, uint32_t NS, uint32_t SRC>
struct MxFew {
  static constexpr bool kRaw = SRC != kMxReady;
  // two turns of U * (4 * NS + 4 * MS) registers (U * 4 * NS, with a in LDS) and what belongs to them, in the 128 of a lane, or 256 (MS > 1)
  static constexpr uint32_t U = (kRaw ? NS <= 2u : NS + MS <= (MS == 1u ? 2u : 5u)) ? 4u : 2u;
  uint4 b[U][NS];
  uint32_t sb[U];
  uint4 a[U][MS];
  uint32_t sa[U][MS];
};

template <uint32_t S>
__device__ __forceinline__ uint32_t mx_scales_at(const uint8_t* p) {
  if constexpr (S == 4) return *reinterpret_cast<const mx_u1u*>(p);
  else if constexpr (S == 2) return *reinterpret_cast<const mx_h1u*>(p);
  else return *p;
}
template <uint32_t J>
__device__ __forceinline__ mx_f4v mx_mfma16(uint4 a, uint4 b, mx_f4v c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(a), mx_operand(b), c, kMxFp4, kMxFp4, 0, (int)sa, J, (int)sb);
}

__device__ __forceinline__ uint32_t mx_pk_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(mx_u16x2, a), __builtin_bit_cast(mx_u16x2, b)));
}

// one block of 32 values, `left` of which exist (a multiple of 8, at least 8), to codes and scale byte
template <uint32_t TYPE>
__device__ __forceinline__ uint4 mx_compress_block(const uint8_t* p, uint32_t left, uint32_t fullrange, uint32_t* byte) {
  constexpr uint32_t N = TYPE == kMxF32 ? 8u : 4u, kEach = 32u / N;  // loads, and values of one
  uint4 v[N];
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) {
    const mx_u4u t = *reinterpret_cast<const mx_u4u*>(p + (i * kEach < left ? 16u * i : 0u));
    v[i] = make_uint4(t.x, t.y, t.z, t.w);
  }
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) {
    const uint32_t keep = i * kEach < left ? ~0u : 0u;
    v[i] = make_uint4(v[i].x & keep, v[i].y & keep, v[i].z & keep, v[i].w & keep);
  }
  uint32_t most = 0u;
  if constexpr (TYPE == kMxF32) {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) most = max(most, max(max(v[i].x & 0x7FFFFFFFu, v[i].y & 0x7FFFFFFFu), max(v[i].z & 0x7FFFFFFFu, v[i].w & 0x7FFFFFFFu)));
  } else {
    uint32_t m2 = 0u;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) m2 = mx_pk_max(m2, mx_pk_max(mx_pk_max(v[i].x & 0x7FFF7FFFu, v[i].y & 0x7FFF7FFFu), mx_pk_max(v[i].z & 0x7FFF7FFFu, v[i].w & 0x7FFF7FFFu)));
    const uint32_t mag = max(m2 & 0xFFFFu, m2 >> 16);
    most = TYPE == kMxBf16 ? mag << 16 : __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)mag));
  }
  *byte = mx_scale_byte(most, fullrange);
  const float s = mx_scale_value(*byte);
  uint32_t o[4];
#pragma unroll
  for (uint32_t k = 0; k < 4u; ++k) {
    uint32_t w = 0u;
    if constexpr (TYPE == kMxF32) {
      const uint4 x = v[(2 * k) % N], y = v[(2 * k + 1) % N];
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x.x), __uint_as_float(x.y), s, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x.z), __uint_as_float(x.w), s, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(y.x), __uint_as_float(y.y), s, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(y.z), __uint_as_float(y.w), s, 3);
    } else if constexpr (TYPE == kMxBf16) {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(mx_bf16x2, v[k % N].x), s, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(mx_bf16x2, v[k % N].y), s, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(mx_bf16x2, v[k % N].z), s, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(mx_bf16x2, v[k % N].w), s, 3);
    } else {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(mx_f16x2, v[k % N].x), s, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(mx_f16x2, v[k % N].y), s, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(mx_f16x2, v[k % N].z), s, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(mx_f16x2, v[k % N].w), s, 3);
    }
    o[k] = *byte == kMxNanByte ? 0u : w;
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

template <uint32_t MS, uint32_t NS, uint32_t SRC>
__global__ __launch_bounds__(mx4_few_waves(MS) * kWave) void mx4_few_kernel(MxProductArgs p) {
  using F = MxFew<MS, NS, SRC>;
  constexpr uint32_t U = F::U;
  extern __shared__ __attribute__((aligned(16))) uint8_t mx_lds[];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const uint32_t waves = blockDim.x / kWave;
  const uint32_t nt = blockIdx.x % p.n_tiles, mt = blockIdx.x / p.n_tiles;
  const MxPlace at = mx_place<false>(p.g, mt, 16u * MS);
  if ((uint64_t)at.unit * (16u * MS) >= (uint64_t)(at.last - at.first)) return;
  const uint32_t row0 = at.first + at.unit * (16u * MS);
  const uint32_t rows = min(at.last - row0, 16u * MS);
  const bool nobody = at.group >= p.g.groups && p.g.offsets != nullptr;
  const uint32_t b_first = nobody ? 0u : at.group * p.n;
  const uint32_t col0 = nt * (16u * NS);  // of the output
  const uint32_t cols = min(p.n - col0, 16u * NS);
  const uint32_t r = lane % 16u, q = lane / 16u;
  const uint32_t steps = nobody ? 0u : p.b.steps;

  mx_f4v acc[MS][NS];
#pragma unroll
  for (uint32_t i = 0; i < MS; ++i)
#pragma unroll
    for (uint32_t j = 0; j < NS; ++j) acc[i][j] = mx_f4v{0.0f, 0.0f, 0.0f, 0.0f};

  // rows behind the last read the last one (of b: results that are not kept; of a: rows that are not kept)
  const uint8_t* b_row[NS];
#pragma unroll
  for (uint32_t j = 0; j < NS; ++j) b_row[j] = p.b.codes + (uint64_t)(b_first + col0 + min(NS * r + j, cols - 1u)) * kMxStepBytes + 16u * q;
  // NS scale bytes at once, within the block column: those of the stack's last rows, where a matrix begins between two words, are the high ones
  const uint64_t b_scale_want = (uint64_t)b_first + col0 + NS * r, b_scale_row = min(b_scale_want, p.b.pitch - NS);
  const uint32_t b_scale_shift = (uint32_t)(b_scale_want - b_scale_row) * 8u % 32u;  // (beyond NS bytes: results that are not kept)
  const uint8_t* b_scale = p.b.scales + (uint64_t)q * p.b.pitch + b_scale_row;
  const uint8_t* a_row[MS];
  const uint8_t* a_scale[MS];
  uint32_t a_step, a_scale_step;  // with a in LDS: [step][row][64], then [step][block][row]
  uint8_t* const lds_scales = mx_lds + steps * rows * kMxStepBytes;
#pragma unroll
  for (uint32_t i = 0; i < MS; ++i) {
    const uint32_t row = min(16u * i + r, rows - 1u);
    a_row[i] = F::kRaw ? mx_lds + row * kMxStepBytes + 16u * q : p.a.codes + (uint64_t)(row0 + row) * kMxStepBytes + 16u * q;
    a_scale[i] = F::kRaw ? lds_scales + q * rows + row : p.a.scales + (uint64_t)q * p.a.pitch + row0 + row;
  }
  a_step = rows * kMxStepBytes;
  a_scale_step = 4u * rows;
  // the U steps from s0 on (behind the last: the last one again, which multiply leaves out)
  const auto load = [&](F& t, uint32_t s0) {
    if constexpr (!F::kRaw) {
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
        const uint32_t s = min(s0 + u, steps - 1u);
#pragma unroll
        for (uint32_t i = 0; i < MS; ++i) {
          t.a[u][i] = *reinterpret_cast<const uint4*>(a_row[i] + (uint64_t)s * p.a.step_bytes);
          t.sa[u][i] = a_scale[i][(uint64_t)(4u * s) * p.a.pitch];
        }
      }
    }
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) {
      const uint32_t s = min(s0 + u, steps - 1u);
      t.sb[u] = mx_scales_at<NS>(b_scale + (uint64_t)(4u * s) * p.b.pitch);
#pragma unroll
      for (uint32_t j = 0; j < NS; ++j) {
        t.b[u][j] = *reinterpret_cast<const uint4*>(b_row[j] + (uint64_t)s * p.b.step_bytes);
      }
    }
  };
  const auto multiply = [&](F& t, uint32_t s0) {
    if constexpr (F::kRaw) {
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
        const uint32_t s = min(s0 + u, steps - 1u);
#pragma unroll
        for (uint32_t i = 0; i < MS; ++i) {
          t.a[u][i] = *reinterpret_cast<const uint4*>(a_row[i] + s * a_step);
          t.sa[u][i] = a_scale[i][s * a_scale_step];
        }
      }
    }
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) {
      if (s0 + u < steps) {  // (uniform)
        const uint32_t sb = NS > 1u ? t.sb[u] >> b_scale_shift : t.sb[u];
#pragma unroll
        for (uint32_t i = 0; i < MS; ++i) {
#define ADACC_MX_AT(J) if constexpr (J < NS) acc[i][J % NS] = mx_mfma16<J>(t.a[u][i], t.b[u][J % NS], acc[i][J % NS], t.sa[u][i], sb);
          ADACC_MX_AT(0) ADACC_MX_AT(1) ADACC_MX_AT(2) ADACC_MX_AT(3)
#undef ADACC_MX_AT
        }
      }
    }
  };
  const uint32_t apart = U * waves;
  uint32_t s0 = U * wave;
  F one, two;
  if constexpr (F::kRaw) {
    const uint32_t blocks = 4u * steps;  // of a row; those behind its end are zeros
    for (uint32_t t = threadIdx.x; t < rows * blocks; t += blockDim.x) {
      const uint32_t row = t / blocks, block = t - row * blocks;
      const uint32_t first = block * kMxBlock;
      uint4 codes = make_uint4(0u, 0u, 0u, 0u);
      uint32_t byte = 0u;
      if (first < p.k)
        codes = mx_compress_block<SRC>(static_cast<const uint8_t*>(p.x) + ((uint64_t)(row0 + row) * p.x_stride + first) * (SRC == kMxF32 ? 4u : 2u),
                                       min(p.k - first, kMxBlock), p.fullrange, &byte);
      const uint32_t step = block / 4u, in = block % 4u;
      *reinterpret_cast<uint4*>(mx_lds + (step * rows + row) * kMxStepBytes + in * 16u) = codes;
      lds_scales[block * rows + row] = (uint8_t)byte;
    }
    if (s0 < steps) load(one, s0);
    __syncthreads();
  } else {
    if (s0 < steps) load(one, s0);
  }
  if (s0 < steps) {  // (uniform in the wavefront)
    for (;;) {
      if (s0 + apart < steps) load(two, s0 + apart);
      multiply(one, s0);
      s0 += apart;
      if (s0 >= steps) break;
      if (s0 + apart < steps) load(one, s0 + apart);
      multiply(two, s0);
      s0 += apart;
      if (s0 >= steps) break;
    }
  }
  if constexpr (F::kRaw) __syncthreads();  // a has been read
  // lane (r, q) holds rows 4 * q + e and column r of a tile; [wave][row][column] in LDS
  float* sums = reinterpret_cast<float*>(mx_lds);
  constexpr uint32_t kCols = 16u * NS, kRows = 16u * MS;
#pragma unroll
  for (uint32_t i = 0; i < MS; ++i)
#pragma unroll
    for (uint32_t e = 0; e < 4u; ++e)
#pragma unroll
      for (uint32_t j = 0; j < NS; ++j) sums[(wave * kRows + 16u * i + 4u * q + e) * kCols + NS * r + j] = acc[i][j][e];
  __syncthreads();
  for (uint32_t t = threadIdx.x; t < rows * kCols; t += blockDim.x) {
    const uint32_t row = t / kCols, col = t % kCols;
    if (col >= cols) continue;
    float v = 0.0f;
    for (uint32_t u = 0; u < waves; ++u) v += sums[(u * kRows + row) * kCols + col];
    mx_store1(p.out, p.out_type, (uint64_t)(row0 + row) * p.out_stride + col0 + col, v);
  }
}

template <uint32_t MS, uint32_t NS>
static MxProductFn few_of(uint32_t src) {
  if constexpr (MS == 1) {  // (sixteen rows and fewer are compressed on the way)
    if (src == kMxBf16) return mx4_few_kernel<MS, NS, kMxBf16>;
    if (src == kMxF16) return mx4_few_kernel<MS, NS, kMxF16>;
    if (src == kMxF32) return mx4_few_kernel<MS, NS, kMxF32>;
  }
  return mx4_few_kernel<MS, NS, kMxReady>;
}
template <uint32_t MS>
static MxProductFn few_by_columns(uint32_t ns, uint32_t src) {
  return ns == 1 ? few_of<MS, 1>(src) : ns == 2 ? few_of<MS, 2>(src) : few_of<MS, 4>(src);
}
MxProductFn mx4_few_fn(uint32_t ms, uint32_t ns, uint32_t src) {
  return ms == 1 ? few_by_columns<1>(ns, src) : ms == 2 ? few_by_columns<2>(ns, src) : few_by_columns<4>(ns, src);
}

// Steps in LDS: four fill it with tiles of 256, and hold two workgroups of 128 a compute unit.  Tiles of 64 are taken where there are few, and wait for
// memory: eight (64 x 4096 x 11008 16.6 us, with four 21.0).  Neither more workgroups nor more wavefronts shorten that: the contraction cut in
// eight, with a launch that joins the parts, takes 16 us, by four teams in a workgroup 17.6.
template <uint32_t TILE>
constexpr uint32_t kMxDepth = TILE == 64u ? 8u : 4u;
template <uint32_t TILE>
static MxProductFn product_of(bool gradient) {
  return gradient ? mx4_gradient_kernel<TILE, TILE, kMxDepth<TILE>> : mx4_product_kernel<TILE, TILE, kMxDepth<TILE>>;
}
MxProductFn mx4_product_fn(uint32_t tile, bool gradient) {
  return tile == 256 ? product_of<256>(gradient) : tile == 128 ? product_of<128>(gradient) : product_of<64>(gradient);
}
uint32_t mx4_product_lds(uint32_t tile) {
  return tile == 256 ? MxTile<256, 256, kMxDepth<256>>::kLds : tile == 128 ? MxTile<128, 128, kMxDepth<128>>::kLds : MxTile<64, 64, kMxDepth<64>>::kLds;
}

}  // namespace adacc
