// libadacc, host code of the layers whose saved activations are compressed (include/adacc.h).  Kernels: adacc_k_norm.hip, adacc_k_act.hip, adacc_k_linear.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "adacc.h"
#include "adacc_fn.hpp"
#include "adacc_layers.hpp"

namespace adacc {

constexpr uint64_t kLayMost = 1ull << 30;         // rows and columns of a matrix: kernels count them in 32 bits
constexpr uint64_t kLayThreads = 0xFFFFFFFFull;   // of a launch: the runtime takes fewer than 2^32
constexpr uint64_t kLayGroupsMost = 1ull << 30;   // groups of 128 in all rows of a call of the kernels that have sixteen lanes for each
constexpr uint64_t kLinStrideMost = 1ull << 23;   // elements between the rows of a product's operands: a tile's offsets have 32 bits
constexpr uint64_t kCus = 256;

static uint64_t lay_align256(uint64_t v) { return (v + 255ull) & ~255ull; }
static uint64_t over(uint64_t v, uint64_t by) { return (v + by - 1) / by; }
static bool lay_misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
static uint64_t lay_size(uint32_t type) { return type == kTypeF32 ? 4u : 2u; }
static bool lay_sizes_ok(uint64_t rows, uint64_t cols) { return rows <= kLayMost && cols <= kLayMost; }
static bool lay_groups_ok(uint64_t rows, uint64_t cols) { return lay_sizes_ok(rows, cols) && rows * over(cols, kR8Group) <= kLayGroupsMost; }

static void rows8_layout(uint64_t rows, uint64_t cols, adacc_rows8_layout* L) {
  L->pitch = over(cols, 16) * 16;
  L->groups = over(cols, kR8Group);
  L->codes_off = 0;
  L->scales_off = lay_align256(rows * L->pitch);
  L->total_bytes = L->scales_off + lay_align256(rows * L->groups * 4);
}
static Rows8 rows8_of(const void* blob, uint64_t rows, uint64_t cols) {
  Rows8 b;
  std::memset(&b, 0, sizeof b);
  if (!blob) return b;
  adacc_rows8_layout L;
  rows8_layout(rows, cols, &L);
  b.codes = static_cast<uint8_t*>(const_cast<void*>(blob)) + L.codes_off;
  b.scales = reinterpret_cast<float*>(static_cast<uint8_t*>(const_cast<void*>(blob)) + L.scales_off);
  b.pitch = L.pitch;
  b.groups = (uint32_t)L.groups;
  return b;
}
static int check_blob(const void* blob, uint64_t bytes, uint64_t rows, uint64_t cols) {
  adacc_rows8_layout L;
  rows8_layout(rows, cols, &L);
  if (!blob) return ADACC_ENULL;
  if (bytes < L.total_bytes) return ADACC_ESIZE;
  return lay_misaligned(blob, 256) ? ADACC_EALIGN : ADACC_OK;
}
static int check_matrix(const void* p, uint32_t type, uint64_t rows, uint64_t cols, uint64_t stride) {
  if (!p) return ADACC_ENULL;
  if (stride < cols && rows > 1) return ADACC_EINVAL;
  return lay_misaligned(p, lay_size(type)) ? ADACC_EALIGN : ADACC_OK;
}
static int check_vector(const void* p, uint32_t type) { return lay_misaligned(p, lay_size(type)) ? ADACC_EALIGN : ADACC_OK; }
static int check_workspace(const void* p, uint64_t bytes, uint64_t need) {
  if (need == 0) return ADACC_OK;
  if (!p) return ADACC_ENULL;
  if (bytes < need) return ADACC_ESIZE;
  return lay_misaligned(p, 256) ? ADACC_EALIGN : ADACC_OK;
}
#define ADACC_TRY(call)               \
  do {                                \
    const int rc_ = (call);           \
    if (rc_ != ADACC_OK) return rc_;  \
  } while (0)

static Strided strided(const void* p, uint64_t stride) { return Strided{const_cast<void*>(p), stride}; }
static void skip(Strided* m, uint64_t rows, uint32_t type) {
  if (m->at) m->at = static_cast<uint8_t*>(m->at) + rows * m->stride * lay_size(type);
}
static void skip(Rows8* b, uint64_t rows) {
  if (!b->codes) return;
  b->codes += rows * b->pitch;
  b->scales += rows * b->groups;
}

template <typename Args>
static int launch(void (*fn)(Args), uint64_t grid, uint32_t threads, uint32_t lds, hipStream_t s, const Args& a, const char* what) {
  if (grid * threads > kLayThreads) return ADACC_ELIMIT;
  if (grid == 0) return ADACC_OK;
  if (lds > 65536u) {  // more than a launch may ask for unless the kernel has been told (nothing is enqueued by it)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return hip_result(e, what);
  }
  hipLaunchKernelGGL(fn, dim3((uint32_t)grid), dim3(threads), lds, s, a);
  return launch_check(what);
}

// groups of 128 columns, 16 lanes each, kR8Units one after the other a lane
static uint64_t group_grid(uint64_t rows, uint64_t cols) { return over(rows * over(cols, kR8Group), (kThreads / kR8Lanes) * kR8Units); }
// ... as many rows at a time as a launch takes; behind(a, n): a's matrices begin n rows further on
template <typename Args, typename Behind>
static int launch_groups(void (*fn)(Args), uint64_t rows, Args a, hipStream_t s, const char* what, Behind&& behind) {
  const uint32_t groups = (uint32_t)over(a.cols, kR8Group), step = kThreads / kR8Lanes;
  a.step_rows = step / groups;
  a.step_groups = step % groups;
  const uint64_t most = kLayThreads / kThreads * (step * kR8Units) / groups;
  for (uint64_t at = 0; at < rows; at += most) {
    const uint64_t now = std::min(rows - at, most);
    a.rows = (uint32_t)now;
    ADACC_TRY(launch(fn, group_grid(now, a.cols), (uint32_t)kThreads, 0, s, a, what));
    behind(&a, now);
  }
  return ADACC_OK;
}

static auto act_behind(uint32_t type) {
  return [type](ActArgs* p, uint64_t n) {
    for (Strided* m : {&p->a, &p->up, &p->y, &p->da, &p->dup}) skip(m, n, type);
    skip(&p->a8, n);
    skip(&p->up8, n);
  };
}

// ------------------------------------------------------------------ layer norm
static NormShape norm_shape(uint64_t cols) {
  if (cols <= 128) return {16, 1};
  if (cols <= 256) return {32, 1};
  if (cols <= 512) return {64, 1};
  if (cols <= 1024) return {64, 2};
  if (cols > kNormWidest) return {1024, 0};
  const uint32_t octets = cols <= kNormThreads * 8 ? 1 : cols <= kNormThreads * 16 ? 2 : 4;
  return {(uint32_t)over(cols, 512 * octets) * kWave, octets};
}
static uint32_t norm_threads(NormShape s) { return s.lanes <= 64 ? (uint32_t)kThreads : s.lanes; }
static uint64_t norm_bunch(NormShape s) { return s.lanes <= 64 ? kThreads / s.lanes : 1; }
// Workgroups, which take rows in turn: as many as the compute units hold, by registers
static uint64_t norm_workgroups(NormShape s, bool backward) {
  const uint64_t waves = backward ? (s.lanes > 64 && s.octets == 1 ? 16 : 8) : s.octets == 1 ? 32 : s.octets == 2 ? 16 : 8;
  return kCus * std::max<uint64_t>(1, waves / (norm_threads(s) / kWave));
}
// Those of the backward pass leave [2][cols] sums each: as many as above, but of fewer than eight rows (or bunches) no more than there are compute units
static uint32_t norm_partials(uint64_t rows, uint64_t cols) {
  const NormShape s = norm_shape(cols);
  if (s.octets == 0) return (uint32_t)std::min({rows, (uint64_t)64, kLayThreads / kThreads / over(cols, 2048)});  // (a workgroup for 2048 columns of each, in one launch)
  const uint64_t bunches = over(rows, norm_bunch(s));
  return (uint32_t)std::min<uint64_t>(bunches, std::max<uint64_t>(kCus, std::min<uint64_t>(norm_workgroups(s, true), bunches / 8)));
}

static int reduce(uint32_t cols, uint32_t partials, uint32_t parts, const float* partial, uint32_t type, void* a, void* b, hipStream_t s) {
  ReduceArgs r;
  r.cols = cols;
  r.partials = partials;
  r.parts = parts;
  r.type = type;
  r.partial = partial;
  r.out[0] = a;
  r.out[1] = b;
  return launch(reduce_fn(), std::min<uint64_t>(over(cols, kReduceCols) * parts, kLayThreads / 1024), 1024, 0, s, r, "reduce_kernel");
}

// ------------------------------------------------------------------ sums of columns
// A strip is as wide as leaves least of it idle: `wide` groups of 128, by 16 / wide rows
static uint32_t strip_wide(uint64_t cols) {
  const uint64_t groups = over(cols, kR8Group);
  return groups >= 16 ? 16u : groups >= 8 ? 8u : groups >= 4 ? 4u : groups >= 2 ? 2u : 1u;
}
static uint32_t strip_partials(uint64_t rows, uint64_t cols) {
  const uint32_t wide = strip_wide(cols);
  const uint64_t strips = over(over(cols, kR8Group), wide), bunch = 16 / wide;
  return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(over(rows, bunch * 4), over(kCus * 4, strips)));
}

// ------------------------------------------------------------------ products
struct LinPlan {
  bool few;
  uint32_t ms, ns, waves;
  uint32_t tile, splits, split_steps;
};
constexpr uint32_t kFewWaves = 8;  // of a workgroup, at most (sixteen: one row by 11008 x 4096 21 us instead of 18, 16 by 4096 x 11008 as many, 26)

// Tiles of 256 or 128, and into how many parts the contraction is cut, by what each way takes: us, fitted to 14 shapes from 64 x 4096 x 4096 to 8192 x 2112 x 8192, which it puts in the
// right order but for differences of a few percent.
//   256   a compute unit has one at a time: 1.6 a step of 64, and 6 for its results
//   128   two share a compute unit at 0.53 a step each, one alone takes 0.64; 4 for the results.  Cut contractions are written in binary32 and read again, at 4 TB/s, by a launch of 4
// Measured (256 / 128 / 128 cut): 4096^3 115 / 146 / -; 3000^3 72 / 91 / 101; 8192 x 2112 x 8192 352 / 315 / -; 2048^3 - / 24 / 35; 13540 x 128 x 1024 - / 13 / 17; 777 x 1003 x 2040
// - / 23 / 19 (in three); 64 x 4096 x 4096 - / 44 / 16 (in eight).
static double lin_time_256(uint64_t m, uint64_t n, uint64_t steps) { return (double)over(over(m, 256) * over(n, 256), kCus) * (1.6 * (double)steps + 6.0); }
static double lin_time_128(uint64_t m, uint64_t n, uint64_t steps, uint64_t splits) {
  const uint64_t each = over(over(m, 128) * over(n, 128) * splits, kCus), part = over(steps, splits);
  const double t = each == 1 ? 0.64 * (double)part + 4.0 : 0.53 * (double)(each * part) + 4.0 * (double)over(each, 2);
  return splits == 1 ? t : t + 4.0 + (double)(splits * m * n) * 8.0 / 4e6;
}
static LinPlan lin_plan(uint64_t m, uint64_t n, uint64_t k, bool may_be_few) {
  LinPlan p;
  std::memset(&p, 0, sizeof p);
  // up to 32 rows: 64 x 4096 x 4096 22 us, in tiles 16; 32 by 4096 x 4096 14, 33 in tiles 15; 32 by 11008 x 4096 26, 33 in tiles 24.  (By 4096 x 11008, 32 rows take 32, 64 in tiles 26.)
  p.few = may_be_few && k >= kLinShort && m <= 32;
  p.splits = 1;
  if (p.few) {
    p.ms = m <= 16 ? 1u : 2u;
    // columns of a workgroup: 64 read x less often, which 17 rows and more gain by where workgroups enough are left (32 by 11008 x 4096: 29 us, of 16 columns 35; by 4096 x 4096 25 and 12)
    p.ns = p.ms == 2 && over(n, 64) >= 160 ? 4u : 1u;
    p.waves = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(kFewWaves, over(k, 4 * 32)));
    if (over(n, 16 * p.ns) * p.waves * kWave <= kLayThreads) return p;  // (a launch's; tiles are taken in turn)
    p.few = false;
  }
  const uint64_t steps = over(k, kLinStep);
  p.tile = 128u;
  uint64_t splits = 1;
  double least = lin_time_128(m, n, steps, 1);
  for (uint64_t s = 2; s <= 16 && s * 4 <= steps; ++s) {
    const double t = lin_time_128(m, n, steps, s);
    if (t < least) {
      least = t;
      splits = s;
    }
  }
  if (lin_time_256(m, n, steps) < least) {
    p.tile = 256u;
    splits = 1;
  }
  p.split_steps = (uint32_t)std::max<uint64_t>(1, over(steps, splits));
  p.splits = (uint32_t)std::max<uint64_t>(1, over(steps, p.split_steps));
  return p;
}

// the operands of a product as they are, and what the workspace has to hold for them
struct LinOperand {
  const void* at;
  uint64_t rows, cols, stride;
};
static uint64_t pad_bytes(uint64_t rows, uint64_t cols) { return cols < kLinShort && cols ? lay_align256(rows * 16) : 0; }
static uint64_t partial_bytes(const LinPlan& p, uint64_t m, uint64_t n) { return p.splits > 1 ? lay_align256((uint64_t)p.splits * m * n * 4) : 0; }

static int pad(LinOperand* o, uint8_t** ws, hipStream_t s) {
  if (o->cols >= kLinShort) return ADACC_OK;
  uint4* dst = reinterpret_cast<uint4*>(*ws);
  *ws += pad_bytes(o->rows, o->cols);
  hipLaunchKernelGGL(pad_fn(), dim3((uint32_t)over(o->rows, kThreads)), dim3(kThreads), 0, s, static_cast<const uint16_t*>(o->at), o->stride, (uint32_t)o->rows,
                     (uint32_t)o->cols, dst);
  const int rc = launch_check("lin_pad_kernel");
  o->at = dst;
  o->cols = o->stride = kLinShort;
  return rc;
}

// out = A B^T; the operands have been checked.  a_mode, b_mode: kAlong ...; b8: instead of b
static int product(const LinPlan& plan, uint32_t type, LinOperand a, uint32_t a_mode, LinOperand b, uint32_t b_mode, const Rows8& b8, uint64_t k, const Epilogue& e, uint8_t* ws,
                   hipStream_t s) {
  ProductArgs p;
  std::memset(&p, 0, sizeof p);
  p.e = e;
  p.k = (uint32_t)k;
  const uint64_t total = plan.few ? 0 : over(e.m, plan.tile) * over(e.n, plan.tile) * plan.splits;
  if (total > 0x7FFFFFFFull) return ADACC_ELIMIT;
  if (plan.few) {
    p.a = strided(a.at, a.stride);
    p.b = strided(b.at, b.stride);
    p.n_tiles = (uint32_t)over(e.n, 16 * plan.ns);
    return launch(linear_few_fn(type, plan.ms, plan.ns), over(e.m, 16 * plan.ms) * p.n_tiles, plan.waves * kWave, plan.waves * 16u * plan.ms * 16u * plan.ns * 4u, s, p, "lin_few_kernel");
  }
  if (k) {
    ADACC_TRY(pad(&a, &ws, s));
    if (b_mode != kAcross8) ADACC_TRY(pad(&b, &ws, s));
  }
  p.a = strided(a.at, a.stride);
  p.b = strided(b.at, b.stride);
  p.b8 = b8;
  p.m_tiles = (uint32_t)over(e.m, plan.tile);
  p.n_tiles = (uint32_t)over(e.n, plan.tile);
  p.splits = plan.splits;
  p.split_steps = plan.split_steps;
  p.partial = reinterpret_cast<float*>(ws);
  const uint64_t room = plan.tile == 256 ? kCus : 2 * kCus;  // as many workgroups as the compute units hold at a time, by LDS
  ADACC_TRY(launch(product_fn(type, a_mode, b_mode, plan.tile), std::min(total, room), (uint32_t)kThreads, product_lds(plan.tile), s, p, "lin_product_kernel"));
  if (plan.splits == 1) return ADACC_OK;
  JoinArgs j;
  j.e = e;
  j.partial = p.partial;
  j.splits = p.splits;
  return launch(join_fn(type), over((uint64_t)e.m * over(e.n, kR8Group), kThreads / kR8Lanes), (uint32_t)kThreads, 0, s, j, "lin_join_kernel");
}

static int check_operand(const void* p, uint64_t rows, uint64_t cols, uint64_t stride) {
  ADACC_TRY(check_matrix(p, kTypeBf16, rows, cols, stride));
  return rows > 1 && stride >= kLinStrideMost ? ADACC_ELIMIT : ADACC_OK;
}

}  // namespace adacc

using namespace adacc;

extern "C" {

// ------------------------------------------------------------------ 8-bit rows
int adacc_rows8_layout_of(uint64_t rows, uint64_t cols, adacc_rows8_layout* out) {
  if (!out) return ADACC_ENULL;
  if (!lay_sizes_ok(rows, cols)) return ADACC_ELIMIT;
  rows8_layout(rows, cols, out);
  return ADACC_OK;
}

static int rows8_call(bool restore, uint32_t type, const void* m, uint64_t rows, uint64_t cols, uint64_t stride, const void* blob, uint64_t blob_bytes, void* hip_stream) {
  if (type > kTypeF32) return ADACC_EINVAL;
  if (!lay_groups_ok(rows, cols)) return ADACC_ELIMIT;
  if (!rows || !cols) return ADACC_OK;
  ADACC_TRY(check_matrix(m, type, rows, cols, stride));
  ADACC_TRY(check_blob(blob, blob_bytes, rows, cols));
  Rows8Args a;
  a.cols = (uint32_t)cols;
  a.m = strided(m, stride);
  a.blob = rows8_of(blob, rows, cols);
  return launch_groups(restore ? rows8_restore_fn(type) : rows8_compress_fn(type), rows, a, static_cast<hipStream_t>(hip_stream), "rows8_kernel", [type](Rows8Args* p, uint64_t n) {
    skip(&p->m, n, type);
    skip(&p->blob, n);
  });
}
int adacc_rows8_compress(uint32_t type, const void* src, uint64_t rows, uint64_t cols, uint64_t row_stride, void* blob, uint64_t blob_bytes, void* hip_stream) {
  return rows8_call(false, type, src, rows, cols, row_stride, blob, blob_bytes, hip_stream);
}
int adacc_rows8_decompress(const void* blob, uint64_t blob_bytes, uint64_t rows, uint64_t cols, void* dst, uint32_t type, uint64_t row_stride, void* hip_stream) {
  return rows8_call(true, type, dst, rows, cols, row_stride, blob, blob_bytes, hip_stream);
}

// ------------------------------------------------------------------ layer norm
int adacc_norm_forward(uint32_t type, const void* x, uint64_t rows, uint64_t cols, uint64_t x_stride, uint32_t weight_type, const void* weight, const void* bias, float eps, void* y,
                       uint64_t y_stride, void* blob, uint64_t blob_bytes, void* stats, void* hip_stream) {
  if (type > kTypeF32 || (weight_type != type && weight_type != kTypeF32) || !(eps >= 0.0f)) return ADACC_EINVAL;
  if (!lay_sizes_ok(rows, cols)) return ADACC_ELIMIT;
  if (!rows || !cols) return ADACC_OK;
  ADACC_TRY(check_matrix(x, type, rows, cols, x_stride));
  ADACC_TRY(check_matrix(y, type, rows, cols, y_stride));
  ADACC_TRY(check_vector(weight, weight_type));
  ADACC_TRY(check_vector(bias, weight_type));
  if (blob) ADACC_TRY(check_blob(blob, blob_bytes, rows, cols));
  if (lay_misaligned(stats, 8)) return ADACC_EALIGN;
  NormArgs a;
  std::memset(&a, 0, sizeof a);
  a.cols = (uint32_t)cols;
  a.wtype = weight_type;
  a.eps = eps;
  a.x = strided(x, x_stride);
  a.y = strided(y, y_stride);
  a.blob = rows8_of(blob, rows, cols);
  a.weight = weight;
  a.bias = bias;
  a.stats = static_cast<float2*>(stats);
  const NormShape shape = norm_shape(cols);
  const NormFn fn = norm_forward_fn(type, shape, blob != nullptr, cols % 8 == 0);
  const uint32_t threads = norm_threads(shape);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  a.rows = (uint32_t)rows;
  if (shape.octets) return launch(fn, std::min<uint64_t>(over(rows, norm_bunch(shape)), norm_workgroups(shape, false)), threads, 0, s, a, "norm_forward_kernel");
  const uint64_t most = kLayThreads / threads;  // rows of a launch, a workgroup each
  for (uint64_t at = 0; at < rows; at += most) {
    const uint64_t now = std::min(rows - at, most);
    a.rows = (uint32_t)now;
    ADACC_TRY(launch(fn, now, threads, 0, s, a, "norm_forward_pieces_kernel"));
    skip(&a.x, now, type);
    skip(&a.y, now, type);
    skip(&a.blob, now);
    if (a.stats) a.stats += now;
  }
  return ADACC_OK;
}

uint64_t adacc_norm_workspace_bytes(uint64_t rows, uint64_t cols) {
  if (!rows || !cols || !lay_sizes_ok(rows, cols)) return 0;
  return lay_align256((uint64_t)norm_partials(rows, cols) * 2 * cols * 4);
}

int adacc_norm_backward(uint32_t type, const void* x, uint64_t x_stride, const void* blob, uint64_t blob_bytes, uint64_t rows, uint64_t cols, uint32_t weight_type, const void* weight,
                        const void* stats, const void* dy, uint64_t dy_stride, void* dx, uint64_t dx_stride, void* dweight, void* dbias, void* workspace, uint64_t workspace_bytes,
                        void* hip_stream) {
  if (type > kTypeF32 || (weight_type != type && weight_type != kTypeF32) || (x && blob)) return ADACC_EINVAL;
  if (!lay_sizes_ok(rows, cols)) return ADACC_ELIMIT;
  if (!cols) return ADACC_OK;
  const bool params = dweight || dbias;
  ADACC_TRY(check_vector(dweight, weight_type));
  ADACC_TRY(check_vector(dbias, weight_type));
  ADACC_TRY(check_vector(weight, weight_type));
  if (rows) {
    if (blob) ADACC_TRY(check_blob(blob, blob_bytes, rows, cols));
    else ADACC_TRY(check_matrix(x, type, rows, cols, x_stride));
    if (!stats) return ADACC_ENULL;
    if (lay_misaligned(stats, 8)) return ADACC_EALIGN;
    ADACC_TRY(check_matrix(dy, type, rows, cols, dy_stride));
    if (dx) ADACC_TRY(check_matrix(dx, type, rows, cols, dx_stride));
    if (params) ADACC_TRY(check_workspace(workspace, workspace_bytes, adacc_norm_workspace_bytes(rows, cols)));
  }
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (!params && !dx) return ADACC_OK;
  NormArgs a;
  std::memset(&a, 0, sizeof a);
  a.rows = (uint32_t)rows;
  a.cols = (uint32_t)cols;
  a.wtype = weight_type;
  a.x = strided(x, x_stride);
  a.dy = strided(dy, dy_stride);
  a.dx = strided(dx, dx_stride);
  a.blob = rows8_of(blob, rows, cols);
  a.weight = weight;
  a.stats = static_cast<float2*>(const_cast<void*>(stats));
  a.partial = params ? static_cast<float*>(workspace) : nullptr;
  if (rows) {
    const NormShape shape = norm_shape(cols);
    a.partials = norm_partials(rows, cols);
    const uint32_t threads = norm_threads(shape);
    if (shape.octets) {
      // the sums of a workgroup's rows, two a column; or the weight
      const uint32_t lds = shape.lanes <= 64 ? (uint32_t)kThreads * shape.octets * 8u * 2u * 4u : shape.octets == 4 ? threads * 4u * 8u * 4u : 0u;
      ADACC_TRY(launch(norm_backward_fn(type, shape, blob != nullptr, cols % 8 == 0), a.partials, threads, lds, s, a, "norm_backward_kernel"));
    } else {
      if (params) ADACC_TRY(launch(norm_columns_fn(type, blob != nullptr), a.partials * over(cols, 2048), (uint32_t)kThreads, 0, s, a, "norm_columns_kernel"));
      NormArgs b = a;
      const uint64_t most = kLayThreads / threads;
      for (uint64_t at = 0; dx && at < rows; at += most) {
        const uint64_t now = std::min(rows - at, most);
        b.rows = (uint32_t)now;
        ADACC_TRY(launch(norm_backward_fn(type, shape, blob != nullptr, cols % 8 == 0), now, threads, 0, s, b, "norm_backward_pieces_kernel"));
        skip(&b.x, now, type);
        skip(&b.dy, now, type);
        skip(&b.dx, now, type);
        skip(&b.blob, now);
        b.stats += now;
      }
    }
  }
  if (!params) return ADACC_OK;
  return reduce(a.cols, a.partials, 2, a.partial, weight_type, dweight, dbias, s);
}

// ------------------------------------------------------------------ activations
int adacc_act_forward(uint32_t type, uint32_t kind, const void* a, uint64_t a_stride, const void* up, uint64_t up_stride, uint64_t rows, uint64_t cols, void* y, uint64_t y_stride, void* a_blob,
                      uint64_t a_blob_bytes, void* up_blob, uint64_t up_blob_bytes, void* hip_stream) {
  if (type > kTypeF32 || kind < kActGelu || kind > kActSilu) return ADACC_EINVAL;
  if ((up_blob != nullptr) != (up && a_blob)) return ADACC_EINVAL;
  if (!lay_groups_ok(rows, cols)) return ADACC_ELIMIT;
  if (!rows || !cols) return ADACC_OK;
  ADACC_TRY(check_matrix(a, type, rows, cols, a_stride));
  if (up) ADACC_TRY(check_matrix(up, type, rows, cols, up_stride));
  ADACC_TRY(check_matrix(y, type, rows, cols, y_stride));
  if (a_blob) ADACC_TRY(check_blob(a_blob, a_blob_bytes, rows, cols));
  if (up_blob) ADACC_TRY(check_blob(up_blob, up_blob_bytes, rows, cols));
  ActArgs p;
  std::memset(&p, 0, sizeof p);
  p.cols = (uint32_t)cols;
  p.a = strided(a, a_stride);
  p.up = strided(up, up_stride);
  p.y = strided(y, y_stride);
  p.a8 = rows8_of(a_blob, rows, cols);
  p.up8 = rows8_of(up_blob, rows, cols);
  return launch_groups(act_forward_fn(type, kind, up != nullptr, a_blob != nullptr, cols % 8 == 0), rows, p, static_cast<hipStream_t>(hip_stream), "act_forward_kernel", act_behind(type));
}

int adacc_act_backward(uint32_t type, uint32_t kind, const void* a, uint64_t a_stride, const void* a_blob, uint64_t a_blob_bytes, const void* up, uint64_t up_stride, const void* up_blob,
                       uint64_t up_blob_bytes, const void* dy, uint64_t dy_stride, uint64_t rows, uint64_t cols, void* da, uint64_t da_stride, void* dup, uint64_t dup_stride, void* hip_stream) {
  if (type > kTypeF32 || kind < kActGelu || kind > kActSilu) return ADACC_EINVAL;
  if ((a && a_blob) || (up && up_blob) || (up && a_blob) || (up_blob && a)) return ADACC_EINVAL;
  const bool gated = up || up_blob;
  if (dup && !gated) return ADACC_EINVAL;
  if (!lay_groups_ok(rows, cols)) return ADACC_ELIMIT;
  if (!rows || !cols || (!da && !dup)) return ADACC_OK;
  if (a_blob) ADACC_TRY(check_blob(a_blob, a_blob_bytes, rows, cols));
  else ADACC_TRY(check_matrix(a, type, rows, cols, a_stride));
  if (up_blob) ADACC_TRY(check_blob(up_blob, up_blob_bytes, rows, cols));
  if (up) ADACC_TRY(check_matrix(up, type, rows, cols, up_stride));
  ADACC_TRY(check_matrix(dy, type, rows, cols, dy_stride));
  if (da) ADACC_TRY(check_matrix(da, type, rows, cols, da_stride));
  if (dup) ADACC_TRY(check_matrix(dup, type, rows, cols, dup_stride));
  ActArgs p;
  std::memset(&p, 0, sizeof p);
  p.cols = (uint32_t)cols;
  p.a = strided(a, a_stride);
  p.up = strided(up, up_stride);
  p.y = strided(dy, dy_stride);
  p.da = strided(da, da_stride);
  p.dup = strided(dup, dup_stride);
  p.a8 = rows8_of(a_blob, rows, cols);
  p.up8 = rows8_of(up_blob, rows, cols);
  return launch_groups(act_backward_fn(type, kind, gated, a_blob != nullptr, cols % 8 == 0), rows, p, static_cast<hipStream_t>(hip_stream), "act_backward_kernel", act_behind(type));
}

// ------------------------------------------------------------------ products
uint64_t adacc_linear_workspace_bytes(uint32_t which, uint64_t m, uint64_t n, uint64_t k) {
  if (which > ADACC_LINEAR_WEIGHT_GRADIENT || !m || !n || !k || m > kLayMost || n > kLayMost || k > kLayMost) return 0;
  if (which == ADACC_LINEAR_ROWS_GRADIENT) return pad_bytes(m, n) + pad_bytes(n, k) + partial_bytes(lin_plan(m, k, n, false), m, k);
  if (which == ADACC_LINEAR_WEIGHT_GRADIENT) return pad_bytes(m, n) + pad_bytes(m, k) + partial_bytes(lin_plan(n, k, m, false), n, k);
  if (lin_plan(m, n, k, which == ADACC_LINEAR_SERVED).few) return 0;
  return pad_bytes(m, k) + pad_bytes(n, k) + partial_bytes(lin_plan(m, n, k, false), m, n);
}

int adacc_linear(uint32_t type, uint32_t kind, const void* x, uint64_t x_stride, const void* w, uint64_t w_stride, uint64_t m, uint64_t n, uint64_t k, uint32_t bias_type, const void* bias,
                 const void* residual, uint64_t residual_stride, void* y, uint64_t y_stride, void* pre, uint64_t pre_stride, void* pre_blob, uint64_t pre_blob_bytes, void* workspace,
                 uint64_t workspace_bytes, void* hip_stream) {
  if (type > kTypeF16 || kind > kActSilu || (bias_type != type && bias_type != kTypeF32)) return ADACC_EINVAL;
  if ((pre || pre_blob) && (kind == kActNone || (pre && pre_blob))) return ADACC_EINVAL;
  if (m > kLayMost || n > kLayMost || k > kLayMost) return ADACC_ELIMIT;
  if (!m || !n) return ADACC_OK;
  if (k) {
    ADACC_TRY(check_operand(x, m, k, x_stride));
    ADACC_TRY(check_operand(w, n, k, w_stride));
  }
  ADACC_TRY(check_vector(bias, bias_type));
  if (residual) ADACC_TRY(check_matrix(residual, type, m, n, residual_stride));
  ADACC_TRY(check_matrix(y, type, m, n, y_stride));
  if (pre) ADACC_TRY(check_matrix(pre, type, m, n, pre_stride));
  if (pre_blob) ADACC_TRY(check_blob(pre_blob, pre_blob_bytes, m, n));
  const bool served = !pre_blob && !pre;
  ADACC_TRY(check_workspace(workspace, workspace_bytes, adacc_linear_workspace_bytes(served ? ADACC_LINEAR_SERVED : ADACC_LINEAR_TRAINED, m, n, k)));
  Epilogue e;
  std::memset(&e, 0, sizeof e);
  e.m = (uint32_t)m;
  e.n = (uint32_t)n;
  e.act = kind;
  e.btype = bias_type;
  e.bias = bias;
  e.residual = strided(residual, residual_stride);
  e.out = strided(y, y_stride);
  e.pre = strided(pre, pre_stride);
  e.pre8 = rows8_of(pre_blob, m, n);
  Rows8 none;
  std::memset(&none, 0, sizeof none);
  return product(lin_plan(m, n, k, served), type, {x, m, k, x_stride}, kAlong, {w, n, k, w_stride}, kAlong, none, k, e, static_cast<uint8_t*>(workspace), static_cast<hipStream_t>(hip_stream));
}

uint64_t adacc_linear_columns_workspace_bytes(uint64_t m, uint64_t n) {
  if (!m || !n || !lay_sizes_ok(m, n)) return 0;
  return lay_align256((uint64_t)strip_partials(m, n) * n * 4);
}

int adacc_linear_columns(uint32_t type, uint32_t kind, const void* dy, uint64_t dy_stride, uint64_t m, uint64_t n, const void* pre, uint64_t pre_stride, const void* pre_blob,
                         uint64_t pre_blob_bytes, void* dpre, uint64_t dpre_stride, uint32_t bias_type, void* dbias, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  if (type > kTypeF16 || kind > kActSilu || (bias_type != type && bias_type != kTypeF32)) return ADACC_EINVAL;
  if ((pre && pre_blob) || (kind == kActNone && (pre || pre_blob || dpre))) return ADACC_EINVAL;
  if (!lay_sizes_ok(m, n)) return ADACC_ELIMIT;
  if (!n) return ADACC_OK;
  ADACC_TRY(check_vector(dbias, bias_type));
  if (m) {
    ADACC_TRY(check_matrix(dy, type, m, n, dy_stride));
    if (kind != kActNone) {
      if (pre_blob) ADACC_TRY(check_blob(pre_blob, pre_blob_bytes, m, n));
      else ADACC_TRY(check_matrix(pre, type, m, n, pre_stride));
      ADACC_TRY(check_matrix(dpre, type, m, n, dpre_stride));
    }
    if (dbias) ADACC_TRY(check_workspace(workspace, workspace_bytes, adacc_linear_columns_workspace_bytes(m, n)));
  }
  if (!dbias && (kind == kActNone || !m)) return ADACC_OK;
  ActArgs p;
  std::memset(&p, 0, sizeof p);
  p.rows = (uint32_t)m;
  p.cols = (uint32_t)n;
  p.a = strided(pre, pre_stride);
  p.a8 = rows8_of(pre_blob, m, n);
  p.y = strided(dy, dy_stride);
  p.da = strided(dpre, dpre_stride);
  p.partial = dbias ? static_cast<float*>(workspace) : nullptr;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (m) {
    p.partials = strip_partials(m, n);
    p.step_groups = strip_wide(n);
    ADACC_TRY(launch(act_columns_fn(type, kind, pre_blob != nullptr), (uint64_t)p.partials * over(over(n, kR8Group), p.step_groups), (uint32_t)kThreads, 0, s, p, "act_columns_kernel"));
  }
  return dbias ? reduce(p.cols, p.partials, 1, p.partial, bias_type, dbias, nullptr, s) : ADACC_OK;
}

int adacc_linear_rows_gradient(uint32_t type, const void* dpre, uint64_t dpre_stride, const void* w, uint64_t w_stride, uint64_t m, uint64_t n, uint64_t k, void* dx, uint64_t dx_stride,
                               void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  if (type > kTypeF16) return ADACC_EINVAL;
  if (m > kLayMost || n > kLayMost || k > kLayMost) return ADACC_ELIMIT;
  if (!m || !k) return ADACC_OK;
  if (n) {
    ADACC_TRY(check_operand(dpre, m, n, dpre_stride));
    ADACC_TRY(check_operand(w, n, k, w_stride));
  }
  ADACC_TRY(check_matrix(dx, type, m, k, dx_stride));
  ADACC_TRY(check_workspace(workspace, workspace_bytes, adacc_linear_workspace_bytes(ADACC_LINEAR_ROWS_GRADIENT, m, n, k)));
  Epilogue e;
  std::memset(&e, 0, sizeof e);
  e.m = (uint32_t)m;
  e.n = (uint32_t)k;
  e.out = strided(dx, dx_stride);
  Rows8 none;
  std::memset(&none, 0, sizeof none);
  return product(lin_plan(m, k, n, false), type, {dpre, m, n, dpre_stride}, kAlong, {w, n, k, w_stride}, kAcross, none, n, e, static_cast<uint8_t*>(workspace), static_cast<hipStream_t>(hip_stream));
}

int adacc_linear_weight_gradient(uint32_t type, const void* dpre, uint64_t dpre_stride, const void* x, uint64_t x_stride, const void* x_blob, uint64_t x_blob_bytes, uint64_t m, uint64_t n,
                                 uint64_t k, void* dw, uint64_t dw_stride, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  if (type > kTypeF16 || (x && x_blob)) return ADACC_EINVAL;
  if (m > kLayMost || n > kLayMost || k > kLayMost) return ADACC_ELIMIT;
  if (!n || !k) return ADACC_OK;
  if (m) {
    ADACC_TRY(check_operand(dpre, m, n, dpre_stride));
    if (x_blob) ADACC_TRY(check_blob(x_blob, x_blob_bytes, m, k));
    else ADACC_TRY(check_operand(x, m, k, x_stride));
    if (x_blob && m > 1 && k >= kLinStrideMost) return ADACC_ELIMIT;
  }
  ADACC_TRY(check_matrix(dw, type, n, k, dw_stride));
  ADACC_TRY(check_workspace(workspace, workspace_bytes, adacc_linear_workspace_bytes(ADACC_LINEAR_WEIGHT_GRADIENT, m, n, k)));
  Epilogue e;
  std::memset(&e, 0, sizeof e);
  e.m = (uint32_t)n;
  e.n = (uint32_t)k;
  e.out = strided(dw, dw_stride);
  return product(lin_plan(n, k, m, false), type, {dpre, m, n, dpre_stride}, kAcross, {x, m, k, x_stride}, x_blob ? kAcross8 : kAcross, rows8_of(x_blob, m, k), m, e,
                 static_cast<uint8_t*>(workspace), static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
