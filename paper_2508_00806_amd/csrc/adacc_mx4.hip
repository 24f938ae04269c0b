// libadacc, host code of the microscaled 4-bit matrices and their products (include/adacc.h).  Kernels: adacc_k_mx4_*.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "adacc.h"
#include "adacc_fn.hpp"
#include "adacc_mx4.hpp"

namespace adacc {

constexpr uint64_t kMxMaxRows = 1ull << 30;      // of a blob, and columns: kernels count them in 32 bits
constexpr uint64_t kMxMaxGrid = 0x7FFFFFFFull;   // workgroups of a call
constexpr uint64_t kMxMaxThreads = 0xFFFFFFFFull;  // of a launch: the runtime takes fewer than 2^32

static uint64_t mx_align256(uint64_t v) { return (v + 255ull) & ~255ull; }
static uint64_t mx_over(uint64_t v, uint64_t by) { return (v + by - 1) / by; }
static bool mx_misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
static uint64_t mx_size(uint32_t type) { return type == ADACC_MX4_F32 ? 4u : 2u; }
static bool mx_sizes_ok(uint64_t rows, uint64_t cols) { return rows <= kMxMaxRows && cols <= kMxMaxRows; }

static void mx_layout(uint64_t rows, uint64_t cols, adacc_mx4_layout* L) {
  L->step_bytes = rows * kMxStepBytes;
  L->scale_pitch = mx_over(rows, 16) * 16;
  L->codes_off = 0;
  L->scales_off = mx_align256(mx_over(cols, kMxStep) * L->step_bytes);
  L->total_bytes = L->scales_off + mx_align256(mx_over(cols, kMxStep) * 4 * L->scale_pitch);
}

static MxMatrix mx_matrix(const void* blob, uint64_t rows, uint64_t cols) {
  adacc_mx4_layout L;
  mx_layout(rows, cols, &L);
  MxMatrix m;
  uint8_t* b = static_cast<uint8_t*>(const_cast<void*>(blob));
  m.codes = b + L.codes_off;
  m.scales = b + L.scales_off;
  m.step_bytes = L.step_bytes;
  m.pitch = L.scale_pitch;
  m.rows = (uint32_t)rows;
  m.steps = (uint32_t)mx_over(cols, kMxStep);
  return m;
}

// a blob that a call reads or writes
static int mx_check_blob(const void* blob, uint64_t bytes, uint64_t rows, uint64_t cols) {
  adacc_mx4_layout L;
  mx_layout(rows, cols, &L);
  if (L.total_bytes == 0) return ADACC_OK;
  if (!blob) return ADACC_ENULL;
  if (bytes < L.total_bytes) return ADACC_ESIZE;
  return mx_misaligned(blob, 256) ? ADACC_EALIGN : ADACC_OK;
}

// rows sorted by group, `per` a tile: no more tiles than this, whatever the offsets are (`lower`: a group's first tile may start up to three rows early).
// The rows behind the last group count as one more.
static uint64_t mx_tiles(uint64_t rows, uint32_t groups, uint64_t per, bool lower) {
  if (groups == 0) return mx_over(rows, per);
  const uint64_t live = std::min<uint64_t>(groups + 1ull, rows);
  return (rows + (lower ? 3 * live : 0)) / per + live;
}

static int mx_check_groups(const int32_t* offsets, uint32_t groups) {
  if (groups > kMxMaxGroups) return ADACC_ELIMIT;
  if ((offsets != nullptr) != (groups != 0)) return offsets ? ADACC_EINVAL : ADACC_ENULL;
  return mx_misaligned(offsets, 4) ? ADACC_EALIGN : ADACC_OK;
}

static int mx_check_out(const void* out, uint32_t type, uint64_t cols, uint64_t stride) {
  if (type > ADACC_MX4_F32 || stride < cols) return ADACC_EINVAL;
  if (!out) return ADACC_ENULL;
  return mx_misaligned(out, mx_size(type)) ? ADACC_EALIGN : ADACC_OK;
}

// ------------------------------------------------------------------ which kernel
struct MxPlan {
  bool few, ready;    // few rows; the left operand has to be compressed before
  uint32_t ms, ns, waves;
  uint32_t tile;
};
constexpr uint64_t kMxCus = 256;
constexpr uint64_t kMxFewTiles = 160;
// Values of a tile's rows that every workgroup compresses for itself rather than reading them from a launch of its own (3.4 us): 16 rows by 4096 x 4096
// 7.0 us, 5.1 and the launch; by 4096 x 11008 12.7, 8.3 and the launch.
constexpr uint64_t kMxFewRaw = 1ull << 16;
static uint32_t mx_few_row_lds(uint64_t k) { return (uint32_t)mx_over(k, kMxStep) * (kMxStepBytes + 4u); }

// Rows and columns of a tile, by the number of tiles that there would be.  us in tiles of 256 / 128 / 64: 4096^3 (256, 1024 ... tiles) 38 / 41 / 64;
// 1024 x 11008 x 4096 (172, 688) 31 / 31 / 45; 1536 x 2048 x 2048 (48, 192, 768) - / 10.9 / 12.0; 1024 x 2048 x 2048 (32, 128, 512) - / 10.2 / 9.8.
// A tile of 256 has no way for a lane whose four columns are not all inside.
static uint32_t mx_tile_of(uint64_t rows, uint64_t n, uint64_t live) {
  const auto tiles = [&](uint64_t t) { return mx_over(rows, t) * mx_over(n, t) * live; };
  return n % 4 == 0 && tiles(256) >= kMxCus ? 256u : tiles(128) >= 144 ? 128u : 64u;
}

static MxPlan mx_plan(uint64_t m, uint64_t n, uint64_t k, uint32_t groups) {
  MxPlan p;
  std::memset(&p, 0, sizeof p);
  const uint64_t rows = groups ? mx_over(m, groups) : m;  // of a group, on average
  const uint64_t live = groups ? std::min<uint64_t>(groups, m) : 1;
  // 33 to 64 rows: by 11008 x 4096 (172 tiles) 8.9 us in tiles, else 11.7; by 4096 x 4096 (64) 7.7, else 6.1; by 4096 x 11008 16.3, else 12.5.
  // 32 rows and fewer, however many tiles: by 11008 x 4096 17 rows 8.4 in tiles, else 8.1; 24 8.4, else 8.3; 32 8.1, else 8.5; by 4096 x 4096 32 rows 7.9, else 4.9
  // (A group of many rows among groups of few goes the way of the few: 64 groups by 2048 x 2048, all 2048 rows in one, 29 us; 32 in each 34; 9 without groups.)
  p.few = rows <= 32 || (rows <= 64 && mx_over(n, 64) * live < 128);
  if (p.few) {
    p.ms = rows <= 16 ? 1u : rows <= 32 ? 2u : 4u;
    const uint64_t m_tiles = groups ? live : mx_over(m, 16 * p.ms);
    // columns a workgroup: 64 or 32 read a's rows less often, where that leaves work for most of the 256 compute units (one row by 11008 x 4096:
    // 172 workgroups of 64 columns 7.3 us, 344 of 32 8.2, 688 of 16 7.9; by 4096 x 11008: 128 of 32 8.9, 256 of 16 7.9)
    p.ns = mx_over(n, 64) * m_tiles >= kMxFewTiles ? 4u : mx_over(n, 32) * m_tiles >= kMxFewTiles ? 2u : 1u;
    // a compute unit holds mx4_few_waves wavefronts: they are shared among the workgroups that come to it, none has less than a turn of two steps
    const uint64_t wgs = mx_over(n, 16 * p.ns) * m_tiles, most = mx4_few_waves(p.ms);
    p.waves = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(most / std::min<uint64_t>(most, mx_over(wgs, kMxCus)), mx_over(k, 2 * kMxStep)));
    p.ready = p.ms != 1 || k % 8 != 0 || (groups ? std::min<uint64_t>(m, 16) : m) * k > kMxFewRaw;
    return p;
  }
  p.tile = mx_tile_of(rows, n, live);
  p.ready = true;
  return p;
}

static int mx_launch(MxProductFn fn, uint64_t grid, uint32_t threads, uint32_t lds, hipStream_t s, const MxProductArgs& a, const char* what) {
  if (grid * threads > kMxMaxThreads) return ADACC_ELIMIT;  // (no product within the limits has so many: tiles 512 workgroups, few rows 2^25 of 64)
  if (grid == 0) return ADACC_OK;
  if (lds > 65536u) {  // more than a launch may ask for unless the kernel has been told (nothing is enqueued by it)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return hip_result(e, what);
  }
  hipLaunchKernelGGL(fn, dim3((uint32_t)grid), dim3(threads), lds, s, a);
  return launch_check(what);
}

// As many workgroups as the compute units hold at a time, by LDS: one of tiles of 256, else two
static int mx_launch_tiles(uint32_t tile, bool gradient, uint64_t tiles, hipStream_t s, const MxProductArgs& a, const char* what) {
  if (tiles > kMxMaxGrid) return ADACC_ELIMIT;
  const uint64_t room = tile == 256 ? kMxCus : 2 * kMxCus;
  return mx_launch(mx4_product_fn(tile, gradient), std::min(tiles, room), kThreads, mx4_product_lds(tile), s, a, what);
}

// a (or x) times b: the operands have been checked
static int mx_product(const MxPlan& plan, MxProductArgs& a, uint32_t src, hipStream_t s) {
  if (plan.few) {
    a.n_tiles = (uint32_t)mx_over(a.n, 16 * plan.ns);
    const uint64_t m_tiles = mx_tiles(a.m, a.g.groups, 16 * plan.ms, false);
    a.m_tiles = (uint32_t)m_tiles;
    const uint32_t lds = std::max<uint32_t>(plan.waves * 16u * plan.ms * 16u * plan.ns * 4u, src != kMxReady ? mx_few_row_lds(a.k) * (uint32_t)std::min<uint64_t>(a.m, 16u * plan.ms) : 0u);
    return mx_launch(mx4_few_fn(plan.ms, plan.ns, src), m_tiles * a.n_tiles, plan.waves * kWave, lds, s, a, "mx4_few_kernel");
  }
  const uint64_t m_tiles = mx_tiles(a.m, a.g.groups, plan.tile, true);
  a.m_tiles = (uint32_t)m_tiles;
  a.n_tiles = (uint32_t)mx_over(a.n + (a.g.groups && a.n % 4 ? 3 : 0), plan.tile);
  return mx_launch_tiles(plan.tile, false, m_tiles * a.n_tiles, s, a, "mx4_product_kernel");
}

// A conversion: one launch, but for matrices of 2^24 workgroups and more (2^29 rows along, 2^24 matrices across), whose launches follow each other
template <typename Args>
static int mx_launch_conversion(void (*fn)(Args), uint64_t grid, hipStream_t s, Args a, const char* what) {
  if (grid > kMxMaxGrid) return ADACC_ELIMIT;
  constexpr uint64_t kMost = kMxMaxThreads / kThreads;
  for (uint64_t at = 0; at < grid; at += kMost) {
    a.first = (uint32_t)at;
    hipLaunchKernelGGL(fn, dim3((uint32_t)std::min(grid - at, kMost)), dim3(kThreads), 0, s, a);
    const int rc = launch_check(what);
    if (rc != ADACC_OK) return rc;
  }
  return ADACC_OK;
}

static void mx_compress_args(uint32_t scale_rule, const void* src, uint64_t mats, uint64_t rows, uint64_t cols,
                                    uint64_t row_stride, uint64_t mat_stride, MxCompressArgs* a) {
  std::memset(a, 0, sizeof *a);
  a->src = src;
  a->row_stride = row_stride;
  a->mat_stride = mat_stride;
  a->mats = (uint32_t)mats;
  a->rows = (uint32_t)rows;
  a->cols = (uint32_t)cols;
  a->fullrange = scale_rule;
  a->g.rows = (uint32_t)rows;
}

static int mx_compress_along(uint32_t type, MxCompressArgs a, void* blob, hipStream_t s) {
  a.col_tiles = (uint32_t)mx_over(a.cols, type == ADACC_MX4_F32 ? 256 : 512);
  if (a.mats > 1 && a.mat_stride == (uint64_t)a.rows * a.row_stride) {  // one after the other: one matrix
    a.rows *= a.mats;
    a.mats = 1;
  }
  a.along = mx_matrix(blob, (uint64_t)a.mats * a.rows, a.cols);
  a.row_tiles = (uint32_t)mx_over(a.rows, kMxWaveRows * kWavesPerWg);
  const bool narrow = a.cols * mx_size(type) < 16;
  return mx_launch_conversion(mx4_compress_fn(type, true, false, narrow), (uint64_t)a.row_tiles * a.mats * a.col_tiles, s, a, "mx4_along_kernel");
}

}  // namespace adacc

using namespace adacc;

extern "C" {

int adacc_mx4_layout_of(uint64_t rows, uint64_t cols, adacc_mx4_layout* out) {
  if (!out) return ADACC_ENULL;
  if (!mx_sizes_ok(rows, cols)) return ADACC_ELIMIT;
  mx_layout(rows, cols, out);
  return ADACC_OK;
}

uint64_t adacc_mx4_grouped_cols(uint64_t rows, uint32_t groups) {
  if (rows > kMxMaxRows || groups > kMxMaxGroups) return 0;
  return (rows + (uint64_t)(kMxTileRows - 1) * std::min<uint64_t>(groups, rows)) / kMxTileRows * kMxTileRows;
}

int adacc_mx4_compress(uint32_t type, uint32_t scale_rule, const void* src, uint64_t mats, uint64_t rows, uint64_t cols, uint64_t row_stride,
                       uint64_t mat_stride, const int32_t* offsets, uint32_t groups, void* along, uint64_t along_bytes, void* across,
                       uint64_t across_bytes, void* hip_stream) {
  if (type > ADACC_MX4_F32 || scale_rule > ADACC_MX4_SCALE_FULLRANGE) return ADACC_EINVAL;
  if (row_stride < cols || (groups && mats != 1)) return ADACC_EINVAL;
  if (!mx_sizes_ok(rows, cols) || mats > kMxMaxRows || mats * std::max(rows, cols) > kMxMaxRows) return ADACC_ELIMIT;
  int rc = mx_check_groups(offsets, groups);
  if (rc != ADACC_OK) return rc;
  const uint64_t positions = groups ? adacc_mx4_grouped_cols(rows, groups) : rows;
  if (positions > kMxMaxRows) return ADACC_ELIMIT;
  if (!mats || !rows || !cols) return ADACC_OK;
  if (!src || (!along && !across)) return ADACC_ENULL;
  if (mx_misaligned(src, mx_size(type))) return ADACC_EALIGN;
  if (along && (rc = mx_check_blob(along, along_bytes, mats * rows, cols)) != ADACC_OK) return rc;
  if (across && (rc = mx_check_blob(across, across_bytes, mats * cols, positions)) != ADACC_OK) return rc;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  MxCompressArgs a;
  mx_compress_args(scale_rule, src, mats, rows, cols, row_stride, mat_stride, &a);
  const bool narrow = cols < 4;  // (a lane of that kernel has four columns)
  if (!across) return mx_compress_along(type, a, along, s);
  MxCompressArgs b = a;
  const bool both = along && !narrow;  // (narrow rows: a pass for either)
  if (both) b.along = mx_matrix(along, mats * rows, cols);
  b.across = mx_matrix(across, mats * cols, positions);
  b.g.offsets = offsets;
  b.g.groups = groups;
  b.col_tiles = (uint32_t)mx_over(cols, 256);
  const uint64_t row_tiles = mx_tiles(rows, groups, kMxTileRows, false);
  b.row_tiles = (uint32_t)row_tiles;
  rc = mx_launch_conversion(mx4_compress_fn(type, both, true, narrow), row_tiles * mats * b.col_tiles, s, b, "mx4_across_kernel");
  if (rc != ADACC_OK || both || !along) return rc;
  return mx_compress_along(type, a, along, s);
}

int adacc_mx4_decompress(const void* blob, uint64_t blob_bytes, uint64_t rows, uint64_t cols, void* dst, uint32_t type, uint64_t row_stride,
                         void* hip_stream) {
  if (type > ADACC_MX4_F32 || row_stride < cols) return ADACC_EINVAL;
  if (!mx_sizes_ok(rows, cols)) return ADACC_ELIMIT;
  if (!rows || !cols) return ADACC_OK;
  if (!dst) return ADACC_ENULL;
  if (mx_misaligned(dst, mx_size(type))) return ADACC_EALIGN;
  const int rc = mx_check_blob(blob, blob_bytes, rows, cols);
  if (rc != ADACC_OK) return rc;
  MxDecompressArgs a;
  std::memset(&a, 0, sizeof a);
  a.m = mx_matrix(blob, rows, cols);
  a.cols = (uint32_t)cols;
  a.dst = dst;
  a.row_stride = row_stride;
  a.col_tiles = (uint32_t)mx_over(cols, type == ADACC_MX4_F32 ? 256 : 512);
  return mx_launch_conversion(mx4_decompress_fn(type), mx_over(rows, kMxWaveRows * kWavesPerWg) * a.col_tiles, static_cast<hipStream_t>(hip_stream), a,
                              "mx4_restore_kernel");
}

// what the three products check alike; the left operand is the caller's matter.  b has the rows of every group.
static int mx_check_product(const void* b, uint64_t b_bytes, uint64_t m, uint64_t n, uint64_t k, const int32_t* offsets, uint32_t groups,
                            const void* out, uint32_t out_type, uint64_t out_stride) {
  if (out_type > ADACC_MX4_F32 || out_stride < n) return ADACC_EINVAL;
  const uint64_t mats = groups ? groups : 1;
  if (m > kMxMaxRows || n > kMxMaxRows || mats * n > kMxMaxRows || k > kMxMaxRows) return ADACC_ELIMIT;
  int rc = mx_check_groups(offsets, groups);
  if (rc != ADACC_OK || !m || !n) return rc;
  rc = mx_check_out(out, out_type, n, out_stride);
  return rc != ADACC_OK ? rc : mx_check_blob(b, b_bytes, mats * n, k);
}

static void mx_product_args(const void* b, uint64_t m, uint64_t n, uint64_t k, const int32_t* offsets, uint32_t groups, void* out,
                            uint32_t out_type, uint64_t out_stride, MxProductArgs* p) {
  std::memset(p, 0, sizeof *p);
  p->b = mx_matrix(b, (groups ? groups : 1) * n, k);
  p->out = out;
  p->out_stride = out_stride;
  p->out_type = out_type;
  p->m = (uint32_t)m;
  p->n = (uint32_t)n;
  p->k = (uint32_t)k;
  p->g.offsets = offsets;
  p->g.groups = groups;
  p->g.rows = (uint32_t)m;
}

int adacc_mx4_product(const void* a, uint64_t a_bytes, uint64_t m, const void* b, uint64_t b_bytes, uint64_t n, uint64_t k,
                      const int32_t* offsets, uint32_t groups, void* out, uint32_t out_type, uint64_t out_stride, void* hip_stream) {
  int rc = mx_check_product(b, b_bytes, m, n, k, offsets, groups, out, out_type, out_stride);
  if (rc != ADACC_OK || !m || !n) return rc;
  rc = mx_check_blob(a, a_bytes, m, k);
  if (rc != ADACC_OK) return rc;
  MxProductArgs p;
  mx_product_args(b, m, n, k, offsets, groups, out, out_type, out_stride, &p);
  p.a = mx_matrix(a, m, k);
  return mx_product(mx_plan(m, n, k, groups), p, kMxReady, static_cast<hipStream_t>(hip_stream));
}

uint64_t adacc_mx4_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, uint32_t groups) {
  if (!m || !n || m > kMxMaxRows || k > kMxMaxRows || !mx_plan(m, n, k, groups).ready) return 0;
  adacc_mx4_layout L;
  mx_layout(m, k, &L);
  return L.total_bytes;
}

int adacc_mx4_linear(uint32_t type, uint32_t scale_rule, const void* x, uint64_t m, uint64_t x_stride, const void* b, uint64_t b_bytes,
                     uint64_t n, uint64_t k, const int32_t* offsets, uint32_t groups, void* out, uint32_t out_type, uint64_t out_stride,
                     void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  if (type > ADACC_MX4_F32 || scale_rule > ADACC_MX4_SCALE_FULLRANGE || x_stride < k) return ADACC_EINVAL;
  int rc = mx_check_product(b, b_bytes, m, n, k, offsets, groups, out, out_type, out_stride);
  if (rc != ADACC_OK || !m || !n) return rc;
  if (k && !x) return ADACC_ENULL;
  if (mx_misaligned(x, mx_size(type))) return ADACC_EALIGN;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const MxPlan plan = mx_plan(m, n, k, groups);
  MxProductArgs p;
  mx_product_args(b, m, n, k, offsets, groups, out, out_type, out_stride, &p);
  if (!plan.ready) {
    p.x = x;
    p.x_stride = x_stride;
    p.fullrange = scale_rule;
    return mx_product(plan, p, type, s);
  }
  rc = mx_check_blob(workspace, workspace_bytes, m, k);
  if (rc != ADACC_OK) return rc;
  if (k) {
    MxCompressArgs c;
    mx_compress_args(scale_rule, x, 1, m, k, x_stride, 0, &c);
    rc = mx_compress_along(type, c, workspace, s);
    if (rc != ADACC_OK) return rc;
  }
  p.a = mx_matrix(workspace, m, k);
  return mx_product(plan, p, kMxReady, s);
}

int adacc_mx4_gradient(const void* a, uint64_t a_bytes, uint64_t m, const void* b, uint64_t b_bytes, uint64_t n, uint64_t rows,
                       const int32_t* offsets, uint32_t groups, void* out, uint32_t out_type, uint64_t out_stride, void* hip_stream) {
  if (out_type > ADACC_MX4_F32 || out_stride < n) return ADACC_EINVAL;
  if (m > kMxMaxRows || n > kMxMaxRows || rows > kMxMaxRows) return ADACC_ELIMIT;
  int rc = mx_check_groups(offsets, groups);
  if (rc != ADACC_OK) return rc;
  const uint64_t positions = groups ? adacc_mx4_grouped_cols(rows, groups) : rows;
  if (positions > kMxMaxRows) return ADACC_ELIMIT;
  if (!m || !n) return ADACC_OK;
  rc = mx_check_out(out, out_type, n, out_stride);
  if (rc == ADACC_OK) rc = mx_check_blob(a, a_bytes, m, positions);
  if (rc == ADACC_OK) rc = mx_check_blob(b, b_bytes, n, positions);
  if (rc != ADACC_OK) return rc;
  MxProductArgs p;
  std::memset(&p, 0, sizeof p);
  p.a = mx_matrix(a, m, positions);
  p.b = mx_matrix(b, n, positions);
  p.out = out;
  p.out_stride = out_stride;
  p.out_group = m * out_stride;
  p.out_type = out_type;
  p.m = (uint32_t)m;
  p.n = (uint32_t)n;
  p.k = (uint32_t)positions;
  p.g.offsets = offsets;
  p.g.groups = groups;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (!groups) {
    p.g.rows = (uint32_t)m;
    return mx_product(mx_plan(m, n, positions, 0), p, kMxReady, s);
  }
  p.g.rows = (uint32_t)rows;
  const uint32_t tile = mx_tile_of(m, n, groups);
  p.m_tiles = (uint32_t)mx_over(m, tile);
  p.n_tiles = (uint32_t)mx_over(n, tile);
  return mx_launch_tiles(tile, true, (uint64_t)p.m_tiles * p.n_tiles * groups, s, p, "mx4_gradient_kernel");
}

}  // extern "C"
