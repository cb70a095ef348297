// Entry points of the 8-bit matrices (dr.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "dr_internal.h"
#include "quant_kernels.h"

namespace dr {
namespace {

bool aligned(const void* p, uintptr_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int64_t padded(int64_t cols) { return ceil_div(cols, kBlock) * kBlock; }

int check_shape(int64_t rows, int64_t cols, int32_t block_rows, const char* what, const char* name) {
  if (rows < 0 || rows >= kMaxQRows || cols < 0 || cols > kMaxQCols)
    return fail(DR_EINVAL, "%s: %s is %lld x %lld (rows are below 2^26, columns at most 2^23)", what, name,
                (long long)rows, (long long)cols);
  if (block_rows != 1 && block_rows != kBlock)
    return fail(DR_EINVAL, "%s: %s has blocks of %d rows (1 or 128)", what, name, block_rows);
  return DR_OK;
}

int check_matrix(const dr_qmatrix* m, const char* what, const char* name) {
  if (!m) return fail(DR_EINVAL, "%s: %s is null", what, name);
  if (int rc = check_shape(m->rows, m->cols, m->block_rows, what, name)) return rc;
  if (m->reserved) return fail(DR_EINVAL, "%s: %s: reserved field is not 0", what, name);
  if (m->stride < padded(m->cols) || m->stride > kMaxQCols || m->stride % 16)
    return fail(DR_EINVAL, "%s: %s: stride %lld (a multiple of 16 from %lld to 2^23)", what, name, (long long)m->stride,
                (long long)padded(m->cols));
  if (m->rows && m->cols && (!aligned(m->data, 16) || !aligned(m->scales, 4)))
    return fail(DR_EINVAL, "%s: %s: data (16-byte) or scales (4-byte) null or misaligned", what, name);
  return DR_OK;
}

QView view(const dr_qmatrix& m) {
  return QView{static_cast<uint8_t*>(m.data),         static_cast<uint8_t*>(m.scales),
               m.stride,                              (uint32_t)m.rows,
               (uint32_t)m.cols,                      (uint32_t)ceil_div(m.rows, m.block_rows),
               m.block_rows == 1 ? 0 : 7};
}

int element_bytes(int32_t type) { return type == DR_TYPE_F32 ? 4 : type == DR_TYPE_BF16 ? 2 : 0; }

// A dense matrix of `type` with rows of row_stride elements.
int check_dense(const void* p, int32_t type, int64_t rows, int64_t cols, int64_t row_stride, const char* what,
                const char* name) {
  const int size = element_bytes(type);
  if (!size) return fail(DR_EINVAL, "%s: %s has unknown type %d", what, name, type);
  if (row_stride < cols || row_stride > (1ll << 40))
    return fail(DR_EINVAL, "%s: %s: row stride %lld for %lld columns", what, name, (long long)row_stride, (long long)cols);
  if (rows && cols && !aligned(p, size)) return fail(DR_EINVAL, "%s: %s is null or misaligned", what, name);
  return DR_OK;
}

// The tiles of a product are counted in 32 bits.
int check_results(int64_t m, int64_t n, const char* what) {
  return m * n <= 1ll << 38 ? DR_OK : fail(DR_EINVAL, "%s: %lld x %lld results (at most 2^38)", what, (long long)m, (long long)n);
}

int hip_result(hipError_t e, const char* what) {
  return e == hipSuccess ? DR_OK : fail(DR_EHIP, "%s: kernel launch: %s", what, hipGetErrorString(e));
}

int quantize(const void* src, int32_t type, int64_t rows, int64_t cols, int64_t row_stride, const dr_qmatrix* q,
             const dr_qmatrix* qt, hipStream_t st, const char* what) {
  const int64_t tiles = ceil_div(rows, kBlock) * ceil_div(cols, kBlock);
  if (tiles > max_workgroups(kTileLanes))
    return fail(DR_EINVAL, "%s: %lld x %lld is %s tiles", what, (long long)rows, (long long)cols,
                tiles > 1 << 24 ? "more than 2^24" : "2^23 or more");
  if (!rows || !cols) return DR_OK;
  QuantizeLaunch l;
  std::memset(&l, 0, sizeof(l));
  l.src = src;
  l.src_stride = row_stride;
  l.rows = (uint32_t)rows;
  l.cols = (uint32_t)cols;
  l.bf16 = type == DR_TYPE_BF16;
  if (q) l.q = view(*q);
  if (qt) l.qt = view(*qt);
  return hip_result(launch_quantize(l, st), what);
}

// Bytes of the splits' sums, whichever sums the caller asks for.
uint64_t product_space(int64_t m, int64_t n, int64_t k) {
  uint64_t bytes = 0;
  for (bool fast : {false, true}) {
    const ProductPlan plan = plan_product(m, n, ceil_div(k, kBlock), fast);
    if (plan.splits > 1) bytes = std::max(bytes, (uint64_t)plan.splits * m * part_stride(n) * sizeof(float));
  }
  return bytes;
}

// Where the quantized rows of a linear layer lie in its workspace.
struct LinearSpace {
  uint64_t data, scales, product, total;
};
LinearSpace linear_space(int64_t m, int64_t n, int64_t k) {
  LinearSpace s{0, 0, 0, 0};
  if (m > kFusedRows) {
    s.scales = s.data + (uint64_t)m * padded(k);
    s.product = s.scales + (uint64_t)ceil_div(padded(k) / kBlock, 4) * m * 4;
    s.product = (s.product + 15) / 16 * 16;
    s.total = s.product + product_space(m, n, k);
  }
  return s;
}

int check_workspace(const void* p, uint64_t have, uint64_t need, const char* what) {
  if (have < need || (need && !aligned(p, 16)))
    return fail(DR_EINVAL, "%s: workspace of %llu bytes null, misaligned or too small (%llu needed)", what,
                (unsigned long long)have, (unsigned long long)need);
  return DR_OK;
}

}  // namespace

// Times in us, measured on random codes.  A step of a 256 x 256 tile takes 1.34 (exact sums 2.7), of one 128 x 128 tile
// alone on its CU 0.63 (0.78; 0.5 with four blocks staged) and of two of them together 0.96 (1.72); what a tile costs beside
// its steps is 8, 3 and, of two together, 4; a second launch 6; joining splits 4 and their sums' bytes, written and read, at
// 6.5 TB/s.  A round of 256 workgroups of the kernel for few rows takes direct_step (by columns and by rows per workgroup)
// for each 128-column block of a wave, beside direct_start and 0.5 for each further round, and no less than the weights at
// 4.5 TB/s.  Over 83 shapes from 48 x 2000 x 2000 to 3000 x 32064 x 4096 the choice takes at most 11 % more than the
// best of eight ways with tiles and three with the kernel for few rows, in another session 19 % (200 x 4096 x 3584); that kernel
// brings 48 x 2000 x 2000 from 10.0 to 6.7, 200 x 688 x 256 from 5.4 to 3.7.
ProductPlan plan_product(int64_t m, int64_t n, int64_t kb, bool fast) {
  if (m <= 32 || !kb) return {ProductPlan::kDirect, 1, 0, m <= 16 ? 1u : 2u};
  constexpr double kCus = 256;
  const double step256 = fast ? 1.34 : 2.7, step128 = fast ? 0.63 : 0.78, pair128 = fast ? 0.96 : 1.72;
  ProductPlan best{ProductPlan::kTile256, 1, 0, 2};
  double least = HUGE_VAL;
  constexpr double direct_step[3][3] = {{1.45, 1.72, 2.45}, {1.88, 2.3, 2.9}, {1.35, 1.75, 2.1}}, direct_start[3] = {1.8, 3, 3};
  const uint32_t columns16 = direct_columns16(n), waves = direct_waves(columns16), wide = columns16 / 2;
  const double blocks = kb < waves ? (double)kb / waves : (double)ceil_div(kb, waves);
  for (uint32_t rows16 = 2; rows16 <= 4; ++rows16) {
    const double rounds = std::ceil((double)ceil_div(n, 16 * columns16) * (double)ceil_div(m, 16 * rows16) / kCus);
    const double us = std::max(direct_start[wide] + rounds * blocks * direct_step[wide][rows16 - 2] + 0.5 * (rounds - 1), 2 + 128.0 * (double)kb * (double)n / 4.5e6);
    if (us < least) least = us, best = {ProductPlan::kDirect, 1, 0, rows16};
  }
  for (const auto kind : {ProductPlan::kTile256, ProductPlan::kTile128}) {
    const int64_t side = kind == ProductPlan::kTile256 ? 256 : 128;
    const double tiles = (double)ceil_div(m, side) * (double)ceil_div(n, side);
    for (uint32_t splits = 1; splits <= 16 && (splits == 1 || (kb >= 2 * (int64_t)splits && part_stride(n) * 4 < kMaxRowBytes)); ++splits) {
      const double steps = (double)ceil_div(kb, splits), rounds = std::ceil(tiles * splits / kCus);
      const double us = splits == 1 ? 0 : 4 + 8.0 * splits * (double)m * (double)part_stride(n) / 6.5e6;
      auto time128 = [&](double n_rounds) {
        const double pairs = std::floor(n_rounds / 2), lone = n_rounds - 2 * pairs;
        const double step = fast && n_rounds == 1 && steps >= 4 ? 0.5 : step128;
        return pairs * (steps * pair128 + 4) + lone * (steps * step + 3);
      };
      auto consider = [&](double time, uint32_t quartered) {
        if (us + time < least) least = us + time, best = {kind, splits, quartered, 2};
      };
      if (kind == ProductPlan::kTile128) {
        consider(time128(rounds), 0);
        continue;
      }
      const double round = steps * step256 + 8, rest = tiles - kCus * (rounds - 1);
      consider(rounds * round, 0);
      // a last round that few tiles share: these by quarters
      if (splits == 1 && rounds > 1 && rest < kCus)
        consider((rounds - 1) * round + 6 + time128(std::ceil(4 * rest / kCus)), (uint32_t)rest);
    }
  }
  return best;
}
}  // namespace dr

using namespace dr;

extern "C" int dr_qmatrix_sizes(int64_t rows, int64_t cols, int32_t block_rows, int64_t* stride, uint64_t* data_bytes,
                                uint64_t* scale_bytes) {
  clear_error();
  if (int rc = check_shape(rows, cols, block_rows, "dr_qmatrix_sizes", "the matrix")) return rc;
  const int64_t s = padded(cols);
  if (stride) *stride = s;
  if (data_bytes) *data_bytes = (uint64_t)rows * s;
  if (scale_bytes) *scale_bytes = (uint64_t)ceil_div(s / kBlock, 4) * ceil_div(rows, block_rows) * 4;
  return DR_OK;
}

extern "C" int dr_quantize(const void* src, int32_t type, int64_t rows, int64_t cols, int64_t row_stride,
                           const dr_qmatrix* q, const dr_qmatrix* qt, void* stream) {
  clear_error();
  const char* what = "dr_quantize";
  if (!q && !qt) return fail(DR_EINVAL, "%s: neither q nor qt given", what);
  if (q) {
    if (int rc = check_matrix(q, what, "q")) return rc;
    if (q->rows != rows || q->cols != cols) return fail(DR_EINVAL, "%s: q is not %lld x %lld", what, (long long)rows, (long long)cols);
  }
  if (qt) {
    if (int rc = check_matrix(qt, what, "qt")) return rc;
    if (qt->rows != cols || qt->cols != rows) return fail(DR_EINVAL, "%s: qt is not %lld x %lld", what, (long long)cols, (long long)rows);
    if (q && q->block_rows != qt->block_rows) return fail(DR_EINVAL, "%s: q and qt differ in block_rows", what);
  }
  if (int rc = check_dense(src, type, rows, cols, row_stride, what, "src")) return rc;
  return quantize(src, type, rows, cols, row_stride, q, qt, static_cast<hipStream_t>(stream), what);
}

extern "C" int dr_qmatmul_workspace(int64_t m, int64_t n, int64_t k, uint64_t* bytes) {
  clear_error();
  const char* what = "dr_qmatmul_workspace";
  if (!bytes) return fail(DR_EINVAL, "%s: null argument", what);
  if (int rc = check_shape(m, k, 1, what, "a")) return rc;
  if (int rc = check_shape(n, k, 1, what, "b")) return rc;
  *bytes = product_space(m, n, k);
  return DR_OK;
}

extern "C" int dr_qlinear_workspace(int64_t m, int64_t n, int64_t k, uint64_t* bytes) {
  clear_error();
  const char* what = "dr_qlinear_workspace";
  if (!bytes) return fail(DR_EINVAL, "%s: null argument", what);
  if (int rc = check_shape(m, k, 1, what, "x")) return rc;
  if (int rc = check_shape(n, k, 1, what, "w")) return rc;
  *bytes = linear_space(m, n, k).total;
  return DR_OK;
}

extern "C" int dr_qmatmul(const dr_qmatrix* a, const dr_qmatrix* b, void* c, int32_t type, int64_t row_stride,
                          int32_t flags, void* workspace, uint64_t workspace_bytes, void* stream) {
  clear_error();
  const char* what = "dr_qmatmul";
  if (int rc = check_matrix(a, what, "a")) return rc;
  if (int rc = check_matrix(b, what, "b")) return rc;
  if (a->cols != b->cols)
    return fail(DR_EINVAL, "%s: a has %lld columns, b %lld", what, (long long)a->cols, (long long)b->cols);
  if (int rc = check_dense(c, type, a->rows, b->rows, row_stride, what, "c")) return rc;
  if (flags & ~(DR_ACCUMULATE | DR_FAST_SUMS)) return fail(DR_EINVAL, "%s: unknown flags %d", what, flags);
  if ((flags & DR_ACCUMULATE) && type != DR_TYPE_F32) return fail(DR_EINVAL, "%s: DR_ACCUMULATE needs an fp32 c", what);
  if (int rc = check_results(a->rows, b->rows, what)) return rc;
  uint64_t need = 0;
  if (int rc = dr_qmatmul_workspace(a->rows, b->rows, a->cols, &need)) return rc;
  if (int rc = check_workspace(workspace, workspace_bytes, need, what)) return rc;
  if (!a->rows || !b->rows) return DR_OK;
  ProductLaunch l;
  std::memset(&l, 0, sizeof(l));
  l.a = view(*a);
  l.b = view(*b);
  l.c = c;
  l.c_stride = row_stride;
  l.m = (uint32_t)a->rows;
  l.n = (uint32_t)b->rows;
  l.kb = (uint32_t)ceil_div(a->cols, kBlock);
  l.c_bf16 = type == DR_TYPE_BF16;
  l.accumulate = (flags & DR_ACCUMULATE) != 0;
  l.fast = (flags & DR_FAST_SUMS) != 0;
  l.workspace = workspace;
  return hip_result(launch_product(l, static_cast<hipStream_t>(stream)), what);
}

extern "C" int dr_qlinear(const void* x, int32_t x_type, int64_t m, int64_t x_row_stride, const dr_qmatrix* w, void* y,
                          int32_t y_type, int64_t y_row_stride, int32_t flags, void* workspace,
                          uint64_t workspace_bytes, void* stream) {
  clear_error();
  const char* what = "dr_qlinear";
  if (int rc = check_matrix(w, what, "w")) return rc;
  const int64_t k = w->cols, n = w->rows;
  if (int rc = check_shape(m, k, 1, what, "x")) return rc;
  if (int rc = check_dense(x, x_type, m, k, x_row_stride, what, "x")) return rc;
  if (int rc = check_dense(y, y_type, m, n, y_row_stride, what, "y")) return rc;
  if (flags & ~DR_FAST_SUMS) return fail(DR_EINVAL, "%s: unknown flags %d", what, flags);
  if (int rc = check_results(m, n, what)) return rc;
  const LinearSpace s = linear_space(m, n, k);
  if (int rc = check_workspace(workspace, workspace_bytes, s.total, what)) return rc;
  if (!m || !n) return DR_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  ProductLaunch l;
  std::memset(&l, 0, sizeof(l));
  l.b = view(*w);
  l.c = y;
  l.c_stride = y_row_stride;
  l.m = (uint32_t)m;
  l.n = (uint32_t)n;
  l.kb = (uint32_t)ceil_div(k, kBlock);
  l.c_bf16 = y_type == DR_TYPE_BF16;
  l.fast = (flags & DR_FAST_SUMS) != 0;
  if (m <= kFusedRows) {
    l.x = x;
    l.x_stride = x_row_stride;
    l.x_bf16 = x_type == DR_TYPE_BF16;
    l.a.cols = (uint32_t)k;
  } else {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const dr_qmatrix q = {ws + s.data, ws + s.scales, m, k, padded(k), 1, 0};
    if (int rc = quantize(x, x_type, m, k, x_row_stride, &q, nullptr, st, what)) return rc;
    l.a = view(q);
    l.workspace = ws + s.product;
  }
  return hip_result(launch_product(l, st), what);
}
