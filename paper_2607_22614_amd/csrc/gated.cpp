// Entry points of the gated feed-forward block (dr.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "dr_internal.h"
#include "gated_kernels.h"
#include "quant_checks.h"

namespace dr {
namespace {

int check_act(int32_t act, const char* what) {
  return act == DR_ACT_SILU || act == DR_ACT_GELU_TANH ? DR_OK : fail(DR_EINVAL, "%s: unknown activation %d", what, act);
}

Act act_of(int32_t act) {
  constexpr double kMinusLog2e = -1.44269504088896340736;
  const double k1 = act == DR_ACT_SILU ? 1.0 : 2.0 * std::sqrt(2.0 / 3.14159265358979323846), k3 = act == DR_ACT_SILU ? 0.0 : 0.044715 * k1;
  return Act{(float)k1, (float)k3, (float)(kMinusLog2e * k1), (float)(kMinusLog2e * k3)};
}

// An 8-bit matrix of rows x cols in blocks of 1 x 128, as activations and gradients are.
int check_rows_matrix(const dr_qmatrix* q, int64_t rows, int64_t cols, const char* what, const char* name) {
  if (int rc = check_matrix(q, what, name)) return rc;
  if (q->rows != rows || q->cols != cols)
    return fail(DR_EINVAL, "%s: %s is %lld x %lld, not %lld x %lld", what, name, (long long)q->rows, (long long)q->cols, (long long)rows, (long long)cols);
  if (q->block_rows != 1) return fail(DR_EINVAL, "%s: %s has blocks of %d rows (1 here)", what, name, q->block_rows);
  return DR_OK;
}

// The fused weights: gate's rows, then as many of up.
int check_halves(const dr_qmatrix* w, const char* what) {
  if (int rc = check_matrix(w, what, "w")) return rc;
  return w->rows % 2 ? fail(DR_EINVAL, "%s: w has %lld rows, not gate's and as many of up", what, (long long)w->rows) : DR_OK;
}

// Where x's codes lie in the workspace of dr_qgated (none where x is quantized in the product's kernel), and behind them the
// sums of gate and up where a product's splits have to be joined.
struct GatedSpace {
  uint64_t data, scales, sums;
};
GatedSpace gated_space(int64_t m, int64_t k, bool fused) {
  if (fused) return {0, 0, 0};
  const uint64_t scales = (uint64_t)m * padded(k);
  return {0, scales, (scales + (uint64_t)ceil_div(padded(k) / kBlock, 4) * m * 4 + 15) / 16 * 16};
}
uint64_t sums_space(int64_t m, int64_t f, uint32_t splits) {
  return splits * (uint64_t)m * part_stride(2 * f) * sizeof(float) + 16;  // the join reads whole 16 bytes
}
uint64_t rows_need(int64_t m, int64_t f, int64_t k, const GatedRowsPlan& plan) {
  return gated_space(m, k, plan.fused).sums + (plan.product.splits > 1 ? sums_space(m, f, plan.product.splits) : 0);
}
// Whatever x's type.
uint64_t rows_most(int64_t m, int64_t f, int64_t k, bool fast) {
  return rows_need(m, f, k, {m <= kFusedRows, plan_product(m, 2 * f, ceil_div(k, kBlock), fast)});
}
uint64_t save_need(int64_t m, int64_t f, const GatedCodesPlan& plan) { return plan.rows ? 0 : sums_space(m, f, plan.sums.splits); }

int check_sizes(int64_t m, int64_t f, int64_t k, const char* what) {
  if (f < 0 || f > kMaxQCols) return fail(DR_EINVAL, "%s: %lld inner columns (at most 2^23)", what, (long long)f);
  if (int rc = check_shape(m, k, 1, what, "x")) return rc;
  if (int rc = check_shape(2 * f, k, 1, what, "w")) return rc;
  return check_results(m, 2 * f, what);
}

// What either kind of sums needs, whichever the caller asks for.
template <class Need>
int workspace_of(int64_t m, int64_t f, int64_t k, uint64_t* bytes, const char* what, Need need) {
  if (!bytes) return fail(DR_EINVAL, "%s: null argument", what);
  if (int rc = check_sizes(m, f, k, what)) return rc;
  *bytes = m && f ? std::max(need(false), need(true)) : 0;
  return DR_OK;
}

ProductLaunch product_with(const dr_qmatrix& w, int64_t m, bool fast) {
  ProductLaunch l;
  std::memset(&l, 0, sizeof(l));
  l.b = view(w);
  l.m = (uint32_t)m;
  l.n = (uint32_t)w.rows;
  l.kb = (uint32_t)ceil_div(w.cols, kBlock);
  l.fast = fast;
  return l;
}

// The product's sums, and the join of their halves into what j holds.
int product_and_join(ProductLaunch l, GatedJoin& j, uint8_t* sums, Act act, hipStream_t st, const char* what) {
  l.c = l.workspace = sums;
  l.c_stride = part_stride(l.n);
  l.c_bf16 = false;
  l.sums = true;
  if (int rc = hip_result(launch_product(l, st), what)) return rc;
  j.sums = reinterpret_cast<const float*>(sums);
  j.stride = l.c_stride;
  j.split_stride = l.m * l.c_stride;
  j.m = l.m;
  j.f = l.n / 2;
  j.splits = l.plan->splits;
  j.act = act;
  return hip_result(launch_gated_join(j, st), what);
}

}  // namespace

// Beyond kFusedRows rows of x a launch of its own quantizes them, which takes 2 us between others and, with the host's calls for
// two launches, 8.5 at least; in the product's kernel, where every workgroup quantizes what it reads, x costs 1.5 and a tenth
// of the product, in fp32 1.8 and seven tenths.  In us, apart / in the product's kernel, launched by the host: 333 x 344 x 256
// fp32 9.0 / 7.3, bf16 9.0 / 6.5; 100 x 1000 x 1000 8.7 / 7.0; 32 x 4864 x 896 8.9 / 7.6; 61 x 4864 x 896 10.5 / 10.9; 20 x 3584 x
// 4096 13.1 / 13.2; 40 x 2000 x 2000 9.2 / 9.9 (profiles/gated_plans.txt: 32 shapes, the choice at most 2 % above the better one).
// With 64 instead of 32 rows a workgroup the latter lose 10 to 50 %.
GatedRowsPlan plan_gated_rows(int64_t m, int64_t f, int64_t k, bool x_bf16, bool fast) {
  const int64_t kb = ceil_div(k, kBlock);
  const GatedRowsPlan plan{m <= kFusedRows, plan_product(m, 2 * f, kb, fast)};
  if (plan.fused || k < 8) return plan;
  const double direct = direct_us(m, 2 * f, kb, 2), inside = x_bf16 ? 1.1 * direct + 1.5 : 1.7 * direct + 1.8;
  const double apart = std::max((m <= 32 ? direct : plan.product.us) + 2, 8.5);
  return inside < apart ? GatedRowsPlan{true, {ProductPlan::kDirect, 1, 0, 2, inside}} : plan;
}

// Times in us as plan_product's: a step of a tile of 256 rows takes 1.34 (exact sums 2.7), of 128 rows, alone on its CU,
// 0.85 (1.5); what a tile costs beside its steps is 12 and 7, the codes' part of it included; a second launch 6.  As a product
// with fp32 sums: that product, a launch of 4, and the sums' and results' 20 bytes an element of h and split at 6.5 TB/s.  In us,
// by sums / 128 / 256 rows a tile: 200 x 688 x 256 7.7 / 10.4 / 15.8; 700 x 4864 x 896 27 / 17 / 23; 512 x 3456 x 5120 33 / 49 / 64;
// 2048 x 3456 x 5120 99 / 124 / 83 (profiles/gated_plans.txt: 20 shapes, the choice at most 2 % above the best way).
GatedCodesPlan plan_gated_codes(int64_t m, int64_t f, int64_t kb, bool fast) {
  const ProductPlan sums = plan_product(m, 2 * f, kb, fast);
  if (m <= 32 || !kb) return {0, 0, sums};
  constexpr double kCus = 256;
  const double step256 = fast ? 1.34 : 2.7, step128 = fast ? 0.85 : 1.5, start256 = 12, start128 = 7;
  GatedCodesPlan best{0, 0, sums};
  double least = sums.us + 4 + 20.0 * sums.splits * (double)m * (double)f / 6.5e6;
  auto consider = [&](double us, GatedCodesPlan plan) {
    if (us < least) least = us, best = plan;
  };
  const double columns = (double)ceil_div(f, 128), lone = (double)kb * step128 + start128, round = (double)kb * step256 + start256;
  consider(std::ceil(columns * (double)ceil_div(m, 128) / kCus) * lone, {128, 0, sums});
  if (kb < 2) return best;
  const double tiles = columns * (double)ceil_div(m, 256), rounds = std::ceil(tiles / kCus), rest = tiles - kCus * (rounds - 1);
  consider(rounds * round, {256, 0, sums});
  if (rounds > 1 && rest < kCus) consider((rounds - 1) * round + 6 + std::ceil(2 * rest / kCus) * lone, {256, (uint32_t)rest, sums});
  return best;
}
}  // namespace dr

using namespace dr;

extern "C" int dr_qgated_workspace(int64_t m, int64_t f, int64_t k, uint64_t* bytes) {
  clear_error();
  return workspace_of(m, f, k, bytes, "dr_qgated_workspace",
                      [=](bool fast) { return rows_most(m, f, k, fast); });
}

extern "C" int dr_qgated_save_workspace(int64_t m, int64_t f, int64_t k, uint64_t* bytes) {
  clear_error();
  return workspace_of(m, f, k, bytes, "dr_qgated_save_workspace",
                      [=](bool fast) { return save_need(m, f, plan_gated_codes(m, f, ceil_div(k, kBlock), fast)); });
}

extern "C" int dr_qgated(const void* x, int32_t x_type, int64_t m, int64_t x_row_stride, const dr_qmatrix* w, int32_t act, void* h, int32_t h_type,
                         int64_t h_row_stride, int32_t flags, void* workspace, uint64_t workspace_bytes, void* stream) {
  clear_error();
  const char* what = "dr_qgated";
  if (int rc = check_halves(w, what)) return rc;
  const int64_t k = w->cols, f = w->rows / 2;
  if (int rc = check_act(act, what)) return rc;
  if (int rc = check_shape(m, k, 1, what, "x")) return rc;
  if (int rc = check_dense(x, x_type, m, k, x_row_stride, what, "x")) return rc;
  if (int rc = check_dense(h, h_type, m, f, h_row_stride, what, "h")) return rc;
  if (flags & ~DR_FAST_SUMS) return fail(DR_EINVAL, "%s: unknown flags %d", what, flags);
  if (int rc = check_sizes(m, f, k, what)) return rc;
  if (!m || !f) return DR_OK;
  ProductLaunch l = product_with(*w, m, (flags & DR_FAST_SUMS) != 0);
  const GatedRowsPlan plan = plan_gated_rows(m, f, k, x_type == DR_TYPE_BF16, l.fast);
  if (int rc = check_workspace(workspace, workspace_bytes, rows_need(m, f, k, plan), what)) return rc;
  l.plan = &plan.product;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const GatedSpace s = gated_space(m, k, plan.fused);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (plan.fused) {
    l.x = x;
    l.x_stride = x_row_stride;
    l.x_bf16 = x_type == DR_TYPE_BF16;
    l.a.cols = (uint32_t)k;
  } else {
    const dr_qmatrix q = {ws + s.data, ws + s.scales, m, k, padded(k), 1, 0};
    if (int rc = quantize_checked(x, x_type, m, k, x_row_stride, &q, nullptr, st, what)) return rc;
    l.a = view(q);
  }
  l.c = h;
  l.c_stride = h_row_stride;
  l.c_bf16 = h_type == DR_TYPE_BF16;
  if (plan.product.splits == 1) {
    GatedProduct g;
    std::memset(&g, 0, sizeof(g));
    g.product = l;
    g.act = act_of(act);
    return hip_result(launch_gated_rows(g, st), what);
  }
  GatedJoin j;
  std::memset(&j, 0, sizeof(j));
  j.h = h;
  j.h_stride = h_row_stride;
  j.h_bf16 = h_type == DR_TYPE_BF16;
  return product_and_join(l, j, ws + s.sums, act_of(act), st, what);
}

extern "C" int dr_qgated_save(const dr_qmatrix* x, const dr_qmatrix* w, int32_t act, const dr_qmatrix* h, const dr_qmatrix* gate, const dr_qmatrix* up,
                              int32_t flags, void* workspace, uint64_t workspace_bytes, void* stream) {
  clear_error();
  const char* what = "dr_qgated_save";
  if (int rc = check_matrix(x, what, "x")) return rc;
  if (int rc = check_halves(w, what)) return rc;
  const int64_t m = x->rows, k = w->cols, f = w->rows / 2;
  if (x->cols != k) return fail(DR_EINVAL, "%s: x has %lld columns, w %lld", what, (long long)x->cols, (long long)k);
  if (int rc = check_act(act, what)) return rc;
  if (int rc = check_rows_matrix(h, m, f, what, "h")) return rc;
  if (!gate != !up) return fail(DR_EINVAL, "%s: one of gate and up without the other", what);
  if (gate) {
    if (int rc = check_rows_matrix(gate, m, f, what, "gate")) return rc;
    if (int rc = check_rows_matrix(up, m, f, what, "up")) return rc;
  }
  if (flags & ~DR_FAST_SUMS) return fail(DR_EINVAL, "%s: unknown flags %d", what, flags);
  if (int rc = check_sizes(m, f, k, what)) return rc;
  if (!m || !f) return DR_OK;
  ProductLaunch l = product_with(*w, m, (flags & DR_FAST_SUMS) != 0);
  const GatedCodesPlan plan = plan_gated_codes(m, f, l.kb, l.fast);
  if (int rc = check_workspace(workspace, workspace_bytes, save_need(m, f, plan), what)) return rc;
  l.plan = &plan.sums;
  hipStream_t st = static_cast<hipStream_t>(stream);
  l.a = view(*x);
  if (plan.rows) {
    GatedProduct g;
    std::memset(&g, 0, sizeof(g));
    g.product = l;
    g.act = act_of(act);
    g.hq = view(*h);
    if (gate) {
      g.gate = view(*gate);
      g.up = view(*up);
    }
    return hip_result(launch_gated_codes(g, plan, st), what);
  }
  GatedJoin j;
  std::memset(&j, 0, sizeof(j));
  j.hq = view(*h);
  if (gate) {
    j.gate = view(*gate);
    j.up = view(*up);
  }
  return product_and_join(l, j, static_cast<uint8_t*>(workspace), act_of(act), st, what);
}

extern "C" int dr_gated_backward(const void* dh, int32_t dh_type, int64_t dh_row_stride, const dr_qmatrix* gate, const dr_qmatrix* up, int32_t act,
                                 const dr_qmatrix* d, const dr_qmatrix* dt, const dr_qmatrix* ht, void* stream) {
  clear_error();
  const char* what = "dr_gated_backward";
  if (int rc = check_matrix(gate, what, "gate")) return rc;
  const int64_t m = gate->rows, f = gate->cols;
  if (int rc = check_rows_matrix(gate, m, f, what, "gate")) return rc;
  if (int rc = check_rows_matrix(up, m, f, what, "up")) return rc;
  if (int rc = check_act(act, what)) return rc;
  if (int rc = check_dense(dh, dh_type, m, f, dh_row_stride, what, "dh")) return rc;
  if (!d && !dt && !ht) return fail(DR_EINVAL, "%s: none of d, dt and ht given", what);
  if (d) {
    if (int rc = check_rows_matrix(d, m, 2 * f, what, "d")) return rc;
  }
  if (dt) {
    if (int rc = check_rows_matrix(dt, 2 * f, m, what, "dt")) return rc;
  }
  if (ht) {
    if (int rc = check_rows_matrix(ht, f, m, what, "ht")) return rc;
  }
  const int64_t tiles = ceil_div(2 * f, kBlock) * ceil_div(m, kBlock);
  if (tiles > max_workgroups(kTileLanes)) return fail(DR_EINVAL, "%s: %lld x %lld is 2^23 or more tiles", what, (long long)m, (long long)f);
  if (!m || !f) return DR_OK;
  GatedBackward l;
  std::memset(&l, 0, sizeof(l));
  l.dh = dh;
  l.dh_stride = dh_row_stride;
  l.dh_bf16 = dh_type == DR_TYPE_BF16;
  l.rows = (uint32_t)m;
  l.f = (uint32_t)f;
  l.act = act_of(act);
  l.gate = view(*gate);
  l.up = view(*up);
  if (d) l.d = view(*d);
  if (dt) l.dt = view(*dt);
  if (ht) l.ht = view(*ht);
  return hip_result(launch_gated_backward(l, static_cast<hipStream_t>(stream)), what);
}

extern "C" int dr_qtranspose(const dr_qmatrix* src, const dr_qmatrix* qt, void* stream) {
  clear_error();
  const char* what = "dr_qtranspose";
  if (int rc = check_matrix(src, what, "src")) return rc;
  if (int rc = check_rows_matrix(qt, src->cols, src->rows, what, "qt")) return rc;
  const int64_t tiles = ceil_div(src->rows, kBlock) * ceil_div(src->cols, kBlock);
  if (tiles > max_workgroups(kTileLanes))
    return fail(DR_EINVAL, "%s: %lld x %lld is 2^23 or more tiles", what, (long long)src->rows, (long long)src->cols);
  if (!src->rows || !src->cols) return DR_OK;
  return hip_result(launch_turn(view(*src), view(*qt), static_cast<hipStream_t>(stream)), what);
}
