// The products of a gated feed-forward block (dr_qgated, dr_qgated_save), with activation and product where their sums stand.
#include <hip/hip_runtime.h>

#include "product_device.h"

namespace dr {
namespace {

void fill_pairs(GatedArgs& a, const GatedProduct& g) {
  fill_args(a, g.product, g.product.n / 2);
  a.half = a.n;
  a.half_bytes = (int64_t)a.n * a.b.stride;
  a.b.rows = a.n;  // gate's; up's lie half_bytes behind them
  a.act = g.act;
}

}  // namespace

hipError_t launch_gated_rows(const GatedProduct& g, hipStream_t st) {
  GatedArgs a;
  fill_pairs(a, g);
  const ProductLaunch& l = g.product;
  const int size = l.c_bf16 ? 2 : 4;
  const ProductPlan plan = plan_product(l.m, l.n, l.kb, l.fast);
  if (l.x || plan.kind == ProductPlan::kDirect || l.c_stride * size >= kMaxRowBytes) {
    launch_direct_kind<kGated>(a, l.x_bf16, plan.rows16, st);
  } else {
    if (a.n * (int64_t)size % 16) a.c_vec = 0;  // whole pieces only
    if (l.c_bf16) launch_tile_kind<2, kGated>(a, plan, l.fast, st);
    else launch_tile_kind<4, kGated>(a, plan, l.fast, st);
  }
  return hipGetLastError();
}

hipError_t launch_gated_codes(const GatedProduct& g, const GatedCodesPlan& plan, hipStream_t st) {
  GatedArgs a;
  fill_pairs(a, g);
  a.hq = g.hq;
  a.gate = g.gate;
  a.up = g.up;
  const bool fast = g.product.fast;
  if (a.kb == 1) launch_tiles<128, 256, 1, true, true, kGatedCodes>(a, 0, fast, st);
  else if (plan.rows == 256) launch_tiles<256, 256, 1, true, false, kGatedCodes>(a, plan.halved, fast, st);
  else launch_tiles<128, 256, 1, true, false, kGatedCodes>(a, 0, fast, st);
  return hipGetLastError();
}

}  // namespace dr
