// Products of 8-bit matrices (dr_qmatmul, dr_qlinear): the launches, and the joining of splits.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "product_device.h"

namespace dr {
namespace {

// c from the sums of the splits, in their order; a lane takes four columns.
__global__ __launch_bounds__(256) void join_splits_kernel(ProductArgs p) {
  const uint32_t groups = (uint32_t)(p.part_stride / 4);
  const uint64_t n = (uint64_t)p.m * groups;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
    const uint32_t m = (uint32_t)(i / groups), n0 = (uint32_t)(i % groups) * 4;
    const float* part = p.part + (int64_t)m * p.part_stride + n0;
    f32x4 s = *reinterpret_cast<const f32x4*>(part);
    for (uint32_t k = 1; k < p.splits; ++k) s += *reinterpret_cast<const f32x4*>(part + (int64_t)k * p.m * p.part_stride);
    store4(p, m, n0, s);
  }
}

// sums: the splits' sums stay in the workspace, unjoined, those of a single one too.
void launch_tile(const ProductArgs& a, const ProductPlan& plan, bool fast, bool sums, hipStream_t st) {
  if (a.splits == 1 && !sums) {
    if (a.c_bf16) launch_tile_kind<2, kSums>(a, plan, fast, st);
    else launch_tile_kind<4, kSums>(a, plan, fast, st);
    return;
  }
  ProductArgs parts = a;
  parts.c = a.part;
  parts.c_stride = a.part_stride;
  parts.split_bytes = (int64_t)a.m * a.part_stride * (int64_t)sizeof(float);
  parts.c_vec = 1;
  parts.n = (uint32_t)a.part_stride;  // columns past b's last one: sums of zeros
  parts.accumulate = 0;
  launch_tile_kind<4, kSums>(parts, plan, fast, st);
  if (sums) return;
  hipLaunchKernelGGL(join_splits_kernel, dim3((uint32_t)std::min<int64_t>(2048, ceil_div(a.m * (a.part_stride / 4), 256))), dim3(256), 0, st, a);
}

}  // namespace

hipError_t launch_product(const ProductLaunch& l, hipStream_t st) {
  ProductArgs a;
  fill_args(a, l, l.n);
  const int size = l.c_bf16 ? 2 : 4;
  const ProductPlan plan = l.plan ? *l.plan : plan_product(l.m, l.n, l.kb, l.fast);
  if (l.x || plan.kind == ProductPlan::kDirect || l.c_stride * size >= kMaxRowBytes) {
    launch_direct_kind<kSums>(a, l.x_bf16, plan.rows16, st);
  } else {
    a.splits = plan.splits;
    if (l.n * (int64_t)size % 16) a.c_vec = 0;  // whole pieces only
    a.part = static_cast<float*>(l.workspace);
    a.part_stride = part_stride(l.n);
    launch_tile(a, plan, l.fast, l.sums, st);
  }
  return hipGetLastError();
}

}  // namespace dr
