// Launches of the gated feed-forward kernels (gated.hip, gated_backward.hip): plain arguments, checked by the host code that
// fills them (gated.cpp).  Each wrapper enqueues on `st` and returns hipGetLastError().
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "quant_kernels.h"

namespace dr {

// act(g) = g / (1 + exp(-z)) with z = g (k1 + k3 g^2): silu with k1 = 1, k3 = 0; the tanh form of gelu, 0.5 g (1 + tanh(z / 2)),
// with k1 = 2 sqrt(2 / pi), k3 = 0.044715 k1.
struct Act {
  float k1, k3;
  float n1, n3;  // times -log2(e): e^-z = 2^(g (n1 + n3 g^2))
};

// The product with the fused weights (b: gate's rows, then up's; n: all of them), with act(gate) * up in place of its sums.
struct GatedProduct {
  ProductLaunch product;
  Act act;
  QView hq, gate, up;  // of launch_gated_codes; gate and up: data null: not wanted
};
// Into rows of c, m x n / 2, by product.plan, which has no splits.
hipError_t launch_gated_rows(const GatedProduct& g, hipStream_t st);
//   fused: x is quantized in the product's kernel (whose plan's rows16 is 1 or 2).
struct GatedRowsPlan {
  bool fused;
  ProductPlan product;
};
GatedRowsPlan plan_gated_rows(int64_t m, int64_t f, int64_t k, bool x_bf16, bool fast);
// Into 8 bits: tiles of 256 or 128 rows by 128 columns, of which the last `halved` ones of 256 rows are cut into two each.
//   rows 0: as a product of fp32 sums, by `sums`, and their join.
struct GatedCodesPlan {
  uint32_t rows, halved;
  ProductPlan sums;
};
GatedCodesPlan plan_gated_codes(int64_t m, int64_t f, int64_t kb, bool fast);
hipError_t launch_gated_codes(const GatedProduct& g, const GatedCodesPlan& plan, hipStream_t st);

// h = act(gate) * up where a product's sums hold gate in columns [0, f) and up in [f, 2f): `splits` parts, split_stride
// elements apart, are added in their order.  Readable are 4 elements behind the last part.
struct GatedJoin {
  const float* sums;
  int64_t stride, split_stride;  // elements
  uint32_t m, f, splits;
  Act act;
  void* h;           // set: rows of bf16 or fp32
  int64_t h_stride;  // elements
  bool h_bf16;
  QView hq, gate, up;  // h null: 8 bits; gate and up: data null: not wanted
};
hipError_t launch_gated_join(const GatedJoin& l, hipStream_t st);

// d = [dgate dup] and its transpose, and h^T, from dh and the checkpoint; data null: not wanted.
struct GatedBackward {
  const void* dh;
  int64_t dh_stride;  // elements
  bool dh_bf16;
  uint32_t rows, f;
  Act act;
  QView gate, up, d, dt, ht;
};
hipError_t launch_gated_backward(const GatedBackward& l, hipStream_t st);

}  // namespace dr
