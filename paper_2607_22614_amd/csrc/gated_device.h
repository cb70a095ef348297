// The activation of the gated feed-forward block and its derivative.
#pragma once

#include <hip/hip_runtime.h>

#include "gated_kernels.h"
#include "quant_device.h"

namespace dr {

// 1 / (1 + e^-z).  g is cut off at 128, where that is 0 or 1 in fp32 for either activation: an infinite g or g^2 would make 0 * inf
// in z.  Each rounding of the exponent costs up to |z| 2^-24 of e^-z; what its last product loses is known, and goes into the sum
// with 1 by e^(z + d) = e^z (1 + d).  What stays is g^2, the inner sum and the constants: 1.02 |z| 2^-23 for gelu, 0.12 |z| 2^-23 for
// silu, whose inner sum is a constant.  The exponential, the reciprocal and the sums between add 3 2^-23, so that the result is
// off by (6 + |z|) 2^-23 of itself at most where e^-z is 2^126 at most, and beyond it may be 0.  With the product's loss left out
// gelu would be off by 1.5 |z| 2^-23, and 8192 rows of 3456 x 5120 would take 1.7 of 272 us less; with that of g^2 taken in too it
// would be 0.6 |z| 2^-23, and 1.8 us more.
//   SILU: k1 = 1, k3 = 0.
template <bool SILU>
__device__ __forceinline__ float logistic(float g, const Act& act) {
  const float c = __builtin_amdgcn_fmed3f(g, -128.0f, 128.0f), n = SILU ? act.n1 : fmaf(c * c, act.n3, act.n1);
  const float t = c * n, lost = fmaf(c, n, -t);  // of -z log2(e), which the constants hold
  return __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_exp2f(t), fmaf(lost, 0.693147181f, 1.0f), 1.0f));
}

__device__ __forceinline__ float gated(float gate, float up, const Act& act) { return gate * logistic<false>(gate, act) * up; }

// act, and act' = s + g s (1 - s) z'.  1 - s is off by 2^-23 at most, and so the slope by |z| 2^-21.  1 - s comes first: it is 0 for
// gates whose product with z' passes fp32.
struct ActSlope {
  float act, slope;
};
template <bool SILU>
__device__ __forceinline__ ActSlope act_slope(float g, const Act& act) {
  const float s = logistic<SILU>(g, act), a = g * s;
  if (SILU) return ActSlope{a, fmaf(a, 1.0f - s, s)};
  const float c = __builtin_amdgcn_fmed3f(g, -128.0f, 128.0f);
  return ActSlope{a, fmaf(a * (1.0f - s), fmaf(c * c, 3.0f * act.k3, act.k1), s)};
}

__device__ __forceinline__ float element(const Raw8<false>& v, int i) { return __uint_as_float(bits_of<false>(v, i)); }
__device__ __forceinline__ void put_element(Raw8<false>& v, int i, float x) { v.w[i / 4][i % 4] = __float_as_uint(x); }

}  // namespace dr
