// The activation of the gated feed-forward block and its derivative.
#pragma once

#include <hip/hip_runtime.h>

#include "gated_kernels.h"
#include "quant_device.h"

namespace dr {

// z of act, times -log2(e), which the constants hold.  g is cut off at 128, where the logistic function is 0 or 1 in fp32 for either activation: an infinite
// g or g^2 would make 0 * inf in z.
__device__ __forceinline__ float exponent(float g, const Act& act) {
  const float c = __builtin_amdgcn_fmed3f(g, -128.0f, 128.0f);
  return c * fmaf(c * c, act.n3, act.n1);
}

// The exponent is rounded to fp32, so the logistic function is off by (6 + |z|) 2^-23 of itself at most, and it is 0 where e^-z
// is infinite.
__device__ __forceinline__ float gated(float gate, float up, const Act& act) {
  return gate * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(exponent(gate, act))) * up;
}

// act, and act' = s + g s (1 - s) z'.  1 - s is off by 2^-23 at most, and so the slope by |z| 2^-21.  SILU: k1 = 1, k3 = 0, at half the
// instructions.
struct ActSlope {
  float act, slope;
};
template <bool SILU>
__device__ __forceinline__ ActSlope act_slope(float g, const Act& act) {
  if (SILU) {
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * act.n1)), a = g * s;
    return ActSlope{a, fmaf(a, 1.0f - s, s)};
  }
  const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(exponent(g, act))), a = g * s, c = __builtin_amdgcn_fmed3f(g, -128.0f, 128.0f);
  return ActSlope{a, fmaf(a * fmaf(c * c, 3.0f * act.k3, act.k1), 1.0f - s, s)};
}

__device__ __forceinline__ float element(const Raw8<false>& v, int i) { return __uint_as_float(bits_of<false>(v, i)); }
__device__ __forceinline__ void put_element(Raw8<false>& v, int i, float x) { v.w[i / 4][i % 4] = __float_as_uint(x); }

}  // namespace dr
