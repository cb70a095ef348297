// The activation of the gated feed-forward block and its derivative.
#pragma once

#include <hip/hip_runtime.h>

#include "gated_kernels.h"
#include "quant_device.h"

namespace dr {

// z of act, times -log2(e).  g is cut off at 128, where the logistic function is 0 or 1 in fp32 for either activation: an infinite
// g or g^2 would make 0 * inf in z.
__device__ __forceinline__ float exponent(float g, const Act& act) {
  const float c = __builtin_amdgcn_fmed3f(g, -128.0f, 128.0f);
  return c * fmaf(c * c, act.k3, act.k1) * -1.44269504088896340736f;
}

// The exponent is rounded to fp32, so the logistic function is off by (6 + |z|) 2^-23 of itself at most, and it is 0 where e^-z
// is infinite.
__device__ __forceinline__ float gated(float gate, float up, const Act& act) {
  return gate * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(exponent(gate, act))) * up;
}

struct GatedGradient {
  float dgate, dup, h;
};
// act' = s + g s (1 - s) z', where 1 - s = e^-z s loses nothing to cancellation; the exponent is cut off at 126, past which s is
// 0, so that no infinity meets it.
__device__ __forceinline__ GatedGradient gated_gradient(float dh, float gate, float up, const Act& act) {
  const float x = exponent(gate, act), e = __builtin_amdgcn_exp2f(fminf(x, 126.0f)), s = x > 126.0f ? 0.0f : __builtin_amdgcn_rcpf(1.0f + e);
  const float c = __builtin_amdgcn_fmed3f(gate, -128.0f, 128.0f), slope = fmaf(c * c, 3.0f * act.k3, act.k1), a = gate * s;
  return GatedGradient{dh * up * fmaf(a * slope, e * s, s), dh * a, a * up};
}

__device__ __forceinline__ float element(const Raw8<false>& v, int i) { return __uint_as_float(bits_of<false>(v, i)); }
__device__ __forceinline__ void put_element(Raw8<false>& v, int i, float x) { v.w[i / 4][i % 4] = __float_as_uint(x); }

}  // namespace dr
