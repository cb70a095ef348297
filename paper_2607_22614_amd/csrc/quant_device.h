// Device helpers of the 8-bit kernels: scales, rounding to e4m3, loads of 8 elements.
#pragma once

#include <hip/hip_runtime.h>

#include "device_common.h"
#include "quant_kernels.h"

namespace dr {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kInfBits = 0x7F800000u;

// The other lanes' largest v within each row of 16 lanes, by DPP moves (quads, the two quads of a
// half row, the two halves).
template <int ctrl>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false));
}
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = dpp_max<0xb1>(v);    // quad_perm [1,0,3,2]
  v = dpp_max<0x4e>(v);    // quad_perm [2,3,0,1]
  v = dpp_max<0x141>(v);   // row_half_mirror
  return dpp_max<0x140>(v);  // row_mirror
}
// ... and across the four rows of a wave.
__device__ __forceinline__ uint32_t max_rows(uint32_t v) {
  v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  return max(v, (uint32_t)__shfl_xor((int)v, 32));
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// |v| as bits, 0 where v is not finite.
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t u = abs_bits(v);
  return u < kInfBits ? u : 0u;
}

// e8m0 code of the smallest power of two, at least 2^-127, by which amax is at most 448 = 1.75 * 2^8:
// the exponent less 8, one more where the mantissa passes 1.75.  1 for amax = 0.
__device__ __forceinline__ uint32_t scale_code(uint32_t amax) {
  const int c = (int)((amax + 0x1FFFFFu) >> 23) - 8;
  return amax == 0 ? 127u : (uint32_t)max(c, 0);
}
// 2^(127 - code), the factor that divides by the scale: exact, since code is at most 247.
__device__ __forceinline__ float inverse_scale(uint32_t code) { return __uint_as_float((254u - code) << 23); }

// Four values times `inv` as e4m3 codes, rounded to even by the hardware convert.  Values are within
// 448 after scaling; CHECK: some may not be finite, and those become NaN.
template <bool CHECK>
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d, float inv) {
  if (CHECK) {
    const float nan = __uint_as_float(0x7FC00000u);
    a = abs_bits(a) < kInfBits ? a : nan;
    b = abs_bits(b) < kInfBits ? b : nan;
    c = abs_bits(c) < kInfBits ? c : nan;
    d = abs_bits(d) < kInfBits ? d : nan;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}

// Elements [0, n) of the 8 at p, n <= 8; the others are 0.  vec: 16-byte loads where all 8 are there.
template <bool BF16>
__device__ __forceinline__ void load8(const void* base, int64_t at, int n, bool vec, float (&v)[8]) {
  if (BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    if (vec && n >= 8) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? __uint_as_float((uint32_t)p[i] << 16) : 0.f;
    }
  } else {
    const float* p = static_cast<const float*>(base) + at;
    if (vec && n >= 8) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[4 + i] = b[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
    }
  }
}

// fp32 -> bf16, ties to even (the hardware convert).
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

// Elements [0, n) of v to the 8 at `at`, n <= 8.  vec: 16-byte stores where all 8 are there.
template <bool BF16>
__device__ __forceinline__ void store8(void* base, int64_t at, int n, bool vec, const float (&v)[8]) {
  if (BF16) {
    uint16_t* p = static_cast<uint16_t*>(base) + at;
    const u32x4 w = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    if (vec && n >= 8) {
      *reinterpret_cast<u32x4*>(p) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
    }
  } else {
    float* p = static_cast<float*>(base) + at;
    if (vec && n >= 8) {
      *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = v[i];
    }
  }
}

}  // namespace dr
