// Device helpers of the 8-bit and gradient kernels: scales, rounding to e4m3, loads of 8 elements.
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

// e8m0 code of the smallest power of two, at least 2^-127, by which amax (its bits) is at most 448 = 1.75 * 2^8:
// the exponent less 8, one more where the mantissa passes 1.75.  1 for amax = 0.
__device__ __forceinline__ uint32_t scale_code(uint32_t amax) {
  const int c = (int)((amax + 0x1FFFFFu) >> 23) - 8;
  return amax == 0 ? 127u : (uint32_t)max(c, 0);
}
// The scale as an operand of the converts, which look at its exponent bits only (0 is 2^-127 to them).
__device__ __forceinline__ float scale_operand(uint32_t code) { return __uint_as_float(code << 23); }

// 8 elements of a row as they lie in memory.
template <bool BF16>
struct Raw8 {
  u32x4 w[BF16 ? 1 : 2];
};

// 16 bytes at any element: the memory takes that
template <bool BF16>
struct AnyElement {
  typedef u32x4 __attribute__((aligned(4))) type;
};
template <>
struct AnyElement<true> {
  typedef u32x4 __attribute__((aligned(2))) type;
};

// Elements col .. col + 7 of the row of `cols` elements at element `row` of base, aligned to the element alone.  The last 8
// of the row stand in for those that are not all there, so that every lane loads and none branches; settle8 puts that
// right.  A row of fewer than 8 is loaded element by element, and is right at once.
// STREAM: rows of whole 16 bytes (whole_pieces), read once.
template <bool BF16, bool STREAM = false>
__device__ __forceinline__ Raw8<BF16> load_row8(const void* base, int64_t row, uint32_t col, uint32_t cols) {
  const uint8_t* p = static_cast<const uint8_t*>(base) + (row + min(col, cols - 8)) * (BF16 ? 2 : 4);
  Raw8<BF16> v;
#pragma unroll
  for (int i = 0; i < (BF16 ? 1 : 2); ++i) {
    if constexpr (STREAM) v.w[i] = load_stream(reinterpret_cast<const u32x4*>(p) + i);
    else v.w[i] = reinterpret_cast<const typename AnyElement<BF16>::type*>(p)[i];
  }
  return v;
}
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> load_short_row8(const void* base, int64_t row, uint32_t col, uint32_t cols) {
  Raw8<BF16> v = {};
#pragma unroll
  for (uint32_t i = 0; i < 7; ++i) {
    if (BF16) v.w[0][i / 2] |= col + i < cols ? (uint32_t)static_cast<const uint16_t*>(base)[row + i] << (i % 2 * 16) : 0u;
    else v.w[BF16 ? 0 : i / 4][i % 4] = col + i < cols ? static_cast<const uint32_t*>(base)[row + i] : 0u;
  }
  return v;
}
// Elements too many in front of those that load_row8 was asked for; 0 in a row of fewer than 8.
__device__ __forceinline__ uint32_t ahead8(uint32_t col, uint32_t cols) { return cols < 8 ? 0 : col - min(col, cols - 8); }
// What load_row8 gave, with s elements too many in front: the elements that are there in their places, zeros behind them.
template <bool BF16>
__device__ __forceinline__ void settle8(Raw8<BF16>& v, uint32_t s) {
  constexpr int kWords = BF16 ? 4 : 8, kPer = 8 / kWords;  // elements in a word
  uint32_t w[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i) w[i] = s < 8 ? v.w[i / 4][i % 4] : 0u;
#pragma unroll
  for (int d = kWords / 2; d; d /= 2)
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = s & (d * kPer) ? (i + d < kWords ? w[i + d] : 0u) : w[i];
  if (BF16) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = s & 1 ? w[i] >> 16 | (i + 1 < kWords ? w[i + 1] << 16 : 0u) : w[i];
  }
#pragma unroll
  for (int i = 0; i < kWords; ++i) v.w[i / 4][i % 4] = w[i];
}

// The 8 elements s places further on (s < 8), zeros in front of them.
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> delayed8(const Raw8<BF16>& v, uint32_t s) {
  constexpr int kWords = BF16 ? 4 : 8, kPer = 8 / kWords;  // elements in a word
  Raw8<BF16> r = v;
#pragma unroll
  for (int d = kWords / 2; d; d /= 2)
#pragma unroll
    for (int i = kWords - 1; i >= 0; --i) r.w[i / 4][i % 4] = s & (d * kPer) ? (i >= d ? r.w[(i - d) / 4][(i - d) % 4] : 0u) : r.w[i / 4][i % 4];
  if (BF16) {
#pragma unroll
    for (int i = kWords - 1; i >= 0; --i) r.w[i / 4][i % 4] = s & 1 ? r.w[i / 4][i % 4] << 16 | (i ? r.w[(i - 1) / 4][(i - 1) % 4] >> 16 : 0u) : r.w[i / 4][i % 4];
  }
  return r;
}

// fp32 bits of element i.
template <bool BF16>
__device__ __forceinline__ uint32_t bits_of(const Raw8<BF16>& v, int i) {
  if (!BF16) return v.w[BF16 ? 0 : i / 4][i % 4];
  const uint32_t w = v.w[0][i / 2];
  return i % 2 ? w & 0xFFFF0000u : w << 16;
}

// Magnitudes of two elements at a time for bf16 (packed 16-bit maxima), of one for fp32.  finite: those that are not
// finite count as 0.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
template <bool BF16>
__device__ __forceinline__ uint32_t magnitude(uint32_t w, bool finite) {
  if (BF16) {
    w &= 0x7FFF7FFFu;
    if (finite) {
      if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
      if ((w & 0x7F800000u) == 0x7F800000u) w &= 0xFFFFu;
    }
    return w;
  }
  w &= 0x7FFFFFFFu;
  return finite && w >= kInfBits ? 0u : w;
}
template <bool BF16>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  if (BF16) return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
  return max(a, b);
}
// Largest of the packed magnitudes, as fp32 bits.
template <bool BF16>
__device__ __forceinline__ uint32_t unpack_max(uint32_t m) {
  return BF16 ? max(m << 16, m & 0xFFFF0000u) : m;
}
template <bool BF16>
__device__ __forceinline__ uint32_t row_max(const Raw8<BF16>& v, bool finite) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < (BF16 ? 4 : 8); ++i) m = larger<BF16>(m, magnitude<BF16>(v.w[BF16 ? 0 : i / 4][i % 4], finite));
  return unpack_max<BF16>(m);
}

typedef short s16x2 __attribute__((ext_vector_type(2)));
// What two converts overwrite, one half each: no instruction sets it.
__device__ __forceinline__ s16x2 any_halves() { return __builtin_nondeterministic_value(s16x2{}); }
// Four values over the scale as e4m3 codes: the hardware converts divide by the power of two exactly, round to even and
// make NaN of what is not finite.  Values are within 448 after scaling.
__device__ __forceinline__ uint32_t to_e4m3_f32(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float scale) {
  s16x2 w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(any_halves(), __uint_as_float(a), __uint_as_float(b), scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, __uint_as_float(c), __uint_as_float(d), scale, true);
  return __builtin_bit_cast(uint32_t, w);
}
__device__ __forceinline__ uint32_t to_e4m3_bf16(uint32_t ab, uint32_t cd, float scale) {
  s16x2 w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(any_halves(), __builtin_bit_cast(bf16x2, ab), scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, cd), scale, true);
  return __builtin_bit_cast(uint32_t, w);
}

// Codes of 8 elements of a row.
template <bool BF16>
__device__ __forceinline__ u32x2 row_codes(const Raw8<BF16>& v, uint32_t code) {
  const float s = scale_operand(code);
  if (BF16) return u32x2{to_e4m3_bf16(v.w[0][0], v.w[0][1], s), to_e4m3_bf16(v.w[0][2], v.w[0][3], s)};
  const u32x4 a = v.w[0], b = v.w[BF16 ? 0 : 1];
  return u32x2{to_e4m3_f32(a[0], a[1], a[2], a[3], s), to_e4m3_f32(b[0], b[1], b[2], b[3], s)};
}

// Codes of column j of 4 rows.
template <bool BF16>
__device__ __forceinline__ uint32_t column_codes(const Raw8<BF16> (&v)[4], int j, uint32_t code) {
  const float s = scale_operand(code);
  if (BF16) {
    uint32_t pair[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)  // (lower, upper) halves of two rows side by side
      pair[i] = __builtin_amdgcn_perm(v[2 * i + 1].w[0][j / 2], v[2 * i].w[0][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
    return to_e4m3_bf16(pair[0], pair[1], s);
  }
  return to_e4m3_f32(bits_of<BF16>(v[0], j), bits_of<BF16>(v[1], j), bits_of<BF16>(v[2], j), bits_of<BF16>(v[3], j), s);
}

// What 8 codes and their scale stand for, in bf16 (exact: 4 significant bits; below 2^-133 it is 0).
__device__ __forceinline__ Raw8<true> bf16_values(u32x2 codes, uint32_t code) {
  const float s = scale_operand(code);
  Raw8<true> v;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v.w[0][2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes[i], s, false));
    v.w[0][2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes[i], s, true));
  }
  return v;
}

// What codes and their scale stand for, in fp32.
struct Values8 {
  float v[8];
};
__device__ __forceinline__ void f32_values4(uint32_t codes, float scale, float* to) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 lo = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)codes, scale, false));
  const f32x2 hi = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)codes, scale, true));
  to[0] = lo[0], to[1] = lo[1], to[2] = hi[0], to[3] = hi[1];
}
__device__ __forceinline__ Values8 f32_values(u32x2 codes, uint32_t code) {
  Values8 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) f32_values4(codes[i], scale_operand(code), r.v + 4 * i);
  return r;
}

// Sum over the wave, in every lane: within rows of 16 lanes by DPP moves, then across the rows.
template <int ctrl>
__device__ __forceinline__ float dpp_sum(float v) {
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), ctrl, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = dpp_sum<0xb1>(v);   // quad_perm [1,0,3,2]
  v = dpp_sum<0x4e>(v);   // quad_perm [2,3,0,1]
  v = dpp_sum<0x141>(v);  // row_half_mirror
  v = dpp_sum<0x140>(v);  // row_mirror
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// fp32 -> bf16, ties to even (the hardware convert).
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

}  // namespace dr
