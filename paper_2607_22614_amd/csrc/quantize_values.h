// Quantization along rows and columns of a tile of 128 x 128 values that a workgroup has computed (gated_backward.hip) or decoded
// (turn_tile_kernel): what quantize_tile does (quantize_tile.h), where the vector units and not the memory would be the bound.
//
// Maxima go through v_max3 on magnitudes, which passes over NaN; infinities are looked for in the result, and only where there
// are any are all maxima taken again.  A scale is carried as amax's bits + 0x1FFFFF: less 8 << 23 (or 0) it is the converts'
// operand, whose exponent alone counts, and its own exponent less 8 the scale's code.
#pragma once

#include <hip/hip_runtime.h>

#include "quantize_tile.h"

namespace dr {

// The workgroup's LDS accesses before it are done; stores to memory stay on their way, which a plain barrier waits for (8192 x
// 14336 of the gated block's gradients 224 us with plain barriers).
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A lane's values: 8 columns of kTileRows rows.
struct TileValues {
  float v[kTileRows][8];
};

struct ValuesSpace {
  __align__(16) uint32_t cmax[3][128];  // of up to three matrices, zero at the start
  __align__(16) uint8_t turned[128 * 128];
};
// The workgroup's first barrier has to follow.
__device__ __forceinline__ void clear_maxima(ValuesSpace& space) {
  if (threadIdx.x < 3 * 128 / 4) reinterpret_cast<u32x4*>(space.cmax)[threadIdx.x] = u32x4{};
}

constexpr uint32_t kRoundUp = 0x1FFFFF, kEight = 8u << 23;
__device__ __forceinline__ uint32_t biased_scale(uint32_t amax) { return amax + kRoundUp; }
__device__ __forceinline__ float biased_operand(uint32_t b) { return __uint_as_float(__builtin_elementwise_sub_sat(b, kEight)); }
__device__ __forceinline__ uint32_t biased_code(uint32_t b) { return b == kRoundUp ? 127u : __builtin_elementwise_sub_sat(b, kEight) >> 23; }

// |v|, or NaN where v is not finite.
__device__ __forceinline__ float finite_magnitude(float v) { return fmaf(v, 0.0f, fabsf(v)); }
template <bool FINITE>
__device__ __forceinline__ float magnitude_of(float v) {
  return FINITE ? finite_magnitude(v) : fabsf(v);
}
template <bool FINITE>
__device__ __forceinline__ void row_maxima(const TileValues& t, float (&most)[kTileRows]) {
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    float m = magnitude_of<FINITE>(t.v[i][0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) m = fmaxf(m, magnitude_of<FINITE>(t.v[i][j]));
    most[i] = fmaxf(m, 0.0f);  // NaN alone counts as nothing
  }
}
template <bool FINITE>
__device__ __forceinline__ void column_maxima(const TileValues& t, float (&most)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float m = magnitude_of<FINITE>(t.v[0][j]);
#pragma unroll
    for (int i = 1; i < kTileRows; ++i) m = fmaxf(m, magnitude_of<FINITE>(t.v[i][j]));
    most[j] = fmaxf(m, 0.0f);
  }
}

// Addresses: a tile's first element is the same for the whole workgroup, and a lane's row of the tile times a stride of
// at most 2^23 bytes fits the 24-bit multiplication and an offset of 32 bits.
__device__ __forceinline__ uint8_t* tile_at(const QView& q, uint32_t row, uint32_t col) { return q.data + (int64_t)row * q.stride + col; }
__device__ __forceinline__ uint32_t row_offset(uint32_t row, int64_t stride) { return __umul24(row, (uint32_t)stride); }

__device__ __forceinline__ void put_rows(const TileValues& t, const TilePlace& at, const QView& q) {
  const uint32_t tx = threadIdx.x & 15, first = threadIdx.x / 16 * kTileRows;
  float most[kTileRows];
  row_maxima<false>(t, most);
  float top = most[0];
#pragma unroll
  for (int i = 1; i < kTileRows; ++i) top = fmaxf(top, most[i]);
  if (__any(__float_as_uint(top) >= kInfBits)) row_maxima<true>(t, most);
  uint8_t* to = tile_at(q, at.rt * 128, at.ct * 128);
  uint32_t mine = 0;  // of the lane's row tx
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    const uint32_t b = biased_scale(max16(__float_as_uint(most[i])));
    const float s = biased_operand(b);
    mine = tx == (uint32_t)i ? b : mine;
    const float* v = t.v[i];
    if (at.row0 + i < q.rows)
      *reinterpret_cast<u32x2*>(to + (row_offset(first + i, q.stride) + tx * 8)) =
          u32x2{to_e4m3_f32(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]), s),
                to_e4m3_f32(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]), s)};
  }
  if (tx < kTileRows && at.row0 + tx < q.rows) put_code(q, at.row0 + tx, at.ct, biased_code(mine));
}

// Two registers whose lanes 32 (or 16) apart are to meet: of a in the lower lanes, of b in the upper ones.
struct Pair {
  uint32_t a, b;
};
__device__ __forceinline__ Pair halves(uint32_t a, uint32_t b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return Pair{r[0], r[1]};
}
__device__ __forceinline__ Pair lines(uint32_t a, uint32_t b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return Pair{r[0], r[1]};
}
__device__ __forceinline__ uint32_t larger_of(Pair p) { return max(p.a, p.b); }
__device__ __forceinline__ uint32_t larger_pairs_of(Pair p) { return larger<true>(p.a, p.b); }

// The columns' codes and scales, their maxima being in the space: codes(j, operand) gives those of the lane's column j of its rows.
template <class Codes>
__device__ __forceinline__ void turn_columns(const TilePlace& at, const QView& qt, ValuesSpace& space, int which, Codes codes) {
  const uint32_t tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  lds_barrier();
  // word ty of a column lies at ty ^ 4 (tx % 8), which keeps its 16-byte pieces together
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const u32x4 most4 = *reinterpret_cast<const u32x4*>(&space.cmax[which][tx * 8 + h * 4]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<uint32_t*>(space.turned + (tx * 8 + h * 4 + e) * 128 + (ty ^ (tx % 8 * 4)) * 4) = codes(h * 4 + e, biased_operand(biased_scale(most4[e])));
  }
  const uint32_t first = at.ct * 128;
  if (tid < 128 && first + tid < qt.rows) put_code(qt, first + tid, at.rt, biased_code(biased_scale(space.cmax[which][tid])));
  lds_barrier();
  uint8_t* to = tile_at(qt, first, at.rt * 128);
#pragma unroll
  for (int r = 0; r < 128 * 8 / kTileLanes; ++r) {
    const uint32_t c = r * (kTileLanes / 8) + tid / 8, piece = tid % 8;
    const u32x4 w = *reinterpret_cast<const u32x4*>(space.turned + c * 128 + (piece ^ (c / 8 % 8)) * 16);
    if (first + c < qt.rows) *reinterpret_cast<u32x4*>(to + (row_offset(c, qt.stride) + piece * 16)) = w;
  }
}

// `which` of the space's maxima are this matrix's, still zero.
__device__ __forceinline__ void put_columns(const TileValues& t, const TilePlace& at, const QView& qt, ValuesSpace& space, int which) {
  const uint32_t tx = threadIdx.x & 15, line = threadIdx.x / 16 & 3;
  float most[8];
  column_maxima<false>(t, most);
  float top = most[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) top = fmaxf(top, most[j]);
  if (__any(__float_as_uint(top) >= kInfBits)) column_maxima<true>(t, most);
  // over the wave's four rows of lanes: columns j and j + 4 meet in a register, lower and upper lanes, then j and j + 2
  uint32_t pair[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) pair[j] = larger_of(halves(__float_as_uint(most[j]), __float_as_uint(most[j + 4])));
#pragma unroll
  for (int j = 0; j < 2; ++j)  // of column j, j + 2, j + 4, j + 6 in lines 0 to 3
    atomicMax(&space.cmax[which][tx * 8 + j + line * 2], larger_of(lines(pair[j], pair[j + 2])));
  turn_columns(at, qt, space, which, [&](int j, float scale) {
    return to_e4m3_f32(__float_as_uint(t.v[0][j]), __float_as_uint(t.v[1][j]), __float_as_uint(t.v[2][j]), __float_as_uint(t.v[3][j]), scale);
  });
}

// Of values in bf16, two of a row to a register.
__device__ __forceinline__ void put_columns(const Raw8<true> (&v)[kTileRows], const TilePlace& at, const QView& qt, ValuesSpace& space, int which) {
  const uint32_t tx = threadIdx.x & 15, line = threadIdx.x / 16 & 3;
  uint32_t most[4], top = 0;
  auto maxima = [&](bool finite) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      most[w] = magnitude<true>(v[0].w[0][w], finite);
#pragma unroll
      for (int i = 1; i < kTileRows; ++i) most[w] = larger<true>(most[w], magnitude<true>(v[i].w[0][w], finite));
    }
  };
  maxima(false);
#pragma unroll
  for (int w = 0; w < 4; ++w) top = larger<true>(top, most[w]);
  if (__any(unpack_max<true>(top) >= kInfBits)) maxima(true);
  // columns 2 w and 2 w + 1 and those 4 further on meet in a register, then those 2 further on: 2 line and 2 line + 1 in the end
  const uint32_t m = larger_pairs_of(lines(larger_pairs_of(halves(most[0], most[2])), larger_pairs_of(halves(most[1], most[3]))));
  atomicMax(&space.cmax[which][tx * 8 + line * 2], m << 16);
  atomicMax(&space.cmax[which][tx * 8 + line * 2 + 1], m & 0xFFFF0000u);
  turn_columns(at, qt, space, which, [&](int j, float scale) {
    const uint32_t pick = j % 2 ? 0x07060302u : 0x05040100u;  // (lower, upper) halves of two rows side by side
    return to_e4m3_bf16(__builtin_amdgcn_perm(v[1].w[0][j / 2], v[0].w[0][j / 2], pick), __builtin_amdgcn_perm(v[3].w[0][j / 2], v[2].w[0][j / 2], pick), scale);
  });
}

// The tile's codes along the rows into q, along the columns into qt, whichever are wanted.  A following call's writes of the
// turned codes stand behind the barrier of its maxima, and so behind this one's reads.
__device__ __forceinline__ void put_tile(const TileValues& t, const TilePlace& at, const QView& q, const QView& qt, ValuesSpace& space, int which) {
  if (q.data) put_rows(t, at, q);
  if (qt.data) put_columns(t, at, qt, space, which);
}

}  // namespace dr
