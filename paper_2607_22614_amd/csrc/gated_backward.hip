// The backward pass of a gated feed-forward block's inner half, from its 8-bit checkpoint (dr_gated_backward).
//
//   s = 1 / (1 + e^-z(g)),  a = g s,  act'(g) = s + a (1 - s) z'(g)
//   dgate = dh u act'(g),   dup = dh a,   h = a u
//
// One pass: a tile of 128 x 128 elements of dh, gate and up gives tiles of dgate, dup and h, each quantized along its rows
// and columns where it stands in registers.
#include <hip/hip_runtime.h>

#include "gated_device.h"
#include "quantize_tile.h"

namespace dr {
namespace {

struct BackwardArgs {
  const void* dh;
  int64_t dh_stride;
  uint32_t rows, f, tiles_x;
  Act act;
  QView gate, up, d, dt, ht;
};

struct Values8 {
  float v[8];
};
// What 8 codes and their scale stand for.
__device__ __forceinline__ Values8 f32_values(u32x2 codes, uint32_t code) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const float s = scale_operand(code);
  Values8 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 lo = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)codes[i], s, false));
    const f32x2 hi = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)codes[i], s, true));
    r.v[4 * i] = lo[0], r.v[4 * i + 1] = lo[1], r.v[4 * i + 2] = hi[0], r.v[4 * i + 3] = hi[1];
  }
  return r;
}

__device__ __forceinline__ uint32_t scale_at(const QView& q, uint32_t row, uint32_t block) {
  return q.scales[((int64_t)(block >> 2) * q.srows + row) * 4 + (block & 3)];
}

// The tile's codes along the rows into q, along the columns into qt, whichever are wanted.
__device__ __forceinline__ void put_tile(const Raw8<false> (&v)[kTileRows], const TilePlace& at, const QView& q, const QView& qt, TileSpace<true>& space) {
  if (q.data && qt.data) quantize_tile<false, false, true, true>(v, at, q, qt, space);
  else if (q.data) quantize_tile<false, false, true, false>(v, at, q, qt, space);
  else quantize_tile<false, false, false, true>(v, at, q, qt, space);
}

// f a multiple of 128: gate's and up's halves of d consist of whole tiles, and a workgroup takes one of either.
template <bool BF16>
__global__ __launch_bounds__(kTileLanes) void gated_backward_kernel(BackwardArgs a) {
  __shared__ TileSpace<true> space;
  const TilePlace at = tile_place(a.tiles_x);
  Raw8<BF16> dh[kTileRows];
  u32x2 gate[kTileRows], up[kTileRows];
  uint32_t gate_code[kTileRows], up_code[kTileRows];
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    const uint32_t row = min(at.row0 + i, a.rows - 1);
    dh[i] = load_row8<BF16>(a.dh, (int64_t)row * a.dh_stride, at.col, a.f);
    gate[i] = *reinterpret_cast<const u32x2*>(a.gate.data + (int64_t)row * a.gate.stride + at.col);
    up[i] = *reinterpret_cast<const u32x2*>(a.up.data + (int64_t)row * a.up.stride + at.col);
    gate_code[i] = scale_at(a.gate, row, at.ct);
    up_code[i] = scale_at(a.up, row, at.ct);
  }
  Raw8<false> dgate[kTileRows], dup[kTileRows], h[kTileRows];
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    const Values8 g = f32_values(gate[i], gate_code[i]), u = f32_values(up[i], up_code[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const GatedGradient r = gated_gradient(__uint_as_float(bits_of<BF16>(dh[i], j)), g.v[j], u.v[j], a.act);
      put_element(dgate[i], j, r.dgate);
      put_element(dup[i], j, r.dup);
      put_element(h[i], j, r.h);
    }
    if (at.row0 + i >= a.rows) dgate[i] = dup[i] = h[i] = Raw8<false>{};
  }
  if (a.d.data || a.dt.data) {
    put_tile(dgate, at, a.d, a.dt, space);
    TilePlace second = at;
    second.ct += a.f / 128;
    second.col += a.f;
    put_tile(dup, second, a.d, a.dt, space);
  }
  if (a.ht.data) put_tile(h, at, QView{}, a.ht, space);
}

// Any f: a workgroup takes one tile of d's 2f columns, of which one holds the end of gate's half and the beginning of up's,
// element by element.
template <bool BF16>
__global__ __launch_bounds__(kTileLanes) void gated_backward_any_kernel(BackwardArgs a) {
  __shared__ TileSpace<true> space;
  const TilePlace at = tile_place(a.tiles_x);
  Raw8<false> d[kTileRows], h[kTileRows];
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    const uint32_t row = min(at.row0 + i, a.rows - 1);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t c = at.col + j, f = min(c - (c < a.f ? 0 : a.f), a.f - 1), block = f / 128;
      const int64_t from = (int64_t)row * a.dh_stride + f;
      const float dh = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.dh)[from] << 16) : static_cast<const float*>(a.dh)[from];
      const uint32_t g = a.gate.data[(int64_t)row * a.gate.stride + f], u = a.up.data[(int64_t)row * a.up.stride + f];
      const GatedGradient r = gated_gradient(dh, f32_values(u32x2{g, 0}, scale_at(a.gate, row, block)).v[0],
                                             f32_values(u32x2{u, 0}, scale_at(a.up, row, block)).v[0], a.act);
      const bool in = at.row0 + i < a.rows;
      put_element(d[i], j, in && c < 2 * a.f ? (c < a.f ? r.dgate : r.dup) : 0.0f);
      put_element(h[i], j, in && c < a.f ? r.h : 0.0f);
    }
  }
  if (a.d.data || a.dt.data) put_tile(d, at, a.d, a.dt, space);
  if (a.ht.data && at.ct * 128 < a.f) put_tile(h, at, QView{}, a.ht, space);
}

}  // namespace

hipError_t launch_gated_backward(const GatedBackward& l, hipStream_t st) {
  const BackwardArgs a = {l.dh, l.dh_stride, l.rows, l.f, (uint32_t)backward_tiles_x(l.f), l.act, l.gate, l.up, l.d, l.dt, l.ht};
  const dim3 grid(a.tiles_x * (uint32_t)ceil_div(l.rows, 128)), block(kTileLanes);
  if (l.f % kBlock == 0) {
    if (l.dh_bf16) hipLaunchKernelGGL(gated_backward_kernel<true>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(gated_backward_kernel<false>, grid, block, 0, st, a);
  } else {
    if (l.dh_bf16) hipLaunchKernelGGL(gated_backward_any_kernel<true>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(gated_backward_any_kernel<false>, grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace dr
