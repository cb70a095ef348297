// The backward pass of a gated feed-forward block's inner half, from its 8-bit checkpoint (dr_gated_backward).
//
//   s = 1 / (1 + e^-z(g)),  a = g s,  act'(g) = s + a (1 - s) z'(g)
//   dgate = dh u act'(g),   dup = dh a,   h = a u
//
// One pass: a tile of 128 x 128 elements of dh, gate and up gives tiles of dgate, dup and h, each quantized along its rows
// and columns where it stands in registers.
#include <hip/hip_runtime.h>

#include "gated_device.h"
#include "quantize_values.h"

namespace dr {
namespace {

struct BackwardArgs {
  const void* dh;
  int64_t dh_stride;
  uint32_t rows, f, tiles_x;
  Act act;
  QView gate, up, d, dt, ht;
};

__device__ __forceinline__ uint32_t scale_at(const QView& q, uint32_t row, uint32_t block) {
  return q.scales[((int64_t)(block >> 2) * q.srows + row) * 4 + (block & 3)];
}

// Holds what is computed from v behind this place.
__device__ __forceinline__ void pin(TileValues& t) {
#pragma unroll
  for (int i = 0; i < kTileRows; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(t.v[i][j]));
}

// f a multiple of 128: gate's and up's halves of d consist of whole tiles, and a workgroup takes one of either.  dup and h are
// computed when dgate has left: all three at once would take the registers of a second workgroup.
template <bool BF16, bool SILU>
__global__ __launch_bounds__(kTileLanes, 4) void gated_backward_kernel(BackwardArgs p) {
  __shared__ ValuesSpace space;
  const TilePlace at = tile_place(p.tiles_x);
  clear_maxima(space);
  Raw8<BF16> dh[kTileRows];
  u32x2 gate[kTileRows], up[kTileRows];
  uint32_t gate_code[kTileRows], up_code[kTileRows];
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    const uint32_t row = min(at.row0 + i, p.rows - 1);
    dh[i] = load_row8<BF16>(p.dh, (int64_t)row * p.dh_stride, at.col, p.f);
    gate[i] = *reinterpret_cast<const u32x2*>(p.gate.data + (int64_t)row * p.gate.stride + at.col);
    up[i] = *reinterpret_cast<const u32x2*>(p.up.data + (int64_t)row * p.up.stride + at.col);
    gate_code[i] = scale_at(p.gate, row, at.ct);
    up_code[i] = scale_at(p.up, row, at.ct);
  }
  __syncthreads();
  TileValues a, t;
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    const Values8 g = f32_values(gate[i], gate_code[i]), u = f32_values(up[i], up_code[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const ActSlope r = act_slope<SILU>(g.v[j], p.act);
      a.v[i][j] = r.act;
      t.v[i][j] = __uint_as_float(bits_of<BF16>(dh[i], j)) * u.v[j] * r.slope;
    }
    if (at.row0 + i >= p.rows) {
#pragma unroll
      for (int j = 0; j < 8; ++j) a.v[i][j] = t.v[i][j] = 0.0f;
      dh[i] = Raw8<BF16>{};
      up[i] = u32x2{};
    }
  }
  if (p.d.data || p.dt.data) {
    put_tile(t, at, p.d, p.dt, space, 0);
    pin(a);
#pragma unroll
    for (int i = 0; i < kTileRows; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) t.v[i][j] = __uint_as_float(bits_of<BF16>(dh[i], j)) * a.v[i][j];
    TilePlace second = at;
    second.ct += p.f / 128;
    second.col += p.f;
    put_tile(t, second, p.d, p.dt, space, 1);
  }
  if (p.ht.data) {
    pin(a);
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
      const Values8 u = f32_values(up[i], up_code[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) t.v[i][j] = a.v[i][j] * u.v[j];
    }
    put_columns(t, at, p.ht, space, 2);
  }
}

// 8 codes of a row from column f on, at any byte: as load_row8 and settle8, for rows of 8 and more.
__device__ __forceinline__ u32x2 load_codes8(const QView& q, uint32_t row, uint32_t f) {
  typedef uint64_t __attribute__((aligned(1))) AnyU64;
  const uint32_t ahead = ahead8(f, q.cols);
  const uint64_t w = *reinterpret_cast<const AnyU64*>(q.data + (int64_t)row * q.stride + min(f, q.cols - 8));
  return __builtin_bit_cast(u32x2, ahead < 8 ? w >> 8 * ahead : 0ull);
}

// Any f: a workgroup takes one tile of d's 2f columns.  A lane's 8 columns begin anywhere in a block of gate or up, so that
// they may have two scales; those with the end of gate's half and the beginning of up's, and rows of fewer than 8, are read
// one by one.
template <bool BF16>
__global__ __launch_bounds__(kTileLanes) void gated_backward_any_kernel(BackwardArgs p) {
  __shared__ ValuesSpace space;
  const TilePlace at = tile_place(p.tiles_x);
  clear_maxima(space);
  const bool of_up = at.col >= p.f, single = p.f < 8 || (!of_up && at.col + 8 > p.f);
  const uint32_t f = at.col - (of_up ? p.f : 0), block = min(f, p.f - 1) / 128, last = min(f + 7, p.f - 1) / 128;
  const uint32_t first = 128 - f % 128;  // columns of the first scale
  Raw8<BF16> dh[kTileRows] = {};
  u32x2 gate[kTileRows] = {}, up[kTileRows] = {};
  uint32_t gate_code[kTileRows][2], up_code[kTileRows][2];
  if (!single) {
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
      const uint32_t row = min(at.row0 + i, p.rows - 1);
      dh[i] = load_row8<BF16>(p.dh, (int64_t)row * p.dh_stride, f, p.f);
      gate[i] = load_codes8(p.gate, row, f);
      up[i] = load_codes8(p.up, row, f);
      gate_code[i][0] = scale_at(p.gate, row, block), gate_code[i][1] = scale_at(p.gate, row, last);
      up_code[i][0] = scale_at(p.up, row, block), up_code[i][1] = scale_at(p.up, row, last);
    }
  }
  __syncthreads();
  TileValues d, h;
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    float dhs[8], gs[8], us[8];
    if (single) {
      const uint32_t row = min(at.row0 + i, p.rows - 1);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = at.col + j, one = min(c - (c < p.f ? 0 : p.f), p.f - 1);
        const int64_t from = (int64_t)row * p.dh_stride + one;
        dhs[j] = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p.dh)[from] << 16) : static_cast<const float*>(p.dh)[from];
        gs[j] = f32_values(u32x2{p.gate.data[(int64_t)row * p.gate.stride + one], 0}, scale_at(p.gate, row, one / 128)).v[0];
        us[j] = f32_values(u32x2{p.up.data[(int64_t)row * p.up.stride + one], 0}, scale_at(p.up, row, one / 128)).v[0];
      }
    } else {
      settle8(dh[i], ahead8(f, p.f));
      const Values8 g0 = f32_values(gate[i], gate_code[i][0]), g1 = f32_values(gate[i], gate_code[i][1]);
      const Values8 u0 = f32_values(up[i], up_code[i][0]), u1 = f32_values(up[i], up_code[i][1]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dhs[j] = __uint_as_float(bits_of<BF16>(dh[i], j));
        gs[j] = (uint32_t)j < first ? g0.v[j] : g1.v[j];
        us[j] = (uint32_t)j < first ? u0.v[j] : u1.v[j];
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t c = at.col + j;
      const bool in = at.row0 + i < p.rows;
      const ActSlope r = act_slope<false>(gs[j], p.act);
      d.v[i][j] = in && c < 2 * p.f ? (c < p.f ? dhs[j] * us[j] * r.slope : dhs[j] * r.act) : 0.0f;
      h.v[i][j] = in && c < p.f ? r.act * us[j] : 0.0f;
    }
  }
  put_tile(d, at, p.d, p.dt, space, 0);
  if (p.ht.data && at.ct * 128 < p.f) put_columns(h, at, p.ht, space, 2);
}

}  // namespace

hipError_t launch_gated_backward(const GatedBackward& l, hipStream_t st) {
  const BackwardArgs a = {l.dh, l.dh_stride, l.rows, l.f, (uint32_t)backward_tiles_x(l.f), l.act, l.gate, l.up, l.d, l.dt, l.ht};
  const dim3 grid(a.tiles_x * (uint32_t)ceil_div(l.rows, 128)), block(kTileLanes);
  const bool silu = l.act.k3 == 0;
  if (l.f % kBlock == 0) {
    if (l.dh_bf16 && silu) hipLaunchKernelGGL((gated_backward_kernel<true, true>), grid, block, 0, st, a);
    else if (l.dh_bf16) hipLaunchKernelGGL((gated_backward_kernel<true, false>), grid, block, 0, st, a);
    else if (silu) hipLaunchKernelGGL((gated_backward_kernel<false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((gated_backward_kernel<false, false>), grid, block, 0, st, a);
  } else {
    if (l.dh_bf16) hipLaunchKernelGGL(gated_backward_any_kernel<true>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(gated_backward_any_kernel<false>, grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace dr
