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

// Bands of sixteen tiles down, a contiguous eighth of them to each XCD: 8192 x 14336 in 218 us, in the order of dr_quantize's
// tiles 226 (bands of 8 and 32: 229, 219).
__device__ __forceinline__ TilePlace backward_place(uint32_t tiles_x) { return place_of<16>(xcd_tile(blockIdx.x, gridDim.x), tiles_x); }

struct BackwardArgs {
  const void* dh;
  int64_t dh_stride;
  uint32_t rows, f, tiles_x;
  int32_t stream;
  Act act;
  QView gate, up, d, dt, ht;
};

__device__ __forceinline__ uint32_t scale_at(const QView& q, uint32_t row, uint32_t block) {
  return q.scales[((int64_t)(block >> 2) * q.srows + row) * 4 + (block & 3)];
}

// What is computed from these is computed behind this place, and not kept from before it.
__device__ __forceinline__ void pin(TileValues& t) {
#pragma unroll
  for (int i = 0; i < kTileRows; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(t.v[i][j]));
}
template <int N>
__device__ __forceinline__ void pin(u32x2 (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(w[i]));
}
template <bool BF16, int N>
__device__ __forceinline__ void pin(Raw8<BF16> (&r)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int h = 0; h < (BF16 ? 1 : 2); ++h) asm volatile("" : "+v"(r[i].w[h]));
}

// f a multiple of 128, rows of dh less than 2^24 bytes apart: gate's and up's halves of d consist of whole tiles, and a workgroup takes one of either.  dup and h are
// computed when dgate has left: all three at once would take the registers of a second workgroup.
template <bool BF16, bool SILU>
__global__ __launch_bounds__(kTileLanes, 4) void gated_backward_kernel(BackwardArgs p) {
  __shared__ ValuesSpace space;
  const TilePlace at = backward_place(p.tiles_x);
  clear_maxima(space);
  const uint32_t first = threadIdx.x / 16 * kTileRows, behind = p.rows - at.rt * 128;  // the lane's first row, of those of the tile
  const uint32_t col = threadIdx.x % 16 * 8;
  const uint8_t* gates = tile_at(p.gate, at.rt * 128, at.ct * 128);
  const uint8_t* ups = tile_at(p.up, at.rt * 128, at.ct * 128);
  const uint8_t* dhs = static_cast<const uint8_t*>(p.dh) + ((int64_t)at.rt * 128 * p.dh_stride + at.ct * 128) * (BF16 ? 2 : 4);
  const uint8_t* gate_codes = p.gate.scales + ((int64_t)(at.ct >> 2) * p.gate.srows + at.rt * 128) * 4 + (at.ct & 3);
  const uint8_t* up_codes = p.up.scales + ((int64_t)(at.ct >> 2) * p.up.srows + at.rt * 128) * 4 + (at.ct & 3);
  Raw8<BF16> dh[kTileRows];
  u32x2 gate[kTileRows], up[kTileRows];
  uint32_t gate_code[kTileRows], up_code[kTileRows];
  auto load = [&](auto load_dh, auto load_codes) {
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
      const uint32_t row = min(first + i, behind - 1);
      const uint8_t* from = dhs + (row_offset(row, p.dh_stride * (BF16 ? 2 : 4)) + col * (BF16 ? 2 : 4));
#pragma unroll
      for (int h = 0; h < (BF16 ? 1 : 2); ++h) dh[i].w[h] = load_dh(from + 16 * h);
      gate[i] = load_codes(gates + (row_offset(row, p.gate.stride) + col));
      up[i] = load_codes(ups + (row_offset(row, p.up.stride) + col));
      gate_code[i] = gate_codes[row * 4];
      up_code[i] = up_codes[row * 4];
    }
  };
  if (p.stream) {
    asm volatile("; a branch");  // the compiler would make the loads of both branches one, ahead of them or behind, without the hint
    load([](const uint8_t* from) { return load_stream(reinterpret_cast<const u32x4*>(from)); },
         [](const uint8_t* from) { return load_stream(reinterpret_cast<const u32x2*>(from)); });
    asm volatile("; its end");
  } else
    load([](const uint8_t* from) -> u32x4 { return *reinterpret_cast<const typename AnyElement<BF16>::type*>(from); },
         [](const uint8_t* from) { return *reinterpret_cast<const u32x2*>(from); });
  lds_barrier();
  TileValues a, t;
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    if (first + i >= behind) dh[i] = Raw8<BF16>{}, gate[i] = up[i] = u32x2{};
    const Values8 g = f32_values(gate[i], gate_code[i]), u = f32_values(up[i], up_code[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const ActSlope r = act_slope<SILU>(g.v[j], p.act);
      a.v[i][j] = r.act;
      t.v[i][j] = __uint_as_float(bits_of<BF16>(dh[i], j)) * u.v[j] * r.slope;
    }
    // a row at a time, whether d or dt is wanted or not: the registers hold no more
#pragma unroll
    for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(t.v[i][j]), "+v"(a.v[i][j]));
  }
  if (p.d.data || p.dt.data) {
    put_tile(t, at, p.d, p.dt, space, 0);
    pin(a), pin(dh), pin(up);
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
    pin(a), pin(up);
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
  const TilePlace at = backward_place(p.tiles_x);
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
  lds_barrier();
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
  BackwardArgs a = {l.dh, l.dh_stride, l.rows, l.f, 0, 0, l.act, l.gate, l.up, l.d, l.dt, l.ht};
  const dim3 block(kTileLanes);
  const bool silu = l.act.k3 == 0;
  if (l.f % kBlock == 0 && l.dh_stride * (l.dh_bf16 ? 2 : 4) < 1 << 24) {
    a.tiles_x = l.f / kBlock;
    // large inputs are streamed past the last cache, which is left to what the products behind this call read: with them
    // 8192 x 3456 735 us, else 740; 2048 x 4864 (less than kCached) 93 and 95
    const int64_t size = l.dh_bf16 ? 2 : 4, outs = 2 * (l.d.data != nullptr) + 2 * (l.dt.data != nullptr) + (l.ht.data != nullptr);
    a.stream = (int64_t)l.rows * l.f * (size + 2 + outs) > kCached && whole_pieces(l.dh, l.dh_stride, l.f, size);
    const dim3 grid(a.tiles_x * (uint32_t)ceil_div(l.rows, 128));
    if (l.dh_bf16 && silu) hipLaunchKernelGGL((gated_backward_kernel<true, true>), grid, block, 0, st, a);
    else if (l.dh_bf16) hipLaunchKernelGGL((gated_backward_kernel<true, false>), grid, block, 0, st, a);
    else if (silu) hipLaunchKernelGGL((gated_backward_kernel<false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((gated_backward_kernel<false, false>), grid, block, 0, st, a);
  } else {
    a.tiles_x = (uint32_t)ceil_div(2 * (int64_t)l.f, kBlock);
    const dim3 grid(a.tiles_x * (uint32_t)ceil_div(l.rows, 128));
    if (l.dh_bf16) hipLaunchKernelGGL(gated_backward_any_kernel<true>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(gated_backward_any_kernel<false>, grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace dr
