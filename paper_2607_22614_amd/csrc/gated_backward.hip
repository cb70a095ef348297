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
  uint32_t rows, f, tiles, tiles_x;
  int32_t split;   // the grid holds every tile once for each matrix it gives (dgate, dup, h; d, h for any f), in this order
  int32_t stream;
  Act act;
  QView gate, up, d, dt, ht;
};

// Bands of sixteen tiles down, a contiguous eighth of them to each XCD: 8192 x 14336 in 218 us as first measured, in the order of
// dr_quantize's tiles 226 (bands of 8 and 32: 229, 219).
__device__ __forceinline__ TilePlace backward_place(const BackwardArgs& p) { return place_of<16>(xcd_tile(blockIdx.x % p.tiles, p.tiles), p.tiles, p.tiles_x); }

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

// f a multiple of 128, rows of dh less than 2^24 bytes apart: gate's and up's halves of d consist of whole tiles, and a workgroup
// takes one of either.  dup and h are computed when dgate has left: all three at once would take the registers of a second
// workgroup (8192 x 14336 341 us with them).
//   Memory-bound: 8192 x 14336 in 219 us, 4.9 TB/s, with the vector units busy 65 % of the time.
template <bool BF16, bool SILU>
__global__ __launch_bounds__(kTileLanes, 4) void gated_backward_kernel(BackwardArgs p) {
  __shared__ ValuesSpace space;
  const TilePlace at = backward_place(p);
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
  const uint32_t role = blockIdx.x / p.tiles;
  if (p.d.data || p.dt.data) {
    if (!p.split || role == 0) put_tile(t, at, p.d, p.dt, space, 0);
    if (!p.split || role == 1) {
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
  }
  if (p.ht.data && (!p.split || role == 2)) {
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

// Any f: a workgroup takes one tile of d's 2f columns, or, for ht alone, of its f (2000 x 2000 7.7 us; of 2f 12.0).  A lane's 8
// columns begin anywhere in a block of gate or up, so that they may have two scales; where gate's half ends among them, up's
// first columns follow (ODD: f no multiple of 8, else neither comes about).  Rows of fewer than 8 are read element by element.
// 2000 x 2000 in 16.7 us; element by element 23.5.
template <bool BF16, bool SILU, bool ODD>
__global__ __launch_bounds__(kTileLanes) void gated_backward_any_kernel(BackwardArgs p) {
  __shared__ ValuesSpace space;
  const TilePlace at = backward_place(p);
  const uint32_t role = blockIdx.x / p.tiles;
  if (role == 1 && at.ct * 128 >= p.f) return;  // nothing of h
  clear_maxima(space);
  const bool of_up = at.col >= p.f, both = !of_up && at.col + 8 > p.f;
  const uint32_t f = at.col - (of_up ? p.f : 0), block = min(f, p.f - 1) / 128, last = min(f + 7, p.f - 1) / 128;
  const uint32_t first = 128 - f % 128, mine = p.f - f;  // columns of the first scale; (both) of gate
  struct Part {
    Raw8<BF16> dh;
    u32x2 gate, up;
    uint32_t gate_code, up_code;
  };
  Part own[kTileRows] = {}, next[kTileRows] = {};  // next: (both) up's first 8
  uint32_t gate_last[kTileRows], up_last[kTileRows];
  auto load = [&](Part& t, uint32_t row, uint32_t from, uint32_t of_block) {
    t.dh = load_row8<BF16>(p.dh, (int64_t)row * p.dh_stride, from, p.f);
    t.gate = load_codes8(p.gate, row, from);
    t.up = load_codes8(p.up, row, from);
    t.gate_code = scale_at(p.gate, row, of_block), t.up_code = scale_at(p.up, row, of_block);
  };
  if (!ODD || p.f >= 8) {
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
      const uint32_t row = min(at.row0 + i, p.rows - 1);
      load(own[i], row, f, block);
      if (ODD) gate_last[i] = scale_at(p.gate, row, last), up_last[i] = scale_at(p.up, row, last);
      if (ODD && both) load(next[i], row, 0, 0);
    }
  }
  lds_barrier();
  const bool two_scales = ODD && __any(first < 8), any_both = ODD && __any(both);
  TileValues d, h;
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    const bool in = at.row0 + i < p.rows;
    Values8 dhs = {}, gs = {}, us = {};
    if (ODD && p.f < 8) {
      const uint32_t row = min(at.row0 + i, p.rows - 1);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = at.col + j, one = min(c - (c < p.f ? 0 : p.f), p.f - 1);
        if (!in || c >= 2 * p.f) continue;
        const int64_t from = (int64_t)row * p.dh_stride + one;
        dhs.v[j] = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p.dh)[from] << 16) : static_cast<const float*>(p.dh)[from];
        gs.v[j] = f32_values(u32x2{p.gate.data[(int64_t)row * p.gate.stride + one], 0}, scale_at(p.gate, row, 0)).v[0];
        us.v[j] = f32_values(u32x2{p.up.data[(int64_t)row * p.up.stride + one], 0}, scale_at(p.up, row, 0)).v[0];
      }
    } else {
      Part& t = own[i];
      if (!in) t.dh = Raw8<BF16>{}, t.gate = t.up = u32x2{};
      settle8(t.dh, ahead8(f, p.f));
      gs = f32_values(t.gate, t.gate_code);
      us = f32_values(t.up, t.up_code);
      if (two_scales) {
        const Values8 g = f32_values(t.gate, gate_last[i]), u = f32_values(t.up, up_last[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          gs.v[j] = (uint32_t)j < first ? gs.v[j] : g.v[j];
          us.v[j] = (uint32_t)j < first ? us.v[j] : u.v[j];
        }
      }
      if (any_both) {
        const Raw8<BF16> after = delayed8(next[i].dh, mine & 7);
        const uint64_t gates = __builtin_bit_cast(uint64_t, next[i].gate) << 8 * (mine & 7), ups = __builtin_bit_cast(uint64_t, next[i].up) << 8 * (mine & 7);
        const Values8 g = f32_values(__builtin_bit_cast(u32x2, gates), next[i].gate_code), u = f32_values(__builtin_bit_cast(u32x2, ups), next[i].up_code);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool theirs = both && in && (uint32_t)j >= mine;
          dhs.v[j] = __uint_as_float(theirs ? bits_of<BF16>(after, j) : bits_of<BF16>(t.dh, j));
          gs.v[j] = theirs ? g.v[j] : gs.v[j];
          us.v[j] = theirs ? u.v[j] : us.v[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) dhs.v[j] = __uint_as_float(bits_of<BF16>(t.dh, j));
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool upper = at.col + j >= p.f;
      const ActSlope r = act_slope<SILU>(gs.v[j], p.act);
      d.v[i][j] = upper ? dhs.v[j] * r.act : dhs.v[j] * us.v[j] * r.slope;
      h.v[i][j] = upper ? 0.0f : r.act * us.v[j];
    }
  }
  if (!p.split || role == 0) put_tile(d, at, p.d, p.dt, space, 0);
  if (p.ht.data && at.ct * 128 < p.f && (!p.split || role == 1)) put_columns(h, at, p.ht, space, 2);
}

}  // namespace

hipError_t launch_gated_backward(const GatedBackward& l, hipStream_t st) {
  BackwardArgs a = {l.dh, l.dh_stride, l.rows, l.f, 0, 0, 0, 0, l.act, l.gate, l.up, l.d, l.dt, l.ht};
  const dim3 block(kTileLanes);
  const bool silu = l.act.k3 == 0, whole = l.f % kBlock == 0 && l.dh_stride * (l.dh_bf16 ? 2 : 4) < 1 << 24;
  a.tiles_x = (uint32_t)ceil_div(whole || !(l.d.data || l.dt.data) ? l.f : 2 * (int64_t)l.f, kBlock);
  a.tiles = a.tiles_x * (uint32_t)ceil_div(l.rows, 128);
  // where the CUs hold every matrix of every tile at once, each is computed by a workgroup of its own: 1024 x 1024 in 6.3 us, by one
  // workgroup a tile 8.4
  const uint32_t each = whole ? 3 : 2;
  a.split = l.ht.data && (l.d.data || l.dt.data) && a.tiles * each <= 256;
  const dim3 grid(a.split ? a.tiles * each : a.tiles);
  if (whole) {
    // large inputs are streamed past the last cache, which is left to what the products behind this call read: with them
    // 8192 x 3456 735 us, else 740; 2048 x 4864 (less than kCached) 93 and 95
    const int64_t size = l.dh_bf16 ? 2 : 4, outs = 2 * (l.d.data != nullptr) + 2 * (l.dt.data != nullptr) + (l.ht.data != nullptr);
    a.stream = (int64_t)l.rows * l.f * (size + 2 + outs) > kCached && whole_pieces(l.dh, l.dh_stride, l.f, size);
    if (l.dh_bf16 && silu) hipLaunchKernelGGL((gated_backward_kernel<true, true>), grid, block, 0, st, a);
    else if (l.dh_bf16) hipLaunchKernelGGL((gated_backward_kernel<true, false>), grid, block, 0, st, a);
    else if (silu) hipLaunchKernelGGL((gated_backward_kernel<false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((gated_backward_kernel<false, false>), grid, block, 0, st, a);
  } else {
    const bool odd = l.f % 8 != 0;
    auto launch = [&](auto any, auto odd_any) {
      if (odd) hipLaunchKernelGGL(odd_any, grid, block, 0, st, a);
      else hipLaunchKernelGGL(any, grid, block, 0, st, a);
    };
    if (l.dh_bf16 && silu) launch(gated_backward_any_kernel<true, true, false>, gated_backward_any_kernel<true, true, true>);
    else if (l.dh_bf16) launch(gated_backward_any_kernel<true, false, false>, gated_backward_any_kernel<true, false, true>);
    else if (silu) launch(gated_backward_any_kernel<false, true, false>, gated_backward_any_kernel<false, true, true>);
    else launch(gated_backward_any_kernel<false, false, false>, gated_backward_any_kernel<false, false, true>);
  }
  return hipGetLastError();
}

}  // namespace dr
