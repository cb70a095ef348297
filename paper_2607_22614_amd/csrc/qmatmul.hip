// Products of 8-bit matrices (dr_qmatmul, dr_qlinear): c = a * b^T with both operands row-major along K.
//
//   c[m, n] = sum over 128-column blocks j of 2^(ea[m, j] + eb[n, j]) * sum over k in block j of qa[m, k] * qb[n, k]
//
// b (the weights' side) is the matrix instructions' first operand: a lane then holds four consecutive columns of one
// row of c.  Which 32 of the 128 columns a lane gives is free as long as both operands agree: lane group g (of four)
// gives columns 16g.. and 64+16g.., so that each 16-byte load of a wave covers 64 consecutive bytes of 16 rows.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "quant_device.h"

namespace dr {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct ProductArgs {
  QView a, b;
  const void* x;
  int64_t x_stride;
  void* c;
  int64_t c_stride;
  uint32_t m, n, kb, tiles_m, tiles_n;
  uint32_t splits;  // of the blocks: workgroups of one tile, whose fp32 sums go to part[split][m][part_stride]
  int32_t c_vec, c_bf16, accumulate;
  float* part;
  int64_t part_stride;
};

__device__ __forceinline__ i32x8 join(u32x4 lo, u32x4 hi) {
  return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// 32 codes of a row's 128-column block: p is the row at the block's first column plus 16 * lane group.
__device__ __forceinline__ i32x8 load_codes(const uint8_t* p) {
  const u32x4 lo = *reinterpret_cast<const u32x4*>(p), hi = *reinterpret_cast<const u32x4*>(p + 64);
  return join(lo, hi);
}

// The 128 columns' share of 16 x 16 outputs with exact products and sums: the values that 32 codes and their scale stand
// for are exact in bf16, and the bf16 matrix instructions add exact products in fp32.
struct Bf16Codes {
  bf16x8 v[4];
};
__device__ __forceinline__ Bf16Codes to_bf16(i32x8 codes, int code) {
  const float scale = __uint_as_float((uint32_t)code << 23);  // the convert takes a power of two by its exponent bits
  Bf16Codes r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * i + h], scale, false);
      const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * i + h], scale, true);
      r.v[i][4 * h] = lo[0], r.v[i][4 * h + 1] = lo[1], r.v[i][4 * h + 2] = hi[0], r.v[i][4 * h + 3] = hi[1];
    }
  return r;
}
// Columns n0 .. n0+3 of row m of c.
__device__ __forceinline__ void store4(const ProductArgs& p, uint32_t m, uint32_t n0, f32x4 v) {
  if (m >= p.m || n0 >= p.n) return;
  const int64_t at = (int64_t)m * p.c_stride + n0;
  const bool whole = p.c_vec && n0 + 4 <= p.n;
  if (p.c_bf16) {
    uint16_t* c = static_cast<uint16_t*>(p.c) + at;
    const u32x2 w = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    if (whole) {
      *reinterpret_cast<u32x2*>(c) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n0 + i < p.n) c[i] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
    }
  } else {
    float* c = static_cast<float*>(p.c) + at;
    if (whole) {
      f32x4* q = reinterpret_cast<f32x4*>(c);
      *q = p.accumulate ? *q + v : v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n0 + i < p.n) c[i] = p.accumulate ? c[i] + v[i] : v[i];
    }
  }
}

// 16 bytes of results, columns n0 on, of row m of c.
template <int BYTES>
__device__ __forceinline__ void store_piece(const ProductArgs& p, uint32_t m, uint32_t n0, u32x4 w) {
  constexpr int kElems = 16 / BYTES;
  if (m >= p.m || n0 >= p.n) return;
  const int64_t at = (int64_t)m * p.c_stride + n0;
  const bool whole = p.c_vec && n0 + kElems <= p.n;
  if (BYTES == 2) {
    uint16_t* c = static_cast<uint16_t*>(p.c) + at;
    if (whole) {
      *reinterpret_cast<u32x4*>(c) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (n0 + i < p.n) c[i] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
    }
  } else {
    float* c = static_cast<float*>(p.c) + at;
    const f32x4 v = __builtin_bit_cast(f32x4, w);
    if (whole) {
      f32x4* q = reinterpret_cast<f32x4*>(c);
      *q = p.accumulate ? *q + v : v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n0 + i < p.n) c[i] = p.accumulate ? c[i] + v[i] : v[i];
    }
  }
}

// A lane's 32 elements of 128 columns of one row of x, as they lie in memory.  How x comes: fp32 or bf16, in rows of whole
// 16-byte pieces (kVec: loads without branches, which the compiler leaves in flight) or any rows; or as codes.
enum XKind { kCodes = 0, kF32 = 1, kBf16 = 2, kVec = 4 };
template <int X>
struct Elements {
  Raw8<(X & kBf16) != 0> v[X == kCodes ? 1 : 4];
};
template <int X>
__device__ __forceinline__ Elements<X> load_elements(const ProductArgs& p, uint32_t row, uint32_t col) {
  constexpr bool BF16 = (X & kBf16) != 0;
  Elements<X> e;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t c = col + (q >> 1) * 64 + (q & 1) * 8;
    const int64_t at = (int64_t)row * p.x_stride;
    if (X & kVec) {
      const u32x4* x = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(p.x) + (at + min(c, p.a.cols - 8)) * (BF16 ? 2 : 4));
#pragma unroll
      for (int i = 0; i < (BF16 ? 1 : 2); ++i) e.v[q].w[i] = x[i];
    } else {
      e.v[q] = load_raw8<BF16>(p.x, at + c, max(0, min(8, (int)p.a.cols - (int)c)), false);
    }
  }
  return e;
}
// Zeros in place of what kVec loads read again from columns that are not there (pieces are all there or not at all).
template <int X>
__device__ __forceinline__ void clear_beyond(const ProductArgs& p, uint32_t col, Elements<X>& e) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int i = 0; i < ((X & kBf16) ? 1 : 2); ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) e.v[q].w[i][w] = col + (q >> 1) * 64 + (q & 1) * 8 < p.a.cols ? e.v[q].w[i][w] : 0u;
}

// Their codes, and the scale of the row's 128 columns, as dr_quantize gives them.
template <int X>
__device__ __forceinline__ i32x8 quantize_block(const Elements<X>& e, int& code) {
  uint32_t m = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) m = max(m, row_max(e.v[q], false));
  if (__any(m >= kInfBits)) {
    m = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) m = max(m, row_max(e.v[q], true));
  }
  code = (int)scale_code(max_rows(m));
  i32x8 w;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const u32x2 c = row_codes(e.v[q], (uint32_t)code);
    w[2 * q] = (int)c[0];
    w[2 * q + 1] = (int)c[1];
  }
  return w;
}

// Few rows: a tile of FT * 16 columns by TT * 16 rows of c per workgroup, operands straight from memory to the matrix
// instructions; the KS waves of the workgroup take the 128-column blocks in turn, each with its next block in flight while
// it multiplies one, and join their sums in LDS, in the order of the waves.  X: a's codes, or rows of x to quantize.
template <int FT, int TT, int KS, int X, bool FAST>
__global__ __launch_bounds__(64 * KS) void product_direct_kernel(ProductArgs p) {
  __shared__ f32x4 part[KS][FT * TT][64];
  const uint32_t lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t n0 = blockIdx.x % p.tiles_n * (FT * 16), m0 = blockIdx.x / p.tiles_n * (TT * 16);
  const uint8_t *bp[FT], *ap[TT], *bcode[FT], *acode[TT];
  uint32_t arow[TT];
#pragma unroll
  for (int f = 0; f < FT; ++f) {
    const uint32_t row = min(n0 + f * 16 + r, p.n - 1);
    bp[f] = p.b.data + (int64_t)row * p.b.stride + g * 16;
    bcode[f] = p.b.scales + 4 * (row >> p.b.sh);
  }
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    arow[t] = min(m0 + t * 16 + r, p.m - 1);
    ap[t] = p.a.data + (int64_t)arow[t] * p.a.stride + g * 16;
    acode[t] = p.a.scales + 4 * (arow[t] >> p.a.sh);
  }
  struct Block {
    i32x8 b[FT], a[X ? 1 : TT];
    int eb[FT], ea[TT];
    Elements<X> x[X ? TT : 1];
  };
  auto load = [&](uint32_t j) {
    Block k;
#pragma unroll
    for (int f = 0; f < FT; ++f) {
      k.b[f] = load_codes(bp[f] + (int64_t)j * 128);
      k.eb[f] = bcode[f][(int64_t)(j >> 2) * p.b.srows * 4 + (j & 3)];
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      if constexpr (X != 0) {
        k.x[t] = load_elements<X>(p, arow[t], j * 128 + g * 16);
      } else {
        k.a[t] = load_codes(ap[t] + (int64_t)j * 128);
        k.ea[t] = acode[t][(int64_t)(j >> 2) * p.a.srows * 4 + (j & 3)];
      }
    }
    return k;
  };
  f32x4 acc[FT][TT] = {};
  auto multiply = [&](Block& k, uint32_t j) {
    i32x8 aw[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      if constexpr (X != 0) {
        if ((X & kVec) && j * 128 + 128 > p.a.cols) clear_beyond<X>(p, j * 128 + g * 16, k.x[t]);
        aw[t] = quantize_block(k.x[t], k.ea[t]);
      } else {
        aw[t] = k.a[t];
      }
    }
    if constexpr (FAST) {
#pragma unroll
      for (int f = 0; f < FT; ++f)
#pragma unroll
        for (int t = 0; t < TT; ++t)
          acc[f][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k.b[f], aw[t], acc[f][t], 0, 0, 0, k.eb[f], 0, k.ea[t]);
    } else {
      Bf16Codes ca[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) ca[t] = to_bf16(aw[t], k.ea[t]);
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        const Bf16Codes cb = to_bf16(k.b[f], k.eb[f]);
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cb.v[i], ca[t].v[i], acc[f][t], 0, 0, 0);
      }
    }
  };
  if (wave < p.kb) {
    Block next = load(wave);
    for (uint32_t j = wave; j < p.kb; j += KS) {
      Block k = next;
      if (j + KS < p.kb) next = load(j + KS);
      multiply(k, j);
    }
  }
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int t = 0; t < TT; ++t) part[wave][f * TT + t][lane] = acc[f][t];
  __syncthreads();
  for (uint32_t i = wave; i < FT * TT; i += KS) {
    f32x4 s = part[0][i][lane];
#pragma unroll
    for (int k = 1; k < KS; ++k) s += part[k][i][lane];
    store4(p, m0 + i % TT * 16 + r, n0 + i / TT * 16 + g * 4, s);
  }
}

template <int FT, int TT, int KS, int X>
void launch_direct(ProductArgs a, bool fast, hipStream_t st) {
  a.tiles_n = (uint32_t)ceil_div(a.n, FT * 16);
  const dim3 grid(a.tiles_n * (uint32_t)ceil_div(a.m, TT * 16)), block(64 * KS);
  if (fast) hipLaunchKernelGGL((product_direct_kernel<FT, TT, KS, X, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((product_direct_kernel<FT, TT, KS, X, false>), grid, block, 0, st, a);
}

// More columns a workgroup read a fewer times, fewer columns give more workgroups.  One tile of 16 columns up to 4096
// (256 workgroups), two up to 16384, then four; eight waves share the blocks, four of the widest.  In us for 1 / 2 / 4:
//   1 row, 4096 x 3584: 5.5 / 7.1 / 10.4     16 rows, 6912 x 5120: 17.0 / 13.0 / 18.3     32 rows, 32064 x 4096: 50 / 37 / 32
// and with 4 / 8 / 16 waves, 1 row, 4096 x 3584: 6.4 / 5.5 / 5.7; four tiles, 16 rows, 151936 x 896: 29 / 38 / 66.
template <int TT, int X>
void launch_few_rows(const ProductArgs& a, bool fast, hipStream_t st) {
  if (a.n <= 4096) launch_direct<1, TT, 8, X>(a, fast, st);
  else if (a.n <= 16384) launch_direct<2, TT, 8, X>(a, fast, st);
  else launch_direct<4, TT, 4, X>(a, fast, st);
}

// ------------------------------------------------------------------ large products

// 16 bytes per lane from memory to LDS, at `to` + 16 * lane; nothing passes through registers.  As a buffer access its
// address is the tile's base, the lane's offset and the step's, with no arithmetic in between.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_at(const uint8_t* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, 0xFFFFFFFFu, 0x00027000);  // raw, 32-bit data
}
__device__ __forceinline__ void copy_to_lds(Buffer from, uint32_t lane_at, uint32_t at, uint8_t* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, (int)lane_at, (int)at, 0, 0);
}

// Tile (tm, tn) of workgroup b: each XCD takes a contiguous eighth of the tiles, in bands of kBand tiles down, so that
// the workgroups running at once on it share rows of both operands in its L2.
constexpr uint32_t kBand = 8;
// Returns the split: whole products of tiles follow one another.
__device__ __forceinline__ uint32_t tile_of(uint32_t b, uint32_t tiles_m, uint32_t tiles_n, uint32_t splits, uint32_t& tm, uint32_t& tn) {
  const uint32_t all = xcd_tile(b, tiles_m * tiles_n * splits), split = all / (tiles_m * tiles_n), t = all % (tiles_m * tiles_n);
  const uint32_t band = t / (kBand * tiles_n), high = min(kBand, tiles_m - band * kBand), i = t - band * kBand * tiles_n;
  tm = band * kBand + i % high;
  tn = i / high;
  return split;
}

// Results of a wave, TM * 32 rows by TN * 32 columns from (m0, n0), through TM * TN * 2 KiB of LDS.
template <int TM, int TN, int BYTES>
__device__ __forceinline__ void store_turned(const ProductArgs& p, const f32x16 (&acc)[TN][TM], uint8_t* lds, uint32_t m0, uint32_t n0, uint32_t lane) {
  constexpr int kPitch = TN * 32 * BYTES, kPiecesRow = kPitch / 16, kPart = TM * 2 / BYTES;  // tiles down that fit at once
  constexpr int kMask = kPiecesRow - 1, kRowsAt = 64 / kPiecesRow, kElems = 16 / BYTES;
  static_assert(kPiecesRow <= 64 && (kPiecesRow & kMask) == 0, "rows of a power of two of pieces");
  const uint32_t r = lane & 31, g = lane >> 5;
#pragma unroll
  for (int y0 = 0; y0 < TM; y0 += kPart) {
#pragma unroll
    for (int x = 0; x < TN; ++x)
#pragma unroll
      for (int y = 0; y < kPart; ++y)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x16& a = acc[x][y0 + y];
          uint8_t* row = lds + (y * 32 + r) * kPitch;
          const uint32_t col = x * 32 + q * 8 + g * 4;
          if (BYTES == 2)
            *reinterpret_cast<u32x2*>(row + (((col / 8) ^ (r & kMask)) * 16) + col % 8 * 2) = u32x2{bf16_pair(a[q * 4], a[q * 4 + 1]), bf16_pair(a[q * 4 + 2], a[q * 4 + 3])};
          else
            *reinterpret_cast<f32x4*>(row + (((col / 4) ^ (r & kMask)) * 16)) = f32x4{a[q * 4], a[q * 4 + 1], a[q * 4 + 2], a[q * 4 + 3]};
        }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < kPart * 32 / kRowsAt; ++i) {
      const uint32_t row = i * kRowsAt + lane / kPiecesRow, piece = lane % kPiecesRow;
      const u32x4 w = *reinterpret_cast<const u32x4*>(lds + row * kPitch + ((piece ^ (row & 31 & kMask)) * 16));
      store_piece<BYTES>(p, m0 + y0 * 32 + row, n0 + piece * kElems, w);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// A tile of BM x BN of c per workgroup of WM * WN waves.  A step stages one 128-column block of BM rows of a and BN rows of
// b in LDS (copied straight there, two buffers in turn), each row's eight 16-byte pieces at piece ^ row / 2 % 8: the
// sixteen lanes that read at once, the same piece of sixteen rows, then meet all 64 banks.
template <int BM, int BN, int WM, int WN, bool FAST>
__global__ __launch_bounds__(64 * WM * WN) void product_tile_kernel(ProductArgs p) {
  constexpr int kWaves = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, kRows = BM + BN, kCopies = kRows / 8 / kWaves;
  static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0 && kRows % (8 * kWaves) == 0 && BM % (8 * kWaves) == 0, "tile");
  __shared__ __align__(16) uint8_t lds[2][kRows * 128];
  const uint32_t lane = threadIdx.x & 63, r = lane & 31, g = lane >> 5;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  uint32_t tm, tn;
  const uint32_t split = tile_of(blockIdx.x, p.tiles_m, p.tiles_n, p.splits, tm, tn);
  const uint32_t m0 = tm * BM, n0 = tn * BN;
  const uint32_t wm = wave % WM * (TM * 32), wn = wave / WM * (TN * 32);
  const Buffer abase = buffer_at(p.a.data + (int64_t)m0 * p.a.stride);
  const Buffer bbase = buffer_at(p.b.data + (int64_t)n0 * p.b.stride);

  // copies: rows [0, BM) of the stage are a's, the others b's; rows past the matrix read its last one
  uint32_t from[kCopies];
#pragma unroll
  for (int i = 0; i < kCopies; ++i) {
    const uint32_t row = (i * kWaves + wave) * 8 + lane / 8, piece = (lane % 8) ^ (row / 2 % 8);
    if (i * kWaves * 8 < BM) from[i] = min(row, p.m - 1 - m0) * (uint32_t)p.a.stride + piece * 16;
    else from[i] = min(row - BM, p.n - 1 - n0) * (uint32_t)p.b.stride + piece * 16;
  }
  auto stage = [&](uint32_t j, uint8_t* to, int i) {
    copy_to_lds(i * kWaves * 8 < BM ? abase : bbase, from[i], j * 128, to + (i * kWaves + wave) * 1024);
  };

  // scale codes of one block column for the lane's rows (a matrix's scales are a 128th of its data: below 2^32 bytes)
  const Buffer ascales = buffer_at(p.a.scales), bscales = buffer_at(p.b.scales);
  uint32_t acode[TM], bcode[TN];
#pragma unroll
  for (int t = 0; t < TM; ++t) acode[t] = 4 * (min(m0 + wm + t * 32 + r, p.m - 1) >> p.a.sh);
#pragma unroll
  for (int t = 0; t < TN; ++t) bcode[t] = 4 * (min(n0 + wn + t * 32 + r, p.n - 1) >> p.b.sh);
  struct Scales {
    int a[TM], b[TN];
  };
  auto load_scales = [&](uint32_t j) {
    Scales s;
#pragma unroll
    for (int t = 0; t < TM; ++t) s.a[t] = __builtin_amdgcn_raw_buffer_load_b8(ascales, (int)acode[t], (int)(j / 4 * p.a.srows * 4 + j % 4), 0);
#pragma unroll
    for (int t = 0; t < TN; ++t) s.b[t] = __builtin_amdgcn_raw_buffer_load_b8(bscales, (int)bcode[t], (int)(j / 4 * p.b.srows * 4 + j % 4), 0);
    return s;
  };

  // the lane's pieces: of each half h of the 128 columns, pieces 4h + 2g and 4h + 2g + 1
  uint32_t at[2][2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 2; ++e) at[h][e] = r * 128 + (((h * 4 + g * 2 + e) ^ (r / 2 % 8)) * 16);
  // 16-byte pieces of one half block: two for each 32 rows, b's first
  constexpr int kPieces = 2 * (TM + TN), kTiles = TM * TN;
  struct Codes {
    u32x4 piece[kPieces];
  };
  auto read_piece = [&](const uint8_t* from_lds, int h, int i) {
    const int t = i / 2;
    return *reinterpret_cast<const u32x4*>(from_lds + (t < TN ? (BM + wn) * 128 + t * 4096 : wm * 128 + (t - TN) * 4096) + at[h][i % 2]);
  };

  // One half block: its matrix instructions, and spread evenly among them what `between(i)` does for i of kTiles.
  // Left alone the compiler would put all reads and copies behind them.
  f32x16 acc[TN][TM] = {};
  auto multiply = [&](const Codes& c, const Scales& s, auto between) {
    Bf16Codes ca[FAST ? 1 : TM], cb;
#pragma unroll
    for (int x = 0; x < TN; ++x)
#pragma unroll
      for (int y = 0; y < TM; ++y) {
        const i32x8 fb = join(c.piece[2 * x], c.piece[2 * x + 1]), fa = join(c.piece[2 * (TN + y)], c.piece[2 * (TN + y) + 1]);
        between(x * TM + y);
        if constexpr (FAST) {
          acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb, fa, acc[x][y], 0, 0, 0, s.b[x], 0, s.a[y]);
        } else {
          if (x == 0) ca[y] = to_bf16(fa, s.a[y]);
          if (y == 0) cb = to_bf16(fb, s.b[x]);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cb.v[i], ca[y].v[i], acc[x][y], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0x6);  // vector and scalar arithmetic may move across
      }
  };

  // Step j: block j's second half is read while its first is multiplied; then, once every wave has read all of block
  // j and block j + 1 has landed, block j + 2 starts on its way into block j's buffer and the first half of block j + 1
  // is read while the second of block j is multiplied.
  Codes first;
  Scales now, next;
  auto step = [&](uint32_t j, auto more, auto last) {
    uint8_t *cur = lds[j & 1], *other = lds[(j + 1) & 1];
    Codes second;
    multiply(first, now, [&](int i) {
#pragma unroll
      for (int k = i * kPieces / kTiles; k < (i + 1) * kPieces / kTiles; ++k) second.piece[k] = read_piece(cur, 1, k);
    });
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
    // used from here on only: copied any earlier, they would be waited for there, and all copies with them
#pragma unroll
    for (int t = 0; t < TM; ++t) asm volatile("" : "+v"(next.a[t]));
#pragma unroll
    for (int t = 0; t < TN; ++t) asm volatile("" : "+v"(next.b[t]));
    const Scales landed = next;
    if constexpr (decltype(more)::value) next = load_scales(j + 2);
    multiply(second, now, [&](int i) {
      if constexpr (!decltype(last)::value) {
#pragma unroll
        for (int k = i * kPieces / kTiles; k < (i + 1) * kPieces / kTiles; ++k) first.piece[k] = read_piece(other, 0, k);
      }
      if constexpr (decltype(more)::value) {
#pragma unroll
        for (int k = i * kCopies / kTiles; k < (i + 1) * kCopies / kTiles; ++k) stage(j + 2, cur, k);
      }
    });
    now = landed;
  };
  const uint32_t j0 = (uint32_t)((uint64_t)p.kb * split / p.splits), j1 = (uint32_t)((uint64_t)p.kb * (split + 1) / p.splits);
  if (j0 < j1) {
    now = load_scales(j0);
    next = load_scales(min(j0 + 1, j1 - 1));
#pragma unroll
    for (int i = 0; i < kCopies; ++i) stage(j0, lds[j0 & 1], i);
    __syncthreads();
    if (j0 + 1 < j1) {
#pragma unroll
      for (int i = 0; i < kCopies; ++i) stage(j0 + 1, lds[(j0 + 1) & 1], i);
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) first.piece[i] = read_piece(lds[j0 & 1], 0, i);
    for (uint32_t j = j0; j + 2 < j1; ++j) step(j, std::true_type{}, std::false_type{});
    if (j0 + 1 < j1) step(j1 - 2, std::false_type{}, std::false_type{});
    step(j1 - 1, std::false_type{}, std::true_type{});
  }
  // Each wave turns its results in its own part of the LDS, so that they leave as whole rows of TN * 32 columns: 16-byte
  // pieces, at piece ^ row % 32 of a row.
  __syncthreads();
  constexpr int kOut = BM * BN / kWaves;  // results of a wave
  uint8_t* mine = lds[0] + wave * (sizeof(lds) / kWaves);
  if (p.splits > 1) {
    p.c = p.part + (int64_t)split * p.m * p.part_stride;
    p.c_stride = p.part_stride;
    p.c_vec = 1;
    p.c_bf16 = p.accumulate = 0;
  }
  if (p.c_bf16) store_turned<TM, TN, 2>(p, acc, mine, m0 + wm, n0 + wn, lane);
  else store_turned<TM, TN, 4>(p, acc, mine, m0 + wm, n0 + wn, lane);
  static_assert(kOut * 2 <= (int)sizeof(lds) / kWaves, "a wave's bf16 results fit its part");
}

// c from the sums of the splits, in their order; a lane takes four columns.
__global__ __launch_bounds__(256) void join_splits_kernel(ProductArgs p) {
  const uint32_t groups = (uint32_t)(p.part_stride / 4);
  const uint64_t n = (uint64_t)p.m * groups;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
    const uint32_t m = (uint32_t)(i / groups), n0 = (uint32_t)(i % groups) * 4;
    const float* part = p.part + (int64_t)m * p.part_stride + n0;
    f32x4 s = *reinterpret_cast<const f32x4*>(part);
    for (uint32_t k = 1; k < p.splits; ++k) s += *reinterpret_cast<const f32x4*>(part + (int64_t)k * p.m * p.part_stride);
    store4(p, m, n0, s);
  }
}

template <int BM, int BN, int WM, int WN>
void launch_tile(ProductArgs a, bool fast, hipStream_t st) {
  a.tiles_m = (uint32_t)ceil_div(a.m, BM);
  a.tiles_n = (uint32_t)ceil_div(a.n, BN);
  const dim3 grid(a.tiles_m * a.tiles_n * a.splits), block(64 * WM * WN);
  if (fast) hipLaunchKernelGGL((product_tile_kernel<BM, BN, WM, WN, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((product_tile_kernel<BM, BN, WM, WN, false>), grid, block, 0, st, a);
  if (a.splits > 1)
    hipLaunchKernelGGL(join_splits_kernel, dim3((uint32_t)std::min<int64_t>(2048, ceil_div(a.m * (a.part_stride / 4), 256))), dim3(256), 0, st, a);
}

}  // namespace

hipError_t launch_product(const ProductLaunch& l, hipStream_t st) {
  ProductArgs a;
  a.a = l.a;
  a.b = l.b;
  a.x = l.x;
  a.x_stride = l.x_stride;
  a.c = l.c;
  a.c_stride = l.c_stride;
  a.m = l.m;
  a.n = l.n;
  a.kb = l.kb;
  a.c_vec = reinterpret_cast<uintptr_t>(l.c) % 16 == 0 && l.c_stride * (l.c_bf16 ? 2 : 4) % 16 == 0;
  a.c_bf16 = l.c_bf16;
  a.accumulate = l.accumulate;
  if (l.x) {
    // rows that are no whole 16-byte pieces are loaded element by element, by one form of the kernel
    const bool vec = l.x_aligned && l.a.cols % 8 == 0;
    if (l.x_bf16) {
      if (vec) launch_few_rows<1, kBf16 | kVec>(a, l.fast, st);
      else launch_direct<1, 1, 8, kBf16>(a, l.fast, st);
    } else {
      if (vec) launch_few_rows<1, kF32 | kVec>(a, l.fast, st);
      else launch_direct<1, 1, 8, kF32>(a, l.fast, st);
    }
  } else if (const ProductPlan plan = plan_product(l.m, l.n, l.kb, l.fast); plan.kind != ProductPlan::kDirect) {
    a.splits = plan.splits;
    a.part = static_cast<float*>(l.workspace);
    a.part_stride = part_stride(l.n);
    if (plan.kind == ProductPlan::kTile256) launch_tile<256, 256, 2, 2>(a, l.fast, st);
    else launch_tile<128, 128, 2, 2>(a, l.fast, st);
  } else {
    if (l.m <= 16) launch_few_rows<1, kCodes>(a, l.fast, st);
    else launch_few_rows<2, kCodes>(a, l.fast, st);
  }
  return hipGetLastError();
}

}  // namespace dr
