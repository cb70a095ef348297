// Products of 8-bit matrices (dr_qmatmul, dr_qlinear): c = a * b^T with both operands row-major along K.
//
//   c[m, n] = sum over 128-column blocks j of 2^(ea[m, j] + eb[n, j]) * sum over k in block j of qa[m, k] * qb[n, k]
//
// b (the weights' side) is the matrix instructions' first operand: a lane then holds four consecutive columns of one
// row of c.  Which 32 of the 128 columns a lane gives is free as long as both operands agree: lane group g (of four)
// gives columns 16g.. and 64+16g.., so that each 16-byte load of a wave covers 64 consecutive bytes of 16 rows.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "product_index.h"
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
  uint32_t first, count, quarters;  // the tiles of the launch (of few rows: the first one), and whether an item is a quarter of one (item_of)
  uint32_t splits;  // of the blocks: items of one tile, whose fp32 sums go to part[split][m][part_stride]
  int64_t split_bytes;  // of c, from one split to the next (0 without them)
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

// How x comes: as codes, or as rows of fp32 or bf16 (kShort: of fewer than 8 elements).
enum XKind { kCodes = 0, kF32 = 1, kBf16 = 2, kShort = 4 };

// A lane's 32 elements of 128 columns of one row of x, as load_row8 gives them.
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
    e.v[q] = X & kShort ? load_short_row8<BF16>(p.x, at, c, p.a.cols) : load_row8<BF16>(p.x, at, c, p.a.cols);
  }
  return e;
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

// Few rows, or few results: a tile of FT * 16 columns by TT * 16 rows of c per workgroup, operands straight from memory to the matrix
// instructions; the KS waves of the workgroup take the 128-column blocks in turn, each with its next block in flight while
// it multiplies one, and join their sums in LDS, in the order of the waves.  X: a's codes, or rows of x to quantize.  The sums
// are the exact ones: the 8-bit instructions' would save 6 % at most here (us, theirs / these: 1 x 4096 x 3584 5.9 / 6.1,
// 16 x 6912 x 5120 13.5 / 13.6, 32 x 6912 x 5120 14.2 / 14.7, 16 x 151936 x 896 33.8 / 34.1, 64 x 2000 x 2000 6.2 / 6.3).
template <int FT, int TT, int KS, int X>
__global__ __launch_bounds__(64 * KS) void product_direct_kernel(ProductArgs p) {
  __shared__ f32x4 part[KS][FT * TT][64];
  const uint32_t lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t tile = p.first + blockIdx.x, n0 = tile % p.tiles_n * (FT * 16), m0 = tile / p.tiles_n * (TT * 16);
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
        if (!(X & kShort) && j * 128 + 128 > p.a.cols) {
#pragma unroll
          for (int q = 0; q < 4; ++q) settle8(k.x[t].v[q], ahead8(j * 128 + g * 16 + (q >> 1) * 64 + (q & 1) * 8, p.a.cols));
        }
        aw[t] = quantize_block(k.x[t], k.ea[t]);
      } else {
        aw[t] = k.a[t];
      }
    }
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
void launch_direct(ProductArgs a, hipStream_t st) {
  a.tiles_n = (uint32_t)ceil_div(a.n, FT * 16);
  const uint32_t tiles = a.tiles_n * (uint32_t)ceil_div(a.m, TT * 16);
  // results of tens of gigabytes are more tiles than a launch holds
  for (a.first = 0; a.first < tiles;) {
    const uint32_t grid = std::min(tiles - a.first, max_workgroups(64 * KS));
    hipLaunchKernelGGL((product_direct_kernel<FT, TT, KS, X>), dim3(grid), dim3(64 * KS), 0, st, a);
    a.first += grid;
  }
}

// More columns a workgroup read a fewer times, fewer columns give more workgroups.  One tile of 16 columns up to 4096
// (256 workgroups), two up to 9216, then four; eight waves share the blocks, four of the widest.  In us for 1 / 2 / 4 tiles:
//   4096 x 3584, 1 row 5.8 / 7.3 / 10.6, 16 rows 8.1 / 9.7 / 12.7     6912 x 5120, 1 row 10.9 / 9.3 / 13.9, 16 rows 17.0 / 12.5 / 16.7
//   14336 x 4096, 1 row 18.2 / 16.4 / 16.5, 16 rows 25.8 / 20.0 / 17.5     32064 x 4096, 16 rows 48 / 36 / 31
// and with 4 / 8 / 16 waves, 1 row, 4096 x 3584: 6.6 / 5.8 / 6.1; four tiles with 2 / 4 / 8, 16 rows, 151936 x 896: 33 / 32 / 41.
//   Bound by how fast the weights come, up to 5.2 TB/s (1 row, 151936 x 896: 26 us), and at 16 rows by x, which every
// workgroup reads: 6912 x 5120 take 9.3 us for one row.  More blocks in flight per wave (2 to 6) lost 5 to 50 %.
template <int TT, int X>
void launch_few_rows(const ProductArgs& a, hipStream_t st) {
  const uint32_t columns16 = direct_columns16(a.n);
  if (columns16 == 1) launch_direct<1, TT, direct_waves(1), X>(a, st);
  else if (columns16 == 2) launch_direct<2, TT, direct_waves(2), X>(a, st);
  else launch_direct<4, TT, direct_waves(4), X>(a, st);
}

// ------------------------------------------------------------------ large products

// 16 bytes per lane from memory to LDS, at `to` + 16 * lane; nothing passes through registers.  As a buffer access its
// address is the tile's base, the lane's offset and the step's, with no arithmetic in between.
typedef __amdgpu_buffer_rsrc_t Buffer;
// What lies `bytes` and more behind its base is not read, and counts as 0.
__device__ __forceinline__ Buffer buffer_at(const uint8_t* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, bytes, 0x00027000);  // raw, 32-bit data
}
__device__ __forceinline__ void copy_to_lds(Buffer from, uint32_t lane_at, uint32_t at, uint8_t* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, (int)lane_at, (int)at, 0, 0);
}
// 4 bytes per lane.
__device__ __forceinline__ void copy_words_to_lds(Buffer from, uint32_t lane_at, uint32_t at, uint8_t* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 4, (int)lane_at, (int)at, 0, 0);
}

// Every wave's copies but the LEFT latest ones have landed, and all of them see that; all LDS reads are done.  The wait is
// written out: a barrier alone orders the LDS accesses that the compiler sees, and leaves copies to LDS on their way.
template <int LEFT = 0>
__device__ __forceinline__ void landed_barrier() {
  static_assert(LEFT < 64, "a 6-bit counter");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (LEFT & 15) | (LEFT >> 4) << 14);  // vmcnt(LEFT), lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Work item b of a product: a tile (m0, n0) and its blocks [j0, j1), one split's.  Each XCD takes a contiguous eighth
// of the items; the tiles of a split follow one another in bands of kBand tiles down, so that the workgroups running at
// once on an XCD share rows of both operands in its L2.  A launch takes `count` tiles from `first` on, in this order; or,
// as `quarters`, the four BM x BN parts of each of that many tiles of twice the size, which may lie outside of c.
constexpr uint32_t kBand = 8;
struct Item {
  uint32_t m0, n0, split, j0, j1;
};
__device__ __forceinline__ uint32_t same(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint32_t items_of(const ProductArgs& p) { return p.count * p.splits << 2 * p.quarters; }
template <int BM, int BN>
__device__ __forceinline__ Item item_of(const ProductArgs& p, uint32_t b) {
  const uint32_t at = xcd_tile(b, items_of(p)), part = at & (p.quarters * 3), all = at >> 2 * p.quarters;
  const uint32_t split = all / p.count, t = p.first + all % p.count;
  const uint32_t band = t / (kBand * p.tiles_n), high = min(kBand, p.tiles_m - band * kBand), i = t - band * kBand * p.tiles_n;
  const uint32_t y = ((band * kBand + i % high) << p.quarters) + part % 2, x = (i / high << p.quarters) + part / 2;
  // the same for the whole workgroup, which the compiler does not see behind the divisions
  return Item{same(y * BM), same(x * BN), same(split), same((uint32_t)((uint64_t)p.kb * split / p.splits)),
              same((uint32_t)((uint64_t)p.kb * (split + 1) / p.splits))};
}

// Results of a wave, TM * 32 rows by TN * 32 columns from (m0, n0), through TN * 2 KiB of LDS of its own: 32 rows of all
// columns in bf16 or of half of them in fp32 at a time, so that they leave as runs of whole lines.  A row's 16-byte pieces
// lie at piece ^ row % pieces.  VEC: rows of c are whole 16-byte pieces and a lane stores one, else one element.
//   Everything is one run of instructions without branches (the accumulators would leave their registers all at once
// ahead of one): c is a buffer, what lies outside of it gets an offset past its end, and where nothing is accumulated
// the buffer that c is read from is empty.
// bf16_pair, but where it stands: the compiler would convert a wave's whole results at once, ahead of all parts.
__device__ __forceinline__ uint32_t bf16_pair_here(float lo, float hi) {
  uint32_t r;
  asm volatile("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(r) : "v"(lo), "v"(hi));
  return r;
}

constexpr uint32_t kOutside = 1u << 31;  // 128 rows of c lie within it (kMaxRowBytes)
template <int TM, int TN, int BYTES, bool VEC>
__device__ __forceinline__ void store_turned(const ProductArgs& p, const f32x16 (&acc)[TN][TM], uint8_t* lds, uint32_t m0, uint32_t n0, uint32_t lane) {
  constexpr int kXs = TN * 2 / BYTES, kPitch = TN * 64, kPiecesRow = kPitch / 16, kMask = kPiecesRow - 1, kElems = 16 / BYTES;
  constexpr int kSize = VEC ? 16 : BYTES, kAcross = kPitch / kSize, kTimes = 32 * kPitch / kSize / 64;
  static_assert((kPiecesRow & kMask) == 0 && kXs * 32 * BYTES == kPitch, "rows of a power of two of pieces");
  const uint32_t r = lane & 31, g = lane >> 5, row_bytes = (uint32_t)p.c_stride * BYTES;
  const uint8_t* base = static_cast<const uint8_t*>(p.c) + ((int64_t)m0 * p.c_stride + n0) * BYTES;
  const Buffer c = buffer_at(base, kOutside), old = buffer_at(base, p.accumulate ? kOutside : 0u);
#pragma unroll
  for (int y = 0; y < TM; ++y)
#pragma unroll
    for (int x0 = 0; x0 < TN; x0 += kXs) {
      __builtin_amdgcn_sched_barrier(0);  // one part at a time: the registers hold no more
      uint32_t at[VEC ? kTimes : 1];
      f32x4 before[VEC && BYTES == 4 ? kTimes : 1];
      // offset in c of what the lane stores at time i, and its place in the LDS
      auto place = [&](int i, uint32_t& from) {
        const uint32_t unit = i * 64 + lane, row = unit / kAcross, col = unit % kAcross * (kSize / BYTES);
        from = row * kPitch + ((col / kElems ^ (row & kMask)) * 16) + col % kElems * BYTES;
        const bool in = m0 + y * 32 + row < p.m && n0 + x0 * 32 + col < p.n;
        return in ? (y * 32 + row) * row_bytes + (x0 * 32 + col) * BYTES : kOutside;
      };
      if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
          uint32_t from;
          at[i] = place(i, from);
          if constexpr (BYTES == 4) before[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(old, (int)at[i], 0, 0));
        }
      }
#pragma unroll
      for (int x = 0; x < kXs; ++x)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x16& a = acc[x0 + x][y];
          const uint32_t col = x * 32 + q * 8 + g * 4;
          uint8_t* to = lds + r * kPitch + ((col / kElems) ^ (r & kMask)) * 16;
          if (BYTES == 2)
            *reinterpret_cast<u32x2*>(to + col % 8 * 2) = u32x2{bf16_pair_here(a[q * 4], a[q * 4 + 1]), bf16_pair_here(a[q * 4 + 2], a[q * 4 + 3])};
          else
            *reinterpret_cast<f32x4*>(to) = f32x4{a[q * 4], a[q * 4 + 1], a[q * 4 + 2], a[q * 4 + 3]};
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < kTimes; ++i) {
        uint32_t from;
        const uint32_t to = place(i, from);
        if constexpr (VEC) {
          u32x4 w = *reinterpret_cast<const u32x4*>(lds + from);
          if constexpr (BYTES == 4) w = __builtin_bit_cast(u32x4, before[i] + __builtin_bit_cast(f32x4, w));
          __builtin_amdgcn_raw_buffer_store_b128(w, c, (int)at[i], 0, 0);
        } else if constexpr (BYTES == 2) {
          __builtin_amdgcn_raw_buffer_store_b16(*reinterpret_cast<const uint16_t*>(lds + from), c, (int)to, 0, 0);
        } else {
          const float v = *reinterpret_cast<const float*>(lds + from) + __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(old, (int)to, 0, 0));
          __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), c, (int)to, 0, 0);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
}

// Tiles of BM x BN of c, one after another per workgroup of WM * WN waves.  A step stages one 128-column block of BM rows of
// a and BN rows of b in LDS (copied straight there, two buffers in turn), each row's eight 16-byte pieces at piece ^ row /
// 2 % 8: the sixteen lanes that read at once, the same piece of sixteen rows, then meet all 64 banks.  The copies run two
// blocks ahead of the products and through the ends of tiles: while a tile's results leave, the next one's first blocks
// are on their way.  Every item has two blocks or more, or (ONE) a single one.
//   S > 2: that many buffers, for workgroups that have a CU to themselves and take one item each.  The copies then run S
// blocks ahead, and the scale codes come with them, a word (four blocks' codes) per row: loaded to registers they would have
// to wait for the copies before them.
//   Long products are bound by power: 8192 x 14336 x 4096 take 385 us (2500 TFLOP/s; 410 on a card that gets less) with the matrix units busy 64 % of the
// cycles at a clock of about 1.8 GHz, exact sums 700 to 750 us.  Few rows are bound by how fast b comes: 61 x 151936 x 896
// 36 us (4.7 TB/s); short K by the start and end of tiles: 768 x 9728 x 896 13 us.
template <int BM, int BN, int WM, int WN, int BYTES, bool VEC, bool FAST, bool ONE, int S>
__global__ __launch_bounds__(64 * WM * WN) void product_tile_kernel(ProductArgs p) {
  constexpr int kWaves = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, kRows = BM + BN, kCopies = kRows / 8 / kWaves;
  static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0 && kRows % (8 * kWaves) == 0 && BM % (8 * kWaves) == 0, "tile");
  // the stages, and each wave's part for its results: one array, since between accesses to arrays that it can tell apart
  // the compiler waits for the copies on their way
  constexpr bool DEEP = S > 2;
  constexpr int kStage = kRows * (DEEP ? 132 : 128), kCodes = kRows * 128, kPerStep = kCopies + 1;  // (DEEP) copies of a step
  static_assert(!DEEP || (kRows == 64 * kWaves && BM % 64 == 0 && !ONE), "a wave copies the codes of 64 rows of one side");
  __shared__ __align__(16) uint8_t lds[S * kStage + kWaves * TN * 2048];
  const uint32_t lane = threadIdx.x & 63, r = lane & 31, g = lane >> 5;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t wm = wave % WM * (TM * 32), wn = wave / WM * (TN * 32);
  const uint32_t items = items_of(p);

  // The copying side.  Rows [0, BM) of a stage are a's, the others b's.  What changes from tile to tile is the same for all
  // lanes (ProductSource).  Rows past the matrix are beyond the buffer; scale codes past it are some other row's (a
  // matrix's scales are a 128th of its data, below 2^32 bytes).
  auto source_of = [&](const Item& t) { return product_source(p.a, p.b, BM, BN, t.m0, t.n0, t.j0, t.j1); };
  ProductSource source, upcoming;
  uint32_t from[kCopies], acode[TM], bcode[TN];
#pragma unroll
  for (int i = 0; i < kCopies; ++i) {
    const uint32_t row = (i * kWaves + wave) * 8 + lane / 8, piece = (lane % 8) ^ (row / 2 % 8);
    from[i] = (i * kWaves * 8 < BM ? row * (uint32_t)p.a.stride : (row - BM) * (uint32_t)p.b.stride) + piece * 16;
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) acode[i] = 4 * ((wm + i * 32 + r) >> p.a.sh);
#pragma unroll
  for (int i = 0; i < TN; ++i) bcode[i] = 4 * ((wn + i * 32 + r) >> p.b.sh);
  const Buffer ascales = buffer_at(p.a.scales, (p.kb + 3) / 4 * p.a.srows * 4), bscales = buffer_at(p.b.scales, (p.kb + 3) / 4 * p.b.srows * 4);
  auto stage = [&](uint8_t* to, int i) {
    copy_to_lds(i * kWaves * 8 < BM ? buffer_at(source.a, source.abytes) : buffer_at(source.b, source.bbytes), from[i], source.block * 128,
                to + (i * kWaves + wave) * 1024);
  };
  const bool a_codes = wave * 64 < BM;
  const uint32_t code_at = 4 * (a_codes ? (wave * 64 + lane) >> p.a.sh : (wave * 64 + lane - BM) >> p.b.sh);
  auto stage_codes = [&](uint8_t* to) {
    if (a_codes) copy_words_to_lds(ascales, code_at, source.acodes + source.block / 4 * p.a.srows * 4, to + kCodes + wave * 256);
    else copy_words_to_lds(bscales, code_at, source.bcodes + source.block / 4 * p.b.srows * 4, to + kCodes + wave * 256);
  };
  auto advance = [&] { next_block(source, upcoming); };
  struct Scales {
    int a[TM], b[TN];
  };
  auto load_scales = [&] {
    const uint32_t aat = source.acodes + source.block / 4 * p.a.srows * 4 + source.block % 4;
    const uint32_t bat = source.bcodes + source.block / 4 * p.b.srows * 4 + source.block % 4;
    Scales s;
#pragma unroll
    for (int t = 0; t < TM; ++t) s.a[t] = __builtin_amdgcn_raw_buffer_load_b8(ascales, (int)acode[t], (int)aat, 0);
#pragma unroll
    for (int t = 0; t < TN; ++t) s.b[t] = __builtin_amdgcn_raw_buffer_load_b8(bscales, (int)bcode[t], (int)bat, 0);
    return s;
  };

  // (DEEP) of the block staged at `from_lds`
  auto read_scales = [&](const uint8_t* from_lds, uint32_t block) {
    const uint32_t* words = reinterpret_cast<const uint32_t*>(from_lds + kCodes);
    Scales s;
#pragma unroll
    for (int t = 0; t < TM; ++t) s.a[t] = (int)(words[wm + t * 32 + r] >> block % 4 * 8 & 255);
#pragma unroll
    for (int t = 0; t < TN; ++t) s.b[t] = (int)(words[BM + wn + t * 32 + r] >> block % 4 * 8 & 255);
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
  f32x16 acc[TN][TM];
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

  // A step: the second half of the block in stage `in` is read while its first is multiplied; then, once every wave has read
  // all of it and the next block has landed in the other buffer, the block after that starts on its way into stage `in` and
  // the first half of the next one is read while the second half of this one is multiplied.
  Codes first;
  Scales now, next;
  uint32_t in = 0;
  auto step = [&](uint32_t following) {  // the block after this one
    const uint32_t in_next = in + 1 == S ? 0 : in + 1;
    uint8_t *cur = lds + in * kStage, *other = lds + in_next * kStage;
    Codes second;
    multiply(first, now, [&](int i) {
#pragma unroll
      for (int k = i * kPieces / kTiles; k < (i + 1) * kPieces / kTiles; ++k) second.piece[k] = read_piece(cur, 1, k);
    });
    landed_barrier<DEEP ? (S - 2) * kPerStep : 0>();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!DEEP) {
      // used from here on only: copied any earlier, they would be waited for there, and all copies with them
#pragma unroll
      for (int t = 0; t < TM; ++t) asm volatile("" : "+v"(next.a[t]));
#pragma unroll
      for (int t = 0; t < TN; ++t) asm volatile("" : "+v"(next.b[t]));
    }
    const Scales landed = DEEP ? read_scales(other, following) : next;
    advance();
    if constexpr (DEEP) stage_codes(cur);
    else next = load_scales();
    multiply(second, now, [&](int i) {
#pragma unroll
      for (int k = i * kPieces / kTiles; k < (i + 1) * kPieces / kTiles; ++k) first.piece[k] = read_piece(other, 0, k);
#pragma unroll
      for (int k = i * kCopies / kTiles; k < (i + 1) * kCopies / kTiles; ++k) stage(cur, k);
    });
    now = landed;
    in = in_next;
  };

  Item t = item_of<BM, BN>(p, blockIdx.x);
  source = upcoming = source_of(t);
  if constexpr (DEEP) {
    no_product_source(upcoming);
#pragma unroll
    for (int b = 0; b < S; ++b) {
      if (b) advance();
      stage_codes(lds + b * kStage);
#pragma unroll
      for (int i = 0; i < kCopies; ++i) stage(lds + b * kStage, i);
    }
    landed_barrier<(S - 1) * kPerStep>();
    now = read_scales(lds, t.j0);
  } else if constexpr (!ONE) {
    now = load_scales();
#pragma unroll
    for (int i = 0; i < kCopies; ++i) stage(lds, i);
    advance();
    next = load_scales();
#pragma unroll
    for (int i = 0; i < kCopies; ++i) stage(lds + kStage, i);
    landed_barrier();
  }
  if constexpr (!ONE) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) first.piece[i] = read_piece(lds, 0, i);
  }
  for (uint32_t b = blockIdx.x; b < items; b += gridDim.x) {
#pragma unroll
    for (int x = 0; x < TN; ++x)
#pragma unroll
      for (int y = 0; y < TM; ++y) acc[x][y] = f32x16{};
    const Item done = t;
    const bool more = b + gridDim.x < items;
    if (more) t = item_of<BM, BN>(p, b + gridDim.x);
    upcoming = source_of(t);
    if (!more) no_product_source(upcoming);
    if constexpr (ONE) {
      __syncthreads();  // every wave has read the block before
      now = load_scales();
#pragma unroll
      for (int i = 0; i < kCopies; ++i) stage(lds, i);
      landed_barrier();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) first.piece[i] = read_piece(lds, h, i);
        multiply(first, now, [](int) {});
      }
      source = upcoming;
    } else {
      uint32_t j = done.j0;
      do step(j + 1);
      while (++j < done.j1);
    }
    // the results are read by instructions written out (bf16_pair_here), whose distance from the matrix instructions that
    // write them, 19 wait states at most, the compiler does not keep by itself
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 15");
    __builtin_amdgcn_sched_barrier(0);
    // the lane as if it were new each time: addresses made from it and kept through the steps would not fit the registers
    uint32_t me = lane;
    asm volatile("" : "+v"(me));
    ProductArgs out = p;
    out.c = static_cast<uint8_t*>(p.c) + done.split * p.split_bytes;
    store_turned<TM, TN, BYTES, VEC>(out, acc, lds + S * kStage + wave * TN * 2048, done.m0 + wm, done.n0 + wn, me);
  }
  landed_barrier();  // no copy is on its way any more when the LDS goes to another workgroup
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

// Workgroups with a CU to themselves stage four blocks, in the LDS of the second one that is not there: fast sums of 512 x
// 6912 x 5120 in 24 us instead of 35 (up to 31 where less of it lies in the last cache), 100 x 32064 x 4096 37 (46), 2048 x 2000 x 2000 14 (17).  Exact sums are not faster (512 x
// 896 x 4864 20.6 and 19.9), nor are items of two or three blocks (200 x 688 x 256 5.7 and 5.4).
constexpr uint32_t kCus = 256;
constexpr int kDeep = 4;
template <int BM, int BN, int BYTES, bool VEC, bool ONE>
void launch_items(const ProductArgs& a, bool fast, hipStream_t st) {
  // as many workgroups as the LDS of all CUs holds; a multiple of the XCDs keeps a workgroup's items on its XCD
  constexpr uint32_t kResident = kCus * (160 / ((BM + BN) / 4 + BN / 8));
  const uint32_t items = a.count * a.splits << 2 * a.quarters;
  const dim3 grid(std::min(items, kResident)), block(256);
  if constexpr (BM + BN == 256 && !ONE) {
    if (fast && items <= kCus && a.kb >= kDeep * a.splits) {
      hipLaunchKernelGGL((product_tile_kernel<BM, BN, 2, 2, BYTES, VEC, true, false, kDeep>), grid, block, 0, st, a);
      return;
    }
  }
  if (fast) hipLaunchKernelGGL((product_tile_kernel<BM, BN, 2, 2, BYTES, VEC, true, ONE, 2>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((product_tile_kernel<BM, BN, 2, 2, BYTES, VEC, false, ONE, 2>), grid, block, 0, st, a);
}

// All tiles but the last `quartered` ones of 256 x 256, and these as tiles of 128 x 128 in a second launch, two to a CU:
// 8192 x 6912 x 5120, 864 tiles for 256 CUs, in 269 us instead of 292 with a fourth round for the last 96.
template <int BM, int BN, int BYTES, bool VEC, bool ONE>
void launch_tiles(ProductArgs a, uint32_t quartered, bool fast, hipStream_t st) {
  a.tiles_m = (uint32_t)ceil_div(a.m, BM);
  a.tiles_n = (uint32_t)ceil_div(a.n, BN);
  a.first = a.quarters = 0;
  a.count = a.tiles_m * a.tiles_n - quartered;
  launch_items<BM, BN, BYTES, VEC, ONE>(a, fast, st);
  if constexpr (BM == 256 && BN == 256) {
    if (!quartered) return;
    a.first = a.count;
    a.count = quartered;
    a.quarters = 1;
    launch_items<128, 128, BYTES, VEC, ONE>(a, fast, st);
  }
}

// Tiles of 256 want rows of whole 16-byte pieces and two blocks or more.
template <int BYTES>
void launch_tile_kind(const ProductArgs& a, const ProductPlan& plan, bool fast, hipStream_t st) {
  if (a.kb == 1) {
    if (a.c_vec) launch_tiles<128, 128, BYTES, true, true>(a, 0, fast, st);
    else launch_tiles<128, 128, BYTES, false, true>(a, 0, fast, st);
  } else if (a.c_vec) {
    if (plan.kind == ProductPlan::kTile256) launch_tiles<256, 256, BYTES, true, false>(a, plan.quartered, fast, st);
    else launch_tiles<128, 128, BYTES, true, false>(a, 0, fast, st);
  } else {
    launch_tiles<128, 128, BYTES, false, false>(a, 0, fast, st);
  }
}

void launch_tile(const ProductArgs& a, const ProductPlan& plan, bool fast, hipStream_t st) {
  if (a.splits == 1) {
    if (a.c_bf16) launch_tile_kind<2>(a, plan, fast, st);
    else launch_tile_kind<4>(a, plan, fast, st);
    return;
  }
  ProductArgs parts = a;
  parts.c = a.part;
  parts.c_stride = a.part_stride;
  parts.split_bytes = (int64_t)a.m * a.part_stride * (int64_t)sizeof(float);
  parts.c_vec = 1;
  parts.n = (uint32_t)a.part_stride;  // columns past b's last one: sums of zeros
  parts.accumulate = 0;
  launch_tile_kind<4>(parts, plan, fast, st);
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
  const int size = l.c_bf16 ? 2 : 4;
  a.c_vec = reinterpret_cast<uintptr_t>(l.c) % 16 == 0 && l.c_stride * size % 16 == 0;
  a.c_bf16 = l.c_bf16;
  a.accumulate = l.accumulate;
  if (l.x) {
    const bool shorter = l.a.cols < 8;
    if (l.x_bf16) {
      if (shorter) launch_direct<1, 1, 8, kBf16 | kShort>(a, st);
      else launch_few_rows<1, kBf16>(a, st);
    } else {
      if (shorter) launch_direct<1, 1, 8, kF32 | kShort>(a, st);
      else launch_few_rows<1, kF32>(a, st);
    }
  } else if (const ProductPlan plan = plan_product(l.m, l.n, l.kb, l.fast); plan.kind != ProductPlan::kDirect && l.c_stride * size < kMaxRowBytes) {
    a.splits = plan.splits;
    a.split_bytes = 0;
    if (l.n * (int64_t)size % 16) a.c_vec = 0;  // whole pieces only
    a.part = static_cast<float*>(l.workspace);
    a.part_stride = part_stride(l.n);
    launch_tile(a, plan, l.fast, st);
  } else {
    switch (plan.rows16) {
      case 1: launch_few_rows<1, kCodes>(a, st); break;
      case 2: launch_few_rows<2, kCodes>(a, st); break;
      case 3: launch_few_rows<3, kCodes>(a, st); break;
      default: launch_few_rows<4, kCodes>(a, st);
    }
  }
  return hipGetLastError();
}

}  // namespace dr
