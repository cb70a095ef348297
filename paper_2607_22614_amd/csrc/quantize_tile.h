// Quantization of a tile of 128 x 128 elements that a workgroup holds in registers as they lie in memory (quantize.hip), and what
// it has in common with that of computed values (quantize_values.h): the places of tiles and lanes, and the scale codes.
#pragma once

#include <hip/hip_runtime.h>

#include "quant_device.h"

namespace dr {

// Scale code of block (i, j) of a matrix with R block rows, and 127 in the unused bytes of its last word.
__device__ __forceinline__ void put_code(const QView& q, uint32_t i, uint32_t j, uint32_t code) {
  const uint32_t blocks = (q.cols + 127) / 128;
  uint8_t* p = q.scales + ((int64_t)(j >> 2) * q.srows + i) * 4;
  p[j & 3] = (uint8_t)code;
  if (j + 1 == blocks)
    for (uint32_t k = (j & 3) + 1; k < 4; ++k) p[k] = 127;
}

// kTileLanes lanes, of which each holds 8 columns (16 lanes side by side) of kTileRows rows.
constexpr int kTileRows = 128 / (kTileLanes / 16), kTileWaves = kTileLanes / 64;

template <bool COLS>
struct TileSpace {
  uint32_t cmax[kTileWaves][128];
  __align__(16) uint8_t turned[COLS ? 128 * 128 : 16];
};

// Tile (rt, ct) of a workgroup, and the lane's first row and column.
//   Tiles go in bands of four down, and 32 of them to an XCD at a time: runs of 512 to 1024 bytes of q's and qt's rows then
// leave one L2 (8192 x 4096 fp32 both ways 43 us, in the order of the rows 45; 3000 x 3001 bf16 10.8 and 11.6).
constexpr uint32_t kBandT = 4, kTurn = 32;
struct TilePlace {
  uint32_t rt, ct, row0, col;
};
// The t-th of `tiles` tiles, in bands of BAND tiles down.
template <uint32_t BAND>
__device__ __forceinline__ TilePlace place_of(uint32_t t, uint32_t tiles, uint32_t tiles_x) {
  const uint32_t tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const uint32_t tiles_y = tiles / tiles_x, band = t / (BAND * tiles_x);
  const uint32_t high = min(BAND, tiles_y - band * BAND), i_band = t - band * BAND * tiles_x;
  const uint32_t rt = band * BAND + i_band % high, ct = i_band / high;
  return TilePlace{rt, ct, rt * 128 + ty * kTileRows, ct * 128 + tx * 8};
}

__device__ __forceinline__ TilePlace tile_place(uint32_t tiles_x) { return place_of<kBandT>(xcd_group<kTurn>(blockIdx.x, gridDim.x), gridDim.x, tiles_x); }

// Codes and scales of a tile whose elements behind the matrix's last row and column are 0: into q as they are (ROWS) and
// into qt, whose rows are q's columns (COLS).  SQUARE: one scale for the tile, else one per row (DPP) and one per column (over
// the four rows of lanes, then over the waves in LDS).  The transpose's codes are packed 4 rows to a word, turned in LDS (one
// 128-byte row per column, its words spread by an exclusive or over the banks), and leave as whole 128-byte rows.
template <bool BF16, bool SQUARE, bool ROWS, bool COLS>
__device__ __forceinline__ void quantize_tile(const Raw8<BF16> (&v)[kTileRows], const TilePlace& at, const QView& q, const QView& qt,
                                              TileSpace<COLS>& space) {
  constexpr int R = kTileRows, kWaves = kTileWaves;
  const uint32_t rows = ROWS ? q.rows : qt.cols, cols = ROWS ? q.cols : qt.rows;
  const uint32_t tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, wave = tid / 64;
  const uint32_t rt = at.rt, ct = at.ct, row0 = at.row0, col = at.col;
  // the lane's largest magnitude of each row; finite ones only if any is not
  uint32_t rmax[R], top = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) top = max(top, rmax[i] = row_max(v[i], false));
  const bool odd = __any(top >= kInfBits);
  if (odd) {
    top = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) top = max(top, rmax[i] = row_max(v[i], true));
  }

  uint32_t square_code = 0;
  if (SQUARE) {
    const uint32_t m = max_rows(max16(top));
    if ((tid & 63) == 0) space.cmax[0][wave] = m;
    __syncthreads();
    uint32_t most = space.cmax[0][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) most = max(most, space.cmax[0][w]);
    square_code = scale_code(most);
    if (tid == 0) {
      if (ROWS) put_code(q, rt, ct, square_code);
      if (COLS) put_code(qt, ct, rt, square_code);
    }
  }

  if (ROWS) {
    uint32_t mine = 0;  // of row row0 + tx
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint32_t code = SQUARE ? square_code : scale_code(max16(rmax[i]));
      mine = tx == (uint32_t)i ? code : mine;
      if (row0 + i < rows)
        *reinterpret_cast<u32x2*>(q.data + (int64_t)(row0 + i) * q.stride + col) = row_codes(v[i], code);
    }
    if (!SQUARE && tx < R && row0 + tx < rows) put_code(q, row0 + tx, ct, mine);
  }

  if (COLS) {
    uint32_t code[8], mine = 0;  // of column col + ty
    if (SQUARE) {
#pragma unroll
      for (int j = 0; j < 8; ++j) code[j] = square_code;
    } else {
      uint32_t most[BF16 ? 4 : 8] = {};
      auto column_max = [&](bool finite) {
#pragma unroll
        for (int w = 0; w < (BF16 ? 4 : 8); ++w)
#pragma unroll
          for (int i = 0; i < R; ++i) most[w] = larger<BF16>(most[w], magnitude<BF16>(v[i].w[BF16 ? 0 : w / 4][w % 4], finite));
      };
      if (odd) column_max(true);
      else column_max(false);
#pragma unroll
      for (int w = 0; w < (BF16 ? 4 : 8); ++w) {
        uint32_t m = most[w];
        m = larger<BF16>(m, (uint32_t)__shfl_xor((int)m, 16));
        m = larger<BF16>(m, (uint32_t)__shfl_xor((int)m, 32));
        if ((tid & 63) < 16) {
          if (BF16) {
            space.cmax[wave][tx * 8 + 2 * w] = m << 16;
            space.cmax[wave][tx * 8 + 2 * w + 1] = m & 0xFFFF0000u;
          } else {
            space.cmax[wave][tx * 8 + w] = m;
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = tx * 8 + j;
        uint32_t m = space.cmax[0][c];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = max(m, space.cmax[w][c]);
        code[j] = scale_code(m);
        mine = ty == (uint32_t)j ? code[j] : mine;
      }
      if (ty < 8 && col + ty < cols) put_code(qt, col + ty, rt, mine);
    }
    // word ty of a column lies at ty ^ 4 (tx % 8), which keeps its 16-byte pieces together
#pragma unroll
    for (int j = 0; j < 8; ++j)
      *reinterpret_cast<uint32_t*>(space.turned + (tx * 8 + j) * 128 + (ty ^ (tx % 8 * 4)) * 4) = column_codes<BF16>(v, j, code[j]);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 128 * 8 / kTileLanes; ++r) {
      const uint32_t c = r * (kTileLanes / 8) + tid / 8, piece = tid % 8;
      const u32x4 w = *reinterpret_cast<const u32x4*>(space.turned + c * 128 + (piece ^ (c / 8 % 8)) * 16);
      if (ct * 128 + c < cols)
        *reinterpret_cast<u32x4*>(qt.data + (int64_t)(ct * 128 + c) * qt.stride + rt * 128 + piece * 16) = w;
    }
  }
}

}  // namespace dr
