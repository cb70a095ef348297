// What a workgroup of the tiled products (qmatmul.hip) copies to LDS, block by block.  Plain arithmetic on the host and on
// the device, so that the CPU tests run what the kernel runs.
#pragma once

#include <hip/hip_runtime.h>

#include "quant_kernels.h"

namespace dr {

// The operands of an item from its next block on: where the tile's rows begin and how many bytes of them there are, where
// their scale codes begin, and the blocks [block, end).
//   The copies are buffer accesses: a lane's offset counts as inside where it is below the length less the scalar offset
// (the block's, or the scale codes'), and a difference below 0 need not count as one.  So that none comes about, every item has
// a row of either operand at least: a tile outside of c (a quarter may lie there) takes the matrix's last row, whose products
// nobody stores, and what stands behind the last item has no bytes and stays at block 0.
struct ProductSource {
  const uint8_t *a, *b;
  uint32_t abytes, bbytes, acodes, bcodes, block, end;
  uint32_t bfirst;  // row of b
};

// Rows of an operand that a tile of `tile` rows from row `at` on reads.
struct StagedRows {
  uint32_t first, count;
};
__host__ __device__ __forceinline__ StagedRows staged_rows(uint32_t at, uint32_t tile, uint32_t rows) {
  const uint32_t first = at < rows ? at : rows - 1;
  return StagedRows{first, rows - first < tile ? rows - first : tile};
}

__host__ __device__ __forceinline__ ProductSource product_source(const QView& a, const QView& b, uint32_t tile_m, uint32_t tile_n, uint32_t m0,
                                                                 uint32_t n0, uint32_t j0, uint32_t j1) {
  const StagedRows m = staged_rows(m0, tile_m, a.rows), n = staged_rows(n0, tile_n, b.rows);
  return ProductSource{a.data + (int64_t)m.first * a.stride, b.data + (int64_t)n.first * b.stride, m.count * (uint32_t)a.stride,
                       n.count * (uint32_t)b.stride, (m.first >> a.sh) * 4, (n.first >> b.sh) * 4, j0, j1, n.first};
}

// Products of pairs (qgated.hip): 32 rows of b's part of a stage are the first rows of 32 pairs, the next 32 their second ones.
// Of row `at` of that part: the pair's place in the tile, and which row of the pair it is.
__host__ __device__ __forceinline__ uint32_t pair_of(uint32_t at) { return at / 64 * 32 + at % 32; }
__host__ __device__ __forceinline__ uint32_t second_of(uint32_t at) { return at / 32 % 2; }
// Offset of the scale code of row first + row among its column block's: the second rows may begin inside a square block.
__host__ __device__ __forceinline__ uint32_t pair_code_at(uint32_t first, uint32_t row, int32_t sh) { return 4 * ((first + row) >> sh); }

// Behind the last item: copies of nothing, which take no memory access.
__host__ __device__ __forceinline__ void no_product_source(ProductSource& s) { s.abytes = s.bbytes = s.block = s.end = 0; }

// To the next block, or the first one of the upcoming item.
__host__ __device__ __forceinline__ void next_block(ProductSource& s, const ProductSource& upcoming) {
  const bool same = ++s.block < s.end;
  s.a = same ? s.a : upcoming.a;
  s.b = same ? s.b : upcoming.b;
  s.abytes = same ? s.abytes : upcoming.abytes;
  s.bbytes = same ? s.bbytes : upcoming.bbytes;
  s.acodes = same ? s.acodes : upcoming.acodes;
  s.bcodes = same ? s.bcodes : upcoming.bcodes;
  s.bfirst = same ? s.bfirst : upcoming.bfirst;
  s.block = same ? s.block : upcoming.block;
  s.end = same ? s.end : upcoming.end;
}

}  // namespace dr
