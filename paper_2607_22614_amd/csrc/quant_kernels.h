// Launches of the 8-bit kernels (quantize.hip, qmatmul.hip) and of the gradient kernels
// (grad_clip.hip): plain arguments, checked by the host code that fills them (quant.cpp,
// grads.cpp).  Each wrapper enqueues on `st` and returns hipGetLastError().
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dr.h"

namespace dr {

constexpr int64_t kBlock = DR_QUANT_BLOCK;
constexpr int64_t kMaxQRows = 1ll << 26;  // exclusive: 16 rows a workgroup of 512 lanes is 2^31 lanes
constexpr int64_t kMaxQCols = 1ll << 23;  // 256 rows of a tile lie within 2^31 bytes

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// One operand as the kernels see it; sh: log2 of block_rows, srows: block rows.
struct QView {
  uint8_t* data;
  uint8_t* scales;
  int64_t stride;
  uint32_t rows, cols, srows;
  int32_t sh;
};

struct QuantizeLaunch {
  const void* src;
  int64_t src_stride;  // elements
  uint32_t rows, cols;
  bool bf16;
  QView q, qt;         // data null: not wanted
};
hipError_t launch_quantize(const QuantizeLaunch& l, hipStream_t st);
// Whether rows begin at whole 16 bytes and consist of them, so that every load of 16 bytes of theirs is aligned.
inline bool whole_pieces(const void* src, int64_t stride, int64_t cols, int64_t size) {
  return reinterpret_cast<uintptr_t>(src) % 16 == 0 && stride * size % 16 == 0 && cols * size % 16 == 0;
}
// Lanes of a workgroup that takes a tile of 128 x 128; a launch of rows alone has fewer of them in all.
constexpr int kTileLanes = 512;

// c (m x n) = a (m x k) * b^T (n x k), kb = ceil(k / 128) column blocks.
struct ProductLaunch {
  QView a, b;
  const void* x;     // set: a is quantized in the kernel from these rows
  int64_t x_stride;  // elements
  bool x_bf16;
  void* c;
  int64_t c_stride;  // elements
  uint32_t m, n, kb;
  bool c_bf16, accumulate, fast;
  void* workspace;
};
hipError_t launch_product(const ProductLaunch& l, hipStream_t st);
// Rows that launch_product quantizes itself.
constexpr uint32_t kFusedRows = 16;

// How a product of 8-bit operands is cut: tiles of one of two sizes, and each tile's blocks over `splits` workgroups
// whose fp32 sums lie in the workspace until a second kernel joins them; or the kernel for few rows, `rows16` times 16 of them
// per workgroup.  The last `quartered` tiles of 256 x 256 are cut into tiles of 128 x 128 each.
struct ProductPlan {
  enum Kind { kDirect, kTile128, kTile256 } kind;
  uint32_t splits;
  uint32_t quartered;
  uint32_t rows16;  // of kDirect: 1 to 4
};
// Tiles of 16 columns per workgroup of the kernel for few rows, and its waves, by the columns of c.
inline uint32_t direct_columns16(int64_t n) { return n <= 4096 ? 1 : n <= 9216 ? 2 : 4; }
constexpr uint32_t direct_waves(uint32_t columns16) { return columns16 == 4 ? 4 : 8; }

// Workgroups of `lanes` lanes that one launch holds: it counts lanes in 32 bits.
constexpr uint32_t max_workgroups(uint32_t lanes) { return 0xFFFFFFFFu / lanes; }

// Bytes from row to row of c that the tiles can store to: the last of 128 rows begins below 2^31 bytes.  The kernel for few rows
// takes what lies further apart.
constexpr int64_t kMaxRowBytes = 1ll << 24;

inline int64_t part_stride(int64_t n) { return ceil_div(n, 4) * 4; }

ProductPlan plan_product(int64_t m, int64_t n, int64_t kb, bool fast);

}  // namespace dr
