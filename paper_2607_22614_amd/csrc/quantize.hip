// Quantization to e4m3 codes with a power of two for each block of 128 columns (dr_quantize).
//
// With amax the largest finite magnitude of a block, its scale is 2^e with e = ceil(log2(amax / 448)) and an
// element's code is x * 2^-e rounded to 4 significant bits.  Both multiplications by powers of two are
// exact, so the codes depend on nothing but the definition.
//
// HBM-bound: 2 or 4 bytes read and 1 byte written per element and orientation.  8192 x 5120 bf16 along the rows take 24.5 us from
// HBM (5.1 TB/s), fp32 42 (5.0); 8192 x 4096 both ways 29 (4.6; 25 where part of it lies in the last cache), fp32 43 (4.7); 8192 x 14336 99
// (4.7): a tile's codes leave only after all of it has come.
#include <hip/hip_runtime.h>

#include "quant_device.h"
#include "quantize_tile.h"
#include "quantize_values.h"

namespace dr {
namespace {

struct QuantizeArgs {
  const void* src;
  int64_t src_stride;
  uint32_t rows, cols, tiles_x;
  int32_t stream;
  QView q, qt;
};

// Eight columns of ROWS rows; rows past the matrix read its last one.  The sources of large calls are streamed past the
// caches, where their rows are whole 16 bytes (those that share lines with others take 13 instead of 10 us for 3000 x
// 3001 that way).  Streamed loads leave the last cache (256 MiB) to what the call writes, and
// do not profit from a source that lies there.  Between calls that go round among a few sets of buffers they win where all
// of the sets together pass the cache: from 128 MiB moved by a call with 2 sets, about 90 with 3, 64 to 72 with 4.  A
// call does not know the others; kCached (quant_kernels.h) is the line for somewhat less than 3.  In us, plain / streamed:
//                                  3 sets         from HBM       just written
//   4096 x 4096 bf16, rows       10.6 / 11.3     12.6 / 11.0     12.5 / 12.7
//   8192 x 4096 bf16, both ways  28.2 / 26.4     28.7 / 29.0     22.7 / 25.9
//   16384 x 4096 bf16, rows      38.7 / 35.5
//   8192 x 14336 bf16, rows                      66.9 / 64.7     57.5 / 61.7
//   16384 x 4096 fp32, rows      63.1 / 60.2
//   16384 x 4096 fp32, both ways 75.3 / 82.0, where it does not pay
template <bool BF16, int ROWS>
__device__ __forceinline__ void load_rows(const QuantizeArgs& a, uint32_t row0, uint32_t col, Raw8<BF16> (&v)[ROWS]) {
  auto each = [&](auto load) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) v[i] = load(a.src, (int64_t)min(row0 + i, a.rows - 1) * a.src_stride, col, a.cols);
  };
  if (a.cols < 8) each(load_short_row8<BF16>);
  else if (a.stream) each(load_row8<BF16, true>);
  else each(load_row8<BF16>);
  const uint32_t s = ahead8(col, a.cols);
  if (__any(s)) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) settle8(v[i], s);
  }
}

// Blocks of 1 x 128, rows only.  A wave takes 512 columns (four blocks, 16 lanes each, 8 elements a lane) of
// ROWS rows, whose loads are all in flight together; a block's maximum is a DPP reduction over its 16
// lanes, and the four codes of a row make the 32-bit word that one lane stores.
constexpr int kRowWaves = 4;

template <bool BF16, int ROWS>
__global__ __launch_bounds__(64 * kRowWaves) void quantize_rows_kernel(QuantizeArgs a) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const uint32_t quad = blockIdx.x % a.tiles_x;
  const uint32_t row0 = (blockIdx.x / a.tiles_x * kRowWaves + wave) * ROWS;
  if (row0 >= a.rows) return;
  const uint32_t col = quad * 512 + lane * 8;
  Raw8<BF16> v[ROWS];
  load_rows(a, row0, col, v);
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    uint32_t m = row_max(v[i], false);
    if (__any(m >= kInfBits)) m = row_max(v[i], true);
    const uint32_t code = scale_code(max16(m));
    const uint32_t codes = (uint32_t)__builtin_amdgcn_readlane((int)code, 0) | (uint32_t)__builtin_amdgcn_readlane((int)code, 16) << 8 |
                           (uint32_t)__builtin_amdgcn_readlane((int)code, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane((int)code, 48) << 24;
    if ((int)lane == i) word = codes;
    if (row0 + i < a.rows && (col & ~127u) < a.cols)
      *reinterpret_cast<u32x2*>(a.q.data + (int64_t)(row0 + i) * a.q.stride + col) = row_codes(v[i], code);
  }
  if (lane < ROWS && row0 + lane < a.rows)
    reinterpret_cast<uint32_t*>(a.q.scales)[(int64_t)quad * a.rows + row0 + lane] = word;
}

// A tile of 128 x 128 per workgroup, each lane 8 columns of 4 rows, kept in registers (of 8 rows by half the lanes: 200 x 256
// bf16 both ways 5.0 us instead of 4.5, 2000 x 4096 fp32 14.1 and 13.4).
template <bool BF16, bool SQUARE, bool ROWS, bool COLS>
__global__ __launch_bounds__(kTileLanes) void quantize_tile_kernel(QuantizeArgs a) {
  __shared__ TileSpace<COLS> space;
  const TilePlace at = tile_place(a.tiles_x);
  Raw8<BF16> v[kTileRows];
  load_rows(a, at.row0, at.col, v);
  if (at.row0 + kTileRows > a.rows) {
#pragma unroll
    for (int i = 0; i < kTileRows; ++i)
      if (at.row0 + i >= a.rows) v[i] = Raw8<BF16>{};
  }
  quantize_tile<BF16, SQUARE, ROWS, COLS>(v, at, a.q, a.qt, space);
}

// The transpose of an 8-bit matrix, quantized anew.  The values go through bf16, which holds them: 4 significant bits, and
// what lies below 2^-133 counts as 0 as in the products.  8192 x 4096 in 12.5 us, 8192 x 14336 in 47.5 (5.0 TB/s), 7 vector
// instructions an element; with those of quantize_tile, 11, 15.6 and 51.
struct TurnArgs {
  QView src, qt;
  uint32_t tiles_x;
};
__global__ __launch_bounds__(kTileLanes) void turn_tile_kernel(TurnArgs a) {
  __shared__ ValuesSpace space;
  const TilePlace at = place_of<16>(xcd_tile(blockIdx.x, gridDim.x), gridDim.x, a.tiles_x);
  clear_maxima(space);
  const uint32_t first = threadIdx.x / 16 * kTileRows, behind = a.src.rows - at.rt * 128, col = threadIdx.x % 16 * 8;
  const uint8_t* from = tile_at(a.src, at.rt * 128, at.ct * 128);
  const uint8_t* scales = a.src.scales + (int64_t)(at.ct >> 2) * a.src.srows * 4 + (at.ct & 3);
  u32x2 codes[kTileRows];
  uint32_t scale[kTileRows];
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    const uint32_t row = min(first + i, behind - 1);
    codes[i] = *reinterpret_cast<const u32x2*>(from + (row_offset(row, a.src.stride) + col));
    scale[i] = scales[(int64_t)((at.rt * 128 + row) >> a.src.sh) * 4];
  }
  lds_barrier();
  Raw8<true> v[kTileRows];
#pragma unroll
  for (int i = 0; i < kTileRows; ++i) {
    if (first + i >= behind) codes[i] = u32x2{};
    v[i] = bf16_values(codes[i], scale[i]);
  }
  put_columns(v, at, a.qt, space, 0);
}

// Eight rows a wave keep the loads of a long matrix in flight; where that leaves CUs without work, one.
template <bool BF16>
void launch_rows(const QuantizeArgs& a, hipStream_t st) {
  const uint32_t grid8 = a.tiles_x * (uint32_t)ceil_div(a.rows, 8 * kRowWaves);
  if (grid8 >= 512)
    hipLaunchKernelGGL((quantize_rows_kernel<BF16, 8>), dim3(grid8), dim3(64 * kRowWaves), 0, st, a);
  else
    hipLaunchKernelGGL((quantize_rows_kernel<BF16, 1>), dim3(a.tiles_x * (uint32_t)ceil_div(a.rows, kRowWaves)), dim3(64 * kRowWaves), 0, st, a);
}

template <bool BF16, bool SQUARE>
void launch_tiles(const QuantizeArgs& a, dim3 grid, hipStream_t st) {
  const dim3 block(kTileLanes);
  if (a.q.data && a.qt.data) {
    hipLaunchKernelGGL((quantize_tile_kernel<BF16, SQUARE, true, true>), grid, block, 0, st, a);
  } else if (a.qt.data) {
    hipLaunchKernelGGL((quantize_tile_kernel<BF16, SQUARE, false, true>), grid, block, 0, st, a);
  } else {
    if constexpr (SQUARE) hipLaunchKernelGGL((quantize_tile_kernel<BF16, true, true, false>), grid, block, 0, st, a);
  }
}

}  // namespace

hipError_t launch_quantize(const QuantizeLaunch& l, hipStream_t st) {
  QuantizeArgs a;
  a.src = l.src;
  a.src_stride = l.src_stride;
  a.rows = l.rows;
  a.cols = l.cols;
  a.q = l.q;
  a.qt = l.qt;
  const int64_t size = l.bf16 ? 2 : 4;
  const int64_t moved = (int64_t)l.rows * l.cols * (size + (l.q.data != nullptr) + (l.qt.data != nullptr));
  a.stream = moved > kCached && whole_pieces(l.src, l.src_stride, l.cols, size);
  const bool square = (l.q.data ? l.q.sh : l.qt.sh) != 0;
  if (!square && !l.qt.data) {
    a.tiles_x = (uint32_t)ceil_div(l.cols, 512);
    if (l.bf16) launch_rows<true>(a, st);
    else launch_rows<false>(a, st);
    return hipGetLastError();
  }
  a.tiles_x = (uint32_t)ceil_div(l.cols, 128);
  const dim3 grid(a.tiles_x * (uint32_t)ceil_div(l.rows, 128));
  if (l.bf16) {
    if (square) launch_tiles<true, true>(a, grid, st);
    else launch_tiles<true, false>(a, grid, st);
  } else {
    if (square) launch_tiles<false, true>(a, grid, st);
    else launch_tiles<false, false>(a, grid, st);
  }
  return hipGetLastError();
}

hipError_t launch_turn(const QView& src, const QView& qt, hipStream_t st) {
  const uint32_t tiles_x = (uint32_t)ceil_div(src.cols, 128);
  hipLaunchKernelGGL(turn_tile_kernel, dim3(tiles_x * (uint32_t)ceil_div(src.rows, 128)), dim3(kTileLanes), 0, st, TurnArgs{src, qt, tiles_x});
  return hipGetLastError();
}

}  // namespace dr
