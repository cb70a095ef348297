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
// call does not know the others; kCached is the line for somewhat less than 3.  In us, plain / streamed:
//                                  3 sets         from HBM       just written
//   4096 x 4096 bf16, rows       10.6 / 11.3     12.6 / 11.0     12.5 / 12.7
//   8192 x 4096 bf16, both ways  28.2 / 26.4     28.7 / 29.0     22.7 / 25.9
//   16384 x 4096 bf16, rows      38.7 / 35.5
//   8192 x 14336 bf16, rows                      66.9 / 64.7     57.5 / 61.7
//   16384 x 4096 fp32, rows      63.1 / 60.2
//   16384 x 4096 fp32, both ways 75.3 / 82.0, where it does not pay
constexpr int64_t kCached = 96ll << 20;
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

// Scale code of block (i, j) of a matrix with R block rows, and 127 in the unused bytes of its last word.
__device__ __forceinline__ void put_code(const QView& q, uint32_t i, uint32_t j, uint32_t code) {
  const uint32_t blocks = (q.cols + 127) / 128;
  uint8_t* p = q.scales + ((int64_t)(j >> 2) * q.srows + i) * 4;
  p[j & 3] = (uint8_t)code;
  if (j + 1 == blocks)
    for (uint32_t k = (j & 3) + 1; k < 4; ++k) p[k] = 127;
}

// A tile of 128 x 128 per workgroup, each lane 8 columns of 4 rows, kept in registers (of 8 rows by half the lanes: 200 x 256
// bf16 both ways 5.0 us instead of 4.5, 2000 x 4096 fp32 14.1 and 13.4).  ROWS writes the codes along the rows, COLS the
// transpose: its codes are packed 4 rows to a word, turned in LDS (one 128-byte row per column, its words spread by an
// exclusive or over the banks), and leave as whole 128-byte rows.  SQUARE: one scale for the tile, else one per row (DPP) and
// one per column (over the four rows of lanes, then over the waves in LDS).
//   Tiles go in bands of four down, and 32 of them to an XCD at a time: runs of 512 to 1024 bytes of q's and qt's rows then
// leave one L2 (8192 x 4096 fp32 both ways 43 us, in the order of the rows 45; 3000 x 3001 bf16 10.8 and 11.6).
constexpr uint32_t kBandT = 4, kTurn = 32;
template <bool BF16, bool SQUARE, bool ROWS, bool COLS>
__global__ __launch_bounds__(kTileLanes) void quantize_tile_kernel(QuantizeArgs a) {
  constexpr int R = 128 / (kTileLanes / 16), kWaves = kTileLanes / 64;
  __shared__ uint32_t cmax[kWaves][128];
  __shared__ __align__(16) uint8_t turned[COLS ? 128 * 128 : 16];
  const uint32_t tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, wave = tid / 64;
  const uint32_t t = xcd_group<kTurn>(blockIdx.x, gridDim.x), tiles_y = gridDim.x / a.tiles_x, band = t / (kBandT * a.tiles_x);
  const uint32_t high = min(kBandT, tiles_y - band * kBandT), i_band = t - band * kBandT * a.tiles_x;
  const uint32_t rt = band * kBandT + i_band % high, ct = i_band / high;
  const uint32_t col = ct * 128 + tx * 8, row0 = rt * 128 + ty * R;
  Raw8<BF16> v[R];
  load_rows(a, row0, col, v);
  if (row0 + R > a.rows) {
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (row0 + i >= a.rows) v[i] = Raw8<BF16>{};
  }
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
    if ((tid & 63) == 0) cmax[0][wave] = m;
    __syncthreads();
    uint32_t most = cmax[0][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) most = max(most, cmax[0][w]);
    square_code = scale_code(most);
    if (tid == 0) {
      if (ROWS) put_code(a.q, rt, ct, square_code);
      if (COLS) put_code(a.qt, ct, rt, square_code);
    }
  }

  if (ROWS) {
    uint32_t mine = 0;  // of row row0 + tx
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint32_t code = SQUARE ? square_code : scale_code(max16(rmax[i]));
      mine = tx == (uint32_t)i ? code : mine;
      if (row0 + i < a.rows)
        *reinterpret_cast<u32x2*>(a.q.data + (int64_t)(row0 + i) * a.q.stride + col) = row_codes(v[i], code);
    }
    if (!SQUARE && tx < R && row0 + tx < a.rows) put_code(a.q, row0 + tx, ct, mine);
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
            cmax[wave][tx * 8 + 2 * w] = m << 16;
            cmax[wave][tx * 8 + 2 * w + 1] = m & 0xFFFF0000u;
          } else {
            cmax[wave][tx * 8 + w] = m;
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = tx * 8 + j;
        uint32_t m = cmax[0][c];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = max(m, cmax[w][c]);
        code[j] = scale_code(m);
        mine = ty == (uint32_t)j ? code[j] : mine;
      }
      if (ty < 8 && col + ty < a.cols) put_code(a.qt, col + ty, rt, mine);
    }
    // word ty of a column lies at ty ^ 4 (tx % 8), which keeps its 16-byte pieces together
#pragma unroll
    for (int j = 0; j < 8; ++j)
      *reinterpret_cast<uint32_t*>(turned + (tx * 8 + j) * 128 + (ty ^ (tx % 8 * 4)) * 4) = column_codes<BF16>(v, j, code[j]);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 128 * 8 / kTileLanes; ++r) {
      const uint32_t c = r * (kTileLanes / 8) + tid / 8, piece = tid % 8;
      const u32x4 w = *reinterpret_cast<const u32x4*>(turned + c * 128 + (piece ^ (c / 8 % 8)) * 16);
      if (ct * 128 + c < a.cols)
        *reinterpret_cast<u32x4*>(a.qt.data + (int64_t)(ct * 128 + c) * a.qt.stride + rt * 128 + piece * 16) = w;
    }
  }
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

}  // namespace dr
