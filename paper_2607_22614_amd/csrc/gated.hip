// The second half of a gated feed-forward block's forward pass where its projections are computed as one product with
// fp32 sums in a workspace: h = act(gate) * up (dr_qgated, dr_qgated_save).
//
// Memory-bound, and for small blocks alone, whose sums lie in the last cache: 8 bytes read for each part and 1 to 4
// written per element of h.  200 x 688 in 8 bits with gate and up take 3.9 us, of which a launch's start and end 2.4.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gated_device.h"

namespace dr {
namespace {

typedef f32x4 __attribute__((aligned(4))) AnyF32x4;

// A lane takes four columns of a row; up's need not begin at 16 bytes.
template <bool BF16>
__global__ __launch_bounds__(256) void gated_join_kernel(GatedJoin p) {
  const uint32_t groups = (p.f + 3) / 4;
  const uint64_t n = (uint64_t)p.m * groups;
  const bool vec = reinterpret_cast<uintptr_t>(p.h) % 16 == 0 && p.h_stride % 8 == 0;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
    const uint32_t m = (uint32_t)(i / groups), f0 = (uint32_t)(i % groups) * 4;
    const float* part = p.sums + (int64_t)m * p.stride + f0;
    f32x4 gate = *reinterpret_cast<const AnyF32x4*>(part), up = *reinterpret_cast<const AnyF32x4*>(part + p.f);
    for (uint32_t k = 1; k < p.splits; ++k) {
      part += p.split_stride;
      gate += *reinterpret_cast<const AnyF32x4*>(part);
      up += *reinterpret_cast<const AnyF32x4*>(part + p.f);
    }
    f32x4 h;
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = gated(gate[j], up[j], p.act);
    const int64_t at = (int64_t)m * p.h_stride + f0;
    const bool whole = vec && f0 + 4 <= p.f;
    if (BF16) {
      uint16_t* c = static_cast<uint16_t*>(p.h) + at;
      const u32x2 w = {bf16_pair(h[0], h[1]), bf16_pair(h[2], h[3])};
      if (whole) {
        *reinterpret_cast<u32x2*>(c) = w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (f0 + j < p.f) c[j] = (uint16_t)(w[j / 2] >> (j % 2 * 16));
      }
    } else {
      float* c = static_cast<float*>(p.h) + at;
      if (whole) {
        *reinterpret_cast<f32x4*>(c) = h;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (f0 + j < p.f) c[j] = h[j];
      }
    }
  }
}

// The sums of 8 columns of a row of gate or up, those behind the last column 0.
__device__ __forceinline__ Raw8<false> joined8(const GatedJoin& p, uint32_t row, uint32_t col, uint32_t half) {
  Raw8<false> v = {};
  for (uint32_t k = 0; k < p.splits; ++k) {
    const int64_t at = (int64_t)row * p.stride + (int64_t)k * p.split_stride + (int64_t)half * p.f;
    const Raw8<false> part = p.f < 8 ? load_short_row8<false>(p.sums, at, col, p.f) : load_row8<false>(p.sums, at, col, p.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) put_element(v, i, k ? element(v, i) + element(part, i) : element(part, i));
  }
  settle8(v, ahead8(col, p.f));
  return v;
}

// Codes of 8 columns of a row by each lane (512 columns a wave, four blocks), and the row's four scale codes as one word.
__device__ __forceinline__ void put_row(const QView& q, uint32_t row, uint32_t quad, uint32_t lane, const Raw8<false>& v) {
  uint32_t m = row_max(v, false);
  if (__any(m >= kInfBits)) m = row_max(v, true);
  const uint32_t code = scale_code(max16(m)), col = quad * 512 + lane * 8;
  const uint32_t word = (uint32_t)__builtin_amdgcn_readlane((int)code, 0) | (uint32_t)__builtin_amdgcn_readlane((int)code, 16) << 8 |
                        (uint32_t)__builtin_amdgcn_readlane((int)code, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane((int)code, 48) << 24;
  if ((col & ~127u) < q.cols) *reinterpret_cast<u32x2*>(q.data + (int64_t)row * q.stride + col) = row_codes(v, code);
  if (lane == 0) reinterpret_cast<uint32_t*>(q.scales)[(int64_t)quad * q.rows + row] = word;
}

// A wave takes 512 columns of a row.
constexpr int kJoinWaves = 4;
__global__ __launch_bounds__(64 * kJoinWaves) void gated_join_quantize_kernel(GatedJoin p) {
  const uint32_t lane = threadIdx.x & 63, quads = (p.f + 511) / 512;
  const uint64_t n = (uint64_t)p.m * quads;
  for (uint64_t i = (uint64_t)blockIdx.x * kJoinWaves + threadIdx.x / 64; i < n; i += (uint64_t)gridDim.x * kJoinWaves) {
    const uint32_t row = (uint32_t)(i / quads), quad = (uint32_t)(i % quads), col = quad * 512 + lane * 8;
    const Raw8<false> gate = joined8(p, row, col, 0), up = joined8(p, row, col, 1);
    Raw8<false> h;
#pragma unroll
    for (int j = 0; j < 8; ++j) put_element(h, j, gated(element(gate, j), element(up, j), p.act));
    put_row(p.hq, row, quad, lane, h);
    if (p.gate.data) {
      put_row(p.gate, row, quad, lane, gate);
      put_row(p.up, row, quad, lane, up);
    }
  }
}

constexpr int64_t kJoinGrid = 2048;

}  // namespace

hipError_t launch_gated_join(const GatedJoin& l, hipStream_t st) {
  if (l.h) {
    const dim3 grid((uint32_t)std::min(kJoinGrid, ceil_div((int64_t)l.m * ceil_div(l.f, 4), 256)));
    if (l.h_bf16) hipLaunchKernelGGL(gated_join_kernel<true>, grid, dim3(256), 0, st, l);
    else hipLaunchKernelGGL(gated_join_kernel<false>, grid, dim3(256), 0, st, l);
  } else {
    const dim3 grid((uint32_t)std::min(kJoinGrid, ceil_div((int64_t)l.m * ceil_div(l.f, 512), kJoinWaves)));
    hipLaunchKernelGGL(gated_join_quantize_kernel, grid, dim3(64 * kJoinWaves), 0, st, l);
  }
  return hipGetLastError();
}

}  // namespace dr
