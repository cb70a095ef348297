// The products of a gated feed-forward block (dr_qgated, dr_qgated_save), with activation and product where their sums stand.
#include <hip/hip_runtime.h>

#include "product_device.h"

namespace dr {
namespace {

void fill_pairs(GatedArgs& a, const GatedProduct& g) {
  fill_args(a, g.product, g.product.n / 2);
  a.half = a.n;
  a.half_bytes = (int64_t)a.n * a.b.stride;
  a.b.rows = a.n;  // gate's; up's lie half_bytes behind them
  a.act = g.act;
}

// One row of x, without the matrix instructions: a wave takes a pair of b's rows, whose columns its lanes read 16 at a time, 1 KiB
// of a row together, and adds products in fp32 in its lanes and then across them.  x stands quantized in LDS, as fp32 values
// in the order in which the lanes read them: of each 1024 columns the first four of every lane's 16, the second four, and
// so on.
//   Bound by how fast the weights come, behind the launch's start and x (about 3 us): in us, this / the kernel for few rows
//   3584 x 4096 7.8 / 9.0   3456 x 5120 8.9 / 9.4   14336 x 4096 25.5 / 28.2   4864 x 896 3.7 / 4.9   1000 x 1000 2.9 / 3.6   300 x 8192 6.1 / 8.5
// Two rows of x take 10.0 / 9.2 at 3584 x 4096.  With 4 / 8 / 16 waves 9.2 / 8.2 / 8.4, with 2 / 4 / 6 steps in flight 7.8 / 8.2 / 8.5.
constexpr int kVectorWaves = 8, kVectorSteps = 2;
constexpr uint32_t kVectorColumns = 1024;  // of a step

template <bool BF16>
__global__ __launch_bounds__(64 * kVectorWaves) void gated_vector_kernel(GatedArgs p) {
  extern __shared__ __align__(16) float xs[];  // [steps][4][64][4]
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t columns = p.kb * 128, steps = (columns + kVectorColumns - 1) / kVectorColumns;
  const uint32_t n = blockIdx.x * kVectorWaves + wave, pair = min(n, p.n - 1);
  const uint32_t rows[2] = {pair, pair + p.half};
  struct Step {
    u32x4 codes[2];
    uint32_t scale[2];
  };
  auto load = [&](uint32_t step) {
    Step s = {};
    const uint32_t col = step * kVectorColumns + lane * 16, block = col / 128;
    if (col < columns) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s.codes[i] = *reinterpret_cast<const u32x4*>(p.b.data + (int64_t)rows[i] * p.b.stride + col);
        s.scale[i] = p.b.scales[((int64_t)(block >> 2) * p.b.srows + (rows[i] >> p.b.sh)) * 4 + (block & 3)];
      }
    }
    return s;
  };
  Step now[kVectorSteps];
#pragma unroll
  for (int i = 0; i < kVectorSteps; ++i) now[i] = load(i);

  // 512 columns of x a wave; those behind the last one are 0
  for (uint32_t part = wave; part < steps * 2; part += kVectorWaves) {
    const uint32_t col = part * 512 + lane * 8;
    Raw8<BF16> v = load_row8<BF16>(p.x, 0, col, p.a.cols);
    settle8(v, ahead8(col, p.a.cols));
    uint32_t m = row_max(v, false);
    if (__any(m >= kInfBits)) m = row_max(v, true);
    const uint32_t code = scale_code(max16(m));
    const Values8 values = f32_values(row_codes(v, code), code);
    float* to = xs + col / kVectorColumns * kVectorColumns + col / 16 % 64 * 4 + col / 8 % 2 * 512;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<f32x4*>(to + h * 256) = f32x4{values.v[4 * h], values.v[4 * h + 1], values.v[4 * h + 2], values.v[4 * h + 3]};
  }
  __syncthreads();

  float sum[2] = {};
  for (uint32_t first = 0; first < steps; first += kVectorSteps) {
#pragma unroll
    for (int i = 0; i < kVectorSteps; ++i) {
      const uint32_t step = first + i;
      if (step >= steps) break;
      const Step s = now[i];
      now[i] = load(step + kVectorSteps);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(xs + step * kVectorColumns + q * 256 + lane * 4);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float w[4];
          f32_values4(s.codes[h][q], scale_operand(s.scale[h]), w);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[h] = fmaf(w[e], x[e], sum[h]);
        }
      }
    }
  }
  const float h = gated(wave_sum(sum[0]), wave_sum(sum[1]), p.act);
  if (lane == 0 && n < p.n) {
    if (p.c_bf16) static_cast<uint16_t*>(p.c)[n] = (uint16_t)bf16_pair(h, h);
    else static_cast<float*>(p.c)[n] = h;
  }
}

// The LDS that x takes, and the most of it: two workgroups stay on a CU.
int64_t vector_bytes(uint32_t kb) { return ceil_div(kb * 128, kVectorColumns) * kVectorColumns * 4; }
constexpr int64_t kVectorBytes = 64 << 10;

void launch_vector(const GatedArgs& a, bool x_bf16, hipStream_t st) {
  const dim3 grid((uint32_t)ceil_div(a.n, kVectorWaves)), block(64 * kVectorWaves);
  if (x_bf16) hipLaunchKernelGGL(gated_vector_kernel<true>, grid, block, (uint32_t)vector_bytes(a.kb), st, a);
  else hipLaunchKernelGGL(gated_vector_kernel<false>, grid, block, (uint32_t)vector_bytes(a.kb), st, a);
}

}  // namespace

hipError_t launch_gated_rows(const GatedProduct& g, hipStream_t st) {
  GatedArgs a;
  fill_pairs(a, g);
  const ProductLaunch& l = g.product;
  const int size = l.c_bf16 ? 2 : 4;
  const ProductPlan& plan = *l.plan;
  if (l.x && l.m == 1 && l.a.cols >= 8 && vector_bytes(l.kb) <= kVectorBytes) {
    launch_vector(a, l.x_bf16, st);
  } else if (l.x || plan.kind == ProductPlan::kDirect || l.c_stride * size >= kMaxRowBytes) {
    launch_direct_kind<kGated>(a, l.x_bf16, plan.rows16, st);
  } else {
    if (a.n * (int64_t)size % 16) a.c_vec = 0;  // whole pieces only
    if (l.c_bf16) launch_tile_kind<2, kGated>(a, plan, l.fast, st);
    else launch_tile_kind<4, kGated>(a, plan, l.fast, st);
  }
  return hipGetLastError();
}

hipError_t launch_gated_codes(const GatedProduct& g, const GatedCodesPlan& plan, hipStream_t st) {
  GatedArgs a;
  fill_pairs(a, g);
  a.hq = g.hq;
  a.gate = g.gate;
  a.up = g.up;
  const bool fast = g.product.fast;
  if (a.kb == 1) launch_tiles<128, 256, 1, true, true, kGatedCodes>(a, 0, fast, st);
  else if (plan.rows == 256) launch_tiles<256, 256, 1, true, false, kGatedCodes>(a, plan.halved, fast, st);
  else launch_tiles<128, 256, 1, true, false, kGatedCodes>(a, 0, fast, st);
  return hipGetLastError();
}

}  // namespace dr
