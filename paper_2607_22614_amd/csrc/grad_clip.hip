// Global gradient norm and clipping over a list of tensors (dr_grad_norm, dr_grad_scale, dr_grad_clip).
//
//   norm = sqrt(sum of g^2),  out = g * min(1, max_norm / (norm + 1e-6))
//
// HBM-bound: the norm reads every gradient, the scaling reads it again and writes it.  The list travels in the kernel
// argument, kGradTensors tensors a launch; a workgroup strides over chunks of kGradChunk elements and finds a
// chunk's tensor by bisection.  Squares are summed in fp64, where no square of an fp32 value overflows or vanishes, at
// one convert and one fma per element; each workgroup leaves one sum in the workspace (a later launch of a
// longer list adds to it), and every workgroup of the scaling adds these up itself, in the same order: no atomics, no
// third launch, and equal inputs give equal bits.  The factor stays in fp64 too: against a norm beyond fp32's range it
// is a number that fp32 holds with few bits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "grad_kernels.h"
#include "quant_device.h"

namespace dr {
namespace {

constexpr int kGradTensors = 112;
constexpr int kThreadsG = 256;
constexpr uint32_t kGradChunk = 16384;  // elements
constexpr uint32_t kTypeShift = 56;     // grad type in bit 56, out type in bit 57 of `numel`

struct GradArgs {
  const double* sums;  // of the norm's workgroups, or one sum of squares
  double* partial;
  float* norm_out;
  double max_norm;
  uint32_t nsums, count, chunks;
  int32_t add;
  uint32_t first[kGradTensors + 1];  // first chunk of each tensor
  uint64_t numel[kGradTensors];
  const void* grad[kGradTensors];
  void* out[kGradTensors];
};
static_assert(sizeof(GradArgs) <= 4096, "kernel argument");

struct Chunk {
  uint32_t tensor, n;
  uint64_t at;
  bool grad_bf16, out_bf16;
};

__device__ __forceinline__ Chunk find_chunk(const GradArgs& a, uint32_t c) {
  uint32_t lo = 0, hi = a.count;  // first[lo] <= c < first[hi]
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (a.first[mid] <= c) lo = mid;
    else hi = mid;
  }
  const uint64_t word = a.numel[lo], numel = word & ((1ull << kTypeShift) - 1);
  const uint64_t at = (uint64_t)(c - a.first[lo]) * kGradChunk;
  return Chunk{lo, (uint32_t)min((uint64_t)kGradChunk, numel - at), at, (word >> kTypeShift & 1) != 0,
               (word >> (kTypeShift + 1) & 1) != 0};
}

__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Sum over the workgroup in a fixed order; every lane gets it.
__device__ __forceinline__ double block_sum(double v, double (&red)[kThreadsG / 64]) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  double s = red[0];
#pragma unroll
  for (int w = 1; w < kThreadsG / 64; ++w) s += red[w];
  __syncthreads();
  return s;
}

// fp32 values of element i of the 4 or 8 in 16 bytes.
template <bool BF16>
__device__ __forceinline__ float value(u32x4 w, int i) {
  return __uint_as_float(!BF16 ? w[BF16 ? 0 : i] : i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}

// Whole chunks move 16 bytes per lane and access, kAhead of them in flight.
constexpr int kAhead = 8;

template <bool BF16>
__device__ __forceinline__ void sum_chunk(const void* grad, uint64_t at, uint32_t n, double (&acc)[2]) {
  constexpr int E = BF16 ? 8 : 4;
  if (n == kGradChunk && aligned16(grad)) {
    const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(grad) + at * (BF16 ? 2 : 4)) + threadIdx.x;
#pragma unroll
    for (uint32_t i = 0; i < kGradChunk / (kThreadsG * E * kAhead); ++i) {
      u32x4 w[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) w[k] = load_stream(p + (i * kAhead + k) * kThreadsG);
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const double d = value<BF16>(w[k], j);
          acc[j & 1] = fma(d, d, acc[j & 1]);
        }
    }
    return;
  }
  const bool vec = aligned16(grad);
  for (uint32_t i = threadIdx.x * 8; i < n; i += kThreadsG * 8) {
    float v[8];
    load8<BF16>(grad, (int64_t)(at + i), (int)min(8u, n - i), vec, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j & 1] = fma((double)v[j], (double)v[j], acc[j & 1]);
  }
}

__global__ __launch_bounds__(kThreadsG) void grad_norm_kernel(GradArgs args) {
  (void)args;  // read through the kernarg segment (same bytes)
  const GradArgs& a = *(const GradArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ double red[kThreadsG / 64];
  double acc[2] = {0, 0};
  for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Chunk k = find_chunk(a, c);
    if (k.grad_bf16) sum_chunk<true>(a.grad[k.tensor], k.at, k.n, acc);
    else sum_chunk<false>(a.grad[k.tensor], k.at, k.n, acc);
  }
  const double s = block_sum(acc[0] + acc[1], red);
  if (threadIdx.x == 0) a.partial[blockIdx.x] = a.add ? a.partial[blockIdx.x] + s : s;
}

__device__ __forceinline__ double total(const double* sums, uint32_t n, double (&red)[kThreadsG / 64]) {
  double s = 0;
  for (uint32_t i = threadIdx.x; i < n; i += kThreadsG) s += sums[i];
  return block_sum(s, red);
}

__global__ __launch_bounds__(kThreadsG) void grad_total_kernel(const double* sums, uint32_t n, double* sum_squares, float* norm) {
  __shared__ double red[kThreadsG / 64];
  const double s = total(sums, n, red);
  if (threadIdx.x == 0) {
    if (sum_squares) *sum_squares = s;
    if (norm) *norm = (float)sqrt(s);
  }
}

template <bool BF16, bool OUT_BF16>
__device__ __forceinline__ void scale_chunk(const void* grad, void* out, uint64_t at, uint32_t n, double f) {
  constexpr int E = BF16 ? 8 : 4;
  const bool vec = aligned16(grad), ovec = aligned16(out);
  if (n == kGradChunk && vec && ovec) {
    const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(grad) + at * (BF16 ? 2 : 4)) + threadIdx.x;
    uint8_t* q = static_cast<uint8_t*>(out) + at * (OUT_BF16 ? 2 : 4);
#pragma unroll
    for (uint32_t i = 0; i < kGradChunk / (kThreadsG * E * kAhead); ++i) {
      u32x4 w[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) w[k] = load_stream(p + (i * kAhead + k) * kThreadsG);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = (float)(value<BF16>(w[k], j) * f);
        const uint32_t to = ((i * kAhead + k) * kThreadsG + threadIdx.x) * E;  // element
#pragma unroll
        for (int j = 0; j < E; j += 4) {
          if constexpr (OUT_BF16) {
            if constexpr (BF16) {
              if (j == 0) store_stream(u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[E - 4], v[E - 3]), bf16_pair(v[E - 2], v[E - 1])}, reinterpret_cast<u32x4*>(q + 2 * to));
            } else {
              store_stream(u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])}, reinterpret_cast<u32x2*>(q + 2 * to));
            }
          } else {
            store_stream(f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]}, reinterpret_cast<f32x4*>(q + 4 * (to + j)));
          }
        }
      }
    }
    return;
  }
  for (uint32_t i = threadIdx.x * 8; i < n; i += kThreadsG * 8) {
    float v[8];
    const int k = (int)min(8u, n - i);
    load8<BF16>(grad, (int64_t)(at + i), k, vec, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)(v[j] * f);
    store8<OUT_BF16>(out, (int64_t)(at + i), k, ovec, v);
  }
}

__global__ __launch_bounds__(kThreadsG) void grad_scale_kernel(GradArgs args) {
  (void)args;
  const GradArgs& a = *(const GradArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ double red[kThreadsG / 64];
  const double norm = sqrt(total(a.sums, a.nsums, red));
  if (a.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *a.norm_out = (float)norm;
  const double ratio = a.max_norm / (norm + 1e-6);
  const double f = a.max_norm == HUGE_VAL || ratio >= 1.0 ? 1.0 : ratio;  // a NaN norm: NaN
  for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Chunk k = find_chunk(a, c);
    const void* grad = a.grad[k.tensor];
    void* out = a.out[k.tensor];
    if (f == 1.0 && grad == out) continue;
    if (k.grad_bf16) {
      if (k.out_bf16) scale_chunk<true, true>(grad, out, k.at, k.n, f);
      else scale_chunk<true, false>(grad, out, k.at, k.n, f);
    } else {
      if (k.out_bf16) scale_chunk<false, true>(grad, out, k.at, k.n, f);
      else scale_chunk<false, false>(grad, out, k.at, k.n, f);
    }
  }
}

// Fills a from grads[at..] and returns how many of them it took (empty ones are passed over).
int64_t fill(GradArgs& a, const dr_grad* grads, int64_t count, int64_t at, bool scale) {
  a.count = 0;
  uint64_t chunks = 0;  // at most 2^31 (kMaxGradElems) and one more per tensor
  int64_t i = at;
  for (; i < count && a.count < (uint32_t)kGradTensors; ++i) {
    const dr_grad& g = grads[i];
    if (!g.numel) continue;
    const uint64_t c = ((uint64_t)g.numel + kGradChunk - 1) / kGradChunk;
    a.first[a.count] = (uint32_t)chunks;
    a.numel[a.count] = (uint64_t)g.numel | (uint64_t)(g.grad_type == DR_TYPE_BF16) << kTypeShift |
                       (uint64_t)(scale && g.out_type == DR_TYPE_BF16) << (kTypeShift + 1);
    a.grad[a.count] = g.grad;
    a.out[a.count] = scale ? g.out : nullptr;
    chunks += c;
    ++a.count;
  }
  a.first[a.count] = (uint32_t)chunks;
  a.chunks = (uint32_t)chunks;
  return i - at;
}

}  // namespace

hipError_t launch_grad_norm(const dr_grad* grads, int64_t count, double* partial, uint32_t* nsums, hipStream_t st) {
  GradArgs a;
  a.partial = partial;
  *nsums = 0;
  for (int64_t at = 0; at < count;) {
    at += fill(a, grads, count, at, false);
    if (!a.chunks) break;
    a.add = *nsums != 0;
    // a longer list's later launches add to the sums that the first one wrote
    const uint32_t grid = a.add ? *nsums : std::min(a.chunks, kGradSums);
    *nsums = grid;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(grid), dim3(kThreadsG), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

hipError_t launch_grad_total(const double* sums, uint32_t nsums, double* sum_squares, float* norm, hipStream_t st) {
  hipLaunchKernelGGL(grad_total_kernel, dim3(1), dim3(kThreadsG), 0, st, sums, nsums, sum_squares, norm);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const dr_grad* grads, int64_t count, const double* sums, uint32_t nsums, double max_norm, float* norm_out,
                             hipStream_t st) {
  GradArgs a;
  a.sums = sums;
  a.nsums = nsums;
  a.max_norm = max_norm;
  a.norm_out = norm_out;
  for (int64_t at = 0; at < count || a.norm_out;) {
    at += fill(a, grads, count, at, true);
    if (!a.chunks && !a.norm_out) break;
    hipLaunchKernelGGL(grad_scale_kernel, dim3(std::max(1u, std::min(a.chunks, kGradSums))), dim3(kThreadsG), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    a.norm_out = nullptr;  // the first launch writes it
  }
  return hipSuccess;
}

}  // namespace dr
