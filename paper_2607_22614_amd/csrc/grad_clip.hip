// Global gradient norm and clipping over a list of tensors (dr_grad_norm, dr_grad_scale, dr_grad_clip).
//
//   norm = sqrt(sum of g^2),  out = g * min(1, max_norm / (norm + 1e-6))
//
// HBM-bound: the norm reads every gradient, the scaling reads it again and writes it.  The list travels in the kernel
// argument, kGradTensors tensors a launch; a workgroup strides over chunks of elements and finds a
// chunk's tensor by bisection.  Squares are summed in fp64, where no square of an fp32 value overflows or vanishes, at
// one convert and one fma per element; each workgroup leaves one sum in the workspace (or adds it to that of an
// earlier launch of a longer list: 0.5B matrices behind 112 vectors are read at 6.6 TB/s, in model order at 6.7).  Every workgroup of the scaling adds these up itself where they are few, else a launch
// between them does: no atomics, and equal inputs give equal bits.  The factor stays in fp64 too: against a norm beyond fp32's range it
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
// Elements of a chunk.  The norm strides over long ones with 2048 workgroups (6.9 TB/s read; 2048 to 8192 elements with a
// workgroup each 6.1-6.7); lists that give at most kGradSums / 2 short ones take those, for more workgroups.  The scaling
// reads and writes, and is fastest with a short chunk per workgroup and the XCDs taking 64 of them in turn: 6.2 TB/s, in
// strides of long chunks 5.2.
constexpr uint32_t kLongChunk = 16384, kShortChunk = 4096, kChunkGroup = 64;
constexpr uint32_t kTypeShift = 56;     // grad type in bit 56, out type in bit 57 of `numel`

struct GradArgs {
  const double* sums;  // of the norm's workgroups, or one sum of squares
  double* partial;
  float* norm_out;
  double max_norm;
  uint32_t nsums, count, chunks;  // nsums of the norm: those that launches before wrote to `partial`
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

template <uint32_t CHUNK>
__device__ __forceinline__ Chunk find_chunk(const GradArgs& a, uint32_t c) {
  uint32_t lo = 0, hi = a.count;  // first[lo] <= c < first[hi]
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (a.first[mid] <= c) lo = mid;
    else hi = mid;
  }
  const uint64_t word = a.numel[lo], numel = word & ((1ull << kTypeShift) - 1);
  const uint64_t at = (uint64_t)(c - a.first[lo]) * CHUNK;
  return Chunk{lo, (uint32_t)min((uint64_t)CHUNK, numel - at), at, (word >> kTypeShift & 1) != 0,
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

// Whole chunks move 16 bytes per lane and access, at most kAhead of them in flight.
constexpr uint32_t kAhead = 8;

// Other chunks: single elements, adjacent lanes adjacent ones, kSingles loads in flight.  Element k is i0 + 256 k of the
// chunk; past its end the last one is read again.
constexpr int kSingles = 16;
template <bool BF16>
__device__ __forceinline__ void load_singles(const void* grad, uint64_t at, uint32_t i0, uint32_t n, float (&v)[kSingles]) {
#pragma unroll
  for (int k = 0; k < kSingles; ++k) {
    const uint64_t i = at + min(i0 + k * kThreadsG, n - 1);
    v[k] = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(grad)[i] << 16) : static_cast<const float*>(grad)[i];
  }
}

template <uint32_t CHUNK, bool BF16>
__device__ __forceinline__ void sum_chunk(const void* grad, uint64_t at, uint32_t n, double (&acc)[2]) {
  constexpr uint32_t E = BF16 ? 8 : 4, kLoads = CHUNK / (kThreadsG * E), kFly = kLoads < kAhead ? kLoads : kAhead;
  if (n == CHUNK && aligned16(grad)) {
    const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(grad) + at * (BF16 ? 2 : 4)) + threadIdx.x;
#pragma unroll
    for (uint32_t i = 0; i < kLoads; i += kFly) {
      u32x4 w[kFly];
#pragma unroll
      for (uint32_t k = 0; k < kFly; ++k) w[k] = load_stream(p + (i + k) * kThreadsG);
#pragma unroll
      for (uint32_t k = 0; k < kFly; ++k)
#pragma unroll
        for (uint32_t j = 0; j < E; ++j) {
          const double d = value<BF16>(w[k], j);
          acc[j & 1] = fma(d, d, acc[j & 1]);
        }
    }
    return;
  }
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kThreadsG * kSingles) {
    float v[kSingles];
    load_singles<BF16>(grad, at, i0, n, v);
#pragma unroll
    for (int k = 0; k < kSingles; ++k) {
      const double d = i0 + k * kThreadsG < n ? v[k] : 0.f;
      acc[k & 1] = fma(d, d, acc[k & 1]);
    }
  }
}

template <uint32_t CHUNK>
__global__ __launch_bounds__(kThreadsG) void grad_norm_kernel(GradArgs args) {
  (void)args;  // read through the kernarg segment (same bytes)
  const GradArgs& a = *(const GradArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ double red[kThreadsG / 64];
  double acc[2] = {0, 0};
  for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Chunk k = find_chunk<CHUNK>(a, c);
    if (k.grad_bf16) sum_chunk<CHUNK, true>(a.grad[k.tensor], k.at, k.n, acc);
    else sum_chunk<CHUNK, false>(a.grad[k.tensor], k.at, k.n, acc);
  }
  const double s = block_sum(acc[0] + acc[1], red);
  if (threadIdx.x == 0) a.partial[blockIdx.x] = blockIdx.x < a.nsums ? a.partial[blockIdx.x] + s : s;
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

// factor() is called once the loads are on their way.
template <bool BF16, bool OUT_BF16, typename Factor>
__device__ __forceinline__ void scale_chunk(const void* grad, void* out, uint64_t at, uint32_t n, Factor factor) {
  // bf16 to fp32 loads 8 bytes a lane, so that a wave's stores are whole lines too
  constexpr int E = BF16 && OUT_BF16 ? 8 : 4, IN = E * (BF16 ? 2 : 4), OUT = E * (OUT_BF16 ? 2 : 4);
  typedef uint32_t In __attribute__((ext_vector_type(IN / 4)));
  typedef uint32_t Out __attribute__((ext_vector_type(OUT / 4)));
  if (n == kShortChunk && aligned16(grad) && aligned16(out)) {
    const In* p = reinterpret_cast<const In*>(static_cast<const uint8_t*>(grad) + at * (BF16 ? 2 : 4)) + threadIdx.x;
    Out* q = reinterpret_cast<Out*>(static_cast<uint8_t*>(out) + at * (OUT_BF16 ? 2 : 4)) + threadIdx.x;
    constexpr int kLoads = kShortChunk / (kThreadsG * E);
    In w[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) w[k] = load_stream(p + k * kThreadsG);
    const double f = factor();
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j)
          v[j] = (float)(__uint_as_float(!BF16 ? w[k][j % (IN / 4)] : j % 2 ? w[k][j / 2 % (IN / 4)] & 0xFFFF0000u : w[k][j / 2 % (IN / 4)] << 16) * f);
        Out o;
#pragma unroll
        for (int j = 0; j < OUT / 4; ++j) o[j] = OUT_BF16 ? bf16_pair(v[2 * j % E], v[(2 * j + 1) % E]) : __float_as_uint(v[j % E]);
        store_stream(o, q + k * kThreadsG);
    }
    return;
  }
  const double f = factor();
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kThreadsG * kSingles) {
    float v[kSingles];
    load_singles<BF16>(grad, at, i0, n, v);
#pragma unroll
    for (int k = 0; k < kSingles; ++k) {
      const uint32_t i = i0 + k * kThreadsG;
      const float x = (float)(v[k] * f);
      if (i < n) {
        if (OUT_BF16) static_cast<uint16_t*>(out)[at + i] = (uint16_t)bf16_pair(x, x);
        else static_cast<float*>(out)[at + i] = x;
      }
    }
  }
}

__global__ __launch_bounds__(kThreadsG) void grad_scale_kernel(GradArgs args) {
  (void)args;
  const GradArgs& a = *(const GradArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ double red[kThreadsG / 64];
  double f = -1;  // not known yet
  auto factor = [&] {
    if (f == -1) {
      const double norm = sqrt(total(a.sums, a.nsums, red));
      if (a.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *a.norm_out = (float)norm;
      const double ratio = a.max_norm / (norm + 1e-6);
      f = a.max_norm == HUGE_VAL || ratio >= 1.0 ? 1.0 : ratio;  // a NaN norm: NaN
    }
    return f;
  };
  if (a.chunks == 0) factor();
  for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Chunk k = find_chunk<kShortChunk>(a, xcd_group<kChunkGroup>(c, a.chunks));
    const void* grad = a.grad[k.tensor];
    void* out = a.out[k.tensor];
    if (grad == out && factor() == 1.0) continue;
    if (k.grad_bf16) {
      if (k.out_bf16) scale_chunk<true, true>(grad, out, k.at, k.n, factor);
      else scale_chunk<true, false>(grad, out, k.at, k.n, factor);
    } else {
      if (k.out_bf16) scale_chunk<false, true>(grad, out, k.at, k.n, factor);
      else scale_chunk<false, false>(grad, out, k.at, k.n, factor);
    }
  }
}

// Fills a from grads[at..], in chunks of `chunk`, and returns how many of them it took (empty ones are passed over).
int64_t fill(GradArgs& a, const dr_grad* grads, int64_t count, int64_t at, uint32_t chunk, bool scale) {
  a.count = 0;
  uint64_t chunks = 0;  // at most 2^30 (kMaxGradElems) and one more per tensor
  int64_t i = at;
  for (; i < count && a.count < (uint32_t)kGradTensors; ++i) {
    const dr_grad& g = grads[i];
    if (!g.numel) continue;
    a.first[a.count] = (uint32_t)chunks;
    a.numel[a.count] = (uint64_t)g.numel | (uint64_t)(g.grad_type == DR_TYPE_BF16) << kTypeShift |
                       (uint64_t)(scale && g.out_type == DR_TYPE_BF16) << (kTypeShift + 1);
    a.grad[a.count] = g.grad;
    a.out[a.count] = scale ? g.out : nullptr;
    chunks += ((uint64_t)g.numel + chunk - 1) / chunk;
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
  uint64_t shorts = 0;
  for (int64_t i = 0; i < count; ++i) shorts += ((uint64_t)grads[i].numel + kShortChunk - 1) / kShortChunk;
  const uint32_t chunk = shorts <= kGradSums / 2 ? kShortChunk : kLongChunk;
  for (int64_t at = 0; at < count;) {
    at += fill(a, grads, count, at, chunk, false);
    if (!a.chunks) break;
    // a longer list's later launches add to the sums that earlier ones wrote, and write those behind them
    const uint32_t grid = std::min(a.chunks, kGradSums);
    a.nsums = *nsums;
    *nsums = std::max(*nsums, grid);
    if (chunk == kShortChunk) hipLaunchKernelGGL(grad_norm_kernel<kShortChunk>, dim3(grid), dim3(kThreadsG), 0, st, a);
    else hipLaunchKernelGGL(grad_norm_kernel<kLongChunk>, dim3(grid), dim3(kThreadsG), 0, st, a);
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
    at += fill(a, grads, count, at, kShortChunk, true);
    if (!a.chunks && !a.norm_out) break;
    hipLaunchKernelGGL(grad_scale_kernel, dim3(std::max(1u, std::min(a.chunks, kMaxGrid))), dim3(kThreadsG), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    a.norm_out = nullptr;  // the first launch writes it
  }
  return hipSuccess;
}

}  // namespace dr
