// Launches of the gradient kernels (grad_clip.hip): arguments checked by grads.cpp.  Each wrapper
// enqueues on `st` and returns hipGetLastError().
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dr.h"

namespace dr {

constexpr int64_t kMaxGradElems = 1ll << 42;  // of a list: its chunks are counted in 32 bits
constexpr uint32_t kGradSums = 2048;  // workgroups of a launch of the norm, and its sums in the workspace
// The most sums that every workgroup of the scaling adds up itself.
constexpr uint32_t kFewSums = kGradSums / 2;

// One sum of squares per workgroup into partial[0 .. *nsums), *nsums <= kGradSums (0: an empty list).
hipError_t launch_grad_norm(const dr_grad* grads, int64_t count, double* partial, uint32_t* nsums, hipStream_t st);
hipError_t launch_grad_total(const double* sums, uint32_t nsums, double* sum_squares, float* norm, hipStream_t st);
// The squares' total is that of sums[0 .. nsums).
hipError_t launch_grad_scale(const dr_grad* grads, int64_t count, const double* sums, uint32_t nsums, double max_norm,
                             float* norm_out, hipStream_t st);

}  // namespace dr
