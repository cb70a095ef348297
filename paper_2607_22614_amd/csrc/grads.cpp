// Entry points of the gradient norm and clipping (dr.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "dr_internal.h"
#include "grad_kernels.h"

namespace dr {
namespace {

bool aligned(const void* p, uintptr_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int element_bytes(int32_t type) { return type == DR_TYPE_F32 ? 4 : type == DR_TYPE_BF16 ? 2 : 0; }

int check_list(const dr_grad* grads, int64_t count, bool out, const char* what) {
  if (count < 0 || (count && !grads)) return fail(DR_EINVAL, "%s: a list of %lld gradients is null", what, (long long)count);
  uint64_t all = 0;
  for (int64_t i = 0; i < count; ++i) {
    const dr_grad& g = grads[i];
    const int size = element_bytes(g.grad_type), out_size = element_bytes(g.out_type);
    if (!size || (out && !out_size)) return fail(DR_EINVAL, "%s: gradient %lld has an unknown type", what, (long long)i);
    if (g.numel < 0 || g.numel > kMaxGradElems || (all += (uint64_t)g.numel) > (uint64_t)kMaxGradElems)
      return fail(DR_EINVAL, "%s: gradient %lld: %lld elements (at most 2^42 in all)", what, (long long)i, (long long)g.numel);
    if (!g.numel) continue;
    if (!aligned(g.grad, size) || (out && !aligned(g.out, out_size)))
      return fail(DR_EINVAL, "%s: gradient %lld: pointer null or misaligned", what, (long long)i);
    if (out && g.grad == g.out && g.grad_type != g.out_type)
      return fail(DR_EINVAL, "%s: gradient %lld is scaled in place to another type", what, (long long)i);
  }
  return DR_OK;
}

int hip_result(hipError_t e, const char* what) {
  return e == hipSuccess ? DR_OK : fail(DR_EHIP, "%s: kernel launch: %s", what, hipGetErrorString(e));
}

int check_max_norm(double max_norm, const char* what) {
  return max_norm >= 0 ? DR_OK : fail(DR_EINVAL, "%s: max_norm is %g", what, max_norm);
}

}  // namespace
}  // namespace dr

using namespace dr;

extern "C" int dr_grad_workspace(uint64_t* bytes) {
  clear_error();
  if (!bytes) return fail(DR_EINVAL, "dr_grad_workspace: null argument");
  *bytes = (kGradSums + 1) * sizeof(double);  // and their total
  return DR_OK;
}

extern "C" int dr_grad_norm(const dr_grad* grads, int64_t count, void* workspace, double* sum_squares, float* norm,
                            void* stream) {
  clear_error();
  const char* what = "dr_grad_norm";
  if (int rc = check_list(grads, count, false, what)) return rc;
  if (!aligned(workspace, 8)) return fail(DR_EINVAL, "%s: workspace is null or misaligned", what);
  if ((sum_squares && !aligned(sum_squares, 8)) || (norm && !aligned(norm, 4)))
    return fail(DR_EINVAL, "%s: misaligned result", what);
  hipStream_t st = static_cast<hipStream_t>(stream);
  double* partial = static_cast<double*>(workspace);
  uint32_t nsums = 0;
  hipError_t e = launch_grad_norm(grads, count, partial, &nsums, st);
  if (e == hipSuccess) e = launch_grad_total(partial, nsums, sum_squares, norm, st);
  return hip_result(e, what);
}

extern "C" int dr_grad_scale(const dr_grad* grads, int64_t count, const double* sum_squares, double max_norm,
                             float* norm_out, void* stream) {
  clear_error();
  const char* what = "dr_grad_scale";
  if (int rc = check_list(grads, count, true, what)) return rc;
  if (int rc = check_max_norm(max_norm, what)) return rc;
  if (!aligned(sum_squares, 8) || (norm_out && !aligned(norm_out, 4)))
    return fail(DR_EINVAL, "%s: sum_squares null or misaligned, or norm_out misaligned", what);
  return hip_result(launch_grad_scale(grads, count, sum_squares, 1, max_norm, norm_out, static_cast<hipStream_t>(stream)),
                    what);
}

extern "C" int dr_grad_clip(const dr_grad* grads, int64_t count, double max_norm, void* workspace, float* norm_out,
                            void* stream) {
  clear_error();
  const char* what = "dr_grad_clip";
  if (int rc = check_list(grads, count, true, what)) return rc;
  if (int rc = check_max_norm(max_norm, what)) return rc;
  if (!aligned(workspace, 8) || (norm_out && !aligned(norm_out, 4)))
    return fail(DR_EINVAL, "%s: workspace null or misaligned, or norm_out misaligned", what);
  hipStream_t st = static_cast<hipStream_t>(stream);
  double* partial = static_cast<double*>(workspace);
  uint32_t nsums = 0;
  hipError_t e = launch_grad_norm(grads, count, partial, &nsums, st);
  const double* sums = partial;
  if (e == hipSuccess && nsums > kFewSums) {
    sums = partial + kGradSums;
    e = launch_grad_total(partial, nsums, partial + kGradSums, nullptr, st);
    nsums = 1;
  }
  if (e == hipSuccess) e = launch_grad_scale(grads, count, sums, nsums, max_norm, norm_out, st);
  return hip_result(e, what);
}
