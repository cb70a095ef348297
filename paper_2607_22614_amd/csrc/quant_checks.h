// Argument checks that the entry points of the 8-bit operators share (quant.cpp, gated.cpp).
#pragma once

#include <hip/hip_runtime.h>

#include "dr_internal.h"
#include "quant_kernels.h"

namespace dr {

inline bool aligned(const void* p, uintptr_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline int64_t padded(int64_t cols) { return ceil_div(cols, kBlock) * kBlock; }

inline int check_shape(int64_t rows, int64_t cols, int32_t block_rows, const char* what, const char* name) {
  if (rows < 0 || rows >= kMaxQRows || cols < 0 || cols > kMaxQCols)
    return fail(DR_EINVAL, "%s: %s is %lld x %lld (rows are below 2^26, columns at most 2^23)", what, name,
                (long long)rows, (long long)cols);
  if (block_rows != 1 && block_rows != kBlock)
    return fail(DR_EINVAL, "%s: %s has blocks of %d rows (1 or 128)", what, name, block_rows);
  return DR_OK;
}

inline int check_matrix(const dr_qmatrix* m, const char* what, const char* name) {
  if (!m) return fail(DR_EINVAL, "%s: %s is null", what, name);
  if (int rc = check_shape(m->rows, m->cols, m->block_rows, what, name)) return rc;
  if (m->reserved) return fail(DR_EINVAL, "%s: %s: reserved field is not 0", what, name);
  if (m->stride < padded(m->cols) || m->stride > kMaxQCols || m->stride % 16)
    return fail(DR_EINVAL, "%s: %s: stride %lld (a multiple of 16 from %lld to 2^23)", what, name, (long long)m->stride,
                (long long)padded(m->cols));
  if (m->rows && m->cols && (!aligned(m->data, 16) || !aligned(m->scales, 4)))
    return fail(DR_EINVAL, "%s: %s: data (16-byte) or scales (4-byte) null or misaligned", what, name);
  return DR_OK;
}

inline QView view(const dr_qmatrix& m) {
  return QView{static_cast<uint8_t*>(m.data),         static_cast<uint8_t*>(m.scales),
               m.stride,                              (uint32_t)m.rows,
               (uint32_t)m.cols,                      (uint32_t)ceil_div(m.rows, m.block_rows),
               m.block_rows == 1 ? 0 : 7};
}

inline int element_bytes(int32_t type) { return type == DR_TYPE_F32 ? 4 : type == DR_TYPE_BF16 ? 2 : 0; }

// A dense matrix of `type` with rows of row_stride elements.
inline int check_dense(const void* p, int32_t type, int64_t rows, int64_t cols, int64_t row_stride, const char* what,
                const char* name) {
  const int size = element_bytes(type);
  if (!size) return fail(DR_EINVAL, "%s: %s has unknown type %d", what, name, type);
  if (row_stride < cols || row_stride > (1ll << 40))
    return fail(DR_EINVAL, "%s: %s: row stride %lld for %lld columns", what, name, (long long)row_stride, (long long)cols);
  if (rows && cols && !aligned(p, size)) return fail(DR_EINVAL, "%s: %s is null or misaligned", what, name);
  return DR_OK;
}

// The tiles of a product are counted in 32 bits.
inline int check_results(int64_t m, int64_t n, const char* what) {
  return m * n <= 1ll << 38 ? DR_OK : fail(DR_EINVAL, "%s: %lld x %lld results (at most 2^38)", what, (long long)m, (long long)n);
}

inline int hip_result(hipError_t e, const char* what) {
  return e == hipSuccess ? DR_OK : fail(DR_EHIP, "%s: kernel launch: %s", what, hipGetErrorString(e));
}

inline int check_workspace(const void* p, uint64_t have, uint64_t need, const char* what) {
  if (have < need || (need && !aligned(p, 16)))
    return fail(DR_EINVAL, "%s: workspace of %llu bytes null, misaligned or too small (%llu needed)", what,
                (unsigned long long)have, (unsigned long long)need);
  return DR_OK;
}

// Quantizes src into q and/or qt, whose shapes and pointers have been checked.
int quantize_checked(const void* src, int32_t type, int64_t rows, int64_t cols, int64_t row_stride, const dr_qmatrix* q, const dr_qmatrix* qt,
                     hipStream_t st, const char* what);

}  // namespace dr
