// Argument checks shared by the C entry points that take matrices of several
// element types (head_api.hip, ends_api.hip). All run on the host before any HIP
// call.
#pragma once

#include <stdint.h>

#include "w2v_internal.h"

namespace w2v {

inline int element_bytes(int32_t dtype) { return dtype == W2V_DTYPE_F32 ? 4 : 2; }

inline bool known_dtype(int32_t dtype) {
  return dtype == W2V_DTYPE_F32 || dtype == W2V_DTYPE_BF16 || dtype == W2V_DTYPE_F16;
}

// A matrix argument of `rows` rows: there, aligned to its elements, and with
// rows that do not overlap. A matrix without rows may be NULL.
inline int check_operand(const void* p, int64_t ld, int64_t rows, int64_t cols, int32_t dtype,
                  const char* name) {
  if (ld < cols) return failf(W2V_EINVAL, "%s: the row stride must be >= its columns", name);
  if (ld > INT64_MAX / 8 / (rows > 0 ? rows : 1))
    return failf(W2V_EINVAL, "%s: the row stride is out of range", name);
  if (rows == 0) return W2V_OK;
  if (p == nullptr) return failf(W2V_EINVAL, "%s is NULL", name);
  if ((uintptr_t)p % (uintptr_t)element_bytes(dtype) != 0)
    return failf(W2V_EINVAL, "%s must be aligned to its elements", name);
  return W2V_OK;
}

inline int check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need == 0) return W2V_OK;
  if (workspace == nullptr || bytes < need)
    return failf(W2V_EINVAL, "workspace must hold %zu bytes", need);
  if (((uintptr_t)workspace & 255u) != 0)
    return fail(W2V_EINVAL, "workspace must be 256-byte aligned");
  return W2V_OK;
}

// A float or int32 array of the call: there if it is needed, and aligned.
inline int check_array(const void* p, bool needed, const char* name) {
  if (needed && p == nullptr) return failf(W2V_EINVAL, "%s is NULL", name);
  if ((uintptr_t)p % 4 != 0)
    return failf(W2V_EINVAL, "%s must be aligned to its elements", name);
  return W2V_OK;
}

}  // namespace w2v
