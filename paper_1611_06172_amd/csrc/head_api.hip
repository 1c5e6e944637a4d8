// C ABI of the vocabulary head (declared in include/w2v.h): argument
// validation and launches. Every check runs on the host before any HIP call.
#include "linear.h"
#include "w2v_internal.h"

namespace w2v {
namespace {

int element_bytes(int32_t dtype) { return dtype == W2V_DTYPE_F32 ? 4 : 2; }

bool known_dtype(int32_t dtype) {
  return dtype == W2V_DTYPE_F32 || dtype == W2V_DTYPE_BF16 || dtype == W2V_DTYPE_F16;
}

// A matrix argument of `rows` rows: there, aligned to its elements, and with
// rows that do not overlap. A matrix without rows may be NULL.
int check_operand(const void* p, int64_t ld, int64_t rows, int64_t cols, int32_t dtype,
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

int check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need == 0) return W2V_OK;
  if (workspace == nullptr || bytes < need)
    return failf(W2V_EINVAL, "workspace must hold %zu bytes", need);
  if (((uintptr_t)workspace & 255u) != 0)
    return fail(W2V_EINVAL, "workspace must be 256-byte aligned");
  return W2V_OK;
}

int check_linear(int32_t M, int32_t N, int32_t K, int32_t dtype, int32_t activation) {
  if (M < 0) return fail(W2V_EINVAL, "M must be >= 0");
  if (N < 1) return fail(W2V_EINVAL, "N must be positive");
  if (K < 1) return fail(W2V_EINVAL, "K must be positive");
  if (!known_dtype(dtype)) return fail(W2V_EINVAL, "dtype must be a W2V_DTYPE_* value");
  if (activation < W2V_ACTIVATION_NONE || activation > W2V_ACTIVATION_SIGMOID)
    return fail(W2V_EINVAL, "activation must be a W2V_ACTIVATION_* value");
  // blocks of 64 x 64 of an output, and its splits, are counted in 31 bits
  const int64_t m = ((int64_t)M + 63) / 64, n = ((int64_t)N + 63) / 64,
                k = ((int64_t)K + 63) / 64;
  const int64_t most = INT32_MAX / 64;
  if (m * n > most || m * k > most || n * k > most)
    return fail(W2V_EUNSUPPORTED, "the product has too many tiles");
  return W2V_OK;
}

}  // namespace
}  // namespace w2v

using namespace w2v;

extern "C" {

size_t w2v_linear_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype) {
  if (check_linear(M, N, K, dtype, W2V_ACTIVATION_NONE) != W2V_OK) return 0;
  return linear_workspace_bytes(M, N, K, dtype);
}

int w2v_linear(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias,
               const void* residual, int64_t ldr, void* y, int64_t ldy, void* pre,
               int64_t ldp, int32_t M, int32_t N, int32_t K, int32_t dtype,
               int32_t out_dtype, int32_t activation, void* workspace,
               size_t workspace_bytes, void* stream) {
  int rc = check_linear(M, N, K, dtype, activation);
  if (rc != W2V_OK) return rc;
  if (out_dtype != dtype && out_dtype != W2V_DTYPE_F32)
    return fail(W2V_EINVAL, "out_dtype must be dtype or W2V_DTYPE_F32");
  if ((rc = check_operand(x, ldx, M, K, dtype, "x")) != W2V_OK) return rc;
  if ((rc = check_operand(w, ldw, N, K, dtype, "w")) != W2V_OK) return rc;
  if ((rc = check_operand(y, ldy, M, N, out_dtype, "y")) != W2V_OK) return rc;
  if (residual != nullptr &&
      (rc = check_operand(residual, ldr, M, N, out_dtype, "residual")) != W2V_OK)
    return rc;
  if (pre != nullptr && (rc = check_operand(pre, ldp, M, N, dtype, "pre")) != W2V_OK)
    return rc;
  if ((uintptr_t)bias % 4 != 0)
    return fail(W2V_EINVAL, "bias must be aligned to its elements");
  rc = check_workspace(workspace, workspace_bytes, linear_workspace_bytes(M, N, K, dtype));
  if (rc != W2V_OK) return rc;
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  if (M == 0) return ok();
  LinearArgs a{};
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.residual = residual;
  a.y = y;
  a.pre = pre;
  a.ldx = ldx;
  a.ldw = ldw;
  a.ldr = ldr;
  a.ldy = ldy;
  a.ldp = ldp;
  a.M = M;
  a.N = N;
  a.K = K;
  a.dtype = dtype;
  a.out_dtype = out_dtype;
  a.activation = activation;
  const hipError_t e = launch_linear(a, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "linear launch");
  return ok();
}

size_t w2v_linear_backward_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype,
                                           int32_t activation) {
  if (check_linear(M, N, K, dtype, activation) != W2V_OK) return 0;
  return linear_backward_workspace_bytes(M, N, K, dtype, activation);
}

int w2v_linear_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                        const void* w, int64_t ldw, const void* pre, int64_t ldp, void* dx,
                        int64_t lddx, void* dw, int64_t lddw, float* db, int32_t M, int32_t N,
                        int32_t K, int32_t dtype, int32_t activation, void* workspace,
                        size_t workspace_bytes, void* stream) {
  int rc = check_linear(M, N, K, dtype, activation);
  if (rc != W2V_OK) return rc;
  if ((rc = check_operand(dy, lddy, M, N, dtype, "dy")) != W2V_OK) return rc;
  if ((rc = check_operand(x, ldx, M, K, dtype, "x")) != W2V_OK) return rc;
  if ((rc = check_operand(w, ldw, N, K, dtype, "w")) != W2V_OK) return rc;
  if (activation != W2V_ACTIVATION_NONE &&
      (rc = check_operand(pre, ldp, M, N, dtype, "pre")) != W2V_OK)
    return rc;
  if (dx != nullptr && (rc = check_operand(dx, lddx, M, K, dtype, "dx")) != W2V_OK) return rc;
  if (dw != nullptr && (rc = check_operand(dw, lddw, N, K, dtype, "dw")) != W2V_OK) return rc;
  if ((uintptr_t)db % 4 != 0) return fail(W2V_EINVAL, "db must be aligned to its elements");
  rc = check_workspace(workspace, workspace_bytes,
                       linear_backward_workspace_bytes(M, N, K, dtype, activation));
  if (rc != W2V_OK) return rc;
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  LinearBackwardArgs a{};
  a.dy = dy;
  a.x = x;
  a.w = w;
  a.pre = pre;
  a.dx = dx;
  a.dw = dw;
  a.db = db;
  a.lddy = lddy;
  a.ldx = ldx;
  a.ldw = ldw;
  a.ldp = ldp;
  a.lddx = lddx;
  a.lddw = lddw;
  a.M = M;
  a.N = N;
  a.K = K;
  a.dtype = dtype;
  a.activation = activation;
  const hipError_t e = launch_linear_backward(a, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "linear backward launch");
  return ok();
}

}  // extern "C"
