// C ABI of the vocabulary head (declared in include/w2v.h): argument
// validation and launches. Every check runs on the host before any HIP call.
#include <math.h>

#include "distill.h"
#include "head_checks.h"
#include "linear.h"
#include "sample.h"
#include "w2v_internal.h"

namespace w2v {
namespace {

int check_linear(int32_t M, int32_t N, int32_t K, int32_t dtype, int32_t activation,
                 bool backward) {
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
  if (!linear_fits(M, N, K, dtype, backward))
    return fail(W2V_EUNSUPPORTED, "the product has too many tiles for a launch");
  return W2V_OK;
}

int check_distill(int32_t rows, int32_t V, int32_t dtype, const int32_t* ids,
                  const void* teacher, int32_t K, int32_t teacher_dtype, float temperature,
                  float soft, float hard) {
  if (rows < 0) return fail(W2V_EINVAL, "rows must be >= 0");
  if (V < 1) return fail(W2V_EINVAL, "V must be positive");
  if (!known_dtype(dtype)) return fail(W2V_EINVAL, "dtype must be a W2V_DTYPE_* value");
  if (!known_dtype(teacher_dtype))
    return fail(W2V_EINVAL, "teacher_dtype must be a W2V_DTYPE_* value");
  if (K < 0 || K > W2V_MAX_TEACHER)
    return failf(W2V_EINVAL, "K must be in [0, %d]", W2V_MAX_TEACHER);
  if (!(temperature >= 0x1p-20f && temperature <= 0x1p20f))
    return fail(W2V_EINVAL, "temperature must be in [2^-20, 2^20]");
  if (!isfinite(soft) || !isfinite(hard))
    return fail(W2V_EINVAL, "soft and hard must be finite");
  if (rows > 0 && K > 0) {
    if (ids == nullptr) return fail(W2V_EINVAL, "ids is NULL");
    if (teacher == nullptr) return fail(W2V_EINVAL, "teacher is NULL");
  }
  if ((uintptr_t)ids % 4 != 0 || (uintptr_t)teacher % element_bytes(teacher_dtype) != 0)
    return fail(W2V_EINVAL, "ids and teacher must be aligned to their elements");
  return W2V_OK;
}

}  // namespace
}  // namespace w2v

using namespace w2v;

extern "C" {

size_t w2v_linear_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype) {
  if (check_linear(M, N, K, dtype, W2V_ACTIVATION_NONE, false) != W2V_OK) return 0;
  return linear_workspace_bytes(M, N, K, dtype);
}

int w2v_linear(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias,
               const void* residual, int64_t ldr, void* y, int64_t ldy, void* pre,
               int64_t ldp, int32_t M, int32_t N, int32_t K, int32_t dtype,
               int32_t out_dtype, int32_t activation, void* workspace,
               size_t workspace_bytes, void* stream) {
  int rc = check_linear(M, N, K, dtype, activation, false);
  if (rc != W2V_OK) return rc;
  if (out_dtype != dtype && out_dtype != W2V_DTYPE_F32)
    return fail(W2V_EINVAL, "out_dtype must be dtype or W2V_DTYPE_F32");
  if ((rc = check_operand(x, ldx, M, K, dtype, "x")) != W2V_OK) return rc;
  if ((rc = check_operand(w, ldw, N, K, dtype, "w")) != W2V_OK) return rc;
  if ((rc = check_operand(y, ldy, M, N, out_dtype, "y")) != W2V_OK) return rc;
  if (residual != nullptr &&
      (rc = check_operand(residual, ldr, M, N, out_dtype, "residual")) != W2V_OK)
    return rc;
  if (residual == y && ldr != ldy && M > 1)
    return fail(W2V_EINVAL, "a residual in y's memory must have its stride");
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
  if (check_linear(M, N, K, dtype, activation, true) != W2V_OK) return 0;
  return linear_backward_workspace_bytes(M, N, K, dtype, activation);
}

int w2v_linear_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                        const void* w, int64_t ldw, const void* pre, int64_t ldp, void* dx,
                        int64_t lddx, void* dw, int64_t lddw, float* db, int32_t M, int32_t N,
                        int32_t K, int32_t dtype, int32_t activation, void* workspace,
                        size_t workspace_bytes, void* stream) {
  int rc = check_linear(M, N, K, dtype, activation, true);
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

size_t w2v_distill_workspace_bytes(int32_t rows, int32_t V, int32_t dtype) {
  if (rows < 0 || V < 1 || !known_dtype(dtype)) return 0;
  return distill_workspace_bytes(rows, V, dtype);
}

int w2v_distill_loss(const void* logits, int64_t ld, int32_t rows, int32_t V, int32_t dtype,
                     const int32_t* ids, const void* teacher, int32_t K,
                     int32_t teacher_dtype, const int32_t* labels, float temperature,
                     float soft, float hard, const float* row_weight, float* loss,
                     float* stats, void* grad, int64_t ldg, void* workspace,
                     size_t workspace_bytes, void* stream) {
  int rc = check_distill(rows, V, dtype, ids, teacher, K, teacher_dtype, temperature, soft,
                         hard);
  if (rc != W2V_OK) return rc;
  if ((rc = check_operand(logits, ld, rows, V, dtype, "logits")) != W2V_OK) return rc;
  if ((rc = check_array(labels, false, "labels")) != W2V_OK) return rc;
  if ((rc = check_array(row_weight, false, "row_weight")) != W2V_OK) return rc;
  if ((rc = check_array(loss, rows > 0, "loss")) != W2V_OK) return rc;
  if ((rc = check_array(stats, rows > 0, "stats")) != W2V_OK) return rc;
  if (grad != nullptr) {
    if ((rc = check_operand(grad, ldg, rows, V, dtype, "grad")) != W2V_OK) return rc;
    if (grad == logits && ldg != ld)
      return fail(W2V_EINVAL, "grad in the logits' memory must have their stride");
  }
  rc = check_workspace(workspace, workspace_bytes, distill_workspace_bytes(rows, V, dtype));
  if (rc != W2V_OK) return rc;
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  if (rows == 0) return ok();
  DistillArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.rows = rows;
  a.V = V;
  a.dtype = dtype;
  a.ids = ids;
  a.teacher = teacher;
  a.K = K;
  a.teacher_dtype = teacher_dtype;
  a.labels = labels;
  a.temperature = temperature;
  a.soft = soft;
  a.hard = hard;
  a.row_weight = row_weight;
  a.loss = loss;
  a.stats = stats;
  a.grad = grad;
  a.ldg = ldg;
  a.status = status;
  const hipError_t e = launch_distill(a, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "distillation launch");
  return ok();
}

int w2v_distill_backward(const float* dloss, const void* logits, int64_t ld, int32_t rows,
                         int32_t V, int32_t dtype, const int32_t* ids, const void* teacher,
                         int32_t K, int32_t teacher_dtype, const int32_t* labels,
                         float temperature, float soft, float hard, const float* stats,
                         void* grad, int64_t ldg, void* stream) {
  int rc = check_distill(rows, V, dtype, ids, teacher, K, teacher_dtype, temperature, soft,
                         hard);
  if (rc != W2V_OK) return rc;
  if ((rc = check_operand(logits, ld, rows, V, dtype, "logits")) != W2V_OK) return rc;
  if ((rc = check_array(labels, false, "labels")) != W2V_OK) return rc;
  if ((rc = check_array(dloss, rows > 0, "dloss")) != W2V_OK) return rc;
  if ((rc = check_array(stats, rows > 0, "stats")) != W2V_OK) return rc;
  if ((rc = check_operand(grad, ldg, rows, V, dtype, "grad")) != W2V_OK) return rc;
  if (grad == logits && ldg != ld)
    return fail(W2V_EINVAL, "grad in the logits' memory must have their stride");
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  if (rows == 0) return ok();
  DistillArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.rows = rows;
  a.V = V;
  a.dtype = dtype;
  a.ids = ids;
  a.teacher = teacher;
  a.K = K;
  a.teacher_dtype = teacher_dtype;
  a.labels = labels;
  a.temperature = temperature;
  a.soft = soft;
  a.hard = hard;
  a.row_weight = dloss;
  a.stats = const_cast<float*>(stats);  // only read by the backward pass
  a.grad = grad;
  a.ldg = ldg;
  a.status = status;
  const hipError_t e = launch_distill_backward(a, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "distillation backward launch");
  return ok();
}

size_t w2v_sample_workspace_bytes(int32_t rows, int32_t V) {
  if (rows < 0 || V < 1) return 0;
  return sample_workspace_bytes(rows, V);
}

int w2v_sample_words(const void* logits, int64_t ld, const float* uniforms, int64_t ldu,
                     int32_t rows, int32_t V, int32_t dtype, const float* temperatures,
                     float temperature, const int32_t* top_ks, int32_t top_k,
                     const float* top_ps, float top_p, const float* min_ps, float min_p,
                     int32_t* ids, float* logprob, void* workspace, size_t workspace_bytes,
                     void* stream) {
  if (rows < 0) return fail(W2V_EINVAL, "rows must be >= 0");
  if (V < 1) return fail(W2V_EINVAL, "V must be positive");
  if (!known_dtype(dtype)) return fail(W2V_EINVAL, "dtype must be a W2V_DTYPE_* value");
  int rc = check_operand(logits, ld, rows, V, dtype, "logits");
  if (rc != W2V_OK) return rc;
  if (temperatures == nullptr && !(temperature >= 0.0f && isfinite(temperature)))
    return fail(W2V_EINVAL, "temperature must be finite and >= 0");
  if (top_ks == nullptr && top_k < 0) return fail(W2V_EINVAL, "top_k must be >= 0");
  if (top_ks == nullptr && top_k > W2V_MAX_TOP_K && top_k < V)
    return failf(W2V_EUNSUPPORTED, "top_k must be at most %d, or V or more (off)",
                 W2V_MAX_TOP_K);
  if (top_ps == nullptr && !(top_p > 0.0f))
    return fail(W2V_EINVAL, "top_p must be positive");
  if (min_ps == nullptr && !(min_p >= 0.0f && min_p <= 1.0f))
    return fail(W2V_EINVAL, "min_p must be in [0, 1]");
  const bool greedy = temperatures == nullptr && temperature == 0.0f;
  if (uniforms != nullptr || !greedy) {
    rc = check_operand(uniforms, ldu, rows, V, W2V_DTYPE_F32, "uniforms");
    if (rc != W2V_OK) return rc;
  }
  if ((rc = check_array(temperatures, false, "temperatures")) != W2V_OK) return rc;
  if ((rc = check_array(top_ks, false, "top_ks")) != W2V_OK) return rc;
  if ((rc = check_array(top_ps, false, "top_ps")) != W2V_OK) return rc;
  if ((rc = check_array(min_ps, false, "min_ps")) != W2V_OK) return rc;
  if ((rc = check_array(ids, rows > 0, "ids")) != W2V_OK) return rc;
  if ((rc = check_array(logprob, false, "logprob")) != W2V_OK) return rc;
  rc = check_workspace(workspace, workspace_bytes, sample_workspace_bytes(rows, V));
  if (rc != W2V_OK) return rc;
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  if (rows == 0) return ok();
  SampleArgs a{};
  a.logits = logits;
  a.uniforms = uniforms;
  a.ld = ld;
  a.ldu = ldu;
  a.rows = rows;
  a.V = V;
  a.dtype = dtype;
  a.temperatures = temperatures;
  a.top_ks = top_ks;
  a.top_ps = top_ps;
  a.min_ps = min_ps;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.ids = ids;
  a.logprob = logprob;
  a.status = status;
  const hipError_t e = launch_sample(a, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "sampling launch");
  return ok();
}

}  // extern "C"
