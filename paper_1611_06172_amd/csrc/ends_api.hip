// C ABI of a word model's ends (declared in include/w2v.h): words in, dropout,
// scores from 4-bit weights, beam search. Argument validation and launches; every
// check runs on the host before any HIP call.
#include <math.h>

#include "beam.h"
#include "dropout.h"
#include "embed.h"
#include "head_checks.h"
#include "linear_q4.h"
#include "w2v_internal.h"

namespace w2v {
namespace {

// Columns whose packs and offsets within a row are counted in 31 bits.
constexpr int32_t kMaxColumns = 1 << 24;

int check_embed(int32_t n, int32_t V, int32_t D, int32_t dtype, int32_t out_dtype,
                const char* out_name, float scale, const int32_t* ids) {
  if (n < 0) return fail(W2V_EINVAL, "n must be >= 0");
  if (V < 1) return fail(W2V_EINVAL, "V must be positive");
  if (D < 1) return fail(W2V_EINVAL, "D must be positive");
  if (D > kMaxColumns) return failf(W2V_EUNSUPPORTED, "D must be at most %d", kMaxColumns);
  if (!known_dtype(dtype)) return fail(W2V_EINVAL, "dtype must be a W2V_DTYPE_* value");
  if (!known_dtype(out_dtype))
    return failf(W2V_EINVAL, "%s must be a W2V_DTYPE_* value", out_name);
  if (!isfinite(scale)) return fail(W2V_EINVAL, "scale must be finite");
  return check_array(ids, n > 0, "ids");
}

int check_q4(int32_t N, int32_t K, int32_t group, int32_t dtype) {
  if (N < 1) return fail(W2V_EINVAL, "N must be positive");
  if (K < 1) return fail(W2V_EINVAL, "K must be positive");
  if (K > kMaxColumns) return failf(W2V_EUNSUPPORTED, "K must be at most %d", kMaxColumns);
  if (group != 32 && group != 64 && group != 128)
    return fail(W2V_EINVAL, "group must be 32, 64 or 128");
  if (!known_dtype(dtype)) return fail(W2V_EINVAL, "dtype must be a W2V_DTYPE_* value");
  return W2V_OK;
}

int check_packed(const void* packed, const void* scales) {
  if (packed == nullptr) return fail(W2V_EINVAL, "packed is NULL");
  if (scales == nullptr) return fail(W2V_EINVAL, "scales is NULL");
  if (((uintptr_t)packed | (uintptr_t)scales) % 16 != 0)
    return fail(W2V_EINVAL, "packed and scales must be 16-byte aligned");
  return W2V_OK;
}

int check_beams(int32_t batch, int32_t beams, int32_t width) {
  if (batch < 0) return fail(W2V_EINVAL, "batch must be >= 0");
  if (beams < 1 || beams > W2V_MAX_BEAMS)
    return failf(W2V_EINVAL, "beams must be in [1, %d]", W2V_MAX_BEAMS);
  if (width < 1 || width > W2V_MAX_BEAMS)
    return failf(W2V_EINVAL, "width must be in [1, %d]", W2V_MAX_BEAMS);
  if (batch > INT32_MAX / W2V_MAX_BEAMS)
    return failf(W2V_EUNSUPPORTED, "batch must be at most %d", INT32_MAX / W2V_MAX_BEAMS);
  return W2V_OK;
}

}  // namespace
}  // namespace w2v

using namespace w2v;

extern "C" {

int w2v_embed(const int32_t* ids, int32_t n, const void* weight, int64_t ldw, int32_t V,
              int32_t D, int32_t dtype, float scale, void* y, int64_t ldy, int32_t out_dtype,
              void* stream) {
  int rc = check_embed(n, V, D, dtype, out_dtype, "out_dtype", scale, ids);
  if (rc != W2V_OK) return rc;
  if ((rc = check_operand(weight, ldw, V, D, dtype, "weight")) != W2V_OK) return rc;
  if ((rc = check_operand(y, ldy, n, D, out_dtype, "y")) != W2V_OK) return rc;
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  if (n == 0) return ok();
  EmbedArgs a{};
  a.ids = ids;
  a.weight = weight;
  a.y = y;
  a.ldw = ldw;
  a.ldy = ldy;
  a.n = n;
  a.V = V;
  a.D = D;
  a.dtype = dtype;
  a.out_dtype = out_dtype;
  a.scale = scale;
  a.status = status;
  const hipError_t e = launch_embed(a, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "embedding launch");
  return ok();
}

size_t w2v_embed_backward_workspace_bytes(int32_t n, int32_t V, int32_t D) {
  if (n < 0 || V < 1 || D < 1 || D > kMaxColumns) return 0;
  return embed_backward_workspace_bytes(n, V, D);
}

int w2v_embed_backward(const void* dy, int64_t lddy, const int32_t* ids, int32_t n,
                       int32_t dtype, float scale, void* grad, int64_t ldg, int32_t V, int32_t D,
                       int32_t grad_dtype, int32_t accumulate, void* workspace,
                       size_t workspace_bytes, void* stream) {
  int rc = check_embed(n, V, D, dtype, grad_dtype, "grad_dtype", scale, ids);
  if (rc != W2V_OK) return rc;
  if (accumulate != 0 && accumulate != 1)
    return fail(W2V_EINVAL, "accumulate must be 0 or 1");
  if ((rc = check_operand(dy, lddy, n, D, dtype, "dy")) != W2V_OK) return rc;
  if ((rc = check_operand(grad, ldg, V, D, grad_dtype, "grad")) != W2V_OK) return rc;
  rc = check_workspace(workspace, workspace_bytes, embed_backward_workspace_bytes(n, V, D));
  if (rc != W2V_OK) return rc;
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  EmbedBackwardArgs a{};
  a.dy = dy;
  a.ids = ids;
  a.grad = grad;
  a.lddy = lddy;
  a.ldg = ldg;
  a.n = n;
  a.V = V;
  a.D = D;
  a.dtype = dtype;
  a.grad_dtype = grad_dtype;
  a.accumulate = accumulate != 0;
  a.scale = scale;
  a.status = status;
  const hipError_t e = launch_embed_backward(a, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "embedding backward launch");
  return ok();
}

int w2v_dropout(const void* x, int64_t ldx, const void* residual, int64_t ldr, void* y,
                int64_t ldy, int32_t rows, int32_t cols, int32_t dtype, double p, uint64_t seed,
                uint64_t offset, const int64_t* offset_dev, void* stream) {
  if (rows < 0) return fail(W2V_EINVAL, "rows must be >= 0");
  if (cols < 1) return fail(W2V_EINVAL, "cols must be positive");
  if (cols > (1 << 30)) return failf(W2V_EUNSUPPORTED, "cols must be at most %d", 1 << 30);
  if (!known_dtype(dtype)) return fail(W2V_EINVAL, "dtype must be a W2V_DTYPE_* value");
  if (!(p >= 0.0 && p <= 1.0)) return fail(W2V_EINVAL, "p must be in [0, 1]");
  int rc = check_operand(x, ldx, rows, cols, dtype, "x");
  if (rc != W2V_OK) return rc;
  if ((rc = check_operand(y, ldy, rows, cols, dtype, "y")) != W2V_OK) return rc;
  if (residual != nullptr &&
      (rc = check_operand(residual, ldr, rows, cols, dtype, "residual")) != W2V_OK)
    return rc;
  if (rows > 1 && ((x == y && ldx != ldy) || (residual == y && ldr != ldy)))
    return fail(W2V_EINVAL, "x or a residual in y's memory must have its stride");
  if ((uintptr_t)offset_dev % 8 != 0)
    return fail(W2V_EINVAL, "offset_dev must be aligned to its element");
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  if (rows == 0) return ok();
  DropoutArgs a{};
  a.x = x;
  a.residual = residual;
  a.y = y;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldy = ldy;
  a.rows = rows;
  a.cols = cols;
  a.dtype = dtype;
  a.below = (uint64_t)floor(p * 0x1p32 + 0.5);
  a.scale = a.below >> 32 != 0 ? 0.0f : (float)(0x1p32 / (0x1p32 - (double)a.below));
  a.seed = seed;
  a.offset = offset;
  a.offset_dev = offset_dev;
  const hipError_t e = launch_dropout(a, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "dropout launch");
  return ok();
}

size_t w2v_q4_packed_bytes(int32_t N, int32_t K, int32_t group) {
  if (check_q4(N, K, group, W2V_DTYPE_F32) != W2V_OK) return 0;
  const Q4Shape q = q4_shape(N, K, group);
  return (size_t)q.tiles * (size_t)q.blocks * 256;
}

size_t w2v_q4_scale_count(int32_t N, int32_t K, int32_t group) {
  if (check_q4(N, K, group, W2V_DTYPE_F32) != W2V_OK) return 0;
  const Q4Shape q = q4_shape(N, K, group);
  return (size_t)q.tiles * (size_t)q.groups * 16;
}

int w2v_quantize_q4(const void* w, int64_t ldw, int32_t N, int32_t K, int32_t dtype,
                    int32_t group, void* packed, void* scales, void* stream) {
  int rc = check_q4(N, K, group, dtype);
  if (rc != W2V_OK) return rc;
  if ((rc = check_operand(w, ldw, N, K, dtype, "w")) != W2V_OK) return rc;
  if ((rc = check_packed(packed, scales)) != W2V_OK) return rc;
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  const QuantizeArgs a{w, ldw, dtype, (uint32_t*)packed, scales};
  const hipError_t e = launch_quantize_q4(a, q4_shape(N, K, group), (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "quantisation launch");
  return ok();
}

int w2v_linear_q4(const void* x, int64_t ldx, const void* packed, const void* scales,
                  const float* bias, void* y, int64_t ldy, int32_t M, int32_t N, int32_t K,
                  int32_t group, int32_t dtype, int32_t out_dtype, void* stream) {
  if (M < 0) return fail(W2V_EINVAL, "M must be >= 0");
  if (M > W2V_MAX_Q4_ROWS)
    return failf(W2V_EUNSUPPORTED, "M must be at most %d", W2V_MAX_Q4_ROWS);
  int rc = check_q4(N, K, group, dtype);
  if (rc != W2V_OK) return rc;
  if (out_dtype != dtype && out_dtype != W2V_DTYPE_F32)
    return fail(W2V_EINVAL, "out_dtype must be dtype or W2V_DTYPE_F32");
  if ((rc = check_operand(x, ldx, M, K, dtype, "x")) != W2V_OK) return rc;
  if ((rc = check_packed(packed, scales)) != W2V_OK) return rc;
  if ((rc = check_operand(y, ldy, M, N, out_dtype, "y")) != W2V_OK) return rc;
  if ((rc = check_array(bias, false, "bias")) != W2V_OK) return rc;
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  if (M == 0) return ok();
  LinearQ4Args a{};
  a.x = x;
  a.packed = (const uint32_t*)packed;
  a.scales = scales;
  a.bias = bias;
  a.y = y;
  a.ldx = ldx;
  a.ldy = ldy;
  a.M = M;
  a.dtype = dtype;
  a.out_dtype = out_dtype;
  const hipError_t e = launch_linear_q4(a, q4_shape(N, K, group), (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "4-bit product launch");
  return ok();
}

size_t w2v_beam_step_workspace_bytes(int32_t batch, int32_t beams, int32_t width, int32_t V,
                                     int32_t dtype) {
  if (check_beams(batch, beams, width) != W2V_OK || V < 1 || !known_dtype(dtype)) return 0;
  return batch == 0 ? 0 : beam_workspace_bytes(batch, beams, width, V, dtype);
}

int w2v_beam_step(const void* logits, int64_t ld, int32_t batch, int32_t beams, int32_t V,
                  int32_t dtype, const float* scores, const uint8_t* finished, int32_t end,
                  int32_t width, int32_t* words, int32_t* parents, float* new_scores,
                  uint8_t* new_finished, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_beams(batch, beams, width);
  if (rc != W2V_OK) return rc;
  if (V < 1) return fail(W2V_EINVAL, "V must be positive");
  if (!known_dtype(dtype)) return fail(W2V_EINVAL, "dtype must be a W2V_DTYPE_* value");
  if (end < -1 || end >= V) return fail(W2V_EINVAL, "end must be a word or -1");
  if (finished != nullptr && end < 0)
    return fail(W2V_EINVAL, "finished needs the word that ends a beam");
  rc = check_operand(logits, ld, (int64_t)batch * beams, V, dtype, "logits");
  if (rc != W2V_OK) return rc;
  if ((rc = check_array(scores, batch > 0, "scores")) != W2V_OK) return rc;
  if ((rc = check_array(words, batch > 0, "words")) != W2V_OK) return rc;
  if ((rc = check_array(parents, batch > 0, "parents")) != W2V_OK) return rc;
  if ((rc = check_array(new_scores, batch > 0, "new_scores")) != W2V_OK) return rc;
  if (batch > 0 && (new_scores == scores || (finished != nullptr && new_finished == finished)))
    return fail(W2V_EINVAL, "the new scores and flags must not replace the old ones in place");
  rc = check_workspace(workspace, workspace_bytes,
                       batch == 0 ? 0 : beam_workspace_bytes(batch, beams, width, V, dtype));
  if (rc != W2V_OK) return rc;
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  if (batch == 0) return ok();
  BeamArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.batch = batch;
  a.beams = beams;
  a.V = V;
  a.dtype = dtype;
  a.width = width;
  a.end = end;
  a.scores = scores;
  a.finished = finished;
  a.words = words;
  a.parents = parents;
  a.new_scores = new_scores;
  a.new_finished = new_finished;
  const hipError_t e = launch_beam_step(a, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "beam search launch");
  return ok();
}

int w2v_beam_reorder(const w2v_beam_state* states, int32_t count, const int32_t* parents,
                     int32_t batch, int32_t beams, int32_t width, void* stream) {
  int rc = check_beams(batch, beams, width);
  if (rc != W2V_OK) return rc;
  if (count < 0 || count > W2V_MAX_BEAM_STATES)
    return failf(W2V_EINVAL, "count must be in [0, %d]", W2V_MAX_BEAM_STATES);
  if (count > 0 && states == nullptr) return fail(W2V_EINVAL, "states is NULL");
  if ((rc = check_array(parents, batch > 0 && count > 0, "parents")) != W2V_OK) return rc;
  ReorderArgs a{};
  for (int32_t i = 0; i < count; i++) {
    const w2v_beam_state& s = states[i];
    if (s.row_bytes < 1) return fail(W2V_EINVAL, "states: row_bytes must be positive");
    if (s.row_bytes > W2V_MAX_STATE_BYTES)
      return fail(W2V_EUNSUPPORTED, "states: a row has too many bytes");
    const int64_t rows = (int64_t)batch * (beams > width ? beams : width);
    if (s.src_stride < s.row_bytes || s.dst_stride < s.row_bytes)
      return fail(W2V_EINVAL, "states: the row strides must be >= the row's bytes");
    const int64_t most = INT64_MAX / 2 / (rows > 0 ? rows : 1);
    if (s.src_stride > most || s.dst_stride > most)
      return fail(W2V_EINVAL, "states: a row stride is out of range");
    if (batch > 0 && (s.src == nullptr || s.dst == nullptr))
      return fail(W2V_EINVAL, "states: src or dst is NULL");
    // also not by states that change places
    for (int32_t j = 0; j < count && batch > 0; j++)
      if (s.dst == states[j].src || (j != i && s.dst == states[j].dst))
        return fail(W2V_EINVAL, "states: rows cannot be reordered in place");
    a.states[i] = s;
  }
  int32_t* status = nullptr;
  rc = enter_call(&status);
  if (rc != W2V_OK) return rc;
  if (batch == 0 || count == 0) return ok();
  a.parents = parents;
  a.count = count;
  a.batch = batch;
  a.beams = beams;
  a.width = width;
  a.status = status;
  const hipError_t e = launch_beam_reorder(a, (hipStream_t)stream);
  if (e != hipSuccess) return launch_failed(e, "beam reorder launch");
  return ok();
}

}  // extern "C"
