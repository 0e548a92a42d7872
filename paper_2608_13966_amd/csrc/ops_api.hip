// ops_api.hip -- the C ABI of quasar_ops.h: argument checks and dispatch.
#include <math.h>

#include "ops_internal.h"
#include "quasar_ops.h"

namespace {

using quasar::size_of;

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int64_t kMaxStride = (int64_t)1 << 40;  // rows * stride stays far inside int64

bool f32_or_bf16(int32_t t) { return t == QUASAR_F32 || t == QUASAR_BF16; }
bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// one matrix operand (p may be NULL: absent)
int check_matrix(const void* p, int64_t rows, int64_t cols, int64_t stride, int32_t dtype) {
  if (p == nullptr) return QUASAR_OK;
  if (rows > 1 && (stride < cols || stride > kMaxStride)) return QUASAR_ERR_SHAPE;
  return misaligned(p, size_of(dtype)) ? QUASAR_ERR_ALIGN : QUASAR_OK;
}

int status_of(hipError_t e) { return e == hipSuccess ? QUASAR_OK : QUASAR_ERR_DEVICE; }

// desc's own checks, through a size query that fails for an invalid one; the
// status itself from a call of quasar_check with stand-in buffers
int check_desc(const quasar_desc* d) {
  if (d == nullptr) return QUASAR_ERR_ARG;
  void* const p = reinterpret_cast<void*>(uintptr_t{16});
  const bool nv = d->format == QUASAR_NVFP4;
  return quasar_check(d, p, reinterpret_cast<float*>(p), nullptr, reinterpret_cast<uint8_t*>(p), p,
                      reinterpret_cast<float*>(p), nullptr, nullptr, nullptr, nv ? reinterpret_cast<float*>(p) : nullptr,
                      nv ? reinterpret_cast<float*>(p) : nullptr, nullptr, 0);
}

#define QUASAR_TRY(X)                      \
  do {                                     \
    const int s_ = (X);                    \
    if (s_ != QUASAR_OK) return s_;        \
  } while (0)

}  // namespace

extern "C" {

int quasar_add_rms_norm_check(const quasar_norm* a) {
  if (a == nullptr) return QUASAR_ERR_ARG;
  if (a->rows < 0 || a->rows > kMaxRows || a->cols < 1 || a->cols > QUASAR_NORM_MAX_COLS) return QUASAR_ERR_SHAPE;
  if (!f32_or_bf16(a->x_dtype) || !f32_or_bf16(a->weight_dtype)) return QUASAR_ERR_FORMAT;
  if (a->residual && !f32_or_bf16(a->residual_dtype)) return QUASAR_ERR_FORMAT;
  if (a->y && !f32_or_bf16(a->y_dtype)) return QUASAR_ERR_FORMAT;
  if (!(a->eps >= 0.0f && a->eps < INFINITY)) return QUASAR_ERR_ARG;
  if (a->rows == 0) return QUASAR_OK;
  if (a->x == nullptr || a->weight == nullptr) return QUASAR_ERR_ARG;
  if ((a->q == nullptr) != (a->scale == nullptr)) return QUASAR_ERR_ARG;
  if (a->h && !a->residual) return QUASAR_ERR_ARG;
  QUASAR_TRY(check_matrix(a->x, a->rows, a->cols, a->x_stride, a->x_dtype));
  QUASAR_TRY(check_matrix(a->residual, a->rows, a->cols, a->residual_stride, a->residual_dtype));
  QUASAR_TRY(check_matrix(a->h, a->rows, a->cols, a->h_stride, a->residual_dtype));
  QUASAR_TRY(check_matrix(a->y, a->rows, a->cols, a->y_stride, a->y_dtype));
  QUASAR_TRY(check_matrix(a->q, a->rows, a->cols, a->q_stride, QUASAR_E4M3));
  if (misaligned(a->weight, size_of(a->weight_dtype)) || misaligned(a->scale, 4) || misaligned(a->rstd, 4))
    return QUASAR_ERR_ALIGN;
  return QUASAR_OK;
}

int quasar_add_rms_norm(const quasar_norm* a, void* stream) {
  QUASAR_TRY(quasar_add_rms_norm_check(a));
  if (a->rows == 0) return QUASAR_OK;
  return status_of(quasar::launch_norm(*a, reinterpret_cast<hipStream_t>(stream)));
}

size_t quasar_add_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 1 || rows > kMaxRows || cols < 1 || cols > QUASAR_NORM_MAX_COLS) return 0;
  return quasar::norm_backward_workspace(rows, cols);
}

int quasar_add_rms_norm_backward_check(const quasar_norm_backward* a) {
  if (a == nullptr) return QUASAR_ERR_ARG;
  if (a->rows < 0 || a->rows > kMaxRows || a->cols < 1 || a->cols > QUASAR_NORM_MAX_COLS) return QUASAR_ERR_SHAPE;
  if (!f32_or_bf16(a->dy_dtype) || !f32_or_bf16(a->h_dtype) || !f32_or_bf16(a->weight_dtype) ||
      !f32_or_bf16(a->dx_dtype))
    return QUASAR_ERR_FORMAT;
  if (a->rows == 0) return QUASAR_OK;
  if (!a->dy || !a->h || !a->weight || !a->rstd || !a->dx) return QUASAR_ERR_ARG;
  QUASAR_TRY(check_matrix(a->dy, a->rows, a->cols, a->dy_stride, a->dy_dtype));
  QUASAR_TRY(check_matrix(a->h, a->rows, a->cols, a->h_stride, a->h_dtype));
  QUASAR_TRY(check_matrix(a->dh, a->rows, a->cols, a->dh_stride, a->dx_dtype));
  QUASAR_TRY(check_matrix(a->dx, a->rows, a->cols, a->dx_stride, a->dx_dtype));
  if (misaligned(a->weight, size_of(a->weight_dtype)) || misaligned(a->rstd, 4) || misaligned(a->dweight, 4) ||
      misaligned(a->workspace, 16))
    return QUASAR_ERR_ALIGN;
  const size_t need = a->dweight ? quasar_add_rms_norm_backward_workspace_bytes(a->rows, a->cols) : 0;
  if (need > 0 && (a->workspace == nullptr || a->workspace_bytes < need)) return QUASAR_ERR_WORKSPACE;
  return QUASAR_OK;
}

int quasar_add_rms_norm_backward(const quasar_norm_backward* a, void* stream) {
  QUASAR_TRY(quasar_add_rms_norm_backward_check(a));
  if (a->rows == 0) return QUASAR_OK;
  return status_of(quasar::launch_norm_backward(*a, reinterpret_cast<hipStream_t>(stream)));
}

size_t quasar_distill_topk_workspace_bytes(int64_t rows, int64_t classes) {
  if (rows < 1 || rows > kMaxRows || classes < 1 || classes >= kMaxRows - 65535) return 0;
  return quasar::distill_workspace(rows, classes);
}

int quasar_distill_topk_check(const quasar_distill* a, int what) {
  if (a == nullptr || what < 0 || what > 2) return QUASAR_ERR_ARG;
  if (a->rows < 0 || a->classes < 1 || a->classes >= kMaxRows - 65535) return QUASAR_ERR_SHAPE;
  // parts of rows, of 2^11 classes or more, are counted in 32 bits
  if (a->rows > kMaxRows / ((a->classes + 1023) / 1024)) return QUASAR_ERR_SHAPE;
  if (a->listed < 1 || a->listed > QUASAR_DISTILL_MAX_LISTED) return QUASAR_ERR_SHAPE;
  if (!f32_or_bf16(a->logits_dtype) || !f32_or_bf16(a->teacher_dtype)) return QUASAR_ERR_FORMAT;
  if (a->index_bits != 32 && a->index_bits != 64) return QUASAR_ERR_FORMAT;
  if (!(a->temperature > 0.0f && a->temperature < INFINITY && 1.0f / a->temperature < INFINITY)) return QUASAR_ERR_ARG;
  if (!(fabsf(a->grad_scale) < INFINITY)) return QUASAR_ERR_ARG;
  if (a->rows == 0) return QUASAR_OK;
  if (!a->logits || !a->index || !a->teacher || !a->lse) return QUASAR_ERR_ARG;
  if ((what != 1) != (a->loss != nullptr) || (what != 0) != (a->grad != nullptr)) return QUASAR_ERR_ARG;
  if (what != 1 && a->grad_loss) return QUASAR_ERR_ARG;
  QUASAR_TRY(check_matrix(a->logits, a->rows, a->classes, a->logits_stride, a->logits_dtype));
  QUASAR_TRY(check_matrix(a->grad, a->rows, a->classes, a->grad_stride, a->logits_dtype));
  if (a->grad == a->logits && a->rows > 1 && a->grad_stride != a->logits_stride) return QUASAR_ERR_ARG;
  if (misaligned(a->index, (uintptr_t)a->index_bits / 8) || misaligned(a->teacher, size_of(a->teacher_dtype)) ||
      misaligned(a->row_weight, 4) || misaligned(a->grad_loss, 4) || misaligned(a->loss, 4) || misaligned(a->lse, 4) ||
      misaligned(a->workspace, 16))
    return QUASAR_ERR_ALIGN;
  if (what != 1) {
    const size_t need = quasar::distill_workspace(a->rows, a->classes);
    if (need > 0 && (a->workspace == nullptr || a->workspace_bytes < need)) return QUASAR_ERR_WORKSPACE;
  }
  return QUASAR_OK;
}

static int distill(const quasar_distill* a, int what, void* stream) {
  QUASAR_TRY(quasar_distill_topk_check(a, what));
  if (a->rows == 0) return QUASAR_OK;
  return status_of(quasar::launch_distill(*a, what, reinterpret_cast<hipStream_t>(stream)));
}
int quasar_distill_topk(const quasar_distill* a, void* stream) { return distill(a, 0, stream); }
int quasar_distill_topk_backward(const quasar_distill* a, void* stream) { return distill(a, 1, stream); }
int quasar_distill_topk_grad(const quasar_distill* a, void* stream) { return distill(a, 2, stream); }

size_t quasar_linear_codes_workspace_bytes(const quasar_desc* d, int64_t tokens, int32_t x_dtype) {
  (void)x_dtype;
  if (check_desc(d) != QUASAR_OK || tokens < 1 || tokens > kMaxRows) return 0;
  return quasar::linear_workspace(*d, tokens);
}

int quasar_linear_codes_check(const quasar_desc* d, const quasar_linear* a) {
  if (a == nullptr) return QUASAR_ERR_ARG;
  QUASAR_TRY(check_desc(d));
  // byte offsets inside 256 rows of r, and grids, stay inside 32 bits (y of 2^27 tiles is beyond the card's memory)
  if (a->tokens < 0 || a->tokens > (int64_t)1 << 28 || d->rows > (int64_t)1 << 28 || d->cols > (int64_t)1 << 22 ||
      ((a->tokens + 127) / 128) * ((d->rows + 127) / 128) > (int64_t)1 << 27)
    return QUASAR_ERR_SHAPE;
  if (a->x_dtype != QUASAR_BF16 && a->x_dtype != QUASAR_E4M3) return QUASAR_ERR_FORMAT;
  if (!f32_or_bf16(a->y_dtype) || (a->bias && !f32_or_bf16(a->bias_dtype)) ||
      (a->residual && !f32_or_bf16(a->residual_dtype)))
    return QUASAR_ERR_FORMAT;
  if (a->act < QUASAR_ACT_NONE || a->act > QUASAR_ACT_GELU) return QUASAR_ERR_ARG;
  if (!a->codes || !a->scales) return QUASAR_ERR_ARG;
  if (d->format == QUASAR_INT && !a->zeros) return QUASAR_ERR_ARG;
  if ((d->format == QUASAR_NVFP4) != (a->tensor_scale != nullptr)) return QUASAR_ERR_ARG;
  if (misaligned(a->codes, 16) || misaligned(a->scales, 16) || misaligned(a->zeros, 16) ||
      misaligned(a->tensor_scale, 4) || misaligned(a->workspace, 16))
    return QUASAR_ERR_ALIGN;
  if (a->tokens == 0) return QUASAR_OK;
  size_t need;
  if (!quasar::linear_fits(*d, a->tokens, a->x_dtype, need)) return QUASAR_ERR_SHAPE;
  if (!a->x || !a->y) return QUASAR_ERR_ARG;
  QUASAR_TRY(check_matrix(a->x, a->tokens, d->cols, a->x_stride, a->x_dtype));
  QUASAR_TRY(check_matrix(a->residual, a->tokens, d->rows, a->residual_stride, a->residual_dtype));
  QUASAR_TRY(check_matrix(a->y, a->tokens, d->rows, a->y_stride, a->y_dtype));
  if (misaligned(a->x_scale, 4) || (a->bias && misaligned(a->bias, size_of(a->bias_dtype)))) return QUASAR_ERR_ALIGN;
  if (need > 0 && (a->workspace == nullptr || a->workspace_bytes < need)) return QUASAR_ERR_WORKSPACE;
  return QUASAR_OK;
}

int quasar_linear_codes(const quasar_desc* d, const quasar_linear* a, void* stream) {
  QUASAR_TRY(quasar_linear_codes_check(d, a));
  if (a->tokens == 0) return QUASAR_OK;
  return status_of(quasar::launch_linear(*d, *a, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
