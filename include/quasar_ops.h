/*
 * quasar_ops.h -- C ABI of the operators of libquasar.so that stand around the
 * reconstruction of quasar.h: the loss against a teacher's top logits that
 * trains the quantised model (the paper's distillation loss is the forward KL
 * divergence to the teacher, Sec. 6.1), the RMS norm with the residual's
 * addition (and an 8-bit output) between its layers, and the layers' product
 * from the packed codes that quasar_reconstruct emits.
 *
 * Conventions: those of quasar.h (device memory of the caller's, nothing
 * allocated or kept, asynchronous on `stream`, reentrant, argument errors
 * found on the host before anything is launched), except that
 *  - pointers need only the alignment of their element type (codes, scales
 *    and zeros of the product: 16 bytes, as quasar_reconstruct writes them;
 *    workspaces: 16 bytes), and matrices have a row stride of their own, in
 *    elements, at least their number of columns;
 *  - a call with no rows (rows or tokens = 0) does nothing and returns
 *    QUASAR_OK;
 *  - NaN and infinity go through the formulas as IEEE arithmetic takes them
 *    unless an argument masks them out.
 * Outputs may not overlap inputs or each other except where it says so.
 */
#ifndef QUASAR_OPS_H
#define QUASAR_OPS_H

#include "quasar.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One byte E4M3FN (4 exponent bits, 3 of the mantissa, largest 448, no
 * infinity): a dtype of 8-bit activations only. */
#define QUASAR_E4M3 3

/* ---- RMS norm with the residual's addition ---------------------------------
 *
 *   h = x + residual                       (fp32)
 *   rstd = 1 / sqrt(mean(h^2) + eps)       (one per row)
 *   y = h * rstd * weight
 *
 * and, as asked for: h in the residual's type (the stream's next value), y in
 * y_dtype, and y in 8 bits, q = E4M3(y / scale) with scale = max|y| / 448 per
 * row (at least 2^-120, so a row of zeros has q = 0).  y and q come from the
 * fp32 h, not from its rounding.  A row whose sum of squares is not finite has
 * scale = NaN and every q NaN.  Sums are in fp32.
 */
#define QUASAR_NORM_MAX_COLS 32768
typedef struct {
  int64_t rows, cols;        /* 0 <= rows < 2^31, 1 <= cols <= QUASAR_NORM_MAX_COLS */
  const void* x;             /* [rows, cols] */
  const void* residual;      /* [rows, cols], or NULL: h = x */
  const void* weight;        /* [cols] */
  void* h;                   /* [rows, cols] in residual_dtype, or NULL; may be `residual` itself, or x where the
                                types agree (with the same stride).  NULL without a residual */
  void* y;                   /* [rows, cols], or NULL */
  uint8_t* q;                /* [rows, cols] E4M3, or NULL */
  float* scale;              /* [rows]; required with q, NULL without */
  float* rstd;               /* [rows], or NULL */
  int64_t x_stride, residual_stride, h_stride, y_stride, q_stride;
  int32_t x_dtype, residual_dtype, weight_dtype, y_dtype;  /* QUASAR_F32 or QUASAR_BF16 each */
  float eps;                 /* finite, >= 0 */
} quasar_norm;

int quasar_add_rms_norm(const quasar_norm* a, void* stream);
int quasar_add_rms_norm_check(const quasar_norm* a);

/*
 * The gradients of the norm, with n = h * rstd and u = dy * weight:
 *   dx = rstd (u - n mean(u n)) + dh       (the gradient of x and of residual)
 *   dweight = sum over rows of dy n        (fp32)
 * q is taken straight through: its gradient is y's.  h and rstd are what the
 * forward pass gave (without a residual h is x).  The sum over rows has a
 * fixed order: the same inputs give the same bits.
 */
typedef struct {
  int64_t rows, cols;
  const void* dy;            /* [rows, cols] */
  const void* h;             /* [rows, cols] */
  const void* weight;        /* [cols] */
  const float* rstd;         /* [rows] */
  const void* dh;            /* [rows, cols] in dx_dtype, the stream's own gradient, or NULL */
  void* dx;                  /* [rows, cols]; may be dh itself with the same stride, or dy or h likewise where the
                                types agree */
  float* dweight;            /* [cols] (with no rows: not written), or NULL */
  void* workspace;           /* quasar_add_rms_norm_backward_workspace_bytes() */
  size_t workspace_bytes;
  int64_t dy_stride, h_stride, dh_stride, dx_stride;
  int32_t dy_dtype, h_dtype, weight_dtype, dx_dtype;
} quasar_norm_backward;

int quasar_add_rms_norm_backward(const quasar_norm_backward* a, void* stream);
int quasar_add_rms_norm_backward_check(const quasar_norm_backward* a);
size_t quasar_add_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols);

/* ---- distillation from a teacher's top logits --------------------------------
 *
 * Per row, with z the student's logits, t the teacher's at K listed classes
 * and tau the temperature:
 *   p_k  = exp(t_k / tau) / sum over listed j of exp(t_j / tau)
 *   lse  = log sum_v exp(z_v / tau)
 *   loss = row_weight sum_k p_k (log p_k - z_{index_k} / tau + lse)
 *   dz_v = G (row_weight / tau) (exp(z_v / tau - lse) - sum_{k: index_k = v} p_k)
 * (forward KL to the teacher restricted to its list and renormalised), G the
 * gradient of the row's loss.  An entry whose index is outside [0, classes) is
 * no entry (-1 fills a short list); one whose t is -inf has p = 0.  A class
 * may be listed more than once.  A row with row_weight 0, or without an entry
 * of p > 0, is masked: loss, lse and gradient are exactly 0 whatever its logits
 * hold.  Sums are in fp32, in a fixed order.
 */
#define QUASAR_DISTILL_MAX_LISTED 1024
typedef struct {
  int64_t rows, classes;     /* 0 <= rows, 1 <= classes < 2^31 - 2^16, rows * ceil(classes / 1024) < 2^31 */
  int32_t listed;            /* K, 1 .. QUASAR_DISTILL_MAX_LISTED */
  int32_t logits_dtype;      /* of logits and grad: QUASAR_F32 or QUASAR_BF16 */
  int32_t teacher_dtype;     /* QUASAR_F32 or QUASAR_BF16 */
  int32_t index_bits;        /* 32 or 64 */
  const void* logits;        /* [rows, classes] */
  const void* index;         /* [rows, listed], contiguous */
  const void* teacher;       /* [rows, listed], contiguous: logits or log-probabilities */
  const float* row_weight;   /* [rows], or NULL: 1 */
  const float* grad_loss;    /* quasar_distill_topk_backward: G per row [rows], or NULL: grad_scale in every row */
  float* loss;               /* [rows] */
  float* lse;                /* [rows]: an output, and what quasar_distill_topk_backward takes */
  void* grad;                /* [rows, classes]; may be `logits` itself with the same stride */
  void* workspace;           /* quasar_distill_topk_workspace_bytes(), not for the backward call */
  size_t workspace_bytes;
  int64_t logits_stride, grad_stride;
  float temperature;         /* finite, > 0, and its reciprocal too */
  float grad_scale;          /* finite: G of quasar_distill_topk_grad, and of the backward call without grad_loss */
} quasar_distill;

/* loss and lse (grad, grad_loss unused: NULL) */
int quasar_distill_topk(const quasar_distill* a, void* stream);
/* grad from lse (loss unused: NULL) */
int quasar_distill_topk_backward(const quasar_distill* a, void* stream);
/* loss, lse and grad with G = grad_scale (grad_loss NULL) */
int quasar_distill_topk_grad(const quasar_distill* a, void* stream);
/* The status that call would return: what = 0 for quasar_distill_topk, 1 for the backward, 2 for both at once. */
int quasar_distill_topk_check(const quasar_distill* a, int what);
size_t quasar_distill_topk_workspace_bytes(int64_t rows, int64_t classes);

/* ---- product from packed codes -------------------------------------------------
 *
 *   y[t, n] = act(x_scale[t] sum_k x[t, k] r[n, k] + bias[n]) + residual[t, n]
 *
 * r [rows = out, cols = in] is the reconstruction that codes, scales, zeros and
 * tensor_scale stand for, in bf16 -- bit for bit the r that quasar_reconstruct
 * gives for a bf16 W and that a layer is trained with -- formed in the kernel
 * from the codes.  desc gives its shape, format, bits and group; its clip and
 * dtype fields are validated but unused.  INT scales are below 2^100 in size (the
 * kernels multiply them by up to 2^24).  Products are accumulated in fp32.
 */
typedef enum {
  QUASAR_ACT_NONE = 0,
  QUASAR_ACT_RELU = 1,       /* max(v, 0) */
  QUASAR_ACT_SILU = 2,       /* v / (1 + exp(-v)) */
  QUASAR_ACT_GELU = 3        /* v (1 + erf(v / sqrt 2)) / 2 */
} quasar_activation;

typedef struct {
  int64_t tokens;            /* 0 <= tokens <= 2^28, with rows <= 2^28 and cols <= 2^22, as far as a grid takes the
                                workgroups: up to 16 tokens (8 bits: 32) rows <= 2^27 - 16; else past 2^37 outputs */
  const void* x;             /* [tokens, cols] */
  const float* x_scale;      /* [tokens], or NULL: 1 */
  const uint8_t* codes;      /* as quasar_reconstruct writes them */
  const void* scales;
  const float* zeros;        /* INT only, else NULL (INT_SYM: not read) */
  const float* tensor_scale; /* NVFP4 only, else NULL */
  const void* bias;          /* [rows], or NULL */
  const void* residual;      /* [tokens, rows], or NULL; may be y itself with the same type and stride */
  void* y;                   /* [tokens, rows] */
  void* workspace;           /* quasar_linear_codes_workspace_bytes() */
  size_t workspace_bytes;
  int64_t x_stride, residual_stride, y_stride;
  int32_t x_dtype;           /* QUASAR_BF16 or QUASAR_E4M3 */
  int32_t bias_dtype, residual_dtype, y_dtype;  /* QUASAR_F32 or QUASAR_BF16 */
  int32_t act;               /* quasar_activation */
} quasar_linear;

int quasar_linear_codes(const quasar_desc* desc, const quasar_linear* a, void* stream);
int quasar_linear_codes_check(const quasar_desc* desc, const quasar_linear* a);
/* Device scratch the call needs for this many tokens, of either x_dtype; 0 where it needs none, or for an invalid desc. */
size_t quasar_linear_codes_workspace_bytes(const quasar_desc* desc, int64_t tokens, int32_t x_dtype);

#ifdef __cplusplus
}
#endif

#endif /* QUASAR_OPS_H */
