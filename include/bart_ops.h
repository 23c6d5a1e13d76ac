/*
 * bart_ops.h -- C ABI of libbart, second part: what a program does with a
 * matrix of class scores (one row per observation, one column per class: the
 * forests of a classifier, or any other model's last layer) and how it trains
 * the weights that made it.
 *
 *  - bart_logprob: log probability of each row's given class, entropy of the
 *    row, its best alternatives, and (optionally, in the same call) the
 *    gradient of a weighted sum of the first two with respect to the scores.
 *  - bart_logprob_grad: that gradient alone, from what bart_logprob kept.
 *  - bart_adamw_*: one AdamW step over all tensors of a model at once, its
 *    moments held in 32 bits or in 8.
 *
 * Conventions are those of bart.h: 0 or a negative BART_E* code, arguments
 * checked before anything is enqueued, bart_last_error() for the message, no
 * device memory allocated by the library.  Calls enqueue on the given stream
 * (a hipStream_t, NULL = default stream) and do not synchronise it, except
 * bart_adamw_init.  They can be captured into a graph, except that
 * bart_adamw_init cannot and that a captured bart_adamw_step repeats one step
 * (see there).
 */
#ifndef BART_OPS_H
#define BART_OPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types */
#define BART_F32 0
#define BART_F16 1
#define BART_BF16 2

#define BART_MAX_TOP 64 /* most alternatives per row */

/* Rows of scores.  Class j of row i is allowed iff mask is NULL or
 * mask[i * ld_mask + j] != 0; the score at a place that is not allowed is
 * never used, whatever it holds. */
typedef struct {
  const void *x;        /* device [n][ld] of dtype */
  int64_t n;            /* rows, >= 0 */
  int64_t ld;           /* elements between rows; 0: one row for all */
  int32_t n_class;      /* in [1, 2^30] */
  int32_t dtype;        /* BART_F32, BART_F16 or BART_BF16 */
  const int64_t *label; /* device, the given class of row i at label[i * label_stride];
                           negative: none.  NULL: no row has one */
  int64_t label_stride; /* >= 0 */
  const uint8_t *mask;  /* device u8, or NULL */
  int64_t ld_mask;      /* bytes between rows of mask; 0: one row for all */
  double temperature;   /* T in [1e-30, 1e30]: scores are divided by it */
} bart_rows;

/* Weights of a gradient: of sum_i (w_logp[i] logp_i + w_entropy[i] H_i).  A
 * stride of 0 gives all rows the same weight; a NULL pointer, weight 0. */
typedef struct {
  const float *w_logp;    /* device, w_logp[i * w_logp_stride] */
  int64_t w_logp_stride;  /* >= 0 */
  const float *w_entropy; /* device, w_entropy[i * w_entropy_stride] */
  int64_t w_entropy_stride;
  void *grad;             /* device [n][ld_grad] of the scores' dtype; may be the scores
                             themselves (same ld, not 0) or lie between their rows (same
                             ld), else apart from them */
  int64_t ld_grad;        /* >= n_class */
} bart_rows_grad;

/* What bart_logprob writes; a NULL pointer: not wanted. */
typedef struct {
  float *logp;        /* device f32 [n] */
  float *entropy;     /* device f32 [n] */
  float *norm;        /* device f32 [n][2]: m_i and log s_i, for bart_logprob_grad */
  int32_t k;          /* alternatives per row, in [0, BART_MAX_TOP] */
  float *top_logp;    /* device f32 [n][k] */
  int32_t *top_class; /* device i32 [n][k] */
} bart_rows_out;

/* With x_j the allowed scores of a row, m = max x_j, z_j = (x_j - m) / T,
 * s = sum exp z_j:
 *   log p_j = z_j - log s;  logp = log p_label;  H = log s - (sum z_j exp z_j) / s;
 *   norm = (m, log s);
 *   alternatives: the k largest x_j, the lowest j first among equal ones;
 *   d/dx_j of w logp + h H = (w ([j = label] - p_j) - h p_j (log p_j + H)) / T.
 * (m and log s are kept apart: where the scores are large their sum would
 * lose log s.)  Sums are held in 32 bits whatever the scores' type; the
 * gradient is rounded to it once, to nearest.
 *
 * Rows that need a rule:
 *  - nothing allowed, or every allowed score -inf: log s, m and logp -inf, H 0,
 *    gradient 0;
 *  - a NaN or +inf among the allowed scores: log s, logp and H NaN, every
 *    alternative (NaN, -1), the gradient NaN at allowed places above -inf;
 *  - the gradient is 0 at every place that is not allowed, and where x_j = -inf;
 *  - label < 0: logp 0, and w counts as 0; where w and h are 0 the whole row's
 *    gradient is 0 (also where the row is NaN);
 *  - label not allowed or its score -inf: logp -inf;
 *  - label >= n_class: logp NaN, and where w is not 0 the gradient NaN at
 *    allowed places above -inf;
 *  - a weight that is not finite (or overflows over T): the gradient NaN at
 *    allowed places above -inf;
 *  - fewer than k allowed scores above -inf: the rest of the alternatives are
 *    (-inf, -1).
 * The same call gives the same bits each time; a row's last bits may differ
 * with the number of rows and with what else is asked for.
 *
 * g may be NULL (no gradient).  workspace: device, at least
 * bart_logprob_workspace_bytes (0 for most calls: only few long rows, which
 * are split over several workgroups, need one), 16-byte aligned, its contents
 * before the call are not used; calls that may overlap need their own. */
int bart_logprob(const bart_rows *rows, const bart_rows_out *out, const bart_rows_grad *g,
                 void *workspace, size_t ws_bytes, void *stream);

/* Bytes of workspace for such a call (0 also for invalid arguments). */
size_t bart_logprob_workspace_bytes(const bart_rows *rows, const bart_rows_out *out,
                                    const bart_rows_grad *g);

/* The same gradient from norm [n][2] and entropy [n] of an earlier
 * bart_logprob on the same rows (entropy may be NULL without w_entropy). */
int bart_logprob_grad(const bart_rows *rows, const float *norm, const float *entropy,
                      const bart_rows_grad *g, void *stream);

/* One tensor of an AdamW step; all arrays are dense.  State of 32 bits: m and
 * v are f32 [n], the scales NULL.  State of 8 bits: m holds e4m3 codes (1
 * sign, 4 exponent, 3 mantissa bits, no infinities) of the first moment, v
 * those of the ROOT of the second, u8 [n]; blocks of 256 consecutive elements
 * share a scale, f32 [ceil(n / 256)]: value = code x scale. */
typedef struct {
  void *param;          /* [n] of param_dtype, read (unless master) and written */
  const void *grad;     /* [n] of grad_dtype */
  float *master;        /* NULL, or f32 [n]: the weights, of which param is a rounded copy */
  void *m, *v;
  float *m_scale, *v_scale;
  int64_t n;            /* >= 0 */
  int32_t param_dtype;  /* BART_F32, BART_F16 or BART_BF16; a master only beside 16 bits */
  int32_t grad_dtype;   /* param_dtype or BART_F32 */
  float weight_decay;   /* finite */
  float lr_scale;       /* finite: this tensor's learning rate is lr x lr_scale */
} bart_adamw_tensor;

typedef struct {
  double lr, beta1, beta2; /* lr finite as f32; betas in [0, 1) */
  double eps;              /* >= 1e-37 */
  double grad_scale;       /* finite as f32: gradients are multiplied by it first */
  int64_t step;            /* t >= 1, the number of this step */
} bart_adamw_hyper;

typedef struct bart_adamw bart_adamw;

/* Bytes of device workspace for these tensors (0: invalid arguments). */
size_t bart_adamw_workspace_bytes(const bart_adamw_tensor *t, int32_t n_tensors,
                                  int32_t state_bits);

/* A plan over n_tensors >= 1 tensors (host array, copied; the device arrays
 * it names are borrowed and must outlive the plan, as must the workspace,
 * 16-byte aligned).  state_bits: 32 or 8.  No array that is written may overlap
 * one of another tensor (BART_EINVAL).  Synchronises the stream.  Steps run on the device that is
 * current now, whichever is current then; they leave it current. */
int bart_adamw_init(const bart_adamw_tensor *t, int32_t n_tensors, int32_t state_bits,
                    void *workspace, size_t ws_bytes, void *stream, bart_adamw **out);

/* Step t, for every element:
 *   g <- grad_scale g;  m <- beta1 m + (1 - beta1) g;  v <- beta2 v + (1 - beta2) g^2;
 *   p <- p (1 - lr wd) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps).
 * All of it is computed in 32 bits.  A param of 16 bits is rounded to nearest
 * once, at the end.  An 8-bit state is rounded after it has been used: a
 * block's scale is its largest magnitude / 448; m goes to the nearest code; the
 * root of v to the code below or above by a threshold that runs through an
 * equidistributed sequence over the elements and the steps (a step changes v
 * by a share of about 1 - beta2, less than half a rounding step, so
 * rounding to nearest would hold it for good), and never to 0 where v > 0.  A
 * block without a magnitude of 2^-100 or more is held as zeros.
 * Such a root follows a slow decay to within a few rounding steps, on the
 * whole up to 1/16 faster in its logarithm (independent random thresholds
 * would leave no such tendency, and about five times the scatter).
 * A gradient that is NaN or infinite makes its element's state NaN; with
 * 8-bit states, possibly its whole block's.
 * What hyper holds is taken at the call.  A graph that captured it repeats step
 * t at every replay: the bias corrections stand still, and with 8-bit states
 * each element meets the same threshold again, so that a root may never move
 * (what the sequence is there to avoid).  Training needs a call per step; the
 * plan, its arrays and the workspace must outlive such a graph. */
int bart_adamw_step(bart_adamw *h, const bart_adamw_hyper *hyper, void *stream);

void bart_adamw_destroy(bart_adamw *h);

#ifdef __cplusplus
}
#endif
#endif /* BART_OPS_H */
