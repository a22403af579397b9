/* falqon_train.h -- what a fine-tuning step runs between and behind the melded layers (falqon.h): the norms around a
 * block with its gate and residual scale, 8-bit checkpoints of activations and the gated MLP that keeps them, and the
 * preference loss of paired sequences with its gradient.
 *
 * Conventions are those of falqon.h: dense row-major device tensors owned by the caller, 16-byte aligned (fp32 vectors
 * of one entry per row, pair or sequence: 4-byte), asynchronous on `stream`, no allocation, no synchronisation, an int
 * status per call.  Arithmetic is fp32 (or wider) whatever the tensors' type; results are rounded to nearest even once.
 * Every call gives the same bits for the same inputs: no sum depends on the order in which thread blocks finish.
 * amax_out arguments (device [1] fp32, nullable) are those of falqon_chain.h: raised to the largest |value| stored, so
 * that a melded layer can take the tensor without an absmax pass of its own. */
#ifndef FALQON_TRAIN_H
#define FALQON_TRAIN_H

#include "falqon.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- 8-bit activation checkpoints
 * A [rows][cols] tensor is held as E4M3 codes [rows][cols] and one scale byte for every 32 consecutive values of a row,
 * [rows][ceil(cols / 32)] (a row's last block may be short).  A scale byte e stands for 2^(e - 127); it is the smallest
 * e >= 0 for which the block's largest |value| * 2^(127 - e) is at most 448, so scaling is exact, nothing saturates, and
 * a value is rounded once (to nearest even).  A block that holds an infinity or a NaN gets e = 255 and NaN codes: it
 * reads back as NaN.  1.03 bytes per value. */
#define FALQON_CHECKPOINT_BLOCK 32

int falqon_checkpoint_save(const void *x, int dtype, int64_t rows, int64_t cols, uint8_t *codes, uint8_t *scales,
                           falqon_stream stream);
int falqon_checkpoint_load(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *x, int dtype,
                           falqon_stream stream);

/* z = silu(g) * u, silu(x) = x / (1 + exp(-x)), and (all four or none) the checkpoints of g and u in the same pass.
 * z is neither g nor u. */
int falqon_gate_forward(const void *g, const void *u, int dtype, int64_t rows, int64_t cols, void *z, uint8_t *g_codes,
                        uint8_t *g_scales, uint8_t *u_codes, uint8_t *u_scales, float *amax_out, falqon_stream stream);
/* Its gradient from the checkpoints: with s = 1 / (1 + exp(-g)):  du = dz * g * s,  dg = dz * u * s * (1 + g * (1 - s)).
 * dg or du may alias dz. */
int falqon_gate_backward(const uint8_t *g_codes, const uint8_t *g_scales, const uint8_t *u_codes, const uint8_t *u_scales,
                         const void *dz, int dtype, int64_t rows, int64_t cols, void *dg, void *du, float *amax_dg,
                         float *amax_du, falqon_stream stream);

/* ---- the norms after and before a block, with the block's gate and the residual scale
 *   n     = y * inv_post[t] * (gain_offset + post_gain)      inv_post[t] = 1 / sqrt(mean(y[t]^2) + eps)     (FALQON_NORM_POST; else n = y)
 *   h_out = res_scale * h + gate * n                         y: what the block gave, h: the residual stream before it
 *   x     = h_out * inv_pre[t] * (gain_offset + pre_gain)    inv_pre[t] = 1 / sqrt(mean(h_out[t]^2) + eps)  (FALQON_NORM_PRE: the next block's input)
 * x and inv_pre come from h_out before its rounding.  A NULL gain or gate is 1 (without gain_offset); a NULL h leaves the
 * residual term out.  rows <= FALQON_NORM_MAX_ROWS, cols <= FALQON_NORM_MAX_COLS. */
#define FALQON_NORM_POST 1
#define FALQON_NORM_PRE 2
#define FALQON_NORM_MAX_COLS 16384
#define FALQON_NORM_MAX_ROWS 2147482624 /* 2^31 - 1024: the kernels count rows in 32 bits and look up to 64 rows ahead */

typedef struct { /* host struct */
  int64_t rows, cols;
  int64_t rows_per_gate;  /* row t uses row t / rows_per_gate of gate [ceil(rows / rows_per_gate)][cols]; >= 1          */
  int32_t dtype;          /* falqon_dtype of h, y, h_out, x and their gradients                                        */
  int32_t gain_dtype;     /* falqon_dtype of post_gain, pre_gain and gate; their gradients are fp32                    */
  int32_t flags;          /* FALQON_NORM_POST | FALQON_NORM_PRE                                                        */
  float res_scale, gain_offset, eps;
  const void *post_gain;  /* device [cols], nullable                                                                   */
  const void *pre_gain;   /* device [cols], nullable                                                                   */
  const void *gate;       /* device, nullable                                                                          */
} falqon_block_norm;

/* h_out may be NULL with FALQON_NORM_PRE (only x is wanted) and may alias h or y; x is not h_out; x, inv_pre / inv_post are
 * needed with their flag and ignored without it.  h_codes, h_scales / y_codes, y_scales (nullable, in pairs): checkpoints of h / y. */
int falqon_block_norm_forward(const falqon_block_norm *p, const void *h, const void *y, void *h_out, void *x, float *inv_post,
                              float *inv_pre, uint8_t *h_codes, uint8_t *h_scales, uint8_t *y_codes, uint8_t *y_scales,
                              float *amax_x, falqon_stream stream);

/* The gradient, with h_out recomputed from the saved inputs: h and y as they were, or (h and y NULL) their checkpoints.
 * dx (NULL without FALQON_NORM_PRE) and dh_out (nullable: 0) are the gradients of x and h_out.  dh (nullable; must be NULL when
 * the forward had no h) and dy (nullable) may alias dx or dh_out.  dpost_gain, dpre_gain [cols], dgate [gates][cols], fp32,
 * nullable: gradients of a frozen gain or gate are not computed.  scratch (needed with any of the three):
 * falqon_block_norm_scratch_bytes(p) bytes, no initialisation. */
size_t falqon_block_norm_scratch_bytes(const falqon_block_norm *p);
int falqon_block_norm_backward(const falqon_block_norm *p, const void *dx, const void *dh_out, const void *h,
                               const uint8_t *h_codes, const uint8_t *h_scales, const void *y, const uint8_t *y_codes,
                               const uint8_t *y_scales, const float *inv_post, const float *inv_pre, void *dh, void *dy,
                               float *dpost_gain, float *dpre_gain, float *dgate, float *amax_dy, void *scratch,
                               size_t scratch_bytes, falqon_stream stream);

/* ---- the preference loss of paired sequences
 * logits [rows][vocab] with a row pitch of ld >= vocab values (aligned to their type only); targets [rows] int64: the token that row predicts, negative: the
 * row is not counted (a prompt's rows, padding) and its logits are not read.  A target >= vocab is not counted either and is
 * reported by falqon_last_device_status as FALQON_ERR_INVALID_ARG.  Sequences are packed: sequence i owns rows cu_rows[i] ..
 * cu_rows[i + 1] (int64 device array, ascending from 0 to rows; rows outside are not counted).
 *   logp[row]   = logits[row][target] - log sum exp(logits[row])      (0 where the row is not counted)
 *   seq_logp[i] = the sum of its rows' logp, or their mean over the counted rows (FALQON_PREFERENCE_AVERAGE; 0 if there are none) */
#define FALQON_PREFERENCE_AVERAGE 1

typedef enum { FALQON_PREFERENCE_SIGMOID = 0, FALQON_PREFERENCE_HINGE = 1, FALQON_PREFERENCE_IPO = 2 } falqon_preference_kind;

/* Pair p is sequences 2p (chosen) and 2p + 1 (rejected):
 *   u = (seq_logp[2p] - ref_logp[2p]) - (seq_logp[2p + 1] - ref_logp[2p + 1]);  D = beta * u - margin
 *   SIGMOID: l = -(1 - label_smoothing) * log sigmoid(D) - label_smoothing * log sigmoid(-D)
 *   HINGE:   l = max(0, 1 - D)            IPO: l = (u - margin - 1 / (2 beta))^2       (label_smoothing must be 0 for both)
 *   pair_loss[p] = l - nll_weight * (mean of the chosen sequence's counted logp);   loss = mean of pair_loss */
typedef struct { /* host struct */
  int64_t rows, vocab, ld, pairs;
  int32_t dtype;          /* falqon_dtype of the logits and their gradient */
  int32_t kind;           /* falqon_preference_kind */
  int32_t flags;          /* FALQON_PREFERENCE_AVERAGE */
  float beta, margin, label_smoothing, nll_weight;
} falqon_preference;

/* Device bytes of scratch for the two forward calls (no initialisation needed); 0: bad sizes. */
size_t falqon_preference_scratch_bytes(int64_t rows, int64_t vocab, int dtype);

/* The log-probabilities alone (a reference model's pass): logp [rows] (nullable) and seq_logp [n_seq]. */
int falqon_sequence_logprob(const void *logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const int64_t *targets,
                            const int64_t *cu_rows, int64_t n_seq, int average, float *logp, float *seq_logp, void *scratch,
                            size_t scratch_bytes, falqon_stream stream);

/* ref_logp [2 * pairs] (nullable: 0).  Results: loss [1], pair_loss [pairs], seq_logp [2 * pairs], logp [rows]; and for the
 * gradient (both or neither) row_stats [rows][2], 8-byte aligned: the row's maximum and its sum of exp(logit - maximum) (of no
 * meaning where the row is not counted), and dlogp [rows]: d loss / d logp of the row, 0 where it is not counted. */
int falqon_preference_forward(const falqon_preference *p, const void *logits, const int64_t *targets, const int64_t *cu_rows,
                              const float *ref_logp, float *loss, float *pair_loss, float *seq_logp, float *logp,
                              float *row_stats, float *dlogp, void *scratch, size_t scratch_bytes, falqon_stream stream);

/* dlogits[row][v] = dloss * dlogp[row] * ([v == target] - softmax(logits[row])[v]), row pitch ld_out; a row whose dlogp is 0
 * gets zeros and is not read, whatever dloss is.  dloss: device [1], nullable (1).  dlogits may be logits (ld_out == ld). */
int falqon_preference_backward(const falqon_preference *p, const void *logits, const int64_t *targets, const float *row_stats,
                               const float *dlogp, const float *dloss, void *dlogits, int64_t ld_out, float *amax_out,
                               falqon_stream stream);

#ifdef __cplusplus
}
#endif
#endif
