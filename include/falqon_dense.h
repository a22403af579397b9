/* falqon_dense.h -- a linear layer held, multiplied and updated in 8 bits by blocks: codes with a scale for each block of
 * 128 values, the three products of training on them and the form for few tokens, and the orthogonalised update that the
 * Muon optimizer takes.
 *
 * Conventions are those of falqon.h: row-major device tensors owned by the caller, 16-byte aligned unless said otherwise,
 * asynchronous on `stream`, no allocation, no synchronisation, an int status per call.  Every call gives the same bits for
 * the same inputs on the same device: no sum depends on the order in which thread blocks finish.  The same row in a tensor of
 * another shape may be added up in another order (short contractions by one tile, long ones by several). */
#ifndef FALQON_DENSE_H
#define FALQON_DENSE_H

#include "falqon.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- 8-bit codes by blocks
 * A [rows][cols] tensor is held as codes [rows][cols] (E4M3 or E5M2) and one scale byte per block.  A byte e stands for
 * 2^(e - 127) and is the smallest e >= 0 for which the block's largest |value| * 2^(127 - e) is at most the type's largest
 * value (448 / 57344): scaling is exact, nothing saturates, a value is rounded once (to nearest even).  A block that holds an
 * infinity or a NaN gets e = 255 and NaN codes: it reads back as NaN.  Blocks at an edge may be short.
 *   FALQON_ALONG_ROW   128 values of a row,    scales [rows][ceil(cols / 128)]: what is contracted along its columns
 *   FALQON_ALONG_COL   128 values of a column, scales [ceil(rows / 128)][cols]: what is contracted along its rows
 *   FALQON_TILE        128 x 128 values,       scales [ceil(rows / 128)][ceil(cols / 128)]: weights, contracted either way
 * Scales need no alignment. */
#define FALQON_BLOCK 128

typedef enum { FALQON_ALONG_ROW = 0, FALQON_ALONG_COL = 1, FALQON_TILE = 2 } falqon_blocking;

/* x has a row pitch of ld >= cols values and is aligned to its type only (16-byte aligned rows are faster).  Codes are dense
 * and need no alignment (8 bytes are faster).  rows, cols <= 2^30, rows * cols <= 2^42, rows * ld <= 2^44. */
int falqon_block_quantize(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, falqon_fp8 fmt, falqon_blocking along,
                          uint8_t *codes, uint8_t *scales, falqon_stream stream);
/* FALQON_ALONG_ROW and FALQON_ALONG_COL of the same tensor in one read: what a training step needs of a layer's input (forward,
 * weight gradient) and of its output's gradient (input gradient, weight gradient). */
int falqon_block_quantize_both(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, falqon_fp8 fmt, uint8_t *row_codes,
                               uint8_t *row_scales, uint8_t *col_codes, uint8_t *col_scales, falqon_stream stream);
/* The values that codes stand for, rounded once: y [rows][cols], dense, aligned to its type only. */
int falqon_block_dequantize(const uint8_t *codes, const uint8_t *scales, falqon_fp8 fmt, falqon_blocking along, int64_t rows, int64_t cols,
                            void *y, int dtype, falqon_stream stream);

/* ---- the products of a linear layer y = x w^T with w [m][n] held as FALQON_TILE E4M3 or E5M2 codes
 * n and m are multiples of 16, T >= 1; codes and results 16-byte aligned and dense.  Sums over the contraction are fp32 as the tensor
 * cores add: cut off instead of rounded, 2e-6 of the result's norm after 4096 terms (bf16's rounding is 1.7e-3).  fp32 results are summed
 * so in parts of at most 2048 terms, which are added up by rounding additions: 1e-6, however long the contraction (a plain fp32 product:
 * 8e-7 after 4096 terms, 1.6e-6 after 16384).  Results are rounded once to their type.  A NaN block makes NaN of what it takes part in. */
/* y [T][m] = x w^T; x [T][n] as FALQON_ALONG_ROW codes */
int falqon_block_forward(const uint8_t *x_codes, const uint8_t *x_scales, falqon_fp8 x_fmt, const uint8_t *w_codes, const uint8_t *w_scales,
                         falqon_fp8 w_fmt, int64_t T, int64_t n, int64_t m, void *y, int y_dtype, falqon_stream stream);
/* dx [T][n] = dy w; dy [T][m] as FALQON_ALONG_ROW codes */
int falqon_block_input_grad(const uint8_t *dy_codes, const uint8_t *dy_scales, falqon_fp8 dy_fmt, const uint8_t *w_codes,
                            const uint8_t *w_scales, falqon_fp8 w_fmt, int64_t T, int64_t n, int64_t m, void *dx, int dx_dtype,
                            falqon_stream stream);
/* dw [m][n] = dy^T x; dy [T][m] and x [T][n] as FALQON_ALONG_COL codes */
int falqon_block_weight_grad(const uint8_t *dy_codes, const uint8_t *dy_scales, falqon_fp8 dy_fmt, const uint8_t *x_codes,
                             const uint8_t *x_scales, falqon_fp8 x_fmt, int64_t T, int64_t n, int64_t m, void *dw, int dw_dtype,
                             falqon_stream stream);
/* y [T][m] = q(x) w^T with x [T][n] bf16 or fp32, dense, quantized to E4M3 by FALQON_ALONG_ROW on the way.  scratch (nullable where
 * falqon_block_linear_scratch_bytes is 0; no initialisation): that many bytes. */
size_t falqon_block_linear_scratch_bytes(int64_t T, int64_t n, int64_t m);
int falqon_block_linear(const void *x, int x_dtype, const uint8_t *w_codes, const uint8_t *w_scales, falqon_fp8 w_fmt, int64_t T, int64_t n,
                        int64_t m, void *y, int y_dtype, void *scratch, size_t scratch_bytes, falqon_stream stream);

/* ---- an update orthogonalised by Newton-Schulz products (the Muon optimizer's)
 *   X = g / (|g|_F + eps);   steps times:  G = X X^T,  X <- a X + (b G + c G G) X;   out = scale * X
 * for each of `batch` matrices [rows][cols]; tall ones are taken from their short side, which gives the same.  The singular
 * values s of X become p(s) = a s + b s^3 + c s^5 at each step.
 * Arithmetic: sums are fp32 (the norm's fp64).  X and the term a X are held in 22 bits (two fp16 numbers, a power of two apart; no
 * finer than 2^-37 of X's norm, of which single values may be a small part), the products' operands in fp16 (11 bits) where the results
 * are bf16 (of B X with a short side up to 96: 22 bits); where they are fp32, each product is three: both operands in 22 bits.  Where |g| is far below eps, so that X is small
 * altogether, its digits are kept by powers of two, a matrix's own.  A step whose polynomial cancels, a + q being small beside
 * q = b s^2 + c s^4, leaves up to 2^-11 |q| / |a + q| of that direction in bf16 results (0.2 % with Muon's coefficients, 2 % with the steepest
 * of published schedules, whose last steps take it away again).  A matrix of zeros gives zeros; an infinity or a NaN makes NaN of its whole matrix. */
#define FALQON_ORTHO_MAX_STEPS 32

typedef struct { /* host struct */
  int64_t batch, rows, cols;     /* >= 1; rows, cols <= 32768, batch <= 65535, batch * rows * cols <= 2^36                     */
  int32_t dtype;                 /* falqon_dtype of g                                                                          */
  int32_t out_dtype;             /* falqon_dtype of out                                                                        */
  int32_t steps;                 /* 1 .. FALQON_ORTHO_MAX_STEPS                                                                */
  float eps, scale;              /* eps >= 0 and finite                                                                        */
  const float *coefficients;     /* host, [steps][3]: a, b, c of each step; NULL: 3.4445, -4.7750, 2.0315 at each.  Refused where
                                    p or s^2 could pass 7.9 in size, or b s^2 + c s^4 7.98, for some 0 <= s <= the bound before the
                                    step (0.1 % more than the step before can give).  The published schedules for singular values
                                    down to 1e-3, which begin with 8.2, -22.9, 16.5, are taken with their safety factor */
} falqon_ortho;

/* Device bytes of scratch, 0: bad sizes.  No initialisation. */
size_t falqon_orthogonalize_scratch_bytes(const falqon_ortho *p);
/* g and out: dense [batch][rows][cols], aligned to their type only; out may be g where the types are the same. */
int falqon_orthogonalize(const falqon_ortho *p, const void *g, void *out, void *scratch, size_t scratch_bytes, falqon_stream stream);

#ifdef __cplusplus
}
#endif
#endif
