/*
 * oz2_lm.h -- operators of liboz2 at the ends of a language model's step, and
 * between its layers, for one NVIDIA GB300 (sm_103a): the lookup of tokens' rows
 * in a table, layer norm, and the losses over a vocabulary that are taken from the
 * last layer's input without keeping the logits; each with its gradient.
 *
 * Conventions are those of oz2_layers.h: tokens are columns (a framework's
 * row-major (tokens, features) array), types and their checks, leading dimensions in
 * elements, base addresses on multiples of the element size, work enqueued on
 * `stream`, workspace allocated and freed stream-ordered, calls on several streams
 * and captured into CUDA graphs, OZ2_OK or a negative oz2_status with nothing
 * enqueued.  An output overlaps no other argument unless it says so.  Sizes of
 * 2^31 - 256 or more are OZ2_ERR_UNSUPPORTED.  Every sum has one order: a call repeated
 * gives the same bits.
 *
 * Tokens name rows of a table or vocabulary by integers of id_bits 64 or 32.
 */
#ifndef OZ2_LM_H
#define OZ2_LM_H

#include "oz2_layers.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Y_t = scale·E[id_t], rounded once: k features of m tokens from a table of n rows
 * (E k×n, lde ≥ k; Y k×m, ldy ≥ k), both of `type` F32, BF16 or F16.  id < 0 (padding):
 * zeros.  id ≥ n: NaN.  m = 0 or k = 0: nothing. */
int oz2_embedding(int64_t m, int64_t n, int64_t k, int type, const void* d_ids, int id_bits,
                  const void* d_E, int64_t lde, float scale, void* d_Y, int64_t ldy, void* stream);

/* Its gradient: dE_j = scale·Σ dY_t over the tokens with id_t = j, summed in FP32 and
 * rounded once; tokens whose id is not in [0, n) count for nothing.
 *   de_type   of dE (k×n, ldde ≥ k): `type` or F32
 *   flags     OZ2_GRAD_ACCUMULATE: the sums are added to dE, whose other rows are left
 *             as they are; else rows without tokens become zeros
 * A row's tokens are summed in ascending order, in stretches that depend on the sorted
 * tokens alone.  (16-bit rows are added to in FP32 and rounded once; sums for F32 ones are rounded and
 * then added in memory, where a result below 2^-126 counts as 0.) */
int oz2_embedding_grad(int64_t m, int64_t n, int64_t k, int type, const void* d_dY, int64_t lddy,
                       const void* d_ids, int id_bits, float scale, void* d_dE, int64_t ldde, int de_type,
                       unsigned flags, void* stream);

/* y = (x - μ)·r·w + b over the k features of each of m tokens, r = 1/√(σ² + eps):
 *   center    μ is the mean and σ² the variance (over k, not k - 1); 0: μ = 0 and σ²
 *             the mean of squares
 *   d_X, d_Y  k×m of `type` F32, BF16 or F16 (ldx, ldy ≥ k); d_Y may be d_X itself (with
 *             its ldx)
 *   d_w, d_b  k values of wtype (`type` or F32), or null: 1 and 0
 *   d_mean, d_rstd  m floats that receive μ and r, or null
 * In FP32, the variance from the deviations.  m = 0: nothing.  k = 0: r and, where centred, μ
 * are NaN, as the mean of nothing is.  eps ≥ 0. */
int oz2_layer_norm(int64_t m, int64_t k, int type, const void* d_X, int64_t ldx, const void* d_w, const void* d_b,
                   int wtype, float eps, int center, void* d_Y, int64_t ldy, float* d_mean, float* d_rstd,
                   void* stream);

/* Its gradient from dY, X and the μ and r that it kept (d_mean null: not centred).
 * With x̂ = (x - μ)·r and g = dy·w:
 *   dx = r·(g - mean g - x̂·mean(g·x̂)) + R   (without mean g where not centred)
 *   dw = Σ_t dy·x̂      db = Σ_t dy
 *   d_R       k×m of `type` (ldr ≥ k), a skip connection's gradient, or null; may be d_dX
 *             itself (with its lddx)
 *   d_dX      k×m of `type` (lddx ≥ k), or null: not wanted
 *   d_dw, d_db  k floats, or null: not wanted
 *   flags     OZ2_GRAD_ACCUMULATE: dw and db are added to
 * m = 0: dw = db = 0 (unchanged when accumulating). */
int oz2_layer_norm_grad(int64_t m, int64_t k, int type, const void* d_dY, int64_t lddy, const void* d_X, int64_t ldx,
                        const float* d_mean, const float* d_rstd, const void* d_w, int wtype, const void* d_R,
                        int64_t ldr, void* d_dX, int64_t lddx, float* d_dw, float* d_db, unsigned flags, void* stream);

/* Cross entropy of m tokens over n rows of W (k×n) from X (k×m), both BF16 or F16:
 *   z = scale·Wᵀ·x      lse = log Σ_j exp z_j      loss = lse - z_target + z_loss·lse²
 *   d_loss, d_lse, d_picked   m floats each: the loss, lse, and the target's logit
 * target < 0: the token does not count, loss and picked are 0, whatever its x is; target ≥ n:
 * loss and picked are NaN.  The logits live on chip, 256 × 256 at a time, as powers of two
 * (scale·log2 e is finite, and a logit beyond 2^127.47, 2.3e38, counts as infinite in lse); the
 * workspace is 8 bytes for 64 of them.  m = 0: nothing.  n < 1: OZ2_ERR_INVALID_ARG.
 * Operands are copied to rows that TMA can read as by oz2_linear. */
int oz2_linear_xent(int64_t m, int64_t n, int64_t k, int type, const void* d_X, int64_t ldx, const void* d_W,
                    int64_t ldw, const void* d_targets, int id_bits, float scale, float z_loss, float* d_loss,
                    float* d_lse, float* d_picked, void* stream);

/* Its gradient from ∂L/∂loss and the lse that it kept:
 *   dz_j = dloss·scale·((1 + 2·z_loss·lse)·exp(z_j - lse) - [j = target])
 *   dX = W·dz      dW = X·dzᵀ
 *   d_dloss   m floats, or with OZ2_GRAD_ONE_DLOSS one that goes for all tokens
 *   d_dX      k×m of `type` (lddx ≥ k), or null: not wanted
 *   d_dW      k×n of dw_type (`type` or F32; lddw ≥ k), or null: not wanted
 *   flags     OZ2_GRAD_ACCUMULATE: dW (F32 only) is added to
 * The logits are formed again, and dz is rounded to `type`, for dW in F32 too (F16: under a power
 * of two that brings the largest dloss into its range, taken out of the sums), in pieces of the
 * vocabulary of at most some 512 MB.  Tokens that do not count have zeros in dX (with W finite: they
 * are 0·W) and no part in dW, whatever their x, lse and dloss are; a target ≥ n makes its dX and all
 * of dW NaN. */
#define OZ2_GRAD_ONE_DLOSS 0x2u
int oz2_linear_xent_grad(int64_t m, int64_t n, int64_t k, int type, const float* d_dloss, const void* d_X, int64_t ldx,
                         const void* d_W, int64_t ldw, const void* d_targets, int id_bits, const float* d_lse,
                         float scale, float z_loss, void* d_dX, int64_t lddx, void* d_dW, int64_t lddw, int dw_type,
                         unsigned flags, void* stream);

/* Distillation: the cross entropy against a teacher's `top` listed rows of each token, less the
 * teacher's own entropy.  With z = Wᵀ·x / T and q the softmax of teacher / T over the rows that
 * are listed (id ≥ 0; the same row twice counts twice):
 *   loss = Σ_i q_i·(log q_i - z_id(i)) + lse
 *   d_ids     `top` rows of each token (top×m, ldi ≥ top), in any order; below 0: none there
 *   d_teacher the teacher's logits of them (top×m, ldt ≥ top) of teacher_type F32, BF16 or F16
 *   d_loss, d_lse   m floats;  d_picked   top×m floats (ld top): the listed rows' z, 0 where none is
 * A token without rows does not count: its loss is 0.  id ≥ n: NaN.  1 ≤ top ≤ 1024;
 * temperature > 0. */
int oz2_linear_distill(int64_t m, int64_t n, int64_t k, int64_t top, int type, const void* d_X, int64_t ldx,
                       const void* d_W, int64_t ldw, const void* d_ids, int64_t ldi, int id_bits,
                       const void* d_teacher, int64_t ldt, int teacher_type, float temperature, float* d_loss,
                       float* d_lse, float* d_picked, void* stream);

/* Its gradient, as oz2_linear_xent_grad:
 *   dz_j = dloss/T·(exp(z_j - lse) - Σ q_i over the entries with id_i = j) */
int oz2_linear_distill_grad(int64_t m, int64_t n, int64_t k, int64_t top, int type, const float* d_dloss,
                            const void* d_X, int64_t ldx, const void* d_W, int64_t ldw, const void* d_ids, int64_t ldi,
                            int id_bits, const void* d_teacher, int64_t ldt, int teacher_type, float temperature,
                            const float* d_lse, void* d_dX, int64_t lddx, void* d_dW, int64_t lddw, int dw_type,
                            unsigned flags, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* OZ2_LM_H */
