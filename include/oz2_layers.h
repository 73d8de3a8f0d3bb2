/*
 * oz2_layers.h -- operators of liboz2 around a product, for a model's layers:
 * a linear layer with its epilogue, that layer's gradient, and the AdamW step
 * that updates the weights, for one NVIDIA GB300 (sm_103a).
 *
 * Conventions are those of oz2.h: matrices are column-major, d_* are device
 * pointers, work is enqueued on `stream` without synchronising the host, the
 * return value is OZ2_OK or a negative oz2_status, errors found on the host
 * enqueue nothing, a kernel's bounded wait that ran out is reported by
 * oz2_check_device_status, and workspace is allocated and freed stream-ordered
 * from the library's pool (oz2_trim_memory); calls on several streams may
 * overlap and calls can be captured into a CUDA graph.
 *
 * Tokens are columns: X is k×m with a token's k features contiguous, which is
 * the row-major (m, k) array that deep-learning frameworks hold.  W is k×n, an
 * output's k weights contiguous: the row-major (n, k) weight of a linear layer.
 *
 * Sums are held in FP32 and rounded once to the output's type.  (The tensor
 * cores' FP32 sums truncate: against 64 bits a sum is low by 1e-9 to 5e-9 of
 * itself for each element summed over, some 2e-5 at 16384, below a 16-bit
 * rounding; it shows in an F32 dW over very many tokens.)  Base addresses
 * are multiples of the element size; leading dimensions are in elements.
 *
 * An operand of a product is copied first (a pass over it, and workspace for it)
 *   - where its base or leading dimension is no multiple of 16 bytes: its rows go to
 *     ones that are multiples of 128.  But weights off the 16-byte grid are read where
 *     they lie for up to 16 tokens, without workspace, unless there are over 4096 rows
 *     of less than 512 bytes;
 *   - where both operands' rows lie on odd multiples of 16 bytes and the product is so
 *     long that it pays: the smaller one of oz2_linear's, dY of oz2_linear_grad.
 */
#ifndef OZ2_LAYERS_H
#define OZ2_LAYERS_H

#include "oz2.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { OZ2_TYPE_F32 = 0, OZ2_TYPE_BF16 = 1, OZ2_TYPE_F16 = 2, OZ2_TYPE_E4M3 = 3 } oz2_type;

/* act(z): z; max(z, 0); z·Φ(z); z·(1 + tanh(√(2/π)(z + 0.044715 z³)))/2;
 * z/(1 + e^-z).  In FP32, off by some 2^-19 of the value and 2^-21 of it for each
 * unit of exp's argument, far into the tails too; a factor of z below 2^-126 counts
 * as 0. */
typedef enum {
  OZ2_ACT_NONE = 0,
  OZ2_ACT_RELU = 1,
  OZ2_ACT_GELU = 2,
  OZ2_ACT_GELU_TANH = 3,
  OZ2_ACT_SILU = 4
} oz2_act;

/* Y = act(Z) + R with Z = Wᵀ·X, scaled and biased:
 *   Z_jt = (Σ_l W_lj X_lt) · w_scale_j · x_scale_t + bias_j
 * for m tokens t, n outputs j and k features l.  In one pass: bias, activation
 * and residual are applied to the sums before they are rounded.
 *   type      of X and W: BF16, F16 or E4M3
 *   d_x_scale m floats, d_w_scale n floats: with E4M3 both or neither; null
 *             otherwise
 *   d_bias    n values of bias_type (F32 or out_type), or null
 *   d_R       n×m of out_type (ldr ≥ n), or null; may be d_Y itself
 *   d_Z       n×m of out_type (ldz ≥ n), written with Z, or null
 *   d_Y       n×m of out_type (ldy ≥ n); not overlapping X or W
 *   out_type  BF16 or F16: X's type where that is a 16-bit one
 * m = 0 or n = 0: nothing; k = 0: Z = bias.  Errors: OZ2_ERR_INVALID_ARG for
 * sizes, leading dimensions, pointers or a combination of types not named here;
 * OZ2_ERR_UNSUPPORTED for a size of 2^31 - 256 or more. */
int oz2_linear(int64_t m, int64_t n, int64_t k, int type,
               const void* d_X, int64_t ldx, const void* d_W, int64_t ldw,
               const float* d_x_scale, const float* d_w_scale,
               const void* d_bias, int bias_type, int act,
               const void* d_R, int64_t ldr, void* d_Z, int64_t ldz,
               void* d_Y, int64_t ldy, int out_type, void* stream);

/* The gradient of oz2_linear (16-bit types) from dY = ∂L/∂Y and the Z it kept:
 *   dZ = dY ∘ act'(Z)    dX = W·dZ    dW = X·dZᵀ    db_j = Σ_t dZ_jt
 * (dR is dY.)  act'(0) of ReLU is 0.
 *   type      of dY, Z, X, W and dX: BF16 or F16
 *   d_Z       n×m (ldz ≥ n); may be null with OZ2_ACT_NONE
 *   d_dX      k×m (lddx ≥ k), or null: not wanted (d_W may then be null)
 *   d_dW      k×n of dw_type (lddw ≥ k), or null: not wanted (d_X may then be
 *             null)
 *   dw_type   `type` or F32
 *   d_db      n floats, or null
 *   flags     OZ2_GRAD_ACCUMULATE: dW (F32 only) and db are added to
 * dZ is rounded to `type` before the products, whose operand it is on the
 * tensor cores (dX and dW then carry two roundings to that type in place of
 * one); db is summed from the unrounded one, in a fixed order.  The outputs overlap no input.  m = 0: dW = 0
 * and db = 0 (unchanged when accumulating). */
#define OZ2_GRAD_ACCUMULATE 0x1u
int oz2_linear_grad(int64_t m, int64_t n, int64_t k, int type,
                    const void* d_dY, int64_t lddy, const void* d_Z, int64_t ldz, int act,
                    const void* d_X, int64_t ldx, const void* d_W, int64_t ldw,
                    void* d_dX, int64_t lddx, void* d_dW, int64_t lddw, int dw_type,
                    float* d_db, unsigned flags, void* stream);

/* One AdamW step over `count` tensors, in one launch for up to 256 of them (twice
 * that where some have a master and some have none):
 *   g' = c·g    m ← β1·m + (1-β1)·g'    v ← β2·v + (1-β2)·g'²
 *   w ← w - lr·λ·w - lr·(m/(1-β1^t))/(√(v/(1-β2^t)) + ε)
 * with t = step, λ = weight_decay, c = *d_grad_scale (1 if null; read on the
 * device, so that a clipping factor needs no host round trip), and lr and λ
 * multiplied by the tensor's own lr_scale and decay_scale.
 *
 * w is `master` (F32) where that is not null, and `param` then receives its
 * copy rounded to param_type (or is null); else w is `param` itself.
 *
 * state_bits 32: m and v are floats.  state_bits 8: m and v are E4M3 values and
 * m_scale, v_scale hold one float per 256 of them (the last block of a tensor
 * may be short): m = value·m_scale and √v = value·v_scale.  The scales are
 * powers of two that bring a block's largest finite magnitude to (224, 448]; a
 * value is rounded to one of its two E4M3 neighbours at random, up with the
 * probability of its distance from the lower one, by 16 bits of a hash of
 * seed, step and the value's number: the list's values are numbered through,
 * every tensor starting a new block of 256 (so a step can be repeated bit for
 * bit, and a tensor's place in the list matters).  w is updated from the
 * unrounded m and v.  An element whose √v is zero has no history: its m counts as
 * zero too.  (So it is with elements whose gradients stay some 10^-5 of their
 * block's largest: √v may be rounded to zero, and their steps are those of single
 * gradients, up to (1-β1)/√(1-β2) of lr.  Tensors where those matter want 32 bits.)
 * States of zero bytes with any finite scales are the initial state.  A value that
 * is not finite is kept as E4M3's NaN; the others of its block are not touched by it.
 *
 * The tensors' addresses and all of `args` but *d_grad_scale go by value: a captured
 * call is this step again at every replay, with its bias corrections and its random
 * bits (8-bit states then are not rounded at random from replay to replay).  Training
 * calls it anew for each step, after the replay of what was captured.
 *
 * param_type F32, BF16 or F16 (a master wants a 16-bit one); grad_type F32 or
 * param_type.  Errors:
 * OZ2_ERR_INVALID_ARG for null pointers, negative sizes, step < 1, betas
 * outside [0, 1), or a combination of types not named here. */
typedef struct {
  int64_t numel;
  void* param;
  const void* grad;
  float* master;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  float lr_scale, decay_scale;
} oz2_adamw_tensor;
typedef struct {
  int64_t step;
  double lr, beta1, beta2, eps, weight_decay;
  const float* d_grad_scale;
  uint32_t seed;
} oz2_adamw_step;
int oz2_adamw(const oz2_adamw_tensor* tensors, int count, int param_type, int grad_type, int state_bits,
              const oz2_adamw_step* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* OZ2_LAYERS_H */
