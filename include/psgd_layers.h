/*
 * psgd_layers.h - C boundary of the learners' layers and losses: the work that produces the gradients G which the averaging step
 * X_out = mix(X) - lr * G of psgd.h takes (Sec. 2, Eq. 2: g(Phi_k, xi_k)).
 *
 * All n learners are computed by one call.  Activations are [n, t, c] arrays (t tokens of each learner), parameters are views of the
 * rows of an [n, d] array (learner i's layer lies at the same columns of row i), and gradients of parameters are written into views of the
 * rows of another.  A single model is n = 1.  In float the arrays are the averaging step's own X and G.  In bf16 G is (the step takes bf16 gradients), and a
 * layer norm reads its gain and bias from X whatever its activations are, but the matrices of psgd_linear have the type of its activations: a learner that
 * computes in bf16 keeps a bf16 copy of X's rows for them and makes it anew after each step.
 *
 * Conventions of psgd.h hold: device pointers of the current device, nothing kept after the enqueued work has run, PSGD_OK or a
 * negative psgd_status with the text in psgd_last_error(), work enqueued on `stream` only.  Beyond them:
 *   - nothing is allocated: what a call needs besides its operands it takes from the caller's workspace, whose size the
 *     *_workspace function beside it returns for the same arguments.  The workspace's contents mean nothing between calls; calls that
 *     may run at the same time need one each.  It starts at 256 bytes.
 *   - sums, statistics and gradients are accumulated in fp32; each output is rounded once to its type.  The order of every sum is fixed: the
 *     same call gives the same bits.
 */
#ifndef PSGD_LAYERS_H
#define PSGD_LAYERS_H

#include <stddef.h>
#include <stdint.h>

#include "psgd.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { PSGD_F32 = 0, PSGD_BF16 = 1, PSGD_I32 = 2 };

/*
 * One operand: element (i, r, c) of learner i, row r and column c lies at data[i * learner + r * row + c], strides in ELEMENTS, columns
 * next to each other.  A learner or row stride of 0 shares an INPUT between learners or rows; outputs may not share a byte.  Data need
 * only be aligned to its elements.  Parameter vectors ([n, c]) have no rows: `row` is ignored.
 */
typedef struct {
    void* data;
    int64_t learner;
    int64_t row;
    int32_t type;
} psgd_view;

/* Activations of the linear layer. */
enum { PSGD_ACT_NONE = 0, PSGD_ACT_RELU = 1, PSGD_ACT_GELU = 2 /* z Phi(z), the normal distribution's */, PSGD_ACT_SILU = 3 };

enum { PSGD_MAX_TOP = 64, PSGD_MAX_SLOTS = 1024 };   /* psgd_token_logprobs: k; psgd_distill: k */

/*
 * psgd_layer_norm - y = (x - m) r gain + bias with m the mean and r = (variance + eps)^-1/2 of each row of c columns.
 *
 *   x, y        [n, t, c], float or bf16 alike; y may be x (same pointer and strides)
 *   gain, bias  [n, c], float or bf16 alike; bias may be NULL
 *   mean, rstd  float [n * t] each, written, or both NULL
 * The variance is that of the differences from the mean, taken in a second pass over values on the chip.
 * n in 1..PSGD_MAX_N, t and c >= 0 (nothing to do if t or c is 0), eps >= 0.
 */
int psgd_layer_norm(const psgd_view* x, const psgd_view* gain, const psgd_view* bias, const psgd_view* y, float* mean, float* rstd,
                    int n, int64_t t, int64_t c, float eps, void* stream);

/*
 * psgd_layer_norm_grad - its backward pass.  With u = dy gain and h = (x - mean) rstd:
 *     dx = rstd (u - mean_c(u) - h mean_c(u h)) [+ add],   dgain = sum_t dy h,   dbias = sum_t dy.
 *
 *   dy, x, dx, add  [n, t, c], one type; add (or NULL) is the gradient that reaches x by another way; dx may be dy or add
 *   gain            [n, c], float or bf16;    mean, rstd  float [n * t] as psgd_layer_norm wrote them
 *   dgain, dbias    [n, c], float or bf16 alike, or NULL (each)
 * With t = 0 the parameter gradients are zero.
 */
size_t psgd_layer_norm_grad_workspace(int n, int64_t t, int64_t c);
int psgd_layer_norm_grad(const psgd_view* dy, const psgd_view* x, const psgd_view* gain, const float* mean, const float* rstd,
                         const psgd_view* add, const psgd_view* dx, const psgd_view* dgain, const psgd_view* dbias, int n, int64_t t,
                         int64_t c, void* workspace, size_t workspace_bytes, void* stream);

/*
 * psgd_linear - y = act(z) [+ residual], z = x W' [+ b], for every learner by its own W and b.
 *
 *   x [n, t, in], w [n, out, in] (row r of w: output r), bias [n, out] or NULL, residual [n, t, out] or NULL (it may be y),
 *   y [n, t, out], z [n, t, out] or NULL (written: what the backward pass needs of an activation).  One type for all, float or bf16.
 * bf16 products are exact and summed in fp32; float products and sums are fp32.  in = 0 gives z = bias.
 */
size_t psgd_linear_workspace(const psgd_view* x, const psgd_view* w, int n, int64_t t, int64_t in, int64_t out);
int psgd_linear(const psgd_view* x, const psgd_view* w, const psgd_view* bias, const psgd_view* residual, const psgd_view* y,
                const psgd_view* z, int act, int n, int64_t t, int64_t in, int64_t out, void* workspace, size_t workspace_bytes,
                void* stream);

/*
 * psgd_linear_grad - its backward pass.  With dz = dy act'(z):  dx = dz W,  dw = dz' x,  db = sum_t dz.
 *
 *   dy, z [n, t, out] (z is needed unless act is PSGD_ACT_NONE), x, w as in psgd_linear; dx [n, t, in], dw [n, out, in], db [n, out],
 *   each may be NULL.  One type for all.  A residual's gradient is dy itself.
 * In bf16, dz is rounded to bf16 where it enters the two products (db sums it before that).
 */
size_t psgd_linear_grad_workspace(const psgd_view* dy, const psgd_view* x, const psgd_view* w, const psgd_view* dx, const psgd_view* dw,
                                  const psgd_view* db, int act, int n, int64_t t, int64_t in, int64_t out);
int psgd_linear_grad(const psgd_view* dy, const psgd_view* z, const psgd_view* x, const psgd_view* w, const psgd_view* dx,
                     const psgd_view* dw, const psgd_view* db, int act, int n, int64_t t, int64_t in, int64_t out, void* workspace,
                     size_t workspace_bytes, void* stream);

/*
 * psgd_token_logprobs - what a model says of given tokens.  With q = softmax(logits) over a row's v columns:
 *
 *   logits    [n, t, v], float or bf16
 *   tokens    [n, t] int32 (PSGD_I32; `row` is the stride between tokens)
 *   logp      float [n * t]: log q(token); 0 where the token is negative (none given)
 *   entropy   float [n * t] or NULL: -sum q log q
 *   top_logp, top_idx   float and int32 [n * t * k], or both NULL with k = 0: the k largest log q and their columns, largest first, equal
 *             logits by ascending column (NaN counts as the largest)
 * A logit of -inf is a masked column (q = 0).  A row of nothing but -inf has log q = -inf everywhere and entropy 0; one with NaN or
 * +inf gives NaN for logp, entropy and top_logp.  A token >= v gives NaN and raises bit 1 of psgd_device_status().
 * v in 1..2^31-1, k in 0..min(v, PSGD_MAX_TOP).
 */
int psgd_token_logprobs(const psgd_view* logits, const psgd_view* tokens, float* logp, float* entropy, float* top_logp, int32_t* top_idx,
                        int k, int n, int64_t t, int64_t v, void* stream);

/*
 * psgd_distill - distillation from a teacher's top logits, loss and gradient.  With p the softmax of a row's given teacher logits / tau
 * over the slots given, and q = softmax(logits / tau) over all v columns:
 *
 *     loss = weight tau^2 sum_s p_s (log p_s - log q(idx_s)),     dlogits = d loss / d logits = weight tau (q - p)
 *
 *   logits, dlogits     [n, t, v], one type, float or bf16; dlogits may be logits, or NULL for the loss alone
 *   top_idx, top_logit  [n, t, k] int32 and float: the teacher's columns and logits (or log probabilities: p is the same).  A negative
 *                       index or a logit of -inf is a slot that is not given; a column given twice counts twice
 *   weight              float [n * t] or NULL (all 1): 1 / tokens for a mean, 0 for a masked row
 *   loss                float [n * t]
 * A row with weight 0 or no slot given has loss 0 and gradient 0 whatever its logits hold.  An index >= v counts as a slot not given and
 * raises bit 1 of psgd_device_status().  tau > 0 and finite, log2(e) / tau too; v in 1..2^31-1, k in
 * 1..PSGD_MAX_SLOTS.
 */
int psgd_distill(const psgd_view* logits, const psgd_view* top_idx, const psgd_view* top_logit, const float* weight, float* loss,
                 const psgd_view* dlogits, float tau, int k, int n, int64_t t, int64_t v, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PSGD_LAYERS_H */
