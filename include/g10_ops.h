/* g10_ops.h - C ABI of the operators of a training step that stand next to the planner (same library, gfx950).
 *
 * The planner of g10.h moves tensors that a step keeps but does not use.  These operators keep fewer: attention whose
 * scores never leave the chip, the norms of queries and keys together with the rotation by position, one AdamW
 * update over all weights with its moments in 8 bits where wanted, norms of rows and the first half of a gated MLP whose
 * backward passes are given the inputs alone, log probabilities whose gradient needs one number a row, and the lookup in a table
 * of embeddings with its gradient.
 *
 * Conventions
 *   - plain C, no exceptions, no state outside the handles of g10_adamw_create; every call but g10_adamw_free returns
 *     G10_OK or a negative error of g10.h (G10_EINVAL for what the argument checks refuse, G10_EDEVICE, G10_ENOMEM).
 *   - pointers are DEVICE pointers owned by the caller unless a comment says host; every call enqueues on `hip_stream`
 *     (NULL = default stream) of the current device and does not wait for it.  No call allocates device memory but
 *     g10_adamw_create; calls that need room besides their outputs are given it (`workspace`, of at least the size that
 *     the operator's *_workspace function says; contents are neither read nor kept).
 *   - strides are in elements, the last dimension is contiguous.  Nothing is written outside the outputs' elements.
 *   - every result is the same from run to run: no sum depends on the order in which work finishes.
 */
#ifndef G10_OPS_H
#define G10_OPS_H

#include <stdint.h>

#include "g10.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { G10_F32 = 0, G10_F16 = 1, G10_BF16 = 2, G10_E4M3 = 3 };   /* element types */

/* ------------------------------------------------------------------------------------------------ norm and rotation
 * For every token and head, x of `dim` values:   r = 1 / sqrt(mean(x^2) + eps),  n = x * r * weight,  and the first
 * `rot` values of n are turned pair by pair by the angles of the token's position, (a, b) -> (a c - b s, b c + a s).
 * Pairs are (i, i + rot/2), or neighbours (2i, 2i + 1) with G10_ROPE_INTERLEAVED.  Queries and keys in one pass.
 * Sums in 32 bits, one rounding at the end. */
#define G10_ROPE_INTERLEAVED 1u
#define G10_ROPE_POSITIONS_64 2u /* positions are int64_t, not int32_t */

typedef struct {
  const void *x;             /* [batch][seq][heads][dim], or NULL with heads = 0               */
  const void *weight;        /* [dim] of weight_type, or NULL: no weight                       */
  const void *dy;            /* backward only: gradient of the output                          */
  void *out;                 /* forward: the output (may be x); backward: gradient of x (may be x or dy) */
  void *dweight;             /* backward only, with a weight: its gradient, [dim] of weight_type, or NULL */
  int64_t x_stride[3], dy_stride[3], out_stride[3]; /* batch, token, head                      */
  uint32_t heads;
} g10_rope_part;

typedef struct {
  g10_rope_part part[2];     /* queries, keys                                                  */
  uint32_t batch, seq, dim, rot; /* dim 1..256; rot even, 0..dim                               */
  const float *table;        /* [n_positions][rot]: cosines of the rot/2 angles, then their sines */
  uint32_t n_positions;
  const void *positions;     /* [batch][seq]; a position outside the table makes its token's outputs (backward:
                                its gradients and its share of dweight) NaN                    */
  float eps;                 /* >= 0                                                           */
  uint32_t type, weight_type;/* of x, dy, out: G10_F32, G10_F16, G10_BF16; of the weights: `type` or G10_F32 */
  uint32_t flags;
} g10_rope_args;

int g10_norm_rope(const g10_rope_args *args, void *hip_stream);
/* Bytes of workspace that g10_norm_rope_backward takes for these arguments (host result). */
int g10_norm_rope_workspace(const g10_rope_args *args, uint64_t *bytes);
int g10_norm_rope_backward(const g10_rope_args *args, void *workspace, uint64_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------------------------------------- attention
 * o_i = sum_j softmax_j(scale q_i k_j) v_j over the keys j that query i sees.  Query i of a sequence of n_q queries and
 * n_k keys stands at position p = i + n_k - n_q (the last query at the last key).  It sees j if j < n_k and
 *   causal:      j <= p  and  (window == 0  or  j > p - window    or  j < sinks)
 *   otherwise:                 window == 0  or  |j - p| < window  or  j < sinks
 * A query that sees nothing has o = 0, lse = -infinity, and no gradient.  `heads` is a multiple of `kv_heads`: query
 * head h reads key head h / (heads / kv_heads), whose gradient is the sum over them.
 * Sequences lie side by side ([batch][seq][head][dim]; q_start = k_start = NULL), k_len then says how many keys each
 * has; or packed one behind the other ([total][head][dim]): q_start and k_start hold where each begins, batch + 1
 * numbers, none below the one before it.  Keys past a sequence's end are not read.  Numbers that point outside the tensors are moved
 * to their border.  Rows of packed tensors before the first sequence and behind the last one (padding) see nothing and are seen by none. */
typedef struct {
  const void *q, *k, *v;
  void *o;                   /* forward: output; backward: the forward pass's                  */
  float *lse;                /* natural logarithm of the sum of exponentials, contiguous: [batch][heads][seq_q], packed:
                                [heads][seq_q]                                                 */
  const void *d_o;           /* backward                                                       */
  void *dq, *dk, *dv;        /* backward                                                       */
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3]; /* batch (not read if packed), token, head */
  int64_t do_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
  uint32_t batch, heads, kv_heads, dim; /* dim: a multiple of 8 up to 128                      */
  uint32_t seq_q, seq_k;     /* tokens per sequence; packed: rows of q and of k in all         */
  const int32_t *q_start, *k_start; /* [batch + 1] or NULL, both or none                       */
  const int32_t *k_len;      /* [batch] or NULL; not with q_start                              */
  uint32_t max_q, max_k;     /* packed: length of the longest sequence; decides how the work is cut, not what is computed */
  uint32_t causal, window, sinks;
  float scale;               /* > 0                                                            */
  uint32_t type;             /* G10_F16 or G10_BF16                                            */
} g10_attention_args;
/* Pointers and strides of q, k, v, o, d_o, dq, dk, dv are multiples of 16 bytes (of 8 elements), token strides at
 * most 2^22 elements; else G10_EINVAL. */

int g10_attention_workspace(const g10_attention_args *args, uint64_t *bytes);
int g10_attention(const g10_attention_args *args, void *workspace, uint64_t workspace_bytes, void *hip_stream);
int g10_attention_backward_workspace(const g10_attention_args *args, uint64_t *bytes);
int g10_attention_backward(const g10_attention_args *args, void *workspace, uint64_t workspace_bytes, void *hip_stream);

/* ----------------------------------------------------------------------------------------------------------- AdamW
 * One update of many tensors, in 32-bit arithmetic, with g' = g * coefficient:
 *   m = beta1 m + (1 - beta1) g'      v = beta2 v + (1 - beta2) g'^2
 *   p = p (1 - lr decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * The moments of all tensors lie in one array each, every tensor's part beginning at a multiple of G10_ADAMW_BLOCK
 * elements.  state_type G10_F32: m and v themselves.  G10_E4M3: m and sqrt(v) in blocks of G10_ADAMW_BLOCK values, 8-bit
 * floats (3 bits of mantissa) times one 32-bit scale a block, largest magnitude / 448; the update of a step works on
 * the moments before they are rounded.  A root above zero is never held as zero; blocks whose largest magnitude is below
 * 1e-30 are held as zeros.  Tensors and copies must not overlap: they are updated side by side.  Steps 1 to G10_ADAMW_NEAREST round to nearest, which is the more exact while the moments come into being (after 16 steps on
 * normal gradients m and the root are off by 4.9 and 6.0 %, else by 5.7 and 6.9).  Later ones round up or down by a threshold that goes by the
 * value's place and the step's number, so that the mean over steps is right: a step moves a root by far less than half of what separates
 * two 8-bit values, and to nearest it would no longer move.  A step that is captured and replayed has the number, and the thresholds, of its capture. */
#define G10_ADAMW_BLOCK 256u
#define G10_ADAMW_NEAREST 16u
#define G10_ADAMW_MAX_TENSORS 1048576u

typedef struct {
  void *p;                   /* n elements, contiguous                                         */
  void *copy;                /* the updated p rounded to copy_type, or NULL                    */
  uint64_t n;                /* may be 0                                                       */
} g10_adamw_tensor;

typedef struct {
  const g10_adamw_tensor *tensors; /* HOST array; what it points to stays the caller's and in place until g10_adamw_free */
  uint32_t count;
  uint32_t type, grad_type, copy_type, state_type; /* of p and the gradients: F32, F16, BF16; copies: F16, BF16 */
  void *m, *v;               /* [G10_ADAMW_BLOCK * blocks], 16-byte aligned                    */
  float *m_scale, *v_scale;  /* [blocks], with G10_E4M3                                        */
} g10_adamw_desc;

typedef struct {
  double lr, beta1, beta2, eps, weight_decay;
  uint64_t step;             /* of this update: 1 for the first                                */
  const float *coefficient;  /* device, or NULL = 1.  If it is not finite nothing is updated   */
} g10_adamw_params;

typedef struct g10_adamw_s g10_adamw_t;

/* Blocks that tensors of these sizes take in the moments' arrays (host result): sum of ceil(n / G10_ADAMW_BLOCK). */
int g10_adamw_blocks(const g10_adamw_tensor *tensors, uint32_t count, uint64_t *blocks);
/* Device tables of the tensors' places.  Allocates, and waits for `hip_stream`. */
int g10_adamw_create(const g10_adamw_desc *desc, void *hip_stream, g10_adamw_t **out);
/* `grads`: HOST array of `count` device pointers, read during the call; NULL: that tensor is left as it is. */
int g10_adamw_step(g10_adamw_t *handle, const void *const *grads, const g10_adamw_params *params, void *hip_stream);
/* out[0] = norm of all gradients together (the ones that are not NULL), summed in 64 bits; out[1] = the coefficient that
 * limits it: min(1, max_norm / (norm + 1e-6)), NaN where the norm is not finite (a step with it changes nothing).
 * out: device, 2 floats; max_norm > 0.  The handle's own workspace: calls on one handle must not overlap in time. */
int g10_grad_norm(g10_adamw_t *handle, const void *const *grads, float max_norm, float *out, void *hip_stream);
void g10_adamw_free(g10_adamw_t *handle); /* after waiting for the device; NULL is allowed */

/* ------------------------------------------------------------------------------------------------------ embeddings
 * out_t = scale * table[ids_t], and of the table: dtable_v = scale * sum over the tokens t with ids_t = v of dout_t, summed in 32 bits.
 * Every row of dtable is written, the ones without a token with zeros.  An id outside the table makes its token's out NaN and
 * has no part in dtable.  The sums' order is that of the tokens, cut into pieces that depend on the sizes and the ids alone. */
typedef struct {
  const void *ids;           /* [tokens], int32_t, or int64_t with ids_64                      */
  const void *table;         /* forward: [vocab][dim]                                          */
  void *out;                 /* forward: [tokens][dim]                                         */
  const void *dout;          /* backward: [tokens][dim]                                        */
  void *dtable;              /* backward: [vocab][dim]                                         */
  int64_t table_stride, out_stride, dout_stride, dtable_stride; /* of rows                      */
  uint32_t tokens, vocab, dim; /* tokens below 2^31, vocab 1 .. 2^31 - 1, dim 1 .. 65536         */
  float scale;
  uint32_t type;             /* of table, out, dout, dtable: G10_F32, G10_F16, G10_BF16        */
  uint32_t ids_64;
} g10_embed_args;

int g10_embed(const g10_embed_args *args, void *hip_stream);
int g10_embed_backward_workspace(const g10_embed_args *args, uint64_t *bytes);
int g10_embed_backward(const g10_embed_args *args, void *workspace, uint64_t workspace_bytes, void *hip_stream);

/* ---------------------------------------------------------------------------------------------------- norms of rows
 * For every row x of `dim` values:   m = mean(x) with `center`, else 0;   r = 1 / sqrt(mean((x - m)^2) + eps);
 *   n = (x - m) r;   y = n * weight + bias.
 * Backward, from x and dy alone, with u = dy * weight:   dx = r (u - n mean(u n) - [center] mean(u)),
 *   dweight = sum of dy n,  dbias = sum of dy  over the rows.
 * Row sums in 32 bits (the squares of what is left after the mean is taken off), sums over rows in 32 and joined in 64.  Squares that add up
 * beyond 32 bits (values of 1.8e19) make a row's n zero. */
typedef struct {
  const void *x, *dy;        /* [rows][dim]; dy: backward                                      */
  const void *weight, *bias; /* [dim] of weight_type, or NULL                                  */
  void *out;                 /* forward: y (may be x); backward: dx (may be x or dy)           */
  void *dweight, *dbias;     /* backward: [dim] of weight_type, or NULL                        */
  int64_t x_stride, dy_stride, out_stride; /* of rows                                           */
  uint32_t rows, dim;        /* rows below 2^31, dim 1 .. 65536                                */
  float eps;                 /* >= 0                                                           */
  uint32_t center;
  uint32_t type, weight_type;/* of x, dy, out: G10_F32, G10_F16, G10_BF16; of the weights: `type` or G10_F32 */
} g10_norm_args;

int g10_norm(const g10_norm_args *args, void *hip_stream);
int g10_norm_backward_workspace(const g10_norm_args *args, uint64_t *bytes);
int g10_norm_backward(const g10_norm_args *args, void *workspace, uint64_t workspace_bytes, void *hip_stream);

/* ---------------------------------------------------------------------------------------------------- log probabilities
 * Of every row z = scale * logits:   lse = log sum_j exp z_j,   p_j = exp(z_j - lse),   logp = z_t - lse for the row's token t,
 *   entropy = - sum p_j log p_j,   and the `top` largest z_j - lse with their places, ties in order of the places.
 * dlogits_j = scale * (dlogp ([j = t] - p_j) - dentropy p_j (log p_j + entropy)).
 * A token equal to `ignore` has logp = 0 and no share in the gradient; any other one outside the row makes logp NaN, and the row's
 * gradient too where dlogp is given and not 0.  Places of -infinity have no probability; a row of nothing else has lse = logp = -infinity, entropy 0 and no gradient.
 * Sums, logp, top_logp, entropy and the gradient go by distances from the row's largest logit and are as exact for a row with a large offset, or at the type's end,
 * as for one around zero; lse is rounded to 32 bits where it lies, and infinite where scale * logits are beyond them.  Where it is 64 or more (16-bit logits: 256),
 * either side of zero, the backward pass sums the row again.
 * A row with a NaN or +infinity has logp, lse, entropy and the gradient NaN (NaN counts as the largest where the top is sought); a row
 * with dlogp = 0 or an ignored token, and dentropy = 0, has the gradient 0 whatever it holds. */
#define G10_LOG_PROBS_TOP 64u

typedef struct {
  const void *logits;        /* [rows][vocab]                                                  */
  const int64_t *tokens;     /* [rows], or NULL: no logp (and no share of it in the gradient)  */
  float *logp, *lse, *entropy; /* forward: [rows]; entropy may be NULL.  Backward reads lse, and entropy with dentropy */
  float *top_logp;           /* forward: [rows][top], with top > 0                             */
  int64_t *top_ids;
  const float *dlogp, *dentropy; /* backward: [rows], or NULL                                  */
  void *dlogits;             /* backward: [rows][vocab], may be logits                         */
  int64_t logits_stride, dlogits_stride; /* of rows                                             */
  uint32_t rows, vocab;      /* vocab 1 .. 2^31 - 1                                            */
  uint32_t top;              /* 0 .. G10_LOG_PROBS_TOP, at most vocab                          */
  float scale;               /* above 0, up to 2e38                                            */
  int64_t ignore;
  uint32_t type;             /* of logits and dlogits: G10_F32, G10_F16, G10_BF16              */
} g10_log_probs_args;

int g10_log_probs_workspace(const g10_log_probs_args *args, uint64_t *bytes);
int g10_log_probs(const g10_log_probs_args *args, void *workspace, uint64_t workspace_bytes, void *hip_stream);
int g10_log_probs_backward(const g10_log_probs_args *args, void *hip_stream);

/* ------------------------------------------------------------------------------------------------------- gated MLP
 * Of tokens x and two weights:   g = x gate,   u = x up,   h = act(g) * u.   act: g / (1 + exp(-g)), or g * Phi(g) with the normal
 * distribution's Phi.  Backward, from x, the weights and dh alone (g and u are computed again):
 *   dg = dh u act'(g),   du = dh act(g),   dx = dg gate^T + du up^T,   dgate = x^T dg,   dup = x^T du.
 * Products of 16-bit factors summed in 32 bits; dg and du are rounded to `type` before their products (the matrix unit takes 16-bit
 * factors), h and the gradients once at their end.  In G10_F16 a dg or du above 65504 is infinite from there on, and one below 6e-5 has fewer bits:
 * dh is scaled so that they lie between. */
#define G10_ACT_SILU 0u
#define G10_ACT_GELU 1u

typedef struct {
  const void *x;             /* [tokens][dim]                                                  */
  const void *gate, *up;     /* [dim][inner], or with out_in [inner][dim]                      */
  void *h;                   /* forward: [tokens][inner]                                       */
  const void *dh;            /* backward: [tokens][inner]                                      */
  void *dx;                  /* backward: [tokens][dim]                                        */
  void *dgate, *dup;         /* backward: laid out as the weights                              */
  int64_t x_stride, gate_stride, up_stride, h_stride, dh_stride, dx_stride, dw_stride; /* of rows, not shorter than they are */
  uint32_t tokens, dim, inner; /* dim and inner 1 .. 2^20, tokens below 2^31                     */
  uint32_t act, out_in;
  uint32_t type;             /* G10_F16 or G10_BF16                                            */
} g10_gated_args;
/* Inputs whose pointers and strides are multiples of 16 bytes (of 8 elements) and whose rows are multiples of 8 elements, with strides up to 2^22 and
 * one stride for both weights, are read where they lie; others are laid out in the workspace first.  Outputs may lie anywhere.
 * A product is cut into tiles of 64 to 256 rows by 64 to 256 columns, and its sum into up to 32 shares; one of more than 2^23 tiles and shares
 * altogether is refused (2^20 inner values: from some 2^18 tokens on), by the call, not by the workspace's. */

int g10_gated_workspace(const g10_gated_args *args, uint64_t *bytes);
int g10_gated(const g10_gated_args *args, void *workspace, uint64_t workspace_bytes, void *hip_stream);
int g10_gated_backward_workspace(const g10_gated_args *args, uint64_t *bytes);
int g10_gated_backward(const g10_gated_args *args, void *workspace, uint64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* G10_OPS_H */
