/*
 * ar_ops.h -- C ABI of the operators around libar's collectives (gfx950).
 *
 * A rank of a tensor- or data-parallel program computes a block on its shard,
 * has the ranks' results joined, adds the join to its residual stream between
 * two norms, and turns joined gradients into weight updates.  The joins are
 * ar.h's collectives; the rest is here:
 *   ar_gated_ffn       act(x Wg^T) * (x Wu^T), and its backward pass
 *   ar_residual_norm   norm of a block's output, gate, scaled residual, norm
 *                      before the next block, and its backward pass
 *   ar_orthogonalize   Newton-Schulz products that orthogonalise an update
 *   ar_attention       attention of a rank's heads over packed sequences, and
 *                      its backward pass
 *   ar_vocab_loss      cross entropy over a vocabulary or a rank's rows of it,
 *                      and its backward pass
 *
 * Conventions.  As in ar.h: device pointers on the current device, sizes in
 * elements unless named *_bytes, `stream` a hipStream_t as void* (NULL = the
 * null stream), AR_OK or an AR_ERR_* code returned, the code of a failure also
 * left in ar_last_error().  Calls are asynchronous on `stream`, allocate
 * nothing, create no stream or event and issue no memset, so they may be
 * captured into a HIP graph and replayed.  They keep nothing between calls, beside
 * which kernels a device has been told about, and may be made from several host
 * threads and for several devices.  Matrices are row-major with a row
 * stride (`ld_*`, elements; 0 = the number of columns; at least that number);
 * elements of a row are contiguous.  Pointers need the alignment of their
 * elements and no more.  Where a function takes a workspace, it is device
 * memory of at least the bytes that the matching *_workspace function names
 * for the same description, 256-byte aligned, owned by the caller and used
 * until the call's work on `stream` is done (AR_ERR_SCRATCH: too small or
 * absent).  Calls that overlap in time need workspaces of their own.
 *
 * Aliasing.  An output must not overlap another output or an input, but where
 * a function says that it may be an input itself: then with the same pointer
 * and row stride.  Column ranges of one buffer that share no element do not
 * overlap.  AR_ERR_ARG otherwise.
 *
 * Arithmetic.  fp32 throughout (sums of squares of ar_orthogonalize in fp64);
 * outputs are rounded to their type once, to nearest even.  Where an operand
 * of a matrix product is rounded on the way, the function says so.  Results
 * depend on the inputs alone: sums are taken in a fixed order and no atomics
 * are used, so repeated calls give the same bits.
 */
#ifndef AR_OPS_H
#define AR_OPS_H

#include "ar.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- residual norm ------------------------------------------------------ */

/* Per row t, with rms(v) = sqrt(mean_j v_j^2 + eps):
 *     n = y / rms(y) * post_weight           (without AR_NORM_POST: n = y)
 *     s = alpha * residual + gate * n        (without a gate: gate = 1)
 *     x = s / rms(s) * pre_weight            (without AR_NORM_PRE: no x)
 * y is a block's output (joined over the ranks), s the new residual stream, x
 * the next block's input.  x is computed from the unrounded s.  A NULL weight
 * stands for ones. */
enum { AR_NORM_POST = 1, AR_NORM_PRE = 2 };

typedef struct ar_norm_desc {
    size_t rows;           /* 0 is a valid no-op (backward: zero parameter gradients) */
    size_t cols;           /* 1 or more */
    int dtype;             /* AR_FLOAT32 or AR_BFLOAT16: y, residual, s, x and
                              their gradients */
    int param_dtype;       /* the same choice for weights, gate and their gradients */
    int flags;             /* AR_NORM_* */
    float alpha;           /* scale of the residual; finite */
    float eps;             /* > 0 and finite; used with AR_NORM_* */
    size_t gate_rows;      /* 0: no gate; otherwise it divides rows, and row k
                              of the gate (gate_rows x cols, contiguous) holds for
                              rows / gate_rows consecutive rows: 1 = one gate for
                              all, one per sequence, rows = one per row */
    size_t ld_y, ld_residual, ld_s, ld_x;  /* row strides (ld_residual: also of dresidual) */
    size_t ld_ds, ld_dx, ld_dy;            /* backward only */
} ar_norm_desc;

/* Forward.  s may be y or residual, x may be y or residual (not both the
 * same).  Errors: AR_ERR_ARG (NULL or misaligned pointer, range, stride,
 * overlap, gate_rows that does not divide rows), AR_ERR_UNSUPPORTED (data
 * type), AR_ERR_HIP. */
int ar_residual_norm(const ar_norm_desc *desc, const void *y, const void *residual, const void *post_weight,
                     const void *gate, const void *pre_weight, void *s, void *x, void *stream);

/* Backward.  From y and s of the forward, ds (gradient of s from its later
 * uses; NULL = zero) and dx (gradient of x; NULL without AR_NORM_PRE):
 *     G         = ds + gradient of x with regard to s, times dx
 *     dresidual = alpha * G
 *     dgate     = sum over the gate row's rows of G * n
 *     dn        = G * gate
 *     dy        = gradient of n with regard to y, times dn
 *     dpost_weight = sum_t dn * y / rms(y),  dpre_weight = sum_t dx * s / rms(s)
 * The norms are taken of y and s again; nothing else is kept by the forward.
 * dpost_weight, dgate and dpre_weight may be NULL (not wanted), and must be
 * where what they belong to is absent from the forward: a gradient for a norm
 * without its flag, or for a gate with gate_rows 0, is AR_ERR_ARG.  A weight
 * that stands for ones (NULL) may have a gradient.  dy and dresidual may each
 * be y, s, ds or dx.  Workspace: partial sums of the parameter gradients. */
int ar_residual_norm_backward(const ar_norm_desc *desc, const void *y, const void *s, const void *ds, const void *dx,
                              const void *post_weight, const void *gate, const void *pre_weight, void *dy,
                              void *dresidual, void *dpost_weight, void *dgate, void *dpre_weight, void *workspace,
                              size_t workspace_bytes, void *stream);
size_t ar_residual_norm_backward_workspace(const ar_norm_desc *desc);

/* ---- gated feed-forward block ------------------------------------------- */

/* Activations: silu g / (1 + e^-g); gelu, the form with tanh,
 * g/2 (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))); relu max(g, 0). */
enum { AR_ACT_SILU = 0, AR_ACT_GELU = 1, AR_ACT_RELU = 2 };

/* With G = x Wg^T and U = x Wu^T (x: tokens x dim; weights: hidden x dim):
 *     h = act(G) * U
 * The block's way back from hidden to dim is a plain product and no part of it. */
typedef struct ar_ffn_desc {
    size_t tokens;         /* 0 is a valid no-op (backward: zero weight gradients) */
    size_t dim, hidden;    /* 1 .. 2^20 */
    int dtype;             /* AR_BFLOAT16 */
    int act;               /* AR_ACT_* */
    size_t ld_x, ld_w_gate, ld_w_up, ld_h;  /* row strides (ld_h: also of dh) */
    size_t ld_dx, ld_dw_gate, ld_dw_up;     /* backward only */
} ar_ffn_desc;

/* Forward, one kernel for both products, the activation and their product.
 * Operands that it cannot read where they lie, not 16-byte aligned or with a
 * dim or row stride that is no multiple of 8, are first copied into the
 * workspace.  Where tokens x hidden is small beside a long dim, the sums over
 * dim are taken in several runs, which a second kernel joins, from the
 * workspace.  Calls that need neither need no workspace; the size named for a
 * description is enough for any alignment of the pointers.  saved: NULL, or
 * 2 * tokens * hidden floats (16-byte aligned) that receive G and U for the
 * backward pass, in fp32.  Errors: AR_ERR_ARG, AR_ERR_UNSUPPORTED,
 * AR_ERR_SCRATCH, AR_ERR_HIP. */
int ar_gated_ffn(const ar_ffn_desc *desc, const void *x, const void *w_gate, const void *w_up, void *h, float *saved,
                 void *workspace, size_t workspace_bytes, void *stream);
size_t ar_gated_ffn_workspace(const ar_ffn_desc *desc);
/* What the call uses with these operands, which is enough for it: the copies that
 * their alignment asks for, and no others.  0: none, or a description that the call
 * refuses. */
size_t ar_gated_ffn_workspace_for(const ar_ffn_desc *desc, const void *x, const void *w_gate, const void *w_up);

/* Backward.  From `saved` of the forward and dh:
 *     dG = dh * U * act'(G),  dU = dh * act(G)
 *     dx = dG Wg + dU Wu,  dWg = dG^T x,  dWu = dU^T x
 * dG and dU are computed in fp32 and rounded to bf16 as operands of these
 * products (the matrix units' operand type).  dx, or both weight gradients,
 * may be NULL (not wanted). */
int ar_gated_ffn_backward(const ar_ffn_desc *desc, const void *dh, const void *x, const void *w_gate,
                          const void *w_up, const float *saved, void *dx, void *dw_gate, void *dw_up,
                          void *workspace, size_t workspace_bytes, void *stream);
size_t ar_gated_ffn_backward_workspace(const ar_ffn_desc *desc);

/* ---- orthogonalised updates --------------------------------------------- */

#define AR_ORTHO_MAX_STEPS 16

/* For each of `batch` matrices M (rows x cols):
 *     X = M / (|M|_F + eps)                       (of M^T where rows > cols)
 *     steps times, with the step's (a, b, c):
 *         A = X X^T,  B = b A + c A A,  X = a X + B X
 *     out = scale * X                              (its transpose there)
 * Each step takes every singular value v to a v + b v^3 + c v^5; with the
 * usual coefficients all come near 1 within five steps. */
typedef struct ar_ortho_desc {
    size_t batch;          /* matrices; 0 is a valid no-op */
    size_t rows, cols;     /* 1 .. 65536 */
    int dtype;             /* AR_FLOAT32 or AR_BFLOAT16: input and output */
    int steps;             /* 1 .. AR_ORTHO_MAX_STEPS */
    const float *coefs;    /* host memory: a, b, c of each step (3 * steps) */
    float eps;             /* 0 or more; finite */
    float scale;           /* finite */
    size_t ld_in, ld_out;  /* row strides */
    size_t stride_in, stride_out;  /* elements between matrices; 0 = rows * ld */
} ar_ortho_desc;

/* out may be `in`.  Operands of the products are held in fp16 planes with
 * power-of-two scales.  fp32, and bf16 with a short side of at most 256: two
 * planes (22 bits) and three products, about fp32's accuracy.  Other bf16:
 * products of one plane (11 bits), with the diagonals of A and B and the a X
 * term kept apart from it in fp32 and in two planes.  With the usual coefficients
 * and five steps that adds, before the result's rounding to bf16 (1.7e-3 of its
 * norm), 0.2e-3 to 0.9e-3 of its norm for a matrix of full rank, up to 1.8e-3 for
 * low rank and up to 2.8e-3 where rows hold few magnitudes; a caller who needs less
 * gives the matrix in fp32.  A matrix of zeros gives
 * zeros; one with an infinity or NaN gives NaN throughout.  AR_ERR_ARG also
 * for coefficients that are not finite or take singular values in [0, 1]
 * beyond 2^12 on the way.  Matrices of a batch may lie one after another or
 * side by side in shared rows, without sharing elements.  Workspace: the
 * planes. */
int ar_orthogonalize(const ar_ortho_desc *desc, const void *in, void *out, void *workspace, size_t workspace_bytes,
                     void *stream);
size_t ar_orthogonalize_workspace(const ar_ortho_desc *desc);

/* ---- attention ------------------------------------------------------------ */

/* Sequences lie one after another in the tokens: sequence i has the queries
 * starts_q[i] .. starts_q[i+1] - 1 and the keys starts_k[i] .. starts_k[i+1] - 1 (device
 * memory, sequences + 1 values each, not decreasing; both NULL for one sequence of all
 * tokens).  Its query i (of lq) sees its key j (of lk) where AR_ATTN_CAUSAL is not set or
 * j <= i + lk - lq: the last query sees every key.  Head h reads key head
 * h / (heads / kv_heads).  With z_ij = scale * q_i . k_j over the keys that i sees:
 *     lse_i = log sum_j e^z_ij,  o_i = sum_j e^(z_ij - lse_i) v_j
 * A query that sees no key has o = 0 and lse = minus infinity.  Tokens of no sequence
 * (before the first start, from the last one on) keep their o and lse, or get zeros
 * with AR_ATTN_CLEAR.  Values of `starts` outside the tokens are taken as the nearest
 * end of them; where they decrease, no output is defined, but nothing else is touched.
 * A sequence may have no queries: unused places between caches that have room to grow are
 * the keys of one such sequence each.  (They count in the mean length by which keys are
 * split into runs, which is best where sequences are alike.)
 * A key that a query does not see has no part in it but for one thing: in a value (v)
 * or, backward, a k, q or dout that is infinite or NaN, 0 times it is NaN, which can
 * reach rows of the same sequence within 256 tokens. */
enum { AR_ATTN_CAUSAL = 1, AR_ATTN_CLEAR = 2 };

/* Element d of head h of token t lies at t * ld + h * hs + d: ld_* strides between
 * tokens (0 = heads * hs), hs_* between heads (0 = dim).  Either a token's heads lie
 * within ld, or a head's tokens within hs; nothing overlaps. */
typedef struct ar_attention_desc {
    size_t sequences;             /* 0, or no tokens: a valid no-op, with AR_ATTN_CLEAR too; times heads at most 2^22 */
    size_t tokens_q, tokens_k;    /* times heads, or kv_heads, at most 2^30 */
    size_t heads, kv_heads, dim;  /* heads a multiple of kv_heads; dim 1 .. 128 (AR_ERR_UNSUPPORTED above) */
    int dtype;                    /* AR_BFLOAT16 */
    int flags;                    /* AR_ATTN_* */
    float scale;                  /* 2^-100 .. 2^100; 1 / sqrt(dim) as a rule */
    size_t ld_q, hs_q, ld_k, hs_k, ld_v, hs_v, ld_o, hs_o;
    size_t ld_dout, hs_dout, ld_dq, hs_dq, ld_dk, hs_dk, ld_dv, hs_dv;  /* backward only */
} ar_attention_desc;

/* Forward.  lse: NULL, or heads * tokens_q floats, a head's tokens after one another,
 * that the backward pass needs.  e^(z - m) is rounded to bf16 as an operand of the product with v (m: within
 * e^5.6 of the row's maximum); its sum is not.  Tensors that cannot be read where
 * they lie, not 16-byte aligned or with a dim or stride that is no multiple of 8, are
 * first copied into the workspace.  Where there are few rows the keys are taken in
 * several runs, which a second kernel joins, from the workspace.  Errors: AR_ERR_ARG,
 * AR_ERR_UNSUPPORTED, AR_ERR_SCRATCH, AR_ERR_HIP. */
int ar_attention(const ar_attention_desc *desc, const void *q, const void *k, const void *v, const int32_t *starts_q,
                 const int32_t *starts_k, void *o, float *lse, void *workspace, size_t workspace_bytes, void *stream);
size_t ar_attention_workspace(const ar_attention_desc *desc);
/* What the call uses with these tensors, which is enough for it (0: none, or refused). */
size_t ar_attention_workspace_for(const ar_attention_desc *desc, const void *q, const void *k, const void *v);

/* Backward.  From dout, o and lse of the forward, with p_ij = e^(z_ij - lse_i):
 *     delta_i = dout_i . o_i,  dz_ij = p_ij (dout_i . v_j - delta_i)
 *     dq_i = scale sum_j dz_ij k_j,  dk_j = scale sum_i dz_ij q_i,  dv_j = sum_i p_ij dout_i
 * dk and dv are summed over the heads that share them.  p and dz are rounded to bf16 as
 * operands of these products.  dq, or both dk and dv, may be NULL (not wanted). */
int ar_attention_backward(const ar_attention_desc *desc, const void *dout, const void *q, const void *k, const void *v,
                          const void *o, const float *lse, const int32_t *starts_q, const int32_t *starts_k, void *dq, void *dk,
                          void *dv, void *workspace, size_t workspace_bytes, void *stream);
size_t ar_attention_backward_workspace(const ar_attention_desc *desc);

/* ---- loss over a vocabulary ----------------------------------------------- */

/* Softmax cross entropy of z = x W^T, one row of W for each class, of each token t:
 *     lse_t = log sum_j e^z_tj,  loss_t = lse_t - z_t,target(t)
 * W is the whole vocabulary, or a rank's rows of it: the classes first .. first + rows - 1
 * of `classes`.  A token whose target is not one of 0 .. classes - 1, a negative one say,
 * has no loss (0) and no gradient, whatever its dloss holds; its row of x has to be finite
 * all the same where dW is wanted (0 times it is added there).  The logits are never in
 * memory. */
typedef struct ar_vocab_desc {
    size_t tokens;         /* 0 is a valid no-op (backward: zero weight gradient); at most
                              2^24, times rows 2^38 */
    size_t dim;            /* 1 .. 2^20 */
    size_t rows;           /* of W: 1 .. 2^26 */
    size_t first, classes; /* first + rows <= classes <= 2^40 */
    int dtype;             /* AR_BFLOAT16: x, W and their gradients */
    int target_bytes;      /* 4 or 8: signed whole numbers */
    size_t ld_x, ld_w, ld_dx, ld_dw;  /* row strides */
} ar_vocab_desc;

/* Forward, of the whole vocabulary (first 0, rows = classes): loss and lse, tokens
 * floats each.  x and W are copied into the workspace where they cannot be read where
 * they lie (not 16-byte aligned, dim or row stride no multiple of 8); the size named is
 * for these pointers.  Errors: AR_ERR_ARG, AR_ERR_UNSUPPORTED, AR_ERR_SCRATCH, AR_ERR_HIP. */
int ar_vocab_loss(const ar_vocab_desc *desc, const void *x, const void *w, const void *target, float *loss, float *lse,
                  void *workspace, size_t workspace_bytes, void *stream);
size_t ar_vocab_loss_workspace(const ar_vocab_desc *desc, const void *x, const void *w);

/* Forward of a rank's rows: part[0 .. tokens - 1] = log sum e^z over them, part[tokens ..]
 * the target's logit, 0 where the target is none of them.  Workspace as above. */
int ar_vocab_loss_part(const ar_vocab_desc *desc, const void *x, const void *w, const void *target, float *part,
                       void *workspace, size_t workspace_bytes, void *stream);
/* Joins the parts of `ranks` ranks (1 .. 65536), one after another, whose rows make up the
 * vocabulary.  Of the description, valid as a whole, tokens, classes and target_bytes
 * count. */
int ar_vocab_loss_join(const ar_vocab_desc *desc, size_t ranks, const float *parts, const void *target, float *loss, float *lse,
                       void *stream);

/* Backward.  From dloss (of token t at dloss[t * dloss_stride]; stride 0: one for all) and
 * lse of the whole vocabulary:
 *     dz_tj = (e^(z_tj - lse_t) - [j = target(t)]) dloss_t
 *     dx = dz W  (of a rank's rows: its part of the sum over the ranks),  dW = dz^T x
 * The logits are computed again.  dz is rounded to bf16 as an operand of these products
 * and kept for a piece of the rows at a time, at most 512 MiB or 1024 rows.  dx or dw may
 * be NULL (not wanted). */
int ar_vocab_loss_backward(const ar_vocab_desc *desc, const float *dloss, size_t dloss_stride, const void *x, const void *w,
                           const void *target, const float *lse, void *dx, void *dw, void *workspace,
                           size_t workspace_bytes, void *stream);
/* For a call with these pointers; dx, dw: whether the gradient is wanted. */
size_t ar_vocab_loss_backward_workspace(const ar_vocab_desc *desc, const void *x, const void *w, int dx, int dw);

#ifdef __cplusplus
}
#endif

#endif /* AR_OPS_H */
