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

#ifdef __cplusplus
}
#endif

#endif /* AR_OPS_H */
