/*
 * detonation_model.h — C ABI of the operators that a training step needs around its library matrix
 * products, next to the optimizer step of detonation.h (same library, same rules):
 *
 *   detonation_token_logprobs, .._backward        log probability of given tokens, entropy, the best
 *                                                 alternatives; gradient of the logits
 *   detonation_norm_residual, .._backward         x + scale * gate (.) norm(f), and the next block's
 *                                                 norm of the sum
 *   detonation_act8_encode, .._decode             activations in 8 bits
 *   detonation_glu_forward, .._backward           act(a) (.) b, saved in 8 bits, and its gradient out
 *                                                 of them
 *   detonation_act8_weight_grad                   a linear layer's weight gradient out of its input in
 *                                                 8 bits: what detonation_compress takes as gradient
 *
 * Common rules are those of detonation.h: data pointers are device pointers on the current device,
 * the structs that describe them are host memory, read before the call returns; nothing is
 * allocated, kept or synchronised; work is enqueued on `stream`; the return value is a deto_status;
 * every pointer is aligned to its element size.  Beyond them:
 *   - A matrix is a deto_rows: T rows of consecutive elements, `ld` elements from one row's start to
 *     the next one's (ld >= row length; any ld for an input of which T <= 1).  Rows need no alignment
 *     beyond the element's; rows that start at multiples of 16 bytes are read fastest.
 *   - Types are DETO_F32, DETO_BF16 and DETO_F16.  Sums, statistics and every intermediate value are
 *     fp32; a result is rounded once (to nearest even), where it is written.
 *   - Outputs must not overlap inputs or each other, except where an entry point says so.
 *   - `workspace` is scratch of at least as many bytes as the matching .._workspace function says,
 *     aligned to 16 bytes.  Its contents need not survive from call to call, and calls that may run at
 *     the same time need one each.  The functions return -1 for sizes that the call refuses.
 *   - T = 0 is allowed: no rows are written, and sums over rows come out as zeros.
 *   - Results do not depend on the order in which workgroups run: the same call on the same data
 *     gives the same bits.
 */
#ifndef DETONATION_MODEL_H
#define DETONATION_MODEL_H

#include <stdint.h>

#include "detonation.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows of a matrix; data == NULL or a NULL pointer to the struct: the matrix is absent. */
typedef struct {
    void* data;
    int64_t ld;       /* elements from row to row */
    int32_t dtype;    /* deto_dtype: F32, BF16 or F16 */
    int32_t reserved; /* 0 */
} deto_rows;

/*
 * A [T, D] matrix in 8 bits.  The 32 consecutive features 32 g ... 32 g + 31 of a row (fewer in the
 * last group) share an exponent:
 *     value = codes[t][d] * 2^(exps[t][d / 32] - 127)
 * codes are two's complement, -127 ... 127, and the exponent is the smallest (126 below zero at
 * least) at which the group's largest magnitude rounds to 127 or less; values are rounded to the
 * nearest code, ties to even.  The scale is a power of two, so values are exact in bf16 and fp32, and
 * encoding is exact arithmetic: every implementation of it gives the same bits.  exps == 255 marks a
 * group that held an infinity or a NaN: all of it decodes to NaN.  exps == 0 is never written and
 * decodes to zeros.
 */
typedef struct {
    int8_t* codes;    /* T rows of D */
    int64_t ld_codes; /* >= D */
    uint8_t* exps;    /* T rows of ceil(D / 32) */
    int64_t ld_exps;  /* >= ceil(D / 32) */
} deto_act8;

enum { DETO_ACT8_GROUP = 32 };

/* ---- log probabilities of given tokens ------------------------------------------------------
 *
 * Per row t of logits [T, V], with z = logit_scale * logits[t]:
 *     lse = log sum_v exp(z_v)          logp = z_y - lse,  y = targets[t]
 *     p_v = exp(z_v - lse)              entropy = -sum_v p_v log p_v      (0 log 0 = 0)
 *     top_idx, top_logp: the `top` tokens of largest logit in falling order, ties by rising index, and
 *     their log probabilities.  A NaN counts as the largest value.
 * A target outside [0, V) (-100, say) is not scored: logp = 0.  A row whose logits are all -infinity
 * has lse = logp = top_logp = -infinity and entropy = 0.  A NaN or +infinity in a row makes its lse,
 * logp and entropy NaN.
 *
 *   targets    device, [T] int32 or int64 (target_bytes 4 or 8)
 *   logp       device, [T] fp32;  lse, entropy: the same, or NULL
 *   top        0 ... 32, at most V; top_idx [T, top] int32, top_logp [T, top] fp32 (may be NULL)
 *   stats      device, [T, 2] fp32 or NULL: a row's largest logit and log sum_v exp(z_v - largest z),
 *              which the backward pass takes.  (lse is their sum: where logits are large, or all at a
 *              type's lowest value, the sum no longer tells them apart.)
 * logit_scale is above 0 and at most 2^127.  V is at most 2^31 - 1.
 */
int detonation_token_logprobs(int64_t T, int64_t V, const deto_rows* logits, float logit_scale,
                              const void* targets, int target_bytes, float* logp, float* lse,
                              float* entropy, int32_t top, int32_t* top_idx, float* top_logp,
                              float* stats, void* workspace, void* stream);

/*
 * Gradient of  sum_t g_logp[t] logp[t] + g_entropy[t] entropy[t]  with respect to the logits:
 *     dlogits_v = logit_scale * ( g_logp (1[v = y] - p_v) - g_entropy p_v (log p_v + entropy) )
 * A row whose target is not scored has no first term; a row of -infinities has a gradient of zeros.
 *
 *   stats, entropy   as detonation_token_logprobs wrote them (entropy only with g_entropy)
 *   g_logp, g_entropy  device, [T] fp32; either may be NULL (zeros), not both
 *   dlogits          [T, V] of the logits' type; may be the logits themselves (same data and ld)
 */
int detonation_token_logprobs_backward(int64_t T, int64_t V, const deto_rows* logits,
                                       float logit_scale, const void* targets, int target_bytes,
                                       const float* stats, const float* entropy,
                                       const float* g_logp, const float* g_entropy,
                                       const deto_rows* dlogits, void* stream);

int64_t detonation_token_logprobs_workspace(int64_t T, int64_t V, int32_t top);

/* ---- norms before and after a block, its gate and the residual ------------------------------
 *
 *     u = post(f)                               the norm after the block that computed f
 *     x_out = x + scale * gate (.) u            gate: one row for all, or one for rows_per_gate rows
 *     y = pre(x_out)                            the norm before the next block
 * RMS:   norm(v) = v / sqrt(mean(v^2) + eps) * w + b
 * LAYER: norm(v) = (v - mean(v)) / sqrt(var(v) + eps) * w + b
 * y is the norm of the sum before that is rounded to x_out's type.
 */
typedef enum { DETO_NORM_NONE = 0, DETO_NORM_RMS = 1, DETO_NORM_LAYER = 2 } deto_norm_kind;

typedef struct {
    int32_t pre, post;      /* deto_norm_kind */
    float eps_pre, eps_post; /* >= 0 */
    float scale;            /* of the branch */
    int32_t param_dtype;    /* of the weights, biases and the gate: F32, BF16 or F16 */
    int64_t rows_per_gate;  /* row t's gate is row t / rows_per_gate of `gate`; 0: row 0 for all */
    const void* w_pre;      /* device, [D]; NULL: ones */
    const void* b_pre;      /* device, [D]; NULL: zeros */
    const void* w_post;
    const void* b_post;
    const void* gate;       /* device, rows of D, ld_gate elements apart; NULL: ones */
    int64_t ld_gate;        /* >= D */
} deto_norm_residual;

/*
 *   x, x_out   [T, D] of one type; x_out may be x itself (same data and ld).  x_out may be absent if f is
 *   f          [T, D]; absent: x_out = x, no branch (cfg->post NONE, no gate)
 *   y          [T, D] of f's type (if f is absent: of x's, or of any where x is fp32); absent if cfg->pre is
 *              NONE
 *   y8         y in 8 bits, encoded from y before that is rounded; may be absent
 * Types: x is fp32 or of f's type.  D is at most 16384 (else DETO_ERR_UNSUPPORTED).  With cfg->pre other
 * than NONE at least one of y and y8 is there.
 */
int detonation_norm_residual(const deto_norm_residual* cfg, int64_t T, int64_t D,
                             const deto_rows* x, const deto_rows* f, const deto_rows* x_out,
                             const deto_rows* y, const deto_act8* y8, void* stream);

/* Sums over rows, device, fp32, written (not added to); NULL: not wanted. */
typedef struct {
    float *w_pre, *b_pre, *w_post, *b_post; /* [D] */
    float* gate;   /* [ceil(T / rows_per_gate), D] dense, or [D] if rows_per_gate is 0 */
} deto_norm_grads;

/*
 * Gradients, given those of y (dy) and of x_out through the residual stream (dx_out):
 *     G = dx_out + (d pre / d x_out)^T dy                    dx = G
 *     df = (d post / d f)^T (scale * gate (.) G)             gate, weights, biases: sums over rows
 * The norms' statistics are computed again from x_out and f as they are given.
 *
 *   dy       of y's type; absent if cfg->pre is NONE        dx_out   of x_out's type; absent: zeros
 *   dx       of x_out's type; may be dx_out itself          df       of f's type; absent iff f is
 *   (dy is of f's type.)  b_post of cfg is needed for the gate's gradient, b_pre is not.
 */
int detonation_norm_residual_backward(const deto_norm_residual* cfg, int64_t T, int64_t D,
                                      const deto_rows* x_out, const deto_rows* f,
                                      const deto_rows* dy, const deto_rows* dx_out,
                                      const deto_rows* dx, const deto_rows* df,
                                      const deto_norm_grads* grads, void* workspace, void* stream);

int64_t detonation_norm_residual_workspace(const deto_norm_residual* cfg, int64_t T, int64_t D);

/* ---- activations in 8 bits -------------------------------------------------------------------*/

int detonation_act8_encode(int64_t T, int64_t D, const deto_rows* x, const deto_act8* x8,
                           void* stream);

int detonation_act8_decode(int64_t T, int64_t D, const deto_act8* x8, const deto_rows* x,
                           void* stream);

/* GELU is x Phi(x) with the error function, GELU_TANH its approximation by a tanh. */
typedef enum { DETO_ACT_SILU = 0, DETO_ACT_GELU = 1, DETO_ACT_GELU_TANH = 2, DETO_ACT_RELU = 3 } deto_act;

/*
 * h = act(a) (.) b, or act(a) if b is absent; a8, b8: a and b in 8 bits (either may be absent).
 * a, b, h are [T, D] of one type; h may be a or b itself (same data and ld).
 */
int detonation_glu_forward(int act, int64_t T, int64_t D, const deto_rows* a, const deto_rows* b,
                           const deto_rows* h, const deto_act8* a8, const deto_act8* b8,
                           void* stream);

/*
 * With a and b decoded from a8 and b8:  da = dh (.) b (.) act'(a),  db = dh (.) act(a); relu'(0) = 0.
 * b8 and db are absent for act alone.  h8, if there, receives act(a) (.) b of the decoded values in 8
 * bits: the input of the next linear layer, whose weight gradient takes it.
 * dh, da, db are [T, D] of one type; da or db may be dh itself (same data and ld).
 */
int detonation_glu_backward(int act, int64_t T, int64_t D, const deto_rows* dh, const deto_act8* a8,
                            const deto_act8* b8, const deto_rows* da, const deto_rows* db,
                            const deto_act8* h8, void* stream);

/*
 * dw = [dw +] dy^T x :  dw[n][k] = sum_t dy[t][n] * x[t][k],  x decoded from x8 (exactly).
 *   dy   [T, N];  x8  [T, K];  dw  [N, K] of any of the three types
 *   accumulate  0: dw is written; 1: the product is added to what dw holds
 * T, N and K are at most 2^30, N * K at most 2^40.
 * Products are exact (fp32 and fp16 dy enter as sums of three or two bf16 numbers), sums are fp32.
 */
int detonation_act8_weight_grad(int64_t T, int64_t N, int64_t K, const deto_rows* dy,
                                const deto_act8* x8, const deto_rows* dw, int accumulate,
                                void* workspace, void* stream);

int64_t detonation_act8_weight_grad_workspace(int64_t T, int64_t N, int64_t K);

#ifdef __cplusplus
}
#endif
#endif /* DETONATION_MODEL_H */
