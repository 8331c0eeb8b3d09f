/*
 * cpdp_q8.h -- C ABI of the 8-bit activation path: the operators of a
 * transformer layer that keep activations as rows of 8-bit numbers, in the
 * forward pass and as checkpoints for the backward pass, on one AMD Instinct
 * MI355X (gfx950).
 *
 * W replicas on one GPU (cpdp.h) keep W sets of activations there; these
 * operators hold them in one byte an element and train from them: the
 * gradients they return go into the replicas' gradient rows.
 *
 * 8-bit rows.  A row x[0..D) is held as int8 numbers q[0..D) and one fp32
 * scale s, and stands for the values s * q:
 *   s    = the smallest bfloat16 number >= 2^-126 with 127 * s >= max |x|
 *   q[d] = x[d] / s rounded to the nearest whole number, ties to even
 * A row that holds an infinity or a NaN gets s = NaN and q = 0, so everything
 * computed from it is NaN.  A scale has 8 significant bits, so s * q has 15: it
 * is exact in fp32 and in the sum of two bfloat16 numbers.  The readers take
 * any fp32 scales and any q in [-128, 127].
 *
 * Layout.  A matrix argument of R rows and C columns has its element (r, c) at
 * base[r * ld + c].  Elements past a row's end are never written, and not used:
 * the gradients of a product, and of the loss, read their operands in whole 16-byte
 * pieces, up to 15 bytes past a row's end, the other calls read nothing there.
 * Every matrix starts on a 16-byte boundary and ld * sizeof(element) is a
 * multiple of 16 (CPDP_ERR_MISALIGNED); ld >= C.  Vectors (scales, w, dw) are
 * contiguous; w and dw start on a 16-byte boundary, scales and rstd on a 4-byte
 * one.  Storage types are CPDP_F32 or CPDP_BF16 of cpdp.h; arithmetic is fp32
 * (sums of 8-bit products: 32-bit integers), each value rounded to nearest-even
 * once, when it is written; but the gradients of a product may round what they sum,
 * as it says there.
 *
 * All pointers are device pointers owned by the caller; the library never
 * allocates, frees or keeps them.  Every argument is checked on the host before
 * any GPU work: a count below 0 or an inner size out of range is
 * CPDP_ERR_INVALID_ARG, a missing pointer CPDP_ERR_NULL, an unknown storage
 * type CPDP_ERR_DTYPE; the ranges of different arguments must not overlap
 * (CPDP_ERR_OVERLAP) but where it says so.  Row strides are at most 2^28 elements;
 * those of the matrices that a product or its gradients read at most 2^23 - 16 (dy:
 * 2^22 - 8), and a gradient sums over at most 2^22 - 72 values (CPDP_ERR_TOO_LARGE).
 * Calls return once their kernels are enqueued on `stream` (a hipStream_t, NULL for
 * the null stream); they copy, clear and allocate nothing through the runtime, so
 * they may be captured in a graph.  Zero rows are a valid no-op (a gradient summed
 * over zero rows is 0).  Results are bitwise reproducible: sums run in an order that
 * is fixed by the sizes.
 *
 * Workspaces.  Calls with a `workspace` need the bytes that the matching
 * *_workspace function returns for the same sizes (0: it may be NULL), on a
 * 16-byte boundary; less is CPDP_ERR_INVALID_ARG (also from calls of these sizes
 * whose storage types let a kernel do without).  The content is not kept from one
 * call to the next; two calls that may run at the same time need two.
 */
#ifndef CPDP_Q8_H
#define CPDP_Q8_H

#include <stdint.h>

#include "cpdp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest inner size of a product: 128 * 128 * 131071 < 2^31, so a 32-bit sum
 * of 8-bit products cannot overflow. */
#define CPDP_Q8_MAX_K 131071

/*
 * Hold the rows of x [T x D] in 8 bits: q [T x D], scale [T].
 * y [T x D] (y_dt), or NULL: also the values s * q.
 */
int cpdp_q8_rows(const void* x, int64_t ldx, int x_dt, int64_t T, int64_t D, int8_t* q,
                 int64_t ldq, float* scale, void* y, int64_t ldy, int y_dt, void* stream);

/* Read 8-bit rows back: y [T x D] (y_dt) <- scale * q. */
int cpdp_q8_values(const int8_t* q, int64_t ldq, const float* scale, int64_t T, int64_t D,
                   void* y, int64_t ldy, int y_dt, void* stream);

/*
 * Root-mean-square norm with the residual's addition, its output in 8 bits.
 * For every row t of x [T x D]:
 *   h    = x + residual                (stored, in act_dt; h = x without one)
 *   rstd = 1 / sqrt(mean(h^2) + eps)
 *   v    = h * w * rstd
 *   q, scale <- v as an 8-bit row;  y <- s * q (y_dt), if y is not NULL
 * x, residual, h in act_dt; w [D] in w_dt; rstd [T] fp32 or NULL.  residual and
 * h are both given or both NULL; h may be the same rows as x or as residual.
 * eps >= 0.  The sum of squares is fp32, as the other arithmetic: one that passes
 * fp32's largest number (|h| about 2^64) makes rstd and the row 0.
 */
int cpdp_q8_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, int act_dt,
                 const void* w, int w_dt, float eps, int64_t T, int64_t D, void* h, int64_t ldh,
                 int8_t* q, int64_t ldq, float* scale, float* rstd, void* y, int64_t ldy,
                 int y_dt, void* stream);

/*
 * Backward pass of cpdp_q8_norm, with dy [T x D] the gradient of v (the
 * rounding to 8 bits passes it on unchanged), and with n = h * rstd:
 *   dx = rstd * (dy * w - n * mean(dy * w * n)) + dres
 *   dw = sum over rows of dy * n
 * dres [T x D] is the gradient that reaches h by the residual path, or NULL; dx
 * is the gradient of x and of the residual.  dy, h, dres, dx in act_dt; dw [D]
 * in dw_dt.
 */
int64_t cpdp_q8_norm_bwd_workspace(int64_t T, int64_t D);
int cpdp_q8_norm_bwd(const void* dy, int64_t lddy, const void* h, int64_t ldh, const void* dres,
                     int64_t lddres, int act_dt, const void* w, int w_dt, const float* rstd,
                     int64_t T, int64_t D, void* dx, int64_t lddx, void* dw, int dw_dt,
                     void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Product of 8-bit rows with 8-bit weights:
 *   y[m, n] = a_scale[m] * b_scale[n] * sum_k a[m, k] * b[n, k]
 * a [M x K] with a scale for each row (token), b [N x K] with a scale for each
 * row (output channel), y [M x N] in y_dt.  The sum is exact (32-bit integers);
 * 1 <= K <= CPDP_Q8_MAX_K.
 */
int64_t cpdp_q8_matmul_workspace(int64_t M, int64_t N, int64_t K);
int cpdp_q8_matmul(const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b,
                   int64_t ldb, const float* b_scale, int64_t M, int64_t N, int64_t K, void* y,
                   int64_t ldy, int y_dt, void* workspace, int64_t workspace_bytes, void* stream);

/* Activations of a layer's inner product.
 *   CPDP_ACT_GELU    a = g * Phi(g), Phi the normal distribution function
 *   CPDP_ACT_SWIGLU  a = g * sigmoid(g) * u */
typedef enum { CPDP_ACT_GELU = 0, CPDP_ACT_SWIGLU = 1 } cpdp_act_kind;

/*
 * Activation with 8-bit output and 8-bit checkpoint:
 *   q, scale   <- a as 8-bit rows;  y <- their values (y_dt), if not NULL
 *   cg, cg_scale <- g as 8-bit rows; cu, cu_scale <- u likewise (SWIGLU)
 * g, u [T x F] in act_dt with the one stride ldg (u is ignored for GELU).  The
 * checkpoint may be left out (cg, cg_scale, cu and cu_scale all NULL); its rows
 * have the one stride ldc.
 */
int cpdp_q8_act(int kind, const void* g, const void* u, int64_t ldg, int act_dt, int64_t T,
                int64_t F, int8_t* q, int64_t ldq, float* scale, void* y, int64_t ldy, int y_dt,
                int8_t* cg, float* cg_scale, int8_t* cu, float* cu_scale, int64_t ldc,
                void* stream);

/*
 * Backward pass of the activation from its checkpoint, with da [T x F] the
 * gradient of a, G = cg_scale * cg and U = cu_scale * cu:
 *   GELU    dg = da * (Phi(G) + G * phi(G)), phi the normal density
 *   SWIGLU  dg = da * U * s * (1 + G * (1 - s)), du = da * G * s, s = sigmoid(G)
 * da, dg, du in act_dt; dg and du have the one stride lddg.
 */
int cpdp_q8_act_bwd(int kind, const void* da, int64_t ldda, int act_dt, const int8_t* cg,
                    const float* cg_scale, const int8_t* cu, const float* cu_scale, int64_t ldc,
                    int64_t T, int64_t F, void* dg, void* du, int64_t lddg, void* stream);

/*
 * The two gradients of y = a * b^T from the 8-bit operands, with dy [T x N] the
 * gradient of y in dy_dt:
 *   cpdp_q8_grad_input   dx[t, k] = sum_n dy[t, n] * b_scale[n] * b[n, k]
 *   cpdp_q8_grad_weight  dw[n, k] = sum_t dy[t, n] * a_scale[t] * a[t, k]
 * dx [T x K], dw [N x K] in out_dt.  Products run on the bfloat16 matrix cores
 * with fp32 sums; what they sum is held in bfloat16 numbers:
 *   fp32 result, or a sum of at most 64 values
 *     fp32 dy   three for each scaled value of dy: all of its 24 bits
 *     bf16 dy   two: all of its bits where the scale has 8 significant ones, as those
 *               that this library writes; with other scales within 2^-16 of it
 *   bf16 result of a sum of more than 64 values
 *     one, for each scaled value of dy (fp32 dy) or of the 8-bit operand (bf16 dy):
 *     within 2^-8 of it, as one rounding of the result is.  These errors are
 *     independent and average out over a sum, but not against one that cancels: whoever
 *     needs that takes an fp32 result.
 */
int64_t cpdp_q8_grad_input_workspace(int64_t T, int64_t N, int64_t K, int dy_dt, int out_dt);
int cpdp_q8_grad_input(const void* dy, int64_t lddy, int dy_dt, const int8_t* b, int64_t ldb,
                       const float* b_scale, int64_t T, int64_t N, int64_t K, void* dx,
                       int64_t lddx, int out_dt, void* workspace, int64_t workspace_bytes,
                       void* stream);
int64_t cpdp_q8_grad_weight_workspace(int64_t T, int64_t N, int64_t K, int dy_dt, int out_dt);
int cpdp_q8_grad_weight(const void* dy, int64_t lddy, int dy_dt, const int8_t* a, int64_t lda,
                        const float* a_scale, int64_t T, int64_t N, int64_t K, void* dw,
                        int64_t lddw, int out_dt, void* workspace, int64_t workspace_bytes,
                        void* stream);

/*
 * Softmax cross entropy over V classes, of the logits
 *   z[t, v] = x_scale[t] * w_scale[v] * sum_k x[t, k] * w[v, k]
 * which are not kept from one pass to the next: the forward pass uses them a tile at a time
 * and holds none, the gradients make them again and hold what they are of a piece of the
 * classes, up to 2^27 of them (with fewer logits that is all), laid out in 2 to 8 bytes a
 * logit, and the piece's weights in 2 or 4 bytes each, up to 512 MB.
 *   cpdp_q8_xent      lse[t]  = log sum_v exp z[t, v]
 *                     loss[t] = lse[t] - z[t, target[t]]
 *   cpdp_q8_xent_bwd  d[t, v] = g[t] * (exp(z[t, v] - lse[t]) - (v == target[t] ? 1 : 0))
 *                     dx[t, k] = sum_v d[t, v] * w_scale[v] * w[v, k]
 *                     dw[v, k] = sum_t d[t, v] * x_scale[t] * x[t, k]
 * x [T x K] with a scale for each row (token), w [V x K] with a scale for each row
 * (class); target [T] int64 on an 8-byte boundary; loss, lse and g [T] fp32, lse as
 * cpdp_q8_xent left it, g the gradient that reaches loss.  A token whose target is
 * negative does not count: its loss and its row of dx are 0 and it adds nothing to dw,
 * whatever its x and g hold.  One whose target is V or more has a NaN for its loss, its
 * row of dx and all of dw.  dx [T x K] in dx_dt, dw [V x K] in dw_dt; either may be NULL
 * and is then not computed.
 * The _miss calls are the same, and hand on, [T] fp32,
 *   miss[t] = 1 - exp(-loss[t])   what the target's probability lacks of 1
 * (0 for a token that does not count, NaN for a target of V or more), from which
 * cpdp_q8_xent_miss_bwd takes -g * miss for the target's d.  cpdp_q8_xent_bwd takes
 * g * (exp(z - lse) - 1) there, of the lse that was rounded to fp32: it is off by up to |lse| *
 * 2^-24 |g|, all that there is of it for a token whose loss is below |lse| * 2^-24.
 * 0 <= T <= CPDP_Q8_MAX_T, 1 <= V <= 2^31 - 9, 1 <= K <= CPDP_Q8_MAX_K.  Logits are exact
 * sums, scaled in fp32, and everything that is taken of them is fp32; a loss is the sum of
 * (the largest logit - the target's) and the logarithm, so its error does not grow with lse,
 * while that of a probability, relative, does: |lse| * 2^-24.  The gradients'
 * products have fp32 sums.  What they sum, with p the factor of g in d:
 *   dx   p[t, v] * w_scale[v], each sum times g[t]
 *   dw   p[t, v] * g[t] * x_scale[t]
 * is held in two fp16 numbers for an fp32 result: 22 bits, but with an error of up to
 * 2^-51 of the largest |w_scale|, or of the largest |g * x_scale| of the tokens that count;
 * in one for a bf16 result: 11 bits, and 2^-39 of the largest.  (Up to 64 tokens: in
 * bfloat16 numbers, as the gradients of a product from fp32 dy.)
 * The gradients' workspace, whatever V is: less than 512 MiB up to 64 tokens, and else less than
 * max(1 GiB, 2048 T) + 640 MiB + 12 (T + 64) (K + 64) bytes.
 */
#define CPDP_Q8_MAX_T 2097088 /* 2^21 - 64: rows of sums that a tile can address */

int64_t cpdp_q8_xent_workspace(int64_t T, int64_t V, int64_t K);
int cpdp_q8_xent(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w, int64_t ldw,
                 const float* w_scale, const int64_t* target, int64_t T, int64_t V, int64_t K,
                 float* loss, float* lse, void* workspace, int64_t workspace_bytes, void* stream);
int cpdp_q8_xent_miss(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w,
                      int64_t ldw, const float* w_scale, const int64_t* target, int64_t T,
                      int64_t V, int64_t K, float* loss, float* lse, float* miss, void* workspace,
                      int64_t workspace_bytes, void* stream);
int64_t cpdp_q8_xent_bwd_workspace(int64_t T, int64_t V, int64_t K, int dx_dt, int dw_dt);
int cpdp_q8_xent_bwd(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w,
                     int64_t ldw, const float* w_scale, const int64_t* target, const float* lse,
                     const float* g, int64_t T, int64_t V, int64_t K, void* dx, int64_t lddx,
                     int dx_dt, void* dw, int64_t lddw, int dw_dt, void* workspace,
                     int64_t workspace_bytes, void* stream);
int cpdp_q8_xent_miss_bwd(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w,
                          int64_t ldw, const float* w_scale, const int64_t* target,
                          const float* lse, const float* miss, const float* g, int64_t T,
                          int64_t V, int64_t K, void* dx, int64_t lddx, int dx_dt, void* dw,
                          int64_t lddw, int dw_dt, void* workspace, int64_t workspace_bytes,
                          void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CPDP_Q8_H */
