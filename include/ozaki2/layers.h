/*
 * layers.h -- products of the feed-forward layers of language models on the
 * CDNA4 (gfx950) matrix cores: a dense layer and a layer of experts, each with
 * bias, activation and residual in the product's epilogue, the order of tokens
 * by expert, and the gradients of all of them.  Part of libozaki2.so; status
 * codes are those of ozaki2.h.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Layout: row-major, one token per row; a leading dimension is the distance of
 * two rows in elements (at least the row's length), any value and any
 * element-aligned pointer.  (Rows that start on 16-byte boundaries are read
 * by direct loads into LDS; others work alike, more slowly.)
 * Types: x, w, bias, residual, y, z and their gradients have one type, `dtype`.
 * Products are summed in 32 bits by the matrix cores, the epilogue is evaluated
 * in 32 bits, and each result is rounded once, to nearest even, when stored.
 * All data pointers are DEVICE pointers owned by the caller; the library keeps
 * none of them after a call.  `stream` is a hipStream_t passed as void*; work
 * is enqueued asynchronously, nothing synchronises, nothing is allocated, and
 * calls may be captured into a graph.
 * Validation happens before any launch: on an error nothing is written
 * (OZ2_E_INVALID for sizes, types, leading dimensions, null pointers and
 * outputs or a workspace that overlap an input or another output; OZ2_E_WORKSPACE for a
 * workspace that is smaller than the _workspace_bytes function says or not
 * 256-byte aligned).  Matrices may lie side by side in the rows of one buffer, and stacks
 * of one stride in between each other.  A workspace of 0 bytes may be null.  Sizes of zero are
 * allowed: an empty sum is zero.  Limits: rows and token-expert pairs up to 2^30,
 * in and out up to 2^21, and matrices (all groups' weights together) below 2^40
 * elements.
 * Results do not depend on timing: no atomics decide the order of a sum.
 * Infinities and NaN follow from the formulas in 32-bit arithmetic.
 */
#ifndef OZAKI2_LAYERS_H
#define OZAKI2_LAYERS_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* dtype */
enum { OZ2_F32 = 0, OZ2_F16 = 1, OZ2_BF16 = 2 };

/* activation f: none x; relu max(x, 0); gelu x Phi(x); gelu_tanh its tanh
 * form 0.5 x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))); silu x / (1 + e^-x) */
enum { OZ2_ACT_NONE = 0, OZ2_ACT_RELU = 1, OZ2_ACT_GELU = 2, OZ2_ACT_GELU_TANH = 3, OZ2_ACT_SILU = 4 };

#define OZ2_MAX_EXPERTS 1024   /* groups of the grouped products, experts of the sort */
#define OZ2_MAX_TOPK 64        /* experts per token */

/* Y = f(X W^T + bias) + residual for X (rows x in), W (out x in), bias (out),
 * residual and Y (rows x out).  gated != 0: W has 2 out rows and bias 2 out
 * entries, the gates first, and Y = f(Z_gate) * Z_up + residual, with
 * Z = X W^T + bias = [Z_gate Z_up].
 * bias, residual and z may be null.  z receives Z (rows x out, gated 2 out),
 * rounded, which ozaki2_linear_backward takes; Y is computed from the unrounded
 * Z.  residual may be Y itself (same pointer and leading dimension). */
int ozaki2_linear(int dtype, int activation, int gated, int rows, int out, int in, const void* x,
                  long long ldx, const void* w, long long ldw, const void* bias,
                  const void* residual, long long ldr, void* y, long long ldy, void* z,
                  long long ldz, void* workspace, size_t ws_bytes, void* stream);
size_t ozaki2_linear_workspace_bytes(int dtype, int gated, int rows, int out, int in);

/* The gradients of ozaki2_linear from dY (rows x out), with Z as it stored it
 * (null where the activation is none and gated is 0):
 *   dZ = dY f'(Z), gated [dY Z_up f'(Z_gate), dY f(Z_gate)];
 *   dX = dZ W, dW = dZ^T X, dbias = the column sums of dZ.
 * The residual's gradient is dY.  Each of dx, dw and dbias may be null (not
 * wanted); x is read for dw alone and w for dx alone, and may be null without
 * them.  dZ is rounded to dtype before the products (the matrix cores take
 * their operands in that type; beyond 65504 fp16 is infinite), but not before its column
 * sums.  OZ2_F32 keeps dZ in 32 bits. */
int ozaki2_linear_backward(int dtype, int activation, int gated, int rows, int out, int in,
                           const void* dy, long long lddy, const void* x, long long ldx,
                           const void* w, long long ldw, const void* z, long long ldz, void* dx,
                           long long lddx, void* dw, long long lddw, void* dbias, void* workspace,
                           size_t ws_bytes, void* stream);
size_t ozaki2_linear_backward_workspace_bytes(int dtype, int activation, int gated, int rows,
                                              int out, int in);

/* ozaki2_linear (without residual) for `groups` layers at once: rows
 * offsets[g] .. offsets[g+1] - 1 of X and Y belong to layer g, whose weights
 * start at w + g stride_w and bias at bias + g stride_bias (elements).
 * offsets is DEVICE memory, int [groups + 1], not read by the host: ascending from 0
 * and at most rows (other values are clamped to [0, rows] and, where groups are
 * added up, to ascending order, so that no access leaves the arrays or the
 * workspace; the results of such a call are undefined).  Rows of X from
 * offsets[groups] on affect nothing, whatever they hold, and those of y and z are
 * written as zeros.  1 <= groups <= OZ2_MAX_EXPERTS. */
int ozaki2_grouped_linear(int dtype, int activation, int gated, int rows, int groups, int out,
                          int in, const int* offsets, const void* x, long long ldx, const void* w,
                          long long ldw, long long stride_w, const void* bias,
                          long long stride_bias, void* y, long long ldy, void* z, long long ldz,
                          void* workspace, size_t ws_bytes, void* stream);
size_t ozaki2_grouped_linear_workspace_bytes(int dtype, int gated, int rows, int groups, int out,
                                             int in);

/* The gradients of ozaki2_grouped_linear: dx as there (rows from
 * offsets[groups] on are zeros), dw (lddw, stride_dw) and dbias (stride_dbias)
 * per group, zeros for a group without rows. */
int ozaki2_grouped_linear_backward(int dtype, int activation, int gated, int rows, int groups,
                                   int out, int in, const int* offsets, const void* dy,
                                   long long lddy, const void* x, long long ldx, const void* w,
                                   long long ldw, long long stride_w, const void* z, long long ldz,
                                   void* dx, long long lddx, void* dw, long long lddw,
                                   long long stride_dw, void* dbias, long long stride_dbias,
                                   void* workspace, size_t ws_bytes, void* stream);
size_t ozaki2_grouped_linear_backward_workspace_bytes(int dtype, int activation, int gated,
                                                      int rows, int groups, int out, int in);

/* Token-expert pairs in the order of their experts.  experts [tokens][top_k]
 * (int, or long long with wide_ids != 0; ldexperts elements between tokens)
 * names the experts of each token; a value outside [0, num_experts) drops the pair
 * (an expert over its capacity, padding).  Pair p = t top_k + j.
 *   offsets [num_experts + 1]: expert e has places offsets[e] .. offsets[e+1] - 1,
 *   rows [tokens top_k]: the pair at each place; within an expert ascending
 *     (a stable sort); dropped pairs follow from offsets[num_experts] on,
 *   slots [tokens][top_k]: the place of each pair (the inverse of rows).
 * All three are written in full. */
int ozaki2_expert_sort(int tokens, int top_k, int num_experts, const void* experts, int wide_ids,
                       long long ldexperts, int* offsets, int* rows, int* slots, void* workspace,
                       size_t ws_bytes, void* stream);
size_t ozaki2_expert_sort_workspace_bytes(int tokens, int top_k, int num_experts);

/* XS[slots[t][j]] = X[t] (weights null) or weights[t][j] X[t]: the tokens' rows
 * at their places, zeros at the places of dropped pairs.  XS has tokens * top_k
 * rows; `kept` points at offsets[num_experts] of the sort (DEVICE memory).
 * weights is float [tokens][top_k], whatever dtype.  A place outside
 * [0, tokens top_k) in slots is ignored. */
int ozaki2_expert_gather(int dtype, int tokens, int top_k, int width, const void* x, long long ldx,
                         const int* slots, const int* kept, const float* weights, void* xs,
                         long long ldxs, void* stream);

/* Y[t] = residual[t] + sum over j ascending of weights[t][j] YS[slots[t][j]],
 * dropped pairs left out (their rows of YS are not read); weights null: 1;
 * residual null: 0; residual may be Y itself.  With residual null it is the gradient
 * of ozaki2_expert_gather with the same weights. */
int ozaki2_expert_combine(int dtype, int tokens, int top_k, int width, const void* ys,
                          long long ldys, const int* slots, const int* kept, const float* weights,
                          const void* residual, long long ldr, void* y, long long ldy,
                          void* stream);

/* The gradients of ozaki2_expert_combine from dY: dys[slots[t][j]] =
 * weights[t][j] dY[t] (zeros for dropped pairs), and dweights[t][j] =
 * <dY[t], YS[slots[t][j]]> (float; 0 for dropped pairs).  weights must be given;
 * dys or dweights may be null (not wanted); ys is read for dweights alone.
 * dweights from X as dy and dXS as ys is the gradient of ozaki2_expert_gather's weights. */
int ozaki2_expert_combine_backward(int dtype, int tokens, int top_k, int width, const void* dy,
                                   long long lddy, const void* ys, long long ldys,
                                   const int* slots, const int* kept, const float* weights,
                                   void* dys, long long lddys, float* dweights, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* OZAKI2_LAYERS_H */
