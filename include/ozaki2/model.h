/*
 * model.h -- what stands before and behind the layers of layers.h in a language
 * model, on CDNA4 (gfx950): the router that gives every token its experts and their
 * weights, layer norm, and the cross entropy over a vocabulary whose logits are never
 * kept; each with its gradients.  Part of libozaki2.so; types (OZ2_F32, ..), limits and
 * status codes are those of layers.h and ozaki2.h.
 *
 * The conventions of layers.h hold: row-major, one token per row; leading dimensions in
 * elements, any element-aligned pointer; DEVICE pointers that the caller owns; work is
 * enqueued on `stream`, nothing synchronises or is allocated, calls may be captured.  A
 * workspace belongs to one call at a time: calls, or replays, that can run at once need one each.
 * Validation happens before any launch: OZ2_E_INVALID for sizes, types, leading dimensions, null pointers
 * and outputs or a workspace that overlap an input or another output, OZ2_E_WORKSPACE for a workspace
 * smaller than the _workspace_bytes function says or not 256-byte aligned.  Sums,
 * statistics and exponentials are in 32 bits, each result is rounded once when stored, and
 * results do not depend on timing.  Infinities and NaN follow from the formulas.
 */
#ifndef OZAKI2_MODEL_H
#define OZAKI2_MODEL_H

#include "layers.h"

#ifdef __cplusplus
extern "C" {
#endif

/* score s of an expert: softmax over all experts, or 1 / (1 + e^-logit) of each */
enum { OZ2_SCORE_SOFTMAX = 0, OZ2_SCORE_SIGMOID = 1 };

/* The experts of every token from its logits (tokens x num_experts, of type dtype).
 * An expert's value is c = s + bias (bias null: s); the bias (float [num_experts]) decides the choice
 * and does not enter the weights.  groups > 1: the experts are `groups` ranges of
 * num_experts / groups; a group's value is the sum of its group_best (1 or 2) largest c, and only
 * experts of the top_groups largest groups can be chosen.
 *   ids [tokens][top_k]: the experts of largest c, descending; of equal ones the lower
 *     index comes first, among groups too.  c is compared as in 64 bits; without a bias, unless
 *     group_best 2 compares groups by sums, by the logits, whose order it has: so also
 *     where two scores are one number in 64 bits (sigmoid: logits beyond 37).
 *   weights [tokens][top_k]: scale s, or with renormalize scale s / (sum of the chosen s),
 *     which is formed from logarithms: scores too small for 32 bits still have weights.
 * An expert whose logit or bias is -infinity is out: it is never chosen, in groups too.  (Masks
 * are better -infinity than a large finite bias: what 32-bit scores may be off grows with the
 * largest |c|, and beside -1e9 all of a token's are formed in 64.)
 * Where none is left (fewer experts than top_k; a padding row of -infinity) the id is -1,
 * which ozaki2_expert_sort drops, and the weight 0.  A NaN is larger than every number:
 * it is chosen, and shows in the weights; with softmax a NaN or +infinity makes all of the
 * token's weights NaN.
 * 1 <= num_experts <= OZ2_MAX_EXPERTS, groups divides num_experts, top_k at most
 * OZ2_MAX_TOPK and the experts of top_groups groups. */
int ozaki2_expert_route(int dtype, int tokens, int num_experts, int top_k, const void* logits,
                        long long ldl, const float* bias, int score, int groups, int top_groups,
                        int group_best, int renormalize, float scale, int* ids, float* weights,
                        void* stream);

/* The gradient of the weights at the logits: dlogits (tokens x num_experts, type dtype) from
 * dweights and the ids that ozaki2_expert_route gave, g = scale dweights:
 *   softmax: s (G - sum of s g over the choices), G the expert's g, 0 where not chosen;
 *   softmax, renormalize: p (g - sum of p g) at the chosen ones, p their share; else 0;
 *   sigmoid: g s (1 - s); sigmoid, renormalize: p (1 - s) (g - sum of p g).
 * Choices outside [0, num_experts) take no part (their dweights are not read as
 * numbers); an expert named twice by a token gets both gradients.  The bias has none. */
int ozaki2_expert_route_backward(int dtype, int tokens, int num_experts, int top_k,
                                 const float* dweights, const void* logits, long long ldl,
                                 const int* ids, int score, int renormalize, float scale,
                                 void* dlogits, long long lddl, void* stream);

/* Y = (X - mean) rstd weight + bias for X and Y (rows x width), mean and variance of each
 * row (the variance about the mean, over width), rstd = 1 / sqrt(variance + eps); weight and bias
 * (width, type dtype) may be null.  stats (float [rows][2], may be null) receives mean and
 * rstd.  Y may be X itself (same pointer and leading dimension).  width 0: nothing is
 * written, stats neither. */
int ozaki2_layer_norm(int dtype, int rows, int width, const void* x, long long ldx,
                      const void* weight, const void* bias, float eps, void* y, long long ldy,
                      float* stats, void* stream);

/* The gradients of ozaki2_layer_norm from dY and the stats it stored, h = (X - mean) rstd,
 * g = dY weight:
 *   dX = rstd (g - mean of g - h mean of (g h)) + residual (what flows past the norm; may
 *   be null, or dX itself), dweight = column sums of dY h, dbias = column sums of dY.
 * dx, dweight and dbias may be null (not wanted); x and stats are needed for dx and dweight. */
int ozaki2_layer_norm_backward(int dtype, int rows, int width, const void* dy, long long lddy,
                               const void* x, long long ldx, const float* stats,
                               const void* weight, const void* residual, long long ldr, void* dx,
                               long long lddx, void* dweight, void* dbias, void* workspace,
                               size_t ws_bytes, void* stream);
size_t ozaki2_layer_norm_backward_workspace_bytes(int dtype, int rows, int width);

/* The cross entropy of tokens X (rows x in) over a vocabulary W (vocab x in), the logits
 * Z = X W^T summed and kept in 32 bits and never stored:
 *   lse [rows] = log of the sum of e^Z over the vocabulary,
 *   loss [rows] = lse - Z[target], 0 where the target is outside [0, vocab) (a token that
 *   does not count).
 * targets [rows]: int, or long long with wide_targets != 0.  loss and lse are float. */
int ozaki2_linear_cross_entropy(int dtype, int rows, int vocab, int in, const void* x,
                                long long ldx, const void* w, long long ldw, const void* targets,
                                int wide_targets, float* loss, float* lse, void* workspace,
                                size_t ws_bytes, void* stream);
size_t ozaki2_linear_cross_entropy_workspace_bytes(int dtype, int rows, int vocab, int in);

/* The gradients from dloss (float [rows]) and the forward call's lse:
 *   dZ = (e^(Z - lse) - [target]) dloss, dX = dZ W, dW = dZ^T X.
 * The logits are computed again, a piece of the vocabulary at a time; dZ is rounded to dtype for
 * the products (fp16: times a power of two that keeps the largest finite dloss near 2^14, taken
 * back in 32 bits; of up to 64 rows in 16 bits what the rounding leaves is added, rounded in turn),
 * and the pieces' shares of dX are added up in 32 bits.  A caller that needs dZ in 32 bits for
 * more rows passes X and W in OZ2_F32.  Tokens that do not
 * count have a zero row of dX and no part in dW, whatever their rows of X, lse and dloss hold.
 * dx or dw may be null (not wanted). */
int ozaki2_linear_cross_entropy_backward(int dtype, int rows, int vocab, int in,
                                         const float* dloss, const void* x, long long ldx,
                                         const void* w, long long ldw, const void* targets,
                                         int wide_targets, const float* lse, void* dx,
                                         long long lddx, void* dw, long long lddw,
                                         void* workspace, size_t ws_bytes, void* stream);
size_t ozaki2_linear_cross_entropy_backward_workspace_bytes(int dtype, int rows, int vocab, int in);

#ifdef __cplusplus
}
#endif
#endif /* OZAKI2_MODEL_H */
