// Arguments and launchers of the model operators' kernels (include/ozaki2/model.h).
// Not part of the public ABI.
#pragma once
#include "../../include/ozaki2/model.h"
#include "oz2_layers.h"

struct Oz2Route {
  const void* logits;
  ll ld;
  const float* bias;
  int tokens, experts, top_k;
  int score, groups, top_groups, group_best;
  bool renormalize;
  float scale;
  int* ids;
  float* weights;
};
hipError_t oz2_launch_route(int dtype, const Oz2Route& a, hipStream_t s);

struct Oz2RouteBack {
  const float* dweights;
  const void* logits;
  ll ld;
  const int* ids;
  int tokens, experts, top_k, score;
  bool renormalize;
  float scale;
  void* dlogits;
  ll ldd;
};
hipError_t oz2_launch_route_backward(int dtype, const Oz2RouteBack& a, hipStream_t s);

struct Oz2Norm {
  const void* x;
  ll ldx;
  const void *weight, *bias;
  float eps;
  int rows, width;
  void* y;
  ll ldy;
  float* stats;
};
hipError_t oz2_launch_norm(int dtype, const Oz2Norm& a, hipStream_t s);

struct Oz2NormBack {
  const void* dy;
  ll lddy;
  const void* x;
  ll ldx;
  const float* stats;
  const void* weight;
  const void* residual;
  ll ldr;
  int rows, width;
  void* dx;
  ll lddx;
  void *dweight, *dbias;
  float* part;          // [parts][2][width]: of dweight, of dbias
  int parts;            // (set by the launcher)
};
int oz2_norm_parts(int dtype, int rows, int width);   // of the column sums
hipError_t oz2_launch_norm_backward(int dtype, const Oz2NormBack& a, hipStream_t s);

// Rows of the loss: X in rows of whole lines, zeros where the token does not count, and
// what the gradient at a row's logits takes; and rows of W in whole lines
struct Oz2LossRows {
  const void* x;
  ll ldx;
  int rows, in, vocab;
  const void* targets;
  int wide;
  const float *lse, *dloss;
  void* dst;
  ll pitch;
  bool twin;            // X once more, from row `rows` on
  Oz2LossRow* out;
  float* scale;         // fp16: [0] the power of two of the slopes, [1] its inverse
  const void* w;        // null: none
  ll ldw;
  int words;
  void* dst_w;
};
#define OZ2_SCALE_ROWS 4096   // up to so many rows each workgroup finds the scale by itself
hipError_t oz2_launch_loss_rows(int dtype, const Oz2LossRows& a, hipStream_t s);
// the forward product's chunks into loss and lse (rows of p)
hipError_t oz2_launch_lse(int dtype, const Oz2Plan& plan, const Oz2Product& p, float* loss, float* lse,
                          hipStream_t s);
hipError_t oz2_launch_loss_slope(int dtype, const Oz2Plan& plan, const Oz2Product& p, hipStream_t s);
// the gradient of X (side DGRAD) or, fp16 with a scale, of W; joined where `last`
hipError_t oz2_launch_loss_sum(int dtype, Oz2Side side, const Oz2Plan& plan, const Oz2Product& p, bool last,
                               hipStream_t s);
inline int oz2_lse_chunk(const Oz2Plan& plan) { return plan.rows ? 16 : 64; }   // the least columns of one

#define OZ2_TYPED(dtype, ...)                                         \
  do {                                                                \
    if ((dtype) == OZ2_F32) { typedef float T; __VA_ARGS__; }         \
    else if ((dtype) == OZ2_F16) { typedef _Float16 T; __VA_ARGS__; } \
    else { typedef __bf16 T; __VA_ARGS__; }                           \
  } while (0)
