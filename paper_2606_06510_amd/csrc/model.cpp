// Host side of the model operators (include/ozaki2/model.h): argument checks,
// workspace layout, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "oz2_model.h"
#include "oz2_operands.h"

namespace {

bool type_ok(int dtype) { return dtype >= OZ2_F32 && dtype <= OZ2_BF16; }

bool route_ok(int dtype, int tokens, int E, int k, int score) {
  return type_ok(dtype) && tokens >= 0 && tokens <= kMaxRows && E >= 1 && E <= OZ2_MAX_EXPERTS && k >= 1 &&
         k <= OZ2_MAX_TOPK && k <= E && (ll)tokens * k <= kMaxRows &&
         (score == OZ2_SCORE_SOFTMAX || score == OZ2_SCORE_SIGMOID);
}

bool norm_ok(int dtype, int rows, int width) {
  return type_ok(dtype) && rows >= 0 && rows <= kMaxRows && width >= 0 && width <= kMaxWidth &&
         (ll)rows * width < kMaxElems;
}

bool loss_ok(int dtype, int rows, int vocab, int in) {
  return type_ok(dtype) && rows >= 0 && rows <= kMaxRows && vocab >= 0 && vocab <= kMaxWidth && in >= 0 &&
         in <= kMaxWidth && (ll)rows * in < kMaxElems && (ll)vocab * in < kMaxElems;
}

Oz2Groups all(int rows) { return Oz2Groups{nullptr, 1, rows}; }

// Rows of the loss at a time: their chunks take no more than half a GiB (W is read
// again for the next ones: 0.2 ms a GiB beside their product)
int lse_rows(int rows, int vocab) {
  const ll per = std::max(1ll, (ll)(vocab + 63) / 64 * (ll)sizeof(Oz2Chunk));
  return (int)std::min<ll>(rows, std::max<ll>(256, (1ll << 29) / per / 256 * 256));
}

struct LseLayout {
  size_t chunks, picked, packed, total;
  int step;
  Oz2Plan plan;
};
LseLayout lse_layout(int dtype, int rows, int vocab, int in) {
  LseLayout L{};
  L.step = lse_rows(rows, vocab);
  L.plan = oz2_plan(dtype, OZ2_FWD, L.step, vocab, in, all(L.step), false, true);
  size_t o = 0;
  const int chunk = oz2_lse_chunk(L.plan);
  L.chunks = o;
  o = align256(o + (size_t)((vocab + chunk - 1) / chunk) * L.step * sizeof(Oz2Chunk));
  L.picked = o;
  o = align256(o + (size_t)L.step * 4);
  L.packed = o;
  L.total = o + align256(L.plan.packed_bytes);
  return L;
}

// The gradients of the loss, `step` words of the vocabulary at a time: so many bytes of slopes,
// half of the memory-side cache, which holds them for the products that read them.  4096 x 65536
// over 4096 bf16 and 8192 x 131072 over 1024: 64 MiB 4498 and 6607 us, 128 4458 and 5859, 256 4610
// and 6266, 1 GiB 4603 and 6671.  Longer batches were not measured: pieces get shorter, and each
// reads and writes all of dX's 32-bit sums (16384 tokens of 131072 words over 4096: 32 pieces, 17
// GB; 65536 tokens: 128, 275 GB).  Nor does a piece of few tokens leave W in the cache for dX: it is
// read twice from memory.
constexpr size_t kSlopeBytes = 128u << 20;

// Up to so many tokens the slopes are kept in two 16-bit parts, for the products are bound by W
// there (65536 x 4096 bf16, all gradients: 16 tokens 389 us instead of 382, 64 tokens 419 instead of
// 399; 100 tokens 508 instead of 408).  Of few tokens one rounding is that of all of dW:
// relatively 2^-8 at most, where it is 0.0017 on average.  With more tokens the gradients' error
// (8192 words over 1024, its norm by theirs) is that of two roundings: bf16 0.0020 of 100 and 0.0025
// of 777 tokens, fp16 0.0003 and 0.0004, of which their own is 0.0017 and 0.0002 to 0.00025; from fp32
// operands 2e-6 at most.
constexpr int kTwinRows = 64;

struct LossLayout {
  size_t rows, scale, x, w, dz, dx, work, total;
  ll pitch, pitch_dz;
  int step, lines;       // lines: rows of the slopes, and of X beside them
  int padded;            // of the products with W: 1, and 2 where W is copied as X is
  bool whole;            // dX of one piece in one product
  Oz2Plan dgrad;         // of the first piece, for all (their parts add up)
};
Oz2Plan slope_plan(int dtype, const LossLayout& L, int rows, int n, int in) {
  return oz2_plan(dtype, OZ2_FWD, rows, n, in, all(rows), L.padded, true);
}
Oz2Plan wgrad_plan(int dtype, const LossLayout& L, int n, int in) {
  return oz2_plan(dtype, OZ2_WGRAD, n, in, L.lines, all(L.lines), 3);
}
size_t piece_bytes(int dtype, const LossLayout& L, int rows, int n, int in) {
  return std::max(
      std::max(align256(slope_plan(dtype, L, rows, n, in).packed_bytes), align256(L.dgrad.packed_bytes)),
      product_bytes(wgrad_plan(dtype, L, n, in), n, in));
}
LossLayout loss_layout(int dtype, int rows, int vocab, int in) {
  const size_t e = element(dtype);
  LossLayout L{};
  L.step = (int)std::min<ll>(vocab, std::max<ll>(256, (ll)(kSlopeBytes / e / std::max(rows, 1)) / 256 * 256));
  L.pitch = oz2_packed_pitch(in, e);
  L.pitch_dz = slope_pitch(L.step, e);
  const bool twin = e == 2 && rows <= kTwinRows;
  L.lines = twin ? 2 * rows : rows;
  // (16-bit rows that are not whole pieces, for both products that read them)
  L.padded = e == 2 && (ll)in * (ll)e % 16 ? 3 : 1;
  L.dgrad = oz2_plan(dtype, OZ2_DGRAD, L.lines, in, L.step, all(L.lines), L.padded);
  L.whole = L.step >= vocab && L.dgrad.splits == 1 && !twin;
  size_t o = 0;
  L.rows = o;
  o = align256(o + (size_t)rows * sizeof(Oz2LossRow));
  L.scale = o;
  o += 256;
  L.x = o;
  o = align256(o + (size_t)L.lines * L.pitch * e);
  L.w = o;
  if (L.padded & 2) o = align256(o + (size_t)L.step * L.pitch * e);
  L.dz = o;
  o = align256(o + (size_t)L.lines * L.pitch_dz * e);
  L.dx = o;
  if (!L.whole) o = align256(o + (size_t)L.dgrad.splits * L.lines * in * 4);
  L.work = o;
  size_t most = piece_bytes(dtype, L, rows, L.step, in);
  if (L.step && vocab % L.step) most = std::max(most, piece_bytes(dtype, L, rows, vocab % L.step, in));
  L.total = o + most;
  return L;
}

bool targets_ok(const void* p, int wide) { return p && (uintptr_t)p % (wide ? 8 : 4) == 0; }

}  // namespace

extern "C" {

int ozaki2_expert_route(int dtype, int tokens, int num_experts, int top_k, const void* logits, ll ldl,
                        const float* bias, int score, int groups, int top_groups, int group_best,
                        int renormalize, float scale, int* ids, float* weights, void* stream) {
  if (!route_ok(dtype, tokens, num_experts, top_k, score)) return OZ2_E_INVALID;
  if (groups < 1 || groups > num_experts || num_experts % groups || top_groups < 1 || top_groups > groups ||
      group_best < 1 || group_best > 2 || top_k > num_experts / groups * top_groups)
    return OZ2_E_INVALID;
  if (tokens == 0) return OZ2_OK;
  const size_t e = element(dtype);
  const ll pairs = (ll)tokens * top_k;
  const Mat l = mat(logits, tokens, num_experts, ldl), b = mat(bias, 1, num_experts, num_experts),
            i = mat(ids, 1, pairs, pairs), w = mat(weights, 1, pairs, pairs);
  if (!good(l, e) || (bias && !good(b, 4)) || !good(i, 4) || !good(w, 4) || !disjoint(i, w, 4))
    return OZ2_E_INVALID;
  for (const Mat* o : {&i, &w})
    if (!disjoint_bytes(l, e, o->p, 4 * pairs) || !disjoint(b, *o, 4)) return OZ2_E_INVALID;
  const int st = oz2_device_ok();
  if (st != OZ2_OK) return st;
  return hip_status(oz2_launch_route(dtype, Oz2Route{logits, ldl, bias, tokens, num_experts, top_k, score, groups,
                                                     top_groups, group_best, renormalize != 0, scale, ids,
                                                     weights},
                                     (hipStream_t)stream));
}

int ozaki2_expert_route_backward(int dtype, int tokens, int num_experts, int top_k, const float* dweights,
                                 const void* logits, ll ldl, const int* ids, int score, int renormalize,
                                 float scale, void* dlogits, ll lddl, void* stream) {
  if (!route_ok(dtype, tokens, num_experts, top_k, score)) return OZ2_E_INVALID;
  if (tokens == 0) return OZ2_OK;
  const size_t e = element(dtype);
  const ll pairs = (ll)tokens * top_k;
  const Mat l = mat(logits, tokens, num_experts, ldl), d = mat(dlogits, tokens, num_experts, lddl);
  if (!good(l, e) || !good(d, e, true) || !int_ok(dweights) || !int_ok(ids) || !disjoint(l, d, e) ||
      !disjoint_bytes(d, e, dweights, 4 * pairs) || !disjoint_bytes(d, e, ids, 4 * pairs))
    return OZ2_E_INVALID;
  const int st = oz2_device_ok();
  if (st != OZ2_OK) return st;
  return hip_status(oz2_launch_route_backward(dtype, Oz2RouteBack{dweights, logits, ldl, ids, tokens, num_experts,
                                                                  top_k, score, renormalize != 0, scale, dlogits,
                                                                  lddl},
                                              (hipStream_t)stream));
}

int ozaki2_layer_norm(int dtype, int rows, int width, const void* x, ll ldx, const void* weight,
                      const void* bias, float eps, void* y, ll ldy, float* stats, void* stream) {
  if (!norm_ok(dtype, rows, width) || !(eps >= 0.0f)) return OZ2_E_INVALID;
  if (rows == 0 || width == 0) return OZ2_OK;
  const size_t e = element(dtype);
  const Mat mx = mat(x, rows, width, ldx), my = mat(y, rows, width, ldy), mw = mat(weight, 1, width, width),
            mb = mat(bias, 1, width, width);
  const size_t sb = stats ? 8 * (size_t)rows : 0;
  if (!good(mx, e) || !good(my, e, true) || (weight && !good(mw, e)) || (bias && !good(mb, e)) ||
      (stats && !int_ok(stats)))
    return OZ2_E_INVALID;
  if (!(x == y && ldx == ldy) && !disjoint(mx, my, e)) return OZ2_E_INVALID;
  if (!disjoint(my, mw, e) || !disjoint(my, mb, e)) return OZ2_E_INVALID;
  for (const Mat* m : {&mx, &my, &mw, &mb})
    if (!disjoint_bytes(*m, e, stats, sb)) return OZ2_E_INVALID;
  const int st = oz2_device_ok();
  if (st != OZ2_OK) return st;
  return hip_status(oz2_launch_norm(dtype, Oz2Norm{x, ldx, weight, bias, eps, rows, width, y, ldy, stats},
                                    (hipStream_t)stream));
}

size_t ozaki2_layer_norm_backward_workspace_bytes(int dtype, int rows, int width) {
  if (!norm_ok(dtype, rows, width)) return 0;
  return align256((size_t)oz2_norm_parts(dtype, rows, width) * 2 * width * 4);
}

int ozaki2_layer_norm_backward(int dtype, int rows, int width, const void* dy, ll lddy, const void* x, ll ldx,
                               const float* stats, const void* weight, const void* residual, ll ldr, void* dx,
                               ll lddx, void* dweight, void* dbias, void* workspace, size_t ws_bytes,
                               void* stream) {
  if (!norm_ok(dtype, rows, width)) return OZ2_E_INVALID;
  if (rows == 0) dx = nullptr;
  if (width == 0 || (!dx && !dweight && !dbias)) return OZ2_OK;
  const size_t e = element(dtype);
  const bool reads = dx || dweight;   // x and its statistics
  if (!dx) residual = nullptr;
  const Mat md = mat(dy, rows, width, lddy), mx = mat(reads ? x : nullptr, rows, width, ldx),
            mw = mat(dx ? weight : nullptr, 1, width, width), mr = mat(residual, rows, width, ldr);
  const Mat gx = mat(dx, rows, width, lddx), gw = mat(dweight, 1, width, width), gb = mat(dbias, 1, width, width);
  if (rows && (!good(md, e) || (reads && (!good(mx, e) || !int_ok(stats))))) return OZ2_E_INVALID;
  if ((mw.p && !good(mw, e)) || (mr.p && !good(mr, e)) || (dx && !good(gx, e, true)) ||
      (dweight && !good(gw, e, true)) || (dbias && !good(gb, e, true)))
    return OZ2_E_INVALID;
  const size_t sb = reads && rows ? 8 * (size_t)rows : 0;
  const Mat* outs[3] = {&gx, &gw, &gb};
  for (int i = 0; i < 3; ++i) {
    for (const Mat* m : {&md, &mx, &mw})
      if (!disjoint(*outs[i], *m, e)) return OZ2_E_INVALID;
    if (!(i == 0 && residual == dx && ldr == lddx) && !disjoint(*outs[i], mr, e)) return OZ2_E_INVALID;
    if (!disjoint_bytes(*outs[i], e, stats, sb)) return OZ2_E_INVALID;
    for (int j = 0; j < i; ++j)
      if (!disjoint(*outs[i], *outs[j], e)) return OZ2_E_INVALID;
  }
  const size_t need = dweight || dbias ? ozaki2_layer_norm_backward_workspace_bytes(dtype, rows, width) : 0;
  int st = check_workspace(workspace, ws_bytes, need);
  if (st != OZ2_OK) return st;
  for (const Mat* m : {&md, &mx, &mw, &mr, &gx, &gw, &gb})
    if (!disjoint_bytes(*m, e, workspace, need)) return OZ2_E_INVALID;
  if (sb && !disjoint_bytes(mat(stats, 1, 2 * (ll)rows, 2 * (ll)rows), 4, workspace, need)) return OZ2_E_INVALID;
  if ((st = oz2_device_ok()) != OZ2_OK) return st;
  return hip_status(oz2_launch_norm_backward(
      dtype, Oz2NormBack{dy, lddy, mx.p, ldx, reads ? stats : nullptr, mw.p, residual, ldr, rows, width, dx, lddx, dweight, dbias,
                         (float*)workspace, 0},
      (hipStream_t)stream));
}

size_t ozaki2_linear_cross_entropy_workspace_bytes(int dtype, int rows, int vocab, int in) {
  if (!loss_ok(dtype, rows, vocab, in) || rows == 0) return 0;
  return lse_layout(dtype, rows, vocab, in).total;
}

int ozaki2_linear_cross_entropy(int dtype, int rows, int vocab, int in, const void* x, ll ldx, const void* w,
                                ll ldw, const void* targets, int wide_targets, float* loss, float* lse,
                                void* workspace, size_t ws_bytes, void* stream) {
  if (!loss_ok(dtype, rows, vocab, in)) return OZ2_E_INVALID;
  if (rows == 0) return OZ2_OK;
  const size_t e = element(dtype), te = wide_targets ? 8 : 4;
  const Mat mx = mat(in ? x : nullptr, rows, in, ldx), mw = mat(in ? w : nullptr, vocab, in, ldw),
            mt = mat(targets, 1, rows, rows), ml = mat(loss, 1, rows, rows), me = mat(lse, 1, rows, rows);
  if (!good(mx, e) || !good(mw, e) || !targets_ok(targets, wide_targets) || !good(ml, 4) || !good(me, 4) ||
      !disjoint(ml, me, 4))
    return OZ2_E_INVALID;
  for (const Mat* o : {&ml, &me})
    if (!disjoint_bytes(mx, e, o->p, 4 * (size_t)rows) || !disjoint_bytes(mw, e, o->p, 4 * (size_t)rows) ||
        !disjoint_bytes(mt, te, o->p, 4 * (size_t)rows))
      return OZ2_E_INVALID;
  const LseLayout L = lse_layout(dtype, rows, vocab, in);
  int st = check_workspace(workspace, ws_bytes, L.total);
  if (st != OZ2_OK) return st;
  if (!disjoint_bytes(mx, e, workspace, L.total) || !disjoint_bytes(mw, e, workspace, L.total) ||
      !disjoint_bytes(mt, te, workspace, L.total) || !disjoint_bytes(ml, 4, workspace, L.total) ||
      !disjoint_bytes(me, 4, workspace, L.total))
    return OZ2_E_INVALID;
  if ((st = oz2_device_ok()) != OZ2_OK) return st;
  uint8_t* base = (uint8_t*)workspace;
  for (ll r = 0; r < rows; r += L.step) {
    const int n = (int)std::min<ll>(L.step, rows - r);
    Oz2Product p{};
    p.A = (const uint8_t*)x + (in ? r * ldx * (ll)e : 0);
    p.lda = ldx;
    p.B = w;
    p.ldb = ldw;
    p.M = n;
    p.N2 = p.N = vocab;
    p.L = in;
    p.gr = all(n);
    p.packed = base + L.packed;
    p.loss.targets = (const uint8_t*)targets + r * (ll)te;
    p.loss.wide = wide_targets != 0;
    p.loss.chunks = (Oz2Chunk*)(base + L.chunks);
    p.loss.picked = (float*)(base + L.picked);
    const hipError_t err = oz2_launch_lse(dtype, L.plan, p, loss + r, lse + r, (hipStream_t)stream);
    if (err != hipSuccess) return hip_status(err);
  }
  return OZ2_OK;
}

size_t ozaki2_linear_cross_entropy_backward_workspace_bytes(int dtype, int rows, int vocab, int in) {
  if (!loss_ok(dtype, rows, vocab, in)) return 0;
  return loss_layout(dtype, rows, vocab, in).total;
}

int ozaki2_linear_cross_entropy_backward(int dtype, int rows, int vocab, int in, const float* dloss,
                                         const void* x, ll ldx, const void* w, ll ldw, const void* targets,
                                         int wide_targets, const float* lse, void* dx, ll lddx, void* dw,
                                         ll lddw, void* workspace, size_t ws_bytes, void* stream) {
  if (!loss_ok(dtype, rows, vocab, in)) return OZ2_E_INVALID;
  if (rows == 0 || in == 0) dx = nullptr;
  if (vocab == 0 || in == 0) dw = nullptr;
  if (!dx && !dw) return OZ2_OK;
  const size_t e = element(dtype), te = wide_targets ? 8 : 4, rb = 4 * (size_t)rows;
  const Mat mx = mat(rows ? x : nullptr, rows, in, ldx), mw = mat(vocab && rows ? w : nullptr, vocab, in, ldw),
            mt = mat(rows ? targets : nullptr, 1, rows, rows), md = mat(rows ? dloss : nullptr, 1, rows, rows),
            me = mat(rows ? lse : nullptr, 1, rows, rows);
  const Mat gx = mat(dx, rows, in, lddx), gw = mat(dw, vocab, in, lddw);
  if (!good(mx, e) || (rows && !good(mw, e)) || (dx && !good(gx, e, true)) || (dw && !good(gw, e, true)) ||
      (rows && (!targets_ok(targets, wide_targets) || !int_ok(dloss) || !int_ok(lse))))
    return OZ2_E_INVALID;
  for (const Mat* o : {&gx, &gw})
    if (!disjoint(*o, mx, e) || !disjoint(*o, mw, e) || !disjoint_bytes(*o, e, mt.p, rows * te) ||
        !disjoint_bytes(*o, e, md.p, rb) || !disjoint_bytes(*o, e, me.p, rb))
      return OZ2_E_INVALID;
  if (!disjoint(gx, gw, e)) return OZ2_E_INVALID;
  const LossLayout L = loss_layout(dtype, rows, vocab, in);
  int st = check_workspace(workspace, ws_bytes, L.total);
  if (st != OZ2_OK) return st;
  for (const Mat* m : {&mx, &mw, &gx, &gw})
    if (!disjoint_bytes(*m, e, workspace, L.total)) return OZ2_E_INVALID;
  if (!disjoint_bytes(mt, te, workspace, L.total) || !disjoint_bytes(md, 4, workspace, L.total) ||
      !disjoint_bytes(me, 4, workspace, L.total))
    return OZ2_E_INVALID;
  if ((st = oz2_device_ok()) != OZ2_OK) return st;
  uint8_t* base = (uint8_t*)workspace;
  hipStream_t s = (hipStream_t)stream;
  float* scale = dtype == OZ2_F16 && rows ? (float*)(base + L.scale) : nullptr;
  hipError_t err = hipSuccess;
  const bool twin = L.lines > rows;
  // (an empty vocabulary: one empty piece, so that dX is written)
  for (ll v = 0; v == 0 || v < vocab; v += L.step) {
    const int n = (int)std::min<ll>(L.step, vocab - v);
    const void* wv = (const uint8_t*)w + (mw.p ? v * ldw * (ll)e : 0);
    ll ldv = ldw;
    const bool last = v + n >= vocab, copied = L.padded & 2 && n;
    // the rows once, W's with each piece
    if (rows && (v == 0 || copied)) {
      Oz2LossRows a{x, ldx, v ? 0 : rows, in, vocab, targets, wide_targets != 0, lse, dloss, base + L.x, L.pitch,
                    twin, (Oz2LossRow*)(base + L.rows), scale, nullptr, 0, 0, nullptr};
      if (copied) {
        a.w = wv;
        a.ldw = ldw;
        a.words = n;
        a.dst_w = base + L.w;
        wv = base + L.w;
        ldv = L.pitch;
      }
      if ((err = oz2_launch_loss_rows(dtype, a, s)) != hipSuccess) return hip_status(err);
    }
    if (rows && n) {
      Oz2Product p{};
      p.A = base + L.x;
      p.lda = L.pitch;
      p.padded = true;
      p.B = wv;
      p.ldb = ldv;
      p.paddedB = L.padded & 2;
      p.M = rows;
      p.N2 = p.N = n;
      p.L = in;
      p.gr = all(rows);
      p.y = base + L.dz;
      p.ldy = L.pitch_dz;
      p.packed = base + L.work;
      p.loss.rows = (const Oz2LossRow*)(base + L.rows);
      p.loss.first = (int)v;
      p.loss.twin = twin;
      if ((err = oz2_launch_loss_slope(dtype, slope_plan(dtype, L, rows, n, in), p, s)) != hipSuccess)
        return hip_status(err);
    }
    Oz2Product p{};
    p.A = base + L.dz;
    p.lda = L.pitch_dz;
    p.padded = true;
    p.gr = all(L.lines);
    p.loss.scale = scale;
    if (dx) {
      Oz2Product d = p;
      d.B = wv;
      d.ldb = ldv;
      d.paddedB = L.padded & 2;
      d.M = L.lines;
      d.N2 = d.N = in;
      d.L = n;
      d.y = dx;
      d.ldy = lddx;
      d.part = (float*)(base + L.dx);
      d.packed = base + L.work;
      d.loss.whole = L.whole;
      d.loss.more = v > 0;
      d.loss.twin = twin;
      if ((err = oz2_launch_loss_sum(dtype, OZ2_DGRAD, L.dgrad, d, last, s)) != hipSuccess) return hip_status(err);
    }
    if (dw) {
      const Oz2Plan plan = wgrad_plan(dtype, L, n, in);
      Oz2Product d = p;
      d.B = base + L.x;
      d.ldb = L.pitch;
      d.M = n;
      d.N2 = d.N = in;
      d.paddedB = true;
      d.L = L.lines;
      d.y = (uint8_t*)dw + v * lddw * (ll)e;
      d.ldy = lddw;
      d.part = (float*)(base + L.work);
      d.packed = base + L.work + part_bytes(plan, n, in);
      d.loss.whole = plan.splits == 1;
      err = scale ? oz2_launch_loss_sum(dtype, OZ2_WGRAD, plan, d, true, s)
                  : oz2_launch_product(dtype, OZ2_WGRAD, plan, d, s);
      if (err != hipSuccess) return hip_status(err);
    }
    if (n == 0) break;
  }
  return OZ2_OK;
}

}  // extern "C"
