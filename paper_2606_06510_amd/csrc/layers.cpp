// Host side of the layer operators (include/ozaki2/layers.h): argument checks,
// workspace layout, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/ozaki2.h"
#include "oz2_layers.h"
#include "oz2_operands.h"

namespace {

bool sizes_ok(int dtype, int act, ll rows, ll groups, ll out, ll in, int gated) {
  if (dtype < OZ2_F32 || dtype > OZ2_BF16 || act < OZ2_ACT_NONE || act > OZ2_ACT_SILU) return false;
  if (rows < 0 || out < 0 || in < 0 || rows > kMaxRows || out > kMaxWidth || in > kMaxWidth) return false;
  if (groups < 1 || groups > OZ2_MAX_EXPERTS) return false;
  const ll n2 = gated ? 2 * out : out;
  return rows * n2 < kMaxElems && rows * in < kMaxElems && (double)n2 * in * groups < (double)kMaxElems;
}

struct BackwardLayout {
  size_t dz, sums, parts, total;
  Oz2Plan dgrad, wgrad;
};
BackwardLayout backward_layout(int dtype, int act, int gated, const Oz2Groups& gr, ll out, ll in) {
  const size_t e = element(dtype);
  const ll n2 = gated ? 2 * out : out;
  BackwardLayout L{};
  size_t o = 0;
  L.dz = o;
  if (act != OZ2_ACT_NONE || gated) o = align256(o + (size_t)gr.rows * slope_pitch(n2, e) * e);
  L.sums = o;
  o = align256(o + (size_t)oz2_row_tiles(gr, OZ2_SUM_ROWS) * n2 * 4);
  L.parts = o;   // of one product after the other
  const bool sloped = act != OZ2_ACT_NONE || gated;
  L.dgrad = oz2_plan(dtype, OZ2_DGRAD, gr.rows, in, n2, gr, sloped);
  L.wgrad = oz2_plan(dtype, OZ2_WGRAD, n2, in, gr.rows, gr, sloped);
  o += std::max(product_bytes(L.dgrad, gr.rows, in), product_bytes(L.wgrad, n2, in));
  L.total = o;
  return L;
}

size_t forward_bytes(int dtype, int gated, const Oz2Groups& gr, ll out, ll in) {
  const ll n2 = gated ? 2 * out : out;
  return product_bytes(oz2_plan(dtype, OZ2_FWD, gr.rows, n2, in, gr), gr.rows, n2);
}

int forward(int dtype, int act, int gated, const Oz2Groups& gr, ll out, ll in, const Mat& x, const Mat& w,
            const Mat& bias, const Mat& res, const Mat& y, const Mat& z, void* ws, size_t ws_bytes,
            hipStream_t s) {
  const size_t e = element(dtype);
  if (gr.rows == 0 || out == 0) return OZ2_OK;
  if (in > 0 && (!good(x, e) || !good(w, e))) return OZ2_E_INVALID;
  if ((bias.p && !good(bias, e)) || (res.p && !good(res, e)) || !good(y, e, true) ||
      (z.p && !good(z, e, true)))
    return OZ2_E_INVALID;
  const bool in_place = res.p == y.p && res.ld == y.ld;
  const Mat* outs[2] = {&y, &z};
  for (const Mat* o : outs) {
    if (in > 0 && (!disjoint(*o, x, e) || !disjoint(*o, w, e))) return OZ2_E_INVALID;
    if (!disjoint(*o, bias, e)) return OZ2_E_INVALID;
    if (!(o == &y && in_place) && !disjoint(*o, res, e)) return OZ2_E_INVALID;
    if (gr.offsets && !disjoint_bytes(*o, e, gr.offsets, 4 * (size_t)(gr.groups + 1))) return OZ2_E_INVALID;
  }
  if (!disjoint(y, z, e)) return OZ2_E_INVALID;
  const size_t need = forward_bytes(dtype, gated, gr, out, in);
  int st = check_workspace(ws, ws_bytes, need);
  if (st != OZ2_OK) return st;
  for (const Mat* m : {&x, &w, &bias, &res, &y, &z})
    if (!disjoint_bytes(*m, e, ws, need)) return OZ2_E_INVALID;
  if (!offsets_apart(gr, ws, need)) return OZ2_E_INVALID;
  if ((st = oz2_device_ok()) != OZ2_OK) return st;
  Oz2Product p{};
  p.A = x.p;
  p.B = w.p;
  p.lda = x.ld;
  p.ldb = w.ld;
  p.M = gr.rows;
  p.N2 = (int)(gated ? 2 * out : out);
  p.L = (int)in;
  p.gr = gr;
  p.strideB = w.stride;
  p.bias = bias.p;
  p.stride_bias = bias.stride;
  p.res = res.p;
  p.ldr = res.ld;
  p.y = const_cast<void*>(y.p);
  p.ldy = y.ld;
  p.z = const_cast<void*>(z.p);
  p.ldz = z.ld;
  p.N = (int)out;
  p.act = act;
  p.gated = gated ? 1 : 0;
  const Oz2Plan plan = oz2_plan(dtype, OZ2_FWD, gr.rows, p.N2, in, gr);
  p.part = (float*)ws;
  p.packed = (uint8_t*)ws + part_bytes(plan, p.M, p.N2);
  return hip_status(oz2_launch_product(dtype, OZ2_FWD, plan, p, s));
}

int backward(int dtype, int act, int gated, const Oz2Groups& gr, ll out, ll in, const Mat& dy, const Mat& x,
             const Mat& w, const Mat& z, const Mat& dx, const Mat& dw, const Mat& db, void* ws,
             size_t ws_bytes, hipStream_t s) {
  const size_t e = element(dtype);
  const ll n2 = gated ? 2 * out : out;
  const bool sloped = act != OZ2_ACT_NONE || gated;
  const bool want_dx = dx.p && gr.rows > 0 && in > 0, want_dw = dw.p && n2 > 0 && in > 0,
             want_db = db.p && n2 > 0;
  if (!want_dx && !want_dw && !want_db) return OZ2_OK;
  const bool sums = gr.rows > 0 && out > 0;   // anything to sum
  if (sums && (!good(dy, e) || (sloped && !good(z, e)))) return OZ2_E_INVALID;
  if ((want_dx && (!good(dx, e, true) || (sums && !good(w, e)))) ||
      (want_dw && (!good(dw, e, true) || (sums && !good(x, e)))) || (want_db && !good(db, e, true)))
    return OZ2_E_INVALID;
  const Mat* ins[4] = {&dy, sloped ? &z : nullptr, want_dx ? &w : nullptr, want_dw ? &x : nullptr};
  const Mat* outs[3] = {want_dx ? &dx : nullptr, want_dw ? &dw : nullptr, want_db ? &db : nullptr};
  for (int i = 0; i < 3; ++i) {
    if (!outs[i]) continue;
    for (const Mat* m : ins)
      if (m && sums && !disjoint(*outs[i], *m, e)) return OZ2_E_INVALID;
    for (int j = 0; j < i; ++j)
      if (outs[j] && !disjoint(*outs[i], *outs[j], e)) return OZ2_E_INVALID;
    if (gr.offsets && !disjoint_bytes(*outs[i], e, gr.offsets, 4 * (size_t)(gr.groups + 1)))
      return OZ2_E_INVALID;
  }
  const BackwardLayout L = backward_layout(dtype, act, gated, gr, out, in);
  int st = check_workspace(ws, ws_bytes, L.total);
  if (st != OZ2_OK) return st;
  for (const Mat* m : ins)
    if (m && sums && !disjoint_bytes(*m, e, ws, L.total)) return OZ2_E_INVALID;
  for (const Mat* m : outs)
    if (m && !disjoint_bytes(*m, e, ws, L.total)) return OZ2_E_INVALID;
  if (!offsets_apart(gr, ws, L.total)) return OZ2_E_INVALID;
  if ((st = oz2_device_ok()) != OZ2_OK) return st;
  uint8_t* base = (uint8_t*)ws;
  hipError_t err = hipSuccess;
  const bool want_dz = sloped && (want_dx || want_dw);
  if (want_dz || want_db) {
    Oz2Slope q{};
    q.dy = dy.p;
    q.lddy = dy.ld;
    q.z = sloped ? z.p : nullptr;
    q.ldz = z.ld;
    q.dz = want_dz ? base + L.dz : nullptr;
    q.ldd = slope_pitch(n2, e);
    q.n = (int)out;
    q.act = act;
    q.gated = gated ? 1 : 0;
    q.gr = gr;
    q.db = want_db ? const_cast<void*>(db.p) : nullptr;
    q.stride_db = db.stride;
    q.part = (float*)(base + L.sums);
    if ((err = oz2_launch_slope(dtype, q, s)) != hipSuccess) return hip_status(err);
  }
  Oz2Product p{};
  p.A = sloped ? base + L.dz : dy.p;
  p.lda = sloped ? slope_pitch(n2, e) : dy.ld;
  p.padded = sloped;
  p.gr = gr;
  p.part = (float*)(base + L.parts);
  if (want_dx) {
    Oz2Product d = p;
    d.B = w.p;
    d.ldb = w.ld;
    d.strideB = w.stride;
    d.M = gr.rows;
    d.N2 = d.N = (int)in;
    d.L = (int)n2;
    d.y = const_cast<void*>(dx.p);
    d.ldy = dx.ld;
    d.packed = base + L.parts + part_bytes(L.dgrad, d.M, d.N2);
    if ((err = oz2_launch_product(dtype, OZ2_DGRAD, L.dgrad, d, s)) != hipSuccess) return hip_status(err);
  }
  if (want_dw) {
    Oz2Product d = p;
    d.B = x.p;
    d.ldb = x.ld;
    d.M = (int)n2;
    d.N2 = d.N = (int)in;
    d.L = gr.rows;
    d.y = const_cast<void*>(dw.p);
    d.ldy = dw.ld;
    d.packed = base + L.parts + part_bytes(L.wgrad, d.M, d.N2);
    d.strideB = dw.stride;
    if ((err = oz2_launch_product(dtype, OZ2_WGRAD, L.wgrad, d, s)) != hipSuccess) return hip_status(err);
  }
  return OZ2_OK;
}

bool tokens_ok(int dtype, int tokens, int top_k, int width) {
  return dtype >= OZ2_F32 && dtype <= OZ2_BF16 && tokens >= 0 && top_k >= 1 && top_k <= OZ2_MAX_TOPK &&
         width >= 0 && width <= kMaxWidth && (ll)tokens * top_k <= kMaxRows &&
         (ll)tokens * top_k * width < kMaxElems;
}

}  // namespace

// The fastest of the tilings by a fit of measured times (us; L in stages of 128 bytes,
// k workgroups on a CU):
//   256 x 256: 6 a launch; a round of tiles 8 + 1.05 a stage, 1.65 on a full chip
//   128 x 128: 5 a launch; k = 1: 0.55 a stage (fp32 2.1); k = 2: 3 + 1.1 (4.2) a stage a
//              round
//   64 x 64:   3.5 a launch; 0.28 (0.67) a stage, from k = 2 to 4 0.21 k (0.61 k), and 2 a
//              round
//   a sum in s parts: 4 for the second launch, the parts written and read at 4 TB/s
//   operands whose rows are not whole 16-byte pieces: copied first (4, and 4 TB/s), or
//   fp32 in pieces of 4 bytes, 15% more a stage, 16 bits in 128 x 128 tiles by way of
//   registers, 2.6 (4.0 two a CU) a stage
// for instance bf16 (256 / 128 / 64): 4096^3 120 / 153 / -, 2048^2 x 4096 82 / 42 / 53,
// 1024^3 27 / 13 / 7.2, 1024^2 x 4096 79 / 36 (two parts 26) / 22, 512^2 x 1024 - / 12.5 /
// 6.6, 128^2 x 8192 145 / 65 (eight 18) / 31 (eight 12), 6144 x 4096 x 1024 67 / 61 / -;
// fp32 (128 / 64): 1024^3 71 (eight 36) / 25, 1500 x 1200 x 776 58 (two 41) / 34, 2048^2 x
// 1024 80 / 83.
//   few rows (k_rows): 2, W at 5.6 TB/s, and for each row 0.05 and 0.003 a megabyte of W
//   (the workgroups' reads of x); bf16 (k_rows / tiles): 4096^2, 1 row 7.5 / 12, 16 rows
//   10.4 / 13, 32 rows 13.9 / 13.6; gated 11008 x 4096, 1 row 34 / 30, 16 rows 39 / 29.
//   Tiles read W at no more than 6.2 TB/s.
// Groups: their sizes are not known here; even ones that end half a tile early are
// assumed, and the sum stays whole.  At most 8 rows a group on average: k_rows.  The same
// rows in k_rows and in tiles, 1 and 8 a group: 16 gated bf16 experts, 4096 -> 2048, 90 and
// 113 against 112; without gates tiles win (64 experts, 4096 -> 2048, 213 and 291 against
// 178; 16 in fp32, 1024 -> 2048, 41 and 42 against 39), and so they do where most rows fall
// to one group (k_rows reads W again for every 32 of them).
Oz2Plan oz2_plan(int dtype, Oz2Side side, ll M, ll N2, ll L, const Oz2Groups& gr, int padded,
                 bool whole) {
  const double cus = oz2_device_cus();
  const bool wide = dtype == OZ2_F32;
  if (side == OZ2_FWD && gr.offsets && M <= 8ll * gr.groups)
    return Oz2Plan{M <= 2ll * gr.groups ? 1 : 2, 0, 1, 0, 0};
  const ll e = wide ? 4 : 2, groups = gr.offsets ? gr.groups : 1;
  const double stages = std::max<double>(1.0, std::ceil((double)L * e / 128.0 /
                                                        (side == OZ2_WGRAD ? groups : 1)));
  // rows of A and B as they lie in memory
  const ll wa = side == OZ2_WGRAD ? M : L, wb = side == OZ2_FWD ? L : N2;
  const ll ra = side == OZ2_WGRAD ? L : M, rb = side == OZ2_FWD ? groups * N2 : side == OZ2_DGRAD ? groups * L : L;
  const int odd = (!(padded & 1) && wa * e % 16 ? 1 : 0) | (!(padded & 2) && wb * e % 16 ? 2 : 0);
  const size_t packed = (odd & 1 ? (size_t)ra * oz2_packed_pitch(wa, e) * e : 0) +
                        (odd & 2 ? (size_t)rb * oz2_packed_pitch(wb, e) * e : 0);
  auto tiles = [&](double t) {
    if (!gr.offsets) return std::ceil(std::ceil(M / t) * std::ceil(N2 / t) / 8.0) * 8.0;   // (as launched)
    if (side == OZ2_WGRAD) return std::ceil(M / t) * std::ceil(N2 / t) * gr.groups;
    // (a group ends half a tile early on average)
    return std::max(1.0, (double)M / gr.groups / t + 0.5) * gr.groups * std::ceil(N2 / t);
  };
  Oz2Plan best{0, 128, 1, 0, 0};
  double t_best = 1e30;
  const double mb = (double)groups * (side == OZ2_WGRAD ? M : L) * N2 * e / 1e6;   // of W (or dW)
  if (side == OZ2_FWD && !gr.offsets && M <= 32) {
    best = Oz2Plan{M <= 16 ? 1 : 2, 0, 1, 0, 0};
    t_best = 2.0 + mb / 5.6 + (double)M * (0.05 + 0.003 * mb);
  }
  const double big = tiles(256.0);
  const int most = gr.offsets || whole ? 1 : (int)std::min(32.0, std::max(1.0, stages / 4.0));
  for (int pack = 0; pack <= (odd ? 1 : 0); ++pack) {
    const double first = pack ? 4.0 + (double)packed / 2e6 : 0.0;
    const bool slow = odd && !pack;
    auto take = [&](double t, int tile, int splits) {
      t = std::max(t, 3.5 + mb / 6.2) + first + (splits > 1 ? 4.0 + splits * (double)M * N2 * 8.0 / 4e6 : 0.0);
      if (t >= t_best) return;
      t_best = t;
      best = Oz2Plan{0, tile, splits, pack ? odd : 0, pack ? packed : 0};
    };
    if (!wide && !slow) {
      const double load = std::min(1.0, big / cus);
      take(6.0 + std::max(1.0, big <= 4.0 * cus ? std::ceil(big / cus) : big / cus) *
                     (8.0 + stages * (1.05 + 0.6 * load)), 256, 1);
    }
    const double f = slow ? 1.15 : 1.0, alone = wide ? 2.1 * f : slow ? 2.6 : 0.55;
    const double full = wide ? 4.2 * f : slow ? 4.0 : 1.1;
    for (int s = 1; s <= most; ++s) {
      const double per = std::ceil(stages / s), w128 = tiles(128.0) * s, w64 = tiles(64.0) * s;
      if (s == 1 || w128 <= 2.0 * cus)
        take(w128 <= cus ? 5.0 + per * alone
                         : 5.0 + (w128 <= 8.0 * cus ? std::ceil(w128 / (2.0 * cus)) : w128 / (2.0 * cus)) *
                                     (3.0 + per * full), 128, s);
      if ((wide || !slow) && (s == 1 || w64 <= 4.0 * cus)) {
        const double k = std::min(4.0, std::ceil(w64 / cus)), rounds = std::max(1.0, w64 / (4.0 * cus));
        take(3.5 + rounds * (per * (wide ? f * std::max(0.67, 0.61 * k) : std::max(0.28, 0.21 * k)) +
                             (rounds > 1.0 ? 2.0 : 0.0)), 64, s);
      }
    }
  }
  return best;
}

extern "C" {

void oz2_plan_of(int dtype, int side, ll M, ll N2, ll L, int rows, int groups, int padded, int* out) {
  static const int any = 0;
  const Oz2Plan p = oz2_plan(dtype, (Oz2Side)side, M, N2, L,
                             Oz2Groups{groups ? &any : nullptr, groups ? groups : 1, rows}, padded ? 1 : 0);
  out[0] = p.rows;
  out[1] = p.tile;
  out[2] = p.splits;
  out[3] = p.pack;
}

size_t ozaki2_linear_workspace_bytes(int dtype, int gated, int rows, int out, int in) {
  if (!sizes_ok(dtype, OZ2_ACT_NONE, rows, 1, out, in, gated)) return 0;
  return forward_bytes(dtype, gated, Oz2Groups{nullptr, 1, rows}, out, in);
}

int ozaki2_linear(int dtype, int activation, int gated, int rows, int out, int in, const void* x, ll ldx,
                  const void* w, ll ldw, const void* bias, const void* residual, ll ldr, void* y, ll ldy,
                  void* z, ll ldz, void* workspace, size_t ws_bytes, void* stream) {
  if (!sizes_ok(dtype, activation, rows, 1, out, in, gated)) return OZ2_E_INVALID;
  const ll n2 = gated ? 2ll * out : out;
  return forward(dtype, activation, gated, Oz2Groups{nullptr, 1, rows}, out, in, mat(x, rows, in, ldx),
                 mat(w, n2, in, ldw), mat(bias, 1, n2, n2), mat(residual, rows, out, ldr),
                 mat(y, rows, out, ldy), mat(z, rows, n2, ldz), workspace, ws_bytes, (hipStream_t)stream);
}

size_t ozaki2_grouped_linear_workspace_bytes(int dtype, int gated, int rows, int groups, int out, int in) {
  if (!sizes_ok(dtype, OZ2_ACT_NONE, rows, groups, out, in, gated)) return 0;
  static const int any = 0;
  return forward_bytes(dtype, gated, Oz2Groups{&any, groups, rows}, out, in);
}

int ozaki2_grouped_linear(int dtype, int activation, int gated, int rows, int groups, int out, int in,
                          const int* offsets, const void* x, ll ldx, const void* w, ll ldw, ll stride_w,
                          const void* bias, ll stride_bias, void* y, ll ldy, void* z, ll ldz,
                          void* workspace, size_t ws_bytes, void* stream) {
  if (!sizes_ok(dtype, activation, rows, groups, out, in, gated) || !int_ok(offsets)) return OZ2_E_INVALID;
  const ll n2 = gated ? 2ll * out : out;
  return forward(dtype, activation, gated, Oz2Groups{offsets, groups, rows}, out, in,
                 mat(x, rows, in, ldx), mat(w, n2, in, ldw, groups, stride_w),
                 mat(bias, 1, n2, n2, groups, stride_bias), Mat{}, mat(y, rows, out, ldy),
                 mat(z, rows, n2, ldz), workspace, ws_bytes, (hipStream_t)stream);
}

size_t ozaki2_linear_backward_workspace_bytes(int dtype, int activation, int gated, int rows, int out,
                                              int in) {
  if (!sizes_ok(dtype, activation, rows, 1, out, in, gated)) return 0;
  return backward_layout(dtype, activation, gated, Oz2Groups{nullptr, 1, rows}, out, in).total;
}

int ozaki2_linear_backward(int dtype, int activation, int gated, int rows, int out, int in, const void* dy,
                           ll lddy, const void* x, ll ldx, const void* w, ll ldw, const void* z, ll ldz,
                           void* dx, ll lddx, void* dw, ll lddw, void* dbias, void* workspace,
                           size_t ws_bytes, void* stream) {
  if (!sizes_ok(dtype, activation, rows, 1, out, in, gated)) return OZ2_E_INVALID;
  const ll n2 = gated ? 2ll * out : out;
  return backward(dtype, activation, gated, Oz2Groups{nullptr, 1, rows}, out, in, mat(dy, rows, out, lddy),
                  mat(x, rows, in, ldx), mat(w, n2, in, ldw), mat(z, rows, n2, ldz),
                  mat(dx, rows, in, lddx), mat(dw, n2, in, lddw), mat(dbias, 1, n2, n2), workspace,
                  ws_bytes, (hipStream_t)stream);
}

size_t ozaki2_grouped_linear_backward_workspace_bytes(int dtype, int activation, int gated, int rows,
                                                      int groups, int out, int in) {
  if (!sizes_ok(dtype, activation, rows, groups, out, in, gated)) return 0;
  static const int any = 0;
  return backward_layout(dtype, activation, gated, Oz2Groups{&any, groups, rows}, out, in).total;
}

int ozaki2_grouped_linear_backward(int dtype, int activation, int gated, int rows, int groups, int out,
                                   int in, const int* offsets, const void* dy, ll lddy, const void* x,
                                   ll ldx, const void* w, ll ldw, ll stride_w, const void* z, ll ldz,
                                   void* dx, ll lddx, void* dw, ll lddw, ll stride_dw, void* dbias,
                                   ll stride_dbias, void* workspace, size_t ws_bytes, void* stream) {
  if (!sizes_ok(dtype, activation, rows, groups, out, in, gated) || !int_ok(offsets)) return OZ2_E_INVALID;
  const ll n2 = gated ? 2ll * out : out;
  return backward(dtype, activation, gated, Oz2Groups{offsets, groups, rows}, out, in,
                  mat(dy, rows, out, lddy), mat(x, rows, in, ldx), mat(w, n2, in, ldw, groups, stride_w),
                  mat(z, rows, n2, ldz), mat(dx, rows, in, lddx), mat(dw, n2, in, lddw, groups, stride_dw),
                  mat(dbias, 1, n2, n2, groups, stride_dbias), workspace, ws_bytes, (hipStream_t)stream);
}

size_t ozaki2_expert_sort_workspace_bytes(int tokens, int top_k, int num_experts) {
  if (!tokens_ok(OZ2_F32, tokens, top_k, 0) || num_experts < 1 || num_experts > OZ2_MAX_EXPERTS) return 0;
  const int nb = oz2_sort_blocks((ll)tokens * top_k);
  return nb > 1 ? align256((size_t)nb * (num_experts + 1) * 4) : 0;
}

int ozaki2_expert_sort(int tokens, int top_k, int num_experts, const void* experts, int wide_ids,
                       ll ldexperts, int* offsets, int* rows, int* slots, void* workspace, size_t ws_bytes,
                       void* stream) {
  if (!tokens_ok(OZ2_F32, tokens, top_k, 0) || num_experts < 1 || num_experts > OZ2_MAX_EXPERTS)
    return OZ2_E_INVALID;
  const size_t ie = wide_ids ? 8 : 4;
  const Mat ids = mat(experts, tokens, top_k, ldexperts);
  const ll pairs = (ll)tokens * top_k;
  const Mat o = mat(offsets, 1, num_experts + 1, num_experts + 1), r = mat(rows, 1, pairs, pairs),
            sl = mat(slots, 1, pairs, pairs);
  if (!good(ids, ie) || !good(o, 4) || !good(r, 4) || !good(sl, 4)) return OZ2_E_INVALID;
  if (!disjoint(o, r, 4) || !disjoint(o, sl, 4) || !disjoint(r, sl, 4)) return OZ2_E_INVALID;
  for (const Mat* m : {&o, &r, &sl})
    if (!ids.empty() && !disjoint_bytes(*m, 4, ids.p, ids.span(ie))) return OZ2_E_INVALID;
  const size_t need = ozaki2_expert_sort_workspace_bytes(tokens, top_k, num_experts);
  int st = check_workspace(workspace, ws_bytes, need);
  if (st != OZ2_OK) return st;
  for (const Mat* m : {&o, &r, &sl})
    if (!disjoint_bytes(*m, 4, workspace, need)) return OZ2_E_INVALID;
  if (!disjoint_bytes(ids, ie, workspace, need)) return OZ2_E_INVALID;
  if ((st = oz2_device_ok()) != OZ2_OK) return st;
  return hip_status(oz2_launch_sort(tokens, top_k, num_experts, experts, wide_ids != 0, ldexperts, offsets,
                                    rows, slots, (int*)workspace, (hipStream_t)stream));
}

int ozaki2_expert_gather(int dtype, int tokens, int top_k, int width, const void* x, ll ldx,
                         const int* slots, const int* kept, const float* weights, void* xs, ll ldxs,
                         void* stream) {
  if (!tokens_ok(dtype, tokens, top_k, width)) return OZ2_E_INVALID;
  if (tokens == 0 || width == 0) return OZ2_OK;
  const size_t e = element(dtype);
  const ll pairs = (ll)tokens * top_k;
  const Mat mx = mat(x, tokens, width, ldx), mo = mat(xs, pairs, width, ldxs);
  if (!good(mx, e) || !good(mo, e, true) || !int_ok(slots) || !int_ok(kept) ||
      (weights && !int_ok(weights)) || !disjoint(mx, mo, e))
    return OZ2_E_INVALID;
  if (!disjoint_bytes(mo, e, slots, 4 * pairs) || !disjoint_bytes(mo, e, kept, 4) ||
      !disjoint_bytes(mo, e, weights, weights ? 4 * pairs : 0))
    return OZ2_E_INVALID;
  const int st = oz2_device_ok();
  if (st != OZ2_OK) return st;
  return hip_status(oz2_launch_gather(dtype, Oz2Tokens{tokens, top_k, width, slots, kept, weights}, x, ldx,
                                      xs, ldxs, (hipStream_t)stream));
}

int ozaki2_expert_combine(int dtype, int tokens, int top_k, int width, const void* ys, ll ldys,
                          const int* slots, const int* kept, const float* weights, const void* residual,
                          ll ldr, void* y, ll ldy, void* stream) {
  if (!tokens_ok(dtype, tokens, top_k, width)) return OZ2_E_INVALID;
  if (tokens == 0 || width == 0) return OZ2_OK;
  const size_t e = element(dtype);
  const ll pairs = (ll)tokens * top_k;
  const Mat mi = mat(ys, pairs, width, ldys), mr = mat(residual, tokens, width, ldr),
            mo = mat(y, tokens, width, ldy);
  if (!good(mi, e) || !good(mo, e, true) || (residual && !good(mr, e)) || !int_ok(slots) || !int_ok(kept) ||
      (weights && !int_ok(weights)) || !disjoint(mi, mo, e))
    return OZ2_E_INVALID;
  if (residual && !(residual == y && ldr == ldy) && !disjoint(mr, mo, e)) return OZ2_E_INVALID;
  if (!disjoint_bytes(mo, e, slots, 4 * pairs) || !disjoint_bytes(mo, e, kept, 4) ||
      !disjoint_bytes(mo, e, weights, weights ? 4 * pairs : 0))
    return OZ2_E_INVALID;
  const int st = oz2_device_ok();
  if (st != OZ2_OK) return st;
  return hip_status(oz2_launch_combine(dtype, Oz2Tokens{tokens, top_k, width, slots, kept, weights}, ys,
                                       ldys, residual, ldr, y, ldy, (hipStream_t)stream));
}

int ozaki2_expert_combine_backward(int dtype, int tokens, int top_k, int width, const void* dy, ll lddy,
                                   const void* ys, ll ldys, const int* slots, const int* kept,
                                   const float* weights, void* dys, ll lddys, float* dweights,
                                   void* stream) {
  if (!tokens_ok(dtype, tokens, top_k, width)) return OZ2_E_INVALID;
  if (tokens == 0 || (!dys && !dweights) || (width == 0 && !dweights)) return OZ2_OK;
  const size_t e = element(dtype);
  const ll pairs = (ll)tokens * top_k;
  const Mat md = mat(dy, tokens, width, lddy), mi = mat(dweights ? ys : nullptr, pairs, width, ldys),
            mo = mat(dys, pairs, width, lddys);
  if (!good(md, e) || (dweights && (!good(mi, e) || !int_ok(dweights))) || (dys && !good(mo, e, true)) ||
      !int_ok(slots) || !int_ok(kept) || !int_ok(weights))
    return OZ2_E_INVALID;
  if (!disjoint(md, mo, e) || !disjoint(mi, mo, e)) return OZ2_E_INVALID;
  const Mat mw = mat(dweights, 1, pairs, pairs);
  for (const void* p : {(const void*)slots, (const void*)weights})
    if (!disjoint_bytes(mo, e, p, 4 * pairs) || !disjoint_bytes(mw, 4, p, 4 * pairs)) return OZ2_E_INVALID;
  if (!disjoint_bytes(mo, e, kept, 4) || !disjoint_bytes(mw, 4, kept, 4) ||
      !disjoint_bytes(mo, e, dweights, dweights ? 4 * pairs : 0) ||
      !disjoint_bytes(md, e, dweights, dweights ? 4 * pairs : 0) ||
      !disjoint_bytes(mi, e, dweights, dweights ? 4 * pairs : 0))
    return OZ2_E_INVALID;
  const int st = oz2_device_ok();
  if (st != OZ2_OK) return st;
  return hip_status(oz2_launch_combine_backward(dtype,
                                                Oz2Tokens{tokens, top_k, width, slots, kept, weights}, dy,
                                                lddy, ys, ldys, dys, lddys, dweights, (hipStream_t)stream));
}

}  // extern "C"
