// Matrices as operands of the layer and model operators, checked before any launch:
// limits, alignment, overlap, workspaces.  Host code.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/ozaki2.h"
#include "oz2_layers.h"

namespace {

constexpr ll kMaxRows = 1ll << 30, kMaxWidth = 1ll << 21, kMaxLd = 1ll << 40, kMaxElems = 1ll << 40;

size_t element(int dtype) { return dtype == OZ2_F32 ? 4 : 2; }
size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// `count` matrices of rows x cols elements
struct Mat {
  const void* p;
  ll rows, cols, ld;
  int count;
  ll stride;
  bool empty() const { return !p || rows <= 0 || cols <= 0 || count <= 0; }
  size_t span(size_t e) const { return (size_t)((count - 1) * stride + (rows - 1) * ld + cols) * e; }
};

Mat mat(const void* p, ll rows, ll cols, ll ld, int count = 1, ll stride = 0) {
  return Mat{p, rows, cols, ld, count, stride};
}

// an operand that is needed: there, aligned to its elements, leading dimension
// and stride in range
bool good(const Mat& m, size_t e, bool output = false) {
  if (m.rows <= 0 || m.cols <= 0 || m.count <= 0) return true;
  if (!m.p || (uintptr_t)m.p % e) return false;
  if (m.ld < m.cols || m.ld > kMaxLd) return false;
  if (m.count == 1) return true;
  if (m.stride < 0 || m.stride > kMaxLd) return false;
  // outputs: one matrix after the other, or all matrices' first rows, then their second ones
  return !output || m.stride >= (m.rows - 1) * m.ld + m.cols ||
         (m.stride >= m.cols && m.ld >= (m.count - 1) * m.stride + m.cols);
}

// bytes at [0, ca) and at [d, d + cb) of every `period`
bool apart(ll d, ll ca, ll cb, ll period) {
  if (period <= 0) return false;
  d %= period;
  if (d < 0) d += period;
  return d >= ca && d + cb <= period;
}

// no element in both.  Matrices of one leading dimension may lie side by side (column
// ranges of one buffer), also where they are stacked in whole rows of it, and stacks of
// one stride may lie in between each other (a layer's parameters one after the other, for
// every layer).
bool disjoint(const Mat& a, const Mat& b, size_t e) {
  if (a.empty() || b.empty()) return true;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  if (a0 + a.span(e) <= b0 || b0 + b.span(e) <= a0) return true;
  const ll d = (ll)b0 - (ll)a0, size = (ll)e;
  auto whole_rows = [](const Mat& m) { return m.count == 1 || m.stride % m.ld == 0; };
  if (a.ld == b.ld && whole_rows(a) && whole_rows(b) &&
      apart(d, a.cols * size, b.cols * size, a.ld * size))
    return true;
  if (a.count == 1 && b.count == 1) return false;
  if (a.count > 1 && b.count > 1 && a.stride != b.stride) return false;
  return apart(d, ((a.rows - 1) * a.ld + a.cols) * size, ((b.rows - 1) * b.ld + b.cols) * size,
               (a.count > 1 ? a.stride : b.stride) * size);
}
bool disjoint_bytes(const Mat& a, size_t e, const void* p, size_t bytes) {
  if (a.empty() || !p || !bytes) return true;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)p;
  return a0 + a.span(e) <= b0 || b0 + bytes <= a0;
}

bool offsets_apart(const Oz2Groups& gr, const void* ws, size_t bytes) {
  return !gr.offsets || disjoint_bytes(mat(gr.offsets, 1, gr.groups + 1, gr.groups + 1), 4, ws, bytes);
}

int hip_status(hipError_t e) { return e == hipSuccess ? OZ2_OK : OZ2_E_DEVICE; }

int check_workspace(const void* ws, size_t bytes, size_t need) {
  if (!need) return OZ2_OK;
  return ws && (uintptr_t)ws % 256 == 0 && bytes >= need ? OZ2_OK : OZ2_E_WORKSPACE;
}

// pitch of dZ in the workspace: whole 64-byte pieces
ll slope_pitch(ll n2, size_t e) {
  const ll per = 64 / (ll)e;
  return (n2 + per - 1) / per * per;
}

// the parts of a split sum, then the packed operands
size_t part_bytes(const Oz2Plan& pl, ll M, ll N2) {
  return pl.splits > 1 ? align256((size_t)pl.splits * M * N2 * 4) : 0;
}
size_t product_bytes(const Oz2Plan& pl, ll M, ll N2) {
  return part_bytes(pl, M, N2) + align256(pl.packed_bytes);
}

bool int_ok(const void* p) { return p && (uintptr_t)p % 4 == 0; }

}  // namespace
