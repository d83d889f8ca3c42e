// Layer norm of rows, y = (x - mean) rstd w + b, and its gradients,
//   dx = rstd (g - mean g - h mean(g h)), g = dy w, h = (x - mean) rstd; dw = sum dy h, db = sum dy.
// Both are bound by memory: every entry is read once and kept in registers while its
// row's sums are taken, the variance about the mean.  16384 x 4096 bf16: forward 53 us a call on
// inputs that no cache holds (5.0 TB/s; the same inputs again 45), the gradients 81, with a
// residual 101-102 (5.0 and 5.3 TB/s, the join of the column sums, 5 of them, included).
//
// L lanes have a row, lane l its 16-byte pieces l, l + L, .., N of them at most.  As few lanes
// as keep N small: many pieces a lane cost more in registers than the barrier of several waves a
// row (16384 x 4096 bf16, forward: 64 lanes of 8 pieces 99 us, 256 of 2 52; with
// loads that wait for nothing 45).  Forward, 1025 to 2048 pieces: 256 lanes of 8, for 512 of 4
// are slower in 16 bits (16384 x 12288 231 us against 304, 4096 x 8200 63 against 77) and faster
// in fp32 (8000 x 8000 116 against 102, 300 x 5000 7.6 against 6.0).  1024 lanes have 128 registers
// each, into which four pieces do not fit but for the forward pass in fp32: 12 spill forward in 16
// bits, and of the gradients 148 in fp32 and 288 in 16 bits (4096 x 12000 fp32 396 us, 1.5 TB/s;
// 4096 x 20000 bf16 982, 0.5).
#include <algorithm>

#include "oz2_lanes.h"
#include "oz2_model.h"

#pragma clang fp contract(fast)

namespace {

constexpr ll ROW_BLOCKS = 1 << 20;

// M sums over the L lanes of each row, in a fixed order, in all of them.  Beyond a wave by way
// of LDS (red: M floats for each wave of the workgroup), and every thread calls it; red may
// be written again after the next barrier.
template <int L, int M>
__device__ __forceinline__ void row_sums(float (&v)[M], float* red) {
#pragma unroll
  for (int i = 0; i < M; ++i) v[i] = across<(L < 64 ? L : 64), true>(v[i]);
  if constexpr (L > 64) {
    const int w = threadIdx.x >> 6, first = w / (L / 64) * (L / 64);
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < M; ++i) red[w * M + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < L / 64; ++k) s += red[(first + k) * M + i];
      v[i] = s;
    }
  }
}

// Piece c / P of a row, without a branch between the loads of a row's pieces (each would wait
// for the ones before): one that ends behind the row's end is read from where it ends with
// the row (a row of a piece at least), and `settle` then moves its entries to their place and
// zeros behind them.  TINY: rows shorter than a piece.
template <class T, bool TINY, bool PAST>
__device__ __forceinline__ Piece<T, 16 / sizeof(T)> row_piece(const T* row, int c, int width) {
  constexpr int P = 16 / sizeof(T);
  if (TINY) return load_piece<T>(row + c, width - c);
  const T* p = row + min(c, width - P);
  return PAST ? load_stream<T>(p, P) : load_piece<T>(p, P);   // (past the caches)
}
template <class T, bool TINY>
__device__ __forceinline__ void settle(Piece<T, 16 / sizeof(T)>& v, int c, int width) {
  constexpr int P = 16 / sizeof(T);
  if (TINY) return;
  struct Halves {
    uint64_t lo, hi;
  } h;
  __builtin_memcpy(&h, &v, sizeof(v));
  const int bits = 8 * (int)sizeof(T) * max(c - (width - P), 0);
  const uint64_t up = bits >= 128 ? 0 : bits >= 64 ? h.hi >> (bits - 64) : bits ? h.lo >> bits | h.hi << (64 - bits) : h.lo;
  h.hi = bits >= 64 ? 0 : h.hi >> bits;
  h.lo = up;
  __builtin_memcpy(&v, &h, sizeof(v));
}

template <class T, int L, int N, bool TINY = false>
__global__ void __launch_bounds__(L < 256 ? 256 : L)
k_norm(Oz2Norm a) {
  constexpr int P = 16 / sizeof(T), NT = L < 256 ? 256 : L, G = NT / L;
  __shared__ float red[2][NT / 64];
  const int lane = threadIdx.x % L;
  const float n = (float)a.width;
  for (ll r = (ll)blockIdx.x * G + threadIdx.x / L; r < a.rows; r += (ll)gridDim.x * G) {
    const T* x = (const T*)a.x + r * a.ldx;
    Piece<T, P> v[N], w[N], b[N];
    float sum[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = row_piece<T, TINY, false>(x, (lane + L * k) * P, a.width);
    if (a.weight) {
#pragma unroll
      for (int k = 0; k < N; ++k) w[k] = row_piece<T, TINY, false>((const T*)a.weight, (lane + L * k) * P, a.width);
    }
    if (a.bias) {
#pragma unroll
      for (int k = 0; k < N; ++k) b[k] = row_piece<T, TINY, false>((const T*)a.bias, (lane + L * k) * P, a.width);
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (L * (k + 1) * P > a.width) {
        settle<T, TINY>(v[k], (lane + L * k) * P, a.width);
        if (a.weight) settle<T, TINY>(w[k], (lane + L * k) * P, a.width);
        if (a.bias) settle<T, TINY>(b[k], (lane + L * k) * P, a.width);
      }
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < P; ++i) sum[0] += to_f(v[k].v[i]);
    row_sums<L>(sum, red[0]);
    const float mean = sum[0] / n;
    sum[0] = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int valid = a.width - (lane + L * k) * P;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float d = to_f(v[k].v[i]) - mean;
        if (i < valid) sum[0] += d * d;
      }
    }
    row_sums<L>(sum, red[1]);
    const float rstd = 1.0f / sqrtf(sum[0] / n + a.eps);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = (lane + L * k) * P, valid = a.width - c;
      Piece<T, P> o;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float q = (to_f(v[k].v[i]) - mean) * rstd;
        if (a.weight) q *= to_f(w[k].v[i]);
        if (a.bias) q += to_f(b[k].v[i]);
        o.v[i] = from_f<T>(q);
      }
      store_stream((T*)a.y + r * a.ldy + c, o, valid);
    }
    if (a.stats && lane == 0) {
      a.stats[2 * r] = mean;
      a.stats[2 * r + 1] = rstd;
    }
  }
}

// Longer rows (beyond 4096 pieces): read three times, the second and third time from a cache
template <class T>
__global__ void __launch_bounds__(1024)
k_norm_long(Oz2Norm a) {
  constexpr int P = 16 / sizeof(T), NT = 1024;
  __shared__ float red[2][NT / 64];
  const float n = (float)a.width;
  for (ll r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.ldx;
    float sum[1] = {0.0f};
    for (int c = threadIdx.x * P; c < a.width; c += NT * P) {
      const Piece<T, P> v = load_piece<T>(x + c, a.width - c);
#pragma unroll
      for (int i = 0; i < P; ++i) sum[0] += to_f(v.v[i]);
    }
    row_sums<NT>(sum, red[0]);
    const float mean = sum[0] / n;
    sum[0] = 0.0f;
    for (int c = threadIdx.x * P; c < a.width; c += NT * P) {
      const Piece<T, P> v = load_piece<T>(x + c, a.width - c);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float d = to_f(v.v[i]) - mean;
        if (c + i < a.width) sum[0] += d * d;
      }
    }
    row_sums<NT>(sum, red[1]);
    const float rstd = 1.0f / sqrtf(sum[0] / n + a.eps);
    for (int c = threadIdx.x * P; c < a.width; c += NT * P) {
      const int valid = a.width - c;
      const Piece<T, P> v = load_piece<T>(x + c, valid);
      Piece<T, P> w, b, o;
      if (a.weight) w = load_piece<T>((const T*)a.weight + c, valid);
      if (a.bias) b = load_piece<T>((const T*)a.bias + c, valid);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float q = (to_f(v.v[i]) - mean) * rstd;
        if (a.weight) q *= to_f(w.v[i]);
        if (a.bias) q += to_f(b.v[i]);
        o.v[i] = from_f<T>(q);
      }
      store_stream((T*)a.y + r * a.ldy + c, o, valid);
    }
    if (a.stats && threadIdx.x == 0) {
      a.stats[2 * r] = mean;
      a.stats[2 * r + 1] = rstd;
    }
  }
}

// ---------------------------------------------------------------- gradients
// A workgroup takes G rows of every gridDim G, and keeps the column sums of its rows in
// registers; they leave as one partial row each of dweight and dbias, which k_norm_join adds
// up in order.  One read of dY and X serves all three gradients (dX and the column sums
// apart: 483 us for 16384 x 4096 bf16 with a residual, together 102).
template <class T, int L, int N, int G, bool TINY = false>
__global__ void __launch_bounds__(L* G)
k_norm_backward(Oz2NormBack a) {
  constexpr int P = 16 / sizeof(T), NT = L * G;
  __shared__ float red[2][NT / 64 * 2];
  __shared__ float others[G > 1 ? (G - 1) * L * N * P : 1];
  const int lane = threadIdx.x % L, grp = threadIdx.x / L;
  const float n = (float)a.width;
  const bool cols = a.dweight || a.dbias;
  float dw[N * P], db[N * P];
#pragma unroll
  for (int i = 0; i < N * P; ++i) dw[i] = db[i] = 0.0f;
  Piece<T, P> w[N];
  if (a.weight) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      w[k] = row_piece<T, TINY, false>((const T*)a.weight, (lane + L * k) * P, a.width);
      settle<T, TINY>(w[k], (lane + L * k) * P, a.width);
    }
  }
  int turn = 0;
  for (ll r0 = (ll)blockIdx.x * G; r0 < a.rows; r0 += (ll)gridDim.x * G, turn ^= 1) {
    const bool on = r0 + grp < a.rows;
    const ll r = on ? r0 + grp : a.rows - 1;   // (read, and not used)
    Piece<T, P> x[N], dy[N], res[N];
    float mean = 0.0f, rstd = 0.0f, sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < N; ++k)
      dy[k] = row_piece<T, TINY, true>((const T*)a.dy + r * a.lddy, (lane + L * k) * P, a.width);
    if (a.x) {
      mean = a.stats[2 * r];
      rstd = a.stats[2 * r + 1];
#pragma unroll
      for (int k = 0; k < N; ++k)
        x[k] = row_piece<T, TINY, true>((const T*)a.x + r * a.ldx, (lane + L * k) * P, a.width);
    }
    if (a.residual) {
#pragma unroll
      for (int k = 0; k < N; ++k)
        res[k] = row_piece<T, TINY, true>((const T*)a.residual + r * a.ldr, (lane + L * k) * P, a.width);
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (L * (k + 1) * P > a.width) {
        settle<T, TINY>(dy[k], (lane + L * k) * P, a.width);
        if (a.x) settle<T, TINY>(x[k], (lane + L * k) * P, a.width);
        if (a.residual) settle<T, TINY>(res[k], (lane + L * k) * P, a.width);
      }
    auto h_of = [&](int k, int i) {
      // (behind the row's end x reads as 0, which is not the mean)
      return a.x && i < a.width - (lane + L * k) * P ? (to_f(x[k].v[i]) - mean) * rstd : 0.0f;
    };
    auto g_of = [&](int k, int i) {
      const float d = to_f(dy[k].v[i]);
      return a.weight ? d * to_f(w[k].v[i]) : d;
    };
    if (on) {
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const float h = h_of(k, i), g = g_of(k, i), d = to_f(dy[k].v[i]);
          sum[0] += g;
          sum[1] += g * h;
          dw[k * P + i] += d * h;
          db[k * P + i] += d;
        }
    }
    if (!a.dx) continue;
    row_sums<L>(sum, red[turn]);
    if (!on) continue;
    const float mg = sum[0] / n, mh = sum[1] / n;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = (lane + L * k) * P;
      Piece<T, P> o;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float d = rstd * (g_of(k, i) - mg - h_of(k, i) * mh);
        if (a.residual) d += to_f(res[k].v[i]);
        o.v[i] = from_f<T>(d);
      }
      store_stream((T*)a.dx + r * a.lddx + c, o, a.width - c);
    }
  }
  if (!cols) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* mine = which ? db : dw;
    if (G > 1) {
      __syncthreads();
      if (grp > 0) {
#pragma unroll
        for (int i = 0; i < N * P; ++i) others[(grp - 1) * L * N * P + i * L + lane] = mine[i];
      }
      __syncthreads();
      if (grp == 0) {
        for (int q = 0; q < G - 1; ++q)
#pragma unroll
          for (int i = 0; i < N * P; ++i) mine[i] += others[q * L * N * P + i * L + lane];
      }
    }
    if (grp == 0) {
      float* to = a.part + (2ll * blockIdx.x + which) * a.width;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int c = (lane + L * k) * P;
        Piece<float, P> o;
#pragma unroll
        for (int i = 0; i < P; ++i) o.v[i] = mine[k * P + i];
        if (c < a.width) store_piece(to + c, o, a.width - c);
      }
    }
  }
}

// Longer rows: dX of a row by a workgroup, and partial column sums of LONG_ROWS rows, a column
// a thread
constexpr int LONG_ROWS = 64;

template <class T>
__global__ void __launch_bounds__(1024)
k_norm_dx_long(Oz2NormBack a) {
  constexpr int P = 16 / sizeof(T), NT = 1024;
  __shared__ float red[2][NT / 64 * 2];
  const float n = (float)a.width;
  int turn = 0;
  for (ll r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    const T *x = (const T*)a.x + r * a.ldx, *dy = (const T*)a.dy + r * a.lddy;
    const float mean = a.stats[2 * r], rstd = a.stats[2 * r + 1];
    auto at = [&](int c, float* g, float* h) {
      const int valid = a.width - c;
      const Piece<T, P> v = load_piece<T>(x + c, valid), d = load_piece<T>(dy + c, valid);
      Piece<T, P> w;
      if (a.weight) w = load_piece<T>((const T*)a.weight + c, valid);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        g[i] = to_f(d.v[i]) * (a.weight ? to_f(w.v[i]) : 1.0f);
        h[i] = i < valid ? (to_f(v.v[i]) - mean) * rstd : 0.0f;
      }
    };
    float sum[2] = {0.0f, 0.0f}, g[P], h[P];
    for (int c = threadIdx.x * P; c < a.width; c += NT * P) {
      at(c, g, h);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        sum[0] += g[i];
        sum[1] += g[i] * h[i];
      }
    }
    row_sums<NT>(sum, red[turn]);
    const float mg = sum[0] / n, mh = sum[1] / n;
    for (int c = threadIdx.x * P; c < a.width; c += NT * P) {
      const int valid = a.width - c;
      at(c, g, h);
      Piece<T, P> o, q;
      if (a.residual) q = load_piece<T>((const T*)a.residual + r * a.ldr + c, valid);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float d = rstd * (g[i] - mg - h[i] * mh);
        if (a.residual) d += to_f(q.v[i]);
        o.v[i] = from_f<T>(d);
      }
      store_stream((T*)a.dx + r * a.lddx + c, o, valid);
    }
  }
}

template <class T>
__global__ void __launch_bounds__(256)
k_norm_columns_long(Oz2NormBack a) {
  const int c = (int)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.width) return;
  for (int q = blockIdx.y; q < a.parts; q += gridDim.y) {
    const ll r0 = (ll)q * LONG_ROWS, r1 = min(r0 + LONG_ROWS, (ll)a.rows);
    float sw = 0.0f, sb = 0.0f;
    for (ll r = r0; r < r1; ++r) {
      const float d = to_f(((const T*)a.dy)[r * a.lddy + c]);
      if (a.dweight) sw += d * ((to_f(((const T*)a.x)[r * a.ldx + c]) - a.stats[2 * r]) * a.stats[2 * r + 1]);
      sb += d;
    }
    a.part[(2ll * q) * a.width + c] = sw;
    a.part[(2ll * q + 1) * a.width + c] = sb;
  }
}

// 32 columns of dweight (grid y 0) or dbias: the parts in eight runs, each in order, then the
// runs in order.  Bound by its launch and a chain of loads: 4.9 us for 512 parts of 4096.
template <class T>
__global__ void __launch_bounds__(256)
k_norm_join(Oz2NormBack a) {
  __shared__ float red[8][32];
  T* to = (T*)(blockIdx.y ? a.dbias : a.dweight);
  if (!to) return;
  const int l = threadIdx.x & 31, run = threadIdx.x >> 5, c = (int)blockIdx.x * 32 + l;
  const int per = (a.parts + 7) / 8, k0 = run * per, k1 = min(a.parts, k0 + per);
  float s = 0.0f;
  if (c < a.width) {
    const ll stride = 2ll * a.width;
    const float* q = a.part + (ll)blockIdx.y * a.width + c + k0 * stride;
    int k = k0;
    for (; k + 8 <= k1; k += 8, q += 8 * stride) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = q[u * stride];
      s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
    for (; k < k1; ++k, q += stride) s += *q;
  }
  red[run][l] = s;
  __syncthreads();
  if (run || c >= a.width) return;
  float sum = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) sum += red[k][l];
  to[c] = from_f<T>(sum);
}

// How the gradients run: lanes a row, pieces a lane (0: longer rows), rows a workgroup
struct Shape {
  int lanes, pieces, rows;
};
Shape backward_shape(int pieces) {
  return pieces <= 16    ? Shape{16, 1, 16}
         : pieces <= 64  ? Shape{64, 1, 8}
         : pieces <= 128 ? Shape{64, 2, 8}
         : pieces <= 256 ? Shape{64, 4, 4}
         : pieces <= 512 ? Shape{256, 2, 2}
         : pieces <= 1024 ? Shape{256, 4, 2}
         : pieces <= 2048 ? Shape{512, 4, 1}
         : pieces <= 4096 ? Shape{1024, 4, 1}
                          : Shape{1024, 0, 1};
}

}  // namespace

// Partial column sums, as many as workgroups: one on a CU, two where each has two turns of
// rows.  More parts cost more than their workgroups save (1000 x 4096 bf16: 500 of them 24.6 us,
// 250 17.8; 16384 x 4096 with a residual: 1024 109, 512 101; 4000 x 2048 fp32 36 and 28).
int oz2_norm_parts(int dtype, int rows, int width) {
  const Shape f = backward_shape((width + (dtype == OZ2_F32 ? 4 : 8) - 1) / (dtype == OZ2_F32 ? 4 : 8));
  if (!f.pieces) return (int)(((ll)rows + LONG_ROWS - 1) / LONG_ROWS);
  const ll cus = oz2_device_cus(), groups = ((ll)rows + f.rows - 1) / f.rows;
  return (int)std::min(groups, std::max(cus, std::min(2 * cus, groups / 2)));
}

namespace {

template <class T>
hipError_t launch_norm(const Oz2Norm& a, hipStream_t s) {
  constexpr int P = 16 / sizeof(T);
  const int pieces = (a.width + P - 1) / P;
  auto go = [&](auto* kernel, int lanes) {
    const int threads = std::max(lanes, 256), g = threads / lanes;
    const dim3 grid((unsigned)std::min<ll>(ROW_BLOCKS, ((ll)a.rows + g - 1) / g));
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, a);
    return hipGetLastError();
  };
  // the fewest lanes, a wave mostly (no barrier), unless that leaves most of the chip idle
  const bool few = (ll)a.rows * 64 <= 1024ll * oz2_device_cus();
  if (a.width < P) return go(k_norm<T, 16, 1, true>, 16);
  if (pieces <= 16) return go(k_norm<T, 16, 1>, 16);
  if (pieces <= 64) return go(k_norm<T, 64, 1>, 64);
  if (pieces <= 128) return go(k_norm<T, 64, 2>, 64);
  if (pieces <= 256 && !few) return go(k_norm<T, 64, 4>, 64);
  if (pieces <= 256) return go(k_norm<T, 256, 1>, 256);
  if (pieces <= 512) return go(k_norm<T, 256, 2>, 256);
  if (pieces <= 1024) return go(k_norm<T, 256, 4>, 256);
  if (pieces <= 2048) return go(k_norm<T, 256, 8>, 256);
  if (pieces <= 4096) return go(k_norm<T, 1024, 4>, 1024);
  return go(k_norm_long<T>, 1024);
}

template <class T>
hipError_t launch_backward(const Oz2NormBack& a, const Shape& f, hipStream_t s) {
  auto go = [&](auto* kernel, int threads) {
    if (a.parts) hipLaunchKernelGGL(kernel, dim3((unsigned)a.parts), dim3(threads), 0, s, a);
    return hipGetLastError();
  };
  switch (f.lanes + f.pieces) {
    case 17:
      return a.width < 16 / (int)sizeof(T) ? go(k_norm_backward<T, 16, 1, 16, true>, 256)
                                           : go(k_norm_backward<T, 16, 1, 16>, 256);
    case 65: return go(k_norm_backward<T, 64, 1, 8>, 512);
    case 66: return go(k_norm_backward<T, 64, 2, 8>, 512);
    case 68: return go(k_norm_backward<T, 64, 4, 4>, 256);
    case 258: return go(k_norm_backward<T, 256, 2, 2>, 512);
    case 260: return go(k_norm_backward<T, 256, 4, 2>, 512);
    case 516: return go(k_norm_backward<T, 512, 4, 1>, 512);
    case 1028: return go(k_norm_backward<T, 1024, 4, 1>, 1024);
  }
  hipError_t e = hipSuccess;
  if ((a.dweight || a.dbias) && a.parts) {
    hipLaunchKernelGGL(k_norm_columns_long<T>,
                       dim3((unsigned)((a.width + 255) / 256), (unsigned)std::min(a.parts, 32768)), dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.dx) {
    hipLaunchKernelGGL(k_norm_dx_long<T>, dim3((unsigned)std::min<ll>(ROW_BLOCKS, a.rows)), dim3(1024), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t oz2_launch_norm(int dtype, const Oz2Norm& a, hipStream_t s) {
  OZ2_TYPED(dtype, return launch_norm<T>(a, s));
}

hipError_t oz2_launch_norm_backward(int dtype, const Oz2NormBack& args, hipStream_t s) {
  Oz2NormBack a = args;
  const int per = dtype == OZ2_F32 ? 4 : 8;
  a.parts = oz2_norm_parts(dtype, a.rows, a.width);
  hipError_t e = hipSuccess;
  OZ2_TYPED(dtype, e = launch_backward<T>(a, backward_shape((a.width + per - 1) / per), s));
  if (e != hipSuccess || (!a.dweight && !a.dbias)) return e;
  const dim3 grid((unsigned)((a.width + 31) / 32), 2);
  OZ2_TYPED(dtype, hipLaunchKernelGGL(k_norm_join<T>, grid, dim3(256), 0, s, a));
  return hipGetLastError();
}
