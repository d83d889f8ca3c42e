// The products of the layer operators, forward and both gradients (the kernels:
// oz2_product.h), and the slope with its column sums.
#include "oz2_product.h"

namespace {

template <class T>
hipError_t launch_product(Oz2Side side, const Oz2Plan& plan, Oz2Product p, hipStream_t s) {
  if (p.M == 0 || p.N2 == 0) return hipSuccess;
  p.esize = sizeof(T);
  p.splits = plan.splits;
  if (plan.rows) return p.gated ? launch_rows<T, true>(plan.rows, p, s) : launch_rows<T, false>(plan.rows, p, s);
  hipError_t e = plan.pack ? pack<T>(side, plan, p, s) : hipSuccess;
  if (e != hipSuccess) return e;
  e = side == OZ2_FWD     ? launch_tiles<T, OZ2_FWD>(plan.tile, p, s)
      : side == OZ2_DGRAD ? launch_tiles<T, OZ2_DGRAD>(plan.tile, p, s)
                          : launch_tiles<T, OZ2_WGRAD>(plan.tile, p, s);
  return e != hipSuccess || p.splits == 1 ? e : launch_join<T>(p, s);
}

// ------------------------------------------------ slope: dZ and its column sums
// dZ = dY f'(Z), in 32 bits; stored for the products in their operands' type.  That
// rounding is of the same size as the ones that X and W have had: in bf16 the gradients'
// error against 64 bits is 0.0024 instead of the 0.0017 of their own rounding (fp16 0.00029
// and 0.00021; fp16 overflows beyond 65504).  dZ in two 16-bit parts would double the
// products (4096^3: 2 x 108 us); a caller who needs more passes fp32 (8e-7).  The column
// sums take dZ unrounded.  A workgroup takes p.sum_rows rows of one group and 32 pieces of 16
// bytes of n, 8 rows at a time; the column sums of its rows leave as one partial row,
// added up in order by k_sums.  Bound by memory: dY and Z read and dZ written once,
// 4096^2 bf16 with gelu in 22.7 us, 4.4 TB/s.
template <class T, int ACT, bool GATED>
__global__ void __launch_bounds__(256)
k_slope(Oz2Slope p) {
  constexpr int P = 16 / sizeof(T), U = 2;
  constexpr bool SLOPED = GATED || ACT != OZ2_ACT_NONE;
  __shared__ float red[8][32 * 2 * P];
  // a row's pieces in a row of workgroups: whole rows are read at a time
  const int cb = (p.n + 32 * P - 1) / (32 * P);
  const unsigned b = blockIdx.x + blockIdx.y * gridDim.x;
  const int tile = (int)(b / cb), cc = (int)(b - (unsigned)tile * cb);
  if (tile >= group_tiles(p.gr, p.sum_rows)) return;
  int group, first, row, end;
  group_tile(p.gr, p.sum_rows, tile, group, first, row, end);
  end = min(end, row + p.sum_rows);
  const int c = (cc * 32 + (int)(threadIdx.x & 31)) * P, rr = threadIdx.x >> 5;
  const int n2 = GATED ? 2 * p.n : p.n, valid = p.n - c;
  float sg[P], su[P];
#pragma unroll
  for (int i = 0; i < P; ++i) sg[i] = su[i] = 0.0f;
  if (valid > 0) {
#pragma clang loop unroll(disable)
    for (int t0 = row + rr; t0 < end; t0 += 8 * U) {
      Piece<T, P> g[U], a[U], u[U];
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const ll t = min(t0 + 8 * q, end - 1);
        g[q] = load_stream<T>((const T*)p.dy + t * p.lddy + c, valid);
        if (SLOPED) a[q] = load_stream<T>((const T*)p.z + t * p.ldz + c, valid);
        if (GATED) u[q] = load_stream<T>((const T*)p.z + t * p.ldz + p.n + c, valid);
      }
      float d[U * P], e[U * P];
#pragma unroll
      for (int i = 0; i < U * P; ++i) d[i] = t0 + 8 * (i / P) < end ? to_f(g[i / P].v[i % P]) : 0.0f;
      if (GATED) {
#pragma unroll
        for (int i = 0; i < U * P; ++i) e[i] = d[i] * act_f<T>(to_f(a[i / P].v[i % P]), ACT);
#pragma unroll
        for (int i = 0; i < U * P; ++i) {
          // (rows past the end: d is 0, but 0 times an infinite f, or a slope of NaN, is not)
          if (t0 + 8 * (i / P) < end) su[i % P] += e[i];
          d[i] *= to_f(u[i / P].v[i % P]);
          u[i / P].v[i % P] = from_f<T>(e[i]);
        }
      }
      if (ACT != OZ2_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < U * P; ++i) d[i] *= act_d<T>(to_f(a[i / P].v[i % P]), ACT);
      }
#pragma unroll
      for (int i = 0; i < U * P; ++i) {
        if (t0 + 8 * (i / P) < end) sg[i % P] += d[i];
        g[i / P].v[i % P] = from_f<T>(d[i]);
      }
      if (SLOPED && p.dz) {
#pragma unroll
        for (int q = 0; q < U; ++q) {
          if (t0 + 8 * q >= end) continue;
          T* z = (T*)p.dz + (t0 + 8 * q) * p.ldd;
          store_stream(z + c, g[q], valid);
          if (GATED) store_stream(z + p.n + c, u[q], valid);
          // the pad of the row is read as part of the last piece: zeros
          if (valid <= P)
            for (int k = n2; k < p.ldd; ++k) z[k] = (T)0.0f;
        }
      }
    }
  }
  if (!p.db) return;
  const int l = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    red[rr][l * 2 * P + i] = sg[i];
    red[rr][l * 2 * P + P + i] = su[i];
  }
  __syncthreads();
  for (int q = threadIdx.x; q < 32 * 2 * P; q += 256) {
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += red[k][q];
    const int piece = q / (2 * P), i = q % (2 * P);
    const int col = (cc * 32 + piece) * P + i % P;
    const bool up = i >= P;
    if (col < p.n && (!up || GATED)) p.part[(ll)tile * n2 + (up ? p.n + col : col)] = s;
  }
}

// db of group blockIdx.y, 32 columns a workgroup: the partial rows of the group's row
// tiles in eight runs, each in order, then the runs in order (4.6 us, its launch and a
// chain of loads)
template <class T>
__global__ void __launch_bounds__(256)
k_sums(Oz2Slope p) {
  __shared__ float red[8][32];
  const int n2 = p.gated ? 2 * p.n : p.n, l = threadIdx.x & 31, run = threadIdx.x >> 5;
  const int c = (int)blockIdx.x * 32 + l, g = (int)blockIdx.y;
  int first, count;
  group_tiles_before(p.gr, p.sum_rows, g, first, count);
  const int per = (count + 7) / 8, k0 = run * per, k1 = min(count, k0 + per);
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c < n2) {
    const float* q = p.part + (ll)first * n2 + c;
    int k = k0;
    for (; k + 4 <= k1; k += 4)
#pragma unroll
      for (int u = 0; u < 4; ++u) s[u] += q[(ll)(k + u) * n2];
    for (; k < k1; ++k) s[0] += q[(ll)k * n2];
  }
  red[run][l] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (run == 0 && c < n2) {
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += red[k][l];
    ((T*)p.db)[g * p.stride_db + c] = from_f<T>(sum);
  }
}

template <class T>
hipError_t launch_slope(Oz2Slope p, hipStream_t s) {
  constexpr int P = 16 / sizeof(T);
  const int cb = (p.n + 32 * P - 1) / (32 * P);
  // long workgroups where there are enough of them: a workgroup's start (its place among
  // the groups) takes as long as 16 rows
  p.sum_rows = OZ2_SUM_ROWS;
  while (p.sum_rows < 128 && (ll)p.gr.rows / p.sum_rows * cb > 8ll * oz2_device_cus()) p.sum_rows *= 2;
  const ll rt = oz2_row_tiles(p.gr, p.sum_rows);
  if (rt > 0 && cb > 0) {
    const Oz2Grid g = oz2_grid(rt * cb);
    const dim3 grid(g.x, g.y);
#define OZ2_SLOPE(ACT)                                                          \
  case ACT:                                                                     \
    if (p.gated)                                                                \
      hipLaunchKernelGGL((k_slope<T, ACT, true>), grid, dim3(256), 0, s, p);    \
    else                                                                        \
      hipLaunchKernelGGL((k_slope<T, ACT, false>), grid, dim3(256), 0, s, p);   \
    break
    switch (p.act) {
      OZ2_SLOPE(OZ2_ACT_NONE);
      OZ2_SLOPE(OZ2_ACT_RELU);
      OZ2_SLOPE(OZ2_ACT_GELU);
      OZ2_SLOPE(OZ2_ACT_GELU_TANH);
      OZ2_SLOPE(OZ2_ACT_SILU);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int n2 = p.gated ? 2 * p.n : p.n;
  if (p.db && n2 > 0) {
    hipLaunchKernelGGL(k_sums<T>, dim3((unsigned)((n2 + 31) / 32), (unsigned)p.gr.groups), dim3(256), 0,
                       s, p);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace

hipError_t oz2_launch_product(int dtype, Oz2Side side, const Oz2Plan& plan, const Oz2Product& p,
                              hipStream_t s) {
  if (dtype == OZ2_F32) return launch_product<float>(side, plan, p, s);
  if (dtype == OZ2_F16) return launch_product<_Float16>(side, plan, p, s);
  return launch_product<__bf16>(side, plan, p, s);
}

hipError_t oz2_launch_slope(int dtype, const Oz2Slope& p, hipStream_t s) {
  if (dtype == OZ2_F32) return launch_slope<float>(p, s);
  if (dtype == OZ2_F16) return launch_slope<_Float16>(p, s);
  return launch_slope<__bf16>(p, s);
}
