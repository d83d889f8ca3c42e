// Layer norm of rows, and its gradients.
#include <algorithm>

#include "oz2_model.h"

#pragma clang fp contract(fast)

namespace {

constexpr int NT = 256, SUM_ROWS = 256;   // rows of a partial column sum
constexpr ll ROW_BLOCKS = 1 << 20;

// The sum of v over the workgroup, in a fixed order, in all threads
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

template <class T>
__global__ void __launch_bounds__(NT)
k_norm(Oz2Norm a) {
  constexpr int P = 16 / sizeof(T);
  __shared__ float red[4];
  for (ll r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.ldx;
    T* y = (T*)a.y + r * a.ldy;
    float sum = 0.0f;
    for (int c = threadIdx.x * P; c < a.width; c += NT * P) {
      const Piece<T, P> v = load_piece<T>(x + c, a.width - c);
#pragma unroll
      for (int i = 0; i < P; ++i) sum += to_f(v.v[i]);
    }
    const float mean = block_sum(sum, red) / (float)a.width;
    sum = 0.0f;
    for (int c = threadIdx.x * P; c < a.width; c += NT * P) {
      const Piece<T, P> v = load_piece<T>(x + c, a.width - c);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float d = to_f(v.v[i]) - mean;
        if (c + i < a.width) sum += d * d;
      }
    }
    const float rstd = 1.0f / sqrtf(block_sum(sum, red) / (float)a.width + a.eps);
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
      store_piece(y + c, o, valid);
    }
    if (a.stats && threadIdx.x == 0) {
      a.stats[2 * r] = mean;
      a.stats[2 * r + 1] = rstd;
    }
    __syncthreads();
  }
}

template <class T>
__global__ void __launch_bounds__(NT)
k_norm_dx(Oz2NormBack a) {
  constexpr int P = 16 / sizeof(T);
  __shared__ float red[4];
  for (ll r = blockIdx.x; r < a.rows; r += gridDim.x) {
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
    float sg = 0.0f, sh = 0.0f, g[P], h[P];
    for (int c = threadIdx.x * P; c < a.width; c += NT * P) {
      at(c, g, h);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        sg += g[i];
        sh += g[i] * h[i];
      }
    }
    sg = block_sum(sg, red) / (float)a.width;
    sh = block_sum(sh, red) / (float)a.width;
    for (int c = threadIdx.x * P; c < a.width; c += NT * P) {
      const int valid = a.width - c;
      at(c, g, h);
      Piece<T, P> o, q;
      if (a.residual) q = load_piece<T>((const T*)a.residual + r * a.ldr + c, valid);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float d = rstd * (g[i] - sg - h[i] * sh);
        if (a.residual) d += to_f(q.v[i]);
        o.v[i] = from_f<T>(d);
      }
      store_piece((T*)a.dx + r * a.lddx + c, o, valid);
    }
    __syncthreads();
  }
}

// partial column sums of SUM_ROWS rows, a column a thread
template <class T>
__global__ void __launch_bounds__(NT)
k_norm_columns(Oz2NormBack a) {
  const int c = (int)blockIdx.x * NT + threadIdx.x;
  if (c >= a.width) return;
  for (int q = blockIdx.y; q < a.parts; q += gridDim.y) {
    const ll r0 = (ll)q * SUM_ROWS, r1 = min(r0 + SUM_ROWS, (ll)a.rows);
    float sw = 0.0f, sb = 0.0f;
    for (ll r = r0; r < r1; ++r) {
      const float d = to_f(((const T*)a.dy)[r * a.lddy + c]);
      if (a.dweight) sw += d * (to_f(((const T*)a.x)[r * a.ldx + c]) - a.stats[2 * r]) * a.stats[2 * r + 1];
      sb += d;
    }
    a.part[(2ll * q) * a.width + c] = sw;
    a.part[(2ll * q + 1) * a.width + c] = sb;
  }
}

template <class T>
__global__ void __launch_bounds__(NT)
k_norm_join(Oz2NormBack a) {
  const int c = (int)blockIdx.x * NT + threadIdx.x;
  if (c >= a.width) return;
  float sw = 0.0f, sb = 0.0f;
  for (int q = 0; q < a.parts; ++q) {
    sw += a.part[(2ll * q) * a.width + c];
    sb += a.part[(2ll * q + 1) * a.width + c];
  }
  if (a.dweight) ((T*)a.dweight)[c] = from_f<T>(sw);
  if (a.dbias) ((T*)a.dbias)[c] = from_f<T>(sb);
}

}  // namespace

int oz2_norm_parts(int, int rows, int) { return (int)(((ll)rows + SUM_ROWS - 1) / SUM_ROWS); }

hipError_t oz2_launch_norm(int dtype, const Oz2Norm& a, hipStream_t s) {
  const dim3 grid((unsigned)std::min<ll>(ROW_BLOCKS, a.rows));
  OZ2_TYPED(dtype, hipLaunchKernelGGL(k_norm<T>, grid, dim3(NT), 0, s, a));
  return hipGetLastError();
}

hipError_t oz2_launch_norm_backward(int dtype, const Oz2NormBack& args, hipStream_t s) {
  Oz2NormBack a = args;
  a.parts = oz2_norm_parts(dtype, a.rows, a.width);
  hipError_t e = hipSuccess;
  if (a.dweight || a.dbias) {
    const unsigned cols = (unsigned)((a.width + NT - 1) / NT);
    if (a.parts) {
      OZ2_TYPED(dtype, hipLaunchKernelGGL(k_norm_columns<T>, dim3(cols, (unsigned)std::min(a.parts, 32768)),
                                          dim3(NT), 0, s, a));
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    OZ2_TYPED(dtype, hipLaunchKernelGGL(k_norm_join<T>, dim3(cols), dim3(NT), 0, s, a));
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.dx && a.rows) {
    const dim3 grid((unsigned)std::min<ll>(ROW_BLOCKS, a.rows));
    OZ2_TYPED(dtype, hipLaunchKernelGGL(k_norm_dx<T>, grid, dim3(NT), 0, s, a));
    e = hipGetLastError();
  }
  return e;
}
