// The loss over a vocabulary: the products whose ends are its statistics, its slopes and
// the gradients' sums (oz2_product.h), and the rows beside them.  With z = x W^T,
//   lse = log sum e^z, loss = lse - z[target], dz = (e^(z - lse) - [target]) dloss,
//   dx = dz W, dW = dz^T x.
// The products are all of it: 8192 x 131072 over 4096 bf16 6.2-6.4 ms by card (1.37-1.42 PFLOP/s,
// the library's rate for a product alone), 4096 x 65536 over 4096 and both gradients 4.5-5.0 ms.
// (Under the profiler with pauses between, the first takes 6.3-6.6 ms and of the second, a quarter
// of the vocabulary each, the slopes 414-442 us, dX 389-428 and dW 414-447.)  fp32: 2048 x 32768
// over 2048 1.97 ms (140 TFLOP/s), its gradients 6.2 (133).
#include "oz2_product.h"

#include "oz2_model.h"

namespace {

constexpr int JT = 256;

// (top, sum) and another one's: the larger top, both sums as seen from it (from 0 where it is
// infinite)
__device__ __forceinline__ void join(float& top, float& sum, float t, float s) {
  const float m = fmaxf(top, t), m0 = fabsf(m) == INFINITY ? 0.0f : m;
  sum = sum * __builtin_amdgcn_exp2f((top - m0) * kLog2e) + s * __builtin_amdgcn_exp2f((t - m0) * kLog2e);
  top = m;
}

// loss and lse of RT rows a workgroup from the n chunks of each: JT / RT threads a row take
// them in turn, and are joined in a fixed order.  Bound by memory (8192 rows of 1024 chunks:
// 67 MB in 22 us), for few rows by its launch (4 us).
template <int RT>
__global__ void __launch_bounds__(JT)
k_lse_join(Oz2Loss l, int rows, int vocab, int n, float* __restrict__ loss, float* __restrict__ lse) {
  constexpr int RUNS = JT / RT;
  __shared__ float top[JT], sum[JT];
  const int lr = threadIdx.x % RT, run = threadIdx.x / RT;
  const ll r = (ll)blockIdx.x * RT + lr;
  float m = -INFINITY, s = 0.0f;
  if (r < rows) {
    int k = run;
    for (; k + 3 * RUNS < n; k += 4 * RUNS) {
      Oz2Chunk c[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) c[u] = l.chunks[(ll)(k + u * RUNS) * rows + r];
#pragma unroll
      for (int u = 0; u < 4; ++u) join(m, s, c[u].top, c[u].sum);
    }
    for (; k < n; k += RUNS) {
      const Oz2Chunk c = l.chunks[(ll)k * rows + r];
      join(m, s, c.top, c.sum);
    }
  }
  top[threadIdx.x] = m;
  sum[threadIdx.x] = s;
  for (int d = RUNS / 2; d; d /= 2) {
    __syncthreads();
    if (run < d) {
      join(m, s, top[threadIdx.x + d * RT], sum[threadIdx.x + d * RT]);
      top[threadIdx.x] = m;
      sum[threadIdx.x] = s;
    }
  }
  if (run || r >= rows) return;
  const ll t = target_of(l, r);
  // (the target's logit from the largest first, in 64 bits: of a large lse and a target close to
  // it little is left)
  const double more = (double)logf(s);
  lse[r] = (float)((double)m + more);
  loss[r] = t >= 0 && t < vocab ? (float)((double)m - (double)l.picked[r] + more) : 0.0f;
}

// The exponent of the power of two that takes the largest finite |dloss| of the rows that count
// to [2^14, 2^15), 0 where there is none: a row whose dloss is infinite or no number has such
// slopes with any factor, and the others' stay in range.  Every one of NT threads calls it.
template <int NT>
__device__ __forceinline__ int slope_exponent(const Oz2LossRows& a, float* red) {
  Oz2Loss l{};
  l.targets = a.targets;
  l.wide = a.wide;
  float m = 0.0f;
  for (ll r = threadIdx.x; r < a.rows; r += NT) {
    const ll t = target_of(l, r);
    if (t < 0 || t >= a.vocab) continue;
    const float g = fabsf(a.dloss[r]);
    if (g < INFINITY) m = fmaxf(m, g);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  m = red[0];
  for (int i = 1; i < NT / 64; ++i) m = fmaxf(m, red[i]);
  int e = 0;
  if (m > 0.0f) {
    frexpf(m, &e);           // m in [2^(e - 1), 2^e)
    e = min(15 - e, 126);
  }
  return e;
}

__global__ void __launch_bounds__(1024)
k_loss_scale(Oz2LossRows a) {
  __shared__ float red[16];
  const int e = slope_exponent<1024>(a, red);
  if (threadIdx.x) return;
  a.scale[0] = ldexpf(1.0f, e);
  a.scale[1] = ldexpf(1.0f, -e);
}

// Rows of X (and of W) at whole lines, zeros at their ends and for rows of X that do not count
// (whatever such a row holds, it meets the slopes' zeros as a zero).  4096 x 4096 bf16 14 us.
template <class T>
__global__ void __launch_bounds__(256)
k_loss_rows(Oz2LossRows a) {
  constexpr int P = 16 / sizeof(T);
  __shared__ float red[4];
  float scale = 1.0f;
  if (a.scale && a.rows) {
    if (a.rows <= OZ2_SCALE_ROWS) {
      const int e = slope_exponent<256>(a, red);
      scale = ldexpf(1.0f, e);
      if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.scale[0] = scale;
        a.scale[1] = ldexpf(1.0f, -e);
      }
    } else {
      scale = a.scale[0];
    }
  }
  Oz2Loss l{};
  l.targets = a.targets;
  l.wide = a.wide;
  const ll all = (ll)a.rows + (a.w ? a.words : 0);
  for (ll r = (ll)blockIdx.x * 4 + (threadIdx.x >> 6); r < all; r += (ll)gridDim.x * 4) {
    const bool of_w = r >= a.rows;
    bool on = true;
    if (!of_w) {
      const ll t = target_of(l, r);
      on = t >= 0 && t < a.vocab;
      if ((threadIdx.x & 63) == 0)
        a.out[r] = Oz2LossRow{on ? a.lse[r] : 0.0f, on ? a.dloss[r] * scale : 0.0f, on ? (int)t : -1, 0};
    }
    const T* from = of_w ? (const T*)a.w + (r - a.rows) * a.ldw : (const T*)a.x + r * a.ldx;
    T* to = of_w ? (T*)a.dst_w + (r - a.rows) * a.pitch : (T*)a.dst + r * a.pitch;
    for (int c = (threadIdx.x & 63) * P; c < a.pitch; c += 64 * P) {
      const Piece<T, P> v = load_piece<T>(from + c, on ? a.in - c : 0);
      store_piece(to + c, v, P);
      if (a.twin && !of_w) store_piece(to + a.rows * a.pitch + c, v, P);
    }
  }
}

template <class T>
hipError_t launch_lse(const Oz2Plan& plan, Oz2Product p, float* loss, float* lse, hipStream_t s) {
  p.esize = sizeof(T);
  p.splits = 1;
  const int vocab = p.N2;
  int chunk = oz2_lse_chunk(plan);
  hipError_t e = hipSuccess;
  if (vocab > 0) {
    if (plan.rows) {
      e = launch_rows<T, false, OZ2_END_LSE>(plan.rows, p, s);
    } else {
      if (plan.pack && (e = pack<T>(OZ2_FWD, plan, p, s)) != hipSuccess) return e;
      if (plan.tile == BT && direct<T>(OZ2_FWD, p, BT)) chunk = 128;   // (as launch_tiles goes)
      e = launch_tiles<T, OZ2_FWD, OZ2_END_LSE>(plan.tile, p, s);
    }
    if (e != hipSuccess) return e;
  }
  const int n = (vocab + chunk - 1) / chunk, rows = p.M;
  auto go = [&](auto* kernel, int rt) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + rt - 1) / rt)), dim3(JT), 0, s, p.loss, rows, vocab, n,
                       loss, lse);
    return hipGetLastError();
  };
  return rows <= 64 ? go(k_lse_join<1>, 1) : rows <= 2048 ? go(k_lse_join<8>, 8) : go(k_lse_join<32>, 32);
}

template <class T>
hipError_t launch_slope(const Oz2Plan& plan, Oz2Product p, hipStream_t s) {
  p.esize = sizeof(T);
  p.splits = 1;
  if (plan.rows) return launch_rows<T, false, OZ2_END_DZ>(plan.rows, p, s);
  hipError_t e = plan.pack ? pack<T>(OZ2_FWD, plan, p, s) : hipSuccess;
  return e != hipSuccess ? e : launch_tiles<T, OZ2_FWD, OZ2_END_DZ>(plan.tile, p, s);
}

template <class T, Oz2Side SIDE>
hipError_t launch_sum(const Oz2Plan& plan, Oz2Product p, bool last, hipStream_t s) {
  p.esize = sizeof(T);
  p.splits = plan.splits;
  hipError_t e = plan.pack ? pack<T>(SIDE, plan, p, s) : hipSuccess;
  if (e == hipSuccess) e = launch_tiles<T, SIDE, OZ2_END_SUM>(plan.tile, p, s);
  if (e != hipSuccess || p.loss.whole || !last) return e;
  if (p.loss.twin) {   // both halves of a part are parts
    p.M /= 2;
    p.splits *= 2;
  }
  return launch_join<T>(p, s);
}

}  // namespace

hipError_t oz2_launch_loss_rows(int dtype, const Oz2LossRows& a, hipStream_t s) {
  if (a.scale && a.rows > OZ2_SCALE_ROWS) {
    hipLaunchKernelGGL(k_loss_scale, dim3(1), dim3(1024), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const ll all = (ll)a.rows + (a.w ? a.words : 0);
  if (all == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<ll>(1 << 20, (all + 3) / 4));
  OZ2_TYPED(dtype, hipLaunchKernelGGL(k_loss_rows<T>, grid, dim3(256), 0, s, a));
  return hipGetLastError();
}

hipError_t oz2_launch_lse(int dtype, const Oz2Plan& plan, const Oz2Product& p, float* loss, float* lse,
                          hipStream_t s) {
  OZ2_TYPED(dtype, return launch_lse<T>(plan, p, loss, lse, s));
}

hipError_t oz2_launch_loss_slope(int dtype, const Oz2Plan& plan, const Oz2Product& p, hipStream_t s) {
  OZ2_TYPED(dtype, return launch_slope<T>(plan, p, s));
}

hipError_t oz2_launch_loss_sum(int dtype, Oz2Side side, const Oz2Plan& plan, const Oz2Product& p, bool last,
                               hipStream_t s) {
  if (side == OZ2_WGRAD) return launch_sum<_Float16, OZ2_WGRAD>(plan, p, last, s);
  OZ2_TYPED(dtype, return (launch_sum<T, OZ2_DGRAD>(plan, p, last, s)));
}
