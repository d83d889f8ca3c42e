// The router: every token's experts and their weights from its logits, and the gradient.
#include <algorithm>

#include "oz2_model.h"

namespace {

constexpr int SLOTS = OZ2_MAX_EXPERTS / 64;   // experts of a lane: lane, lane + 64, ..
constexpr int WAVES = 4;                      // tokens of a workgroup

// Order of values as order of whole numbers: NaN first, then as numbers (no negative
// zero).  0 is less than any value's.
__device__ __forceinline__ uint64_t rank_of(double c) {
  if (c != c) return ~0ull;
  const uint64_t b = __builtin_bit_cast(uint64_t, c + 0.0);
  return b >> 63 ? ~b : b | 1ull << 63;
}

// The largest of all lanes' (key, index), of equal keys the lowest index
__device__ __forceinline__ void largest(uint64_t& key, int& at) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t k = __shfl_xor(key, d);
    const int i = __shfl_xor(at, d);
    if (k > key || (k == key && i < at)) {
      key = k;
      at = i;
    }
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

__device__ __forceinline__ float log_sigmoid(float l) { return fminf(l, 0.0f) - log1pf(expf(-fabsf(l))); }

template <class T>
__global__ void __launch_bounds__(64 * WAVES)
k_route(Oz2Route a) {
  __shared__ double value[WAVES][OZ2_MAX_EXPERTS];
  __shared__ bool stays[WAVES][OZ2_MAX_EXPERTS];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, E = a.experts;
  for (ll t = (ll)blockIdx.x * WAVES + w; t < a.tokens; t += (ll)gridDim.x * WAVES) {
  const T* row = (const T*)a.logits + t * a.ld;
  float l[SLOTS];
  float top = -INFINITY;
  bool bad = false;   // a logit that makes a softmax NaN
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    const int e = lane + 64 * i;
    l[i] = e < E ? to_f(row[e]) : -INFINITY;
    bad |= !(l[i] < INFINITY);
    top = fmaxf(top, l[i]);
  }
  bad = __any(bad);
  top = wave_max(top);
  const bool soft = a.score == OZ2_SCORE_SOFTMAX;
  // scores keep the order of the logits: they are asked for only where they are added to
  const bool scored = a.bias || (a.groups > 1 && a.group_best > 1);
  double total = 0.0;
  float total32 = 0.0f;
  if (soft) {
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      if (l[i] == -INFINITY) continue;
      total32 += expf(l[i] - top);
      if (scored) total += exp((double)l[i] - (double)top);
    }
    total32 = wave_sum(total32);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
  }
  uint64_t key[SLOTS];
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    const int e = lane + 64 * i;
    key[i] = 0;
    if (e >= E) continue;
    double c = (double)l[i];
    if (scored) {
      c = soft ? exp((double)l[i] - (double)top) / total : 1.0 / (1.0 + exp(-(double)l[i]));
      if (soft && bad) c = __builtin_nan("");
      if (a.bias) c += (double)a.bias[e];
    }
    const bool out = l[i] == -INFINITY || c == -INFINITY;
    if (!out) key[i] = rank_of(c);
    if (a.groups > 1) value[w][e] = out ? -INFINITY : c;
  }
  if (a.groups > 1) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int per = E / a.groups;
    uint64_t gk[SLOTS];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      const int g = lane + 64 * i;
      gk[i] = 0;
      if (g >= a.groups) continue;
      double b1 = -INFINITY, b2 = -INFINITY;
      bool nan = false;
      for (int e = 0; e < per; ++e) {
        const double c = value[w][g * per + e];
        nan |= c != c;
        if (c > b1) {
          b2 = b1;
          b1 = c;
        } else if (c > b2) {
          b2 = c;
        }
      }
      if (nan)
        gk[i] = ~0ull;
      else if (b1 > -INFINITY)
        gk[i] = rank_of(a.group_best > 1 && b2 > -INFINITY ? b1 + b2 : b1);
      stays[w][g] = false;
    }
    for (int r = 0; r < a.top_groups; ++r) {
      uint64_t best = 0;
      int at = OZ2_MAX_EXPERTS;
#pragma unroll
      for (int i = 0; i < SLOTS; ++i)
        if (gk[i] > best) {
          best = gk[i];
          at = lane + 64 * i;
        }
      largest(best, at);
      if (best == 0) break;
#pragma unroll
      for (int i = 0; i < SLOTS; ++i)
        if (at == lane + 64 * i) {
          gk[i] = 0;
          stays[w][at] = true;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      const int e = lane + 64 * i;
      if (e < E && !stays[w][e / per]) key[i] = 0;
    }
  }
  int mine = -1;   // choice `lane`
  for (int r = 0; r < a.top_k; ++r) {
    uint64_t best = 0;
    int at = OZ2_MAX_EXPERTS;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i)
      if (key[i] > best) {
        best = key[i];
        at = lane + 64 * i;
      }
    largest(best, at);
    if (best == 0) break;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i)
      if (at == lane + 64 * i) key[i] = 0;
    if (lane == r) mine = at;
  }
  const float z = mine >= 0 ? to_f(row[mine]) : -INFINITY;
  float weight;
  if (a.renormalize) {
    const float q = soft || mine < 0 ? z : log_sigmoid(z);
    const float most = wave_max(q);
    const float e = mine >= 0 ? expf(q - most) : 0.0f;
    weight = e / wave_sum(e);
  } else {
    weight = soft ? expf(z - top) / total32 : 1.0f / (1.0f + expf(-z));
  }
  if (soft && bad) weight = __builtin_nanf("");
  if (lane < a.top_k) {
    a.ids[t * a.top_k + lane] = mine;
    a.weights[t * a.top_k + lane] = mine >= 0 ? a.scale * weight : 0.0f;
  }
  }
}

template <class T>
__global__ void __launch_bounds__(64 * WAVES)
k_route_backward(Oz2RouteBack a) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, E = a.experts;
  for (ll t = (ll)blockIdx.x * WAVES + w; t < a.tokens; t += (ll)gridDim.x * WAVES) {
  const T* row = (const T*)a.logits + t * a.ld;
  const bool soft = a.score == OZ2_SCORE_SOFTMAX;
  int id = lane < a.top_k ? a.ids[t * a.top_k + lane] : -1;
  if (id >= E) id = -1;
  const float g = id >= 0 ? a.scale * a.dweights[t * a.top_k + lane] : 0.0f;
  const float z = id >= 0 ? to_f(row[id]) : -INFINITY;
  float top = 0.0f, total = 1.0f, dot = 0.0f, part;   // part: the choice's own gradient
  float l[SLOTS];
  if (a.renormalize) {
    const float q = soft || id < 0 ? z : log_sigmoid(z);
    const float most = wave_max(q);
    const float e = q == -INFINITY ? 0.0f : expf(q - most), sum = wave_sum(e);
    const float p = sum == 0.0f ? 0.0f : e / sum;   // (no choice at all)
    dot = wave_sum(p * g);
    part = p * (g - dot);
    if (!soft) part *= 1.0f / (1.0f + expf(z));
  } else if (soft) {
    top = -INFINITY;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      const int e = lane + 64 * i;
      l[i] = e < E ? to_f(row[e]) : -INFINITY;
      top = fmaxf(top, l[i]);
    }
    top = wave_max(top);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i)
      if (l[i] != -INFINITY) sum += expf(l[i] - top);
    total = wave_sum(sum);
    const float s = id >= 0 && z != -INFINITY ? expf(z - top) / total : 0.0f;
    dot = wave_sum(s * g);
    part = g;
  } else {
    const float s = 1.0f / (1.0f + expf(-z));
    part = g * s / (1.0f + expf(z));
  }
  if (id < 0) part = 0.0f;
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    const int e = lane + 64 * i;
    if (64 * i >= E) break;
    float d = 0.0f;
    for (int j = 0; j < a.top_k; ++j) {
      const float pj = __shfl(part, j);
      if (__shfl(id, j) == e) d += pj;
    }
    if (e >= E) continue;
    if (soft && !a.renormalize) d = l[i] == -INFINITY ? 0.0f : expf(l[i] - top) / total * (d - dot);
    ((T*)a.dlogits)[t * a.ldd + e] = from_f<T>(d);
  }
  }
}

}  // namespace

hipError_t oz2_launch_route(int dtype, const Oz2Route& a, hipStream_t s) {
  const dim3 grid((unsigned)std::min(1 << 20, (a.tokens + WAVES - 1) / WAVES));
  OZ2_TYPED(dtype, hipLaunchKernelGGL(k_route<T>, grid, dim3(64 * WAVES), 0, s, a));
  return hipGetLastError();
}

hipError_t oz2_launch_route_backward(int dtype, const Oz2RouteBack& a, hipStream_t s) {
  const dim3 grid((unsigned)std::min(1 << 20, (a.tokens + WAVES - 1) / WAVES));
  OZ2_TYPED(dtype, hipLaunchKernelGGL(k_route_backward<T>, grid, dim3(64 * WAVES), 0, s, a));
  return hipGetLastError();
}
