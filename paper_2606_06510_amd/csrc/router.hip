// The router: every token's experts and their weights from its logits, and the gradient.
//
// L lanes have a token, lane l of them its experts l V .. l V + V - 1, in registers; a wave has
// 64 / L tokens.  Rows of logits are read once.
#include <algorithm>

#include "oz2_lanes.h"
#include "oz2_model.h"

namespace {

constexpr int NT = 256;
constexpr ll ROW_BLOCKS = 1 << 20;

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------- keys
// Values as keys of a total order: NaN before all, then as numbers, those that are out last
// (none).  Logits alone, where the order is theirs, as whole numbers of 32 bits; scores in
// 64 bits, among which +infinity is the largest number, for +infinity is NaN's.
constexpr double kMost = 1.7976931348623157e308;

__device__ __forceinline__ void none(uint32_t& k) { k = 0; }
__device__ __forceinline__ void none(double& k) { k = -INFINITY; }
__device__ __forceinline__ void key_of(float l, uint32_t& k) {
  const uint32_t b = __builtin_bit_cast(uint32_t, l + 0.0f);   // (no negative zero)
  k = l != l ? ~0u : b >> 31 ? ~b : b | 1u << 31;
}
__device__ __forceinline__ void key_of(double c, double& k) {
  k = c != c ? INFINITY : fmin(c, kMost);
}
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }

template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
template <int CTRL>
__device__ __forceinline__ double moved(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = moved<CTRL>((uint32_t)b), hi = moved<CTRL>((uint32_t)(b >> 32));
  return __builtin_bit_cast(double, hi << 32 | lo);
}
// the largest key (the sum, in a fixed order) of a token's lanes, in all of them
template <int L, class KEY>
__device__ __forceinline__ KEY largest(KEY k) {
  k = larger(k, moved<0xB1>(k));
  k = larger(k, moved<0x4E>(k));
  k = larger(k, moved<0x141>(k));
  k = larger(k, moved<0x140>(k));
#pragma unroll
  for (int d = 16; d < L; d *= 2) k = larger(k, __shfl_xor(k, d));
  return k;
}
template <int L>
__device__ __forceinline__ double total_of(double v) {
  v += moved<0xB1>(v);
  v += moved<0x4E>(v);
  v += moved<0x141>(v);
  v += moved<0x140>(v);
#pragma unroll
  for (int d = 16; d < L; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// a token's bits of a ballot
template <int L>
__device__ __forceinline__ uint64_t of_token(uint64_t ballot) {
  if (L == 64) return ballot;
  return ballot >> (threadIdx.x & 63 & ~(L - 1)) & ((1ull << (L & 63)) - 1);
}

// The `n` largest of a token's keys, largest first, of equal ones the lower index, each taken
// out of them: take(r, index) is called by the lane that has it.  Fewer where none are left.
template <int L, int V, class KEY, class F>
__device__ __forceinline__ void take_largest(KEY (&key)[V], int n, int lane, F take) {
  KEY no;
  none(no);
  for (int r = 0; r < n; ++r) {
    KEY mine = key[0];
#pragma unroll
    for (int i = 1; i < V; ++i) mine = larger(mine, key[i]);
    const KEY best = largest<L>(mine);
    const uint64_t have = of_token<L>(__ballot(mine == best));
    if (best != no && lane == __ffsll((unsigned long long)have) - 1) {
      int at = V - 1;
#pragma unroll
      for (int i = V - 2; i >= 0; --i) at = key[i] == best ? i : at;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i == at) key[i] = no;
      take(r, lane * V + at);
    }
  }
}

__device__ __forceinline__ float log_sigmoid(float l) { return fminf(l, 0.0f) - log1pf(expf(-fabsf(l))); }

// V logits of a lane, -infinity behind the row's end
template <class T, int V>
__device__ __forceinline__ void load_logits(const T* row, int first, int E, float (&l)[V]) {
  if (first + V <= E) {
    const Piece<T, V> p = load_piece<T, V>(row + first, V);
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = to_f(p.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = first + i < E ? to_f(row[first + i]) : -INFINITY;
  }
}

// KEY: uint32_t where the order is that of the logits, double where scores are compared
template <class T, class KEY, int L, int V>
__global__ void __launch_bounds__(NT)
k_route(Oz2Route a) {
  constexpr int TOKENS = NT / L, Q = OZ2_MAX_TOPK / L;
  constexpr bool SCORED = sizeof(KEY) == 8;
  extern __shared__ double lds[];
  int* const chosen = (int*)lds + threadIdx.x / L * OZ2_MAX_TOPK;
  // groups: a token's keys, then which groups stay
  KEY* const keys = (KEY*)((int*)lds + TOKENS * OZ2_MAX_TOPK) + threadIdx.x / L * (L * V);
  uint8_t* const stays = (uint8_t*)((KEY*)((int*)lds + TOKENS * OZ2_MAX_TOPK) + NT * V) + threadIdx.x / L * (L * V);
  const int lane = threadIdx.x % L, E = a.experts, first = lane * V;
  const bool soft = a.score == OZ2_SCORE_SOFTMAX;
  const ll last = a.tokens - 1;
  for (ll t0 = (ll)blockIdx.x * TOKENS; t0 <= last; t0 += (ll)gridDim.x * TOKENS) {
    const bool live = t0 + threadIdx.x / L <= last;
    const ll t = live ? t0 + threadIdx.x / L : last;
    const T* row = (const T*)a.logits + t * a.ld;
    float l[V];
    load_logits<T, V>(row, first, E, l);
    float top = l[0];
    bool bad = !(l[0] < INFINITY);   // a logit that makes a softmax NaN
#pragma unroll
    for (int i = 1; i < V; ++i) {
      bad |= !(l[i] < INFINITY);
      top = fmaxf(top, l[i]);
    }
    bad = soft && of_token<L>(__ballot(bad));
    float total = 1.0f;
    KEY key[V], no;
    none(no);
    if constexpr (SCORED) {
      float b[V];
#pragma unroll
      for (int i = 0; i < V; ++i) b[i] = a.bias && first + i < E ? a.bias[first + i] : 0.0f;
      double s[V];
      if (soft) {
        top = across<L, false>(top);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          s[i] = l[i] == -INFINITY ? 0.0 : exp((double)l[i] - (double)top);
          sum += s[i];
        }
        sum = total_of<L>(sum);
        total = (float)sum;
        const double share = bad ? __builtin_nan("") : 1.0;
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = s[i] / sum * share;
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = 1.0 / (1.0 + exp(-(double)l[i]));
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const double c = s[i] + (double)b[i];
        key_of(c, key[i]);
        if (l[i] == -INFINITY || b[i] == -INFINITY) key[i] = no;
      }
    } else {
      if (soft && !a.renormalize) {
        top = across<L, false>(top);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) sum += l[i] == -INFINITY ? 0.0f : expf(l[i] - top);
        total = across<L, true>(sum);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        key_of(l[i], key[i]);
        if (l[i] == -INFINITY) key[i] = no;
      }
    }
    for (int j = lane; j < a.top_k; j += L) chosen[j] = -1;
    if (a.groups > 1) {
      const int per = E / a.groups;
#pragma unroll
      for (int i = 0; i < V; ++i) keys[first + i] = key[i];
      for (int g = lane; g < a.groups; g += L) stays[g] = 0;
      wave_fence();
      // lane l's groups: l W .. l W + W - 1, each lane starting elsewhere in them (LDS's banks)
      auto group_key = [&](int g) {
        KEY b1 = no, b2 = no;
        int e = lane % per;
        for (int n = 0; n < per; ++n) {
          const KEY c = keys[g * per + e];
          e = e + 1 == per ? 0 : e + 1;
          if constexpr (SCORED) b2 = fmax(b2, fmin(b1, c));
          b1 = larger(b1, c);
        }
        if constexpr (SCORED) {
          if (a.group_best > 1 && b2 > -INFINITY && b1 < INFINITY) b1 = fmin(b1 + b2, kMost);
        }
        return b1;
      };
      auto stay = [&](int, int g) { stays[g] = 1; };
      if (a.groups <= L) {
        KEY gk[1] = {no};
        if (lane < a.groups) gk[0] = group_key(lane);
        take_largest<L, 1>(gk, a.top_groups, lane, stay);
      } else {
        KEY gk[V];
#pragma unroll
        for (int i = 0; i < V; ++i) gk[i] = first + i < a.groups ? group_key(first + i) : no;
        take_largest<L, V>(gk, a.top_groups, lane, stay);
      }
      wave_fence();
      const uint32_t inverse = per > 1 ? 0xffffffffu / per + 1 : 0;   // e / per = e inverse / 2^32
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = min(first + i, E - 1);
        if (!stays[per > 1 ? (int)__umulhi(e, inverse) : e]) key[i] = no;
      }
    }
    wave_fence();
    take_largest<L, V>(key, a.top_k, lane, [&](int r, int e) { chosen[r] = e; });
    wave_fence();
    // the weights of choices lane, lane + L, ..
    int id[Q];
    float z[Q], w[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = lane + L * q;
      id[q] = j < a.top_k ? chosen[j] : -1;
      z[q] = id[q] >= 0 ? to_f(row[id[q]]) : -INFINITY;
    }
    if (a.renormalize) {
      float most = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        w[q] = soft || id[q] < 0 ? z[q] : log_sigmoid(z[q]);
        most = fmaxf(most, w[q]);
      }
      most = across<L, false>(most);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        w[q] = id[q] >= 0 ? expf(w[q] - most) : 0.0f;
        sum += w[q];
      }
      sum = across<L, true>(sum);
#pragma unroll
      for (int q = 0; q < Q; ++q) w[q] /= sum;
    } else {
#pragma unroll
      for (int q = 0; q < Q; ++q) w[q] = soft ? expf(z[q] - top) / total : 1.0f / (1.0f + expf(-z[q]));
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = lane + L * q;
      if (!live || j >= a.top_k) continue;
      a.ids[t * a.top_k + j] = id[q];
      a.weights[t * a.top_k + j] = id[q] < 0 ? 0.0f : bad ? __builtin_nanf("") : a.scale * w[q];
    }
    wave_fence();
  }
}

// ---------------------------------------------------------------- gradient
template <class T, int L, int V>
__global__ void __launch_bounds__(NT)
k_route_backward(Oz2RouteBack a) {
  constexpr int TOKENS = NT / L, Q = OZ2_MAX_TOPK / L;
  __shared__ int2 parts[TOKENS][OZ2_MAX_TOPK];   // of each choice: its expert, its gradient
  int2* const part = parts[threadIdx.x / L];
  const int lane = threadIdx.x % L, E = a.experts, first = lane * V;
  const bool soft = a.score == OZ2_SCORE_SOFTMAX, all = soft && !a.renormalize;
  const ll last = a.tokens - 1;
  for (ll t0 = (ll)blockIdx.x * TOKENS; t0 <= last; t0 += (ll)gridDim.x * TOKENS) {
    const bool live = t0 + threadIdx.x / L <= last;
    const ll t = live ? t0 + threadIdx.x / L : last;
    const T* row = (const T*)a.logits + t * a.ld;
    float l[V], top = -INFINITY, total = 1.0f;
    if (all) {   // every expert's score
      load_logits<T, V>(row, first, E, l);
#pragma unroll
      for (int i = 0; i < V; ++i) top = fmaxf(top, l[i]);
      top = across<L, false>(top);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        l[i] = l[i] == -INFINITY ? 0.0f : expf(l[i] - top);
        sum += l[i];
      }
      total = across<L, true>(sum);
    }
    int id[Q];
    float g[Q], z[Q], p[Q], own[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = lane + L * q;
      id[q] = j < a.top_k ? a.ids[t * a.top_k + j] : -1;
      if (id[q] >= E) id[q] = -1;
      g[q] = id[q] >= 0 ? a.scale * a.dweights[t * a.top_k + j] : 0.0f;
      z[q] = id[q] >= 0 ? to_f(row[id[q]]) : -INFINITY;
    }
    float dot = 0.0f;
    if (a.renormalize) {
      float most = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        p[q] = soft || id[q] < 0 ? z[q] : log_sigmoid(z[q]);
        most = fmaxf(most, p[q]);
      }
      most = across<L, false>(most);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        p[q] = p[q] == -INFINITY ? 0.0f : expf(p[q] - most);
        sum += p[q];
      }
      sum = across<L, true>(sum);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        p[q] = sum == 0.0f ? 0.0f : p[q] / sum;   // (no choice at all)
        dot += p[q] * g[q];
      }
      dot = across<L, true>(dot);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        own[q] = p[q] * (g[q] - dot);
        if (!soft) own[q] *= 1.0f / (1.0f + expf(z[q]));
      }
    } else if (soft) {
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        dot += z[q] == -INFINITY ? 0.0f : expf(z[q] - top) / total * g[q];
        own[q] = g[q];
      }
      dot = across<L, true>(dot);
    } else {
#pragma unroll
      for (int q = 0; q < Q; ++q) own[q] = g[q] / (1.0f + expf(-z[q])) / (1.0f + expf(z[q]));
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = lane + L * q;
      if (j < a.top_k) part[j] = make_int2(id[q], __float_as_int(own[q]));
    }
    wave_fence();
    float d[V];
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = 0.0f;
    for (int j = 0; j < a.top_k; ++j) {
      const int2 c = part[j];
      const int at = c.x < 0 ? -1 : c.x - first;
      const float v = __int_as_float(c.y);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (at == i) d[i] += v;
    }
    if (all) {
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] = l[i] == 0.0f ? 0.0f : l[i] / total * (d[i] - dot);
    }
    Piece<T, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.v[i] = from_f<T>(d[i]);
    if (live && first < E) store_piece((T*)a.dlogits + t * a.ldd + first, o, E - first);
    wave_fence();
  }
}

// f(lanes a token, experts a lane) as types
template <class F>
hipError_t for_experts(int E, F f) {
  using std::integral_constant;
  if (E <= 16) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (E <= 32) return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  if (E <= 64) return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if (E <= 128) return f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  if (E <= 256) return f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
  if (E <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  return f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

template <class T, class KEY>
hipError_t launch_route(const Oz2Route& a, hipStream_t s) {
  return for_experts(a.experts, [&](auto lanes, auto each) {
    constexpr int L = decltype(lanes)::value, V = decltype(each)::value, TOKENS = NT / L;
    const size_t lds = TOKENS * OZ2_MAX_TOPK * 4 + (a.groups > 1 ? NT * V * (sizeof(KEY) + 1) : 0);
    const dim3 grid((unsigned)std::min<ll>(ROW_BLOCKS, ((ll)a.tokens + TOKENS - 1) / TOKENS));
    hipLaunchKernelGGL((k_route<T, KEY, L, V>), grid, dim3(NT), lds, s, a);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t oz2_launch_route(int dtype, const Oz2Route& a, hipStream_t s) {
  // scores keep the order of the logits: they are formed only where they are added to
  const bool scored = a.bias || (a.groups > 1 && a.group_best > 1);
  OZ2_TYPED(dtype, return scored ? (launch_route<T, double>(a, s)) : (launch_route<T, uint32_t>(a, s)));
}

hipError_t oz2_launch_route_backward(int dtype, const Oz2RouteBack& a, hipStream_t s) {
  OZ2_TYPED(dtype, return for_experts(a.experts, [&](auto lanes, auto each) {
              constexpr int L = decltype(lanes)::value, V = decltype(each)::value, TOKENS = NT / L;
              const dim3 grid((unsigned)std::min<ll>(ROW_BLOCKS, ((ll)a.tokens + TOKENS - 1) / TOKENS));
              hipLaunchKernelGGL((k_route_backward<T, L, V>), grid, dim3(NT), 0, s, a);
              return hipGetLastError();
            }));
}
