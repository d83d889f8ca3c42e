// Tokens in the order of their experts and back: a stable counting sort of the
// token-expert pairs, the tokens' rows at their places, their weighted sum, and
// the gradients.  All of it moves data once; nothing here is bound by arithmetic.
#include <algorithm>

#include "oz2_layers.h"

namespace {

// ---------------------------------------------------------------- sort
// Key of pair p: its expert, or E where dropped.  The stable order of keys
// 0..E by counting: place = (pairs of lower keys) + (earlier pairs of the key).
// A workgroup takes a contiguous range of pairs, each of its waves a contiguous
// part, so "earlier" is: earlier workgroups (counted by a first launch), earlier
// waves (counted in LDS), and earlier lanes (a ballot per bit of the key).  Bound by
// the two launches and the chains of waits in them: 131072 pairs of 64 experts 4.8 and 7.0
// us, 16 pairs (one launch) 3.2.
constexpr int SORT_NT = 512, SORT_W = SORT_NT / 64;
constexpr int SORT_KEYS = 4;                      // of a thread, kept in registers
constexpr int SORT_CHUNK = SORT_NT * SORT_KEYS;   // pairs of a workgroup, or a multiple

struct SortArgs {
  const void* ids;
  ll ld;
  int k, E, pairs, chunk;   // chunk: pairs per workgroup, a multiple of SORT_CHUNK
  bool wide;
};

__device__ __forceinline__ int key_of(const SortArgs& a, int p) {
  const int t = p / a.k;
  const ll at = (ll)t * a.ld + (p - t * a.k);
  const ll v = a.wide ? ((const ll*)a.ids)[at] : (ll)((const int*)a.ids)[at];
  return v >= 0 && v < a.E ? (int)v : a.E;
}

__global__ void __launch_bounds__(SORT_NT)
k_sort_count(SortArgs a, int* __restrict__ counts) {
  __shared__ int h[OZ2_MAX_EXPERTS + 1];
  for (int e = threadIdx.x; e <= a.E; e += SORT_NT) h[e] = 0;
  __syncthreads();
  const int p0 = blockIdx.x * a.chunk, p1 = min(a.pairs, p0 + a.chunk);
  for (int p = p0 + (int)threadIdx.x; p < p1; p += SORT_NT) atomicAdd(&h[key_of(a, p)], 1);
  __syncthreads();
  for (int e = threadIdx.x; e <= a.E; e += SORT_NT) counts[(ll)blockIdx.x * (a.E + 1) + e] = h[e];
}

__global__ void __launch_bounds__(SORT_NT)
k_sort_place(SortArgs a, const int* __restrict__ counts, int* __restrict__ offsets,
             int* __restrict__ rows, int* __restrict__ slots) {
  __shared__ int at[SORT_W][OZ2_MAX_EXPERTS + 1];   // counts, then next place, of each wave and key
  __shared__ int tot[OZ2_MAX_EXPERTS + 1], before[OZ2_MAX_EXPERTS + 1];
  __shared__ int wsum[SORT_W];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, K = a.E + 1;
  const int part = a.chunk / SORT_W, p0 = blockIdx.x * a.chunk + w * part;
  const int p1 = min(a.pairs, p0 + part);
  // the wave's first SORT_KEYS steps' keys (all, unless there are a great many pairs)
  int keys[SORT_KEYS];
#pragma unroll
  for (int i = 0; i < SORT_KEYS; ++i) {
    const int p = p0 + 64 * i + lane;
    keys[i] = p < p1 ? key_of(a, p) : -1;
  }
  for (int e = tid; e < K; e += SORT_NT) {
    tot[e] = before[e] = 0;
#pragma unroll
    for (int v = 0; v < SORT_W; ++v) at[v][e] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SORT_KEYS; ++i)
    if (keys[i] >= 0) atomicAdd(&at[w][keys[i]], 1);
  for (int p = p0 + 64 * SORT_KEYS + lane; p < p1; p += 64) atomicAdd(&at[w][key_of(a, p)], 1);
  // pairs of each key in all, and in earlier workgroups: every eighth one a wave's
  if (gridDim.x > 1) {
    for (int e = lane; e < K; e += 64) {
      int all = 0, early = 0;
#pragma unroll 4
      for (int b = w; b < (int)gridDim.x; b += SORT_W) {
        const int c = counts[(ll)b * K + e];
        all += c;
        early += b < (int)blockIdx.x ? c : 0;
      }
      atomicAdd(&tot[e], all);
      atomicAdd(&before[e], early);
    }
  }
  __syncthreads();
  for (int e = tid; e < K; e += SORT_NT) {
    // exclusive over the waves, from the earlier workgroups' pairs on
    int n = before[e];
#pragma unroll
    for (int v = 0; v < SORT_W; ++v) {
      const int c = at[v][e];
      at[v][e] = n;
      n += c;
    }
    if (gridDim.x == 1) tot[e] = n;
  }
  __syncthreads();
  // exclusive sums of tot: each thread `per` consecutive keys
  const int per = (K + SORT_NT - 1) / SORT_NT;
  int mine = 0;
  for (int i = 0; i < per; ++i) {
    const int e = tid * per + i;
    if (e < K) mine += tot[e];
  }
  int incl = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(incl, d);
    if (lane >= d) incl += up;
  }
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  int excl = incl - mine;
  for (int v = 0; v < w; ++v) excl += wsum[v];
  for (int i = 0; i < per; ++i) {
    const int e = tid * per + i;
    if (e < K) {
      const int c = tot[e];
      tot[e] = excl;
      if (blockIdx.x == 0) offsets[e] = excl;   // offsets[E]: the pairs kept
      excl += c;
    }
  }
  __syncthreads();
  const int bits = 32 - __clz(a.E);   // of keys 0..E
  auto place = [&](int p, int key) {  // key < 0: no pair
    const bool live = key >= 0;
    unsigned long long same = __ballot(live);
    for (int b = 0; b < bits; ++b) {
      const bool one = (key >> b) & 1;
      const unsigned long long m = __ballot(one);
      same &= one ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (live) {
      const int to = tot[key] + at[w][key] + rank;
      rows[to] = p;
      slots[p] = to;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (live && rank == 0) at[w][key] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
#pragma unroll
  for (int i = 0; i < SORT_KEYS; ++i)
    if (p0 + 64 * i < p1) place(p0 + 64 * i + lane, keys[i]);
  for (int q = p0 + 64 * SORT_KEYS; q < p1; q += 64)
    place(q + lane, q + lane < p1 ? key_of(a, q + lane) : -1);
}

// ---------------------------------------------------------------- rows
// LPR lanes walk the 16-byte pieces of one token's row; a token's row is read once and
// meets all of its places.  All rows may start at any element.  Grids are bounded: a
// workgroup goes on to the tokens a grid further.  Bound by memory: k_gather of 16384
// tokens to 8 places each, 4096 wide in bf16 (0.13 GB read, 1.05 written), 208 us, 5.7
// TB/s; 5000 tokens, 4 places, 2001 wide in fp16: k_combine 23.4 us (117 MB, 5.0 TB/s),
// k_combine_backward 39 (176 MB, 4.5).  Loads past the caches, which help the stores, cost
// these 5 to 17%.
constexpr ll ROW_BLOCKS = 1 << 20;
#define OZ2_TOKENS(t, lane)                                                                     \
  const int lane = (int)(threadIdx.x % LPR);                                                    \
  for (ll t = ((ll)blockIdx.x * 256 + threadIdx.x) / LPR; t < a.tokens; t += (ll)gridDim.x * 256 / LPR)

// Xs at each of a token's places = (weight x) X; zeros at those of dropped pairs
template <class T, int LPR>
__global__ void __launch_bounds__(256)
k_gather(Oz2Tokens a, const T* __restrict__ x, ll ldx, T* __restrict__ xs, ll ldxs) {
  constexpr int P = 16 / sizeof(T);
  const int pairs = a.tokens * a.top_k, kept = min(*a.kept, pairs);
  const int pieces = (a.width + P - 1) / P;
  OZ2_TOKENS(t, lane) {
    const int* sl = a.slots + t * a.top_k;
    const float* wt = a.weights ? a.weights + t * a.top_k : nullptr;
    for (int c = lane + LPR * (int)blockIdx.y; c < pieces; c += LPR * (int)gridDim.y) {
      const int valid = a.width - c * P;
      const Piece<T, P> v = load_piece<T>(x + t * ldx + (ll)c * P, valid);
      for (int j = 0; j < a.top_k; ++j) {
        const int s = sl[j];
        if (s < 0 || s >= pairs) continue;
        Piece<T, P> o = v;
        if (s >= kept) {
#pragma unroll
          for (int i = 0; i < P; ++i) o.v[i] = (T)0.0f;
        } else if (wt) {
          const float f = wt[j];
#pragma unroll
          for (int i = 0; i < P; ++i) o.v[i] = from_f<T>(f * to_f(v.v[i]));
        }
        store_stream(xs + s * ldxs + (ll)c * P, o, valid);
      }
    }
  }
}

// Y = residual + sum over the places of weight x Ys, in 32 bits and in the order of the
// choices
template <class T, int LPR>
__global__ void __launch_bounds__(256)
k_combine(Oz2Tokens a, const T* __restrict__ ys, ll ldys, const T* res, ll ldr, T* y, ll ldy) {
  constexpr int P = 16 / sizeof(T), UN = 4;
  const int kept = min(*a.kept, a.tokens * a.top_k);
  const int pieces = (a.width + P - 1) / P;
  OZ2_TOKENS(t, lane) {
    const int* sl = a.slots + t * a.top_k;
    const float* wt = a.weights ? a.weights + t * a.top_k : nullptr;
    for (int c = lane + LPR * (int)blockIdx.y; c < pieces; c += LPR * (int)gridDim.y) {
      const int valid = a.width - c * P;
      float sum[P];
      if (res) {
        const Piece<T, P> r = load_piece<T>(res + t * ldr + (ll)c * P, valid);
#pragma unroll
        for (int i = 0; i < P; ++i) sum[i] = to_f(r.v[i]);
      } else {
#pragma unroll
        for (int i = 0; i < P; ++i) sum[i] = 0.0f;
      }
      for (int j0 = 0; j0 < a.top_k; j0 += UN) {   // UN rows in flight
        Piece<T, P> v[UN];
        float f[UN];
        bool on[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          const int j = j0 + u;
          const int s = j < a.top_k ? sl[j] : -1;
          on[u] = s >= 0 && s < kept;
          f[u] = on[u] && wt ? wt[j] : 1.0f;
          if (on[u]) v[u] = load_piece<T>(ys + s * ldys + (ll)c * P, valid);
        }
#pragma unroll
        for (int u = 0; u < UN; ++u)
          if (on[u]) {
#pragma unroll
            for (int i = 0; i < P; ++i) sum[i] += f[u] * to_f(v[u].v[i]);
          }
      }
      Piece<T, P> o;
#pragma unroll
      for (int i = 0; i < P; ++i) o.v[i] = from_f<T>(sum[i]);
      store_stream(y + t * ldy + (ll)c * P, o, valid);
    }
  }
}

// dYs = weight x dY at a place, dweight = <dY, Ys there>.  UN places at a time: dY's
// piece is read once for them.  The dot products are
// joined over the LPR lanes in a fixed order.
template <class T, int LPR>
__global__ void __launch_bounds__(256)
k_combine_backward(Oz2Tokens a, const T* __restrict__ dy, ll lddy, const T* __restrict__ ys, ll ldys,
                   T* __restrict__ dys, ll lddys, float* __restrict__ dw) {
  constexpr int P = 16 / sizeof(T), UN = 4;
  __shared__ float red[4][UN];
  const int pairs = a.tokens * a.top_k, kept = min(*a.kept, pairs);
  const int pieces = (a.width + P - 1) / P;
  OZ2_TOKENS(t, lane) {   // (LPR = 256: one token a workgroup, so its barriers are met by all)
    const int* sl = a.slots + t * a.top_k;
    const float* wt = a.weights + t * a.top_k;
    for (int j0 = 0; j0 < a.top_k; j0 += UN) {
      int s[UN];
      float f[UN], dot[UN];
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const int j = j0 + u;
        s[u] = j < a.top_k ? sl[j] : -1;
        if (s[u] >= pairs) s[u] = -1;
        f[u] = s[u] >= 0 && s[u] < kept ? wt[j] : 0.0f;
        dot[u] = 0.0f;
      }
      for (int c = lane; c < pieces; c += LPR) {
        const int valid = a.width - c * P;
        const Piece<T, P> g = load_piece<T>(dy + t * lddy + (ll)c * P, valid);
        Piece<T, P> v[UN];
        if (dw) {
#pragma unroll
          for (int u = 0; u < UN; ++u)
            if (s[u] >= 0 && s[u] < kept) v[u] = load_piece<T>(ys + s[u] * ldys + (ll)c * P, valid);
        }
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          if (s[u] < 0) continue;
          const bool on = s[u] < kept;
          if (dw && on) {
#pragma unroll
            for (int i = 0; i < P; ++i) dot[u] += to_f(g.v[i]) * to_f(v[u].v[i]);
          }
          if (dys) {
            Piece<T, P> o;
#pragma unroll
            for (int i = 0; i < P; ++i) o.v[i] = from_f<T>(on ? f[u] * to_f(g.v[i]) : 0.0f);
            store_stream(dys + s[u] * lddys + (ll)c * P, o, valid);
          }
        }
      }
      if (!dw) continue;
#pragma unroll
      for (int u = 0; u < UN; ++u)
#pragma unroll
        for (int d = 1; d < (LPR < 64 ? LPR : 64); d <<= 1) dot[u] += __shfl_xor(dot[u], d);
      if (LPR > 64) {
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
          for (int u = 0; u < UN; ++u) red[threadIdx.x >> 6][u] = dot[u];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < UN; ++u) dot[u] = (red[0][u] + red[1][u]) + (red[2][u] + red[3][u]);
        __syncthreads();
      }
      if (lane == 0) {
#pragma unroll
        for (int u = 0; u < UN; ++u)
          if (j0 + u < a.top_k) dw[t * a.top_k + j0 + u] = dot[u];
      }
    }
  }
}

// workgroups over the tokens, and over pieces of long rows until the chip is full
dim3 row_grid(int tokens, int lpr, int pieces) {
  const ll bx = std::min(ROW_BLOCKS, ((ll)tokens * lpr + 255) / 256);
  const int want = (int)std::max<ll>(1, 2 * oz2_device_cus() / bx);
  return dim3((unsigned)bx, (unsigned)std::min(want, (pieces + lpr - 1) / lpr));
}

int lanes_per_row(int pieces) { return pieces <= 8 ? 8 : pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64; }

}  // namespace

#define OZ2_TYPE(dtype, ...)                               \
  do {                                                     \
    if ((dtype) == OZ2_F32) { typedef float T; __VA_ARGS__; }    \
    else if ((dtype) == OZ2_F16) { typedef _Float16 T; __VA_ARGS__; } \
    else { typedef __bf16 T; __VA_ARGS__; }                \
  } while (0)
#define OZ2_LANES(lpr, kern, ...)                          \
  do {                                                     \
    if ((lpr) == 8) { auto* f = kern<T, 8>; __VA_ARGS__; }       \
    else if ((lpr) == 16) { auto* f = kern<T, 16>; __VA_ARGS__; } \
    else if ((lpr) == 32) { auto* f = kern<T, 32>; __VA_ARGS__; } \
    else { auto* f = kern<T, 64>; __VA_ARGS__; }                 \
  } while (0)

// workgroups of the sort: one where its own loop is shorter than a second launch, at
// most 256 (each adds up the counts of all)
int oz2_sort_blocks(ll pairs) {
  if (pairs <= 2 * SORT_CHUNK) return 1;
  return (int)std::min<ll>(256, (pairs + SORT_CHUNK - 1) / SORT_CHUNK);
}

hipError_t oz2_launch_sort(int tokens, int top_k, int E, const void* ids, bool wide, ll ld, int* offsets,
                           int* rows, int* slots, int* counts, hipStream_t s) {
  const ll pairs = (ll)tokens * top_k;
  int nb = oz2_sort_blocks(pairs);
  const ll chunk = std::max<ll>(1, ((pairs + nb - 1) / nb + SORT_CHUNK - 1) / SORT_CHUNK) * SORT_CHUNK;
  nb = std::max(1, (int)((pairs + chunk - 1) / chunk));
  SortArgs a{ids, ld, top_k, E, (int)pairs, (int)chunk, wide};
  if (nb > 1) {
    hipLaunchKernelGGL(k_sort_count, dim3(nb), dim3(SORT_NT), 0, s, a, counts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_sort_place, dim3(nb), dim3(SORT_NT), 0, s, a, counts, offsets, rows, slots);
  return hipGetLastError();
}

hipError_t oz2_launch_gather(int dtype, const Oz2Tokens& t, const void* x, ll ldx, void* xs, ll ldxs,
                             hipStream_t s) {
  OZ2_TYPE(dtype, {
    const int pieces = (t.width + 16 / (int)sizeof(T) - 1) / (16 / (int)sizeof(T));
    const int lpr = lanes_per_row(pieces);
    OZ2_LANES(lpr, k_gather, hipLaunchKernelGGL(f, row_grid(t.tokens, lpr, pieces), dim3(256), 0, s, t,
                                                (const T*)x, ldx, (T*)xs, ldxs));
  });
  return hipGetLastError();
}

hipError_t oz2_launch_combine(int dtype, const Oz2Tokens& t, const void* ys, ll ldys, const void* res,
                              ll ldr, void* y, ll ldy, hipStream_t s) {
  OZ2_TYPE(dtype, {
    const int pieces = (t.width + 16 / (int)sizeof(T) - 1) / (16 / (int)sizeof(T));
    const int lpr = lanes_per_row(pieces);
    OZ2_LANES(lpr, k_combine, hipLaunchKernelGGL(f, row_grid(t.tokens, lpr, pieces), dim3(256), 0, s, t,
                                                 (const T*)ys, ldys, (const T*)res, ldr, (T*)y, ldy));
  });
  return hipGetLastError();
}

hipError_t oz2_launch_combine_backward(int dtype, const Oz2Tokens& t, const void* dy, ll lddy,
                                       const void* ys, ll ldys, void* dys, ll lddys, float* dw,
                                       hipStream_t s) {
  OZ2_TYPE(dtype, {
    const int pieces = (t.width + 16 / (int)sizeof(T) - 1) / (16 / (int)sizeof(T));
    if (pieces > 128) {
      hipLaunchKernelGGL((k_combine_backward<T, 256>), dim3((unsigned)std::min<ll>(t.tokens, ROW_BLOCKS)), dim3(256), 0, s,
                         t, (const T*)dy,
                         lddy, (const T*)ys, ldys, (T*)dys, lddys, dw);
    } else {
      const int lpr = lanes_per_row(pieces);
      const unsigned bx = (unsigned)std::min(ROW_BLOCKS, ((ll)t.tokens * lpr + 255) / 256);
      OZ2_LANES(lpr, k_combine_backward, hipLaunchKernelGGL(f, dim3(bx), dim3(256), 0, s, t, (const T*)dy,
                                                            lddy, (const T*)ys, ldys, (T*)dys, lddys, dw));
    }
  });
  return hipGetLastError();
}
