// The router: every token's experts and their weights from its logits, and the gradient.
//
// L lanes have a token, lane l of them its experts l V .. l V + V - 1, in registers; a wave has
// 64 / L tokens.  Rows of logits are read once, and the bytes are few (16384 tokens of 256
// experts: 17 MB, 3 us): what bounds it is the search for the largest values, some 30
// instructions a choice and token.  16384 tokens, 8 choices: of 256 experts by the logits'
// order 10 us, by scores with a bias 19, in 8 groups 24-27 by card (a group's two largest are one
// lane's search in LDS, so that 8 of a token's 32 lanes work); of 64 experts 5.9, 8.8 and 11.  (All
// scores in 64 bits and a wave a token: 169 us in groups.)  Gradient, 16384 x 128 bf16: 7 us.
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
// (keys are no NaN: nothing is to be made quiet first)
__device__ __forceinline__ double larger(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ double smaller(double a, double b) {
  double r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ uint32_t smaller(uint32_t a, uint32_t b) { return min(a, b); }
__device__ __forceinline__ float value_of(uint32_t k) { return __builtin_bit_cast(float, k >> 31 ? k ^ 1u << 31 : ~k); }

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
// Returns the last one.
template <int L, int V, class KEY, class F>
__device__ __forceinline__ KEY take_largest(KEY (&key)[V], int n, int lane, F take) {
  KEY no, last;
  none(no);
  none(last);
  for (int r = 0; r < n; ++r) {
    KEY mine = key[0];
#pragma unroll
    for (int i = 1; i < V; ++i) mine = larger(mine, key[i]);
    const KEY best = largest<L>(mine);
    if (best != no) last = best;
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
  return last;
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
    for (int i = 0; i < V; ++i) l[i] = to_f(row[min(first + i, E - 1)]);
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = first + i < E ? l[i] : -INFINITY;
  }
}

__device__ __forceinline__ double sigmoid64(float l) { return 1.0 / (1.0 + exp(-(double)l)); }

// The keys of groups first .. end - 1 of `per` keys each; sum: of the two largest, joined by
// add.  (Each lane starts elsewhere in its group: LDS's banks.)
template <int L, class KEY, class F, class G>
__device__ __forceinline__ void group_keys(const KEY* keys, int per, int first, int end, bool sum, int lane, F add,
                                           G give) {
  KEY no;
  none(no);
#pragma clang loop unroll(disable)
  for (int g = first; g < end; ++g) {
    KEY b1 = no, b2 = no;
    int e = lane % per;
#pragma clang loop unroll_count(4)
    for (int n = 0; n < per; ++n) {
      const KEY c = keys[g * per + e];
      e = e + 1 == per ? 0 : e + 1;
      b2 = larger(b2, smaller(b1, c));
      b1 = larger(b1, c);
    }
    give(g, sum && b2 != no ? add(b1, b2) : b1);
  }
}

// Keys of experts in groups (of two at least) that do not stay are taken out
template <int L, int V>
__device__ __forceinline__ void drop_groups(uint32_t (&key)[V], const uint8_t* stays, int E, int groups, int lane) {
  const uint32_t inverse = 0xffffffffu / (uint32_t)(E / groups) + 1;   // e / per = e inverse / 2^32
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (!stays[__umulhi(min(lane * V + i, E - 1), inverse)]) key[i] = 0;
}

// The same from the keys themselves.  Returns the last group's value
// that stays, and in *next the largest that does not (none: there is none).
template <int L, int V, class F>
__device__ __forceinline__ uint32_t keep_groups(uint32_t (&key)[V], uint32_t* keys, uint8_t* stays, int E, int groups,
                                                int top_groups, bool sum, int lane, uint32_t* next, F add) {
  const int per = E / groups, first = lane * V;
#pragma unroll
  for (int i = 0; i < V; ++i) keys[first + i] = key[i];
  for (int g = lane; g < groups; g += L) stays[g] = 0;
  wave_fence();
  auto stay = [&](int, int g) { stays[g] = 1; };
  uint32_t last;
  if (groups <= L) {
    uint32_t gk[1] = {0};
    group_keys<L>(keys, per, lane, min(groups, lane + 1), sum, lane, add, [&](int, uint32_t k) { gk[0] = k; });
    last = take_largest<L, 1>(gk, top_groups, lane, stay);
    *next = largest<L>(gk[0]);
  } else {
    // (by way of LDS, behind the experts' keys: there is room for V a lane)
    uint32_t* const values = keys + L * V;
    group_keys<L>(keys, per, first, min(groups, first + V), sum, lane, add, [&](int g, uint32_t k) { values[g] = k; });
    wave_fence();
    uint32_t gk[V], rest = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) gk[i] = first + i < groups ? values[first + i] : 0;
    last = take_largest<L, V>(gk, top_groups, lane, stay);
#pragma unroll
    for (int i = 0; i < V; ++i) rest = larger(rest, gk[i]);
    *next = largest<L>(rest);
  }
  wave_fence();
  drop_groups<L, V>(key, stays, E, groups, lane);
  wave_fence();
  return last;
}

// The groups that stay, where 32 bits do not tell them from the next one: their values from the
// scores in 64 bits of the experts that can be a group's two largest.  keys: as keep_groups left them.
// False where there are too many of either (a lane has a group and four such experts).
template <int L, int V, class F>
__device__ __forceinline__ bool settle_groups(uint32_t (&key)[V], const uint32_t* keys, uint8_t* stays, int E,
                                              int groups, int top_groups, bool sum, float near, int lane, F score64) {
  if (groups > L) return false;
  const int per = E / groups;
  double value[1] = {-INFINITY};
  int hits = 0;
  if (lane < groups) {
    const uint32_t* mine = keys + lane * per;
    uint32_t b1 = 0, b2 = 0;
    for (int e = 0; e < per; ++e) {
      b2 = max(b2, min(b1, mine[e]));
      b1 = max(b1, mine[e]);
    }
    const float least = value_of(sum && b2 ? b2 : b1) - near;
    uint64_t which = 0;
    for (int e = 0; e < per; ++e)
      if (mine[e] && value_of(mine[e]) >= least) {
        if (hits < 4) which |= (uint64_t)(lane * per + e) << 16 * hits;
        ++hits;
      }
    double d1 = -INFINITY, d2 = -INFINITY;
#pragma clang loop unroll(disable)
    for (int h = 0; h < min(hits, 4); ++h) {
      const double s = score64((int)(which >> 16 * h) & 0xffff);
      d2 = larger(d2, smaller(d1, s));
      d1 = larger(d1, s);
    }
    value[0] = sum && d2 > -INFINITY ? d1 + d2 : d1;
    stays[lane] = 0;
  }
  if (of_token<L>(__ballot(hits > 4))) return false;
  take_largest<L, 1>(value, top_groups, lane, [&](int, int g) { stays[g] = 1; });
  wave_fence();
#pragma unroll
  for (int i = 0; i < V; ++i) key[i] = keys[lane * V + i];
  drop_groups<L, V>(key, stays, E, groups, lane);
  return true;
}

// take_largest of n keys in LDS (each lane a run of them): seldom called, and in few registers,
// which the rest would have to do without
template <int L, class F>
__device__ __forceinline__ void take_largest_lds(double* keys, int n, int k, int lane, F take) {
  const int each = (n + L - 1) / L, first = lane * each, end = min(n, first + each);
#pragma clang loop unroll(disable)
  for (int r = 0; r < k; ++r) {
    double mine = -INFINITY;
    int at = first;
#pragma clang loop unroll_count(4)
    for (int e = first; e < end; ++e) {
      const double c = keys[e];
      at = c > mine ? e : at;
      mine = larger(mine, c);
    }
    const double best = largest<L>(mine);
    const uint64_t have = of_token<L>(__ballot(mine == best));
    if (best > -INFINITY && lane == __ffsll((unsigned long long)have) - 1) {
      keys[at] = -INFINITY;
      take(r, at);
    }
    wave_fence();
  }
}

// LDS of a wave: its tokens' choices, which of their groups stay, and room for one thing after the
// other: of each token the keys of experts and groups of 32 bits, or candidates with
// their scores; keys of 64 bits of one token at a time.  (Groups are of two experts at least.)
constexpr int CAND = 64;
template <int L, int V>
struct Lds {
  static constexpr int TOKENS = 64 / L, STAYS = TOKENS * OZ2_MAX_TOPK * 4, ROOM = STAYS + TOKENS * L * V;
  static constexpr int EACH = std::max(L * V * (L < 64 ? 6 : 12), CAND * 12), WAVE = ROOM + TOKENS * EACH;
  static_assert(TOKENS * EACH >= L * V * 12 && ROOM % 8 == 0 && EACH % 8 == 0 && WAVE % 8 == 0, "room");
};

// Choices by scores (SCORED) or by the logits, whose order is that of scores without a bias.
// Scores are compared as in 64 bits, for biased ones lie closer together than 32 bits tell, but
// 64 bits are formed for few: 32 bits find those that can be among the largest, within `near`
// of the last of them, and those are ranked.  near is twice the error of c = s + b: A of the score
// (sigmoid: s (1 - s) (|l| 2^-24 + 2^-23) and two roundings, 3e-7 at most; softmax: of its
// largest score, |x| e^x being below 0.37), and of the sum 2^-24 |c|, c the largest of the token's
// experts: a finite bias of -1e9 makes all others candidates (16384 tokens of 256 experts 20 -> 57
// us, in groups 25 -> 93), -infinity does not (19 and 27).  Groups whose values are
// that close are settled by the scores that can be their two largest.  Where none of that decides
// (a NaN, an infinity, more than 64 so close), a token's scores are all formed, in LDS
// and in loops: unrolled in registers they slowed down the rest (15 us to 35).
template <class T, bool SCORED, int L, int V>
__global__ void __launch_bounds__(NT, 4)
k_route(Oz2Route a) {
  constexpr int TOKENS = NT / L, Q = OZ2_MAX_TOPK / L;
  typedef Lds<L, V> Part;
  __shared__ __attribute__((aligned(8))) uint8_t lds[NT / 64 * Part::WAVE];
  const int lane = threadIdx.x % L, tok = threadIdx.x % 64 / L, E = a.experts, first = lane * V;
  uint8_t* const mine = lds + threadIdx.x / 64 * Part::WAVE;
  int* const chosen = (int*)mine + tok * OZ2_MAX_TOPK;
  uint8_t* const stays = mine + Part::STAYS + tok * L * V;
  uint8_t* const room = mine + Part::ROOM + tok * Part::EACH;
  const bool grouped = a.groups > 1 && a.groups < E;   // (groups of one: the experts themselves)
  const bool soft = a.score == OZ2_SCORE_SOFTMAX;
  {
    const int own = (int)blockIdx.x * TOKENS + (int)threadIdx.x / L;
    const bool live = own < a.tokens;
    const ll t = live ? own : a.tokens - 1;
    const T* row = (const T*)a.logits + t * a.ld;
    float l[V], b[V];
    load_logits<T, V>(row, first, E, l);
    if (SCORED) {
      if (a.bias) {
        load_logits<float, V>(a.bias, first, E, b);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) b[i] = 0.0f;
      }
    }
    float top = l[0], total = 1.0f;
    bool bad = !(l[0] < INFINITY);   // a logit that makes a softmax NaN
#pragma unroll
    for (int i = 1; i < V; ++i) {
      bad |= !(l[i] < INFINITY);
      top = fmaxf(top, l[i]);
    }
    bad = soft && of_token<L>(__ballot(bad));
    for (int j = lane; j < a.top_k; j += L) chosen[j] = -1;
    uint32_t key[V], after = 0;
    if (!SCORED) {
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
        if (l[i] == -INFINITY) key[i] = 0;
      }
      if (grouped)
        keep_groups<L, V>(key, (uint32_t*)room, stays, E, a.groups, a.top_groups, false, lane, &after,
                          [](uint32_t x, uint32_t) { return x; });
      wave_fence();
      take_largest<L, V>(key, a.top_k, lane, [&](int r, int e) { chosen[r] = e; });
    } else {
      float c[V], far = 0.0f, A = 5e-7f;
      double sum = 1.0;
      if (soft) {
        top = across<L, false>(top);
        sum = 0.0;
        // (a loop, its logits in LDS: the exponential of 64 bits is long)
        float* const z = (float*)room;
#pragma unroll
        for (int i = 0; i < V; ++i) z[first + i] = l[i];
        wave_fence();
#pragma clang loop unroll(disable)
        for (int i = 0; i < V; ++i) {
          const float v = z[first + i];
          sum += v == -INFINITY ? 0.0 : exp((double)v - (double)top);
        }
        wave_fence();
        sum = total_of<L>(sum);
        total = (float)sum;
        A /= total;   // (of the largest score; e^x in 32 bits is off by |x| 2^-24, and |x| e^x below 1)
        const float share = 1.0f / total;
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = __expf(l[i] - top) * share;
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = __builtin_amdgcn_rcpf(1.0f + __expf(-l[i]));
      }
      bool exact = false;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        c[i] += b[i];
        key_of(c[i], key[i]);
        if (l[i] == -INFINITY || b[i] == -INFINITY) {
          key[i] = 0;
          c[i] = -INFINITY;
        } else {
          exact |= !(fabsf(c[i]) < INFINITY);
          far = fmaxf(far, fabsf(c[i]));
        }
      }
      exact = of_token<L>(__ballot(exact));
      far = across<L, false>(far);
      const float near = 2.0f * (A + 2.4e-7f * far);
      // expert e's score and bias in 64 bits
      auto score64 = [&](int e) {
        const float z = to_f(row[e]);
        const double s = soft ? exp((double)z - (double)top) / sum : sigmoid64(z);
        return s + (a.bias ? (double)a.bias[e] : 0.0);
      };
      if (grouped) {
        const uint32_t least = keep_groups<L, V>(
            key, (uint32_t*)room, stays, E, a.groups, a.top_groups, a.group_best > 1, lane, &after,
            [](uint32_t x, uint32_t y) {
              uint32_t k;
              key_of(value_of(x) + value_of(y), k);
              return k;
            });
        // (sums of two; where both are beyond 32 bits their difference is no number)
        if (!exact && after && !(value_of(least) - value_of(after) > 3.0f * near))
          exact = !settle_groups<L, V>(key, (uint32_t*)room, stays, E, a.groups, a.top_groups, a.group_best > 1, near,
                                       lane, score64);
      }
      // the k-th value, or the least there is
      uint32_t kth = ~0u;
      for (int r = 0; r < a.top_k; ++r) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) m = max(m, key[i] < kth ? key[i] : 0u);
        m = largest<L>(m);
        kth = m ? m : kth;
      }
      const float least = value_of(kth) - near;
      int n = 0, before;
      bool in[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        in[i] = key[i] && c[i] >= least;
        n += in[i];
      }
      before = n;
#pragma unroll
      for (int d = 1; d < L; d *= 2) {
        const int up = __shfl_up(before, d, L);
        if (lane >= d) before += up;
      }
      const int count = __shfl(before, L - 1, L);
      exact |= count > CAND;
      wave_fence();
      if (!exact) {
        double* const score = (double*)room;
        int* const who = (int*)(score + CAND);
        int at = before - n;
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (in[i]) who[at++] = first + i;
        wave_fence();
        for (int j = lane; j < count; j += L) score[j] = score64(who[j]);
        wave_fence();
        for (int j = lane; j < count; j += L) {
          const double mine = score[j];
          const int e = who[j];
          int rank = 0;
          for (int i = 0; i < count; ++i) rank += score[i] > mine || (score[i] == mine && who[i] < e);
          if (rank < a.top_k) chosen[rank] = e;
        }
      }
      wave_fence();
      for (int q = 0; q < 64 / L; ++q) {
        if (q != tok || !exact) continue;
        // all of a token's keys in 64 bits: in few registers, which the rest would have to do without
        double* const keys = (double*)(mine + Part::ROOM);
#pragma clang loop unroll(disable)
        for (int e = lane; e < E; e += L) {
          const float z = to_f(row[e]), d = a.bias ? a.bias[e] : 0.0f;
          key_of(soft && bad ? __builtin_nan("") : score64(e), keys[e]);
          if (z == -INFINITY || d == -INFINITY) none(keys[e]);
        }
        wave_fence();
        if (grouped) {
          const int per = E / a.groups, each = (a.groups + L - 1) / L;
          double* const values = keys + L * V;
          for (int g = lane; g < a.groups; g += L) stays[g] = 0;
          group_keys<L>(keys, per, min(a.groups, lane * each), min(a.groups, lane * each + each), a.group_best > 1,
                        lane, [](double x, double y) { return x < INFINITY ? fmin(x + y, kMost) : x; },
                        [&](int g, double v) { values[g] = v; });
          wave_fence();
          take_largest_lds<L>(values, a.groups, a.top_groups, lane, [&](int, int g) { stays[g] = 1; });
#pragma clang loop unroll(disable)
          for (int e = lane; e < E; e += L)
            if (!stays[e / per]) keys[e] = -INFINITY;
          wave_fence();
        }
        take_largest_lds<L>(keys, E, a.top_k, lane, [&](int r, int e) { chosen[r] = e; });
        wave_fence();
      }
    }
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

// f(lanes a token, experts a lane) as types.  The fewest lanes that keep a lane's experts in
// registers: 16 experts and their scores do not fit beside what scores take
template <bool SCORED, class F>
hipError_t for_experts(int E, F f) {
  using std::integral_constant;
  if (E <= 16) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (E <= 32) return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  if (E <= 64) return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if (E <= 128) return f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  if (E <= 256) return f(integral_constant<int, SCORED ? 32 : 16>{}, integral_constant<int, SCORED ? 8 : 16>{});
  if (E <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  return f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

template <class T, bool SCORED>
hipError_t launch_route(const Oz2Route& a, hipStream_t s) {
  return for_experts<SCORED>(a.experts, [&](auto lanes, auto each) {
    constexpr int L = decltype(lanes)::value, V = decltype(each)::value, TOKENS = NT / L;
    hipError_t e = hipSuccess;
    // (launches of no more than a grid's workgroups)
    for (ll t = 0; t < a.tokens && e == hipSuccess; t += ROW_BLOCKS * TOKENS) {
      Oz2Route part = a;
      part.tokens = (int)std::min<ll>(ROW_BLOCKS * TOKENS, a.tokens - t);
      part.logits = (const T*)a.logits + t * a.ld;
      part.ids += t * a.top_k;
      part.weights += t * a.top_k;
      hipLaunchKernelGGL((k_route<T, SCORED, L, V>), dim3((unsigned)((part.tokens + TOKENS - 1) / TOKENS)), dim3(NT),
                         0, s, part);
      e = hipGetLastError();
    }
    return e;
  });
}

}  // namespace

hipError_t oz2_launch_route(int dtype, const Oz2Route& a, hipStream_t s) {
  const bool scored = a.bias || (a.groups > 1 && a.group_best > 1);
  OZ2_TYPED(dtype, return scored ? (launch_route<T, true>(a, s)) : (launch_route<T, false>(a, s)));
}

hipError_t oz2_launch_route_backward(int dtype, const Oz2RouteBack& a, hipStream_t s) {
  OZ2_TYPED(dtype, return for_experts<false>(a.experts, [&](auto lanes, auto each) {
              constexpr int L = decltype(lanes)::value, V = decltype(each)::value, TOKENS = NT / L;
              const dim3 grid((unsigned)std::min<ll>(ROW_BLOCKS, ((ll)a.tokens + TOKENS - 1) / TOKENS));
              hipLaunchKernelGGL((k_route_backward<T, L, V>), grid, dim3(NT), 0, s, a);
              return hipGetLastError();
            }));
}
