// Definitions shared by the host code and the kernels of the layer operators
// (include/ozaki2/layers.h): element types, activations, 16-byte pieces of rows,
// the groups of rows, and the launchers.  Not part of the public ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ozaki2/layers.h"

typedef long long ll;

int oz2_device_cus();   // as in oz2_internal.h
int oz2_device_ok();

// Groups of rows: group g is rows [offsets[g], offsets[g+1]) of `rows`, clamped
// so that whatever the array holds, no row index leaves [0, rows] and no count of rows
// over several groups passes `rows`.
// offsets null: one group of all rows.
struct Oz2Groups {
  const int* offsets;
  int groups;
  int rows;
};

// D[i][j] = sum over l < L of A(i, l) B(j, l), i < M, j < N2.
enum Oz2Side {
  OZ2_FWD,     // A = X, B = W: both with l contiguous; epilogue
  OZ2_DGRAD,   // A = dZ (l contiguous), B = W (j contiguous)
  OZ2_WGRAD    // A = dZ, B = X: i and j contiguous
};

// What becomes of a product's sums
enum Oz2End {
  OZ2_END_Y,     // y (and z) with bias, activation and residual, or parts of a split sum
  OZ2_END_LSE,   // FWD: of each row's columns, a chunk at a time, the largest and the sum of exponentials
  OZ2_END_DZ,    // FWD: the gradient of the loss at the logits
  OZ2_END_SUM    // DGRAD, WGRAD: y, or added to the parts of the sum so far
};

// The loss over a vocabulary: its rows, and how far its sums have come
struct Oz2Chunk {
  float top, sum;        // the largest z; the sum of e^(z - top)
};
struct alignas(16) Oz2LossRow {
  float lse, factor;
  int target;            // -1: the row does not count
  int unused;
};
struct Oz2Loss {
  const void* targets;   // LSE: one for each row, int or long long
  int wide;
  Oz2Chunk* chunks;      // LSE: [chunk][M]
  float* picked;         // LSE: [M], the target's logit (where the row has one)
  const Oz2LossRow* rows;   // DZ: [M]
  bool twin;             // DZ: what the rounding leaves of row t goes to row M + t
  int first;             // DZ: the vocabulary's index of column 0
  const float* scale;    // SUM: null, or [1] is what the sums are multiplied by at last
  int whole, more;       // SUM: y at once; added to what part holds already
};

struct Oz2Product {
  const void *A, *B;
  ll lda, ldb;           // elements between rows of A and B as they lie in memory
  int M, N2, L;          // WGRAD: L = all rows, its groups give each product its own range
  Oz2Groups gr;          // FWD, DGRAD: groups of rows i; WGRAD: of l
  ll strideB;            // FWD, DGRAD: elements between the groups' B; WGRAD: between their D
  const void* bias;
  ll stride_bias;
  const void* res;
  ll ldr;
  void* y;               // D, or f(..) of it in FWD: N columns
  ll ldy;
  void* z;
  ll ldz;
  int N;                 // columns of y (N2, gated N2 / 2)
  int act, gated;
  bool padded, paddedB;  // A's (B's) rows go on, in zeros, to a multiple of 16 bytes
  void* packed;          // room for the copies that the plan asks for
  float* part;           // splits > 1: [split][M][N2] partial sums
  int splits, esize;     // (set by the launcher)
  Oz2Loss loss;
};

// How a product runs: `rows` > 0: the kernel of few rows, that many blocks of 16 at a
// time (1 or 2; FWD); else tiles of 256 (16 bits), 128 or 64 rows and columns, the sum in
// how many parts, joined by a second launch.
struct Oz2Plan {
  int rows;
  int tile;
  int splits;
  int pack;              // 1: A, 2: B is first copied into rows of whole lines
  size_t packed_bytes;
};
inline ll oz2_packed_pitch(ll cols, size_t e) { return (cols * (ll)e + 127) / 128 * 128 / (ll)e; }
// padded: 1 A, 2 B, as in Oz2Product; whole: the sum is not split
Oz2Plan oz2_plan(int dtype, Oz2Side side, ll M, ll N2, ll L, const Oz2Groups& gr,
                 int padded = 0, bool whole = false);
// the plan of a product (side 0, 1, 2; groups 0: one product) as rows, tile, splits and
// pack: a diagnostic for tests, not part of the public ABI
extern "C" void oz2_plan_of(int dtype, int side, ll M, ll N2, ll L, int rows, int groups, int padded,
                            int* out);

#ifdef __HIPCC__
// products and sums of the epilogues may be fused; nothing here is compared bit for bit
#pragma clang fp contract(fast)
namespace {

template <class T>
__device__ __forceinline__ float to_f(T v) {
  return (float)v;
}
template <class T>
__device__ __forceinline__ T from_f(float v) {
  return (T)v;   // to nearest even; fp16 overflows to infinity
}

// N elements that move as one piece, from and to any element-aligned address
// (gfx950 serves unaligned 16-byte accesses in one instruction)
template <class T, int N>
struct Piece {
  T v[N];
};
template <class T, int N = 16 / (int)sizeof(T)>
__device__ __forceinline__ Piece<T, N> load_piece(const T* p, int valid) {
  Piece<T, N> r;
  if (valid >= N) {
    __builtin_memcpy(&r, p, sizeof(r));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = i < valid ? p[i] : (T)0.0f;
  }
  return r;
}
template <class T, int N>
__device__ __forceinline__ void store_piece(T* p, const Piece<T, N>& r, int valid) {
  if (valid >= N) {
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < valid) p[i] = r.v[i];
  }
}
// The same past the caches, for outputs written once (8-byte pieces and ends of rows
// go the ordinary way): a gather of 1 GiB 387 -> 206 us, 16384^2 outputs of a product over
// 4096 1740 -> 1582.
template <class T, int N>
__device__ __forceinline__ void store_stream(T* p, const Piece<T, N>& r, int valid) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
  if constexpr (sizeof(r) == 16) {
    if (valid >= N) {
      __builtin_nontemporal_store(__builtin_bit_cast(u4, r), reinterpret_cast<u4*>(p));
      return;
    }
  }
  store_piece(p, r, valid);
}
// A piece that nobody reads again soon, past the caches likewise (the slope of 16384 x 2048
// entries 62 -> 54 us)
template <class T, int N = 16 / (int)sizeof(T)>
__device__ __forceinline__ Piece<T, N> load_stream(const T* p, int valid) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
  if (valid >= N)
    return __builtin_bit_cast(Piece<T, N>, __builtin_nontemporal_load(reinterpret_cast<const u4*>(p)));
  return load_piece<T, N>(p, valid);
}

// f(x) and f'(x).  16-bit results take the hardware's exponential, fp32 ones the
// library's.  The former takes x log2(e) rounded to 32 bits, which alone is off by some |x|
// 2^-24 relatively (e^-80: 2^-18), beside the instruction's own 2^-23: little against the
// 2^-11 and 2^-8 that the results keep.
template <class T>
__device__ __forceinline__ float exp_for(float x) {
  return sizeof(T) == 4 ? expf(x) : __expf(x);
}
// 1 / (1 + e^-x): 0 and 1 at the ends (e^-x may be infinite)
template <class T>
__device__ __forceinline__ float sigmoid(float x) {
  return sizeof(T) == 4 ? 1.0f / (1.0f + expf(-x)) : __builtin_amdgcn_rcpf(1.0f + __expf(-x));
}

constexpr float kHalfRoot = 0.70710678118654752f;      // 1 / sqrt 2
constexpr float kGauss = 0.39894228040143268f;         // 1 / sqrt(2 pi)
constexpr float kTanh = 1.5957691216057308f;           // 2 sqrt(2 / pi)

// Phi(x), the normal distribution, and in *bell e^(-x^2/2).  16 bits: Abramowitz and
// Stegun's 7.1.26, erfc(q) = e^(-q^2) (a1 t + .. + a5 t^5), t = 1 / (1 + 0.3275911 q), q
// >= 0, good to 1.5e-7, which shares its exponential with the slope and takes a
// quarter of the library's erfc (the slope of 4096^2 bf16 entries: 58 us with that).  Of
// the value itself that is 0.05% at x = -4 (a result of 1e-4) and, by the fit's asymptote,
// 1% at -8 (5e-15) and 3% at -12: 1 + erf in 32 bits holds nothing there.
template <class T>
__device__ __forceinline__ float gauss_tail(float x, float* bell) {
  if (sizeof(T) == 4) {
    if (bell) *bell = expf(-0.5f * x * x);
    return 0.5f * erfcf(-x * kHalfRoot);
  }
  const float q = fabsf(x) * kHalfRoot, e = __expf(-0.5f * x * x);
  const float t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * q);
  const float half = 0.5f * e * t *
      (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
  if (bell) *bell = e;
  return x > 0.0f ? 1.0f - half : half;
}

template <class T>
__device__ __forceinline__ float act_f(float x, int act) {
  switch (act) {
    case OZ2_ACT_RELU:
      return x < 0.0f ? 0.0f : x;          // NaN stays
    case OZ2_ACT_GELU:
      return x * gauss_tail<T>(x, nullptr);
    case OZ2_ACT_GELU_TANH:                // 0.5 (1 + tanh(q)) = sigmoid(2 q)
      return x * sigmoid<T>(kTanh * (x + 0.044715f * x * x * x));
    case OZ2_ACT_SILU:
      return x * sigmoid<T>(x);
    default:
      return x;
  }
}

// Where the bell-shaped factor of the second term has underflowed the term is 0,
// whatever the powers of x beside it.
template <class T>
__device__ __forceinline__ float act_d(float x, int act) {
  switch (act) {
    case OZ2_ACT_RELU:
      return x > 0.0f ? 1.0f : (x <= 0.0f ? 0.0f : x);
    case OZ2_ACT_GELU: {
      float b;
      const float s = gauss_tail<T>(x, &b);
      return b == 0.0f ? s : s + x * kGauss * b;
    }
    case OZ2_ACT_GELU_TANH: {
      const float s = sigmoid<T>(kTanh * (x + 0.044715f * x * x * x)), b = s * (1.0f - s);
      return b == 0.0f ? s : s + x * b * kTanh * (1.0f + 0.134145f * x * x);
    }
    case OZ2_ACT_SILU: {
      const float s = sigmoid<T>(x), b = s * (1.0f - s);
      return b == 0.0f ? s : s + x * b;
    }
    default:
      return 1.0f;
  }
}

__device__ __forceinline__ int group_start(const Oz2Groups& g, int i) {
  return min(max(g.offsets[i], 0), g.rows);
}
// rows [start, end) of group i
__device__ __forceinline__ void group_range(const Oz2Groups& g, int i, int& start, int& end) {
  if (!g.offsets) {
    start = 0;
    end = g.rows;
    return;
  }
  start = group_start(g, i);
  end = max(start, group_start(g, i + 1));
}

// Rows [start, end) of group i = g0 + lane, g0 = 0, 64, .. in turn, where what all groups
// have is added up: a group starts no earlier than the ones before it, so that whatever
// the array holds, all of them together are at most `rows` (ascending offsets: as
// group_range).  high: 0 at first, then the end of the groups before.  Every lane of the
// wave calls it; groups that do not exist are empty.
__device__ __forceinline__ void ascending_ranges(const Oz2Groups& g, int g0, int& high, int& start,
                                                 int& end) {
  const int lane = threadIdx.x & 63, i = g0 + lane;
  start = i < g.groups ? group_start(g, i) : 0;
  end = i < g.groups ? group_start(g, i + 1) : 0;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(start, d);
    if (lane >= d) start = max(start, up);
  }
  start = max(start, high);
  end = max(start, end);
  high = __shfl(end, 63);
}

// Row tiles of `tile` rows that the groups have.  Every lane of the wave calls it;
// the result is uniform.
__device__ __forceinline__ int group_tiles(const Oz2Groups& g, int tile) {
  if (!g.offsets) return (int)(((ll)g.rows + tile - 1) / tile);
  int n = 0, high = 0;
  for (int g0 = 0; g0 < g.groups; g0 += 64) {
    int s, e;
    ascending_ranges(g, g0, high, s, e);
    n += (e - s + tile - 1) / tile;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) n += __shfl_xor(n, d);
  return __builtin_amdgcn_readfirstlane(n);
}

// Tile t < group_tiles() of the row tiles of all groups in turn: its group, that group's
// first tile, and its rows [row, end).  Likewise uniform.
__device__ __forceinline__ void group_tile(const Oz2Groups& g, int tile, int t, int& group, int& first,
                                           int& row, int& end) {
  group = first = 0;
  row = t * tile;
  end = g.rows;
  if (!g.offsets) return;
  const int lane = threadIdx.x & 63;
  int before = 0, high = 0;
  for (int g0 = 0; g0 < g.groups; g0 += 64) {
    int s, e;
    ascending_ranges(g, g0, high, s, e);
    const int mine = (e - s + tile - 1) / tile;
    int sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(sum, d);
      if (lane >= d) sum += up;
    }
    const unsigned long long hit = __ballot(before + sum > t);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;
      group = __builtin_amdgcn_readfirstlane(g0 + l);
      first = __builtin_amdgcn_readfirstlane(__shfl(before + sum - mine, l));
      row = __builtin_amdgcn_readfirstlane(__shfl(s, l) + (t - first) * tile);
      end = __builtin_amdgcn_readfirstlane(__shfl(e, l));
      return;
    }
    before += __shfl(sum, 63);
  }
}

// The row tiles of the groups before `group`, and its own.  Likewise uniform.
__device__ __forceinline__ void group_tiles_before(const Oz2Groups& g, int tile, int group, int& first,
                                                   int& count) {
  first = 0;
  if (!g.offsets) {
    count = (int)(((ll)g.rows + tile - 1) / tile);
    return;
  }
  const int lane = threadIdx.x & 63;
  int high = 0;
  for (int g0 = 0; g0 <= group; g0 += 64) {
    int s, e;
    ascending_ranges(g, g0, high, s, e);
    const int mine = (e - s + tile - 1) / tile;
    if (g0 + lane < group) first += mine;
    count = __shfl(mine, (group - g0) & 63);   // (the last round's: of group itself)
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) first += __shfl_xor(first, d);
}

// Workgroup b's place in an order of n items in which each XCD (workgroups go
// round-robin over the eight of them, each with an L2 of its own) has a contiguous
// eighth.  -1 where it has none; items take 8 ceil(n / 8) workgroups.
__device__ __forceinline__ ll xcd_order(ll b, ll n) {
  const ll per = (n + 7) >> 3, p = (b & 7) * per + (b >> 3);
  return (b >> 3) < per && p < n ? p : -1;
}

// Tile p of nrow x ncol tiles in bands of four rows of tiles, the last of up to seven, a
// band column by column: 32 workgroups that run together (an XCD's) share 4 to 7 panels
// of A and 8 to 5 of B.
__device__ __forceinline__ void banded(ll p, int nrow, int ncol, int& r, int& c) {
  const int last = max(nrow / 4 - 1, 0), band = (int)min(p / (4ll * ncol), (ll)last);
  const int in = (int)(p - band * 4ll * ncol), h = band == last ? nrow - 4 * band : 4;
  c = in / h;
  r = band * 4 + in - c * h;
}

}  // namespace
#endif

// most row tiles of `tile` rows that groups of `rows` rows in all can make, with
// those of the rows outside
inline ll oz2_row_tiles(const Oz2Groups& g, int tile) {
  return g.offsets ? (ll)g.rows / tile + g.groups + 1 : ((ll)g.rows + tile - 1) / tile;
}
// workgroups for them and ncol tiles across: a multiple of eight in the groups' order,
// then those of the rows outside
inline ll oz2_tile_blocks(const Oz2Groups& g, int tile, int ncol) {
  return (oz2_row_tiles(g, tile) * ncol + 7) / 8 * 8 + (g.offsets ? 8 : 0);
}

// A grid of `blocks` workgroups of 256 threads: HIP takes fewer than 2^32 threads along x
// (2^30 rows in 64-row tiles are that many), so beyond 2^24 - 8 workgroups it goes on
// along y, in whole rounds of the XCDs.
struct Oz2Grid {
  unsigned x, y;
};
inline Oz2Grid oz2_grid(ll blocks) {
  const ll most = (1 << 24) - 8;
  return blocks <= most ? Oz2Grid{(unsigned)blocks, 1u}
                        : Oz2Grid{(unsigned)most, (unsigned)((blocks + most - 1) / most)};
}

// ---------------------------------------------------------------- launchers
hipError_t oz2_launch_product(int dtype, Oz2Side side, const Oz2Plan& plan, const Oz2Product& p,
                              hipStream_t s);
// dZ (pitch ldd, a multiple of 64 bytes; entries beyond n2 zero) from dY and Z,
// or nothing of it where dz is null; column sums of dZ into db where not null,
// by way of part ([row tile][n2])
struct Oz2Slope {
  const void* dy;
  ll lddy;
  const void* z;
  ll ldz;
  void* dz;
  ll ldd;
  int n, act, gated;
  Oz2Groups gr;
  void* db;
  ll stride_db;
  float* part;
  int sum_rows;          // rows per partial column sum (set by the launcher)
};
#define OZ2_SUM_ROWS 32   // the least of it: part holds a row for each of as many
hipError_t oz2_launch_slope(int dtype, const Oz2Slope& p, hipStream_t s);

struct Oz2Tokens {
  int tokens, top_k, width;
  const int* slots;
  const int* kept;
  const float* weights;
};
hipError_t oz2_launch_sort(int tokens, int top_k, int E, const void* ids, bool wide, ll ld, int* offsets,
                           int* rows, int* slots, int* counts, hipStream_t s);
int oz2_sort_blocks(ll pairs);
hipError_t oz2_launch_gather(int dtype, const Oz2Tokens& t, const void* x, ll ldx, void* xs, ll ldxs,
                             hipStream_t s);
hipError_t oz2_launch_combine(int dtype, const Oz2Tokens& t, const void* ys, ll ldys, const void* res,
                              ll ldr, void* y, ll ldy, hipStream_t s);
hipError_t oz2_launch_combine_backward(int dtype, const Oz2Tokens& t, const void* dy, ll lddy,
                                       const void* ys, ll ldys, void* dys, ll lddys, float* dw,
                                       hipStream_t s);
