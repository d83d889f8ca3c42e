// Products of the layer operators on the matrix cores:
//   D[i][j] = sum over l of A(i, l) B(j, l),
// forward (A = X, B = W, both contiguous along l), the gradient of X (B = W
// contiguous along j) and of W (A = dZ contiguous along i, B = X along j), each
// for one product or for groups of rows.
//
// A step is 64 bytes of l (32 entries of 16 bits, 16 of 32), a stage two steps,
// for all rows of the workgroup's tiles, in LDS in the layout of its source, read as
// 16-byte fragments: lane (r = L%16, g = L/16) of a block of 16 rows holds row r and
// l = 8 g .. 8 g + 7 (16 bits) or 4 g .. 4 g + 3 (32 bits) of the step, which is one
// 16x16x32 instruction or four 16x16x4 ones.  Rows contiguous along l give a
// fragment as one read; the others through the transposing LDS read (16 bits:
// its 16 lanes read 4 l x 16 columns and each receives one column) or as four
// words (32 bits).
//
// The instruction's first operand is B, so that a lane's accumulators are four
// consecutive columns j of one row i of D.  They leave by way of LDS, a few rows of a
// wave's outputs at a time, so that the epilogue is a short loop over whole 16-byte
// pieces of rows (unrolled over the accumulators it was 330 KB of code, run once a
// tile: 30 us of instruction fetches).
#include <algorithm>
#include <type_traits>

#include "oz2_layers.h"

#pragma clang fp contract(fast)

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) uint8_t lds8;
typedef __attribute__((address_space(3))) v4s lds_v4s;

constexpr int SB2 = 128;   // bytes of l in a stage

// 16 bytes of operand
template <class T>
struct Frag;
template <>
struct Frag<__bf16> {
  v8b v;
};
template <>
struct Frag<_Float16> {
  v8h v;
};
template <>
struct Frag<float> {
  v4f v;
};

__device__ __forceinline__ v4f mma(const Frag<__bf16>& a, const Frag<__bf16>& b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ v4f mma(const Frag<_Float16>& a, const Frag<_Float16>& b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ v4f mma(const Frag<float>& a, const Frag<float>& b, v4f c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
  return c;
}

// The same with the accumulators in the accumulation registers for good: the compiler
// moves them to and fro where they take all of that half of the register file.  It
// sees no matrix instruction here, so the wait states before a result is read are
// the caller's (acc_settle).
__device__ __forceinline__ void mma_acc(const Frag<__bf16>& a, const Frag<__bf16>& b, v4f& c) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a.v), "v"(b.v));
}
__device__ __forceinline__ void mma_acc(const Frag<_Float16>& a, const Frag<_Float16>& b, v4f& c) {
  asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a.v), "v"(b.v));
}
__device__ __forceinline__ void acc_settle() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// ------------------------------------------------------------ LDS layouts
// Rows contiguous along l: [row][128 B], the row's 16-byte pieces permuted by an
// exclusive or so that the pieces a read serves together (rows 0-3, 12-15 of one
// piece and 4-11 of the next) lie in different banks.
__device__ __forceinline__ int row_swz(int r) { return (r >> 1) & 7; }

// Rows contiguous along the tile's other dimension: [l][R entries], the 16-byte pieces
// of row l permuted so that the rows read together lie in different banks: blocks of
// 16 columns (2 pieces of 16 bits, 4 of 32) by an exclusive or with col_swz, less than
// the R / 16 blocks of a row.
template <class T, int R>
__device__ __forceinline__ int col_swz(int l) {
  if (sizeof(T) == 4) return (l >> 2) & 3;
  return R == 64 ? (l & 3) ^ ((l >> 3) & 1) : (l & 3) | ((l >> 3) & 1) << 2;
}
template <class T, int R>
__device__ __forceinline__ int col_piece(int l, int piece) {
  static_assert(R % 64 == 0 && (sizeof(T) == 4 || R == 64 || R >= 128), "col_swz");
  return piece ^ (col_swz<T, R>(l) * (sizeof(T) == 2 ? 2 : 4));
}

// The fragment of block b (16 rows) and step h of a stage of a tile of R rows at LDS address `base`.
template <class T, bool ROWS, int R>
struct Reader {
  uint32_t at;   // lane's address within block 0
  int sw;        // !ROWS: the lane's block permutation
  __device__ __forceinline__ Reader(int lane) {
    const int r = lane & 15, g = lane >> 4;
    if (ROWS) {
      at = (uint32_t)(r * SB2 + 16 * (g ^ row_swz(r)));
      sw = 0;
    } else if (sizeof(T) == 2) {
      const int l = 8 * g + (r >> 2);   // and + 4 in the second read
      sw = col_swz<T, R>(l);
      at = (uint32_t)(l * R * 2 + 8 * (r & 3));
    } else {
      sw = col_swz<T, R>(4 * g);
      at = (uint32_t)(4 * g * R * 4 + 4 * r);
    }
  }
  __device__ __forceinline__ Frag<T> get(const uint8_t* base, int b, int h = 0) const {
    Frag<T> f;
    if constexpr (ROWS) {
      f.v = *reinterpret_cast<const decltype(f.v)*>(base + (at ^ 64u * h) + b * 16 * SB2);
    } else if constexpr (sizeof(T) == 2) {
      const uint8_t* p = base + at + ((b ^ sw) << 5) + h * 64 * R;
      typedef short v8s __attribute__((ext_vector_type(8)));
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p));
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 4 * R * 2));
      const v8s both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      f.v = __builtin_bit_cast(decltype(f.v), both);
    } else {
      const uint8_t* p = base + at + ((b ^ sw) << 6) + h * 64 * R;
#pragma unroll
      for (int e = 0; e < 4; ++e) f.v[e] = *reinterpret_cast<const float*>(p + e * R * 4);
    }
    return f;
  }
};

// ------------------------------------------------------------ direct loads
// A wave's load of 1 KiB of a stage straight into LDS (lane L's 16 bytes to m0 + 16 L; of
// 256 bytes, lane L's 4 to m0 + 4 L).
// Lanes whose offset is at or beyond kRecords read zeros: that is how rows, columns
// and ends of the sum that do not exist become zeros without a branch.
constexpr uint32_t kRecords = 0x80000000u, kNowhere = 0x80000000u;
typedef int v4i __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void bar() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ const uint8_t* uniform(const void* p) {
  const uint64_t a = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return (const uint8_t*)((uint64_t)hi << 32 | lo);
}

// (one wait state between writing m0 and the load that reads it)
template <int BYTES>
__device__ __forceinline__ void load_lds(const uint8_t* base, uint32_t voff, uint32_t m0) {
  const uint64_t a = (uint64_t)base;
  const v4i rsrc = {(int)(uint32_t)a, (int)(uint32_t)(a >> 32), (int)kRecords, 0x00027000};
  if constexpr (BYTES == 16)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff),
                 "s"(rsrc), "s"(m0)
                 : "memory");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff),
                 "s"(rsrc), "s"(m0)
                 : "memory");
}

// One operand's stages: a wave's share is the blocks w, w + W, .. of a stage, each 64
// pieces of PB bytes, W waves.  16 bytes a piece; 4 for fp32 rows that start anywhere or
// end within 16 bytes: four times the loads, 15% more time a stage, which is less than a
// copy to whole lines first where the product is small (333 x 1001 x 555 15.5 us against
// 19.3; 2047 x 2047 x 2048 168 against 151).
template <class T, bool ROWS, int R, int W, int PB = 16>
struct Stream {
  static constexpr int BLOCK = 64 * PB, N = R * SB2 / BLOCK / W, KE = SB2 / sizeof(T), P = 16 / sizeof(T);
  static constexpr int Q = 16 / PB, E = PB / sizeof(T);   // pieces of 16 bytes; entries of one
  const uint8_t* base;   // uniform
  ll step;
  ll alt;                // gated: from the gates' rows to the values' (32 rows in turn)
  uint32_t vo[N];
  int l[N];              // the lane's first l of the stage
  // src: the tile's first row (ROWS) or first l (else, at its first column) ; row(q)
  // gives the offset in rows from src of LDS row q, or -1; cols: columns from there on
  template <class F>
  __device__ __forceinline__ void init(const T* src, ll ld, int w, int lane, F row, int cols) {
    base = uniform(src);
    alt = 0;
    const int part = lane % Q * E;   // the lane's entries of 16 bytes start here
    if (ROWS) {
      constexpr int PR = SB2 / 16;   // 16 bytes of a row
      step = SB2;
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const int q16 = (w + W * u) * (64 / Q) + lane / Q, q = q16 / PR, at = row(q);
        l[u] = ((q16 % PR) ^ row_swz(q)) * P + part;
        vo[u] = at < 0 ? kNowhere : (uint32_t)((at * ld + l[u]) * (ll)sizeof(T));
      }
    } else {
      constexpr int PR = R / P;   // 16 bytes of an l
      step = KE * ld * (ll)sizeof(T);
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const int q16 = (w + W * u) * (64 / Q) + lane / Q;
        l[u] = q16 / PR;
        const int c = col_piece<T, R>(l[u], q16 % PR) * P + part;
        vo[u] = c >= cols ? kNowhere : (uint32_t)((l[u] * ld + c) * (ll)sizeof(T));
      }
    }
  }
  // block u of the next stage, of which `left` entries of l exist, to LDS at `at` (the
  // stage + the wave's first block); the last one moves on to the stage after it
  __device__ __forceinline__ void issue(int u, uint32_t at, int left) {
    const bool other = ROWS && W * BLOCK * u / SB2 & 32;
    load_lds<PB>(other ? base + alt : base, l[u] < left ? vo[u] : kNowhere, at + (uint32_t)BLOCK * W * u);
    if (u == N - 1) base += step;
  }
};

// ------------------------------------------------------------ rows of W
// The column of y (from the tile's first on) of LDS row q of a tile of W; gated: in
// blocks of 64 rows, 32 gates and the 32 values they gate (8 rows a load, so a wave's
// loads are of gates and of values in turn).
__device__ __forceinline__ int w_col(int q, bool gated) {
  return gated ? (q >> 6) * 32 + (q & 31) : q;
}

// ------------------------------------------------ tiles
constexpr int TM = 128, NT = 256;   // of the smaller tiles; threads of all

struct Tile {
  int group, row, end;   // rows of D; group -1: rows of no group
  int col0;              // first column of y
  int l0, l1;            // range of the sum
  int split;
};

template <Oz2Side SIDE>
__device__ __forceinline__ bool tile_of(const Oz2Product& p, int tile, int ncol, Tile& t) {
  const int cols = p.gated ? tile / 2 : tile;
  // (grid y: the parts of a split sum, else the rest of a grid too long for x)
  const ll b = blockIdx.x + (p.splits > 1 ? 0ll : (ll)blockIdx.y * gridDim.x);
  int r, c;
  t.split = 0;
  if (SIDE == OZ2_WGRAD) {
    const int nrow = (p.M + tile - 1) / tile;
    const ll q = xcd_order(b, (ll)nrow * ncol);
    if (q < 0) return false;
    banded(q, nrow, ncol, r, c);
    t.group = (int)blockIdx.z;
    t.row = r * tile;
    t.end = p.M;
    group_range(p.gr, t.group, t.l0, t.l1);
  } else {
    const int nrow = group_tiles(p.gr, tile);
    const ll n = (ll)nrow * ncol, q = xcd_order(b, n);
    t.l0 = 0;
    t.l1 = p.L;
    if (q >= 0) {
      // in bands of one group's tiles
      const int any = (int)(q / ncol);
      int first;
      group_tile(p.gr, tile, any, t.group, first, t.row, t.end);
      const int start = t.row - (any - first) * tile;
      banded(q - (ll)first * ncol, (t.end - start + tile - 1) / tile, ncol, r, c);
      t.row = start + r * tile;
    } else {   // the rows outside the groups
      const ll k = b - (n + 7) / 8 * 8;
      if (k < 0 || !p.gr.offsets) return false;
      c = (int)(k % ncol);
      t.group = -1;
      const ll row = group_start(p.gr, p.gr.groups) + k / ncol * tile;
      if (row >= p.gr.rows) return false;
      t.row = (int)row;
      t.end = p.gr.rows;
    }
  }
  t.col0 = c * cols;
  if (p.splits > 1) {   // (one group) whole stages, as even as they go
    const int st = SB2 / (p.esize), n = (t.l1 - t.l0 + st - 1) / st;
    t.split = (int)blockIdx.y;
    const int a = (int)((ll)n * t.split / p.splits), e = (int)((ll)n * (t.split + 1) / p.splits);
    t.l1 = min(t.l1, t.l0 + e * st);
    t.l0 += a * st;
  }
  return true;
}

// ------------------------------------------------------------ epilogue
template <class T, int W>
__device__ __forceinline__ void activate(float (&v)[W], int act) {
  if (act == OZ2_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = act_f<T>(v[i], OZ2_ACT_RELU);
  } else if (act == OZ2_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = act_f<T>(v[i], OZ2_ACT_GELU);
  } else if (act == OZ2_ACT_GELU_TANH) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = act_f<T>(v[i], OZ2_ACT_GELU_TANH);
  } else if (act == OZ2_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = act_f<T>(v[i], OZ2_ACT_SILU);
  }
}

// W entries at p, all of them there (ALL) or `valid`
template <class T, int W, bool ALL>
__device__ __forceinline__ void put(T* p, const float* v, int valid) {
  Piece<T, W> o;
#pragma unroll
  for (int i = 0; i < W; ++i) o.v[i] = from_f<T>(v[i]);
  store_stream(p, o, ALL ? W : valid);
}
template <class T, int W, bool ALL>
__device__ __forceinline__ void add_to(float* v, const T* p, int valid) {
  const Piece<T, W> o = load_piece<T, W>(p, ALL ? W : valid);
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] += to_f(o.v[i]);
}

// `steps` rows of a lane from `row` on, STRIDE apart (those before `end`): W columns
// from col on, read from lw (PITCH floats a row), U rows in flight.  y may be res.
template <class T, Oz2Side SIDE, bool GATED, bool ALL, int W, int STRIDE, int STEPS, int PITCH>
__device__ __forceinline__ void emit(const Oz2Product& p, const Tile& t, const float* lw, int row, int col,
                                     int valid, const float* b, const float* bu) {
  constexpr int U = STEPS < 4 ? STEPS : 4;
#pragma clang loop unroll(disable)
  for (int s = 0; s < STEPS; s += U) {
    if (row + s * STRIDE >= t.end) return;
    float v[U * W], u[GATED ? U * W : 1];
    Piece<T, W> r[U];
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int at = row + (s + q) * STRIDE;
      if (SIDE == OZ2_FWD && p.res && at < t.end)
        r[q] = load_piece<T, W>((const T*)p.res + at * p.ldr + col, ALL ? W : valid);
#pragma unroll
      for (int i = 0; i < W; i += 4) {
        const v4f x = *reinterpret_cast<const v4f*>(lw + (s + q) * STRIDE * PITCH + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[q * W + i + e] = SIDE == OZ2_FWD ? x[e] + b[i + e] : x[e];
        if (GATED) {
          const v4f y = *reinterpret_cast<const v4f*>(lw + (s + q) * STRIDE * PITCH + 32 + i);
#pragma unroll
          for (int e = 0; e < 4; ++e) u[q * W + i + e] = y[e] + bu[i + e];
        }
      }
    }
    if (p.splits > 1) {
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const int at = row + (s + q) * STRIDE;
        if (at >= t.end) continue;
        float* d = p.part + ((ll)t.split * p.M + at) * p.N2 + col;
        put<float, W, ALL>(d, v + q * W, valid);
        if (GATED) put<float, W, ALL>(d + p.N, u + q * W, valid);
      }
      continue;
    }
    if (SIDE == OZ2_FWD) {
      if (p.z) {
#pragma unroll
        for (int q = 0; q < U; ++q) {
          const int at = row + (s + q) * STRIDE;
          if (at >= t.end) continue;
          T* z = (T*)p.z + at * p.ldz + col;
          put<T, W, ALL>(z, v + q * W, valid);
          if (GATED) put<T, W, ALL>(z + p.N, u + q * W, valid);
        }
      }
      activate<T, U * W>(v, p.act);
      if (GATED) {
#pragma unroll
        for (int i = 0; i < U * W; ++i) v[i] *= u[i];
      }
      if (p.res) {
#pragma unroll
        for (int i = 0; i < U * W; ++i) v[i] += to_f(r[i / W].v[i % W]);
      }
    }
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int at = row + (s + q) * STRIDE;
      if (at >= t.end) continue;
      put<T, W, ALL>((T*)p.y + (SIDE == OZ2_WGRAD ? t.group * p.strideB : 0) + at * p.ldy + col, v + q * W,
                     valid);
    }
  }
}

// Accumulators acc[j][i] of a wave: 16 MI rows from `row` on (they end before t.end),
// LDS rows wn .. wn + 64 NB - 1 of B.  PI blocks of 16 rows at a time go through the
// wave's own part of LDS, lw: 16 PI rows of 64 NB + 4 floats.
template <class T, Oz2Side SIDE, bool GATED, int MI, int NB, int PI>
__device__ __forceinline__ void epilogue_of(const Oz2Product& p, const v4f (&acc)[4 * NB][MI], float* lw,
                                            const Tile& t, int row, int wn, int lane) {
  constexpr int W = 16 / sizeof(T), PITCH = 64 * NB + 4;
  constexpr int LPR = (GATED ? 32 : 64) * NB / W;   // lanes a row
  constexpr int STRIDE = 64 / LPR, STEPS = 16 * PI / STRIDE;
  const int lr = lane / LPR, c = lane % LPR * W;
  const int col = t.col0 + (GATED ? wn / 2 : wn) + c;
  const int at = GATED ? (c >> 5) * 64 + (c & 31) : c;   // of the (gate's) columns in lw
  const int valid = (SIDE == OZ2_FWD ? p.N : p.N2) - col;
  float b[W], bu[W];
#pragma unroll
  for (int i = 0; i < W; ++i) b[i] = bu[i] = 0.0f;
  if (SIDE == OZ2_FWD && p.bias && p.splits == 1 && valid > 0) {
    const T* bp = (const T*)p.bias + t.group * p.stride_bias + col;
    add_to<T, W, false>(b, bp, valid);
    if (GATED) add_to<T, W, false>(bu, bp + p.N, valid);
  }
  float* lq = lw + (lane & 15) * PITCH + 4 * (lane >> 4);
#pragma clang loop unroll(disable)
  for (int ps = 0; ps < MI / PI; ++ps) {
#pragma unroll
    for (int k = 0; k < MI / PI; ++k)
      if (k == ps) {
#pragma unroll
        for (int i = 0; i < PI; ++i)
#pragma unroll
          for (int j = 0; j < 4 * NB; ++j)
            *reinterpret_cast<v4f*>(lq + 16 * i * PITCH + 16 * j) = acc[j][k * PI + i];
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int r0 = row + 16 * PI * ps + lr;
    const float* lr0 = lw + lr * PITCH + at;
    if (valid >= W)
      emit<T, SIDE, GATED, true, W, STRIDE, STEPS, PITCH>(p, t, lr0, r0, col, W, b, bu);
    else if (valid > 0)
      emit<T, SIDE, GATED, false, W, STRIDE, STEPS, PITCH>(p, t, lr0, r0, col, valid, b, bu);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <class T, Oz2Side SIDE, int MI, int NB, int PI>
__device__ __forceinline__ void epilogue(const Oz2Product& p, const v4f (&acc)[4 * NB][MI], float* lw,
                                         const Tile& t, int row, int wn, int lane) {
  if (SIDE == OZ2_FWD && p.gated)
    epilogue_of<T, SIDE, true, MI, NB, PI>(p, acc, lw, t, row, wn, lane);
  else
    epilogue_of<T, SIDE, false, MI, NB, PI>(p, acc, lw, t, row, wn, lane);
}

// rows [row, row + tile) below end of y (and z) are zeros: columns col .. col + n
template <class T>
__device__ __forceinline__ void zero_rows(const Oz2Product& p, int row, int end, int col, int n, int tile,
                                          int threads) {
  const int w = min(n, p.N - col);
  for (int q = threadIdx.x; q < tile * n; q += threads) {
    const int t = row + q / n, c = q % n;
    if (t >= end || c >= w) continue;
    ((T*)p.y)[t * p.ldy + col + c] = (T)0.0f;
    if (p.z) {
      ((T*)p.z)[t * p.ldz + col + c] = (T)0.0f;
      if (p.gated) ((T*)p.z)[t * p.ldz + p.N + col + c] = (T)0.0f;
    }
  }
}

// Where the operands' tiles start
template <class T, Oz2Side SIDE>
__device__ __forceinline__ void origins(const Oz2Product& p, const Tile& t, const T*& A, const T*& B) {
  A = (const T*)p.A;
  B = (const T*)p.B;
  if (SIDE == OZ2_WGRAD) {
    A += t.l0 * p.lda;
    B += t.l0 * p.ldb;
  } else {
    A += t.l0;
    B += t.group * p.strideB + (SIDE == OZ2_FWD ? (ll)t.l0 : t.l0 * p.ldb);
  }
}

template <class T, Oz2Side SIDE, int R, class SA, class SBT>
__device__ __forceinline__ void streams(const Oz2Product& p, const Tile& t, int w, int lane, SA& sa, SBT& sb) {
  const T *A, *B;
  origins<T, SIDE>(p, t, A, B);
  if (SIDE != OZ2_WGRAD)
    sa.init(A + t.row * p.lda, p.lda, w, lane, [&](int q) { return t.row + q < t.end ? q : -1; }, 0);
  else
    sa.init(A + t.row, p.lda, w, lane, [](int) { return 0; }, t.end - t.row);
  if (SIDE == OZ2_FWD) {
    sb.init(B + t.col0 * p.ldb, p.ldb, w, lane, [&](int q) {
      const int c = w_col(q, p.gated != 0);
      return t.col0 + c < p.N ? c : -1;
    }, 0);
    if (p.gated) sb.alt = p.N * p.ldb * (ll)sizeof(T);
  } else {
    sb.init(B + t.col0, p.ldb, w, lane, [](int) { return 0; }, p.N2 - t.col0);
  }
}

// ------------------------------------------------ 256 x 256 tiles (16 bits)
// 4 waves, one per SIMD, 128 x 128 outputs each: 16 fragment reads feed the 64 products
// of a step.  Stages of two steps, 64 KiB (whole 128-byte lines of rows that are
// contiguous along l; stages of half of that took 0.84 us a step against 0.65 of
// operands that read whole lines anyway); LDS holds two of A's and three of B's.  While
// a step is multiplied, the next one's fragments are read into the other set of
// registers; once every wave holds a stage's last fragments, the loads of A's stage
// after the next and of B's after that go out into its place (W comes from memory where A
// mostly comes from a cache: 2% less time than with two stages of each).  One barrier a
// stage.  Bound by the matrix cores, which the power limit holds at the rate of the
// library's products: 16384 x 4096 x 16384 bf16, gated, 1.57-1.62 ms (1.36-1.40 PFLOP/s);
// 4096^3 108 us for either gradient.  8-12 us of a tile are its first loads and its
// epilogue, which nothing covers: groups of 1000 rows, 2 x 2048 x 4096, reach 1.08.
constexpr int BT = 256, BOP = BT * SB2;

template <class T, Oz2Side SIDE>
__global__ void __launch_bounds__(NT, 1)
k_product256(Oz2Product p, int ncol) {
  constexpr bool AR = SIDE != OZ2_WGRAD, BR = SIDE == OZ2_FWD;
  constexpr int KE = SB2 / sizeof(T);
  __shared__ __attribute__((aligned(16))) uint8_t LB[5 * BOP];   // 2 stages of A, 3 of B
  Tile t;
  if (!tile_of<SIDE>(p, BT, ncol, t)) return;
  if (SIDE != OZ2_WGRAD && t.group < 0) {
    zero_rows<T>(p, t.row, t.end, t.col0, p.gated ? BT / 2 : BT, BT, NT);
    return;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds8*)LB;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Stream<T, AR, BT, 4> sa;
  Stream<T, BR, BT, 4> sb;
  streams<T, SIDE, BT>(p, t, w, lane, sa, sb);
  const int len = t.l1 - t.l0, n = (len + KE - 1) / KE;
  // the wave's share of stage it of A, and of B into place `at`
  auto issue_a = [&](int u, int it) { sa.issue(u, lds0 + (it & 1) * BOP + 1024u * w, len - it * KE); };
  auto issue_b = [&](int u, int it, int at) { sb.issue(u, lds0 + 2 * BOP + at + 1024u * w, len - it * KE); };
  // stages beyond the last one are loaded too, as zeros (nothing is read for them)
#pragma unroll
  for (int u = 0; u < 8; ++u) issue_a(u, 0);
#pragma unroll
  for (int u = 0; u < 16; ++u) issue_b(u & 7, u >> 3, (u >> 3) * BOP);
#pragma unroll
  for (int u = 0; u < 8; ++u) issue_a(u, 1);
#pragma unroll
  for (int u = 0; u < 8; ++u) issue_b(u, 2, 2 * BOP);
  const int wr = w >> 1, wc = w & 1;
  const Reader<T, AR, BT> ra(lane);
  const Reader<T, BR, BT> rb(lane);
  v4f acc[8][8];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  Frag<T> fa[2][8], fb[2][8];   // of the two steps of a stage
  wait_vm<24>();
  bar();
#pragma unroll
  for (int j = 0; j < 8; ++j) fb[0][j] = rb.get(LB + 2 * BOP, 8 * wc + j);
#pragma unroll
  for (int i = 0; i < 8; ++i) fa[0][i] = ra.get(LB, 8 * wr + i);
  int at = 0;   // of B's stage it
  for (int it = 0; it < n; ++it) {
    const int next = at == 2 * BOP ? 0 : at + BOP;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      wait_lds();
      if (h) {
        // all waves hold the last fragments of stage it, and stage it + 1 has landed
        wait_vm<8>();
        bar();
      }
      const uint8_t *ta = LB + ((it + h) & 1) * BOP, *tb = LB + 2 * BOP + (h ? next : at);
      // a read or a load between two products, hardly ever more: the next product is
      // issued before the matrix unit has done with the last
#pragma unroll
      for (int m = 0; m < 64; ++m) {
        mma_acc(fb[h][m & 7], fa[h][m >> 3], acc[m & 7][m >> 3]);
        if (m % 3 == 0 && m < 48) {
          const int k = m / 3;
          if (k < 8)
            fb[1 - h][k] = rb.get(tb, 8 * wc + k, 1 - h);
          else
            fa[1 - h][k - 8] = ra.get(ta, 8 * wr + k - 8, 1 - h);
        }
        if (h && m % 3 == 1 && m < 48) {
          if (m < 24)
            issue_a(m / 3, it + 2);
          else
            issue_b(m / 3 - 8, it + 3, at);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    at = next;
  }
  wait_vm<0>();
  acc_settle();
  __syncthreads();
  epilogue<T, SIDE, 8, 2, 2>(p, acc, reinterpret_cast<float*>(LB) + w * 32 * 132, t, t.row + 128 * wr,
                             128 * wc, lane);
}

// ------------------------------------------------ 128 x 128 and 64 x 64 tiles
// For products with few large tiles, and all of fp32.  4 waves, 64 x 64 (16 x 64)
// outputs each; two stages of 128 bytes of l, 32 (16) KiB each, so that two (four)
// workgroups of a CU cover each other's waits.  Bound by those waits and by reads of LDS
// (a fragment read feeds 2 (0.8) products, the 256 wide tiles' 4): bf16 2048 x 1024 x
// 2048 16 us (540 TFLOP/s), 1024^3 7.2; fp32 1024^3 26 (83), 2048 x 1024 x 2048 74 (116).
template <class T, Oz2Side SIDE, int TILE, int PB>
__global__ void __launch_bounds__(NT, TILE == 128 ? 2 : 4)
k_product128(Oz2Product p, int ncol) {
  constexpr bool AR = SIDE != OZ2_WGRAD, BR = SIDE == OZ2_FWD;
  constexpr int KE = SB2 / sizeof(T), OP = TILE * SB2, ST = 2 * OP, MI = TILE == 128 ? 4 : 1;
  constexpr int EP = 4 * 16 * 68 * 4;   // of the epilogue
  __shared__ __attribute__((aligned(16))) uint8_t LB[2 * ST > EP ? 2 * ST : EP];
  Tile t;
  if (!tile_of<SIDE>(p, TILE, ncol, t)) return;
  if (SIDE != OZ2_WGRAD && t.group < 0) {
    zero_rows<T>(p, t.row, t.end, t.col0, p.gated ? TILE / 2 : TILE, TILE, NT);
    return;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds8*)LB;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = TILE == 128 ? w >> 1 : w, wc = TILE == 128 ? w & 1 : 0;
  Stream<T, AR, TILE, 4, PB> sa;
  Stream<T, BR, TILE, 4, PB> sb;
  streams<T, SIDE, TILE>(p, t, w, lane, sa, sb);
  constexpr int N = Stream<T, AR, TILE, 4, PB>::N;
  const int len = t.l1 - t.l0, n = (len + KE - 1) / KE;
  auto issue = [&](int it) {
    const uint32_t at = lds0 + (it & 1) * ST + 64u * PB * w;
#pragma unroll
    for (int u = 0; u < N; ++u) sa.issue(u, at, len - it * KE);
#pragma unroll
    for (int u = 0; u < N; ++u) sb.issue(u, at + OP, len - it * KE);
  };
  issue(0);   // (stages beyond the last are loaded as zeros)
  issue(1);
  const Reader<T, AR, TILE> ra(lane);
  const Reader<T, BR, TILE> rb(lane);
  v4f acc[4][MI];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < MI; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  for (int it = 0; it < n; ++it) {
    const uint8_t* st = LB + (it & 1) * ST;
    Frag<T> fa[2][MI], fb[2][4];
    wait_vm<2 * N>();
    bar();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < 4; ++j) fb[h][j] = rb.get(st + OP, 4 * wc + j, h);
#pragma unroll
      for (int i = 0; i < MI; ++i) fa[h][i] = ra.get(st, MI * wr + i, h);
    }
    wait_lds();
    bar();
    issue(it + 2);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j][i] = mma(fb[h][j], fa[h][i], acc[j][i]);
  }
  wait_vm<0>();
  __syncthreads();
  epilogue<T, SIDE, MI, 1, 1>(p, acc, reinterpret_cast<float*>(LB) + w * 16 * 68, t, t.row + 16 * MI * wr,
                              64 * wc, lane);
}

// ------------------------------------------------ 128 x 128 tiles, by way of registers
// The same for operands that direct loads do not take: 16-bit rows of any length from any
// address where a copy would cost more, and rows more than 8 MiB apart.  A stage waits in
// LDS, the next two on their way in registers.  Bound by the loads, which fall on no
// boundary: 2.6 us a stage against 0.55.

constexpr int DOP = TM * SB2, DST = 2 * DOP;

// A thread's four 16-byte pieces of an operand's stage
template <class T, bool ROWS>
struct Loader {
  static constexpr int P = 16 / sizeof(T), KE = SB2 / sizeof(T), N = 4;
  typedef Piece<T, P> Set[N];
  const T* src[N];
  int valid[N];          // ROWS: the row exists; else entries of the piece that exist
  int l[N];              // ROWS: first l of the piece; else its l
  uint32_t dst[N];
  ll step;
  template <class F>
  __device__ __forceinline__ void init(const T* base, ll ld, int tid, F row, int cols) {
    step = ROWS ? KE : KE * ld;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int q = tid + NT * u;
      if (ROWS) {
        const int c = q & 7;
        const ll at = row(q >> 3);
        src[u] = base + at * ld + c * P;
        valid[u] = at >= 0;
        l[u] = c * P;
        dst[u] = (uint32_t)((q >> 3) * SB2 + 16 * (c ^ row_swz(q >> 3)));
      } else {
        constexpr int PR = TM / P;   // pieces per l
        l[u] = q / PR;
        const int c = q % PR;
        src[u] = base + l[u] * ld + c * P;
        valid[u] = cols - c * P;
        dst[u] = (uint32_t)(l[u] * TM * sizeof(T) + 16 * col_piece<T, TM>(l[u], c));
      }
    }
  }
  // the next stage, of which `left` entries of l exist
  __device__ __forceinline__ void fetch(Set& s, int left) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int n = ROWS ? (valid[u] ? left - l[u] : 0) : (l[u] < left ? valid[u] : 0);
      s[u] = load_piece<T>(src[u], n);
      src[u] += step;
    }
  }
  __device__ __forceinline__ void store(uint8_t* at, const Set& s) const {
#pragma unroll
    for (int u = 0; u < N; ++u) __builtin_memcpy(__builtin_assume_aligned(at + dst[u], 16), &s[u], 16);
  }
};

template <class T, Oz2Side SIDE>
__global__ void __launch_bounds__(NT, 2)
k_product(Oz2Product p, int ncol) {
  constexpr bool AR = SIDE != OZ2_WGRAD, BR = SIDE == OZ2_FWD;
  constexpr int KE = SB2 / sizeof(T);
  __shared__ __attribute__((aligned(16))) uint8_t LB[2 * DST];
  Tile t;
  if (!tile_of<SIDE>(p, TM, ncol, t)) return;
  if (SIDE != OZ2_WGRAD && t.group < 0) {
    zero_rows<T>(p, t.row, t.end, t.col0, p.gated ? TM / 2 : TM, TM, NT);
    return;
  }
  const T *A, *B;
  origins<T, SIDE>(p, t, A, B);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wr = w >> 1, wc = w & 1;
  Loader<T, AR> la;
  Loader<T, BR> lb;
  if (AR)
    la.init(A, p.lda, tid, [&](int q) { return t.row + q < t.end ? (ll)t.row + q : -1ll; }, 0);
  else
    la.init(A + t.row, p.lda, tid, [](int) { return 0ll; }, t.end - t.row);
  if (BR)
    lb.init(B, p.ldb, tid, [&](int q) {
      const int c = t.col0 + w_col(q, p.gated != 0);
      return c < p.N ? (ll)c + (p.gated && (q & 32) ? p.N : 0) : -1ll;
    }, 0);
  else
    lb.init(B + t.col0, p.ldb, tid, [](int) { return 0ll; }, p.N2 - t.col0);
  v4f acc[4][4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  const Reader<T, AR, TM> ra(lane);
  const Reader<T, BR, TM> rb(lane);
  const int len = t.l1 - t.l0, n = (len + KE - 1) / KE;
  typename Loader<T, AR>::Set pa[2];
  typename Loader<T, BR>::Set pb[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    la.fetch(pa[u], len - u * KE);
    lb.fetch(pb[u], len - u * KE);
  }
  // (an even number of stages: those beyond the last are zeros)
  for (int it0 = 0; it0 < n; it0 += 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint8_t* st = LB + u * DST;
      la.store(st, pa[u]);
      lb.store(st + DOP, pb[u]);
      __syncthreads();
      la.fetch(pa[u], len - (it0 + u + 2) * KE);
      lb.fetch(pb[u], len - (it0 + u + 2) * KE);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Frag<T> fa[4], fb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) fb[j] = rb.get(st + DOP, 4 * wc + j, h);
#pragma unroll
        for (int i = 0; i < 4; ++i) fa[i] = ra.get(st, 4 * wr + i, h);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j][i] = mma(fb[j], fa[i], acc[j][i]);
      }
    }
  }
  __syncthreads();
  epilogue<T, SIDE, 4, 1, 1>(p, acc, reinterpret_cast<float*>(LB) + w * 16 * 68, t, t.row + 64 * wr, 64 * wc,
                             lane);
}

// The pieces in which direct loads can take an operand: 16 bytes where its rows start
// and end on them, 4 bytes of fp32, else (or where offsets within a stage's rows pass
// kRecords) none, 0.
template <class T>
int direct_side(const void* x, ll ld, bool rows, ll extent, int tile) {
  constexpr int P = 16 / sizeof(T);
  if (ld * (rows ? (ll)sizeof(T) * tile : SB2) >= (ll)kRecords - 65536) return 0;
  if ((uintptr_t)x % 16 == 0 && ld % P == 0 && extent % P == 0) return 16;
  return sizeof(T) == 4 ? 4 : 0;
}
template <class T>
int direct(Oz2Side side, const Oz2Product& p, int tile) {
  constexpr int P = 16 / sizeof(T);
  const ll acols = side == OZ2_WGRAD ? p.M : p.L;
  const int a = direct_side<T>(p.A, p.lda, side != OZ2_WGRAD, p.padded ? 0 : acols, tile);
  const int b = direct_side<T>(p.B, p.ldb, side == OZ2_FWD, p.paddedB ? 0 : side == OZ2_FWD ? p.L : p.N2, tile);
  const int group = side == OZ2_WGRAD || p.strideB % P == 0 ? 16 : sizeof(T) == 4 ? 4 : 0;
  return std::min(std::min(a, b), group);
}

#define OZ2_SIDES(kern, ...)                                                            \
  do {                                                                                  \
    if (side == OZ2_FWD)                                                                \
      hipLaunchKernelGGL((kern<T, OZ2_FWD __VA_ARGS__>), grid, dim3(NT), 0, s, p, ncol);   \
    else if (side == OZ2_DGRAD)                                                         \
      hipLaunchKernelGGL((kern<T, OZ2_DGRAD __VA_ARGS__>), grid, dim3(NT), 0, s, p, ncol); \
    else                                                                                \
      hipLaunchKernelGGL((kern<T, OZ2_WGRAD __VA_ARGS__>), grid, dim3(NT), 0, s, p, ncol); \
    return hipGetLastError();                                                           \
  } while (0)

// columns of tiles and the grid of a product in `tile` x `tile` tiles
dim3 tile_grid(Oz2Side side, const Oz2Product& p, int tile, int& ncol) {
  const int cols = p.gated && side == OZ2_FWD ? tile / 2 : tile, n = side == OZ2_FWD ? p.N : p.N2;
  ncol = (n + cols - 1) / cols;
  const Oz2Grid g = oz2_grid(side == OZ2_WGRAD ? ((ll)((p.M + tile - 1) / tile) * ncol + 7) / 8 * 8
                                               : oz2_tile_blocks(p.gr, tile, ncol));
  // (split sums are of few tiles)
  return dim3(g.x, p.splits > 1 ? p.splits : g.y, side == OZ2_WGRAD ? p.gr.groups : 1);
}

// The epilogue of W columns of one row from column col on (valid of them exist), v and
// u the sums
template <class T, int W>
__device__ __forceinline__ void finish(const Oz2Product& p, int group, ll row, int col, int valid,
                                       float (&v)[W], float (&u)[W]) {
  if (p.bias) {
    const T* b = (const T*)p.bias + group * p.stride_bias + col;
    add_to<T, W, false>(v, b, valid);
    if (p.gated) add_to<T, W, false>(u, b + p.N, valid);
  }
  if (p.z) {
    T* z = (T*)p.z + row * p.ldz + col;
    put<T, W, false>(z, v, valid);
    if (p.gated) put<T, W, false>(z + p.N, u, valid);
  }
  activate<T, W>(v, p.act);
  if (p.gated) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] *= u[i];
  }
  if (p.res) add_to<T, W, false>(v, (const T*)p.res + row * p.ldr + col, valid);
  put<T, W, false>((T*)p.y + row * p.ldy + col, v, valid);
}

// The sum of a product's splits, in order, and the epilogue: 16 bytes of y a thread.  Bound
// by the launch and the parts' bytes (4 us and 4 TB/s); one part of 128^2 x 8192 bf16
// takes 31 us, eight 12.
template <class T>
__global__ void __launch_bounds__(256)
k_join(Oz2Product p) {
  constexpr int W = 16 / sizeof(T);
  const int pieces = (p.N + W - 1) / W;
  const ll id = (ll)blockIdx.x * 256 + threadIdx.x, row = id / pieces;
  if (row >= p.M) return;
  const int col = (int)(id - row * pieces) * W, valid = p.N - col;
  float v[W], u[W];
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = u[i] = 0.0f;
  for (int s = 0; s < p.splits; ++s) {
    const float* q = p.part + ((ll)s * p.M + row) * p.N2 + col;
    add_to<float, W, false>(v, q, valid);
    if (p.gated) add_to<float, W, false>(u, q + p.N, valid);
  }
  finish<T, W>(p, 0, row, col, valid, v, u);
}

// ------------------------------------------------ few rows: one read of W
// y = f(x W^T ..) for groups of a few rows each (single tokens, decoding): the bytes of
// W bound it (4096 x 4096 bf16, one row: 8.2-8.5 us, 4.0 TB/s; 14 experts of 2 x 2048 x
// 4096: 75 us, 6.2 TB/s).  A workgroup takes 16 columns of y of one group (gated: their gates and
// values), its eight waves share out the 128-byte chunks of l and read their rows of
// W straight into fragments, UN chunks in flight; 16 TB rows of x at a time are the
// other operand.  The waves' sums meet in LDS and are added in order.
constexpr int RNT = 512, RW = RNT / 64;

template <class T, int TB, bool GATED>
__global__ void __launch_bounds__(RNT)
k_rows(Oz2Product p) {
  constexpr int P = 16 / sizeof(T), KC = SB2 / sizeof(T), G = GATED ? 2 : 1;
  constexpr int UN = TB == 1 && !GATED ? 8 : 4;
  __shared__ v4f red[RW][G * TB][64];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = (int)blockIdx.x * 16, group = (int)blockIdx.y;
  if (group == p.gr.groups) {   // the rows of no group
    for (int t = group_start(p.gr, group) + (tid >> 4); t < p.gr.rows; t += RNT / 16) {
      const int c = n0 + (tid & 15);
      if (c >= p.N) continue;
      ((T*)p.y)[t * p.ldy + c] = (T)0.0f;
      if (p.z) {
        ((T*)p.z)[t * p.ldz + c] = (T)0.0f;
        if (GATED) ((T*)p.z)[t * p.ldz + p.N + c] = (T)0.0f;
      }
    }
    return;
  }
  int r0, r1;
  group_range(p.gr, group, r0, r1);
  // rows that do not exist are read as the last one: their results are not stored
  const T* wp = (const T*)p.B + group * p.strideB + min(n0 + r, p.N - 1) * p.ldb + g * P;
  const ll up = GATED ? p.N * p.ldb : 0;
  const int nch = (p.L + KC - 1) / KC, full = p.L / KC;
  for (int row = r0; row < r1; row += 16 * TB) {
    const T* xp[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) xp[b] = (const T*)p.A + min(row + 16 * b + r, r1 - 1) * p.lda + g * P;
    v4f acc[G][TB];
#pragma unroll
    for (int k = 0; k < G; ++k)
#pragma unroll
      for (int b = 0; b < TB; ++b) acc[k][b] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    typedef decltype(Frag<T>::v) V;
    // UN chunks of the wave from c0 on (WHOLE: all there).  One beyond the last full one
    // must not meet W, whose infinities times zero are NaN: gated, it is the last one
    // again and its products are left out (no branch between the loads and one loop's
    // registers: 14 experts of 2 x 2048 x 4096 76 us against 83); else, where short sums
    // count, zeros for both (5 x 1000 x 777 fp16 4.5 us against 6.5).
    auto batch = [&](auto whole, int c0) {
      constexpr bool WHOLE = decltype(whole)::value;
      Frag<T> wf[UN][2][G], xf[UN][2][TB];
#pragma unroll
      for (int q = 0; q < UN; ++q) {
        const bool on = GATED || WHOLE || c0 + RW * q < full;
        const int k = (GATED ? min(c0 + RW * q, full - 1) : c0 + RW * q) * KC;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int e = 0; e < G; ++e) {
            if (on)
              __builtin_memcpy(&wf[q][h][e].v, wp + e * up + k + 4 * h * P, 16);
            else
              wf[q][h][e].v = V{};
          }
#pragma unroll
          for (int b = 0; b < TB; ++b) {
            if (on)
              __builtin_memcpy(&xf[q][h][b].v, xp[b] + k + 4 * h * P, 16);
            else
              xf[q][h][b].v = V{};
          }
        }
      }
      if (!GATED) __builtin_amdgcn_sched_barrier(0);   // all loads first
#pragma unroll
      for (int q = 0; q < UN; ++q)
        if (!GATED || c0 + RW * q < full)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < G; ++e)
#pragma unroll
              for (int b = 0; b < TB; ++b) acc[e][b] = mma(wf[q][h][e], xf[q][h][b], acc[e][b]);
    };
    int c0 = w;
    if (!GATED)
      for (; c0 + RW * (UN - 1) < full; c0 += RW * UN) batch(std::true_type{}, c0);
    for (; c0 < full; c0 += RW * UN) batch(std::false_type{}, c0);
    if (nch > full && full % RW == w) {   // the last chunk, in part
      const int k = full * KC;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int valid = p.L - k - (g + 4 * h) * P;
        Frag<T> wf[G], xf[TB];
#pragma unroll
        for (int e = 0; e < G; ++e)
          wf[e].v = __builtin_bit_cast(V, load_piece<T>(wp + e * up + k + 4 * h * P, valid));
#pragma unroll
        for (int b = 0; b < TB; ++b)
          xf[b].v = __builtin_bit_cast(V, load_piece<T>(xp[b] + k + 4 * h * P, valid));
#pragma unroll
        for (int e = 0; e < G; ++e)
#pragma unroll
          for (int b = 0; b < TB; ++b) acc[e][b] = mma(wf[e], xf[b], acc[e][b]);
      }
    }
#pragma unroll
    for (int e = 0; e < G; ++e)
#pragma unroll
      for (int b = 0; b < TB; ++b) red[w][e * TB + b][lane] = acc[e][b];
    __syncthreads();
    if (tid < TB * 64) {   // entry tid: accumulators of lane `lane` of block w
      v4f s[2] = {v4f{0.0f, 0.0f, 0.0f, 0.0f}, v4f{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
      for (int k = 0; k < RW; ++k)
#pragma unroll
        for (int e = 0; e < G; ++e) s[e] += red[k][e * TB + w][lane];
      const int t = row + 16 * w + r, col = n0 + 4 * g, valid = p.N - col;
      if (t < r1 && valid > 0) {
        float v[4], u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = s[0][i];
          u[i] = s[1][i];
        }
        finish<T, 4>(p, group, t, col, valid, v, u);
      }
    }
    __syncthreads();
  }
}

template <class T, bool GATED>
hipError_t launch_rows(int blocks, const Oz2Product& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.N + 15) / 16), (unsigned)(p.gr.groups + (p.gr.offsets ? 1 : 0)));
  if (blocks == 1)
    hipLaunchKernelGGL((k_rows<T, 1, GATED>), grid, dim3(RNT), 0, s, p);
  else
    hipLaunchKernelGGL((k_rows<T, 2, GATED>), grid, dim3(RNT), 0, s, p);
  return hipGetLastError();
}

// ------------------------------------------------ operands in whole lines
// Rows that are not whole 16-byte pieces, copied to rows of whole 128-byte lines with
// zeros at their ends, for the direct loads: 16-bit rows from any address take 2.6 us
// a stage of 128 x 128 tiles, direct loads 0.55.  64 lanes a row, both operands.  Bound by
// its launch for small ones: 777 and 1301 rows of 995 fp16 6.2 us.
struct Rows {
  const void* src;
  ll ld, stride;     // elements between rows, and between matrices of `per` rows
  ll rows;
  int per, cols;
  void* dst;
  ll pitch;
};

template <class T>
__global__ void __launch_bounds__(256)
k_pack(Rows a, Rows b) {
  constexpr int P = 16 / sizeof(T);
  for (ll row = (ll)blockIdx.x * 4 + (threadIdx.x >> 6); row < a.rows + b.rows; row += (ll)gridDim.x * 4) {
    const bool second = row >= a.rows;
    const Rows& m = second ? b : a;
    const ll r = second ? row - a.rows : row, k = r / m.per;
    const T* src = (const T*)m.src + k * m.stride + (r - k * m.per) * m.ld;
    T* dst = (T*)m.dst + r * m.pitch;
    for (int c = (threadIdx.x & 63) * P; c < m.pitch; c += 64 * P)
      store_piece(dst + c, load_piece<T>(src + c, m.cols - c), P);
  }
}

template <class T>
hipError_t pack(Oz2Side side, const Oz2Plan& plan, Oz2Product& p, hipStream_t s) {
  Rows r[2] = {};
  const int groups = p.gr.offsets ? p.gr.groups : 1;
  T* at = (T*)p.packed;
  if (plan.pack & 1) {
    const int cols = side == OZ2_WGRAD ? p.M : p.L, rows = side == OZ2_WGRAD ? p.L : p.M;
    r[0] = Rows{p.A, p.lda, 0, rows, std::max(rows, 1), cols, at, (ll)(oz2_packed_pitch(cols, sizeof(T)))};
    p.A = at;
    p.lda = r[0].pitch;
    at += rows * r[0].pitch;
    p.padded = true;
  }
  if (plan.pack & 2) {
    const int cols = side == OZ2_FWD ? p.L : p.N2;
    const int per = side == OZ2_FWD ? p.N2 : p.L, count = side == OZ2_WGRAD ? 1 : groups;
    Rows& q = r[1];
    q = Rows{p.B, p.ldb, p.strideB, (ll)per * count, std::max(per, 1), cols, at, oz2_packed_pitch(cols, sizeof(T))};
    p.B = at;
    p.ldb = q.pitch;
    if (side != OZ2_WGRAD) p.strideB = per * q.pitch;
    p.paddedB = true;
  }
  const ll rows = r[0].rows + r[1].rows;
  if (rows == 0) return hipSuccess;
  hipLaunchKernelGGL(k_pack<T>, dim3((unsigned)std::min<ll>(1 << 20, (rows + 3) / 4)), dim3(256), 0, s, r[0],
                     r[1]);
  return hipGetLastError();
}

template <class T>
hipError_t launch_tiles(Oz2Side side, int tile, const Oz2Product& p, hipStream_t s) {
  int ncol;
  // (operands that direct loads do not take: 128 x 128 whatever the plan)
  const int pieces = direct<T>(side, p, tile);
  if (!pieces) tile = 0;
  const dim3 grid = tile_grid(side, p, tile ? tile : TM, ncol);
  if constexpr (sizeof(T) == 2) {
    if (tile == BT) OZ2_SIDES(k_product256);
  }
  if constexpr (sizeof(T) == 4) {
    if (tile == 128 && pieces == 4) OZ2_SIDES(k_product128, , 128, 4);
    if (tile == 64 && pieces == 4) OZ2_SIDES(k_product128, , 64, 4);
  }
  if (tile == 128) OZ2_SIDES(k_product128, , 128, 16);
  if (tile == 64) OZ2_SIDES(k_product128, , 64, 16);
  OZ2_SIDES(k_product);
}

template <class T>
hipError_t launch_product(Oz2Side side, const Oz2Plan& plan, Oz2Product p, hipStream_t s) {
  if (p.M == 0 || p.N2 == 0) return hipSuccess;
  p.esize = sizeof(T);
  p.splits = plan.splits;
  if (plan.rows) return p.gated ? launch_rows<T, true>(plan.rows, p, s) : launch_rows<T, false>(plan.rows, p, s);
  hipError_t e = plan.pack ? pack<T>(side, plan, p, s) : hipSuccess;
  if (e != hipSuccess) return e;
  e = launch_tiles<T>(side, plan.tile, p, s);
  if (e != hipSuccess || p.splits == 1) return e;
  constexpr int W = 16 / sizeof(T);
  const ll items = (ll)p.M * ((p.N + W - 1) / W);
  hipLaunchKernelGGL(k_join<T>, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, s, p);
  return hipGetLastError();
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
