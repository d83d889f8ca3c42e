// Sums and maxima over neighbouring lanes of a wave, in a fixed order, in all of them.
// Device code.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

namespace {

// The largest (sum) of v over N neighbouring lanes (8, 16, 32 or 64, from a multiple of N
// on): pairs, quads, then halves of a row of 16 and rows mirrored, which the arithmetic
// instructions do by themselves, then rows by way of LDS's crossbar.
template <int N, bool SUM>
__device__ __forceinline__ float across(float v) {
  auto with = [&](auto ctrl) {
    const int u = __builtin_bit_cast(int, v);
    const float o = __builtin_bit_cast(
        float, __builtin_amdgcn_update_dpp(u, u, decltype(ctrl)::value, 0xf, 0xf, false));
    v = SUM ? v + o : fmaxf(v, o);
  };
  with(std::integral_constant<int, 0xB1>{});
  with(std::integral_constant<int, 0x4E>{});
  with(std::integral_constant<int, 0x141>{});
  if (N >= 16) with(std::integral_constant<int, 0x140>{});
#pragma unroll
  for (int d = 16; d < N; d *= 2) {
    const float o = __shfl_xor(v, d);
    v = SUM ? v + o : fmaxf(v, o);
  }
  return v;
}

}  // namespace
