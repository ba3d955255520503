// Shared by the kernels between the layers.
// Reductions across lanes without LDS: within a row of 16 lanes by data-parallel moves, across rows by
// the row swaps of gfx950. Every lane receives the result.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace aqmb {

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, kCtrl, 0xF, 0xF, true);
}

// One step of a butterfly over lanes; f combines two bit patterns. D is the distance 1, 2, 4, 8, 16 or 32.
// 4 and 8 pair lane i with 7 - i and 15 - i of its row: after the steps below them the same values.
template <int D, class F>
__device__ __forceinline__ uint32_t butterfly(uint32_t x, F f) {
  if constexpr (D == 1) return f(x, dpp<0xB1>(x));         // quad_perm 1, 0, 3, 2
  else if constexpr (D == 2) return f(x, dpp<0x4E>(x));    // quad_perm 2, 3, 0, 1
  else if constexpr (D == 4) return f(x, dpp<0x141>(x));   // row_half_mirror
  else if constexpr (D == 8) return f(x, dpp<0x140>(x));   // row_mirror
  else if constexpr (D == 16) {
    const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return f((uint32_t)p[0], (uint32_t)p[1]);
  } else {
    const auto p = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return f((uint32_t)p[0], (uint32_t)p[1]);
  }
}

// f over groups of N neighbouring lanes (a power of two up to 64, from a multiple of N).
template <int N, int D = 1, class F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t x, F f) {
  if constexpr (D >= N) return x;
  else return over_lanes<N, 2 * D>(butterfly<D>(x, f), f);
}

__device__ __forceinline__ uint32_t max_bits(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t add_floats(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
}

// How a group of values is brought to 8 bits: from the largest magnitude's bits (those of infinity and NaN are
// above every finite value's) the factor of the values and the scale that the results stand for, each the rounded
// quotient, so that every kernel that scales does it alike. The floor keeps both normal numbers.
struct Scaling {
  float mul, scale;
  bool finite;
};
__device__ __forceinline__ Scaling scaling_of(uint32_t largest, float top) {
  const bool finite = largest < 0x7F800000u;
  const float a = fmaxf(__builtin_bit_cast(float, largest), 0x1p-100f);
  return {top / a, finite ? a / top : __builtin_nanf(""), finite};
}

}  // namespace aqmb
