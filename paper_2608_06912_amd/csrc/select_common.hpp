// Device helpers of the hard selections (routing, beams, cache entries):
// elements of three types, an order on floats, and lanes that work on one row
// together.
#pragma once

#include <float.h>
#include <math.h>

#include <type_traits>
#include <utility>

#include "common.hpp"
#include "kernels.hpp"

namespace lapsum {

// ---------------------------------------------------------------- types ----
// Elements by lapsum_dtype: float32, bfloat16, float16.
template <int DT>
struct Elem;
template <>
struct Elem<0> {
  using raw = uint32_t;
  static __device__ __forceinline__ float get(uint32_t u) { return __uint_as_float(u); }
  static __device__ __forceinline__ uint32_t put(float f) { return __float_as_uint(f); }
};
template <>
struct Elem<1> {
  using raw = uint16_t;
  static __device__ __forceinline__ float get(uint32_t u) { return __uint_as_float(u << 16); }
  // to nearest even, as torch rounds
  static __device__ __forceinline__ uint16_t put(float f) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));
  }
};
template <>
struct Elem<2> {
  using raw = uint16_t;
  static __device__ __forceinline__ float get(uint32_t u) {
    return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(u)));
  }
  static __device__ __forceinline__ uint16_t put(float f) {
    return __builtin_bit_cast(uint16_t, static_cast<_Float16>(f));
  }
};

// Words that are moved as they are (vectors of the compiler's own, which stay
// in registers).
typedef uint32_t Move16 __attribute__((ext_vector_type(4)));
typedef uint32_t Move8 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- order ----
// uint32 key whose ascending order is the ascending order of the float, equal
// for both zeros; NaN as low as can be (0 is below every float's key).
__device__ __forceinline__ uint32_t asc_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);
  const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return f == f ? k : 0u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}

// ------------------------------------------------------------ wave order ---
// LDS written by some lanes of a wave and read by others: a wave's LDS
// operations complete in order, so the compiler alone has to keep them so.
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The value of the lane that a control names where every lane has one in its
// row of 16 (rotations, permutations of four, mirrors): nothing to keep, so
// that the move becomes part of the operation that reads it.
template <int CTRL, typename T>
__device__ __forceinline__ T row_move(T x) {
  static_assert(sizeof(T) == 4 || sizeof(T) == 8, "32- or 64-bit values");
  const auto word = [](uint32_t w) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(w), CTRL, 0xf, 0xf, true));
  };
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, word(__builtin_bit_cast(uint32_t, x)));
  } else {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(T, (static_cast<uint64_t>(word(static_cast<uint32_t>(b >> 32))) << 32) |
                                     word(static_cast<uint32_t>(b)));
  }
}

// f(control) for the 15 rotations of a row of 16 lanes.
template <class F, int... D>
__device__ __forceinline__ void each_rotation(F&& f, std::integer_sequence<int, D...>) {
  (f(std::integral_constant<int, 0x121 + D>{}), ...);
}
template <class F>
__device__ __forceinline__ void each_rotation(F&& f) {
  each_rotation(f, std::make_integer_sequence<int, 15>{});
}

// Reductions over groups of LT lanes (16: a row of the wave, by rotations; 64:
// the wave), the result in every lane.  Every lane of the wave takes part.
template <int LT, typename T, typename Op>
__device__ __forceinline__ T team_reduce(T v, Op op) {
  static_assert(LT == 16 || LT == 64, "a row of lanes or a wave");
  v = op(v, row_move<0x128>(v));
  v = op(v, row_move<0x124>(v));
  v = op(v, row_move<0x122>(v));
  v = op(v, row_move<0x121>(v));
  if constexpr (LT == 64)
    v = op(op(readlane_as(v, 0), readlane_as(v, 16)), op(readlane_as(v, 32), readlane_as(v, 48)));
  return v;
}
// (floats as the middle of three, one instruction; no NaN comes here)
__device__ __forceinline__ float max_f32(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }
__device__ __forceinline__ float min_f32(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, -INFINITY); }
template <int LT, typename T>
__device__ __forceinline__ T team_max(T v) {
  if constexpr (std::is_same_v<T, float>) return team_reduce<LT>(v, max_f32);
  else return team_reduce<LT>(v, [](T a, T b) { return a > b ? a : b; });
}
template <int LT, typename T>
__device__ __forceinline__ T team_min(T v) {
  if constexpr (std::is_same_v<T, float>) return team_reduce<LT>(v, min_f32);
  else return team_reduce<LT>(v, [](T a, T b) { return a < b ? a : b; });
}
// bits, with the sign of f for a new lowest bit.
__device__ __forceinline__ uint32_t push_sign(uint32_t bits, float f) {
  return __builtin_amdgcn_alignbit(bits, __float_as_uint(f), 31);
}
// 0 - x, +0 for both zeros; the sum it goes into is not to be made a difference
// with x, whose sign is another for zeros.
__device__ __forceinline__ float minus(float x) {
  float y = 0.0f - x;
  asm("" : "+v"(y));
  return y;
}
// How many of the row's 16 lanes hold a larger value than this one.  The values
// are finite, so that the sign of a difference is the comparison (a
// difference of zeros is +0); one instruction subtracts and one
// keeps the sign, where a comparison and its count take three.
__device__ __forceinline__ int row_count_above(float x) {
  const float neg = minus(x);
  float d[15];
  each_rotation([&](auto ctl) { d[decltype(ctl)::value - 0x121] = x + row_move<decltype(ctl)::value>(neg); });
  asm("" : "+v"(d[0]), "+v"(d[1]), "+v"(d[2]), "+v"(d[3]), "+v"(d[4]));
  asm("" : "+v"(d[5]), "+v"(d[6]), "+v"(d[7]), "+v"(d[8]), "+v"(d[9]));
  asm("" : "+v"(d[10]), "+v"(d[11]), "+v"(d[12]), "+v"(d[13]), "+v"(d[14]));
  uint32_t bits = 0u;
#pragma unroll
  for (int i = 0; i < 15; ++i) bits = push_sign(bits, d[i]);
  return __popc(bits);
}
template <int LT, typename T>
__device__ __forceinline__ T team_sum(T v) {
  return team_reduce<LT>(v, [](T a, T b) { return a + b; });
}
// Inclusive sum over the lanes of the team up to this one.
template <int LT>
__device__ __forceinline__ int team_incl_add(int x) {
  if constexpr (LT == 64) return wave_incl_add(x);
  x += dpp_move<0x111>(x, 0);
  x += dpp_move<0x112>(x, 0);
  x += dpp_move<0x114>(x, 0);
  x += dpp_move<0x118>(x, 0);
  return x;
}

}  // namespace lapsum
