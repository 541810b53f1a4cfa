// Elements of a paged cache: where an entry is, and eight-bit codes.
#pragma once

#include "select_common.hpp"

namespace lapsum {

// Types of a cache: the three of Elem, and codes of 8 bits with a scale per row.
constexpr int kInt8 = 3, kE4m3 = 4;
template <int KIND>
constexpr int kCacheBytes = KIND == 0 ? 4 : KIND <= 2 ? 2 : 1;

// The page and the slot in it of position `at` of sequence b; page -1 where the
// sequence has none.
__device__ __forceinline__ void find_slot(const PageTable& t, int b, int at, int* page, int* slot) {
  if (!t.table) {
    *page = at < t.size ? b : -1;
    *slot = at;
    return;
  }
  const int p = static_cast<int>(divide(static_cast<uint32_t>(at), t.by));
  *slot = at - p * t.size;
  int64_t page_no = -1;
  if (p < t.width) page_no = t.table[static_cast<int64_t>(b) * t.width + p];
  *page = page_no >= 0 && page_no < t.pages ? static_cast<int>(page_no) : -1;
}

// Four codes as floats.
template <int KIND>
__device__ __forceinline__ void decode4(uint32_t w, float* x) {
  if constexpr (KIND == kInt8) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = static_cast<float>(static_cast<int8_t>(w >> (8 * j)));
  } else {
    typedef float Two __attribute__((ext_vector_type(2)));
    const Two a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
    const Two b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    x[0] = a[0];
    x[1] = a[1];
    x[2] = b[0];
    x[3] = b[1];
  }
}
// Four floats within the codes' range, each to the nearest code, ties to even.
template <int KIND>
__device__ __forceinline__ uint32_t encode4(const float* x) {
  static_assert(KIND == kE4m3, "the others are whole numbers");
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
  return static_cast<uint32_t>(w);
}

}  // namespace lapsum
