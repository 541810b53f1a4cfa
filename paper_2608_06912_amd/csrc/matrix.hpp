// Tiles of a matrix product on the matrix cores: operands in LDS as chunks of 16
// bytes, and the fragments of a 16 x 16 tile of results read from them.
//
// The contraction goes in stages of one or two steps of four chunks (32 elements
// of 16 bits, 16 floats).  Lane l of a wave holds, of row l & 15, the chunk l >> 4
// of a step: eight elements for one 16x16x32 instruction, or four floats for four
// 16x16x4 ones (the order of the contraction is the operands' own business, as
// long as it is the same for both).
#pragma once

#include "select_common.hpp"

namespace lapsum {

typedef float Acc __attribute__((ext_vector_type(4)));
typedef __bf16 Bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 F16x8 __attribute__((ext_vector_type(8)));
typedef short Half4 __attribute__((ext_vector_type(4)));

// c += a b^T of a step: rows of a and b as above; c[i] of lane l is row
// 4 (l >> 4) + i of a and row l & 15 of b.
template <int DT>
__device__ __forceinline__ Acc mma(Move16 a, Move16 b, Acc c) {
  if constexpr (DT == 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
    return c;
  } else if constexpr (DT == 1) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16x8, a), __builtin_bit_cast(Bf16x8, b),
                                                   c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(F16x8, a), __builtin_bit_cast(F16x8, b), c,
                                                  0, 0, 0);
  }
}

// The chunk at p of which `left` elements exist, the end of a line of `width` elements.
// Elements of 16 bits: a line's last chunk is read as the whole vector that the line ends
// with, and trim_chunk moves it to its place, zeros behind, once it is there (element by
// element, each load waited for, 16384 rows of 8 experts 2047 -> 1023 cost 275 us instead
// of 158).  Floats, and lines shorter than a chunk: by elements, all of them at once (48 rows
// of 7 experts 443 -> 2960 in float32 19 us, as vectors 32).
template <int DT>
__device__ __forceinline__ Move16 load_chunk(const typename Elem<DT>::raw* p, int64_t left, int width) {
  constexpr int N = 16 / sizeof(typename Elem<DT>::raw);
  Move16 v = {0u, 0u, 0u, 0u};
  if (left <= 0) return v;
  if (DT == 0 ? left >= N : width >= N) {
    // (global memory serves vectors at any alignment of their elements)
    struct __attribute__((packed, aligned(sizeof(*p)))) Any {
      uint32_t x, y, z, w;
    };
    const Any u = *reinterpret_cast<const Any*>(left < N ? p + (left - N) : p);
    v = Move16{u.x, u.y, u.z, u.w};
  } else {
    uint32_t e[N];
#pragma unroll
    for (int j = 0; j < N; ++j) e[j] = p[j < left ? j : left - 1];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (DT == 0) v[j] = j < left ? e[j] : 0u;
      else v[j / 2] |= (j < left ? e[j] : 0u) << (16 * (j % 2));
    }
  }
  return v;
}
template <int DT>
__device__ __forceinline__ Move16 trim_chunk(Move16 v, int64_t left, int width) {
  constexpr int N = 16 / sizeof(typename Elem<DT>::raw);
  if (DT == 0 || width < N || left >= N || left <= 0) return v;
  const int back = N - static_cast<int>(left);
  if (back & 4) v = Move16{v[2], v[3], 0u, 0u};
  if (back & 2) v = Move16{v[1], v[2], v[3], 0u};
  if (back & 1)
    v = Move16{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  return v;
}

// A stage of an operand of R rows in LDS.  Dense along the contraction (TR false): R rows
// of four or eight chunks.  Dense along the rows (TR true): a row of R elements for each
// element of the contraction.  Chunks are permuted within a row by the row's
// number, so that the lanes that read together meet different banks.
template <int DT, int R, bool TR, int STEPS>
struct Operand {
  static constexpr int E = DT == 0 ? 4 : 2;              // bytes of an element
  static constexpr int N = 16 / E;                       // elements of a chunk
  static constexpr int Steps = STEPS;
  static constexpr int Stage = STEPS * 4 * N;            // contraction of a stage
  static constexpr int Rows = TR ? Stage : R;
  static constexpr int Chunks = TR ? R / N : STEPS * 4;  // of a row
  static constexpr int Reads = TR ? (DT == 0 ? 4 : 2) : 1;   // of LDS, for a fragment
  static constexpr int Total = Rows * Chunks;
  static constexpr int Bytes = Total * 16;

  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (!TR) return STEPS == 2 ? r & 7 : (r >> 1) & 3;
    else if constexpr (DT == 0) return (((r >> 2) & 3) << 2) & (Chunks - 1);
    else return (((r & 3) | ((r >> 1) & 4)) << 1) & (Chunks - 1);
  }
  static __device__ __forceinline__ int slot(int r, int c) { return r * Chunks + (c ^ swizzle(r)); }

  // The fragment of rows r0 .. r0 + 15 (a multiple of 16) and step s.
  static __device__ __forceinline__ Move16 fragment(const char* lds, int r0, int s) {
    const int i = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
    if constexpr (!TR) {
      return *reinterpret_cast<const Move16*>(lds + 16 * slot(r0 + i, 4 * s + g));
    } else if constexpr (DT == 0) {
      Move16 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 16 * s + 4 * g + j, c = r0 + i;
        v[j] = *reinterpret_cast<const uint32_t*>(lds + 16 * slot(r, c / 4) + 4 * (c % 4));
      }
      return v;
    } else {
      // 16 lanes read four rows of 16 elements, and each gets a column of them
      Move16 v;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = 32 * s + 8 * g + 4 * h + (i >> 2), c = r0 + 4 * (i & 3);
        const char* p = lds + 16 * slot(r, c / 8) + 2 * (c % 8);
        const Half4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) Half4*)(p));
        const Move8 w = __builtin_bit_cast(Move8, t);
        v[2 * h] = w[0];
        v[2 * h + 1] = w[1];
      }
      return v;
    }
  }
};

}  // namespace lapsum
