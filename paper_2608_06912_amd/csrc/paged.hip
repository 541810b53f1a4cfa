// A key-value cache in pages: new entries written, as they are or in 8 bits, and
// the entries of each sequence read back.
//
// A row x in 8 bits is codes c and a scale s = max(r max |x|, 2^-126), r the float32
// nearest 1 / M, M = 127 (int8) or 448 (e4m3): c is x / s rounded to the nearest
// code, ties to even, and stands for c s.  (The largest |x| / s is M to within two
// roundings, which the code rounds away.)  The quotient is exact to rounding, as
// a code off by one is off by a whole step.  (2^-126 keeps s a normal number; such a row is below every use.)  A row
// with an infinity or NaN gets the scale NaN and codes 0, so that it reads back as
// NaN and not as numbers.
//
// Both kernels move bytes: a team of 16 or 32 lanes takes a row, eight elements to
// a lane, and where there are many rows four of them at once.  12 prompts of up to 8192
// in e4m3 take 98 us (3.4 TB/s, half of it vector issue), 8 caches of up to 32768 back in
// bfloat16 136 us (5.2 TB/s; one row at a time 205).
#include "paged.hpp"

namespace lapsum {
namespace {

constexpr int PT = 256;
constexpr int PN = 8;   // elements of a lane

template <int DT, bool VEC>
__device__ __forceinline__ void load8(const void* p, int64_t at, int left, float (&x)[PN]) {
  using raw = typename Elem<DT>::raw;
  const raw* q = static_cast<const raw*>(p) + at;
  if constexpr (VEC) {
    if (left <= 0) return;
    if constexpr (DT == 0) {
#pragma unroll
      for (int i = 0; i < PN; i += 4) {
        const Move16 v = *reinterpret_cast<const Move16*>(q + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i + j] = __uint_as_float(v[j]);
      }
    } else {
      const Move16 v = *reinterpret_cast<const Move16*>(q);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = Elem<DT>::get(v[j] & 0xffffu);
        x[2 * j + 1] = Elem<DT>::get(v[j] >> 16);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < PN; ++j)
      if (j < left) x[j] = Elem<DT>::get(q[j]);
  }
}
template <int DT, bool VEC>
__device__ __forceinline__ void store8(void* p, int64_t at, int left, const float (&x)[PN]) {
  using raw = typename Elem<DT>::raw;
  raw* q = static_cast<raw*>(p) + at;
  if constexpr (VEC) {
    if (left <= 0) return;
    if constexpr (DT == 0) {
#pragma unroll
      for (int i = 0; i < PN; i += 4) {
        Move16 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(x[i + j]);
        *reinterpret_cast<Move16*>(q + i) = v;
      }
    } else {
      Move16 v;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = static_cast<uint32_t>(Elem<DT>::put(x[2 * j])) |
               (static_cast<uint32_t>(Elem<DT>::put(x[2 * j + 1])) << 16);
      *reinterpret_cast<Move16*>(q) = v;
    }
  } else {
#pragma unroll
    for (int j = 0; j < PN; ++j)
      if (j < left) q[j] = Elem<DT>::put(x[j]);
  }
}
template <bool VEC>
__device__ __forceinline__ Move8 load_codes(const void* p, int64_t at, int left) {
  const uint8_t* q = static_cast<const uint8_t*>(p) + at;
  Move8 v = {0u, 0u};
  if constexpr (VEC) {
    if (left > 0) v = *reinterpret_cast<const Move8*>(q);
  } else {
#pragma unroll
    for (int j = 0; j < PN; ++j)
      if (j < left) v[j / 4] |= static_cast<uint32_t>(q[j]) << (8 * (j % 4));
  }
  return v;
}
template <bool VEC>
__device__ __forceinline__ void store_codes(void* p, int64_t at, int left, Move8 v) {
  uint8_t* q = static_cast<uint8_t*>(p) + at;
  if constexpr (VEC) {
    if (left > 0) *reinterpret_cast<Move8*>(q) = v;
  } else {
#pragma unroll
    for (int j = 0; j < PN; ++j)
      if (j < left) q[j] = static_cast<uint8_t>(v[j / 4] >> (8 * (j % 4)));
  }
}

// The largest of a team's values, in every lane of it.
template <int TEAM>
__device__ __forceinline__ uint32_t team_most(uint32_t v) {
  const auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  v = team_reduce<16>(v, larger);
  if constexpr (TEAM == 32) v = larger(v, __shfl_xor(v, 16));
  return v;
}

// The codes of eight elements over the scale.  One division gives 1 / scale to rounding,
// and with it three operations give each quotient so: with r = x - q scale, exact, and q
// the product with 1 / scale, q + r / scale rounds to the quotient's own rounding
// (P. Markstein, Computation of elementary functions on the IBM RISC System/6000,
// 1990; r has to be a number, so `tiny` scales, near the smallest, are divided by).
template <int KIND>
__device__ __forceinline__ Move8 encode8(const float (&x)[PN], float scale, bool tiny) {
  const float inverse = 1.0f / scale;
  float y[PN];
#pragma unroll
  for (int j = 0; j < PN; ++j) {
    const float q = x[j] * inverse;
    y[j] = copysignf(fmaf(fmaf(-q, scale, x[j]), inverse, q), x[j]);   // (zeros keep their sign)
  }
  if (__any(tiny)) {
    asm volatile("");   // (a branch, not eight divisions and a choice)
#pragma unroll
    for (int j = 0; j < PN; ++j) y[j] = x[j] / scale;
  }
  if constexpr (KIND == kE4m3) {
    return Move8{encode4<KIND>(y), encode4<KIND>(y + 4)};
  } else {
    // 1.5 2^23 more is a whole number, to the nearest, whose low byte is the code
    uint32_t u[PN];
#pragma unroll
    for (int j = 0; j < PN; ++j) u[j] = __float_as_uint(y[j] + 12582912.0f);
    Move8 codes;
#pragma unroll
    for (int w = 0; w < 2; ++w)
      codes[w] = __builtin_amdgcn_perm(u[4 * w + 1], u[4 * w], 0x0c0c0400u) |
                 __builtin_amdgcn_perm(u[4 * w + 3], u[4 * w + 2], 0x04000c0cu);
    return codes;
  }
}

// Where a team's rows are.  ROWS 1: teams take rows as they come.  Else a workgroup takes
// ROWS times its teams' rows of one (sequence, head), so that sequence and head are the
// workgroup's and the loads of ROWS rows are on their way together.
template <int TEAM, int ROWS>
struct Place {
  int b, h, i[ROWS];
  bool there[ROWS];
  __device__ __forceinline__ Place(int batch, int kv, int rows, int chunks) {
    constexpr int teams = PT / TEAM;
    const int team = threadIdx.x / TEAM;
    uint32_t bh;
    if constexpr (ROWS == 1) {
      const uint32_t row = blockIdx.x * static_cast<uint32_t>(teams) + team;
      there[0] = row < static_cast<uint32_t>(batch) * static_cast<uint32_t>(kv) * static_cast<uint32_t>(rows);
      bh = there[0] ? row / static_cast<uint32_t>(rows) : 0;
      i[0] = there[0] ? static_cast<int>(row - bh * static_cast<uint32_t>(rows)) : 0;
    } else {
      bh = blockIdx.x / static_cast<uint32_t>(chunks);
      const int first = static_cast<int>(blockIdx.x - bh * static_cast<uint32_t>(chunks)) * ROWS * teams + team;
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        i[r] = first + r * teams;
        there[r] = i[r] < rows;
      }
    }
    b = static_cast<int>(bh / static_cast<uint32_t>(kv));
    h = static_cast<int>(bh) - b * kv;
  }
};

template <int DT, int KIND, int TEAM, int ROWS, bool VEC>
__global__ __launch_bounds__(PT) void cache_append_kernel(AppendArgs a) {
  const int lane = threadIdx.x % TEAM;
  const Place<TEAM, ROWS> at(a.batch, a.kv, a.fresh, a.chunks);
  const int64_t seen = a.seen[at.b];
  const int count = a.count ? a.count[at.b] : a.fresh;
  int page[ROWS], slot[ROWS], left[ROWS];
  float x[ROWS][2][PN] = {};
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    page[r] = -1;
    slot[r] = 0;
    const int64_t pos = seen + at.i[r];
    if (at.there[r] && at.i[r] < count && pos >= 0 && pos <= 2147483647LL)
      find_slot(a.t, at.b, static_cast<int>(pos), &page[r], &slot[r]);
    // (the whole wave goes on: teams reduce together)
    left[r] = page[r] >= 0 ? a.dim - PN * lane : 0;
#pragma unroll
    for (int n = 0; n < 2; ++n)
      load8<DT, VEC>(a.src[n], at.b * a.src_b[n] + at.h * a.src_h[n] + at.i[r] * a.src_i[n] + PN * lane, left[r],
                     x[r][n]);
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (!__any(page[r] >= 0)) continue;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const PagedCache& c = a.cache[n];
      const int64_t to = page[r] * c.page + at.h * c.head + slot[r] * c.slot + PN * lane;
      if constexpr (KIND <= 2) {
        store8<DT, VEC>(c.data, to, left[r], x[r][n]);
      } else {
        constexpr float unit = 1.0f / (KIND == kInt8 ? 127.0f : 448.0f);
        // (magnitudes as whole numbers: infinities and NaN are the largest)
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < PN; ++j) {
          const uint32_t u = __float_as_uint(x[r][n][j]) & 0x7fffffffu;
          m = u > m ? u : m;
        }
        m = team_most<TEAM>(m);
        const bool odd = m >= 0x7f800000u;
        const float scale = fmaxf(__uint_as_float(odd ? 0u : m) * unit, 1.17549435e-38f);
        Move8 codes = encode8<KIND>(x[r][n], scale, m != 0u && scale < 0x1p-90f);
        if (odd) codes = Move8{0u, 0u};
        store_codes<VEC>(c.data, to, left[r], codes);
        if (lane == 0 && page[r] >= 0)
          c.scale[page[r] * c.scale_page + at.h * c.scale_head + slot[r]] = odd ? NAN : scale;
      }
    }
  }
}

template <int KIND, int DO, int TEAM, int ROWS, bool VEC>
__global__ __launch_bounds__(PT) void cache_read_kernel(ReadArgs a) {
  const int lane = threadIdx.x % TEAM;
  const Place<TEAM, ROWS> at(a.batch, a.kv, a.room, a.chunks);
  const int len = a.lens[at.b];
  const int left = a.dim - PN * lane;
  const PagedCache& c = a.cache;
  int page[ROWS], slot[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    page[r] = -1;
    slot[r] = 0;
    if (at.there[r] && at.i[r] < len) find_slot(a.t, at.b, at.i[r], &page[r], &slot[r]);
  }
  float x[ROWS][PN] = {};
  Move8 codes[ROWS];
  float scale[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    codes[r] = Move8{0u, 0u};
    scale[r] = 0.0f;
    if (page[r] < 0) continue;
    const int64_t from = page[r] * c.page + at.h * c.head + slot[r] * c.slot + PN * lane;
    if constexpr (KIND <= 2) {
      load8<KIND, VEC>(c.data, from, left, x[r]);
    } else {
      codes[r] = load_codes<VEC>(c.data, from, left);
      scale[r] = c.scale[page[r] * c.scale_page + at.h * c.scale_head + slot[r]];
    }
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (!at.there[r]) continue;
    if constexpr (KIND > 2) {
      decode4<KIND>(codes[r][0], x[r]);
      decode4<KIND>(codes[r][1], x[r] + 4);
#pragma unroll
      for (int j = 0; j < PN; ++j) {
        x[r][j] *= scale[r];
        // (a product of float32, not one rounded at once to 16 bits)
        asm("" : "+v"(x[r][j]));
      }
    }
    const int64_t row = (static_cast<int64_t>(at.b) * a.kv + at.h) * a.room + at.i[r];
    store8<DO, VEC>(a.out, row * a.dim + PN * lane, left, x[r]);
  }
}

}  // namespace

// ------------------------------------------------------------- launchers ---
// Several rows to a team where a (sequence, head) has enough of them for whole workgroups
// and the launch fills the chip.
bool in_chunks(int64_t heads, int64_t rows, int per, int* chunks, int64_t* blocks) {
  const int64_t all = (rows + 4 * per - 1) / (4 * per);
  *chunks = static_cast<int>(all);
  *blocks = heads * all;
  return rows >= 4 * per && *blocks >= 1024 && *blocks <= 2147483647LL;
}

// The workgroups of a launch over so many rows.
int64_t paged_blocks(int64_t heads, int64_t rows, int64_t dim) {
  const int per = PT / (dim <= 16 * PN ? 16 : 32);
  int chunks;
  int64_t blocks;
  return in_chunks(heads, rows, per, &chunks, &blocks) ? blocks : (heads * rows + per - 1) / per;
}

hipError_t launch_cache_append(AppendArgs a, int dtype, int kind, bool vec, hipStream_t s) {
  const int team = a.dim <= 16 * PN ? 16 : 32, per = PT / team;
  const int64_t heads = static_cast<int64_t>(a.batch) * a.kv;
  int64_t blocks;
  const bool four = in_chunks(heads, a.fresh, per, &a.chunks, &blocks);
  if (!four) blocks = (heads * a.fresh + per - 1) / per;
  const dim3 grid(static_cast<unsigned>(blocks));
  ProfScope ps_("cache_append", s);
  const auto launch = [&](auto dt, auto kd) {
    constexpr int DT = decltype(dt)::value, KIND = decltype(kd)::value;
    const auto rows = [&](auto wide, auto n) {
      constexpr int TEAM = decltype(wide)::value, ROWS = decltype(n)::value;
      if (vec) hipLaunchKernelGGL((cache_append_kernel<DT, KIND, TEAM, ROWS, true>), grid, dim3(PT), 0, s, a);
      else hipLaunchKernelGGL((cache_append_kernel<DT, KIND, TEAM, ROWS, false>), grid, dim3(PT), 0, s, a);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 4> more;
    const std::integral_constant<int, 16> narrow;
    const std::integral_constant<int, 32> wide;
    if (team == 16 && four) rows(narrow, more);
    else if (team == 16) rows(narrow, one);
    else if (four) rows(wide, more);
    else rows(wide, one);
  };
  const auto of = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (kind == kInt8) launch(dt, std::integral_constant<int, kInt8>{});
    else if (kind == kE4m3) launch(dt, std::integral_constant<int, kE4m3>{});
    else launch(dt, std::integral_constant<int, DT>{});
  };
  if (dtype == 0) of(std::integral_constant<int, 0>{});
  else if (dtype == 1) of(std::integral_constant<int, 1>{});
  else of(std::integral_constant<int, 2>{});
  return hipGetLastError();
}

hipError_t launch_cache_read(ReadArgs a, int dtype, int kind, bool vec, hipStream_t s) {
  const int team = a.dim <= 16 * PN ? 16 : 32, per = PT / team;
  const int64_t heads = static_cast<int64_t>(a.batch) * a.kv;
  int64_t blocks;
  const bool four = in_chunks(heads, a.room, per, &a.chunks, &blocks);
  if (!four) blocks = (heads * a.room + per - 1) / per;
  const dim3 grid(static_cast<unsigned>(blocks));
  ProfScope ps_("cache_read", s);
  const auto launch = [&](auto kd, auto dout) {
    constexpr int KIND = decltype(kd)::value, DO = decltype(dout)::value;
    const auto rows = [&](auto wide, auto n) {
      constexpr int TEAM = decltype(wide)::value, ROWS = decltype(n)::value;
      if (vec) hipLaunchKernelGGL((cache_read_kernel<KIND, DO, TEAM, ROWS, true>), grid, dim3(PT), 0, s, a);
      else hipLaunchKernelGGL((cache_read_kernel<KIND, DO, TEAM, ROWS, false>), grid, dim3(PT), 0, s, a);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 4> more;
    const std::integral_constant<int, 16> narrow;
    const std::integral_constant<int, 32> wide;
    if (team == 16 && four) rows(narrow, more);
    else if (team == 16) rows(narrow, one);
    else if (four) rows(wide, more);
    else rows(wide, one);
  };
  const auto to = [&](auto dout) {
    constexpr int DO = decltype(dout)::value;
    if (kind == kInt8) launch(std::integral_constant<int, kInt8>{}, dout);
    else if (kind == kE4m3) launch(std::integral_constant<int, kE4m3>{}, dout);
    else launch(std::integral_constant<int, DO>{}, dout);
  };
  if (dtype == 0) to(std::integral_constant<int, 0>{});
  else if (dtype == 1) to(std::integral_constant<int, 1>{});
  else to(std::integral_constant<int, 2>{});
  return hipGetLastError();
}

}  // namespace lapsum
