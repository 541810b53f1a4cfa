// A key-value cache in pages: new entries written, as they are or in 8 bits, and
// the entries of each sequence read back.
//
// A row x in 8 bits is codes c and a scale s = max(r max |x|, 2^-126), r the float32
// nearest 1 / M, M = 127 (int8) or 448 (e4m3): c is x / s rounded to the nearest
// code, ties to even, and stands for c s.  (The largest |x| / s is M to within two
// roundings, which the code rounds away.)  The division is exact to rounding, as
// a code off by one is off by a whole step.  (2^-126 keeps s a normal number; such a row is below every use.)  A row
// with an infinity or NaN gets the scale NaN and codes 0, so that it reads back as
// NaN and not as numbers.
//
// Both kernels move bytes: a team of 16 or 32 lanes takes a row, eight elements to
// a lane.
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

template <int DT, int KIND, int TEAM, bool VEC>
__global__ __launch_bounds__(PT) void cache_append_kernel(AppendArgs a) {
  const int lane = threadIdx.x % TEAM;
  const uint32_t row = blockIdx.x * static_cast<uint32_t>(PT / TEAM) + threadIdx.x / TEAM;
  const uint32_t total = static_cast<uint32_t>(a.batch) * static_cast<uint32_t>(a.kv) * static_cast<uint32_t>(a.fresh);
  const bool there = row < total;
  const uint32_t bh = there ? row / static_cast<uint32_t>(a.fresh) : 0;
  const int i = there ? static_cast<int>(row - bh * static_cast<uint32_t>(a.fresh)) : 0;
  const int b = static_cast<int>(bh / static_cast<uint32_t>(a.kv));
  const int h = static_cast<int>(bh) - b * a.kv;
  int page = -1, slot = 0;
  const int64_t at = static_cast<int64_t>(a.seen[b]) + i;
  if (there && (!a.count || i < a.count[b]) && at >= 0 && at <= 2147483647LL)
    find_slot(a.t, b, static_cast<int>(at), &page, &slot);
  // (the whole wave goes on: teams reduce together)
  const int left = page >= 0 ? a.dim - PN * lane : 0;
  float x[2][PN] = {};
#pragma unroll
  for (int n = 0; n < 2; ++n)
    load8<DT, VEC>(a.src[n], b * a.src_b[n] + h * a.src_h[n] + i * a.src_i[n] + PN * lane, left, x[n]);
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const PagedCache& c = a.cache[n];
    const int64_t to = page * c.page + h * c.head + slot * c.slot + PN * lane;
    if constexpr (KIND <= 2) {
      store8<DT, VEC>(c.data, to, left, x[n]);
    } else {
      constexpr float unit = 1.0f / (KIND == kInt8 ? 127.0f : 448.0f);
      // (magnitudes as whole numbers: infinities and NaN are the largest)
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < PN; ++j) {
        const uint32_t u = __float_as_uint(x[n][j]) & 0x7fffffffu;
        m = u > m ? u : m;
      }
      m = team_most<TEAM>(m);
      const bool odd = m >= 0x7f800000u;
      const float scale = fmaxf(__uint_as_float(odd ? 0u : m) * unit, 1.17549435e-38f);
      float y[PN];
#pragma unroll
      for (int j = 0; j < PN; ++j) y[j] = odd ? 0.0f : x[n][j] / scale;
      const Move8 codes = {encode4<KIND>(y), encode4<KIND>(y + 4)};
      store_codes<VEC>(c.data, to, left, codes);
      if (lane == 0 && page >= 0)
        c.scale[page * c.scale_page + h * c.scale_head + slot] = odd ? NAN : scale;
    }
  }
}

template <int KIND, int DO, int TEAM, bool VEC>
__global__ __launch_bounds__(PT) void cache_read_kernel(ReadArgs a) {
  const int lane = threadIdx.x % TEAM;
  const uint32_t row = blockIdx.x * static_cast<uint32_t>(PT / TEAM) + threadIdx.x / TEAM;
  const uint32_t total = static_cast<uint32_t>(a.batch) * static_cast<uint32_t>(a.kv) * static_cast<uint32_t>(a.room);
  if (row >= total) return;
  const uint32_t bh = row / static_cast<uint32_t>(a.room);
  const int i = static_cast<int>(row - bh * static_cast<uint32_t>(a.room));
  const int b = static_cast<int>(bh / static_cast<uint32_t>(a.kv));
  const int h = static_cast<int>(bh) - b * a.kv;
  int page = -1, slot = 0;
  if (i < a.lens[b]) find_slot(a.t, b, i, &page, &slot);
  const int left = a.dim - PN * lane;
  float x[PN] = {};
  if (page >= 0) {
    const PagedCache& c = a.cache;
    const int64_t from = page * c.page + h * c.head + slot * c.slot + PN * lane;
    if constexpr (KIND <= 2) {
      load8<KIND, VEC>(c.data, from, left, x);
    } else {
      const Move8 codes = load_codes<VEC>(c.data, from, left);
      const float scale = c.scale[page * c.scale_page + h * c.scale_head + slot];
      decode4<KIND>(codes[0], x);
      decode4<KIND>(codes[1], x + 4);
#pragma unroll
      for (int j = 0; j < PN; ++j) x[j] *= scale;
    }
  }
  store8<DO, VEC>(a.out, static_cast<int64_t>(row) * a.dim + PN * lane, left, x);
}

}  // namespace

// ------------------------------------------------------------- launchers ---
hipError_t launch_cache_append(AppendArgs a, int dtype, int kind, bool vec, hipStream_t s) {
  const int team = a.dim <= 16 * PN ? 16 : 32;
  const int64_t rows = static_cast<int64_t>(a.batch) * a.kv * a.fresh;
  const dim3 grid(static_cast<unsigned>((rows + PT / team - 1) / (PT / team)));
  ProfScope ps_("cache_append", s);
  const auto launch = [&](auto dt, auto kd) {
    constexpr int DT = decltype(dt)::value, KIND = decltype(kd)::value;
    if (team == 16 && vec) hipLaunchKernelGGL((cache_append_kernel<DT, KIND, 16, true>), grid, dim3(PT), 0, s, a);
    else if (team == 16) hipLaunchKernelGGL((cache_append_kernel<DT, KIND, 16, false>), grid, dim3(PT), 0, s, a);
    else if (vec) hipLaunchKernelGGL((cache_append_kernel<DT, KIND, 32, true>), grid, dim3(PT), 0, s, a);
    else hipLaunchKernelGGL((cache_append_kernel<DT, KIND, 32, false>), grid, dim3(PT), 0, s, a);
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
  const int team = a.dim <= 16 * PN ? 16 : 32;
  const int64_t rows = static_cast<int64_t>(a.batch) * a.kv * a.room;
  const dim3 grid(static_cast<unsigned>((rows + PT / team - 1) / (PT / team)));
  ProfScope ps_("cache_read", s);
  const auto launch = [&](auto kd, auto dout) {
    constexpr int KIND = decltype(kd)::value, DO = decltype(dout)::value;
    if (team == 16 && vec) hipLaunchKernelGGL((cache_read_kernel<KIND, DO, 16, true>), grid, dim3(PT), 0, s, a);
    else if (team == 16) hipLaunchKernelGGL((cache_read_kernel<KIND, DO, 16, false>), grid, dim3(PT), 0, s, a);
    else if (vec) hipLaunchKernelGGL((cache_read_kernel<KIND, DO, 32, true>), grid, dim3(PT), 0, s, a);
    else hipLaunchKernelGGL((cache_read_kernel<KIND, DO, 32, false>), grid, dim3(PT), 0, s, a);
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
