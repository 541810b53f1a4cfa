// Attention of one new token over the cache of its sequence, for query heads that
// share key heads (group of them to one):
//
//   s_j = scale <q, k_j>,  m = max s,  l = sum e^(s_j - m),
//   y = sum e^(s_j - m) v_j / l,  lse = m + log l,  w_j = e^(s_j - lse)
//
// in one pass over the keys with the running m and l (in powers of two: s
// log2 e).  Keys and values are read once, straight into the fragments of the matrix
// cores, without LDS: a wave takes 32 keys, whose products with sixteen query
// heads are two tiles, keys by heads; a lane then holds its head's weights
// of the same eight keys that the second product, heads by dims, contracts over.
// Of a value row a lane takes neighbouring dims, so that sixteen lanes read the row whole;
// eight such rows are transposed in registers.  The cost is that of the bytes:
// 4 heads dim operations per 2 kv_heads dim elements are far below what the
// matrix cores do in that time, even where most of the sixteen heads are none.
//
// The keys of a sequence are split over workgroups of four waves, whose parts
// (unnormalised sums, m and l) attend_join_kernel joins.
//
// Types.  Scores, m, l and sums are float32.  The weights go into the second
// product as 16-bit terms of their own sum (two, which is 16 bits or more; three
// for float32 queries), which costs matrix instructions that are free here and leaves the
// outputs' own rounding as the only one.  Codes of 8 bits are whole numbers that
// bfloat16 holds exactly; their scales multiply scores and weights in float32, and
// queries of another type are split into bfloat16 terms too.  A float32 cache uses
// the float32 instructions.
#include "matrix.hpp"
#include "paged.hpp"

namespace lapsum {
namespace {

constexpr int AW = 4;                  // waves
constexpr int AT = AW * kWave;
constexpr int AK = 32;                 // keys of a wave's step

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x05040100u);
}
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}

// N elements of a cache as they lie in memory; the elements past `left` are 0.
template <int KIND, int N, bool VEC>
struct Raw {
  static constexpr int Words = N * kCacheBytes<KIND> / 4;
  uint32_t w[Words];
  __device__ __forceinline__ void load(const void* data, int64_t at, int left) {
    constexpr int B = kCacheBytes<KIND>;
    const char* p = static_cast<const char*>(data) + at * B;
#pragma unroll
    for (int i = 0; i < Words; ++i) w[i] = 0u;
    if constexpr (VEC) {
      if (left <= 0) return;
      if constexpr (Words % 4 == 0) {
#pragma unroll
        for (int i = 0; i < Words; i += 4) {
          const Move16 v = *reinterpret_cast<const Move16*>(p + 4 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) w[i + j] = v[j];
        }
      } else if constexpr (Words == 2) {
        const Move8 v = *reinterpret_cast<const Move8*>(p);
        w[0] = v[0];
        w[1] = v[1];
      } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < left) {
          if constexpr (B == 4) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
          else if constexpr (B == 2)
            w[j / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[j]) << (16 * (j % 2));
          else w[j / 4] |= static_cast<uint32_t>(reinterpret_cast<const uint8_t*>(p)[j]) << (8 * (j % 4));
        }
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < Words; ++i) w[i] = 0u;
  }
  // Elements 2 i and 2 i + 1 in 16 bits each.
  __device__ __forceinline__ void halves(uint32_t (&h)[N / 2]) const {
    if constexpr (kCacheBytes<KIND> == 2) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) h[i] = w[i];
    } else {
#pragma unroll
      for (int i = 0; i < Words; ++i) {
        float x[4];
        decode4<KIND>(w[i], x);   // (exact in bfloat16: the upper halves)
        h[2 * i] = high_halves(__float_as_uint(x[0]), __float_as_uint(x[1]));
        h[2 * i + 1] = high_halves(__float_as_uint(x[2]), __float_as_uint(x[3]));
      }
    }
  }
};

// Eight floats as T fragments of type MT whose sum they are.
template <int MT, int T>
__device__ __forceinline__ void split8(const float (&x)[8], Move16 (&f)[T]) {
  float rest[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) rest[j] = x[j];
#pragma unroll
  for (int t = 0; t < T; ++t) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t a = Elem<MT>::put(rest[2 * j]), b = Elem<MT>::put(rest[2 * j + 1]);
      f[t][j] = a | (b << 16);
      if (t + 1 < T) {
        rest[2 * j] -= Elem<MT>::get(a);
        rest[2 * j + 1] -= Elem<MT>::get(b);
      }
    }
  }
}

// The larger of a value and those of the lanes 16, 32 and 48 away; their sum.
template <class Op>
__device__ __forceinline__ float across_rows(float x, Op op) {
  x = op(x, __shfl_xor(x, 16));
  return op(x, __shfl_xor(x, 32));
}

// dim at most 32 ND.
template <int QT, int KIND, int ND, bool VEC>
__global__ __launch_bounds__(AT) void cache_attend_kernel(AttendArgs a) {
  constexpr bool F32 = KIND == 0;
  constexpr int MT = KIND <= 2 ? KIND : 1;
  constexpr int TQ = KIND <= 2 ? 1 : QT == 1 ? 1 : QT == 2 ? 2 : 3;   // terms of a query
  constexpr int TP = QT == 0 ? 3 : 2;                                   // and of a weight
  constexpr int KN = F32 ? 4 : 8;                  // dims of a lane in a step of the first product
  constexpr int KS = ND * 32 / (4 * KN);           // its steps
  constexpr int VN = F32 || ND <= 2 ? 4 : 8;       // dims of a lane in a piece of a value row
  constexpr int VC = (ND * 32 + 16 * VN - 1) / (16 * VN);
  // float16 weights are scaled to the upper end of their range, where small ones keep their bits
  constexpr float kUp = MT == 2 ? 15.0f : 0.0f;
  __shared__ float parts[AW][16][ND * 32 + 2];

  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i16 = lane & 15, g = lane >> 4;
  const int rows = a.kv * a.tiles;
  const int split = blockIdx.x / (a.batch * rows), at = blockIdx.x % (a.batch * rows);
  const int b = at / rows, h = at % rows / a.tiles, tile = at % a.tiles;
  const int head0 = h * a.group + 16 * tile;
  const int live = min(16, a.group - 16 * tile);

  // the keys [from, to) of this workgroup, in steps from a multiple of 32 on
  const int64_t len = min(static_cast<int64_t>(max(a.lens[b], 0)), a.room);
  const int64_t start = a.window > 0 && len > a.window ? len - a.window : 0;
  const int64_t base = start / AK * AK + static_cast<int64_t>(split) * a.chunk;
  const int from = static_cast<int>(max(start, base));
  const int to = static_cast<int>(min(len, base + a.chunk));

  Move16 q[KS][TQ];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int d = s * 4 * KN + KN * g;
    const int64_t from_q = b * a.q_b + (head0 + i16) * a.q_h + d;
    const int left = i16 < live ? a.dim - d : 0;
    using raw = typename Elem<QT>::raw;
    const raw* p = static_cast<const raw*>(a.q) + from_q;
    float x[8] = {};
#pragma unroll
    for (int j = 0; j < KN; ++j)
      if (j < left) x[j] = Elem<QT>::get(p[j]);
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) q[s][0][j] = __float_as_uint(x[j]);
    } else {
      split8<MT, TQ>(x, q[s]);
    }
  }

  float m = -INFINITY, l = 0.0f;
  Acc out[VC][VN] = {};
  const float scale2 = a.scale * static_cast<float>(kLog2e);
  const bool uniform = !a.t.table || a.t.size % 16 == 0;   // sixteen keys are in one page
  float* scores = a.weights ? a.weights + (static_cast<int64_t>(b) * a.heads + head0 + i16) * a.room : nullptr;

  for (int64_t k0 = base + AK * wave; k0 < to; k0 += AK * AW) {
    const int key0 = static_cast<int>(k0);
    // where the rows are; a row that does not exist is read as the cache's first, and not used
    int64_t k_at[2], v_at[2][4], ks_at[2][4], vs_at[2][4];
    bool ok[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      int page, slot;
      if (uniform) {
        find_slot(a.t, b, key0 + 16 * u, &page, &slot);
        const bool in = page >= 0;
        const int64_t pk = in ? page * a.k.page + slot * a.k.slot : 0;
        const int64_t pv = in ? page * a.v.page + slot * a.v.slot : 0;
        const int key = key0 + 16 * u + i16;
        k_at[u] = in && key < to ? pk + i16 * a.k.slot : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * g + i, kv = key0 + 16 * u + r;
          ok[u][i] = in && kv >= from && kv < to;
          v_at[u][i] = in && kv < to ? pv + r * a.v.slot : 0;
          if constexpr (KIND > 2) {
            ks_at[u][i] = in && kv < to ? page * a.k.scale_page + slot + r : 0;
            vs_at[u][i] = in && kv < to ? page * a.v.scale_page + slot + r : 0;
          }
        }
      } else {
        const int key = key0 + 16 * u + i16;
        find_slot(a.t, b, key, &page, &slot);
        k_at[u] = page >= 0 && key < to ? page * a.k.page + slot * a.k.slot : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int kv = key0 + 16 * u + 4 * g + i;
          find_slot(a.t, b, kv, &page, &slot);
          const bool in = page >= 0 && kv < to;
          ok[u][i] = in && kv >= from;
          v_at[u][i] = in ? page * a.v.page + slot * a.v.slot : 0;
          if constexpr (KIND > 2) {
            ks_at[u][i] = in ? page * a.k.scale_page + slot : 0;
            vs_at[u][i] = in ? page * a.v.scale_page + slot : 0;
          }
        }
      }
    }
    Raw<KIND, KN, VEC> kr[2][KS];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int d = s * 4 * KN + KN * g;
        kr[u][s].load(a.k.data, k_at[u] + h * a.k.head + d, a.dim - d);
      }
    Raw<KIND, VN, VEC> vr[VC][2][4];
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = c * 16 * VN + VN * i16;
          vr[c][u][i].load(a.v.data, v_at[u][i] + h * a.v.head + d, a.dim - d);
        }
    float ks[2][4], vs[2][4];
    if constexpr (KIND > 2) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ks[u][i] = a.k.scale[h * a.k.scale_head + ks_at[u][i]] * scale2;
          vs[u][i] = a.v.scale[h * a.v.scale_head + vs_at[u][i]];
        }
    }

    Acc sc[2] = {};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        Move16 f;
        if constexpr (F32) {
          f = Move16{kr[u][s].w[0], kr[u][s].w[1], kr[u][s].w[2], kr[u][s].w[3]};
        } else {
          uint32_t hv[4];
          kr[u][s].halves(hv);
          f = Move16{hv[0], hv[1], hv[2], hv[3]};
        }
#pragma unroll
        for (int t = 0; t < TQ; ++t) sc[u] = mma<MT>(f, q[s][t], sc[u]);
      }
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = KIND > 2 ? sc[u][i] * ks[u][i] : sc[u][i] * scale2;
        sc[u][i] = ok[u][i] ? x : -INFINITY;
        most = fmaxf(most, sc[u][i]);
      }
    if (scores && i16 < live) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (key0 + 16 * u + 4 * g + i < to) scores[key0 + 16 * u + 4 * g + i] = sc[u][i];
    }
    if (__any(most > m)) {
      const float now = across_rows(fmaxf(m, most), [](float x, float y) { return fmaxf(x, y); });
      const float shrink = now == -INFINITY ? 1.0f : exp2_fast(m - now);
      m = now;
      l *= shrink;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = __shfl(shrink, 4 * g + i);
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
          for (int e = 0; e < VN; ++e) out[c][e][i] *= f;
      }
    }
    const float ref = m == -INFINITY ? 0.0f : m - kUp;
    float p[8];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = exp2_fast(sc[u][i] - ref);
        l += x;
        p[4 * u + i] = x;
        if constexpr (KIND > 2) p[4 * u + i] = ok[u][i] ? x * vs[u][i] : 0.0f;
      }
    // (a value that is not there may hold anything, and 0 of it may be NaN)
    bool all = true;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) all = all && ok[u][i];
    if (!__all(all)) {
#pragma unroll
      for (int c = 0; c < VC; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!ok[u][i]) vr[c][u][i].clear();
    }
    if constexpr (F32) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < VC; ++c)
#pragma unroll
            for (int e = 0; e < VN; ++e)
              out[c][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[4 * u + i], __uint_as_float(vr[c][u][i].w[e]),
                                                               out[c][e], 0, 0, 0);
    } else {
      Move16 w[TP];
      split8<MT, TP>(p, w);
#pragma unroll
      for (int c = 0; c < VC; ++c) {
        uint32_t hv[8][VN / 2];
#pragma unroll
        for (int j = 0; j < 8; ++j) vr[c][j / 4][j % 4].halves(hv[j]);
#pragma unroll
        for (int e = 0; e < VN; ++e) {
          Move16 f;
#pragma unroll
          for (int d = 0; d < 4; ++d)
            f[d] = e % 2 ? high_halves(hv[2 * d][e / 2], hv[2 * d + 1][e / 2])
                         : low_halves(hv[2 * d][e / 2], hv[2 * d + 1][e / 2]);
#pragma unroll
          for (int t = 0; t < TP; ++t) out[c][e] = mma<MT>(w[t], f, out[c][e]);
        }
      }
    }
  }

  // the waves' parts, joined
  l = across_rows(l, [](float x, float y) { return x + y; });
  if (g == 0) {
    parts[wave][i16][ND * 32] = m;
    parts[wave][i16][ND * 32 + 1] = l;
  }
#pragma unroll
  for (int c = 0; c < VC; ++c)
#pragma unroll
    for (int e = 0; e < VN; ++e) {
      const int d = c * 16 * VN + VN * i16 + e;
      if (d < ND * 32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) parts[wave][4 * g + i][d] = out[c][e][i];
      }
    }
  __syncthreads();
  using raw = typename Elem<QT>::raw;
  for (int r = wave; r < live; r += AW) {
    float mw[AW], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < AW; ++w) {
      mw[w] = parts[w][r][ND * 32];
      top = fmaxf(top, mw[w]);
    }
#pragma unroll
    for (int w = 0; w < AW; ++w) {
      mw[w] = mw[w] == -INFINITY ? 0.0f : exp2_fast(mw[w] - top);
      sum += mw[w] * parts[w][r][ND * 32 + 1];
    }
    const int64_t row = static_cast<int64_t>(b) * a.heads + head0 + r;
    float* part = a.part ? a.part + (static_cast<int64_t>(split) * a.batch * a.heads + row) * (a.dim + 2) : nullptr;
    for (int d = lane; d < a.dim; d += kWave) {
      float y = 0.0f;
#pragma unroll
      for (int w = 0; w < AW; ++w) y += mw[w] * parts[w][r][d];
      if (part) part[d] = y;
      else static_cast<raw*>(a.out)[row * a.dim + d] = Elem<QT>::put(sum == 0.0f ? 0.0f : y / sum);
    }
    if (lane == 0) {
      if (part) {
        part[a.dim] = top;
        part[a.dim + 1] = sum;
      } else if (a.lse) {
        a.lse[row] = sum == 0.0f ? -INFINITY : (top + __log2f(sum) - kUp) * static_cast<float>(1.0 / kLog2e);
      }
    }
  }
}

// The parts of a row (b, head) joined; a wave to each.
template <int QT>
__global__ __launch_bounds__(kWave) void cache_attend_join_kernel(AttendArgs a, float up) {
  const int64_t row = blockIdx.x, rows = static_cast<int64_t>(a.batch) * a.heads;
  const int lane = lane_id();
  const int64_t step = rows * (a.dim + 2);
  const float* part = a.part + row * (a.dim + 2);
  float top = -INFINITY;
  for (int s = lane; s < a.splits; s += kWave) top = fmaxf(top, part[s * step + a.dim]);
  top = wave_max(top, -INFINITY);
  float sum = 0.0f;
  for (int s = lane; s < a.splits; s += kWave) {
    const float m = part[s * step + a.dim];
    if (m != -INFINITY) sum += exp2_fast(m - top) * part[s * step + a.dim + 1];
  }
  sum = wave_sum(sum);
  using raw = typename Elem<QT>::raw;
  for (int d = lane; d < a.dim; d += kWave) {
    float y = 0.0f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
      const float m = part[s * step + a.dim];
      y += (m == -INFINITY ? 0.0f : exp2_fast(m - top)) * part[s * step + d];
    }
    static_cast<raw*>(a.out)[row * a.dim + d] = Elem<QT>::put(sum == 0.0f ? 0.0f : y / sum);
  }
  if (lane == 0 && a.lse)
    a.lse[row] = sum == 0.0f ? -INFINITY : (top + __log2f(sum) - up) * static_cast<float>(1.0 / kLog2e);
}

// Scores in powers of two to weights, by the row's lse; 0 outside its keys.
__global__ __launch_bounds__(256) void cache_weights_kernel(AttendArgs a) {
  const int64_t pieces = (a.room + 255) / 256;
  const int64_t row = blockIdx.x / pieces, j = blockIdx.x % pieces * 256 + threadIdx.x;
  if (j >= a.room) return;
  const int b = static_cast<int>(row / a.heads);
  const int64_t len = min(static_cast<int64_t>(max(a.lens[b], 0)), a.room);
  const int64_t start = a.window > 0 && len > a.window ? len - a.window : 0;
  const float lse = a.lse[row] * static_cast<float>(kLog2e);
  float w = 0.0f;
  if (j >= start && j < len && a.lse[row] != -INFINITY) w = exp2_fast(a.weights[row * a.room + j] - lse);
  a.weights[row * a.room + j] = w;
}

}  // namespace

// ------------------------------------------------------------- launchers ---
void attend_plan(int64_t batch, int64_t heads, int64_t kv, int64_t room, int64_t window, int* splits,
                 int* chunk) {
  constexpr int64_t step = AK * AW;
  const int64_t rows = batch * kv * ((heads / kv + 15) / 16);
  const int64_t keys = window > 0 && window < room ? (window + AK < room ? window + AK : room) : room;
  int64_t each = (keys * rows + 2047) / 2048;
  each = (each + step - 1) / step * step;
  if (each < step) each = step;
  *chunk = static_cast<int>(each);
  *splits = static_cast<int>(keys < 1 ? 1 : (keys + each - 1) / each);
}

hipError_t launch_cache_attend(const AttendArgs& a, int dtype, int kind, bool vec, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.splits) * a.batch * a.kv * a.tiles));
  {
    ProfScope ps_("cache_attend", s);
    const auto launch = [&](auto qt, auto kd) {
      constexpr int QT = decltype(qt)::value, KIND = decltype(kd)::value;
      if (!vec) hipLaunchKernelGGL((cache_attend_kernel<QT, KIND, 8, false>), grid, dim3(AT), 0, s, a);
      else if (a.dim <= 64) hipLaunchKernelGGL((cache_attend_kernel<QT, KIND, 2, true>), grid, dim3(AT), 0, s, a);
      else if (a.dim <= 96) hipLaunchKernelGGL((cache_attend_kernel<QT, KIND, 3, true>), grid, dim3(AT), 0, s, a);
      else if (a.dim <= 128) hipLaunchKernelGGL((cache_attend_kernel<QT, KIND, 4, true>), grid, dim3(AT), 0, s, a);
      else hipLaunchKernelGGL((cache_attend_kernel<QT, KIND, 8, true>), grid, dim3(AT), 0, s, a);
    };
    const auto of = [&](auto qt) {
      if (kind == kInt8) launch(qt, std::integral_constant<int, kInt8>{});
      else if (kind == kE4m3) launch(qt, std::integral_constant<int, kE4m3>{});
      else launch(qt, std::integral_constant<int, decltype(qt)::value>{});
    };
    if (dtype == 0) of(std::integral_constant<int, 0>{});
    else if (dtype == 1) of(std::integral_constant<int, 1>{});
    else of(std::integral_constant<int, 2>{});
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned rows = static_cast<unsigned>(static_cast<int64_t>(a.batch) * a.heads);
  if (a.part) {
    ProfScope ps_("cache_attend_join", s);
    const float up = kind == 2 ? 15.0f : 0.0f;
    if (dtype == 0) hipLaunchKernelGGL((cache_attend_join_kernel<0>), dim3(rows), dim3(kWave), 0, s, a, up);
    else if (dtype == 1) hipLaunchKernelGGL((cache_attend_join_kernel<1>), dim3(rows), dim3(kWave), 0, s, a, up);
    else hipLaunchKernelGGL((cache_attend_join_kernel<2>), dim3(rows), dim3(kWave), 0, s, a, up);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.weights) {
    ProfScope ps_("cache_weights", s);
    const int64_t pieces = (a.room + 255) / 256;
    hipLaunchKernelGGL(cache_weights_kernel, dim3(static_cast<unsigned>(rows * pieces)), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace lapsum
