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
// (unnormalised sums, m and l) cache_attend_join_kernel joins.
//
// A 16-bit cache is read at the memory's rate (four of 131072 keys 331 us, 5.7 TB/s).
// 64 ragged ones of up to 8192 keys in int8 take 145 us (3.8 TB/s; longest sequences first
// 135): 451 vector and 176 scalar instructions a step, some 190 of the former the codes'
// conversion.  The next step's loads go out before a step is used, and the table is looked up a
// step before them (with a join by four waves 163 us, 214 without).
//
// Types.  Scores, m, l and sums are float32.  The weights go into the second
// product as 16-bit terms of their own sum (two, which is 16 bits or more; three
// for float32 queries), which costs matrix instructions that are free here and leaves the
// outputs' own rounding as the only one.  (Infinity times such terms is NaN where one of them is 0
// or below, so sums that infinite values spoil are formed anew, see infinite_values.)  Codes of 8 bits are whole numbers that
// bfloat16 holds exactly; their scales multiply scores and weights in float32, and
// queries of another type are cut into bfloat16 terms too.  A float32 cache uses
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

// N elements of a cache as they lie in memory.
template <int KIND, int N, bool VEC>
struct Raw {
  static constexpr int B = kCacheBytes<KIND>, Words = N * B / 4;
  uint32_t w[Words];
  // VEC: all of them, at a multiple of their bytes; else the elements from `left` on are 0.
  __device__ __forceinline__ void load(const char* p, int left) {
    if constexpr (VEC) {
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
      clear();
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
    if constexpr (B == 2) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) h[i] = w[i];
    } else if constexpr (KIND == kE4m3) {
#pragma unroll
      for (int i = 0; i < Words; ++i) {
        h[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false));
        h[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true));
      }
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
// Any floats as T fragments of bfloat16: eight bits of each after the others, towards zero, so that
// no term and no sum of some is larger than the whole; infinity and zeros (three are a float's 24 bits,
// two more than float16's 11).
template <int T>
__device__ __forceinline__ void split8_any(const float (&x)[8], Move16 (&f)[T]) {
  float rest[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) rest[j] = x[j];
#pragma unroll
  for (int t = 0; t < T; ++t) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[t][j] = high_halves(__float_as_uint(rest[2 * j]), __float_as_uint(rest[2 * j + 1]));
#pragma unroll
    for (int j = 0; j < 8; ++j)
      rest[j] = fabsf(rest[j]) == INFINITY ? 0.0f : rest[j] - __uint_as_float(__float_as_uint(rest[j]) & 0xffff0000u);
  }
}

// The larger of a value and those of the lanes 16, 32 and 48 away; their sum.
template <class Op>
__device__ __forceinline__ float across_rows(float x, Op op) {
  x = op(x, __shfl_xor(x, 16));
  return op(x, __shfl_xor(x, 32));
}

// What a step has on its way: 32 keys' and values' elements and scales.
template <int QT, int KIND, int ND, bool VEC>
struct Step {
  static constexpr bool F32 = KIND == 0;
  static constexpr int KN = F32 ? 4 : 8;           // dims of a lane in a part of the first product
  static constexpr int KS = ND * 32 / (4 * KN);    // its parts
  static constexpr int VN = F32 || ND <= 2 ? 4 : 8;   // dims of a lane in a piece of a value row
  static constexpr int VC = (ND * 32 + 16 * VN - 1) / (16 * VN);
  Raw<KIND, KN, VEC> k[2][KS];
  Raw<KIND, VN, VEC> v[VC][2][4];
  float ks[2][4], vs[2][4];
  // the keys' pages exist: of a tile (UNIFORM), or of a lane's own four
  bool page[2], there[2][4];
};

// Sums of a wave that values which are not numbers take part in: what these alone make of
// them, infinity of their sign or NaN, by the whole weights.  Goes through the wave's keys, eight
// at once, and looks at the weights of those with infinite values; lanes share the dims.  parts:
// the wave's sums, and each head's largest score in powers of two and total behind them.
//
// Four bfloat16 caches of 131072 keys with an infinity in every 64th value take 1370 us; without
// any, and with NaN in as many or in all of them, or in keys, 335 to 345.
template <int QT, int KIND, int ND>
__device__ __forceinline__ void infinite_values(const AttendArgs& a, float (*parts)[ND * 32 + 2], float up, float scale2,
                                                int b, int h, int head0, int live, int64_t first, int from, int to) {
  static_assert(QT == KIND, "8-bit codes are numbers");
  using raw = typename Elem<KIND>::raw;
  constexpr int NT = (ND * 32 + kWave - 1) / kWave, Ahead = 8;
  const int lane = lane_id();
  // (a total that is NaN has left nothing but NaN)
  uint32_t heads = 0;
  for (int r = 0; r < live; ++r) heads |= parts[r][ND * 32 + 1] >= 0.0f ? 1u << r : 0u;
  heads = __builtin_amdgcn_readfirstlane(heads);
  if (!heads) return;
  const float turn = a.scale < 0.0f ? -1.0f : a.scale > 0.0f ? 1.0f : 0.0f;
  const auto is_nan = [](float x) { return x != x; };
  // bit t: such a value of the lane's t-th dim has been met; one that is NaN, or there is none
  uint32_t before = 0, done = (1u << NT) - 1u;
  for (int r = 0; r < live; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int d = lane + kWave * t;
      if ((heads >> r & 1u) && d < a.dim && !(fabsf(parts[r][d]) < INFINITY)) done &= ~(1u << t);
    }
  const auto load = [&](int key, const raw** k, float (&v)[NT]) {
    int page = -1, slot = 0;
    if (key >= from && key < to) find_slot(a.t, b, key, &page, &slot);
    const bool there = page >= 0;
    if (!there) page = slot = 0;
    *k = static_cast<const raw*>(a.k.data) + (page * a.k.page + h * a.k.head + slot * a.k.slot);
    const raw* p = static_cast<const raw*>(a.v.data) + (page * a.v.page + h * a.v.head + slot * a.v.slot);
    uint32_t odd = 0;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int d = lane + kWave * t;
      v[t] = Elem<KIND>::get(p[d < a.dim ? d : 0]);
      odd |= there && !(fabsf(v[t]) < INFINITY) ? 1u << t : 0u;
    }
    return odd & ~done;
  };
  for (int64_t k0 = first; k0 < to; k0 += AK * AW)
    for (int j0 = 0; j0 < AK; j0 += Ahead) {
      const raw* k;
      float v[NT];
      uint32_t some = 0;
#pragma unroll
      for (int j = 0; j < Ahead; ++j) some |= load(static_cast<int>(min(k0 + j0 + j, int64_t(to))), &k, v);
      if (!__any(some != 0u)) continue;
      for (int j = 0; j < Ahead; ++j) {
        const uint32_t odd = load(static_cast<int>(min(k0 + j0 + j, int64_t(to))), &k, v);
        if (!__any(odd != 0u)) continue;
        bool weigh = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) weigh = weigh || ((odd >> t & 1u) && !is_nan(v[t]));
        weigh = __any(weigh);
        for (int r = 0; r < live; ++r) {
          if (!(heads >> r & 1u)) continue;
          float p = 1.0f;
          if (weigh) {
            const raw* q = static_cast<const raw*>(a.q) + b * a.q_b + (head0 + r) * a.q_h;
            float s = 0.0f;
            for (int d = lane; d < a.dim; d += kWave) s = fmaf(Elem<KIND>::get(q[d]) * turn, Elem<KIND>::get(k[d]), s);
            const float top = parts[r][ND * 32];
            p = exp2_fast(fmaf(wave_sum(s), scale2, up - (top == -INFINITY ? 0.0f : top)));
          }
#pragma unroll
          for (int t = 0; t < NT; ++t)
            if (odd >> t & 1u) {
              float* sum = &parts[r][lane + kWave * t];
              *sum = (before >> t & 1u ? *sum : 0.0f) + p * v[t];
            }
        }
        before |= odd;
#pragma unroll
        for (int t = 0; t < NT; ++t) done |= (odd >> t & 1u) && is_nan(v[t]) ? 1u << t : 0u;
        if (__all(done == (1u << NT) - 1u)) return;
      }
    }
}

// dim at most 32 ND.  UNIFORM: sixteen keys that begin at a multiple of 16 are in one page, and
// 15 slots are less than 2^31 bytes.
template <int QT, int KIND, int ND, bool VEC, bool UNIFORM>
__global__ __launch_bounds__(AT, ND == 8 || (QT == 0 && ND > 2) ? 1 : 2) void cache_attend_kernel(AttendArgs a) {
  using St = Step<QT, KIND, ND, VEC>;
  constexpr bool F32 = St::F32;
  constexpr int MT = KIND <= 2 ? KIND : 1;
  constexpr int TQ = KIND <= 2 ? 1 : QT == 1 ? 1 : QT == 2 ? 2 : 3;   // terms of a query
  constexpr int TP = QT == 0 ? 3 : 2;                                   // and of a weight
  constexpr int KN = St::KN, KS = St::KS, VN = St::VN, VC = St::VC, B = kCacheBytes<KIND>;
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

  const int64_t first_row = static_cast<int64_t>(b) * a.heads + head0;
  if (a.part && from >= to) {
    float* part = a.part + (static_cast<int64_t>(split) * a.batch * a.heads + first_row) * (a.dim + 2);
    for (int r = wave; r < live; r += AW)
      for (int d = lane; d < a.dim + 2; d += kWave) part[r * (a.dim + 2) + d] = d == a.dim ? -INFINITY : 0.0f;
    return;
  }

  Move16 q[KS][TQ];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int d = s * 4 * KN + KN * g;
    const int left = i16 < live ? a.dim - d : 0;
    using raw = typename Elem<QT>::raw;
    const raw* p = static_cast<const raw*>(a.q) + b * a.q_b + (head0 + i16) * a.q_h + d;
    float x[8] = {};
    if (a.q_whole) {
      if (left > 0) {
        constexpr int N = 16 / sizeof(raw);
#pragma unroll
        for (int j0 = 0; j0 < KN; j0 += N) {
          const Move16 v = *reinterpret_cast<const Move16*>(p + j0);
#pragma unroll
          for (int j = 0; j < N && j < KN; ++j)
            x[j0 + j] = Elem<QT>::get(QT == 0 ? v[j % 4] : (v[j / 2 % 4] >> (16 * (j % 2))) & 0xffffu);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < KN; ++j)
        if (j < left) x[j] = Elem<QT>::get(p[j]);
    }
    if (a.scale <= 0.0f) {   // (so that larger products are larger scores)
#pragma unroll
      for (int j = 0; j < KN; ++j) x[j] = a.scale < 0.0f ? -x[j] : 0.0f;
    }
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) q[s][0][j] = __float_as_uint(x[j]);
    } else {
      if constexpr (TQ > 1) split8_any<TQ>(x, q[s]);
      else split8<MT, TQ>(x, q[s]);
    }
  }

  // A lane's dims within a row, in bytes; dims that may not exist are the last ones
  // again (of keys in 16 and 32 bits they count as 0, like their part of q: a product of 0 and
  // infinity is none; codes of 8 bits have no infinities; results of them are not stored).  UNIFORM: with the
  // lane's row of the sixteen, or the first of its four.
  constexpr int kSure = ND == 2 ? 0 : ND == 8 ? 128 : 32 * (ND - 1);   // the smallest dim of this ND, less 1
  const int slot_k = static_cast<int>(a.k.slot) * B, slot_v = static_cast<int>(a.v.slot) * B;
  const uint32_t row_k = UNIFORM ? i16 * slot_k : 0, row_v = UNIFORM ? 4 * g * slot_v : 0;
  const uint32_t first_k = row_k + KN * g * B;
  uint32_t k_end[KS], v_at[VC];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int d = s * 4 * KN + KN * g;
    k_end[s] = row_k + static_cast<uint32_t>((VEC ? min(d, a.dim - KN) : d) * B);
  }
  const auto k_at = [&](int s) {
    return 4 * KN * (s + 1) <= kSure ? first_k + static_cast<uint32_t>(4 * KN * B * s) : k_end[s];
  };
#pragma unroll
  for (int c = 0; c < VC; ++c) {
    const int d = c * 16 * VN + VN * i16;
    v_at[c] = row_v + static_cast<uint32_t>((VEC ? min(d, a.dim - VN) : d) * B);
  }
  const char* head_k = static_cast<const char*>(a.k.data) + h * a.k.head * B;
  const char* head_v = static_cast<const char*>(a.v.data) + h * a.v.head * B;
  const float* scale_k = KIND > 2 ? a.k.scale + h * a.k.scale_head : nullptr;
  const float* scale_v = KIND > 2 ? a.v.scale + h * a.v.scale_head : nullptr;

  // the pages of a step, looked up a step before its loads
  const int32_t* table = a.t.table ? a.t.table + static_cast<int64_t>(b) * a.t.width : nullptr;
  int32_t page_of[2] = {b, b};
  const auto look = [&](int64_t k0) {
    if (UNIFORM && table) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int64_t p = divide(static_cast<uint32_t>(min(k0 + 16 * u, a.room)), a.by);
        page_of[u] = p < a.t.width ? table[p] : -1;
      }
    }
  };
  const auto load = [&](St& st, int key0) {
    const char *pk = nullptr, *pv = nullptr;
    const float *sk = nullptr, *sv = nullptr;
    int last = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (UNIFORM) {
        // The second sixteen follow the first on its page, if that is there (one that is not is
        // read from slot 0, wherever in it the first sixteen would be).
        if (u == 1 && st.page[0] && last >= 31) {
          st.page[1] = true;
          pk += 16 * slot_k;
          pv += 16 * slot_v;
          sk += 16;
          sv += 16;
          last -= 16;
        } else {
          const int key = key0 + 16 * u;
          int page = page_of[u];
          int slot = key;
          if (table) slot = key - static_cast<int>(divide(static_cast<uint32_t>(key), a.by)) * a.t.size;
          else page = key < a.t.size ? b : -1;
          page = __builtin_amdgcn_readfirstlane(page);
          st.page[u] = page >= 0 && page < a.t.pages;
          if (!st.page[u]) page = slot = 0;
          pk = head_k + (page * a.k.page + slot * a.k.slot) * B;
          pv = head_v + (page * a.v.page + slot * a.v.slot) * B;
          sk = KIND > 2 ? scale_k + (page * a.k.scale_page + slot) : nullptr;
          sv = KIND > 2 ? scale_v + (page * a.v.scale_page + slot) : nullptr;
          last = a.t.size - 1 - slot;
        }
        if (last >= 15) {
#pragma unroll
          for (int s = 0; s < KS; ++s) st.k[u][s].load(pk + k_at(s), 0);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < VC; ++c) st.v[c][u][i].load(pv + i * slot_v + v_at[c], 0);
          if constexpr (KIND > 2) {
            const float4 fk = load_quad(sk + 4 * g), fv = load_quad(sv + 4 * g);
            st.ks[u][0] = fk.x, st.ks[u][1] = fk.y, st.ks[u][2] = fk.z, st.ks[u][3] = fk.w;
            st.vs[u][0] = fv.x, st.vs[u][1] = fv.y, st.vs[u][2] = fv.z, st.vs[u][3] = fv.w;
          }
        } else {   // (the end of a cache without a table: its last row stands for those past it)
          const uint32_t back = static_cast<uint32_t>((i16 - min(i16, last)) * slot_k);
#pragma unroll
          for (int s = 0; s < KS; ++s) st.k[u][s].load(pk + (k_at(s) - back), 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = min(4 * g + i, last);
#pragma unroll
            for (int c = 0; c < VC; ++c)
              st.v[c][u][i].load(pv + (v_at[c] + static_cast<uint32_t>((r - 4 * g) * slot_v)), 0);
            if constexpr (KIND > 2) {
              st.ks[u][i] = sk[r];
              st.vs[u][i] = sv[r];
            }
          }
        }
      } else {
        const auto find = [&](int key, int* slot) {
          int page;
          if (table) {
            const int p = static_cast<int>(divide(static_cast<uint32_t>(key), a.by));
            *slot = key - p * a.t.size;
            page = p < a.t.width ? table[p] : -1;
          } else {
            *slot = key;
            page = key < a.t.size ? b : -1;
          }
          return page >= 0 && page < a.t.pages && key < to ? page : -1;
        };
        int slot;
        int page = find(key0 + 16 * u + i16, &slot);
        if (page < 0) page = slot = 0;
        const char* pk = head_k + (page * a.k.page + slot * a.k.slot) * B;
#pragma unroll
        for (int s = 0; s < KS; ++s) st.k[u][s].load(pk + k_at(s), a.dim - (s * 4 * KN + KN * g));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          page = find(key0 + 16 * u + 4 * g + i, &slot);
          st.there[u][i] = page >= 0;
          if (page < 0) page = slot = 0;
          const char* pv = head_v + (page * a.v.page + slot * a.v.slot) * B;
#pragma unroll
          for (int c = 0; c < VC; ++c) st.v[c][u][i].load(pv + v_at[c], a.dim - (c * 16 * VN + VN * i16));
          if constexpr (KIND > 2) {
            st.ks[u][i] = scale_k[page * a.k.scale_page + slot];
            st.vs[u][i] = scale_v[page * a.v.scale_page + slot];
          }
        }
      }
    }
  };

  float m = -INFINITY, l = 0.0f;
  Acc out[VC][VN] = {};
  const float scale2 = (a.scale == 0.0f ? 1.0f : fabsf(a.scale)) * static_cast<float>(kLog2e);
  float* scores = a.weights ? a.weights + (first_row + i16) * a.room : nullptr;

  const auto use = [&](St& st, int key0) {
    Acc sc[2] = {};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        Move16 f;
        if constexpr (F32) {
          f = Move16{st.k[u][s].w[0], st.k[u][s].w[1], st.k[u][s].w[2], st.k[u][s].w[3]};
        } else {
          uint32_t hv[4];
          st.k[u][s].halves(hv);
          f = Move16{hv[0], hv[1], hv[2], hv[3]};
        }
        if (VEC && KIND <= 2 && 4 * KN * (s + 1) > kSure && s * 4 * KN + KN * g >= a.dim) f = Move16{0u, 0u, 0u, 0u};
#pragma unroll
        for (int t = 0; t < TQ; ++t) sc[u] = mma<MT>(f, q[s][t], sc[u]);
      }
    if constexpr (KIND > 2) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[u][i] *= st.ks[u][i];
    }
    // Keys that are not there count for nothing, whatever was read for them (and 0 of
    // that may be NaN).
    bool whole = key0 >= from && key0 + AK <= to;
    if constexpr (UNIFORM) {
      whole = whole && st.page[0] && st.page[1];
    } else {
      bool all = true;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) all = all && st.there[u][i];
      whole = whole && __all(all);
    }
    if (!whole) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = key0 + 16 * u + 4 * g + i;
          if (key >= from && key < to && (UNIFORM ? st.page[u] : st.there[u][i])) continue;
          sc[u][i] = -INFINITY;
          st.vs[u][i] = 0.0f;
#pragma unroll
          for (int c = 0; c < VC; ++c) st.v[c][u][i].clear();
        }
    }
    // (the running maximum is one of products, which `scale2` times are powers of two)
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, sc[u][i]);
    if (scores && i16 < live) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (key0 + 16 * u + 4 * g + i < to) scores[key0 + 16 * u + 4 * g + i] = sc[u][i] * scale2;
    }
    if (__any(most > m)) {
      const float now = across_rows(fmaxf(m, most), [](float x, float y) { return fmaxf(x, y); });
      const float shrink = now == -INFINITY ? 1.0f : exp2_fast((m - now) * scale2);
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
    const float ref = m == -INFINITY ? 0.0f : m;
    float p[8];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (a difference first: what is far from zero is near the maximum)
        const float x = exp2_fast(fmaf(sc[u][i] - ref, scale2, kUp));
        l += x;
        p[4 * u + i] = KIND > 2 ? x * st.vs[u][i] : x;
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
              out[c][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[4 * u + i], __uint_as_float(st.v[c][u][i].w[e]),
                                                               out[c][e], 0, 0, 0);
    } else {
      Move16 w[TP];
      split8<MT, TP>(p, w);
#pragma unroll
      for (int c = 0; c < VC; ++c) {
        uint32_t hv[8][VN / 2];
#pragma unroll
        for (int j = 0; j < 8; ++j) st.v[c][j / 4][j % 4].halves(hv[j]);
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
  };

  // a step's loads go out before the step before it is used
  constexpr int stride = AK * AW;
  // (a step's registers are too many to have two of the widest rows)
  constexpr bool two = QT == 0 ? ND <= 2 : ND <= 4;
  int64_t k0 = base + AK * wave;
  if constexpr (two) {
    St even, odd;
    if (k0 < to) {
      look(k0);
      load(even, static_cast<int>(k0));
      look(k0 + stride);
    }
    while (k0 < to) {
      if (k0 + stride < to) {
        load(odd, static_cast<int>(k0 + stride));
        look(k0 + 2 * stride);
      }
      use(even, static_cast<int>(k0));
      k0 += stride;
      if (k0 >= to) break;
      if (k0 + stride < to) {
        load(even, static_cast<int>(k0 + stride));
        look(k0 + 2 * stride);
      }
      use(odd, static_cast<int>(k0));
      k0 += stride;
    }
  } else {
    St st;
    if (k0 < to) look(k0);
    for (; k0 < to; k0 += stride) {
      load(st, static_cast<int>(k0));
      look(k0 + stride);
      use(st, static_cast<int>(k0));
    }
  }

  // the waves' parts, joined
  l = across_rows(l, [](float x, float y) { return x + y; });
  if (g == 0) {
    parts[wave][i16][ND * 32] = m * scale2;   // (in powers of two; scale2 is above 0)
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
  if constexpr (KIND == 1 || KIND == 2) {
    float none = 0.0f;   // NaN where a sum is not a number
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
      for (int e = 0; e < VN; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) none = 4 * g + i < live ? fmaf(out[c][e][i], 0.0f, none) : none;
    if (__any(none != 0.0f)) {
      wave_lds_sync();
      infinite_values<QT, KIND, ND>(a, parts[wave], kUp, scale2, b, h, head0, live, base + AK * wave, from, to);
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
    const int64_t row = first_row + r;
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

// The parts of a row (b, head) joined: their factors e^(m - top) in LDS, then a wave to every
// fourth part, its lanes to the dims.
constexpr int JT = 256;
template <int QT>
__global__ __launch_bounds__(JT) void cache_attend_join_kernel(AttendArgs a, float up) {
  extern __shared__ float lds[];
  float* factor = lds;                                  // [splits]
  float* sums = lds + a.splits;                         // [4][dim]
  __shared__ float shared[2][JT / kWave];
  const int64_t row = blockIdx.x, rows = static_cast<int64_t>(a.batch) * a.heads;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t step = rows * (a.dim + 2);
  const float* part = a.part + row * (a.dim + 2);
  float top = -INFINITY;
  for (int s = threadIdx.x; s < a.splits; s += JT) {
    factor[s] = part[s * step + a.dim];
    top = fmaxf(top, factor[s]);
  }
  top = wave_max(top, -INFINITY);
  if (lane == 0) shared[0][wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < JT / kWave; ++w) top = fmaxf(top, shared[0][w]);
  float sum = 0.0f;
  for (int s = threadIdx.x; s < a.splits; s += JT) {
    const float m = factor[s], f = m == -INFINITY ? 0.0f : exp2_fast(m - top);
    factor[s] = f;
    sum += f * part[s * step + a.dim + 1];   // (a part without keys is all zeros)
  }
  sum = wave_sum(sum);
  if (lane == 0) shared[1][wave] = sum;
  __syncthreads();
  sum = 0.0f;
#pragma unroll
  for (int w = 0; w < JT / kWave; ++w) sum += shared[1][w];
  for (int d = lane; d < a.dim; d += kWave) {
    float y = 0.0f;
#pragma unroll 8
    for (int s = wave; s < a.splits; s += JT / kWave) y = fmaf(factor[s], part[s * step + d], y);
    sums[wave * a.dim + d] = y;
  }
  __syncthreads();
  using raw = typename Elem<QT>::raw;
  for (int d = threadIdx.x; d < a.dim; d += JT) {
    float y = 0.0f;
#pragma unroll
    for (int w = 0; w < JT / kWave; ++w) y += sums[w * a.dim + d];
    static_cast<raw*>(a.out)[row * a.dim + d] = Elem<QT>::put(sum == 0.0f ? 0.0f : y / sum);
  }
  if (threadIdx.x == 0 && a.lse)
    a.lse[row] = sum == 0.0f ? -INFINITY : (top + __log2f(sum) - up) * static_cast<float>(1.0 / kLog2e);
}

// Scores in powers of two to weights, by the row's lse; 0 outside its keys.
__global__ __launch_bounds__(256) void cache_weights_kernel(AttendArgs a) {
  const int64_t pieces = (a.room + 255) / 256, all = static_cast<int64_t>(a.batch) * a.heads * pieces;
  for (int64_t at = blockIdx.x; at < all; at += gridDim.x) {
    const int64_t row = at / pieces, j = at % pieces * 256 + threadIdx.x;
    if (j >= a.room) continue;
    const int b = static_cast<int>(row / a.heads);
    const int64_t len = min(static_cast<int64_t>(max(a.lens[b], 0)), a.room);
    const int64_t start = a.window > 0 && len > a.window ? len - a.window : 0;
    const float lse = a.lse[row] * static_cast<float>(kLog2e);
    float w = 0.0f;
    if (j >= start && j < len && a.lse[row] != -INFINITY) w = exp2_fast(a.weights[row * a.room + j] - lse);
    a.weights[row * a.room + j] = w;
  }
}

}  // namespace

// ------------------------------------------------------------- launchers ---
// A workgroup's keys: as many workgroups as are on the chip twice over, of at least a step
// for each wave.  More of them begin and end more often: four contexts of 131072 take
// 335 us with 1024 workgroups, 346 with 2048, 361 with 4096, 382 with 8192.
void attend_plan(int64_t batch, int64_t heads, int64_t kv, int64_t room, int64_t window, int* splits,
                 int* chunk) {
  constexpr int64_t step = AK * AW;
  const int64_t rows = batch * kv * ((heads / kv + 15) / 16);
  const int64_t keys = window > 0 && window < room ? (window + AK < room ? window + AK : room) : room;
  int64_t each = (keys * rows + 1023) / 1024;
  // (no more than there are: the product is past 32 bits where rows and room are large)
  each = ((each < keys ? each : keys) + step - 1) / step * step;
  if (each < step) each = step;
  *chunk = static_cast<int>(each);
  *splits = static_cast<int>(keys < 1 ? 1 : (keys + each - 1) / each);
}

hipError_t launch_cache_attend(const AttendArgs& a, int dtype, int kind, bool vec, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.splits) * a.batch * a.kv * a.tiles));
  const int64_t bytes = kind == 0 ? 4 : kind <= 2 ? 2 : 1;
  const bool uniform = (!a.t.table || a.t.size % 16 == 0) && 16 * a.k.slot * bytes < (int64_t(1) << 31) - 65536 &&
                       16 * a.v.slot * bytes < (int64_t(1) << 31) - 65536;
  {
    ProfScope ps_("cache_attend", s);
    const auto launch = [&](auto qt, auto kd) {
      constexpr int QT = decltype(qt)::value, KIND = decltype(kd)::value;
      const auto go = [&](auto nd, auto uni) {
        hipLaunchKernelGGL((cache_attend_kernel<QT, KIND, decltype(nd)::value, true, decltype(uni)::value>), grid,
                           dim3(AT), 0, s, a);
      };
      const auto dims = [&](auto uni) {
        if (a.dim <= 64) go(std::integral_constant<int, 2>{}, uni);
        else if (a.dim <= 96) go(std::integral_constant<int, 3>{}, uni);
        else if (a.dim <= 128) go(std::integral_constant<int, 4>{}, uni);
        else go(std::integral_constant<int, 8>{}, uni);
      };
      if (!vec) hipLaunchKernelGGL((cache_attend_kernel<QT, KIND, 8, false, false>), grid, dim3(AT), 0, s, a);
      else if (uniform) dims(std::true_type{});
      else dims(std::false_type{});
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
    const size_t lds = sizeof(float) * (static_cast<size_t>(a.splits) + 4 * static_cast<size_t>(a.dim));
    if (dtype == 0) hipLaunchKernelGGL((cache_attend_join_kernel<0>), dim3(rows), dim3(JT), lds, s, a, up);
    else if (dtype == 1) hipLaunchKernelGGL((cache_attend_join_kernel<1>), dim3(rows), dim3(JT), lds, s, a, up);
    else hipLaunchKernelGGL((cache_attend_join_kernel<2>), dim3(rows), dim3(JT), lds, s, a, up);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.weights) {
    ProfScope ps_("cache_weights", s);
    const int64_t all = rows * ((a.room + 255) / 256);
    hipLaunchKernelGGL(cache_weights_kernel, dim3(static_cast<unsigned>(all < (1 << 20) ? all : (1 << 20))), dim3(256),
                       0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace lapsum
