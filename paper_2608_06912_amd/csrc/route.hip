// Routing of tokens to experts: per token the best `top_k` of E experts, their
// weights, and the gradient of the weights with respect to the logits.
//
// With x the token's logits, s = softmax(x) or sigma(x) = 1/(1 + e^-x) and c =
// s + bias what the selection compares (softmax without a bias: c = x, whose
// order is that of s):
//   groups     E/groups consecutive experts; a group's score is the sum of its
//              `group_top` largest c (softmax without a bias: of e^{x - max},
//              or x itself for one), and the best `topk_groups` groups stay
//   experts    the top_k largest c in them, equal values by the lowest index
//   weights    scale s_j, or scale s_j / sum of the chosen s
// An expert whose logit or c is NaN or -inf is never chosen; a place that no
// expert takes has index -1 and weight 0.
//
// Backward, for g = dL/dw and the indices held fixed:
//   sigmoid             dx_j = scale g_j s_j (1 - s_j)
//   sigmoid, renorm     dx_j = scale s_j (1 - s_j) (g_j - sum g_i s_i / S) / S,
//                       S = sum of the chosen s
//   softmax             dx_e = scale s_e ([e chosen] g_e - sum_j g_j s_j), all e
//   softmax, renorm     dx_j = scale q_j (g_j - sum g_i q_i), q = softmax over
//                       the chosen
//
// A team of LT lanes takes a token: 16 lanes (four tokens a wave) for up to 512
// experts and 8 chosen, else the wave.  A lane holds every LT-th dword of the
// row, so the best experts of a group are spread over the team.  The k-th
// largest of the lanes' maxima bounds the k-th largest c from below; what is
// not below it, little more than k values, goes one to a lane and is ranked by
// counting.  A row with more such values than lanes gets a higher bound, and
// where equal values do not allow one it is chosen one maximum at a time.
//
// Sigmoid scores are compared in float32, so the choice depends on their
// rounding: 1/(1 + e^-x) by expf and a correctly rounded division.  Two exact
// scores per logit would be most of the work, so all of a row gets an
// approximate one first (the hardware's 2^x and 1/x, within kNear), which
// settles what cannot be chosen; the candidates, and rows whose groups are
// closer than that, get the exact one.
//
// Bound: vector issue, about half, and the waits between its steps.  65536
// tokens of 256 bfloat16 logits in eight groups, 8 chosen: 30 us, 17 without
// groups; with counts 32 and 4.7 for their kernel (the bytes take 7.4 at the rate
// of a copy); 673 vector instructions for four tokens, 18 us.  With comparisons
// counted as such, not as the sign of a difference, and the groups' scores passed
// through LDS, it took 785 instructions and 3 us more; with the exact score of
// every logit as well twice the time.  16 tokens: 4.3 us, one wave's chain of
// steps.  Backward: 32768 tokens of 128 float32 logits, dense, 10.8 us (bytes 6.6).
#include "select_common.hpp"

namespace lapsum {

namespace {
constexpr int BT = 256;

// Elements of a dword: what a lane holds of a row at a time.
template <int DT>
constexpr int kPer = DT == 0 ? 1 : 2;

__device__ __forceinline__ float sigmoid_f32(float x) { return 1.0f / (1.0f + expf(-x)); }

// An approximate sigmoid, 1 / (1 + 2^(-x log2 e)) by the hardware's functions,
// is within kNear of the exact one: the product's, the exponential's, the sum's
// and the reciprocal's rounding, each weighted by s (1 - s) or s, are below
// 3e-7 (over all float32, 1.8e-7 at most).  Comparisons of c leave twice that
// much, and four roundings of c itself.  A group's score of two terms is off by
// twice kNear and, its terms and their sum each rounded on both sides, 2^-22 of
// |t1| + |t2|, which can be far above the score where the biases' signs differ; the
// rest of 4e-7 is for the roundings of the comparison.
constexpr float kNear = 1e-6f;
__device__ __forceinline__ float near_margin(float c) { return 2.0f * kNear + 5e-7f * fabsf(c); }
__device__ __forceinline__ float group_margin(float size) { return 2.0f * kNear + 4e-7f * fminf(size, FLT_MAX); }

// A logit as it counts: NaN is masked, +inf the largest float.
__device__ __forceinline__ float clean(float x) { return x > -INFINITY ? fminf(x, FLT_MAX) : -INFINITY; }

// The team's row, a lane every LT-th dword; what lies past the row is of its
// end, no masked value.
template <int DT, int IT, int LT>
__device__ __forceinline__ void load_row(const typename Elem<DT>::raw* __restrict__ row, int E, int l,
                                         float (&x)[IT][kPer<DT>]) {
  constexpr int V = kPer<DT>;
  uint32_t u[IT];
  if (E == IT * LT * V) {   // (the whole of every lane: one address, fixed offsets)
    const char* p = reinterpret_cast<const char*>(row) + l * 4;
#pragma unroll
    for (int i = 0; i < IT; ++i) __builtin_memcpy(&u[i], p + i * LT * 4, 4);
  } else {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int e = (i * LT + l) * V;
      // an odd row's last element is the upper half of the last whole dword
      const int at = e + V <= E ? e : E - V;
      if (V == 2 && E == 1) u[i] = row[0];
      else __builtin_memcpy(&u[i], row + at, 4);
      if (V == 2 && e + 1 == E && E > 1) u[i] >>= 16;
    }
  }
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    if constexpr (V == 2) {
      x[i][0] = Elem<DT>::get(u[i] & 0xffffu);
      x[i][1] = Elem<DT>::get(u[i] >> 16);
    } else {
      x[i][0] = Elem<DT>::get(u[i]);
    }
  }
}
// f(value, expert) for all of a lane's places, past the row too.
template <int IT, int LT, int V, class F>
__device__ __forceinline__ void each_item(float (&x)[IT][V], int l, F&& f) {
#pragma unroll
  for (int i = 0; i < IT; ++i)
#pragma unroll
    for (int v = 0; v < V; ++v) f(x[i][v], (i * LT + l) * V + v);
}

// max and sum of e^{x - max} over the team's row; a row without a finite logit
// has max 0 and sum 0.  NaN and +inf, which make the sum NaN, are cleaned from
// x first where there are any.  compared: a selection reads the sum, which is then
// added up in float64 and rounded once, so that it is the same for every
// arrangement of the row over lanes.
template <int IT, int LT, int V>
__device__ __forceinline__ void softmax_stats(float (&x)[IT][V], int l, float* m_out, float* sum_out,
                                              bool compared = false) {
  for (;;) {
    float m = -INFINITY;
    each_item<IT, LT>(x, l, [&](float& y, int) { m = fmaxf(m, y); });
    m = team_max<LT>(m);
    m = m == -INFINITY ? 0.0f : m;
    float s;
    if (compared) {
      double t = 0.0;
      float most = m;
      asm volatile("" : "+v"(most));   // (exponentials formed for both ways would take registers)
      each_item<IT, LT>(x, l, [&](float& y, int) { t += static_cast<double>(expf(y - most)); });
      s = static_cast<float>(team_sum<LT>(t));
    } else {
      s = 0.0f;
      each_item<IT, LT>(x, l, [&](float& y, int) { s += expf(y - m); });
      s = team_sum<LT>(s);
    }
    if (!__any(s != s)) {
      *m_out = m;
      *sum_out = s;
      return;
    }
    each_item<IT, LT>(x, l, [&](float& y, int) { y = clean(y); });
  }
}

// LDS of a team.
template <int LT>
struct RouteTeam {
  int at[LT];
  float gscore[LT];   // (no more groups than lanes)
};

// Floats from one token's c in LDS to the next (whole 16-byte words).
template <int DT, int IT, int LT>
constexpr int kRow = IT * LT * kPer<DT> + 4;

// Whether the group that this lane takes part in (2^sub lanes to a group)
// stays, on the lane that speaks for it, the first of them, from the row's
// values in LDS; *score_out: the group's score, *size_out: its terms' sizes added up.
template <int LT>
__device__ __forceinline__ bool group_kept(const RouteArgs& a, const float* crow, float* gscore, int l,
                                           float* score_out, float* size_out) {
  const int sub = 1 << a.sub, size = a.group_size;
  const int g = l >> a.sub, q = l & (sub - 1);
  float t1 = -INFINITY, t2 = -INFINITY;
  const auto take = [&](float y) {   // (no NaN comes here)
    t2 = __builtin_amdgcn_fmed3f(t1, t2, y);
    t1 = fmaxf(t1, y);
  };
  if (g < a.groups) {
    if (a.wide) {   // whole 16-byte words of a group for each lane
      const int part = size >> a.sub;
      const float4* from = reinterpret_cast<const float4*>(crow + g * size + q * part);
      for (int j = 0; j < part / 4; ++j) {
        const float4 y = from[j];
        take(y.x);
        take(y.y);
        take(y.z);
        take(y.w);
      }
    } else {
      for (int j = q; j < size; j += sub) take(crow[g * size + j]);
    }
  }
  const auto join = [&](float o1, float o2) {
    t2 = __builtin_amdgcn_fmed3f(t1, o1, max_f32(t2, o2));
    t1 = max_f32(t1, o1);
  };
  if constexpr (LT == 16) {   // pairs, fours, and mirrors of eight and sixteen
    if (sub > 1) join(row_move<0xb1>(t1), row_move<0xb1>(t2));
    if (sub > 2) join(row_move<0x4e>(t1), row_move<0x4e>(t2));
    if (sub > 4) join(row_move<0x141>(t1), row_move<0x141>(t2));
    if (sub > 8) join(row_move<0x140>(t1), row_move<0x140>(t2));
  } else {
    for (int d = 1; d < sub; d *= 2) join(__shfl_xor(t1, d, LT), __shfl_xor(t2, d, LT));
  }
  // (an expert that cannot be chosen adds nothing)
  const bool two = a.group_top > 1 && t2 > -INFINITY;
  const float score = two ? t1 + t2 : t1;
  const bool speaks = q == 0 && g < a.groups;
  *score_out = score;
  *size_out = fabsf(t1) + (two ? fabsf(t2) : 0.0f);
  if constexpr (LT == 16) {
    // by score alone; where equal ones do not leave topk_groups, by index too
    const float s = speaks ? __builtin_amdgcn_fmed3f(score, -FLT_MAX, FLT_MAX) : -FLT_MAX;
    const int above = row_count_above(s);   // (of every lane: the others' values come from it)
    const bool stays = speaks && above < a.topk_groups;
    const uint32_t row = static_cast<uint32_t>(__ballot(stays) >> (threadIdx.x & 48)) & 0xffffu;
    if (!__any(__popc(row) != a.topk_groups)) return stays;
  }
  if (speaks) gscore[g] = score;
  wave_lds_sync();
  int before = 0;
  for (int j = 0; j < a.groups; ++j) {
    const float o = gscore[j];
    before += o > score || (o == score && j < g) ? 1 : 0;
  }
  wave_lds_sync();
  return speaks && before < a.topk_groups;
}
// The bit of expert e's group in the ballot of the lanes that speak for the
// team's groups.
template <int LT>
using lanes_t = std::conditional_t<LT == 16, uint32_t, uint64_t>;
template <int LT>
__device__ __forceinline__ bool group_bit(const RouteArgs& a, lanes_t<LT> stay, int e) {
  const int lane = static_cast<int>((static_cast<uint32_t>(e) * a.group_inv) >> 21) << a.sub;
  return (stay >> (lane & (sizeof(stay) * 8 - 1))) & 1u;
}

// Waves per SIMD that the registers of a lane's values leave room for.
constexpr int route_waves(int values) { return values <= 8 ? 6 : (values <= 16 ? 5 : (values <= 32 ? 3 : 2)); }
}  // namespace

// SIG: sigmoid scores, else softmax.
template <int DT, int IT, int LT, bool SIG>
__global__ __launch_bounds__(BT, route_waves(IT * kPer<DT>)) void route_forward_kernel(RouteArgs a) {
  constexpr int R = BT / LT;   // tokens a workgroup takes at a time
  constexpr int V = kPer<DT>;
  using raw = typename Elem<DT>::raw;
  using mask_t = std::conditional_t<(IT * V > 32), uint64_t, uint32_t>;
  __shared__ RouteTeam<LT> teams[R];
  extern __shared__ __align__(16) float dyn[];   // [R][kRow] c, [kRow] bias, [E] counts
  const int r = threadIdx.x / LT;
  const int k = a.top_k;
  RouteTeam<LT>& tm = teams[r];
  float* crow = dyn + r * kRow<DT, IT, LT>;
  float* bias = dyn + R * kRow<DT, IT, LT>;
  int* hist = reinterpret_cast<int*>(bias + kRow<DT, IT, LT>);
  // (past the row -inf, which masks what is there; NaN forbids as -inf does)
  for (int e = threadIdx.x; e < IT * LT * V; e += BT)
    bias[e] = e >= a.experts ? -INFINITY : (a.bias ? fmaxf(a.bias[e], -INFINITY) : 0.0f);
  if (a.counts)
    for (int e = threadIdx.x; e < a.experts; e += BT) hist[e] = 0;
  __syncthreads();
  const bool raw_order = !SIG && !a.bias;
  const bool exps = raw_order && a.group_top > 1;   // a group's score is a sum of e^{x - max}
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * R; base < a.tokens;
       base += static_cast<int64_t>(gridDim.x) * R) {
    // what follows from the lane and E is formed anew for each token: kept over the
    // loop it would take the registers that the values need
    int l = threadIdx.x % LT, E = a.experts;
    asm volatile("" : "+v"(l), "+s"(E));
    const bool on = base + r < a.tokens;
    const int64_t token = on ? base + r : a.tokens - 1;
    const raw* row = static_cast<const raw*>(a.logits) + token * a.stride;
    float c[IT][V];
    float m = 0.0f, sum = 1.0f;
    // the exact score of a clean logit, and what the selection compares
    const auto score_of = [&](float x) -> float {
      if constexpr (SIG) return sigmoid_f32(x);
      else return raw_order ? x : expf(x - m) / sum;
    };
    const auto value_of = [&](float x, float s, float b) -> float {
      return x > -INFINITY ? fmaxf(s + b, -INFINITY) : -INFINITY;
    };
    load_row<DT, IT, LT>(row, E, l, c);
    if constexpr (SIG) {
      float dmax = 0.0f;
      each_item<IT, LT>(c, l, [&](float& y, int) {
        const float d = 1.0f + exp2_fast(y * -static_cast<float>(kLog2e));
        dmax = fmaxf(dmax, d);
        y = __builtin_amdgcn_rcpf(d);
      });
      // a score of 0 may be that of a masked logit: which it is is seen again
      if (__any(dmax == INFINITY)) {
        float x[IT][V];
        load_row<DT, IT, LT>(row, E, l, x);
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int v = 0; v < V; ++v) c[i][v] = x[i][v] > -INFINITY ? c[i][v] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v)   // (NaN, of a logit or of -inf + inf: -inf)
          c[i][v] = fmaxf(c[i][v] + bias[(i * LT + l) * V + v], -INFINITY);
    } else {
      each_item<IT, LT>(c, l, [&](float& y, int e) { y = e < E ? clean(y) : -INFINITY; });
      if (!a.renorm || a.bias || (a.groups > 1 && exps)) softmax_stats<IT, LT>(c, l, &m, &sum, !raw_order);
      if (!raw_order) {
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int v = 0; v < V; ++v) c[i][v] = value_of(c[i][v], score_of(c[i][v]), bias[(i * LT + l) * V + v]);
      }
    }
    bool slow = false;   // of a team of this wave
    // the expert of item q, part v: l's dwords, or `first` on
    bool packed = false;
    int first = 0;
    if (a.groups > 1) {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        float y[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
          y[v] = !SIG && exps && c[i][v] > -INFINITY ? expf(c[i][v] - m) : c[i][v];
        __builtin_memcpy(crow + (i * LT + l) * V, y, sizeof(y));
      }
      wave_lds_sync();
      float score, size;
      const bool kept = group_kept<LT>(a, crow, tm.gscore, l, &score, &size);
      const uint64_t all = __ballot(kept);
      if constexpr (SIG) {
        // approximate scores settle it where every group that stays is above every
        // one that does not by more than the two may be off
        const bool speaks = (l & ((1 << a.sub) - 1)) == 0 && l >> a.sub < a.groups;
        const float off = group_margin(size);
        const float in = team_min<LT>(kept ? score - off : INFINITY);
        const float out = team_max<LT>(speaks && !kept ? score + off : -INFINITY);
        slow = __any(!(in > out));
      }
      const lanes_t<LT> stay =
          static_cast<lanes_t<LT>>(LT == 16 ? (all >> (threadIdx.x & 48)) & 0xffffull : all);
      packed = a.packed != 0;
      if (packed) {
        // the groups that stay, over all of the team: 2^lanes lanes to a group,
        // `part` consecutive experts to a lane
        const int part = a.group_size >> a.lanes;
        lanes_t<LT> rest = stay;   // the speaking lanes, in the order of their groups
        for (int j = l >> a.lanes; j > 0; --j) rest &= rest - 1;
        const int lane = LT == 16 ? __ffs(static_cast<uint32_t>(rest))
                                  : __ffsll(static_cast<unsigned long long>(rest));
        const int g = rest ? (lane - 1) >> a.sub : 0;
        first = g * a.group_size + (l & ((1 << a.lanes) - 1)) * part;
#pragma unroll
        for (int q = 0; q < IT * V; q += 4) {
          float4 y = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
          if (q < part) y = *reinterpret_cast<const float4*>(crow + first + q);
          const float w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int v = 0; v < 4 && q + v < IT * V; ++v) c[(q + v) / V][(q + v) % V] = w[v];
        }
      } else {
        each_item<IT, LT>(c, l, [&](float& y, int e) { y = group_bit<LT>(a, stay, e) ? y : -INFINITY; });
      }
    }

    // the candidates: nothing below the k-th largest of the lanes' maxima
    float best = -INFINITY;
    each_item<IT, LT>(c, l, [&](float& y, int) { best = fmaxf(best, y); });
    float bound;
    if constexpr (LT == 16) {
      const float b = __builtin_amdgcn_fmed3f(best, -FLT_MAX, FLT_MAX);
      bound = team_min<LT>(row_count_above(b) < k ? b : INFINITY);
    } else {
      const uint32_t key = asc_key(best);
      uint32_t K = 0u;
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t cand = K | (1u << bit);
        if (__popcll(__ballot(key >= cand)) >= k) K = cand;
      }
      bound = key_value(K);
    }
    // where that leaves more candidates than lanes, a higher bound that still
    // leaves k: halving towards the maximum (equal values may not allow one)
    mask_t mine;
    int have, incl, count;
    float top = 0.0f;
    for (int turn = 0;; ++turn) {
      float b = bound;
      if (SIG && fabsf(b) <= FLT_MAX) b -= near_margin(b);
      b = minus(__builtin_amdgcn_fmed3f(b, -FLT_MAX, FLT_MAX));
      // from the last item, in the highest bit, to the first; a bit is clear where
      // c - b is not below zero
      uint32_t below[2] = {~0u, ~0u};
#pragma unroll
      for (int q = IT * V - 1; q >= 0; --q) below[q / 32] = push_sign(below[q / 32], c[q / V][q % V] + b);
      mine = static_cast<mask_t>(~((static_cast<uint64_t>(below[1]) << 32) | below[0]));
      have = IT * V > 32 ? __popcll(mine) : __popc(static_cast<uint32_t>(mine));
      incl = team_incl_add<LT>(have);
      count = team_max<LT>(incl);
      if (turn == 8 || !__any(count > LT)) break;
      if (turn == 0) top = fminf(team_max<LT>(best), FLT_MAX);
      const float mid = 0.5f * fmaxf(bound, -FLT_MAX) + 0.5f * top;
      int n = 0;
      each_item<IT, LT>(c, l, [&](float& y, int) { n += y >= mid ? 1 : 0; });
      n = team_sum<LT>(n);
      bound = n >= k ? mid : bound;
      top = n >= k ? top : mid;
    }
    int at = INT32_MAX;
    slow = slow || __any(count > LT);
    if (!slow) {
      int pos = incl - have;
      while (__any(mine != 0)) {
        if (mine != 0) {
          const int q = IT * V > 32 ? __ffsll(static_cast<unsigned long long>(mine)) - 1
                                    : __ffs(static_cast<uint32_t>(mine)) - 1;
          mine &= mine - 1;
          tm.at[pos] = packed ? first + q : (q / V * LT + l) * V + q % V;
          ++pos;
        }
      }
      wave_lds_sync();
      if (l < count) at = tm.at[l];
    } else {
      // exact values of the whole row in LDS, and one maximum at a time: lane j
      // gets the j-th
      wave_lds_sync();
#pragma unroll 1
      for (int e = l; e < E; e += LT) {
        const float x = clean(Elem<DT>::get(row[e]));
        const float y = value_of(x, score_of(x), bias[e]);
        crow[e] = exps && y > -INFINITY ? expf(y - m) : y;
      }
      wave_lds_sync();
      lanes_t<LT> stay = 0;
      if (a.groups > 1) {
        float score, size;
        const uint64_t all = __ballot(group_kept<LT>(a, crow, tm.gscore, l, &score, &size));
        stay = static_cast<lanes_t<LT>>(LT == 16 ? all >> (threadIdx.x & 48) : all);
      }
#pragma unroll 1
      for (int e = l; e < E; e += LT) {
        if (exps) crow[e] = clean(Elem<DT>::get(row[e]));
        if (a.groups > 1 && !group_bit<LT>(a, stay, e)) crow[e] = -INFINITY;
      }
      count = 0;
      for (int j = 0; j < k; ++j) {
        float v1 = -INFINITY;
        int a1 = INT32_MAX;
#pragma unroll 1
        for (int e = l; e < E; e += LT)
          if (crow[e] > v1) {
            v1 = crow[e];
            a1 = e;
          }
        const float most = team_max<LT>(v1);
        const int got = team_min<LT>(v1 == most && most > -INFINITY ? a1 : INT32_MAX);
        if (got != INT32_MAX) {
          if (a1 == got) crow[got] = -INFINITY;   // (its own lane's entry)
          if (l == j) at = got;
          ++count;
        }
      }
    }

    // a candidate to a lane: its exact c, its rank, its weight
    const bool is = at != INT32_MAX;
    const float x = clean(Elem<DT>::get(row[is ? at : 0]));
    const float s = score_of(x);
    const float val = is ? value_of(x, s, bias[at]) : -INFINITY;
    int rank = 0;
    const auto rank_by = [&](auto key) {
      rank = 0;
      if constexpr (LT == 16 && std::is_same_v<decltype(key), float>) {
        rank = row_count_above(__builtin_amdgcn_fmed3f(key, -FLT_MAX, FLT_MAX));
      } else if constexpr (LT == 16) {
        each_rotation([&](auto ctl) { rank += row_move<decltype(ctl)::value>(key) > key ? 1 : 0; });
      } else {
        for (int j = 0; j < count; ++j) rank += readlane_as(key, j) > key ? 1 : 0;
      }
    };
    // by value alone; where two are equal (their ranks are then fewer than the
    // candidates), by value and index
    rank_by(val);
    uint32_t lo = is && rank < 32 ? 1u << rank : 0u, hi = is && rank >= 32 ? 1u << (rank - 32) : 0u;
    lo = team_reduce<LT>(lo, [](uint32_t p, uint32_t q) { return p | q; });
    if constexpr (LT == 64) hi = team_reduce<LT>(hi, [](uint32_t p, uint32_t q) { return p | q; });
    if (__any(__popc(lo) + (LT == 64 ? __popc(hi) : 0) != count))
      rank_by((static_cast<uint64_t>(asc_key(val)) << 32) | static_cast<uint32_t>(~at));
    const bool chosen = is && rank < k;
    float w;
    if (SIG || !a.renorm) {
      w = chosen ? (raw_order ? expf(x - m) / sum : s) : 0.0f;
    } else {
      const float most = team_max<LT>(chosen ? x : -INFINITY);
      w = chosen ? expf(x - most) : 0.0f;
    }
    if (a.renorm) {
      const float total = team_sum<LT>(w);
      w = total > 0.0f ? w / total : 0.0f;
    }
    if (on) {
      const int64_t o = token * k;
      if (chosen) {
        a.weights[o + rank] = a.scale * w;
        a.indices[o + rank] = at;
        if (a.counts) atomicAdd(&hist[at], 1);
      }
      if (l >= count && l < k) {   // places that no expert is left for
        a.weights[o + l] = 0.0f;
        a.indices[o + l] = -1;
      }
    }
    wave_lds_sync();   // what the team wrote has been read
  }
  if (a.counts) {
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += BT)
      a.counts[static_cast<int64_t>(blockIdx.x) * a.experts + e] = hist[e];
  }
}

// counts[e] = sum of the workgroups' counts: eight experts a workgroup.  (Atomics
// on the counts themselves would need them cleared first, a launch as this is
// one.)
__global__ __launch_bounds__(1024) void route_counts_kernel(const int* __restrict__ parts, int blocks,
                                                            int E, int* __restrict__ counts) {
  __shared__ int sums[16][8];
  const int e = blockIdx.x * 8 + threadIdx.x % 8;
  int s = 0;
  if (e < E) {
#pragma unroll 4
    for (int b = threadIdx.x / 8; b < blocks; b += 128) s += parts[static_cast<int64_t>(b) * E + e];
  }
#pragma unroll
  for (int d = 8; d < kWave; d *= 2) s += __shfl_xor(s, d);
  if (lane_id() < 8) sums[threadIdx.x / kWave][lane_id()] = s;
  __syncthreads();
  if (threadIdx.x < 8 && e < E) {
    int t = 0;
    for (int q = 0; q < 16; ++q) t += sums[q][threadIdx.x];
    counts[e] = t;
  }
}

// The gradient of a token's logits, composed in LDS: the chosen experts'
// entries, zero (or the softmax's common term) elsewhere.
template <int DT, int IT, int LT>
__global__ __launch_bounds__(BT) void route_backward_kernel(RouteGradArgs a) {
  constexpr int R = BT / LT;
  constexpr int V = kPer<DT>;
  using raw = typename Elem<DT>::raw;
  extern __shared__ __align__(16) float dyn[];   // [R][kRow] entries of the chosen
  const int l = threadIdx.x % LT;
  const int r = threadIdx.x / LT;
  const int E = a.experts, k = a.top_k;
  float* grow = dyn + r * kRow<DT, IT, LT>;
  const bool softmax = a.score == 0;
  const bool dense = softmax && !a.renorm;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * R; base < a.tokens;
       base += static_cast<int64_t>(gridDim.x) * R) {
    const bool on = base + r < a.tokens;
    const int64_t token = on ? base + r : a.tokens - 1;
    const raw* row = static_cast<const raw*>(a.logits) + token * a.stride;
    float p[IT][V], m = 0.0f, sum = 1.0f, common = 0.0f, entry;
    if (dense) load_row<DT, IT, LT>(row, E, l, p);
    int at = l < k ? a.indices[token * k + l] : -1;
    if (at < 0 || at >= E) at = -1;
    const float g = at >= 0 ? a.grad[token * k + l] * a.scale : 0.0f;
    const float x = clean(Elem<DT>::get(row[at >= 0 ? at : 0]));
    const float none[V] = {};
#pragma unroll
    for (int i = 0; i < IT; ++i) __builtin_memcpy(grow + (i * LT + l) * V, none, sizeof(none));
    wave_lds_sync();
    if (dense) {
      each_item<IT, LT>(p, l, [&](float& y, int e) { y = e < E ? y : -INFINITY; });
      softmax_stats<IT, LT>(p, l, &m, &sum);
      const float q = at >= 0 && sum > 0.0f ? expf(x - m) / sum : 0.0f;
      common = team_sum<LT>(g * q);
      entry = g;
    } else if (softmax) {
      const float top = team_max<LT>(at >= 0 ? x : -INFINITY);
      float q = at >= 0 && top > -INFINITY ? expf(x - top) : 0.0f;
      const float total = team_sum<LT>(q);
      q = total > 0.0f ? q / total : 0.0f;
      entry = q * (g - team_sum<LT>(g * q));
    } else {
      // s (1 - s) = t / (1 + t)^2 with t = e^-|x|, which loses nothing near 1
      const float t = expf(-fabsf(x));
      const float d = at >= 0 ? t / ((1.0f + t) * (1.0f + t)) : 0.0f;
      if (a.renorm) {
        const float s = at >= 0 ? sigmoid_f32(x) : 0.0f;
        const float total = team_sum<LT>(s);
        const float mean = team_sum<LT>(g * s) / total;
        entry = total > 0.0f ? d * ((g - mean) / total) : 0.0f;
      } else {
        entry = d * g;
      }
    }
    if (at >= 0) grow[at] = entry;
    wave_lds_sync();
    raw* out = static_cast<raw*>(a.grad_logits) + token * E;
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int e = (i * LT + l) * V;
      float y[V];
      __builtin_memcpy(y, grow + e, sizeof(y));
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (dense) y[v] = sum > 0.0f ? expf(p[i][v] - m) * inv * (y[v] - common) : 0.0f;
      if constexpr (V == 2) {
        const uint32_t u = static_cast<uint32_t>(Elem<DT>::put(y[0])) |
                           (static_cast<uint32_t>(Elem<DT>::put(y[1])) << 16);
        if (on && e + 1 < E) __builtin_memcpy(out + e, &u, 4);
        else if (on && e < E) out[e] = static_cast<raw>(u);
      } else {
        if (on && e < E) out[e] = Elem<DT>::put(y[0]);
      }
    }
    wave_lds_sync();   // the row has been read
  }
}

// ------------------------------------------------------------- launchers ---
namespace {
// 16 lanes hold a token of up to 512 experts (32 values each); a team has to
// have a lane per chosen expert and per group, and to leave most rows fewer
// candidates than lanes.  65536 tokens of 256, sigmoid: 18 us with 8 chosen, and
// by the wave 51 with 9, 60 with 16; 32768 of 512: 15 with 8, 32 with 10.
bool narrow_team(int experts, int top_k, int groups) {
  return experts <= 512 && top_k <= 8 && groups <= 16;
}

// f(items, lanes of a team) for this many experts.
template <int DT, class F>
bool by_team(int experts, bool narrow, F&& f) {
  const int dwords = (experts + kPer<DT> - 1) / kPer<DT>;
  const int items = (dwords + (narrow ? 15 : 63)) / (narrow ? 16 : 64);
  const auto pick = [&](auto lt) {
    if (items <= 1) f(std::integral_constant<int, 1>{}, lt);
    else if (items <= 2) f(std::integral_constant<int, 2>{}, lt);
    else if (items <= 4) f(std::integral_constant<int, 4>{}, lt);
    else if (items <= 8) f(std::integral_constant<int, 8>{}, lt);
    else if (items <= 16) f(std::integral_constant<int, 16>{}, lt);
    else if constexpr (DT == 0) {
      if (items > 32) return false;
      f(std::integral_constant<int, 32>{}, lt);
    } else {
      return false;
    }
    return true;
  };
  return narrow ? pick(std::integral_constant<int, 16>{}) : pick(std::integral_constant<int, 64>{});
}

// Workgroups, each with the same number of turns: a turn each, so that a compute
// unit that is done takes the next (65536 tokens of 256 in eight groups: 30.2 us,
// 33.7 with those that fit the device together), but with counts, which each has
// to clear, add up and leave to the second kernel, no more than fit (38.4 in all,
// 39.6 with a turn each).
int64_t route_grid(int64_t tokens, bool narrow, bool counts) {
  const int64_t per = BT / (narrow ? 16 : 64);
  const int64_t want = (tokens + per - 1) / per;
  const int64_t most = counts ? kRouteBlocks : kRouteMost;
  const int64_t turns = (want + most - 1) / most;
  return (want + turns - 1) / turns;
}

template <int DT>
bool forward_type(const RouteArgs& a, bool narrow, int64_t grid, hipStream_t s) {
  return by_team<DT>(a.experts, narrow, [&](auto it, auto lt) {
    constexpr int IT = decltype(it)::value, LT = decltype(lt)::value;
    const unsigned lds = 4u * static_cast<unsigned>((BT / LT + 1) * kRow<DT, IT, LT> + (a.counts ? a.experts : 0));
    if (a.score)
      hipLaunchKernelGGL((route_forward_kernel<DT, IT, LT, true>), dim3(static_cast<unsigned>(grid)),
                         dim3(BT), lds, s, a);
    else
      hipLaunchKernelGGL((route_forward_kernel<DT, IT, LT, false>), dim3(static_cast<unsigned>(grid)),
                         dim3(BT), lds, s, a);
  });
}
template <int DT>
bool backward_type(const RouteGradArgs& a, bool narrow, int64_t grid, hipStream_t s) {
  return by_team<DT>(a.experts, narrow, [&](auto it, auto lt) {
    constexpr int IT = decltype(it)::value, LT = decltype(lt)::value;
    const unsigned lds = 4u * static_cast<unsigned>(BT / LT * kRow<DT, IT, LT>);
    hipLaunchKernelGGL((route_backward_kernel<DT, IT, LT>), dim3(static_cast<unsigned>(grid)),
                       dim3(BT), lds, s, a);
  });
}
}  // namespace

int64_t route_blocks(int64_t tokens, int experts, int top_k, int groups) {
  return route_grid(tokens, narrow_team(experts, top_k, groups), true);
}

hipError_t launch_route_forward(RouteArgs a, int dtype, int* parts, hipStream_t s) {
  const bool narrow = narrow_team(a.experts, a.top_k, a.groups);
  const int64_t grid = route_grid(a.tokens, narrow, a.counts != nullptr);
  int* const counts = a.counts;
  if (counts && grid > 1) a.counts = parts;
  const int team = narrow ? 16 : 64;
  a.sub = 0;
  while ((2 << a.sub) * a.groups <= team) ++a.sub;
  a.group_size = a.experts / a.groups;
  a.wide = a.experts % 4 == 0 && a.group_size % (4 << a.sub) == 0;
  // the experts of the chosen groups dealt out to the whole team, where that comes
  // out even and LDS holds what the selection compares
  a.lanes = 0;
  while ((2 << a.lanes) * a.topk_groups <= team) ++a.lanes;
  a.packed = a.groups > 1 && a.experts % 4 == 0 && (a.topk_groups << a.lanes) == team &&
             a.group_size % (4 << a.lanes) == 0 && !(a.score == 0 && !a.bias && a.group_top > 1);
  // e / size by a product: exact where e (size - 1) < 2^21, that is for the experts
  // of two groups or more and the places past them
  a.group_inv = static_cast<uint32_t>(((1u << 21) + a.group_size - 1) / a.group_size);
  bool done;
  { ProfScope ps_("route_forward", s);
  done = dtype == 0 ? forward_type<0>(a, narrow, grid, s)
       : dtype == 1 ? forward_type<1>(a, narrow, grid, s)
                    : forward_type<2>(a, narrow, grid, s); }
  if (!done) return hipErrorInvalidValue;
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !counts || grid <= 1) return e;
  { ProfScope ps_("route_counts", s);
  hipLaunchKernelGGL(route_counts_kernel, dim3(static_cast<unsigned>((a.experts + 7) / 8)),
                     dim3(1024), 0, s, parts, static_cast<int>(grid), a.experts, counts); }
  return hipGetLastError();
}

hipError_t launch_route_backward(const RouteGradArgs& a, int dtype, hipStream_t s) {
  const bool narrow = narrow_team(a.experts, a.top_k, 1);
  const int64_t grid = route_grid(a.tokens, narrow, false);
  bool done;
  { ProfScope ps_("route_backward", s);
  done = dtype == 0 ? backward_type<0>(a, narrow, grid, s)
       : dtype == 1 ? backward_type<1>(a, narrow, grid, s)
                    : backward_type<2>(a, narrow, grid, s); }
  if (!done) return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace lapsum
