// Routing of tokens to experts: per token the best `top_k` of E experts, their
// weights, and the gradient of the weights with respect to the logits.
//
// With x the token's logits, s = softmax(x) or sigma(x) = 1/(1 + e^-x) and
// c = s + bias what the selection compares (softmax without a bias: c = x,
// whose order is that of s):
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
// A team of LT lanes takes a token: 16 lanes (four tokens a wave) for up to
// 512 experts and 8 chosen, else the wave.  A lane holds every LT-th dword of the row, so
// the best experts of a group are spread over the team.  The k-th largest of the lanes'
// maxima bounds the k-th largest c from below; what is not below it, little
// more than k values, is ranked by counting.  The rare row with more such
// values than lanes is chosen one maximum at a time.
//
// Sigmoid scores are compared in float32, so the selection depends on their
// rounding: 1/(1 + e^-x) is formed by expf and a correctly rounded division.
#include "select_common.hpp"

namespace lapsum {

namespace {
constexpr int BT = 256;

__device__ __forceinline__ float sigmoid_f32(float x) { return 1.0f / (1.0f + expf(-x)); }

// Experts' logits of a lane's items: item i, part v is expert (i LT + l) V + v.
template <int DT, int V, int IT, int LT>
__device__ __forceinline__ void load_row(const typename Elem<DT>::raw* __restrict__ row, int E, int l,
                                         float (&x)[IT][V]) {
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int e = (i * LT + l) * V;
    const int at = e < E ? e : 0;   // (V divides E)
    if constexpr (V == 2) {
      uint32_t u;
      __builtin_memcpy(&u, row + at, 4);
      x[i][0] = Elem<DT>::get(u & 0xffffu);
      x[i][1] = Elem<DT>::get(u >> 16);
    } else {
      x[i][0] = Elem<DT>::get(row[at]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      // NaN counts as -inf (not chosen, no share), +inf as the largest float
      x[i][v] = x[i][v] == x[i][v] ? fminf(x[i][v], FLT_MAX) : -INFINITY;
      if (e >= E) x[i][v] = -INFINITY;
    }
  }
}

// max and sum of e^{x - max} over the team's row; a row without a finite
// logit has sum 0.
template <int V, int IT, int LT>
__device__ __forceinline__ void softmax_stats(const float (&x)[IT][V], float* m_out, float* sum_out) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < IT; ++i)
#pragma unroll
    for (int v = 0; v < V; ++v) m = fmaxf(m, x[i][v]);
  m = team_max<LT>(m);
  const float at = m == -INFINITY ? 0.0f : m;
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < IT; ++i)
#pragma unroll
    for (int v = 0; v < V; ++v) s += expf(x[i][v] - at);
  *m_out = at;
  *sum_out = team_sum<LT>(s);
}
}  // namespace

// LDS of a team.
template <int LT>
struct RouteTeam {
  float cand[LT];
  int at[LT];
  int sel[LT];
  float gscore[LT];
};

template <int DT, int V, int IT, int LT>
__global__ __launch_bounds__(BT) void route_forward_kernel(RouteArgs a) {
  constexpr int R = BT / LT;   // tokens a workgroup takes at a time
  using raw = typename Elem<DT>::raw;
  __shared__ RouteTeam<LT> teams[R];
  extern __shared__ float dyn[];   // [R][E] c (groups), then [E] counts
  const int l = threadIdx.x % LT;
  const int r = threadIdx.x / LT;
  const int E = a.experts, k = a.top_k;
  RouteTeam<LT>& tm = teams[r];
  float* crow = dyn + static_cast<int64_t>(r) * (E | 1);
  int* hist = reinterpret_cast<int*>(dyn + (a.groups > 1 ? R * (E | 1) : 0));
  if (a.counts) {
    for (int e = threadIdx.x; e < E; e += BT) hist[e] = 0;
    __syncthreads();
  }
  const bool softmax = a.score == 0;
  const bool raw_order = softmax && !a.bias;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * R; base < a.tokens;
       base += static_cast<int64_t>(gridDim.x) * R) {
    const bool on = base + r < a.tokens;
    const int64_t token = on ? base + r : a.tokens - 1;
    const raw* row = static_cast<const raw*>(a.logits) + token * a.stride;
    float c[IT][V];
    load_row<DT, V, IT, LT>(row, E, l, c);
    float m = 0.0f, sum = 1.0f;
    if (softmax && (!a.renorm || a.bias || (a.groups > 1 && a.group_top > 1)))
      softmax_stats<V, IT, LT>(c, &m, &sum);
    if (!raw_order) {
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int e = (i * LT + l) * V + v;
          const float x = c[i][v];
          const float s = softmax ? expf(x - m) / sum : sigmoid_f32(x);
          const float y = a.bias ? s + a.bias[e < E ? e : 0] : s;
          c[i][v] = x == -INFINITY ? -INFINITY : fmaxf(y, -INFINITY);   // (NaN: -inf)
        }
    }
    if (a.groups > 1) {
      // the groups' scores: `sub` lanes take a group, a lane every sub-th member
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int e = (i * LT + l) * V + v;
          const bool exps = raw_order && a.group_top > 1 && c[i][v] > -INFINITY;
          if (e < E) crow[e] = exps ? expf(c[i][v] - m) : c[i][v];
        }
      wave_lds_sync();
      const int sub = a.sub, size = a.group_size;
      const int g = l / sub;
      float t1 = -INFINITY, t2 = -INFINITY;
      if (g < a.groups)
        for (int j = l % sub; j < size; j += sub) {
          const float y = crow[g * size + j];
          t2 = fmaxf(t2, fminf(t1, y));
          t1 = fmaxf(t1, y);
        }
      for (int d = 1; d < sub; d *= 2) {
        const float o1 = __shfl_xor(t1, d, LT), o2 = __shfl_xor(t2, d, LT);
        t2 = fmaxf(fminf(t1, o1), fmaxf(t2, o2));
        t1 = fmaxf(t1, o1);
      }
      // (an expert that cannot be chosen adds nothing)
      const float score = a.group_top > 1 && t2 > -INFINITY ? t1 + t2 : t1;
      if (l % sub == 0 && g < a.groups) tm.gscore[g] = score;
      wave_lds_sync();
      int before = 0;
      for (int j = 0; j < a.groups; ++j) {
        const float o = tm.gscore[j];
        before += o > score || (o == score && j < g) ? 1 : 0;
      }
      wave_lds_sync();
      if (l % sub == 0 && g < a.groups) tm.gscore[g] = before < a.topk_groups ? 1.0f : 0.0f;
      wave_lds_sync();
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int e = (i * LT + l) * V + v;
          if (e < E && tm.gscore[e / size] == 0.0f) c[i][v] = -INFINITY;
        }
      wave_lds_sync();
    }

    // the candidates: nothing below the k-th largest of the lanes' maxima
    float best = -INFINITY;
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) best = fmaxf(best, c[i][v]);
    float bound;
    if constexpr (LT == 16) {
      int above = 0;
      each_rotation([&](auto ctl) {
        above += dpp_move<decltype(ctl)::value>(best, best) > best ? 1 : 0;
      });
      bound = team_min<LT>(above < k ? best : INFINITY);
    } else {
      const uint32_t key = asc_key(best);
      uint32_t K = 0u;
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t cand = K | (1u << bit);
        if (__popcll(__ballot(key >= cand)) >= k) K = cand;
      }
      bound = key_value(K);
    }
    bound = fmaxf(bound, -FLT_MAX);
    int mine = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) mine += c[i][v] >= bound ? 1 : 0;
    const int incl = team_incl_add<LT>(mine);
    const int count = team_max<LT>(incl);
    tm.sel[l] = -1;
    if (!__any(count > LT)) {
      int pos = incl - mine;
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (c[i][v] >= bound) {
            tm.cand[pos] = c[i][v];
            tm.at[pos] = (i * LT + l) * V + v;
            ++pos;
          }
      wave_lds_sync();
      const bool is = l < count;
      const float val = is ? tm.cand[l] : -INFINITY;
      const int at = is ? tm.at[l] : INT32_MAX;
      int rank = 0;
      if constexpr (LT == 16) {
        each_rotation([&](auto ctl) {
          const float ov = dpp_move<decltype(ctl)::value>(val, val);
          const int oa = dpp_move<decltype(ctl)::value>(at, at);
          rank += ov > val || (ov == val && oa < at) ? 1 : 0;
        });
      } else {
        for (int j = 0; j < count; ++j) {
          const float ov = readlane_as(val, j);
          const int oa = readlane_as(at, j);
          rank += ov > val || (ov == val && oa < at) ? 1 : 0;
        }
      }
      if (is && rank < k) tm.sel[rank] = at;
    } else {
      // one maximum at a time
      for (int j = 0; j < k; ++j) {
        float v1 = -INFINITY;
        int a1 = INT32_MAX;
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (c[i][v] > v1) {
              v1 = c[i][v];
              a1 = (i * LT + l) * V + v;
            }
        const float top = team_max<LT>(v1);
        const int at = team_min<LT>(v1 == top && top > -INFINITY ? a1 : INT32_MAX);
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int v = 0; v < V; ++v)
            if ((i * LT + l) * V + v == at) c[i][v] = -INFINITY;
        if (l == 0) tm.sel[j] = at == INT32_MAX ? -1 : at;
      }
    }
    wave_lds_sync();

    // lane j: the j-th chosen expert and its weight
    const int at = l < k ? tm.sel[l] : -1;
    float x = Elem<DT>::get(row[at >= 0 ? at : 0]);
    x = fminf(x, FLT_MAX);
    float w = 0.0f;
    if (!softmax) {
      w = at >= 0 ? sigmoid_f32(x) : 0.0f;
    } else if (!a.renorm) {
      w = at >= 0 ? expf(x - m) / sum : 0.0f;
    } else {
      const float top = team_max<LT>(at >= 0 ? x : -INFINITY);
      w = at >= 0 ? expf(x - top) : 0.0f;
    }
    if (a.renorm) {
      const float total = team_sum<LT>(w);
      w = total > 0.0f ? w / total : 0.0f;
    }
    if (on && l < k) {
      a.weights[token * k + l] = a.scale * w;
      a.indices[token * k + l] = at;
      if (a.counts && at >= 0) atomicAdd(&hist[at], 1);
    }
    wave_lds_sync();   // sel has been read
  }
  if (a.counts) {
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += BT)
      a.counts[static_cast<int64_t>(blockIdx.x) * E + e] = hist[e];
  }
}

// counts[e] = sum of the workgroups' counts: 32 experts a workgroup.
__global__ __launch_bounds__(1024) void route_counts_kernel(const int* __restrict__ parts, int blocks,
                                                            int E, int* __restrict__ counts) {
  __shared__ int sums[32][33];
  const int e = blockIdx.x * 32 + threadIdx.x % 32;
  const int part = threadIdx.x / 32;
  int s = 0;
  if (e < E)
    for (int b = part; b < blocks; b += 32) s += parts[static_cast<int64_t>(b) * E + e];
  sums[part][threadIdx.x % 32] = s;
  __syncthreads();
  if (part == 0 && e < E) {
    int t = 0;
    for (int q = 0; q < 32; ++q) t += sums[q][threadIdx.x];
    counts[e] = t;
  }
}

// The gradient of a token's logits, composed in LDS: the chosen experts'
// entries, zero (or the softmax's common term) elsewhere.
template <int DT, int V, int IT, int LT>
__global__ __launch_bounds__(BT) void route_backward_kernel(RouteGradArgs a) {
  constexpr int R = BT / LT;
  using raw = typename Elem<DT>::raw;
  extern __shared__ float dyn[];   // [R][E] entries of the chosen
  const int l = threadIdx.x % LT;
  const int r = threadIdx.x / LT;
  const int E = a.experts, k = a.top_k;
  float* grow = dyn + static_cast<int64_t>(r) * (E | 1);
  const bool softmax = a.score == 0;
  const bool dense = softmax && !a.renorm;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * R; base < a.tokens;
       base += static_cast<int64_t>(gridDim.x) * R) {
    const bool on = base + r < a.tokens;
    const int64_t token = on ? base + r : a.tokens - 1;
    const raw* row = static_cast<const raw*>(a.logits) + token * a.stride;
    for (int e = l; e < E; e += LT) grow[e] = 0.0f;
    wave_lds_sync();
    int at = l < k ? a.indices[token * k + l] : -1;
    if (at < 0 || at >= E) at = -1;
    const float g = at >= 0 ? a.grad[token * k + l] * a.scale : 0.0f;
    float x = Elem<DT>::get(row[at >= 0 ? at : 0]);
    x = x == x ? fminf(x, FLT_MAX) : -INFINITY;
    float p[IT][V], m = 0.0f, sum = 1.0f, common = 0.0f, entry;
    if (dense) {
      load_row<DT, V, IT, LT>(row, E, l, p);
      softmax_stats<V, IT, LT>(p, &m, &sum);
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
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int e = (i * LT + l) * V;
      if (!on || e >= E) continue;
      float y[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        y[v] = grow[e + v];
        if (dense) y[v] = sum > 0.0f ? expf(p[i][v] - m) / sum * (y[v] - common) : 0.0f;
      }
      if constexpr (V == 2) {
        const uint32_t u = static_cast<uint32_t>(Elem<DT>::put(y[0])) |
                           (static_cast<uint32_t>(Elem<DT>::put(y[1])) << 16);
        __builtin_memcpy(out + e, &u, 4);
      } else {
        out[e] = Elem<DT>::put(y[0]);
      }
    }
    wave_lds_sync();   // the row has been read
  }
}

// ------------------------------------------------------------- launchers ---
namespace {
// 16 lanes hold a token of up to 512 experts (32 items each); a team has to
// have a lane per chosen expert and per group, and to leave most rows fewer
// candidates than lanes.
bool narrow_team(int experts, int top_k, int groups) {
  return experts <= 512 && top_k <= 8 && groups <= 16;
}

template <int DT, int V, int LT, class F>
bool by_items(int experts, F&& f) {
  const int items = (experts / V + LT - 1) / LT;
  if (items <= 2) f(std::integral_constant<int, 2>{});
  else if (items <= 4) f(std::integral_constant<int, 4>{});
  else if (items <= 8) f(std::integral_constant<int, 8>{});
  else if (items <= 16) f(std::integral_constant<int, 16>{});
  else if (items <= 32) f(std::integral_constant<int, 32>{});
  else return false;
  return true;
}

int64_t route_grid(int64_t tokens, int team) {
  const int64_t per = BT / team;
  const int64_t want = (tokens + per - 1) / per;
  return want < kRouteBlocks ? want : kRouteBlocks;
}

template <int DT, int V, int LT>
bool forward_team(const RouteArgs& a, int64_t grid, hipStream_t s) {
  const int rows = BT / LT;
  const size_t lds = 4 * (static_cast<size_t>(a.groups > 1 ? rows * (a.experts | 1) : 0) +
                          static_cast<size_t>(a.counts ? a.experts : 0));
  return by_items<DT, V, LT>(a.experts, [&](auto it) {
    constexpr int IT = decltype(it)::value;
    hipLaunchKernelGGL((route_forward_kernel<DT, V, IT, LT>), dim3(static_cast<unsigned>(grid)),
                       dim3(BT), static_cast<unsigned>(lds), s, a);
  });
}
template <int DT, int V, int LT>
bool backward_team(const RouteGradArgs& a, int64_t grid, hipStream_t s) {
  const size_t lds = 4 * static_cast<size_t>(BT / LT) * (a.experts | 1);
  return by_items<DT, V, LT>(a.experts, [&](auto it) {
    constexpr int IT = decltype(it)::value;
    hipLaunchKernelGGL((route_backward_kernel<DT, V, IT, LT>), dim3(static_cast<unsigned>(grid)),
                       dim3(BT), static_cast<unsigned>(lds), s, a);
  });
}

template <int DT>
bool forward_type(const RouteArgs& a, bool narrow, bool pairs, int64_t grid, hipStream_t s) {
  if constexpr (DT != 0)
    if (pairs) return narrow ? forward_team<DT, 2, 16>(a, grid, s) : forward_team<DT, 2, 64>(a, grid, s);
  return narrow ? forward_team<DT, 1, 16>(a, grid, s) : forward_team<DT, 1, 64>(a, grid, s);
}
template <int DT>
bool backward_type(const RouteGradArgs& a, bool narrow, bool pairs, int64_t grid, hipStream_t s) {
  if constexpr (DT != 0)
    if (pairs) return narrow ? backward_team<DT, 2, 16>(a, grid, s) : backward_team<DT, 2, 64>(a, grid, s);
  return narrow ? backward_team<DT, 1, 16>(a, grid, s) : backward_team<DT, 1, 64>(a, grid, s);
}

}  // namespace

int64_t route_blocks(int64_t tokens, int experts, int top_k, int groups) {
  return route_grid(tokens, narrow_team(experts, top_k, groups) ? 16 : 64);
}

hipError_t launch_route_forward(RouteArgs a, int dtype, int* parts, hipStream_t s) {
  const bool narrow = narrow_team(a.experts, a.top_k, a.groups);
  const int team = narrow ? 16 : 64;
  const int64_t grid = route_grid(a.tokens, team);
  int* const counts = a.counts;
  if (counts && grid > 1) a.counts = parts;
  a.sub = 1;
  while (a.sub * 2 * a.groups <= team) a.sub *= 2;
  a.group_size = a.experts / a.groups;
  // 16-bit logits of an even number of experts are read as pairs (dwords, at
  // any alignment: a token's result does not depend on where its row lies)
  const bool pairs = a.experts % 2 == 0;
  bool done;
  { ProfScope ps_("route_forward", s);
  done = dtype == 0 ? forward_type<0>(a, narrow, pairs, grid, s)
       : dtype == 1 ? forward_type<1>(a, narrow, pairs, grid, s)
                    : forward_type<2>(a, narrow, pairs, grid, s); }
  if (!done) return hipErrorInvalidValue;
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !counts || grid <= 1) return e;
  { ProfScope ps_("route_counts", s);
  hipLaunchKernelGGL(route_counts_kernel, dim3(static_cast<unsigned>((a.experts + 31) / 32)),
                     dim3(1024), 0, s, parts, static_cast<int>(grid), a.experts, counts); }
  return hipGetLastError();
}

hipError_t launch_route_backward(const RouteGradArgs& a, int dtype, hipStream_t s) {
  const bool narrow = narrow_team(a.experts, a.top_k, 1);
  const int64_t grid = route_grid(a.tokens, narrow ? 16 : 64);
  const bool pairs = a.experts % 2 == 0;
  bool done;
  { ProfScope ps_("route_backward", s);
  done = dtype == 0 ? backward_type<0>(a, narrow, pairs, grid, s)
       : dtype == 1 ? backward_type<1>(a, narrow, pairs, grid, s)
                    : backward_type<2>(a, narrow, pairs, grid, s); }
  if (!done) return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace lapsum
