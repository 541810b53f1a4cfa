// One step of a beam search: the best `num` continuations over a request's
// beams and the vocabulary, and the states moved to the beams they go on in.
//
// With x the logits of beam w and cum_w its score so far,
//   lse_w = log sum_v e^{x_wv},   s(w, v) = cum_w + (x_wv - lse_w),
// in float32 at each step; larger s first, equal s by the lowest w V + v.  A
// continuation whose s is NaN or -inf is none.
//
// The logits are read once.  A wave takes a contiguous part of a row, holds
// its 2048 logits of a step in registers, adds e^{x - R} to its lanes' sums (R the
// wave's first maximum, moved only when a logit exceeds it by 60, so the sum
// is hardly ever scaled) and keeps the best `num` logits: what reaches the
// current num-th best goes to a list of 64 in LDS, which is cut to the best
// num, by counting, when it is full.  The first threshold is the num-th largest of the
// lanes' maxima.  The finish has one workgroup per request: lse from the
// parts, s of the kept, the best num of them.  s is a monotone function of x, but
// rounding can make it equal for different x (a beam at the lowest float, say), and
// then the index decides among logits that were not kept; the finish
// sees that (a full list ends at the last s taken) and looks for them in the logits.
//
// The sums are held in float64: eight terms in float32, then added.
#include "select_common.hpp"

namespace lapsum {

namespace {
constexpr int BT = 256;
constexpr int BW = BT / kWave;
constexpr int kList = 64;           // entries of a wave's list
constexpr float kMove = 60.0f;      // e^60 times 2^31 terms stays below the largest float
static_assert(kBeamMaxNum * 2 <= kList, "a cut list leaves room");

// Entry: larger value first, then the lower index; 0 is none.
__device__ __forceinline__ uint64_t entry(float v, uint32_t at) {
  return (static_cast<uint64_t>(asc_key(v)) << 32) | (0xffffffffu - at);
}
__device__ __forceinline__ float entry_value(uint64_t e) { return key_value(static_cast<uint32_t>(e >> 32)); }
__device__ __forceinline__ uint32_t entry_index(uint64_t e) { return 0xffffffffu - static_cast<uint32_t>(e); }

__device__ __forceinline__ float next_up(float f) {   // f > -inf
  uint32_t u = __float_as_uint(f + 0.0f);
  return __uint_as_float((u & 0x80000000u) ? u - 1u : u + 1u);
}

// A wave's list of the best entries.
struct BestList {
  uint64_t* buf;   // [kList] in LDS, this wave's
  int count;       // entries in it
  int num;
  float base;      // once num entries are in, num of them are not below it
  float admit;     // values from here on are wanted

  __device__ __forceinline__ void start(uint64_t* b, int n) {
    buf = b;
    count = 0;
    num = n;
    base = admit = -FLT_MAX;
  }
  // Cut to the best num, in order.
  __device__ __forceinline__ void cut() {
    wave_lds_sync();
    const int l = lane_id();
    const uint64_t e = l < count ? buf[l] : 0ull;
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += readlane_as(e, j) > e ? 1 : 0;
    wave_lds_sync();
    if (e && rank < num) buf[rank] = e;
    wave_lds_sync();
    if (count >= num) {
      count = num;
      base = fmaxf(base, entry_value(buf[num - 1]));
    }
    admit = base;
  }
  // The entries (v, at) of the lanes with pred, all of them v >= admit.
  __device__ __forceinline__ void push(bool pred, float v, uint32_t at) {
    for (;;) {
      const uint64_t mask = __ballot(pred);
      if (!mask) return;
      const int pos = count + __popcll(mask & ((1ull << lane_id()) - 1ull));
      if (pred && pos < kList) buf[pos] = entry(v, at);
      const int after = count + __popcll(mask);
      if (after <= kList) {
        count = after;
        return;
      }
      count = kList;
      pred = pred && pos >= kList;
      cut();
      pred = pred && v >= admit;
    }
  }
  // All that follows has a higher index: what equals the num-th best is not
  // wanted any more.
  __device__ __forceinline__ void all_later() {
    if (count >= num) admit = next_up(base);
  }
};

// A value that at least `num` lanes' reach: the largest but for its low bits,
// which are not looked for once few more lanes do.
__device__ __forceinline__ float nth_bound(float mx, int num) {
  const uint32_t key = asc_key(mx);
  const uint32_t differ = wave_max_u32(key) ^ wave_min_u32(key);
  const int bits = differ ? 32 - __clz(static_cast<int>(differ)) : 0;   // that are not common
  uint32_t K = bits < 32 ? (wave_max_u32(key) >> bits) << bits : 0u;
  int count = kWave;
  for (int bit = bits - 1; bit >= 0 && count > num + 4; --bit) {
    const uint32_t cand = K | (1u << bit);
    const int c = __popcll(__ballot(key >= cand));
    if (c >= num) {
      K = cand;
      count = c;
    }
  }
  return key_value(K);
}

// The VE elements of a row from `first` on; past the row -inf.  (A row starts at
// any element: the loads are as wide as they are at any alignment, and a
// row's parts do not depend on its address, so equal rows get equal sums.)
template <int DT>
struct RowVec {
  static constexpr int VE = DT == 0 ? 4 : 8;
};
template <int DT>
__device__ __forceinline__ void load_vec(const typename Elem<DT>::raw* __restrict__ row, int64_t first,
                                         int64_t V, uint32_t (&w)[4]) {
  constexpr int VE = RowVec<DT>::VE;
  if (first + VE <= V) {
    __builtin_memcpy(w, row + first, 16);
  } else {
    typename Elem<DT>::raw r[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) r[j] = first + j < V ? row[first + j] : Elem<DT>::put(-INFINITY);
    __builtin_memcpy(w, r, 16);
  }
}
template <int DT>
__device__ __forceinline__ void get_vec(const uint32_t (&w)[4], float* x) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (DT == 0) {
      x[q] = Elem<0>::get(w[q]);
    } else {
      x[2 * q] = Elem<DT>::get(w[q] & 0xffffu);
      x[2 * q + 1] = Elem<DT>::get(w[q] >> 16);
    }
  }
}

// e^d for d <= kMove to about a float's rounding of d log2(e).
__device__ __forceinline__ float exp_term(float d) {
  constexpr float hi = 1.44269502162933349609375f;
  constexpr float lo = 1.925963033500011e-8f;
  return exp2_fast(__builtin_fmaf(d, hi, d * lo));
}
}  // namespace

// grid (parts, rows).  part p of a row: its steps [p per, (p+1) per).
template <int DT>
__global__ __launch_bounds__(BT) void beam_scan_kernel(BeamArgs a) {
  using raw = typename Elem<DT>::raw;
  constexpr int VE = RowVec<DT>::VE;
  constexpr int U = 32 / VE;   // vectors of a lane and step
  __shared__ uint64_t lists[BW][kList];
  __shared__ float refs[BW];
  __shared__ double sums[BW];
  const int lane = lane_id();
  const int wid = threadIdx.x / kWave;
  const int64_t r = blockIdx.y;
  const raw* row = static_cast<const raw*>(a.logits) + r * a.stride;
  BestList best;
  best.start(lists[wid], a.num);
  float R = -INFINITY;
  double sum = 0.0;
  bool first = true;
  // (a wave's steps are consecutive: later ones hold higher indices)
  const int64_t s0 = (static_cast<int64_t>(blockIdx.x) * BW + wid) * a.steps;
  const int64_t s1 = s0 + a.steps < a.row_steps ? s0 + a.steps : a.row_steps;
  uint32_t next[U][4];   // the next step's logits, under way while one is worked on
  const auto fetch = [&](int64_t st) {
#pragma unroll
    for (int u = 0; u < U; ++u) load_vec<DT>(row, ((st * U + u) * kWave + lane) * VE, a.vocab, next[u]);
  };
  if (s0 < s1) fetch(s0);
  for (int64_t st = s0; st < s1; ++st) {
    float x[U][VE];
    const int64_t at = (st * U * kWave + lane) * VE;   // of u = 0
#pragma unroll
    for (int u = 0; u < U; ++u) get_vec<DT>(next[u], x[u]);
    if (st + 1 < s1) fetch(st + 1);
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < VE; ++j) mx = fmaxf(mx, x[u][j]);
    const float top = wave_max(mx, -INFINITY);
    if (top > R + kMove) {
      sum = R == -INFINITY ? 0.0 : sum * exp(static_cast<double>(R) - static_cast<double>(top));
      R = top;
    }
    const float ref = R == -INFINITY ? 0.0f : R;
#pragma unroll
    for (int u = 0; u < U; u += 8 / VE) {
      float t = 0.0f;
#pragma unroll
      for (int q = 0; q < 8 / VE; ++q)
#pragma unroll
        for (int j = 0; j < VE; ++j) t += exp_term(x[u + q][j] - ref);
      sum += static_cast<double>(t);
    }
    if (first) {
      best.base = best.admit = fmaxf(nth_bound(mx, a.num), -FLT_MAX);
      first = false;
    }
    if (__ballot(mx >= best.admit)) {
      // each lane's wanted logits as bits, then one of each lane at a time (its
      // value read again: registers have no index)
      uint32_t bits = 0u;
#pragma unroll
      for (int u = U - 1; u >= 0; --u)
#pragma unroll
        for (int j = VE - 1; j >= 0; --j) bits = bits + bits + (x[u][j] >= best.admit ? 1u : 0u);
      while (__ballot(bits != 0u)) {
        const int q = bits ? __ffs(bits) - 1 : 0;
        const int64_t v = at + static_cast<int64_t>(q / VE) * (kWave * VE) + q % VE;
        const float y = bits ? Elem<DT>::get(row[v]) : -INFINITY;
        best.push(y >= best.admit, y, static_cast<uint32_t>(v));
        bits &= bits - 1u;
      }
    }
    best.all_later();
  }
  best.cut();
  sum = wave_sum(sum);
  if (lane == 0) {
    refs[wid] = R;
    sums[wid] = sum;
  }
  for (int j = best.count + lane; j < kBeamMaxNum; j += kWave) lists[wid][j] = 0ull;
  __syncthreads();
  if (wid != 0) return;
  // one list and one sum for the workgroup
  uint64_t e[BW];
#pragma unroll
  for (int w = 0; w < BW; ++w) e[w] = lane < kBeamMaxNum ? lists[w][lane] : 0ull;
#pragma unroll
  for (int w = 1; w < BW; ++w)
    best.push(e[w] && entry_value(e[w]) >= best.admit, entry_value(e[w]), entry_index(e[w]));
  best.cut();
  const int64_t part = r * gridDim.x + blockIdx.x;
  if (lane < a.num)
    a.lists[part * a.num + lane] = lane < best.count ? best.buf[lane] : 0ull;
  if (lane == 0) {
    float m = refs[0];
    for (int w = 1; w < BW; ++w) m = fmaxf(m, refs[w]);
    double t = 0.0;
    for (int w = 0; w < BW; ++w)
      if (sums[w] != 0.0)   // (NaN too)
        t += sums[w] * exp(static_cast<double>(refs[w]) - static_cast<double>(m));
    a.refs[part] = m;
    a.sums[part] = t;
  }
}

// One workgroup per request.
template <int DT>
__global__ __launch_bounds__(BT) void beam_finish_kernel(BeamArgs a) {
  using raw = typename Elem<DT>::raw;
  __shared__ uint64_t list[kList];
  __shared__ float lse[kBeamMaxBeams];
  __shared__ int again;
  __shared__ int wcount[BW];
  const int lane = lane_id();
  const int wid = threadIdx.x / kWave;
  const int64_t req = blockIdx.x;
  const int W = a.beams, P = a.parts, num = a.num;
  const float* cum = a.cum + req * W;
  for (int w = wid; w < W; w += BW) {
    const int64_t o = (req * W + w) * P;
    float m = -INFINITY;
    for (int p = lane; p < P; p += kWave) m = fmaxf(m, a.refs[o + p]);
    m = wave_max(m, -INFINITY);
    double t = 0.0;
    for (int p = lane; p < P; p += kWave) {
      const double s = a.sums[o + p];
      if (s != 0.0) t += s * exp(static_cast<double>(a.refs[o + p]) - static_cast<double>(m));
    }
    t = wave_sum(t);
    // (no finite logit: -inf + log 0, and every s is NaN)
    if (lane == 0) lse[w] = static_cast<float>(static_cast<double>(m) + log(t));
  }
  if (threadIdx.x == 0) again = 0;
  __syncthreads();

  // one wave chooses: a lane holds 16 kept entries at a time, the first bound
  // from the lanes' largest
  const uint64_t* kept = a.lists + req * W * P * num;
  const int total = W * P * num;
  if (wid == 0) {
    constexpr int H = 16;
    BestList best;
    best.start(list, num);
    const float per = 1.0f / static_cast<float>(P * num);
    const auto score = [&](int c, uint32_t* at) -> float {
      const uint64_t e = c < total ? kept[c] : 0ull;
      // c / (P num): the product may be off by one either way
      int w = static_cast<int>(static_cast<float>(c) * per);
      w += (w + 1) * P * num <= c ? 1 : 0;
      w -= w * P * num > c ? 1 : 0;
      w = w < W ? w : W - 1;
      *at = static_cast<uint32_t>(w) * static_cast<uint32_t>(a.vocab) + entry_index(e);
      return e ? cum[w] + (entry_value(e) - lse[w]) : -INFINITY;
    };
    for (int c0 = 0; c0 < total; c0 += H * kWave) {
      float s[H], mx = -INFINITY;
      uint32_t at;
#pragma unroll
      for (int h = 0; h < H; ++h) s[h] = score(c0 + h * kWave + lane, &at);
#pragma unroll
      for (int h = 0; h < H; ++h) mx = fmaxf(mx, s[h]);
      if (c0 == 0) best.base = best.admit = fmaxf(nth_bound(mx, num), -FLT_MAX);
      uint32_t bits = 0u;
#pragma unroll
      for (int h = H - 1; h >= 0; --h) bits = bits + bits + (s[h] >= best.admit ? 1u : 0u);
      while (__ballot(bits != 0u)) {
        const int h = bits ? __ffs(bits) - 1 : 0;
        const float y = score(bits ? c0 + h * kWave + lane : total, &at);
        best.push(y >= best.admit, y, at);
        bits &= bits - 1u;
      }
    }
    best.cut();
    for (int j = best.count + lane; j < kBeamMaxNum; j += kWave) list[j] = 0ull;
  }
  __syncthreads();
  uint64_t* out = list;

  // A full list whose last entry has the last s taken may have left out
  // equal ones of a lower index.
  const uint64_t last = out[num - 1];
  if (last) {
    const float least = entry_value(last);
    for (int q = threadIdx.x; q < W * P; q += BT) {
      const uint64_t e = kept[static_cast<int64_t>(q) * num + num - 1];
      const int w = q / P;
      if (e && cum[w] + (entry_value(e) - lse[w]) == least) again = 1;
    }
    __syncthreads();
    if (again) {
      // what is above `least` stays; then the lowest indices that equal it
      int have = 0;
      while (have < num && entry_value(out[have]) > least) ++have;
      __syncthreads();
      for (int w = 0; w < W && have < num; ++w) {
        const raw* row = static_cast<const raw*>(a.logits) + (req * W + w) * a.stride;
        for (int64_t v0 = 0; v0 < a.vocab && have < num; v0 += BT) {
          const int64_t v = v0 + threadIdx.x;
          const float x = v < a.vocab ? Elem<DT>::get(row[v]) : -INFINITY;
          const bool is = x > -INFINITY && cum[w] + (x - lse[w]) == least;
          const uint64_t mask = __ballot(is);
          if (lane == 0) wcount[wid] = __popcll(mask);
          __syncthreads();
          int pos = have + __popcll(mask & ((1ull << lane) - 1ull));
#pragma unroll
          for (int q = 0; q < BW; ++q) {
            if (q < wid) pos += wcount[q];
            have += wcount[q];
          }
          if (is && pos < num)
            out[pos] = entry(least, static_cast<uint32_t>(w) * static_cast<uint32_t>(a.vocab) + static_cast<uint32_t>(v));
          __syncthreads();
        }
      }
    }
  }
  if (threadIdx.x < num) {
    const uint64_t e = out[threadIdx.x];
    const int64_t o = req * num + threadIdx.x;
    const uint32_t at = entry_index(e);
    const uint32_t w = at / static_cast<uint32_t>(a.vocab);
    a.scores[o] = e ? entry_value(e) : -INFINITY;
    a.parents[o] = e ? static_cast<int32_t>(w) : -1;
    a.tokens[o] = e ? static_cast<int32_t>(at - w * static_cast<uint32_t>(a.vocab)) : -1;
  }
}

// --------------------------------------------------------------- reorder ---
// A thread owns a column of 16 bytes (or what the alignment allows) of all of a request's beams:
// it reads every beam's parent before it writes a beam, so the states may be
// reordered in place, and a parent of several beams comes from the caches after its
// first read.
template <typename Vec, int WMAX>
__global__ __launch_bounds__(BT) void beam_reorder_kernel(ReorderArgs a) {
  int t = 0;
  while (t + 1 < a.count && blockIdx.x >= a.state[t + 1].block0) ++t;
  const ReorderState& st = a.state[t];
  const int64_t req = blockIdx.y;
  const int W = a.beams;
  const int64_t c = static_cast<int64_t>(blockIdx.x - st.block0) * BT + threadIdx.x;
  if (c >= st.outer * st.live) return;
  const int64_t o = c / st.live;
  const int64_t at = o * st.outer_stride + (c - o * st.live);
  const Vec* in = static_cast<const Vec*>(st.in) + req * W * st.row + at;
  Vec* out = static_cast<Vec*>(st.out) + req * W * st.row + at;
  const bool same = st.in == st.out;
  const int32_t* parents = a.parents + req * a.parent_stride;
  // (A row that is not needed, because it stays or there is no such beam, is
  // replaced by one that is: no branch stands between the loads.)
  int from[WMAX];
  int some = 0;
#pragma unroll
  for (int i = 0; i < WMAX; ++i) {
    const int32_t p = parents[i < W ? i : 0];
    from[i] = i < W ? (p >= 0 && p < W ? p : i) : -1;
    if (i < W && from[i] != i) some = from[i];
  }
  Vec v[WMAX];
#pragma unroll
  for (int i = 0; i < WMAX; ++i) {
    const bool wanted = from[i] >= 0 && !(same && from[i] == i);
    v[i] = in[(wanted ? from[i] : some) * st.row];
  }
#pragma unroll
  for (int i = 0; i < WMAX; ++i)
    if (from[i] >= 0 && !(same && from[i] == i)) out[i * st.row] = v[i];
}

// ------------------------------------------------------------- launchers ---
void beam_plan(int64_t rows, int64_t vocab, int* steps, int64_t* row_steps, int* parts) {
  const int64_t step = 32 * kWave;
  const int64_t n = (vocab + step - 1) / step;
  // about 16 waves per compute unit, and at least one step each
  int64_t waves = (256 * 16 + rows - 1) / rows;
  if (waves > n) waves = n;
  if (waves > kBeamMaxParts * BW) waves = kBeamMaxParts * BW;
  const int64_t per = (n + waves - 1) / waves;
  *steps = static_cast<int>(per);
  *row_steps = n;
  *parts = static_cast<int>((n + per * BW - 1) / (per * BW));
}

hipError_t launch_beam_select(BeamArgs a, int dtype, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.parts), static_cast<unsigned>(a.batch * a.beams));
  { ProfScope ps_("beam_scan", s);
  if (dtype == 0) hipLaunchKernelGGL((beam_scan_kernel<0>), grid, dim3(BT), 0, s, a);
  else if (dtype == 1) hipLaunchKernelGGL((beam_scan_kernel<1>), grid, dim3(BT), 0, s, a);
  else hipLaunchKernelGGL((beam_scan_kernel<2>), grid, dim3(BT), 0, s, a); }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 one(static_cast<unsigned>(a.batch));
  { ProfScope ps_("beam_finish", s);
  if (dtype == 0) hipLaunchKernelGGL((beam_finish_kernel<0>), one, dim3(BT), 0, s, a);
  else if (dtype == 1) hipLaunchKernelGGL((beam_finish_kernel<1>), one, dim3(BT), 0, s, a);
  else hipLaunchKernelGGL((beam_finish_kernel<2>), one, dim3(BT), 0, s, a); }
  return hipGetLastError();
}

namespace {
template <typename Vec>
void reorder_width(const ReorderArgs& a, dim3 grid, hipStream_t s) {
  if (a.beams <= 4) hipLaunchKernelGGL((beam_reorder_kernel<Vec, 4>), grid, dim3(BT), 0, s, a);
  else if (a.beams <= 8) hipLaunchKernelGGL((beam_reorder_kernel<Vec, 8>), grid, dim3(BT), 0, s, a);
  else if (a.beams <= 16) hipLaunchKernelGGL((beam_reorder_kernel<Vec, 16>), grid, dim3(BT), 0, s, a);
  else hipLaunchKernelGGL((beam_reorder_kernel<Vec, 32>), grid, dim3(BT), 0, s, a);
}
}  // namespace

// Sizes of a.state in vectors of `width` bytes.
hipError_t launch_beam_reorder(ReorderArgs& a, int64_t batch, int width, hipStream_t s) {
  int64_t blocks = 0;
  for (int t = 0; t < a.count; ++t) {
    a.state[t].block0 = static_cast<uint32_t>(blocks);
    blocks += (a.state[t].outer * a.state[t].live + BT - 1) / BT;
  }
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(batch));
  { ProfScope ps_("beam_reorder", s);
  if (width == 16) reorder_width<Move16>(a, grid, s);
  else if (width == 8) reorder_width<Move8>(a, grid, s);
  else if (width == 4) reorder_width<uint32_t>(a, grid, s);
  else if (width == 2) reorder_width<uint16_t>(a, grid, s);
  else reorder_width<uint8_t>(a, grid, s); }
  return hipGetLastError();
}

}  // namespace lapsum
