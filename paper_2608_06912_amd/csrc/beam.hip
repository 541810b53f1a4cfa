// One step of a beam search: the best `num` continuations over a request's
// beams and the vocabulary, and the states moved to the beams they go on in.
//
// With x the logits of beam w and cum_w its score so far,
//   lse_w = log sum_v e^{x_wv},   s(w, v) = cum_w + (x_wv - lse_w),
// in float32 at each step; larger s first, equal s by the lowest w V + v.  A
// continuation whose s is NaN or -inf is none.
//
// beam_scan reads the logits once, as a stream: a wave takes consecutive steps
// of 2048 logits, adds their exponentials to its lanes' sums and keeps each
// step's largest logit, no more.  beam_finish, one workgroup per request, has
// lse from the waves' sums and s of every step's largest.  The num-th largest
// of those bounds the num-th best continuation from below, so only the steps
// that reach the bound, little more than num, are read again (they are in the
// caches), and their continuations that reach it go to lists of 64, cut to the
// best num by counting.  Nothing that could be chosen is left out before its s
// is known: where rounding makes s equal for different logits (a beam at the
// lowest float, say) the index decides.
//
// The choice compares beams by lse, so it is that of the exact sum, rounded once:
// each e^x is formed in float64, within 2e-12 of itself and the same wherever a
// row is divided (the parts depend on how many rows there are), and summed in
// float64 over a power of two that moves only when a logit exceeds it by far.
//
// Bound: the scan by vector issue, 16 operations a logit of which 14 are float64
// (they issue at nearly the rate of float32 ones): 256 rows of 128000 bfloat16
// 36 us, 1.8 TB/s; 29 where part of the logits is in the caches.  Float32
// exponentials, eight added in float32 at a time, took 22 and left lse up to
// 1e-6 off, by another amount for other parts.  Lists of the best logits kept
// in the scan, as a first form had them, took 43: the candidates' steps wait on
// each other.  The finish is such a chain (lse, bound, the steps' second read,
// the lists): 14 us for 32 requests of 8 beams, 7.1 for one of 4.
#include "select_common.hpp"

namespace lapsum {

namespace {
constexpr int BT = 256;
constexpr int BW = BT / kWave;
constexpr int FT = 1024;            // threads of the finish
constexpr int FW = FT / kWave;
constexpr int kFinishSteps = 2048;  // steps the finish looks at together
constexpr int kList = 64;           // entries of a wave's list
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
  // All that follows has a higher index: what equals the num-th best is not wanted
  // any more.
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

// The VE elements of a row from `first` on; past the row -inf.  (A row may
// start at any element: the loads are as wide at any alignment.)
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

// A wave's step: 32 logits a lane.
template <int DT>
struct Step {
  static constexpr int VE = RowVec<DT>::VE;
  static constexpr int U = 32 / VE;   // vectors
  uint32_t w[U][4];
  // The first logit of vector u, which lane 0 .. 63 continue.
  static __device__ __forceinline__ int64_t first(int64_t st, int u) {
    return ((st * U + u) * kWave + lane_id()) * VE;
  }
  __device__ __forceinline__ void fetch(const typename Elem<DT>::raw* row, int64_t st, int64_t V) {
#pragma unroll
    for (int u = 0; u < U; ++u) load_vec<DT>(row, first(st, u), V, w[u]);
  }
  __device__ __forceinline__ void get(float (&x)[U][VE]) const {
#pragma unroll
    for (int u = 0; u < U; ++u) get_vec<DT>(w[u], x[u]);
  }
};

// e^x / 2^N for x from kLow below a reference to kRise above it, N the integer
// nearest its log2 e: with n the integer nearest x log2 e, 2^(n - N) 2^f, where
// 2^f = 1 + f q(f) and q interpolates (2^f - 1) / f at eight Chebyshev nodes of
// [-1/2, 1/2] (relative error of 2^f 2e-12).  shift is 1.5 2^52 - N: the sum
// with it rounds to an integer and leaves n - N in the low bits.
constexpr float kRise = 300.0f;
constexpr float kLow = 600.0f;
constexpr float kFar = 1073741824.0f;   // from here on a float is 64 above the one before it at least
constexpr double kShift = 6755399441055744.0;
constexpr double kLn2 = 0.69314718055994530942;
__device__ __forceinline__ double exp_by(float x, double shift) {
  const double y = static_cast<double>(x);
  const double t = __builtin_fma(y, kLog2e, shift);
  const double f = __builtin_fma(y, kLog2e, shift - t);
  double q = 1.325080551750225e-06;
  q = __builtin_fma(q, f, 1.5303700711365693e-05);
  q = __builtin_fma(q, f, 1.5403475186530786e-04);
  q = __builtin_fma(q, f, 1.3333478473685416e-03);
  q = __builtin_fma(q, f, 9.61812913523614e-03);
  q = __builtin_fma(q, f, 5.5504109063258665e-02);
  q = __builtin_fma(q, f, 2.4022650695888503e-01);
  q = __builtin_fma(q, f, 6.931471805568324e-01);
  const double p = __builtin_fma(q, f, 1.0);
  return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
}

}  // namespace

// grid (parts, rows), a wave a part of `steps` steps.  refs and sums: sum of
// e^{x - ref} over the part.
template <int DT>
__global__ __launch_bounds__(BT) void beam_scan_kernel(BeamArgs a) {
  using S = Step<DT>;
  const int lane = lane_id();
  const int64_t r = blockIdx.y;
  const auto* row = static_cast<const typename Elem<DT>::raw*>(a.logits) + r * a.stride;
  const int64_t part = static_cast<int64_t>(blockIdx.x) * BW + threadIdx.x / kWave;
  if (part >= a.parts) return;   // (whole waves; no barrier below)
  const int64_t s0 = part * a.steps;
  const int64_t s1 = s0 + a.steps < a.row_steps ? s0 + a.steps : a.row_steps;
  float kept = -INFINITY;
  bool none = false;                // a logit of NaN or +inf
  bool have = false, far = false;   // a reference, one past kFar
  float ref = 0.0f;
  double N = 0.0, sum = 0.0;        // the sum over 2^N, or e^ref where it is far
  S next;
  next.fetch(row, s0, a.vocab);
  for (int64_t st = s0; st < s1; ++st) {
    float x[S::U][S::VE];
    next.get(x);
    if (st + 1 < s1) next.fetch(row, st + 1, a.vocab);   // under way while this one is worked on
    float mx = -INFINITY;   // (NaN where one is)
#pragma unroll
    for (int u = 0; u < S::U; ++u)
#pragma unroll
      for (int j = 0; j < S::VE; ++j) mx = __builtin_elementwise_maximum(mx, x[u][j]);
    none = none || __any(!(mx < INFINITY));
    const float top = wave_max(mx, -INFINITY);
    const int at = static_cast<int>(st - s0);
    kept = lane == (at & 63) ? top : kept;
    if ((at & 63) == 63 || st + 1 == s1) {
      if (lane <= (at & 63)) a.tops[r * a.row_steps + s0 + (at & ~63) + lane] = kept;
    }
    if (!(top > -INFINITY)) continue;   // (all of it masked)
    // the reference: the first largest that is no mask, moved where one is far above it
    if (!have || (far ? top > ref : top - ref > kRise)) {
      const bool now_far = fabsf(top) >= kFar;
      const double old = N;
      N = rint(static_cast<double>(top) * kLog2e);
      // (what lies 64 below has no weight in a float64 sum)
      sum = far || now_far ? 0.0 : ldexp(sum, static_cast<int>(fmax(old - N, -4000.0)));
      have = true;
      far = now_far;
      ref = top;
    }
    if (!far) {
      const float low = ref - kLow;
      const double shift = kShift - N;
      double t[4] = {};
#pragma unroll
      for (int u = 0; u < S::U; ++u)
#pragma unroll
        for (int j = 0; j < S::VE; ++j) t[j % 4] += exp_by(__builtin_elementwise_maximum(x[u][j], low), shift);
      sum += (t[0] + t[1]) + (t[2] + t[3]);
    } else {
      int same = 0;
#pragma unroll
      for (int u = 0; u < S::U; ++u)
#pragma unroll
        for (int j = 0; j < S::VE; ++j) same += x[u][j] == ref ? 1 : 0;
      sum += static_cast<double>(same);
    }
  }
  if (none) sum = static_cast<double>(NAN);
  sum = wave_sum(sum);
  if (lane == 0) {
    a.refs[r * a.parts + part] = far ? static_cast<double>(ref) : N * kLn2;
    a.sums[r * a.parts + part] = sum;
  }
}

// One workgroup per request.
template <int DT>
__global__ __launch_bounds__(FT) void beam_finish_kernel(BeamArgs a) {
  using S = Step<DT>;
  using raw = typename Elem<DT>::raw;
  __shared__ uint64_t lists[FW][kList];
  __shared__ float lse[kBeamMaxBeams];
  __shared__ uint64_t merged[FW * kBeamMaxNum];
  __shared__ float score[kFinishSteps];
  __shared__ uint32_t wanted[kFinishSteps];
  __shared__ int count, counts[FW];
  __shared__ float bound;
  const int lane = lane_id();
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t req = blockIdx.x;
  const int W = a.beams, P = a.parts, num = a.num;
  const int steps = static_cast<int>(a.row_steps);
  const float* cum = a.cum + req * W;
  for (int w = wid; w < W; w += FW) {
    const int64_t o = (req * W + w) * P;
    double m = -INFINITY;
    for (int p = lane; p < P; p += kWave) m = a.sums[o + p] != 0.0 ? fmax(m, a.refs[o + p]) : m;
    m = wave_max(m, -static_cast<double>(INFINITY));
    double t = 0.0;
    for (int p = lane; p < P; p += kWave) {
      const double s = a.sums[o + p];
      if (s != 0.0) t += s * exp(a.refs[o + p] - m);   // (NaN too)
    }
    t = wave_sum(t);
    // (nothing but masked logits: -inf, and every s is NaN)
    if (lane == 0) lse[w] = t == 0.0 ? -INFINITY : static_cast<float>(m + log(t));
  }
  __syncthreads();

  // s of step q's largest logit: steps of one beam after another
  const float* tops = a.tops + req * W * static_cast<int64_t>(steps);
  const int total = W * steps;
  const float inv = 1.0f / static_cast<float>(steps);
  const auto beam_of = [&](int q) {   // q / steps: the product may be off by one either way
    int w = static_cast<int>(static_cast<float>(q) * inv);
    w += w + 1 < W && (w + 1) * steps <= q ? 1 : 0;
    w -= w * steps > q ? 1 : 0;
    return w < W ? w : W - 1;
  };
  BestList best;
  best.start(lists[wid], num);
  for (int q0 = 0; q0 < total; q0 += kFinishSteps) {
    const int q1 = total - q0 < kFinishSteps ? total : q0 + kFinishSteps;
    for (int q = q0 + threadIdx.x; q < q1; q += FT) {
      const int w = beam_of(q);
      score[q - q0] = cum[w] + (tops[q] - lse[w]);
    }
    __syncthreads();
    if (wid == 0) {
      const int size = q1 - q0;
      if (q0 == 0) {
        float mx = -INFINITY;
        for (int q = lane; q < size; q += kWave) mx = fmaxf(mx, score[q]);
        const float b = fmaxf(nth_bound(mx, num), -FLT_MAX);
        if (lane == 0) bound = b;
        best.base = best.admit = b;
      }
      int n = 0;   // the steps that reach the bound, in order
      const float b = best.base;
      for (int q = lane; q - lane < size; q += kWave) {
        const bool is = q < size && score[q] >= b;
        const uint64_t mask = __ballot(is);
        if (is) wanted[n + __popcll(mask & ((1ull << lane) - 1ull))] = static_cast<uint32_t>(q0 + q);
        n += __popcll(mask);
      }
      if (lane == 0) count = n;
    }
    __syncthreads();
    if (q0 == 0) best.base = best.admit = bound;
    const int n = count;
    for (int i = wid; i < n; i += FW) {
      const int q = static_cast<int>(wanted[i]);
      const int w = beam_of(q);
      const int64_t st = q - w * steps;
      const raw* row = static_cast<const raw*>(a.logits) + (req * W + w) * a.stride;
      const float c = cum[w], l = lse[w];
      const uint32_t base = static_cast<uint32_t>(w) * static_cast<uint32_t>(a.vocab);
      S step;
      step.fetch(row, st, a.vocab);
      float x[S::U][S::VE];
      step.get(x);
      // each lane's wanted ones as bits, then one of each lane at a time (its value
      // read again: registers have no index)
      if (total < 2 * num && best.count < num) {
        // so few steps bound little: the num-th largest of this one's lanes
        float mx = -INFINITY;
#pragma unroll
        for (int u = 0; u < S::U; ++u)
#pragma unroll
          for (int j = 0; j < S::VE; ++j) mx = fmaxf(mx, c + (x[u][j] - l));
        best.base = best.admit = fmaxf(best.base, nth_bound(mx, num));
      }
      uint32_t bits = 0u;
#pragma unroll
      for (int u = S::U - 1; u >= 0; --u)
#pragma unroll
        for (int j = S::VE - 1; j >= 0; --j) bits = bits + bits + (c + (x[u][j] - l) >= best.admit ? 1u : 0u);
      while (__ballot(bits != 0u)) {
        const int k = bits ? __ffs(bits) - 1 : 0;
        const int64_t v = S::first(st, k / S::VE) + k % S::VE;
        const float s = bits ? c + (Elem<DT>::get(row[v]) - l) : -INFINITY;
        best.push(s >= best.admit, s, base + static_cast<uint32_t>(v));
        bits &= bits - 1u;
      }
      best.all_later();
    }
    __syncthreads();   // wanted and count have been read
  }
  // the waves' lists together, and the best of them
  if (best.count > num) best.cut();
  if (lane == 0) counts[wid] = best.count;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int f = 0; f < FW; ++f) {
    before += f < wid ? counts[f] : 0;
    all += counts[f];
  }
  wave_lds_sync();   // (this wave's list)
  if (lane < best.count) merged[before + lane] = best.buf[lane];
  __syncthreads();
  if (wid != 0) return;
  best.start(lists[0], num);
  for (int j = 0; j < all; j += kWave) {
    const uint64_t e = j + lane < all ? merged[j + lane] : 0ull;
    best.push(e && entry_value(e) >= best.admit, entry_value(e), entry_index(e));
  }
  best.cut();
  if (lane < num) {
    const uint64_t e = lane < best.count ? best.buf[lane] : 0ull;
    const int64_t o = req * num + lane;
    const uint32_t at = entry_index(e);
    const uint32_t w = at / static_cast<uint32_t>(a.vocab);
    a.scores[o] = e ? entry_value(e) : -INFINITY;
    a.parents[o] = e ? static_cast<int32_t>(w) : -1;
    a.tokens[o] = e ? static_cast<int32_t>(at - w * static_cast<uint32_t>(a.vocab)) : -1;
  }
}

// --------------------------------------------------------------- reorder ---
// A thread owns a column of 16 bytes (or what the alignment allows) of all of a
// request's beams: it reads every beam's parent before it writes a beam, so the
// states may be reordered in place, and a parent of several beams comes from
// the caches after its first read.  Bound: memory.  32 x 8 rows of 258 KiB in
// two states 37 us (135 MB written, up to as much read), 16 x 4 rows of 517 KiB
// in eight 77 us (271 MB). A branch around each load took the first from 37 to
// 73: its registers.
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
  if (waves > kBeamMaxParts) waves = kBeamMaxParts;
  const int64_t per = (n + waves - 1) / waves;
  *steps = static_cast<int>(per);
  *row_steps = n;
  *parts = static_cast<int>((n + per - 1) / per);
}

hipError_t launch_beam_select(BeamArgs a, int dtype, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.parts + BW - 1) / BW), static_cast<unsigned>(a.batch * a.beams));
  { ProfScope ps_("beam_scan", s);
  if (dtype == 0) hipLaunchKernelGGL((beam_scan_kernel<0>), grid, dim3(BT), 0, s, a);
  else if (dtype == 1) hipLaunchKernelGGL((beam_scan_kernel<1>), grid, dim3(BT), 0, s, a);
  else hipLaunchKernelGGL((beam_scan_kernel<2>), grid, dim3(BT), 0, s, a); }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 one(static_cast<unsigned>(a.batch));
  { ProfScope ps_("beam_finish", s);
  if (dtype == 0) hipLaunchKernelGGL((beam_finish_kernel<0>), one, dim3(FT), 0, s, a);
  else if (dtype == 1) hipLaunchKernelGGL((beam_finish_kernel<1>), one, dim3(FT), 0, s, a);
  else hipLaunchKernelGGL((beam_finish_kernel<2>), one, dim3(FT), 0, s, a); }
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
