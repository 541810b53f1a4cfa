// Eviction from a key-value cache by accumulated attention weight.
//
//   accumulate  acc[b,h,s] (+)= sum over the query heads of h and the queries
//               of w[b, h G + g, q, s]; a column sum, each weight read once
//   evict       of each (sequence, head) the best `budget` entries: the first
//               `sink` and the last `recent` positions, then the largest acc,
//               equal ones by the lowest slot; copied in slot order
//   step        one token: acc += its weights, the first empty slot or else
//               the smallest acc outside sink and recent gets the new entry
//
// A selection compares acc, so it is formed in float64 and rounded once: its
// value does not depend on the order of the sum.
//
// Selection key of an entry (uint32, larger stays longer): empty 0, NaN 1, then
// the float's order, and the largest for what always stays.
#include "select_common.hpp"

namespace lapsum {

namespace {
constexpr uint32_t kStays = 0xffffffffu;
constexpr uint32_t kTopKey = 0xff800000u;   // of +inf, the largest of a number
constexpr uint32_t kLowKey = 0x007fffffu;   // of -inf, the smallest

__device__ __forceinline__ uint32_t stay_key(float acc, int32_t pos, int32_t first_old, int sink) {
  if (pos < 0) return 0u;
  if (pos < sink || pos >= first_old) return kStays;
  const uint32_t k = asc_key(acc);
  return k == 0u ? 1u : k;
}

template <int DT>
struct Wide {
  static constexpr int VE = DT == 0 ? 4 : 8;
};

template <int DT>
__device__ __forceinline__ void get_words(const uint32_t (&w)[4], float* x) {
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
}  // namespace

// ------------------------------------------------------------ accumulate ---
// A workgroup takes 64 VE columns of one (sequence, head); its waves take the
// rows of weights (query heads x queries) in turn.  Bound: the read of the
// weights (32 heads x 32 queries over 131072 bfloat16: 50 us, 5.4 TB/s; 12 x 53
// rows of 130789, which start at any element, 29 us); with few columns the
// latency of the rows in flight (1000 columns, 512 rows: 7 us with sixteen
// waves, 9 with four).
template <int DT, int T>
__global__ __launch_bounds__(T) void cache_accumulate_kernel(AccumulateArgs a) {
  using raw = typename Elem<DT>::raw;
  constexpr int VE = Wide<DT>::VE;
  constexpr int W = T / kWave;
  constexpr int U = T == 1024 ? 4 : 8;   // rows in flight
  __shared__ double part[W - 1][kWave][VE + 1];
  const int lane = lane_id();
  const int wid = threadIdx.x / kWave;
  const int64_t bh = blockIdx.x / a.tiles;
  const int64_t tile = blockIdx.x - bh * a.tiles;
  const int64_t b = bh / a.kv, h = bh - b * a.kv;
  const int64_t s = (tile * kWave + lane) * VE;
  int64_t seen = a.seen ? a.seen[b] : a.keys;
  seen = seen < 0 ? 0 : (seen < a.keys ? seen : a.keys);
  const int live = s >= seen ? 0 : (seen - s < VE ? static_cast<int>(seen - s) : VE);
  double sum[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) sum[j] = 0.0;
  const raw* base = static_cast<const raw*>(a.weights) + b * a.stride_b + h * a.group * a.stride_h + s;
  const int rows = static_cast<int>(a.group * a.queries), queries = static_cast<int>(a.queries);
  // the wave's next row: query q of head g, counted on without a division
  int g = 0, q = __builtin_amdgcn_readfirstlane(wid);
  const auto row = [&]() -> const raw* {
    while (q >= queries && g + 1 < a.group) {
      q -= queries;
      ++g;
    }
    const raw* p = base + g * a.stride_h + (q < queries ? q : queries - 1) * a.stride_q;
    q += W;
    return p;
  };
  if (a.keys >= VE) {
    // A lane at the row's end adds up the row's last VE columns and moves its sums
    // into place afterwards, and columns that are not seen are added up with the
    // others and left out: every lane's loads are whole, and none waits for a
    // branch.
    const int64_t over = s + VE > a.keys ? s + VE - a.keys : 0;
    if (tile * kWave * VE < seen) {   // (columns of this workgroup are seen)
      for (int r0 = wid; r0 < rows; r0 += W * U) {
        uint32_t x[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u)   // (past the last row that one again)
          __builtin_memcpy(x[u], row() - over, 16);
        const int in = (rows - r0 + W - 1) / W;   // of the U, rows there are
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float y[VE];
          get_words<DT>(x[u], y);
          const bool is = u < in;
#pragma unroll
          for (int j = 0; j < VE; ++j) sum[j] += static_cast<double>(is ? y[j] : 0.0f);
        }
      }
    }
    const int back = over < VE ? static_cast<int>(over) : 0;
#pragma unroll
    for (int d = 1; d < VE; d *= 2)   // sum[j] <- sum[j + back]
#pragma unroll
      for (int j = 0; j < VE; ++j)
        if (back & d) sum[j] = sum[j + d < VE ? j + d : j];
  } else if (live > 0) {
    for (int r = wid; r < rows; r += W) {
      const raw* p = row();
#pragma unroll
      for (int j = 0; j < VE; ++j)
        if (j < live) sum[j] += static_cast<double>(Elem<DT>::get(p[j]));
    }
  }
  if (wid > 0) {
#pragma unroll
    for (int j = 0; j < VE; ++j) part[wid - 1][lane][j] = sum[j];
  }
  __syncthreads();
  if (wid > 0) return;
  float* acc = a.out + bh * a.keys + s;
  const float* old = a.acc ? a.acc + bh * a.keys + s : nullptr;
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    if (s + j >= a.keys) continue;
    double t = sum[j];
#pragma unroll
    for (int w = 0; w < W - 1; ++w) t += part[w][lane][j];
    if (old) {
      const float o = old[j];
      acc[j] = j < live ? static_cast<float>(static_cast<double>(o) + t) : o;
    } else {
      acc[j] = j < live ? static_cast<float>(t) : 0.0f;
    }
  }
}

// ----------------------------------------------------------------- evict ---
// The slots that stay, one workgroup per (sequence, head): the budget-th
// largest key, then the kept slots in order.
//
// The key is found digit by digit from histograms in LDS, 2048 bins over the
// range that still holds it (the keys of positive sums are spread like their
// logarithms, so few share a bin).  Rows of up to 32768 slots keep their keys
// in registers.  A longer row is read once: 8192 of its entries give a window
// that holds the last kept value, one pass marks what is above it and what is
// in it, as bits in LDS, and only the window's entries (a few percent) are
// looked at again.  What that does not settle (a window that misses, or too
// many equal values in it), and a row past 262144 slots, takes a pass over the
// row per digit.
//
// Bound: one compute unit per row, its barriers and its instructions.  8 rows
// of 131072, 4096 kept: 34 us (sample and window 5, marking 7.4, list 3, its
// digits 6, slots 3, the rest loads and launch), 255 where every digit took a
// pass and the bins were the floats' top bits; half of that row kept 57.  96
// rows of 6007: 11.4 us; 8 of 1000: 8.4.
constexpr int kEvictBins = 2048;
constexpr int kEvictSample = 8192;
constexpr int kEvictList = 12288;            // entries of the window
constexpr int kEvictWords = 4096;            // 64 slots each
constexpr int kEvictRound = 16;              // loads in flight per lane
constexpr double kEvictSigmas = 4.0;

namespace {
// What the threads of a workgroup of T exchange; the pairs alternate, so that
// one round's values may still be read while the next are written.
template <int T>
struct EvictSmem {
  uint32_t bins[2][kEvictBins];
  uint32_t wsum[2][T / kWave];
  uint32_t bin[2], above[2];
  uint32_t live, stays, lo, hi;
};

template <int T>
struct EvictBlock {
  EvictSmem<T>& sm;
  int turn = 0;

  // Once, with a barrier before the first histogram.
  __device__ __forceinline__ void start() {
    for (int e = threadIdx.x; e < kEvictBins; e += T) sm.bins[0][e] = sm.bins[1][e] = 0u;
    if (threadIdx.x == 0) {
      sm.live = sm.stays = sm.hi = 0u;
      sm.lo = 0xffffffffu;
    }
    __syncthreads();
  }
  // Inclusive sum over the workgroup, and the total.  One barrier.
  __device__ __forceinline__ uint32_t incl(uint32_t x, uint32_t* total) {
    const int wid = threadIdx.x / kWave;
    uint32_t* wsum = sm.wsum[turn];
    turn ^= 1;
    uint32_t s = wave_incl_add<uint32_t>(x);
    if (lane_id() == kWave - 1) wsum[wid] = s;
    __syncthreads();
    uint32_t all = 0u;
#pragma unroll
    for (int w = 0; w < T / kWave; ++w) {
      const uint32_t v = wsum[w];
      if (w < wid) s += v;
      all += v;
    }
    *total = all;
    return s;
  }
  __device__ __forceinline__ uint32_t sum(uint32_t x) {
    uint32_t all;
    incl(x, &all);
    return all;
  }
  // The bin of bins[which] (from the last downwards) where the count reaches
  // `want`, from 1 to the total, and what is in the bins after it; the bins are
  // zero again afterwards.  After a barrier; two barriers.
  __device__ __forceinline__ void find_bin(int which, uint32_t want, uint32_t* bin, uint32_t* above) {
    constexpr int B = kEvictBins / T;
    const int hi = kEvictBins - 1 - B * static_cast<int>(threadIdx.x);
    uint32_t c[B], s = 0u, all;
#pragma unroll
    for (int q = 0; q < B; ++q) {
      c[q] = sm.bins[which][hi - q];
      sm.bins[which][hi - q] = 0u;
      s += c[q];
    }
    const int slot = turn;
    uint32_t run = incl(s, &all) - s;
    if (run < want && want <= run + s) {
      bool found = false;
#pragma unroll
      for (int q = 0; q < B; ++q) {
        if (!found && want <= run + c[q]) {
          sm.bin[slot] = static_cast<uint32_t>(hi - q);
          sm.above[slot] = run;
          found = true;
        }
        run += c[q];
      }
    }
    __syncthreads();
    *bin = sm.bin[slot];
    *above = sm.above[slot];
  }
  // The live entries, those that always stay, and the range of the others' keys, of
  // each(f): f(key) for this thread's.  Once; one barrier.
  template <class F>
  __device__ __forceinline__ void look(F&& each, uint32_t* live, uint32_t* stays, uint32_t* lo, uint32_t* hi) {
    uint32_t n = 0u, s = 0u, a = 0xffffffffu, b = 0u;
    each([&](uint32_t k) {
      n += k != 0u ? 1u : 0u;
      s += k == kStays ? 1u : 0u;
      const bool some = k != 0u && k != kStays;
      a = some && k < a ? k : a;
      b = some && k > b ? k : b;
    });
    n = wave_sum(n);
    s = wave_sum(s);
    a = wave_min_u32(a);
    b = wave_max_u32(b);
    if (lane_id() == 0) {
      atomicAdd(&sm.live, n);
      atomicAdd(&sm.stays, s);
      atomicMin(&sm.lo, a);
      atomicMax(&sm.hi, b);
    }
    __syncthreads();
    *live = sm.live;
    *stays = sm.stays;
    *lo = sm.lo;
    *hi = sm.hi;
  }
  static __device__ __forceinline__ int shift_of(uint32_t lo, uint32_t hi) {
    const int bits = hi > lo ? 32 - __clz(static_cast<int>(hi - lo)) : 0;
    return bits > 11 ? bits - 11 : 0;
  }
  // The `want`-th largest of the keys in [lo, hi] (at least that many), and how
  // many that equal it are among the first `want`.
  template <class F>
  __device__ __forceinline__ void kth(F&& each, uint32_t want, uint32_t lo, uint32_t hi, uint32_t* key,
                                      uint32_t* equal) {
    for (int which = 0;; which ^= 1) {
      const int shift = shift_of(lo, hi);
      each([&](uint32_t k) {
        if (k >= lo && k <= hi) atomicAdd(&sm.bins[which][(k - lo) >> shift], 1u);
      });
      __syncthreads();
      uint32_t bin, above;
      find_bin(which, want, &bin, &above);
      want -= above;
      lo += bin << shift;
      const uint32_t end = lo + ((1u << shift) - 1u);
      hi = end < hi ? end : hi;
      if (shift == 0) break;
    }
    *key = lo;
    *equal = want;
  }
  // The last key that stays and how many equal ones do, for `budget` of the entries
  // of each(f); key 0 and none equal where all of them stay.
  template <class F>
  __device__ __forceinline__ void last_key(F&& each, uint32_t budget, uint32_t* key, uint32_t* equal) {
    uint32_t live, stays, lo, hi;
    look(each, &live, &stays, &lo, &hi);
    *key = *equal = 0u;
    if (live <= budget) return;
    if (stays >= budget) {   // (positions that are not distinct)
      *key = kStays;
      *equal = budget;
      return;
    }
    kth(each, budget - stays, lo, hi, key, equal);
  }
};

// Which entries of the row are there, and which always stay.
struct EvictRow {
  const float* acc;
  const int32_t* pos;   // null: positions are the slots
  int64_t n;            // slots to look at
  int32_t first_old;    // positions from here on are the last `recent`
  int sink;
  __device__ __forceinline__ uint32_t key(int64_t i) const {
    return stay_key(acc[i], pos ? pos[i] : static_cast<int32_t>(i), first_old, sink);
  }
};
__device__ __forceinline__ EvictRow evict_row(const EvictArgs& a, int64_t bh) {
  const int32_t seen = a.seen[bh / a.kv] < 0 ? 0 : a.seen[bh / a.kv];
  EvictRow r;
  r.acc = a.acc + bh * a.room;
  r.pos = a.pos ? a.pos + bh * a.room : nullptr;
  r.n = !a.pos && seen < a.room ? seen : a.room;
  r.first_old = seen - a.recent > 0 ? seen - a.recent : 0;
  r.sink = a.sink;
  return r;
}
}  // namespace

// Rows of up to T PER slots: slot i T + t is item i of thread t.
template <int T, int PER>
__global__ __launch_bounds__(T) void cache_select_kernel(EvictArgs a) {
  constexpr int W = T / kWave;
  static_assert(PER * W <= T, "a thread per 64 slots");
  __shared__ EvictSmem<T> sm;
  __shared__ uint32_t counts[PER * W];   // kept and equal ones per 64 slots, then before them
  EvictBlock<T> block{sm};
  const int tid = threadIdx.x, lane = lane_id(), wid = tid / kWave;
  const int64_t bh = blockIdx.x;
  const EvictRow row = evict_row(a, bh);
  uint32_t k[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) k[i] = i * T + tid < row.n ? row.key(i * T + tid) : 0u;
  block.start();
  uint32_t last, want;
  block.last_key([&](auto&& f) {
#pragma unroll
    for (int i = 0; i < PER; ++i) f(k[i]);
  }, static_cast<uint32_t>(a.budget), &last, &want);
  // above the last key in the low half, equal to it in the high half (at most 32768
  // of each)
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint64_t gt = __ballot(k[i] > last), eq = __ballot(k[i] == last && k[i] != 0u);
    if (lane == 0)
      counts[i * W + wid] = static_cast<uint32_t>(__popcll(gt)) | (static_cast<uint32_t>(__popcll(eq)) << 16);
  }
  __syncthreads();
  const uint32_t c = tid < PER * W ? counts[tid] : 0u;
  uint32_t all;
  const uint32_t before = block.incl(c, &all) - c;
  if (tid < PER * W) counts[tid] = before;
  __syncthreads();
  int32_t* slots = a.slots + bh * a.budget;
  const uint64_t below = (1ull << lane) - 1ull;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint64_t gt = __ballot(k[i] > last), eq = __ballot(k[i] == last && k[i] != 0u);
    const uint32_t b = counts[i * W + wid];
    const uint32_t e = (b >> 16) + static_cast<uint32_t>(__popcll(eq & below));
    const uint32_t at = (b & 0xffffu) + static_cast<uint32_t>(__popcll(gt & below)) + (e < want ? e : want);
    if (k[i] > last || (k[i] == last && k[i] != 0u && e < want)) slots[at] = i * T + tid;
  }
  const uint32_t eq_all = all >> 16;
  const int64_t kept = (all & 0xffffu) + (eq_all < want ? eq_all : want);
  for (int64_t j = kept + tid; j < a.budget; j += T) slots[j] = -1;
}

// Longer rows.
constexpr int ET = 1024;
constexpr int EW = ET / kWave;

__global__ __launch_bounds__(ET) void cache_select_long_kernel(EvictArgs a) {
  __shared__ EvictSmem<ET> sm;
  __shared__ uint64_t keep[kEvictWords], window[kEvictWords];
  __shared__ int32_t list_at[kEvictList];
  EvictBlock<ET> block{sm};
  const int tid = threadIdx.x, lane = lane_id(), wid = tid / kWave;
  const int64_t bh = blockIdx.x;
  const EvictRow row = evict_row(a, bh);
  const int64_t n = row.n;
  const uint32_t budget = static_cast<uint32_t>(a.budget);
  int32_t* slots = a.slots + bh * a.budget;
  const int words = static_cast<int>((n + 63) / 64);
  bool done = words <= kEvictWords;
  if (done) {
    // 1. a window from the sample
    constexpr int PER = kEvictSample / ET;
    uint32_t k[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      k[i] = n > 0 ? row.key((static_cast<int64_t>(i) * ET + tid) * n / kEvictSample) : 0u;
      if (k[i] == kStays) k[i] = 0u;
    }
    block.start();
    uint32_t got, none, lo, hi;
    const auto sample = [&](auto&& f) {
#pragma unroll
      for (int i = 0; i < PER; ++i) f(k[i]);
    };
    block.look(sample, &got, &none, &lo, &hi);
    // ranks of its ends in the sample, from the largest: kEvictSigmas standard
    // deviations of a binomial around the share that stays (of the entries that do
    // not always stay)
    const double always = static_cast<double>(a.sink) + static_cast<double>(a.recent);
    const double total = row.pos ? static_cast<double>(n) * got / kEvictSample : n - always;
    const double share = total > a.budget - always ? (a.budget - always) / total : 1.0;
    const double mid = share * got, dev = kEvictSigmas * sqrt(got * (share * (1.0 - share))) + 2.0;
    uint32_t wlo = 0u, whi = kTopKey;   // window of keys, both ends in it
    // (a list that holds all that stays as well needs no upper end)
    const bool top = mid - dev >= 1.0 && (mid + dev) * (static_cast<double>(n) / kEvictSample) > 0.9 * kEvictList;
    const bool bottom = mid + dev <= got;
    if (got > 0u) {
      // ends rounded outwards to a bin: about two entries of the sample
      const int shift = block.shift_of(lo, hi);
      sample([&](uint32_t v) {
        if (v != 0u) atomicAdd(&sm.bins[0][(v - lo) >> shift], 1u);
        if (v != 0u && top) atomicAdd(&sm.bins[1][(v - lo) >> shift], 1u);
      });
      __syncthreads();
      uint32_t bin, unused;
      block.find_bin(0, bottom ? static_cast<uint32_t>(mid + dev) : got, &bin, &unused);
      if (bottom) wlo = lo + (bin << shift);
      if (top) {
        block.find_bin(1, static_cast<uint32_t>(mid - dev), &bin, &unused);
        whi = lo + (bin << shift) + ((1u << shift) - 1u);
        whi = whi < kTopKey ? whi : kTopKey;
      }
    }
    // Ends that are no number's key (below -inf, and that of a zero's lower
    // neighbour, which would read -0) go up to the next that is: the comparison of
    // the values is then that of the keys, so an entry above the window by the one
    // is above it by the other.
    if (wlo > 1u && wlo < kLowKey) wlo = kLowKey;
    if (whi < kLowKey) whi = kLowKey;
    if (whi == 0x7fffffffu) whi = 0x80000000u;
    // 2. one pass: what is above the window stays, what is in it is marked. As
    // floats; NaN (key 1) is below every window but an open one.
    const bool open = wlo <= 1u;
    const float vlo = open ? -INFINITY : key_value(wlo);
    const float vhi = key_value(whi);
    // One compute unit's instructions bound the pass, so a wave takes 64 words in a
    // row: loads at fixed offsets, two comparisons, and the masks into the lanes of
    // a register.  (Words past the last may be marked.)
    const int w1 = __builtin_amdgcn_readfirstlane(wid);
    const uint32_t end = static_cast<uint32_t>(n - 1);
    const auto pass = [&](auto both) {   // both ends of the window, or the lower alone
      for (int s = w1; s * 64 < words; s += EW) {
        uint32_t k0 = 0u, k1 = 0u, i0 = 0u, i1 = 0u;
        const auto mark = [&](const float (&x)[kEvictRound], int b) {
#pragma unroll
          for (int u = 0; u < kEvictRound; ++u) {
            const uint64_t ws = __ballot(x[u] >= vlo);
            const int to = b * kEvictRound + u;
            i0 = lane == to ? static_cast<uint32_t>(ws) : i0;
            i1 = lane == to ? static_cast<uint32_t>(ws >> 32) : i1;
            if constexpr (decltype(both)::value) {
              const uint64_t ks = __ballot(x[u] > vhi);
              k0 = lane == to ? static_cast<uint32_t>(ks) : k0;
              k1 = lane == to ? static_cast<uint32_t>(ks >> 32) : k1;
            }
          }
        };
        constexpr int rounds = 64 / kEvictRound;
        float x[2][kEvictRound];
        if (static_cast<int64_t>(s + 1) * 4096 <= n) {
          const float* from = row.acc + static_cast<int64_t>(s) * 4096 + lane;
          const auto fetch = [&](float (&y)[kEvictRound], int b) {
#pragma unroll
            for (int u = 0; u < kEvictRound; ++u) y[u] = from[(b * kEvictRound + u) * 64];
          };
          fetch(x[0], 0);
#pragma unroll
          for (int b = 0; b < rounds; ++b) {
            if (b + 1 < rounds) fetch(x[(b + 1) % 2], b + 1);
            mark(x[b % 2], b);
          }
        } else {
#pragma unroll 1
          for (int b = 0; b < rounds; ++b) {
#pragma unroll
            for (int u = 0; u < kEvictRound; ++u) {
              const uint32_t i = static_cast<uint32_t>(s * 64 + b * kEvictRound + u) * 64u + static_cast<uint32_t>(lane);
              x[0][u] = row.acc[i < end ? i : end];
            }
            mark(x[0], b);
          }
        }
        keep[s * 64 + lane] = (static_cast<uint64_t>(k1) << 32) | k0;
        window[s * 64 + lane] = open ? ~0ull : (static_cast<uint64_t>(i1) << 32) | i0;
      }
    };
    if (top) pass(std::true_type{});
    else pass(std::false_type{});
    if (row.pos) __syncthreads();   // (other waves' words)
    if (row.pos)   // by their positions: what always stays, and what is there
      for (int w0 = w1; w0 < words; w0 += EW * kEvictRound) {
        int32_t ps[kEvictRound];
#pragma unroll
        for (int u = 0; u < kEvictRound; ++u) {
          const uint32_t i = static_cast<uint32_t>(w0 + u * EW) * 64u + static_cast<uint32_t>(lane);
          ps[u] = row.pos[i < end ? i : end];
        }
#pragma unroll
        for (int u = 0; u < kEvictRound; ++u) {
          const uint64_t there = __ballot(ps[u] >= 0);
          const uint64_t stays = __ballot(ps[u] < row.sink || ps[u] >= row.first_old);
          if (lane == 0 && w0 + u * EW < words) {
            keep[w0 + u * EW] = (keep[w0 + u * EW] | stays) & there;
            window[w0 + u * EW] &= there;
          }
        }
      }
    __syncthreads();
    // 3. the window's entries, in order
    constexpr int WPT = kEvictWords / ET;
    const int per = (words + ET - 1) / ET;   // words a thread takes, consecutive ones
    const auto from = [](int64_t first) -> uint64_t {   // bits `first` on
      return first <= 0 ? ~0ull : (first >= 64 ? 0ull : ~0ull << first);
    };
    uint32_t nk = 0u, nw = 0u;
#pragma unroll
    for (int q = 0; q < WPT; ++q) {
      const int w = tid * per + q;
      if (q < per && w < words) {
        const int64_t s0 = static_cast<int64_t>(w) * 64;
        uint64_t ks = keep[w];
        if (!row.pos) ks |= ~from(row.sink - s0) | from(row.first_old - s0);
        ks &= ~from(n - s0);
        const uint64_t ws = window[w] & ~from(n - s0) & ~ks;
        keep[w] = ks;
        window[w] = ws;
        nk += static_cast<uint32_t>(__popcll(ks));
        nw += static_cast<uint32_t>(__popcll(ws));
      }
    }
    const uint32_t sure = block.sum(nk);
    uint32_t found;
    uint32_t at = block.incl(nw, &found) - nw;
    const uint32_t want = budget - sure;
    done = sure <= budget && want <= found && found <= kEvictList;
    if (done && want > 0u) {
#pragma unroll
      for (int q = 0; q < WPT; ++q) {
        const int w = tid * per + q;
        if (q < per && w < words) {
          uint64_t bits = window[w];
          while (bits) {
            list_at[at++] = w * 64 + __ffsll(static_cast<unsigned long long>(bits)) - 1;
            bits &= bits - 1;
          }
        }
      }
      __syncthreads();
      constexpr int LPT = kEvictList / ET;
      uint32_t key[LPT];
#pragma unroll
      for (int i = 0; i < LPT; ++i) {
        const uint32_t j = i * ET + tid;
        key[i] = j < found ? row.key(list_at[j]) : 0u;
      }
      const auto each = [&](auto&& f) {
#pragma unroll
        for (int i = 0; i < LPT; ++i) f(key[i]);
      };
      // (the window as it was asked for; a lower end at 1 leaves out no entry)
      uint32_t last, equal;
      block.kth(each, want, wlo > 1u ? wlo : 1u, whi, &last, &equal);
      uint32_t eq = 0u;
      each([&](uint32_t v) { eq += v == last ? 1u : 0u; });
      if (block.sum(eq) == equal) {
#pragma unroll
        for (int i = 0; i < LPT; ++i)
          if (key[i] >= last) {
            const int32_t s = list_at[i * ET + tid];
            atomicOr(reinterpret_cast<uint32_t*>(keep) + s / 32, 1u << (s % 32));
          }
      } else {   // the first of the equal ones
        uint32_t before = 0u;
#pragma unroll
        for (int i = 0; i < LPT; ++i) {
          const bool is = key[i] == last;
          uint32_t all;
          const uint32_t rank = before + block.incl(is ? 1u : 0u, &all) - (is ? 1u : 0u);
          before += all;
          if (key[i] > last || (is && rank < equal)) {
            const int32_t s = list_at[i * ET + tid];
            atomicOr(reinterpret_cast<uint32_t*>(keep) + s / 32, 1u << (s % 32));
          }
        }
      }
    }
    __syncthreads();
    if (done) {
      // 4. the slots
      uint32_t c = 0u, all;
#pragma unroll
      for (int q = 0; q < WPT; ++q) {
        const int w = tid * per + q;
        if (q < per && w < words) c += static_cast<uint32_t>(__popcll(keep[w]));
      }
      uint32_t out = block.incl(c, &all) - c;
#pragma unroll
      for (int q = 0; q < WPT; ++q) {
        const int w = tid * per + q;
        if (q < per && w < words) {
          uint64_t bits = keep[w];
          while (bits) {
            slots[out++] = w * 64 + __ffsll(static_cast<unsigned long long>(bits)) - 1;
            bits &= bits - 1;
          }
        }
      }
      for (int64_t j = static_cast<int64_t>(all) + tid; j < a.budget; j += ET) slots[j] = -1;
      return;
    }
  }
  // every digit by a pass over the row, and one more for the slots, a wave's part
  // of the row consecutive
  __syncthreads();
  block.start();
  uint32_t last, want;
  block.last_key([&](auto&& f) {
    for (int64_t i = tid; i < n; i += ET) f(row.key(i));
  }, budget, &last, &want);
  const int64_t part = (n + 64 * EW - 1) / (64 * EW) * 64;
  const int64_t i0 = wid * part, i1 = i0 + part < n ? i0 + part : n;
  uint32_t gt = 0u, eq = 0u;
  for (int64_t i = i0 + lane; i < i1; i += kWave) {
    const uint32_t k = row.key(i);
    gt += k > last ? 1u : 0u;
    eq += k == last && k != 0u ? 1u : 0u;
  }
  gt = wave_sum(gt);
  eq = wave_sum(eq);
  __shared__ uint32_t wgt[EW], weq[EW];
  if (lane == 0) {
    wgt[wid] = gt;
    weq[wid] = eq;
  }
  __syncthreads();
  uint32_t g = 0u, e = 0u, all_g = 0u, all_e = 0u;
  for (int w = 0; w < EW; ++w) {
    if (w < wid) {
      g += wgt[w];
      e += weq[w];
    }
    all_g += wgt[w];
    all_e += weq[w];
  }
  const uint64_t below = (1ull << lane) - 1ull;
  for (int64_t j = i0; j < i1; j += kWave) {
    const int64_t i = j + lane;
    const uint32_t k = i < i1 ? row.key(i) : 0u;
    const uint64_t mg = __ballot(k > last), me = __ballot(k == last && k != 0u);
    const uint32_t er = e + static_cast<uint32_t>(__popcll(me & below));
    const uint32_t at = g + static_cast<uint32_t>(__popcll(mg & below)) + (er < want ? er : want);
    if (k > last || (k == last && k != 0u && er < want)) slots[at] = static_cast<int32_t>(i);
    g += static_cast<uint32_t>(__popcll(mg));
    e += static_cast<uint32_t>(__popcll(me));
  }
  const int64_t kept = static_cast<int64_t>(all_g) + (all_e < want ? all_e : want);
  for (int64_t j = kept + tid; j < a.budget; j += ET) slots[j] = -1;
}

// Rows of K and V, acc and positions of the kept slots: a team of `team` lanes
// copies a row of each, in vectors.  Bound: memory (96 x 1024 rows of 192
// bytes, twice: 75 MB in 17 us, 4.4 TB/s; 8 x 4096 of 256 bytes 9.4 us).
template <typename Vec>
__global__ __launch_bounds__(256) void cache_gather_kernel(EvictArgs a) {
  const int team = a.team;
  const int l = threadIdx.x % team;
  const int64_t per = 256 / team;
  const int64_t rows = a.batch * a.kv * a.budget;
  for (int64_t j = blockIdx.x * per + threadIdx.x / team; j < rows; j += gridDim.x * per) {
    const int64_t bh = j / a.budget;
    const int64_t b = bh / a.kv, h = bh - b * a.kv;
    const int64_t slot = a.slots[j];
    const int64_t from = slot < 0 ? 0 : slot;
    const Vec* k = static_cast<const Vec*>(a.k) + b * a.k_b + h * a.k_h + from * a.k_s;
    const Vec* v = static_cast<const Vec*>(a.v) + b * a.v_b + h * a.v_h + from * a.v_s;
    Vec* ko = static_cast<Vec*>(a.k_out) + j * a.row;
    Vec* vo = static_cast<Vec*>(a.v_out) + j * a.row;
    for (int c = l; c < a.row; c += team) {
      Vec x{}, y{};
      if (slot >= 0) {
        x = k[c];
        y = v[c];
      }
      ko[c] = x;
      vo[c] = y;
    }
    if (l == 0) {
      const int64_t at = bh * a.room + from;
      a.acc_out[j] = slot < 0 ? 0.0f : a.acc[at];
      a.pos_out[j] = slot < 0 || !a.pos ? static_cast<int32_t>(slot) : a.pos[at];
    }
  }
}

// ------------------------------------------------------------------ step ---
// One workgroup per (sequence, head): its row of sums stays in registers
// between the addition and the choice, so one launch and one pass do both.
// Bound: the read of the weights where there are many rows (512 of 4096 slots,
// 8 heads each: 59 MB in 12 to 13 us, 4.7 TB/s), else the launch (8 rows of
// 2048: 4.8 us).
template <int DT, int T>
__global__ __launch_bounds__(T) void cache_step_kernel(StepArgs a) {
  using raw = typename Elem<DT>::raw;
  constexpr int NW = T / kWave;
  constexpr int VE = 4;
  constexpr int U = 8;   // rows of weights in flight
  __shared__ uint64_t least[NW];
  const int tid = threadIdx.x;
  const int64_t bh = blockIdx.x;
  const int64_t b = bh / a.kv, h = bh - b * a.kv;
  float* acc = a.acc + bh * a.room;
  int32_t* pos = a.pos + bh * a.room;
  const int32_t now = a.seen[b];
  const int32_t first_old = now - a.recent + 1;   // the new token is one of `recent`
  const raw* w = static_cast<const raw*>(a.weights) + b * a.stride_b + h * a.group * a.stride_h;
  uint64_t best = ~0ull;
  for (int64_t s = static_cast<int64_t>(tid) * VE; s < a.room; s += T * VE) {
    const int live = a.room - s < VE ? static_cast<int>(a.room - s) : VE;
    float o[VE];
    int32_t p[VE];
    if (live == VE) {
      __builtin_memcpy(o, acc + s, sizeof(o));
      __builtin_memcpy(p, pos + s, sizeof(p));
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        o[j] = j < live ? acc[s + j] : 0.0f;
        p[j] = j < live ? pos[s + j] : -1;
      }
    }
    double t[VE] = {};
    for (int g0 = 0; g0 < a.group; g0 += U) {
      raw x[U][VE];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        // (past the last head its row again, left out below)
        const int g = g0 + u < a.group ? g0 + u : static_cast<int>(a.group) - 1;
        const raw* wp = w + g * a.stride_h + s;
        if (live == VE) {
          __builtin_memcpy(x[u], wp, sizeof(x[u]));
        } else {
#pragma unroll
          for (int j = 0; j < VE; ++j) x[u][j] = j < live ? wp[j] : raw(0);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g0 + u < a.group) {
#pragma unroll
          for (int j = 0; j < VE; ++j) t[j] += static_cast<double>(Elem<DT>::get(x[u][j]));
        }
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      if (p[j] >= 0) o[j] = static_cast<float>(static_cast<double>(o[j]) + t[j]);
      const uint64_t k = (static_cast<uint64_t>(stay_key(o[j], p[j], first_old, a.sink)) << 32) |
                         static_cast<uint64_t>(s + j);
      if (j < live && k < best) best = k;
    }
    if (live == VE) {
      __builtin_memcpy(acc + s, o, sizeof(o));
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j)
        if (j < live) acc[s + j] = o[j];
    }
  }
  best = wave_min(best, static_cast<uint64_t>(~0ull));
  if (lane_id() == 0) least[tid / kWave] = best;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < NW; ++q) best = least[q] < best ? least[q] : best;
  const int64_t slot = static_cast<int64_t>(best & 0xffffffffull);
  // (every acc of the row has been stored)
  char* k = static_cast<char*>(a.k) + b * a.k_b + h * a.k_h + slot * a.k_s;
  char* v = static_cast<char*>(a.v) + b * a.v_b + h * a.v_h + slot * a.v_s;
  const char* k1 = static_cast<const char*>(a.k_new) + bh * a.row;
  const char* v1 = static_cast<const char*>(a.v_new) + bh * a.row;
  if (a.words) {
    for (int64_t c = tid; c < a.row / 4; c += T) {
      reinterpret_cast<uint32_t*>(k)[c] = reinterpret_cast<const uint32_t*>(k1)[c];
      reinterpret_cast<uint32_t*>(v)[c] = reinterpret_cast<const uint32_t*>(v1)[c];
    }
  } else {
    for (int64_t c = tid; c < a.row; c += T) {
      k[c] = k1[c];
      v[c] = v1[c];
    }
  }
  if (tid == 0) {
    acc[slot] = 0.0f;
    pos[slot] = now;
    a.slot[bh] = static_cast<int32_t>(slot);
  }
}

// ------------------------------------------------------------- launchers ---
hipError_t launch_cache_accumulate(AccumulateArgs a, int dtype, hipStream_t s) {
  const int64_t cols = kWave * (dtype == 0 ? 4 : 8);
  a.tiles = (a.keys + cols - 1) / cols;
  const dim3 grid(static_cast<unsigned>(a.tiles * a.batch * a.kv));
  // with fewer workgroups than compute units a workgroup's waves are the only ones
  // that share the rows: sixteen of them
  const bool few = a.tiles * a.batch * a.kv < 256 && a.group * a.queries > 32;
  ProfScope ps_("cache_accumulate", s);
  const auto launch = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (few) hipLaunchKernelGGL((cache_accumulate_kernel<DT, 1024>), grid, dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((cache_accumulate_kernel<DT, 256>), grid, dim3(256), 0, s, a);
  };
  if (dtype == 0) launch(std::integral_constant<int, 0>{});
  else if (dtype == 1) launch(std::integral_constant<int, 1>{});
  else launch(std::integral_constant<int, 2>{});
  return hipGetLastError();
}

// Sizes and strides of K and V in vectors of `width` bytes.
hipError_t launch_cache_evict(EvictArgs a, int width, hipStream_t s) {
  const dim3 rows(static_cast<unsigned>(a.batch * a.kv));
  { ProfScope ps_("cache_select", s);
  if (a.room <= 1024) hipLaunchKernelGGL((cache_select_kernel<256, 4>), rows, dim3(256), 0, s, a);
  else if (a.room <= 4096) hipLaunchKernelGGL((cache_select_kernel<512, 8>), rows, dim3(512), 0, s, a);
  else if (a.room <= 8192) hipLaunchKernelGGL((cache_select_kernel<1024, 8>), rows, dim3(1024), 0, s, a);
  else if (a.room <= 32768) hipLaunchKernelGGL((cache_select_kernel<1024, 32>), rows, dim3(1024), 0, s, a);
  else hipLaunchKernelGGL(cache_select_long_kernel, rows, dim3(ET), 0, s, a); }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.team = 1;
  while (a.team < a.row && a.team < 64) a.team *= 2;
  const int64_t per = 256 / a.team;
  const int64_t want = (a.batch * a.kv * a.budget + per - 1) / per;
  const dim3 grid(static_cast<unsigned>(want < (int64_t(1) << 20) ? want : (int64_t(1) << 20)));
  { ProfScope ps_("cache_gather", s);
  if (width == 16) hipLaunchKernelGGL((cache_gather_kernel<Move16>), grid, dim3(256), 0, s, a);
  else if (width == 8) hipLaunchKernelGGL((cache_gather_kernel<Move8>), grid, dim3(256), 0, s, a);
  else if (width == 4) hipLaunchKernelGGL((cache_gather_kernel<uint32_t>), grid, dim3(256), 0, s, a);
  else if (width == 2) hipLaunchKernelGGL((cache_gather_kernel<uint16_t>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((cache_gather_kernel<uint8_t>), grid, dim3(256), 0, s, a); }
  return hipGetLastError();
}

hipError_t launch_cache_step(const StepArgs& a, int dtype, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.batch * a.kv));
  ProfScope ps_("cache_step", s);
  const auto launch = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    // 512 rows of 4096 slots, 8 heads each: 512 threads with eight rows of weights
    // in flight 11.9 us, 256 threads 14.9, 1024 14.4; eight slots a thread 15.2
    if (a.room <= 1024) hipLaunchKernelGGL((cache_step_kernel<DT, 256>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cache_step_kernel<DT, 512>), grid, dim3(512), 0, s, a);
  };
  if (dtype == 0) launch(std::integral_constant<int, 0>{});
  else if (dtype == 1) launch(std::integral_constant<int, 1>{});
  else launch(std::integral_constant<int, 2>{});
  return hipGetLastError();
}

}  // namespace lapsum
