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
// Selection key of an entry (uint32, larger stays longer): empty 0, NaN 1,
// then the float's order, and the largest for what always stays.
#include "select_common.hpp"

namespace lapsum {

namespace {
constexpr uint32_t kStays = 0xffffffffu;

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

// VE weights at p (their own alignment only), those from `live` on as 0.
template <int DT>
__device__ __forceinline__ void load_weights(const typename Elem<DT>::raw* __restrict__ p, int live,
                                             float* x) {
  constexpr int VE = Wide<DT>::VE;
  if (live >= VE) {
    uint32_t w[4];
    __builtin_memcpy(w, p, 16);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (DT == 0) {
        x[q] = Elem<0>::get(w[q]);
      } else {
        x[2 * q] = Elem<DT>::get(w[q] & 0xffffu);
        x[2 * q + 1] = Elem<DT>::get(w[q] >> 16);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j) x[j] = j < live ? Elem<DT>::get(p[j]) : 0.0f;
  }
}
}  // namespace

// ------------------------------------------------------------ accumulate ---
// A workgroup takes 64 VE columns of one (sequence, head); its waves take the
// rows of weights (query heads x queries) in turn.
constexpr int AT = 256;
constexpr int AW = AT / kWave;

template <int DT>
__global__ __launch_bounds__(AT) void cache_accumulate_kernel(AccumulateArgs a) {
  using raw = typename Elem<DT>::raw;
  constexpr int VE = Wide<DT>::VE;
  constexpr int U = 4;   // rows in flight per lane
  __shared__ double part[AW - 1][kWave][VE + 1];
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
  const int64_t rows = a.group * a.queries;
  if (live > 0) {
    for (int64_t r0 = wid; r0 < rows; r0 += AW * U) {
      float x[U][VE];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * AW;
        if (r < rows) {
          const int64_t g = r / a.queries, q = r - g * a.queries;
          load_weights<DT>(base + g * a.stride_h + q * a.stride_q, live, x[u]);
        } else {
#pragma unroll
          for (int j = 0; j < VE; ++j) x[u][j] = 0.0f;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < VE; ++j) sum[j] += static_cast<double>(x[u][j]);
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
    for (int w = 0; w < AW - 1; ++w) t += part[w][lane][j];
    if (old) {
      const float o = old[j];
      acc[j] = j < live ? static_cast<float>(static_cast<double>(o) + t) : o;
    } else {
      acc[j] = j < live ? static_cast<float>(t) : 0.0f;
    }
  }
}

// ----------------------------------------------------------------- evict ---
// One workgroup per (sequence, head): the digits of the budget-th largest key
// (11, 11 and 10 bits) from histograms in LDS, then the kept slots in order.
constexpr int ET = 1024;
constexpr int EW = ET / kWave;
constexpr int kEvictBins = 2048;

namespace {
struct EvictSmem {
  uint32_t bins[kEvictBins];
  uint32_t wsum[EW];
  uint32_t digit, above, live;
  uint32_t wg[EW], we[EW];   // kept for sure, and equal to the last key, per wave
};
}  // namespace

__global__ __launch_bounds__(ET) void cache_select_kernel(EvictArgs a) {
  __shared__ EvictSmem sm;
  const int tid = threadIdx.x, lane = lane_id(), wid = tid / kWave;
  const int64_t bh = blockIdx.x;
  const int64_t b = bh / a.kv;
  const float* acc = a.acc + bh * a.room;
  const int32_t* pos = a.pos ? a.pos + bh * a.room : nullptr;
  const int32_t seen = a.seen[b] < 0 ? 0 : a.seen[b];
  const int32_t first_old = seen - a.recent > 0 ? seen - a.recent : 0;
  // (positions are the slots where none are given)
  const int64_t n = !pos && seen < a.room ? seen : a.room;
  auto key_of = [&](int64_t i) -> uint32_t {
    return stay_key(acc[i], pos ? pos[i] : static_cast<int32_t>(i), first_old, a.sink);
  };
  // digits from the top; want: entries still to be found among those that
  // share the digits so far
  uint32_t want = static_cast<uint32_t>(a.budget), prefix = 0u;
  bool all = false;   // no more live entries than the budget
  for (int p = 0; p < 3 && !all; ++p) {
    const int shift = p == 0 ? 21 : (p == 1 ? 10 : 0);
    const int upper = p == 0 ? 32 : (p == 1 ? 21 : 10);
    const uint32_t mask = p == 2 ? 1023u : 2047u;
    for (int e = tid; e < kEvictBins; e += ET) sm.bins[e] = 0u;
    if (tid == 0) sm.live = 0u;
    __syncthreads();
    uint32_t mine = 0u;
    for (int64_t i = tid; i < n; i += ET) {
      const uint32_t k = key_of(i);
      if (k != 0u && (p == 0 || (k >> (upper & 31)) == prefix)) {
        atomicAdd(&sm.bins[(k >> shift) & mask], 1u);
        ++mine;
      }
    }
    if (p == 0) {
      mine = wave_sum(mine);
      if (lane == 0) atomicAdd(&sm.live, mine);
    }
    __syncthreads();
    if (p == 0 && sm.live <= want) {
      all = true;
      break;
    }
    // the bin where the count from the largest key down reaches `want`
    const int hi = kEvictBins - 1 - 2 * tid;   // two bins a thread, downwards
    const uint32_t c0 = sm.bins[hi], c1 = sm.bins[hi - 1];
    const uint32_t incl = wave_incl_add<uint32_t>(c0 + c1);
    if (lane == kWave - 1) sm.wsum[wid] = incl;
    __syncthreads();
    uint32_t run = incl - c0 - c1;
#pragma unroll
    for (int w = 0; w < EW; ++w)
      if (w < wid) run += sm.wsum[w];
    if (run < want && want <= run + c0) {
      sm.digit = static_cast<uint32_t>(hi);
      sm.above = run;
    } else if (run + c0 < want && want <= run + c0 + c1) {
      sm.digit = static_cast<uint32_t>(hi - 1);
      sm.above = run + c0;
    }
    __syncthreads();
    want -= sm.above;
    prefix = (prefix << (p == 2 ? 10 : 11)) | sm.digit;
    __syncthreads();
  }
  // kept: above the last key, and the first `want` that equal it
  const uint32_t last = all ? 1u : prefix;
  if (all) want = 0xffffffffu;
  int32_t* slots = a.slots + bh * a.budget;
  uint32_t out = 0u, equal = 0u;   // kept, and equal ones seen, before this round
  const int64_t rounds = (n + ET - 1) / ET;
  for (int64_t q = 0; q < rounds; ++q) {
    const int64_t i = q * ET + tid;
    const uint32_t k = i < n ? key_of(i) : 0u;
    const uint64_t gt = __ballot(k > last), eq = __ballot(k == last && k != 0u);
    if (lane == 0) {
      sm.wg[wid] = static_cast<uint32_t>(__popcll(gt));
      sm.we[wid] = static_cast<uint32_t>(__popcll(eq));
    }
    __syncthreads();
    const uint64_t before = (1ull << lane) - 1ull;
    uint32_t g = static_cast<uint32_t>(__popcll(gt & before)), e = static_cast<uint32_t>(__popcll(eq & before));
    uint32_t tg = 0u, te = 0u;
#pragma unroll
    for (int w = 0; w < EW; ++w) {
      if (w < wid) {
        g += sm.wg[w];
        e += sm.we[w];
      }
      tg += sm.wg[w];
      te += sm.we[w];
    }
    // equal ones kept before this lane: at most `want` in all
    const uint32_t eb = equal + e < want ? equal + e : want;
    const uint32_t e0 = equal < want ? equal : want;
    const bool keep = k > last || (k == last && k != 0u && equal + e < want);
    const uint32_t at = out + g + (eb - e0);
    if (keep && at < static_cast<uint32_t>(a.budget)) slots[at] = static_cast<int32_t>(i);
    const uint32_t e1 = equal + te < want ? equal + te : want;
    out += tg + (e1 - e0);
    equal += te;
    __syncthreads();
  }
  for (int64_t j = out + tid; j < a.budget; j += ET) slots[j] = -1;
}

// Rows of K and V, acc and positions of the kept slots: a team of `team`
// lanes copies a row of each, in vectors.
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
// One workgroup per (sequence, head).
template <int DT, int T>
__global__ __launch_bounds__(T) void cache_step_kernel(StepArgs a) {
  using raw = typename Elem<DT>::raw;
  constexpr int NW = T / kWave;
  constexpr int VE = 4;
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
      __builtin_memcpy(o, acc + s, 16);
      __builtin_memcpy(p, pos + s, 16);
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        o[j] = j < live ? acc[s + j] : 0.0f;
        p[j] = j < live ? pos[s + j] : -1;
      }
    }
    double t[VE] = {0.0, 0.0, 0.0, 0.0};
    for (int64_t g = 0; g < a.group; ++g) {
      const raw* wp = w + g * a.stride_h + s;
      if (live == VE) {
        raw x[VE];
        __builtin_memcpy(x, wp, sizeof(x));
#pragma unroll
        for (int j = 0; j < VE; ++j) t[j] += static_cast<double>(Elem<DT>::get(x[j]));
      } else {
#pragma unroll
        for (int j = 0; j < VE; ++j)
          if (j < live) t[j] += static_cast<double>(Elem<DT>::get(wp[j]));
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
      __builtin_memcpy(acc + s, o, 16);
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
  ProfScope ps_("cache_accumulate", s);
  if (dtype == 0) hipLaunchKernelGGL((cache_accumulate_kernel<0>), grid, dim3(AT), 0, s, a);
  else if (dtype == 1) hipLaunchKernelGGL((cache_accumulate_kernel<1>), grid, dim3(AT), 0, s, a);
  else hipLaunchKernelGGL((cache_accumulate_kernel<2>), grid, dim3(AT), 0, s, a);
  return hipGetLastError();
}

// Sizes and strides of K and V in vectors of `width` bytes.
hipError_t launch_cache_evict(EvictArgs a, int width, hipStream_t s) {
  { ProfScope ps_("cache_select", s);
  hipLaunchKernelGGL(cache_select_kernel, dim3(static_cast<unsigned>(a.batch * a.kv)), dim3(ET), 0, s, a); }
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
  if (a.room <= 1024) {
    if (dtype == 0) hipLaunchKernelGGL((cache_step_kernel<0, 256>), grid, dim3(256), 0, s, a);
    else if (dtype == 1) hipLaunchKernelGGL((cache_step_kernel<1, 256>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cache_step_kernel<2, 256>), grid, dim3(256), 0, s, a);
  } else {
    if (dtype == 0) hipLaunchKernelGGL((cache_step_kernel<0, 512>), grid, dim3(512), 0, s, a);
    else if (dtype == 1) hipLaunchKernelGGL((cache_step_kernel<1, 512>), grid, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((cache_step_kernel<2, 512>), grid, dim3(512), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace lapsum
