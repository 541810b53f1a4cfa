// Experts' rows: the order of the places (token, slot) by the expert that a
// router chose for them, and the weighted sum of the experts' outputs back to
// tokens with its gradient.
//
// Order.  A stable counting sort of small whole numbers.  Every wave owns a run
// of consecutive places; it counts its run by expert in LDS, the counts of the
// runs before it give its first position for each expert, and a second walk over the
// run hands positions out, 64 places at a time: a place's rank among
// the 64 is the number of lower lanes with its expert, from one ballot per bit of
// the expert's number.  Counts are whole numbers, so atomics' order changes
// nothing.  Places without an expert are those of one expert more, so they come
// last.
//
// 131072 places of 128 experts take 17 us in two launches, 64 places of 64 2.9 in one:
// chains of loads, counts and ballots.
//
// Sum.  out_t = sum_j w_tj y_row(t, j): a gather of rows, without atomics, in the order
// of the slots.  Backward: dy_row(t, j) = w_tj g_t and dw_tj = <g_t, y_row(t, j)>
// from one read of g_t and y.  Both are bound by memory: 16384 tokens of 8 rows of 2048
// in bfloat16 take 140 us (4.3 TB/s) and 214 us (5.3 TB/s).
#include "select_common.hpp"

namespace lapsum {
namespace {

constexpr int OW = 8;                  // waves of a workgroup of the order
constexpr int OT = OW * kWave;

__device__ __forceinline__ int bin_of(const int32_t* indices, int64_t i, int experts) {
  const int e = indices[i];
  return e >= 0 && e < experts ? e : experts;
}

// parts[block][experts + 1]: places per expert of each workgroup's run.
__global__ __launch_bounds__(OT) void expert_count_kernel(OrderArgs a) {
  extern __shared__ int lds[];
  const int bins = a.experts + 1;
  for (int e = threadIdx.x; e < bins; e += OT) lds[e] = 0;
  __syncthreads();
  const int64_t lo = static_cast<int64_t>(blockIdx.x) * a.run;
  const int64_t hi = lo + a.run < a.count ? lo + a.run : a.count;
  for (int64_t i = lo + threadIdx.x; i < hi; i += OT) atomicAdd(&lds[bin_of(a.indices, i, a.experts)], 1);
  __syncthreads();
  for (int e = threadIdx.x; e < bins; e += OT) a.parts[static_cast<int64_t>(blockIdx.x) * bins + e] = lds[e];
}

// LDS: [OW][bins] counts of the waves' runs, then their positions; with several
// workgroups [bins] totals and [bins] counts of the workgroups before.
__global__ __launch_bounds__(OT) void expert_order_kernel(OrderArgs a) {
  extern __shared__ int lds[];
  const int bins = a.experts + 1, blocks = gridDim.x;
  const int wave = threadIdx.x / kWave, lane = lane_id();
  int* mine = lds + wave * bins;
  int* total = lds + OW * bins;
  int* before = total + bins;
  for (int e = threadIdx.x; e < (OW + 2) * bins; e += OT) lds[e] = 0;
  __syncthreads();
  const int64_t run = a.run / OW;
  const int64_t lo = (static_cast<int64_t>(blockIdx.x) * OW + wave) * run;
  const int64_t hi = lo + run < a.count ? lo + run : a.count;
  for (int64_t i = lo + lane; i < hi; i += kWave) atomicAdd(&mine[bin_of(a.indices, i, a.experts)], 1);
  if (blocks > 1) {
    // (consecutive threads take consecutive experts, the rest of them other workgroups)
    const int teams = OT / bins > 0 ? OT / bins : 1;
    const int team = threadIdx.x / bins;
    if (teams > 1 ? team < teams : true) {
      for (int e = teams > 1 ? threadIdx.x % bins : threadIdx.x; e < bins; e += teams > 1 ? bins : OT) {
        int all = 0, ahead = 0;
        for (int b = teams > 1 ? team : 0; b < blocks; b += teams) {
          const int c = a.parts[static_cast<int64_t>(b) * bins + e];
          all += c;
          ahead += b < static_cast<int>(blockIdx.x) ? c : 0;
        }
        atomicAdd(&total[e], all);
        atomicAdd(&before[e], ahead);
      }
    }
  }
  __syncthreads();
  // each expert's first position in the order; each wave's from it
  if (wave == 0) {
    int carry = 0;
    for (int e0 = 0; e0 < bins; e0 += kWave) {
      const int e = e0 + lane;
      int c = 0;
      if (e < bins) {
        if (blocks > 1) c = total[e];
        else for (int w = 0; w < OW; ++w) c += lds[w * bins + e];
      }
      const int end = carry + wave_incl_add(c);
      if (e < bins) {
        if (blockIdx.x == 0) a.offsets[e] = end - c;   // (of the last bin: the end of the others)
        int at = end - c + (blocks > 1 ? before[e] : 0);
        for (int w = 0; w < OW; ++w) {
          const int n = lds[w * bins + e];
          lds[w * bins + e] = at;
          at += n;
        }
      }
      carry = __builtin_amdgcn_readlane(end, kWave - 1);
    }
  }
  __syncthreads();
  const int bits = 32 - __clz(a.experts);
  for (int64_t i0 = lo; i0 < hi; i0 += kWave) {
    const int64_t i = i0 + lane;
    const bool here = i < hi;
    const int e = here ? bin_of(a.indices, i, a.experts) : 0;
    uint64_t same = __ballot(here);
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot((e >> b) & 1);
      same &= (e >> b) & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((uint64_t(1) << lane) - 1));
    int at = 0;
    if (here) at = mine[e] + rank;
    wave_lds_sync();
    // (the last of the expert's lanes knows how many there are)
    if (here && (same >> lane) == 1) mine[e] = at + 1;
    wave_lds_sync();
    if (here) {
      a.order[at] = static_cast<int32_t>(i);
      a.place[i] = e < a.experts ? at : -1;
    }
  }
}

// ------------------------------------------------------------------ sum ----
// N elements of a row from column c0, as floats; the columns past dim are 0.
template <int DT, int N, bool VEC>
__device__ __forceinline__ void load_row(const void* p, int64_t at, int left, float (&x)[N]) {
  using raw = typename Elem<DT>::raw;
  const raw* q = static_cast<const raw*>(p) + at;
  if constexpr (VEC) {
    if constexpr (DT == 0) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const Move16 v = *reinterpret_cast<const Move16*>(q + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i + j] = __uint_as_float(v[j]);
      }
    } else {
      static_assert(N == 8, "one vector");
      const Move16 v = *reinterpret_cast<const Move16*>(q);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = Elem<DT>::get(v[j] & 0xffffu);
        x[2 * j + 1] = Elem<DT>::get(v[j] >> 16);
      }
    }
  } else if (left == N) {
    // (global memory serves vectors at any alignment of their elements)
    struct __attribute__((packed, aligned(sizeof(raw)))) Any {
      uint32_t w[N * sizeof(raw) / 4];
    };
    const Any v = *reinterpret_cast<const Any*>(q);
#pragma unroll
    for (int j = 0; j < N; ++j)
      x[j] = DT == 0 ? __uint_as_float(v.w[j % (N * sizeof(raw) / 4)])
                     : Elem<DT>::get((v.w[j / 2] >> (16 * (j % 2))) & 0xffffu);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = j < left ? Elem<DT>::get(q[j]) : 0.0f;
  }
}
template <int DT, int N, bool VEC>
__device__ __forceinline__ void store_row(void* p, int64_t at, int left, const float (&x)[N]) {
  using raw = typename Elem<DT>::raw;
  raw* q = static_cast<raw*>(p) + at;
  if constexpr (VEC) {
    if constexpr (DT == 0) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
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
  } else if (left == N) {
    struct __attribute__((packed, aligned(sizeof(raw)))) Any {
      uint32_t w[N * sizeof(raw) / 4];
    };
    Any v;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (DT == 0) v.w[j] = __float_as_uint(x[j]);
      else if (j % 2 == 0) v.w[j / 2] = Elem<DT>::put(x[j]);
      else v.w[j / 2] |= static_cast<uint32_t>(Elem<DT>::put(x[j])) << 16;
    }
    *reinterpret_cast<Any*>(q) = v;
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < left) q[j] = Elem<DT>::put(x[j]);
  }
}

// Eight columns to a lane, a wave to 512 columns of a token.
constexpr int CN = 8;
constexpr int CW = CN * kWave;

// y of type DT, out of type DO; weights null: 1 each.
template <int DT, int DO, bool VEC>
__global__ __launch_bounds__(256) void expert_combine_kernel(CombineArgs a) {
  const int64_t items = a.tokens * a.pieces;
  for (int64_t item = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / kWave; item < items;
       item += static_cast<int64_t>(gridDim.x) * (256 / kWave)) {
    const int64_t t = item / a.pieces;
    const int64_t c = (item - t * a.pieces) * CW + lane_id() * CN;
    if (c >= a.dim) continue;
    const int left = static_cast<int>(a.dim - c < CN ? a.dim - c : CN);
    float sum[CN] = {};
#pragma unroll 4
    for (int j = 0; j < a.top_k; ++j) {
      const int32_t row = a.place[t * a.top_k + j];
      if (row < 0 || row >= a.rows) continue;
      const float w = a.weights ? a.weights[t * a.top_k + j] : 1.0f;
      float y[CN];
      load_row<DT, CN, VEC>(a.y, row * a.dim + c, left, y);
#pragma unroll
      for (int i = 0; i < CN; ++i) sum[i] = fmaf(w, y[i], sum[i]);
    }
    store_row<DO, CN, VEC>(a.out, t * a.dim + c, left, sum);
  }
}

// A wave to a token: g in registers where the row has at most NC pieces.
template <int DT, int NC, bool VEC>
__global__ __launch_bounds__(256) void expert_combine_backward_kernel(CombineGradArgs a) {
  const int lane = lane_id();
  const int64_t waves = static_cast<int64_t>(gridDim.x) * (256 / kWave);
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / kWave;
  for (int64_t t = first; t < a.tokens; t += waves) {
    for (int64_t c0 = 0; c0 < a.dim; c0 += NC * CW) {
      float g[NC][CN];
      int left[NC];
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        const int64_t c = c0 + n * CW + lane * CN;
        left[n] = c >= a.dim ? 0 : static_cast<int>(a.dim - c < CN ? a.dim - c : CN);
        if (left[n]) load_row<DT, CN, VEC>(a.grad, t * a.dim + c, left[n], g[n]);
      }
      for (int j = 0; j < a.top_k; ++j) {
        const int64_t at = t * a.top_k + j;
        const int32_t row = a.place[at];
        if (row < 0 || row >= a.rows) {
          if (lane == 0 && c0 == 0) a.grad_weights[at] = 0.0f;
          continue;
        }
        const float w = a.weights[at];
        float dot = 0.0f;
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          if (!left[n]) continue;
          const int64_t c = row * a.dim + c0 + n * CW + lane * CN;
          float y[CN];
          load_row<DT, CN, VEC>(a.y, c, left[n], y);
#pragma unroll
          for (int i = 0; i < CN; ++i)
            if (VEC || i < left[n]) dot = fmaf(g[n][i], y[i], dot);
#pragma unroll
          for (int i = 0; i < CN; ++i) y[i] = w * g[n][i];
          store_row<DT, CN, VEC>(a.grad_y, c, left[n], y);
        }
        dot = team_sum<kWave>(dot);
        if (lane == 0) a.grad_weights[at] = c0 == 0 ? dot : a.grad_weights[at] + dot;
      }
    }
  }
  // rows that are no token's
  const int32_t end = a.ends[a.experts];
  const int64_t from = end < 0 ? 0 : end;
  for (int64_t r = from + first; r < a.rows; r += waves) {
    const float zero[CN] = {};
    for (int64_t c = lane * CN; c < a.dim; c += CW)
      store_row<DT, CN, VEC>(a.grad_y, r * a.dim + c, static_cast<int>(a.dim - c < CN ? a.dim - c : CN), zero);
  }
}

}  // namespace

// ------------------------------------------------------------- launchers ---
// One workgroup up to 8192 places, which is one launch less; else 2048 places to one,
// more where that would be more than 256 of them: each reads all others' counts.
int64_t order_run(int64_t count) {
  const int64_t want = count <= 16 * OT ? count : (count + 255) / 256;
  const int64_t least = count <= 16 * OT ? OT : 4 * OT;
  return (want < least ? least : want + OT - 1) / OT * OT;
}
int64_t order_blocks(int64_t count) {
  const int64_t run = order_run(count);
  return (count + run - 1) / run;
}

hipError_t launch_expert_order(OrderArgs a, hipStream_t s) {
  const unsigned blocks = static_cast<unsigned>(order_blocks(a.count));
  a.run = order_run(a.count);
  const size_t bins = static_cast<size_t>(a.experts) + 1;
  if (blocks > 1) {
    ProfScope ps_("expert_count", s);
    hipLaunchKernelGGL(expert_count_kernel, dim3(blocks), dim3(OT), bins * sizeof(int), s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  ProfScope ps_("expert_order", s);
  hipLaunchKernelGGL(expert_order_kernel, dim3(blocks), dim3(OT), (OW + 2) * bins * sizeof(int), s, a);
  return hipGetLastError();
}

hipError_t launch_expert_combine(CombineArgs a, int dtype, int out_dtype, bool vec, hipStream_t s) {
  a.pieces = (a.dim + CW - 1) / CW;
  const int64_t want = (a.tokens * a.pieces + 3) / 4;
  const dim3 grid(static_cast<unsigned>(want < (int64_t(1) << 20) ? want : (int64_t(1) << 20)));
  ProfScope ps_("expert_combine", s);
  const auto launch = [&](auto dt, auto dout) {
    constexpr int DT = decltype(dt)::value, DO = decltype(dout)::value;
    if (vec) hipLaunchKernelGGL((expert_combine_kernel<DT, DO, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((expert_combine_kernel<DT, DO, false>), grid, dim3(256), 0, s, a);
  };
  const std::integral_constant<int, 0> f32;
  const std::integral_constant<int, 1> b16;
  const std::integral_constant<int, 2> h16;
  if (dtype == 0 && out_dtype == 0) launch(f32, f32);
  else if (dtype == 0 && out_dtype == 1) launch(f32, b16);
  else if (dtype == 0) launch(f32, h16);
  else if (dtype == 1) launch(b16, b16);
  else launch(h16, h16);
  return hipGetLastError();
}

hipError_t launch_expert_combine_backward(const CombineGradArgs& a, int dtype, bool vec, hipStream_t s) {
  const int64_t most = a.tokens > a.rows ? a.tokens : a.rows;
  const int64_t want = ((a.tokens > 0 ? a.tokens : most) + 3) / 4;
  const dim3 grid(static_cast<unsigned>(want < (int64_t(1) << 20) ? want : (int64_t(1) << 20)));
  ProfScope ps_("expert_combine_backward", s);
  const auto launch = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (!vec && a.dim <= CW)
      hipLaunchKernelGGL((expert_combine_backward_kernel<DT, 1, false>), grid, dim3(256), 0, s, a);
    else if (!vec) hipLaunchKernelGGL((expert_combine_backward_kernel<DT, 4, false>), grid, dim3(256), 0, s, a);
    else if (a.dim <= CW) hipLaunchKernelGGL((expert_combine_backward_kernel<DT, 1, true>), grid, dim3(256), 0, s, a);
    else if (a.dim <= 2 * CW) hipLaunchKernelGGL((expert_combine_backward_kernel<DT, 2, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((expert_combine_backward_kernel<DT, 4, true>), grid, dim3(256), 0, s, a);
  };
  if (dtype == 0) launch(std::integral_constant<int, 0>{});
  else if (dtype == 1) launch(std::integral_constant<int, 1>{});
  else launch(std::integral_constant<int, 2>{});
  return hipGetLastError();
}

}  // namespace lapsum
