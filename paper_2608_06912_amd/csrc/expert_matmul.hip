// Matrix products grouped by expert: the rows of each expert, consecutive after
// the order, times the expert's matrix; and the matrices' gradient, a product over
// each expert's rows.
//
//   rows   y[i][n] = sum_k x[row(i)][k] w_e[k][n],      offsets[e] <= i < offsets[e+1]
//   grad   c_e[m][n] = sum_i a[row(i)][m] b[row(i)][n], the same i
//
// The gradient of the rows is the first one with w read the other way round, so
// w may be dense along k or along n.  A workgroup computes a tile of 128 x 128
// results of one expert; which one it finds by itself from the offsets, as the
// host does not know them.
#include "matrix.hpp"

namespace lapsum {
namespace {

constexpr int BM = 128, BN = 128, PT = 256;

// The expert and the first row of the t-th tile of M rows, experts' tiles one
// after another, the rows of no expert last.
struct Tile {
  int expert;      // experts: rows of none; -1: no such tile
  int row, end;    // the tile's first row, the end of the expert's
};
__device__ __forceinline__ Tile find_tile(const int32_t* offsets, int experts, int rows, int t) {
  const int lane = lane_id();
  int before = 0;
  for (int e0 = 0; e0 <= experts; e0 += kWave) {
    const int e = e0 + lane;
    int lo = 0, hi = 0;
    if (e <= experts) {
      // (whatever the offsets hold, rows stay rows)
      lo = e == 0 ? 0 : min(max(offsets[e], 0), rows);
      hi = e == experts ? rows : min(max(offsets[e + 1], lo), rows);
    }
    const int mine = (hi - lo + BM - 1) / BM;
    const int upto = before + wave_incl_add(mine);
    const uint64_t past = __ballot(upto > t);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int first = __builtin_amdgcn_readlane(upto - mine, l);
      const int row = __builtin_amdgcn_readlane(lo, l) + (t - first) * BM;
      return Tile{e0 + l, row, __builtin_amdgcn_readlane(hi, l)};
    }
    before = __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return Tile{-1, 0, 0};
}

// The row of the tensor that row i of the order stands for, or -1.
__device__ __forceinline__ int64_t source_row(const int32_t* order, int top_k, int64_t count, int i) {
  int64_t r = i;
  if (order) {
    const int32_t at = order[i];
    r = at < 0 ? -1 : at / top_k;
  }
  return r < count ? r : -1;
}

// Four results of a row that lie side by side, at column n of `width`.
template <int DT, bool VEC>
__device__ __forceinline__ void store4(typename Elem<DT>::raw* p, Acc v, int left) {
  if (VEC && left >= 4) {
    if constexpr (DT == 0) {
      *reinterpret_cast<Acc*>(p) = v;
    } else {
      Move8 u;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        u[j] = static_cast<uint32_t>(Elem<DT>::put(v[2 * j])) |
               (static_cast<uint32_t>(Elem<DT>::put(v[2 * j + 1])) << 16);
      *reinterpret_cast<Move8*>(p) = u;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) p[j] = Elem<DT>::put(v[j]);
  }
}

// A stage of an operand on its way to LDS: PT threads, chunk by chunk.
template <class Op>
struct Stage {
  static constexpr int Each = Op::Total / PT;
  Move16 v[Each];
  static __device__ __forceinline__ int row(int i) { return (threadIdx.x + PT * i) / Op::Chunks; }
  static __device__ __forceinline__ int chunk(int i) { return (threadIdx.x + PT * i) % Op::Chunks; }
  __device__ __forceinline__ void put(char* lds) const {
#pragma unroll
    for (int i = 0; i < Each; ++i)
      *reinterpret_cast<Move16*>(lds + 16 * Op::slot(row(i), chunk(i))) = v[i];
  }
};

// The products of a stage in LDS: the wave's 64 x 64 results, four by four tiles.
// (b goes first, so that a lane holds four results of one row, side by side)
template <int DT, class A, class B>
__device__ __forceinline__ void multiply(const char* la, const char* lb, int m0, int n0, Acc (&acc)[4][4]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    Move16 fa[4], fb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) fa[i] = A::fragment(la, m0 + 16 * i, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) fb[i] = B::fragment(lb, n0 + 16 * i, s);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = mma<DT>(fb[j], fa[i], acc[i][j]);
  }
}

template <int DT, int DO, bool N_DENSE, bool VEC>
__global__ __launch_bounds__(PT) void expert_rows_kernel(RowsArgs a) {
  using A = Operand<DT, BM, false>;
  using B = Operand<DT, BN, N_DENSE>;
  using raw = typename Elem<DT>::raw;
  __shared__ __attribute__((aligned(16))) char lds[A::Bytes + B::Bytes];
  const int tn = blockIdx.x % a.tiles_n;
  const Tile t = find_tile(a.offsets, a.experts, a.rows, blockIdx.x / a.tiles_n);
  if (t.expert < 0) return;
  const int n0 = tn * BN;
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int wm = wave / 2 * 64, wn = wave % 2 * 64;
  Acc acc[4][4] = {};
  if (t.expert < a.experts) {
    const raw* x = static_cast<const raw*>(a.x);
    const raw* w = static_cast<const raw*>(a.w) + a.w_expert * t.expert;
    Stage<A> sa;
    Stage<B> sb;
    int64_t at[Stage<A>::Each];
#pragma unroll
    for (int i = 0; i < Stage<A>::Each; ++i) {
      const int r = t.row + Stage<A>::row(i);
      const int64_t src = r < t.end ? source_row(a.order, a.top_k, a.x_rows, r) : -1;
      at[i] = src < 0 ? -1 : src * a.x_stride;
    }
    const auto load = [&](int k0) {
#pragma unroll
      for (int i = 0; i < Stage<A>::Each; ++i) {
        const int k = k0 + A::N * Stage<A>::chunk(i);
        sa.v[i] = load_chunk<DT, VEC>(x + at[i] + k, at[i] < 0 ? 0 : a.k - k);
      }
#pragma unroll
      for (int i = 0; i < Stage<B>::Each; ++i) {
        const int r = Stage<B>::row(i), c = B::N * Stage<B>::chunk(i);
        const int64_t row = N_DENSE ? k0 + r : n0 + r;
        const int col = N_DENSE ? n0 + c : k0 + c;
        const bool in = row < (N_DENSE ? a.k : a.n);
        sb.v[i] = load_chunk<DT, VEC>(w + row * a.w_row + col, in ? (N_DENSE ? a.n : a.k) - col : 0);
      }
    };
    load(0);
    for (int k0 = 0; k0 < a.k; k0 += A::Stage) {
      sa.put(lds);
      sb.put(lds + A::Bytes);
      __syncthreads();
      if (k0 + A::Stage < a.k) load(k0 + A::Stage);
      multiply<DT, A, B>(lds, lds + A::Bytes, wm, wn, acc);
      __syncthreads();
    }
  }
  using out = typename Elem<DO>::raw;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = t.row + wm + 16 * i + (lane & 15);
    if (r >= t.end) continue;
    out* y = static_cast<out*>(a.y) + static_cast<int64_t>(r) * a.n;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + wn + 16 * j + 4 * (lane >> 4);
      if (n < a.n) store4<DO, VEC>(y + n, acc[i][j], a.n - n);
    }
  }
}

template <int DT, bool VEC>
__global__ __launch_bounds__(PT) void expert_grad_kernel(GradArgs a) {
  using A = Operand<DT, BM, true>;
  using B = Operand<DT, BN, true>;
  using raw = typename Elem<DT>::raw;
  __shared__ __attribute__((aligned(16))) char lds[A::Bytes + B::Bytes];
  const int tiles = a.tiles_m * a.tiles_n;
  const int e = blockIdx.x / tiles, t = blockIdx.x % tiles;
  const int m0 = t / a.tiles_n * BM, n0 = t % a.tiles_n * BN;
  const int lo = e == 0 ? 0 : min(max(a.offsets[e], 0), a.rows);
  const int hi = min(max(a.offsets[e + 1], lo), a.rows);
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int wm = wave / 2 * 64, wn = wave % 2 * 64;
  Acc acc[4][4] = {};
  Stage<A> sa;
  Stage<B> sb;
  const auto side = [&](auto& s, const void* p, const int32_t* order, int64_t count, int64_t stride, int r0,
                        int first, int width) {
    using S = std::remove_reference_t<decltype(s)>;
#pragma unroll
    for (int i = 0; i < S::Each; ++i) {
      const int r = r0 + S::row(i), c = first + A::N * S::chunk(i);
      const int64_t src = r < hi ? source_row(order, a.top_k, count, r) : -1;
      s.v[i] = load_chunk<DT, VEC>(static_cast<const raw*>(p) + src * stride + c, src < 0 ? 0 : width - c);
    }
  };
  const auto load = [&](int r0) {
    side(sa, a.a, a.gather == 1 ? a.order : nullptr, a.a_rows, a.a_stride, r0, m0, a.m);
    side(sb, a.b, a.gather == 2 ? a.order : nullptr, a.b_rows, a.b_stride, r0, n0, a.n);
  };
  load(lo);
  for (int r0 = lo; r0 < hi; r0 += A::Stage) {
    sa.put(lds);
    sb.put(lds + A::Bytes);
    __syncthreads();
    if (r0 + A::Stage < hi) load(r0 + A::Stage);
    multiply<DT, A, B>(lds, lds + A::Bytes, wm, wn, acc);
    __syncthreads();
  }
  raw* c = static_cast<raw*>(a.c) + a.c_expert * e;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + wm + 16 * i + (lane & 15);
    if (m >= a.m) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + wn + 16 * j + 4 * (lane >> 4);
      if (n < a.n) store4<DT, VEC>(c + m * a.c_row + n, acc[i][j], a.n - n);
    }
  }
}

}  // namespace

// ------------------------------------------------------------- launchers ---
hipError_t launch_expert_rows(RowsArgs a, int dtype, bool w_n_dense, bool out_f32, bool vec, hipStream_t s) {
  a.tiles_n = (a.n + BN - 1) / BN;
  // an expert's last tile is not full, and neither is that of the rows of none
  const int64_t most = a.rows / BM + (a.experts + 1 < a.rows ? a.experts + 1 : a.rows);
  const dim3 grid(static_cast<unsigned>(most * a.tiles_n));
  ProfScope ps_("expert_rows", s);
  const auto launch = [&](auto dt, auto dout) {
    constexpr int DT = decltype(dt)::value, DO = decltype(dout)::value;
    if (w_n_dense && vec) hipLaunchKernelGGL((expert_rows_kernel<DT, DO, true, true>), grid, dim3(PT), 0, s, a);
    else if (w_n_dense) hipLaunchKernelGGL((expert_rows_kernel<DT, DO, true, false>), grid, dim3(PT), 0, s, a);
    else if (vec) hipLaunchKernelGGL((expert_rows_kernel<DT, DO, false, true>), grid, dim3(PT), 0, s, a);
    else hipLaunchKernelGGL((expert_rows_kernel<DT, DO, false, false>), grid, dim3(PT), 0, s, a);
  };
  const std::integral_constant<int, 0> f32;
  const std::integral_constant<int, 1> b16;
  const std::integral_constant<int, 2> h16;
  if (dtype == 0) launch(f32, f32);
  else if (dtype == 1 && out_f32) launch(b16, f32);
  else if (dtype == 1) launch(b16, b16);
  else if (out_f32) launch(h16, f32);
  else launch(h16, h16);
  return hipGetLastError();
}

hipError_t launch_expert_grad(GradArgs a, int dtype, bool vec, hipStream_t s) {
  a.tiles_m = (a.m + BM - 1) / BM;
  a.tiles_n = (a.n + BN - 1) / BN;
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.experts) * a.tiles_m * a.tiles_n));
  ProfScope ps_("expert_grad", s);
  const auto launch = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (vec) hipLaunchKernelGGL((expert_grad_kernel<DT, true>), grid, dim3(PT), 0, s, a);
    else hipLaunchKernelGGL((expert_grad_kernel<DT, false>), grid, dim3(PT), 0, s, a);
  };
  if (dtype == 0) launch(std::integral_constant<int, 0>{});
  else if (dtype == 1) launch(std::integral_constant<int, 1>{});
  else launch(std::integral_constant<int, 2>{});
  return hipGetLastError();
}

}  // namespace lapsum
