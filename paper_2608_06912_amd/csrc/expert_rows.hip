// Products grouped by expert: the rows of each expert, consecutive after the order,
// times the expert's matrix,
//
//   y[i][n] = sum_k x[row(i)][k] w_e[k][n],      offsets[e] <= i < offsets[e+1].
//
// The gradient of the rows is the same with w read the other way round, so w may
// be dense along k or along n.  A workgroup computes a tile of one expert's
// results; which one it finds by itself from the offsets, as the host does not know
// them.
//
// Many rows are bound by the way into LDS and by the ends of tiles (131072 rows of 128
// experts 2048 -> 1536 in float16 835 to 853 us, 967 to 988 TFLOP/s; 128 x 128 tiles without
// loads 1390), few rows by the matrices' bytes (64 rows of 41 experts 2048 -> 1024 in
// bfloat16 29 us, 5.9 TB/s: a tile of 16 rows and 64 columns, so that 650 workgroups
// read them).  Rows of y of odd lengths do not keep operands from the direct way (70 rows of
// 16 experts 1512 -> 2187 and back in float16 69 us, through registers 79).
#include "expert_tile.hpp"

namespace lapsum {
namespace {

// The expert and the first row of the t-th tile of `height` rows, experts' tiles one
// after another, the rows of no expert last.
struct Tile {
  int expert;      // experts: rows of none; -1: no such tile
  int row, end;    // the tile's first row, the end of the expert's
};
__device__ __forceinline__ Tile find_tile(const int32_t* offsets, int experts, int rows, int height, int t) {
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
    const int mine = (hi - lo + height - 1) / height;
    const int upto = before + wave_incl_add(mine);
    const uint64_t past = __ballot(upto > t);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int first = __builtin_amdgcn_readlane(upto - mine, l);
      const int row = __builtin_amdgcn_readlane(lo, l) + (t - first) * height;
      return Tile{e0 + l, row, __builtin_amdgcn_readlane(hi, l)};
    }
    before = __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return Tile{-1, 0, 0};
}

template <int DT, bool N_DENSE, class S>
struct Product {
  using A = Operand<DT, S::M, false, S::Steps>;
  using B = Operand<DT, S::N, N_DENSE, S::Steps>;
  using raw = typename Elem<DT>::raw;
};

template <int DT, bool N_DENSE, class S>
__device__ __forceinline__ void direct(const RowsArgs& a, const Tile& t, int n0, int wm, int wn,
                                       Acc (&acc)[S::TM / 16][S::TN / 16]) {
  using P = Product<DT, N_DENSE, S>;
  using A = typename P::A;
  using B = typename P::B;
  __shared__ __attribute__((aligned(16))) char lds[S::Buffers * (A::Bytes + B::Bytes)];
  constexpr int E = A::E;
  Direct<A, S::T> da;
  Direct<B, S::T> db;
  // rows that follow one another are counted from the tile's first
  const int64_t first = a.order ? 0 : t.row;
  da.from = buffer_of(static_cast<const typename P::raw*>(a.x) + first * a.x_stride,
                      ((a.x_rows - first - 1) * a.x_stride + a.k) * E);
  da.step = E;
#pragma unroll
  for (int i = 0; i < da.Each; ++i) {
    const int r = t.row + da.row(i), k = A::N * da.chunk(i);
    const int64_t src = r < t.end ? source_row(a.order, a.by, a.x_rows, r) : -1;
    da.at[i] = static_cast<uint32_t>(((src - first) * a.x_stride + k) * E);
    da.past[i] = src < 0 ? 0 : a.k - k;
  }
  const int64_t lines = N_DENSE ? a.k : a.n, length = N_DENSE ? a.n : a.k;
  db.from = buffer_of(static_cast<const typename P::raw*>(a.w) + a.w_expert * t.expert,
                      ((lines - 1) * a.w_row + length) * E);
  db.step = static_cast<uint32_t>(N_DENSE ? a.w_row * E : E);
#pragma unroll
  for (int i = 0; i < db.Each; ++i) {
    const int r = db.row(i), c = B::N * db.chunk(i);
    const int k = N_DENSE ? r : c, n = n0 + (N_DENSE ? c : r);
    db.at[i] = static_cast<uint32_t>((N_DENSE ? k * a.w_row + n : n * a.w_row + k) * E);
    db.past[i] = n < a.n ? a.k - k : 0;
  }
  const auto bring = [&](char* la, char* lb, int k0) {
    da.bring(la, k0);
    db.bring(lb, k0);
  };
  contract<DT, A, B, S, Chunks<A, S::T>::Each + Chunks<B, S::T>::Each>(lds, bring, a.k, wm, wn, acc);
}

template <int DT, bool N_DENSE, class S>
__device__ __forceinline__ void staged(const RowsArgs& a, const Tile& t, int n0, int wm, int wn,
                                       Acc (&acc)[S::TM / 16][S::TN / 16]) {
  using P = Product<DT, N_DENSE, S>;
  using A = typename P::A;
  using B = typename P::B;
  __shared__ __attribute__((aligned(16))) char lds[A::Bytes + B::Bytes];
  const auto* x = static_cast<const typename P::raw*>(a.x);
  const auto* w = static_cast<const typename P::raw*>(a.w) + a.w_expert * t.expert;
  Staged<A, S::T> sa;
  Staged<B, S::T> sb;
  sa.width = a.k;
  sb.width = N_DENSE ? a.n : a.k;
  int64_t at[sa.Each];
#pragma unroll
  for (int i = 0; i < sa.Each; ++i) {
    const int r = t.row + sa.row(i);
    const int64_t src = r < t.end ? source_row(a.order, a.by, a.x_rows, r) : -1;
    at[i] = src < 0 ? -1 : src * a.x_stride;
  }
  const auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < sa.Each; ++i) {
      const int k = k0 + A::N * sa.chunk(i);
      sa.template load<DT>(i, x + at[i] + k, at[i] < 0 ? 0 : a.k - k);
    }
#pragma unroll
    for (int i = 0; i < sb.Each; ++i) {
      const int r = sb.row(i), c = B::N * sb.chunk(i);
      const int64_t line = N_DENSE ? k0 + r : n0 + r;
      const int col = N_DENSE ? n0 + c : k0 + c;
      const bool in = line < (N_DENSE ? a.k : a.n);
      sb.template load<DT>(i, w + line * a.w_row + col, in ? sb.width - col : 0);
    }
  };
  load(0);
  for (int k0 = 0; k0 < a.k; k0 += A::Stage) {
    sa.template put<DT>(lds);
    sb.template put<DT>(lds + A::Bytes);
    __syncthreads();
    if (k0 + A::Stage < a.k) load(k0 + A::Stage);
    multiply<DT, A, B, S>(lds, wm, wn, acc);
    __syncthreads();
  }
}

template <int DT, int DO, bool N_DENSE, bool DIRECT, class S>
__global__ __launch_bounds__(S::T, S::M >= 128 ? 2 : 4) void expert_rows_kernel(RowsArgs a) {
  const TileAt at = tile_of_block(a.tiles_n);
  const Tile t = find_tile(a.offsets, a.experts, a.rows, S::M, at.m);
  if (t.expert < 0) return;
  const int n0 = at.n * S::N;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = wave / S::WavesN * S::TM, wn = wave % S::WavesN * S::TN;
  Acc acc[S::TM / 16][S::TN / 16] = {};
  if (t.expert < a.experts) {
    if constexpr (DIRECT) direct<DT, N_DENSE, S>(a, t, n0, wm, wn, acc);
    else staged<DT, N_DENSE, S>(a, t, n0, wm, wn, acc);
  }
  using out = typename Elem<DO>::raw;
  constexpr bool lines = DIRECT && DO != 0 && S::TN % 64 == 0;
#pragma unroll
  for (int i = 0; i < S::TM / 16; ++i) {
    const int r = t.row + wm + 16 * i + (lane & 15);
    const bool in = r < t.end;   // (all lanes take part in an exchange)
    out* y = static_cast<out*>(a.y) + static_cast<int64_t>(r) * a.n;
    if (lines && a.y_lines) {
#pragma unroll
      for (int j = 0; j < S::TN / 16; j += 4) {
        const int n = n0 + wn + 16 * j;
        if constexpr (lines) store_line<DO>(y + n, &acc[i][j], in ? a.n - n : 0);
      }
    } else if (in) {
#pragma unroll
      for (int j = 0; j < S::TN / 16; ++j) {
        const int n = n0 + wn + 16 * j + 4 * (lane >> 4);
        if (n < a.n) store4<DO>(y + n, acc[i][j], a.n - n);
      }
    }
  }
}

}  // namespace

// ------------------------------------------------------------- launchers ---
// The way and the shape of tiles of a product: f(way, shape).  What is launched and what is
// checked before come from here both.
template <int DT, bool N_DENSE, class F>
static auto with_shape(const RowsArgs& a, bool vec, F&& f) {
  const int64_t size = DT == 0 ? 4 : 2;
  const bool direct = vec && (a.order ? a.x_rows * a.x_stride : 256 * a.x_stride + a.k) * size < kMostBytes &&
                      ((N_DENSE ? a.k : a.n) + 1) * a.w_row * size < kMostBytes;
  const int64_t tiles = (a.rows / 128 + (a.experts < a.rows ? a.experts : a.rows)) * ((a.n + 127) / 128);
  const std::true_type yes;
  const std::false_type no;
  // (most of a taller tile would be rows of none)
  const bool few = a.rows <= static_cast<int64_t>(a.experts) * 16;
  // Few large tiles leave compute units idle, small ones read more than the die's
  // cache delivers.  Rows of 128 bytes are two steps of 64 and want both at
  // once; where w is dense along n one step's rows of it are long.  16384 rows of
  // 8 experts 2048 -> 4096 in bfloat16 (and 131072 of 128, 2048 -> 1536), us:
  //   w dense along n   256 x 256 307 (854), 128 x 256 284 (856), 128 x 128 301 (1001)
  //   w dense along k   256 x 256 284 (847), 128 x 256 316 (942), 128 x 128 290 (990)
  const int64_t each = a.rows / a.experts;
  if constexpr (DT != 0) {
    if (direct && (N_DENSE ? tiles >= 1024 && each >= 128 : tiles >= 2048 && each >= 256)) {
      if constexpr (N_DENSE) return f(yes, Shape<128, 256, 128, 64, 1, 3>{});
      else return f(yes, Shape<256, 256, 128, 64, 2, 2>{});
    }
  }
  if (direct && tiles >= 512 && !few) return f(yes, Shape<128, 128, 64, 64, 2, 2>{});
  if (direct && !few) return f(yes, Shape<64, 64, 32, 32, 2, 2>{});
  if (direct) return f(yes, Shape<16, 64, 16, 32, 2, 2>{});
  if (few) return f(no, Shape<16, 64, 16, 32, 2, 1>{});
  // (float32, 128 x 128 and 64 x 64, us: 100320 rows 75 -> 691 221 and 206, 16384 rows
  // 2047 -> 1023 794 and 757, 32768 rows 511 -> 2049 695 and 701)
  if constexpr (DT != 0) {
    if (tiles >= 512) return f(no, Shape<128, 128, 64, 64, 2, 1>{});
  }
  return f(no, Shape<64, 64, 32, 32, 2, 1>{});
}
template <class S>
static int64_t blocks_of(const RowsArgs& a) {
  // an expert's last tile is not full, and neither is that of the rows of none
  const int64_t most = (a.rows / S::M + (a.experts + 1 < a.rows ? a.experts + 1 : a.rows) + 3) / 4 * 4;
  return most * ((a.n + S::N - 1) / S::N);
}

int64_t expert_rows_threads(const RowsArgs& a, int dtype, bool w_n_dense, bool vec) {
  const auto count = [&](auto, auto shape) { return blocks_of<decltype(shape)>(a) * decltype(shape)::T; };
  const auto of = [&](auto dt) {
    return w_n_dense ? with_shape<decltype(dt)::value, true>(a, vec, count)
                     : with_shape<decltype(dt)::value, false>(a, vec, count);
  };
  return dtype == 0 ? of(std::integral_constant<int, 0>{}) : of(std::integral_constant<int, 1>{});
}

hipError_t launch_expert_rows(RowsArgs a, int dtype, bool w_n_dense, bool out_f32, bool vec, hipStream_t s) {
  ProfScope ps_("expert_rows", s);
  const auto types = [&](auto dt, auto dout) {
    constexpr int DT = decltype(dt)::value, DO = decltype(dout)::value;
    const auto go = [&](auto dense) {
      constexpr bool N_DENSE = decltype(dense)::value;
      with_shape<DT, N_DENSE>(a, vec, [&](auto way, auto shape) {
        using S = decltype(shape);
        a.tiles_n = (a.n + S::N - 1) / S::N;
        hipLaunchKernelGGL((expert_rows_kernel<DT, DO, N_DENSE, decltype(way)::value, S>),
                           dim3(static_cast<unsigned>(blocks_of<S>(a))), dim3(S::T), 0, s, a);
      });
    };
    if (w_n_dense) go(std::true_type{});
    else go(std::false_type{});
  };
  const std::integral_constant<int, 0> f32;
  const std::integral_constant<int, 1> b16;
  const std::integral_constant<int, 2> h16;
  if (dtype == 0) types(f32, f32);
  else if (dtype == 1 && out_f32) types(b16, f32);
  else if (dtype == 1) types(b16, b16);
  else if (out_f32) types(h16, f32);
  else types(h16, h16);
  return hipGetLastError();
}

}  // namespace lapsum
