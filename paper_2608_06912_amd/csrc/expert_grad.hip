// The gradient of the experts' matrices: for each expert a product over its rows,
//
//   c_e[m][n] = sum_i a[row(i)][m] b[row(i)][n],      offsets[e] <= i < offsets[e+1].
//
// Both operands are dense along the results, so both are transposed on their way out
// of LDS.  Where the matrices are too few to fill the chip, an expert's rows are
// split over several workgroups, whose float32 parts expert_grad_join_kernel adds in
// their order.  8 matrices of 2048 x 4096 from 16384 rows in bfloat16 take 266 us
// (1034 TFLOP/s), bound as the products are; 4 of 283 x 184 from 31538 rows in float32
// 55 + 9 us with 30 splits, 375 without.
#include "expert_tile.hpp"

namespace lapsum {
namespace {

// A side of the product on the direct way.  One whose rows follow one another is counted
// from the first, `lo`; one that comes through the order looks the rows of a stage up a
// stage ahead of their loads.
template <int DT, class Op, int T, bool GATHER>
struct Side : Direct<Op, T> {
  using D = Direct<Op, T>;
  int32_t place[D::Each];
  const int32_t* order;
  int64_t count;
  Divider by;
  int lo, hi;
  __device__ __forceinline__ void look(int k0) {
#pragma unroll
    for (int i = 0; i < D::Each; ++i) place[i] = order[min(lo + k0 + D::row(i), hi - 1)];
  }
  __device__ __forceinline__ void set(const GradArgs& a, const void* p, int64_t rows, int64_t stride, int first,
                                      int width, int lo_, int hi_) {
    constexpr int E = Op::E;
    lo = lo_;
    hi = hi_;
    order = a.order;
    count = rows;
    by = a.by;
    const int64_t base = GATHER ? 0 : lo;
    D::from = buffer_of(static_cast<const typename Elem<DT>::raw*>(p) + base * stride,
                        ((rows - base - 1) * stride + width) * E);
    D::step = static_cast<uint32_t>(stride * E);
#pragma unroll
    for (int i = 0; i < D::Each; ++i) {
      const int r = D::row(i), c = first + Op::N * D::chunk(i);
      D::at[i] = static_cast<uint32_t>((GATHER ? c : r * stride + c) * E);
      D::past[i] = c < width ? hi - lo - r : 0;
    }
    if constexpr (GATHER) look(0);
  }
  __device__ __forceinline__ void bring(char* lds, int k0) {
    if constexpr (!GATHER) {
      D::bring(lds, k0);
    } else {
      uint32_t to[D::Each];
#pragma unroll
      for (int i = 0; i < D::Each; ++i) {
        const int64_t r = place_row(place[i], by, count);
        to[i] = k0 < D::past[i] && r >= 0 ? D::at[i] + static_cast<uint32_t>(r) * D::step : kBeyond;
      }
      // (the lookups go out before this stage's loads: they are waited for in order)
      look(k0 + Op::Stage);
#pragma unroll
      for (int i = 0; i < D::Each; ++i) D::put(lds, i, to[i]);
    }
  }
};

template <int DT, int GATHER, class S>
__device__ __forceinline__ void direct(const GradArgs& a, int lo, int hi, int m0, int n0, int wm, int wn,
                                       Acc (&acc)[S::TM / 16][S::TN / 16]) {
  using A = Operand<DT, S::M, true, S::Steps>;
  using B = Operand<DT, S::N, true, S::Steps>;
  __shared__ __attribute__((aligned(16))) char lds[S::Buffers * (A::Bytes + B::Bytes)];
  if (lo >= hi) return;
  Side<DT, A, S::T, GATHER == 1> da;
  Side<DT, B, S::T, GATHER == 2> db;
  da.set(a, a.a, a.a_rows, a.a_stride, m0, a.m, lo, hi);
  db.set(a, a.b, a.b_rows, a.b_stride, n0, a.n, lo, hi);
  const auto bring = [&](char* la, char* lb, int k0) {
    da.bring(la, k0);
    db.bring(lb, k0);
  };
  contract<DT, A, B, S, Chunks<A, S::T>::Each + Chunks<B, S::T>::Each>(lds, bring, hi - lo, wm, wn, acc);
}

template <int DT, class S>
__device__ __forceinline__ void staged(const GradArgs& a, int lo, int hi, int m0, int n0, int wm, int wn,
                                       Acc (&acc)[S::TM / 16][S::TN / 16]) {
  using A = Operand<DT, S::M, true, S::Steps>;
  using B = Operand<DT, S::N, true, S::Steps>;
  using raw = typename Elem<DT>::raw;
  __shared__ __attribute__((aligned(16))) char lds[A::Bytes + B::Bytes];
  Staged<A, S::T> sa;
  Staged<B, S::T> sb;
  const auto side = [&](auto& s, const void* p, const int32_t* order, int64_t count, int64_t stride, int r0,
                        int first, int width) {
    s.width = width;
#pragma unroll
    for (int i = 0; i < s.Each; ++i) {
      const int r = r0 + s.row(i), c = first + A::N * s.chunk(i);
      const int64_t src = r < hi ? source_row(order, a.by, count, r) : -1;
      s.template load<DT>(i, static_cast<const raw*>(p) + src * stride + c, src < 0 ? 0 : width - c);
    }
  };
  const auto load = [&](int r0) {
    side(sa, a.a, a.gather == 1 ? a.order : nullptr, a.a_rows, a.a_stride, r0, m0, a.m);
    side(sb, a.b, a.gather == 2 ? a.order : nullptr, a.b_rows, a.b_stride, r0, n0, a.n);
  };
  load(lo);
  for (int r0 = lo; r0 < hi; r0 += A::Stage) {
    sa.template put<DT>(lds);
    sb.template put<DT>(lds + A::Bytes);
    __syncthreads();
    if (r0 + A::Stage < hi) load(r0 + A::Stage);
    multiply<DT, A, B, S>(lds, wm, wn, acc);
    __syncthreads();
  }
}

// WAY: operands straight to LDS, a's or b's through the order (0, 1, 2), or not (-1).
template <int DT, int WAY, class S>
__global__ __launch_bounds__(S::T, S::M >= 128 ? 2 : 4) void expert_grad_kernel(GradArgs a) {
  const int tiles_m = (a.m + S::M - 1) / S::M, tiles_n = (a.n + S::N - 1) / S::N;
  const TileAt at = tile_of_block(tiles_n);
  const int piece = at.m / tiles_m;
  if (piece >= a.experts * a.splits) return;
  const int e = piece / a.splits, split = piece % a.splits;
  const int m0 = at.m % tiles_m * S::M, n0 = at.n * S::N;
  int lo = e == 0 ? 0 : min(max(a.offsets[e], 0), a.rows);
  int hi = min(max(a.offsets[e + 1], lo), a.rows);
  if (a.splits > 1) {   // whole stages each
    constexpr int stage = S::Steps * (DT == 0 ? 16 : 32);
    const int each = ((hi - lo + a.splits - 1) / a.splits + stage - 1) / stage * stage;
    const int end = hi;
    lo = static_cast<int>(min(static_cast<int64_t>(end), lo + static_cast<int64_t>(each) * split));
    hi = min(end, lo + each);
  }
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = wave / S::WavesN * S::TM, wn = wave % S::WavesN * S::TN;
  Acc acc[S::TM / 16][S::TN / 16] = {};
  constexpr bool DIRECT = WAY >= 0;
  if constexpr (DIRECT) direct<DT, WAY, S>(a, lo, hi, m0, n0, wm, wn, acc);
  else staged<DT, S>(a, lo, hi, m0, n0, wm, wn, acc);
  using raw = typename Elem<DT>::raw;
  constexpr bool lines = DIRECT && DT != 0 && S::TN % 64 == 0;   // (such tiles have no splits)
#pragma unroll
  for (int i = 0; i < S::TM / 16; ++i) {
    const int m = m0 + wm + 16 * i + (lane & 15);
    raw* c = static_cast<raw*>(a.c) + a.c_expert * e + m * a.c_row;
    if constexpr (lines) {
#pragma unroll
      for (int j = 0; j < S::TN / 16; j += 4) {
        const int n = n0 + wn + 16 * j;
        store_line<DT>(c + n, &acc[i][j], m < a.m ? a.n - n : 0);
      }
    } else if (m < a.m) {
#pragma unroll
      for (int j = 0; j < S::TN / 16; ++j) {
        const int n = n0 + wn + 16 * j + 4 * (lane >> 4);
        if (n >= a.n) continue;
        if (a.splits > 1)
          store4<0>(reinterpret_cast<uint32_t*>(a.part) +
                        ((static_cast<int64_t>(split) * a.experts + e) * a.m + m) * a.n + n,
                    acc[i][j], a.n - n);
        else store4<DT>(c + n, acc[i][j], a.n - n);
      }
    }
  }
}

// The splits' parts, added in their order.
template <int DT>
__global__ __launch_bounds__(256) void expert_grad_join_kernel(GradArgs a) {
  const int64_t each = static_cast<int64_t>(a.m) * a.n, total = a.experts * each;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    float sum = 0.0f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) sum += a.part[s * total + i];
    const int64_t e = i / each, m = (i - e * each) / a.n, n = i - e * each - m * a.n;
    static_cast<typename Elem<DT>::raw*>(a.c)[a.c_expert * e + m * a.c_row + n] = Elem<DT>::put(sum);
  }
}

}  // namespace

// ------------------------------------------------------------- launchers ---
// How many workgroups share an expert's rows: enough for eight of 64 x 64 results per
// compute unit, as long as each has 256 rows.
int grad_splits(int64_t experts, int64_t rows, int64_t m, int64_t n) {
  const int64_t tiles = experts * ((m + 63) / 64) * ((n + 63) / 64);
  if (tiles >= 1024) return 1;
  const int64_t most = rows / experts / 256;
  const int64_t want = (2047 + tiles) / tiles;
  return static_cast<int>(want < most ? (want < 1 ? 1 : want) : (most < 1 ? 1 : most));
}

// The way and the shape of tiles of a gradient: f(way, shape).
template <int DT, class F>
static auto with_shape(const GradArgs& a, bool vec, F&& f) {
  const int64_t size = DT == 0 ? 4 : 2;
  const auto spans = [&](int64_t rows, int64_t stride, bool gather) {
    return (gather ? rows : a.rows + int64_t(1)) * stride * size < kMostBytes;
  };
  const bool direct = vec && spans(a.a_rows, a.a_stride, a.gather == 1) && spans(a.b_rows, a.b_stride, a.gather == 2);
  const int64_t tiles = static_cast<int64_t>(a.experts) * ((a.m + 127) / 128) * ((a.n + 127) / 128);
  const std::integral_constant<int, -1> no;
  const auto big = [&](auto yes) {
    // the training layer's 8 matrices of 2048 x 4096 (and 128 of 2048 x 1536 from 131072
    // rows), us: 256 x 256 338 (1072), 128 x 256 266 (956), 128 x 128 301 (1168)
    if constexpr (DT != 0) {
      if (tiles >= 1024 && a.splits == 1) return f(yes, Shape<128, 256, 128, 64, 1, 3>{});
    }
    if (tiles >= 512 && a.splits == 1) return f(yes, Shape<128, 128, 64, 64, 2, 2>{});
    return f(yes, Shape<64, 64, 32, 32, 2, 2>{});
  };
  if (direct && a.gather == 0) return big(std::integral_constant<int, 0>{});
  if (direct && a.gather == 1) return big(std::integral_constant<int, 1>{});
  if (direct) return big(std::integral_constant<int, 2>{});
  if (tiles >= 512 && a.splits == 1) return f(no, Shape<128, 128, 64, 64, 2, 1>{});
  return f(no, Shape<64, 64, 32, 32, 2, 1>{});
}
template <class S>
static int64_t blocks_of(const GradArgs& a) {
  const int64_t lines = static_cast<int64_t>(a.experts) * a.splits * ((a.m + S::M - 1) / S::M);
  return (lines + 3) / 4 * 4 * ((a.n + S::N - 1) / S::N);
}

int64_t expert_grad_threads(const GradArgs& a, int dtype, bool vec) {
  const auto count = [&](auto, auto shape) { return blocks_of<decltype(shape)>(a) * decltype(shape)::T; };
  return dtype == 0 ? with_shape<0>(a, vec, count) : with_shape<1>(a, vec, count);
}

hipError_t launch_expert_grad(GradArgs a, int dtype, bool vec, hipStream_t s) {
  const auto types = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    {
      ProfScope ps_("expert_grad", s);
      with_shape<DT>(a, vec, [&](auto way, auto shape) {
        using S = decltype(shape);
        hipLaunchKernelGGL((expert_grad_kernel<DT, decltype(way)::value, S>), dim3(static_cast<unsigned>(blocks_of<S>(a))),
                           dim3(S::T), 0, s, a);
      });
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    ProfScope ps_("expert_grad_join", s);
    const int64_t blocks = (static_cast<int64_t>(a.experts) * a.m * a.n + 255) / 256;
    hipLaunchKernelGGL((expert_grad_join_kernel<DT>), dim3(static_cast<unsigned>(blocks < (1 << 16) ? blocks : (1 << 16))),
                       dim3(256), 0, s, a);
    return hipGetLastError();
  };
  if (dtype == 0) return types(std::integral_constant<int, 0>{});
  if (dtype == 1) return types(std::integral_constant<int, 1>{});
  return types(std::integral_constant<int, 2>{});
}

}  // namespace lapsum
