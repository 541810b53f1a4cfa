// What the products grouped by expert share: a workgroup's tile of results, its
// operands on their way to LDS, and the products of a stage.
//
// Two ways to LDS.  Direct: the memory unit writes what it loads to LDS by itself
// (16 bytes a lane, at the wave's address and on), so the next stages are on their way
// while one is multiplied, in buffers of their own, and take no registers.  Elements
// that do not exist are asked for beyond the buffer's end, where loads give 0.
// The fragments of a step are read from LDS while the step before it is multiplied, also
// across the barrier that a stage ends with: reading them when they are due cost
// 131072 rows of 128 experts 2048 -> 1536 973 us, ahead 880.
// That needs lines of whole, aligned vectors, and operands of less than 4 GiB.  Else:
// through registers.
#pragma once

#include "matrix.hpp"

namespace lapsum {

// Tiles of M x N results of several waves, each TM x TN of them; stages of STEPS steps,
// BUFFERS of them in LDS where operands go there directly.
template <int M_, int N_, int TM_, int TN_, int STEPS_, int BUFFERS_>
struct Shape {
  static constexpr int M = M_, N = N_, TM = TM_, TN = TN_, Steps = STEPS_, Buffers = BUFFERS_;
  static constexpr int WavesN = N / TN, Waves = M / TM * WavesN, T = Waves * kWave;
};

constexpr uint32_t kBeyond = 0xfffffff0u;   // past the end of every buffer
constexpr int64_t kMostBytes = (int64_t(1) << 32) - (int64_t(1) << 20);

typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void* base, int64_t bytes) {
  const int64_t n = bytes < 0 ? 0 : bytes < kMostBytes ? bytes : kMostBytes;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, static_cast<int>(static_cast<uint32_t>(n)),
                                           0x00020000);
}

// The chunks of a stage that a thread brings: chunk i of thread t is slot
// t + T i of the operand in LDS.
template <class Op, int T>
struct Chunks {
  static constexpr int Each = Op::Total / T;
  static_assert(Op::Total % T == 0, "whole turns");
  static __device__ __forceinline__ int slot(int i) { return threadIdx.x + T * i; }
  static __device__ __forceinline__ int row(int i) { return slot(i) / Op::Chunks; }
  static __device__ __forceinline__ int chunk(int i) { return (slot(i) % Op::Chunks) ^ Op::swizzle(row(i)); }
};

// An operand on the direct way.  at: where its chunks are at the contraction's
// start; past: from which element of the contraction on a chunk does not exist.
template <class Op, int T>
struct Direct : Chunks<Op, T> {
  using C = Chunks<Op, T>;
  Buffer from;
  uint32_t at[C::Each], step;   // step: bytes of an element of the contraction
  int past[C::Each];
  __device__ __forceinline__ void bring(char* lds, int k0) const {
#pragma unroll
    for (int i = 0; i < C::Each; ++i) put(lds, i, k0 < past[i] ? at[i] + static_cast<uint32_t>(k0) * step : kBeyond);
  }
  __device__ __forceinline__ void put(char* lds, int i, uint32_t offset) const {
    char* to = lds + 16 * (threadIdx.x / kWave * kWave + T * i);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16,
                                             static_cast<int>(offset), 0, 0, 0);
  }
};

// And through registers.
template <class Op, int T>
struct Staged : Chunks<Op, T> {
  using C = Chunks<Op, T>;
  Move16 v[C::Each];
  int left[C::Each], width;   // of the lines that the chunks are from
  template <int DT>
  __device__ __forceinline__ void load(int i, const typename Elem<DT>::raw* p, int exist) {
    left[i] = exist;
    v[i] = load_chunk<DT>(p, exist, width);
  }
  template <int DT>
  __device__ __forceinline__ void put(char* lds) const {
#pragma unroll
    for (int i = 0; i < C::Each; ++i)
      *reinterpret_cast<Move16*>(lds + 16 * C::slot(i)) = trim_chunk<DT>(v[i], left[i], width);
  }
};

// The row of the tensor that a place of the order stands for, or -1: place / top_k by a
// product with floor(2^shift / top_k) + 1, exact for places below 2^31 (shift = 31 +
// the bits of top_k - 1).
__device__ __forceinline__ int64_t place_row(int32_t place, const Divider& by, int64_t count) {
  const int64_t r = divide(static_cast<uint32_t>(place), by);
  return place >= 0 && r < count ? r : -1;
}
__device__ __forceinline__ int64_t source_row(const int32_t* order, const Divider& by, int64_t count, int i) {
  if (order) return place_row(order[i], by, count);
  return i < count ? i : -1;
}

// The fragments of a step: those of the wave's TM rows of a and TN of b.
template <int DT, class A, class B, class S>
struct Fragments {
  static constexpr int MI = S::TM / 16, NI = S::TN / 16;
  static constexpr int Reads = MI * A::Reads + NI * B::Reads;
  Move16 a[MI], b[NI];
  __device__ __forceinline__ void read(const char* __restrict lds, int m0, int n0, int s) {
#pragma unroll
    for (int i = 0; i < NI; ++i) b[i] = B::fragment(lds + A::Bytes, n0 + 16 * i, s);
#pragma unroll
    for (int i = 0; i < MI; ++i) a[i] = A::fragment(lds, m0 + 16 * i, s);
  }
  // (b goes first, so that a lane holds four results of one row, side by side)
  __device__ __forceinline__ void multiply(Acc (&acc)[MI][NI]) const {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = mma<DT>(b[j], a[i], acc[i][j]);
  }
};

// Through registers: the products of a stage.
template <int DT, class A, class B, class S>
__device__ __forceinline__ void multiply(const char* lds, int m0, int n0, Acc (&acc)[S::TM / 16][S::TN / 16]) {
#pragma unroll
  for (int s = 0; s < A::Steps; ++s) {
    Fragments<DT, A, B, S> f;
    f.read(lds, m0, n0, s);
    f.multiply(acc);
  }
}

// All waves have read what they read of LDS, and all but the last N loads of each have
// arrived.  (Loads arrive in the order of their issue.)
template <int N>
__device__ __forceinline__ void arrive() {
  static_assert(N < 64, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The schedule of a step: its matrix instructions, with the reads of the next step's
// fragments spread between them.
template <int READS, int PRODUCTS>
__device__ __forceinline__ void spread() {
  constexpr int each = PRODUCTS / READS > 0 ? PRODUCTS / READS : 1;
#pragma unroll
  for (int i = 0; i < READS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // an LDS read
    __builtin_amdgcn_sched_group_barrier(0x008, each, 0);   // matrix instructions
  }
}

// The products of a step whose fragments are read, while stage `after` arrives, the loads
// from k0 on start to the buffer `to` that the step was read from, and the next
// fragments are read.  What is read is not part of what the loads write: they start
// behind the barrier after which no wave reads that buffer.
template <int DT, class A, class B, class S, int LOADS, class Bring>
__device__ __forceinline__ void pass_on(const char* __restrict after, char* to, Bring& bring, int k0, int count,
                                        int m0, int n0, const Fragments<DT, A, B, S>& have,
                                        Fragments<DT, A, B, S>& next, Acc (&acc)[S::TM / 16][S::TN / 16]) {
  using F = Fragments<DT, A, B, S>;
  if (S::Buffers > 2 && k0 < count) arrive<LOADS * (S::Buffers - 2)>();
  else arrive<0>();
  if (k0 < count) bring(to, to + A::Bytes, k0);
  next.read(after, m0, n0, 0);
  have.multiply(acc);
  spread<F::Reads, F::MI * F::NI * (DT == 0 ? 4 : 1)>();
}
// Stage `now` of two steps, the first one's fragments read already.
template <int DT, class A, class B, class S, int LOADS, class Bring>
__device__ __forceinline__ void two_steps(const char* __restrict now, const char* __restrict after, char* to,
                                          Bring& bring, int k0, int count, int m0, int n0,
                                          Fragments<DT, A, B, S>& first, Acc (&acc)[S::TM / 16][S::TN / 16]) {
  using F = Fragments<DT, A, B, S>;
  F second;
  second.read(now, m0, n0, 1);
  first.multiply(acc);
  spread<F::Reads, F::MI * F::NI * (DT == 0 ? 4 : 1)>();
  pass_on<DT, A, B, S, LOADS>(after, to, bring, k0, count, m0, n0, second, first, acc);
}

// The contraction of `count` elements; lds: S::Buffers stages of both operands.
// bring(lds_a, lds_b, k0) starts a stage's loads, at least LOADS of them; so once no
// more than LOADS times the stages after a stage are on their way, it is there.
template <int DT, class A, class B, class S, int LOADS, class Bring>
__device__ __forceinline__ void contract(char* lds, Bring& bring, int count, int m0, int n0,
                                         Acc (&acc)[S::TM / 16][S::TN / 16]) {
  constexpr int bytes = A::Bytes + B::Bytes, K = A::Stage;
  static_assert(S::Buffers >= 2, "one to multiply, one to fill");
  if (count <= 0) return;
#pragma unroll
  for (int s = 0; s < S::Buffers; ++s)
    if (s * K < count) bring(lds + s * bytes, lds + s * bytes + A::Bytes, s * K);
  if (count > (S::Buffers - 1) * K) arrive<LOADS * (S::Buffers - 1)>();
  else arrive<0>();
  Fragments<DT, A, B, S> first;
  first.read(lds, m0, n0, 0);
  int now = 0;
  const auto turn = [](int b) { return b + 1 < S::Buffers ? b + 1 : 0; };
  if constexpr (A::Steps == 2) {
    for (int k0 = 0; k0 < count; k0 += K) {
      const int after = turn(now);
      two_steps<DT, A, B, S, LOADS>(lds + now * bytes, lds + after * bytes, lds + now * bytes, bring,
                                    k0 + S::Buffers * K, count, m0, n0, first, acc);
      now = after;
    }
  } else {
    Fragments<DT, A, B, S> second;
    int k0 = 0;
    const auto pass = [&](const Fragments<DT, A, B, S>& have, Fragments<DT, A, B, S>& next) {
      const int after = turn(now);
      pass_on<DT, A, B, S, LOADS>(lds + after * bytes, lds + now * bytes, bring, k0 + S::Buffers * K, count, m0, n0,
                                  have, next, acc);
      k0 += K;
      now = after;
    };
    if ((count + K - 1) / K % 2) {   // the rest in pairs
      pass(first, second);
      first = second;
    }
    while (k0 < count) {
      pass(first, second);
      pass(second, first);
    }
  }
}

// Four results of a row that lie side by side (memory serves vectors at any alignment of
// their elements).
template <int DT>
__device__ __forceinline__ void store4(typename Elem<DT>::raw* p, Acc v, int left) {
  using raw = typename Elem<DT>::raw;
  constexpr int words = sizeof(raw);
  struct __attribute__((packed, aligned(sizeof(raw)))) Any {
    uint32_t w[words];
  };
  Any u;
#pragma unroll
  for (int j = 0; j < words; ++j) {
    if constexpr (DT == 0) u.w[j] = __float_as_uint(v[j]);
    else
      u.w[j] = static_cast<uint32_t>(Elem<DT>::put(v[2 * j])) |
               (static_cast<uint32_t>(Elem<DT>::put(v[2 * j + 1])) << 16);
  }
  if (left >= 4) {
    *reinterpret_cast<Any*>(p) = u;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) p[j] = Elem<DT>::put(v[j]);
  }
}

// The results of a row in four tiles side by side, 16-bit and in whole vectors: lanes
// exchange quarters, so that each has 16 neighbouring ones and a row's four lanes a line
// of 128 bytes (32 bytes of it at a time otherwise).  p: the first tile's first column,
// of which `left` exist.
template <int DT>
__device__ __forceinline__ void store_line(typename Elem<DT>::raw* p, const Acc* v, int left) {
  uint32_t w[4][2];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h)
      w[j][h] = static_cast<uint32_t>(Elem<DT>::put(v[j][2 * h])) |
                (static_cast<uint32_t>(Elem<DT>::put(v[j][2 * h + 1])) << 16);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto a = __builtin_amdgcn_permlane32_swap(w[0][h], w[2][h], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(w[1][h], w[3][h], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    w[0][h] = c[0];
    w[1][h] = c[1];
    w[2][h] = d[0];
    w[3][h] = d[1];
  }
  const int first = 16 * (lane_id() >> 4);
  if (first < left) *reinterpret_cast<Move16*>(p + first) = Move16{w[0][0], w[0][1], w[1][0], w[1][1]};
  if (first + 8 < left) *reinterpret_cast<Move16*>(p + first + 8) = Move16{w[2][0], w[2][1], w[3][0], w[3][1]};
}

// Workgroups are dealt out to the eight dies in turn, each with a cache of its own: in
// every 256 of them a die takes 32 tiles that follow one another.  Tiles follow one
// another in blocks of four rows and eight columns of them, which share rows
// and matrices in as few lines as 32 tiles can.  (tile row, tile column)
struct TileAt {
  int m, n;
};
__device__ __forceinline__ TileAt tile_of_block(int tiles_n) {
  constexpr uint32_t dies = 8, run = 32;
  uint32_t b = blockIdx.x;
  const uint32_t whole = gridDim.x / (dies * run) * (dies * run);
  if (b < whole) {
    const uint32_t in = b % (dies * run);
    b = b - in + in % dies * run + in / dies;
  }
  const uint32_t strip = b / (4u * tiles_n), in = b - strip * 4u * tiles_n;
  const uint32_t block = in / 32u, at = in - block * 32u;
  const uint32_t width = min(8u, tiles_n - block * 8u);
  return TileAt{static_cast<int>(strip * 4u + at / width), static_cast<int>(block * 8u + at % width)};
}

}  // namespace lapsum
