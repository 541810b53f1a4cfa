// What the C entry points share: workspace carving, argument checks and the
// device check.
#pragma once

#include <stdint.h>
#include <string.h>

#include <mutex>

#include "../../include/lapsum.h"

namespace lapsum {

constexpr size_t kAlign = 256;

// Bump allocator over the caller's workspace; a null base only measures.
struct Carve {
  char* base;
  size_t off = 0;
  explicit Carve(void* b) : base(static_cast<char*>(b)) {}
  template <typename T>
  T* take(size_t count) {
    off = (off + kAlign - 1) / kAlign * kAlign;
    T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
    off += count * sizeof(T);
    return p;
  }
  size_t size() const { return (off + kAlign - 1) / kAlign * kAlign; }
};

// ------------------------------------------------------------ device check --
inline int check_device() {
  static std::mutex mu;
  static int known[64] = {0};   // 0 unknown, 1 gfx950, 2 other
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return LAPSUM_ERR_HIP;
  if (dev < 0 || dev >= 64) return LAPSUM_ERR_DEVICE;
  std::lock_guard<std::mutex> g(mu);
  if (known[dev] == 0) {
    hipDeviceProp_t prop;
    if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return LAPSUM_ERR_HIP;
    known[dev] = (strncmp(prop.gcnArchName, "gfx950", 6) == 0) ? 1 : 2;
  }
  return known[dev] == 1 ? LAPSUM_OK : LAPSUM_ERR_DEVICE;
}

inline int check_ws(void* ws, size_t have, size_t need) {
  if (need == 0) return LAPSUM_OK;
  if (ws == nullptr || have < need) return LAPSUM_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) % kAlign != 0) return LAPSUM_ERR_WORKSPACE;
  return LAPSUM_OK;
}

// -------------------------------------------------------- argument checks --
constexpr int64_t kMaxBlocks = int64_t(1) << 23;   // workgroups of a launch
constexpr int64_t kMaxThreads = int64_t(1) << 32;  // a launch has less

inline bool valid_dtype(int dtype) { return dtype >= LAPSUM_F32 && dtype <= LAPSUM_F16; }

inline bool int32_range(int64_t v) { return v >= 0 && v <= 2147483647LL; }

// The widest power of two, up to 16, that divides everything or'ed into bits.
inline int vector_width(uint64_t bits) {
  int w = 16;
  while (w > 1 && bits % static_cast<uint64_t>(w)) w /= 2;
  return w;
}
inline uint64_t bits_of(const void* p) { return reinterpret_cast<uintptr_t>(p); }
inline uint64_t bits_of(const int64_t* strides) {
  return static_cast<uint64_t>(strides[0] | strides[1] | strides[2]);
}

#define LAPSUM_TRY(expr)                         \
  do {                                           \
    if ((expr) != hipSuccess) return LAPSUM_ERR_HIP; \
  } while (0)

}  // namespace lapsum
