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

#define LAPSUM_TRY(expr)                         \
  do {                                           \
    if ((expr) != hipSuccess) return LAPSUM_ERR_HIP; \
  } while (0)

}  // namespace lapsum
