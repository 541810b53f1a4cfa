// What the native nodes share: failures as the binding's own exceptions, the
// caller's stream, workspaces.
#pragma once

#include <torch/extension.h>

#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/DeviceGuard.h>

#include <torch/csrc/Exceptions.h>

#include <stdexcept>

#include "../../include/lapsum.h"

namespace lapsum_node {

using torch::Tensor;

// A library call that failed, as the binding's own exception: LapsumError with
// the status and the entry point's name.
struct Failed : std::runtime_error {
  Failed(int status, const char* where) : std::runtime_error(where), status(status) {}
  int status;
};

inline void check(int status, const char* where) {
  if (status != LAPSUM_OK) throw Failed(status, where);
}

// Sets it as the current Python error (with the GIL held).
inline void set_error(const Failed& f) {
  const py::object type = py::module_::import("paper_2608_06912_amd").attr("LapsumError");
  PyErr_SetObject(type.ptr(), type(f.status, f.what()).ptr());
}

// f() on the engine's thread, a failure as the Python error.
template <class F>
auto in_engine(F&& f) -> decltype(f()) {
  try {
    return f();
  } catch (const Failed& failed) {
    const py::gil_scoped_acquire gil;
    set_error(failed);
    python_error e;
    e.persist();
    throw e;
  }
}

// A function called from Python: without the GIL, as a ctypes call runs (an
// allocation or a launch can wait for the device), a failure as the Python
// error.
template <class R, class... A>
auto entry(R (*f)(A...)) {
  return [f](A... args) -> R {
    try {
      const py::gil_scoped_release nogil;
      return f(std::forward<A>(args)...);
    } catch (const Failed& failed) {
      set_error(failed);
      throw py::error_already_set();
    }
  };
}

inline hipStream_t stream_of(const Tensor& x) {
  return c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(x.device().index()).stream();
}

inline Tensor bytes(size_t n, const Tensor& like) {
  return n ? at::empty({static_cast<int64_t>(n)}, like.options().dtype(at::kByte).requires_grad(false)) : Tensor();
}

inline void* ptr(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

using OptTensor = std::optional<Tensor>;

inline int dtype_of(const Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return LAPSUM_F32;
    case at::kBFloat16: return LAPSUM_BF16;
    case at::kHalf: return LAPSUM_F16;
    default: return -1;
  }
}
inline bool plain(const Tensor& t) { return t.is_cuda() && t.layout() == at::kStrided && !t.is_quantized(); }
inline bool dense(const Tensor& t, at::ScalarType type, const Tensor& like) {
  return plain(t) && t.scalar_type() == type && t.is_contiguous() && t.device() == like.device();
}

// What a call writes in place: nothing that requires grad in grad mode (the
// binding says so), and autograd is told afterwards, as after an in-place call of
// torch's.
inline bool may_write(const Tensor& t) { return !(t.requires_grad() && at::GradMode::is_enabled()); }
inline void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

}  // namespace lapsum_node

void bind_selection(py::module_& m);
void bind_products(py::module_& m);
