// The calls of the experts' rows and of the paged cache in native code: the common
// case of each straight to the C ABI.  Whatever a function here does not take (it
// returns None) goes to the bindings in experts.py and paged.py, where it is checked
// and refused.
#include "node.hpp"

#include <torch/csrc/autograd/functions/basic_ops.h>

#include <cmath>

namespace {

using namespace lapsum_node;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// Rows of a matrix, dense, evenly apart.
bool matrix(const Tensor& x) {
  return plain(x) && x.dim() == 2 && (x.stride(1) == 1 || x.size(1) <= 1) &&
         (x.stride(0) >= x.size(1) || x.size(0) <= 1);
}
int64_t row_stride(const Tensor& x) { return x.size(0) > 1 ? x.stride(0) : x.size(1); }

std::optional<std::tuple<Tensor, Tensor, Tensor>> expert_order(const Tensor& at, int64_t experts) {
  if (!plain(at) || at.scalar_type() != at::kInt || !at.is_contiguous() || experts < 1) return std::nullopt;
  const c10::DeviceGuard guard(at.device());
  const auto opt = at.options().requires_grad(false);
  const int64_t n = at.numel();
  Tensor order = at::empty({n}, opt), place = at::empty(at.sizes(), opt), offsets = at::empty({experts + 1}, opt);
  const size_t need = lapsum_expert_order_workspace_size(n, experts);
  Tensor ws = bytes(need, at);
  check(lapsum_expert_order(at.data_ptr<int32_t>(), n, experts, order.data_ptr<int32_t>(),
                            place.data_ptr<int32_t>(), offsets.data_ptr<int32_t>(), ptr(ws), need, stream_of(at)),
        "lapsum_expert_order");
  return std::make_tuple(order, place, offsets);
}

// The arguments of a product that both its directions take, checked.
struct Product {
  bool ok = false;
  int64_t in = 0, out = 0, rows = 0, strides[3] = {0, 0, 0};
  Product(const Tensor& x, const Tensor& w, const Tensor& offsets, const OptTensor& order) {
    if (!matrix(x) || dtype_of(x) < 0 || !plain(w) || w.dim() != 3 || w.scalar_type() != x.scalar_type() ||
        w.device() != x.device() || w.size(1) != x.size(1) || !dense(offsets, at::kInt, x) || offsets.dim() != 1 ||
        offsets.size(0) != w.size(0) + 1 || (order && (!dense(*order, at::kInt, x) || order->dim() != 1)))
      return;
    in = w.size(1);
    out = w.size(2);
    for (int i = 0; i < 3; ++i) strides[i] = w.stride(i);
    ok = (strides[2] == 1 && strides[1] >= out) || (strides[1] == 1 && strides[2] >= in);
    rows = order ? order->numel() : x.size(0);
  }
};

Tensor product(const Tensor& x, const Tensor& w, const Tensor& offsets, const OptTensor& order, int64_t top_k,
               const Product& p, at::ScalarType type) {
  const c10::DeviceGuard guard(x.device());
  Tensor y = at::empty({p.rows, p.out}, x.options().dtype(type).requires_grad(false));
  check(lapsum_expert_matmul(x.data_ptr(), dtype_of(x), x.size(0), row_stride(x),
                             order ? order->data_ptr<int32_t>() : nullptr, top_k, offsets.data_ptr<int32_t>(),
                             w.size(0), p.rows, p.in, p.out, w.data_ptr(), p.strides, y.data_ptr(), dtype_of(y),
                             stream_of(x)),
        "lapsum_expert_matmul");
  return y;
}

OptTensor expert_matmul(const Tensor& x, const Tensor& w, const Tensor& offsets, const OptTensor& order,
                        int64_t top_k) {
  const Product p(x, w, offsets, order);
  if (!p.ok) return std::nullopt;
  return product(x, w, offsets, order, top_k, p, x.scalar_type());
}

Tensor combine(const Tensor& y, const Tensor& place, const OptTensor& weights, at::ScalarType type) {
  const c10::DeviceGuard guard(y.device());
  Tensor out = at::empty({place.size(0), y.size(1)}, y.options().dtype(type).requires_grad(false));
  check(lapsum_expert_combine(y.data_ptr(), dtype_of(y), y.size(0), y.size(1),
                              weights ? weights->data_ptr<float>() : nullptr, place.data_ptr<int32_t>(),
                              place.size(0), place.size(1), out.data_ptr(), dtype_of(out), stream_of(y)),
        "lapsum_expert_combine");
  return out;
}
bool of_combine(const Tensor& y, const Tensor& place, const OptTensor& weights) {
  return plain(y) && dtype_of(y) >= 0 && y.dim() == 2 && y.is_contiguous() && dense(place, at::kInt, y) &&
         place.dim() == 2 && (!weights || (dense(*weights, at::kFloat, y) && weights->sizes() == place.sizes()));
}
OptTensor expert_combine(const Tensor& y, const Tensor& place, const OptTensor& weights) {
  if (!of_combine(y, place, weights)) return std::nullopt;
  return combine(y, place, weights, y.scalar_type());
}

// What comes out of a backward has no gradient of its own: asking for one is an error.
void no_second(variable_list& grads, const char* what) {
  if (!at::GradMode::is_enabled()) return;
  for (Tensor& g : grads)
    if (g.defined())
      g = (*std::make_shared<torch::autograd::DelayedError>(what, 1))({g.detach().requires_grad_()})[0];
}

// autograd.ExpertMatmulFunction in native code.
struct MatmulNode : public torch::autograd::Function<MatmulNode> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, const Tensor& offsets,
                        const OptTensor& order, const OptTensor& place, int64_t top_k) {
    const Tensor xd = x.detach(), wd = w.detach();
    const Product p(xd, wd, offsets, order);
    ctx->save_for_backward({x, w, offsets, order ? *order : Tensor(), place ? *place : Tensor()});
    ctx->saved_data["top_k"] = top_k;
    ctx->set_materialize_grads(false);
    return product(xd, wd, offsets, order, top_k, p, x.scalar_type());
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    variable_list out(6);
    if (grads[0].defined()) in_engine([&] { vjp(ctx, grads[0], out); });
    no_second(out, "the gradient of expert_matmul is not differentiable");
    return out;
  }
  static void vjp(AutogradContext* ctx, Tensor g, variable_list& out) {
    const auto saved = ctx->get_saved_variables();
    const Tensor x = saved[0].detach(), w = saved[1].detach(), offsets = saved[2];
    const OptTensor order = saved[3].defined() ? OptTensor(saved[3]) : std::nullopt;
    const Product p(x, w, offsets, order);
    // (a saved-tensor hook can hand back any tensor)
    TORCH_CHECK_VALUE(p.ok && plain(g) && g.device() == x.device() && g.dim() == 2 && g.size(0) == p.rows &&
                          g.size(1) == p.out,
                      "the saved tensors must be those of the forward");
    const c10::DeviceGuard guard(x.device());
    const at::AutoDispatchBelowADInplaceOrView below;
    g = g.to(x.scalar_type()).contiguous();
    const int64_t top_k = ctx->saved_data["top_k"].toInt();
    if (ctx->needs_input_grad(0)) {
      const Tensor back = w.transpose(1, 2);
      const Product q(g, back, offsets, std::nullopt);
      TORCH_CHECK_VALUE(q.ok, "the saved weight must be that of the forward");
      if (!order) {
        out[0] = product(g, back, offsets, std::nullopt, 1, q, x.scalar_type());
      } else {   // a token's rows are summed before they are rounded
        const Tensor rows = product(g, back, offsets, std::nullopt, 1, q, at::kFloat);
        TORCH_CHECK_VALUE(of_combine(rows, saved[4], std::nullopt), "the saved place must be that of the forward");
        out[0] = combine(rows, saved[4], std::nullopt, x.scalar_type());
      }
    }
    if (ctx->needs_input_grad(1)) {
      const auto opt = w.options().requires_grad(false);
      const bool other = w.stride(1) == 1 && w.stride(2) != 1;
      Tensor grad = other ? at::empty({w.size(0), p.out, p.in}, opt).transpose(1, 2)
                          : at::empty({w.size(0), p.in, p.out}, opt);
      const int64_t strides[3] = {grad.stride(0), grad.stride(1), grad.stride(2)};
      const size_t need = lapsum_expert_matmul_weights_workspace_size(w.size(0), p.rows, p.in, p.out);
      Tensor ws = bytes(need, x);
      check(lapsum_expert_matmul_weights(x.data_ptr(), dtype_of(x), x.size(0), row_stride(x),
                                         order ? order->data_ptr<int32_t>() : nullptr, top_k,
                                         offsets.data_ptr<int32_t>(), w.size(0), p.rows, p.in, p.out, g.data_ptr(),
                                         p.out, grad.data_ptr(), strides, ptr(ws), need, stream_of(x)),
            "lapsum_expert_matmul_weights");
      out[1] = grad;
    }
  }
};

OptTensor expert_matmul_grad(const Tensor& x, const Tensor& w, const Tensor& offsets, const OptTensor& order,
                             const OptTensor& place, int64_t top_k) {
  const Product p(x, w, offsets, order);
  if (!p.ok || order.has_value() != place.has_value() ||
      (place && (!dense(*place, at::kInt, x) || place->dim() != 2 || place->size(0) != x.size(0))))
    return std::nullopt;
  return MatmulNode::apply(x, w, offsets, order, place, top_k);
}

// autograd.ExpertCombineFunction in native code.
struct CombineNode : public torch::autograd::Function<CombineNode> {
  static Tensor forward(AutogradContext* ctx, const Tensor& y, const Tensor& weights, const Tensor& place,
                        const Tensor& offsets) {
    ctx->save_for_backward({y, weights, place, offsets});
    ctx->set_materialize_grads(false);
    return combine(y.detach(), place, weights.detach(), y.scalar_type());
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    variable_list out(4);
    if (grads[0].defined()) in_engine([&] { vjp(ctx, grads[0], out); });
    no_second(out, "the gradient of expert_combine is not differentiable");
    return out;
  }
  static void vjp(AutogradContext* ctx, Tensor g, variable_list& out) {
    const auto saved = ctx->get_saved_variables();
    const Tensor y = saved[0].detach(), weights = saved[1].detach(), place = saved[2], offsets = saved[3];
    TORCH_CHECK_VALUE(of_combine(y, place, weights) && dense(offsets, at::kInt, y) && plain(g) &&
                          g.device() == y.device() && g.dim() == 2 && g.size(0) == place.size(0) &&
                          g.size(1) == y.size(1),
                      "the saved tensors must be those of the forward");
    const c10::DeviceGuard guard(y.device());
    const at::AutoDispatchBelowADInplaceOrView below;
    g = g.to(y.scalar_type()).contiguous();
    Tensor grad_y = at::empty(y.sizes(), y.options().requires_grad(false));
    Tensor grad_w = at::empty(weights.sizes(), weights.options().requires_grad(false));
    check(lapsum_expert_combine_backward(g.data_ptr(), y.data_ptr(), dtype_of(y), y.size(0), y.size(1),
                                         weights.data_ptr<float>(), place.data_ptr<int32_t>(),
                                         offsets.data_ptr<int32_t>(), offsets.numel() - 1, place.size(0),
                                         place.size(1), grad_y.data_ptr(), grad_w.data_ptr<float>(), stream_of(y)),
          "lapsum_expert_combine_backward");
    out[0] = grad_y;
    out[1] = grad_w;
  }
};

OptTensor expert_combine_grad(const Tensor& y, const Tensor& weights, const Tensor& place, const Tensor& offsets) {
  if (!of_combine(y, place, weights) || !dense(offsets, at::kInt, y) || offsets.dim() != 1 || offsets.numel() < 2)
    return std::nullopt;
  return CombineNode::apply(y, weights, place, offsets);
}

// A cache [pages, kv_heads, slots, dim] with dense rows, with its scales.
struct Paged {
  lapsum_paged c{};
  int kind = -1;
  Paged(const Tensor& x, const OptTensor& scale, bool written) {
    if (!plain(x) || x.dim() != 4 || (x.stride(3) != 1 && x.size(3) > 1)) return;
    const auto type = x.scalar_type();
    const int k = type == at::kChar ? LAPSUM_I8 : type == at::kFloat8_e4m3fn ? LAPSUM_E4M3 : dtype_of(x);
    if (k < 0 || (k >= LAPSUM_I8) != scale.has_value()) return;
    for (int i = 0; written && i < 3; ++i)
      if (x.stride(i) == 0 && x.size(i) > 1) return;
    c.data = x.data_ptr();
    c.pages = x.size(0);
    c.slots = x.size(2);
    c.stride_page = x.stride(0);
    c.stride_head = x.stride(1);
    c.stride_slot = x.stride(2);
    if (scale) {
      if (!dense(*scale, at::kFloat, x) || scale->dim() != 3 || scale->size(0) != x.size(0) ||
          scale->size(1) != x.size(1) || scale->size(2) != x.size(2))
        return;
      c.scale = scale->data_ptr<float>();
      c.scale_stride_page = scale->stride(0);
      c.scale_stride_head = scale->stride(1);
    }
    kind = k;
  }
};
bool of_batch(const Tensor& t, int64_t batch, const Tensor& like) {
  return dense(t, at::kInt, like) && t.dim() == 1 && t.size(0) == batch;
}
bool of_table(const OptTensor& t, int64_t batch, const Tensor& like) {
  return !t || (dense(*t, at::kInt, like) && t->dim() == 2 && t->size(0) == batch);
}
// (a table without pages has no address, and is not to be taken for none)
const int32_t* pages_of(const OptTensor& t) {
  static const int32_t none = 0;
  if (!t) return nullptr;
  return t->numel() ? t->data_ptr<int32_t>() : &none;
}
bool alike(const Tensor& a, const Tensor& b) {
  return a.sizes() == b.sizes() && a.scalar_type() == b.scalar_type() && a.device() == b.device();
}

bool cache_append(const Tensor& k_new, const Tensor& v_new, const Tensor& seen, const Tensor& k, const Tensor& v,
                  const OptTensor& table, const OptTensor& count, const OptTensor& k_scale,
                  const OptTensor& v_scale) {
  const Paged kc(k, k_scale, true), vc(v, v_scale, true);
  if (kc.kind < 0 || vc.kind < 0 || !alike(k, v) || !may_write(k) || !may_write(v) ||
      (k_scale && (!may_write(*k_scale) || !may_write(*v_scale))))
    return false;
  const int64_t nd = k_new.dim();
  if (!plain(k_new) || !plain(v_new) || !alike(k_new, v_new) || dtype_of(k_new) < 0 ||
      k_new.device() != k.device() || (nd != 3 && nd != 4) || k_new.size(1) != k.size(1) ||
      k_new.size(-1) != k.size(3) || (kc.kind < LAPSUM_I8 && kc.kind != dtype_of(k_new)))
    return false;
  const int64_t batch = k_new.size(0), fresh = nd == 4 ? k_new.size(2) : 1;
  int64_t strides[2][3];
  const Tensor* rows[2] = {&k_new, &v_new};
  for (int n = 0; n < 2; ++n) {
    const Tensor& x = *rows[n];
    if (x.stride(-1) != 1 && x.size(-1) > 1) return false;
    strides[n][0] = x.stride(0);
    strides[n][1] = x.stride(1);
    strides[n][2] = nd == 4 ? x.stride(2) : 0;
  }
  if (!of_batch(seen, batch, k) || (count && !of_batch(*count, batch, k)) || !of_table(table, batch, k))
    return false;
  const c10::DeviceGuard guard(k.device());
  check(lapsum_cache_append(k_new.data_ptr(), strides[0], v_new.data_ptr(), strides[1], dtype_of(k_new), batch,
                            k.size(1), fresh, k.size(3), seen.data_ptr<int32_t>(),
                            count ? count->data_ptr<int32_t>() : nullptr, &kc.c, &vc.c, kc.kind,
                            pages_of(table), table ? table->size(1) : 0,
                            stream_of(k)),
        "lapsum_cache_append");
  written(k);
  written(v);
  if (k_scale) {
    written(*k_scale);
    written(*v_scale);
  }
  return true;
}

// What has no gradient, from inputs of which one requires it in grad mode: asking for it is an error.
bool recorded(std::initializer_list<const Tensor*> inputs) {
  if (!at::GradMode::is_enabled()) return false;
  for (const Tensor* t : inputs)
    if (t && t->requires_grad()) return true;
  return false;
}
const Tensor* maybe(const OptTensor& t) { return t ? &*t : nullptr; }
variable_list no_gradient(variable_list outputs, const char* what) {
  for (Tensor& t : outputs) t = t.detach().requires_grad_();
  const auto count = static_cast<int64_t>(outputs.size());
  return (*std::make_shared<torch::autograd::DelayedError>(what, count))(std::move(outputs));
}

OptTensor cache_read(const Tensor& x, const Tensor& lens, int64_t room, const OptTensor& table,
                     const OptTensor& scale, const std::optional<at::ScalarType>& dtype) {
  const Paged c(x, scale, false);
  if (c.kind < 0 || !plain(lens) || lens.dim() != 1 || room < 0) return std::nullopt;
  const int64_t batch = lens.size(0);
  const at::ScalarType to = dtype ? *dtype : c.kind >= LAPSUM_I8 ? at::kFloat : x.scalar_type();
  if (!of_batch(lens, batch, x) || !of_table(table, batch, x) || (c.kind < LAPSUM_I8 && to != x.scalar_type()) ||
      (to != at::kFloat && to != at::kBFloat16 && to != at::kHalf))
    return std::nullopt;
  const c10::DeviceGuard guard(x.device());
  Tensor out = at::empty({batch, x.size(1), room, x.size(3)}, x.options().dtype(to).requires_grad(false));
  check(lapsum_cache_read(&c.c, c.kind, batch, x.size(1), room, x.size(3), lens.data_ptr<int32_t>(),
                          pages_of(table), table ? table->size(1) : 0,
                          out.data_ptr(), dtype_of(out), stream_of(x)),
        "lapsum_cache_read");
  if (recorded({&x, maybe(scale)})) return no_gradient({out}, "lapsum_cache_read has no gradient")[0];
  return out;
}

std::optional<std::vector<Tensor>> cache_attend(const Tensor& q, const Tensor& k, const Tensor& v,
                                                const Tensor& lens, const OptTensor& table,
                                                const OptTensor& k_scale, const OptTensor& v_scale,
                                                std::optional<double> scale, int64_t window, bool lse,
                                                bool weights) {
  const Paged kc(k, k_scale, false), vc(v, v_scale, false);
  const int64_t nd = q.dim();
  if (kc.kind < 0 || vc.kind < 0 || !alike(k, v) || !plain(q) || dtype_of(q) < 0 || q.device() != k.device() ||
      !(nd == 3 || (nd == 4 && q.size(2) == 1)) || q.size(-1) != k.size(3) ||
      (q.stride(-1) != 1 && q.size(-1) > 1) || (kc.kind < LAPSUM_I8 && kc.kind != dtype_of(q)) || window < 0)
    return std::nullopt;
  const int64_t batch = q.size(0), heads = q.size(1), kv = k.size(1), dim = k.size(3);
  const double by = scale ? *scale : 1.0 / std::sqrt(static_cast<double>(dim));
  if (kv < 1 || heads % kv || !of_batch(lens, batch, q) || !of_table(table, batch, q) || !std::isfinite(by))
    return std::nullopt;
  const c10::DeviceGuard guard(q.device());
  const auto opt = q.options().requires_grad(false);
  const int64_t width = table ? table->size(1) : 0, room = table ? width * k.size(2) : k.size(2);
  std::vector<Tensor> found{at::empty(q.sizes(), opt)};
  Tensor total, w;
  if (lse || weights) total = at::empty({batch, heads}, opt.dtype(at::kFloat));
  if (weights) w = at::empty({batch, heads, room}, opt.dtype(at::kFloat));
  const size_t need = lapsum_cache_attend_workspace_size(batch, heads, kv, dim, room, window);
  Tensor ws = bytes(need, q);
  check(lapsum_cache_attend(q.data_ptr(), q.stride(0), q.stride(1), dtype_of(q), &kc.c, &vc.c, kc.kind, batch, heads,
                            kv, dim, lens.data_ptr<int32_t>(), pages_of(table), width,
                            by, window, found[0].data_ptr(), static_cast<float*>(ptr(total)),
                            static_cast<float*>(ptr(w)), ptr(ws), need, stream_of(q)),
        "lapsum_cache_attend");
  if (lse) found.push_back(total);
  if (weights) found.push_back(w);
  if (recorded({&q, &k, &v, maybe(k_scale), maybe(v_scale)}))
    return no_gradient(std::move(found), "lapsum_cache_attend has no gradient");
  return found;
}

}  // namespace

void bind_products(py::module_& m) {
  m.def("expert_order", lapsum_node::entry(expert_order));
  m.def("expert_matmul", lapsum_node::entry(expert_matmul));
  m.def("expert_matmul_grad", lapsum_node::entry(expert_matmul_grad));
  m.def("expert_combine", lapsum_node::entry(expert_combine));
  m.def("expert_combine_grad", lapsum_node::entry(expert_combine_grad));
  m.def("cache_append", lapsum_node::entry(cache_append));
  m.def("cache_read", lapsum_node::entry(cache_read));
  m.def("cache_attend", lapsum_node::entry(cache_attend));
}
