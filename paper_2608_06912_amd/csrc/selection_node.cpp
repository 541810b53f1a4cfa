// The hard selections' calls in native code: the common case of each (plain
// tensors of the right type, shape and device) straight to the C ABI, and the
// autograd node of the routing's weights.  The binding in selection.py does the
// same through ctypes with 5 to 10 us more host time per call, which is more
// than the kernels of a single-token step take; whatever a function here does
// not take (it returns None) goes there, where it is checked and refused.
#include "node.hpp"

#include <torch/csrc/autograd/functions/basic_ops.h>

namespace {

using namespace lapsum_node;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// Logits as rows: contiguous, or two dimensions with dense rows.
struct Rows {
  int64_t rows = 0, n = 0, stride = 0;
  bool ok = false;
  explicit Rows(const Tensor& x) {
    if (!plain(x) || x.dim() < 1 || dtype_of(x) < 0) return;
    n = x.size(-1);
    if (n < 1) return;
    if (x.is_contiguous()) {
      rows = x.numel() / n;
      stride = n;
      ok = true;
    } else if (x.dim() == 2 && x.stride(1) == 1 && x.stride(0) >= n) {
      rows = x.size(0);
      stride = x.stride(0);
      ok = true;
    }
  }
};

struct RouteOptions {
  int64_t top_k;
  int score;
  int64_t groups, topk_groups, group_top;
  bool renormalise;
  double scale;
  bool counts;
};

variable_list route_forward(const Tensor& logits, const OptTensor& bias, const RouteOptions& o) {
  const c10::DeviceGuard guard(logits.device());
  const Rows x(logits);
  const auto opt = logits.options().requires_grad(false);
  std::vector<int64_t> size(logits.sizes().begin(), logits.sizes().end());
  size.back() = o.top_k;
  Tensor weights = at::empty(size, opt.dtype(at::kFloat));
  Tensor indices = at::empty(size, opt.dtype(at::kInt));
  Tensor counts, ws;
  size_t need = 0;
  if (o.counts) {
    counts = at::empty({x.n}, opt.dtype(at::kInt));
    need = lapsum_route_forward_workspace_size(x.rows, x.n, o.top_k, o.groups, 1);
    ws = bytes(need, logits);
  }
  check(lapsum_route_forward(logits.data_ptr(), dtype_of(logits), x.rows, x.n, x.stride, o.score,
                             bias ? bias->data_ptr<float>() : nullptr, o.groups, o.topk_groups,
                             o.group_top, o.top_k, o.renormalise, o.scale, weights.data_ptr<float>(),
                             indices.data_ptr<int32_t>(), static_cast<int32_t*>(ptr(counts)), ptr(ws),
                             need, stream_of(logits)),
        "lapsum_route_forward");
  variable_list out{weights, indices};
  if (o.counts) out.push_back(counts);
  return out;
}

struct RouteNode : public torch::autograd::Function<RouteNode> {
  static variable_list forward(AutogradContext* ctx, const Tensor& logits, const OptTensor& bias,
                               const RouteOptions* o) {
    variable_list out = route_forward(logits.detach(), bias, *o);
    ctx->save_for_backward({logits, out[1]});
    ctx->set_materialize_grads(false);
    ctx->saved_data["score"] = static_cast<int64_t>(o->score);
    ctx->saved_data["renormalise"] = o->renormalise;
    ctx->saved_data["scale"] = o->scale;
    ctx->mark_non_differentiable(variable_list(out.begin() + 1, out.end()));
    return out;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    Tensor grad;
    if (grads[0].defined())
      grad = lapsum_node::in_engine([&] { return vjp(ctx, grads[0]); });
    // what comes out has no gradient of its own: asking for one is an error
    if (grad.defined() && at::GradMode::is_enabled()) {
      auto error = std::make_shared<torch::autograd::DelayedError>(
          "the gradient of route_topk is not differentiable", 1);
      grad = (*error)({grad.detach().requires_grad_()})[0];
    }
    return {grad, Tensor(), Tensor()};
  }

  static Tensor vjp(AutogradContext* ctx, Tensor g) {
    const auto saved = ctx->get_saved_variables();
    const Tensor logits = saved[0].detach(), indices = saved[1];
    const Rows x(logits);
    // (a saved-tensor hook can hand back any tensor)
    TORCH_CHECK_VALUE(x.ok && dense(indices, at::kInt, logits) && plain(g) && g.device() == logits.device() &&
                          g.sizes() == indices.sizes() && indices.numel() / indices.size(-1) == x.rows,
                      "the saved logits and indices must be those of the forward");
    const c10::DeviceGuard guard(logits.device());
    const at::AutoDispatchBelowADInplaceOrView below;
    if (g.scalar_type() != at::kFloat) g = g.to(at::kFloat);
    g = g.contiguous();
    Tensor grad = at::empty(logits.sizes(), logits.options().requires_grad(false));
    check(lapsum_route_backward(g.data_ptr<float>(), logits.data_ptr(), dtype_of(logits), x.rows, x.n,
                                x.stride, indices.data_ptr<int32_t>(),
                                static_cast<int>(ctx->saved_data["score"].toInt()), indices.size(-1),
                                ctx->saved_data["renormalise"].toBool(),
                                ctx->saved_data["scale"].toDouble(), grad.data_ptr(), stream_of(logits)),
          "lapsum_route_backward");
    return grad;
  }
};

std::optional<variable_list> route(const Tensor& logits, int64_t top_k, int score, const OptTensor& bias,
                                   int64_t groups, int64_t topk_groups, int64_t group_top,
                                   bool renormalise, double scale, bool counts, bool grad) {
  const Rows x(logits);
  if (!x.ok || top_k < 1 || top_k > x.n) return std::nullopt;
  if (bias && !(dense(*bias, at::kFloat, logits) && bias->dim() == 1 && bias->size(0) == x.n))
    return std::nullopt;
  const RouteOptions o{top_k, score, groups, topk_groups, group_top, renormalise, scale, counts};
  if (!grad) return route_forward(logits, bias, o);
  if (!logits.is_contiguous()) return std::nullopt;
  return RouteNode::apply(logits, bias, &o);
}

std::optional<std::tuple<Tensor, Tensor, Tensor>> beam_select(const Tensor& logits, const Tensor& cum,
                                                              int64_t num) {
  const Rows x(logits);
  if (!x.ok || !dense(cum, at::kFloat, logits) || cum.dim() != 2 || x.rows != cum.numel() || num < 1)
    return std::nullopt;
  const c10::DeviceGuard guard(logits.device());
  const int64_t batch = cum.size(0), beams = cum.size(1);
  const auto opt = logits.options().requires_grad(false);
  Tensor scores = at::empty({batch, num}, opt.dtype(at::kFloat));
  Tensor both = at::empty({2, batch, num}, opt.dtype(at::kInt));
  Tensor tokens = both.select(0, 0), parents = both.select(0, 1);
  const size_t need = lapsum_beam_select_workspace_size(batch, beams, x.n, num);
  Tensor ws = bytes(need, logits);
  check(lapsum_beam_select(logits.data_ptr(), dtype_of(logits), batch, beams, x.n, x.stride,
                           cum.data_ptr<float>(), num, scores.data_ptr<float>(),
                           tokens.data_ptr<int32_t>(), parents.data_ptr<int32_t>(), ptr(ws), need,
                           stream_of(logits)),
        "lapsum_beam_select");
  return std::make_tuple(scores, tokens, parents);
}

bool beam_reorder(const std::vector<Tensor>& states, const Tensor& parents, std::optional<int64_t> length,
                  const std::vector<Tensor>& outs) {
  if (!plain(parents) || parents.scalar_type() != at::kInt || parents.dim() != 2 ||
      (parents.size(1) > 1 && parents.stride(1) != 1) || states.size() != outs.size() || states.empty())
    return false;
  const int64_t batch = parents.size(0), beams = parents.size(1);
  if (batch < 1) return false;
  std::vector<lapsum_beam_state> items(states.size());
  for (size_t i = 0; i < states.size(); ++i) {
    const Tensor &s = states[i], &o = outs[i];
    if (!dense(s, s.scalar_type(), parents) || s.dim() < 1 || s.size(0) != batch * beams ||
        !dense(o, s.scalar_type(), parents) || o.sizes() != s.sizes() || !may_write(o))
      return false;
    const int64_t size = s.element_size(), row = s.numel() / s.size(0) * size;
    items[i] = {s.data_ptr(), o.data_ptr(), row, 1, row, row};
    if (length) {
      if (s.dim() < 3 || *length < 0 || *length > s.size(-2)) return false;
      const int64_t piece = s.size(-2) * s.size(-1) * size;
      items[i].outer = piece ? row / piece : 0;
      items[i].outer_stride = piece;
      items[i].live_bytes = *length * s.size(-1) * size;
    }
  }
  const c10::DeviceGuard guard(parents.device());
  check(lapsum_beam_reorder(items.data(), static_cast<int64_t>(items.size()), parents.data_ptr<int32_t>(),
                            batch > 1 ? parents.stride(0) : beams, batch, beams, stream_of(parents)),
        "lapsum_beam_reorder");
  for (const Tensor& o : outs) written(o);
  return true;
}

OptTensor cache_accumulate(const Tensor& w, int64_t kv, const OptTensor& seen, const OptTensor& acc) {
  if (!plain(w) || dtype_of(w) < 0 || w.dim() != 4 || kv < 1 || (w.stride(3) != 1 && w.size(3) > 1))
    return std::nullopt;
  const int64_t batch = w.size(0), keys = w.size(3);
  if (seen && !(dense(*seen, at::kInt, w) && seen->dim() == 1 && seen->size(0) == batch)) return std::nullopt;
  if (acc && !(dense(*acc, at::kFloat, w) && acc->dim() == 3 && acc->size(0) == batch &&
               acc->size(1) == kv && acc->size(2) == keys && may_write(*acc)))
    return std::nullopt;
  const c10::DeviceGuard guard(w.device());
  Tensor out = acc ? *acc : at::empty({batch, kv, keys}, w.options().dtype(at::kFloat).requires_grad(false));
  check(lapsum_cache_accumulate(w.data_ptr(), dtype_of(w), batch, w.size(1), kv, w.size(2), keys,
                                w.stride(0), w.stride(1), w.stride(2),
                                seen ? seen->data_ptr<int32_t>() : nullptr,
                                acc ? acc->data_ptr<float>() : nullptr, out.data_ptr<float>(),
                                stream_of(w)),
        "lapsum_cache_accumulate");
  if (acc) written(out);
  return out;
}

// A cache [batch, kv_heads, slots, dim] with dense rows, its strides in bytes.
struct Cache {
  int64_t strides[3];
  bool ok = false;
  Cache(const Tensor& x, bool written) {
    if (!plain(x) || x.dim() != 4 || (x.stride(3) != 1 && x.size(3) > 1) || x.size(3) < 1) return;
    for (int i = 0; i < 3; ++i) {
      if (written && x.stride(i) == 0 && x.size(i) > 1) return;
      strides[i] = x.stride(i) * x.element_size();
    }
    ok = true;
  }
};
bool of_cache(const Tensor& t, at::ScalarType type, const Tensor& k) {
  return dense(t, type, k) && t.dim() == 3 && t.size(0) == k.size(0) && t.size(1) == k.size(1) &&
         t.size(2) == k.size(2);
}

std::optional<std::tuple<Tensor, Tensor, Tensor, Tensor>> cache_evict(
    const Tensor& k, const Tensor& v, const Tensor& acc, const Tensor& seen, int64_t budget, int64_t sink,
    int64_t recent, const OptTensor& pos) {
  const Cache kc(k, false), vc(v, false);
  if (!kc.ok || !vc.ok || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type() ||
      v.device() != k.device() || !of_cache(acc, at::kFloat, k) || !dense(seen, at::kInt, k) ||
      seen.dim() != 1 || seen.size(0) != k.size(0) || (pos && !of_cache(*pos, at::kInt, k)) || budget < 1)
    return std::nullopt;
  const int64_t batch = k.size(0), kv = k.size(1), slots = k.size(2), dim = k.size(3);
  const c10::DeviceGuard guard(k.device());
  const auto opt = k.options().requires_grad(false);
  Tensor k_out = at::empty({batch, kv, budget, dim}, opt), v_out = at::empty({batch, kv, budget, dim}, opt);
  Tensor acc_out = at::empty({batch, kv, budget}, opt.dtype(at::kFloat));
  Tensor pos_out = at::empty({batch, kv, budget}, opt.dtype(at::kInt));
  const size_t need = lapsum_cache_evict_workspace_size(batch, kv, slots, budget);
  Tensor ws = bytes(need, k);
  check(lapsum_cache_evict(k.data_ptr(), kc.strides, v.data_ptr(), vc.strides, dim * k.element_size(),
                           acc.data_ptr<float>(), pos ? pos->data_ptr<int32_t>() : nullptr,
                           seen.data_ptr<int32_t>(), batch, kv, slots, budget, sink, recent,
                           k_out.data_ptr(), v_out.data_ptr(), acc_out.data_ptr<float>(),
                           pos_out.data_ptr<int32_t>(), ptr(ws), need, stream_of(k)),
        "lapsum_cache_evict");
  return std::make_tuple(k_out, v_out, acc_out, pos_out);
}

OptTensor cache_step(const Tensor& weights, const Tensor& k_new, const Tensor& v_new, const Tensor& seen,
                     const Tensor& k, const Tensor& v, const Tensor& acc, const Tensor& pos, int64_t sink,
                     int64_t recent) {
  const Cache kc(k, true), vc(v, true);
  if (!kc.ok || !vc.ok || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type() ||
      v.device() != k.device() || !of_cache(acc, at::kFloat, k) || !of_cache(pos, at::kInt, k) ||
      !dense(seen, at::kInt, k) || seen.dim() != 1 || seen.size(0) != k.size(0) || !may_write(k) ||
      !may_write(v) || !may_write(acc))
    return std::nullopt;
  const int64_t batch = k.size(0), kv = k.size(1), slots = k.size(2), dim = k.size(3);
  const int64_t wd = weights.dim();
  if (!plain(weights) || dtype_of(weights) < 0 || weights.device() != k.device() ||
      !(wd == 3 || (wd == 4 && weights.size(2) == 1)) || weights.size(0) != batch ||
      weights.size(-1) != slots || (weights.stride(-1) != 1 && slots > 1))
    return std::nullopt;
  for (const Tensor* x : {&k_new, &v_new})
    if (!dense(*x, k.scalar_type(), k) || !(x->dim() == 3 || (x->dim() == 4 && x->size(2) == 1)) ||
        x->size(0) != batch || x->size(1) != kv || x->size(-1) != dim)
      return std::nullopt;
  const c10::DeviceGuard guard(k.device());
  Tensor slot = at::empty({batch, kv}, k.options().dtype(at::kInt).requires_grad(false));
  check(lapsum_cache_step(weights.data_ptr(), dtype_of(weights), weights.stride(0), weights.stride(1),
                          k_new.data_ptr(), v_new.data_ptr(), seen.data_ptr<int32_t>(), k.data_ptr(),
                          kc.strides, v.data_ptr(), vc.strides, dim * k.element_size(),
                          acc.data_ptr<float>(), pos.data_ptr<int32_t>(), batch, weights.size(1), kv,
                          slots, sink, recent, slot.data_ptr<int32_t>(), stream_of(k)),
        "lapsum_cache_step");
  for (const Tensor* t : {&k, &v, &acc, &pos}) written(*t);
  return slot;
}

}  // namespace

void bind_selection(py::module_& m) {
  m.def("route", lapsum_node::entry(route));
  m.def("beam_select", lapsum_node::entry(beam_select));
  m.def("beam_reorder", lapsum_node::entry(beam_reorder));
  m.def("cache_accumulate", lapsum_node::entry(cache_accumulate));
  m.def("cache_evict", lapsum_node::entry(cache_evict));
  m.def("cache_step", lapsum_node::entry(cache_step));
}
