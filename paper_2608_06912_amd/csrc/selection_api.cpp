// Host side of the hard selections: argument checks, workspace carving and
// launch order of routing, beam search and the bounded cache.
#include <math.h>

#include <algorithm>
#include <memory>
#include <new>

#include "host.hpp"
#include "kernels.hpp"

using namespace lapsum;

namespace {

constexpr int64_t kMaxBlocks = int64_t(1) << 23;   // workgroups of a launch

bool valid_dtype(int dtype) { return dtype >= LAPSUM_F32 && dtype <= LAPSUM_F16; }

bool int32_range(int64_t v) { return v >= 0 && v <= 2147483647LL; }

// The widest power of two, up to 16, that divides everything or'ed into bits.
int vector_width(uint64_t bits) {
  int w = 16;
  while (w > 1 && bits % static_cast<uint64_t>(w)) w /= 2;
  return w;
}
uint64_t bits_of(const void* p) { return reinterpret_cast<uintptr_t>(p); }
uint64_t bits_of(const int64_t* strides) {
  return static_cast<uint64_t>(strides[0] | strides[1] | strides[2]);
}

bool valid_route(int dtype, int64_t tokens, int64_t experts, int64_t row_stride, int score,
                 int64_t top_k, double scale) {
  return valid_dtype(dtype) && tokens >= 0 && experts >= 1 && experts <= kRouteMaxExperts &&
         row_stride >= experts && (score == 0 || score == 1) && top_k >= 1 && top_k <= experts &&
         top_k <= kRouteMaxTop && isfinite(scale);
}

struct BeamWs {
  float* tops;
  double *refs, *sums;
};
BeamWs carve_beam(Carve& c, int64_t rows, int64_t row_steps, int64_t parts) {
  BeamWs w{};
  w.tops = c.take<float>(static_cast<size_t>(rows * row_steps));
  w.refs = c.take<double>(static_cast<size_t>(rows * parts));
  w.sums = c.take<double>(static_cast<size_t>(rows * parts));
  return w;
}
bool valid_beam(int64_t batch, int64_t beams, int64_t vocab, int64_t num) {
  return batch >= 0 && beams >= 1 && beams <= kBeamMaxBeams && batch <= 65535 / beams && vocab >= 1 &&
         vocab <= 2147483647LL / beams && num >= 1 && num <= kBeamMaxNum;
}

// What a reorder reads or writes of a state: `rows` rows, of each `outer` pieces.
struct Region {
  uint64_t begin, row, outer, stride, live;
  bool write;
  uint64_t extent() const { return (outer - 1) * stride + live; }   // of a row
  unsigned __int128 end(uint64_t rows) const {
    return static_cast<unsigned __int128>(rows - 1) * row + begin + extent();
  }
};
// Two that begin in this order and have no byte in common: one ends before the
// other begins, or they lie side by side in each row, or in each piece's stride
// (regions of other strides that reach into one another count as overlapping).
bool apart(const Region& a, const Region& b, uint64_t rows) {
  if (a.end(rows) <= b.begin) return true;
  uint64_t d = b.begin - a.begin;
  if (rows > 1) {
    if (a.row != b.row) return false;
    d %= a.row;   // (a row holds a piece: not 0)
    if (d >= a.extent() && d + b.extent() <= a.row) return true;
  }
  const uint64_t stride = a.outer > 1 ? a.stride : b.stride;
  if ((a.outer == 1 && b.outer == 1) || (a.outer > 1 && b.outer > 1 && a.stride != b.stride) ||
      (rows > 1 && a.row % stride))
    return false;
  d %= stride;
  return d >= a.live && d + b.live <= stride;
}
// Whether nothing that is written is read or written as another state, as the
// same state's other side or as the parents (4-byte, `parents_count` from the
// first to the last): the threads that move a column know only their own.
bool none_shared(const lapsum_beam_state* states, int64_t count, uint64_t rows, const int32_t* parents,
                 uint64_t parents_count) {
  const std::unique_ptr<Region[]> all(new (std::nothrow) Region[2 * static_cast<size_t>(count) + 1]);
  if (!all) return false;
  all[0] = Region{bits_of(parents), 0, 1, 0, 4 * parents_count, false};
  size_t n = 1;
  for (int64_t t = 0; t < count; ++t) {
    const lapsum_beam_state& s = states[t];
    if (s.outer == 0 || s.live_bytes == 0) continue;
    const Region r{bits_of(s.out), static_cast<uint64_t>(s.row_bytes), static_cast<uint64_t>(s.outer),
                   static_cast<uint64_t>(s.outer > 1 ? s.outer_stride : 0),
                   static_cast<uint64_t>(s.live_bytes), true};
    all[n++] = r;
    if (s.in == s.out) continue;
    all[n] = r;
    all[n].begin = bits_of(s.in);
    all[n++].write = false;
  }
  std::sort(all.get(), all.get() + n, [](const Region& a, const Region& b) { return a.begin < b.begin; });
  for (size_t i = 0; i < n; ++i) {
    const unsigned __int128 end = all[i].end(rows);
    for (size_t j = i + 1; j < n && all[j].begin < end; ++j)
      if ((all[i].write || all[j].write) && !apart(all[i], all[j], rows)) return false;
  }
  return true;
}

bool valid_cache(int64_t batch, int64_t kv, int64_t slots, int64_t sink, int64_t recent) {
  return batch >= 0 && kv >= 1 && slots >= 1 && int32_range(slots) && int32_range(sink) &&
         int32_range(recent) && (batch == 0 || kv <= kMaxBlocks / batch);
}

}  // namespace

extern "C" {

// --------------------------------------------------------------- routing --
size_t lapsum_route_forward_workspace_size(int64_t tokens, int64_t experts, int64_t top_k,
                                           int64_t groups, int with_counts) {
  if (!with_counts || tokens < 1 || experts < 1 || experts > kRouteMaxExperts) return 0;
  const int64_t blocks = route_blocks(tokens, static_cast<int>(experts), static_cast<int>(top_k),
                                      static_cast<int>(groups));
  if (blocks <= 1) return 0;
  Carve c(nullptr);
  c.take<int>(static_cast<size_t>(blocks * experts));
  return c.size();
}

int lapsum_route_forward(const void* logits, int dtype, int64_t tokens, int64_t experts,
                         int64_t row_stride, int score, const float* bias, int64_t groups,
                         int64_t topk_groups, int64_t group_top, int64_t top_k, int renormalise,
                         double scale, float* weights, int32_t* indices, int32_t* counts,
                         void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!valid_route(dtype, tokens, experts, row_stride, score, top_k, scale))
    return LAPSUM_ERR_INVALID_ARG;
  if (groups < 1 || groups > kRouteMaxGroups || experts % groups || topk_groups < 1 ||
      topk_groups > groups || group_top < 1 || group_top > 2 || group_top > experts / groups ||
      top_k > topk_groups * (experts / groups))
    return LAPSUM_ERR_INVALID_ARG;
  if (tokens > 0 && (!logits || !weights || !indices)) return LAPSUM_ERR_INVALID_ARG;
  const int wst = check_ws(workspace, workspace_bytes,
                           lapsum_route_forward_workspace_size(tokens, experts, top_k, groups, counts != nullptr));
  if (wst != LAPSUM_OK) return wst;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (tokens == 0) {
    if (counts) LAPSUM_TRY(launch_fill_u32(reinterpret_cast<uint32_t*>(counts), experts, 0u, stream));
    return LAPSUM_OK;
  }
  RouteArgs a{};
  a.logits = logits;
  a.tokens = tokens;
  a.stride = row_stride;
  a.experts = static_cast<int>(experts);
  a.score = score;
  a.renorm = renormalise != 0;
  a.top_k = static_cast<int>(top_k);
  // (all groups chosen: no group is left out)
  a.groups = topk_groups == groups ? 1 : static_cast<int>(groups);
  a.topk_groups = static_cast<int>(topk_groups);
  a.group_top = static_cast<int>(group_top);
  a.scale = static_cast<float>(scale);
  a.bias = bias;
  a.weights = weights;
  a.indices = indices;
  a.counts = counts;
  LAPSUM_TRY(launch_route_forward(a, dtype, static_cast<int*>(workspace), stream));
  return LAPSUM_OK;
}

int lapsum_route_backward(const float* grad_weights, const void* logits, int dtype, int64_t tokens,
                          int64_t experts, int64_t row_stride, const int32_t* indices, int score,
                          int64_t top_k, int renormalise, double scale, void* grad_logits,
                          hipStream_t stream) {
  if (!valid_route(dtype, tokens, experts, row_stride, score, top_k, scale))
    return LAPSUM_ERR_INVALID_ARG;
  if (tokens > 0 && (!grad_weights || !logits || !indices || !grad_logits))
    return LAPSUM_ERR_INVALID_ARG;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (tokens == 0) return LAPSUM_OK;
  RouteGradArgs a{};
  a.logits = logits;
  a.tokens = tokens;
  a.stride = row_stride;
  a.experts = static_cast<int>(experts);
  a.score = score;
  a.renorm = renormalise != 0;
  a.top_k = static_cast<int>(top_k);
  a.scale = static_cast<float>(scale);
  a.grad = grad_weights;
  a.indices = indices;
  a.grad_logits = grad_logits;
  LAPSUM_TRY(launch_route_backward(a, dtype, stream));
  return LAPSUM_OK;
}

// ----------------------------------------------------------- beam search --
size_t lapsum_beam_select_workspace_size(int64_t batch, int64_t beams, int64_t vocab, int64_t num) {
  if (batch < 1 || !valid_beam(batch, beams, vocab, num)) return 0;
  int steps = 0, parts = 0;
  int64_t row_steps = 0;
  beam_plan(batch * beams, vocab, &steps, &row_steps, &parts);
  Carve c(nullptr);
  carve_beam(c, batch * beams, row_steps, parts);
  return c.size();
}

int lapsum_beam_select(const void* logits, int dtype, int64_t batch, int64_t beams, int64_t vocab,
                       int64_t row_stride, const float* beam_scores, int64_t num, float* scores,
                       int32_t* tokens, int32_t* parents, void* workspace, size_t workspace_bytes,
                       hipStream_t stream) {
  if (!valid_dtype(dtype) || !valid_beam(batch, beams, vocab, num) || row_stride < vocab)
    return LAPSUM_ERR_INVALID_ARG;
  if (batch > 0 && (!logits || !beam_scores || !scores || !tokens || !parents))
    return LAPSUM_ERR_INVALID_ARG;
  const int wst = check_ws(workspace, workspace_bytes,
                           lapsum_beam_select_workspace_size(batch, beams, vocab, num));
  if (wst != LAPSUM_OK) return wst;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (batch == 0) return LAPSUM_OK;
  BeamArgs a{};
  a.logits = logits;
  a.stride = row_stride;
  a.vocab = vocab;
  a.batch = batch;
  a.beams = static_cast<int>(beams);
  a.num = static_cast<int>(num);
  a.cum = beam_scores;
  a.scores = scores;
  a.tokens = tokens;
  a.parents = parents;
  beam_plan(batch * beams, vocab, &a.steps, &a.row_steps, &a.parts);
  Carve c(workspace);
  const BeamWs w = carve_beam(c, batch * beams, a.row_steps, a.parts);
  a.tops = w.tops;
  a.refs = w.refs;
  a.sums = w.sums;
  LAPSUM_TRY(launch_beam_select(a, dtype, stream));
  return LAPSUM_OK;
}

int lapsum_beam_reorder(const lapsum_beam_state* states, int64_t count, const int32_t* parents,
                        int64_t parent_stride, int64_t batch, int64_t beams, hipStream_t stream) {
  if (count < 0 || batch < 0 || batch > 65535 || beams < 1 || beams > kBeamMaxBeams ||
      parent_stride < beams || (count > 0 && !states) || (batch > 0 && !parents))
    return LAPSUM_ERR_INVALID_ARG;
  for (int64_t t = 0; t < count; ++t) {
    const lapsum_beam_state& s = states[t];
    if (s.outer < 0 || s.live_bytes < 0 || s.outer_stride < 0 || s.row_bytes < 0)
      return LAPSUM_ERR_INVALID_ARG;
    if (s.outer == 0 || s.live_bytes == 0) continue;
    // (pieces that overlap would be written twice)
    if (!s.in || !s.out || (s.outer > 1 && s.outer_stride < s.live_bytes) ||
        s.outer > (int64_t(1) << 40) / s.live_bytes || s.outer_stride > (int64_t(1) << 50) / s.outer ||
        s.row_bytes < (s.outer - 1) * s.outer_stride + s.live_bytes)
      return LAPSUM_ERR_INVALID_ARG;
  }
  if (batch > 0 && !none_shared(states, count, static_cast<uint64_t>(batch * beams), parents,
                                static_cast<uint64_t>((batch - 1) * parent_stride + beams)))
    return LAPSUM_ERR_INVALID_ARG;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (batch == 0) return LAPSUM_OK;
  // states of one launch share a vector width, the widest that fits all
  ReorderArgs a{};
  a.beams = static_cast<int>(beams);
  a.parents = parents;
  a.parent_stride = parent_stride;
  uint64_t bits = 0;
  int64_t bytes = 0;
  const auto flush = [&]() -> hipError_t {
    if (a.count == 0) return hipSuccess;
    const int width = vector_width(bits);
    for (int q = 0; q < a.count; ++q) {
      a.state[q].row /= width;
      a.state[q].outer_stride /= width;
      a.state[q].live /= width;
    }
    const hipError_t e = launch_beam_reorder(a, batch, width, stream);
    a.count = 0;
    bits = 0;
    bytes = 0;
    return e;
  };
  for (int64_t t = 0; t < count; ++t) {
    const lapsum_beam_state& s = states[t];
    if (s.outer == 0 || s.live_bytes == 0) continue;
    // a launch's workgroups stay below 2^23 even where its vectors are bytes
    if (a.count == kReorderStates || bytes + s.outer * s.live_bytes > (int64_t(1) << 30))
      LAPSUM_TRY(flush());
    ReorderState& r = a.state[a.count++];
    r.in = s.in;
    r.out = s.out;
    r.row = s.row_bytes;
    r.outer = s.outer;
    r.outer_stride = s.outer > 1 ? s.outer_stride : 0;
    r.live = s.live_bytes;
    bits |= bits_of(s.in) | bits_of(s.out) | static_cast<uint64_t>(r.row | r.outer_stride | r.live);
    bytes += s.outer * s.live_bytes;
  }
  LAPSUM_TRY(flush());
  return LAPSUM_OK;
}

// ----------------------------------------------------------------- cache --
int lapsum_cache_accumulate(const void* weights, int dtype, int64_t batch, int64_t heads,
                            int64_t kv_heads, int64_t queries, int64_t keys, int64_t stride_batch,
                            int64_t stride_head, int64_t stride_query, const int32_t* seen,
                            const float* acc_in, float* acc, hipStream_t stream) {
  if (!valid_dtype(dtype) || batch < 0 || kv_heads < 1 || heads < 1 || heads % kv_heads ||
      queries < 0 || keys < 0 || !int32_range(keys) || stride_batch < 0 || stride_head < 0 ||
      stride_query < 0)
    return LAPSUM_ERR_INVALID_ARG;
  // (the rows of one sum are counted in 32 bits)
  if (queries > (int64_t(1) << 30) / (heads / kv_heads)) return LAPSUM_ERR_INVALID_ARG;
  const bool work = batch > 0 && keys > 0;
  if (work && (!acc || (queries > 0 && !weights))) return LAPSUM_ERR_INVALID_ARG;
  if (work && (kv_heads > kMaxBlocks / batch || batch * kv_heads > kMaxBlocks / ((keys + 255) / 256)))
    return LAPSUM_ERR_INVALID_ARG;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (!work) return LAPSUM_OK;
  AccumulateArgs a{};
  a.weights = weights;
  a.stride_b = stride_batch;
  a.stride_h = stride_head;
  a.stride_q = stride_query;
  a.batch = batch;
  a.kv = kv_heads;
  a.group = heads / kv_heads;
  a.queries = queries;
  a.keys = keys;
  a.seen = seen;
  a.acc = acc_in;
  a.out = acc;
  LAPSUM_TRY(launch_cache_accumulate(a, dtype, stream));
  return LAPSUM_OK;
}

size_t lapsum_cache_evict_workspace_size(int64_t batch, int64_t kv_heads, int64_t slots,
                                         int64_t budget) {
  if (batch < 1 || kv_heads < 1 || slots < 1 || budget < 1) return 0;
  Carve c(nullptr);
  c.take<int32_t>(static_cast<size_t>(batch * kv_heads * budget));
  return c.size();
}

int lapsum_cache_evict(const void* k, const int64_t* k_strides, const void* v,
                       const int64_t* v_strides, int64_t row_bytes, const float* acc,
                       const int32_t* pos, const int32_t* seen, int64_t batch, int64_t kv_heads,
                       int64_t slots, int64_t budget, int64_t sink, int64_t recent, void* k_out,
                       void* v_out, float* acc_out, int32_t* pos_out, void* workspace,
                       size_t workspace_bytes, hipStream_t stream) {
  if (!k_strides || !v_strides || !valid_cache(batch, kv_heads, slots, sink, recent) || budget < 1 ||
      !int32_range(budget) || sink + recent > budget || row_bytes < 1 || !int32_range(row_bytes))
    return LAPSUM_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i)
    if (k_strides[i] < 0 || v_strides[i] < 0) return LAPSUM_ERR_INVALID_ARG;
  if (batch > 0 && (!k || !v || !acc || !seen || !k_out || !v_out || !acc_out || !pos_out))
    return LAPSUM_ERR_INVALID_ARG;
  const int wst = check_ws(workspace, workspace_bytes,
                           lapsum_cache_evict_workspace_size(batch, kv_heads, slots, budget));
  if (wst != LAPSUM_OK) return wst;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (batch == 0) return LAPSUM_OK;
  const int width = vector_width(bits_of(k) | bits_of(v) | bits_of(k_out) | bits_of(v_out) |
                                 bits_of(k_strides) | bits_of(v_strides) |
                                 static_cast<uint64_t>(row_bytes));
  EvictArgs a{};
  a.k = k;
  a.v = v;
  a.k_b = k_strides[0] / width;
  a.k_h = k_strides[1] / width;
  a.k_s = k_strides[2] / width;
  a.v_b = v_strides[0] / width;
  a.v_h = v_strides[1] / width;
  a.v_s = v_strides[2] / width;
  a.row = row_bytes / width;
  a.acc = acc;
  a.pos = pos;
  a.seen = seen;
  a.batch = batch;
  a.kv = kv_heads;
  a.room = slots;
  a.budget = budget;
  a.sink = static_cast<int>(sink);
  a.recent = static_cast<int>(recent);
  a.k_out = k_out;
  a.v_out = v_out;
  a.acc_out = acc_out;
  a.pos_out = pos_out;
  a.slots = static_cast<int32_t*>(workspace);
  LAPSUM_TRY(launch_cache_evict(a, width, stream));
  return LAPSUM_OK;
}

int lapsum_cache_step(const void* weights, int dtype, int64_t stride_batch, int64_t stride_head,
                      const void* k_new, const void* v_new, const int32_t* seen, void* k,
                      const int64_t* k_strides, void* v, const int64_t* v_strides,
                      int64_t row_bytes, float* acc, int32_t* pos, int64_t batch, int64_t heads,
                      int64_t kv_heads, int64_t slots, int64_t sink, int64_t recent, int32_t* slot,
                      hipStream_t stream) {
  if (!valid_dtype(dtype) || !k_strides || !v_strides ||
      !valid_cache(batch, kv_heads, slots, sink, recent) || heads < 1 || heads % kv_heads ||
      recent < 1 || sink + recent > slots || row_bytes < 1 || !int32_range(row_bytes) ||
      stride_batch < 0 || stride_head < 0)
    return LAPSUM_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i)
    if (k_strides[i] < 0 || v_strides[i] < 0) return LAPSUM_ERR_INVALID_ARG;
  if (batch > 0 && (!weights || !k_new || !v_new || !seen || !k || !v || !acc || !pos || !slot))
    return LAPSUM_ERR_INVALID_ARG;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (batch == 0) return LAPSUM_OK;
  StepArgs a{};
  a.weights = weights;
  a.stride_b = stride_batch;
  a.stride_h = stride_head;
  a.batch = batch;
  a.kv = kv_heads;
  a.group = heads / kv_heads;
  a.room = slots;
  a.k_new = k_new;
  a.v_new = v_new;
  a.seen = seen;
  a.k = k;
  a.v = v;
  a.k_b = k_strides[0];
  a.k_h = k_strides[1];
  a.k_s = k_strides[2];
  a.v_b = v_strides[0];
  a.v_h = v_strides[1];
  a.v_s = v_strides[2];
  a.row = row_bytes;
  a.words = vector_width(bits_of(k) | bits_of(v) | bits_of(k_new) | bits_of(v_new) |
                         bits_of(k_strides) | bits_of(v_strides) |
                         static_cast<uint64_t>(row_bytes)) >= 4;
  a.acc = acc;
  a.pos = pos;
  a.sink = static_cast<int>(sink);
  a.recent = static_cast<int>(recent);
  a.slot = slot;
  LAPSUM_TRY(launch_cache_step(a, dtype, stream));
  return LAPSUM_OK;
}

}  // extern "C"
