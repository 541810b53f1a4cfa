// Host side of the experts' rows: argument checks, workspaces and launch order of
// their order, products and weighted sums.
#include "host.hpp"
#include "kernels.hpp"

using namespace lapsum;

namespace {

bool whole_vectors(int dtype, uint64_t bytes, int64_t elements) {
  return vector_width(bytes) == 16 && elements % (dtype == LAPSUM_F32 ? 4 : 8) == 0;
}
int64_t size_of(int dtype) { return dtype == LAPSUM_F32 ? 4 : 2; }

// A matrix per expert: [inner, outer] by strides of which one is 1.
struct Matrices {
  bool ok, out_dense;
  int64_t row;
  Matrices(const int64_t* strides, int64_t in, int64_t out) : ok(false), out_dense(false), row(0) {
    if (!strides || strides[0] < 0 || strides[1] < 0 || strides[2] < 0) return;
    if ((strides[2] == 1 || out == 1) && (strides[1] >= out || in == 1)) {
      ok = out_dense = true;
      row = strides[1];
    } else if ((strides[1] == 1 || in == 1) && (strides[2] >= in || out == 1)) {
      ok = true;
      row = strides[2];
    }
  }
};

bool valid_product(int dtype, int64_t x_rows, int64_t x_stride, const int32_t* order, int64_t top_k,
                   int64_t experts, int64_t rows, int64_t in, int64_t out) {
  return valid_dtype(dtype) && x_rows >= 0 && int32_range(x_rows) && top_k >= 1 && int32_range(top_k) &&
         experts >= 1 && experts <= kExpertMost && rows >= 0 && rows <= (int64_t(1) << 30) && in >= 1 &&
         in <= (int64_t(1) << 24) && out >= 1 && out <= (int64_t(1) << 24) && x_stride >= in &&
         (order || rows <= x_rows);
}

}  // namespace

extern "C" {

// ----------------------------------------------------------------- order --
size_t lapsum_expert_order_workspace_size(int64_t count, int64_t experts) {
  if (count < 1 || experts < 1 || experts > kExpertMost) return 0;
  const int64_t blocks = order_blocks(count);
  if (blocks <= 1) return 0;
  Carve c(nullptr);
  c.take<int>(static_cast<size_t>(blocks * (experts + 1)));
  return c.size();
}

int lapsum_expert_order(const int32_t* indices, int64_t count, int64_t experts, int32_t* order,
                        int32_t* place, int32_t* offsets, void* workspace, size_t workspace_bytes,
                        hipStream_t stream) {
  if (count < 0 || count > (int64_t(1) << 30) || experts < 1 || experts > kExpertMost || !offsets ||
      (count > 0 && (!indices || !order || !place)))
    return LAPSUM_ERR_INVALID_ARG;
  const int wst = check_ws(workspace, workspace_bytes, lapsum_expert_order_workspace_size(count, experts));
  if (wst != LAPSUM_OK) return wst;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (count == 0) {
    LAPSUM_TRY(launch_fill_u32(reinterpret_cast<uint32_t*>(offsets), experts + 1, 0u, stream));
    return LAPSUM_OK;
  }
  OrderArgs a{};
  a.indices = indices;
  a.count = count;
  a.experts = static_cast<int>(experts);
  a.order = order;
  a.place = place;
  a.offsets = offsets;
  a.parts = static_cast<int*>(workspace);
  LAPSUM_TRY(launch_expert_order(a, stream));
  return LAPSUM_OK;
}

// -------------------------------------------------------------- products --
int lapsum_expert_matmul(const void* x, int dtype, int64_t x_rows, int64_t x_stride,
                         const int32_t* order, int64_t top_k, const int32_t* offsets,
                         int64_t experts, int64_t rows, int64_t in, int64_t out, const void* w,
                         const int64_t* w_strides, void* y, int y_dtype, hipStream_t stream) {
  if (!valid_product(dtype, x_rows, x_stride, order, top_k, experts, rows, in, out) ||
      (y_dtype != dtype && y_dtype != LAPSUM_F32))
    return LAPSUM_ERR_INVALID_ARG;
  const Matrices m(w_strides, in, out);
  if (!m.ok || (rows > 0 && (!offsets || !w || !y || (x_rows > 0 && !x)))) return LAPSUM_ERR_INVALID_ARG;
  // (the documented bound; what is launched is counted below)
  const bool few = rows <= experts * 16;
  const int64_t lines = (few ? rows / 16 : rows / 128) + (experts < rows ? experts : rows) + 4;
  if (lines * (few ? (out + 63) / 64 : (out + 127) / 128) >= (few ? 4 : 2) * kMaxBlocks) return LAPSUM_ERR_INVALID_ARG;
  RowsArgs a{};
  a.x = x;
  a.w = w;
  a.y = y;
  a.order = order;
  a.offsets = offsets;
  a.x_rows = x_rows;
  a.x_stride = x_stride;
  a.w_expert = w_strides[0];
  a.w_row = m.row;
  a.rows = static_cast<int>(rows);
  a.k = static_cast<int>(in);
  a.n = static_cast<int>(out);
  a.experts = static_cast<int>(experts);
  a.by = divider(top_k);
  const int64_t size = size_of(dtype);
  a.y_lines = vector_width(bits_of(y)) == 16 && out % 8 == 0;
  const bool vec = whole_vectors(dtype, bits_of(x) | bits_of(w) |
                                 static_cast<uint64_t>((x_stride | w_strides[0] | m.row) * size),
                                 m.out_dense ? in | out : in);
  if (expert_rows_threads(a, dtype, m.out_dense, vec) >= kMaxThreads) return LAPSUM_ERR_INVALID_ARG;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (rows == 0) return LAPSUM_OK;
  LAPSUM_TRY(launch_expert_rows(a, dtype, m.out_dense, y_dtype == LAPSUM_F32, vec, stream));
  return LAPSUM_OK;
}

size_t lapsum_expert_matmul_weights_workspace_size(int64_t experts, int64_t rows, int64_t in, int64_t out) {
  if (experts < 1 || experts > kExpertMost || rows < 1 || rows > (int64_t(1) << 30) || in < 1 ||
      in > (int64_t(1) << 24) || out < 1 || out > (int64_t(1) << 24))
    return 0;
  const int splits = grad_splits(experts, rows, in, out);
  if (splits <= 1) return 0;
  Carve c(nullptr);
  c.take<float>(static_cast<size_t>(splits * experts) * static_cast<size_t>(in) * static_cast<size_t>(out));
  return c.size();
}

int lapsum_expert_matmul_weights(const void* x, int dtype, int64_t x_rows, int64_t x_stride,
                                 const int32_t* order, int64_t top_k, const int32_t* offsets,
                                 int64_t experts, int64_t rows, int64_t in, int64_t out,
                                 const void* grad_y, int64_t grad_stride, void* grad_w,
                                 const int64_t* w_strides, void* workspace,
                                 size_t workspace_bytes, hipStream_t stream) {
  if (!valid_product(dtype, x_rows, x_stride, order, top_k, experts, rows, in, out) || grad_stride < out)
    return LAPSUM_ERR_INVALID_ARG;
  const Matrices m(w_strides, in, out);
  if (!m.ok || !offsets || !grad_w || (rows > 0 && (!grad_y || (x_rows > 0 && !x))) ||
      (experts > 1 && w_strides[0] < (m.out_dense ? (in - 1) * m.row + out : (out - 1) * m.row + in)))
    return LAPSUM_ERR_INVALID_ARG;
  if ((experts * ((in + 127) / 128) + 3) * ((out + 127) / 128) >= 2 * kMaxBlocks) return LAPSUM_ERR_INVALID_ARG;
  GradArgs a{};
  const bool swap = !m.out_dense;   // the gradient's rows are those of w in memory
  a.a = swap ? grad_y : x;
  a.b = swap ? x : grad_y;
  a.a_stride = swap ? grad_stride : x_stride;
  a.b_stride = swap ? x_stride : grad_stride;
  a.a_rows = swap ? rows : x_rows;
  a.b_rows = swap ? x_rows : rows;
  a.m = static_cast<int>(swap ? out : in);
  a.n = static_cast<int>(swap ? in : out);
  a.gather = order ? (swap ? 2 : 1) : 0;
  a.c = grad_w;
  a.c_expert = w_strides[0];
  a.c_row = m.row;
  a.order = order;
  a.offsets = offsets;
  a.rows = static_cast<int>(rows);
  a.experts = static_cast<int>(experts);
  a.by = divider(top_k);
  a.splits = rows > 0 ? grad_splits(experts, rows, in, out) : 1;
  a.part = static_cast<float*>(workspace);
  const int64_t size = size_of(dtype);
  const bool vec = whole_vectors(dtype, bits_of(x) | bits_of(grad_y) | bits_of(grad_w) |
                                 static_cast<uint64_t>((x_stride | grad_stride | w_strides[0] | m.row) * size),
                                 in | out);
  if (expert_grad_threads(a, dtype, vec) >= kMaxThreads) return LAPSUM_ERR_INVALID_ARG;
  const int wst = check_ws(workspace, workspace_bytes,
                           lapsum_expert_matmul_weights_workspace_size(experts, rows, in, out));
  if (wst != LAPSUM_OK) return wst;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  LAPSUM_TRY(launch_expert_grad(a, dtype, vec, stream));
  return LAPSUM_OK;
}

// ------------------------------------------------------------------ sums --
int lapsum_expert_combine(const void* y, int dtype, int64_t rows, int64_t dim, const float* weights,
                          const int32_t* place, int64_t tokens, int64_t top_k, void* out,
                          int out_dtype, hipStream_t stream) {
  if (!valid_dtype(dtype) || !valid_dtype(out_dtype) || (out_dtype != dtype && dtype != LAPSUM_F32) ||
      rows < 0 || !int32_range(rows) || dim < 1 || dim > (int64_t(1) << 24) || tokens < 0 ||
      tokens > (int64_t(1) << 30) || top_k < 1 || !int32_range(top_k) || tokens > (int64_t(1) << 40) / top_k)
    return LAPSUM_ERR_INVALID_ARG;
  if (tokens > 0 && (!place || !out || (rows > 0 && !y))) return LAPSUM_ERR_INVALID_ARG;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (tokens == 0) return LAPSUM_OK;
  CombineArgs a{};
  a.y = y;
  a.weights = weights;
  a.place = place;
  a.out = out;
  a.tokens = tokens;
  a.dim = dim;
  a.rows = rows;
  a.top_k = static_cast<int>(top_k);
  const bool vec = vector_width(bits_of(y) | bits_of(out)) == 16 && dim % 8 == 0;
  LAPSUM_TRY(launch_expert_combine(a, dtype, out_dtype, vec, stream));
  return LAPSUM_OK;
}

int lapsum_expert_combine_backward(const void* grad_out, const void* y, int dtype, int64_t rows,
                                   int64_t dim, const float* weights, const int32_t* place,
                                   const int32_t* offsets, int64_t experts, int64_t tokens,
                                   int64_t top_k, void* grad_y, float* grad_weights,
                                   hipStream_t stream) {
  if (!valid_dtype(dtype) || rows < 0 || !int32_range(rows) || dim < 1 || dim > (int64_t(1) << 24) ||
      experts < 1 || experts > kExpertMost || tokens < 0 || tokens > (int64_t(1) << 30) || top_k < 1 ||
      !int32_range(top_k) || tokens > (int64_t(1) << 40) / top_k || !offsets)
    return LAPSUM_ERR_INVALID_ARG;
  if ((tokens > 0 && (!grad_out || !weights || !place || !grad_weights)) || (rows > 0 && (!y || !grad_y)))
    return LAPSUM_ERR_INVALID_ARG;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (tokens == 0 && rows == 0) return LAPSUM_OK;
  CombineGradArgs a{};
  a.grad = grad_out;
  a.y = y;
  a.weights = weights;
  a.place = place;
  a.ends = offsets;
  a.grad_y = grad_y;
  a.grad_weights = grad_weights;
  a.tokens = tokens;
  a.dim = dim;
  a.rows = rows;
  a.top_k = static_cast<int>(top_k);
  a.experts = static_cast<int>(experts);
  const bool vec = vector_width(bits_of(y) | bits_of(grad_out) | bits_of(grad_y)) == 16 && dim % 8 == 0;
  LAPSUM_TRY(launch_expert_combine_backward(a, dtype, vec, stream));
  return LAPSUM_OK;
}

}  // extern "C"
