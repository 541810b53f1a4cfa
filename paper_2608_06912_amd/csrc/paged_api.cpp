// Host side of the paged cache: argument checks, workspaces and launch order of
// writing, reading back and attending.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "host.hpp"
#include "kernels.hpp"

using namespace lapsum;

namespace {

bool valid_kind(int kind, int dtype) {
  return kind == LAPSUM_I8 || kind == LAPSUM_E4M3 || kind == dtype;
}
int64_t bytes_of(int kind) { return kind == LAPSUM_F32 ? 4 : kind <= LAPSUM_F16 ? 2 : 1; }

// The caller's description of a cache; written: no two entries in one place.
bool valid_paged(const lapsum_paged* c, int kind, int64_t kv, int64_t dim) {
  if (!c || c->pages < 1 || !int32_range(c->pages) || c->slots < 1 || c->slots > (int64_t(1) << 30) ||
      c->stride_page < 0 || c->stride_head < 0 || c->stride_slot < 0 || kv < 1 || dim < 1 || dim > kPagedMaxDim)
    return false;
  return kind <= LAPSUM_F16 || (c->scale && c->scale_stride_page >= 0 && c->scale_stride_head >= 0);
}
// No two entries in one place (two that one call may write).
bool apart(const lapsum_paged* c, int kind, int64_t kv, int64_t dim) {
  return (c->slots == 1 || c->stride_slot >= dim) && (kv == 1 || c->stride_head != 0) &&
         (c->pages == 1 || c->stride_page != 0) &&
         (kind <= LAPSUM_F16 || ((kv == 1 || c->scale_stride_head >= c->slots) &&
                                 (c->pages == 1 || c->scale_stride_page != 0)));
}
bool whole(const lapsum_paged* c, int kind, int64_t dim) {
  const uint64_t size = static_cast<uint64_t>(bytes_of(kind));
  const uint64_t bits = bits_of(c->data) |
                        static_cast<uint64_t>(c->stride_page | c->stride_head | c->stride_slot) * size;
  return dim % 8 == 0 && vector_width(bits) >= (kind <= LAPSUM_F16 ? 16 : 8);
}
PagedCache cache_of(const lapsum_paged* c) {
  return PagedCache{c->data, c->scale, c->stride_page, c->stride_head, c->stride_slot, c->scale_stride_page,
                    c->scale_stride_head};
}
// The positions of a sequence, or -1 where the table cannot be.
int64_t room_of(const lapsum_paged* c, const int32_t* table, int64_t width, int64_t batch) {
  if (!table) return c->pages >= batch ? c->slots : -1;
  if (width < 0 || !int32_range(width) || width > (int64_t(1) << 30) / c->slots) return -1;
  return width * c->slots;
}
PageTable table_of(const lapsum_paged* c, const int32_t* table, int64_t width) {
  return PageTable{table, c->pages, static_cast<int>(table ? width : 1), static_cast<int>(c->slots),
                   divider(c->slots)};
}

}  // namespace

extern "C" {

int lapsum_cache_append(const void* k_new, const int64_t* k_strides, const void* v_new,
                        const int64_t* v_strides, int dtype, int64_t batch, int64_t kv_heads,
                        int64_t fresh, int64_t dim, const int32_t* seen, const int32_t* count,
                        const lapsum_paged* k, const lapsum_paged* v, int kind,
                        const int32_t* table, int64_t width, hipStream_t stream) {
  if (!valid_dtype(dtype) || !valid_kind(kind, dtype) || batch < 0 || fresh < 0 || !k_strides || !v_strides ||
      !valid_paged(k, kind, kv_heads, dim) || !valid_paged(v, kind, kv_heads, dim) || k->pages != v->pages ||
      k->slots != v->slots || !apart(k, kind, kv_heads, dim) || !apart(v, kind, kv_heads, dim) ||
      room_of(k, table, width, batch) < 0)
    return LAPSUM_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i)
    if (k_strides[i] < 0 || v_strides[i] < 0) return LAPSUM_ERR_INVALID_ARG;
  const bool work = batch > 0 && fresh > 0;
  if (work && (!k_new || !v_new || !seen || !k->data || !v->data)) return LAPSUM_ERR_INVALID_ARG;
  // one cache for both takes what is one for both
  if (work && (k->data == v->data || (kind > LAPSUM_F16 && k->scale == v->scale)) &&
      (k_new != v_new || !std::equal(k_strides, k_strides + 3, v_strides) || memcmp(k, v, sizeof *k) != 0))
    return LAPSUM_ERR_INVALID_ARG;
  if (work && (kv_heads > 2147483647LL / batch || batch * kv_heads > 2147483647LL / fresh ||
               paged_blocks(batch * kv_heads, fresh, dim) >= 2 * kMaxBlocks))
    return LAPSUM_ERR_INVALID_ARG;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (!work) return LAPSUM_OK;
  AppendArgs a{};
  a.src[0] = k_new;
  a.src[1] = v_new;
  const int64_t* strides[2] = {k_strides, v_strides};
  for (int n = 0; n < 2; ++n) {
    a.src_b[n] = strides[n][0];
    a.src_h[n] = strides[n][1];
    a.src_i[n] = strides[n][2];
  }
  a.cache[0] = cache_of(k);
  a.cache[1] = cache_of(v);
  a.t = table_of(k, table, width);
  a.seen = seen;
  a.count = count;
  a.batch = static_cast<int>(batch);
  a.kv = static_cast<int>(kv_heads);
  a.fresh = static_cast<int>(fresh);
  a.dim = static_cast<int>(dim);
  const uint64_t bits = bits_of(k_new) | bits_of(v_new) |
                        (bits_of(k_strides) | bits_of(v_strides)) * static_cast<uint64_t>(bytes_of(dtype));
  const bool vec = vector_width(bits) == 16 && whole(k, kind, dim) && whole(v, kind, dim);
  LAPSUM_TRY(launch_cache_append(a, dtype, kind, vec, stream));
  return LAPSUM_OK;
}

int lapsum_cache_read(const lapsum_paged* cache, int kind, int64_t batch, int64_t kv_heads,
                      int64_t room, int64_t dim, const int32_t* lens, const int32_t* table,
                      int64_t width, void* out, int dtype, hipStream_t stream) {
  if (!valid_dtype(dtype) || !valid_kind(kind, dtype) || batch < 0 || room < 0 ||
      !valid_paged(cache, kind, kv_heads, dim) || room_of(cache, table, width, batch) < 0)
    return LAPSUM_ERR_INVALID_ARG;
  const bool work = batch > 0 && room > 0;
  if (work && (!cache->data || !lens || !out)) return LAPSUM_ERR_INVALID_ARG;
  if (work && (kv_heads > 2147483647LL / batch || batch * kv_heads > 2147483647LL / room ||
               paged_blocks(batch * kv_heads, room, dim) >= 2 * kMaxBlocks))
    return LAPSUM_ERR_INVALID_ARG;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (!work) return LAPSUM_OK;
  ReadArgs a{};
  a.cache = cache_of(cache);
  a.t = table_of(cache, table, width);
  a.lens = lens;
  a.out = out;
  a.batch = static_cast<int>(batch);
  a.kv = static_cast<int>(kv_heads);
  a.room = static_cast<int>(room);
  a.dim = static_cast<int>(dim);
  const bool vec = vector_width(bits_of(out)) == 16 && whole(cache, kind, dim);
  LAPSUM_TRY(launch_cache_read(a, dtype, kind, vec, stream));
  return LAPSUM_OK;
}

size_t lapsum_cache_attend_workspace_size(int64_t batch, int64_t heads, int64_t kv_heads, int64_t dim,
                                          int64_t room, int64_t window) {
  if (batch < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads || dim < 1 || dim > kPagedMaxDim || room < 0 ||
      room > (int64_t(1) << 30) || window < 0 || heads > (int64_t(1) << 30) / batch)
    return 0;
  int splits = 0, chunk = 0;
  attend_plan(batch, heads, kv_heads, room, window, &splits, &chunk);
  if (splits <= 1) return 0;
  Carve c(nullptr);
  c.take<float>(static_cast<size_t>(splits) * static_cast<size_t>(batch * heads) * static_cast<size_t>(dim + 2));
  return c.size();
}

int lapsum_cache_attend(const void* q, int64_t q_stride_batch, int64_t q_stride_head, int dtype,
                        const lapsum_paged* k, const lapsum_paged* v, int kind, int64_t batch,
                        int64_t heads, int64_t kv_heads, int64_t dim, const int32_t* lens,
                        const int32_t* table, int64_t width, double scale, int64_t window,
                        void* out, float* lse, float* weights, void* workspace,
                        size_t workspace_bytes, hipStream_t stream) {
  if (!valid_dtype(dtype) || !valid_kind(kind, dtype) || batch < 0 || heads < 1 || q_stride_batch < 0 ||
      q_stride_head < 0 || !valid_paged(k, kind, kv_heads, dim) || !valid_paged(v, kind, kv_heads, dim) ||
      heads % kv_heads || k->pages != v->pages || k->slots != v->slots || !isfinite(scale) || window < 0 ||
      !int32_range(window))
    return LAPSUM_ERR_INVALID_ARG;
  const int64_t room = room_of(k, table, width, batch);
  if (room < 0 || (weights && !lse)) return LAPSUM_ERR_INVALID_ARG;
  if (batch > 0 && (heads > kMaxBlocks / batch || !q || !lens || !out || (room > 0 && (!k->data || !v->data))))
    return LAPSUM_ERR_INVALID_ARG;
  const int wst = check_ws(workspace, workspace_bytes,
                           lapsum_cache_attend_workspace_size(batch, heads, kv_heads, dim, room, window));
  if (wst != LAPSUM_OK) return wst;
  const int dst = check_device();
  if (dst != LAPSUM_OK) return dst;
  if (batch == 0) return LAPSUM_OK;
  AttendArgs a{};
  a.q = q;
  a.q_b = q_stride_batch;
  a.q_h = q_stride_head;
  a.k = cache_of(k);
  a.v = cache_of(v);
  a.t = table_of(k, table, width);
  a.lens = lens;
  a.out = out;
  a.lse = lse;
  a.weights = room > 0 ? weights : nullptr;
  a.batch = static_cast<int>(batch);
  a.heads = static_cast<int>(heads);
  a.kv = static_cast<int>(kv_heads);
  a.dim = static_cast<int>(dim);
  a.group = static_cast<int>(heads / kv_heads);
  a.tiles = (a.group + 15) / 16;
  a.window = static_cast<int>(window);
  a.room = room;
  a.by = a.t.by;
  a.q_whole = dim % 8 == 0 && vector_width(bits_of(q) | static_cast<uint64_t>((q_stride_batch | q_stride_head) *
                                                                              bytes_of(dtype))) == 16;
  a.scale = static_cast<float>(scale);
  attend_plan(batch, heads, kv_heads, room, window, &a.splits, &a.chunk);
  a.part = a.splits > 1 ? static_cast<float*>(workspace) : nullptr;
  const bool vec = whole(k, kind, dim) && whole(v, kind, dim);
  LAPSUM_TRY(launch_cache_attend(a, dtype, kind, vec, stream));
  return LAPSUM_OK;
}

}  // extern "C"
