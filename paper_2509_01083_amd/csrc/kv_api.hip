// C ABI of the paged key-value cache: host-side argument validation (before any
// HIP call), workspace sizing and dispatch.
#include <math.h>

#include "kv.hpp"

namespace {

int shift_of(int32_t page_size) {
  if (page_size < dsde::kMinPage || page_size > dsde::kMaxPage || (page_size & (page_size - 1)) != 0) return -1;
  return __builtin_ctz(unsigned(page_size));
}
int32_t size_of(int32_t dtype) { return dtype == DSDE_FP32 ? 4 : dtype == DSDE_BF16 ? 2 : 1; }
bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// Rows of dim elements that start at multiples of 16 bytes.
bool rows_ok(const void *p, int64_t token_stride, int64_t head_stride, int32_t dtype) {
  const int64_t limit = int64_t(1) << 40;
  if (token_stride < 0 || head_stride < 0 || token_stride > limit || head_stride > limit) return false;
  return !misaligned(p) && ((token_stride | head_stride) * size_of(dtype)) % 16 == 0;
}
// Sizes first; whether three strides keep all rows of a cache apart.
struct Axis {
  int64_t n, stride;
};
bool apart(Axis a, Axis b, Axis c, int64_t dim) {
  Axis x[3] = {a, b, c};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (x[j].stride > x[j + 1].stride) {
        const Axis t = x[j];
        x[j] = x[j + 1];
        x[j + 1] = t;
      }
  __int128 reach = dim;  // elements from a row's start to the end of what the smaller axes span
  for (const Axis &y : x) {
    if (y.n == 1) continue;
    if (y.stride < reach) return false;
    reach += __int128(y.n - 1) * y.stride;
  }
  return true;
}
bool cache_ok(const dsde_kv_cache *c) {
  if (!c || !c->k || !c->v || shift_of(c->page_size) < 0) return false;
  if (c->dtype != DSDE_FP32 && c->dtype != DSDE_BF16 && c->dtype != DSDE_E4M3) return false;
  if (c->dim < 16 || c->dim > DSDE_MAX_DIM || c->dim % 16 != 0) return false;
  if (c->heads < 1 || c->heads > DSDE_MAX_HEADS) return false;
  if (c->pages < 1 || int64_t(c->pages) * c->page_size >= (int64_t(1) << 31)) return false;
  if ((c->dtype == DSDE_E4M3) != (c->k_scale != nullptr) || (c->dtype == DSDE_E4M3) != (c->v_scale != nullptr)) return false;
  const int64_t e = size_of(c->dtype), limit = int64_t(1) << 40;
  if (c->page_stride < 0 || c->head_stride < 0 || c->token_stride < 0 || c->page_stride > limit ||
      c->head_stride > limit)
    return false;
  // a lane's offset inside a page is a 32-bit number
  if (c->token_stride > (int64_t(1) << 30) / (c->page_size * e)) return false;
  if (misaligned(c->k) || misaligned(c->v) || ((c->page_stride | c->head_stride | c->token_stride) * e) % 16 != 0)
    return false;
  return apart({c->pages, c->page_stride}, {c->heads, c->head_stride}, {c->page_size, c->token_stride}, c->dim);
}
bool types_match(const dsde_kv_cache *c, int32_t dtype) {
  return c->dtype == DSDE_E4M3 ? dtype == DSDE_BF16 : dtype == c->dtype;
}
dsde::CacheView view(const dsde_kv_cache *c) {
  const int64_t e = size_of(c->dtype);
  dsde::CacheView v;
  v.k = static_cast<char *>(c->k);
  v.v = static_cast<char *>(c->v);
  v.dtype = c->dtype;
  v.pages = c->pages;
  v.shift = shift_of(c->page_size);
  v.heads = c->heads;
  v.dim = c->dim;
  v.page_stride = c->page_stride * e;
  v.head_stride = c->head_stride * e;
  v.token_stride = int32_t(c->token_stride * e);
  v.k_scale = c->k_scale;
  v.v_scale = c->v_scale;
  return v;
}
dsde::KvRows kv_rows(const void *p, int64_t token_stride, int64_t head_stride, int32_t dtype) {
  return dsde::KvRows{static_cast<const char *>(p), token_stride * size_of(dtype), head_stride * size_of(dtype)};
}
bool attend_sizes_ok(int32_t B, int32_t heads, int64_t group, int32_t max_rows, int32_t dim) {
  return B >= 1 && B <= dsde::kMaxKvSeqs && heads >= 1 && heads <= DSDE_MAX_HEADS && group >= 1 &&
         heads * group <= DSDE_MAX_HEADS && max_rows >= 1 && max_rows <= DSDE_MAX_ROWS && dim >= 16 &&
         dim <= DSDE_MAX_DIM && dim % 16 == 0;
}

}  // namespace

extern "C" {

size_t dsde_kv_map_workspace_bytes(int32_t B) {
  return B >= 1 && B <= dsde::kMaxKvSeqs ? dsde::map_layout(B).total : 0;
}

int32_t dsde_kv_map(int32_t B, int32_t page_size, int32_t pages, int32_t width, int64_t rows, const int32_t *sl,
                    int32_t extra, const int32_t *kv_len, const int32_t *accepted, int32_t *table, int32_t *held,
                    int32_t *free_pages, int32_t *n_free, int32_t *base, int32_t *context, int32_t *cu_rows,
                    int32_t *slots, int32_t *positions, uint32_t *seq_err, void *workspace, size_t workspace_bytes,
                    void *stream) {
  return dsde_kv_map_next(B, page_size, pages, width, rows, sl, extra, kv_len, accepted, nullptr, table, held, free_pages,
                          n_free, base, context, cu_rows, slots, positions, seq_err, workspace, workspace_bytes, stream);
}

int32_t dsde_kv_map_next(int32_t B, int32_t page_size, int32_t pages, int32_t width, int64_t rows, const int32_t *sl,
                         int32_t extra, const int32_t *kv_len, const int32_t *accepted, const uint32_t *last_err,
                         int32_t *table, int32_t *held, int32_t *free_pages, int32_t *n_free, int32_t *base,
                         int32_t *context, int32_t *cu_rows, int32_t *slots, int32_t *positions, uint32_t *seq_err,
                         void *workspace, size_t workspace_bytes, void *stream) {
  const int64_t limit = int64_t(1) << 31;
  if (B < 1 || B > dsde::kMaxKvSeqs || shift_of(page_size) < 0 || pages < 1 || int64_t(pages) * page_size >= limit)
    return DSDE_INVALID_ARG;
  if (width < 1 || int64_t(width) * page_size > dsde::kMaxTokens || rows < 0 || rows >= limit) return DSDE_INVALID_ARG;
  if (!sl || !kv_len || !table || !held || !free_pages || !n_free || !base || !context || !cu_rows || !seq_err || !workspace)
    return DSDE_INVALID_ARG;
  if (rows > 0 && (!slots || !positions)) return DSDE_INVALID_ARG;
  const dsde::MapLayout l = dsde::map_layout(B);
  if (workspace_bytes < l.total) return DSDE_WORKSPACE_TOO_SMALL;
  if (misaligned(workspace)) return DSDE_INVALID_ARG;
  char *ws = static_cast<char *>(workspace);
  const auto part = [&](size_t at) { return reinterpret_cast<int32_t *>(ws + at); };
  const dsde::MapArgs a{B, shift_of(page_size), pages, width, rows, sl, extra, kv_len, accepted, last_err, table,
                        held, free_pages, n_free, base, context, cu_rows, slots, positions, seq_err, part(l.top),
                        part(l.from), part(l.taken), part(l.back)};
  return dsde::launch_kv_map(a, static_cast<hipStream_t>(stream));
}

int32_t dsde_kv_write(const dsde_kv_cache *cache, const void *k, int64_t k_token_stride, int64_t k_head_stride,
                      const void *v, int64_t v_token_stride, int64_t v_head_stride, int32_t dtype, int64_t T,
                      const int32_t *slots, uint32_t *row_err, void *stream) {
  if (!cache_ok(cache) || cache->k == cache->v || (dtype != DSDE_FP32 && dtype != DSDE_BF16) || !types_match(cache, dtype))
    return DSDE_INVALID_ARG;
  if (T < 0 || T >= (int64_t(1) << 31)) return DSDE_INVALID_ARG;
  if (T == 0) return DSDE_OK;
  if (!k || !v || !slots || !row_err) return DSDE_INVALID_ARG;
  if (!rows_ok(k, k_token_stride, k_head_stride, dtype) || !rows_ok(v, v_token_stride, v_head_stride, dtype))
    return DSDE_INVALID_ARG;
  dsde::KvWriteArgs a;
  a.cache = view(cache);
  a.k = kv_rows(k, k_token_stride, k_head_stride, dtype);
  a.v = kv_rows(v, v_token_stride, v_head_stride, dtype);
  a.dtype = dtype;
  a.T = T;
  a.slots = slots;
  a.row_err = row_err;
  return dsde::launch_kv_write(a, static_cast<hipStream_t>(stream));
}

size_t dsde_kv_attention_workspace_bytes(int32_t B, int32_t heads, int32_t group, int32_t max_rows, int32_t dim) {
  return attend_sizes_ok(B, heads, group, max_rows, dim) ? dsde::attend_layout(dim, int64_t(group) * max_rows).total : 0;
}

int32_t dsde_kv_attention(const dsde_kv_cache *cache, const void *q, int64_t q_token_stride, int64_t q_head_stride,
                          int32_t dtype, int32_t q_heads, int64_t T, int32_t B, int32_t max_rows, const int32_t *table,
                          int32_t width, const int32_t *context, const int32_t *cu_rows, float scale, int32_t window,
                          void *out, int64_t out_token_stride, int64_t out_head_stride, float *lse, uint32_t *seq_err,
                          void *workspace, size_t workspace_bytes, void *stream) {
  if (!cache_ok(cache) || (dtype != DSDE_FP32 && dtype != DSDE_BF16) || !types_match(cache, dtype))
    return DSDE_INVALID_ARG;
  if (q_heads < 1 || q_heads % cache->heads != 0 ||
      !attend_sizes_ok(B, cache->heads, q_heads / cache->heads, max_rows, cache->dim))
    return DSDE_INVALID_ARG;
  if (T < 0 || T >= (int64_t(1) << 31) || width < 1 || int64_t(width) * cache->page_size > dsde::kMaxTokens)
    return DSDE_INVALID_ARG;
  if (!isfinite(scale * 1.4426950f) || window < 0) return DSDE_INVALID_ARG;  // the kernel's scale is log2(e) times that
  if (!table || !context || !cu_rows || !seq_err || !workspace || (T > 0 && (!q || !out))) return DSDE_INVALID_ARG;
  if (T > 0 && (!rows_ok(q, q_token_stride, q_head_stride, dtype) || !rows_ok(out, out_token_stride, out_head_stride, dtype)))
    return DSDE_INVALID_ARG;
  // rows that are written must not overlap
  if (T > 0 && !apart({T, out_token_stride}, {q_heads, out_head_stride}, {1, 0}, cache->dim)) return DSDE_INVALID_ARG;
  const int32_t group = q_heads / cache->heads;
  if (workspace_bytes < dsde::attend_layout(cache->dim, int64_t(group) * max_rows).total) return DSDE_WORKSPACE_TOO_SMALL;
  if (misaligned(workspace)) return DSDE_INVALID_ARG;
  dsde::AttendArgs a;
  a.cache = view(cache);
  a.q = kv_rows(q, q_token_stride, q_head_stride, dtype);
  a.dtype = dtype;
  a.group = group;
  a.B = B;
  a.max_rows = max_rows;
  a.T = T;
  a.table = table;
  a.width = width;
  a.context = context;
  a.cu_rows = cu_rows;
  a.scale = scale;
  a.window = window;
  a.out = static_cast<char *>(out);
  a.out_token_stride = out_token_stride * size_of(dtype);
  a.out_head_stride = out_head_stride * size_of(dtype);
  a.lse = lse;
  a.seq_err = seq_err;
  a.workspace = workspace;
  return dsde::launch_kv_attention(a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
