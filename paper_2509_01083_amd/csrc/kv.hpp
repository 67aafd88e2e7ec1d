// Arguments, workspaces and launchers of the paged key-value cache.
#pragma once

#include "common.hpp"

namespace dsde {

constexpr int32_t kMaxKvSeqs = 1 << 20;
constexpr int64_t kMaxTokens = int64_t(1) << 30;  // of one sequence: a tile behind the last stays below 2^31
constexpr int32_t kMinPage = 16, kMaxPage = 1024;

// dsde_kv_map's workspace: the stack's height behind the pages given back, then per
// sequence the pages it held and the prefix sums of pages taken and given back.
struct MapLayout {
  size_t top, from, taken, back, total;
};
inline MapLayout map_layout(int32_t B) {
  MapLayout l;
  l.top = 0;
  l.from = align_up(sizeof(int32_t));
  l.taken = l.from + align_up(sizeof(int32_t) * size_t(B));
  l.back = l.taken + align_up(sizeof(int32_t) * (size_t(B) + 1));
  l.total = l.back + align_up(sizeof(int32_t) * (size_t(B) + 1));
  return l;
}
struct MapArgs {
  int32_t B, shift, pages, width;
  int64_t rows;
  const int32_t *sl;
  int32_t extra;
  const int32_t *kv_len, *accepted;  // accepted may be null
  const uint32_t *last_err;          // may be null, may be seq_err
  int32_t *table, *held, *stack, *n_free, *base, *context, *cu_rows, *slots, *positions;
  uint32_t *seq_err;
  int32_t *top, *from, *taken, *back;  // workspace
};
int launch_kv_map(const MapArgs &a, hipStream_t stream);

// Rows [T, heads, dim] of one array, strides in bytes.
struct KvRows {
  const char *data;
  int64_t token_stride, head_stride;
};
struct CacheView {
  char *k, *v;
  int32_t dtype, pages, shift, heads, dim;
  int64_t page_stride, head_stride;  // bytes
  int32_t token_stride;              // bytes
  const float *k_scale, *v_scale;
};
struct KvWriteArgs {
  CacheView cache;
  KvRows k, v;
  int32_t dtype;
  int64_t T;
  const int32_t *slots;
  uint32_t *row_err;
};
int launch_kv_write(const KvWriteArgs &a, hipStream_t stream);

struct AttendArgs {
  CacheView cache;
  KvRows q;
  int32_t dtype, group, B, max_rows;
  int64_t T;
  const int32_t *table;
  int32_t width;
  const int32_t *context, *cu_rows;
  float scale;
  int32_t window;
  char *out;
  int64_t out_token_stride, out_head_stride;  // bytes
  float *lse;
  uint32_t *seq_err;
  void *workspace;
};
constexpr int kAttendWorkers = 1024;  // wavefronts of a launch
// Rows that one of them takes at once, at most, of so many of a sequence and key head.
constexpr int kAttendRows = 64;
inline int attend_rows(int64_t rows) { return rows < kAttendRows ? int(rows + 15) / 16 * 16 : kAttendRows; }
inline int padded_dim(int32_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
struct AttendLayout {
  size_t starts, parts, total;
};
inline AttendLayout attend_layout(int32_t dim, int64_t rows) {
  AttendLayout l;
  l.starts = 0;  // where each wavefront's share begins
  l.parts = align_up(size_t(32) * kAttendWorkers);
  // two parts of a wavefront: for each of its rows the values, a reference and a sum
  l.total = l.parts + align_up(sizeof(float) * 2 * kAttendWorkers * size_t(attend_rows(rows)) * size_t(padded_dim(dim) + 2));
  return l;
}
int launch_kv_attention(const AttendArgs &a, hipStream_t stream);

}  // namespace dsde
