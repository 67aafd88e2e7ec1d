// Arguments, workspaces and launchers of the operators on single rows of logits.
#pragma once

#include "rows.hpp"

namespace dsde {

// Workspace of the rows that one pair of launches takes; larger calls run
// their rows in several passes.  The cap also keeps a pass's keys (an eighth of
// its logits) inside the last-level cache.
constexpr size_t kSelectBytes = size_t(192) << 20;
// The weights of a segment's logits against the largest logit of its chunk: how many logits are that
// one, and the sum of all others.  A row's log-normaliser is log(ones) + log1p(rest / ones), and the
// log-probability of a token with nearly all mass is its rest alone, which one fp32 sum with the
// largest weight, 1, among its terms would round to 2^-24.
struct SegWeight {
  float ones, rest;
};
// The same of a whole row against its largest logit.
struct RowSum {
  double ones, rest;
};
// A row left to the cuts over many tokens, with its maximum and the weight of all its logits.
struct WideRow {
  int32_t row;
  float max;
  RowSum sum;
};
inline size_t select_row_bytes(int64_t V) {
  return size_t(num_chunks(V)) * (sizeof(float) + sizeof(SegWeight) * kSegs + sizeof(uint16_t) * kChunkGroups) +
         sizeof(WideRow);
}
inline int64_t select_rows_per_pass(int64_t R, int64_t V) {
  const int64_t n = int64_t((kSelectBytes - 1024) / select_row_bytes(V));
  return n < R ? n : R;
}
static_assert(kSelectBytes - 1024 >= (DSDE_MAX_VOCAB / kChunk) * (4 + 8 * kSegs + 2 * kChunkGroups) + sizeof(WideRow), "one row fits");
struct SelectLayout {
  size_t max, seg, keys, wide, n_wide, total;
};
inline SelectLayout select_layout(int64_t R, int64_t V) {
  const size_t n = size_t(select_rows_per_pass(R, V)) * size_t(num_chunks(V));
  const size_t all = size_t(R) * select_row_bytes(V);
  SelectLayout l;
  l.max = 0;
  l.seg = l.max + align_up(sizeof(float) * n);
  l.keys = l.seg + align_up(sizeof(SegWeight) * kSegs * n);
  l.wide = l.keys + align_up(sizeof(uint16_t) * kChunkGroups * n);
  l.n_wide = l.wide + align_up(sizeof(WideRow) * size_t(select_rows_per_pass(R, V)));
  // grows with R and with V; each of the five parts is padded to 256 bytes
  const size_t whole = align_up(all) + 6 * 256, most = kSelectBytes + 1024;
  l.total = whole < most ? whole : most;
  return l;
}

struct SelectArgs {
  RowsView rows;
  int32_t dtype;
  int64_t V;
  // per-row settings; a null pointer stands for one value or for no filter
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p, *u;
  float one_temperature;
  int32_t one_k;
  bool keys_always;
  struct {
    float *max;      // [R, nc] largest logit of each chunk; NaN: a NaN in it
    SegWeight *seg;  // [R, nc, 16] weights of its segments against that
    uint16_t *keys;  // [R, nc, 1024] high halves of its groups' largest ordered keys
    WideRow *wide;   // [*n_wide] rows left to wide_kernel
    uint32_t *n_wide;
  } scan;
  void *workspace;
  uint32_t *row_err;
  // sample
  int32_t pad_id;
  int32_t *tokens;
  float *logprob;  // may be null
  int32_t *kept;   // may be null
  // top logits
  float *values;
  int32_t *ids;
  float *lse;
};
int launch_sample(const SelectArgs &a, int64_t R, hipStream_t stream);
int launch_top_logits(const SelectArgs &a, int64_t R, hipStream_t stream);

// Distillation: the teacher's entries and the row records that the loss leaves
// for the gradient.
struct DistillPartial {
  float max;       // a chunk's largest logit outside the teacher's entries; NaN: a NaN in it
  uint32_t bad;    // 1: a teacher's token twice in the chunk
  double sum;      // sum of its weights against that
};
struct DistillArgs {
  RowsView rows;
  int32_t dtype;
  int64_t V;
  int32_t K;
  const int32_t *ids;        // [N, K], -1: unused
  const float *teacher;      // [N, K]
  const float *teacher_lse;  // [N], may be null: the entries are the whole distribution
  float temperature;
  const float *weight;       // [N] gradient weights; null in the loss
  bool skip_zero;            // rows of weight 0 are left out of the loss too
  DistillPartial *part;      // [N, nc]
  dsde_distill_row *record;  // [N]
  float *loss;               // [N]
  uint32_t *row_err;         // [N]
  char *grad;                // [N, V], grad_stride bytes from row to row
  int64_t grad_stride;
};
inline size_t distill_part_bytes(int64_t N, int64_t V) {
  return align_up(sizeof(DistillPartial) * size_t(N) * size_t(num_chunks(V)));
}
int launch_distill_loss(const DistillArgs &a, int64_t N, hipStream_t stream);
int launch_distill_grad(const DistillArgs &a, int64_t N, hipStream_t stream);
int launch_distill_step(const DistillArgs &a, int64_t N, hipStream_t stream);

}  // namespace dsde
