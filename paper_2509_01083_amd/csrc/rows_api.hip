// C ABI of the operators on single rows of logits: host-side argument
// validation (before any HIP call), workspace sizing and dispatch.
#include <math.h>

#include "rows_args.hpp"

namespace {

bool rows_ok(int64_t R, int64_t V, int64_t stride, int32_t dtype) {
  if (dtype != DSDE_FP32 && dtype != DSDE_BF16) return false;
  if (V < 1 || V > DSDE_MAX_VOCAB || R < 0 || R > 0x7fffffff) return false;
  if (R > 1 && stride < V) return false;
  // byte offsets of every row in 64 bits, and one launch dimension over the chunks
  if (stride < 0 || stride > (int64_t(1) << 40)) return false;
  return R * dsde::num_chunks(V) < (int64_t(1) << 31);
}
int64_t row_bytes(int64_t stride, int32_t dtype) { return stride * (dtype == DSDE_BF16 ? 2 : 4); }
bool temperature_ok(float T) { return T >= dsde::kMinTemp && T <= dsde::kMaxTemp; }
bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

dsde::SelectArgs select_args(const void *logits, int64_t stride, int32_t dtype, int64_t V, void *workspace,
                             uint32_t *row_err) {
  dsde::SelectArgs a{};
  a.rows = dsde::RowsView{static_cast<const char *>(logits), row_bytes(stride, dtype), V};
  a.dtype = dtype;
  a.V = V;
  a.one_temperature = 1.0f;
  a.workspace = workspace;
  a.row_err = row_err;
  return a;
}

dsde::DistillArgs distill_args(const void *logits, int64_t stride, int32_t dtype, int64_t V, int32_t K,
                               const int32_t *ids, const float *teacher, float temperature) {
  dsde::DistillArgs a{};
  a.rows = dsde::RowsView{static_cast<const char *>(logits), row_bytes(stride, dtype), V};
  a.dtype = dtype;
  a.V = V;
  a.K = K;
  a.ids = ids;
  a.teacher = teacher;
  a.temperature = temperature;
  return a;
}
size_t distill_workspace(int64_t N, int64_t V) {
  return dsde::distill_part_bytes(N, V) + dsde::align_up(sizeof(dsde_distill_row) * size_t(N)) + 256;
}

}  // namespace

extern "C" {

size_t dsde_sample_workspace_bytes(int64_t R, int64_t V) {
  return rows_ok(R, V, V, DSDE_BF16) ? dsde::select_layout(R, V).total : 0;
}

int32_t dsde_sample(const void *logits, int64_t row_stride, int32_t dtype, int64_t V, int64_t R,
                    const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                    const float *u, int32_t pad_id, int32_t *tokens, float *logprob, int32_t *kept,
                    uint32_t *row_err, void *workspace, size_t workspace_bytes, void *stream) {
  if (!rows_ok(R, V, row_stride, dtype)) return DSDE_INVALID_ARG;
  if (R == 0) return DSDE_OK;
  if (!logits || !temperature || !u || !tokens || !row_err || !workspace) return DSDE_INVALID_ARG;
  if (workspace_bytes < dsde::select_layout(R, V).total) return DSDE_WORKSPACE_TOO_SMALL;
  if (misaligned(workspace)) return DSDE_INVALID_ARG;
  dsde::SelectArgs a = select_args(logits, row_stride, dtype, V, workspace, row_err);
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.u = u;
  a.pad_id = pad_id;
  a.tokens = tokens;
  a.logprob = logprob;
  a.kept = kept;
  return dsde::launch_sample(a, R, static_cast<hipStream_t>(stream));
}

int32_t dsde_top_logits(const void *logits, int64_t row_stride, int32_t dtype, int64_t V, int64_t R, int32_t k,
                        float temperature, float *values, int32_t *ids, float *lse, uint32_t *row_err,
                        void *workspace, size_t workspace_bytes, void *stream) {
  if (!rows_ok(R, V, row_stride, dtype) || k < 1 || k > DSDE_MAX_TOP || !temperature_ok(temperature))
    return DSDE_INVALID_ARG;
  if (R == 0) return DSDE_OK;
  if (!logits || !values || !ids || !lse || !row_err || !workspace) return DSDE_INVALID_ARG;
  if (workspace_bytes < dsde::select_layout(R, V).total) return DSDE_WORKSPACE_TOO_SMALL;
  if (misaligned(workspace)) return DSDE_INVALID_ARG;
  dsde::SelectArgs a = select_args(logits, row_stride, dtype, V, workspace, row_err);
  a.one_temperature = temperature;
  a.one_k = k;
  a.values = values;
  a.ids = ids;
  a.lse = lse;
  return dsde::launch_top_logits(a, R, static_cast<hipStream_t>(stream));
}

size_t dsde_distill_workspace_bytes(int64_t N, int64_t V) {
  return rows_ok(N, V, V, DSDE_BF16) ? distill_workspace(N, V) : 0;
}

int32_t dsde_distill_loss(const void *logits, int64_t row_stride, int32_t dtype, int64_t V, int64_t N, int32_t K,
                          const int32_t *ids, const float *teacher, const float *teacher_lse, float temperature,
                          float *loss, dsde_distill_row *record, uint32_t *row_err, void *workspace,
                          size_t workspace_bytes, void *stream) {
  if (!rows_ok(N, V, row_stride, dtype) || K < 1 || K > DSDE_MAX_TOP || !temperature_ok(temperature))
    return DSDE_INVALID_ARG;
  if (N == 0) return DSDE_OK;
  if (!logits || !ids || !teacher || !loss || !record || !row_err || !workspace) return DSDE_INVALID_ARG;
  if (workspace_bytes < distill_workspace(N, V)) return DSDE_WORKSPACE_TOO_SMALL;
  if (misaligned(workspace)) return DSDE_INVALID_ARG;
  dsde::DistillArgs a = distill_args(logits, row_stride, dtype, V, K, ids, teacher, temperature);
  a.teacher_lse = teacher_lse;
  a.part = static_cast<dsde::DistillPartial *>(workspace);
  a.loss = loss;
  a.record = record;
  a.row_err = row_err;
  return dsde::launch_distill_loss(a, N, static_cast<hipStream_t>(stream));
}

int32_t dsde_distill_grad(const void *logits, int64_t row_stride, int32_t dtype, int64_t V, int64_t N, int32_t K,
                          const int32_t *ids, const float *teacher, float temperature,
                          const dsde_distill_row *record, const float *weight, void *grad, int64_t grad_stride,
                          void *stream) {
  if (!rows_ok(N, V, row_stride, dtype) || !rows_ok(N, V, grad_stride, dtype) || K < 1 || K > DSDE_MAX_TOP ||
      !temperature_ok(temperature))
    return DSDE_INVALID_ARG;
  if (N == 0) return DSDE_OK;
  if (!logits || !ids || !teacher || !record || !weight || !grad) return DSDE_INVALID_ARG;
  if (grad == logits && grad_stride != row_stride) return DSDE_INVALID_ARG;
  dsde::DistillArgs a = distill_args(logits, row_stride, dtype, V, K, ids, teacher, temperature);
  a.record = const_cast<dsde_distill_row *>(record);
  a.weight = weight;
  a.grad = static_cast<char *>(grad);
  a.grad_stride = row_bytes(grad_stride, dtype);
  return dsde::launch_distill_grad(a, N, static_cast<hipStream_t>(stream));
}

int32_t dsde_distill_step(const void *logits, int64_t row_stride, int32_t dtype, int64_t V, int64_t N, int32_t K,
                          const int32_t *ids, const float *teacher, const float *teacher_lse, float temperature,
                          const float *weight, float *loss, void *grad, int64_t grad_stride, uint32_t *row_err,
                          void *workspace, size_t workspace_bytes, void *stream) {
  if (!rows_ok(N, V, row_stride, dtype) || !rows_ok(N, V, grad_stride, dtype) || K < 1 || K > DSDE_MAX_TOP ||
      !temperature_ok(temperature))
    return DSDE_INVALID_ARG;
  if (N == 0) return DSDE_OK;
  if (!logits || !ids || !teacher || !weight || !loss || !grad || !row_err || !workspace) return DSDE_INVALID_ARG;
  if (grad == logits && grad_stride != row_stride) return DSDE_INVALID_ARG;
  if (workspace_bytes < distill_workspace(N, V)) return DSDE_WORKSPACE_TOO_SMALL;
  if (misaligned(workspace)) return DSDE_INVALID_ARG;
  dsde::DistillArgs a = distill_args(logits, row_stride, dtype, V, K, ids, teacher, temperature);
  a.teacher_lse = teacher_lse;
  a.weight = weight;
  a.skip_zero = true;
  a.part = static_cast<dsde::DistillPartial *>(workspace);
  a.record = reinterpret_cast<dsde_distill_row *>(static_cast<char *>(workspace) + dsde::distill_part_bytes(N, V));
  a.loss = loss;
  a.row_err = row_err;
  a.grad = static_cast<char *>(grad);
  a.grad_stride = row_bytes(grad_stride, dtype);
  return dsde::launch_distill_step(a, N, static_cast<hipStream_t>(stream));
}

}  // extern "C"
