// Distillation from a teacher's top logits: the divergence of a row's softmax
// from the teacher's K entries (and, with the teacher's log-normaliser, the
// mass it gives to all other tokens together), and its gradient.
//
// With q = softmax(s / T) over the row, I the teacher's tokens and, of the
// others together, q_r = sum of q outside I and r = 1 - sum of p:
//   loss = sum_k p_k (log p_k - log q_k) + r (log r - log q_r)
//   T dloss/ds_v = q_v - p_k for v = i_k, and (q_v / q_r) (q_r - r) for the rest
// (without the normaliser: p a softmax over the entries, r = 0).  The rest is
// summed apart from the entries, against a maximum of its own: a student that agrees with
// its teacher leaves it 1e-4 of the row and less, which a difference of
// whole-row sums in fp32 would lose, and q_v / q_r keeps its scale where q_r is 0 in fp32.
#include "rows.hpp"
#include "rows_args.hpp"

namespace dsde {
namespace {

// The teacher's tokens in one chunk: a bit per logit, eight logits (a group) to
// a byte, and for the gradient their list.
struct ChunkTokens {
  uint32_t map[kChunkGroups / 4];
  uint32_t n, twice;
  uint16_t at[DSDE_MAX_TOP];
  float p[DSDE_MAX_TOP];
};

// Fills the chunk's map (and list) with 256 threads; ends with a barrier.
template <typename P>
__device__ __forceinline__ void mark_tokens(ChunkTokens &c, const int32_t *ids, int32_t K, int32_t chunk, int64_t V,
                                            P probability) {
  const int t = threadIdx.x;
  c.map[t] = 0;
  if (t == 0) c.n = c.twice = 0;
  const int32_t id = t < K ? ids[t] : -1;
  __syncthreads();
  const uint32_t local = uint32_t(id) - uint32_t(chunk) * kChunk;
  if (id >= 0 && id < V && local < uint32_t(kChunk)) {
    const uint32_t bit = 1u << (local & 31);
    if (atomicOr(&c.map[local >> 5], bit) & bit) c.twice = 1;
    probability(c, t, local);
  }
  __syncthreads();
}
static_assert(DSDE_MAX_TOP <= kThreads, "one entry per thread");
__device__ __forceinline__ uint32_t token_bits(const ChunkTokens &c, int group) {
  return reinterpret_cast<const uint8_t *>(c.map)[group];
}

// Sums of one chunk of a row over the tokens outside the teacher's entries.
template <int DT, int ROW>
__global__ __launch_bounds__(kThreads) void distill_scan_kernel(const DistillArgs a, int32_t nc) {
  __shared__ ChunkTokens tokens;
  __shared__ float redf[kWaves];
  __shared__ double red[kWaves];
  const int64_t unit = blockIdx.x, n = unit / nc;
  const int32_t chunk = int32_t(unit - n * nc);
  if (a.skip_zero && a.weight[n] == 0.0f) return;
  const int t = threadIdx.x;
  const uint32_t V = uint32_t(a.V), w0 = uint32_t(chunk) * kChunkGroups + t;
  const char *row = a.rows.row(n);
  Group<DT, ROW> g[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i].get(row, V, w0 + 256 * i);
  mark_tokens(tokens, a.ids + n * a.K, a.K, chunk, a.V, [](ChunkTokens &, int, uint32_t) {});
  float tm = -INFINITY;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    g[i].place(V, w0 + 256 * i);
    const uint32_t bits = token_bits(tokens, 256 * i + t);
    if (bits) {
#pragma unroll
      for (int e = 0; e < kGroup; ++e)
        if (bits >> e & 1) g[i].drop(e);
    }
    tm = max_nan(tm, g[i].max());
  }
  const bool bad = __syncthreads_or(tm != tm);
  const float M = block_max(tm, redf);
  const float ref = finite_ref(M), c = kLog2e / a.temperature;
  // pairs in fp32, their sums in fp64: the loss is a small difference of logarithms
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < kGroup; e += 2)
      sum += double(row_weight(g[i].at(e), ref, c) + row_weight(g[i].at(e + 1), ref, c));
  sum = block_reduce<kWaves>(sum, red, lanes::Add{});
  if (t == 0) a.part[unit] = DistillPartial{bad ? NAN : M, tokens.twice, sum};
}

// One wavefront per row: the loss, and the record that the gradient takes its
// exponentials against.
__global__ __launch_bounds__(kThreads) void distill_finish_kernel(const DistillArgs a, int64_t N, int32_t nc) {
  const int64_t n = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (n >= N) return;
  const int lane = threadIdx.x & 63;
  constexpr int kPer = DSDE_MAX_TOP / 64;
  constexpr float kInf = __builtin_inff();
  if (a.skip_zero && a.weight[n] == 0.0f) {
    if (lane == 0) {
      a.loss[n] = 0.f;
      a.row_err[n] = 0;
      a.record[n] = dsde_distill_row{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 1, 0};
    }
    return;
  }
  uint32_t err = 0;
  bool used[kPer];
  float z[kPer], q[kPer];  // teacher and student logits
  float tmax = -kInf, smax = -kInf;
  const char *row = a.rows.row(n);
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int32_t k = lane + 64 * j;
    const int32_t id = k < a.K ? a.ids[n * a.K + k] : -1;
    if (id < -1 || id >= a.V) err |= DSDE_ERR_TOKEN;
    used[j] = id >= 0 && id < a.V;
    z[j] = used[j] ? a.teacher[n * a.K + k] : -kInf;
    q[j] = used[j] ? load_logit(row, a.dtype, id) : -kInf;
    if (!(z[j] < kInf) || !(q[j] < kInf) || (z[j] > -kInf && q[j] == -kInf)) err |= DSDE_ERR_LOGIT;
    tmax = fmaxf(tmax, z[j]);
    smax = fmaxf(smax, q[j]);
  }
  float rmax = -kInf;
  for (int32_t i = lane; i < nc; i += 64) {
    const DistillPartial x = a.part[n * nc + i];
    if (!(x.max < kInf)) err |= DSDE_ERR_LOGIT;
    if (x.bad) err |= DSDE_ERR_TOKEN;
    rmax = fmaxf(rmax, x.max);
  }
  const bool tail = a.teacher_lse != nullptr;
  const double L = tail ? double(a.teacher_lse[n]) : 0.0;
  if (!(fabs(L) < double(kInf))) err |= DSDE_ERR_LOGIT;
  err = lanes::wave_or(err);
  tmax = lanes::wave_max(tmax);
  smax = lanes::wave_max(smax);
  rmax = lanes::wave_max(rmax);
  const float m = fmaxf(smax, rmax);
  if (m == -kInf) err |= DSDE_ERR_LOGIT;
  const bool nothing = !tail && tmax == -kInf;  // no teacher at all
  if (err || nothing) {
    if (lane == 0) {
      a.loss[n] = err ? NAN : 0.f;
      a.row_err[n] = err;
      a.record[n] = dsde_distill_row{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 1, 0};
    }
    return;
  }
  const double iT = 1.0 / double(a.temperature);
  double rest = 0.0;  // against rmax
  if (rmax > -kInf)
    for (int32_t i = lane; i < nc; i += 64) {
      const DistillPartial x = a.part[n * nc + i];
      if (x.max > -kInf) rest += x.sum * exp((double(x.max) - double(rmax)) * iT);
    }
  rest = lanes::wave_sum(rest);
  double top = 0.0, tsum = 0.0, e[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    e[j] = z[j] > -kInf ? exp((double(z[j]) - double(tmax)) * iT) : 0.0;
    tsum += e[j];
    if (q[j] > -kInf) top += exp((double(q[j]) - double(m)) * iT);
  }
  top = lanes::wave_sum(top);
  tsum = lanes::wave_sum(tsum);
  const double rest_at = rmax > -kInf ? exp((double(rmax) - double(m)) * iT) : 0.0;
  const double S = top + rest * rest_at, logS = log(S);
  // log p_k = (z_k - tmax) / T + log t0, p_k = e_k t0
  const double logt0 = tmax == -kInf ? 0.0 : tail ? double(tmax) * iT - L : -log(tsum), t0 = exp(logt0);
  double loss = 0.0, psum = 0.0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const double p = e[j] * t0;
    psum += p;
    if (p > 0.0)
      loss += p * ((double(z[j]) - double(tmax)) * iT + logt0 - ((double(q[j]) - double(m)) * iT - logS));
  }
  loss = lanes::wave_sum(loss);
  psum = lanes::wave_sum(psum);
  double r = tail && psum < 1.0 ? 1.0 - psum : 0.0, share = 0.0;  // share: what the rest's gradient adds up to
  if (rmax > -kInf) {
    const double qr = rest * rest_at / S;
    if (r > 0.0) loss += r * (log(r) - ((double(rmax) - double(m)) * iT + log(rest) - logS));
    share = qr - r;
  }
  if (lane == 0) {
    a.loss[n] = float(loss);
    a.row_err[n] = 0;
    a.record[n] = dsde_distill_row{finite_ref(rmax), rest > 0.0 ? float(share / rest) : 0.f, m, float(1.0 / S),
                                   finite_ref(tmax), float(t0), 0, 0};
  }
}

// Eight gradients of a row, rounded once to its type; the last group of a row may be shorter.
template <int DT>
__device__ __forceinline__ void put_group(char *row, uint32_t V, uint32_t w, const float (&x)[kGroup]) {
  const uint32_t v0 = w * kGroup;
  if (v0 >= V) return;
  if constexpr (DT == DSDE_BF16) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    u32x4_t o;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      o[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
    if (v0 + kGroup <= V) {
      __builtin_nontemporal_store(o, reinterpret_cast<u32x4_a2_t *>(row + 2 * size_t(v0)));
    } else {
#pragma unroll
      for (int i = 0; i < kGroup; ++i)
        if (v0 + i < V) reinterpret_cast<uint16_t *>(row)[v0 + i] = uint16_t(o[i / 2] >> (16 * (i & 1)));
    }
  } else {
    float *p = reinterpret_cast<float *>(row) + v0;
    if (v0 + kGroup <= V) {
      __builtin_nontemporal_store(f32x4_t{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4_a4_t *>(p));
      __builtin_nontemporal_store(f32x4_t{x[4], x[5], x[6], x[7]}, reinterpret_cast<f32x4_a4_t *>(p + 4));
    } else {
#pragma unroll
      for (int i = 0; i < kGroup; ++i)
        if (v0 + i < V) p[i] = x[i];
    }
  }
}

// The gradient of one chunk of a row.  It may overwrite the logits: every
// logit is read by the thread that writes its gradient.
template <int DT, int ROW>
__global__ __launch_bounds__(kThreads) void distill_grad_kernel(const DistillArgs a, int32_t nc) {
  __shared__ ChunkTokens tokens;
  const int64_t unit = blockIdx.x, n = unit / nc;
  const int32_t chunk = int32_t(unit - n * nc);
  const int t = threadIdx.x;
  const uint32_t V = uint32_t(a.V), w0 = uint32_t(chunk) * kChunkGroups + t;
  char *out = a.grad + n * a.grad_stride;
  const dsde_distill_row rec = a.record[n];
  const float weight = a.weight[n];
  float x[kGroup];
  if (rec.empty || weight == 0.0f) {
#pragma unroll
    for (int e = 0; e < kGroup; ++e) x[e] = 0.f;
    for (int i = 0; i < 4; ++i) put_group<DT>(out, V, w0 + 256 * i, x);
    return;
  }
  const char *row = a.rows.row(n);
  Group<DT, ROW> g[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i].get(row, V, w0 + 256 * i);
  const float c = kLog2e / a.temperature, scale = weight / a.temperature;
  const float *teacher = a.teacher + n * a.K;
  mark_tokens(tokens, a.ids + n * a.K, a.K, chunk, a.V, [&](ChunkTokens &s, int k, uint32_t local) {
    const uint32_t j = atomicAdd(&s.n, 1u);
    s.at[j] = uint16_t(local);
    s.p[j] = row_weight(teacher[k], rec.teacher_ref, c) * rec.teacher_scale;
  });
  const float coef = rec.rest_scale * scale;
  const uint32_t listed = tokens.n;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    g[i].place(V, w0 + 256 * i);
#pragma unroll
    for (int e = 0; e < kGroup; ++e) x[e] = coef * row_weight(g[i].at(e), rec.rest_ref, c);
    const uint32_t bits = token_bits(tokens, 256 * i + t);
    if (bits) {
      for (uint32_t j = 0; j < listed; ++j) {
        const uint32_t off = uint32_t(tokens.at[j]) - uint32_t(256 * i + t) * kGroup;
        if (off < uint32_t(kGroup)) {
#pragma unroll
          for (int e = 0; e < kGroup; ++e)
            if (off == uint32_t(e)) x[e] = scale * (row_weight(g[i].at(e), rec.ref, c) * rec.scale - tokens.p[j]);
        }
      }
    }
    put_group<DT>(out, V, w0 + 256 * i, x);
  }
}

}  // namespace

int launch_distill_loss(const DistillArgs &a, int64_t N, hipStream_t stream) {
  (void)hipGetLastError();
  const int32_t nc = int32_t(num_chunks(a.V));
  by_rows(a.dtype, strided_rows_form(a.rows.base, a.rows.stride, a.dtype, a.V), [&](auto dt, auto row) {
    distill_scan_kernel<decltype(dt)::value, decltype(row)::value>
        <<<dim3(unsigned(N * nc)), dim3(kThreads), 0, stream>>>(a, nc);
  });
  distill_finish_kernel<<<dim3(unsigned((N + kWaves - 1) / kWaves)), dim3(kThreads), 0, stream>>>(a, N, nc);
  return hipGetLastError() == hipSuccess ? DSDE_OK : DSDE_DEVICE_ERROR;
}

int launch_distill_grad(const DistillArgs &a, int64_t N, hipStream_t stream) {
  (void)hipGetLastError();
  const int32_t nc = int32_t(num_chunks(a.V));
  by_rows(a.dtype, strided_rows_form(a.rows.base, a.rows.stride, a.dtype, a.V), [&](auto dt, auto row) {
    distill_grad_kernel<decltype(dt)::value, decltype(row)::value>
        <<<dim3(unsigned(N * nc)), dim3(kThreads), 0, stream>>>(a, nc);
  });
  return hipGetLastError() == hipSuccess ? DSDE_OK : DSDE_DEVICE_ERROR;
}

int launch_distill_step(const DistillArgs &a, int64_t N, hipStream_t stream) {
  const int rc = launch_distill_loss(a, N, stream);
  return rc != DSDE_OK ? rc : launch_distill_grad(a, N, stream);
}

}  // namespace dsde
