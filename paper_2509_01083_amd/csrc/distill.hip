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

// 2^(z c - ref c), one fused operation and an exponential.  ref c is rounded, by up to
// half a unit of its last place, but to the same number for every token that is weighed
// against it: a weight against ref itself is then 2^(ref c - scaled), within 2^(1/32) of 1 as long
// as |ref c| < 2^20.  Beyond that (chunks masked throughout, with -1e9 or the type's lowest
// value, say) the difference is taken first; the rounding would soon carry weights out of fp32's range.
struct Weigher {
  float ref, c, scaled;
  bool far;
  __device__ __forceinline__ Weigher(float M, float c_) : ref(finite_ref(M)), c(c_) {
    scaled = ref * c;
    far = !(fabsf(scaled) < 0x1p20f);
  }
  template <bool FAR>
  __device__ __forceinline__ float of(float z) const {
    return FAR ? row_weight(z, ref, c) : fast_exp2(fmaf(z, c, -scaled));
  }
  // the log2 that weights of 1 stand for
  __device__ __forceinline__ double base() const { return far ? double(ref) * double(c) : double(scaled); }
};
// A group's weights: four pairs in fp32, added in fp32.
template <bool FAR, typename G>
__device__ __forceinline__ float group_weight(const G &g, const Weigher &w) {
  const float a = w.template of<FAR>(g.at(0)) + w.template of<FAR>(g.at(1));
  const float b = w.template of<FAR>(g.at(2)) + w.template of<FAR>(g.at(3));
  const float d = w.template of<FAR>(g.at(4)) + w.template of<FAR>(g.at(5));
  const float e = w.template of<FAR>(g.at(6)) + w.template of<FAR>(g.at(7));
  return (a + b) + (d + e);
}

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

// Sums of one chunk of a row over the tokens outside the teacher's entries.  HBM-bound:
// 1,152 rows of 128,256 bf16 logits in 50 us (5.9 TB/s); behind the gradient's writes
// of an earlier call 4,096 rows take 200 us (5.3 TB/s).  With a difference and a
// product for each exponent, and pairs added in fp64, 55 and 219.
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
  const Weigher weigh(M, kLog2e / a.temperature);
  // groups in fp32, their sums in fp64: the loss is a small difference of logarithms
  double sum = 0.0;
  if (weigh.far) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += double(group_weight<true>(g[i], weigh));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += double(group_weight<false>(g[i], weigh));
  }
  sum = block_reduce<kWaves>(sum, red, lanes::Add{});
  if (t == 0) a.part[unit] = DistillPartial{bad ? NAN : M, tokens.twice, sum};
}

// The log2 of what a weight of 1 against `ref` stands for, against 2^(m c), and the factor that
// takes sums against `ref` to sums against `to`.
__device__ __forceinline__ double ref_log2(float ref, float m, float c) {
  return Weigher(ref, c).base() - double(m) * double(c);
}
__device__ __forceinline__ double ref_factor(float ref, float to, float c) {
  return exp2(Weigher(ref, c).base() - Weigher(to, c).base());
}

// The teacher's side of one row and the student's logits at its tokens, by one
// wavefront (entry k in lane k % 64), the same in every lane.  A row's few scalars take fp64's exp and
// log: 1 - sum p of a teacher of nearly one token, and the logarithm of a student's sum just over 1, are
// small differences, of which functions good to 1e-7 would leave a loss of 1e-5 two or three digits.
constexpr int kPerLane = DSDE_MAX_TOP / 64;
constexpr float kInf = __builtin_inff();
struct TeacherRow {
  uint32_t err;
  bool nothing;      // no entry with weight, and no mass outside the entries either
  float tmax, smax;  // largest logits of the teacher's entries and of the student's at them
  double scale;      // p_k = scale 2^((t_k - tmax) c)
  double sum;        // sum of p
  double cross;      // sum of p_k (log p_k - (s_k - smax) / T)
  double student;    // sum of exp((s_k - smax) / T)
};
__device__ __forceinline__ double entry_cross(float z, float tmax, float q, float smax, double iT) {
  return ((double(z) - double(tmax)) - (double(q) - double(smax))) * iT;
}
__device__ __forceinline__ TeacherRow teacher_row(const DistillArgs &a, int64_t n) {
  const int lane = threadIdx.x & 63;
  const char *row = a.rows.row(n);
  TeacherRow r;
  r.err = 0;
  float z[kPerLane], q[kPerLane];  // teacher and student logits
  r.tmax = r.smax = -kInf;
#pragma unroll
  for (int j = 0; j < kPerLane; ++j) {
    const int32_t k = lane + 64 * j;
    const int32_t id = k < a.K ? a.ids[n * a.K + k] : -1;
    if (id < -1 || id >= a.V) r.err |= DSDE_ERR_TOKEN;
    const bool used = id >= 0 && id < a.V;
    z[j] = used ? a.teacher[n * a.K + k] : -kInf;
    q[j] = used ? load_logit(row, a.dtype, id) : -kInf;
    if (!(z[j] < kInf) || !(q[j] < kInf) || (z[j] > -kInf && q[j] == -kInf)) r.err |= DSDE_ERR_LOGIT;
    r.tmax = fmaxf(r.tmax, z[j]);
    r.smax = fmaxf(r.smax, q[j]);
  }
  const bool tail = a.teacher_lse != nullptr;
  const double L = tail ? double(a.teacher_lse[n]) : 0.0;
  if (!(fabs(L) < double(kInf))) r.err |= DSDE_ERR_LOGIT;
  r.err = lanes::wave_or(r.err);
  r.tmax = lanes::wave_max(r.tmax);
  r.smax = lanes::wave_max(r.smax);
  r.nothing = !tail && r.tmax == -kInf;
  const double iT = 1.0 / double(a.temperature);
  const float c = kLog2e / a.temperature;
  double e[kPerLane], esum = 0.0;
  r.student = 0.0;
#pragma unroll
  for (int j = 0; j < kPerLane; ++j) {
    e[j] = 0.0;
    if (64 * j < a.K) {
      if (z[j] > -kInf) e[j] = double(row_weight(z[j], r.tmax, c));
      if (q[j] > -kInf) r.student += double(row_weight(q[j], r.smax, c));
    }
    esum += e[j];
  }
  r.student = lanes::wave_sum(r.student);
  esum = lanes::wave_sum(esum);
  // log p_k = (t_k - tmax) / T + log scale
  const double logs = r.tmax == -kInf ? 0.0 : tail ? double(r.tmax) * iT - L : -log(esum);
  r.scale = exp(logs);
  r.sum = esum * r.scale;
  double cross = 0.0;
#pragma unroll
  for (int j = 0; j < kPerLane; ++j)
    if (e[j] > 0.0) cross += e[j] * entry_cross(z[j], r.tmax, q[j], r.smax, iT);
  r.cross = lanes::wave_sum(cross) * r.scale + logs * r.sum;
  return r;
}

// The loss and the record of one row, from its teacher's side and the sums
// over the rest (the largest logit rmax there, and the sum of weights against
// it), in every lane of a wavefront.
struct RowLoss {
  float loss;
  uint32_t err;
  dsde_distill_row record;
};
__device__ __forceinline__ RowLoss row_loss(const DistillArgs &a, const TeacherRow &r, uint32_t err, float rmax,
                                            double rest) {
  const float m = fmaxf(r.smax, rmax);
  err |= r.err;
  if (m == -kInf) err |= DSDE_ERR_LOGIT;
  if (err || r.nothing)
    return RowLoss{err ? __builtin_nanf("") : 0.f, err, dsde_distill_row{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 1, 0}};
  const float c = kLog2e / a.temperature;
  const double ds = r.smax > -kInf ? (double(r.smax) - double(m)) * double(c) * kLn2 : 0.0;
  const double dr = rmax > -kInf ? ref_log2(rmax, m, c) * kLn2 : 0.0;
  const double es = exp(ds), er = rmax > -kInf ? exp(dr) : 0.0;
  const double S = r.student * es + rest * er, logS = log(S);
  const double tail = a.teacher_lse && r.sum < 1.0 ? 1.0 - r.sum : 0.0;
  double loss = r.cross - r.sum * (ds - logS), share = 0.0;  // share: what the rest's gradient adds up to
  if (rest > 0.0) {
    if (tail > 0.0) loss += tail * (log(tail) - (dr + log(rest) - logS));
    share = rest * er / S - tail;
  }
  return RowLoss{float(loss), 0,
                 dsde_distill_row{finite_ref(rmax), rest > 0.0 ? float(share / rest) : 0.f, m, float(1.0 / S),
                                  finite_ref(r.tmax), float(r.scale), 0, 0}};
}

// One wavefront per row: the loss, and the record that the gradient takes its
// exponentials against.
__global__ __launch_bounds__(kThreads) void distill_finish_kernel(const DistillArgs a, int64_t N, int32_t nc) {
  const int64_t n = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (n >= N) return;
  const int lane = threadIdx.x & 63;
  RowLoss out{0.f, 0, dsde_distill_row{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 1, 0}};
  if (!(a.skip_zero && a.weight[n] == 0.0f)) {
    uint32_t err = 0;
    float rmax = -kInf;
    const float c = kLog2e / a.temperature;
    const DistillPartial *part = a.part + n * nc;
    for (int32_t i = lane; i < nc; i += 64) {
      const DistillPartial x = part[i];
      if (!(x.max < kInf)) err |= DSDE_ERR_LOGIT;
      if (x.bad) err |= DSDE_ERR_TOKEN;
      rmax = fmaxf(rmax, x.max);
    }
    err = lanes::wave_or(err);
    rmax = lanes::wave_max(rmax);
    double rest = 0.0;  // against rmax
    if (rmax > -kInf && rmax < kInf)
      for (int32_t i = lane; i < nc; i += 64) {
        const DistillPartial x = part[i];
        if (x.max > -kInf) rest += x.sum * ref_factor(x.max, rmax, c);
      }
    rest = lanes::wave_sum(rest);
    out = row_loss(a, teacher_row(a, n), err, rmax, rest);
  }
  if (lane == 0) {
    a.loss[n] = out.loss;
    a.row_err[n] = out.err;
    a.record[n] = out.record;
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

// The teacher's probability of an entry, and the gradient there.
__device__ __forceinline__ float teacher_p(float logit, const dsde_distill_row &r, float c) {
  return row_weight(logit, r.teacher_ref, c) * r.teacher_scale;
}
__device__ __forceinline__ float entry_gradient(float z, float p, const dsde_distill_row &r, float c, float scale) {
  return scale * (row_weight(z, r.ref, c) * r.scale - p);
}

// The gradient of one chunk of a row.  It may overwrite the logits: every
// logit is read by the thread that writes its gradient.  HBM-bound: 4,096 rows of
// 128,256 bf16 logits in 352 us (6.0 TB/s read and written; torch's copy of 4 GiB
// runs at 4.6).  A form that held a row in the registers of 1,024 threads, to read it
// once for the sums and the gradient, took 628 us for both against 570: its CU's exponentials
// (two for every logit) and barriers did not hide behind its one row's traffic.
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
    s.p[j] = teacher_p(teacher[k], rec, c);
  });
  const float coef = rec.rest_scale * scale;
  const Weigher weigh(rec.rest_ref, c);
  const uint32_t listed = tokens.n;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    g[i].place(V, w0 + 256 * i);
    if (weigh.far) {
#pragma unroll
      for (int e = 0; e < kGroup; ++e) x[e] = coef * weigh.of<true>(g[i].at(e));
    } else {
#pragma unroll
      for (int e = 0; e < kGroup; ++e) x[e] = coef * weigh.of<false>(g[i].at(e));
    }
    const uint32_t bits = token_bits(tokens, 256 * i + t);
    if (bits) {
      for (uint32_t j = 0; j < listed; ++j) {
        const uint32_t off = uint32_t(tokens.at[j]) - uint32_t(256 * i + t) * kGroup;
        if (off < uint32_t(kGroup)) {
#pragma unroll
          for (int e = 0; e < kGroup; ++e)
            if (off == uint32_t(e)) x[e] = entry_gradient(g[i].at(e), tokens.p[j], rec, c, scale);
        }
      }
    }
    put_group<DT>(out, V, w0 + 256 * i, x);
  }
}

}  // namespace

// A launch takes fewer than 2^32 threads: rows of 2^23 chunks at a time (2^31 threads).
template <typename F>
static void each_pass(const DistillArgs &a0, int64_t N, F f) {
  const int64_t nc = num_chunks(a0.V), per_pass = (int64_t(1) << 23) / nc;
  for (int64_t r0 = 0; r0 < N; r0 += per_pass) {
    DistillArgs a = a0;
    a.rows.base += r0 * a.rows.stride;
    a.ids += r0 * a.K;
    a.teacher += r0 * a.K;
    if (a.teacher_lse) a.teacher_lse += r0;
    if (a.weight) a.weight += r0;
    if (a.part) a.part += r0 * nc;
    a.record += r0;
    if (a.loss) a.loss += r0;
    if (a.row_err) a.row_err += r0;
    if (a.grad) a.grad += r0 * a.grad_stride;
    f(a, N - r0 < per_pass ? N - r0 : per_pass, int32_t(nc));
  }
}
static_assert((int64_t(1) << 23) / (DSDE_MAX_VOCAB / kChunk) > 0, "a row fits a launch");

int launch_distill_loss(const DistillArgs &a0, int64_t N, hipStream_t stream) {
  (void)hipGetLastError();
  const int form = strided_rows_form(a0.rows.base, a0.rows.stride, a0.dtype, a0.V);
  each_pass(a0, N, [&](const DistillArgs &a, int64_t n, int32_t nc) {
    by_rows(a.dtype, form, [&](auto dt, auto row) {
      distill_scan_kernel<decltype(dt)::value, decltype(row)::value>
          <<<dim3(unsigned(n * nc)), dim3(kThreads), 0, stream>>>(a, nc);
    });
    distill_finish_kernel<<<dim3(unsigned((n + kWaves - 1) / kWaves)), dim3(kThreads), 0, stream>>>(a, n, nc);
  });
  return hipGetLastError() == hipSuccess ? DSDE_OK : DSDE_DEVICE_ERROR;
}

int launch_distill_grad(const DistillArgs &a0, int64_t N, hipStream_t stream) {
  (void)hipGetLastError();
  const int form = strided_rows_form(a0.rows.base, a0.rows.stride, a0.dtype, a0.V);
  each_pass(a0, N, [&](const DistillArgs &a, int64_t n, int32_t nc) {
    by_rows(a.dtype, form, [&](auto dt, auto row) {
      distill_grad_kernel<decltype(dt)::value, decltype(row)::value>
          <<<dim3(unsigned(n * nc)), dim3(kThreads), 0, stream>>>(a, nc);
    });
  });
  return hipGetLastError() == hipSuccess ? DSDE_OK : DSDE_DEVICE_ERROR;
}

int launch_distill_step(const DistillArgs &a, int64_t N, hipStream_t stream) {
  const int rc = launch_distill_loss(a, N, stream);
  return rc != DSDE_OK ? rc : launch_distill_grad(a, N, stream);
}

}  // namespace dsde
