// Sampling (temperature, top-k, top-p, min-p) and the k largest logits of rows.
//
// Both order a row by (logit descending, id ascending) and need its first
// tokens: the kept set of every filter is a prefix of that order.
//   row_scan_kernel  reads each row once, one workgroup per chunk of 8,192 logits, and
//                    leaves per chunk its maximum, the weight of each of its 16 segments
//                    of 512 logits (the largest logits apart from the rest), and the
//                    16-bit ordered key of the largest logit of each group of 8: an
//                    eighth of the row's length in keys;
//   select_kernel    one workgroup per row: draws without filters from the segments'
//                    weights; else finds from the keys alone a threshold that enough groups
//                    reach, reads those groups again, sorts the few logits that reach it too, and cuts;
//   wide_kernel      rows whose filters keep more tokens than that: cuts by histograms.
#include "rows.hpp"
#include "rows_args.hpp"
#include "select_device.hpp"

namespace dsde {
namespace {

constexpr int kMostNeed = 256;      // groups asked for at most: about 1.4 times as many reach their threshold
constexpr int kFirstNeed = 56;      // groups that a row without a top-k asks for: about 60 candidates, one wavefront's sort
constexpr int32_t kUndecided = 0x7fffffff;

// One row's settings, checked.  Greedy rows (T = 0) are rows with top_k = 1.
struct Setting {
  float T, c;  // c = log2(e) / T
  int32_t k;
  float p, m, u;
  uint32_t err;
  bool filtered;
};
__device__ __forceinline__ Setting row_setting(const SelectArgs &a, int64_t r) {
  Setting s;
  s.err = 0;
  float T = a.temperature ? a.temperature[r] : a.one_temperature;
  s.k = a.top_k ? a.top_k[r] : a.one_k;
  s.p = a.top_p ? a.top_p[r] : 1.0f;
  s.m = a.min_p ? a.min_p[r] : 0.0f;
  s.u = a.u ? a.u[r] : 0.0f;
  if (T == 0.0f) {
    T = 1.0f;
    s.k = 1;
    s.p = 1.0f;
    s.m = 0.0f;
    s.u = 0.0f;
  }
  if (!(T >= kMinTemp && T <= kMaxTemp)) s.err |= DSDE_ERR_TEMP;
  if (!(s.p > 0.0f && s.p <= 1.0f) || !(s.m >= 0.0f && s.m <= 1.0f)) s.err |= DSDE_ERR_FILTER;
  if (!(s.u >= 0.0f && s.u < 1.0f)) s.err |= DSDE_ERR_UNIFORM;
  s.T = s.err ? 1.0f : T;
  s.c = kLog2e / s.T;
  if (s.k < 0 || s.k >= a.V) s.k = 0;
  s.filtered = s.k > 0 || s.p < 1.0f || s.m > 0.0f;
  return s;
}

// ---------------------------------------------------------------------------
// the pass over the logits
// ---------------------------------------------------------------------------

// Per logit a subtraction, a product, an exponential and an addition, against the
// chunk's own maximum, so that no chunk waits for another; HBM-bound.  1,024 rows of
// 128,256 bf16 logits take 42.6 us (6.2 TB/s; a plain read of that size runs at 6.9).
// With keys (an eighth of the bytes, written) 1,408 rows take 68 us.  The weights are added
// in fp32, over the eight of a group and then across the wavefront: a segment is good to 6e-7 of itself at
// worst.  The largest logits, weights of 1, stay out of its sum (SegWeight).
template <int DT, int ROW>
__global__ __launch_bounds__(kThreads) void row_scan_kernel(const SelectArgs a, int64_t row0, int32_t nc) {
  __shared__ float red[kWaves];
  const int64_t unit = blockIdx.x, r = unit / nc;
  const int32_t chunk = int32_t(unit - r * nc);
  const int t = threadIdx.x;
  const uint32_t V = uint32_t(a.V), w0 = uint32_t(chunk) * kChunkGroups + t;
  const char *row = a.rows.row(row0 + r);
  Group<DT, ROW> g[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i].get(row, V, w0 + 256 * i);
  const Setting s = row_setting(a, row0 + r);
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i].place(V, w0 + 256 * i);
  float gm[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) gm[i] = g[i].max();
  const float tm = max_nan(max_nan(gm[0], gm[1]), max_nan(gm[2], gm[3]));
  // a NaN must reach the maximum whatever the lanes' order
  const bool bad = __syncthreads_or(tm != tm);
  const float M = block_max(tm, red);
  float seg[4];
  const float ref = finite_ref(M);
  const int wave = t >> 6, lane = t & 63;
  uint32_t ones = 0;  // in lane i: of segment i of the wavefront
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x = 0.f, y = 0.f;
#pragma unroll
    for (int e = 0; e < kGroup; e += 2) {
      x += row_weight(g[i].at(e), ref, s.c);
      y += row_weight(g[i].at(e + 1), ref, s.c);
    }
    seg[i] = x + y;
    if (__ballot(gm[i] == ref)) {  // one wavefront of the chunk, as a rule: the largest logits apart
      uint32_t n = 0;
      x = 0.f;
#pragma unroll
      for (int e = 0; e < kGroup; ++e) {
        const float z = g[i].at(e);
        n += z == ref;
        x += z == ref ? 0.f : row_weight(z, ref, s.c);
      }
      seg[i] = x;
      n = lanes::wave_sum(n);
      if (lane == i) ones = n;
    }
  }
  const float rest = lanes::wave_sum4(seg);
  // segment 4 i + wave of the chunk: groups 256 i + 64 wave ...
  if (lane < 4) a.scan.seg[unit * kSegs + 4 * lane + wave] = SegWeight{float(ones), rest};
  if (t == 0) a.scan.max[unit] = bad ? NAN : M;
  if (t == 0 && unit == 0) *a.scan.n_wide = 0;
  if (a.keys_always || s.filtered) {
    // a thread's four keys together: group 256 i + t of the chunk at place 4 t + i (place_group)
    const uint32_t lo = (order_key(gm[0]) >> 16) | (order_key(gm[1]) & 0xffff0000u);
    const uint32_t hi = (order_key(gm[2]) >> 16) | (order_key(gm[3]) & 0xffff0000u);
    reinterpret_cast<uint2 *>(a.scan.keys + unit * kChunkGroups)[t] = make_uint2(lo, hi);
  }
}

// ---------------------------------------------------------------------------
// the two kernels behind it
// ---------------------------------------------------------------------------

__device__ __forceinline__ double log_of(const RowSum &s) {
  return s.ones == 1.0 ? log1p(s.rest) : log(s.ones) + log1p(s.rest / s.ones);
}
__device__ __forceinline__ float row_logprob(float z, float m, float T, const RowSum &s) {
  return float((double(z) - double(m)) / double(T) - log_of(s));
}

// A little below the smallest logit that min_p keeps, as the upper half of a key.
__device__ __forceinline__ uint32_t min_p_key(const Setting &s, float m) {
  if (!(s.m > 0.f)) return 0;
  const float d = log2f(s.m) / s.c;
  return order_key(m + d - 1e-5f * (1.f + fabsf(m) + fabsf(d))) >> 16;
}

// One row per workgroup of 512 threads: 40 keys of a 163,840-token row per thread,
// and one thread for each candidate.  Bound by a chain of some ten dependent steps
// (round trips to the last-level cache for the row's sums, keys and groups; barriers): 11.1 us for a row with a nucleus.
// With many rows it is the instructions of its eight wavefronts: the 64 largest of
// 1,408 rows take 28.7 us.  (With 1,024 threads and a histogram of all keys: 53 us
// and 103 us.)
template <int DT, int ROW, bool TOP>
__global__ __launch_bounds__(kSelThreads, 4) void select_kernel(const SelectArgs a, int64_t row0, int32_t nc) {
  using LDS = std::conditional_t<TOP, TopLds, DrawLds>;
  constexpr int W = LDS::kWaves;
  __shared__ LDS L;
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x, out = row0 + r;
  const Setting s = row_setting(a, out);
  const float *cmax = a.scan.max + r * nc;
  const SegWeight *seg = a.scan.seg + r * nc * kSegs;
  const int32_t nseg = nc * kSegs;
  const uint32_t V = uint32_t(a.V);
  Selector<DT, ROW, LDS> sel{a.rows.row(out), a.scan.keys + r * nc * kChunkGroups, V, (V + kGroup - 1) / kGroup,
                        uint32_t(nc) * kChunkGroups, 0.f, s.c, L, {}, false, false, 0, 9};
  // the loads that the kernel starts with, together
  float first_max = -INFINITY, first_ref = -INFINITY;
  SegWeight first_seg{0.f, 0.f};
  if (t < nc) first_max = cmax[t];
  if (t < nseg) {
    first_seg = seg[t];
    first_ref = cmax[t / kSegs];
  }
  if (TOP || s.filtered) sel.tile.load(sel.keys, sel.places, 0);

  float mt = first_max;
  bool bad = !(mt < INFINITY);
  // (a row has at most 512 chunks: one per thread)
  bad = __syncthreads_or(bad);
  const float m = block_reduce<W>(mt, L.redf, lanes::Max{});
  const uint32_t err = s.err | (bad || m == -INFINITY ? DSDE_ERR_LOGIT : 0u);
  if (t == 0) a.row_err[out] = err;
  if (err) {
    if constexpr (TOP) {
      for (int32_t i = t; i < a.one_k; i += kSelThreads) {
        a.values[out * a.one_k + i] = NAN;
        a.ids[out * a.one_k + i] = -1;
      }
      if (t == 0) a.lse[out] = NAN;
    } else if (t == 0) {
      a.tokens[out] = a.pad_id;
      if (a.logprob) a.logprob[out] = NAN;
      if (a.kept) a.kept[out] = 0;
    }
    return;
  }
  sel.m = m;
  // a segment's weight against m
  auto seg_weight = [&](const SegWeight &x, float ref) {
    return (double(x.ones) + double(x.rest)) * double(row_weight(ref, m, s.c));
  };
  const double part0 = seg_weight(first_seg, first_ref);
  RowSum S{0.0, 0.0};
  auto add = [&](const SegWeight &x, float ref, double weight) {
    S.ones += ref == m ? double(x.ones) : 0.0;
    S.rest += ref == m ? double(x.rest) : weight;
  };
  add(first_seg, first_ref, part0);
  for (int32_t i = t + kSelThreads; i < nseg; i += kSelThreads) {
    const float ref = cmax[i / kSegs];
    add(seg[i], ref, seg_weight(seg[i], ref));
  }
  block_sum2<W>(S.ones, S.rest, reinterpret_cast<double *>(L.red64));

  auto emit = [&](int32_t token, float z, int32_t kept) {
    a.tokens[out] = token;
    if (a.logprob) a.logprob[out] = row_logprob(z, m, s.T, S);
    if (a.kept) a.kept[out] = kept;
  };

  if constexpr (TOP) {
    if (t == 0) a.lse[out] = float(double(m) / double(s.T) + log_of(S));
    const int32_t k = a.one_k;
    uint64_t v = 0;
    int32_t n = sel.gather(sel.threshold(uint32_t(k)), &v);
    if (n < 0) {
      // more logits than threads reach that threshold: long runs of equal or nearby ones
      sel.list_logits(sel.exact_threshold(uint32_t(k)));
      const uint64_t cut = sel.template key_cut<false>(uint64_t(k)).at;
      if (t == 0) L.n_cand = 0;
      __syncthreads();
      sel.each([&](uint32_t key, float, uint32_t id) {
        const uint64_t x = packed(key, id);
        if (x >= cut) {
          const uint32_t i = atomicAdd(&L.n_cand, 1u);
          if (i < kSelThreads) L.cand[i] = x;
        }
      });
      __syncthreads();
      n = int32_t(min(L.n_cand, uint32_t(kSelThreads)));
      v = t < n ? L.cand[t] : 0;
      __syncthreads();
      block_sort<kSelThreads>(v, uint32_t(n), L.cand);
    }
    if (t < k) {
      a.values[out * k + t] = t < n ? key_logit(uint32_t(v >> 32)) : -INFINITY;
      a.ids[out * k + t] = t < n ? int32_t(~uint32_t(v)) : -1;
    }
    return;
  } else {
    if (!s.filtered) {
      const uint32_t n = a.kept ? block_reduce<W>(sel.unmasked(), L.red32, lanes::Add{}) : 0u;
      // A segment's weight is a product of two, of which the smaller may be of any size, while its
      // tokens are weighed against m at once and vanish under 2^-126: of 512 that add up to 2^-116 one does not.
      sel.draw_segment(nseg, s.u, [&](int32_t i) {
        const double x = i == t ? part0 : seg_weight(seg[i], cmax[i / kSegs]);
        return x >= 0x1p-116 ? x : 0.0;
      });
      if (t < 64) {
        int32_t token;
        float z;
        sel.draw_token(1, kEvery, 0.f, &token, &z);
        if (t == 0) emit(token, z, int32_t(n));
      }
      return;
    }

    const uint32_t min_key = min_p_key(s, m);
    // Few tokens kept: candidates, a prefix of the row's order, sorted.  Where its
    // length does not settle every filter, the cuts of wide_kernel.
    if (s.k <= kMostNeed) {
      uint32_t kappa = sel.threshold(s.k > 0 ? s.k : kFirstNeed);
      const bool min_decided = min_key >= kappa;
      if (min_decided) kappa = min_key;
      const bool all = kappa == kAll;
      uint64_t v = 0;
      const int32_t n = sel.gather(kappa, &v);
      int32_t kept = kUndecided;
      if (n >= 0) {
        const float e = t < n ? sel.weight(key_logit(uint32_t(v >> 32))) : 0.f;
        const BlockScan<double> cs = block_scan<W>(double(e), reinterpret_cast<double *>(L.red64));
        const bool k_in = s.k > 0 && s.k <= n;
        if (k_in && t == s.k - 1) L.mass = cs.incl;
        const int32_t n_min = __syncthreads_count(t < n && e >= s.m);
        const double mass = k_in ? L.mass : all ? cs.total : S.ones + S.rest;
        const int32_t n_below = __syncthreads_count(t < n && cs.incl < double(s.p) * mass);
        int32_t lim = kUndecided;
        if (k_in) lim = s.k;
        if (all) lim = min(lim, n);
        if (s.m > 0.f && (n_min < n || all || min_decided)) lim = min(lim, n_min);
        bool known = true;
        if (s.p < 1.f) {
          known = k_in || all || s.k == 0;  // else top_p's share is of a mass beyond the candidates
          if (n_below < n) lim = min(lim, n_below + 1);
        }
        if (known && lim != kUndecided) kept = max(lim, 1);
      }
      if (kept != kUndecided) {
        // the draw walks the kept tokens in the order of their ids; up to 64 of them lie in one wavefront
        const bool one_wave = kept <= 64;
        if (one_wave && t >= 64) return;
        uint64_t x = t < kept ? (v << 32) | uint32_t(t) : 0;  // (~id, rank)
        if (!one_wave) L.elems[t] = v;
        block_sort<kSelThreads>(x, uint32_t(kept), L.cand);
        const uint32_t key = one_wave ? __shfl(uint32_t(v >> 32), int(uint32_t(x)))
                                      : uint32_t(L.elems[uint32_t(x)] >> 32);
        const float z = key_logit(key);
        const double e = t < kept ? double(sel.weight(z)) : 0.0;
        int32_t at;
        if (one_wave) {
          const double incl = lanes::wave_scan(e).incl, total = lanes::readlane(incl, 63);
          at = __popcll(__ballot(t < kept && incl <= double(s.u) * total));
        } else {
          const BlockScan<double> cs = block_scan<W>(e, reinterpret_cast<double *>(L.red64));
          at = __syncthreads_count(t < kept && cs.incl <= double(s.u) * cs.total);
        }
        if (t == min(at, kept - 1)) emit(int32_t(~uint32_t(x >> 32)), z, kept);
        return;
      }
    }
    if (t == 0) a.scan.wide[atomicAdd(a.scan.n_wide, 1u)] = WideRow{int32_t(r), m, S};
  }
}

// The rows that the select kernel has left: cuts by histograms over the logits
// that may lie above them, then the draw over segments.  A kernel of its own, since
// its lists take the LDS of a CU: with them in the select kernel, 256 mixed rows
// took 105 us in two kernels, 74 in three; a call none of whose rows needs it pays 2 to 4 us.
// A row whose cut lies within the 10,000 largest logits takes about 28 us on its CU for V =
// 50,257 and 42 for V = 128,256, about half of it the listing; beyond that its passes over all logits are
// bound by their instructions (by the code's count, some 280 per group of 8): 92 us for V = 128,256.
// Rows with fewer unmasked tokens than top_k end in key_cut, a pass over all logits for every 2,048
// values of the keys' upper halves from the maximum down: 256 rows of V = 128,256 masked to 300
// tokens, with top_k = 500, take 410 us (-inf) and 720 (the type's lowest value) against 55 unmasked.
template <int DT, int ROW>
__global__ __launch_bounds__(kWideThreads) void wide_kernel(const SelectArgs a, int64_t row0, int32_t nc) {
  __shared__ WideLds L;
  const int t = threadIdx.x;
  const uint32_t n = *a.scan.n_wide, V = uint32_t(a.V);
  for (uint32_t i = blockIdx.x; i < n; i += gridDim.x) {
    const WideRow w = a.scan.wide[i];
    const int64_t out = row0 + w.row;
    const Setting s = row_setting(a, out);
    Selector<DT, ROW, WideLds> sel{a.rows.row(out), a.scan.keys + int64_t(w.row) * nc * kChunkGroups, V,
                                   (V + kGroup - 1) / kGroup, uint32_t(nc) * kChunkGroups, w.max, s.c, L, {}, false,
                                   false, 0, 9};
    sel.tile.load(sel.keys, sel.places, 0);
    int32_t kept = 0;
    const double sum = w.sum.ones + w.sum.rest;
    sel.list_relevant(s.k, s.p, float(sum), min_p_key(s, w.max));
    Cut cut{kEvery, uint64_t(sum * double(kFixed))};
    const bool by_p = s.p < 1.f;
    if (s.k > 0 || by_p) sel.histogram();
    if (s.k > 0) cut = sel.template weight_cut<false>(uint64_t(s.k), !by_p, s.m, &kept);
    if (by_p) {
      const uint64_t target = uint64_t(double(s.p) * double(cut.mass));
      if (s.k > 0) sel.histogram();
      cut = sel.template weight_cut<true>(target ? target : 1, true, s.m, &kept);
    } else if (s.k == 0) {
      sel.add_segments(kEvery, s.m, &kept);
    }
    const uint32_t count = block_reduce<WideLds::kWaves>(uint32_t(kept), L.red32, lanes::Add{});
    sel.draw_segment(sel.nseg, s.u, [&](int32_t j) { return double(L.segs[j]) * (1.0 / double(kFixed)); });
    if (t < 64) {
      int32_t token;
      float z;
      sel.draw_token(1 << (sel.seg_shift - 9), cut.at, s.m, &token, &z);
      if (t == 0) {
        a.tokens[out] = token;
        if (a.logprob) a.logprob[out] = row_logprob(z, w.max, s.T, w.sum);
        if (a.kept) a.kept[out] = int32_t(count);
      }
    }
    __syncthreads();
  }
}

template <bool TOP>
int launch(const SelectArgs &a0, int64_t R, hipStream_t stream) {
  (void)hipGetLastError();
  const int32_t nc = int32_t(num_chunks(a0.V));
  const int64_t per_pass = select_rows_per_pass(R, a0.V);
  const int form = strided_rows_form(a0.rows.base, a0.rows.stride, a0.dtype, a0.V);
  SelectArgs a = a0;
  a.keys_always = TOP;
  const SelectLayout l = select_layout(R, a.V);
  char *ws = static_cast<char *>(a.workspace);
  a.scan.max = reinterpret_cast<float *>(ws + l.max);
  a.scan.seg = reinterpret_cast<SegWeight *>(ws + l.seg);
  a.scan.keys = reinterpret_cast<uint16_t *>(ws + l.keys);
  a.scan.wide = reinterpret_cast<WideRow *>(ws + l.wide);
  a.scan.n_wide = reinterpret_cast<uint32_t *>(ws + l.n_wide);
  for (int64_t r0 = 0; r0 < R; r0 += per_pass) {
    const int64_t n = R - r0 < per_pass ? R - r0 : per_pass;
    by_rows(a.dtype, form, [&](auto dt, auto row) {
      constexpr int DT = decltype(dt)::value, ROW = decltype(row)::value;
      row_scan_kernel<DT, ROW><<<dim3(unsigned(n * nc)), dim3(kThreads), 0, stream>>>(a, r0, nc);
      select_kernel<DT, ROW, TOP><<<dim3(unsigned(n)), dim3(kSelThreads), 0, stream>>>(a, r0, nc);
      if constexpr (!TOP)  // without filters too: a greedy row of equal logits may be among its rows
        wide_kernel<DT, ROW><<<dim3(unsigned(n < 256 ? n : 256)), dim3(kWideThreads), 0, stream>>>(a, r0, nc);
    });
  }
  return hipGetLastError() == hipSuccess ? DSDE_OK : DSDE_DEVICE_ERROR;
}

}  // namespace

int launch_sample(const SelectArgs &a, int64_t R, hipStream_t stream) { return launch<false>(a, R, stream); }
int launch_top_logits(const SelectArgs &a, int64_t R, hipStream_t stream) { return launch<true>(a, R, stream); }

}  // namespace dsde
