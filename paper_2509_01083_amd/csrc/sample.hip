// Sampling (temperature, top-k, top-p, min-p) and the k largest logits of rows.
//
// Both order a row by (logit descending, id ascending) and need its first
// tokens: the kept set of every filter is a prefix of that order.  A scan kernel
// reads each row once, at one workgroup per chunk of 8,192 logits, and leaves
// per chunk its maximum, the weight of each of its 16 segments of 512 logits, and the
// 16-bit ordered key of the maximum of each group of 8 logits: an eighth of the
// row's length in keys.  A select kernel, one workgroup per row, finds from the keys alone a
// threshold that at least `need` groups reach; the logits that reach it, a few
// more than `need`, are all in those groups, which it reads again, sorts, and cuts.
#include "rows.hpp"
#include "rows_args.hpp"

namespace dsde {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kCand = kSelThreads;  // candidates that the select kernel sorts, one per thread
constexpr int kNeed = 512;          // groups that a row without a smaller top-k asks for
constexpr int kBins = 4096;
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
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x = 0.f, y = 0.f;
#pragma unroll
    for (int e = 0; e < kGroup; e += 2) {
      x += row_weight(g[i].at(e), ref, s.c);
      y += row_weight(g[i].at(e + 1), ref, s.c);
    }
    seg[i] = x + y;
  }
  const float total = lanes::wave_sum4(seg);
  const int wave = t >> 6, lane = t & 63;
  // segment 4 i + wave of the chunk: groups 256 i + 64 wave ...
  if (lane < 4) a.scan.seg[unit * kSegs + 4 * lane + wave] = total;
  if (t == 0) a.scan.max[unit] = bad ? NAN : M;
  if (a.keys_always || s.filtered) {
    uint16_t *keys = a.scan.keys + unit * kChunkGroups + t;
#pragma unroll
    for (int i = 0; i < 4; ++i) keys[256 * i] = uint16_t(order_key(gm[i]) >> 16);
  }
}

// ---------------------------------------------------------------------------
// selection
// ---------------------------------------------------------------------------

// Everything the select kernel keeps in LDS.  The histogram's two arrays, the
// candidates and the segment arrays are never needed at once.
struct SelectLds {
  union {
    struct {
      unsigned long long mass[kBins];
      uint32_t count[kBins];
    } hist;
    struct {
      uint64_t cand[kCand];
      uint32_t groups[kCand];
    } list;
    struct {
      float weight[2 * kBins];
      uint16_t ties[2 * kBins];
    } segs;
  };
  double red64[kSelWaves];
  uint32_t red32[kSelWaves];
  float redf[kSelWaves];
  uint32_t n_groups, n_cand;
  int32_t found;
  uint32_t found_before, found_count;
  uint64_t mass_before, mass_count;
  double mass, target;
  int32_t seg;
  uint32_t seg_ties;
};

// Sorts one value per thread, descending over the first P threads (a power of
// two; the others pass through).  Partners in one wavefront exchange by
// shuffles, others through LDS.
__device__ __forceinline__ uint64_t block_sort(uint64_t v, uint32_t P, uint64_t *lds) {
  const uint32_t t = threadIdx.x;
  for (uint32_t size = 2; size <= P; size *= 2) {
    for (uint32_t stride = size / 2; stride > 0; stride /= 2) {
      uint64_t o;
      if (stride >= 64) {
        lds[t] = v;
        __syncthreads();
        o = lds[t ^ stride];
        __syncthreads();
      } else {
        o = __shfl_xor((unsigned long long)v, int(stride));
      }
      const bool first = (t & stride) == 0, desc = (t & size) == 0;
      v = (first == desc) == (v < o) ? o : v;
    }
  }
  return v;
}
__device__ __forceinline__ uint32_t sort_width(uint32_t n) { return n <= 2 ? 2 : 1u << (32 - __builtin_clz(n - 1)); }

// The bin of a descending histogram at which the running total (count, or mass
// with MASS) reaches the target, given the total before its first bin.  Leaves
// found, found_before / found_count and mass_before / mass_count; found = -1
// when the window does not reach it, with the totals over it in *_before.
template <bool MASS>
__device__ __forceinline__ void find_bin(SelectLds &L, uint64_t target, uint32_t count0, uint64_t mass0) {
  const int t = threadIdx.x;
  uint32_t c[4];
  uint64_t m[4];
  uint32_t cs = 0;
  uint64_t ms = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = L.hist.count[4 * t + i];
    m[i] = L.hist.mass[4 * t + i];
    cs += c[i];
    ms += m[i];
  }
  if (t == 0) L.found = -1;
  const BlockScan<uint32_t> bc = block_scan<kSelWaves>(cs, L.red32);
  const BlockScan<uint64_t> bm = block_scan<kSelWaves>(ms, reinterpret_cast<uint64_t *>(L.red64));
  uint32_t nc = count0 + bc.excl;
  uint64_t nm = mass0 + bm.excl;
  const uint64_t before = MASS ? nm : nc, after = MASS ? mass0 + bm.incl : count0 + bc.incl;
  if (before < target && target <= after) {
    bool done = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t next = MASS ? nm + m[i] : nc + c[i];
      if (!done && next >= target) {
        done = true;
        L.found = 4 * t + i;
        L.found_before = nc;
        L.found_count = c[i];
        L.mass_before = nm;
        L.mass_count = m[i];
      }
      nc += c[i];
      nm += m[i];
    }
  }
  __syncthreads();
  if (L.found < 0 && t == 0) {
    L.found_before = count0 + bc.total;
    L.mass_before = mass0 + bm.total;
  }
  __syncthreads();
}

__device__ __forceinline__ void clear_hist(SelectLds &L) {
  for (int i = threadIdx.x; i < kBins; i += kSelThreads) {
    L.hist.count[i] = 0;
    L.hist.mass[i] = 0;
  }
  __syncthreads();
}

// Tokens that a cut keeps: those with a larger key, and the first `ties` of
// those with this key.
struct Cut {
  uint32_t key, ties;
  uint64_t mass;  // of what it keeps, in units of 2^-40 of the largest weight
};
constexpr float kFixed = 1099511627776.0f;  // 2^40: 2^22 weights of at most 1 stay below 2^63

template <int DT, int ROW>
struct Selector {
  const SelectArgs &a;
  const char *row;
  const uint16_t *keys;
  uint32_t V, ng;
  float m, c;
  SelectLds &L;

  __device__ __forceinline__ float weight(float z) const { return row_weight(z, m, c); }

  // Calls f(key, weight) on every finite logit of the groups that reach the key `lo` (16 bits).
  template <typename F>
  __device__ __forceinline__ void each(uint32_t lo, F f) {
    for (uint32_t w = threadIdx.x; w < ng; w += kSelThreads) {
      if (keys[w] < lo) continue;
      Group<DT, ROW> g;
      g.get(row, V, w);
      g.place(V, w);
#pragma unroll
      for (int i = 0; i < kGroup; ++i) {
        const uint32_t key = order_key(g.at(i));
        if (key > kKeyNegInf) f(key, g.at(i));
      }
    }
  }

  // Tokens that are not masked (this thread's share).
  __device__ uint32_t unmasked() {
    uint32_t n = 0;
    for (uint32_t w = threadIdx.x; w < ng; w += kSelThreads) {
      Group<DT, ROW> g;
      g.get(row, V, w);
      g.place(V, w);
#pragma unroll
      for (int i = 0; i < kGroup; ++i) n += g.at(i) != -__builtin_inff();
    }
    return n;
  }

  // The cut at which the running count (or mass) over the whole row reaches the target.
  // Windows of 4,096 values of the 16-bit key from the row's maximum down: 32
  // octaves of a logit's size, at bf16's resolution, so that bf16 rows are done
  // and few logits share a bin; fp32 rows look into the bin twice more.
  // Integer masses add up to the same bits in any order.
  template <bool MASS>
  __device__ Cut find_cut(uint64_t target) {
    const uint32_t km = order_key(m) >> 16;
    uint32_t count0 = 0, key = 0;
    uint64_t mass0 = 0;
    for (uint32_t off0 = 0;; off0 += kBins) {
      if (off0 > km) return Cut{kKeyNegInf, 0, mass0};  // every finite logit
      clear_hist(L);
      const uint32_t end = off0 + kBins;
      each(km >= end ? km - end + 1 : 0, [&](uint32_t k, float z) {
        const uint32_t b = km - (k >> 16) - off0;
        if (b < kBins) {
          atomicAdd(&L.hist.count[b], 1u);
          atomicAdd(&L.hist.mass[b], (unsigned long long)(weight(z) * kFixed + 0.5f));
        }
      });
      __syncthreads();
      find_bin<MASS>(L, target, count0, mass0);
      count0 = L.found_before;
      mass0 = L.mass_before;
      const int32_t found = L.found;
      __syncthreads();
      if (found >= 0) {
        key = km - off0 - uint32_t(found);
        break;
      }
    }
    if constexpr (DT == DSDE_FP32) {
      // the next 12 bits, then the last 4
      for (int last = 0; last < 2; ++last) {
        const uint32_t prefix = key, below = last ? 4 : 16, shift = last ? 0 : 4, most = last ? 15 : kBins - 1;
        clear_hist(L);
        each(last ? prefix >> 12 : prefix, [&](uint32_t k, float z) {
          if (k >> below == prefix) {
            const uint32_t b = most - ((k >> shift) & most);
            atomicAdd(&L.hist.count[b], 1u);
            atomicAdd(&L.hist.mass[b], (unsigned long long)(weight(z) * kFixed + 0.5f));
          }
        });
        __syncthreads();
        find_bin<MASS>(L, target, count0, mass0);
        count0 = L.found_before;
        mass0 = L.mass_before;
        key = (prefix << (last ? 4 : 12)) | (most - uint32_t(L.found));
        __syncthreads();
      }
    } else {
      key = (key << 16) | ((key & 0x8000u) ? 0u : 0xffffu);
    }
    const uint32_t in_bin = L.found_count;
    const uint64_t unit = L.mass_count / in_bin;
    uint64_t ties = target - (MASS ? mass0 : count0);
    if (MASS) ties = unit ? (ties + unit - 1) / unit : in_bin;
    if (ties > in_bin) ties = in_bin;
    __syncthreads();
    return Cut{key, uint32_t(ties), mass0 + ties * unit};
  }

  // Ties (and, for a draw, weights above the cut) of every segment, into LDS.
  // Returns how many tokens above the cut this thread kept.
  template <bool WEIGHTS>
  __device__ int32_t scan_segments(const Cut &cut, float min_p, int32_t nseg) {
    const int t = threadIdx.x, lane = t & 63;
    int32_t count = 0;
    for (int32_t s = t >> 6; s < nseg; s += kSelWaves) {
      const uint32_t w = uint32_t(s) * 64 + lane;
      uint32_t ties = 0;
      float sum = 0.f;
      if (w < ng) {
        Group<DT, ROW> g;
        g.get(row, V, w);
        g.place(V, w);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
          const uint32_t key = order_key(g.at(i));
          ties += key == cut.key;
          if (WEIGHTS) {
            const float e = weight(g.at(i));
            const bool in = key > cut.key && e >= min_p;
            sum += in ? e : 0.f;
            count += in;
          }
        }
      }
      ties = lanes::wave_sum(ties);
      if (WEIGHTS) sum = lanes::wave_sum(sum);
      if (lane == 0) {
        L.segs.ties[s] = uint16_t(ties);
        if (WEIGHTS) L.segs.weight[s] = sum;
      }
    }
    __syncthreads();
    return count;
  }

  // The inverse-CDF draw over segment weights: the last segment of positive
  // weight whose exclusive prefix is at most u times the total.  weight_of(s, ties
  // before s) gives a segment's weight; ties_of(s) its ties.  Leaves the segment,
  // the ties before it and the weight left in LDS.
  template <typename WF, typename TF>
  __device__ void draw_segment(int32_t nseg, float u, WF weight_of, TF ties_of) {
    const int t = threadIdx.x;
    const int32_t per = (nseg + kSelThreads - 1) / kSelThreads;  // consecutive segments of one thread
    const int32_t s0 = t * per, s1 = min(s0 + per, nseg);
    uint32_t ties = 0;
    for (int32_t s = s0; s < s1; ++s) ties += ties_of(s);
    const uint32_t ties0 = block_scan<kSelWaves>(ties, L.red32).excl;
    double w = 0.0;
    uint32_t before = ties0;
    for (int32_t s = s0; s < s1; ++s) {
      w += weight_of(s, before);
      before += ties_of(s);
    }
    if (t == 0) L.seg = -1;
    const BlockScan<double> bw = block_scan<kSelWaves>(w, L.red64);
    const double target = double(u) * bw.total;
    int32_t best = -1;
    uint32_t best_ties = 0;
    double best_rem = 0.0;
    double at = bw.excl;
    before = ties0;
    for (int32_t s = s0; s < s1; ++s) {
      const double x = weight_of(s, before);
      if (x > 0.0 && at <= target) {
        best = s;
        best_ties = before;
        best_rem = target - at;
      }
      at += x;
      before += ties_of(s);
    }
    if (best >= 0) atomicMax(&L.seg, best);
    __syncthreads();
    if (best >= 0 && L.seg == best) {
      L.seg_ties = best_ties;
      L.target = best_rem;
    }
    __syncthreads();
  }

  // The token of the chosen segment, by wavefront 0: keep(key, weight, tie
  // rank) says whether a logit belongs to the kept set.  Every lane returns (token, logit).
  template <typename K>
  __device__ void draw_token(K keep, uint32_t tie_key, int32_t *token, float *logit) {
    const int lane = threadIdx.x & 63;
    const uint32_t w = uint32_t(L.seg) * 64 + lane;
    Group<DT, ROW> g;
    g.get(row, V, min(w, ng - 1));
    g.place(V, min(w, ng - 1));
    uint32_t ties = 0;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) ties += w < ng && order_key(g.at(i)) == tie_key;
    uint32_t rank = L.seg_ties + lanes::wave_scan(ties).excl;
    float e[kGroup];
    double sum = 0.0;
    int last = -1;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
      const uint32_t key = order_key(g.at(i));
      const float x = weight(g.at(i));
      e[i] = w < ng && key > kKeyNegInf && keep(key, x, rank) ? x : 0.f;
      rank += key == tie_key;
      sum += double(e[i]);
      if (e[i] > 0.f) last = i;
    }
    const lanes::Scan<double> sc = lanes::wave_scan(sum);
    const double rem = L.target;
    const uint64_t can = __ballot(last >= 0 && sc.excl <= rem);
    const int winner = can ? 63 - __builtin_clzll(can) : 0;
    int pick = last >= 0 ? last : 0;
    double acc = sc.excl;
    bool done = false;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
      acc += double(e[i]);
      if (!done && acc > rem) {
        pick = i;
        done = true;
      }
    }
    float z = g.at(0);
#pragma unroll
    for (int i = 1; i < kGroup; ++i)
      if (pick == i) z = g.at(i);
    *token = lanes::readlane(int32_t(w * kGroup) + pick, winner);
    *logit = lanes::readlane(z, winner);
  }

  // The groups that reach a key, and from them the logits that do, sorted in
  // the row's order.  -1 when there are more than one per thread.
  __device__ int32_t gather(uint32_t kappa, uint64_t *sorted) {
    const int t = threadIdx.x;
    if (t == 0) L.n_groups = L.n_cand = 0;
    __syncthreads();
    for (uint32_t w = t; w < ng; w += kSelThreads)
      if (keys[w] >= kappa) {
        const uint32_t i = atomicAdd(&L.n_groups, 1u);
        if (i < kCand) L.list.groups[i] = w;
      }
    __syncthreads();
    if (L.n_groups > kCand) return -1;
    if (uint32_t(t) < L.n_groups) {
      const uint32_t w = L.list.groups[t];
      Group<DT, ROW> g;
      g.get(row, V, w);
      g.place(V, w);
#pragma unroll
      for (int e = 0; e < kGroup; ++e) {
        const uint32_t key = order_key(g.at(e));
        if (key >> 16 >= kappa) {
          const uint32_t i = atomicAdd(&L.n_cand, 1u);
          if (i < kCand) L.list.cand[i] = (uint64_t(key) << 32) | uint32_t(~(w * kGroup + e));
        }
      }
    }
    __syncthreads();
    const uint32_t n = L.n_cand;
    if (n > kCand) return -1;
    uint64_t v = uint32_t(t) < n ? L.list.cand[t] : 0;
    __syncthreads();
    *sorted = block_sort(v, sort_width(n), L.list.cand);
    return int32_t(n);
  }

  // The largest 16-bit key that at least `need` groups reach (kAll when fewer
  // than that lie in the histogram's window).
  static constexpr uint32_t kAll = (kKeyNegInf >> 16) + 1;  // every finite logit
  __device__ uint32_t threshold(uint32_t need) {
    const uint32_t km = order_key(m) >> 16;
    clear_hist(L);
    for (uint32_t w = threadIdx.x; w < ng; w += kSelThreads) {
      const uint32_t b = km - keys[w];
      if (b < kBins) atomicAdd(&L.hist.count[b], 1u);
    }
    __syncthreads();
    find_bin<false>(L, need, 0, 0);
    const int32_t f = L.found;
    __syncthreads();
    if (f < 0) return kAll;
    const uint32_t k = km - uint32_t(f);
    return k < kAll ? kAll : k;
  }
};

// One row per workgroup.
template <int DT, int ROW, bool TOP>
__global__ __launch_bounds__(kSelThreads) void select_kernel(const SelectArgs a, int64_t row0, int32_t nc) {
  __shared__ SelectLds L;
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x, out = row0 + r;
  const Setting s = row_setting(a, out);
  const float *cmax = a.scan.max + r * nc;
  const float *seg = a.scan.seg + r * nc * kSegs;
  const int32_t nseg = nc * kSegs;

  float mt = -INFINITY;
  bool bad = false;
  for (int32_t i = t; i < nc; i += kSelThreads) {
    const float x = cmax[i];
    bad |= !(x < INFINITY);
    mt = fmaxf(mt, x);
  }
  bad = __syncthreads_or(bad);
  const float m = block_reduce<kSelWaves>(mt, L.redf, lanes::Max{});
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
  double part = 0.0;
  for (int32_t i = t; i < nseg; i += kSelThreads) part += double(seg[i]) * double(row_weight(cmax[i / kSegs], m, s.c));
  const double S = block_reduce<kSelWaves>(part, L.red64, lanes::Add{});

  const uint32_t V = uint32_t(a.V);
  Selector<DT, ROW> sel{a, a.rows.row(out), a.scan.keys + r * nc * kChunkGroups, V, (V + kGroup - 1) / kGroup, m, s.c, L};

  auto emit = [&](int32_t token, float z, int32_t kept) {
    a.tokens[out] = token;
    if (a.logprob) a.logprob[out] = float((double(z) - double(m)) / double(s.T) - log(S));
    if (a.kept) a.kept[out] = kept;
  };

  if constexpr (TOP) {
    if (t == 0) a.lse[out] = float(double(m) / double(s.T) + log(S));
    const int32_t k = a.one_k;
    const uint32_t kappa = sel.threshold(uint32_t(k));
    uint64_t v = 0;
    int32_t n = sel.gather(kappa, &v);
    if (n < 0) {
      const Cut cut = sel.template find_cut<false>(uint64_t(k));
      sel.template scan_segments<false>(cut, 0.f, nseg);
      // ties before every segment, clamped (at most k <= 256 of them are taken)
      const int32_t per = (nseg + kSelThreads - 1) / kSelThreads, s0 = t * per, s1 = min(s0 + per, nseg);
      uint32_t ties = 0;
      for (int32_t i = s0; i < s1; ++i) ties += L.segs.ties[i];
      uint32_t before = block_scan<kSelWaves>(ties, L.red32).excl;
      for (int32_t i = s0; i < s1; ++i) {
        const uint32_t x = L.segs.ties[i];
        L.segs.ties[i] = uint16_t(min(before, 65535u));
        before += x;
      }
      if (t == 0) L.n_cand = 0;
      __syncthreads();
      uint64_t *picked = reinterpret_cast<uint64_t *>(L.segs.weight);  // not used here: 8 KB of its 32
      for (int32_t i = t >> 6; i < nseg; i += kSelWaves) {
        const uint32_t w = uint32_t(i) * 64 + (t & 63);
        uint32_t key[kGroup], own = 0;
        Group<DT, ROW> g;
        g.get(sel.row, V, min(w, sel.ng - 1));
        g.place(V, min(w, sel.ng - 1));
#pragma unroll
        for (int e = 0; e < kGroup; ++e) {
          key[e] = w < sel.ng ? order_key(g.at(e)) : 0u;
          own += key[e] == cut.key;
        }
        uint32_t rank = L.segs.ties[i] + lanes::wave_scan(own).excl;
#pragma unroll
        for (int e = 0; e < kGroup; ++e) {
          const bool tie = key[e] == cut.key;
          if (key[e] > kKeyNegInf && (key[e] > cut.key || (tie && rank < cut.ties))) {
            const uint32_t j = atomicAdd(&L.n_cand, 1u);
            if (j < kCand) picked[j] = (uint64_t(key[e]) << 32) | uint32_t(~(w * kGroup + e));
          }
          rank += tie;
        }
      }
      __syncthreads();
      n = int32_t(min(L.n_cand, uint32_t(kCand)));
      v = t < n ? picked[t] : 0;
      __syncthreads();
      v = block_sort(v, sort_width(uint32_t(n)), picked);
    }
    if (t < k) {
      a.values[out * k + t] = t < n ? key_logit(uint32_t(v >> 32)) : -INFINITY;
      a.ids[out * k + t] = t < n ? int32_t(~uint32_t(v)) : -1;
    }
    return;
  } else {
    if (!s.filtered) {
      const uint32_t n = a.kept ? block_reduce<kSelWaves>(sel.unmasked(), L.red32, lanes::Add{}) : 0u;
      sel.draw_segment(
          nseg, s.u,
          [&](int32_t i, uint32_t) { return double(seg[i]) * double(row_weight(cmax[i / kSegs], m, s.c)); },
          [](int32_t) { return 0u; });
      if (t < 64) {
        int32_t token;
        float z;
        sel.draw_token([](uint32_t, float, uint32_t) { return true; }, 0u, &token, &z);
        if (t == 0) emit(token, z, int32_t(n));
      }
      return;
    }

    // candidates: a prefix of the row's order
    const uint32_t need = s.k > 0 && s.k < kNeed ? uint32_t(s.k) : uint32_t(kNeed);
    uint32_t kappa = sel.threshold(need);
    bool min_decided = false;
    if (s.m > 0.f) {
      // a little below the smallest logit that min_p keeps
      const float d = log2f(s.m) / s.c, z = m + d - 1e-5f * (1.f + fabsf(m) + fabsf(d));
      const uint32_t low = order_key(z) >> 16;
      if (low >= kappa) {
        kappa = low;
        min_decided = true;
      }
    }
    const bool all = kappa == sel.kAll;
    uint64_t v = 0;
    const int32_t n = sel.gather(kappa, &v);
    int32_t kept = kUndecided;
    if (n >= 0) {
      const float e = t < n ? sel.weight(key_logit(uint32_t(v >> 32))) : 0.f;
      const BlockScan<double> cs = block_scan<kSelWaves>(double(e), L.red64);
      const bool k_in = s.k > 0 && s.k <= n;
      if (k_in && t == s.k - 1) L.mass = cs.incl;
      const int32_t n_min = __syncthreads_count(t < n && e >= s.m);
      const double mass = k_in ? L.mass : all ? cs.total : S;
      const int32_t n_below = __syncthreads_count(t < n && cs.incl < double(s.p) * mass);
      int32_t lim = kUndecided;
      if (k_in) lim = s.k;
      if (all) lim = min(lim, n);
      if (s.m > 0.f && (n_min < n || all || min_decided)) lim = min(lim, n_min);
      bool known = true;
      if (s.p < 1.f) {
        known = k_in || all || s.k == 0;
        if (n_below < n) lim = min(lim, n_below + 1);
      }
      if (known && lim != kUndecided) kept = max(lim, 1);
    }
    if (kept != kUndecided) {
      // the draw walks the kept tokens in the order of their ids
      const uint32_t id = ~uint32_t(v);
      const float e = t < kept ? sel.weight(key_logit(uint32_t(v >> 32))) : 0.f;
      uint64_t x = t < kept ? (uint64_t(~id) << 32) | __float_as_uint(e) : 0;
      if (kept > 1) x = block_sort(x, sort_width(uint32_t(kept)), L.list.cand);
      const float ex = __uint_as_float(uint32_t(x));
      const BlockScan<double> cs = block_scan<kSelWaves>(double(ex), L.red64);
      const int32_t at = min(__syncthreads_count(t < kept && cs.incl <= double(s.u) * cs.total), kept - 1);
      if (t == at) {
        const int32_t token = int32_t(~uint32_t(x >> 32));
        emit(token, load_logit(sel.row, DT, token), kept);
      }
      return;
    }

    // more tokens than candidates: cuts over the whole row
    __syncthreads();
    Cut cut{kKeyNegInf, 0, uint64_t(S * double(kFixed))};
    if (s.k > 0) cut = sel.template find_cut<false>(uint64_t(s.k));
    if (s.p < 1.f) {
      const uint64_t target = uint64_t(double(s.p) * double(cut.mass));
      cut = sel.template find_cut<true>(target ? target : 1);
    }
    const int32_t above = sel.template scan_segments<true>(cut, s.m, nseg);
    const uint32_t count = block_reduce<kSelWaves>(uint32_t(above), L.red32, lanes::Add{});
    const float tie_weight = sel.weight(key_logit(cut.key));
    const uint32_t tie_limit = tie_weight >= s.m ? cut.ties : 0u;
    auto ties_of = [&](int32_t i) { return uint32_t(L.segs.ties[i]); };
    auto weight_of = [&](int32_t i, uint32_t before) {
      const uint32_t left = before < tie_limit ? tie_limit - before : 0u, here = ties_of(i);
      return double(L.segs.weight[i]) + double(tie_weight) * double(here < left ? here : left);
    };
    sel.draw_segment(nseg, s.u, weight_of, ties_of);
    if (t < 64) {
      int32_t token;
      float z;
      const float min_p = s.m;
      sel.draw_token(
          [&](uint32_t key, float e, uint32_t rank) {
            return e >= min_p && (key > cut.key || (key == cut.key && rank < tie_limit));
          },
          cut.key, &token, &z);
      if (t == 0) emit(token, z, int32_t(count + tie_limit));
    }
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
  a.scan.seg = reinterpret_cast<float *>(ws + l.seg);
  a.scan.keys = reinterpret_cast<uint16_t *>(ws + l.keys);
  for (int64_t r0 = 0; r0 < R; r0 += per_pass) {
    const int64_t n = R - r0 < per_pass ? R - r0 : per_pass;
    by_rows(a.dtype, form, [&](auto dt, auto row) {
      constexpr int DT = decltype(dt)::value, ROW = decltype(row)::value;
      row_scan_kernel<DT, ROW><<<dim3(unsigned(n * nc)), dim3(kThreads), 0, stream>>>(a, r0, nc);
      select_kernel<DT, ROW, TOP><<<dim3(unsigned(n)), dim3(kSelThreads), 0, stream>>>(a, r0, nc);
    });
  }
  return hipGetLastError() == hipSuccess ? DSDE_OK : DSDE_DEVICE_ERROR;
}

}  // namespace

int launch_sample(const SelectArgs &a, int64_t R, hipStream_t stream) { return launch<false>(a, R, stream); }
int launch_top_logits(const SelectArgs &a, int64_t R, hipStream_t stream) { return launch<true>(a, R, stream); }

}  // namespace dsde
