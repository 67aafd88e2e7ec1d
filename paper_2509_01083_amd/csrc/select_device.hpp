// Device code of the selection inside one row, by one workgroup: thresholds and
// lists from the keys of the row's groups, sorts, the cuts of a count or of a
// share of the weight, and the draw over segments.  Internal to sample.hip.
#pragma once

#include "rows.hpp"
#include "rows_args.hpp"

namespace dsde {
namespace {

constexpr int kSelThreads = 512;    // threads per row of the select kernel,
constexpr int kWideThreads = 1024;  // and of the cuts over many tokens
constexpr int kBins = 2048;
constexpr int kPerOctave = 64;  // bins per octave of a weight: 32 octaves below the largest
constexpr int kMostSegs = 2048;

// The group whose key lies at this place of a row's keys.
__device__ __forceinline__ uint32_t place_group(uint32_t q) {
  return (q & ~uint32_t(kChunkGroups - 1)) + 256 * (q & 3) + ((q & (kChunkGroups - 1)) >> 2);
}
constexpr uint32_t kAll = (kKeyNegInf >> 16) + 1;  // the smallest key (high half) of a finite logit

// What a workgroup of T threads keeps in LDS.  The histogram, the segments, the list of GROUPS
// groups and the arrays of the search for few tokens are never needed at once.
template <int T, int BINS, int GROUPS, int ELEMS>
struct SelectLdsOf {
  static constexpr int kThreads = T, kWaves = T / 64;
  static constexpr uint32_t kGroups = GROUPS, kElems = ELEMS;
  union {
    struct {
      unsigned long long mass[BINS];
      uint32_t count[BINS];
    } hist;
    unsigned long long segs[BINS];
    uint32_t list[GROUPS];
    uint32_t tmax[T];
  };
  uint64_t cand[T];  // what the workgroup sorts, one per thread
  uint64_t elems[ELEMS];
  uint64_t red64[2 * kWaves];
  uint32_t red32[kWaves];
  float redf[kWaves];
  uint32_t n_groups, n_cand, n_elems;
  int32_t found;
  uint32_t found_before, found_count;
  uint64_t mass_before, mass_count;
  double mass, rem;
  int32_t seg;
  uint32_t seg_ties;
  uint64_t cut;
};
// The draw's select kernel has no histogram; the top logits', whose rows hardly ever need one, keeps the
// whole of it and short lists (45 KB: three workgroups per CU).  The cuts over many tokens take one CU.
using DrawLds = SelectLdsOf<kSelThreads, 1, kSelThreads, kSelThreads>;
using TopLds = SelectLdsOf<kSelThreads, kBins, 2048, 2048>;
using WideLds = SelectLdsOf<kWideThreads, kBins, 8192, 12288>;
static_assert(kBins == kMostSegs, "one array holds either");
static_assert(sizeof(WideLds) <= 160 * 1024, "LDS of a CU");

// The value of lane ^ STRIDE.
template <int STRIDE>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v) {
  if constexpr (STRIDE == 1) return lanes::dpp<lanes::kQuadSwap1>(v);
  if constexpr (STRIDE == 2) return lanes::dpp<lanes::kQuadSwap2>(v);
  if constexpr (STRIDE == 4) return lanes::dpp<0x1B>(lanes::dpp<lanes::kRowHalfMirror>(v));  // i ^ 7, then i ^ 3
  if constexpr (STRIDE == 8) return lanes::dpp<lanes::kRowRor8>(v);
  return __shfl_xor((unsigned long long)v, STRIDE);
}
template <int SIZE, int STRIDE>
__device__ __forceinline__ void sort_steps(uint64_t &v, bool used, uint64_t *lds) {
  const uint32_t t = threadIdx.x;
  const bool larger = ((t & STRIDE) == 0) == ((t & SIZE) == 0);  // this thread keeps the larger of the two
  if constexpr (STRIDE >= 64) {
    lds[t] = v;
    __syncthreads();
    const uint64_t o = lds[t ^ STRIDE];
    __syncthreads();
    v = larger == (v < o) ? o : v;
    sort_steps<SIZE, STRIDE / 2>(v, used, lds);
  } else if (used) {
    const uint64_t o = lane_xor<STRIDE>(v);
    v = larger == (v < o) ? o : v;
    if constexpr (STRIDE > 1) sort_steps<SIZE, STRIDE / 2>(v, used, lds);
  }
}
// Sorts one value per thread, descending over the first P threads (P the
// smallest power of two >= n, at least 64; the other wavefronts only keep the
// barriers): a bitonic network whose partners inside one wavefront exchange by DPP moves
// and shuffles, others through LDS.
template <int T, int SIZE = 2>
__device__ __forceinline__ void block_sort(uint64_t &v, uint32_t n, uint64_t *lds) {
  const bool used = n > 1 && (threadIdx.x & ~63u) < (1u << (32 - __builtin_clz(n - 1)));
  sort_steps<SIZE, SIZE / 2>(v, used, lds);
  if constexpr (SIZE < T) {
    if (n > SIZE) block_sort<T, SIZE * 2>(v, n, lds);
  }
}

// The bin of a descending histogram at which the running total (count, or mass
// with MASS) reaches the target, given the totals before its first bin.  Leaves
// found, found_before / found_count and mass_before / mass_count; found = -1
// when the window does not reach it, with the totals behind it in *_before.
template <bool MASS, typename LDS>
__device__ __forceinline__ void find_bin(LDS &L, uint64_t target, uint32_t count0, uint64_t mass0) {
  constexpr int kPer = kBins / LDS::kThreads;
  const int t = threadIdx.x;
  uint32_t c[kPer], cs = 0;
  uint64_t m[kPer], ms = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    c[i] = L.hist.count[kPer * t + i];
    m[i] = L.hist.mass[kPer * t + i];
    cs += c[i];
    ms += m[i];
  }
  if (t == 0) L.found = -1;
  const BlockScan<uint32_t> bc = block_scan<LDS::kWaves>(cs, L.red32);
  const BlockScan<uint64_t> bm = block_scan<LDS::kWaves>(ms, L.red64);
  uint32_t nc = count0 + bc.excl;
  uint64_t nm = mass0 + bm.excl;
  const uint64_t before = MASS ? nm : nc, after = MASS ? mass0 + bm.incl : count0 + bc.incl;
  if (before < target && target <= after) {
    bool done = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint64_t next = MASS ? nm + m[i] : nc + c[i];
      if (!done && next >= target) {
        done = true;
        L.found = kPer * t + i;
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

template <typename LDS>
__device__ __forceinline__ void clear_hist(LDS &L) {
  for (int i = threadIdx.x; i < kBins; i += LDS::kThreads) {
    L.hist.count[i] = 0;
    L.hist.mass[i] = 0;
  }
  __syncthreads();
}

// A token's place in its row's order: larger packed values come first.
__device__ __forceinline__ uint64_t packed(uint32_t key, uint32_t id) { return (uint64_t(key) << 32) | uint32_t(~id); }
constexpr uint64_t kEvery = uint64_t(kKeyNegInf + 1) << 32;  // below every token that is not masked

// The last kept token of a row, and the weight of all kept ones.
struct Cut {
  uint64_t at;
  uint64_t mass;  // in units of 2^-40 of the largest weight
};
constexpr float kFixed = 1099511627776.0f;  // 2^40: 2^22 weights of at most 1 stay below 2^63
__device__ __forceinline__ unsigned long long fixed_weight(float w) { return (unsigned long long)(w * kFixed + 0.5f); }

// Keys of a row that a thread holds: 8 consecutive places in each load of a
// tile (20,480 groups with 512 threads, one tile up to V = 163,840), the first tile from the start on.
template <int T>
struct KeyTile {
  static constexpr int kKeyLoads = T == kSelThreads ? 5 : 3;
  static constexpr uint32_t kTile = kKeyLoads * 8 * T;
  uint4 q[kKeyLoads];
  // `places` keys of the row (a multiple of 1,024); missing ones are 0
  __device__ __forceinline__ void load(const uint16_t *keys, uint32_t places, uint32_t base) {
#pragma unroll
    for (int j = 0; j < kKeyLoads; ++j) {
      const uint32_t at = base + 8 * (uint32_t(j) * T + threadIdx.x);
      q[j] = *reinterpret_cast<const uint4 *>(keys + min(at, places - 8));
      if (at >= places) q[j] = make_uint4(0, 0, 0, 0);
    }
  }
  __device__ __forceinline__ uint32_t largest() const {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = {0, 0};
#pragma unroll
    for (int j = 0; j < kKeyLoads; ++j)
#pragma unroll
      for (uint32_t w : {q[j].x, q[j].y, q[j].z, q[j].w})
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w));
    return m.x > m.y ? m.x : m.y;
  }
  // The keys that reach kappa (> 0), a bit each: bits w and 16 + w of mask i stand for the two
  // keys of word 16 i + w.
  static constexpr int kMasks = (4 * kKeyLoads + 15) / 16;
  __device__ __forceinline__ void reaching(uint32_t kappa, uint32_t (&mask)[kMasks]) const {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const u16x2 below = {uint16_t(kappa - 1), uint16_t(kappa - 1)}, one = {1, 1};
#pragma unroll
    for (int i = 0; i < kMasks; ++i) mask[i] = 0;
#pragma unroll
    for (int j = 0; j < kKeyLoads; ++j) {
      const uint32_t w[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u16x2 d = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, w[i]), below);
        const u16x2 b = __builtin_elementwise_min(d, one);
        mask[(4 * j + i) / 16] |= __builtin_bit_cast(uint32_t, b) << ((4 * j + i) % 16);
      }
    }
  }
  __device__ __forceinline__ static uint32_t mask_place(uint32_t base, int i, int bit) {
    const uint32_t word = uint32_t(16 * i + (bit & 15));
    return base + 8 * ((word >> 2) * T + threadIdx.x) + 2 * (word & 3) + uint32_t(bit >> 4);
  }
  // f(key, place) on every key
  template <typename F>
  __device__ __forceinline__ void each(uint32_t base, F f) const {
#pragma unroll
    for (int j = 0; j < kKeyLoads; ++j) {
      // opaque to the compiler, which would otherwise keep all unpacked keys and
      // places of one use for the next (and spill)
      uint32_t at = base + 8 * (uint32_t(j) * T + threadIdx.x);
      uint32_t w[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
      asm volatile("" : "+v"(at), "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
#pragma unroll
      for (int i = 0; i < 8; ++i) f((w[i / 2] >> (16 * (i & 1))) & 0xffffu, at + i);
    }
  }
};

static_assert(DSDE_MAX_VOCAB / kChunk <= kSelThreads, "one chunk per thread at most");
static_assert(DSDE_MAX_VOCAB <= kMostSegs << 11, "segments of the cuts fit the LDS array");

template <int DT, int ROW, typename LDS>
struct Selector {
  static constexpr int T = LDS::kThreads, W = LDS::kWaves;
  using Tile = KeyTile<T>;
  const char *row;
  const uint16_t *keys;
  uint32_t V, ng, places;
  float m, c;
  LDS &L;
  Tile tile;          // the first tile's keys
  bool listed = false;     // the logits to look at are in L.elems
  bool min_bound = false;  // they are those that min_p may keep

  __device__ __forceinline__ float weight(float z) const { return row_weight(z, m, c); }

  // f(tile, base) on every tile of keys
  template <typename F>
  __device__ __forceinline__ void tiles(F f) {
    f(tile, 0u);
    for (uint32_t base = Tile::kTile; base < places; base += Tile::kTile) {
      Tile x;
      x.load(keys, places, base);
      f(x, base);
    }
  }

  // Lists the groups whose key reaches kappa (as far as there is room) and returns how many there are, in every thread.
  __device__ __forceinline__ uint32_t groups_reaching(uint32_t kappa) {
    if (threadIdx.x == 0) L.n_groups = 0;
    __syncthreads();
    tiles([&](const Tile &x, uint32_t base) {
      uint32_t mask[Tile::kMasks], n = 0;
      x.reaching(kappa, mask);
#pragma unroll
      for (int i = 0; i < Tile::kMasks; ++i) n += __popc(mask[i]);
      if (__ballot(n != 0) == 0) return;
      const lanes::Scan<uint32_t> sc = lanes::wave_scan(n);
      uint32_t at = 0;
      if ((threadIdx.x & 63) == 63) at = atomicAdd(&L.n_groups, sc.incl);
      at = lanes::readlane(at, 63) + sc.excl;
#pragma unroll
      for (int i = 0; i < Tile::kMasks; ++i)
        for (; mask[i]; mask[i] &= mask[i] - 1, ++at)
          if (at < LDS::kGroups) L.list[at] = place_group(Tile::mask_place(base, i, __ffs(mask[i]) - 1));
    });
    __syncthreads();
    return L.n_groups;
  }

  // A key that at least `need` groups reach: the need-th largest of the
  // threads' largest keys.  (Of 512 threads, 64 with a key that reaches it hold about 69 such
  // keys, and 256 about 355.)  kAll when fewer threads than that hold a finite one.
  __device__ __forceinline__ uint32_t threshold(uint32_t need) {
    uint32_t top = 0;
    tiles([&](const Tile &x, uint32_t) { top = max(top, x.largest()); });
    L.tmax[threadIdx.x] = top;
    __syncthreads();
    uint32_t v[W];
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = L.tmax[64 * j + (threadIdx.x & 63)];
    uint32_t kappa = 0;
    for (uint32_t bit = 0x8000u; bit; bit >>= 1) {
      uint32_t n = 0;
#pragma unroll
      for (int j = 0; j < W; ++j) n += __popcll(__ballot(v[j] >= (kappa | bit)));
      if (n >= need) kappa |= bit;
    }
    return max(kappa, kAll);
  }

  // The largest key that at least `need` groups reach, or kAll.
  __device__ __forceinline__ uint32_t exact_threshold(uint32_t need) {
    uint32_t kappa = 0;
    for (uint32_t bit = 0x8000u; bit; bit >>= 1) {
      uint32_t n = 0;
      tiles([&](const Tile &x, uint32_t base) { x.each(base, [&](uint32_t k, uint32_t) { n += k >= (kappa | bit); }); });
      if (block_reduce<W>(n, L.red32, lanes::Add{}) >= need) kappa |= bit;
    }
    return max(kappa, kAll);
  }

  // The logits that reach kappa, one per thread, in the row's order.  -1 when
  // there are more groups or logits than threads.
  __device__ __forceinline__ int32_t gather(uint32_t kappa, uint64_t *sorted) {
    const int t = threadIdx.x;
    const uint32_t n_groups = groups_reaching(kappa);
    if (n_groups > T) return -1;
    uint32_t key[kGroup], n = 0, w = 0;
    if (uint32_t(t) < n_groups) {
      w = L.list[t];
      Group<DT, ROW> g;
      g.get(row, V, w);
      g.place(V, w);
#pragma unroll
      for (int e = 0; e < kGroup; ++e) {
        key[e] = order_key(g.at(e));
        n += key[e] >> 16 >= kappa;
      }
    }
    const BlockScan<uint32_t> sc = block_scan<W>(n, L.red32);
    if (sc.total > T) return -1;
    if (n) {
      uint32_t at = sc.excl;
#pragma unroll
      for (int e = 0; e < kGroup; ++e)
        if (key[e] >> 16 >= kappa) L.cand[at++] = (uint64_t(key[e]) << 32) | uint32_t(~(w * kGroup + e));
    }
    __syncthreads();
    uint64_t v = uint32_t(t) < sc.total ? L.cand[t] : 0;
    __syncthreads();
    block_sort<T>(v, sc.total, L.cand);
    *sorted = v;
    return int32_t(sc.total);
  }

  // Calls f(group, its number, whether it counts) on the groups that list(i) names,
  // or on all, in order: then the lanes of a wavefront hold the 64 groups of one segment.
  template <typename F, typename I>
  __device__ __forceinline__ void each_group(uint32_t n, I list, F f) {
    constexpr int kBatch = 4;
    for (uint32_t i = threadIdx.x & ~63u; i < n; i += kBatch * T) {
      Group<DT, ROW> g[kBatch];
      uint32_t w[kBatch];
      const uint32_t j0 = i + (threadIdx.x & 63);
#pragma unroll
      for (int b = 0; b < kBatch; ++b) w[b] = list(min(j0 + uint32_t(b) * T, n - 1));
#pragma unroll
      for (int b = 0; b < kBatch; ++b) g[b].get(row, V, w[b]);
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        if (i + uint32_t(b) * T >= n) break;
        g[b].place(V, w[b]);
        f(g[b], w[b], j0 + uint32_t(b) * T < n);
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void all_groups(F f) {
    each_group(ng, [](uint32_t i) { return i; }, f);
  }
  // Calls f(key, logit, id) on the listed logits, or on all that are not masked.
  template <typename F>
  __device__ __forceinline__ void each(F f) {
    if (listed) {
      for (uint32_t i = threadIdx.x; i < L.n_elems; i += T) {
        const uint64_t x = L.elems[i];
        f(uint32_t(x >> 32), key_logit(uint32_t(x >> 32)), ~uint32_t(x));
      }
    } else {
      all_groups([&](const Group<DT, ROW> &g, uint32_t w, bool in) {
#pragma unroll
        for (int e = 0; e < kGroup; ++e) {
          const uint32_t key = order_key(g.at(e));
          if (in && key > kKeyNegInf) f(key, g.at(e), w * kGroup + e);
        }
      });
    }
  }

  // Lists the logits that reach `low` (a key's upper half); where they, or their
  // groups, are too many, all logits are looked at.
  __device__ __forceinline__ void list_logits(uint32_t low) {
    const uint32_t n = groups_reaching(low);
    listed = n <= LDS::kGroups;
    if (!listed) return;
    if (threadIdx.x == 0) L.n_elems = 0;
    __syncthreads();
    const uint32_t least = low << 16;
    each_group(n, [&](uint32_t i) { return L.list[i]; }, [&](const Group<DT, ROW> &g, uint32_t w, bool in) {
      uint32_t key[kGroup], own = 0;
#pragma unroll
      for (int e = 0; e < kGroup; ++e) {
        key[e] = order_key(g.at(e));
        own += in && key[e] >= least;
      }
      const lanes::Scan<uint32_t> sc = lanes::wave_scan(own);
      uint32_t at = 0;
      if ((threadIdx.x & 63) == 63) at = atomicAdd(&L.n_elems, sc.incl);
      at = lanes::readlane(at, 63) + sc.excl;
#pragma unroll
      for (int e = 0; e < kGroup; ++e)
        if (in && key[e] >= least) {
          if (at < LDS::kElems) L.elems[at] = packed(key[e], w * kGroup + e);
          ++at;
        }
    });
    __syncthreads();
    listed = L.n_elems <= LDS::kElems;
  }

  // The smallest logit with this upper half of a key (bf16 has no other).
  __device__ __forceinline__ static float key_floor(uint32_t key) {
    return key_logit((key << 16) | (DT == DSDE_BF16 && !(key & 0x8000u) ? 0xffffu : 0u));
  }
  // The bin of a logit on a scale of its weight: equal logits share one, and larger
  // ones never come behind smaller ones.
  __device__ __forceinline__ uint32_t weight_bin(float z) const {
    return uint32_t(fminf((m - z) * c * float(kPerOctave), float(kBins)));
  }

  // Lists the logits from which the cuts are found, from the groups' largest
  // keys.  Any key will do whose logits turn out to hold the cut (weight_cut
  // looks): k groups whose largest lies in the first b bins do for a count of
  // k; for a weight, the first bins whose groups' largest alone weigh enough, or as many bins as
  // the list has room for.
  __device__ __forceinline__ void list_relevant(int32_t k, float p, float S, uint32_t min_key) {
    constexpr int kPer = kBins / T;
    const int t = threadIdx.x;
    clear_hist(L);
    tiles([&](const Tile &x, uint32_t base) {
      x.each(base, [&](uint32_t key, uint32_t) {
        if (key < kAll) return;
        const uint32_t b = weight_bin(key_floor(key));
        if (b < uint32_t(kBins)) atomicAdd(&L.hist.count[b], 1u);
      });
    });
    if (t == 0) L.found = kBins;
    __syncthreads();
    uint32_t n[kPer], own = 0;
    float mass = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      n[i] = L.hist.count[kPer * t + i];
      own += n[i];
      mass += float(n[i]) * fast_exp2(-float(kPer * t + i + 1) / kPerOctave);
    }
    const BlockScan<uint32_t> sn = block_scan<W>(own, L.red32);
    const BlockScan<float> sm = block_scan<W>(mass, L.redf);
    // about as many logits as there is room for reach the key that these groups reach, when the
    // larger ones fall into the groups at random
    const uint32_t room = min(LDS::kGroups, uint32_t(float(ng) * (1.f - __expf(-0.85f * LDS::kElems / float(ng)))));
    uint32_t inside = sn.excl;
    float weighs = sm.excl;
    int32_t best = kBins;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {  // the first kPer t + i + 1 bins
      inside += n[i];
      weighs += float(n[i]) * fast_exp2(-float(kPer * t + i + 1) / kPerOctave);
      const uint32_t next = T * kPer > kPer * t + i + 1 ? L.hist.count[kPer * t + i + 1] : 0u;
      const bool ok = k > 0 ? inside >= uint32_t(k) : weighs >= 1.00001f * p * S || inside + next > room;
      if (ok && best == kBins) best = kPer * t + i + 1;
    }
    if (best < kBins) atomicMin(&L.found, best);
    __syncthreads();
    const int32_t b = L.found;
    uint32_t low = kAll;
    if (b < kBins) {
      const float d = float(b + 1) / (kPerOctave * c);  // a bin more than needed, for its rounding
      low = max(low, order_key(m - d - 1e-5f * (fabsf(m) + d)) >> 16);
    }
    // (with both, top_p's share is of all top_k's weight; with neither, min_p alone decides)
    min_bound = k > 0 ? min_key > low && p >= 1.f : min_key > low || p >= 1.f;
    if (min_bound) low = max(min_key, kAll);
    __syncthreads();
    list_logits(low);
  }

  // Counts and weights of the listed logits by bin.  Integer weights add up to
  // the same bits in any order.
  __device__ __forceinline__ void histogram() {
    clear_hist(L);
    auto add = [&](float z) {
      const float d = (m - z) * c;
      if (d < float(kBins / kPerOctave)) {
        const uint32_t b = uint32_t(d * float(kPerOctave));
        atomicAdd(&L.hist.count[b], 1u);
        atomicAdd(&L.hist.mass[b], fixed_weight(fast_exp2(-d)));
      }
    };
    if (listed)
      each([&](uint32_t, float z, uint32_t) { add(z); });
    else
      all_groups([&](const Group<DT, ROW> &g, uint32_t, bool in) {
#pragma unroll
        for (int e = 0; e < kGroup; ++e)
          if (in) add(g.at(e));
      });
    __syncthreads();
  }

  // The cut at which the running count (or weight) reaches the target, from
  // the histogram and the logits of one bin, sorted.  With `last`, the segments'
  // weights of what it and min_p keep are left in LDS.
  template <bool MASS>
  __device__ __forceinline__ Cut weight_cut(uint64_t target, bool last, float min_p, int32_t *kept) {
    const int t = threadIdx.x;
    find_bin<MASS>(L, target, 0, 0);
    if (L.found < 0 && listed && !min_bound) {  // the lists were too short
      listed = false;
      __syncthreads();
      histogram();
      find_bin<MASS>(L, target, 0, 0);
    }
    const int32_t bin = L.found;
    const uint32_t in_bin = L.found_count;
    const uint64_t count0 = L.found_before, mass0 = L.mass_before;
    __syncthreads();
    Cut cut;
    // min_p's tokens, which are listed, end before the cut; that the histogram does not reach it says so
    // only where it holds all of them (weights over 2^-32), and key_cut looks further where it does not
    if (bin < 0 && min_bound && min_p >= 0x1p-31f) {
      if (last) add_segments(kEvery, min_p, kept);
      return Cut{kEvery, 0};
    }
    if (bin < 0 || in_bin > uint32_t(T)) {
      // outside the histogram's range, or a long run of nearly equal logits
      if (bin >= 0 && !listed && in_bin <= LDS::kElems) {
        if (t == 0) L.n_elems = 0;
        __syncthreads();
        pass([&](float z, uint32_t id, bool in) -> unsigned long long {
          if (in && weight_bin(z) == uint32_t(bin)) L.elems[atomicAdd(&L.n_elems, 1u)] = packed(order_key(z), id);
          return 0;
        });
        __syncthreads();
        listed = true;
        cut = key_cut<MASS>(target - (MASS ? mass0 : count0));
        cut.mass += mass0;
        listed = false;
      } else {
        cut = key_cut<MASS>(target);
      }
      if (last) add_segments(cut.at, min_p, kept);
      return cut;
    }
    if (t == 0) L.n_cand = 0;
    if (last) clear_segments();
    __syncthreads();
    int32_t n = 0;
    pass([&](float z, uint32_t id, bool in) -> unsigned long long {
      const uint32_t b = weight_bin(z);
      if (in && b == uint32_t(bin)) L.cand[atomicAdd(&L.n_cand, 1u)] = packed(order_key(z), id);
      if (!last) return 0;
      const float x = weight(z);
      const bool keep = in && b < uint32_t(bin) && x >= min_p;
      n += keep;
      return keep ? fixed_weight(x) : 0ull;
    });
    __syncthreads();
    uint64_t v = uint32_t(t) < in_bin ? L.cand[t] : 0;
    __syncthreads();
    block_sort<T>(v, in_bin, L.cand);
    const float x = uint32_t(t) < in_bin ? weight(key_logit(uint32_t(v >> 32))) : 0.f;
    const uint64_t f = fixed_weight(x);
    const BlockScan<uint64_t> sc = block_scan<W>(uint32_t(t) < in_bin ? f : 0, L.red64);
    const uint32_t end = MASS ? min(uint32_t(__syncthreads_count(uint32_t(t) < in_bin && mass0 + sc.incl < target)), in_bin - 1)
                              : uint32_t(target - count0) - 1;
    if (uint32_t(t) == end) {
      L.cut = v;
      L.mass_before = mass0 + sc.incl;
    }
    if (last && uint32_t(t) <= end && x >= min_p) {
      const uint32_t id = ~uint32_t(v);
      atomicAdd(&L.segs[id >> seg_shift], (unsigned long long)f);
      ++n;
    }
    __syncthreads();
    cut.at = L.cut;
    cut.mass = L.mass_before;
    __syncthreads();
    if (last) *kept = n;
    return cut;
  }

  // The same cut by the logits' keys, for any row, in windows of 2,048 values of the keys' upper
  // halves from the maximum down (16 octaves of a logit's size, at bf16's
  // resolution), then, in fp32, by the rest of the key; among equal logits by their ids.
  template <bool MASS>
  __device__ __forceinline__ Cut key_cut(uint64_t target) {
    const uint32_t km = order_key(m) >> 16;
    uint32_t count0 = 0, key = 0;
    uint64_t mass0 = 0;
    for (uint32_t off0 = 0;; off0 += kBins) {
      if (off0 > km) return Cut{kEvery, mass0};
      clear_hist(L);
      each([&](uint32_t k, float z, uint32_t) {
        const uint32_t b = km - (k >> 16) - off0;
        if (b < uint32_t(kBins)) {
          atomicAdd(&L.hist.count[b], 1u);
          atomicAdd(&L.hist.mass[b], fixed_weight(weight(z)));
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
      // the next 11 bits, then the last 5
      for (int last = 0; last < 2; ++last) {
        const uint32_t prefix = key, below = last ? 5 : 16, shift = last ? 0 : 5, most = last ? 31 : kBins - 1;
        clear_hist(L);
        each([&](uint32_t k, float z, uint32_t) {
          if (k >> below == prefix) {
            const uint32_t b = most - ((k >> shift) & most);
            atomicAdd(&L.hist.count[b], 1u);
            atomicAdd(&L.hist.mass[b], fixed_weight(weight(z)));
          }
        });
        __syncthreads();
        find_bin<MASS>(L, target, count0, mass0);
        count0 = L.found_before;
        mass0 = L.mass_before;
        key = (prefix << (last ? 5 : 11)) | (most - uint32_t(L.found));
        __syncthreads();
      }
    } else {
      key = (key << 16) | ((key & 0x8000u) ? 0u : 0xffffu);
    }
    const uint32_t in_bin = L.found_count;
    const uint64_t unit = L.mass_count / in_bin;  // the bin's logits are equal
    uint64_t ties = target - (MASS ? mass0 : count0);
    if (MASS) ties = unit ? (ties + unit - 1) / unit : in_bin;
    if (ties > in_bin) ties = in_bin;
    __syncthreads();
    return Cut{packed(key, tie_id(key, uint32_t(ties))), mass0 + ties * unit};
  }

  // The id of the n-th token, in id order, whose key is this (there are as many).
  __device__ __forceinline__ uint32_t tie_id(uint32_t key, uint32_t n) {
    const int t = threadIdx.x;
    clear_segments();
    each([&](uint32_t k, float, uint32_t id) {
      if (k == key) atomicAdd(&L.segs[id >> seg_shift], 1ull);
    });
    __syncthreads();
    const int32_t per = (nseg + T - 1) / T, s0 = t * per, s1 = min(s0 + per, nseg);
    uint32_t own = 0;
    for (int32_t i = s0; i < s1; ++i) own += uint32_t(L.segs[i]);
    uint32_t before = block_scan<W>(own, L.red32).excl;
    for (int32_t i = s0; i < s1; ++i) {
      const uint32_t x = uint32_t(L.segs[i]);
      if (before < n && n <= before + x) {
        L.seg = i;
        L.seg_ties = before;
      }
      before += x;
    }
    __syncthreads();
    if (t < 64) {
      uint32_t rank = L.seg_ties;
      for (uint32_t b = 0; b < 1u << (seg_shift - 9); ++b) {
        const uint32_t w = ((uint32_t(L.seg) << (seg_shift - 9)) + b) * 64 + t;
        Group<DT, ROW> g;
        g.get(row, V, min(w, ng - 1));
        g.place(V, min(w, ng - 1));
        uint32_t here = 0;
#pragma unroll
        for (int e = 0; e < kGroup; ++e) here += w < ng && order_key(g.at(e)) == key;
        const lanes::Scan<uint32_t> sc = lanes::wave_scan(here);
        uint32_t at = rank + sc.excl;
#pragma unroll
        for (int e = 0; e < kGroup; ++e)
          if (w < ng && order_key(g.at(e)) == key && ++at == n) L.found_count = w * kGroup + e;
        rank += lanes::readlane(sc.incl, 63);
      }
    }
    __syncthreads();
    const uint32_t id = L.found_count;
    __syncthreads();
    return id;
  }

  // Segments of the cuts: 512 logits, or as many more as keep them within the LDS array.
  __device__ __forceinline__ void clear_segments() {
    seg_shift = V <= 512u * kMostSegs ? 9 : V <= 1024u * kMostSegs ? 10 : 11;
    nseg = int32_t((V + (1u << seg_shift) - 1) >> seg_shift);
    for (int32_t i = threadIdx.x; i < nseg; i += T) L.segs[i] = 0;
    __syncthreads();
  }
  // Calls f(logit, id, whether it counts) on the listed logits, or on all, and adds the
  // weights that it returns to their segments.  Where all are looked at, a
  // wavefront's 64 groups lie in one segment and are added first.
  template <typename F>
  __device__ __forceinline__ void pass(F f) {
    if (listed) {
      for (uint32_t i = threadIdx.x; i < L.n_elems; i += T) {
        const uint64_t x = L.elems[i];
        const unsigned long long sum = f(key_logit(uint32_t(x >> 32)), ~uint32_t(x), true);
        if (sum) atomicAdd(&L.segs[~uint32_t(x) >> seg_shift], sum);
      }
    } else {
      all_groups([&](const Group<DT, ROW> &g, uint32_t w, bool in) {
        unsigned long long sum = 0;
#pragma unroll
        for (int e = 0; e < kGroup; ++e) sum += f(g.at(e), w * kGroup + e, in);
        sum = lanes::wave_sum(uint64_t(sum));
        if (sum && (threadIdx.x & 63) == 0) atomicAdd(&L.segs[w >> (seg_shift - 3)], sum);
      });
    }
  }
  // Weights of every segment under a cut and min_p, and this thread's share of the kept tokens.
  __device__ __forceinline__ void add_segments(uint64_t cut, float min_p, int32_t *kept) {
    clear_segments();
    int32_t n = 0;
    pass([&](float z, uint32_t id, bool in) -> unsigned long long {
      const float x = weight(z);
      const bool keep = in && packed(order_key(z), id) >= cut && x >= min_p;
      n += keep;
      return keep ? fixed_weight(x) : 0ull;
    });
    __syncthreads();
    *kept = n;
  }

  // The segment of the draw: the last one of positive weight whose exclusive
  // prefix is at most u times the total.  Leaves it and the weight left in LDS.
  template <typename WF>
  __device__ __forceinline__ void draw_segment(int32_t n, float u, WF weight_of) {
    const int t = threadIdx.x;
    const int32_t per = (n + T - 1) / T;  // consecutive segments of one thread
    const int32_t s0 = t * per, s1 = min(s0 + per, n);
    double w = 0.0;
    for (int32_t s = s0; s < s1; ++s) w += weight_of(s);
    if (t == 0) L.seg = -1;
    const BlockScan<double> bw = block_scan<W>(w, reinterpret_cast<double *>(L.red64));
    const double target = double(u) * bw.total;
    int32_t best = -1;
    double rem = 0.0, at = bw.excl;
    if (w > 0.0 && at <= target)
      for (int32_t s = s0; s < s1; ++s) {
        const double x = weight_of(s);
        if (x > 0.0 && at <= target) {
          best = s;
          rem = target - at;
        }
        at += x;
      }
    if (best >= 0) atomicMax(&L.seg, best);
    __syncthreads();
    if (best >= 0 && L.seg == best) L.rem = rem;
    __syncthreads();
  }

  // The token of the drawn segment of `blocks` times 64 groups, by one
  // wavefront, among those above the cut that min_p keeps.  Every lane returns (token, logit).
  __device__ __forceinline__ void draw_token(int32_t blocks, uint64_t cut, float min_p, int32_t *token, float *logit) {
    const int lane = threadIdx.x & 63;
    double base = 0.0;
    const double rem = L.rem;
    *token = 0;
    *logit = 0.f;
    for (int32_t b = 0; b < blocks; ++b) {
      const uint32_t w = uint32_t(L.seg * blocks + b) * 64 + lane;
      if (w - lane >= ng) break;
      Group<DT, ROW> g;
      g.get(row, V, min(w, ng - 1));
      g.place(V, min(w, ng - 1));
      float e[kGroup];
      double sum = 0.0;
      int last = -1;
#pragma unroll
      for (int i = 0; i < kGroup; ++i) {
        const float x = weight(g.at(i));
        e[i] = w < ng && packed(order_key(g.at(i)), w * kGroup + i) >= cut && x >= min_p ? x : 0.f;
        sum += double(e[i]);
        if (e[i] > 0.f) last = i;
      }
      const lanes::Scan<double> sc = lanes::wave_scan(sum);
      const uint64_t can = __ballot(last >= 0 && base + sc.excl <= rem);
      if (can) {  // a later block takes over where it begins at or before the place
        const int winner = 63 - __builtin_clzll(can);
        int pick = last >= 0 ? last : 0;
        double acc = base + sc.excl;
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
      base += lanes::readlane(sc.incl, 63);
    }
  }

  int32_t nseg;
  uint32_t seg_shift;

  // Tokens that are not masked (this thread's share).
  __device__ __forceinline__ uint32_t unmasked() {
    uint32_t n = 0;
    each([&](uint32_t, float, uint32_t) { ++n; });
    return n;
  }
};

}  // namespace
}  // namespace dsde
