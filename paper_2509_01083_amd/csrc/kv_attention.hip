// Attention of each sequence's newest rows over its paged cache.
//
// With x_t = scale log2(e) q . k_t for the tokens t that a row sees, and any reference m:
//   l = sum_t 2^(x_t - m),  o = sum_t 2^(x_t - m) v_t,  out = o / l,  lse = (m + log2 l) ln 2
// and of parts of the tokens with references m_i the whole has m = max m_i, l = sum 2^(m_i - m) l_i,
// o likewise.  So a wavefront goes over its share of the tokens once, with its keys, values and
// accumulators in registers; what is joined is (m, l, o).
//
// Bound by HBM: every key and value is read once, and the rows of all query heads of a key head
// (and of all its newest tokens) share that read.  The matrix instructions hold 16 rows at a time:
//   scores^T (16 keys x 16 rows)  = K (16 x d) Q^T (d x 16)
//   out^T    (16 dims x 16 rows) += V^T (16 x 32 keys) P^T (32 x 16)
// Scores come out with a row's keys in the registers of four lanes, in the order that the second
// product takes P in: its contraction runs over keys in whatever order both operands have, so the
// probabilities never leave their lane.  V^T wants eight keys of one dimension in a lane:
// lane (c, g) loads dimensions 8c .. 8c+7 of its eight keys, whole rows of 256 bytes per four
// lanes' keys, and picks halves of registers with v_perm (one per two elements).
#include "kv.hpp"

namespace dsde {
namespace {

using f32x4 = __attribute__((ext_vector_type(4))) float;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;

constexpr int kAttendThreads = 256, kAttendWaves = 4;
constexpr float kLn2f = 0.69314718f;
// A row's reference is raised once a score passes it by this much (weights stay under 2^8).
constexpr float kSlack = 8.0f;

// A call's integer arrays through scalar loads where the index is the same in all lanes (nothing writes them
// meanwhile): a page that lay in vector registers would take two of them for every load's address.
using ConstInt = const int32_t __attribute__((address_space(4))) *;
__device__ __forceinline__ ConstInt constant(const int32_t *p) { return (ConstInt) reinterpret_cast<uintptr_t>(p); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Elements of a cache type, DP the head size rounded up to 64, 128 or 256.  Lane (r, g) = (lane & 15, lane >> 4).
template <int CACHE, int DP>
struct Shape {
  static constexpr int kElt = CACHE == DSDE_FP32 ? 4 : CACHE == DSDE_BF16 ? 2 : 1;
  static constexpr int kSub = CACHE == DSDE_FP32 ? 1 : 2;      // subtiles of 16 keys
  static constexpr int kTile = 16 * kSub;                      // keys of a step
  static constexpr int kPer16 = 16 / kElt;                     // elements in 16 bytes
  static constexpr int kChunks = DP * kElt / 64;               // 16-byte chunks of a key per lane: chunk j at 16 (4 j + g)
  static constexpr int kVec = CACHE == DSDE_FP32 ? 4 : DP == 64 ? 4 : 8;  // dimensions of a value that a lane loads at once
  static constexpr int kSets = DP / (16 * kVec);               // sets of 16 kVec dimensions
  static constexpr int kVecBytes = kVec * kElt;
  static constexpr int kVecWords = kVecBytes / 4;
  static constexpr int kKeys = 4 * kSub;                       // keys of a tile in a lane: 16 t + 4 g + i
  static constexpr int kQWords = CACHE == DSDE_FP32 ? DP / 4 : DP / 8;  // words of a row's share in a lane
};

template <int WORDS>
struct Words {
  uint32_t w[WORDS];
};
// Memory that lanes read through one scalar descriptor and 32-bit offsets; what lies at or behind `bytes` reads as 0.
using Buffer = __amdgpu_buffer_rsrc_t;
__device__ __forceinline__ Buffer buffer(const char *base, int32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, bytes, 0x00020000);
}
constexpr uint32_t kOutside = 0x40000000;  // an offset behind every buffer here
template <int WORDS>
__device__ __forceinline__ Words<WORDS> load_words(Buffer from, uint32_t off, uint32_t base = 0) {
  Words<WORDS> r;
  if constexpr (WORDS == 4) {
    const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, off, base, 0));
    r.w[0] = x.x, r.w[1] = x.y, r.w[2] = x.z, r.w[3] = x.w;
  } else if constexpr (WORDS == 2) {
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(from, off, base, 0));
    r.w[0] = x.x, r.w[1] = x.y;
  } else {
    r.w[0] = __builtin_amdgcn_raw_buffer_load_b32(from, off, base, 0);
  }
  return r;
}
// Two of four 8-bit floats as bf16, exact.
template <bool HIGH>
__device__ __forceinline__ uint32_t widen(uint32_t x) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, HIGH));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf16x2 p{__bf16(a), __bf16(b)};
  return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ bf16x8 operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const u32x4 x{a, b, c, d};
  return __builtin_bit_cast(bf16x8, x);
}
template <int CACHE>
__device__ __forceinline__ bool not_finite(uint32_t x) {
  if constexpr (CACHE == DSDE_FP32) return (x & 0x7f800000u) == 0x7f800000u;
  if constexpr (CACHE == DSDE_BF16) return (x & 0x7f800000u) == 0x7f800000u || (x & 0x7f80u) == 0x7f80u;
  const uint32_t y = ~x & 0x7f7f7f7fu;  // a byte of 0: NaN
  return ((y - 0x01010101u) & ~y & 0x80808080u) != 0;
}

// One sequence of a call.
struct Seq {
  int32_t row0, n, context;  // its rows, tokens in the cache
  int32_t tile0, tiles;      // tiles that any of its rows sees, one at least
  int32_t blocks;            // blocks of rows
  uint32_t err;
};
template <int TILE>
__device__ __forceinline__ Seq sequence(const AttendArgs &a, int32_t b, int32_t block_rows) {
  Seq s;
  s.row0 = constant(a.cu_rows)[b];
  const int64_t end = constant(a.cu_rows)[b + 1];
  s.n = int32_t(end - s.row0);
  s.context = constant(a.context)[b];
  s.err = 0;
  if (s.row0 < 0 || end < s.row0 || end > a.T || end - s.row0 > a.max_rows) {
    s.err = DSDE_ERR_LAYOUT;
    s.n = 0;
  }
  if (s.context < 0 || s.context > (int64_t(a.width) << a.cache.shift)) {
    s.err |= DSDE_ERR_LAYOUT;
    s.context = 0;
  }
  const int64_t first = a.window > 0 ? int64_t(s.context) - s.n - a.window + 1 : 0;
  s.tile0 = first > 0 ? int32_t(first) / TILE : 0;
  s.tiles = (s.context + TILE - 1) / TILE - s.tile0;
  if (s.tiles < 1) s.tiles = 1;
  s.blocks = (s.n * a.group + block_rows - 1) / block_rows;
  return s;
}
template <int TILE>
__device__ __forceinline__ int64_t units_of(const AttendArgs &a, int32_t b, int32_t block_rows) {
  const Seq s = sequence<TILE>(a, b, block_rows);
  return int64_t(s.tiles) * s.blocks * a.cache.heads;
}

// Units of work (a tile of one head and one row block) that each workgroup takes: a tile per
// wavefront at least, so that short calls do not end in joining many parts.
__device__ __forceinline__ int64_t share_of(int64_t all, int32_t groups) {
  const int64_t n = (all + groups - 1) / groups;
  return n > kAttendWaves ? n : kAttendWaves;
}

// A row's reference, sum and values where parts meet.
struct Joined {
  float m, l;
};

// Writes columns d .. d+3 of a finished row, and with `stats` its log-normaliser.
template <int CACHE>
__device__ __forceinline__ void finish(const AttendArgs &a, const Seq &s, int32_t h, int32_t row, Joined x, f32x4 o, int32_t d,
                                       bool stats) {
  const int32_t j = row / a.group, head = h * a.group + (row - j * a.group);
  const int64_t t = int64_t(s.row0) + j;
  if (stats && a.lse) a.lse[t * (int64_t(a.group) * a.cache.heads) + head] = x.l == 0.0f ? -INFINITY : (x.m + __builtin_amdgcn_logf(x.l)) * kLn2f;
  if (d >= a.cache.dim) return;
  float inv = x.l == 0.0f ? 0.0f : 1.0f / x.l;
  if constexpr (CACHE == DSDE_E4M3) inv *= a.cache.v_scale[h];
  char *to = a.out + t * a.out_token_stride + int64_t(head) * a.out_head_stride;
  if constexpr (CACHE == DSDE_FP32)
    *reinterpret_cast<f32x4 *>(to + d * 4) = o * inv;
  else
    *reinterpret_cast<u32x2 *>(to + d * 2) = u32x2{pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv)};
}

// The wavefront's view of its rows.
template <int MT>
struct Rows {
  int32_t hi[MT], lo[MT];      // tokens that lane r's row of each block sees: lo .. hi
  int32_t hi_all, lo_all;      // seen by every row
  int32_t hi_any, lo_any;      // seen by any
};

template <int CACHE, int DP, int MT>
struct Wave {
  using S = Shape<CACHE, DP>;
  const AttendArgs &a;
  const Seq &s;
  int lane, r, g;
  const char *k_head, *v_head;  // of the head, from the cache's start
  ConstInt table;               // of the sequence
  float c;                      // scale log2(e), with the keys' scale
  int32_t mtiles;               // row tiles of this block that have rows
  Rows<MT> rows;
  uint32_t k_off, v_off;

  uint32_t q[MT][S::kQWords];
  f32x4 o[MT][S::kSets][S::kVec];
  float m[MT], l[MT];
  // keys and values of a tile, and where its subtiles are bad
  Words<4> k[S::kSub][S::kChunks];
  Words<S::kVecWords> v[S::kKeys][S::kSets];

  // A subtile's place in the cache.
  struct At {
    int64_t offset;
    bool bad;    // its page is none
    bool there;  // it is to be read
  };
  __device__ __forceinline__ At locate(int32_t tile, int t, bool wanted) const {
    const int32_t key = tile * S::kTile + 16 * t;
    const int32_t page = wanted && key < s.context ? table[key >> a.cache.shift] : 0;
    At x;
    x.bad = uint32_t(page) >= uint32_t(a.cache.pages);
    x.there = wanted && !x.bad;
    x.offset = (x.bad ? 0 : int64_t(page) * a.cache.page_stride) + int64_t(key & ((1 << a.cache.shift) - 1)) * a.cache.token_stride;
    return x;
  }
  // Bytes of a subtile's 16 rows; none of one that is not to be read, whose loads give 0 without memory.
  __device__ __forceinline__ int32_t span(const At &x) const { return x.there ? 15 * a.cache.token_stride + a.cache.dim * S::kElt : 0; }

  __device__ __forceinline__ void load_k(const At (&at)[S::kSub]) {
#pragma unroll
    for (int t = 0; t < S::kSub; ++t) {
      const Buffer from = buffer(k_head + at[t].offset, span(at[t]));
#pragma unroll
      for (int j = 0; j < S::kChunks; ++j)  // 0 behind the row's end
        k[t][j] = load_words<4>(from, (4 * j + g) * S::kPer16 < a.cache.dim ? k_off + 64 * j : kOutside);
    }
  }
  __device__ __forceinline__ void load_v(const At (&at)[S::kSub]) {
#pragma unroll
    for (int t = 0; t < S::kSub; ++t) {
      const Buffer from = buffer(v_head + at[t].offset, span(at[t]));
#pragma unroll
      for (int e = 0; e < S::kSets; ++e) {
        const uint32_t off = (16 * e + r) * S::kVec < a.cache.dim ? v_off + 16 * S::kVecBytes * e : kOutside;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * t + i][e] = load_words<S::kVecWords>(from, off, i * a.cache.token_stride);
      }
    }
  }

  __device__ __forceinline__ void load_q(const char *base, int32_t row, int32_t count, int mt) {
    // lane r's row; rows behind the last are zero
    const bool live = row < count;
    const int32_t j = live ? row / a.group : 0, head = live ? row - j * a.group : 0;
    const char *p = base + j * a.q.token_stride + head * a.q.head_stride;
    constexpr int kQElt = CACHE == DSDE_FP32 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < S::kQWords / 4; ++i) {
      // the dimensions that the keys' chunks hold
      int32_t d;
      if constexpr (CACHE == DSDE_E4M3)
        d = (4 * (i / 2) + g) * 16 + 8 * (i % 2);
      else
        d = (4 * i + g) * S::kPer16;
      Words<4> x{};
      if (live && d < a.cache.dim) {
        const u32x4 y = *reinterpret_cast<const u32x4 *>(p + d * kQElt);
        x = Words<4>{{y.x, y.y, y.z, y.w}};
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) q[mt][4 * i + e] = x.w[e];
    }
    rows.hi[mt] = live ? s.context - s.n + j : -1;
    rows.lo[mt] = a.window > 0 && rows.hi[mt] >= a.window ? rows.hi[mt] - a.window + 1 : 0;
  }

  // Scores of a tile, in the log2 domain; NaN of a bad page (its keys are 0).
  __device__ __forceinline__ void scores(f32x4 (&x)[MT][S::kSub], const At (&at)[S::kSub]) {
#pragma unroll
    for (int t = 0; t < S::kSub; ++t) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) x[mt][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < S::kChunks; ++j) {
        const Words<4> &w = k[t][j];
        if constexpr (CACHE == DSDE_FP32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
              x[mt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.w[e]), __uint_as_float(q[mt][4 * j + e]), x[mt][t], 0, 0, 0);
        } else if constexpr (CACHE == DSDE_BF16) {
          const bf16x8 kk = operand(w.w[0], w.w[1], w.w[2], w.w[3]);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const uint32_t *p = &q[mt][4 * j];
            x[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, operand(p[0], p[1], p[2], p[3]), x[mt][t], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const bf16x8 kk = operand(widen<false>(w.w[2 * e]), widen<true>(w.w[2 * e]), widen<false>(w.w[2 * e + 1]),
                                      widen<true>(w.w[2 * e + 1]));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              const uint32_t *p = &q[mt][8 * j + 4 * e];
              x[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, operand(p[0], p[1], p[2], p[3]), x[mt][t], 0, 0, 0);
            }
          }
        }
      }
      const float f = at[t].bad ? NAN : c;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) x[mt][t] *= f;
    }
  }

  // Raises references where scores pass them, and turns scores into weights.
  __device__ __forceinline__ void weigh(f32x4 (&x)[MT][S::kSub]) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < S::kSub; ++t) top = fmaxf(fmaxf(fmaxf(x[mt][t].x, x[mt][t].y), fmaxf(x[mt][t].z, x[mt][t].w)), top);
      if (__any(top > m[mt] + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m[mt], top);
        const float f = now == -INFINITY ? 1.0f : exp2_fast(m[mt] - now);
        m[mt] = now;
        l[mt] *= f;
#pragma unroll
        for (int e = 0; e < S::kSets; ++e)
#pragma unroll
          for (int j = 0; j < S::kVec; ++j) o[mt][e][j] *= f;
      }
      const float ref = m[mt] == -INFINITY ? 0.0f : m[mt];
      float sum = 0.0f;
#pragma unroll
      for (int t = 0; t < S::kSub; ++t) {
        x[mt][t] = f32x4{exp2_fast(x[mt][t].x - ref), exp2_fast(x[mt][t].y - ref), exp2_fast(x[mt][t].z - ref), exp2_fast(x[mt][t].w - ref)};
        sum += (x[mt][t].x + x[mt][t].y) + (x[mt][t].z + x[mt][t].w);
      }
      l[mt] += sum;
    }
  }

  // Adds the weights' values.  The weights are rounded to the type of the values for the matrix instruction: half a
  // unit of the last place each, as the output's own rounding, and independent of each other.
  // ONLY: to the rows of token `token` alone (a weight of 0 would not keep a NaN from the others).
  template <bool ONLY = false>
  __device__ __forceinline__ void add(const f32x4 (&p)[MT][S::kSub], int32_t token = 0) {
    const auto put = [&](int mt, int e, int j, f32x4 x) { o[mt][e][j] = !ONLY || rows.hi[mt] == token ? x : o[mt][e][j]; };
    if constexpr (CACHE == DSDE_FP32) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < S::kSets; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
              put(mt, e, j, __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][e].w[j]), p[mt][0][i], o[mt][e][j], 0, 0, 0));
    } else {
      bf16x8 w[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        w[mt] = operand(pack_bf16(p[mt][0].x, p[mt][0].y), pack_bf16(p[mt][0].z, p[mt][0].w),
                        pack_bf16(p[mt][1].x, p[mt][1].y), pack_bf16(p[mt][1].z, p[mt][1].w));
#pragma unroll
      for (int e = 0; e < S::kSets; ++e)
#pragma unroll
        for (int j2 = 0; j2 < S::kVec / 2; ++j2) {  // two dimensions from one word of each key
          uint32_t x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if constexpr (CACHE == DSDE_BF16)
              x[i] = v[i][e].w[j2];
            else
              x[i] = j2 & 1 ? widen<true>(v[i][e].w[j2 / 2]) : widen<false>(v[i][e].w[j2 / 2]);
          }
          uint32_t lo[4], hi[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            lo[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);
            hi[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
          }
          const bf16x8 a0 = operand(lo[0], lo[1], lo[2], lo[3]), a1 = operand(hi[0], hi[1], hi[2], hi[3]);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            put(mt, e, 2 * j2, __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, w[mt], o[mt][e][2 * j2], 0, 0, 0));
            put(mt, e, 2 * j2 + 1, __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, w[mt], o[mt][e][2 * j2 + 1], 0, 0, 0));
          }
        }
    }
  }

  // Scores that some row does not see.
  __device__ __forceinline__ void mask(f32x4 (&x)[MT][S::kSub], int32_t tile) {
#pragma unroll
    for (int t = 0; t < S::kSub; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t key = tile * S::kTile + 16 * t + 4 * g + i;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) x[mt][t][i] = key >= rows.lo[mt] && key <= rows.hi[mt] ? x[mt][t][i] : -INFINITY;
      }
  }
  __device__ __forceinline__ bool keep(int32_t tile, int32_t lo, int32_t hi) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < S::kKeys; ++i) {
      const int32_t key = tile * S::kTile + 16 * (i / 4) + 4 * g + i % 4;
      const bool seen = key >= lo && key <= hi;
#pragma unroll
      for (int e = 0; e < S::kSets; ++e)
#pragma unroll
        for (int w = 0; w < S::kVecWords; ++w) {
          v[i][e].w[w] = seen ? v[i][e].w[w] : 0;
          odd |= not_finite<CACHE>(v[i][e].w[w]);
        }
    }
    return __any(odd);
  }
  // The same for values: a weight of 0 takes no part only beside finite ones.  Values that no row sees become 0; where
  // one that some rows see is not finite (rare), the tile's values are read again for each of the sequence's tokens,
  // which adds what it sees, and then all become 0.
  __device__ __forceinline__ void mask_values(const f32x4 (&p)[MT][S::kSub], int32_t tile, const At (&from)[S::kSub]) {
    if (!keep(tile, rows.lo_any, rows.hi_any)) return;
    for (int32_t token = s.context - s.n; token < s.context; ++token) {
      load_v(from);
      keep(tile, a.window > 0 && token >= a.window ? token - a.window + 1 : 0, token);
      add<true>(p, token);
    }
    keep(tile, 0, -1);
  }

  // Tiles first, first + step, ... below end.
  __device__ __forceinline__ void run(int32_t first, int32_t end, int32_t step) {
    if (first >= end) return;
    At at[S::kSub], next[S::kSub];
#pragma unroll
    for (int t = 0; t < S::kSub; ++t) at[t] = locate(first, t, true);
    load_k(at);
    load_v(at);
    // The next tile's keys are on their way while this one's values are weighed, and its values while the next scores
    // are taken, into registers that have just been read; a tile behind the last is none.  No load stands behind a
    // branch: waits could not be counted then.
    for (int32_t tile = first; tile < end; tile += step) {
#pragma unroll
      for (int t = 0; t < S::kSub; ++t) next[t] = locate(tile + step, t, tile + step < end);
      f32x4 x[MT][S::kSub];
      scores(x, at);
      load_k(next);
      const bool clear = tile * S::kTile >= rows.lo_all && tile * S::kTile + S::kTile - 1 <= rows.hi_all;
      if (!clear) mask(x, tile);
      weigh(x);
      if (!clear) mask_values(x, tile, at);
      add(x);
      load_v(next);
#pragma unroll
      for (int t = 0; t < S::kSub; ++t) at[t] = next[t];
    }
  }
};

// A place in the order of all work: sequence, key head, row block, tile.
struct Cursor {
  int32_t b, h, block, tile;
};

template <int CACHE, int DP, int MT, int OCC>
__global__ __launch_bounds__(kAttendThreads, OCC) void attend_kernel(AttendArgs a) {
  using S = Shape<CACHE, DP>;
  constexpr int kRows = 16 * MT;
  constexpr int kPitch = DP + 4;
  __shared__ float s_o[kAttendWaves][16][kPitch];
  __shared__ float s_m[kAttendWaves][kRows], s_l[kAttendWaves][kRows];
  __shared__ int64_t s_sum[kAttendWaves];
  __shared__ Cursor s_at;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);

  // where this workgroup's share of the work begins
  const int32_t per = (a.B + kAttendThreads - 1) / kAttendThreads;
  const int32_t b0 = tid * per < a.B ? tid * per : a.B, b1 = b0 + per < a.B ? b0 + per : a.B;
  int64_t own = 0;
  for (int32_t b = b0; b < b1; ++b) own += units_of<S::kTile>(a, b, kRows);
  int64_t upto = own;
  for (int n = 1; n < 64; n <<= 1) {
    const int64_t o = __shfl_up(upto, n);
    if (lane >= n) upto += o;
  }
  if (lane == 63) s_sum[wave] = upto;
  __syncthreads();
  int64_t all = 0;
  for (int i = 0; i < kAttendWaves; ++i) {
    if (i < wave) upto += s_sum[i];
    all += s_sum[i];
  }
  const int64_t share = share_of(all, gridDim.x);
  const int64_t begin = int64_t(blockIdx.x) * share, end = begin + share < all ? begin + share : all;
  int64_t before = upto - own;
  const bool mine = begin >= before && begin < upto;
  if (mine || blockIdx.x == 0) {
    int64_t *units = static_cast<int64_t *>(a.workspace);
    for (int32_t b = b0; b < b1; ++b) {
      const Seq s = sequence<S::kTile>(a, b, kRows);
      const int64_t n = int64_t(s.tiles) * s.blocks * a.cache.heads;
      if (begin >= before && begin < before + n) {
        const int64_t x = begin - before;
        const int32_t item = int32_t(x / s.tiles);
        s_at = Cursor{b, item / s.blocks, item % s.blocks, int32_t(x % s.tiles)};
      }
      if (blockIdx.x == 0) units[b] = before;
      before += n;
    }
    if (blockIdx.x == 0 && tid == 0) units[a.B] = all;
  }
  if (begin >= end) return;
  __syncthreads();

  int64_t left = end - begin;
  Cursor at = s_at;
  at.b = uniform(at.b), at.h = uniform(at.h), at.block = uniform(at.block), at.tile = uniform(at.tile);
  bool first = true;
  while (left > 0 && at.b < a.B) {
    Seq s = sequence<S::kTile>(a, at.b, kRows);
    if (s.blocks == 0) {
      at = Cursor{at.b + 1, 0, 0, 0};
      continue;
    }
    const int32_t count = int32_t(left < s.tiles - at.tile ? left : s.tiles - at.tile);
    const int32_t rows = s.n * a.group, row0 = at.block * kRows;

    Wave<CACHE, DP, MT> w{a, s};
    w.lane = lane, w.r = lane & 15, w.g = lane >> 4;
    w.k_head = a.cache.k + at.h * a.cache.head_stride;
    w.v_head = a.cache.v + at.h * a.cache.head_stride;
    w.table = constant(a.table + int64_t(at.b) * a.width);
    w.c = a.scale * kLog2e;
    if constexpr (CACHE == DSDE_E4M3) w.c *= a.cache.k_scale[at.h];
    w.k_off = uint32_t(w.r * a.cache.token_stride + 16 * w.g);
    w.v_off = uint32_t(4 * w.g * a.cache.token_stride + S::kVecBytes * w.r);
    const char *q = a.q.data + s.row0 * a.q.token_stride + int64_t(at.h) * a.group * a.q.head_stride;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      w.load_q(q, row0 + 16 * mt + w.r, rows, mt);
      w.m[mt] = -INFINITY, w.l[mt] = 0.0f;
#pragma unroll
      for (int e = 0; e < S::kSets; ++e)
#pragma unroll
        for (int j = 0; j < S::kVec; ++j) w.o[mt][e][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int32_t newest = s.context - 1, oldest = s.context - s.n;
    w.rows.hi_all = oldest, w.rows.hi_any = newest;
    w.rows.lo_all = a.window > 0 && newest >= a.window ? newest - a.window + 1 : 0;
    w.rows.lo_any = a.window > 0 && oldest >= a.window ? oldest - a.window + 1 : 0;
    const int32_t t0 = s.tile0 + at.tile;
    w.run(t0 + wave, t0 + count, kAttendWaves);

    // join the wavefronts
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float l = w.l[mt];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (w.g == 0) s_m[wave][16 * mt + w.r] = w.m[mt], s_l[wave][16 * mt + w.r] = l;
    }
    const bool done = count == s.tiles;
    float *partial = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + attend_layout_partial(a.B)) +
                     (int64_t(blockIdx.x) * 2 + (first ? 0 : 1)) * (kRows * (DP + 2));
    for (int mt = 0; mt < MT; ++mt) {
      if (row0 + 16 * mt >= rows) break;
#pragma unroll
      for (int x = 0; x < MT; ++x)
        if (x == mt) {
#pragma unroll
          for (int e = 0; e < S::kSets; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int j = 0; j < S::kVec; j += 4)
                *reinterpret_cast<f32x4 *>(&s_o[wave][w.r][(16 * e + 4 * w.g + i) * S::kVec + j]) =
                    f32x4{w.o[x][e][j][i], w.o[x][e][j + 1][i], w.o[x][e][j + 2][i], w.o[x][e][j + 3][i]};
        }
      __syncthreads();
      const int32_t rr = tid >> 4, cc = tid & 15, row = row0 + 16 * mt + rr;
      if (row < rows) {
        float top = -INFINITY;
        for (int i = 0; i < kAttendWaves; ++i) top = fmaxf(top, s_m[i][16 * mt + rr]);
        const float ref = top == -INFINITY ? 0.0f : top;
        float f[kAttendWaves], sum = 0.0f;
        for (int i = 0; i < kAttendWaves; ++i) {
          f[i] = exp2_fast(s_m[i][16 * mt + rr] - ref);
          sum += f[i] * s_l[i][16 * mt + rr];
        }
        if (s.err) sum = NAN;  // a context that is none
#pragma unroll
        for (int k = 0; k < DP / 64; ++k) {
          const int32_t d = 64 * k + 4 * cc;
          f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
          for (int i = 0; i < kAttendWaves; ++i) o += f[i] * *reinterpret_cast<const f32x4 *>(&s_o[i][rr][d]);
          if (done)
            finish<CACHE>(a, s, at.h, row, Joined{top, sum}, o, d, k == 0 && cc == 0);
          else
            *reinterpret_cast<f32x4 *>(&partial[(16 * mt + rr) * DP + d]) = o;
        }
        if (!done && cc == 0) partial[kRows * DP + 16 * mt + rr] = top, partial[kRows * (DP + 1) + 16 * mt + rr] = sum;
      }
      __syncthreads();
    }

    left -= count;
    first = false;
    at.tile = 0;
    if (++at.block == s.blocks) {
      at.block = 0;
      if (++at.h == a.cache.heads) at = Cursor{at.b + 1, 0, 0, 0};
    }
  }
}

// Joins the parts of rows whose tokens more than one workgroup had, and checks every sequence.
template <int CACHE, int DP, int MT>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a, int32_t groups, int32_t max_blocks) {
  using S = Shape<CACHE, DP>;
  constexpr int kRows = 16 * MT;
  constexpr int64_t kPart = kRows * (DP + 2);
  __shared__ int s_bad;
  const int64_t *units = static_cast<const int64_t *>(a.workspace);
  const float *parts = reinterpret_cast<const float *>(static_cast<const char *>(a.workspace) + attend_layout_partial(a.B));
  const int64_t share = share_of(units[a.B], groups);
  const int tid = threadIdx.x, rr = tid >> 4, cc = tid & 15;
  const int32_t per_seq = a.cache.heads * max_blocks;
  for (int64_t item = blockIdx.x; item < int64_t(a.B) * per_seq; item += gridDim.x) {
    const int32_t b = int32_t(item / per_seq), x = int32_t(item % per_seq), h = x / max_blocks, block = x % max_blocks;
    const Seq s = sequence<S::kTile>(a, b, kRows);
    if (x == 0) {
      if (tid == 0) s_bad = 0;
      __syncthreads();
      if (s.n > 0 && s.context > 0) {
        const int64_t first = a.window > 0 ? int64_t(s.context) - s.n - a.window + 1 : 0;
        bool bad = false;
        for (int32_t i = int32_t((first > 0 ? first : 0) >> a.cache.shift) + tid; i <= (s.context - 1) >> a.cache.shift; i += 256)
          bad |= uint32_t(a.table[int64_t(b) * a.width + i]) >= uint32_t(a.cache.pages);
        if (bad) s_bad = 1;
      }
      __syncthreads();
      if (tid == 0) a.seq_err[b] = s.err | (s_bad ? DSDE_ERR_PAGES : 0u);
      __syncthreads();
    }
    if (block >= s.blocks) continue;
    const int64_t from = units[b] + (int64_t(h) * s.blocks + block) * s.tiles, to = from + s.tiles;
    const int64_t w0 = from / share, w1 = (to - 1) / share;
    if (w0 == w1) continue;
    const int32_t rows = s.n * a.group;
    const float *start = parts + (2 * w0 + (from > w0 * share ? 1 : 0)) * kPart;
    for (int32_t i = rr; i < kRows && block * kRows + i < rows; i += 16) {
      float top = start[kRows * DP + i];
      for (int64_t w = w0 + 1; w <= w1; ++w) top = fmaxf(top, parts[2 * w * kPart + kRows * DP + i]);
      const float ref = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f;
      f32x4 o[DP / 64];
      for (int k = 0; k < DP / 64; ++k) o[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      for (int64_t w = w0; w <= w1; ++w) {
        const float *p = w == w0 ? start : parts + 2 * w * kPart;
        const float f = exp2_fast(p[kRows * DP + i] - ref);
        sum += f * p[kRows * (DP + 1) + i];
#pragma unroll
        for (int k = 0; k < DP / 64; ++k) o[k] += f * *reinterpret_cast<const f32x4 *>(&p[i * DP + 64 * k + 4 * cc]);
      }
#pragma unroll
      for (int k = 0; k < DP / 64; ++k)
        finish<CACHE>(a, s, h, block * kRows + i, Joined{top, sum}, o[k], 64 * k + 4 * cc, k == 0 && cc == 0);
    }
  }
}

template <int CACHE, int DP, int MT, int OCC>
void launch(const AttendArgs &a, hipStream_t stream) {
  const int32_t groups = 256 * OCC < kAttendGroups ? 256 * OCC : kAttendGroups;
  attend_kernel<CACHE, DP, MT, OCC><<<groups, kAttendThreads, 0, stream>>>(a);
  const int32_t max_blocks = (a.max_rows * a.group + 16 * MT - 1) / (16 * MT);
  const int64_t items = int64_t(a.B) * a.cache.heads * max_blocks;
  join_kernel<CACHE, DP, MT><<<uint32_t(items < 4096 ? items : 4096), 256, 0, stream>>>(a, groups, max_blocks);
}
template <int CACHE, int DP>
void by_tiles(const AttendArgs &a, hipStream_t stream) {
  const int tiles = row_tiles(a.group, a.max_rows, a.cache.dim);
  // workgroups per CU by the registers that each form takes
  if (tiles == 1)
    launch<CACHE, DP, 1, DP == 256 || (CACHE == DSDE_FP32 && DP == 128) ? 1 : 2>(a, stream);
  else if (tiles == 2)
    launch<CACHE, DP, 2, DP == 256 || CACHE == DSDE_FP32 ? 1 : 2>(a, stream);
  else if constexpr (DP <= 128)
    launch<CACHE, DP, 4, 1>(a, stream);
}
template <int CACHE>
void by_dim(const AttendArgs &a, hipStream_t stream) {
  if (a.cache.dim <= 64)
    by_tiles<CACHE, 64>(a, stream);
  else if (a.cache.dim <= 128)
    by_tiles<CACHE, 128>(a, stream);
  else
    by_tiles<CACHE, 256>(a, stream);
}

}  // namespace

int launch_kv_attention(const AttendArgs &a, hipStream_t stream) {
  if (a.cache.dtype == DSDE_FP32)
    by_dim<DSDE_FP32>(a, stream);
  else if (a.cache.dtype == DSDE_BF16)
    by_dim<DSDE_BF16>(a, stream);
  else
    by_dim<DSDE_E4M3>(a, stream);
  return hipGetLastError() == hipSuccess ? DSDE_OK : DSDE_DEVICE_ERROR;
}

}  // namespace dsde
