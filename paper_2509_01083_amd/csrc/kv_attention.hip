// Attention of each sequence's newest rows over its paged cache.
//
// With x_t = scale log2(e) q . k_t for the tokens t that a row sees, and any reference m:
//   l = sum_t 2^(x_t - m),  o = sum_t 2^(x_t - m) v_t,  out = o / l,  lse = (m + log2 l) ln 2
// and of parts of the tokens with references m_i the whole has m = max m_i, l = sum 2^(m_i - m) l_i,
// o likewise.  So a wavefront goes over its share of the tokens once, with its keys, values and
// accumulators in registers; what is joined is (m, l, o).
//
// Bound by HBM: every key and value is read once for a block of rows, in which the query heads of a key head and
// their newest tokens share that read.  A block is as many rows as registers hold: 64 of heads up to 128 (32 in fp32 above
// 64), of larger ones 32 (16 in fp32).  A key head with more rows has several blocks, each of which reads all it sees: 72
// rows of 128 in bf16 (256 sequences, 2.4 GB) take 883 us, 64 take 513.  The matrix instructions hold 16 rows at a time:
//   scores^T (16 keys x 16 rows)  = K (16 x d) Q^T (d x 16)
//   out^T    (16 dims x 16 rows) += V^T (16 x 32 keys) P^T (32 x 16)
// Scores come out with a row's keys in the registers of four lanes, in the order that the second
// product takes P in: its contraction runs over keys in whatever order both operands have, so the
// probabilities never leave their lane.  V^T wants eight keys of one dimension in a lane:
// lane (c, g) loads eight dimensions of its eight keys, whole rows of 256 bytes in sixteen lanes,
// and picks halves of registers with v_perm (one per two elements).
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
template <int CACHE, int DP, int MT>
struct Shape {
  static constexpr int kElt = CACHE == DSDE_FP32 ? 4 : CACHE == DSDE_BF16 ? 2 : 1;
  // subtiles of 16 keys: 16 KiB of keys and values at a time where registers allow (heads of 64 with 48 rows and more: 433
  // and 488 us with four subtiles, 446 and 512 with two)
  static constexpr int kLeastSub = CACHE == DSDE_FP32 ? 1 : 2;
  static constexpr int kMostSub = MT > 2 && DP > 64 ? 2 : 4;
  static constexpr int kSub = 512 / (DP * kElt) < kLeastSub ? kLeastSub : 512 / (DP * kElt) > kMostSub ? kMostSub : 512 / (DP * kElt);
  static constexpr int kTile = 16 * kSub;                      // keys of a step
  static constexpr int kPer16 = 16 / kElt;                     // elements in 16 bytes
  static constexpr int kChunks = DP * kElt / 64;               // 16-byte chunks of a key per lane: chunk j at 16 (4 j + g)
  static constexpr int kVec = CACHE == DSDE_FP32 ? 4 : DP == 64 ? 4 : 8;  // dimensions of a value that a lane loads at once
  static constexpr int kSets = DP / (16 * kVec);               // sets of 16 kVec dimensions
  static constexpr int kVecBytes = kVec * kElt;
  static constexpr int kVecWords = kVecBytes / 4;
  static constexpr int kKeys = 4 * kSub;                       // keys of a tile in a lane: 16 t + 4 g + i
  static constexpr int kQElt = CACHE == DSDE_FP32 ? 4 : 2;
  static constexpr int kQChunks = DP * kQElt / 64;             // 16-byte chunks of a query row in a lane
  // where rows and accumulators are many, the rows at hand are in LDS, or the next item's are not fetched early either:
  // a spill of a few registers in the loop costs more (12 % with 48 rows of 128)
  static constexpr bool kRowsInLds = MT * DP * kQElt > 512;
  static constexpr bool kAhead = MT * DP * kQElt <= 768;
  // first dimension of a chunk: those that the keys' chunks hold
  __device__ static __forceinline__ int32_t q_dim(int i, int g) {
    if constexpr (CACHE == DSDE_E4M3) return (4 * (i / 2) + g) * 16 + 8 * (i % 2);
    return (4 * i + g) * kPer16;
  }
};

template <int WORDS>
struct alignas(4 * WORDS) Words {
  uint32_t w[WORDS];
};
// Memory that lanes read through one scalar descriptor and 32-bit offsets; what lies at or behind `bytes` reads as 0.
using Buffer = __amdgpu_buffer_rsrc_t;
__device__ __forceinline__ Buffer buffer(const char *base, int32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, bytes, 0x00020000);
}
// Cache hint (nt): keys and values are read once.  With it 2.1 GB go at 6.3 TB/s, without at 5.7.
constexpr int kStream = 2;
constexpr uint32_t kOutside = 0x40000000;  // an offset behind every buffer here
template <int WORDS>
__device__ __forceinline__ Words<WORDS> load_words(Buffer from, uint32_t off, uint32_t base = 0) {
  Words<WORDS> r;
  if constexpr (WORDS == 4) {
    const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, off, base, kStream));
    r.w[0] = x.x, r.w[1] = x.y, r.w[2] = x.z, r.w[3] = x.w;
  } else if constexpr (WORDS == 2) {
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(from, off, base, kStream));
    r.w[0] = x.x, r.w[1] = x.y;
  } else {
    r.w[0] = __builtin_amdgcn_raw_buffer_load_b32(from, off, base, kStream);
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
__device__ __forceinline__ bf16x8 operand(const Words<4> &x) { return __builtin_bit_cast(bf16x8, x); }
// The values of a word that are not finite: the highest bit of each.  Their exponent (e4m3: all but the sign) is all ones.
template <int CACHE>
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {
  if constexpr (CACHE == DSDE_FP32) return ((x & 0x7f800000u) + 0x00800000u) & 0x80000000u;
  if constexpr (CACHE == DSDE_BF16) return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}
// The same word with those values at 0.
template <int CACHE>
__device__ __forceinline__ uint32_t finite_only(uint32_t x) {
  constexpr int kTop = CACHE == DSDE_FP32 ? 31 : CACHE == DSDE_BF16 ? 15 : 7;
  return x & ~((not_finite<CACHE>(x) >> kTop) * ((2u << kTop) - 1));
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
// The work in one line: for every sequence, key head and row block an item of kStart units (what it costs to begin
// and end one, in tiles: with 0, 1, 2, 4 units 256 sequences took 465, 449, 440, 434 us, 1,024 over e4m3 460, 408, 390,
// 400, 64 in fp32 46, 36, 39, 41) and a unit for each tile.  Every wavefront takes an equal share of the line, whatever the
// lengths are, so that all end together; items that it has a part of leave that part to join_kernel.
constexpr int32_t kStart = 2;
// units of a share at least: short calls do not end in joining many parts (1,000 tokens: 12.4 us, with 1 13.2, with 4 13.8)
constexpr int32_t kLeast = 2;
__device__ __forceinline__ int64_t units_of(const AttendArgs &a, const Seq &s) {
  return int64_t(s.tiles + kStart) * s.blocks * a.cache.heads;
}
// Where a wavefront's share begins inside an item (tile > 0), and the wavefronts that have parts of that item.
struct Start {
  int32_t h, block, tile, w0, w1, row0, rows, b;
};
// A wavefront has two places for parts: 0 for one that another began, 1 for one that it began and did not end.
__device__ __forceinline__ float *part_of(const AttendArgs &a, size_t at, int64_t worker, int slot, size_t floats) {
  return reinterpret_cast<float *>(static_cast<char *>(a.workspace) + at) + size_t(2 * worker + slot) * floats;
}

// Finished values: stored past the cache (nt), where reads that fill it keep a write waiting for microseconds, and with
// it, waits being counted in order, every load behind it.
template <typename T>
__device__ __forceinline__ void store_past(char *to, T x) {
  __builtin_nontemporal_store(x, reinterpret_cast<T *>(to));
}
// kVec values of a finished row, from dimension d on.
template <int CACHE, int VEC>
__device__ __forceinline__ void store_row(char *row, int32_t d, const float (&x)[VEC]) {
  if constexpr (CACHE == DSDE_FP32)
    store_past(row + d * 4, f32x4{x[0], x[1], x[2], x[3]});
  else if constexpr (VEC == 8)
    store_past(row + d * 2, u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])});
  else
    store_past(row + d * 2, u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])});
}
// A finished row's place, its factor and its log-normaliser.
template <int CACHE>
__device__ __forceinline__ char *finished(const AttendArgs &a, int32_t row0, int32_t h, int32_t row, float m, float l, bool stats,
                                          float *factor) {
  const int32_t j = row / a.group, head = h * a.group + (row - j * a.group);
  const int64_t t = int64_t(row0) + j;
  if (stats && a.lse)
    a.lse[t * (int64_t(a.group) * a.cache.heads) + head] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2f;
  float f = l == 0.0f ? 0.0f : 1.0f / l;
  if constexpr (CACHE == DSDE_E4M3) f *= a.cache.v_scale[h];
  *factor = f;
  return a.out + t * a.out_token_stride + int64_t(head) * a.out_head_stride;
}

// A join's sums.  What is not finite among them is NaN once its factor is 0, and is then taken again (`again`, rare) by
// products in which it stays what it is, whatever part of the whole it has (NaN: none is known).  To take them like
// this always costs a join of 128 parts 0.9 us; the finite ones keep their bits.
__device__ __forceinline__ bool finite(f32x4 o) {
  const float t = fmaf(o.x, 0.0f, fmaf(o.y, 0.0f, fmaf(o.z, 0.0f, o.w * 0.0f)));
  return t == t;
}
__device__ __forceinline__ f32x4 carried(f32x4 o, float f) {
  const auto one = [f](float x) { return fabsf(x) < INFINITY || f != f ? x * f : x; };
  return f32x4{one(o.x), one(o.y), one(o.z), one(o.w)};
}
__device__ __forceinline__ f32x4 again(f32x4 o, f32x4 odd) {
  const auto one = [](float x, float y) { return fabsf(x) < INFINITY ? x : y; };
  return f32x4{one(o.x, odd.x), one(o.y, odd.y), one(o.z, odd.z), one(o.w, odd.w)};
}

// One item of a wavefront's share: tiles first .. end - 1 of a sequence, key head and row block.
struct Item {
  int32_t b, h, block, first, end;
  Seq s;
};
// A subtile's keys in memory; its values are as far from the values' start.
struct At {
  const char *keys;
  int32_t bytes;  // 0: not to be read, loads give 0 without memory
  bool bad;       // its page is none
};

template <int CACHE, int DP, int MT>
struct Wave {
  using S = Shape<CACHE, DP, MT>;
  const AttendArgs &a;
  int r, g;
  uint32_t k_off, v_off;

  // of the item at hand
  int32_t hi[MT], lo[MT];  // tokens that lane r's row of each block sees: lo .. hi
  int32_t hi_all, lo_all;  // seen by every row
  int32_t hi_any, lo_any;  // seen by any
  int32_t live;            // blocks of 16 that have rows, the first ones
  float c;                 // scale log2(e), with the keys' scale, positive
  Words<4> q[S::kRowsInLds ? 1 : MT][S::kRowsInLds ? 1 : S::kQChunks];
  Words<4> (*q_lds)[64];   // [MT * kQChunks][64]: each lane its own
  f32x4 o[MT][S::kSets][S::kVec];
  float m[MT], l[MT];
  bool odd;                // mask_values left values out that are not finite
  static constexpr int kBits = (DP + 127) / 128;  // words with a bit for each of a lane's values
  // keys and values of a tile
  Words<4> k[S::kSub][S::kChunks];
  Words<S::kVecWords> v[S::kKeys][S::kSets];

  __device__ __forceinline__ Words<4> &row(int mt, int i) {
    if constexpr (!S::kRowsInLds) return q[mt][i];
    return q_lds[mt * S::kQChunks + i][16 * g + r];
  }

  __device__ __forceinline__ Wave(const AttendArgs &args, int lane, Words<4> (*lds)[64])
      : a(args), r(lane & 15), g(lane >> 4), q_lds(lds) {
    k_off = uint32_t(r * a.cache.token_stride + 16 * g);
    v_off = uint32_t(4 * g * a.cache.token_stride + S::kVecBytes * piece(r));
  }

  // Which kVec dimensions of a set lane r loads.  Its sums come out in register r % 4 of the lanes of g = r / 4: in
  // this order the four lanes of a row hold 64 bytes in a row (bf16) in each register, and store them together.
  __device__ static __forceinline__ int piece(int r) { return 4 * (r % 4) + r / 4; }

  // Subtile t of a tile; nothing is read of those that no row sees.
  __device__ __forceinline__ At locate(const Item &x, int32_t tile, int t, bool wanted) const {
    const int32_t key = tile * S::kTile + 16 * t;
    const int64_t oldest = int64_t(x.s.context) - x.s.n - a.window + 1;  // with a window, what the first row sees
    wanted = wanted && key < x.s.context && (a.window == 0 || key + 15 >= oldest);
    const int32_t page = wanted ? constant(a.table + int64_t(x.b) * a.width)[key >> a.cache.shift] : 0;
    At y;
    y.bad = uint32_t(page) >= uint32_t(a.cache.pages);
    wanted = wanted && !y.bad;
    y.keys = a.cache.k + (wanted ? int64_t(page) * a.cache.page_stride + int64_t(x.h) * a.cache.head_stride +
                                       int64_t(key & ((1 << a.cache.shift) - 1)) * a.cache.token_stride
                                 : 0);
    y.bytes = wanted ? 15 * a.cache.token_stride + a.cache.dim * S::kElt : 0;
    return y;
  }
  __device__ __forceinline__ void load_k(const At (&at)[S::kSub]) {
#pragma unroll
    for (int t = 0; t < S::kSub; ++t) {
      const Buffer from = buffer(at[t].keys, at[t].bytes);
#pragma unroll
      for (int j = 0; j < S::kChunks; ++j)  // 0 behind the row's end
        k[t][j] = load_words<4>(from, (4 * j + g) * S::kPer16 < a.cache.dim ? k_off + 64 * j : kOutside);
    }
  }
  __device__ __forceinline__ void load_v(const At (&at)[S::kSub]) {
#pragma unroll
    for (int t = 0; t < S::kSub; ++t) {
      const Buffer from = buffer(at[t].keys + (a.cache.v - a.cache.k), at[t].bytes);
#pragma unroll
      for (int e = 0; e < S::kSets; ++e) {
        const uint32_t off = (16 * e + piece(r)) * S::kVec < a.cache.dim ? v_off + 16 * S::kVecBytes * e : kOutside;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * t + i][e] = load_words<S::kVecWords>(from, off, i * a.cache.token_stride);
      }
    }
  }
  // An item's rows: a lane's chunk of one, in memory; for rows and dimensions that are none, another one's.
  __device__ __forceinline__ const u32x4 *q_chunk(const Item &x, int mt, int i) const {
    const char *base = a.q.data + x.s.row0 * a.q.token_stride + int64_t(x.h) * a.group * a.q.head_stride;
    const int32_t row = (x.block * MT + mt) * 16 + r, at = row < x.s.n * a.group ? row : 0, j = at / a.group, d = S::q_dim(i, g);
    return reinterpret_cast<const u32x4 *>(base + j * a.q.token_stride + (at - j * a.group) * a.q.head_stride +
                                           (d < a.cache.dim ? d : 0) * S::kQElt);
  }
  __device__ __forceinline__ void load_q(const Item &x, Words<4> (&ahead)[MT][S::kQChunks]) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < S::kQChunks; ++i) ahead[mt][i] = __builtin_bit_cast(Words<4>, *q_chunk(x, mt, i));
  }
  // Takes over an item's rows, loaded or (kAhead false) from memory.  A negative scale turns their signs, one of 0 makes
  // them 0.
  __device__ __forceinline__ void take_q(const Item &x, const Words<4> (&ahead)[MT][S::kQChunks]) {
    const float f = a.scale * kLog2e * (CACHE == DSDE_E4M3 ? a.cache.k_scale[x.h] : 1.0f);
    const bool flat = fabsf(f) < 0x1p-126f;
    const uint32_t flip = f < 0.0f ? (CACHE == DSDE_FP32 ? 0x80000000u : 0x80008000u) : 0u;
    c = flat ? 1.0f : fabsf(f);
    const auto put = [&](int mt, int i, const Words<4> &y) {
      const bool there = (x.block * MT + mt) * 16 + r < x.s.n * a.group && !flat && S::q_dim(i, g) < a.cache.dim;
      Words<4> z;
#pragma unroll
      for (int e = 0; e < 4; ++e) z.w[e] = there ? y.w[e] ^ flip : 0u;
      row(mt, i) = z;
    };
    if constexpr (S::kAhead) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < S::kQChunks; ++i) put(mt, i, ahead[mt][i]);
    } else {  // eight chunks at a time
      static_assert(S::kAhead || MT * S::kQChunks % 8 == 0, "whole turns");
#pragma unroll 1
      for (int k = 0; k < MT * S::kQChunks; k += 8) {
        Words<4> y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __builtin_bit_cast(Words<4>, *q_chunk(x, (k + i) / S::kQChunks, (k + i) % S::kQChunks));
#pragma unroll
        for (int i = 0; i < 8; ++i) put((k + i) / S::kQChunks, (k + i) % S::kQChunks, y[i]);
      }
    }
  }
  // What an item's rows see, and empty accumulators.
  __device__ __forceinline__ void begin(const Item &x) {
    const int32_t newest = x.s.context - 1, oldest = x.s.context - x.s.n;
    hi_all = oldest, hi_any = newest;
    const int32_t blocks = (x.s.n * a.group + 15) / 16 - x.block * MT;
    live = blocks < MT ? blocks : MT;
    lo_all = a.window > 0 && newest >= a.window ? newest - a.window + 1 : 0;
    lo_any = a.window > 0 && oldest >= a.window ? oldest - a.window + 1 : 0;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      // the quotient of every lane, no branch around it: where lanes without a row leave one, the compiler has saved
      // other values with those lanes still off (build_lib.py, partial_copies), and a later load went astray
      const int32_t row = (x.block * MT + mt) * 16 + r;
      const bool there = row < x.s.n * a.group;
      const int32_t j = (there ? row : 0) / a.group;
      hi[mt] = there ? oldest + j : -1;
      lo[mt] = a.window > 0 && hi[mt] >= a.window ? hi[mt] - a.window + 1 : 0;
      m[mt] = -INFINITY, l[mt] = 0.0f;
#pragma unroll
      for (int e = 0; e < S::kSets; ++e)
#pragma unroll
        for (int j = 0; j < S::kVec; ++j) o[mt][e][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    odd = false;
  }

  // f for the blocks of 16 that have rows.  The fp32 instructions take eight times as long as bf16's, so that an empty
  // second block is left out: 4 to 32 rows of 64 take 371 us instead of 439, of 128 404 instead of 502 (always 32 rows: 474 and
  // 479 instead of 467 and 457).  With three or four blocks, or 16-bit products, the branches cost more than they save (3 to
  // 6 %, or spills).
  template <typename F>
  __device__ __forceinline__ void of_live(F f) const {
    if constexpr (CACHE == DSDE_FP32 && MT == 2)
      if (live == 1) return f(std::integral_constant<int, 1>{});
    f(std::integral_constant<int, MT>{});
  }
  // Scores of a tile, without their scale.
  template <int L>
  __device__ __forceinline__ void scores(f32x4 (&x)[MT][S::kSub]) {
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
            for (int mt = 0; mt < L; ++mt)
              x[mt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.w[e]), __uint_as_float(row(mt, j).w[e]), x[mt][t], 0, 0, 0);
        } else if constexpr (CACHE == DSDE_BF16) {
#pragma unroll
          for (int mt = 0; mt < L; ++mt) x[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(w), operand(row(mt, j)), x[mt][t], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const bf16x8 kk = operand(Words<4>{{widen<false>(w.w[2 * e]), widen<true>(w.w[2 * e]), widen<false>(w.w[2 * e + 1]),
                                                widen<true>(w.w[2 * e + 1])}});
#pragma unroll
            for (int mt = 0; mt < L; ++mt) x[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, operand(row(mt, 2 * j + e)), x[mt][t], 0, 0, 0);
          }
        }
      }
    }
  }

  // Raises references (in the log2 domain) where scores pass them, and turns scores into weights.
  template <int L>
  __device__ __forceinline__ void weigh(f32x4 (&x)[MT][S::kSub]) {
#pragma unroll
    for (int mt = 0; mt < L; ++mt) {
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < S::kSub; ++t) top = fmaxf(fmaxf(fmaxf(x[mt][t].x, x[mt][t].y), fmaxf(x[mt][t].z, x[mt][t].w)), top);
      top *= c;
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
        x[mt][t] = f32x4{exp2_fast(fmaf(x[mt][t].x, c, -ref)), exp2_fast(fmaf(x[mt][t].y, c, -ref)),
                         exp2_fast(fmaf(x[mt][t].z, c, -ref)), exp2_fast(fmaf(x[mt][t].w, c, -ref))};
        sum += (x[mt][t].x + x[mt][t].y) + (x[mt][t].z + x[mt][t].w);
      }
      l[mt] += sum;
    }
  }

  // Two dimensions, 2 j2 and 2 j2 + 1 of set e, of the eight keys of subtiles t and t + 1: one word of each key.
  __device__ __forceinline__ void pick(int t, int e, int j2, Words<4> &even, Words<4> &odd) const {
    uint32_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Words<S::kVecWords> &y = v[4 * t + i][e];
      if constexpr (CACHE == DSDE_BF16)
        x[i] = y.w[j2];
      else
        x[i] = j2 & 1 ? widen<true>(y.w[j2 / 2]) : widen<false>(y.w[j2 / 2]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      even.w[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);
      odd.w[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
    }
  }

  // Adds the weights' values.  For 16-bit matrix instructions a weight is the sum of two bf16 numbers, good to 2^-17: one
  // alone would be off by as much as the output's own rounding (2.2e-3 of the norm of random rows' outputs instead of
  // 1.6e-3), and the second product takes no time that memory does not (0 to 1 % with up to 48 rows, 6 % with 64).
  template <int L>
  __device__ __forceinline__ void add(const f32x4 (&p)[MT][S::kSub]) {
    if constexpr (CACHE == DSDE_FP32) {
#pragma unroll
      for (int i = 0; i < S::kKeys; ++i)
#pragma unroll
        for (int e = 0; e < S::kSets; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int mt = 0; mt < L; ++mt)
              o[mt][e][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][e].w[j]), p[mt][i / 4][i % 4], o[mt][e][j], 0, 0, 0);
    } else {
#pragma unroll
      for (int t = 0; t < S::kSub; t += 2) {
        bf16x8 w[L], rest[L];
#pragma unroll
        for (int mt = 0; mt < L; ++mt) {
          Words<4> hi, lo;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = p[mt][t + i / 2][2 * (i % 2)], y = p[mt][t + i / 2][2 * (i % 2) + 1];
            hi.w[i] = pack_bf16(x, y);
            lo.w[i] = pack_bf16(x - __uint_as_float(hi.w[i] << 16), y - __uint_as_float(hi.w[i] & 0xffff0000u));
          }
          w[mt] = operand(hi), rest[mt] = operand(lo);
        }
#pragma unroll
        for (int e = 0; e < S::kSets; ++e)
#pragma unroll
          for (int j2 = 0; j2 < S::kVec / 2; ++j2) {
            Words<4> even, odd;
            pick(t, e, j2, even, odd);
#pragma unroll
            for (int mt = 0; mt < L; ++mt) {
              const auto both = [&](const Words<4> &v, f32x4 to) {
                to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(v), w[mt], to, 0, 0, 0);
                return __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(v), rest[mt], to, 0, 0, 0);
              };
              o[mt][e][2 * j2] = both(even, o[mt][e][2 * j2]);
              o[mt][e][2 * j2 + 1] = both(odd, o[mt][e][2 * j2 + 1]);
            }
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
        for (int mt = 0; mt < MT; ++mt) x[mt][t][i] = key >= lo[mt] && key <= hi[mt] ? x[mt][t][i] : -INFINITY;
      }
  }
  // Scores of a bad page: NaN where mask has left any, to rows that see them.  Apart from mask, where a factor for every
  // score kept registers that the loop needs (256 sequences of 32 rows of 256 542 us, of 64 over e4m3 464; behind a branch of
  // their own 517 and 425).
  __device__ __forceinline__ void spoil(f32x4 (&x)[MT][S::kSub], const At (&at)[S::kSub]) {
#pragma unroll
    for (int t = 0; t < S::kSub; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) x[mt][t][i] = at[t].bad && x[mt][t][i] != -INFINITY ? NAN : x[mt][t][i];
  }
  // The same for values, as a weight of 0 takes no part only beside finite ones.  Values that no row sees become 0;
  // others that are not finite (rare) too, for find_odd.
  __device__ __forceinline__ void mask_values(int32_t tile) {
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < S::kKeys; ++i) {
      const int32_t key = tile * S::kTile + 16 * (i / 4) + 4 * g + i % 4;
      const bool seen = key >= lo_any && key <= hi_any;
#pragma unroll
      for (int e = 0; e < S::kSets; ++e)
#pragma unroll
        for (int w = 0; w < S::kVecWords; ++w) {
          v[i][e].w[w] = seen ? v[i][e].w[w] : 0;
          any |= not_finite<CACHE>(v[i][e].w[w]);
        }
    }
    if (__any(any != 0)) {
      odd = true;
#pragma unroll
      for (int i = 0; i < S::kKeys; ++i)
#pragma unroll
        for (int e = 0; e < S::kSets; ++e)
#pragma unroll
          for (int w = 0; w < S::kVecWords; ++w) v[i][e].w[w] = finite_only<CACHE>(v[i][e].w[w]);
    }
  }
  // Whether some row may see a value that is not finite: one was left out, or reached an accumulator (which is inf
  // or NaN ever after, whatever it is multiplied by or added to).
  __device__ __forceinline__ bool maybe_odd() const {
    f32x4 t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < S::kSets; ++e)
#pragma unroll
        for (int j = 0; j < S::kVec; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) t[i] = fmaf(o[mt][e][j][i], 0.0f, t[i]);
    const float u = (t.x + t.y) + (t.z + t.w);
    return __any(odd || u != u);
  }
  __device__ static constexpr int bit(int e, int j, int i) { return (e * S::kVec + j) * 4 + i; }
  // Which of a lane's values have +inf (bits[0]), and which -inf (bits[1]) among what their row sees of the item, NaN as
  // both: a sum with one of them is it, whatever the weights (NaN with both).  The accumulators cannot tell: the sum of two
  // bf16 numbers that a weight is makes inf NaN where the second is not positive, as do weights and factors that underflow
  // to 0.  So the values are read once more, and what each row sees of either kind is counted: a product of ones and zeros
  // (256 sequences of 256 to 8,192 tokens, up to 36 rows: an infinity in each 610 us, in one 541, in none 428 to 455).
  __device__ __forceinline__ void find_odd(const Item &x, uint32_t (&bits)[2][MT][kBits]) {
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < kBits; ++i) bits[kind][mt][i] = 0;
#pragma unroll 1
    for (int32_t tile = x.first; tile < x.end; ++tile) {
      At at[S::kSub];
#pragma unroll
      for (int t = 0; t < S::kSub; ++t) at[t] = locate(x, tile, t, true);
      load_v(at);
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < S::kKeys; ++i)
#pragma unroll
        for (int e = 0; e < S::kSets; ++e)
#pragma unroll
          for (int w = 0; w < S::kVecWords; ++w) any |= not_finite<CACHE>(v[i][e].w[w]);
      if (__any(any != 0)) count_odd(tile, bits);
    }
  }
  __device__ __forceinline__ void count_odd(int32_t tile, uint32_t (&bits)[2][MT][kBits]) {
    const auto sees = [&](int mt, int t, int i) {
      const int32_t key = tile * S::kTile + 16 * t + 4 * g + i;
      return key >= lo[mt] && key <= hi[mt];
    };
#pragma unroll 1
    for (int kind = 0; kind < 2; ++kind) {
      // nothing is to be worked out before the loop and kept: registers are scarce
#pragma unroll
      for (int i = 0; i < S::kKeys; ++i)
#pragma unroll
        for (int e = 0; e < S::kSets; ++e)
#pragma unroll
          for (int w = 0; w < S::kVecWords; ++w) asm volatile("" : "+v"(v[i][e].w[w]));
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) asm volatile("" : "+v"(lo[mt]), "+v"(hi[mt]));
      const auto put = [&](int mt, int e, int j, f32x4 count) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t one = count[i] > 0.0f ? 1u << bit(e, j, i) % 32 : 0u;
          bits[0][mt][bit(e, j, i) / 32] |= kind == 0 ? one : 0u;
          bits[1][mt][bit(e, j, i) / 32] |= kind == 1 ? one : 0u;
        }
      };
      if constexpr (CACHE == DSDE_FP32) {
#pragma unroll
        for (int e = 0; e < S::kSets; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              f32x4 count{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
              for (int i = 0; i < S::kKeys; ++i) {
                const float y = __uint_as_float(v[i][e].w[j]);
                const bool is = y != y || y == (kind == 0 ? INFINITY : -INFINITY);
                count = __builtin_amdgcn_mfma_f32_16x16x4f32(is ? 1.0f : 0.0f, sees(mt, i / 4, i % 4) ? 1.0f : 0.0f, count, 0, 0, 0);
              }
              put(mt, e, j, count);
            }
      } else {
        // halves of a word that are of the kind, as ones
        const auto ones = [&](Words<4> x) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const auto one = [&](uint32_t h) {
              return (h & 0x7fffu) > 0x7f80u || h == (kind == 0 ? 0x7f80u : 0xff80u) ? 0x3f80u : 0u;
            };
            x.w[i] = one(x.w[i] & 0xffffu) | one(x.w[i] >> 16) << 16;
          }
          return x;
        };
#pragma unroll
        for (int t = 0; t < S::kSub; t += 2) {
          bf16x8 seen[MT];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            Words<4> x;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              x.w[i] = (sees(mt, t + i / 2, 2 * (i % 2)) ? 0x3f80u : 0u) | (sees(mt, t + i / 2, 2 * (i % 2) + 1) ? 0x3f800000u : 0u);
            seen[mt] = operand(x);
          }
#pragma unroll
          for (int e = 0; e < S::kSets; ++e)
#pragma unroll
            for (int j2 = 0; j2 < S::kVec / 2; ++j2) {
              Words<4> even, odd;
              pick(t, e, j2, even, odd);
              even = ones(even), odd = ones(odd);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                const f32x4 none{0.0f, 0.0f, 0.0f, 0.0f};
                put(mt, e, 2 * j2, __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(even), seen[mt], none, 0, 0, 0));
                put(mt, e, 2 * j2 + 1, __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(odd), seen[mt], none, 0, 0, 0));
              }
            }
        }
      }
    }
  }

  // The item's rows, or its part of them.
  __device__ __forceinline__ void end(const Item &x, float *part) {
    constexpr int kRows = 16 * MT;
    const bool done = x.end - x.first == x.s.tiles;
    uint32_t bits[2][MT][kBits];
    const bool some = maybe_odd();
    if (some) find_odd(x, bits);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int32_t row = x.block * kRows + 16 * mt + r;
      float sum = l[mt];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (x.s.err) sum = NAN;  // a context that is none
      if (row < x.s.n * a.group) {
        float f = 1.0f;
        char *to = nullptr;
        if (done) to = finished<CACHE>(a, x.s.row0, x.h, row, m[mt], sum, g == 0, &f);
#pragma unroll
        for (int e = 0; e < S::kSets; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int32_t d = (16 * e + piece(4 * g + i)) * S::kVec;
            float y[S::kVec];
#pragma unroll
            for (int j = 0; j < S::kVec; ++j) y[j] = o[mt][e][j][i] * f;
            if (some) {
#pragma unroll
              for (int j = 0; j < S::kVec; ++j) {
                const int w = bit(e, j, i) / 32, at = bit(e, j, i) % 32;
                const bool plus = bits[0][mt][w] >> at & 1, minus = bits[1][mt][w] >> at & 1;
                if (plus || minus) y[j] = sum != sum || (plus && minus) ? NAN : plus ? INFINITY : -INFINITY;
              }
            }
            if (done) {
              if (d < a.cache.dim) store_row<CACHE, S::kVec>(to, d, y);
            } else {
#pragma unroll
              for (int j = 0; j < S::kVec; j += 4)
                *reinterpret_cast<f32x4 *>(part + (16 * mt + r) * DP + d + j) = f32x4{y[j], y[j + 1], y[j + 2], y[j + 3]};
            }
          }
        if (!done && g == 0) {
          part[kRows * DP + 16 * mt + r] = m[mt];
          part[kRows * (DP + 1) + 16 * mt + r] = sum;
        }
      }
    }
  }
};

// Quotients of the work's line, in 32 bits where it is that short (64 take ten times the instructions).
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y, bool small) {
  return small ? int64_t(uint32_t(x) / uint32_t(y)) : x / y;
}

template <int CACHE, int DP, int MT>
__global__ __launch_bounds__(kAttendThreads, 1) void attend_kernel(AttendArgs a, AttendLayout at) {
  using S = Shape<CACHE, DP, MT>;
  constexpr int kRows = 16 * MT;
  constexpr size_t kPart = kRows * (DP + 2);
  struct Begin {
    Start at;
    int32_t used;  // units of its item's start that lie before the share
    Seq s;
  };
  __shared__ int64_t s_sum[kAttendWaves];
  __shared__ Begin s_begin[kAttendWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);

  // where each wavefront's share begins; neighbours in the line are in different workgroups, so that few shares
  // spread over many CUs
  const int32_t per = (a.B + kAttendThreads - 1) / kAttendThreads;
  const int32_t b0 = tid * per < a.B ? tid * per : a.B, b1 = b0 + per < a.B ? b0 + per : a.B;
  int64_t own = 0;
  Seq mine;  // a thread's last sequence, its only one in batches up to 256
  for (int32_t b = b0; b < b1; ++b) {
    mine = sequence<S::kTile>(a, b, kRows);
    own += units_of(a, mine);
  }
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
  const int32_t workers = int32_t(gridDim.x) * kAttendWaves;
  const bool small = all + workers < (int64_t(1) << 31);
  int64_t share = quotient(all + workers - 1, workers, small);
  if (share < kLeast) share = kLeast;
  for (int i = 0; i < kAttendWaves; ++i) {
    const int64_t begin = (int64_t(i) * gridDim.x + blockIdx.x) * share;
    int64_t before = upto - own;
    if (begin < before || begin >= upto) continue;
    for (int32_t b = b0; b < b1; ++b) {
      const Seq s = per == 1 ? mine : sequence<S::kTile>(a, b, kRows);
      const int64_t n = units_of(a, s);
      if (begin < before + n) {
        const int64_t x = begin - before;
        const int32_t size = s.tiles + kStart, item = int32_t(quotient(x, size, small)), u = int32_t(x - int64_t(item) * size);
        const int64_t unit = before + int64_t(item) * size + kStart;  // of the item's first tile
        const int32_t h = item / s.blocks;
        s_begin[i] = Begin{Start{h, item - h * s.blocks, u > kStart ? u - kStart : 0, int32_t(quotient(unit, share, small)),
                                 int32_t(quotient(unit + s.tiles - 1, share, small)), s.row0, s.n * a.group, b}, u < kStart ? u : kStart, s};
        break;
      }
      before += n;
    }
  }
  __syncthreads();
  const int64_t worker = int64_t(wave) * gridDim.x + blockIdx.x;
  const int64_t begin = worker * share, end = begin + share < all ? begin + share : all;
  Start *starts = reinterpret_cast<Start *>(static_cast<char *>(a.workspace) + at.starts);
  if (begin >= end) {
    if (lane == 0) starts[worker].tile = 0;
    return;
  }
  const Begin &from = s_begin[wave];
  if (lane == 0) starts[worker] = from.at;
  int64_t left = end - begin - (kStart - uniform(from.used));
  if (left <= 0) return;  // the end of an item's start alone

  Item x{uniform(from.at.b), uniform(from.at.h), uniform(from.at.block), 0, 0,
         Seq{uniform(from.s.row0), uniform(from.s.n), uniform(from.s.context), uniform(from.s.tile0), uniform(from.s.tiles),
             uniform(from.s.blocks), uint32_t(uniform(int(from.s.err)))}};
  int32_t tile = uniform(from.at.tile);  // of the sequence's tiles; above 0 in the first item alone
  const auto take = [&](Item &y, int32_t tile) {
    y.first = y.s.tile0 + tile;
    y.end = y.first + int32_t(left < y.s.tiles - tile ? left : y.s.tiles - tile);
    left -= y.end - y.first + kStart;
  };
  take(x, tile);

  constexpr int kLds = S::kRowsInLds ? MT * S::kQChunks : 1;
  __shared__ Words<4> s_q[S::kRowsInLds ? kAttendWaves : 1][kLds][64];
  Wave<CACHE, DP, MT> w(a, lane, s_q[S::kRowsInLds ? wave : 0]);
  At now[S::kSub], next[S::kSub];
  Words<4> ahead[MT][S::kQChunks];
  if (S::kAhead) w.load_q(x, ahead);
#pragma unroll
  for (int t = 0; t < S::kSub; ++t) now[t] = w.locate(x, x.first, t, true);
  w.load_k(now);
  w.take_q(x, ahead);
  for (;;) {
    // what comes behind this item
    Item y = x;
    bool more = left > 0;
    if (more && ++y.block == y.s.blocks) {
      y.block = 0;
      if (++y.h == a.cache.heads) {
        y.h = 0;
        do {
          if (++y.b >= a.B) {
            more = false;
            break;
          }
          y.s = sequence<S::kTile>(a, y.b, kRows);
        } while (y.s.blocks == 0);
      }
    }
    if (more)
      take(y, 0);
    else
      y = x;
    w.begin(x);
    if (S::kAhead) w.load_q(y, ahead);
    // A tile's values are on their way while its scores are taken, and the next tile's keys while its values are
    // weighed, into registers that have just been read; behind an item's last tile come the next item's first keys.
    // No load stands behind a branch, and a loop has a tile at least: waits could not be counted otherwise.  A tile
    // behind the last of all is none.
    int32_t tile = x.first;
    do {
      if (S::kRowsInLds) asm volatile("" : : : "memory");  // rows are read from LDS for every tile, not kept
      w.load_v(now);
      const bool last = tile + 1 == x.end;
#pragma unroll
      for (int t = 0; t < S::kSub; ++t) next[t] = w.locate(last ? y : x, last ? y.first : tile + 1, t, !last || more);
      f32x4 p[MT][S::kSub];
      w.of_live([&](auto n) { w.template scores<n.value>(p); });
      w.load_k(next);
      bool bad = false;
#pragma unroll
      for (int t = 0; t < S::kSub; ++t) bad |= now[t].bad;
      const bool clear = !bad && tile * S::kTile >= w.lo_all && tile * S::kTile + S::kTile - 1 <= w.hi_all;
      if (!clear) w.mask(p, tile);
      if (bad) w.spoil(p, now);
      w.of_live([&](auto n) { w.template weigh<n.value>(p); });
      if (!clear) w.mask_values(tile);
      w.of_live([&](auto n) { w.template add<n.value>(p); });
#pragma unroll
      for (int t = 0; t < S::kSub; ++t) now[t] = next[t];
    } while (++tile < x.end);
    w.take_q(y, ahead);  // before the stores, which its wait would count
    w.end(x, part_of(a, at.parts, worker, x.first > x.s.tile0 ? 0 : 1, kPart));
    if (!more) return;
    x = y;
  }
}

// Joins the parts of items that more than one wavefront had.  A workgroup for each wavefront whose share begins
// inside an item; those of one item divide its values among them, and a value's parts among lanes.  The workgroups
// behind them check the sequences.
template <int CACHE, int DP, int MT>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a, AttendLayout at, int32_t workers) {
  using S = Shape<CACHE, DP, MT>;
  constexpr int kRows = 16 * MT;
  constexpr size_t kPart = kRows * (DP + 2);
  const int tid = threadIdx.x;
  if (int32_t(blockIdx.x) >= workers) {
    __shared__ int s_bad;
    for (int32_t b = int32_t(blockIdx.x) - workers; b < a.B; b += int32_t(gridDim.x) - workers) {
      const Seq s = sequence<S::kTile>(a, b, kRows);
      __syncthreads();
      if (tid == 0) s_bad = 0;
      __syncthreads();
      if (s.n > 0 && s.context > 0) {
        const int64_t first = a.window > 0 ? int64_t(s.context) - s.n - a.window + 1 : 0;
        bool bad = false;
        // eight loads at once: one workgroup has all pages of a sequence (8,192 of them: the whole kernel 7.4 us instead of 9.6)
        const int32_t last = (s.context - 1) >> a.cache.shift;
        for (int32_t i = int32_t((first > 0 ? first : 0) >> a.cache.shift) + tid; i <= last; i += 256 * 8) {
          int32_t id[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) id[k] = a.table[int64_t(b) * a.width + (i + 256 * k < last ? i + 256 * k : last)];
#pragma unroll
          for (int k = 0; k < 8; ++k) bad |= uint32_t(id[k]) >= uint32_t(a.cache.pages);
        }
        if (bad) s_bad = 1;
      }
      __syncthreads();
      if (tid == 0) a.seq_err[b] = s.err | (s_bad ? DSDE_ERR_PAGES : 0u);
    }
    return;
  }
  const int32_t worker = blockIdx.x;
  const Start x = reinterpret_cast<const Start *>(static_cast<const char *>(a.workspace) + at.starts)[worker];
  if (x.tile == 0) return;
  const int32_t row0 = x.block * kRows, live = x.rows - row0 < kRows ? x.rows - row0 : kRows;
  // cells of four values, at least 4 (64 bytes) for each workgroup: the fewer they are, the more lanes share a cell's parts
  // and the fewer loads come one after another (128 parts of 8 items: 9.5 us, with 16 cells 12)
  const int32_t cells = live * (DP / 4), parts = x.w1 - x.w0 + 1, sharers = parts - 1;
  if (parts == 2) {  // most often: all loads at once
    constexpr int kTimes = (kRows * DP / 4 + 255) / 256;
    const float *p0 = part_of(a, at.parts, x.w0, 1, kPart), *p1 = part_of(a, at.parts, x.w1, 0, kPart);
    float m0[kTimes], m1[kTimes], l0[kTimes], l1[kTimes];
    f32x4 o0[kTimes], o1[kTimes];
#pragma unroll
    for (int k = 0; k < kTimes; ++k) {
      const int32_t c = tid + 256 * k < cells ? tid + 256 * k : 0, i = c / (DP / 4), d = c % (DP / 4) * 4;
      m0[k] = p0[kRows * DP + i], m1[k] = p1[kRows * DP + i];
      l0[k] = p0[kRows * (DP + 1) + i], l1[k] = p1[kRows * (DP + 1) + i];
      o0[k] = *reinterpret_cast<const f32x4 *>(p0 + i * DP + d), o1[k] = *reinterpret_cast<const f32x4 *>(p1 + i * DP + d);
    }
#pragma unroll
    for (int k = 0; k < kTimes; ++k) {
      const int32_t c = tid + 256 * k, i = c / (DP / 4), d = c % (DP / 4) * 4;
      if (c >= cells) break;
      const float m = fmaxf(m0[k], m1[k]), ref = m == -INFINITY ? 0.0f : m;
      const float f0 = exp2_fast(m0[k] - ref), f1 = exp2_fast(m1[k] - ref);
      float f;
      char *to = finished<CACHE>(a, x.row0, x.h, row0 + i, m, l0[k] * f0 + l1[k] * f1, d == 0, &f);
      f32x4 o = (o0[k] * f0 + o1[k] * f1) * f;
      if (!finite(o)) o = again(o, carried(carried(o0[k], f0) + carried(o1[k], f1), f));
      const float y[4] = {o.x, o.y, o.z, o.w};
      if (d < a.cache.dim) store_row<CACHE, 4>(to, d, y);
    }
    return;
  }
  int32_t n = (cells + sharers - 1) / sharers;
  n = n < 4 ? 4 : n;
  const int32_t c0 = (worker - x.w0 - 1) * n, c1 = c0 + n < cells ? c0 + n : cells;
  // lanes that share a cell's parts
  int32_t span = 1;
  while (span < 64 && span < parts && span * 2 * n <= 256) span *= 2;
  const int32_t groups = 256 / span, lane = tid % span;
  for (int32_t c = c0 + tid / span; c - tid / span < c1; c += groups) {  // all lanes stay for the shuffles
    const bool mine = c < c1;
    const int32_t i = (mine ? c : c0 < cells ? c0 : 0) / (DP / 4), d = (mine ? c : 0) % (DP / 4) * 4;
    const auto total = [&](auto odd, float &m, float &l) {
      m = -INFINITY, l = 0.0f;
      f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
      const auto with = [&](float pm, float pl, f32x4 po) {
        const float now = fmaxf(m, pm), ref = now == -INFINITY ? 0.0f : now;
        const float f0 = exp2_fast(m - ref), f1 = exp2_fast(pm - ref);
        m = now;
        l = l * f0 + pl * f1;
        if constexpr (odd.value)
          o = carried(o, f0) + carried(po, f1);
        else
          o = o * f0 + po * f1;
      };
#pragma unroll 4
      for (int32_t k = lane; k < parts; k += span) {
        const float *p = part_of(a, at.parts, x.w0 + k, k == 0 ? 1 : 0, kPart);
        with(p[kRows * DP + i], p[kRows * (DP + 1) + i], *reinterpret_cast<const f32x4 *>(p + i * DP + d));
      }
      for (int32_t step = 1; step < span; step *= 2) {
        const float pm = __shfl_xor(m, step), pl = __shfl_xor(l, step);
        with(pm, pl, f32x4{__shfl_xor(o.x, step), __shfl_xor(o.y, step), __shfl_xor(o.z, step), __shfl_xor(o.w, step)});
      }
      return o;
    };
    float m, l, m2, l2;
    f32x4 o = total(std::false_type{}, m, l), odd = o;
    if (__any(!finite(o))) odd = total(std::true_type{}, m2, l2);
    if (mine && lane == 0) {
      float f;
      char *to = finished<CACHE>(a, x.row0, x.h, row0 + i, m, l, d == 0, &f);
      o = again(o * f, carried(odd, f));
      const float y[4] = {o.x, o.y, o.z, o.w};
      if (d < a.cache.dim) store_row<CACHE, 4>(to, d, y);
    }
  }
}

// One workgroup per CU, a wavefront per SIMD: 64 KiB of loads in flight on each CU.  With two workgroups the same
// 2.1 GB took 340 us instead of 330, with three 373.
template <int CACHE, int DP, int MT>
void launch(const AttendArgs &a, hipStream_t stream) {
  const AttendLayout at = attend_layout(a.cache.dim, int64_t(a.group) * a.max_rows);
  constexpr int32_t groups = 256, workers = groups * kAttendWaves;
  static_assert(workers <= kAttendWorkers && 16 * MT <= kAttendRows, "workspace");
  attend_kernel<CACHE, DP, MT><<<groups, kAttendThreads, 0, stream>>>(a, at);
  join_kernel<CACHE, DP, MT><<<workers + (a.B < 1024 ? a.B : 1024), 256, 0, stream>>>(a, at, workers);
}
template <int CACHE, int DP>
void by_tiles(const AttendArgs &a, hipStream_t stream) {
  // as many row blocks as fit the registers, and no more than the rows fill (the workspace has room for those)
  constexpr int most = DP == 256 ? (CACHE == DSDE_FP32 ? 1 : 2) : CACHE == DSDE_FP32 && DP == 128 ? 2 : 4;
  const int32_t rows = a.group * a.max_rows;
  if (rows <= 16 || most == 1)
    launch<CACHE, DP, 1>(a, stream);
  else if (rows <= 32 || most == 2)
    launch<CACHE, DP, most < 2 ? 1 : 2>(a, stream);
  else if (rows <= 48)
    launch<CACHE, DP, most < 4 ? 1 : 3>(a, stream);
  else
    launch<CACHE, DP, most < 4 ? 1 : 4>(a, stream);
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
