// Pages and slots of a ragged step's rows, and their keys and values into the cache.
//
// The map is integer arithmetic on a few numbers per sequence: three prefix sums
// (rows, pages given back, pages taken) decide where each sequence's rows and pages lie, so any
// number of threads can move pages at once and the result is the one of a loop over the
// sequences.  It is bound by dependent round trips to memory, not by bytes (0.1 MB for 1,024 sequences).
#include "kv.hpp"

namespace dsde {
namespace {

constexpr int kMapThreads = 1024, kMapWaves = kMapThreads / 64;
constexpr int kSmallSeqs = 1024;     // sequences whose prefix sums stay in LDS
constexpr int64_t kSmallRows = 6144;  // rows that the planning workgroup maps itself
constexpr int32_t kManyPages = 4096;  // more pages than it gives back itself where it can leave them

struct Sums {
  int64_t rows, taken, back;
  __device__ Sums operator+(const Sums &o) const { return Sums{rows + o.rows, taken + o.taken, back + o.back}; }
};
__device__ __forceinline__ Sums shift_up(const Sums &s, int n) {
  return Sums{__shfl_up(s.rows, n), __shfl_up(s.taken, n), __shfl_up(s.back, n)};
}
// Inclusive sums over the workgroup's threads, and their total.
__device__ Sums block_scan(Sums s, Sums *total) {
  __shared__ Sums wave[kMapWaves];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int n = 1; n < 64; n <<= 1) {
    const Sums o = shift_up(s, n);
    if (lane >= n) s = s + o;
  }
  __syncthreads();  // the last call's sums have been read
  if (lane == 63) wave[w] = s;
  __syncthreads();
  Sums all{0, 0, 0};
  for (int i = 0; i < kMapWaves; ++i) {
    if (i == w) s = s + all;
    all = all + wave[i];
  }
  *total = all;
  return s;
}

// Prefix sums as they are kept: sums that reach 2^31 are beyond any page or row there is.
__device__ __forceinline__ int32_t kept(int64_t x) { return int32_t(x < 0x7fffffff ? x : 0x7fffffff); }

// One sequence's share of the call.
struct Want {
  int64_t n, base;
  int32_t from, to;  // pages held before and wanted after
  uint32_t err;
};
__device__ __forceinline__ Want wanted(const MapArgs &a, int32_t b) {
  Want x;
  // a sequence without rows in the last step has none to keep; last_err may be seq_err, of which a thread reads what
  // it writes later
  const int64_t len = a.kv_len[b], acc = a.accepted && !(a.last_err && a.last_err[b]) ? a.accepted[b] : -1;
  x.n = int64_t(a.sl[b]) + a.extra;
  x.base = len + acc + 1;
  x.from = a.held[b];
  x.err = 0;
  if (x.n < 0 || len < 0 || acc < -1) x.err |= DSDE_ERR_LAYOUT;
  if (len < 0 || acc < -1) x.base = len;  // as it was
  if (x.n < 0) x.n = 0;
  if (x.from < 0 || x.from > a.width) x.err |= DSDE_ERR_STATE;
  x.to = x.from;
  if (!x.err) {
    const int64_t need = (x.base + x.n + (int64_t(1) << a.shift) - 1) >> a.shift;
    if (need > a.width)
      x.err |= DSDE_ERR_PAGES;
    else
      x.to = int32_t(need);
  }
  return x;
}
// Pages that a sequence takes and gives back; none where its rows do not fit.
__device__ __forceinline__ Sums moved(const Want &x, bool fits) {
  const bool ok = !x.err && fits;
  return Sums{x.n, ok && x.to > x.from ? x.to - x.from : 0, ok && x.to < x.from ? x.from - x.to : 0};
}

// The sequence whose range of the prefix sums pre [B+1] holds i: pre[0] <= i < pre[B].
__device__ __forceinline__ int32_t find(const int32_t *pre, int32_t B, int32_t i) {
  int32_t lo = 0, hi = B;  // pre[lo] <= i < pre[hi]
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (pre[mid] <= i)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// What the second half of the plan needs of every sequence: in LDS for batches up to kSmallSeqs.
struct Plan {
  const int32_t *cu, *taken, *from, *base, *context;
};
// A row's slot: its page is in the table or, taken in this call, on the stack.
__device__ __forceinline__ void map_row(const MapArgs &a, const Plan &p, int32_t top, int64_t t) {
  int32_t slot = -1, pos = -1;
  if (t < p.cu[a.B]) {
    const int32_t b = find(p.cu, a.B, int32_t(t));
    if (p.context[b] > 0) {  // a sequence with rows that is not flagged
      pos = p.base[b] + (int32_t(t) - p.cu[b]);
      const int32_t c = pos >> a.shift, grown = c - p.from[b];
      const int32_t page = grown >= 0 ? a.stack[top - 1 - (p.taken[b] + grown)] : a.table[int64_t(b) * a.width + c];
      if (page >= 0 && page < a.pages)
        slot = (page << a.shift) | (pos & ((1 << a.shift) - 1));
      else
        a.seq_err[b] = DSDE_ERR_PAGES;  // every thread that comes here stores the same
    }
  }
  a.slots[t] = slot;
  a.positions[t] = pos;
}
// The i-th page taken, of those that there are.
__device__ __forceinline__ void take_page(const MapArgs &a, const Plan &p, int32_t top, int32_t i) {
  const int32_t b = find(p.taken, a.B, i);
  // not of a sequence that went without
  if (p.context[b] > 0) a.table[int64_t(b) * a.width + p.from[b] + (i - p.taken[b])] = a.stack[top - 1 - i];
}
// The i-th page of F given back onto a stack of `have`; those of the sequences behind come first.
__device__ __forceinline__ void give_page(const MapArgs &a, const int32_t *back, const int32_t *from, int32_t have, int32_t F,
                                          int32_t i) {
  const int32_t b = find(back, a.B, i);
  int32_t *entry = a.table + int64_t(b) * a.width + from[b] - (back[b + 1] - i);  // ascending pages, descending places
  a.stack[have + (F - 1 - i)] = *entry;
  *entry = -1;
}

// The plan, by one workgroup: a chain of round trips to memory (the sequences' numbers, the pages that move, the pages
// of the rows) and prefix sums between them.  ALL: it also takes the pages and maps the rows, which saves a launch
// where they are few (512 rows: 6.1 us instead of 8.9, 4,096 of 1,024 sequences 10.1 instead of 10.8, and where many take a
// page 1.5 less); more take one CU longer (8,192: 14.4 instead of 10.5, with pages 2 more; the two meet at 4,600 and 7,000).  LOCAL: one sequence to a thread, kept in
// registers and LDS.  SHARED: give_kernel runs behind it (37,000 pages took this workgroup 31 us).
template <bool ALL, bool LOCAL, bool SHARED>
__global__ __launch_bounds__(kMapThreads) void map_plan_kernel(MapArgs a) {
  constexpr int kHeld = LOCAL ? kSmallSeqs : 1;
  __shared__ int32_t s_cu[kHeld + 1], s_taken[kHeld + 1], s_back[kHeld + 1], s_from[kHeld], s_base[kHeld], s_context[kHeld];
  const int32_t have = a.n_free[0];
  int32_t *cu = LOCAL ? s_cu : a.cu_rows, *taken = LOCAL ? s_taken : a.taken, *back = LOCAL ? s_back : a.back;
  // rows as they are packed, and what moves for sequences whose rows fit
  Sums before{0, 0, 0}, total;
  Want x{0, 0, 0, 0, 0};
  Sums own{0, 0, 0};
  for (int32_t b0 = 0; b0 < a.B; b0 += kMapThreads) {
    const int32_t b = b0 + threadIdx.x;
    x = Want{0, 0, 0, 0, 0};
    if (b < a.B) x = wanted(a, b);
    own = moved(x, true);
    Sums end = block_scan(own, &total);
    if (before.rows + total.rows > a.rows) {  // some do not fit: once more, without what they move
      own = moved(x, before.rows + end.rows <= a.rows);
      end = block_scan(own, &total);
    }
    if (b < a.B) {
      const Sums last = before + end;
      const auto store = [&](int32_t i, int64_t r, int64_t t, int64_t g) {
        a.cu_rows[i] = kept(r);
        cu[i] = kept(r), taken[i] = kept(t), back[i] = kept(g);
        if (LOCAL && !ALL) a.taken[i] = kept(t);
        if (LOCAL && SHARED) a.back[i] = kept(g);
      };
      store(b, last.rows - x.n, last.taken - own.taken, last.back - own.back);
      if (b == a.B - 1) store(a.B, last.rows, last.taken, last.back);
      if (LOCAL) s_from[b] = x.from;
      if (!LOCAL || !ALL || SHARED) a.from[b] = x.from;
    }
    before = before + total;
  }
  __syncthreads();
  const bool sound = have >= 0 && have <= a.pages && before.back <= a.pages - have;
  const int32_t F = sound ? int32_t(before.back) : 0, top = sound ? have + F : 0;
  const int32_t *from = LOCAL ? s_from : a.from;
  // many pages given back by a call that takes none are left to the whole card
  const bool leave = SHARED && before.taken == 0 && F > kManyPages;
  if (!leave)
    for (int32_t i = threadIdx.x; i < F; i += kMapThreads) give_page(a, back, from, have, F, i);
  // every sequence's outcome
  int32_t used = 0;
  for (int32_t b0 = 0; b0 < a.B; b0 += kMapThreads) {
    const int32_t b = b0 + threadIdx.x;
    if (b >= a.B) break;
    if (!LOCAL) x = wanted(a, b);
    const bool fits = int64_t(cu[b]) + x.n <= a.rows;
    if (!LOCAL) own = moved(x, fits);
    if (!fits) x.err |= DSDE_ERR_LAYOUT;
    if (own.taken + own.back > 0 && !sound) x.err |= DSDE_ERR_STATE;
    if (own.taken > 0 && sound && taken[b + 1] > top) x.err |= DSDE_ERR_PAGES;
    if (!x.err) {
      if (own.taken > 0) used = taken[b + 1];
      if (x.to != x.from) a.held[b] = x.to;
    }
    const int32_t base = kept(x.base), context = x.err ? 0 : int32_t(x.base + x.n);
    a.base[b] = base;
    a.context[b] = context;
    a.seq_err[b] = x.err;
    if (LOCAL) s_base[b] = base, s_context[b] = context;
  }
  __shared__ int32_t s_used;
  if (threadIdx.x == 0) s_used = 0;
  __syncthreads();
  if (used > 0) atomicMax(&s_used, used);
  __syncthreads();
  if (threadIdx.x == 0) {
    if (sound) a.n_free[0] = top - s_used;
    a.top[0] = top;
    a.top[1] = leave ? F : 0;
  }
  if (!ALL) return;
  const Plan p{cu, taken, from, LOCAL ? s_base : a.base, LOCAL ? s_context : a.context};
  const int32_t n = s_used;
  for (int32_t i = threadIdx.x; i < n; i += kMapThreads) take_page(a, p, top, i);
  for (int64_t t = threadIdx.x; t < a.rows; t += kMapThreads) map_row(a, p, top, t);
}

// Pages taken and rows mapped by the whole card.
__global__ __launch_bounds__(256) void map_rows_kernel(MapArgs a) {
  const int64_t stride = int64_t(gridDim.x) * 256, at = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const Plan p{a.cu_rows, a.taken, a.from, a.base, a.context};
  const int32_t top = a.top[0], n = top > 0 ? top - a.n_free[0] : 0;
  for (int64_t i = at; i < n; i += stride) take_page(a, p, top, int32_t(i));
  for (int64_t t = at; t < a.rows; t += stride) map_row(a, p, top, t);
}
// Pages given back that the plan left.
__global__ __launch_bounds__(256) void give_kernel(MapArgs a) {
  const int32_t F = a.top[1];
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < F; i += int64_t(gridDim.x) * 256)
    give_page(a, a.back, a.from, a.top[0] - F, F, int32_t(i));
}

// Rows into slots, a wavefront per row of keys or values: 16 bytes of the cache per lane.  Bound by HBM: 81,000 rows of
// 4 KiB take 140 to 148 us, 4.5 to 4.75 TB/s, the rate of a large copy.  PAST: stores past the L2s (nt), 2 to 7 % faster
// for more than twice what those hold (32 MiB); fewer rows are read sooner than they would leave them (a reader of
// 17 MiB right behind took 10 us longer).
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
__device__ __forceinline__ u32x4 load16(const char *from) { return *reinterpret_cast<const u32x4 *>(from); }
// Four numbers over their scale, in 8 bits.
__device__ __forceinline__ uint32_t narrow(uint32_t lo, uint32_t hi, float scale) {
  float f[4] = {__uint_as_float(lo << 16), __uint_as_float(lo & 0xffff0000u), __uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u)};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float y = f[i] / scale;
    f[i] = y != y ? y : fminf(fmaxf(y, -448.0f), 448.0f);  // the conversion alone would make what is larger NaN
  }
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false), true));
}
template <bool E4M3, bool PAST>
__global__ __launch_bounds__(256) void kv_write_kernel(KvWriteArgs a, int64_t first, uint32_t per_head, uint32_t magic) {
  const int64_t t = first + int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= a.T) return;
  const int lane = threadIdx.x & 63;
  const bool values = blockIdx.y != 0;
  const CacheView &c = a.cache;
  const int32_t slot = a.slots[t];
  const bool inside = slot >= 0 && (slot >> c.shift) < c.pages;
  if (!values && lane == 0) a.row_err[t] = slot >= -1 && (slot < 0 || inside) ? 0u : DSDE_ERR_PAGES;
  if (!inside) return;
  const KvRows &rows = values ? a.v : a.k;
  const char *src = rows.data + t * rows.token_stride;
  char *dst = (values ? c.v : c.k) + int64_t(slot >> c.shift) * c.page_stride +
              int64_t(slot & ((1 << c.shift) - 1)) * c.token_stride;
  const uint32_t n = per_head * uint32_t(c.heads);
  for (uint32_t i = lane; i < n; i += 64) {
    const uint32_t h = per_head == 1 ? i : __umulhi(i, magic), j = i - h * per_head;
    const char *from = src + int64_t(h) * rows.head_stride + j * (E4M3 ? 32 : 16);
    u32x4 x = load16(from);
    if constexpr (E4M3) {
      const u32x4 y = load16(from + 16);
      const float s = (values ? c.v_scale : c.k_scale)[h];
      x = u32x4{narrow(x.x, x.y, s), narrow(x.z, x.w, s), narrow(y.x, y.y, s), narrow(y.z, y.w, s)};
    }
    u32x4 *to = reinterpret_cast<u32x4 *>(dst + int64_t(h) * c.head_stride + j * 16);
    if constexpr (PAST)
      __builtin_nontemporal_store(x, to);
    else
      *to = x;
  }
}

}  // namespace

int launch_kv_map(const MapArgs &a, hipStream_t stream) {
  const auto plan = [&](auto all, auto shared) {
    if (a.B <= kSmallSeqs)
      map_plan_kernel<all.value, true, shared.value><<<1, kMapThreads, 0, stream>>>(a);
    else
      map_plan_kernel<all.value, false, shared.value><<<1, kMapThreads, 0, stream>>>(a);
  };
  if (a.rows == 0 && int64_t(a.B) * a.width > 4 * kManyPages) {  // sequences that end: maybe many pages
    plan(std::true_type{}, std::true_type{});
    give_kernel<<<256, 256, 0, stream>>>(a);
  } else if (a.rows <= kSmallRows) {
    plan(std::true_type{}, std::false_type{});
  } else {
    plan(std::false_type{}, std::false_type{});
    const int64_t blocks = (a.rows + 255) / 256;
    map_rows_kernel<<<uint32_t(blocks < 2048 ? blocks : 2048), 256, 0, stream>>>(a);
  }
  return hipGetLastError() == hipSuccess ? DSDE_OK : DSDE_DEVICE_ERROR;
}

int launch_kv_write(const KvWriteArgs &a, hipStream_t stream) {
  const int32_t e = a.cache.dtype == DSDE_FP32 ? 4 : a.cache.dtype == DSDE_BF16 ? 2 : 1;
  const uint32_t per_head = uint32_t(a.cache.dim * e / 16);  // lanes of a head
  // i / per_head as a high product: exact below 2^27 (and for one lane to a head, i itself)
  const uint32_t magic = uint32_t(((uint64_t(1) << 32) + per_head - 1) / per_head);
  const bool past = a.T * a.cache.heads * a.cache.dim * e * 2 > (int64_t(64) << 20);
  // a launch takes fewer than 2^32 threads
  constexpr int64_t kPass = int64_t(1) << 24;
  for (int64_t first = 0; first < a.T; first += kPass) {
    const int64_t n = a.T - first < kPass ? a.T - first : kPass;
    const dim3 grid(uint32_t((n + 3) / 4), 2);
    const auto launch = [&](auto e4m3) {
      if (past)
        kv_write_kernel<e4m3.value, true><<<grid, 256, 0, stream>>>(a, first, per_head, magic);
      else
        kv_write_kernel<e4m3.value, false><<<grid, 256, 0, stream>>>(a, first, per_head, magic);
    };
    if (a.cache.dtype == DSDE_E4M3)
      launch(std::true_type{});
    else
      launch(std::false_type{});
  }
  return hipGetLastError() == hipSuccess ? DSDE_OK : DSDE_DEVICE_ERROR;
}

}  // namespace dsde
