// Device helpers of the operators on single rows of logits (sampling, top
// logits, distillation): groups of eight consecutive logits with -inf past the
// row's end, ordered keys, and reductions over one workgroup.
#pragma once

#include "common.hpp"
#include "lanes.hpp"
#include "row_io.hpp"

namespace dsde {

// A row is read in groups of eight consecutive logits; a chunk is 1,024 groups
// (8,192 logits).  Thread t of a 256-thread workgroup owns groups
// 1024 k + 256 i + t, i = 0..3, of chunk k, and thread t of a 1,024-thread one
// group 1024 k + t, so the 64 groups of one wavefront and i are 512
// consecutive logits (a segment) in both.
constexpr int kGroup = 8;
constexpr int kChunkGroups = kChunk / kGroup;
constexpr int kSegs = kChunkGroups / 64;  // segments of a chunk

// Rows of a strided array.
struct RowsView {
  const char *base;
  int64_t stride;  // bytes
  int64_t V;
  __device__ __forceinline__ const char *row(int64_t r) const { return base + r * stride; }
};

// How the rows are read, as rows_form: 2 aligned, 1 any alignment, 0 narrower
// than one load.
inline int strided_rows_form(const void *p, int64_t stride_bytes, int32_t dtype, int64_t V) {
  const int64_t per_load = dtype == DSDE_BF16 ? 8 : 4;
  if (((reinterpret_cast<uintptr_t>(p) | uintptr_t(stride_bytes)) & 15u) == 0 && V % per_load == 0) return 2;
  return V >= 8 ? 1 : 0;
}

// Group w of a row: get() loads it from inside the row, place() puts the
// logits in their places and -inf past V.
template <int DT, int ROW>
struct Group {
  static constexpr bool kBf16 = DT == DSDE_BF16;
  u32x4_t h[1];  // bf16 rows
  f32x4_t f[2];  // fp32 rows, and any narrower than one load
  __device__ __forceinline__ void get(const char *row, uint32_t V, uint32_t w) {
    if constexpr (ROW == kScalarRows) {
#pragma unroll
      for (int i = 0; i < kGroup; ++i) {
        const uint32_t v = kGroup * w + i;
        f[i / 4][i % 4] = load_logit(row, DT, v < V ? v : V - 1);
      }
    } else if constexpr (kBf16) {
      h[0] = load_words<ROW>(row, V, w);
    } else {
      f[0] = load_quad<ROW>(row, V, 2 * w);
      f[1] = load_quad<ROW>(row, V, 2 * w + 1);
    }
  }
  __device__ __forceinline__ void place(uint32_t V, uint32_t w) {
    if constexpr (ROW == kScalarRows) {
#pragma unroll
      for (int i = 0; i < kGroup; ++i)
        if (kGroup * w + i >= V) f[i / 4][i % 4] = -__builtin_inff();
    } else if constexpr (kBf16) {
      place_words<ROW, kInfBf16x2>(h[0], V, w);
    } else {
      place_quad<ROW, true>(f[0], V, 2 * w);
      place_quad<ROW, true>(f[1], V, 2 * w + 1);
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (ROW != kScalarRows && kBf16) {
      const uint32_t x = h[0][i >> 1];
      return (i & 1) ? bf_hi(x) : bf_lo(x);
    }
    return f[i >> 2][i & 3];
  }
  __device__ __forceinline__ float max() const {
    return max_nan(max_nan(max_nan(at(0), at(1)), max_nan(at(2), at(3))),
                   max_nan(max_nan(at(4), at(5)), max_nan(at(6), at(7))));
  }
  // Takes logit i out of the row.
  __device__ __forceinline__ void drop(int i) {
    if constexpr (ROW != kScalarRows && kBf16)
      h[0][i >> 1] = (i & 1) ? (h[0][i >> 1] & 0xffffu) | (kInfBf16x2 << 16) : (h[0][i >> 1] & 0xffff0000u) | 0xff80u;
    else
      f[i >> 2][i & 3] = -__builtin_inff();
  }
};

// Unsigned keys in the order of the logits; +0 and -0 have one key.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}
constexpr uint32_t kKeyNegInf = 0x007fffffu;  // order_key(-inf)

// The weight of a logit against the reference M (at least the logit, or 0 where
// that is -inf).  The difference is taken first: z c alone may overflow for
// masks of the type's lowest value.
__device__ __forceinline__ float row_weight(float z, float M, float c) { return fast_exp2((z - M) * c); }
__device__ __forceinline__ float finite_ref(float M) { return M == -__builtin_inff() ? 0.0f : M; }

// Reductions and scans of a workgroup of WAVES wavefronts, in a fixed order;
// `red` holds WAVES entries and may be used again after the next barrier that
// follows the call (each call ends with one).
template <int WAVES, typename T, typename OP>
__device__ __forceinline__ T block_reduce(T v, T *red, OP op) {
  v = lanes::group_reduce<64>(v, op);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  T r = red[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) r = op(r, red[w]);
  __syncthreads();
  return r;
}
// Two sums with one pair of barriers; `red` holds 2 WAVES entries.
template <int WAVES>
__device__ __forceinline__ void block_sum2(double &a, double &b, double *red) {
  a = lanes::wave_sum(a);
  b = lanes::wave_sum(b);
  if ((threadIdx.x & 63) == 0) {
    red[threadIdx.x >> 6] = a;
    red[WAVES + (threadIdx.x >> 6)] = b;
  }
  __syncthreads();
  a = red[0];
  b = red[WAVES];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) {
    a += red[w];
    b += red[WAVES + w];
  }
  __syncthreads();
}
// Prefix sums in thread order and their total.
template <typename T>
struct BlockScan {
  T incl, excl, total;
};
template <int WAVES, typename T>
__device__ __forceinline__ BlockScan<T> block_scan(T v, T *red) {
  const lanes::Scan<T> s = lanes::wave_scan(v);
  const int wave = threadIdx.x >> 6;
  const T last = lanes::readlane(s.incl, 63);
  if ((threadIdx.x & 63) == 0) red[wave] = last;
  __syncthreads();
  T base = T(0), total = T(0);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w == wave) base = total;
    total += red[w];
  }
  __syncthreads();
  // a wavefront's last inclusive sum is the next one's base, bit for bit
  return BlockScan<T>{base + s.incl, (threadIdx.x & 63) == 0 ? base : base + s.excl, total};
}

}  // namespace dsde
