// Rows of logits of either type, their order and their weights: shared by the truncated draws
// and the distillation (row_cut.hip, verify.hip, distill.hip).
#pragma once

#include "common.hpp"

namespace hdf {

// A row of V logits read 16 bytes at a time.  Rows start at any element (odd vocabularies, strides,
// views): vector j holds columns j * N - shift .. + N - 1 and is aligned; the first and the last,
// which reach past the row, are read element by element.  `load_raw` and `raw` give the values as
// they are, `load` and `at` those of a row to choose from: NaN is -inf (masked).
template <typename T>
struct LogitRow {
  static constexpr int N = 16 / int(sizeof(T));
  const T* p;
  int V, shift;

  __device__ __forceinline__ LogitRow(const T* row, int V_) : p(row), V(V_) {
    shift = int((reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (N - 1));
  }
  __device__ __forceinline__ int vectors() const { return (V + shift + N - 1) / N; }
  __device__ __forceinline__ int column(int j) const { return j * N - shift; }
  // Whether vectors j .. j + n - 1 lie within the row.
  __device__ __forceinline__ bool inside(int j, int n) const {
    return column(j) >= 0 && column(j + n) <= V;
  }
  // Vector j, which lies within the row: its bits, and as fp32.
  __device__ __forceinline__ u32x4 bits_inside(int j) const { return ld16(p + column(j)); }
  __device__ __forceinline__ void load_inside(int j, float x[N]) const { unpack(bits_inside(j), x); }
  static __device__ __forceinline__ void unpack(u32x4 v, float x[N]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2) {
        x[2 * e] = lo_bf(v[e]);
        x[2 * e + 1] = hi_bf(v[e]);
      } else {
        x[e] = __uint_as_float(v[e]);
      }
    }
  }
  // Vector j as fp32; columns outside the row are -inf.
  __device__ __forceinline__ void load_raw(int j, float x[N]) const {
    const int c = column(j);
    if (c >= 0 && c + N <= V) {
      load_inside(j, x);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = c + e >= 0 && c + e < V ? raw(c + e) : -INFINITY;
    }
  }
  __device__ __forceinline__ void load(int j, float x[N]) const {
    load_raw(j, x);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = fmaxf(x[e], -INFINITY);
  }
  __device__ __forceinline__ float raw(int c) const {
    if constexpr (sizeof(T) == 2)
      return bf2f(p[c]);
    else
      return p[c];
  }
  __device__ __forceinline__ float at(int c) const { return fmaxf(raw(c), -INFINITY); }
};

// The order of a row's entries (largest value first, ties to the lowest column) as 52-bit keys,
// greater for an earlier entry: the value's order key (-0 as +0: they are equal logits) over the
// complement of the column.
constexpr int kColumnBits = 20;
constexpr uint32_t kColumnMask = (1u << kColumnBits) - 1;   // columns 0 .. 2^20 - 1

__device__ __forceinline__ uint64_t entry_key(float z, int c) {
  return (uint64_t(f32_order_key(z + 0.f)) << kColumnBits) | (kColumnMask - uint32_t(c));
}
__device__ __forceinline__ float entry_logit(uint64_t k) {
  return f32_from_order_key(uint32_t(k >> kColumnBits));
}
__device__ __forceinline__ int entry_column(uint64_t k) {
  return int(kColumnMask - (uint32_t(k) & kColumnMask));
}

// The greatest of three or two values, none of them NaN.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

__device__ __forceinline__ float max2(float a, float b) {
  float d;
  asm("v_max_f32 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
  return d;
}

// a * b + k with k the same for all lanes: a scalar operand.  (The compiler would copy k into the
// result first, two moves a product, and take three times as long over a series.)
__device__ __forceinline__ double fma_k(double a, double b, double k) {
  double d;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "s"(k));
  return d;
}

// 2^t in 64 bits for t <= 0 (and the few ulps above it that rounding leaves): 2^n times the
// exponential series of f ln 2, |f| <= 1/2, whose first dropped term is 0.35^12 / 12! = 6e-15.
// Which entry a draw or a cut falls on is decided by sums of these; with 32-bit exponentials one
// row in a few thousand would fall on a neighbour.
__device__ __forceinline__ double exp2_64(double t) {
  t = fmax(t, -1100.);   // below the least double; also what an infinite difference gives
  const double n = rint(t);
  const double x = (t - n) * 0.69314718055994530942;
  double p = 1. / 39916800.;
  p = fma_k(p, x, 1. / 3628800.);
  p = fma_k(p, x, 1. / 362880.);
  p = fma_k(p, x, 1. / 40320.);
  p = fma_k(p, x, 1. / 5040.);
  p = fma_k(p, x, 1. / 720.);
  p = fma_k(p, x, 1. / 120.);
  p = fma_k(p, x, 1. / 24.);
  p = fma_k(p, x, 1. / 6.);
  p = fma_k(p, x, 0.5);
  p = fma_k(p, x, 1.);
  p = fma_k(p, x, 1.);
  return ldexp(p, int(n));
}

// Weight e^((z - m) / T) of an entry, c2 = log2(e) / T, m >= z (both may be +inf: weight 1);
// 0 for a masked one.
__device__ __forceinline__ double entry_weight(float z, float m, double c2) {
  if (z == -INFINITY) return 0.;
  return z == m ? 1. : exp2_64((double(z) - double(m)) * c2);
}

// Whether a row's log-sum-exp is so far from 0 that its rounding, up to 2^-53 of it, is more than
// 2^-27 of the probabilities that are taken from it: where T is about 1e-6 (or the logits are as
// large).  At 2^53, T = 1e-14, nothing of them would be left.
__device__ __forceinline__ bool far_lse(double lse) { return fabs(lse) > 67108864. && lse > -INFINITY; }

// Another lane's value within the row of 16 (a DPP move; 64-bit values in two).
template <int CTRL, int ROWS, typename X>
__device__ __forceinline__ X dpp(X v) {
  constexpr int D = sizeof(X) / 4;
  int w[D];
  __builtin_memcpy(w, &v, sizeof(X));
#pragma unroll
  for (int i = 0; i < D; ++i) w[i] = __builtin_amdgcn_update_dpp(0, w[i], CTRL, ROWS, 0xf, true);
  __builtin_memcpy(&v, w, sizeof(X));
  return v;
}
template <typename X>
__device__ __forceinline__ X read_lane(X v, int lane) {
  constexpr int D = sizeof(X) / 4;
  int w[D];
  __builtin_memcpy(w, &v, sizeof(X));
#pragma unroll
  for (int i = 0; i < D; ++i) w[i] = __builtin_amdgcn_readlane(w[i], lane);
  __builtin_memcpy(&v, w, sizeof(X));
  return v;
}

// The value of the lane D apart (D a power of two): moves between lanes, no shared memory.
template <int D>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v) {
  if constexpr (D == 1) return dpp<0xB1, 0xf>(v);
  if constexpr (D == 2) return dpp<0x4E, 0xf>(v);
  if constexpr (D == 4) return dpp<0x1B, 0xf>(dpp<0x141, 0xf>(v));   // 7 apart, then 3
  if constexpr (D == 8) return dpp<0x128, 0xf>(v);                   // turned by 8 of 16
  if constexpr (D >= 16) {   // rows, or halves, change places between two copies
    uint32_t w[2];
    __builtin_memcpy(w, &v, 8);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const auto p = D == 16 ? __builtin_amdgcn_permlane16_swap(w[i], w[i], false, false)
                             : __builtin_amdgcn_permlane32_swap(w[i], w[i], false, false);
      w[i] = (threadIdx.x & D) != 0 ? p[0] : p[1];
    }
    __builtin_memcpy(&v, w, 8);
    return v;
  }
}

// All lanes' values under f (commutative, associative but for rounding), the same to every lane:
// within rows of 16 by moves between lanes, then the four rows.  The whole wave takes part.
template <typename X, typename F>
__device__ __forceinline__ X wave_fold(X v, F f) {
  v = f(v, dpp<0xB1, 0xf>(v));    // lanes 1 apart
  v = f(v, dpp<0x4E, 0xf>(v));    // 2 apart
  v = f(v, dpp<0x141, 0xf>(v));   // mirrored in 8
  v = f(v, dpp<0x140, 0xf>(v));   // mirrored in 16
  return f(f(read_lane(v, 0), read_lane(v, 16)), f(read_lane(v, 32), read_lane(v, 48)));
}

// Inclusive running sum over a wave's lanes.
template <typename X>
__device__ __forceinline__ X wave_scan(X v) {
  v += dpp<0x111, 0xf>(v);   // from 1, 2, 4, 8 lanes before in the row, zero past its start
  v += dpp<0x112, 0xf>(v);
  v += dpp<0x114, 0xf>(v);
  v += dpp<0x118, 0xf>(v);
  v += dpp<0x142, 0xa>(v);   // the last lane of rows 0 and 2 to rows 1 and 3
  v += dpp<0x143, 0xc>(v);   // lane 31 to rows 2 and 3
  return v;
}

// Least (greatest) i of the lanes for which c holds into *dst, one atomic a wave; i rises with the
// lane.  (A wave's 64 atomics of different values to one word are done one by one: 45 thousand cycles
// for the eight entries a thread of a draw.)
__device__ __forceinline__ void note_first(bool c, int i, int* dst) {
  const unsigned long long m = __ballot(c);
  if (m == 0ull) return;
  const int v = read_lane(i, __ffsll(static_cast<long long>(m)) - 1);
  if ((threadIdx.x & 63) == 0) atomicMin(dst, v);
}
__device__ __forceinline__ void note_last(bool c, int i, int* dst) {
  const unsigned long long m = __ballot(c);
  if (m == 0ull) return;
  const int v = read_lane(i, 63 - __clzll(static_cast<long long>(m)));
  if ((threadIdx.x & 63) == 0) atomicMax(dst, v);
}

// f over a workgroup of W waves in a fixed order; every thread gets the result.  `sh` holds W values
// and is free again on return.
template <int W, typename X, typename F>
__device__ __forceinline__ X block_fold(X v, X* sh, F f) {
  static_assert(W == 4 || W == 8 || W == 16);
  v = wave_fold(v, f);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  X t = sh[threadIdx.x & (W - 1)];   // a lane a wave, and as within rows of 16
  t = f(t, dpp<0xB1, 0xf>(t));
  t = f(t, dpp<0x4E, 0xf>(t));
  if constexpr (W > 4) t = f(t, dpp<0x141, 0xf>(t));
  if constexpr (W > 8) t = f(t, dpp<0x140, 0xf>(t));
  t = read_lane(t, 0);   // one order of the sum for all
  __syncthreads();
  return t;
}

// Inclusive running sum over the workgroup's threads, in their order; `total` gets the whole.
template <int W, typename X>
__device__ __forceinline__ X block_scan(X v, X* sh, X& total) {
  static_assert(W == 4 || W == 8 || W == 16);
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  v = wave_scan(v);
  if (lane == 63) sh[wid] = v;
  __syncthreads();
  X t = sh[lane & (W - 1)];   // a lane a wave, and as within rows of 16
  t += dpp<0x111, 0xf>(t);
  t += dpp<0x112, 0xf>(t);
  if constexpr (W > 4) t += dpp<0x114, 0xf>(t);
  if constexpr (W > 8) t += dpp<0x118, 0xf>(t);
  const int w = __builtin_amdgcn_readfirstlane(wid);
  X before = X(0);
  if (w > 0) before = read_lane(t, w - 1);
  total = read_lane(t, W - 1);
  __syncthreads();
  return before + v;
}

}  // namespace hdf
