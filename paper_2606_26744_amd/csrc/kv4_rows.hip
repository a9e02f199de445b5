// Rows of keys and values quantised into the 4-bit cache as they are written, and read back
// (layout and codes: kv4.hpp).
//
// Scales.  Keys, of 32 dims with greatest magnitude a: 2^e with the least e for which a <= 7 * 2^e
// (-125 <= e <= 125).  Between 6 and 7 units an element becomes 6, off by no more than the half
// step of the codes above 4; one exponent more would double every other element's step.  Values, of
// a row's head: the least bfloat16 s with a <= 6 * s (s >= 2^-126).  A block or head that holds a
// NaN or an infinity takes a NaN for its scale and reads back as NaN.
// Codes: the nearest of x / scale, ties to the even code, decided without error.  For keys the
// division is a change of exponent.  For values q = x / s is made from q0 = x * fl(1/s) and the
// residual r = x - s * q0 (exact in an fma), q = q0 + r * fl(1/s), with x and s first scaled by
// the power of two that brings s into [1, 2): s has 8 significant bits and the borders between
// codes 3, so an x that is not on a border is off it by 2^-24 of itself or more, and an x on one
// gives the border exactly.
//
// A wave takes eight rows x one head, lane 8i + j the dims (hd/8)*j .. of row i.  Keys leave as they
// come, a lane's codes side by side.  Eight values of one dim in eight rows share a word of the
// cache: the codes of eight rows are transposed by three lane exchanges (halves, bytes, nibbles).
// Rows in a run start at a multiple of 8 of the cache (the wave then owns its words and stores
// them, merged with what is there where the run covers a part).  A list's rows may share a word with
// another wave's: unless eight entries fill a word, its bits are cleared and set by atomics, so
// that the order of the waves does not matter.
//
// Bound by the memory: writing reads the rows once (bf16: 4 bytes a pair of elements against 1.05
// written).
#include <type_traits>

#include "kernels.hpp"
#include "kv4.hpp"

namespace hdf {

namespace {

constexpr int kRowThreads = 256;
constexpr int kGroupRows = 8;

template <typename T, int N>
__device__ __forceinline__ void load_row(const T* p, float* x) {
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    if constexpr (sizeof(T) == 2) {
      const u32x4 v = ld16(p + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[i + 2 * k] = lo_bf(v[k]);
        x[i + 2 * k + 1] = hi_bf(v[k]);
      }
    } else {
      const u32x4 a = ld16(p + i), b = ld16(p + i + 4);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[i + k] = __uint_as_float(a[k]);
        x[i + 4 + k] = __uint_as_float(b[k]);
      }
    }
  }
}

// A bf16 of any float (NaN stays NaN; an overflow becomes an infinity).
__device__ __forceinline__ uint32_t pack_any(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2_t));
}

template <typename T, int N>
__device__ __forceinline__ void store_row(T* p, const float* x) {
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    if constexpr (sizeof(T) == 2) {
      st16(p + i, u32x4{pack_any(x[i], x[i + 1]), pack_any(x[i + 2], x[i + 3]),
                        pack_any(x[i + 4], x[i + 5]), pack_any(x[i + 6], x[i + 7])});
    } else {
      st16(p + i, __builtin_bit_cast(u32x4, f32x4_t{x[i], x[i + 1], x[i + 2], x[i + 3]}));
      st16(p + i + 4, __builtin_bit_cast(u32x4, f32x4_t{x[i + 4], x[i + 5], x[i + 6], x[i + 7]}));
    }
  }
}

// Bits of the greatest magnitude (an infinity's or more where one is not finite).
template <int N>
__device__ __forceinline__ uint32_t top_bits(const float* x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  return m;
}

// Lanes 8i + j hold eight nibbles of row i; afterwards lane 8i + j holds nibble i of rows 0..7.
__device__ __forceinline__ uint32_t transpose8(uint32_t w, int i) {
  uint32_t o = __shfl_xor(w, 32, kWave);
  w = (i & 4) ? (w & 0xFFFF0000u) | (o >> 16) : (w & 0x0000FFFFu) | (o << 16);
  o = __shfl_xor(w, 16, kWave);
  w = (i & 2) ? (w & 0xFF00FF00u) | ((o >> 8) & 0x00FF00FFu) : (w & 0x00FF00FFu) | ((o & 0x00FF00FFu) << 8);
  o = __shfl_xor(w, 8, kWave);
  w = (i & 1) ? (w & 0xF0F0F0F0u) | ((o >> 4) & 0x0F0F0F0Fu) : (w & 0x0F0F0F0Fu) | ((o & 0x0F0F0F0Fu) << 4);
  return w;
}

struct Group {
  int64_t in;      // this lane's input row (-1: none)
  int64_t row;     // its cache row (-1: none)
};

// Rows of group g: of a run, cache rows 8 * (row0 / 8 + g) ..; of a list, entries 8g ...
__device__ __forceinline__ Group group_row(const Kv4RowArgs& a, int64_t g, int i) {
  Group r;
  if (a.rows != nullptr) {
    r.in = kGroupRows * g + i;
    if (r.in >= a.n) return {-1, -1};
    r.row = a.rows[r.in];
    if (r.row < 0 || r.row >= a.cap) r.row = -1;
  } else {
    r.row = (a.row0 & ~int64_t(7)) + kGroupRows * g + i;
    r.in = r.row - a.row0;
    if (r.in < 0 || r.in >= a.n) return {-1, -1};
  }
  return r;
}

template <typename T, int HD>
__global__ void __launch_bounds__(kRowThreads) kv4_write_kernel(Kv4RowArgs a) {
  constexpr int N = HD / 8;        // dims a lane
  constexpr int W = N / 8;         // words of codes a lane
  const int lane = threadIdx.x & 63, i = lane >> 3, j = lane & 7;
  const int64_t items = a.groups * a.nh;
  for (int64_t it = int64_t(blockIdx.x) * (kRowThreads / kWave) + (threadIdx.x >> 6); it < items;
       it += int64_t(gridDim.x) * (kRowThreads / kWave)) {
    const int64_t g = it / a.nh;
    const int h = int(it - g * a.nh);
    const Group gr = group_row(a, g, i);
    const bool live = gr.row >= 0;
    const int r = int(gr.row & 63);
    char* head = a.tiles + int64_t(h) * (a.cap >> 6) * kv4_tile_bytes(HD);
    char* tile = head + (live ? gr.row >> 6 : 0) * kv4_tile_bytes(HD);
    float x[N];
    if (a.k != nullptr) {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = 0.f;
      if (live) load_row<T, N>(static_cast<const T*>(a.k) + gr.in * a.ld_k + h * HD + N * j, x);
      uint32_t m = top_bits<N>(x);
      // 32 dims are two lanes (heads of 128 dims) or four.
      m = max(m, uint32_t(__shfl_xor(m, 1, kWave)));
      if constexpr (HD == 64) m = max(m, uint32_t(__shfl_xor(m, 2, kWave)));
      // a = f * 2^(E - 127), 1 <= f < 2: a <= 7 * 2^e from e = E - 129 on where f <= 1.75, else E - 128
      int e = int(m >> 23) - 129 + ((m & 0x7FFFFFu) > 0x600000u ? 1 : 0);
      e = min(max(e, -125), 125);
      const uint32_t byte = m >= 0x7F800000u ? 255u : uint32_t(e + 127);
      const float scale = __uint_as_float(uint32_t(e + 127) << 23);
      if (live) {
        char* dst = tile + kv4_key_at<HD>(r, j >> 1) + (j & 1) * (4 * W);
        if constexpr (W == 2)
          *reinterpret_cast<uint2*>(dst) = make_uint2(kv4_codes8(x, scale), kv4_codes8(x + 8, scale));
        else
          *reinterpret_cast<uint32_t*>(dst) = kv4_codes8(x, scale);
        constexpr int per = 32 / N;   // lanes of a block
        if (j % per == 0) tile[kv4_kscale_at<HD>(r, j / per)] = char(byte);
      }
    }
    if (a.v != nullptr) {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = 0.f;
      if (live) load_row<T, N>(static_cast<const T*>(a.v) + gr.in * a.ld_v + h * HD + N * j, x);
      uint32_t m = top_bits<N>(x);
      m = max(m, uint32_t(__shfl_xor(m, 1, kWave)));
      m = max(m, uint32_t(__shfl_xor(m, 2, kWave)));
      m = max(m, uint32_t(__shfl_xor(m, 4, kWave)));
      const float amax = __uint_as_float(m);
      const bool finite = m < 0x7F800000u;
      // The least bf16 with amax <= 6 * s: the quotient's upper half, or one or two steps more.
      uint32_t sb = max(__float_as_uint((finite ? amax : 0.f) / 6.f) & 0xFFFF0000u, 0x00800000u);
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (finite && 6.f * __uint_as_float(sb) < amax) sb += 0x10000u;
      const float unit = __uint_as_float((254u - (sb >> 23)) << 23);   // 2^-E of s
      const float s = __uint_as_float(sb) * unit, inv = 1.f / s;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float y = x[e] * unit, q = y * inv;
        x[e] = fmaf(fmaf(-s, q, y), inv, q);
      }
      uint32_t w[W];
#pragma unroll
      for (int k = 0; k < W; ++k) w[k] = transpose8(kv4_codes8(x + 8 * k, 1.f), i);
      if (live && j == 0)
        *reinterpret_cast<bf16_t*>(tile + kv4_vscale_at<HD>(r)) = finite ? bf16_t(sb >> 16) : bf16_t(0x7FC0);
      // Word k of lane 8i + j: dim N*j + 8k + i of the group's eight rows.
      const int64_t first = __shfl(gr.row, 0, kWave);
      const uint64_t there = __ballot(live);
      const bool run = a.rows == nullptr ||
                       (there == ~uint64_t(0) && (first & 7) == 0 && __all(gr.row == first + i));
      if (run) {
        const int64_t base = a.rows != nullptr ? first : (a.row0 & ~int64_t(7)) + kGroupRows * g;
        char* t = head + (base >> 6) * kv4_tile_bytes(HD);
        uint32_t keep = 0;           // bits of rows that the run does not cover
#pragma unroll
        for (int e = 0; e < 8; ++e) keep |= (there >> (8 * e)) & 1 ? 0u : 15u << (4 * e);
#pragma unroll
        for (int k = 0; k < W; ++k) {
          uint32_t* p = reinterpret_cast<uint32_t*>(t + kv4_value_at<HD>(int(base & 63), N * j + 8 * k + i));
          *p = keep == 0 ? w[k] : (*p & keep) | (w[k] & ~keep);
        }
      } else {
        // The words that the group's rows belong to, one after the other.
        uint64_t left = there;
        while (left != 0) {
          const int lead = __ffsll(static_cast<unsigned long long>(left)) - 1;
          const int64_t oct = __shfl(gr.row, lead, kWave) >> 3;
          const uint64_t mine = __ballot(live && (gr.row >> 3) == oct);
          left &= ~mine;
          uint32_t mask = 0, v[W];
#pragma unroll
          for (int k = 0; k < W; ++k) v[k] = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (((mine >> (8 * e)) & 1) == 0) continue;
            const int sh = 4 * int(__shfl(gr.row, 8 * e, kWave) & 7);
            mask |= 15u << sh;
#pragma unroll
            for (int k = 0; k < W; ++k)
              v[k] = (v[k] & ~(15u << sh)) | (((w[k] >> (4 * e)) & 15u) << sh);
          }
          char* t = head + (oct >> 3) * kv4_tile_bytes(HD);
#pragma unroll
          for (int k = 0; k < W; ++k) {
            uint32_t* p = reinterpret_cast<uint32_t*>(
                t + kv4_value_at<HD>(int((oct & 7) * 8), N * j + 8 * k + i));
            atomicAnd(p, ~mask);
            atomicOr(p, v[k]);
          }
        }
      }
    }
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(kRowThreads) kv4_read_kernel(Kv4RowArgs a) {
  constexpr int N = HD / 8, W = N / 8;
  const int lane = threadIdx.x & 63, i = lane >> 3, j = lane & 7;
  const int64_t items = a.groups * a.nh;
  for (int64_t it = int64_t(blockIdx.x) * (kRowThreads / kWave) + (threadIdx.x >> 6); it < items;
       it += int64_t(gridDim.x) * (kRowThreads / kWave)) {
    const int64_t g = it / a.nh;
    const int h = int(it - g * a.nh);
    const Group gr = group_row(a, g, i);
    const bool live = gr.row >= 0;
    const int r = live ? int(gr.row & 63) : 0;
    const char* head = a.tiles + int64_t(h) * (a.cap >> 6) * kv4_tile_bytes(HD);
    const char* tile = head + (live ? gr.row >> 6 : 0) * kv4_tile_bytes(HD);
    float x[N];
    if (a.k != nullptr) {
      const char* src = tile + kv4_key_at<HD>(r, j >> 1) + (j & 1) * (4 * W);
      const uint32_t byte = static_cast<unsigned char>(tile[kv4_kscale_at<HD>(r, j / (32 / N))]);
      const float scale = __uint_as_float(byte << 23);
      if constexpr (W == 2) {
        const uint2 c = *reinterpret_cast<const uint2*>(src);
        kv4_floats8(c.x, scale, x);
        kv4_floats8(c.y, scale, x + 8);
      } else {
        kv4_floats8(*reinterpret_cast<const uint32_t*>(src), scale, x);
      }
      if (!live) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = 0.f;
      }
      if (gr.in >= 0) store_row<T, N>(static_cast<T*>(a.k) + gr.in * a.ld_k + h * HD + N * j, x);
    }
    if (a.v != nullptr) {
      const int64_t first = __shfl(gr.row, 0, kWave);
      const bool run = (first & 7) == 0 && __all(gr.row == first + i);
      uint32_t w[W];
      if (run) {
        const char* t = head + (first >> 6) * kv4_tile_bytes(HD);
#pragma unroll
        for (int k = 0; k < W; ++k)
          w[k] = *reinterpret_cast<const uint32_t*>(
              t + kv4_value_at<HD>(int(first & 63), N * j + 8 * k + i));
#pragma unroll
        for (int k = 0; k < W; ++k) w[k] = transpose8(w[k], i);
      } else {
        const int sh = 4 * (r & 7);
#pragma unroll
        for (int k = 0; k < W; ++k) {
          w[k] = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t c = *reinterpret_cast<const uint32_t*>(
                tile + kv4_value_at<HD>(r, N * j + 8 * k + e));
            w[k] |= ((c >> sh) & 15u) << (4 * e);
          }
        }
      }
      const float s = bf2f(*reinterpret_cast<const bf16_t*>(tile + kv4_vscale_at<HD>(r)));
#pragma unroll
      for (int k = 0; k < W; ++k) kv4_floats8(w[k], 1.f, x + 8 * k);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = live ? x[e] * s : 0.f;
      if (gr.in >= 0) store_row<T, N>(static_cast<T*>(a.v) + gr.in * a.ld_v + h * HD + N * j, x);
    }
  }
}

template <typename T, int HD>
hipError_t rows_t(bool write, const Kv4RowArgs& a, hipStream_t s) {
  const int64_t wgs = (a.groups * a.nh + 3) / 4;
  const dim3 grid(unsigned(wgs < (int64_t(1) << 20) ? wgs : int64_t(1) << 20));
  if (write)
    hipLaunchKernelGGL((kv4_write_kernel<T, HD>), grid, dim3(kRowThreads), 0, s, a);
  else
    hipLaunchKernelGGL((kv4_read_kernel<T, HD>), grid, dim3(kRowThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_rows(bool bf16, bool write, int hd, const Kv4RowArgs& args, hipStream_t s) {
  Kv4RowArgs a = args;
  if (a.n <= 0) return hipSuccess;
  a.groups = a.rows != nullptr ? (a.n + 7) / 8 : (a.row0 % 8 + a.n + 7) / 8;
  if (bf16)
    return hd == 128 ? rows_t<bf16_t, 128>(write, a, s) : rows_t<bf16_t, 64>(write, a, s);
  return hd == 128 ? rows_t<float, 128>(write, a, s) : rows_t<float, 64>(write, a, s);
}

}  // namespace hdf
