// Rows of keys and values quantised into the 4-bit cache as they are written, and read back
// (layout and codes: kv4.hpp).
//
// Scales.  Keys, of 32 dims with greatest magnitude a: 2^e with the least e for which a <= 7 * 2^e
// (-125 <= e <= 125).  Between 6 and 7 units an element becomes 6, off by no more than the half
// step of the codes above 4; one exponent more would double every other element's step.  Values, of
// a row's head: the least bfloat16 s with a <= 6 * s (s >= 2^-126).  A block or head that holds a
// NaN or an infinity takes a NaN for its scale and reads back as NaN.
// Codes: the nearest of x / scale, ties to the even code, decided without error.  For keys the
// division is a change of exponent.  For values, s has 8 significant bits and a border between
// codes 3:
//   bf16  an x that is not on a border t is off it by 2^-11 of itself or more, so x * fl(1/s)
//         rounded to multiples of 2^-15 (by adding 384 and taking it off) stays on its side, and
//         one on a border becomes it;
//   fp32  q0 = x * fl(1/s), r = x - s * q0 (exact in an fma), q = q0 + r * fl(1/s), with x and s
//         first scaled by the power of two that brings s into [1, 2): an x off a border is off it by
//         2^-24 of itself or more, and one on a border gives it exactly.
//
// A wave takes eight rows x one head, lane 8i + j dims 8j .. 8j+7 (and 64 + 8j ..) of row i, so a load
// or store of the rows covers 128 contiguous bytes a row.  Keys leave as they come, a lane's codes in
// a word.  Eight values of one dim in eight rows share a word of the cache: the codes of eight rows
// are transposed by three lane exchanges (halves, bytes, nibbles).  Rows of a run are grouped from a
// multiple of 8 of the cache on (the wave then owns its words and stores them, merged with what is
// there where the run covers a part).  A list's rows may share a word with another wave's: unless
// eight entries fill a word, its bits are cleared and set by atomics, so that the order of the waves
// does not matter.
//
// Bound by the memory: 65536 rows of 32 heads of 128 in bf16, 1.36 GB, are written in 221 us (6.1 TB/s,
// four parts read to one written) and read back in 239 (5.7 TB/s, one part read to four written); a copy
// of 4 GiB moves 4.7 TB/s.  Rows that a call reads back are stored through the caches: past them takes
// the same time, and a few rows are what the next kernel reads.
#include <type_traits>

#include "kernels.hpp"
#include "kv4.hpp"

namespace hdf {

namespace {

constexpr int kHeads = 4, kReadGroups = 4;   // of a workgroup, at most: a wave each
constexpr int kGroupRows = 8;

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Eight consecutive elements of a row as they are stored.
template <typename T>
struct Eight {
  u32x4 w[sizeof(T) / 2];
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 2)
      return (e & 1) ? hi_bf(w[0][e >> 1]) : lo_bf(w[0][e >> 1]);
    else
      return __uint_as_float(w[e >> 2][e & 3]);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; ++i) w[i] = u32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; ++i) w[i] = ld_nt16(p + 4 * i);
  }
  // x rounded to the type (NaN stays NaN, an overflow becomes an infinity).
  __device__ __forceinline__ void set(const float* x) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[0][k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{x[2 * k], x[2 * k + 1]}, bf16x2_t));
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k >> 2][k & 3] = __float_as_uint(x[k]);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; ++i) st16(p + 4 * i, w[i]);
  }
  // fp32 bits of the greatest magnitude (an infinity's or more where one is not finite).
  __device__ __forceinline__ uint32_t top() const {
    if constexpr (sizeof(T) == 2) {
      u16x2_t m = {0, 0};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, uint32_t(w[0][k] & 0x7FFF7FFFu)));
      return uint32_t(max(m[0], m[1])) << 16;
    } else {
      uint32_t m = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) m = max(m, uint32_t(w[k >> 2][k & 3]) & 0x7FFFFFFFu);
      return m;
    }
  }
};

// Codes of x / scale, scale a power of two.
__device__ __forceinline__ uint32_t codes(const Eight<bf16_t>& x, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, uint32_t(x.w[0][0])), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, uint32_t(x.w[0][1])), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, uint32_t(x.w[0][2])), scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, uint32_t(x.w[0][3])), scale, 3);
  return w;
}
__device__ __forceinline__ uint32_t codes(const Eight<float>& x, float scale) {
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = x.get(e);
  return kv4_codes8(y, scale);
}

// Maximum over groups of four (EIGHT: eight) neighbouring lanes.
template <bool EIGHT>
__device__ __forceinline__ uint32_t near_max(uint32_t m) {
  m = max(m, uint32_t(__builtin_amdgcn_update_dpp(0, int(m), 0xB1, 0xF, 0xF, false)));   // lane ^ 1
  m = max(m, uint32_t(__builtin_amdgcn_update_dpp(0, int(m), 0x4E, 0xF, 0xF, false)));   // lane ^ 2
  if constexpr (EIGHT)
    m = max(m, uint32_t(__builtin_amdgcn_update_dpp(0, int(m), 0x141, 0xF, 0xF, false)));   // mirrored in eight
  return m;
}

// Lanes 8i + j hold eight nibbles of row i; afterwards lane 8i + j holds nibble i of rows 0..7 (and
// the same call takes it back).
__device__ __forceinline__ uint32_t transpose8(uint32_t w, int i) {
  // Lanes 32 apart: both get (lower lane's, upper lane's) word.
  auto p = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  w = __builtin_amdgcn_perm(p[1], p[0], (i & 4) ? 0x07060302u : 0x05040100u);
  p = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  w = __builtin_amdgcn_perm(p[1], p[0], (i & 2) ? 0x07030501u : 0x06020400u);
  const uint32_t o = uint32_t(__builtin_amdgcn_update_dpp(0, int(w), 0x128, 0xF, 0xF, false));   // lane ^ 8
  const uint32_t mask = (i & 1) ? 0xF0F0F0F0u : 0x0F0F0F0Fu;
  return (w & mask) | (__builtin_amdgcn_alignbit(o, o, (i & 1) ? 4 : 28) & ~mask);
}

// What a wave works on: its head's tiles, and each lane's rows.
struct Place {
  char* head;
  int64_t in;      // this lane's row of k, v (-1: none)
  int64_t row;     // its cache row (-1: none)
};

// Group g of a run: cache rows 8 * (row0 / 8 + g) ..; of a list: entries 8g ...
template <bool LIST>
__device__ __forceinline__ void place_row(const Kv4RowArgs& a, int64_t g, int i, Place& p) {
  if constexpr (LIST) {
    p.in = kGroupRows * g + i;
    p.row = -1;
    if (p.in >= a.n) {
      p.in = -1;
    } else {
      p.row = a.rows[p.in];
      if (p.row < 0 || p.row >= a.cap) p.row = -1;
    }
  } else {
    p.row = (a.row0 & ~int64_t(7)) + kGroupRows * g + i;
    p.in = p.row - a.row0;
    if (p.in < 0 || p.in >= a.n) p.in = p.row = -1;
  }
}

template <typename T, int HD, bool LIST>
__global__ void __launch_bounds__(kHeads * kWave) kv4_write_kernel(Kv4RowArgs a) {
  constexpr int H = HD / 64;       // eights of dims a lane
  constexpr int TB = kv4_tile_bytes(HD);
  const int lane = threadIdx.x & 63, i = lane >> 3, j = lane & 7;
  const int h = blockIdx.x * kHeads + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (h >= a.nh) return;
  Place pl;
  pl.head = a.tiles + int64_t(h) * (a.cap >> 6) * TB;
  for (int64_t g = blockIdx.y; g < a.groups; g += gridDim.y) {
    place_row<LIST>(a, g, i, pl);
    const bool live = pl.row >= 0;
    const int r = int(pl.row & 63);
    char* tile = pl.head + (live ? pl.row >> 6 : 0) * TB;
    Eight<T> xk[H], xv[H];
#pragma unroll
    for (int q = 0; q < H; ++q) {
      xk[q].clear();
      xv[q].clear();
      if (live && a.k != nullptr) xk[q].load(static_cast<const T*>(a.k) + pl.in * a.ld_k + h * HD + 64 * q + 8 * j);
      if (live && a.v != nullptr) xv[q].load(static_cast<const T*>(a.v) + pl.in * a.ld_v + h * HD + 64 * q + 8 * j);
    }
    if (a.k != nullptr) {
#pragma unroll
      for (int q = 0; q < H; ++q) {
        const uint32_t m = near_max<false>(xk[q].top());   // of 32 dims
        // a = f * 2^(E - 127), 1 <= f < 2: a <= 7 * 2^e from e = E - 129 on where f <= 1.75, else E - 128
        int e = int(m >> 23) - 129 + ((m & 0x7FFFFFu) > 0x600000u ? 1 : 0);
        e = min(max(e, -125), 125);
        const uint32_t byte = m >= 0x7F800000u ? 255u : uint32_t(e + 127);
        const uint32_t w = codes(xk[q], __uint_as_float(uint32_t(e + 127) << 23));
        if (live) {
          const int g4 = (64 * q + 8 * j) / (HD / 4), at = (8 * j) % (HD / 4) / 2;
          *reinterpret_cast<uint32_t*>(tile + kv4_key_at<HD>(r, g4) + at) = w;
          if (j % 4 == 0) tile[kv4_kscale_at<HD>(r, 2 * q + j / 4)] = char(byte);
        }
      }
    }
    if (a.v != nullptr) {
      uint32_t m = xv[0].top();
#pragma unroll
      for (int q = 1; q < H; ++q) m = max(m, xv[q].top());
      m = near_max<true>(m);
      const float amax = __uint_as_float(m);
      const bool finite = m < 0x7F800000u;
      // The least bf16 with amax <= 6 * s: the quotient's upper half, or one or two steps more.
      uint32_t sb = max(__float_as_uint((finite ? amax : 0.f) * (1.f / 6.f)) & 0xFFFF0000u, 0x00800000u);
      if (sb > 0x00800000u) sb -= 0x10000u;    // the product may be a step too far
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (finite && 6.f * __uint_as_float(sb) < amax) sb += 0x10000u;
      const float s = __uint_as_float(sb);
      uint32_t w[H];
      if constexpr (sizeof(T) == 2) {
        const float inv = 1.f / s;
#pragma unroll
        for (int q = 0; q < H; ++q) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = fmaf(xv[q].get(e), inv, 384.f) - 384.f;
          w[q] = kv4_codes8(y, 1.f);
        }
      } else {
        const float unit = __uint_as_float((254u - (sb >> 23)) << 23);   // 2^-E of s
        const float sn = s * unit, inv = 1.f / sn;
#pragma unroll
        for (int q = 0; q < H; ++q) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = xv[q].get(e) * unit, q0 = x * inv;
            y[e] = fmaf(fmaf(-sn, q0, x), inv, q0);
          }
          w[q] = kv4_codes8(y, 1.f);
        }
      }
#pragma unroll
      for (int q = 0; q < H; ++q) w[q] = transpose8(w[q], i);
      if (live && j == 0)
        *reinterpret_cast<bf16_t*>(tile + kv4_vscale_at<HD>(r)) = finite ? bf16_t(sb >> 16) : bf16_t(0x7FC0);
      // Word q of lane 8i + j: dim 64q + 8j + i of the group's eight rows.
      const uint64_t there = __ballot(live);
      int64_t first;
      bool run = true;
      if constexpr (LIST) {
        first = __shfl(pl.row, 0, kWave);
        run = there == ~uint64_t(0) && (first & 7) == 0 && __all(pl.row == first + i);
      } else {
        first = (a.row0 & ~int64_t(7)) + kGroupRows * g;
      }
      if (run) {
        char* t = pl.head + (first >> 6) * TB;
        uint32_t keep = 0;           // bits of rows that the run does not cover
        if constexpr (!LIST) {
          if (there != ~uint64_t(0)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) keep |= (there >> (8 * e)) & 1 ? 0u : 15u << (4 * e);
          }
        }
#pragma unroll
        for (int q = 0; q < H; ++q) {
          uint32_t* p = reinterpret_cast<uint32_t*>(t + kv4_value_at<HD>(int(first & 63), 64 * q + 8 * j + i));
          *p = keep == 0 ? w[q] : (*p & keep) | (w[q] & ~keep);
        }
      } else {
        // The words that the group's rows belong to, one after the other.
        uint64_t left = there;
        while (left != 0) {
          const int lead = __ffsll(static_cast<unsigned long long>(left)) - 1;
          const int64_t oct = __shfl(pl.row, lead, kWave) >> 3;
          const uint64_t mine = __ballot(live && (pl.row >> 3) == oct);
          left &= ~mine;
          uint32_t mask = 0, v[H];
#pragma unroll
          for (int q = 0; q < H; ++q) v[q] = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (((mine >> (8 * e)) & 1) == 0) continue;
            const int sh = 4 * int(__shfl(pl.row, 8 * e, kWave) & 7);
            mask |= 15u << sh;
#pragma unroll
            for (int q = 0; q < H; ++q)
              v[q] = (v[q] & ~(15u << sh)) | (((w[q] >> (4 * e)) & 15u) << sh);
          }
          char* t = pl.head + (oct >> 3) * TB;
#pragma unroll
          for (int q = 0; q < H; ++q) {
            uint32_t* p = reinterpret_cast<uint32_t*>(
                t + kv4_value_at<HD>(int((oct & 7) * 8), 64 * q + 8 * j + i));
            atomicAnd(p, ~mask);
            atomicOr(p, v[q]);
          }
        }
      }
    }
  }
}

template <typename T, int HD, bool LIST>
__global__ void __launch_bounds__(kHeads * kReadGroups * kWave) kv4_read_kernel(Kv4RowArgs a) {
  constexpr int H = HD / 64, TB = kv4_tile_bytes(HD);
  const int lane = threadIdx.x & 63, i = lane >> 3, j = lane & 7;
  const int h = blockIdx.x * kHeads + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (h >= a.nh) return;
  Place pl;
  pl.head = a.tiles + int64_t(h) * (a.cap >> 6) * TB;
  const int in_wg = __builtin_amdgcn_readfirstlane(threadIdx.y), gw = blockDim.y;
  for (int64_t g = int64_t(blockIdx.y) * gw + in_wg; g < a.groups; g += int64_t(gridDim.y) * gw) {
    place_row<LIST>(a, g, i, pl);
    const bool live = pl.row >= 0;
    const int r = live ? int(pl.row & 63) : 0;
    const char* tile = pl.head + (live ? pl.row >> 6 : 0) * TB;
    uint32_t ck[H], cv[H], ks[H];
    bf16_t vs = 0;
    bool run = true;
    int64_t first = 0;
    if (a.k != nullptr) {
#pragma unroll
      for (int q = 0; q < H; ++q) {
        const int g4 = (64 * q + 8 * j) / (HD / 4), at = (8 * j) % (HD / 4) / 2;
        ck[q] = *reinterpret_cast<const uint32_t*>(tile + kv4_key_at<HD>(r, g4) + at);
        ks[q] = static_cast<unsigned char>(tile[kv4_kscale_at<HD>(r, 2 * q + j / 4)]);
      }
    }
    if (a.v != nullptr) {
      if constexpr (LIST) {
        first = __shfl(pl.row, 0, kWave);
        run = (first & 7) == 0 && __all(pl.row == first + i);
      } else {
        first = (a.row0 & ~int64_t(7)) + kGroupRows * g;
      }
      vs = *reinterpret_cast<const bf16_t*>(tile + kv4_vscale_at<HD>(r));
      if (run) {
        const char* t = pl.head + (first >> 6) * TB;
#pragma unroll
        for (int q = 0; q < H; ++q)
          cv[q] = *reinterpret_cast<const uint32_t*>(
              t + kv4_value_at<HD>(int(first & 63), 64 * q + 8 * j + i));
      } else {
        const int sh = 4 * (r & 7);
#pragma unroll
        for (int q = 0; q < H; ++q) {
          cv[q] = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t c = *reinterpret_cast<const uint32_t*>(
                tile + kv4_value_at<HD>(r, 64 * q + 8 * j + e));
            cv[q] |= ((c >> sh) & 15u) << (4 * e);
          }
        }
      }
    }
    float x[8];
    Eight<T> o;
    if (a.k != nullptr) {
#pragma unroll
      for (int q = 0; q < H; ++q) {
        kv4_floats8(ck[q], __uint_as_float(ks[q] << 23), x);
        o.set(x);
        if (!live) o.clear();
        if (pl.in >= 0) o.store(static_cast<T*>(a.k) + pl.in * a.ld_k + h * HD + 64 * q + 8 * j);
      }
    }
    if (a.v != nullptr) {
      const float s = bf2f(vs);
#pragma unroll
      for (int q = 0; q < H; ++q) {
        kv4_floats8(run ? transpose8(cv[q], i) : cv[q], 1.f, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= s;
        o.set(x);
        if (!live) o.clear();
        if (pl.in >= 0) o.store(static_cast<T*>(a.v) + pl.in * a.ld_v + h * HD + 64 * q + 8 * j);
      }
    }
  }
}

template <typename T, int HD, bool LIST>
hipError_t rows_t(bool write, const Kv4RowArgs& a, hipStream_t s) {
  // Four heads of a group a workgroup; in long reads of four neighbouring groups, which share lines of
  // the cache's tiles (the keys of 8 rows lie in runs of 64 bytes): (heads, groups) (4, 1), (16, 1),
  // (2, 8), (4, 4) read 65536 rows of 32 x 128 in bf16 back in 266 us, 248, 249, 239, and 16384 in 68.8,
  // 66.5, 67.1, 64.6; 4096 rows take 20 in all.  Written by 4, 8, 16 heads: 65536 rows 221, 234, 240.
  const int gw = !write && a.groups * a.nh > 32768 ? kReadGroups : 1;
  const int64_t gy = (a.groups + gw - 1) / gw;
  const dim3 grid((a.nh + kHeads - 1) / kHeads, unsigned(gy < 65535 ? gy : 65535)), block(kHeads * kWave, gw);
  if (write)
    hipLaunchKernelGGL((kv4_write_kernel<T, HD, LIST>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((kv4_read_kernel<T, HD, LIST>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t rows_of(bool write, const Kv4RowArgs& a, hipStream_t s) {
  return a.rows != nullptr ? rows_t<T, HD, true>(write, a, s) : rows_t<T, HD, false>(write, a, s);
}

}  // namespace

hipError_t launch_kv4_rows(bool bf16, bool write, int hd, const Kv4RowArgs& args, hipStream_t s) {
  Kv4RowArgs a = args;
  if (a.n <= 0) return hipSuccess;
  a.groups = a.rows != nullptr ? (a.n + 7) / 8 : (a.row0 % 8 + a.n + 7) / 8;
  if (bf16) return hd == 128 ? rows_of<bf16_t, 128>(write, a, s) : rows_of<bf16_t, 64>(write, a, s);
  return hd == 128 ? rows_of<float, 128>(write, a, s) : rows_of<float, 64>(write, a, s);
}

}  // namespace hdf
