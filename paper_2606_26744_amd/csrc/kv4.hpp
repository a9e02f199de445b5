// Layout and arithmetic of the 4-bit KV cache (hdf_kv4_*).
//
// An element is an e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign, bit 3) times a scale: for
// keys a power of two for 32 consecutive dims of a row's head (a biased exponent in a byte), for
// values a bfloat16 for the whole head of a row.  The scales differ because the attention contracts
// keys over dims and values over positions: a key's scale lies along its contraction, where the
// matrix cores and the conversion instructions take powers of two a block, while a value's scale
// multiplies the row's probability once, so it is one number a row and may be any.
//
// A tile of 64 rows of one head is one piece of memory (8576 bytes for heads of 128 dims, 4352
// for 64): keys, values, key scales, value scales.  With row r of the tile in sub-tile
// st = 2*(r/32) + (r/4)%2 at ql = 4*((r%32)/8) + r%4, as in the wider cache (common.hpp):
//   keys    lane 16g + ql of sub-tile st holds dims (hd/4)*g .. of its row, hd/8 bytes, dim
//           0 in the low half of byte 0; 16-byte pieces ordered (sub-tiles, lane)
//   values  lane 16g + m holds, for k-slice ks and 16-dim tile dt, rows 32ks + 8g + 0..7 of dim
//           16dt + m in one word, row e in bits 4e..4e+3; words of four (ks, dt) make a
//           16-byte piece, pieces ordered ((ks, dt)/4, lane)
//   key scales    byte st of word 16b + ql, b the block of 32 dims
//   value scales  one bfloat16 a row, in row order
// so every load of the attention kernel is 16 contiguous bytes a lane.
#pragma once

#include "common.hpp"

namespace hdf {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// Bytes at which a tile's parts start, and its size.
__host__ __device__ constexpr int kv4_values_at(int hd) { return 32 * hd; }
__host__ __device__ constexpr int kv4_kscales_at(int hd) { return 64 * hd; }
__host__ __device__ constexpr int kv4_vscales_at(int hd) { return 66 * hd; }
__host__ __device__ constexpr int kv4_tile_bytes(int hd) { return 66 * hd + 128; }

// Sub-tile and place within it of row r (0..63) of a tile.
__host__ __device__ __forceinline__ int kv4_st(int r) { return 2 * (r >> 5) + ((r >> 2) & 1); }
__host__ __device__ __forceinline__ int kv4_ql(int r) { return 4 * ((r & 31) >> 3) + (r & 3); }

// Byte of the codes of dims (hd/4)*g .. of row r.
template <int HD>
__host__ __device__ __forceinline__ int kv4_key_at(int r, int g) {
  constexpr int KB = HD / 8, P = 16 / KB;   // bytes a lane and sub-tile, sub-tiles a piece
  const int st = kv4_st(r);
  return ((st / P) * 64 + 16 * g + kv4_ql(r)) * 16 + (st % P) * KB;
}
// Byte of the scale of block b of row r.
template <int HD>
__host__ __device__ __forceinline__ int kv4_kscale_at(int r, int b) {
  return kv4_kscales_at(HD) + (16 * b + kv4_ql(r)) * 4 + kv4_st(r);
}
// Byte of the word of rows 8*(r/8) .. of a dim.
template <int HD>
__host__ __device__ __forceinline__ int kv4_value_at(int r, int dim) {
  const int idx = (r >> 5) * (HD / 16) + (dim >> 4);
  return kv4_values_at(HD) + ((idx >> 2) * 64 + 16 * ((r >> 3) & 3) + (dim & 15)) * 16 + (idx & 3) * 4;
}
template <int HD>
__host__ __device__ __forceinline__ int kv4_vscale_at(int r) { return kv4_vscales_at(HD) + 2 * r; }

// Eight codes (a word) as bf16, exact; scale: its exponent field alone counts (0xFF gives NaN).
__device__ __forceinline__ bf16x8_t kv4_bf16x8(uint32_t w, float scale) {
  const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  const uint32_t d = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return __builtin_bit_cast(bf16x8_t, u32x4{a, b, c, d});
}
// ... as fp16 without a scale, exact.
__device__ __forceinline__ f16x8_t kv4_f16x8(uint32_t w) {
  const f16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 0);
  const f16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 1);
  const f16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 2);
  const f16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 3);
  return f16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Eight values as codes of x / scale (a power of two), to the nearest, ties to even, 6 at most.
__device__ __forceinline__ uint32_t kv4_codes8(const float* x, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return w;
}
__device__ __forceinline__ void kv4_floats8(uint32_t w, float scale, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto v = i == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0)
                   : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1)
                   : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2)
                            : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    x[2 * i] = v[0];
    x[2 * i + 1] = v[1];
  }
}

}  // namespace hdf
