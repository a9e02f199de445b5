// Attention of blocks of queries over the 4-bit cache (layout: kv4.hpp) and over the block's own
// keys and values, which are not quantised.
//
//   O = softmax(scale * Q [K, K_b]^T) [V, V_b],   lse = log of the softmax's sum
// G = n_heads / n_kv_heads query heads share a head of keys, so a (sequence, head of keys) has
// G * B query rows, row k * G + j being slot k of its j-th head.
//
// A workgroup of eight waves (or four: few_waves) takes 16 query rows, or 32 as two tiles a wave, of
// a (sequence, head of keys) over a chunk of the context; a wave takes every eighth of its 64-row
// tiles and keeps its own running maximum and sum, so the loop has no barrier and no LDS, and the
// waves' states are joined once.  The products are S^T = K Q^T and O^T = V^T P^T: the keys of a 64-row
// tile are laid out so that the lane that has a score has its probability where the second product
// wants it.
// Codes go from their 16-byte loads through the conversion instructions into the matrix
// instructions.  Keys become bf16 (exactly, scale and all); values fp16 or bf16 codes, their scales in
// the probabilities (struct Unit); 32-bit queries and probabilities are three bf16 terms.
//
// Bound by the memory where a workgroup has enough tiles: 64 contexts of 1024 to 16384 positions, 32
// heads, B = 16, 363 us for 2.32 GB (6.4 TB/s; vector issue 51% of the cycles, matrix cores 17%);
// 8 x 2048 positions 14 to 15.5 us for 70 MB, 3 of them start and join.  Bound by instruction issue where 32
// queries share a head of keys: 16 contexts of one length, 32 heads over 8, B = 16 (256 workgroups), take
// 10 us and 2.4 for every tile a wave, 5800 cycles in which the SIMD's two waves have a tile each, about
// 4300 of them vector issue (500 instructions a tile) and 2050 of the matrix cores (64).  Contexts of 512 to
// 8192 positions take 39 us (2.0 TB/s on average) where the longest has 6656, 13 tiles a wave: 41 by that.
// A conversion costs what any vector instruction does (4.6 cycles; to fp16 as to bf16), an
// exponential two, a matrix instruction 16 of the matrix core and about half of them of the issue.
// Measured and not kept: products of fp4 keys with two fp8 terms of a query (products 2^-11 below an
// instruction's greatest are dropped: log-sum-exps 1e-3 off); loads for the next tile behind a branch
// (the waits then cover them too: 17 us for 14.7 in the 8 x 2048 case); barriers a round or priorities
// so that a SIMD's waves alternate (42 for 41 us, 40 for 40); 2, 6, 12 or 16 waves a workgroup;
// the block's keys read by its wave from memory, without LDS (no gain, and the 32-bit form spills).
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "kv4.hpp"

namespace hdf {

namespace {

constexpr int kTile = 64;
constexpr int kWaves = 8, kFewWaves = 4;    // of a workgroup (attn_t)
constexpr int kJoinThreads = 256;

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t to_bf2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, bf16x2_t));
}

// Eight floats as NT bf16 terms that sum to them (one: rounded; three: all 24 bits).
template <int NT>
__device__ __forceinline__ void split8(const float* x, bf16x8_t* t) {
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = x[e];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = to_bf2(y[2 * e], y[2 * e + 1]);
      if (n + 1 < NT) {
        y[2 * e] -= lo_bf(w[e]);
        y[2 * e + 1] -= hi_bf(w[e]);
      }
    }
    t[n] = __builtin_bit_cast(bf16x8_t, u32x4{w[0], w[1], w[2], w[3]});
  }
}

// Eight consecutive elements of a row as floats.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 v = ld16(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = lo_bf(v[k]);
      x[2 * k + 1] = hi_bf(v[k]);
    }
  } else {
    const u32x4 a = ld16(p), b = ld16(p + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = __uint_as_float(a[k]);
      x[4 + k] = __uint_as_float(b[k]);
    }
  }
}

// A tile of the cache as a wave's lanes hold it.
template <int HD>
struct Tile {
  u32x4 k[HD / 32], v[HD / 32];
  uint32_t ks;      // scales of four sub-tiles' keys
  u32x4 vs[2];      // scales of the lane's sixteen values' rows
  __device__ __forceinline__ uint32_t key_word(int st, int j) const {
    constexpr int WL = HD / 32;   // words a lane and sub-tile
    return k[(st * WL + j) / 4][(st * WL + j) % 4];
  }
  __device__ __forceinline__ uint32_t value_word(int ks_, int dt) const {
    const int idx = ks_ * (HD / 16) + dt;
    return v[idx / 4][idx % 4];
  }
};

// The tile at p (the same for all lanes), or zeros, without a fetch, where there is none.  Buffer
// loads: one 32-bit offset a lane serves them all, where 64-bit addresses of every part cost registers
// that the loop needs; and a tile that is not there takes the same instructions, so that the waits
// before a tile's use count exactly the loads behind it (behind a branch they wait for those too).
// The codes are read once a call, past the caches.
template <int HD>
__device__ __forceinline__ void load_tile(Tile<HD>& t, const char* p, bool there, int lane) {
  const int g = lane >> 4, ql = lane & 15;
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, there ? kv4_tile_bytes(HD) : 0, 0x00027000);
  constexpr int NT = 2;   // non-temporal
#pragma unroll
  for (int l = 0; l < HD / 32; ++l)
    t.k[l] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane * 16, 1024 * l, NT);
#pragma unroll
  for (int l = 0; l < HD / 32; ++l)
    t.v[l] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane * 16, kv4_values_at(HD) + 1024 * l, NT);
  const int word = HD == 128 ? lane : (lane >> 5) * 16 + ql;   // block g, or g / 2, of row ql
  t.ks = __builtin_amdgcn_raw_buffer_load_b32(rsrc, word * 4, kv4_kscales_at(HD), 0);
  t.vs[0] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, g * 16, kv4_vscales_at(HD), 0);
  t.vs[1] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, g * 16, kv4_vscales_at(HD) + 64, 0);
}

// Context chunks of a sequence of T positions.
__device__ __forceinline__ int chunks_of(const Kv4AttnArgs& a, int T) {
  return max(1, min(a.n_chunks, (T + a.chunk_len - 1) / a.chunk_len));
}
__device__ __forceinline__ int context_of(const Kv4AttnArgs& a, int s) {
  return min(max(a.ctx_len[s], 0), a.max_ctx);
}
__device__ __forceinline__ int block_of(const Kv4AttnArgs& a, int s) {
  return a.block_len != nullptr ? min(max(a.block_len[s], 0), a.B) : a.B;
}

// Slot of query row r: r / G (rows are below 2^21, where this quotient is exact).
__device__ __forceinline__ int slot_of(const Kv4AttnArgs& a, int r) {
  return int((float(r) + 0.5f) * a.inv_g);
}

// 2^k, |k| <= 126.
__device__ __forceinline__ float power(int k) { return __uint_as_float(uint32_t(127 + k) << 23); }

// Four dims of an output row: o / l, o held times 2^k; zeros where no key was seen.
template <typename T>
__device__ __forceinline__ void store_out(T* dst, f32x4_t o, float l, int k) {
  const float inv = l == 0.f ? 0.f : power(-k) / l;
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<f32x4_t*>(dst) = f32x4_t{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  else
    *reinterpret_cast<uint2*>(dst) = make_uint2(to_bf2(o[0] * inv, o[1] * inv), to_bf2(o[2] * inv, o[3] * inv));
}

// Maximum over the four lane groups of a query.
__device__ __forceinline__ float groups_max(float x) {
  const uint32_t u = __float_as_uint(x);
  auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1])));
  p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// Running softmax of one 16-row query tile in a wave: lane (g, ql) keeps query ql.  o and l are
// relative to 2^m, m a score (base 2): the greatest so far, or one that the greatest is at most kSlack
// above.  Moving the reference costs a product an element of o, and with 16 queries a tile some query's
// greatest rises in most tiles, by little.
constexpr int kSlack = 4;
template <int HD>
struct State {
  f32x4_t o[HD / 16];    // O^T: dim 16dt + 4g + e of query ql, times 2^k (struct Unit)
  float m, l;            // l: this lane group's part of the sum
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt) o[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[dt][e] *= f;
  }
  // Another state of the same queries; the sums are then held times the lesser unit.
  __device__ __forceinline__ void join(const State& b, int k, int kb) {
    const float m1 = fmaxf(m, b.m), base = m1 == -INFINITY ? 0.f : m1;
    const float f = __builtin_amdgcn_exp2f(m - base), fb = __builtin_amdgcn_exp2f(b.m - base);
    const float u = power(min(k, kb) - k), ub = power(min(k, kb) - kb);
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[dt][e] = fmaf(o[dt][e] * f, u, b.o[dt][e] * fb * ub);
    l = fmaf(l, f, b.l * fb);
    m = m1;
  }
};

// Products of 64 keys (a lane's sixteen, -inf where masked) into the state's reference and sum; x
// leaves as exp2(c * x - m).
template <int HD>
__device__ __forceinline__ void soft_step(State<HD>& st, float (&x)[16], float c) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
  const float seen = groups_max(top) * c;
  if (__any(seen > st.m + float(kSlack))) {
    const float m = fmaxf(st.m, seen);
    const float f = m > st.m ? __builtin_amdgcn_exp2f(st.m - m) : 1.f;   // st.m -inf: 0
    st.l *= f;
    st.scale(f);
    st.m = m;
  }
  const float base = st.m == -INFINITY ? 0.f : st.m;   // no key yet
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c, -base));
    sum += x[i];
  }
  st.l += sum;
}

// Sums of values are held times a unit 2^k, |k| <= kMost, so that they stay within fp32 where their
// quotients do: k is -kMost from values on that are beyond 2^kTop in the unit at the start, so that sums
// of 2^30 keys at 2^kSlack are below 2^123.
//
// With bf16 queries a context factor, a
// probability times its value's scale, is fp16 in tiles whose scales are all within [2^kLow, 2^kHigh) in
// that unit: 11 bits, a rounding an eighth of the output's own, in one product with the codes.  With the
// reference's slack a factor is below 2^15, and the greatest probability's at least 2^kLow, so that
// the half step of fp16's subnormals, 2^-25, is 2^-23 of that one or less.
// Tiles whose scales lie further apart, or elsewhere, are left out and go into a state of their own
// behind the others, with factors of two bf16 terms, 16 bits of any size: a row of large values may have
// no weight, one of small values all of it, and 2^-23 of another's scale is then no small part of the
// output.  Those tiles are fetched twice: a context of nothing else takes 1.5 to 2.6 times as long (16 x 16
// queries over 512 to 8192 positions, 32 heads over 8: 98 us for 38.8).  Two terms in every tile took
// 47 us there, and 385 for 364 in the 64 contexts above.
constexpr int kMost = 40, kTop = 80, kLow = -2, kHigh = 11, kWindow = (kHigh - kLow) << 7;   // kWindow: in steps of bf16
template <typename T>
constexpr int kStart = sizeof(T) == 4 ? 0 : kMost;
struct Unit {
  int k;
  uint32_t low = 0;      // bits of the window's first scale, in both halves
};

// The window that a tile of nval rows sets: 16 times above the greatest scale of its first eight rows
// (the first row's, where there are fewer) it ends.
template <int HD>
__device__ __forceinline__ Unit window_of(const Tile<HD>& t, int nval) {
  u16x2_t m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, uint32_t(t.vs[0][i])));
  const int eight = __builtin_amdgcn_readfirstlane(max(m[0], m[1]));
  const int one = __builtin_amdgcn_readfirstlane(int(t.vs[0][0])) & 0xFFFF;
  Unit u;
  u.k = min(max(kHigh - 5 - (((nval < 8 ? one : eight) >> 7) - 127), -kMost), kMost);
  u.low = uint32_t(127 + kLow - u.k) * 0x00800080u;
  return u;
}

// A query tile as the operand of the products with keys: lane (g, ql) holds dims (HD/4)g + 8j .. of
// query ql, fp32 in three bf16 terms.  (The fp4 x fp8 products would take the keys as they lie and a
// bf16 query as two e4m3 terms, exactly, but drop what is 2^-11 of an instruction's greatest product
// or less, so that scores come out 2^-17 of sum |q k| off, and the log-sum-exps 1e-3.)
template <typename T, int HD>
struct Query {
  static constexpr int QT = sizeof(T) == 4 ? 3 : 1;   // bf16 terms of an element
  bf16x8_t f[HD / 32][QT];
  __device__ __forceinline__ void load(const T* p, int g) {   // p NULL: zeros
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) {
      if constexpr (sizeof(T) == 2) {
        f[j][0] = __builtin_bit_cast(bf16x8_t, u32x4{0, 0, 0, 0});
        if (p != nullptr) f[j][0] = __builtin_bit_cast(bf16x8_t, ld16(p + (HD / 4) * g + 8 * j));
      } else {
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (p != nullptr) load8(p + (HD / 4) * g + 8 * j, x);
        split8<QT>(x, f[j]);
      }
    }
  }
};

// Products of sub-tile st's sixteen keys with the queries: lane (g, ql) gets keys 4g .. 4g+3.
template <typename T, int HD, int NQ>
__device__ __forceinline__ void score(const Tile<HD>& t, int st, const Query<T, HD> (&q)[NQ], f32x4_t (&acc)[NQ]) {
  const float scale = __uint_as_float(((t.ks >> (8 * st)) & 255u) << 23);
#pragma unroll
  for (int n = 0; n < NQ; ++n) acc[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < HD / 32; ++j) {
    const bf16x8_t kf = kv4_bf16x8(t.key_word(st, j), scale);
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int k = 0; k < Query<T, HD>::QT; ++k)
        acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[n].f[j][k], acc[n], 0, 0, 0);
  }
}

// Values of a tile times factors p, in NT bf16 terms, into the sums.
template <int NT, int HD, int NQ>
__device__ __forceinline__ void values_bf16(const Tile<HD>& t, const float (&p)[NQ][16], State<HD> (&st)[NQ]) {
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    bf16x8_t pf[NQ][NT];
#pragma unroll
    for (int n = 0; n < NQ; ++n) split8<NT>(p[n] + 8 * ks, pf[n]);
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt) {
      const bf16x8_t vf = kv4_bf16x8(t.value_word(ks, dt), 1.f);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int k = 0; k < NT; ++k)
          st[n].o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n][k], st[n].o[dt], 0, 0, 0);
    }
  }
}

// A tile of the cache into the states of NQ query tiles; nval of its 64 keys count.  NARROW: factors of
// fp16; false, and the states as they were, where the tile does not take them.
template <typename T, int HD, int NQ, bool NARROW>
__device__ __forceinline__ bool tile_step(Tile<HD>& t, const Query<T, HD> (&q)[NQ], State<HD> (&st)[NQ],
                                          Unit& unit, int nval, int g, float c) {
  constexpr bool F32 = sizeof(T) == 4;
  float x[NQ][16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x4_t acc[NQ];
    score<T, HD, NQ>(t, i, q, acc);
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[n][4 * i + e] = acc[n][e];
  }
  // x[i] is key 32 * (i/8) + 8g + i%8.  Behind the last key anything may stand, in the values'
  // scales too: they become the window's first.
  auto hide = [&](int nval) {
    const int left = nval - 8 * g;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bool off = 32 * (i >> 3) + (i & 7) >= left;
#pragma unroll
      for (int n = 0; n < NQ; ++n) x[n][i] = off ? -INFINITY : x[n][i];
      const uint32_t w = t.vs[i >> 3][(i & 7) >> 1], keep = (i & 1) ? 0x0000FFFFu : 0xFFFF0000u;
      t.vs[i >> 3][(i & 7) >> 1] = off ? (w & keep) | (unit.low & ~keep) : w;
    }
  };
  if (nval < kTile) hide(nval);
  bool in = true;
  u16x2_t scale[8], most = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    scale[i] = __builtin_bit_cast(u16x2_t, uint32_t(t.vs[i >> 2][i & 3]));
    if constexpr (NARROW) scale[i] -= __builtin_bit_cast(u16x2_t, unit.low);   // those below the window wrap
    most = __builtin_elementwise_max(most, scale[i]);
  }
  if constexpr (NARROW) {
    in = !__any(max(most[0], most[1]) >= kWindow);
    if (!in) {
      hide(0);
#pragma unroll
      for (int i = 0; i < 8; ++i) scale[i] = u16x2_t{0, 0};
    }
  } else {
    if (__any((max(most[0], most[1]) >> 7) - 127 + unit.k >= kTop) && unit.k > -kMost) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) st[n].scale(power(-kMost - unit.k));
      unit.k = -kMost;
    }
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n) soft_step<HD>(st[n], x[n], c);
  const float up = power(unit.k);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    constexpr unsigned short kFirst = (127 + kLow) << 7;   // the window's first scale, in its unit
    const uint32_t w = __builtin_bit_cast(uint32_t, NARROW ? u16x2_t(scale[i] + u16x2_t{kFirst, kFirst}) : scale[i]);
    float s0 = lo_bf(w), s1 = hi_bf(w);
    if constexpr (!NARROW) {
      s0 *= up;
      s1 *= up;
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      x[n][2 * i] *= s0;
      x[n][2 * i + 1] *= s1;
    }
  }
  if constexpr (!NARROW) {
    values_bf16<F32 ? 3 : 2, HD, NQ>(t, x, st);
  } else {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      f16x8_t pf[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const f16x2_t p = __builtin_convertvector(f32x2_t{x[n][8 * ks + e], x[n][8 * ks + e + 1]}, f16x2_t);
          pf[n][e] = p[0];
          pf[n][e + 1] = p[1];
        }
#pragma unroll
      for (int dt = 0; dt < HD / 16; ++dt) {
        const f16x8_t vf = kv4_f16x8(t.value_word(ks, dt));
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          st[n].o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[n], st[n].o[dt], 0, 0, 0);
      }
    }
  }
  return in;
}

// The block's own keys and values in LDS: rows of keys, values by dim, zeros behind the last row up
// to a multiple of 32.
template <typename T, int HD>
struct BlockRows {
  static constexpr int E = 16 / sizeof(T);   // elements of 16 bytes
  T k[64][HD + E];
  T v[HD][64 + E];
};

// nbk of them into the state of a query tile, whose sums are held times `unit`; a query sees those up
// to `last`.
template <typename T, int HD>
__device__ __forceinline__ void block_step(const Query<T, HD>& q, const BlockRows<T, HD>& b, State<HD>& st,
                                           int nbk, int last, int lane, float c, float unit) {
  constexpr bool F32 = sizeof(T) == 4;
  const int g = lane >> 4, ql = lane & 15;
  float x[16];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    if (32 * (t >> 1) + 4 * (t & 1) < nbk) {
      const T* kr = b.k[32 * (t >> 1) + 8 * (ql >> 2) + 4 * (t & 1) + (ql & 3)];   // this lane's key
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) {
        if constexpr (F32) {
          float u[8];
          load8(kr + (HD / 4) * g + 8 * j, u);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            // The three terms are the query's element.
            const float w = (bf2f(q.f[j][0][e]) + bf2f(q.f[j][1][e])) + bf2f(q.f[j][2][e]);
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(u[e], w, acc, 0, 0, 0);
          }
        } else {
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8_t, ld16(kr + (HD / 4) * g + 8 * j)), q.f[j][0], acc, 0, 0, 0);
        }
      }
    }
    const int left = min(nbk, last + 1) - 8 * g;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[4 * t + e] = 32 * (t >> 1) + 4 * (t & 1) + e < left ? acc[e] : -INFINITY;
  }
  soft_step<HD>(st, x, c);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] *= unit;
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    if (32 * ks >= nbk) break;
    bf16x8_t pf[2];
    if constexpr (!F32) split8<2>(x + 8 * ks, pf);
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt) {
      const T* vr = b.v[16 * dt + ql] + 32 * ks + 8 * g;
      if constexpr (F32) {
        float v[8];
        load8(vr, v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], x[8 * ks + e], st.o[dt], 0, 0, 0);
      } else {
        const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, ld16(vr));
        st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[0], st.o[dt], 0, 0, 0);
        st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[1], st.o[dt], 0, 0, 0);
      }
    }
  }
}

// Greatest biased exponent of a thread's items of the block's values (255: one is no number).
template <bool F32, int NI>
__device__ __forceinline__ int block_top(const u32x4 (&v)[NI]) {
  u16x2_t w = {0, 0};
  uint32_t u = 0;
#pragma unroll
  for (int n = 0; n < NI; ++n)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (F32)
        u = max(u, uint32_t(v[n][k] & 0x7FFFFFFFu));
      else
        w = __builtin_elementwise_max(w, __builtin_bit_cast(u16x2_t, uint32_t(v[n][k] & 0x7FFF7FFFu)));
    }
  return F32 ? int(u >> 23) : max(w[0], w[1]) >> 7;
}
template <bool F32, int NI>
__device__ __forceinline__ void numbers_only(u32x4 (&v)[NI]) {
#pragma unroll
  for (int n = 0; n < NI; ++n)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t w = v[n][k];
      if ((w & 0x7F800000u) == 0x7F800000u) w &= F32 ? 0u : 0xFFFFu;
      if (!F32 && (w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
      v[n][k] = w;
    }
}
// The block's values (rows of v) that are no numbers into the state of a query tile: a query's sums
// become what those that it sees, up to slot `last`, make of them.
template <typename T, int HD>
__device__ __forceinline__ void no_numbers(State<HD>& st, const T* v, int64_t ld, int last, int nbk, int g) {
  for (int r = 0; r < nbk; ++r)
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x;
        if constexpr (sizeof(T) == 2)
          x = bf2f(v[r * ld + 16 * dt + 4 * g + e]);
        else
          x = v[r * ld + 16 * dt + 4 * g + e];
        const bool number = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
        st.o[dt][e] += number || r > last ? 0.f : x;
      }
}

template <typename T, int HD, int NQ, int W>
__global__ void __launch_bounds__(W * kWave) __attribute__((amdgpu_waves_per_eu(2)))
kv4_attn_kernel(Kv4AttnArgs a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NDT = HD / 16, kThreads = W * kWave;
  // The block's keys and values, later the waves' states.
  __shared__ __align__(16) union {
    BlockRows<T, HD> blk;
    float o[W][16][HD + 4];
  } pool;
  __shared__ float red_m[W][16], red_l[W][16];
  __shared__ int red_k[W];
  // The block's states, joined like a wave's: its keys and values take no part in a context's reference
  // or unit.
  __shared__ __align__(16) float blk_o[NQ][16][HD + 4];
  __shared__ float blk_m[NQ][16], blk_l[NQ][16];
  __shared__ int blk_k;
  __shared__ int blk_top[W];   // greatest biased exponent of the block's numbers; 256: not all are, by wave
  const int chunk = blockIdx.z, hk = blockIdx.x;
  const int G = a.G, R = G * a.B;
  const int s = blockIdx.y / a.n_groups, row0 = 16 * NQ * (blockIdx.y - s * a.n_groups);
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, ql = lane & 15;

  // Lane l keeps the place of the wave's l-th tile, tile wid + W * l of the chunk: read
  // beside the lengths, not behind them.  -1 for a page outside the pool, whose keys count as absent.
  const int t0 = chunk * (a.chunk_len >> 6);
  int page = -1;
  {
    const int t = t0 + wid + W * lane;
    if (a.page_table != nullptr) {
      if (t < a.max_pages) page = a.page_table[int64_t(s) * a.max_pages + t];
    } else if (a.kv_offsets != nullptr) {
      page = int(min(int64_t(a.kv_offsets[s] >> 6) + t, int64_t(INT32_MAX)));
    }
    if (page >= a.n_tiles) page = -1;
  }
  const int n_ctx = context_of(a, s);
  const int nc = chunks_of(a, n_ctx);
  if (chunk >= nc) return;
  const int blen = block_of(a, s);
  if (row0 >= G * blen) return;   // rows of no slot
  const int k_lo = min(n_ctx, t0 << 6), k_hi = min(n_ctx, k_lo + a.chunk_len);
  const int nct = (k_hi - k_lo + kTile - 1) / kTile;
  const int nbk = a.kb != nullptr && chunk == 0 ? blen : 0;   // keys of the block
  const char* head = a.tiles + int64_t(hk) * a.n_tiles * kv4_tile_bytes(HD);

  // Row of query ql of tile n (NULL behind the last).
  auto q_row = [&](int n) -> const T* {
    const int row = row0 + 16 * n + ql;
    const int slot = slot_of(a, row);
    return row < R ? static_cast<const T*>(a.q) + (int64_t(s) * a.B + slot) * a.ld_q +
                         (int64_t(hk) * G + (row - slot * G)) * HD
                   : nullptr;
  };
  // The block's rows, 16 bytes a thread and item, on their way before anything larger.
  constexpr int E = 16 / sizeof(T), P = HD / E, NI = 64 * P / kThreads;   // items of 64 rows
  u32x4 bw[2][NI];
  if (nbk > 0) {
    const T* kb = static_cast<const T*>(a.kb) + int64_t(s) * a.B * a.ld_kb + int64_t(hk) * HD;
    const T* vb = static_cast<const T*>(a.vb) + int64_t(s) * a.B * a.ld_vb + int64_t(hk) * HD;
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int e = n * kThreads + threadIdx.x, r = e / P, i = (e % P) * E;
      bw[0][n] = bw[1][n] = u32x4{0, 0, 0, 0};
      if (r < nbk) {
        bw[0][n] = ld16(kb + r * a.ld_kb + i);
        bw[1][n] = ld16(vb + r * a.ld_vb + i);
      }
    }
  }
  Query<T, HD> q[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) q[n].load(q_row(n), g);
  // This wave's tiles, its l-th into t.
  const int mine = (nct - wid + W - 1) / W;
  auto fetch = [&](Tile<HD>& t, int l) {
    const int at = l < mine ? __builtin_amdgcn_readlane(page, l) : -1;
    load_tile<HD>(t, head + int64_t(max(at, 0)) * kv4_tile_bytes(HD), at >= 0, lane);
  };
  Tile<HD> even, odd;
  fetch(even, 0);
  // A query tile's state to LDS.
  auto keep = [&](const State<HD>& b, float (&o)[16][HD + 4], float (&m)[16], float (&l)[16]) {
    float l_sum = b.l;
    l_sum += __shfl_xor(l_sum, 16, kWave);
    l_sum += __shfl_xor(l_sum, 32, kWave);
    if (g == 0) {
      m[ql] = b.m;
      l[ql] = l_sum;
    }
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) *reinterpret_cast<f32x4_t*>(&o[ql][16 * dt + 4 * g]) = b.o[dt];
  };
  // Through LDS into states by the wave that has the fewest tiles.
  if (nbk > 0) {
    const int rows = (nbk + 31) & ~31;
    // What is no number among the values leaves as 0: a product with a masked probability's 0 would be NaN.
    int top = block_top<F32, NI>(bw[1]), odd_ones = 0;
    if (__any(top == 255)) {
      odd_ones = 256;
      numbers_only<F32, NI>(bw[1]);
      top = block_top<F32, NI>(bw[1]);
    }
    int all = top;
    if (__any(top - 127 + kStart<T> >= kTop)) {   // below, the unit stays what it is
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) all = max(all, __shfl_xor(all, d, kWave));
    }
    all |= odd_ones;
    if (lane == 0) blk_top[wid] = all;
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int e = n * kThreads + threadIdx.x, r = e / P, i = (e % P) * E;
      if (r < rows) {
        st16(&pool.blk.k[r][i], bw[0][n]);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          if constexpr (F32)
            pool.blk.v[i + k][r] = __uint_as_float(bw[1][n][k]);
          else
            pool.blk.v[i + k][r] = T(bw[1][n][k / 2] >> (16 * (k & 1)));
        }
      }
    }
    lds_barrier();
    if (wid == nct % W) {
      int most = 0, odd = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        most = max(most, blk_top[w] & 255);
        odd |= blk_top[w] & 256;
      }
      most = __builtin_amdgcn_readfirstlane(most);
      odd = __builtin_amdgcn_readfirstlane(odd);
      const int k = most - 127 + kStart<T> >= kTop ? -kMost : kStart<T>;
      if (lane == 0) blk_k = k;
      const T* vb = static_cast<const T*>(a.vb) + int64_t(s) * a.B * a.ld_vb + int64_t(hk) * HD;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int last = a.causal != 0 ? slot_of(a, row0 + 16 * n + ql) : a.B;
        State<HD> b;
        b.clear();
        block_step<T, HD>(q[n], pool.blk, b, nbk, last, lane, a.scale_log2, power(k));
        if (odd != 0) no_numbers<T, HD>(b, vb, a.ld_vb, last, nbk, g);
        keep(b, blk_o[n], blk_m[n], blk_l[n]);
      }
    }
  }
  State<HD> st[NQ];
  Unit unit;
  unit.k = kStart<T>;
#pragma unroll
  for (int n = 0; n < NQ; ++n) st[n].clear();
  auto valid = [&](int l) {   // keys of the wave's l-th tile
    return __builtin_amdgcn_readlane(page, l) < 0 ? 0 : min(kTile, k_hi - k_lo - (wid + W * l) * kTile);
  };
  uint64_t left = 0;   // tiles that fp16 factors do not take
  fetch(odd, 1);                       // the next tile always on its way
  __builtin_amdgcn_sched_barrier(0);   // loads first, not sunk between the products
  if constexpr (!F32) unit = window_of<HD>(even, mine > 0 ? valid(0) : 0);
  for (int l = 0; l < mine; l += 2) {
    if (!tile_step<T, HD, NQ, !F32>(even, q, st, unit, valid(l), g, a.scale_log2)) left |= uint64_t(1) << l;
    if (l + 1 >= mine) break;
    fetch(even, l + 2);
    __builtin_amdgcn_sched_barrier(0);
    if (!tile_step<T, HD, NQ, !F32>(odd, q, st, unit, valid(l + 1), g, a.scale_log2)) left |= uint64_t(2) << l;
    fetch(odd, l + 3);
    __builtin_amdgcn_sched_barrier(0);
  }

  // The waves' states of a query tile side by side, then joined: four dims of a row a thread.
  const bool direct = nc == 1;   // nothing to join
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    if (n > 0 || nbk > 0) __syncthreads();
    keep(st[n], pool.o[wid], red_m[wid], red_l[wid]);
    int k = unit.k;
    if constexpr (!F32) {
      // The tiles that were left out, a query tile at a time, while this one's state lies in LDS: both at
      // once would spill in the loop above.
      if (left != 0) {
        const Query<T, HD> one[1] = {q[n]};
        State<HD> own[1], rest;
        own[0].clear();
        Unit wide;
        wide.k = kStart<T>;
        uint64_t todo = left;
        auto next = [&]() {   // kTile: none
          const int l = todo != 0 ? __builtin_ctzll(todo) : kTile;
          todo &= todo - 1;
          return l;
        };
        int l = next();
        fetch(even, l);
        while (l < kTile) {
          const int l1 = next();
          fetch(odd, l1);
          __builtin_amdgcn_sched_barrier(0);
          tile_step<T, HD, 1, false>(even, one, own, wide, valid(l), g, a.scale_log2);
          even = odd;
          l = l1;
        }
        asm volatile("" ::: "memory");   // read back, not kept in registers
        rest.m = st[n].m;
        rest.l = st[n].l;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) rest.o[dt] = *reinterpret_cast<const f32x4_t*>(&pool.o[wid][ql][16 * dt + 4 * g]);
        own[0].join(rest, wide.k, k);
        keep(own[0], pool.o[wid], red_m[wid], red_l[wid]);
        k = min(k, wide.k);
      }
    }
    if (lane == 0) red_k[wid] = k;
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * (HD / 4); e += kThreads) {
      const int qq = e / (HD / 4), dim = 4 * (e % (HD / 4));
      const int qr = row0 + 16 * n + qq, slot = slot_of(a, qr);
      if (slot >= blen) continue;
      float mm = red_m[0][qq];
#pragma unroll
      for (int w = 1; w < W; ++w) mm = fmaxf(mm, red_m[w][qq]);
      int k_min = red_k[0];        // the sums' unit: the least
#pragma unroll
      for (int w = 1; w < W; ++w) k_min = min(k_min, red_k[w]);
      if (nbk > 0) {
        mm = fmaxf(mm, blk_m[n][qq]);
        k_min = min(k_min, blk_k);
      }
      const float base = mm == -INFINITY ? 0.f : mm;
      f32x4_t o = {0.f, 0.f, 0.f, 0.f};
      float l = 0.f;
      auto join = [&](float m, float lw, int kw, const float* from) {
        const float f = __builtin_amdgcn_exp2f(m - base), u = power(k_min - kw);
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(from);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(v[i] * f, u, o[i]);
        l = fmaf(f, lw, l);
      };
#pragma unroll
      for (int w = 0; w < W; ++w) join(red_m[w][qq], red_l[w][qq], red_k[w], &pool.o[w][qq][dim]);
      if (nbk > 0) join(blk_m[n][qq], blk_l[n][qq], blk_k, &blk_o[n][qq][dim]);
      if (direct) {
        const int64_t orow = int64_t(s) * a.B + slot;
        const int h = hk * G + (qr - slot * G);
        store_out<T>(static_cast<T*>(a.out) + orow * a.ld_out + int64_t(h) * HD + dim, o, l, k_min);
        if (dim == 0 && a.lse != nullptr) a.lse[orow * a.nh + h] = (mm + __log2f(l)) * 0.6931471805599453f;
      } else {
        const int64_t p = ((int64_t(s) * a.nkv + hk) * a.n_chunks + chunk) * R + qr;
        *reinterpret_cast<f32x4_t*>(a.part_o + p * HD + dim) = o;
        if (dim == 0) *reinterpret_cast<float4*>(a.part_ml + 4 * p) = make_float4(mm, l, float(k_min), 0.f);
      }
    }
  }
}

// The chunks' partial outputs of a query row joined, where the sequence has more than one: threads
// (row, slice of the row's chunks, four dims), S slices a row and as many rows a workgroup as fit.
template <typename T, int HD, int S>
__global__ void __launch_bounds__(kJoinThreads) kv4_join_kernel(Kv4AttnArgs a) {
  constexpr int Q = HD / 4, N = kJoinThreads / (Q * S);
  __shared__ f32x4_t so[N * S][Q];
  __shared__ float sm[N * S], sl[N * S];
  __shared__ int sk[N * S];
  const int G = a.G, R = G * a.B;
  const int hk = blockIdx.y, s = blockIdx.z;
  const int nc = chunks_of(a, context_of(a, s));
  if (nc == 1) return;
  const int d = threadIdx.x % Q, at = threadIdx.x / Q, sl_ = at % S;
  const int qr = min(int(blockIdx.x) * N + at / S, R - 1);   // rows behind the last: the last's again
  const int k = slot_of(a, qr);
  if (N == 1 && k >= block_of(a, s)) return;
  const int64_t base = (int64_t(s) * a.nkv + hk) * a.n_chunks;
  float m = -INFINITY, l = 0.f;
  int ko = kMost;              // o is held times 2^ko, the least of the chunks'
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  for (int c = sl_; c < nc; c += S) {
    const int64_t p = (base + c) * R + qr;
    const float4 ml = *reinterpret_cast<const float4*>(a.part_ml + 4 * p);
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.part_o + p * HD + 4 * d);
    const float mn = fmaxf(m, ml.x);
    const float b = mn == -INFINITY ? 0.f : mn;
    const int kc = int(ml.z), kn = min(ko, kc);
    const float f0 = __builtin_amdgcn_exp2f(m - b), f1 = __builtin_amdgcn_exp2f(ml.x - b);
    const float u0 = power(kn - ko), u1 = power(kn - kc);
    l = fmaf(l, f0, ml.y * f1);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = fmaf(o[i] * f0, u0, v[i] * f1 * u1);
    m = mn;
    ko = kn;
  }
  so[at][d] = o;
  if (d == 0) {
    sm[at] = m;
    sl[at] = l;
    sk[at] = ko;
  }
  __syncthreads();
  if (sl_ != 0 || k >= block_of(a, s)) return;
  float mm = sm[at];
  ko = sk[at];
#pragma unroll
  for (int w = 1; w < S; ++w) {
    mm = fmaxf(mm, sm[at + w]);
    ko = min(ko, sk[at + w]);
  }
  const float b = mm == -INFINITY ? 0.f : mm;
  float sum = 0.f;
  o = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < S; ++w) {
    const float f = __builtin_amdgcn_exp2f(sm[at + w] - b), u = power(ko - sk[at + w]);
    sum = fmaf(f, sl[at + w], sum);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = fmaf(so[at + w][d][i] * f, u, o[i]);
  }
  const int64_t orow = int64_t(s) * a.B + k;
  const int h = hk * G + (qr - k * G);
  store_out<T>(static_cast<T*>(a.out) + orow * a.ld_out + int64_t(h) * HD + 4 * d,
               o, sum, ko);
  if (d == 0 && a.lse != nullptr) a.lse[orow * a.nh + h] = (mm + __log2f(sum)) * 0.6931471805599453f;
}

// Four waves a workgroup, of which a CU holds two so that one's start and join pass beside the other's
// tiles, where there is more than a round of eight waves' and contexts are short; long ones of
// unequal lengths leave CUs with one workgroup for longer.  us a call with eight and four, bf16, 16
// queries, 32 heads of 128 with keys of their own, lengths from a tenth on:
//   up to               300          2000         4000          8000          16384
//   12 contexts (1.5)                19, 17       28, 32        49, 53
//   16          (2)     13, 10       20, 16       36, 33        64, 65
//   24          (3)     19, 14       32, 24       45, 44        97, 100
//   64          (8)     52, 33 (500) 68, 50       127, 114      221, 209      363, 383
// and all of one length: 16 of 2000 31, 26, of 8000 100, 97; 12 of 8000 80, 79.
// The other forms, 16 queries, up to 300, 1000, 2000, 8000 positions, eight / four:
//   bf16, heads of 64, 32 heads, 16 contexts    8 / 7    10 / 9    13 / 13   34 / 34
//   fp32, heads of 64, 32 heads, 16 contexts   13 / 9    16 / 13   21 / 18   47 / 50
//   fp32, 32 heads, 16 contexts                21 / 14   26 / 20   33 / 28   77 / 78
//   bf16, 32 heads over 8, 32 contexts         21 / 14   25 / 20   32 / 27   69 / 73
//   bf16, 32 heads over 8, 128 contexts        79 / 47   97 / 63  120 / 83  252 / 235
bool few_waves(int64_t wgs, int max_ctx) {
  const int64_t rounds = wgs / device_cu_count();
  return wgs > device_cu_count() && max_ctx <= 2048 * std::min<int64_t>(rounds, 4);
}

template <typename T, int HD>
hipError_t attn_t(Kv4AttnArgs a, hipStream_t s) {
  const int R = a.G * a.B;
  // Two query tiles a wave where there are two (32-bit heads of 128 dims would spill).
  constexpr int MQ = sizeof(T) == 4 && HD == 128 ? 1 : 2;
  const int nq = R > 16 ? MQ : 1;
  a.n_groups = (R + 16 * nq - 1) / (16 * nq);
  const dim3 grid(a.nkv, unsigned(a.n_seq * a.n_groups), a.n_chunks);
  const bool few = few_waves(int64_t(grid.x) * grid.y * grid.z, a.max_ctx);
  const dim3 block((few ? kFewWaves : kWaves) * kWave);
  if (nq == 1 && few)
    hipLaunchKernelGGL((kv4_attn_kernel<T, HD, 1, kFewWaves>), grid, block, 0, s, a);
  else if (nq == 1)
    hipLaunchKernelGGL((kv4_attn_kernel<T, HD, 1, kWaves>), grid, block, 0, s, a);
  else if (few)
    hipLaunchKernelGGL((kv4_attn_kernel<T, HD, MQ, kFewWaves>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((kv4_attn_kernel<T, HD, MQ, kWaves>), grid, block, 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_chunks == 1) return e;
  // Two slices for up to eight chunks (four rows a workgroup at 128 dims), else a workgroup a row: the
  // call takes 32.1 us in the place of 33.3 for 2 contexts of 8192 positions, 32 heads over 8, B = 64
  // (2048 rows of two chunks), 22.7 in the place of 23.0 for 4 contexts, B = 16.
  constexpr int Q = HD / 4, most = kJoinThreads / Q, two = 2;
  const dim3 rows((R + most / two - 1) / (most / two), a.nkv, a.n_seq);
  if (a.n_chunks <= 8)
    hipLaunchKernelGGL((kv4_join_kernel<T, HD, two>), rows, dim3(kJoinThreads), 0, s, a);
  else
    hipLaunchKernelGGL((kv4_join_kernel<T, HD, most>), dim3(R, a.nkv, a.n_seq), dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// Chunks: as many as leave one round of workgroups over the card, of 512 positions at least (a tile a
// wave), and none for contexts of up to 1536.  us a call by chunk length, whole context last:
//   1 query, 32 heads over 8        512    1024   2048   whole
//     1024 positions                9.1                  8.4
//     1500                          9.4    10.5          9.7
//     4096                          9.5    10.5   13.2   16.8
//     16384 (256 workgroups: 512)  11.3    11.8   13.6   49.7
//   16 queries, 32 heads, 1 context
//     1024                          9.9                  9.1
//     4096 (256: 512)              12.2    12.1   14.1   17.3
//     16384 (256: 2048)            32.8    23.5   17.5   50.4
// From 1024 to 1536 positions chunks of 512 and the whole context are within 0.8 us of one another, now
// the one ahead and now the other (1 query, in a graph: 1024 9.4 and 9.0, 1300 9.8 and 10.4, 1500 9.9 and
// 10.4; 16 queries: 10.6 and 9.8, 11.2 and 11.3, 11.1 and 11.2); whole ones need no workspace.
// More than a round pays nowhere: 64 contexts of up to 16384 take 607, 493, 423, 389, 361 us in chunks
// of 1024, 2048, 4096, 8192, 16384 (2048 workgroups), 16 of 512 to 8192 in 256 workgroups 39, in twice
// and four times as many 45 and 48.
constexpr int kMinChunk = 512, kWholeCtx = 1536;
constexpr int kMaxChunk = kWaves * kWave * kTile;   // a lane keeps the place of one tile

static int64_t chunks_wanted(int n_seq, int nkv, int64_t q_rows, int max_ctx) {
  const int64_t wgs = std::max<int64_t>(1, int64_t(n_seq) * nkv * ((q_rows + 31) / 32));
  if (max_ctx <= kWholeCtx) return 1;
  const int64_t most = (int64_t(max_ctx) + kMinChunk - 1) / kMinChunk;
  return std::max<int64_t>(1, std::min(int64_t(device_cu_count()) / wgs, most));
}

void kv4_attn_plan(int n_seq, int nkv, int64_t q_rows, int hd, int max_ctx, int* n_chunks,
                   int* chunk_len) {
  const int64_t ctx = std::max(max_ctx, 1), want = chunks_wanted(n_seq, nkv, q_rows, max_ctx);
  int64_t len = (ctx + want - 1) / want;
  len = std::min<int64_t>((len + 511) / 512 * 512, kMaxChunk);
  *chunk_len = int(len);
  *n_chunks = int((ctx + len - 1) / len);
}

size_t kv4_attn_ws_bytes(int n_seq, int nkv, int64_t q_rows, int hd, int max_ctx) {
  // A shorter context takes as many chunks as are wanted for it, or as many of the greatest length
  // as it needs: neither grows as it gets shorter.
  const int64_t longest = (int64_t(max_ctx) + kMaxChunk - 1) / kMaxChunk;
  const int64_t most = std::max(chunks_wanted(n_seq, nkv, q_rows, max_ctx), longest);
  if (most <= 1) return 0;
  return size_t(n_seq) * nkv * size_t(most) * size_t(q_rows) * (hd + 4) * 4;
}

hipError_t launch_kv4_attention(bool bf16, int hd, const Kv4AttnArgs& args, void* ws, hipStream_t s) {
  Kv4AttnArgs a = args;
  if (a.n_seq <= 0) return hipSuccess;
  a.G = a.nh / a.nkv;
  a.inv_g = 1.f / float(a.G);
  const int64_t R = int64_t(a.G) * a.B;
  kv4_attn_plan(a.n_seq, a.nkv, R, hd, a.max_ctx, &a.n_chunks, &a.chunk_len);
  a.part_o = static_cast<float*>(ws);
  a.part_ml = a.part_o + size_t(a.n_seq) * a.nkv * a.n_chunks * R * hd;
  if (bf16) return hd == 128 ? attn_t<bf16_t, 128>(a, s) : attn_t<bf16_t, 64>(a, s);
  return hd == 128 ? attn_t<float, 128>(a, s) : attn_t<float, 64>(a, s);
}

}  // namespace hdf
