// Attention of blocks of queries over the 4-bit cache (layout: kv4.hpp) and over the block's own
// keys and values, which are not quantised.
//
//   O = softmax(scale * Q [K, K_b]^T) [V, V_b],   lse = log of the softmax's sum
// G = n_heads / n_kv_heads query heads share a head of keys, so a (sequence, head of keys) has
// G * B query rows, row k * G + j being slot k of its j-th head.
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "kv4.hpp"

namespace hdf {

namespace {

constexpr int kTile = 64;
constexpr int kAttnWaves = 8;
constexpr int kAttnThreads = kAttnWaves * kWave;
constexpr int kMaxTiles = 512;            // tiles of a chunk
constexpr int kJoinThreads = 256;

typedef float f32x2_t __attribute__((ext_vector_type(2)));

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

__device__ __forceinline__ float load1(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ float load1(const float* p) { return *p; }

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

template <int HD>
__device__ __forceinline__ void load_tile(Tile<HD>& t, const char* p, int lane) {
  const int g = lane >> 4, ql = lane & 15;
#pragma unroll
  for (int l = 0; l < HD / 32; ++l) t.k[l] = ld_nt16(p + (l * 64 + lane) * 16);
#pragma unroll
  for (int l = 0; l < HD / 32; ++l) t.v[l] = ld_nt16(p + kv4_values_at(HD) + (l * 64 + lane) * 16);
  const int b = HD == 128 ? g : g >> 1;
  t.ks = *reinterpret_cast<const uint32_t*>(p + kv4_kscales_at(HD) + (16 * b + ql) * 4);
  t.vs[0] = ld16(p + kv4_vscales_at(HD) + 16 * g);
  t.vs[1] = ld16(p + kv4_vscales_at(HD) + 64 + 16 * g);
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

// Running softmax of one 16-row query tile in a wave: lane (g, ql) keeps query ql.
template <int HD>
struct State {
  f32x4_t o[HD / 16];    // O^T: dim 16dt + 4g + e of query ql
  float m, l;            // base-2 maximum; this lane group's part of the sum
};

// Scores of 64 keys (a lane's sixteen, -inf where masked) into the state's maximum and sum; sv
// leaves as the probabilities relative to the new maximum.
template <int HD>
__device__ __forceinline__ void soft_step(State<HD>& st, float (&sv)[4][4]) {
  float top = sv[0][0];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = fmaxf(top, sv[i][e]);
  top = fmaxf(top, __shfl_xor(top, 16, kWave));
  top = fmaxf(top, __shfl_xor(top, 32, kWave));
  const float m = fmaxf(st.m, top);
  if (__any(m > st.m)) {
    const float alpha = m > st.m ? __builtin_amdgcn_exp2f(st.m - m) : 1.f;   // st.m -inf: 0
    st.l *= alpha;
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) st.o[dt][e] *= alpha;
    st.m = m;
  }
  const float base = m == -INFINITY ? 0.f : m;   // no key yet
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sv[i][e] = __builtin_amdgcn_exp2f(sv[i][e] - base);
      sum += sv[i][e];
    }
  st.l += sum;
}

template <typename T, int HD>
__global__ void __launch_bounds__(kAttnThreads) kv4_attn_kernel(Kv4AttnArgs a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int QT = F32 ? 3 : 1;   // bf16 terms of a query's element
  constexpr int PT = F32 ? 3 : 2;   // ... of a probability
  constexpr int NJ = HD / 32;       // products over the dims of a score
  constexpr int NDT = HD / 16;
  __shared__ float red_o[kAttnWaves][16][HD + 1];
  __shared__ float red_m[kAttnWaves][16], red_l[kAttnWaves][16];
  __shared__ int32_t page[kMaxTiles];
  const int chunk = blockIdx.z, hk = blockIdx.x;
  const int G = a.nh / a.nkv, R = G * a.B;
  const int nqt = (R + 15) / 16;
  const int s = blockIdx.y / nqt, qt = blockIdx.y - s * nqt;
  const int n_ctx = context_of(a, s);
  if (chunk >= chunks_of(a, n_ctx)) return;
  const int blen = block_of(a, s);
  if (16 * qt >= G * blen) return;   // rows of no slot
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int g = lane >> 4, ql = lane & 15;
  const int k_lo = min(n_ctx, chunk * a.chunk_len), k_hi = min(n_ctx, k_lo + a.chunk_len);
  const int nct = (k_hi - k_lo + kTile - 1) / kTile;
  const int nbk = a.kb != nullptr && chunk == 0 ? blen : 0;   // keys of the block

  // The chunk's tiles; -1 for a page outside the pool, whose keys count as absent.
  for (int j = threadIdx.x; j < nct; j += kAttnThreads) {
    const int t = (k_lo >> 6) + j;
    const int64_t p = a.page_table != nullptr ? int64_t(a.page_table[int64_t(s) * a.max_pages + t])
                                              : int64_t(a.kv_offsets[s] >> 6) + t;
    page[j] = p >= 0 && p < a.n_tiles ? int32_t(p) : -1;
  }
  __syncthreads();
  const char* head = a.tiles + int64_t(hk) * a.n_tiles * kv4_tile_bytes(HD);

  // Query operand: lane (g, ql) holds dims (HD/4)g + 8j .. of query ql.
  const int row = 16 * qt + ql;
  const int slot = row / G;
  bf16x8_t qf[NJ][QT];
  float qx[F32 ? NJ : 1][8];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (row < R)
      load8(static_cast<const T*>(a.q) + (int64_t(s) * a.B + slot) * a.ld_q +
                (int64_t(hk) * G + (row - slot * G)) * HD + (HD / 4) * g + 8 * j, x);
    split8<QT>(x, qf[j]);
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qx[j][e] = x[e];
    }
  }

  State<HD> st;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) st.o[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  st.m = -INFINITY;
  st.l = 0.f;

  Tile<HD> cur, nxt;
  if (wid < nct) load_tile<HD>(cur, head + int64_t(max(page[wid], 0)) * kv4_tile_bytes(HD), lane);
  for (int i = wid; i < nct; i += kAttnWaves) {
    if (i + kAttnWaves < nct)
      load_tile<HD>(nxt, head + int64_t(max(page[i + kAttnWaves], 0)) * kv4_tile_bytes(HD), lane);
    const int nval = page[i] < 0 ? 0 : min(kTile, k_hi - k_lo - i * kTile);
    float sv[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float scale = __uint_as_float(((cur.ks >> (8 * t)) & 255u) << 23);
      f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const bf16x8_t kf = kv4_bf16x8(cur.key_word(t, j), scale);
#pragma unroll
        for (int n = 0; n < QT; ++n)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[j][n], acc, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = 32 * (t >> 1) + 8 * g + 4 * (t & 1) + e;
        sv[t][e] = key < nval ? acc[e] * a.scale_log2 : -INFINITY;
      }
    }
    soft_step<HD>(st, sv);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = cur.vs[ks][e >> 1];
        const float s_v = (e & 1) ? hi_bf(w) : lo_bf(w);
        const float x = sv[2 * ks + (e >> 2)][e & 3];
        p[e] = 32 * ks + 8 * g + e < nval ? x * s_v : 0.f;   // a scale of no row may be anything
      }
      bf16x8_t pf[PT];
      split8<PT>(p, pf);
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        const bf16x8_t vf = kv4_bf16x8(cur.value_word(ks, dt), 1.f);
#pragma unroll
        for (int n = 0; n < PT; ++n)
          st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], st.o[dt], 0, 0, 0);
      }
    }
    cur = nxt;
  }

  // The block's keys, by the wave that would take the next tile.
  if (nbk > 0 && wid == nct % kAttnWaves) {
    const T* kb = static_cast<const T*>(a.kb) + int64_t(s) * a.B * a.ld_kb + int64_t(hk) * HD;
    const T* vb = static_cast<const T*>(a.vb) + int64_t(s) * a.B * a.ld_vb + int64_t(hk) * HD;
    float sv[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int r = 32 * (t >> 1) + 8 * (ql >> 2) + 4 * (t & 1) + (ql & 3);   // this lane's key
      f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (r < nbk) load8(kb + r * a.ld_kb + (HD / 4) * g + 8 * j, x);
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], qx[j][e], acc, 0, 0, 0);
        } else {
          bf16x8_t kf[1];
          split8<1>(x, kf);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[0], qf[j][0], acc, 0, 0, 0);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = 32 * (t >> 1) + 8 * g + 4 * (t & 1) + e;
        const bool seen = key < nbk && (a.causal == 0 || key <= slot);
        sv[t][e] = seen ? acc[e] * a.scale_log2 : -INFINITY;
      }
    }
    soft_step<HD>(st, sv);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if (32 * ks >= nbk) break;
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = sv[2 * ks + (e >> 2)][e & 3];
      bf16x8_t pf[PT];
      if constexpr (!F32) split8<PT>(p, pf);
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int r = 32 * ks + 8 * g + e;
          x[e] = r < nbk ? load1(vb + r * a.ld_vb + 16 * dt + ql) : 0.f;
        }
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], p[e], st.o[dt], 0, 0, 0);
        } else {
          bf16x8_t vf[1];
          split8<1>(x, vf);
#pragma unroll
          for (int n = 0; n < PT; ++n)
            st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[0], pf[n], st.o[dt], 0, 0, 0);
        }
      }
    }
  }

  // The waves' states side by side, then joined.
  st.l += __shfl_xor(st.l, 16, kWave);
  st.l += __shfl_xor(st.l, 32, kWave);
  if (g == 0) {
    red_m[wid][ql] = st.m;
    red_l[wid][ql] = st.l;
  }
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int e = 0; e < 4; ++e) red_o[wid][ql][16 * dt + 4 * g + e] = st.o[dt][e];
  __syncthreads();
  const bool direct = a.n_chunks == 1;
  for (int e = threadIdx.x; e < 16 * (HD / 2); e += kAttnThreads) {
    const int qq = e / (HD / 2), dim = 2 * (e - qq * (HD / 2));
    const int qr = 16 * qt + qq, k = qr / G;
    if (k >= blen) continue;
    float mm = red_m[0][qq];
#pragma unroll
    for (int w = 1; w < kAttnWaves; ++w) mm = fmaxf(mm, red_m[w][qq]);
    float o0 = 0.f, o1 = 0.f, l = 0.f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
      const float f = red_m[w][qq] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(red_m[w][qq] - mm);
      o0 += f * red_o[w][qq][dim];
      o1 += f * red_o[w][qq][dim + 1];
      l += f * red_l[w][qq];
    }
    if (direct) {
      const int64_t orow = int64_t(s) * a.B + k;
      const int h = hk * G + (qr - k * G);
      const float inv = l == 0.f ? 0.f : 1.f / l;   // no key: zeros
      T* dst = static_cast<T*>(a.out) + orow * a.ld_out + int64_t(h) * HD + dim;
      if constexpr (F32)
        *reinterpret_cast<float2*>(dst) = make_float2(o0 * inv, o1 * inv);
      else
        *reinterpret_cast<uint32_t*>(dst) = to_bf2(o0 * inv, o1 * inv);
      if (dim == 0 && a.lse != nullptr)
        a.lse[orow * a.nh + h] = (mm + __log2f(l)) * 0.6931471805599453f;
    } else {
      const int64_t p = ((int64_t(s) * a.nkv + hk) * a.n_chunks + chunk) * R + qr;
      *reinterpret_cast<float2*>(a.part_o + p * HD + dim) = make_float2(o0, o1);
      if (dim == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * p) = make_float2(mm, l);
    }
  }
}

// The chunks' partial outputs of a query row joined: a workgroup a row, its threads (slice of the
// chunks, four dims).
template <typename T, int HD>
__global__ void __launch_bounds__(kJoinThreads) kv4_join_kernel(Kv4AttnArgs a) {
  constexpr int Q = HD / 4, S = kJoinThreads / Q;
  __shared__ float4 so[S][Q];
  __shared__ float sm[S], sl[S];
  const int G = a.nh / a.nkv, R = G * a.B;
  const int qr = blockIdx.x, hk = blockIdx.y, s = blockIdx.z;
  const int k = qr / G;
  if (k >= block_of(a, s)) return;
  const int nc = chunks_of(a, context_of(a, s));
  const int d = threadIdx.x % Q, sl_ = threadIdx.x / Q;
  const int64_t base = (int64_t(s) * a.nkv + hk) * a.n_chunks;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int c = sl_; c < nc; c += S) {
    const int64_t p = (base + c) * R + qr;
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * p);
    const float4 v = *reinterpret_cast<const float4*>(a.part_o + p * HD + 4 * d);
    const float mn = fmaxf(m, ml.x);
    const float b = mn == -INFINITY ? 0.f : mn;
    const float f0 = __builtin_amdgcn_exp2f(m - b), f1 = __builtin_amdgcn_exp2f(ml.x - b);
    l = l * f0 + ml.y * f1;
    o.x = o.x * f0 + v.x * f1;
    o.y = o.y * f0 + v.y * f1;
    o.z = o.z * f0 + v.z * f1;
    o.w = o.w * f0 + v.w * f1;
    m = mn;
  }
  so[sl_][d] = o;
  if (d == 0) {
    sm[sl_] = m;
    sl[sl_] = l;
  }
  __syncthreads();
  if (sl_ != 0) return;
  float mm = sm[0];
#pragma unroll
  for (int w = 1; w < S; ++w) mm = fmaxf(mm, sm[w]);
  const float b = mm == -INFINITY ? 0.f : mm;
  float sum = 0.f;
  o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < S; ++w) {
    const float f = __builtin_amdgcn_exp2f(sm[w] - b);
    sum += f * sl[w];
    o.x += f * so[w][d].x;
    o.y += f * so[w][d].y;
    o.z += f * so[w][d].z;
    o.w += f * so[w][d].w;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t orow = int64_t(s) * a.B + k;
  const int h = hk * G + (qr - k * G);
  T* dst = static_cast<T*>(a.out) + orow * a.ld_out + int64_t(h) * HD + 4 * d;
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<float4*>(dst) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else
    *reinterpret_cast<uint2*>(dst) = make_uint2(to_bf2(o.x * inv, o.y * inv), to_bf2(o.z * inv, o.w * inv));
  if (d == 0 && a.lse != nullptr) a.lse[orow * a.nh + h] = (mm + __log2f(sum)) * 0.6931471805599453f;
}

template <typename T, int HD>
hipError_t attn_t(const Kv4AttnArgs& a, hipStream_t s) {
  const int R = a.nh / a.nkv * a.B;
  const dim3 grid(a.nkv, unsigned(a.n_seq * ((R + 15) / 16)), a.n_chunks);
  hipLaunchKernelGGL((kv4_attn_kernel<T, HD>), grid, dim3(kAttnThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_chunks == 1) return e;
  hipLaunchKernelGGL((kv4_join_kernel<T, HD>), dim3(R, a.nkv, a.n_seq), dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

void kv4_attn_plan(int n_seq, int nkv, int64_t q_rows, int hd, int max_ctx, int* n_chunks,
                   int* chunk_len) {
  const int64_t wgs = int64_t(n_seq) * nkv * ((q_rows + 15) / 16);
  const int64_t want = std::max<int64_t>(1, 2 * int64_t(device_cu_count()) / std::max<int64_t>(1, wgs));
  int64_t len = (std::max(max_ctx, 1) + want - 1) / want;
  len = std::min<int64_t>(std::max<int64_t>((len + 511) / 512 * 512, 512), kMaxTiles * kTile);
  *chunk_len = int(len);
  *n_chunks = int((std::max(max_ctx, 1) + len - 1) / len);
}

size_t kv4_attn_ws_bytes(int n_seq, int nkv, int64_t q_rows, int hd, int max_ctx) {
  // A shorter context has no more chunks: at most as many as fill the card, or one each 512 positions.
  int n, len;
  kv4_attn_plan(n_seq, nkv, q_rows, hd, max_ctx, &n, &len);
  const int64_t wgs = int64_t(n_seq) * nkv * ((q_rows + 15) / 16);
  const int64_t want = std::max<int64_t>(1, 2 * int64_t(device_cu_count()) / std::max<int64_t>(1, wgs));
  const int64_t most = std::max<int64_t>(n, std::min<int64_t>(want, (int64_t(std::max(max_ctx, 1)) + 511) / 512));
  if (most <= 1) return 0;
  return size_t(n_seq) * nkv * size_t(most) * size_t(q_rows) * (hd + 2) * 4;
}

hipError_t launch_kv4_attention(bool bf16, int hd, const Kv4AttnArgs& args, void* ws, hipStream_t s) {
  Kv4AttnArgs a = args;
  if (a.n_seq <= 0) return hipSuccess;
  const int64_t R = int64_t(a.nh / a.nkv) * a.B;
  kv4_attn_plan(a.n_seq, a.nkv, R, hd, a.max_ctx, &a.n_chunks, &a.chunk_len);
  a.part_o = static_cast<float*>(ws);
  a.part_ml = a.part_o + size_t(a.n_seq) * a.nkv * a.n_chunks * R * hd;
  if (bf16) return hd == 128 ? attn_t<bf16_t, 128>(a, s) : attn_t<bf16_t, 64>(a, s);
  return hd == 128 ? attn_t<float, 128>(a, s) : attn_t<float, 64>(a, s);
}

}  // namespace hdf
