// First launch of a row's cut (row_cut.hpp).  Vector instructions bound it: of 27 an entry of a
// nucleus 11 for its bin and weight, 5 for the order, the others a thread's share of the masks, folds and
// lists; 1024 rows of 129280 16-bit logits take 130 us at 87% of the issue slots (reading them alone,
// greedy: 50), the top logits of 960 99 at 93%.  32 entries a thread: 64 were no faster (half the waves),
// 8 serve where rows are few.
#include "row_cut.hpp"

#include <type_traits>

namespace hdf {

constexpr int kHeadWaves = kHeadThreads / kWave;

// a * B + c of 24-bit a; B an inline constant.
template <int B>
__device__ __forceinline__ int mad24(int a, int c) {
  int d;
  asm("v_mad_i32_i24 %0, %1, %2, %3" : "=v"(d) : "v"(a), "n"(B), "v"(c));
  return d;
}

// bits * 2 + (x >= lo), which is false for NaN.
__device__ __forceinline__ uint32_t push_at_least(uint32_t bits, float x, float lo) {
  uint32_t d;
  asm("v_cmp_ge_f32 vcc, %2, %3\n\tv_addc_co_u32 %0, vcc, %1, %1, vcc"
      : "=v"(d)
      : "v"(bits), "v"(x), "v"(lo)
      : "vcc");
  return d;
}

// A chunk of a row: E entries a thread.
template <typename T, int E, bool TOP>
__global__ void __launch_bounds__(kHeadThreads)
row_head_kernel(CutArgs a, HeadArgs h) {
  constexpr int N = LogitRow<T>::N, G = E / N;
  __shared__ unsigned long long mass[kMassBins];
  __shared__ uint32_t count[kHeadThreads];
  __shared__ union {
    double d[kHeadWaves];
    float f[kHeadWaves];
    uint32_t i[kHeadWaves];
  } red;
  __shared__ uint32_t wave_n[kHeadWaves];
  __shared__ int best_col, end_bin;
  __shared__ uint16_t picked[kHeadThreads / kWave][kWave];
  const int64_t at = blockIdx.x / h.chunks, row = a.row0 + at;   // in the launch, in the call
  const int chunk = int(blockIdx.x - at * h.chunks), tid = threadIdx.x;
  const int lane = tid & 63, wid = tid >> 6;
  const LogitRow<T> r(static_cast<const T*>(a.z) + row * a.ld, a.V);
  const int j0 = chunk * G * kHeadThreads, nv = r.vectors();
  float x[G][N];
  if (r.inside(j0, G * kHeadThreads)) {   // all but a row's first and last chunk
#pragma unroll
    for (int g = 0; g < G; ++g) r.load_inside(j0 + g * kHeadThreads + tid, x[g]);
  } else {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int j = j0 + g * kHeadThreads + tid;
#pragma unroll
      for (int e = 0; e < N; ++e) x[g][e] = -INFINITY;
      if (j < nv) r.load_raw(j, x[g]);
    }
  }
  const RowSettings s = settings_of<TOP>(a, row);
  auto col = [&](int g, int e) { return r.column(j0 + g * kHeadThreads + tid) + e; };
  auto add = [](auto u, auto v) { return u + v; };
  auto most = [](float u, float v) { return fmaxf(u, v); };
  auto least = [](float u, float v) { return fminf(u, v); };
  // Unmasked entries (NaN is masked: no comparison holds for it), the greatest one.
  uint32_t live = 0;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < N; ++e)
      // (A ballot of "> -inf" comes out as "unequal or NaN" here: the least value instead.)
      live += uint32_t(__popcll(__ballot(x[g][e] >= kLeast)));
  if (live != uint32_t(kWave * E)) {   // of this wave
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < N; ++e) x[g][e] = x[g][e] >= kLeast ? x[g][e] : -INFINITY;
  }
  float top = -INFINITY;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < N; e += 2) top = max3(top, x[g][e], x[g][e + 1]);
  if (tid == 0) best_col = a.V, end_bin = 0;
  if (lane == 0) wave_n[wid] = live;
  const float m = block_fold<kHeadWaves>(top, red.f, most);
  uint32_t valid = 0;
#pragma unroll
  for (int w = 0; w < kHeadWaves; ++w) valid += wave_n[w];
  if (s.greedy) {
    if (top == m && m > -INFINITY) {
      int first = a.V;
#pragma unroll
      for (int g = G - 1; g >= 0; --g)
#pragma unroll
        for (int e = N - 1; e >= 0; --e) first = x[g][e] == m ? col(g, e) : first;
      atomicMin(&best_col, first);
    }
    __syncthreads();
  }

  // The list: all entries >= lo, lo a thread's greatest value such that `want` threads reach it; so
  // at least `want` entries do, and hardly more unless the great ones crowd into few threads (then
  // fewer threads are asked for).  A histogram of the 512 greatest values finds it.  Values far
  // below the chunk's greatest (masks by the type's lowest value) would widen its bins: they take
  // no part.  near: the same for the few entries a chunk has to contribute on the average.
  float lo = INFINITY, near = INFINITY;
  uint32_t listed = 0;
  if (!s.greedy && !s.open && valid > 0) {
    const float far = m - 64.f * fmaxf(s.t, 1.f);
    const bool in = top > far;
    const float low = block_fold<kHeadWaves>(in ? top : INFINITY, red.f, least);
    const float scale = float(kHeadThreads) / (m - low);
    const int mine = top == m ? 0 : int(fminf((m - top) * scale, float(kHeadThreads - 1)));
    int want = s.top_k > 0 ? int(fminf(float(s.top_k) + 4.f, float(kHeadThreads))) : h.cap;
    const int most_wanted = 2 * h.cap / 3 > 0 ? 2 * h.cap / 3 : 1;
    want = want < most_wanted ? want : most_wanted;
    const int few = s.top_k > 0 ? (s.top_k + h.chunks - 1) / h.chunks : 1;
    count[tid] = 0;
    __syncthreads();
    if (in) atomicAdd(&count[mine], 1u);
    __syncthreads();
    uint32_t all;
    const uint32_t upto = block_scan<kHeadWaves>(count[tid], red.i, all);
    count[tid] = upto;
    __syncthreads();
    const uint32_t first = in && mine > 0 ? count[mine - 1] : 0u;   // threads in the bins before
    if (s.top_k > 0)
      near = block_fold<kHeadWaves>(in && first < uint32_t(few) ? top : INFINITY, red.f, least);
    const bool every = valid <= uint32_t(h.cap);
    uint32_t bits = 0, before = 0;   // this thread's listed entries, the first one's bit the highest
    for (; want > 0; want /= 2) {
      lo = every ? kLeast
                 : block_fold<kHeadWaves>(in && first < uint32_t(want) ? top : INFINITY, red.f, least);
      bits = 0;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < N; ++e) bits = push_at_least(bits, x[g][e], lo);
      const uint32_t n = __popc(bits);
      before = block_scan<kHeadWaves>(n, red.i, listed) - n;
      if (listed <= uint32_t(h.cap)) break;
    }
    if (want == 0) {
      lo = INFINITY;
      listed = bits = before = 0;   // of the last attempt
    }
    // Few of a wave's entries are listed: brought together, a lane takes one, whose value is read
    // again, not picked from registers.
    uint64_t* list = h.list + (at * h.chunks + chunk) * h.cap;
    const uint32_t wave0 = read_lane(before, 0);
    const uint32_t in_wave = read_lane(before + uint32_t(__popc(bits)), kWave - 1) - wave0;
#pragma unroll 1
    for (uint32_t b0 = 0; b0 < in_wave; b0 += kWave) {
      uint32_t i = before - wave0 - b0;
      while (bits != 0 && i < uint32_t(kWave)) {
        const int q = E - __ffs(bits);
        bits &= bits - 1;
        picked[wid][i++] = uint16_t(q * kWave + lane);
      }
      before = wave0 + b0 + i;
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      if (b0 + lane < in_wave) {
        const int p = picked[wid][lane], q = p / kWave;
        const int c = r.column(j0 + q / N * kHeadThreads + wid * kWave + p % kWave) + q % N;
        list[wave0 + b0 + lane] = entry_key(r.raw(c), c);
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  }

  HeadStat st{m, s.greedy ? best_col : 0, valid == listed ? -INFINITY : lo, near, valid, listed, 0, 0, 0., 0.};
  if (s.binned && valid > 0) {
    const double k16 = 16. * s.c2;
    // Masked and far entries go to the last bins, which are not kept, all lanes to different ones:
    // cheaper than leaving them out.  (A bin is at least half a unit in the last place of m wide.)
    const float step = float(double(s.t) * kLog16);   // a bin's width
    const float end = m - step * float(kKeptBins + 4 + (lane & 31));
    if (fabs(double(m)) * k16 < 8e6 && step > 1e-37f && m - step * float(kMassBins - 1) >= kLeast) {
      for (int b = tid; b < kMassBins; b += kHeadThreads) mass[b] = 0;
      __syncthreads();
      const double c5 = mass_coefficient(kBits);
      const int top_bin = weight_bin(m, k16);
      st.top_bin = top_bin;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          int n;   // of 24 bits, top_bin - 1023 .. top_bin
          const uint64_t w = weight_in_bin(max2(x[g][e], end), k16, c5, n);
          auto* bin = reinterpret_cast<unsigned long long*>(reinterpret_cast<char*>(mass) +
                                                            mad24<-8>(n, 8 * top_bin));
          atomicAdd(bin, static_cast<unsigned long long>(w));
        }
      __syncthreads();
      for (int b0 = 0; b0 < kKeptBins; b0 += kHeadThreads) {   // whole waves
        const int b = b0 + tid;
        note_last(b < kKeptBins && mass[b < kKeptBins ? b : 0] != 0, b + 1, &end_bin);
      }
      __syncthreads();
      const int bins = end_bin;
      uint64_t* out = h.mass + (at * h.chunks + chunk) * kMassBins;
      for (int b = tid; b < bins; b += kHeadThreads) out[b] = mass[b];
      st.bins = bins;
    } else {
      st.bins = -1;
    }
  } else if (TOP && a.rest != nullptr && valid > listed) {
    // The others of the top logits: 32-bit exponentials, each to 2^-23 and, by its exponent's rounding,
    // 2^-24 of that at the most, 32 added in 32 bits; a logarithm off by 2e-6 at the worst, stored in 32
    // bits.  Relative to lo, which they stay below; where nearly all vanish so, to their greatest.  The
    // reference is what the rounded product of lo and log2(e) / T stands for, so that an entry
    // costs one product, rounded once; where that rounding is no small part of an octave, z - ref
    // first, in 64 bits.
    const float c2 = float(s.c2);
    for (int turn = 0; turn < 2; ++turn) {
      float ref = lo;
      if (turn == 1 || !(lo < INFINITY)) {
        float g_top = -INFINITY;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int e = 0; e < N; ++e) g_top = fmaxf(g_top, x[g][e] < lo ? x[g][e] : -INFINITY);
        ref = block_fold<kHeadWaves>(g_top, red.f, most);
      }
      const bool far = !(fmax(fabs(double(ref)), 1e-32) * s.c2 < 1e6);   // c2 past 1e38 too
      const float k = ref * c2;
      auto others = [&](auto is_far) __attribute__((always_inline)) {
        float f = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float t = decltype(is_far)::value ? float((double(x[g][e]) - double(ref)) * s.c2)
                                                    : fmaf(x[g][e], c2, -k);
            f += x[g][e] < lo ? __builtin_amdgcn_exp2f(t) : 0.f;
          }
        return f;
      };
      const float f = far ? others(std::true_type()) : others(std::false_type());
      st.rest_ref = far ? double(ref) : double(k) / double(c2);
      st.rest = block_fold<kHeadWaves>(double(f), red.d, add);
      if (st.rest > 1e-25 || !(lo < INFINITY)) break;
    }
  }
  if (tid == 0) h.stats[at * h.chunks + chunk] = st;
}

template <typename T>
static hipError_t launch_head(bool top, bool small, const CutArgs& a, const HeadArgs& h, hipStream_t s) {
  const dim3 grid(unsigned(a.rows) * h.chunks), wg(kHeadThreads);
  if (top && small)
    hipLaunchKernelGGL((row_head_kernel<T, 8, true>), grid, wg, 0, s, a, h);
  else if (top)
    hipLaunchKernelGGL((row_head_kernel<T, 32, true>), grid, wg, 0, s, a, h);
  else if (small)
    hipLaunchKernelGGL((row_head_kernel<T, 8, false>), grid, wg, 0, s, a, h);
  else
    hipLaunchKernelGGL((row_head_kernel<T, 32, false>), grid, wg, 0, s, a, h);
  return hipGetLastError();
}

hipError_t launch_row_head(bool bf16, bool top, bool small, const CutArgs& a, const HeadArgs& h, hipStream_t s) {
  return bf16 ? launch_head<bf16_t>(top, small, a, h, s) : launch_head<float>(top, small, a, h, s);
}

}  // namespace hdf
