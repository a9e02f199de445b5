// Rows of logits cut to the head of their distribution: truncated draws (temperature, top-k,
// top-p, min-p), the verification of drafts under such distributions, and a row's top logits.
//
// The entries of a row are ordered by value, ties to the lowest column; masked ones (-inf) have
// no place.  With m the greatest and w_v = e^((z_v - m) / T), the kept entries are the first
//     n = min(n_k, n_p, n_m):  n_k = top_k;  n_p = the fewest of those whose weights sum to top_p
//     of the first n_k entries' sum;  n_m = those with w_v >= min_p.
// The draw is the lowest column whose running sum of kept weights, in column order, passes
// u times their whole.  Sums are 64-bit throughout: a cut or a draw falls between neighbours that
// may be 1e-6 of the whole apart.
#include "kernels.hpp"
#include "rows.hpp"

namespace hdf {

constexpr int kCutThreads = 1024;
constexpr int kCutWaves = kCutThreads / kWave;
constexpr int kBins = 2 * kCutThreads;
constexpr int kListMax = 2 * kCutThreads;      // entries sorted at once
constexpr int kMaxGroups = (1 << kColumnBits) / (4 * kCutThreads) + 1;
constexpr double kMassUnit = 1.0 / 8796093022208.0;   // 2^-43: sums of up to 2^20 weights fit 64 bits
constexpr uint64_t kKeyTop = (uint64_t(1) << (32 + kColumnBits)) - 1;

// First launch: workgroup (row, chunk) keeps a chunk of a row in registers, lists its greatest
// entries and, where the cut depends on the others, sums them up: in a histogram of weights for a
// nucleus (top_p without top_k), in one sum otherwise.  Second launch: a workgroup a row finds how
// far down the order the cut lies and sorts the listed entries up to there; a cut below the lists
// takes one more pass over the row.
constexpr int kHeadThreads = 512;
constexpr int kHeadWaves = kHeadThreads / kWave;
constexpr int kMaxChunks = 66;
constexpr float kLeast = -3.402823466e38f;   // the least finite value

// The nucleus histogram: bins of 1/16 octave of weight.  Entry z has t = 16 z log2(e) / T, bin
// n = rint(t) and within it the weight 2^((t - n) / 16), 0.978 .. 1.022, as a multiple of 2^-48;
// integers, so that the sums do not depend on their order.  1024 bins from the chunk's greatest
// entry down; entries more than 62 octaves below it weigh nothing.
constexpr int kMassBins = 1024;

struct HeadStat {
  float best;        // greatest value, its lowest column
  int32_t best_col;
  float floor;       // every entry >= floor is listed (-inf: all are)
  float near;        // a value that at least `few` entries reach (HeadArgs)
  uint32_t valid;    // unmasked entries, listed ones
  uint32_t listed;
  int32_t top_bin;   // bin of the greatest value, and how many bins from it down are stored
  int32_t bins;      // (-1: values beyond the bins' range)
  double rest_ref;   // rest: sum of e^((z - rest_ref) / T) over the unlisted entries
  double rest;
};

struct CutNote;   // what one phase of a row's cut leaves for the next

struct HeadArgs {
  int chunks, cap, vectors;   // of a row; entries a chunk may list; vectors of a chunk
  uint64_t* list;             // [rows][chunks][cap]
  HeadStat* stats;            // [rows][chunks]
  uint64_t* mass;             // [rows][chunks][kMassBins]
  CutNote* notes;             // [rows]
};

// A row's settings.
struct RowSettings {
  float t, top_p, min_p;
  int top_k;
  bool greedy, nucleus, open;
  double inv_t, c2;
};
template <bool TOP>
__device__ __forceinline__ RowSettings settings_of(const CutArgs& a, int64_t row) {
  RowSettings s;
  const int64_t i = TOP ? 0 : row / a.per;
  s.t = !TOP && a.ts != nullptr ? a.ts[i] : a.t;
  s.greedy = !(s.t > 0.f);
  s.top_k = TOP ? a.K : a.ks != nullptr ? a.ks[i] : a.k;
  s.top_p = TOP ? 1.f : a.ps != nullptr ? a.ps[i] : a.p;
  s.min_p = TOP ? 0.f : a.mps != nullptr ? a.mps[i] : a.mp;
  if (!TOP && s.top_k >= a.V) s.top_k = 0;
  s.nucleus = !s.greedy && s.top_k <= 0 && s.top_p < 1.f;
  s.open = !s.greedy && s.top_k <= 0 && !s.nucleus && !(s.min_p > 0.f);
  s.inv_t = s.greedy ? 1. : 1. / double(s.t);
  s.c2 = 1.4426950408889634074 * s.inv_t;
  return s;
}

// Bin of a value and the weight within it (a multiple of 2^-48 in the low bits).  The magic
// constants round to an integer in the low bits of the sum; the series is that of 2^(g / 16),
// |g| <= 1/2, whose first dropped term is 0.022^7 / 7! = 4e-16.
__device__ __forceinline__ int weight_bin(float z, double k16) {
  const double t = fma(double(z), k16, 6755399441055744.);   // 1.5 * 2^52
  return int(uint32_t(__builtin_bit_cast(uint64_t, t)));
}
__device__ __forceinline__ uint64_t weight_in_bin(float z, double k16, int& n) {
  const double t = fma(double(z), k16, 6755399441055744.);
  n = int(uint32_t(__builtin_bit_cast(uint64_t, t)));
  const double g = fma(double(z), k16, -(t - 6755399441055744.));
  constexpr double c = 0.69314718055994530942 / 16.;
  double p = c * c * c * c * c * c / 720.;
  p = fma_k(p, g, c * c * c * c * c / 120.);
  p = fma_k(p, g, c * c * c * c / 24.);
  p = fma_k(p, g, c * c * c / 6.);
  p = fma_k(p, g, c * c / 2.);
  p = fma_k(p, g, c);
  p = fma_k(p, g, 17.);   // 16 + 1: a unit of 16's last place is 2^-48
  return __builtin_bit_cast(uint64_t, p) - 0x4030000000000000ull;
}

template <int NT, bool SEARCH = true>
struct CutShared {
  static constexpr int W = NT / kWave;
  union {
    struct {
      uint64_t list[kListMax];
      union {
        struct {
          uint64_t mass[SEARCH ? kBins : 1];
          uint32_t count[SEARCH ? kBins : 1];
        };
        double weight[kListMax];
      };
    };
    double group[W][kMaxGroups];
  };
  double chunk[kMaxChunks];
  struct {
    int listed, top_bin, bins;
    double rest_ref, rest;
  } part[kMaxChunks];   // of the chunks' statistics
  union {
    double d[W];
    uint64_t u[W];
    uint32_t i[W];
    float f[W];
  } red;
  uint64_t before, best;
  double sum;
  float floor, near;
  uint32_t n, valid, listed;
  int pick, last, top_bin, bins;
};

// Calls f(group, value, column) for every unmasked entry of vectors j0 .. j1-1 of the row; group g
// is the g-th run of NT of them, and after(g) follows a group's entries with all lanes together.  A
// thread has AHEAD entries in flight.
template <int NT, int AHEAD, typename T, typename F, typename G>
__device__ __forceinline__ void each_entry(const LogitRow<T>& r, int j0, int j1, F f, G after) {
  constexpr int N = LogitRow<T>::N, Q = AHEAD / N;
  for (int b = 0; j0 + b < j1; b += Q * NT) {
    float x[Q][N];
    if (j0 + b + Q * NT <= j1 && r.inside(j0 + b, Q * NT)) {
#pragma unroll
      for (int q = 0; q < Q; ++q) r.load_inside(j0 + b + q * NT + int(threadIdx.x), x[q]);
    } else {
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int j = j0 + b + q * NT + int(threadIdx.x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[q][e] = -INFINITY;
        if (j < j1) r.load_raw(j, x[q]);
      }
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int g = b / NT + q;
      const int c = r.column(j0 + g * NT + int(threadIdx.x));
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (x[q][e] > -INFINITY) f(g, x[q][e], c + e);   // false for NaN
      if (j0 + g * NT < j1) after(g);
    }
  }
}
template <typename T, typename F>
__device__ __forceinline__ void each_entry(const LogitRow<T>& r, F f) {
  each_entry<kCutThreads, 16>(r, 0, r.vectors(), f, [](int) {});
}

// The list's first n entries (n <= kListMax) from the greatest key down: a bitonic sort whose
// exchanges within 64 entries stay in a wave's registers.
template <int NT>
__device__ __forceinline__ void sort_list(uint64_t* list, int n) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  int P = 64;
  while (P < n) P *= 2;
  for (int i = n + int(threadIdx.x); i < P; i += NT) list[i] = 0;
  __syncthreads();
  auto in_waves = [&](int from, int to) {   // sizes from .. to, their exchanges of up to 32 apart
    for (int s = wid; s * 64 < P; s += NT / kWave) {
      const int i = s * 64 + lane;
      uint64_t k = list[i];
      for (int size = from; size <= to; size *= 2)
        for (int d = size / 2 < 32 ? size / 2 : 32; d > 0; d /= 2) {
          const uint64_t o = __shfl_xor(k, d, kWave);
          const bool greater = ((lane & d) == 0) == ((i & size) == 0);
          k = (o > k) == greater ? o : k;
        }
      list[i] = k;
    }
    __syncthreads();
  };
  in_waves(2, 64);
  for (int size = 128; size <= P; size *= 2) {
    for (int d = size / 2; d >= 64; d /= 2) {
      for (int t = threadIdx.x; t < P / 2; t += NT) {
        const int i = 2 * d * (t / d) + t % d;
        const uint64_t a = list[i], b = list[i + d];
        if ((a < b) == ((i & size) == 0)) {
          list[i] = b;
          list[i + d] = a;
        }
      }
      __syncthreads();
    }
    in_waves(size, size);
  }
}

// First-level bin of a value below the row's greatest one: 64 bins a unit of (m - z) / T, so
// monotone in the value.
__device__ __forceinline__ int value_bin(float z, float m, float scale) {
  return z == m ? 0 : int(fminf((m - z) * scale, float(kBins - 1)));
}

// Least order key of a value in (-inf, m] for which `holds` is true, which it is from there on and
// for m: each wave for itself, 64 candidates a round.
template <typename F>
__device__ __forceinline__ uint32_t least_value_key(float m, F holds) {
  uint32_t l = 0x007FFFFFu, h = f32_order_key(m);   // the key of -inf: not among the candidates
  while (h - l > 1) {
    const uint32_t step = (h - l - 1) / 64 + 1;
    const uint64_t k = uint64_t(l) + uint64_t(step) * ((threadIdx.x & 63) + 1);
    const bool in = k < h && holds(f32_from_order_key(uint32_t(k)));
    const unsigned long long is = __ballot(in);
    // Lanes past h count as true: the first true one bounds the answer from above.
    const unsigned long long past = __ballot(k >= h);
    const unsigned long long any = is | past;
    const int f = any != 0ull ? __ffsll(static_cast<long long>(any)) - 1 : 64;
    const uint64_t up = uint64_t(l) + uint64_t(step) * (f + 1);
    l += step * uint32_t(f);
    h = up < h ? uint32_t(up) : h;
  }
  return h;
}

// Key of the entry with which the running sum, in order, of ones (BY_MASS false) or weights over
// the entries with keys >= floor reaches `target`; the last of them if rounding leaves none.
// Histograms of 2048 bins over ever smaller ranges of the order, until a bin's entries fit the
// list: the first by value, further ones by key, where the last range is one key.  A caller that
// knows the range of keys and the sum `above` it starts there (lo > 0).
template <bool BY_MASS, typename T>
__device__ uint64_t select_entry(const LogitRow<T>& r, double target, uint64_t floor, float m,
                                 double c2, float scale, CutShared<kCutThreads>& sh, uint64_t lo = 0,
                                 uint64_t hi = kKeyTop, double above = 0.) {
  auto shift_of = [&]() {
    int sh_ = 0;
    while (((hi - lo) >> sh_) >= uint64_t(kBins)) ++sh_;
    return sh_;
  };
  int shift = lo > 0 ? shift_of() : -1, bin = 0;   // shift -1: the bins by value
  for (;;) {
    for (int b = threadIdx.x; b < kBins; b += kCutThreads) {
      sh.count[b] = 0;
      sh.mass[b] = 0;
    }
    if (threadIdx.x == 0) sh.pick = -1, sh.last = 0;
    __syncthreads();
    auto bin_of = [&](float z, uint64_t k) {
      return shift < 0 ? value_bin(z, m, scale) : int((hi - k) >> shift);
    };
    each_entry(r, [&](int, float z, int c) {
      const uint64_t k = entry_key(z, c);
      if (k < floor || k < lo || k > hi) return;
      const int b = bin_of(z, k);
      atomicAdd(&sh.count[b], 1u);
      if (BY_MASS)
        atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]),
                  static_cast<unsigned long long>(entry_weight(z, m, c2) / kMassUnit + 0.5));
    });
    __syncthreads();
    const int b0 = 2 * threadIdx.x;
    const uint64_t v0 = BY_MASS ? sh.mass[b0] : sh.count[b0];
    const uint64_t v1 = BY_MASS ? sh.mass[b0 + 1] : sh.count[b0 + 1];
    uint64_t whole;
    const uint64_t at1 = block_scan<kCutWaves>(v0 + v1, sh.red.u, whole);
    const double unit = BY_MASS ? kMassUnit : 1.;
    auto reached = [&](uint64_t s) { return above + double(s) * unit >= target; };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint64_t after = h == 0 ? at1 - v1 : at1, before = after - (h == 0 ? v0 : v1);
      if (reached(after) && !reached(before)) {
        sh.pick = b0 + h;
        sh.before = before;
      }
      if (sh.count[b0 + h] != 0) atomicMax(&sh.last, b0 + h);
    }
    __syncthreads();
    if (sh.pick < 0 && int(threadIdx.x) == sh.last / 2) {
      sh.before = (sh.last & 1) ? at1 - v1 : at1 - v1 - v0;
    }
    bin = sh.pick < 0 ? sh.last : sh.pick;
    __syncthreads();
    above += double(sh.before) * unit;
    const uint32_t here = sh.count[bin];
    if (threadIdx.x == 0) sh.n = 0, sh.pick = kListMax;
    __syncthreads();
    if (here <= uint32_t(kListMax)) {
      each_entry(r, [&](int, float z, int c) {
        const uint64_t k = entry_key(z, c);
        if (k < floor || k < lo || k > hi || bin_of(z, k) != bin) return;
        sh.list[atomicAdd(&sh.n, 1u)] = k;
      });
      __syncthreads();
      const int n = int(sh.n);
      sort_list<kCutThreads>(sh.list, n);
      int at;
      if (BY_MASS) {
        const int i = 2 * threadIdx.x;
        const double w0 = i < n ? entry_weight(entry_logit(sh.list[i]), m, c2) : 0.;
        const double w1 = i + 1 < n ? entry_weight(entry_logit(sh.list[i + 1]), m, c2) : 0.;
        double all;
        const double sum = block_scan<kCutWaves>(w0 + w1, sh.red.d, all);
        if (i < n && above + (sum - w1) >= target) atomicMin(&sh.pick, i);
        if (i + 1 < n && above + sum >= target) atomicMin(&sh.pick, i + 1);
        __syncthreads();
        at = min(sh.pick, n - 1);
      } else {
        at = min(max(int(target - above) - 1, 0), n - 1);
      }
      const uint64_t k = sh.list[at];
      __syncthreads();
      return k;
    }
    if (shift < 0) {
      // The bin's range of keys: value_bin falls as keys rise.
      auto least = [&](int b) {
        return uint64_t(least_value_key(m, [&](float z) { return value_bin(z, m, scale) <= b; }))
               << kColumnBits;
      };
      lo = least(bin);
      hi = bin == 0 ? kKeyTop : least(bin - 1) - 1;
    } else {
      hi -= uint64_t(bin) << shift;
      const uint64_t l = hi - ((uint64_t(1) << shift) - 1);
      lo = l > lo ? l : lo;
    }
    shift = shift_of();
    __syncthreads();
  }
}

// The weights of a row's kept entries (keys >= cut) among vectors j0 .. j1-1, a group and wave a
// sum in sh.group; returns their whole, `run` this thread's group's running sum and `mine` its own.
template <int NT, bool S, typename T>
__device__ __forceinline__ double kept_masses(const LogitRow<T>& r, int j0, int j1, uint64_t cut,
                                              float m, double c2, CutShared<NT, S>& sh,
                                              uint32_t& kept,
                                              uint64_t& low, double& run, double& mine) {
  kept = 0;
  low = kKeyTop;
  double s = 0.;
  each_entry<NT, 16>(
      r, j0, j1,
      [&](int, float z, int c) {
        const uint64_t k = entry_key(z, c);
        if (k < cut) return;
        low = k < low ? k : low;
        ++kept;
        s += entry_weight(z, m, c2);
      },
      [&](int g) {
        const double w = wave_sum(s);
        if ((threadIdx.x & 63) == 0) sh.group[threadIdx.x >> 6][g] = w;
        s = 0.;
      });
  __syncthreads();
  const int groups = (j1 - j0 + NT - 1) / NT;
  mine = 0.;
  if (int(threadIdx.x) < groups)
    for (int w = 0; w < NT / kWave; ++w) mine += sh.group[w][threadIdx.x];
  double all;
  run = block_scan<NT / kWave>(mine, sh.red.d, all);
  return all;
}

// The draw among the kept entries of vectors j0 .. j1-1, after kept_masses: the group in which
// `base` and the running sum pass the target, then the entry; the last one where rounding leaves
// none.
template <int NT, bool S, typename T>
__device__ __forceinline__ int draw_entry(const LogitRow<T>& r, int j0, int j1, uint64_t cut, float m,
                                          double c2, double base, double target, double run,
                                          double mine, CutShared<NT, S>& sh) {
  if (threadIdx.x == 0) sh.pick = NT, sh.last = 0;
  __syncthreads();
  if (mine > 0.) {
    if (base + run > target) atomicMin(&sh.pick, int(threadIdx.x));
    atomicMax(&sh.last, int(threadIdx.x));
  }
  __syncthreads();
  const int g = min(sh.pick, sh.last);
  __syncthreads();
  if (int(threadIdx.x) == g) sh.sum = base + (run - mine);
  if (threadIdx.x == 0) sh.pick = NT, sh.last = -1;
  __syncthreads();
  const int j = j0 + g * NT + int(threadIdx.x), c = r.column(j);
  float x[LogitRow<T>::N];
  double own = 0., all;
#pragma unroll
  for (int e = 0; e < LogitRow<T>::N; ++e) x[e] = -INFINITY;
  if (j < j1) {
    r.load(j, x);
#pragma unroll
    for (int e = 0; e < LogitRow<T>::N; ++e) {
      if (!(x[e] > -INFINITY && entry_key(x[e], c + e) >= cut)) {
        x[e] = -INFINITY;
        continue;
      }
      own += entry_weight(x[e], m, c2);
      atomicMax(&sh.last, c + e);
    }
  }
  const double upto = sh.sum + block_scan<NT / kWave>(own, sh.red.d, all);
  if (own > 0. && upto > target) atomicMin(&sh.pick, int(threadIdx.x));
  __syncthreads();
  const int who = sh.pick;
  __syncthreads();
  if (int(threadIdx.x) == who) {
    double before = upto - own;
    int tok = -1;
#pragma unroll
    for (int e = 0; e < LogitRow<T>::N; ++e) {
      const double w = entry_weight(x[e], m, c2);
      if (w > 0. && (tok < 0 || before <= target)) tok = c + e;
      before += w;
    }
    sh.last = tok;
  }
  __syncthreads();
  return sh.last;
}

// The greatest of three values, none of them NaN.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
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
  __shared__ int best_col;
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
  float top = -INFINITY;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      // (A ballot of "> -inf" comes out as "unequal or NaN" here: the least value instead.)
      const bool is0 = x[g][e] >= kLeast, is1 = x[g][e + 1] >= kLeast;
      live += uint32_t(__popcll(__ballot(is0))) + uint32_t(__popcll(__ballot(is1)));
      x[g][e] = is0 ? x[g][e] : -INFINITY;
      x[g][e + 1] = is1 ? x[g][e + 1] : -INFINITY;
      top = max3(top, x[g][e], x[g][e + 1]);
    }
  if (tid == 0) best_col = a.V;
  if (lane == 0) wave_n[wid] = live;
  const float m = block_fold<kHeadWaves>(top, red.f, most);
  uint32_t valid = 0;
#pragma unroll
  for (int w = 0; w < kHeadWaves; ++w) valid += wave_n[w];
  if (top == m && m > -INFINITY) {
    int first = a.V;
#pragma unroll
    for (int g = G - 1; g >= 0; --g)
#pragma unroll
      for (int e = N - 1; e >= 0; --e) first = x[g][e] == m ? col(g, e) : first;
    atomicMin(&best_col, first);
  }
  __syncthreads();

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
      listed = bits = 0;
    }
    // Few threads have more than one or two: their values are read again, not picked from registers.
    uint64_t* list = h.list + (at * h.chunks + chunk) * h.cap + before;
    while (bits != 0) {
      const int q = E - __ffs(bits);
      bits &= bits - 1;
      const int c = r.column(j0 + q / N * kHeadThreads + tid) + q % N;
      *list++ = entry_key(r.raw(c), c);
    }
  }

  HeadStat st{m, best_col, valid == listed ? -INFINITY : lo, near, valid, listed, 0, 0, 0., 0.};
  if (s.nucleus && valid > 0) {
    const double k16 = 16. * s.c2;
    const float range = float(992. / k16);   // 62 octaves
    if (fabs(double(m)) * k16 < 1e9 && range < INFINITY) {
      for (int b = tid; b < kMassBins; b += kHeadThreads) mass[b] = 0;
      __syncthreads();
      const float end = m - range;
      st.top_bin = weight_bin(m, k16);
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < N; ++e)
        {
          int n;   // of top_bin - 993 .. top_bin
          const uint64_t w = weight_in_bin(fmaxf(x[g][e], end), k16, n);
          if (x[g][e] >= end) atomicAdd(&mass[st.top_bin - n], static_cast<unsigned long long>(w));
        }
      __syncthreads();
      uint32_t end_bin = 0;
      for (int b = tid; b < kMassBins; b += kHeadThreads)
        if (mass[b] != 0) end_bin = uint32_t(b) + 1;
      end_bin = block_fold<kHeadWaves>(end_bin, red.i, [](uint32_t u, uint32_t v) { return u > v ? u : v; });
      uint64_t* out = h.mass + (at * h.chunks + chunk) * kMassBins;
      for (int b = tid; b < int(end_bin); b += kHeadThreads) out[b] = mass[b];
      st.bins = int(end_bin);
    } else {
      st.bins = -1;
    }
  } else if (TOP && a.rest != nullptr && valid > listed) {
    // The others of the top logits: 32-bit exponentials, as their logarithm is stored in 32 bits.
    // Relative to lo, which they stay below; where nearly all vanish so, to their greatest.  The
    // reference is what the rounded product of lo and log2(e) / T stands for, so that an entry
    // costs one product, rounded once.
    const float c2 = fminf(float(s.c2), 3e38f);
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
      const float k = fmaxf(fminf(ref * c2, 3e38f), -3e38f);
      float f = 0.f;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < N; ++e) f += x[g][e] < lo ? __builtin_amdgcn_exp2f(fmaf(x[g][e], c2, -k)) : 0.f;
      st.rest_ref = double(k) / double(c2);
      st.rest = block_fold<kHeadWaves>(double(f), red.d, add);
      if (st.rest > 1e-25 || !(lo < INFINITY)) break;
    }
  } else if (!TOP && s.open && valid > 0) {
    double sum = 0.;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < N; ++e) sum += entry_weight(x[g][e], m, s.c2);
    st.rest_ref = double(m);
    st.rest = block_fold<kHeadWaves>(sum, red.d, add);
  }
  if (tid == 0) h.stats[at * h.chunks + chunk] = st;
}

// First place, in the order of places 0 .. n-1, whose running sum of w(i) reaches (STRICT: passes)
// the target, n where none does; `sum_to` gets the sum of the first n_sum of them.
template <int NT, bool STRICT, bool S, typename F>
__device__ __forceinline__ int reach(int n, double target, int n_sum, double& sum_to,
                                     CutShared<NT, S>& sh, F w) {
  if (threadIdx.x == 0) sh.pick = n;
  double before = 0.;
  for (int b = 0; b < n; b += NT) {
    const int i = b + int(threadIdx.x);
    const double v = i < n ? w(i) : 0.;
    double all;
    const double run = before + block_scan<NT / kWave>(v, sh.red.d, all);
    if (i < n && (STRICT ? v > 0. && run > target : run >= target)) atomicMin(&sh.pick, i);
    if (i == n_sum - 1) sh.sum = run;
    before += all;
  }
  __syncthreads();
  const int at = sh.pick;
  sum_to = n_sum > 0 ? sh.sum : 0.;
  __syncthreads();
  return at;
}

// A row's share of the second launch's work.  With few rows one launch of large workgroups does all
// of it; with many the lists are handled by small ones, several to a CU, and two more launches take
// what those leave: the rows that need one more pass, and those that need the search.
enum CutPhase { kAll, kLists, kBorder, kSearch };
enum { kDone = 0, kLeftBorder = 1, kLeftSearch = 2 };

// Between the phases: a nucleus' border bin, the weights above it and in the whole.
struct CutNote {
  double whole, above;
  int32_t border, left;
};

// One row a workgroup.  TOP: the first K entries and the log-sum-exp of the others; else the
// truncation and the draw.
template <typename T, bool TOP, int NT, CutPhase PHASE>
__global__ void __launch_bounds__(NT)
row_cut_kernel(CutArgs a, HeadArgs h) {
  constexpr bool LISTS = PHASE == kAll || PHASE == kLists, BORDER = PHASE == kAll || PHASE == kBorder,
                 SEARCH = PHASE == kAll || PHASE == kSearch;
  using Shared = CutShared<NT, SEARCH>;
  constexpr int W = Shared::W;
  __shared__ Shared sh;
  const int64_t at = blockIdx.x, row = a.row0 + at;   // in the launch, in the call
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  CutNote* note = h.notes + at;
  if (PHASE == kBorder && note->left != kLeftBorder) return;
  if (PHASE == kSearch && note->left != kLeftSearch) return;
  const LogitRow<T> r(static_cast<const T*>(a.z) + row * a.ld, a.V);
  const RowSettings s = settings_of<TOP>(a, row);
  const float scale = float(64. * s.inv_t);
  auto add = [](auto u, auto v) { return u + v; };
  auto most64 = [](uint64_t u, uint64_t v) { return u > v ? u : v; };
  auto leave = [&](int left) {
    if (tid == 0) note->left = left;
  };

  // The chunks together, by the first wave.
  if (wid == 0) {
    uint64_t best = 0;
    uint32_t valid = 0, listed = 0;
    float floor = -INFINITY, near = INFINITY;
    int top_bin = -2147483647, bins = 0;
    const HeadStat* hs = h.stats + at * h.chunks;
    for (int c0 = 0; c0 < h.chunks; c0 += 64) {
      if (c0 + lane < h.chunks) {
        const HeadStat st = hs[c0 + lane];
        sh.part[c0 + lane] = {int(st.listed), st.top_bin, st.bins, st.rest_ref, st.rest};
        if (st.valid != 0) {
          best = most64(best, entry_key(st.best, st.best_col));
          valid += st.valid;
          listed += st.listed;
          floor = fmaxf(floor, st.floor);
          near = fminf(near, st.near);
          top_bin = st.bins > 0 ? max(top_bin, st.top_bin) : top_bin;
          bins = st.bins < 0 ? -1 : bins;
        }
      }
    }
    best = wave_fold(best, most64);
    valid = wave_fold(valid, add);
    listed = wave_fold(listed, add);
    floor = wave_fold(floor, [](float u, float v) { return fmaxf(u, v); });
    near = wave_fold(near, [](float u, float v) { return fminf(u, v); });
    top_bin = wave_fold(top_bin, [](int u, int v) { return max(u, v); });
    bins = wave_fold(bins, [](int u, int v) { return min(u, v); });
    if (lane == 0) {
      sh.best = best;
      sh.valid = valid;
      sh.listed = listed;
      sh.floor = floor;
      sh.near = near;
      sh.top_bin = top_bin;
      sh.bins = bins;
    }
  }
  __syncthreads();
  const uint64_t best = sh.best;
  const uint32_t valid = sh.valid, listed = sh.listed;
  const float m = entry_logit(best), floor = sh.floor;
  const bool whole = listed == valid;   // nothing is unlisted
  if (PHASE == kLists) leave(kDone);

  if (!TOP && LISTS && (valid == 0 || s.greedy)) {
    if (tid == 0) {
      if (a.tok != nullptr) a.tok[row] = valid != 0 ? entry_column(best) : -1;
      a.kept[row] = valid != 0 ? 1 : 0;
      a.cut_logit[row] = valid > 1 ? m : -INFINITY;
      a.cut_index[row] = valid > 1 ? entry_column(best) : -1;
      a.lse[row] = valid != 0 ? 0. : -INFINITY;
    }
    return;
  }

  // The listed entries, all in flight together: this thread's places of the row's lists.
  constexpr int LISTED = LISTS ? kListMax / NT : 1;
  uint64_t mine[LISTED];
  if constexpr (LISTS) {
    const uint64_t* list = h.list + at * h.chunks * h.cap;
#pragma unroll
    for (int q = 0; q < LISTED; ++q) {
      const int i = q * NT + tid, c = i / h.cap;
      const bool is = c < h.chunks && i - c * h.cap < sh.part[c].listed;
      mine[q] = list[is ? i : 0];
      mine[q] = is ? mine[q] : 0ull;
    }
  }
  // Those of value >= t into the list; all of the row's where t >= floor.
  auto gather = [&](float t) {
    __syncthreads();
    if (tid == 0) sh.n = 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < LISTED; ++q)
      if (mine[q] != 0 && entry_logit(mine[q]) >= t) sh.list[atomicAdd(&sh.n, 1u)] = mine[q];
    __syncthreads();
    const int n = int(sh.n);
    __syncthreads();
    return n;
  };

  if constexpr (TOP) {
    const int K = a.K;
    const int n = int(min(uint32_t(K), valid));
    bool done = false;
    if constexpr (LISTS) {
      int have = gather(fmaxf(floor, sh.near));
      if (have < n && sh.near > floor) have = gather(floor);
      if (have >= n) {
        done = true;
        sort_list<NT>(sh.list, have);
        if (a.rest != nullptr) {
          const uint64_t last = n > 0 ? sh.list[n - 1] : 0;
          uint64_t next = 0;
#pragma unroll
          for (int q = 0; q < LISTED; ++q) next = mine[q] < last ? most64(next, mine[q]) : next;
          double ref = next != 0 ? double(entry_logit(next)) : -INFINITY;
          const bool rest = tid < h.chunks && sh.part[tid].rest > 0.;
          if (rest) ref = fmax(ref, sh.part[tid].rest_ref);
          ref = block_fold<W>(ref, sh.red.d, [](double u, double v) { return fmax(u, v); });
          double sum = 0.;
#pragma unroll
          for (int q = 0; q < LISTED; ++q)
            if (mine[q] != 0 && mine[q] < last)
              sum += exp2_64((double(entry_logit(mine[q])) - ref) * s.c2);
          if (rest) sum += sh.part[tid].rest * exp2_64((sh.part[tid].rest_ref - ref) * s.c2);
          sum = block_fold<W>(sum, sh.red.d, add);
          if (tid == 0) a.rest[row] = sum > 0. ? float(ref * s.inv_t + log(sum)) : -INFINITY;
        }
      } else if (PHASE == kLists) {
        leave(kLeftSearch);
        return;
      }
    }
    if constexpr (SEARCH) {
      if (!done) {
        const uint64_t cut =
            valid > uint32_t(K) ? select_entry<false>(r, double(K), 0, m, s.c2, scale, sh) : 0;
        if (tid == 0) sh.n = 0;
        __syncthreads();
        uint64_t next = 0;   // the first entry past the list
        each_entry(r, [&](int, float z, int c) {
          const uint64_t k = entry_key(z, c);
          if (k >= cut)
            sh.list[atomicAdd(&sh.n, 1u)] = k;
          else
            next = k > next ? k : next;
        });
        __syncthreads();
        sort_list<NT>(sh.list, n);
        if (a.rest != nullptr) {
          next = block_fold<W>(next, sh.red.u, most64);
          const float top = entry_logit(next);
          double sum = 0.;
          if (next != 0)
            each_entry(r, [&](int, float z, int c) {
              if (entry_key(z, c) < cut) sum += entry_weight(z, top, s.c2);
            });
          sum = block_fold<W>(sum, sh.red.d, add);
          if (tid == 0)
            a.rest[row] = next != 0 ? float(double(top) * s.inv_t + log(sum)) : -INFINITY;
        }
      }
    }
    for (int i = tid; i < K; i += NT) {
      const uint64_t k = sh.list[i < n ? i : 0];
      a.ids[row * K + i] = i < n ? entry_column(k) : -1;
      a.vals[row * K + i] = i < n ? entry_logit(k) : -INFINITY;
    }
  } else {
    const bool has_k = s.top_k > 0 && uint32_t(s.top_k) < valid;
    const bool has_p = s.top_p < 1.f, has_m = s.min_p > 0.f;
    const double least_w = has_m ? fmin(double(s.min_p), 1.) : 0.;
    const double u = a.u != nullptr ? fmin(fmax(double(a.u[row]), 0.), 1.) : 0.;
    auto write = [&](uint32_t kept, uint64_t low, double mass, int tok) {
      if (tid != 0) return;
      const bool every = kept == valid;
      a.kept[row] = int32_t(kept);
      a.cut_logit[row] = every ? -INFINITY : entry_logit(low);
      a.cut_index[row] = every ? -1 : entry_column(low);
      a.lse[row] = double(m) * s.inv_t + log(mass);
      if (a.tok != nullptr) a.tok[row] = tok;
    };
    // Least value of weight min_p.
    auto value_of_min_p = [&]() {
      return f32_from_order_key(
          least_value_key(m, [&](float z) { return entry_weight(z, m, s.c2) >= least_w; }));
    };
    // The draw when the chunks' masses are known (thread c has chunk c's): only the chunk that the
    // running sum passes the target in is read.
    auto draw_in_chunks = [&](double w, double run, double mass, uint64_t cut) {
      const double target = u * mass;
      if (tid == 0) sh.pick = NT, sh.last = 0;
      __syncthreads();
      if (w > 0.) {
        if (run > target) atomicMin(&sh.pick, tid);
        atomicMax(&sh.last, tid);
      }
      __syncthreads();
      const int c = min(sh.pick, sh.last);
      __syncthreads();
      if (tid == c) sh.sum = run - w;
      __syncthreads();
      const double base = sh.sum;
      const int j0 = c * h.vectors, j1 = min(r.vectors(), j0 + h.vectors);
      uint32_t n;
      uint64_t l;
      double grun, gmine;
      kept_masses<NT, SEARCH>(r, j0, j1, cut, m, s.c2, sh, n, l, grun, gmine);
      return draw_entry<NT, SEARCH>(r, j0, j1, cut, m, s.c2, base, target, grun, gmine, sh);
    };

    if (s.open) {
      // Everything is kept: the chunks' sums are the masses.
      const bool is = tid < h.chunks && sh.part[tid].rest > 0.;
      const double w = is ? sh.part[tid].rest * exp2_64((sh.part[tid].rest_ref - double(m)) * s.c2) : 0.;
      double mass;
      const double run = block_scan<W>(w, sh.red.d, mass);
      if constexpr (PHASE == kLists) {
        if (a.tok != nullptr)
          leave(kLeftBorder);
        else
          write(valid, 0, mass, -1);
      } else if constexpr (BORDER) {
        write(valid, 0, mass, a.tok != nullptr ? draw_in_chunks(w, run, mass, 0) : -1);
      }
      return;
    }

    // The nucleus' border bin: the histograms joined, their running sum against top_p of the whole.
    const double k16 = 16. * s.c2;
    const bool binned = s.nucleus && sh.bins == 0;
    double zk = 0., above = 0.;   // relative to the greatest entry: the whole, the bins above it
    int border = 0;
    const int top_bin = sh.top_bin;
    auto bin_weight = [&](int b) { return exp2_64(-double(b) / 16.); };
    // 2^-48 of the top bin's middle, relative to the greatest entry's weight.
    const double unit =
        binned ? exp2((double(top_bin) - double(m) * k16) / 16.) * 3.552713678800501e-15 : 0.;
    const uint64_t* masses = h.mass + at * h.chunks * kMassBins;
    auto mass_at = [&](int c, int b) -> double {   // of chunk c in the row's bin b
      const int i = b - (top_bin - sh.part[c].top_bin);
      const bool is = i >= 0 && i < sh.part[c].bins;
      const uint64_t n = masses[int64_t(c) * kMassBins + (is ? i : 0)];   // loaded in any case
      return is ? double(n) : 0.;
    };
    if constexpr (LISTS) {
      if (binned) {
        constexpr int PER = kMassBins / NT;
        double v[PER], sum = 0.;
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = 0.;
#pragma unroll 8
        for (int c = 0; c < h.chunks; ++c) {
#pragma unroll
          for (int e = 0; e < PER; ++e) v[e] += mass_at(c, PER * tid + e);
        }
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          v[e] *= bin_weight(PER * tid + e) * unit;
          sum += v[e];
        }
        const double run = block_scan<W>(sum, sh.red.d, zk);
        if (tid == 0) sh.pick = kMassBins, sh.last = 0;
        __syncthreads();
        const double target = fmax(double(s.top_p) * zk, 1e-300);
        double upto = run - sum;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          upto += v[e];
          if (v[e] > 0.) {
            if (upto >= target) atomicMin(&sh.pick, PER * tid + e);
            atomicMax(&sh.last, PER * tid + e);
          }
        }
        __syncthreads();
        border = min(sh.pick, sh.last);
        upto = run - sum;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          if (PER * tid + e == border) sh.sum = upto;
          upto += v[e];
        }
        __syncthreads();
        above = sh.sum;
        __syncthreads();
        if (PHASE == kLists && tid == 0) note->whole = zk, note->above = above, note->border = border;
      }
    } else if (binned) {
      zk = note->whole;
      above = note->above;
      border = note->border;
    }
    // Least value of bin b or a greater one.
    auto bin_edge = [&](int b) {
      return f32_from_order_key(least_value_key(m, [&](float z) {   // far values have no bin
        return double(z) * k16 > double(top_bin) - 2048. && weight_bin(z, k16) >= top_bin - b;
      }));
    };

    const uint64_t cut_m =
        has_m ? uint64_t(f32_order_key(value_of_min_p() + 0.f)) << kColumnBits : 0;
    uint64_t cut = 0;
    // Among the border bin's n entries in the list, sorted: the first to reach the target.
    auto cut_of_border = [&](int n, int& kept) {
      sort_list<NT>(sh.list, n);
      double sum;
      const int p = reach<NT, false, SEARCH>(
          n, fmax(double(s.top_p) * zk, 1e-300) - above, 0, sum, sh,
          [&](int i) { return entry_weight(entry_logit(sh.list[i]), m, s.c2); });
      kept = min(p + 1, n);
      return sh.list[kept - 1];
    };
    const float border_end = binned ? bin_edge(border) : 0.f;
    const float border_over = binned && border > 0 ? bin_edge(border - 1) : INFINITY;

    if constexpr (LISTS) {
      // The cut, where the lists hold all that lies above it.
      bool quick;
      if (has_k) {
        int have = gather(fmaxf(floor, sh.near));
        if (have < s.top_k && sh.near > floor) have = gather(floor);
        quick = have >= s.top_k;
        if (quick) {
          sort_list<NT>(sh.list, have);
          auto weight = [&](int i) { return entry_weight(entry_logit(sh.list[i]), m, s.c2); };
          int n = s.top_k;
          if (has_p) {
            double sum;
            reach<NT, false, SEARCH>(n, 1e300, n, zk, sh, weight);   // of all n
            const int p =
                reach<NT, false, SEARCH>(n, fmax(double(s.top_p) * zk, 1e-300), 0, sum, sh, weight);
            n = min(n, p + 1);
          }
          cut = sh.list[n - 1];
        }
      } else if (binned) {
        quick = border_end >= floor;
        if (quick) {
          __syncthreads();
          if (tid == 0) sh.n = 0;
          __syncthreads();
#pragma unroll
          for (int q = 0; q < LISTED; ++q) {
            const float z = entry_logit(mine[q]);
            if (mine[q] != 0 && z >= border_end && (z < border_over || border == 0))
              sh.list[atomicAdd(&sh.n, 1u)] = mine[q];
          }
          __syncthreads();
          const int n = int(sh.n);
          __syncthreads();
          int k;
          cut = cut_of_border(n, k);
        }
      } else {
        // min_p alone; a nucleus or a top_k of all that is left, with everything listed.
        quick = whole || (!has_p && s.top_k <= 0 && entry_logit(cut_m) >= floor);
        if (quick && has_p) {
          const int n = gather(floor);
          sort_list<NT>(sh.list, n);
          auto weight = [&](int i) { return entry_weight(entry_logit(sh.list[i]), m, s.c2); };
          double sum;
          reach<NT, false, SEARCH>(n, 1e300, n, zk, sh, weight);
          const int p =
              reach<NT, false, SEARCH>(n, fmax(double(s.top_p) * zk, 1e-300), 0, sum, sh, weight);
          cut = sh.list[min(p, n - 1)];
        }
      }
      if (quick) {
        // The kept entries in token order: columns with their places as keys, the weights beside
        // them.
        __syncthreads();
        if (tid == 0) sh.n = 0;
        __syncthreads();
        cut = most64(cut, cut_m);
        uint64_t low = kKeyTop;
        uint32_t many = 0;
#pragma unroll
        for (int q = 0; q < LISTED; ++q)
          if (mine[q] != 0 && mine[q] >= cut) {
            low = mine[q] < low ? mine[q] : low;
            ++many;
          }
        many = block_fold<W>(many, sh.red.i, add);
        // (A nucleus of many is left to the next phase, which need not sort it.)
        if (PHASE == kLists && binned && many > 2 * NT) {
          leave(kLeftBorder);
          return;
        }
        low = block_fold<W>(low, sh.red.u, [](uint64_t x, uint64_t y) { return x < y ? x : y; });
#pragma unroll
        for (int q = 0; q < LISTED; ++q)
          if (mine[q] != 0 && mine[q] >= cut) {
            const uint32_t i = atomicAdd(&sh.n, 1u);
            sh.list[i] = ((mine[q] & kColumnMask) << 12) | uint64_t(i);
            sh.weight[i] = entry_weight(entry_logit(mine[q]), m, s.c2);
          }
        __syncthreads();
        const int n = int(many);
        sort_list<NT>(sh.list, n);
        auto in_order = [&](int i) { return sh.weight[sh.list[i] & 4095u]; };
        double mass;
        int tok = -1;
        reach<NT, true, SEARCH>(n, 1e300, n, mass, sh, in_order);
        if (a.tok != nullptr) {
          double sum;
          int i = reach<NT, true, SEARCH>(n, u * mass, 0, sum, sh, in_order);
          if (i == n) {   // the last with a weight
            if (tid == 0) sh.last = 0;
            __syncthreads();
            for (int q = tid; q < n; q += NT)
              if (in_order(q) > 0.) atomicMax(&sh.last, q);
            __syncthreads();
            i = sh.last;
          }
          tok = int(kColumnMask - uint32_t(sh.list[i] >> 12));
        }
        write(uint32_t(n), low, mass, tok);
        return;
      }
      if (PHASE == kLists) {
        leave(binned ? kLeftBorder : kLeftSearch);
        return;
      }
    }

    // The lists do not reach the cut: the row is read again.
    if constexpr (BORDER) {
      if (binned) {
        // The border bin's entries, and how many lie above it.
        __syncthreads();
        if (tid == 0) sh.n = 0;
        __syncthreads();
        uint32_t greater = 0;
        constexpr int N = LogitRow<T>::N, Q = 32 / N;
        const int nv = r.vectors();
        for (int b = 0; b < nv; b += Q * NT) {
          float x[Q][N];
          if (r.inside(b, Q * NT)) {
#pragma unroll
            for (int q = 0; q < Q; ++q) r.load_inside(b + q * NT + tid, x[q]);
          } else {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
#pragma unroll
              for (int e = 0; e < N; ++e) x[q][e] = -INFINITY;
              if (b + q * NT + tid < nv) r.load_raw(b + q * NT + tid, x[q]);
            }
          }
          uint32_t bits = 0;   // of the border bin, the first entry's bit the highest
#pragma unroll
          for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int e = 0; e < N; ++e) {
              const bool over = x[q][e] >= border_over;
              greater += uint32_t(__popcll(__ballot(over)));
              bits = 2 * bits + uint32_t(x[q][e] >= border_end && !over);
            }
          while (bits != 0) {
            const int q = 32 - __ffs(bits);
            bits &= bits - 1;
            const int c = r.column(b + q / N * NT + tid) + q % N;
            const uint32_t i = atomicAdd(&sh.n, 1u);
            if (i < uint32_t(kListMax)) sh.list[i] = entry_key(r.raw(c), c);
          }
        }
        greater = block_fold<W>(lane == 0 ? greater : 0u, sh.red.i, add);
        const uint32_t in = sh.n;
        __syncthreads();
        if (in <= uint32_t(kListMax) && in > 0) {
          int n;
          cut = cut_of_border(int(in), n);
          if (cut_m <= cut) {
            // The chunks' masses: their bins above the border, and their part of its entries.
            for (int c = wid; c < h.chunks; c += W) {
              double w = 0.;
              for (int b = lane; b < border; b += 64) w += mass_at(c, b) * bin_weight(b) * unit;
              for (int i = lane; i < n; i += 64) {
                const uint64_t k = sh.list[i];
                const int j = (entry_column(k) + r.shift) / N;
                if (j / h.vectors == c) w += entry_weight(entry_logit(k), m, s.c2);
              }
              w = wave_fold(w, add);
              if (lane == 0) sh.chunk[c] = w;
            }
            __syncthreads();
            const double w = tid < h.chunks ? sh.chunk[tid] : 0.;
            double mass;
            const double run = block_scan<W>(w, sh.red.d, mass);
            const int tok = a.tok != nullptr ? draw_in_chunks(w, run, mass, cut) : -1;
            write(greater + uint32_t(n), cut, mass, tok);
            return;
          }
        }
      }
      if (PHASE == kBorder) {
        leave(kLeftSearch);
        return;
      }
    }
    if constexpr (SEARCH) {
      cut = has_k ? select_entry<false>(r, double(s.top_k), 0, m, s.c2, scale, sh) : 0;
      if (binned) {
        // A border bin of many entries: the cut among them.
        const uint64_t end = entry_key(border_end, a.V - 1);
        const uint64_t over = border > 0 ? entry_key(border_over, kColumnMask) - 1 : kKeyTop;
        cut = select_entry<true>(r, fmax(double(s.top_p) * zk, 1e-300), 0, m, s.c2, scale, sh, end,
                                 over, above);
      } else if (has_p) {
        double all = 0.;
        each_entry(r, [&](int, float z, int c) {
          if (entry_key(z, c) >= cut) all += entry_weight(z, m, s.c2);
        });
        all = block_fold<W>(all, sh.red.d, add);
        // A target of 0 is reached by the first entry, not before it.
        cut = most64(cut, select_entry<true>(r, fmax(double(s.top_p) * all, 1e-300), cut, m, s.c2,
                                             scale, sh));
      }
      cut = most64(cut, cut_m);
      double run, mine_w;
      uint32_t kept;
      uint64_t low;
      const double mass = kept_masses<NT, SEARCH>(r, 0, r.vectors(), cut, m, s.c2, sh, kept, low, run, mine_w);
      kept = block_fold<W>(kept, sh.red.i, add);
      low = block_fold<W>(low, sh.red.u, [](uint64_t x, uint64_t y) { return x < y ? x : y; });
      const int tok = a.tok != nullptr ? draw_entry<NT, SEARCH>(r, 0, r.vectors(), cut, m, s.c2, 0., u * mass,
                                                        run, mine_w, sh)
                                       : -1;
      write(kept, low, mass, tok);
    }
  }
}

// ------------------------------------------------------------------------- verification
// Draft x_i of a sequence is accepted if u_i q_i(x_i) < p_i(x_i), p and q the truncated
// distributions of the target's and the drafter's row; after n acceptances the next token is drawn
// from max(0, p_n - q_n) by its running sum in column order (from p_n where that is zero
// throughout, or after K acceptances).

constexpr int kVerifyThreads = 256;    // one vector of a part each
constexpr int kVerifyWaves = kVerifyThreads / kWave;

// Probability of an entry under a row's truncation; lse2 = lse * log2(e).
struct RowCut {
  float logit;
  int index;
  double lse2;
};
__device__ __forceinline__ double cut_prob(const RowCut& k, float z, int c, bool greedy, double c2) {
  if (!(z > k.logit || (z == k.logit && c <= k.index)) || z == -INFINITY) return 0.;
  return greedy ? 1. : exp2_64(double(z) * c2 - k.lse2);
}

template <typename TD, typename TT>
struct VerifyRows {
  const VerifyArgs& a;
  int s;
  bool greedy;
  double c2;
  __device__ VerifyRows(const VerifyArgs& a_, int s_) : a(a_), s(s_) {
    const float t = a.ts != nullptr ? a.ts[s] : a.t;
    greedy = !(t > 0.f);
    c2 = greedy ? 0. : 1.4426950408889634074 / double(t);
  }
  __device__ const TT* target(int i) const {
    return static_cast<const TT*>(a.tz) + (int64_t(s) * (a.K + 1) + i) * a.V;
  }
  __device__ const TD* draft(int i) const {
    return static_cast<const TD*>(a.dz) + (int64_t(s) * a.stride + i) * a.ld;
  }
  __device__ RowCut target_cut(int i) const {
    const int64_t r = int64_t(s) * (a.K + 1) + i;
    return {a.t_logit[r], a.t_index[r], a.t_lse[r] * 1.4426950408889634074};
  }
  __device__ RowCut draft_cut(int i) const {
    const int64_t r = int64_t(s) * a.stride + i;
    return {a.d_logit[r], a.d_index[r], a.d_lse[r] * 1.4426950408889634074};
  }
  // Weights of the next token's draw in vector j of target row n: the residual w and the target's
  // own p.
  __device__ void weights(int n, int j, double w[LogitRow<TT>::N], double p[LogitRow<TT>::N]) const {
    constexpr int N = LogitRow<TT>::N;
    const LogitRow<TT> t(target(n), a.V);
    const LogitRow<TD> d(n < a.K ? draft(n) : nullptr, a.V);
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = p[e] = 0.;
    if (j >= t.vectors()) return;
    t.load(j, x);
    const RowCut tc = target_cut(n), dc = n < a.K ? draft_cut(n) : tc;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int c = t.column(j) + e;
      p[e] = cut_prob(tc, x[e], c, greedy, c2);
      w[e] = p[e];
      if (n < a.K && p[e] > 0.) w[e] = fmax(p[e] - cut_prob(dc, d.at(c), c, greedy, c2), 0.);
    }
  }
};

// Workgroup (part, sequence): the sequence's decisions (each workgroup makes them for itself: a
// launch between would cost more than the few dependent loads), then the sums of both weights over
// 256 vectors of row n.
template <typename TD, typename TT>
__global__ void __launch_bounds__(kVerifyThreads)
verify_sum_kernel(VerifyArgs a) {
  __shared__ int decided;
  __shared__ double sh[kVerifyWaves];
  const int s = blockIdx.y, part = blockIdx.x;
  const VerifyRows<TD, TT> v(a, s);
  if (threadIdx.x < 64) {
    int n = a.K;
    for (int c0 = 0; c0 < a.K; c0 += 64) {
      const int i = c0 + int(threadIdx.x);
      bool reject = false;
      if (i < a.K) {
        const int x = a.draft[int64_t(s) * a.stride + i];
        double p = 0., q = 0.;
        if (x >= 0 && x < a.V) {
          p = cut_prob(v.target_cut(i), LogitRow<TT>(v.target(i), a.V).at(x), x, v.greedy, v.c2);
          q = cut_prob(v.draft_cut(i), LogitRow<TD>(v.draft(i), a.V).at(x), x, v.greedy, v.c2);
        }
        reject = !(double(a.u[int64_t(s) * (a.K + 1) + i]) * q < p);
      }
      const unsigned long long miss = __ballot(reject);
      if (miss != 0ull) {
        n = c0 + __ffsll(static_cast<long long>(miss)) - 1;
        break;
      }
    }
    if (threadIdx.x == 0) {
      decided = n;
      if (part == 0) a.n_buf[s] = n;
    }
  }
  __syncthreads();
  double w[LogitRow<TT>::N], p[LogitRow<TT>::N], sw = 0., sp = 0.;
  v.weights(decided, part * kVerifyThreads + int(threadIdx.x), w, p);
#pragma unroll
  for (int e = 0; e < LogitRow<TT>::N; ++e) {
    sw += w[e];
    sp += p[e];
  }
  auto add = [](double x, double y) { return x + y; };
  sw = block_fold<kVerifyWaves>(sw, sh, add);
  sp = block_fold<kVerifyWaves>(sp, sh, add);
  if (threadIdx.x == 0) {
    double* o = a.sums + (int64_t(s) * gridDim.x + part) * 2;
    o[0] = sw;
    o[1] = sp;
  }
}

// One workgroup a sequence: the part in which the running sum passes u times the whole, the entry
// within it, and the sequence's commits behind those of the sequences before it.
template <typename TD, typename TT>
__global__ void __launch_bounds__(kVerifyThreads)
verify_pick_kernel(VerifyArgs a, int parts) {
  __shared__ double sh[kVerifyWaves];
  __shared__ int shi[kVerifyWaves];
  __shared__ double base;
  __shared__ int pick, last, token;
  const int s = blockIdx.x, tid = threadIdx.x;
  const VerifyRows<TD, TT> v(a, s);
  const int n = a.n_buf[s];
  const double* sums = a.sums + int64_t(s) * parts * 2;
  auto add = [](auto x, auto y) { return x + y; };
  double sw = 0., sp = 0.;
  for (int i = tid; i < parts; i += kVerifyThreads) {
    sw += sums[2 * i];
    sp += sums[2 * i + 1];
  }
  sw = block_fold<kVerifyWaves>(sw, sh, add);
  sp = block_fold<kVerifyWaves>(sp, sh, add);
  const int which = sw > 0. ? 0 : 1;
  const double target = fmin(fmax(double(a.u[int64_t(s) * (a.K + 1) + a.K]), 0.), 1.) *
                        (which == 0 ? sw : sp);
  if (tid == 0) pick = parts, last = 0, token = -1, base = 0.;
  __syncthreads();
  double before = 0.;   // of the parts ahead of this round's
  for (int b = 0; b < parts; b += kVerifyThreads) {
    const int i = b + tid;
    const double mine = i < parts ? sums[2 * i + which] : 0.;
    double all;
    const double run = before + block_scan<kVerifyWaves>(mine, sh, all);
    if (mine > 0.) {
      if (run > target) atomicMin(&pick, i);
      atomicMax(&last, i);
    }
    __syncthreads();
    const bool found = pick < parts;
    if (found || b + kVerifyThreads >= parts) {
      if (i == (found ? pick : last)) base = run - mine;
    }
    before += all;
    __syncthreads();
    if (found) break;
  }
  const int part = pick < parts ? pick : last;
  // `last` may lie in an earlier round than the final one: its base is then not the one stored.
  // The draw below takes the part's last entry in that case, whatever the base.
  const bool tail = pick >= parts;
  __syncthreads();
  if (tid == 0) pick = kVerifyThreads, last = -1;
  __syncthreads();
  double w[LogitRow<TT>::N], p[LogitRow<TT>::N], mine = 0., all;
  const int j = part * kVerifyThreads + tid;
  v.weights(n, j, w, p);
  const int c = LogitRow<TT>(v.target(n), a.V).column(j);
#pragma unroll
  for (int e = 0; e < LogitRow<TT>::N; ++e) {
    w[e] = which == 0 ? w[e] : p[e];
    mine += w[e];
    if (w[e] > 0.) atomicMax(&last, c + e);
  }
  const double upto = base + block_scan<kVerifyWaves>(mine, sh, all);
  if (!tail && mine > 0. && upto > target) atomicMin(&pick, tid);
  __syncthreads();
  if (pick < kVerifyThreads) {
    if (tid == pick) {
      double sum = upto - mine;
      int tok = -1;
#pragma unroll
      for (int e = 0; e < LogitRow<TT>::N; ++e) {
        sum += w[e];
        if (w[e] > 0. && (tok < 0 || sum - w[e] <= target)) tok = c + e;
      }
      token = tok;
    }
  } else if (tid == 0) {
    token = last;
  }
  int ahead = 0;
  if (a.offs != nullptr || a.toks != nullptr) {
    for (int i = tid; i < s; i += kVerifyThreads) ahead += a.n_buf[i] + 1;
    ahead = block_fold<kVerifyWaves>(ahead, shi, add);
  }
  __syncthreads();
  if (tid == 0) {
    a.acc[s] = n;
    a.anchor[s] = token;
    if (a.offs != nullptr) {
      a.offs[s] = ahead;
      if (s == int(gridDim.x) - 1) a.offs[s + 1] = ahead + n + 1;
    }
  }
  if (a.toks != nullptr)
    for (int i = tid; i <= n; i += kVerifyThreads)
      a.toks[ahead + i] = i < n ? a.draft[int64_t(s) * a.stride + i] : token;
}

static size_t al256(size_t x) { return (x + 255) / 256 * 256; }

// The first launch's chunks: 16384 columns each, or 4096 where those would leave CUs idle (and the
// lists of so many chunks still hold enough).
struct HeadPlan {
  int chunks, elems;
};
static HeadPlan head_plan(bool bf16, int64_t rows, int V) {
  const int N = bf16 ? 8 : 4, span = (V + 2 * N - 2) / N * N;
  const int large = (span + 32 * kHeadThreads - 1) / (32 * kHeadThreads);
  const int small = (span + 8 * kHeadThreads - 1) / (8 * kHeadThreads);
  if (rows * large < device_cu_count() && small <= 64) return {small, 8};
  return {large, 32};
}
// Rows of one group of launches; more run in turns over the same workspace.
constexpr int64_t kCutChunks = 8192;
static int64_t cut_rows(bool bf16, int64_t rows, int V) {
  const int64_t most = kCutChunks / head_plan(bf16, kCutChunks, V).chunks;
  return rows < most ? rows : most;
}
// Above this many rows (a workgroup a CU) the second launch's phases run apart.
constexpr int64_t kCombinedRows = 256;
constexpr int kListThreads = 256, kBorderThreads = 512;

size_t cut_ws_bytes(bool bf16, int64_t rows, int V, bool top) {
  const int64_t n = cut_rows(bf16, rows, V);
  // The lists of a row hold kListMax entries whatever its chunks.  Small chunks are more of them, but
  // only of few rows.
  int64_t chunks = n * head_plan(bf16, kCutChunks, V).chunks;
  const int64_t few = n < device_cu_count() ? n : device_cu_count();
  const HeadPlan fine = head_plan(bf16, 0, V);
  const int64_t fine_chunks = few * fine.chunks;
  chunks = chunks > fine_chunks ? chunks : fine_chunks;
  return al256(size_t(n) * kListMax * 8) + al256(size_t(n) * sizeof(CutNote)) + al256(size_t(chunks) * sizeof(HeadStat)) +
         (top ? 0 : al256(size_t(chunks) * kMassBins * 8));
}

template <typename T, bool TOP>
static hipError_t launch_cut(const CutArgs& all, void* ws, hipStream_t s) {
  const bool bf16 = sizeof(T) == 2;
  const int64_t most = cut_rows(bf16, all.rows, all.V);
  for (int64_t r0 = 0; r0 < all.rows; r0 += most) {
    CutArgs a = all;
    a.rows = all.rows - r0 < most ? all.rows - r0 : most;
    a.row0 = r0;
    const HeadPlan pl = head_plan(bf16, a.rows, a.V);
    char* p = static_cast<char*>(ws);
    auto take = [&](size_t bytes) {
      char* q = p;
      p += al256(bytes);
      return q;
    };
    HeadArgs h;
    h.chunks = pl.chunks;
    h.cap = kListMax / pl.chunks;
    h.vectors = pl.elems * kHeadThreads / LogitRow<T>::N;
    h.list = reinterpret_cast<uint64_t*>(take(size_t(a.rows) * kListMax * 8));
    h.notes = reinterpret_cast<CutNote*>(take(size_t(a.rows) * sizeof(CutNote)));
    h.stats = reinterpret_cast<HeadStat*>(take(size_t(a.rows) * pl.chunks * sizeof(HeadStat)));
    h.mass = reinterpret_cast<uint64_t*>(p);
    const dim3 grid(unsigned(a.rows) * pl.chunks), rows(unsigned(a.rows));
    if (pl.elems == 8)
      hipLaunchKernelGGL((row_head_kernel<T, 8, TOP>), grid, dim3(kHeadThreads), 0, s, a, h);
    else
      hipLaunchKernelGGL((row_head_kernel<T, 32, TOP>), grid, dim3(kHeadThreads), 0, s, a, h);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.rows <= kCombinedRows) {
      hipLaunchKernelGGL((row_cut_kernel<T, TOP, kCutThreads, kAll>), rows, dim3(kCutThreads), 0, s, a, h);
    } else {
      hipLaunchKernelGGL((row_cut_kernel<T, TOP, kListThreads, kLists>), rows, dim3(kListThreads), 0, s, a, h);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      if constexpr (!TOP) {
        hipLaunchKernelGGL((row_cut_kernel<T, TOP, kBorderThreads, kBorder>), rows, dim3(kBorderThreads), 0, s, a, h);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
      hipLaunchKernelGGL((row_cut_kernel<T, TOP, kCutThreads, kSearch>), rows, dim3(kCutThreads), 0, s, a, h);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_truncate(bool bf16, const CutArgs& a, void* ws, hipStream_t s) {
  return bf16 ? launch_cut<bf16_t, false>(a, ws, s) : launch_cut<float, false>(a, ws, s);
}
hipError_t launch_top_logits(bool bf16, const CutArgs& a, void* ws, hipStream_t s) {
  return bf16 ? launch_cut<bf16_t, true>(a, ws, s) : launch_cut<float, true>(a, ws, s);
}

// Parts of a target row: 256 vectors each, of its least vectors and one for a row that starts
// inside one.
static int verify_parts(bool bf16, int V) {
  const int N = bf16 ? 8 : 4;
  return ((V + 2 * N - 2) / N + kVerifyThreads - 1) / kVerifyThreads;
}

size_t accept_truncated_ws_bytes(bool bf16, int n_seq, int K, int V) {
  const size_t rows = size_t(n_seq) * (K + 1);
  return cut_ws_bytes(bf16, int64_t(rows), V, false) + al256(rows * 8) + 3 * al256(rows * 4) + al256(size_t(n_seq) * 4) +
         al256(size_t(n_seq) * verify_parts(bf16, V) * 16);
}

template <typename TD, typename TT>
static hipError_t launch_verify(const VerifyArgs& a, int n_seq, int parts, hipStream_t s) {
  hipLaunchKernelGGL((verify_sum_kernel<TD, TT>), dim3(parts, n_seq), dim3(kVerifyThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((verify_pick_kernel<TD, TT>), dim3(n_seq), dim3(kVerifyThreads), 0, s, a, parts);
  return hipGetLastError();
}

hipError_t launch_accept_truncated(bool draft_bf16, bool target_bf16, VerifyArgs a, CutArgs c,
                                   int n_seq, void* ws, hipStream_t s) {
  const size_t rows = size_t(n_seq) * (a.K + 1);
  char* p = static_cast<char*>(ws);
  auto take = [&](size_t bytes) {
    char* q = p;
    p += al256(bytes);
    return q;
  };
  c.lse = reinterpret_cast<double*>(take(rows * 8));
  c.cut_logit = reinterpret_cast<float*>(take(rows * 4));
  c.cut_index = reinterpret_cast<int32_t*>(take(rows * 4));
  c.kept = reinterpret_cast<int32_t*>(take(rows * 4));
  a.n_buf = reinterpret_cast<int32_t*>(take(size_t(n_seq) * 4));
  const int parts = verify_parts(target_bf16, a.V);
  a.sums = reinterpret_cast<double*>(take(size_t(n_seq) * parts * 16));
  a.t_logit = c.cut_logit;
  a.t_index = c.cut_index;
  a.t_lse = c.lse;
  const hipError_t e = launch_truncate(target_bf16, c, take(cut_ws_bytes(target_bf16, int64_t(rows), a.V, false)), s);
  if (e != hipSuccess) return e;
  if (draft_bf16)
    return target_bf16 ? launch_verify<bf16_t, bf16_t>(a, n_seq, parts, s)
                       : launch_verify<bf16_t, float>(a, n_seq, parts, s);
  return target_bf16 ? launch_verify<float, bf16_t>(a, n_seq, parts, s)
                     : launch_verify<float, float>(a, n_seq, parts, s);
}

}  // namespace hdf
