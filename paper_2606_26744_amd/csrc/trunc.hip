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
constexpr int kListMax = kCutThreads;          // entries sorted at once
constexpr int kAhead = 4;                      // vectors a thread loads before it uses them
constexpr int kMaxGroups = (1 << kColumnBits) / (4 * kCutThreads) + 1;
constexpr double kMassUnit = 1.0 / 8796093022208.0;   // 2^-43: sums of up to 2^20 weights fit 64 bits
constexpr uint64_t kKeyTop = (uint64_t(1) << (32 + kColumnBits)) - 1;

struct CutShared {
  union {
    struct {
      uint64_t mass[kBins];
      uint32_t count[kBins];
      uint64_t list[kListMax];
    };
    double group[kCutWaves][kMaxGroups];
  };
  union {
    double d[kCutWaves];
    uint64_t u[kCutWaves];
    uint32_t i[kCutWaves];
  } red;
  uint64_t before;
  uint32_t n;
  int pick, last;
};

// Calls f(group, value, column) for every unmasked entry of the row; group g is the g-th run of
// kCutThreads vectors, and after(g) follows a group's entries with all lanes together.
template <typename T, typename F, typename G>
__device__ __forceinline__ void each_entry(const LogitRow<T>& r, F f, G after) {
  constexpr int N = LogitRow<T>::N;
  const int nv = r.vectors();
  for (int b = 0; b < nv; b += kAhead * kCutThreads) {
    float x[kAhead][N];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const int j = b + q * kCutThreads + int(threadIdx.x);
#pragma unroll
      for (int e = 0; e < N; ++e) x[q][e] = -INFINITY;
      if (j < nv) r.load(j, x[q]);
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const int g = b / kCutThreads + q;
      const int c = r.column(g * kCutThreads + int(threadIdx.x));
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (x[q][e] > -INFINITY) f(g, x[q][e], c + e);
      if (g * kCutThreads < nv) after(g);
    }
  }
}
template <typename T, typename F>
__device__ __forceinline__ void each_entry(const LogitRow<T>& r, F f) {
  each_entry(r, f, [](int) {});
}

// The list's first n entries (n <= kListMax) from the greatest key down.
__device__ __forceinline__ void sort_list(uint64_t* list, int n) {
  int P = 2;
  while (P < n) P *= 2;
  for (int i = threadIdx.x; i < P; i += kCutThreads)
    if (i >= n) list[i] = 0;
  __syncthreads();
  for (int size = 2; size <= P; size *= 2)
    for (int d = size / 2; d > 0; d /= 2) {
      const int i = 2 * d * (int(threadIdx.x) / d) + int(threadIdx.x) % d;
      if (i + d < P) {
        const uint64_t a = list[i], b = list[i + d];
        if ((a < b) == ((i & size) == 0)) {
          list[i] = b;
          list[i + d] = a;
        }
      }
      __syncthreads();
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
// list: the first by value, further ones by key, where the last range is one key.
template <bool BY_MASS, typename T>
__device__ uint64_t select_entry(const LogitRow<T>& r, double target, uint64_t floor, float m,
                                 double c2, float scale, CutShared& sh) {
  double above = 0.;
  uint64_t lo = 0, hi = kKeyTop;
  int shift = -1, bin = 0;   // shift -1: the bins by value
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
      sort_list(sh.list, n);
      int at;
      if (BY_MASS) {
        const uint64_t k = sh.list[threadIdx.x];
        const double w = int(threadIdx.x) < n ? entry_weight(entry_logit(k), m, c2) : 0.;
        double all;
        const double sum = block_scan<kCutWaves>(w, sh.red.d, all);
        if (int(threadIdx.x) < n && above + sum >= target) atomicMin(&sh.pick, int(threadIdx.x));
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
    shift = 0;
    while (((hi - lo) >> shift) >= uint64_t(kBins)) ++shift;
    __syncthreads();
  }
}

// One row a workgroup.  TOP: the first K entries and the log-sum-exp of the others; else the
// truncation and the draw.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kCutThreads)
row_cut_kernel(CutArgs a) {
  __shared__ CutShared sh;
  const int64_t row = blockIdx.x;
  const LogitRow<T> r(static_cast<const T*>(a.z) + row * a.ld, a.V);
  const int64_t si = TOP ? 0 : row / a.per;
  const float t = a.ts != nullptr ? a.ts[si] : a.t;
  const bool greedy = !(t > 0.f);
  const double inv_t = greedy ? 1. : 1. / double(t);
  const double c2 = 1.4426950408889634074 * inv_t;
  const float scale = float(64. * inv_t);

  uint64_t best = 0;
  uint32_t valid = 0;
  each_entry(r, [&](int, float z, int c) {
    const uint64_t k = entry_key(z, c);
    best = k > best ? k : best;
    ++valid;
  });
  best = block_fold<kCutWaves>(best, sh.red.u, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
  valid = block_fold<kCutWaves>(valid, sh.red.i, [](uint32_t x, uint32_t y) { return x + y; });
  const float m = entry_logit(best);

  if constexpr (TOP) {
    const int K = a.K;
    const int n = int(min(uint32_t(K), valid));
    uint64_t cut = 0;
    if (valid > uint32_t(K)) cut = select_entry<false>(r, double(K), 0, m, c2, scale, sh);
    if (threadIdx.x == 0) sh.n = 0;
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
    sort_list(sh.list, n);
    for (int i = threadIdx.x; i < K; i += kCutThreads) {
      const uint64_t k = sh.list[i < n ? i : 0];
      a.ids[row * K + i] = i < n ? entry_column(k) : -1;
      a.vals[row * K + i] = i < n ? entry_logit(k) : -INFINITY;
    }
    if (a.rest == nullptr) return;
    next = block_fold<kCutWaves>(next, sh.red.u, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
    const float top = entry_logit(next);
    double s = 0.;
    if (next != 0)
      each_entry(r, [&](int, float z, int c) {
        if (entry_key(z, c) < cut) s += entry_weight(z, top, c2);
      });
    s = block_fold<kCutWaves>(s, sh.red.d, [](double x, double y) { return x + y; });
    if (threadIdx.x == 0)
      a.rest[row] = next != 0 ? float(double(top) * inv_t + log(s)) : -INFINITY;
  } else {
    if (valid == 0 || greedy) {
      if (threadIdx.x == 0) {
        if (a.tok != nullptr) a.tok[row] = valid != 0 ? entry_column(best) : -1;
        a.kept[row] = valid != 0 ? 1 : 0;
        a.cut_logit[row] = valid > 1 ? m : -INFINITY;
        a.cut_index[row] = valid > 1 ? entry_column(best) : -1;
        a.lse[row] = valid != 0 ? 0. : -INFINITY;
      }
      return;
    }
    const int top_k = a.ks != nullptr ? a.ks[si] : a.k;
    const float top_p = a.ps != nullptr ? a.ps[si] : a.p;
    const float min_p = a.mps != nullptr ? a.mps[si] : a.mp;
    uint64_t cut = 0;
    if (top_k > 0 && uint32_t(top_k) < valid)
      cut = select_entry<false>(r, double(top_k), 0, m, c2, scale, sh);
    if (top_p < 1.f) {
      double s = 0.;
      each_entry(r, [&](int, float z, int c) {
        if (entry_key(z, c) >= cut) s += entry_weight(z, m, c2);
      });
      s = block_fold<kCutWaves>(s, sh.red.d, [](double x, double y) { return x + y; });
      // A target of 0 is reached by the first entry, not before it.
      const double target = fmax(double(top_p) * s, 1e-300);
      const uint64_t k = select_entry<true>(r, target, cut, m, c2, scale, sh);
      cut = k > cut ? k : cut;
    }
    if (min_p > 0.f) {
      const double least = fmin(double(min_p), 1.);
      const uint64_t k = uint64_t(least_value_key(m, [&](float z) {
                           return entry_weight(z, m, c2) >= least;
                         })) << kColumnBits;
      cut = k > cut ? k : cut;
    }

    // The kept entries: how many, the last of them, their weights' sums a group and wave.
    uint32_t kept = 0;
    uint64_t low = kKeyTop;
    double s = 0.;
    auto keeps = [&](float z, int c) { return entry_key(z, c) >= cut; };
    each_entry(
        r,
        [&](int, float z, int c) {
          if (!keeps(z, c)) return;
          const uint64_t k = entry_key(z, c);
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
    kept = block_fold<kCutWaves>(kept, sh.red.i, [](uint32_t x, uint32_t y) { return x + y; });
    low = block_fold<kCutWaves>(low, sh.red.u, [](uint64_t x, uint64_t y) { return x < y ? x : y; });
    const int groups = (r.vectors() + kCutThreads - 1) / kCutThreads;
    double gs = 0., mass;
    if (int(threadIdx.x) < groups)
      for (int w = 0; w < kCutWaves; ++w) gs += sh.group[w][threadIdx.x];
    const double run = block_scan<kCutWaves>(gs, sh.red.d, mass);
    if (threadIdx.x == 0) {
      const bool every = kept == valid;
      a.kept[row] = int32_t(kept);
      a.cut_logit[row] = every ? -INFINITY : entry_logit(low);
      a.cut_index[row] = every ? -1 : entry_column(low);
      a.lse[row] = double(m) * inv_t + log(mass);
    }
    if (a.tok == nullptr) return;
    // The draw: the group in which the running sum passes the target, then the entry.
    const double target = fmin(fmax(double(a.u[row]), 0.), 1.) * mass;
    if (threadIdx.x == 0) sh.pick = kCutThreads, sh.last = 0;
    __syncthreads();
    if (int(threadIdx.x) < groups && gs > 0.) {
      if (run > target) atomicMin(&sh.pick, int(threadIdx.x));
      atomicMax(&sh.last, int(threadIdx.x));
    }
    __syncthreads();
    const int g = min(sh.pick, sh.last);
    __syncthreads();
    if (int(threadIdx.x) == g) sh.group[0][0] = run - gs;
    if (threadIdx.x == 0) sh.pick = kCutThreads, sh.last = -1;
    __syncthreads();
    const double base = sh.group[0][0];
    float x[LogitRow<T>::N];
    const int j = g * kCutThreads + int(threadIdx.x), c = r.column(j);
    double mine = 0., all;
    if (j < r.vectors()) {
      r.load(j, x);
#pragma unroll
      for (int e = 0; e < LogitRow<T>::N; ++e) {
        const bool k = x[e] > -INFINITY && keeps(x[e], c + e);
        x[e] = k ? x[e] : -INFINITY;
        mine += entry_weight(x[e], m, c2);
        if (k) atomicMax(&sh.last, c + e);
      }
    }
    const double upto = base + block_scan<kCutWaves>(mine, sh.red.d, all);
    if (mine > 0. && upto > target) atomicMin(&sh.pick, int(threadIdx.x));
    __syncthreads();
    if (sh.pick < kCutThreads) {
      if (int(threadIdx.x) == sh.pick) {
        double before = upto - mine;
        int tok = -1;
#pragma unroll
        for (int e = 0; e < LogitRow<T>::N; ++e) {
          const double w = entry_weight(x[e], m, c2);
          before += w;
          if (w > 0. && (tok < 0 || before - w <= target)) tok = c + e;
        }
        a.tok[row] = tok;
      }
    } else if (threadIdx.x == 0) {
      a.tok[row] = sh.last;
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

template <bool TOP>
static hipError_t launch_cut(bool bf16, const CutArgs& a, hipStream_t s) {
  if (bf16)
    hipLaunchKernelGGL((row_cut_kernel<bf16_t, TOP>), dim3(unsigned(a.rows)), dim3(kCutThreads), 0, s, a);
  else
    hipLaunchKernelGGL((row_cut_kernel<float, TOP>), dim3(unsigned(a.rows)), dim3(kCutThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_truncate(bool bf16, const CutArgs& a, hipStream_t s) {
  return launch_cut<false>(bf16, a, s);
}
hipError_t launch_top_logits(bool bf16, const CutArgs& a, hipStream_t s) {
  return launch_cut<true>(bf16, a, s);
}

static size_t al256(size_t x) { return (x + 255) / 256 * 256; }

// Parts of a target row: 256 vectors each, of its least vectors and one for a row that starts
// inside one.
static int verify_parts(bool bf16, int V) {
  const int N = bf16 ? 8 : 4;
  return ((V + 2 * N - 2) / N + kVerifyThreads - 1) / kVerifyThreads;
}

size_t accept_truncated_ws_bytes(bool bf16, int n_seq, int K, int V) {
  const size_t rows = size_t(n_seq) * (K + 1);
  return al256(rows * 8) + 3 * al256(rows * 4) + al256(size_t(n_seq) * 4) +
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
  const hipError_t e = launch_truncate(target_bf16, c, s);
  if (e != hipSuccess) return e;
  if (draft_bf16)
    return target_bf16 ? launch_verify<bf16_t, bf16_t>(a, n_seq, parts, s)
                       : launch_verify<bf16_t, float>(a, n_seq, parts, s);
  return target_bf16 ? launch_verify<float, bf16_t>(a, n_seq, parts, s)
                     : launch_verify<float, float>(a, n_seq, parts, s);
}

}  // namespace hdf
