// Second launch of a row's cut (row_cut.hpp): a workgroup a row.  Its code runs once a row, mostly on
// the way to the next memory access or barrier, so it is kept short: the same few loops for all
// settings, nothing unrolled that memory does not need in flight.  What bounds it is the latency of
// those steps, 1 to 6 thousand cycles each, and for a nucleus beyond the lists the row's second pass,
// 18 vector instructions an entry.  Of 128 rows of 129280 fp32 logits it takes 10 us with top_k = 50, 14
// us for a nucleus of 5 entries, 42 us for one of 4000; of 1024 rows of 16 bits, a nucleus of 4600, 123
// us (the second pass, 99, at 2.7 TB/s and 72% of the vector issue).
#include "row_cut.hpp"

#include <type_traits>

namespace hdf {

constexpr int kBins = 2048;   // of the search
constexpr int kSearchBits = 43;   // of a weight: sums of up to 2^20 of them fit 64 bits
constexpr uint64_t kKeyTop = (uint64_t(1) << (32 + kColumnBits)) - 1;

// Entries of a border bin that are held at once.
constexpr int kBorderMax = 4096;

template <int NT, bool SEARCH, bool BORDER>
struct CutShared {
  static constexpr int W = NT / kWave;
  union {
    struct {
      uint64_t border[BORDER ? kBorderMax : 1];
      unsigned long long fine[BORDER ? NT : 1];
    };
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
    double group[W][(1 << kColumnBits) / (4 * NT) + 1];
  };
  union {
    double chunk[kMaxChunks];
    unsigned long long chunk_n[kMaxChunks];
  };
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
  double run[kWave];
  uint64_t before, best;
  double sum;
  float floor, near, edge[2];
  uint32_t n, valid, listed;
  int pick, last, last_m, top_bin, bins, span;   // span: of the bins of all chunks
};

// Calls f(value, column) for every unmasked entry of vectors j0 .. j1-1 of the row and after(g) with
// all lanes together behind the g-th run of NT of them; the loads of the next runs, 16 entries a
// thread, are in flight.
template <int NT, typename T, typename F, typename G>
__device__ __forceinline__ void each_entry(const LogitRow<T>& r, int j0, int j1, F f, G after) {
  constexpr int N = LogitRow<T>::N, Q = 16 / N;
  float x[Q][N], y[Q][N];
  auto load = [&](int g, float v[Q][N]) {
    const int first = j0 + g * NT;
    if (r.inside(first, Q * NT) && first + Q * NT <= j1) {
#pragma unroll
      for (int q = 0; q < Q; ++q) r.load_inside(first + q * NT + int(threadIdx.x), v[q]);
    } else {
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int j = first + q * NT + int(threadIdx.x);
#pragma unroll
        for (int e = 0; e < N; ++e) v[q][e] = -INFINITY;
        if (j < j1) r.load_raw(j, v[q]);
      }
    }
  };
  const int groups = (j1 - j0 + NT - 1) / NT;
  load(0, x);
#pragma unroll 1
  for (int g0 = 0; g0 < groups; g0 += Q) {
    load(g0 + Q, y);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int g = g0 + q, c = r.column(j0 + g * NT + int(threadIdx.x));
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (x[q][e] > -INFINITY) f(x[q][e], c + e);   // false for NaN
        x[q][e] = y[q][e];
      }
      if (g < groups) after(g);
    }
  }
}
template <int NT, typename T, typename F>
__device__ __forceinline__ void each_entry(const LogitRow<T>& r, F f) {
  each_entry<NT>(r, 0, r.vectors(), f, [](int) {});
}

// Exchanges of a bitonic sort within a wave, FROM, FROM / 2 .. 1 lanes apart, the greater key to the
// lower lane where `down`.
template <int FROM>
__device__ __forceinline__ uint64_t wave_merge(uint64_t k, bool down) {
  const uint64_t o = lane_xor<FROM>(k);
  k = (o > k) == (((threadIdx.x & FROM) == 0) == down) ? o : k;
  if constexpr (FROM > 1)
    return wave_merge<FROM / 2>(k, down);
  else
    return k;
}

// The wave's keys from the greatest down.
__device__ __forceinline__ uint64_t wave_sort(uint64_t k, bool down = true) {
  const uint32_t lane = threadIdx.x & 63;
  k = wave_merge<1>(k, (lane & 2) == 0);
  k = wave_merge<2>(k, (lane & 4) == 0);
  k = wave_merge<4>(k, (lane & 8) == 0);
  k = wave_merge<8>(k, (lane & 16) == 0);
  k = wave_merge<16>(k, (lane & 32) == 0);
  return wave_merge<32>(k, down);
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
#pragma unroll 1
  for (int s = wid; s * 64 < P; s += NT / kWave)
    list[s * 64 + lane] = wave_sort(list[s * 64 + lane], (s & 1) == 0);
  __syncthreads();
#pragma unroll 1
  for (int size = 128; size <= P; size *= 2) {
#pragma unroll 1
    for (int d = size / 2; d >= 64; d /= 2) {
      for (int t = threadIdx.x; t < P / 2; t += NT) {
        const int i = 2 * t - (t & (d - 1));
        const uint64_t a = list[i], b = list[i + d];
        if ((a < b) == ((i & size) == 0)) {
          list[i] = b;
          list[i + d] = a;
        }
      }
      __syncthreads();
    }
#pragma unroll 1
    for (int s = wid; s * 64 < P; s += NT / kWave)
      list[s * 64 + lane] = wave_merge<32>(list[s * 64 + lane], (s * 64 & size) == 0);
    __syncthreads();
  }
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

// The same where an estimate is at hand: the 64 values around it first.
template <typename F>
__device__ __forceinline__ uint32_t least_value_key(float m, float near, F holds) {
  const uint32_t h = f32_order_key(m), k = f32_order_key(near) - 32 + (threadIdx.x & 63);
  const bool in = k >= h || (k > 0x007FFFFFu && holds(f32_from_order_key(k)));
  const unsigned long long is = __ballot(in);
  if (is != 0ull && (is & 1ull) == 0ull)
    return read_lane(k, __ffsll(static_cast<long long>(is)) - 1);
  return least_value_key(m, holds);
}

// First-level bin of a value below the row's greatest one: 64 bins a unit of (m - z) / T, so
// monotone in the value.  Halves: the difference of two finite values may not be one.
__device__ __forceinline__ int value_bin(float z, float m, float scale) {
  return z == m ? 0 : int(fminf((0.5f * m - 0.5f * z) * (2.f * scale), float(kBins - 1)));
}

// Key of the entry with which the running sum, in order, of ones (BY_MASS false) or weights over
// the entries with keys >= floor reaches `target`; the last of them if rounding leaves none.
// Histograms of 2048 bins over ever smaller ranges of the order, until a bin's entries fit the
// list: the first by value, further ones by key, where the last range is one key.  A caller that
// knows the range of keys and the sum `above` it starts there (lo > 0).
// A weight counts as a multiple of 2^-(43 + e), e the whole octaves by which all of its bin (of the
// range, in those by key) stay below the row's greatest: to 2^-43 of itself, however light, down to
// 2^-46 of the greatest; lighter ones, all in the last bin by value, to 2^-89.  Integers, so that a
// bin's sum does not depend on its order; the bins' sums are added in 64-bit floating point.
template <int NT, bool BY_MASS, typename T, typename Shared>
__device__ uint64_t select_entry(const LogitRow<T>& r, double target, uint64_t floor, float m,
                                 double c2, float scale, Shared& sh, uint64_t lo = 0,
                                 uint64_t hi = kKeyTop, double above = 0.) {
  constexpr int W = NT / kWave, PER = kBins / NT, LISTED = kListMax / NT;
  auto shift_of = [&]() {
    int sh_ = 0;
    while (((hi - lo) >> sh_) >= uint64_t(kBins)) ++sh_;
    return sh_;
  };
  scale = fminf(scale, 1e38f);   // a finite one: no entry in a bin of lighter ones
  auto octaves_of = [&]() {   // of the range; kKeyTop is no value's
    return int(fmin((double(m) - double(fminf(entry_logit(hi), m))) * c2, 900.));
  };
  int shift = lo > 0 ? shift_of() : -1, bin = 0;   // shift -1: the bins by value
  int octaves = lo > 0 && BY_MASS ? octaves_of() : 0;
  for (;;) {
    for (int b = threadIdx.x; b < kBins; b += NT) {
      sh.count[b] = 0;
      sh.mass[b] = 0;
    }
    if (threadIdx.x == 0) sh.pick = kBins, sh.last = 0;
    __syncthreads();
    auto bin_of = [&](float z, uint64_t k) {
      return shift < 0 ? value_bin(z, m, scale) : int((hi - k) >> shift);
    };
    auto bits_of = [&](int b) {   // log2(e) / 64 octaves a bin by value
      return kSearchBits + (shift < 0 ? int(float(b) * 0.0225421f) : octaves);
    };
    each_entry<NT>(r, [&](float z, int c) {
      const uint64_t k = entry_key(z, c);
      if (k < floor || k < lo || k > hi) return;
      const int b = bin_of(z, k);
      atomicAdd(&sh.count[b], 1u);
      if (BY_MASS)
        atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]),
                  static_cast<unsigned long long>(ldexp(entry_weight(z, m, c2), bits_of(b)) + 0.5));
    });
    __syncthreads();
    const int b0 = PER * threadIdx.x;
    auto sum_of = [&](int b) { return BY_MASS ? ldexp(double(sh.mass[b]), -bits_of(b)) : double(sh.count[b]); };
    double own = 0., whole;
    int end = -1;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      own += sum_of(b0 + e);
      end = sh.count[b0 + e] != 0 ? b0 + e : end;
    }
    const double before = above + (block_scan<W>(own, sh.red.d, whole) - own);
    double upto = before;
    int first = -1;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const double v = sum_of(b0 + e);
      upto += v;
      first = first < 0 && v > 0. && upto >= target ? b0 + e : first;
    }
    note_first(first >= 0, first, &sh.pick);
    note_last(end >= 0, end, &sh.last);
    __syncthreads();
    bin = min(sh.pick, sh.last);
    if (int(threadIdx.x) == bin / PER) {
      upto = before;
      for (int b = b0; b < bin; ++b) upto += sum_of(b);
      sh.sum = upto;
    }
    __syncthreads();
    above = sh.sum;
    const uint32_t here = sh.count[bin];
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0, sh.pick = kListMax;
    __syncthreads();
    if (here <= uint32_t(kListMax)) {
      each_entry<NT>(r, [&](float z, int c) {
        const uint64_t k = entry_key(z, c);
        if (k < floor || k < lo || k > hi || bin_of(z, k) != bin) return;
        sh.list[atomicAdd(&sh.n, 1u)] = k;
      });
      __syncthreads();
      const int n = int(sh.n);
      sort_list<NT>(sh.list, n);
      int at;
      if (BY_MASS) {
        const int i0 = LISTED * threadIdx.x;
        double own_w = 0., all;
#pragma unroll 1
        for (int e = 0; e < LISTED; ++e)
          own_w += i0 + e < n ? entry_weight(entry_logit(sh.list[i0 + e]), m, c2) : 0.;
        double run = above + (block_scan<W>(own_w, sh.red.d, all) - own_w);
        int first = -1;
#pragma unroll 1
        for (int e = 0; e < LISTED; ++e)
          if (i0 + e < n) {
            run += entry_weight(entry_logit(sh.list[i0 + e]), m, c2);
            first = first < 0 && run >= target ? i0 + e : first;
          }
        note_first(first >= 0, first, &sh.pick);
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
    if (BY_MASS) octaves = octaves_of();
    __syncthreads();
  }
}

// The weights of a row's kept entries (those before or at `cut` in the order) among vectors
// j0 .. j1-1, a sum a group and wave in sh.group; returns their whole, `run` this thread's group's
// running sum and `mine` its own.  COUNT: also how many, and the last one's key, of this thread.
template <int NT, bool COUNT, typename Shared, typename T>
__device__ __forceinline__ double kept_masses(const LogitRow<T>& r, int j0, int j1, uint64_t cut,
                                              float m, double c2, Shared& sh, double& run,
                                              double& mine, uint32_t* kept = nullptr,
                                              uint64_t* low = nullptr) {
  double s = 0.;
  const float cz = entry_logit(cut);
  const int cc = entry_column(cut);
  each_entry<NT>(
      r, j0, j1,
      [&](float z, int c) {
        if (cut != 0 && !(z > cz || (z == cz && c <= cc))) return;
        if constexpr (COUNT) {
          const uint64_t k = entry_key(z, c);
          *low = k < *low ? k : *low;
          ++*kept;
        }
        s += entry_weight(z, m, c2);
      },
      [&](int g) {
        s = wave_fold(s, [](double u, double v) { return u + v; });
        if ((threadIdx.x & 63) == 0) sh.group[threadIdx.x >> 6][g] = s;
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
template <int NT, typename Shared, typename T>
__device__ __forceinline__ int draw_entry(const LogitRow<T>& r, int j0, int j1, uint64_t cut, float m,
                                          double c2, double base, double target, double run,
                                          double mine, Shared& sh) {
  if (threadIdx.x == 0) sh.pick = NT, sh.last = 0;
  __syncthreads();
  note_first(mine > 0. && base + run > target, threadIdx.x, &sh.pick);
  note_last(mine > 0., threadIdx.x, &sh.last);
  __syncthreads();
  const int g = min(sh.pick, sh.last);
  __syncthreads();
  if (int(threadIdx.x) == g) sh.sum = base + (run - mine);
  if (threadIdx.x == 0) sh.pick = NT, sh.last = -1;
  __syncthreads();
  const int j = j0 + g * NT + int(threadIdx.x), c = r.column(j);
  const float cz = entry_logit(cut);
  const int cc = entry_column(cut);
  constexpr int N = LogitRow<T>::N;
  float x[N];
  double w[N], own = 0., all;
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = -INFINITY;
  if (j < j1) r.load(j, x);
  int end = -1;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const bool is = x[e] > -INFINITY && (cut == 0 || x[e] > cz || (x[e] == cz && c + e <= cc));
    w[e] = entry_weight(is ? x[e] : -INFINITY, m, c2);
    own += w[e];
    end = is ? c + e : end;
  }
  note_last(end >= 0, end, &sh.last);
  const double upto = sh.sum + block_scan<NT / kWave>(own, sh.red.d, all);
  note_first(own > 0. && upto > target, threadIdx.x, &sh.pick);
  __syncthreads();
  const int who = sh.pick;
  __syncthreads();
  if (int(threadIdx.x) == who) {
    double before = upto - own;
    int tok = -1;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (w[e] > 0. && (tok < 0 || before <= target)) tok = c + e;
      before += w[e];
    }
    sh.last = tok;
  }
  __syncthreads();
  return sh.last;
}

// First place, among 0 .. n-1, whose running sum of w(i) reaches (STRICT: passes) `from` times the
// whole sum; n where none does.  `sum` gets the whole, sh.last the last place with a weight.
template <int NT, bool STRICT, typename Shared, typename F>
__device__ __forceinline__ int reach(int n, double from, double& sum, Shared& sh, F w) {
  const bool once = n <= NT;   // the sum and the place of one scan
  double target = 0.;
#pragma unroll 1
  for (int pass = once ? 1 : 0; pass < 2; ++pass) {   // the sum, then the place
    if (threadIdx.x == 0) sh.pick = n, sh.last = 0;
    double before = 0.;
#pragma unroll 1
    for (int b = 0; b < n; b += NT) {
      const int i = b + int(threadIdx.x);
      const double v = i < n ? w(i) : 0.;
      double all;
      const double run = before + block_scan<NT / kWave>(v, sh.red.d, all);
      before += all;
      if (once || pass == 0)   // 0 is reached by the first, not before
        target = STRICT ? from * before : fmax(from * before, 1e-300);
      if (pass == 1) {
        note_first(i < n && (STRICT ? v > 0. && run > target : run >= target), i, &sh.pick);
        note_last(v > 0., i, &sh.last);
      }
    }
    __syncthreads();
    sum = before;
  }
  return sh.pick;
}

// The second launch's work in phases.  Of few rows one launch does it all, 512 threads a row (128 rows
// of 129280, a nucleus of 4000 entries 65 us in all, 81 with 256 threads, 62 with 1024; 60 rows of
// 32003, one of 4 entries 21, 22 and 23 us; in three launches 78 and 24).  Of many rows those that the
// lists do not settle are left to further launches of larger workgroups: one more pass, with few
// enough registers for many rows at a time, and the search (lists by 256 threads a row: 1024 rows, a
// nucleus of 5 entries 148 us in all, 153 by 512).
enum CutPhase { kAll, kLists, kBorder, kSearch };
enum { kDone = 0, kLeftBorder = 1, kLeftSearch = 2 };

// The chunks' statistics joined, by the first wave.
template <typename Shared>
__device__ __forceinline__ void join_chunks(const HeadStat* hs, int chunks, Shared& sh) {
  auto add = [](uint32_t u, uint32_t v) { return u + v; };
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    uint64_t best = 0;
    uint32_t valid = 0, listed = 0;
    float floor = -INFINITY, near = INFINITY;
    int top_bin = -2147483647, bins = 0;
#pragma unroll 1
    for (int c = lane; c < chunks; c += 64) {
      const HeadStat st = hs[c];
      sh.part[c] = {int(st.listed), st.top_bin, st.bins, st.rest_ref, st.rest};
      if (st.valid == 0) continue;
      const uint64_t k = entry_key(st.best, st.best_col);
      best = k > best ? k : best;
      valid += st.valid;
      listed += st.listed;
      floor = fmaxf(floor, st.floor);
      near = fminf(near, st.near);
      top_bin = st.bins > 0 ? max(top_bin, st.top_bin) : top_bin;
      bins = st.bins < 0 ? -1 : bins;
    }
    best = wave_fold(best, [](uint64_t u, uint64_t v) { return u > v ? u : v; });
    valid = wave_fold(valid, add);
    listed = wave_fold(listed, add);
    floor = wave_fold(floor, [](float u, float v) { return fmaxf(u, v); });
    near = wave_fold(near, [](float u, float v) { return fminf(u, v); });
    top_bin = wave_fold(top_bin, [](int u, int v) { return max(u, v); });
    bins = wave_fold(bins, [](int u, int v) { return min(u, v); });
    int span = 0;
#pragma unroll 1
    for (int c = lane; c < chunks; c += 64)
      if (sh.part[c].bins > 0) span = max(span, top_bin - sh.part[c].top_bin + sh.part[c].bins);
    span = wave_fold(span, [](int u, int v) { return max(u, v); });
    if (lane == 0) {
      sh.span = span;
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
}

// This thread's places of a row's lists, all in flight together; only_listed() masks those past a
// chunk's list, once the chunks' statistics are known.
template <int NT>
__device__ __forceinline__ void load_listed(const HeadArgs& h, int64_t at, uint64_t mine[kListMax / NT]) {
  const uint64_t* list = h.list + at * h.chunks * h.cap;
#pragma unroll
  for (int q = 0; q < kListMax / NT; ++q) {
    const int i = q * NT + int(threadIdx.x);
    mine[q] = list[i < h.chunks * h.cap ? i : 0];
  }
}
template <int NT, typename Shared>
__device__ __forceinline__ void only_listed(const HeadArgs& h, const Shared& sh, uint64_t mine[kListMax / NT]) {
#pragma unroll
  for (int q = 0; q < kListMax / NT; ++q) {
    const uint32_t i = q * NT + threadIdx.x, c = i / uint32_t(h.cap);
    const bool is = c < uint32_t(h.chunks) && int(i - c * h.cap) < sh.part[c < uint32_t(h.chunks) ? c : 0].listed;
    mine[q] = is ? mine[q] : 0ull;
  }
}
// The listed entries of value >= t into the list; how many.
template <int NT, typename Shared>
__device__ __forceinline__ int gather(const uint64_t mine[kListMax / NT], float t, Shared& sh) {
  __syncthreads();
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
  uint32_t own = 0;
#pragma unroll
  for (int q = 0; q < kListMax / NT; ++q) own += mine[q] != 0 && entry_logit(mine[q]) >= t;
  const uint32_t upto = wave_scan(own);
  uint32_t at = 0;
  if ((threadIdx.x & 63) == 63) at = atomicAdd(&sh.n, upto);
  at = read_lane(at, 63) + upto - own;
#pragma unroll
  for (int q = 0; q < kListMax / NT; ++q)
    if (mine[q] != 0 && entry_logit(mine[q]) >= t) sh.list[at++] = mine[q];
  __syncthreads();
  return int(sh.n);
}

// The first K entries of a row and the log-sum-exp of the others.
template <typename T, int NT, CutPhase PHASE>
__global__ void __launch_bounds__(NT)
row_top_kernel(CutArgs a, HeadArgs h) {
  constexpr bool LISTS = PHASE != kSearch, SEARCH = PHASE != kLists;
  constexpr int W = NT / kWave;
  __shared__ CutShared<NT, SEARCH, false> sh;
  const int64_t at = blockIdx.x, row = a.row0 + at;   // in the launch, in the call
  const int tid = threadIdx.x, K = a.K;
  if (PHASE == kSearch && h.notes[at].left != kLeftSearch) return;
  const LogitRow<T> r(static_cast<const T*>(a.z) + row * a.ld, a.V);
  const RowSettings s = settings_of<true>(a, row);
  auto add = [](double u, double v) { return u + v; };
  auto most64 = [](uint64_t u, uint64_t v) { return u > v ? u : v; };
  uint64_t mine[kListMax / NT];
  if constexpr (LISTS) load_listed<NT>(h, at, mine);
  join_chunks(h.stats + at * h.chunks, h.chunks, sh);
  const uint32_t valid = sh.valid;
  const int n = int(min(uint32_t(K), valid));
  int have = 0;
  bool done = false;
  if constexpr (LISTS) {
    only_listed<NT>(h, sh, mine);
    const float floor = sh.floor;
    // As far down as the chunks' shares go (every entry >= floor is listed), or to the floor.
    float t = fmaxf(floor, sh.near);
#pragma unroll 1
    for (;;) {
      have = gather<NT>(mine, t, sh);
      if (have >= n || t <= floor) break;
      t = floor;
    }
    done = have >= n;
    if (PHASE == kLists && tid == 0) h.notes[at].left = done ? kDone : kLeftSearch;
    if (done) {
      sort_list<NT>(sh.list, have);
      if (a.rest != nullptr) {
        const uint64_t last = n > 0 ? sh.list[n - 1] : 0;
        double ref = -INFINITY;
#pragma unroll
        for (int q = 0; q < kListMax / NT; ++q)
          if (mine[q] != 0 && mine[q] < last) ref = fmax(ref, double(entry_logit(mine[q])));
        const bool rest = tid < h.chunks && sh.part[tid].rest > 0.;
        if (rest) ref = fmax(ref, sh.part[tid].rest_ref);
        ref = block_fold<W>(ref, sh.red.d, [](double u, double v) { return fmax(u, v); });
        double sum = rest ? sh.part[tid].rest * exp2_64((sh.part[tid].rest_ref - ref) * s.c2) : 0.;
#pragma unroll
        for (int q = 0; q < kListMax / NT; ++q)
          if (mine[q] != 0 && mine[q] < last)
            sum += exp2_64((double(entry_logit(mine[q])) - ref) * s.c2);
        sum = block_fold<W>(sum, sh.red.d, add);
        if (tid == 0) a.rest[row] = sum > 0. ? float(ref * s.inv_t + log(sum)) : -INFINITY;
      }
    } else if (PHASE == kLists) {
      return;
    }
  }
  if constexpr (SEARCH) {
    if (!done) {
      __syncthreads();
      const uint64_t cut = valid > uint32_t(K) ? select_entry<NT, false>(r, double(K), 0, entry_logit(sh.best),
                                                                     s.c2, float(64. * s.inv_t), sh)
                                               : 0;
      if (tid == 0) sh.n = 0;
      __syncthreads();
      uint64_t next = 0;   // the first entry past the list
      each_entry<NT>(r, [&](float z, int c) {
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
          each_entry<NT>(r, [&](float z, int c) {
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
}

// The row's entries with end <= z < over, up to kBorderMax of them, in sh.border: how many there are.
// greater: how many lie above.  First their columns, then the values of all at once.
template <int NT, typename T, typename Shared>
__device__ __forceinline__ int border_entries(const LogitRow<T>& r, float end, float over,
                                              uint32_t& greater, Shared& sh) {
  constexpr int N = LogitRow<T>::N, Q = 32 / N;
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid == 0) sh.n = 0;
  __syncthreads();
  uint32_t up = 0;
  const int nv = r.vectors();
#pragma unroll 1
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
        const bool is = x[q][e] >= over;
        up += uint32_t(__popcll(__ballot(is)));
        bits = 2 * bits + uint32_t(x[q][e] >= end && !is);
      }
    const uint32_t own = __popc(bits), upto = wave_scan(own);
    uint32_t at = 0;
    if (lane == 63) at = atomicAdd(&sh.n, upto);
    at = read_lane(at, 63) + upto - own;
    while (bits != 0) {
      const int q = 32 - __ffs(bits);
      bits &= bits - 1;
      if (at < uint32_t(kBorderMax)) sh.border[at] = uint64_t(r.column(b + q / N * NT + tid) + q % N);
      ++at;
    }
  }
  greater = block_fold<NT / kWave>(lane == 0 ? up : 0u, sh.red.i,
                                   [](uint32_t u, uint32_t v) { return u + v; });
  const int n = int(sh.n);
  for (int i = tid; i < min(n, kBorderMax); i += NT) {
    const int c = int(sh.border[i]);
    sh.border[i] = entry_key(r.raw(c), c);
  }
  __syncthreads();
  return n;
}

// Masses relative to the greatest entry's weight: integers of a bin over that of the greatest entry,
// which is w0.  Correctly rounded, from two exact halves, so that n equal entries at the top weigh n
// and a cut or a draw among them falls where their count says.
struct TopWeight {
  double w0, inv;
  __device__ __forceinline__ double over(double hi, double lo) const {   // (2^32 hi + lo) / w0
    const double s = fma(hi, 4294967296., lo), rest = lo - fma(hi, -4294967296., s);
    const double q = s * inv;
    return fma(fma(-q, w0, s) + rest, inv, q);
  }
  __device__ __forceinline__ double over(uint64_t n) const {
    return over(double(uint32_t(n >> 32)), double(uint32_t(n)));
  }
};

// Key, among the n border entries, all of one bin, at which `above` and the running sum of their
// weights in the order, times w_bin, reach the target; the last one if rounding leaves none.  Masses
// over ever smaller ranges of keys; sorting the entries instead took three times as long.
template <int NT, typename Shared>
__device__ __forceinline__ uint64_t border_entry(int n, uint64_t lo, uint64_t hi, double k16, double above,
                                                 const TopWeight& top, double w_bin, double target,
                                                 Shared& sh) {
  const int tid = threadIdx.x;
  const double c5 = mass_coefficient(kBits);
  uint64_t base = 0;
#pragma unroll 1
  while (lo < hi) {
    int shift = 0;
    while (((hi - lo) >> shift) >= uint64_t(NT)) ++shift;
    sh.fine[tid] = 0;
    if (tid == 0) sh.pick = NT, sh.last = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
      const uint64_t k = sh.border[i];
      int bin;
      if (k >= lo && k <= hi)
        atomicAdd(&sh.fine[(hi - k) >> shift],
                  static_cast<unsigned long long>(weight_in_bin(entry_logit(k), k16, c5, bin)));
    }
    __syncthreads();
    const uint64_t own = sh.fine[tid];
    uint64_t all;
    const uint64_t upto = base + block_scan<NT / kWave>(own, sh.red.u, all);
    note_first(own > 0 && above + top.over(upto) * w_bin >= target, tid, &sh.pick);
    note_last(own > 0, tid, &sh.last);
    __syncthreads();
    const int at = min(sh.pick, sh.last);
    const bool few = sh.fine[at] < (uint64_t(62) << 48);   // fewer than 64: they weigh 0.978 at least
    if (tid == at) sh.before = upto - own;
    hi -= uint64_t(at) << shift;
    const uint64_t least = hi - ((uint64_t(1) << shift) - 1);
    lo = least > lo ? least : lo;
    if (few) {   // every wave sorts and sums them for itself
      if (tid == 0) sh.n = 0;
      __syncthreads();
      base = sh.before;
      for (int i = tid; i < n; i += NT) {
        const uint64_t k = sh.border[i];
        if (k >= lo && k <= hi) sh.fine[atomicAdd(&sh.n, 1u)] = k;
      }
      __syncthreads();
      const int lane = tid & 63;
      uint64_t k = wave_sort(lane < int(sh.n) ? sh.fine[lane] : 0ull);
      int bin;
      const uint64_t w = k != 0 ? weight_in_bin(entry_logit(k), k16, c5, bin) : 0ull;
      const unsigned long long some = __ballot(k != 0);
      const double run = above + top.over(base + wave_scan(w)) * w_bin;
      const unsigned long long past = __ballot(k != 0 && run >= target);
      k = read_lane(k, past != 0ull ? __ffsll(static_cast<long long>(past)) - 1
                                    : 63 - __clzll(static_cast<long long>(some | 1ull)));
      __syncthreads();
      return k;
    }
    // The range that its entries take.
    uint64_t first = 0, last = kKeyTop;
    for (int i = tid; i < n; i += NT) {
      const uint64_t k = sh.border[i];
      const bool in = k >= lo && k <= hi;
      first = in && k > first ? k : first;
      last = in && k < last ? k : last;
    }
    hi = block_fold<NT / kWave>(first, sh.red.u, [](uint64_t u, uint64_t v) { return u > v ? u : v; });
    lo = block_fold<NT / kWave>(last, sh.red.u, [](uint64_t u, uint64_t v) { return u < v ? u : v; });
    base = sh.before;
  }
  __syncthreads();
  return hi;
}

// The draw among a row's kept entries of vectors j0 .. j1-1 (a chunk's, up to 64 runs of 64 a wave):
// the entry at which `base` and the running sum pass the target, the last one where rounding leaves
// none.  table: the weights of the bins' middles over the greatest entry's, which is 1 exactly; from
// `end` down entries have none.  A sum a run,
// gone through by every wave, then the run's entries by one.  A loop with D vectors in flight; all in
// registers was 5 KB of code, run once: 13 thousand cycles for 4096 entries where this takes 9.
template <int NT, int D, typename T, typename Shared>
__device__ __forceinline__ int draw_binned(const LogitRow<T>& r, int j0, int j1, uint64_t cut, float m,
                                           double k16, int top_bin, float end, const double* table,
                                           double base, double target, Shared& sh) {
  constexpr int N = LogitRow<T>::N, W = NT / kWave;
  static_assert(32 * kHeadThreads / N / NT * W <= kWave);
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const float cz = entry_logit(cut);
  const int cc = entry_column(cut);
  const double c5 = mass_coefficient(1.);
  auto add = [](double u, double v) { return u + v; };
  auto load = [&](int j, float x[N]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = -INFINITY;
    if (j < j1) r.load_raw(j, x);
  };
  auto weights = [&](int j, const float x[N], double w[N]) __attribute__((always_inline)) {
    double s = 0.;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      int n;
      const float z = x[e];
      const double p = bin_series<false>(fmaxf(z, end), k16, c5, n) * table[top_bin - n];
      const bool kept = z > end && (cut == 0 || z > cz || (z == cz && r.column(j) + e <= cc));
      w[e] = kept ? z == m ? 1. : p : 0.;
      s += w[e];
    }
    return s;
  };
  float x[D][N];
  double w[N];
#pragma unroll
  for (int d = 0; d < D; ++d) load(j0 + d * NT + tid, x[d]);
  const int groups = (j1 - j0 + NT - 1) / NT;
#pragma unroll 1
  for (int g = 0; g < groups; ++g) {
    const double s = wave_fold(weights(j0 + g * NT + tid, x[0], w), add);
    if (lane == 0) sh.run[g * W + wid] = s;
#pragma unroll
    for (int d = 0; d + 1 < D; ++d)
#pragma unroll
      for (int e = 0; e < N; ++e) x[d][e] = x[d + 1][e];
    load(j0 + (g + D) * NT + tid, x[D - 1]);
  }
  __syncthreads();
  const double v = lane < groups * W ? sh.run[lane] : 0., run = base + wave_scan(v);
  const unsigned long long any = __ballot(v > 0.), past = __ballot(v > 0. && run > target);
  const int at = past != 0ull ? __ffsll(static_cast<long long>(past)) - 1
                              : any != 0ull ? 63 - __clzll(static_cast<long long>(any)) : 0;
  if (wid == at % W) {
    const int j = j0 + at / W * NT + tid, c = r.column(j);
    load(j, x[0]);
    const double own = weights(j, x[0], w), before = read_lane(run, at) - read_lane(v, at);
    const double upto = before + wave_scan(own);
    const unsigned long long some = __ballot(own > 0.), over = __ballot(own > 0. && upto > target);
    const int who = over != 0ull ? __ffsll(static_cast<long long>(over)) - 1
                                 : 63 - __clzll(static_cast<long long>(some | 1ull));
    if (lane == who) {
      double sum = upto - own;
      int tok = -1;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (w[e] > 0. && (tok < 0 || sum <= target)) tok = c + e;
        sum += w[e];
      }
      sh.last = tok;
    }
  }
  __syncthreads();
  return sh.last;
}

// A draft's row of a verification: what its probabilities are taken from where its log-sum-exp is too
// far from 0 to tell them.  One workgroup a row, beside those that cut the target's rows: 8 sequences of
// 16 rows of 129280 take 103 us at T = 1e-8, 100 at 1e-6, where no row is far (45 at 1).
template <int NT, typename T, typename Shared>
__device__ __forceinline__ void far_draft(const CutArgs& a, int64_t e, Shared& sh) {
  const DraftRows& d = a.drafts;
  const int64_t s = e / d.K, row = s * d.stride + (e - s * d.K);
  const float t = a.ts != nullptr ? a.ts[s] : a.t;
  if (!(t > 0.f) || !far_lse(d.lse[row])) return;
  const LogitRow<T> r(static_cast<const T*>(d.z) + row * d.ld, a.V);
  const float cz = d.logit[row];
  const int cc = d.index[row];
  const double c2 = 1.4426950408889634074 / double(t);
  float m = -INFINITY;
  each_entry<NT>(r, [&](float z, int) { m = fmaxf(m, z); });
  m = block_fold<NT / kWave>(m, sh.red.f, [](float u, float v) { return fmaxf(u, v); });
  double sum = 0.;
  each_entry<NT>(r, [&](float z, int c) {
    if (z > cz || (z == cz && c <= cc)) sum += entry_weight(z, m, c2);
  });
  sum = block_fold<NT / kWave>(sum, sh.red.d, [](double u, double v) { return u + v; });
  if (threadIdx.x == 0) {
    d.top[e] = m;
    d.log_sum[e] = log(sum);
  }
}

// A row's truncation and draw; workgroups behind the rows' take a verification's drafts.
template <typename T, int NT, CutPhase PHASE>
__global__ void __launch_bounds__(NT, PHASE == kBorder ? 8 : 1)
row_cut_kernel(CutArgs a, HeadArgs h) {
  constexpr bool LISTS = PHASE == kAll || PHASE == kLists, BORDER = PHASE == kAll || PHASE == kBorder,
                 SEARCH = PHASE == kAll || PHASE == kSearch;
  constexpr int W = NT / kWave, PER = kMassBins / NT, LISTED = kListMax / NT;
  // Kept entries that are brought into token order to draw among them; of more (of a cut by weight),
  // whose masses the histograms hold, one chunk is read instead.  An entry a thread, so at most NT.
  // (One launch, min_p: 60 rows of 32003 that keep up to 747, 28.5 us by 512, 35.7 by 256; 200 rows, up
  // to 554, 40 by 512, 46 by 256.)
  constexpr int kInOrder = PHASE == kAll ? 512 : 256;
  __shared__ CutShared<NT, SEARCH, BORDER> sh;
  const int64_t at = blockIdx.x, row = a.row0 + at;   // in the launch, in the call
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  if (LISTS && at >= a.rows) {
    if (a.drafts.bf16)
      far_draft<NT, bf16_t>(a, at - a.rows, sh);
    else
      far_draft<NT, float>(a, at - a.rows, sh);
    return;
  }
  CutNote* note = h.notes + at;
  if (PHASE == kBorder && note->left != kLeftBorder) return;
  if (PHASE == kSearch && note->left != kLeftSearch) return;
  const LogitRow<T> r(static_cast<const T*>(a.z) + row * a.ld, a.V);
  const RowSettings s = settings_of<false>(a, row);
  auto add = [](auto u, auto v) { return u + v; };
  auto most64 = [](uint64_t u, uint64_t v) { return u > v ? u : v; };
  auto least64 = [](uint64_t u, uint64_t v) { return u < v ? u : v; };
  auto leave = [&](int left) {
    if (tid == 0) note->left = left;
  };
  uint64_t mine[LISTED];
  if (LISTS && !s.greedy && !s.open) load_listed<NT>(h, at, mine);
  join_chunks(h.stats + at * h.chunks, h.chunks, sh);
  const uint64_t best = sh.best;
  const uint32_t valid = sh.valid, listed = sh.listed;
  const float m = entry_logit(best), floor = sh.floor;
  const int top_bin = sh.top_bin;
  const bool whole = listed == valid;   // nothing is unlisted
  const bool binned = s.binned && sh.bins == 0;
  if (PHASE == kLists) leave(kDone);

  if (LISTS && (valid == 0 || s.greedy)) {
    if (tid == 0) {
      if (a.tok != nullptr) a.tok[row] = valid != 0 ? entry_column(best) : -1;
      a.kept[row] = valid != 0 ? 1 : 0;
      a.cut_logit[row] = valid > 1 ? m : -INFINITY;
      a.cut_index[row] = valid > 1 ? entry_column(best) : -1;
      a.lse[row] = valid != 0 ? 0. : -INFINITY;
    }
    return;
  }
  const bool has_k = s.top_k > 0 && uint32_t(s.top_k) < valid;
  const bool has_p = s.top_p < 1.f, has_m = s.min_p > 0.f;
  const double u = a.u != nullptr ? fmin(fmax(double(a.u[row]), 0.), 1.) : 0.;
  auto write = [&](uint32_t kept, uint64_t low, double mass, int tok) {
    if (tid != 0) return;
    const bool every = kept == valid;
    a.kept[row] = int32_t(kept);
    a.cut_logit[row] = every ? -INFINITY : entry_logit(low);
    a.cut_index[row] = every ? -1 : entry_column(low);
    const double rel = log(mass);
    a.lse[row] = double(m) * s.inv_t + rel;
    if (a.top != nullptr) {
      a.top[row] = m;
      a.log_sum[row] = rel;
    }
    if (a.tok != nullptr) a.tok[row] = tok;
  };

  if constexpr (LISTS) only_listed<NT>(h, sh, mine);

  // Least value of weight min_p, as the key of its last possible entry.
  uint64_t cut_m = 0;
  if (has_m && (LISTS || !binned)) {
    const double least = fmin(double(s.min_p), 1.);
    const uint32_t k = least_value_key(m, float(double(m) + log(least) / s.inv_t), [&](float z) {
      return entry_weight(z, m, s.c2) >= least;
    });
    cut_m = uint64_t(f32_order_key(f32_from_order_key(k) + 0.f)) << kColumnBits;
  } else if (has_m) {
    cut_m = note->cut_m;
  }

  // A cut by weight: the histograms joined.  The border bin is that of top_p's cut or of min_p's.
  const double k16 = 16. * s.c2;
  double whole_w = 0., above = 0.;   // relative to the greatest entry: the whole, the bins above
  int border = 0;
  float end = 0.f, over = INFINITY;   // the values of the border bin: end <= z < over
  bool by_p = false;   // whether top_p's cut lies in it
  auto bin_weight = [&](int b) { return exp2_64(-double(b) / 16.); };
  TopWeight top{1., 1.};
  if (binned) {
    int n;
    top.w0 = double(weight_in_bin(m, k16, mass_coefficient(kBits), n));
    top.inv = 1. / top.w0;
  }
  const uint64_t* masses = h.mass + at * h.chunks * kMassBins;
  auto mass_at = [&](int c, int b) -> uint64_t {   // of chunk c in the row's bin b
    const int i = b - (top_bin - sh.part[c].top_bin);
    const bool is = i >= 0 && i < sh.part[c].bins;
    const uint64_t n = masses[int64_t(c) * kMassBins + (is ? i : 0)];   // loaded in any case
    return is ? n : 0ull;
  };
  if constexpr (LISTS) {
    // P consecutive bins a thread, of sixteen loads in flight together.
    auto join_masses = [&](auto bins_each) __attribute__((always_inline)) {
      constexpr int P = decltype(bins_each)::value, AHEAD = 16 / P;
      double v[P], lo[P], sum = 0.;   // high and low halves: exact sums
#pragma unroll
      for (int e = 0; e < P; ++e) v[e] = lo[e] = 0.;
#pragma unroll 1
      for (int c0 = 0; c0 < h.chunks; c0 += AHEAD) {
        uint64_t x[AHEAD][P];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
          for (int e = 0; e < P; ++e) x[i][e] = mass_at(min(c0 + i, h.chunks - 1), P * tid + e);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const uint64_t n = c0 + i < h.chunks ? x[i][e] : 0ull;
            v[e] += double(uint32_t(n >> 32));
            lo[e] += double(uint32_t(n));
          }
      }
      if (tid == 0) sh.pick = kMassBins, sh.last = 0, sh.last_m = 0;
#pragma unroll
      for (int e = 0; e < P; ++e) {
        v[e] = top.over(v[e], lo[e]) * bin_weight(P * tid + e);
        sum += v[e];
      }
      const double run = block_scan<W>(sum, sh.red.d, whole_w);
      const double target = has_p ? fmax(double(s.top_p) * whole_w, 1e-300) : INFINITY;
      // min_p's bin: the last one with entries up to that of its least value.
      const int bin_m = has_m ? min(top_bin - weight_bin(entry_logit(cut_m), k16), kMassBins - 1) : -1;
      double upto = run - sum;
      int first = -1, last = -1, last_m = -1;
#pragma unroll
      for (int e = 0; e < P; ++e) {
        const int b = P * tid + e;
        upto += v[e];
        last = v[e] > 0. ? b : last;
        last_m = v[e] > 0. && b <= bin_m ? b : last_m;
        first = first < 0 && v[e] > 0. && upto >= target ? b : first;
      }
      note_first(first >= 0, first, &sh.pick);
      note_last(last >= 0, last, &sh.last);
      if (has_m) note_last(last_m >= 0, last_m, &sh.last_m);
      __syncthreads();
      border = min(sh.pick, sh.last);
      by_p = has_p && (!has_m || border <= sh.last_m);
      if (has_m) border = min(border, sh.last_m);
      upto = run - sum;
#pragma unroll
      for (int e = 0; e < P; ++e) {
        if (P * tid + e == border) sh.sum = upto;
        upto += v[e];
      }
      __syncthreads();
      above = sh.sum;
    };
    if (binned && !s.open) {
      if (sh.span <= 2 * NT)
        join_masses(std::integral_constant<int, 2>());
      else
        join_masses(std::integral_constant<int, PER>());
      if (PHASE == kLists && tid == 0)
        note->whole = whole_w, note->above = above, note->border = border, note->by_p = by_p,
        note->cut_m = cut_m;
    }
  } else if (binned) {
    whole_w = note->whole;
    above = note->above;
    border = note->border;
    by_p = note->by_p != 0;
    end = note->end;
    over = note->over;
  }
  // The least values of the border bin and of the bin before: end <= z < over.
  auto find_edges = [&]() {
    if (wid < 2) {
      const int b = border - wid;
      const float near = float((double(top_bin - b) - 0.5) * (double(s.t) * kLog16));
      const float z = b < 0 ? INFINITY : f32_from_order_key(least_value_key(m, near, [&](float z) {
        return double(z) * k16 > double(top_bin) - 2048. && weight_bin(z, k16) >= top_bin - b;
      }));   // (far values have no bin)
      if (lane == 0) sh.edge[wid] = z;
    }
    __syncthreads();
    end = sh.edge[0];
    over = sh.edge[1];
    __syncthreads();
  };
  const double target_p = fmax(double(s.top_p) * whole_w, 1e-300);   // 0 is reached by the first

  uint64_t cut = 0;
  if constexpr (LISTS) {
    if (binned && !s.open) find_edges();
    // The kept entries and those that the cut lies among, if they are listed, sorted.  Under a cut by
    // weight only a few: of more, whose masses the histograms hold, one chunk is read instead.
    int n = 0, k = 0;
    if (binned ? !s.open && end >= floor : has_k || whole) {
      float t = binned ? end : has_k ? fmaxf(floor, sh.near) : floor;
#pragma unroll 1
      for (;;) {
        n = gather<NT>(mine, t, sh);
        if (!has_k || n >= s.top_k || t <= floor) break;
        t = floor;
      }
    }
    // The greatest entry is among them and is kept.
    if (n > 0 && !(has_k && n < s.top_k) && !(binned && n > kInOrder)) {
      sort_list<NT>(sh.list, n);
      for (int i = tid; i < n; i += NT) sh.weight[i] = entry_weight(entry_logit(sh.list[i]), m, s.c2);
      __syncthreads();
      k = has_k ? s.top_k : n;
      if (binned && by_p) {   // as the histograms count them
        static_assert(kInOrder <= NT);
        int bin;
        const float z = tid < n ? entry_logit(sh.list[tid]) : INFINITY;
        const uint64_t own = z < over ? weight_in_bin(z, k16, mass_coefficient(kBits), bin) : 0ull;
        uint64_t all;
        if (tid == 0) sh.pick = n - 1;
        const uint64_t run = block_scan<W>(own, sh.red.u, all);
        note_first(own != 0 && above + top.over(run) * bin_weight(border) >= target_p, tid, &sh.pick);
        __syncthreads();
        k = min(k, sh.pick + 1);
      } else if (!binned && has_p) {
        double sum;
        const int p = reach<NT, false>(k, double(s.top_p), sum, sh, [&](int i) { return sh.weight[i]; });
        k = min(k, p + 1);
      }
      if (cut_m != 0) {
        uint32_t c = 0;
        for (int i = tid; i < k; i += NT) c += sh.list[i] >= cut_m;
        k = int(block_fold<W>(c, sh.red.i, add));
      }
    }
    if (k > 0) {
      // In token order: columns with the weights' places as keys.
      const uint64_t low = sh.list[k - 1];
      __syncthreads();
      for (int i = tid; i < k; i += NT) sh.list[i] = ((sh.list[i] & kColumnMask) << 12) | uint64_t(i);
      __syncthreads();
      sort_list<NT>(sh.list, k);
      double mass;
      int i = reach<NT, true>(k, u, mass, sh, [&](int q) { return sh.weight[sh.list[q] & 4095u]; });
      if (i == k) i = sh.last;   // rounding left none: the last with a weight
      write(uint32_t(k), low, mass, int(kColumnMask - uint32_t(sh.list[i] >> 12)));
      return;
    }
    if (PHASE == kLists && tid == 0) {
      note->border = border, note->by_p = by_p, note->end = end, note->over = over;
      note->left = binned ? kLeftBorder : kLeftSearch;
    }
  }
  if (PHASE == kAll) __syncthreads();
  if constexpr (BORDER) {
    if (binned) {
      // min_p's cut may lie above all of its bin's entries, if it has any: the last bin before that has.
      auto bin_before = [&]() {
        if (tid == 0) sh.last = 0;
        __syncthreads();
        for (int b0 = 0; b0 < border; b0 += NT) {   // whole waves
          const int b = b0 + tid;
          uint64_t any = 0;
          for (int c = 0; b < border && c < h.chunks; ++c) any |= mass_at(c, b);
          note_last(any != 0, b, &sh.last);
        }
        __syncthreads();
        border = sh.last;
        by_p = false;
        __syncthreads();
        find_edges();
      };
      uint32_t greater = valid;
      int n = 0;
      const bool fits = s.open || [&]() {
        for (;;) {
          n = border_entries<NT>(r, end, over, greater, sh);
          if (n > kBorderMax) return false;
          cut = cut_m;
          if (by_p)
            cut = most64(cut, border_entry<NT>(n, uint64_t(f32_order_key(end)) << kColumnBits,
                                               uint64_t(f32_order_key(over)) << kColumnBits, k16, above,
                                               top, bin_weight(border), target_p, sh));
          uint64_t low = kKeyTop;
          uint32_t kept = 0;
          for (int i = tid; i < n; i += NT) {
            const uint64_t k = sh.border[i];
            kept += k >= cut;
            low = k >= cut && k < low ? k : low;
          }
          kept = block_fold<W>(kept, sh.red.i, add);
          cut = block_fold<W>(low, sh.red.u, least64);
          greater += kept;
          if (kept > 0) return true;
          bin_before();
        }
      }();
      if (fits) {
        // The chunks' masses: their part of the border's entries, their bins above it.
        if (s.open) border = min(sh.span, kMassBins);
        for (int c = tid; c < h.chunks; c += NT) sh.chunk_n[c] = 0;
        __syncthreads();
        const double c5 = mass_coefficient(kBits);
        for (int i = tid; i < n; i += NT) {
          const uint64_t k = sh.border[i];
          const int j = (entry_column(k) + r.shift) / LogitRow<T>::N;
          int b;
          if (k >= cut)
            atomicAdd(&sh.chunk_n[j / h.vectors],
                      static_cast<unsigned long long>(weight_in_bin(entry_logit(k), k16, c5, b)));
        }
        __syncthreads();
        // Weights of the bins' middles, relative to the greatest entry's, over the border's entries.
        double* table = reinterpret_cast<double*>(sh.border);
        for (int b = tid; b < kMassBins; b += NT)
          table[b] = b < kKeptBins ? bin_weight(b) : 0.;
        __syncthreads();
#pragma unroll 1
        for (int c = wid; c < h.chunks; c += W) {
          double w = lane == 0 && n > 0 ? top.over(sh.chunk_n[c]) * table[border] : 0.;
#pragma unroll 1
          for (int b0 = lane; b0 < border; b0 += 256) {
            uint64_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = b0 + 64 * i < border ? mass_at(c, b0 + 64 * i) : 0ull;
#pragma unroll
            for (int i = 0; i < 4; ++i) w += top.over(v[i]) * table[min(b0 + 64 * i, kMassBins - 1)];
          }
          w = wave_fold(w, add);
          if (lane == 0) sh.chunk[c] = w;
        }
        __syncthreads();
        for (int b = tid; b < kMassBins; b += NT) table[b] *= top.inv / kMassUnit;   // for the draw
        // The draw: only the chunk that the running sum passes the target in is read.
        const double w = tid < h.chunks ? sh.chunk[tid] : 0.;
        double mass;
        const double run = block_scan<W>(w, sh.red.d, mass);
        int tok = -1;
        if (a.tok != nullptr) {
          const double target = u * mass;
          if (tid == 0) sh.pick = NT, sh.last = 0;
          __syncthreads();
          note_first(w > 0. && run > target, tid, &sh.pick);
          note_last(w > 0., tid, &sh.last);
          __syncthreads();
          const int c = min(sh.pick, sh.last);
          if (tid == c) sh.sum = run - w;
          __syncthreads();
          const int j0 = c * h.vectors, j1 = min(r.vectors(), j0 + h.vectors);
          const float far = m - float(double(s.t) * kLog16) * float(kKeptBins + 4);
          tok = draw_binned<NT, PHASE == kAll ? 4 : 2>(r, j0, j1, cut, m, k16, top_bin, far, table,
                                                           sh.sum, target, sh);
        }
        write(greater, cut, mass, tok);
        return;
      }
    }
    if (PHASE == kBorder) {
      leave(kLeftSearch);
      return;
    }
  }
  if constexpr (SEARCH) {
    // Neither the lists nor the histograms tell: counts of very many entries, values beyond the
    // bins, border bins of more entries than are sorted.
    const float scale = float(64. * s.inv_t);
    cut = has_k ? select_entry<NT, false>(r, double(s.top_k), 0, m, s.c2, scale, sh) : 0;
    if (binned ? by_p : has_p) {
      uint64_t from = 0, to = kKeyTop;
      double all = whole_w;
      if (binned) {
        from = entry_key(end, a.V - 1);
        to = border > 0 ? (uint64_t(f32_order_key(over)) << kColumnBits) - 1 : kKeyTop;
      } else {
        all = 0.;
        each_entry<NT>(r, [&](float z, int c) {
          if (entry_key(z, c) >= cut) all += entry_weight(z, m, s.c2);
        });
        all = block_fold<W>(all, sh.red.d, add);
      }
      // A target of 0 is reached by the first entry, not before it.
      cut = most64(cut, select_entry<NT, true>(r, fmax(double(s.top_p) * all, 1e-300), cut, m, s.c2, scale,
                                           sh, from, to, binned ? above : 0.));
    }
    cut = most64(cut, cut_m);
    double run, own;
    uint32_t kept = 0;
    uint64_t low = kKeyTop;
    const double mass =
        kept_masses<NT, true>(r, 0, r.vectors(), cut, m, s.c2, sh, run, own, &kept, &low);
    kept = block_fold<W>(kept, sh.red.i, add);
    low = block_fold<W>(low, sh.red.u, least64);
    const int tok = a.tok != nullptr ? draw_entry<NT>(r, 0, r.vectors(), cut, m, s.c2, 0., u * mass, run,
                                                      own, sh)
                                     : -1;
    write(kept, low, mass, tok);
  }
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
constexpr int kListThreads = 256, kBorderThreads = 512, kSearchThreads = 1024;
constexpr int kAllThreads = 512;
// Whether one launch does all: up to a row a CU, whose running sums a workgroup's threads hold.
constexpr int64_t kAllRows = 256;
static bool all_at_once(bool bf16, int64_t rows, int V) {
  return rows <= kAllRows && V <= kAllThreads * kAllThreads * (bf16 ? 8 : 4) - 16;
}

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
    hipError_t e = launch_row_head(bf16, TOP, pl.elems == 8, a, h, s);
    if (e != hipSuccess) return e;
    const dim3 rows{unsigned(a.rows)}, first{unsigned(a.rows + (r0 == 0 ? a.drafts.n : 0))};
    if (all_at_once(bf16, a.rows, a.V)) {
      if constexpr (TOP)
        hipLaunchKernelGGL((row_top_kernel<T, kAllThreads, kAll>), rows, dim3(kAllThreads), 0, s, a, h);
      else
        hipLaunchKernelGGL((row_cut_kernel<T, kAllThreads, kAll>), first, dim3(kAllThreads), 0, s, a, h);
    } else if constexpr (TOP) {
      hipLaunchKernelGGL((row_top_kernel<T, kListThreads, kLists>), rows, dim3(kListThreads), 0, s, a, h);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL((row_top_kernel<T, kSearchThreads, kSearch>), rows, dim3(kSearchThreads), 0, s, a, h);
    } else {
      hipLaunchKernelGGL((row_cut_kernel<T, kListThreads, kLists>), first, dim3(kListThreads), 0, s, a, h);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL((row_cut_kernel<T, kBorderThreads, kBorder>), rows, dim3(kBorderThreads), 0, s, a, h);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL((row_cut_kernel<T, kSearchThreads, kSearch>), rows, dim3(kSearchThreads), 0, s, a, h);
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

}  // namespace hdf
