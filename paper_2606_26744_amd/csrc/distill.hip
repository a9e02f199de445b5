// Distillation from a teacher's stored top logits, forward and backward.  For draft slot k <= P of
// a block, p is the softmax at temperature T over the teacher's listed tokens S and, if given, the
// bucket of all others (whose log-sum-exp was stored with them); q = softmax(z / T) the student's:
//     kl = sum_S p_i (log p_i - log q_i) + p_r (log p_r - log q_r),   q_r = sum_{v not in S} q_v
//     T dkl/dz_v = q_v - p_v in S,   q_v (1 - p_r / q_r) outside (q_v without the bucket)
//     ce = log sum_v e^z_v - z_label,   dce/dz_v = softmax(z)_v - [v = label]
// Forward: one pass over the logits, whose workgroups keep a part of a row in registers between its
// greatest value and the sums; the rows' losses; their means.  Backward: one pass that forms every
// gradient from the row's statistics and then overwrites the few listed tokens'.  Memory bounds both
// of a large batch: 960 slots of 129280 16-bit logits 46 us forward alone (5.4 TB/s), 72 behind the
// backward pass of the step before, whose gradients still have to leave the caches; backward 98 us
// for 513 MB, 5.2 TB/s (a copy of the logits: 108).  Latency bounds a few dozen slots: 5 us the pass, 8
// to 11 the losses and their means, 6 the gradients.
#include "kernels.hpp"
#include "rows.hpp"

#include <type_traits>

namespace hdf {

constexpr int kDistThreads = 256;
constexpr int kDistWaves = kDistThreads / kWave;
constexpr int kDistElems = 32;                              // of a part, a thread
constexpr int kDistPart = kDistThreads * kDistElems;        // columns of a part
constexpr int kMaxTop = 1024;                               // K at most

// What a part of a row adds, with a bucket its unlisted columns alone (they may all lie hundreds of
// octaves below the listed ones, and the bucket's gradient is spread by their softmax): the greatest
// logit m, the sums of e^((z - mt) / T) and of e^(z - m1), mt and m1 being m but for rounding.
struct DistPart {
  float m;
  double mt, m1, st, s1;
};

// A supervised slot's statistics for the backward pass.
struct DistRow {
  float m, inv_t, inv_1;   // greatest logit; one over the sums at temperatures T and 1, relative to it
  float mu, unlisted;      // the columns' greatest, with a bucket the unlisted ones'; relative to it,
                           // 1 / (sum at T) less p_r / (unlisted sum)
  float shift;             // e^(mu - m)
  int kl, ce;              // whether the slot has either loss
};

// Saved between the passes: the number of labelled slots, the slots' statistics, p of the listed
// tokens (-1: no token, or one that stood before it in the list).
struct DistSaved {
  int* labelled;
  DistRow* rows;
  float* p;
};
static size_t al256(size_t x) { return (x + 255) / 256 * 256; }
static DistSaved saved_of(void* saved, int n_seq, int B) {
  char* s = static_cast<char*>(saved);
  return {reinterpret_cast<int*>(s), reinterpret_cast<DistRow*>(s + 256),
          reinterpret_cast<float*>(s + 256 + al256(size_t(n_seq) * (B - 1) * sizeof(DistRow)))};
}
size_t distill_saved_bytes(int n_seq, int B, int P, int K) {
  return 256 + al256(size_t(n_seq) * (B - 1) * sizeof(DistRow)) + al256(size_t(n_seq) * P * K * 4);
}

static int dist_parts(bool bf16, int V) {
  const int N = bf16 ? 8 : 4;
  return ((V + 2 * N - 2) / N * N + kDistPart - 1) / kDistPart;
}
size_t distill_ws_bytes(bool bf16, int n_seq, int B, int V) {
  return 256 + al256(size_t(n_seq) * (B - 1) * dist_parts(bf16, V) * sizeof(DistPart));
}

// Workgroup (part, slot): the slots are k = 1 .. slots of every block.
template <typename T>
__global__ void __launch_bounds__(kDistThreads)
distill_part_kernel(DistArgs a, int slots, DistPart* __restrict__ parts, uint32_t* done) {
  constexpr int N = LogitRow<T>::N, G = kDistElems / N;
  __shared__ uint32_t listed[kDistPart / 32];
  __shared__ float shf[kDistWaves], sums[kDistWaves][2];
  const int part = blockIdx.x;
  const int64_t i = blockIdx.y, s = i / slots;
  const int k = int(i - s * slots) + 1;
  const LogitRow<T> r(static_cast<const T*>(a.z) + (s * a.B + k) * a.ld, a.V);
  const int j0 = part * (kDistPart / N), nv = r.vectors();
  const bool soft = k <= a.P, bucket = soft && a.rest != nullptr;
  float x[G][N];
  if (r.inside(j0, G * kDistThreads)) {   // all but a row's first and last part
#pragma unroll
    for (int g = 0; g < G; ++g) r.load_inside(j0 + g * kDistThreads + int(threadIdx.x), x[g]);
  } else {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int j = j0 + g * kDistThreads + int(threadIdx.x);
#pragma unroll
      for (int e = 0; e < N; ++e) x[g][e] = -INFINITY;
      if (j < nv) r.load_raw(j, x[g]);
    }
  }
  if (bucket) {
    for (int w = threadIdx.x; w < kDistPart / 32; w += kDistThreads) listed[w] = 0;
    __syncthreads();
    const int32_t* ids = a.ids + (s * a.P + k - 1) * a.K;
    const int c0 = r.column(j0);
    for (int t = threadIdx.x; t < a.K; t += kDistThreads) {
      const int id = ids[t];
      const int b = id - c0;
      if (id >= 0 && id < a.V && b >= 0 && b < kDistPart) atomicOr(&listed[b >> 5], 1u << (b & 31));
    }
  }
  if (bucket) {
    __syncthreads();
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int at = (g * kDistThreads + int(threadIdx.x)) * N;
      const uint32_t is = listed[at >> 5] >> (at & 31) & ((1u << N) - 1);
      if (is != 0) {   // few
#pragma unroll
        for (int e = 0; e < N; ++e) x[g][e] = (is >> e) & 1u ? -INFINITY : x[g][e];
      }
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < N; e += 2) m = max3(m, x[g][e], x[g][e + 1]);
  m = block_fold<kDistWaves>(m, shf, [](float u, float v) { return fmaxf(u, v); });
  // An exponential costs one product, rounded once: 2^(z c - b), b the rounded product of m and c,
  // so relative to b / c.  Where that rounding is no small part of an octave (rows of the type's
  // lowest value), z - m first.
  const float ref = m == -INFINITY ? 0.f : m, log2e = 1.44269504f;
  const bool far = !(fabsf(ref) * fmaxf(soft ? a.c2 : 0.f, log2e) < 1e6f);
  const bool hard = a.labels != nullptr && !(soft && a.t == 1.f);
  // At T = 1 and at T: 32-bit sums of N values, then of few of those and over the wave, at most 15
  // additions in a row; 64-bit beyond.
  float sum[2] = {0.f, 0.f};
  auto weight = [&](bool is_far, float z, float c, float b) {
    return __builtin_amdgcn_exp2f(is_far ? (z - ref) * c : fmaf(z, c, -b));
  };
  auto exps_of = [&](auto is_far, float c) __attribute__((always_inline)) {
    const float b = ref * c;
    float v[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      v[g] = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) v[g] += weight(decltype(is_far)::value, x[g][e], c, b);
    }
#pragma unroll
    for (int d = 1; d < G; d *= 2)
#pragma unroll
      for (int g = 0; g < G; g += 2 * d) v[g] += v[g + d];
    return v[0];
  };
  auto exps = [&](float c) __attribute__((always_inline)) {
    return far ? exps_of(std::true_type(), c) : exps_of(std::false_type(), c);
  };
  if (hard) sum[0] = exps(log2e);
  if (soft) sum[1] = exps(a.c2);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float t = wave_fold(sum[i], [](float u, float v) { return u + v; });
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6][i] = t;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  if (part == 0 && i == 0) *done = 0;   // of the next launch
  double t[2] = {0., 0.};
#pragma unroll
  for (int w = 0; w < kDistWaves; ++w)
#pragma unroll
    for (int i = 0; i < 2; ++i) t[i] += double(sums[w][i]);
  DistPart o;
  o.m = m;
  o.mt = far ? double(ref) : double(ref * a.c2) / double(a.c2);
  o.m1 = far ? double(ref) : double(ref * log2e) / double(log2e);
  o.st = t[1];
  o.s1 = hard ? t[0] : o.st;
  parts[i * gridDim.x + part] = o;
}

// Values of all waves folded at once, f[i] into v[i]: one barrier, so `sh` is not to be written again
// before the next one.
template <int W, int N, typename F>
__device__ __forceinline__ void fold_all(double (&v)[N], double (&sh)[W][N], F f) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = wave_fold(v[i], [&](double x, double y) { return f(i, x, y); });
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = sh[0][i];
#pragma unroll
    for (int w = 1; w < W; ++w) v[i] = f(i, v[i], sh[w][i]);
  }
}

// loss = { L_KL = T^2 / P * mean over blocks of the sum of kl, L_CE = mean ce of the labelled
// slots, L_CE + alpha L_KL }, by one workgroup in a fixed order.  FRESH: kl and ce come from
// workgroups of the same launch, so past the caches.
template <int NT, bool FRESH>
__device__ __forceinline__ void distill_loss(const DistArgs& a, const DistSaved& sv,
                                             double (&sh)[NT / kWave][3]) {
  double v[3] = {0., 0., 0.};   // kl, ce; labelled slots
  auto sum = [&](const float* p, int n, double& s) {
    constexpr int Q = 4;   // loads in flight
    for (int i0 = threadIdx.x; i0 < n; i0 += Q * NT) {
      float x[Q];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const float* at = p + min(i0 + q * NT, n - 1);
        x[q] = FRESH ? __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : *at;
      }
#pragma unroll
      for (int q = 0; q < Q; ++q) s += i0 + q * NT < n ? double(x[q]) : 0.;
    }
  };
  sum(a.kl, a.n_seq * a.P, v[0]);
  if (a.labels != nullptr) {
    sum(a.ce, a.n_seq * (a.B - 1), v[1]);
    for (int i = threadIdx.x; i < a.n_seq * (a.B - 1); i += NT)
      v[2] += a.labels[i] >= 0 && a.labels[i] < a.V ? 1. : 0.;
  }
  fold_all(v, sh, [](int, double x, double y) { return x + y; });
  const double kl = v[0], ce = v[1], n = v[2];
  if (threadIdx.x == 0) {
    const double l_kl = double(a.t) * double(a.t) / a.P * kl / a.n_seq;
    const double l_ce = n > 0. ? ce / n : 0.;
    *sv.labelled = int(n);
    a.loss[0] = float(l_kl);
    a.loss[1] = float(l_ce);
    a.loss[2] = float(l_ce + double(a.alpha) * l_kl);
  }
}
constexpr int kLossThreads = 1024;
__global__ void __launch_bounds__(kLossThreads)
distill_loss_kernel(DistArgs a, DistSaved sv) {
  __shared__ double sh[kLossThreads / kWave][3];
  distill_loss<kLossThreads, false>(a, sv, sh);
}

// One workgroup a slot: the parts joined, the teacher's distribution, the losses; the one that ends
// last, by `done` (unless null), the losses' means.  A matter of
// latency: all loads but the listed logits' go out first, and five barriers separate its steps.
template <typename T, int NT>
__global__ void __launch_bounds__(NT)
distill_row_kernel(DistArgs a, int slots, const DistPart* __restrict__ parts, int n_parts,
                   DistSaved sv, uint32_t* done) {
  constexpr int Q = 4, W = NT / kWave;   // listed tokens of a thread, at most
  __shared__ int hash_id[2 * Q * NT], hash_at[2 * Q * NT];
  __shared__ double sh3[W][3], sh4[W][4], sh5[W][5], sh1[W][1];
  __shared__ uint32_t order;
  const int64_t i = blockIdx.x, s = i / slots;
  const int k = int(i - s * slots) + 1, tid = threadIdx.x;
  const LogitRow<T> r(static_cast<const T*>(a.z) + (s * a.B + k) * a.ld, a.V);
  const bool soft = k <= a.P, bucket = soft && a.rest != nullptr, one = soft && a.t == 1.f;
  const int64_t q = s * a.P + k - 1;
  int id[Q], slot[Q];
  double l[Q], z[Q];   // the teacher's logits over T, the student's
  double lr = -INFINITY;
  auto put = [](float* p, float x) {   // through the caches
    __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  const double inv_t = 1. / double(a.t);
  if (soft) {
    const int32_t* ids = a.ids + q * a.K;
    const float* tl = a.tl + q * a.K;
#pragma unroll
    for (int e = 0; e < Q; ++e) {
      const int t = e * NT + tid;
      id[e] = t < a.K ? ids[t] : -1;
      l[e] = t < a.K ? double(tl[t]) * inv_t : -INFINITY;
      if (id[e] >= a.V) id[e] = -1;
    }
    if (bucket) lr = double(a.rest[q]);
  }
  const DistPart* pt = parts + i * n_parts;
  DistPart first;
  first.m = -INFINITY;
  if (tid < n_parts) first = pt[tid];
  double label_z = 0.;
  int label = -1;
  if (a.labels != nullptr) {
    label = a.labels[s * (a.B - 1) + k - 1];
    if (label >= 0 && label < a.V) label_z = double(r.raw(label));
  }
  double v[4] = {-INFINITY, -INFINITY, 0., -INFINITY};   // greatest logit of the parts, the teacher's;
                                                         // its NaNs; the greatest of all
  v[0] = double(first.m);
  for (int j = tid + NT; j < n_parts; j += NT) v[0] = fmax(v[0], double(pt[j].m));
  int mask = 127;   // of the hash table: at least twice as many slots as tokens
  if (soft) {
#pragma unroll
    for (int e = 0; e < Q; ++e) z[e] = id[e] >= 0 ? double(r.raw(id[e])) : 0.;
    // A token's first place in the list holds: a table of tokens with their least place.
    while (mask + 1 < 2 * a.K) mask = 2 * mask + 1;
    for (int h = tid; h <= mask; h += NT) {
      hash_id[h] = -1;
      hash_at[h] = kMaxTop;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < Q; ++e) {
      if (id[e] < 0) continue;
      uint32_t h = (uint32_t(id[e]) * 2654435761u) >> 20 & uint32_t(mask);
      for (;;) {
        const int was = atomicCAS(&hash_id[h], -1, id[e]);
        if (was == -1 || was == id[e]) break;
        h = (h + 1) & uint32_t(mask);
      }
      slot[e] = int(h);
      atomicMin(&hash_at[h], e * NT + tid);
    }
    __syncthreads();
    v[1] = tid == 0 ? lr : -INFINITY;
    v[2] = tid == 0 && lr != -INFINITY ? lr - lr : 0.;   // NaN of NaN and +inf, else 0
#pragma unroll
    for (int e = 0; e < Q; ++e) {
      if (id[e] >= 0 && hash_at[slot[e]] != e * NT + tid) id[e] = -1;
      if (id[e] < 0) continue;
      v[1] = fmax(v[1], l[e]);
      v[3] = fmax(v[3], z[e]);
      v[2] += l[e] != -INFINITY ? l[e] - l[e] : 0.;
    }
  }
  fold_all(v, sh4, [](int e, double x, double y) { return e != 2 ? fmax(x, y) : x + y; });
  const double top = v[1], bad = v[2];
  const double most = fmax(v[0], v[3]), ref = most == -INFINITY ? 0. : most;
  // Without a column in the parts (all that are not listed are masked) the greatest of all: powers of
  // mu - ref are then 1, where another value's could pass the range and make NaNs of zero sums.
  const double mu = v[0] == -INFINITY ? ref : v[0];
  const bool taught = soft && (top > -INFINITY || bad != 0.);   // some mass, or a NaN to pass on
  const double c2 = 1.4426950408889634074 / double(a.t);
  constexpr double log2e = 1.4426950408889634074;
  // The parts' sums at T and at 1 (relative to mu), the teacher's, the listed tokens' (to the greatest).
  double u[5] = {0., 0., 0., 0., 0.};
  auto join = [&](const DistPart& o) {
    if (o.m == -INFINITY && o.st == o.st && o.s1 == o.s1) return;
    const double wt = exp2_64((o.mt - mu) * c2);
    u[0] += o.st * wt;
    u[1] += one ? o.s1 * wt : o.s1 * exp2_64((o.m1 - mu) * log2e);
  };
  if (tid < n_parts) join(first);
  for (int j = tid + NT; j < n_parts; j += NT) join(pt[j]);
  const double er = lr == -INFINITY || !taught ? 0. : exp(lr - top);
  double w[Q];
  if (taught) {
    u[2] = tid == 0 ? er : 0.;
#pragma unroll
    for (int e = 0; e < Q; ++e) {
      w[e] = id[e] >= 0 ? exp(l[e] - top) : 0.;
      u[2] += w[e];
    }
  }
  if (bucket) {
#pragma unroll
    for (int e = 0; e < Q; ++e) {
      if (id[e] < 0 || z[e] == -INFINITY) continue;
      const double nan = z[e] - z[e];   // of NaN and +inf, which the powers do not pass on; else 0
      u[3] += exp2_64((z[e] - ref) * c2) + nan;
      u[4] += exp2_64((z[e] - ref) * log2e) + nan;
    }
  }
  fold_all(u, sh5, [](int, double x, double y) { return x + y; });
  const double out = u[0], sum = u[2], to = (mu - ref) * inv_t;   // log of e^(mu / T) over e^(ref / T)
  const double st = out * exp2_64((mu - ref) * c2) + u[3];
  const double s1 = u[1] * exp2_64((mu - ref) * log2e) + u[4];
  // A row masked throughout has no softmax: its factors are 0, as its exponentials.
  DistRow row{float(ref), st == 0. ? 0.f : float(1. / st), s1 == 0. ? 0.f : float(1. / s1), float(mu),
              0.f, float(exp2_64((mu - ref) * log2e)), 0, 0};
  double unlisted = (st == 0. ? 0. : exp2_64((mu - ref) * c2) / st) + bad;
  if (soft) {
    float* ps = sv.p + q * a.K;
    double kl[1] = {0.};
    if (taught) {
      const double log_sum = log(sum), log_st = log(st);
#pragma unroll
      for (int e = 0; e < Q; ++e) {
        const int t = e * NT + tid;
        if (t >= a.K) continue;
        float stored = -1.f;
        if (id[e] >= 0) {
          const double p = w[e] / sum;
          const double lq = z[e] == -INFINITY ? -INFINITY : (z[e] - ref) * inv_t - log_st;
          kl[0] += p == 0. ? 0. : p * (l[e] - top - log_sum - lq);
          stored = float(p);
        }
        ps[t] = stored;
      }
      if (tid == 0 && er != 0.) {
        const double p = er / sum;
        const double lq = out == 0. ? -INFINITY : log(out) + to - log_st;
        kl[0] += p * (lr - top - log_sum - lq);
        if (out != 0.) unlisted -= p / out;
      }
      row.kl = 1;
    } else {
      for (int t = tid; t < a.K; t += NT) ps[t] = -1.f;
    }
    fold_all(kl, sh1, [](int, double x, double y) { return x + y; });
    if (tid == 0) put(a.kl + q, float(kl[0] + bad));
  }
  if (tid == 0) {
    if (a.labels != nullptr) {
      double ce = 0.;
      if (label >= 0 && label < a.V) {
        ce = label_z == -INFINITY ? INFINITY : (ref - label_z) + log(s1);
        row.ce = 1;
      }
      put(a.ce + s * (a.B - 1) + k - 1, float(ce));
    }
    row.unlisted = float(unlisted);
    sv.rows[s * (a.B - 1) + k - 1] = row;
    if (done != nullptr) {   // counted once they are in memory
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      order = __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (done == nullptr) return;
  __syncthreads();
  if (order == gridDim.x - 1) distill_loss<NT, true>(a, sv, sh3);
}

// Rounded by the conversion instruction, which keeps a NaN of any bits one.
__device__ __forceinline__ uint32_t bf16_bits(float v) {
  return __builtin_bit_cast(uint16_t, __bf16(v));
}
template <typename T>
__device__ __forceinline__ void store_grad(T* p, float v) {
  if constexpr (sizeof(T) == 2)
    *p = bf16_t(bf16_bits(v));
  else
    *p = v;
}

// Workgroup (part, row): the gradients of a part of a row; rows without a loss get zeros.
template <typename T>
__global__ void __launch_bounds__(kDistThreads)
distill_grad_kernel(DistArgs a, DistGrad g, DistSaved sv) {
  constexpr int N = LogitRow<T>::N, G = kDistElems / N;
  __shared__ int label_done;
  const int part = blockIdx.x, tid = threadIdx.x;
  const int64_t row = blockIdx.y, s = row / a.B;
  const int k = int(row - s * a.B);
  const LogitRow<T> r(static_cast<const T*>(a.z) + row * a.ld, a.V);
  T* d = static_cast<T*>(g.d) + row * g.ld;
  const bool vec = LogitRow<T>(d, a.V).shift == r.shift;
  const int j0 = part * (kDistPart / N), nv = r.vectors();
  // Weights of the slot's losses: the means' upstream gradients and the losses' own.
  float wk = 0.f, wc = 0.f;
  DistRow st{0.f, 0.f, 0.f, 0.f, 0.f, 1.f, 0, 0};
  int label = -1;
  if (k >= 1) {
    const int64_t q = s * (a.B - 1) + k - 1;
    const float g0 = g.loss != nullptr ? g.loss[0] + a.alpha * g.loss[2] : 0.f;
    const float g1 = g.loss != nullptr ? g.loss[1] + g.loss[2] : 0.f;
    const bool labels = a.labels != nullptr && *sv.labelled > 0;
    if (k <= a.P || labels) st = sv.rows[q];
    if (k <= a.P && st.kl) {
      wk = g0 * a.t / (float(a.P) * float(a.n_seq));
      if (g.kl != nullptr) wk += g.kl[s * a.P + k - 1] / a.t;
    }
    if (labels && st.ce) {
      wc = g1 / float(*sv.labelled);
      if (g.ce != nullptr) wc += g.ce[q];
      label = a.labels[q];
    }
  }
  const bool soft = wk != 0.f, hard = wc != 0.f, one = a.t == 1.f;
  const float log2e = 1.44269504f;
  const float ct = wk * st.inv_t, cu = wk * st.unlisted, c1 = wc * st.inv_1;
  // What the columns' exponentials are relative to: with a bucket the greatest unlisted one (the
  // listed ones are written after).
  const float mu = soft ? st.mu : st.m, shift = soft ? st.shift : 1.f;
  auto at_t = [&](float x) { return soft ? __builtin_amdgcn_exp2f((x - st.m) * a.c2) : 0.f; };
  auto at_1 = [&](float x) { return hard ? __builtin_amdgcn_exp2f((x - st.m) * log2e) : 0.f; };
  float x[G][N];
  const bool inside = r.inside(j0, G * kDistThreads);   // all but a row's first and last part
  if (inside && (soft || hard)) {
#pragma unroll
    for (int h = 0; h < G; ++h) r.load_inside(j0 + h * kDistThreads + tid, x[h]);
  } else {
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const int j = j0 + h * kDistThreads + tid;
#pragma unroll
      for (int e = 0; e < N; ++e) x[h][e] = -INFINITY;
      if ((soft || hard) && j < nv) r.load_raw(j, x[h]);
    }
  }
  // As in the forward pass, an exponential costs one product where z c is not too far out; what
  // rounding adds to the product of m and c goes into the factor.
  const bool far = !(fmaxf(fabsf(mu), fabsf(st.m)) * fmaxf(soft ? a.c2 : 0.f, log2e) < 1e6f);
  auto sums = [&](auto is_far, auto two, float c, float k, float k1) __attribute__((always_inline)) {
    constexpr bool FAR = decltype(is_far)::value;
    const float b = mu * c, b1 = st.m * log2e;
    if (!FAR) {
      k *= __builtin_amdgcn_exp2f(-fmaf(mu, c, -b));
      k1 *= __builtin_amdgcn_exp2f(-fmaf(st.m, log2e, -b1));
    }
#pragma unroll
    for (int h = 0; h < G; ++h)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float z = x[h][e];
        float v = __builtin_amdgcn_exp2f(FAR ? (z - mu) * c : fmaf(z, c, -b)) * k;
        if (decltype(two)::value)
          v = fmaf(__builtin_amdgcn_exp2f(FAR ? (z - st.m) * log2e : fmaf(z, log2e, -b1)), k1, v);
        x[h][e] = v;
      }
  };
  const bool two = soft && hard && !one;
  const float c = soft ? a.c2 : log2e, k1 = hard ? c1 : 0.f, kt = (soft ? cu : 0.f) + (two ? 0.f : k1 * shift);
  if (two && far)
    sums(std::true_type(), std::true_type(), c, kt, k1);
  else if (two)
    sums(std::false_type(), std::true_type(), c, kt, k1);
  else if (far)
    sums(std::true_type(), std::false_type(), c, kt, 0.f);
  else
    sums(std::false_type(), std::false_type(), c, kt, 0.f);   // zeros where there is no loss
#pragma unroll
  for (int h = 0; h < G; ++h) {
    const int j = j0 + h * kDistThreads + tid, c = r.column(j);
    if (vec && (inside || (j < nv && c >= 0 && c + N <= a.V))) {
      u32x4 q;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2)
          q[e] = bf16_bits(x[h][2 * e]) | bf16_bits(x[h][2 * e + 1]) << 16;
        else
          q[e] = __float_as_uint(x[h][e]);
      }
      st16(d + c, q);
    } else if (j < nv) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (c + e >= 0 && c + e < a.V) store_grad(d + c + e, x[h][e]);
    }
  }
  if (!soft && !hard) return;
  // The listed tokens and the label of this part, over what was just stored.
  if (tid == 0) label_done = 0;
  __syncthreads();
  const int c0 = max(r.column(j0), 0), c1_ = min(r.column(j0) + kDistPart, a.V);
  if (soft) {
    const int64_t q = s * a.P + k - 1;
    for (int t = tid; t < a.K; t += kDistThreads) {
      const int id = a.ids[q * a.K + t];
      const float p = sv.p[q * a.K + t];
      if (id < c0 || id >= c1_ || p == -1.f) continue;
      const float z = r.raw(id);
      float v = at_t(z) * ct - wk * p;
      if (hard) v += at_1(z) * c1;
      if (id == label) {
        v -= wc;
        label_done = 1;
      }
      store_grad(d + id, v);
    }
  }
  __syncthreads();
  if (tid == 0 && hard && !label_done && label >= c0 && label < c1_) {
    const float z = r.raw(label);
    const float u = soft ? __builtin_amdgcn_exp2f((z - mu) * a.c2) * cu : 0.f;
    store_grad(d + label, u + at_1(z) * c1 - wc);
  }
}

// Up to this many slots the means take no launch of their own (a step of 28 slots 31.4 -> 28.9 us, an
// evaluation of 60 21.1 -> 18.1, of 120 22.7 -> 22.4).  For more, one wave would sum them too slowly.
// (A release fence in place of stores past the caches: 960 slots 10 -> 39 us, it writes back all that
// the launches before left there.)
constexpr unsigned kFewSlots = 256;

template <typename T>
static hipError_t forward(const DistArgs& a, const DistSaved& sv, int n_parts, void* ws, hipStream_t s) {
  uint32_t* done = static_cast<uint32_t*>(ws);
  DistPart* parts = reinterpret_cast<DistPart*>(static_cast<char*>(ws) + 256);
  const int slots = a.labels != nullptr ? a.B - 1 : a.P;
  const unsigned rows = unsigned(a.n_seq) * slots;
  hipLaunchKernelGGL((distill_part_kernel<T>), dim3(n_parts, rows), dim3(kDistThreads), 0, s, a, slots, parts, done);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const bool few = rows <= kFewSlots;
  uint32_t* count = few ? done : nullptr;
  if (a.K <= kMaxTop / 4)   // one wave
    hipLaunchKernelGGL((distill_row_kernel<T, 64>), dim3(rows), dim3(64), 0, s, a, slots, parts, n_parts, sv, count);
  else
    hipLaunchKernelGGL((distill_row_kernel<T, 256>), dim3(rows), dim3(256), 0, s, a, slots, parts, n_parts, sv, count);
  e = hipGetLastError();
  if (e != hipSuccess || few) return e;
  hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(kLossThreads), 0, s, a, sv);
  return hipGetLastError();
}

hipError_t launch_distill_forward(bool bf16, const DistArgs& a, void* saved, void* ws, hipStream_t s) {
  const DistSaved sv = saved_of(saved, a.n_seq, a.B);
  const int n_parts = dist_parts(bf16, a.V);
  return bf16 ? forward<bf16_t>(a, sv, n_parts, ws, s) : forward<float>(a, sv, n_parts, ws, s);
}

hipError_t launch_distill_backward(bool bf16, const DistArgs& a, const DistGrad& g, const void* saved,
                                   hipStream_t s) {
  const DistSaved sv = saved_of(const_cast<void*>(saved), a.n_seq, a.B);
  const dim3 grid(dist_parts(bf16, a.V), unsigned(a.n_seq) * a.B);
  if (bf16)
    hipLaunchKernelGGL((distill_grad_kernel<bf16_t>), grid, dim3(kDistThreads), 0, s, a, g, sv);
  else
    hipLaunchKernelGGL((distill_grad_kernel<float>), grid, dim3(kDistThreads), 0, s, a, g, sv);
  return hipGetLastError();
}

}  // namespace hdf
