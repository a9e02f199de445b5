// Speculative verification between truncated distributions: draft x_i of a sequence is accepted if
// u_i q_i(x_i) < p_i(x_i), p and q the truncated distributions of the target's and the drafter's
// row; after n acceptances the next token is drawn from max(0, p_n - q_n) by its running sum in
// column order (from p_n where that is zero throughout, or after K acceptances).  The target rows
// are truncated first (row_cut.hip); the draw reads one row, or two, a sequence.  Latency bounds the
// two launches, 7 to 8 us each for 8 sequences of 129280 logits, 6 for one of 32000: chains of dependent
// loads (draft, cut, logits; sums, part, entries) between barriers.
#include "kernels.hpp"
#include "rows.hpp"

namespace hdf {

constexpr int kVerifyThreads = 256;    // one vector of a part each
constexpr int kVerifyWaves = kVerifyThreads / kWave;

// A row's truncation: the probability of a kept entry is e^((z - ref) / T - lse).  ref = 0 and lse the
// stored log-sum-exp, or, where that is far from 0 (far_lse), the row's greatest logit and the
// log-sum-exp relative to it.
struct RowCut {
  float logit;
  int index;
  double ref, lse;
};
__device__ __forceinline__ double cut_prob(const RowCut& k, float z, int c, bool greedy, double inv_t) {
  if (!(z > k.logit || (z == k.logit && c <= k.index)) || z == -INFINITY) return 0.;
  return greedy ? 1. : exp2_64(fma(double(z) - k.ref, inv_t, -k.lse) * 1.4426950408889634074);
}

template <typename TD, typename TT>
struct VerifyRows {
  const VerifyArgs& a;
  int s;
  bool greedy;
  double inv_t;
  __device__ VerifyRows(const VerifyArgs& a_, int s_) : a(a_), s(s_) {
    const float t = a.ts != nullptr ? a.ts[s] : a.t;
    greedy = !(t > 0.f);
    inv_t = greedy ? 0. : 1. / double(t);   // as the truncation took it: its rounding cancels
  }
  __device__ LogitRow<TT> target(int i) const {
    return {static_cast<const TT*>(a.tz) + (int64_t(s) * (a.K + 1) + i) * a.V, a.V};
  }
  __device__ LogitRow<TD> draft(int i) const {
    return {static_cast<const TD*>(a.dz) + (int64_t(s) * a.stride + i) * a.ld, a.V};
  }
  __device__ RowCut target_cut(int i) const {
    const int64_t r = int64_t(s) * (a.K + 1) + i;
    const double lse = a.t_lse[r];
    const bool far = !greedy && far_lse(lse);
    return {a.t_logit[r], a.t_index[r], far ? double(a.t_top[r]) : 0., far ? a.t_log[r] : lse};
  }
  __device__ RowCut draft_cut(int i) const {
    const int64_t r = int64_t(s) * a.stride + i, e = int64_t(s) * a.K + i;
    const double lse = a.d_lse[r];
    const bool far = !greedy && far_lse(lse);
    return {a.d_logit[r], a.d_index[r], far ? double(a.d_top[e]) : 0., far ? a.d_log[e] : lse};
  }
  // Weights of the next token's draw in vector j of target row n: the residual w and the target's
  // own p.
  __device__ void weights(int n, int j, const RowCut& tc, const RowCut& dc, double w[LogitRow<TT>::N],
                          double p[LogitRow<TT>::N]) const {
    constexpr int N = LogitRow<TT>::N;
    const LogitRow<TT> t = target(n);
    const LogitRow<TD> d = draft(n < a.K ? n : 0);
    // Sums of equal rows that were taken in different orders differ by less than this, of the
    // probabilities; stored ones do not differ.
    const double least = tc.ref != 0. && dc.ref != 0. ? 0x1p-40 : 0.;
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = p[e] = 0.;
    if (j >= t.vectors()) return;
    t.load(j, x);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int c = t.column(j) + e;
      p[e] = cut_prob(tc, x[e], c, greedy, inv_t);
      w[e] = p[e];
      if (n < a.K && p[e] > 0.) {
        w[e] = p[e] - cut_prob(dc, d.at(c), c, greedy, inv_t);
        w[e] = w[e] > least * p[e] ? w[e] : 0.;
      }
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
          p = cut_prob(v.target_cut(i), v.target(i).at(x), x, v.greedy, v.inv_t);
          q = cut_prob(v.draft_cut(i), v.draft(i).at(x), x, v.greedy, v.inv_t);
        }
        reject = !(double(a.u[int64_t(s) * (a.K + 1) + i]) * q < p);
      }
      const unsigned long long miss = __ballot(reject);
      if (miss != 0ull) {
        n = c0 + __ffsll(static_cast<long long>(miss)) - 1;
        break;
      }
    }
    if (threadIdx.x == 0) decided = n;
  }
  __syncthreads();
  const int n = decided;
  const RowCut t = v.target_cut(n), d = n < a.K ? v.draft_cut(n) : t;
  if (part == 0 && threadIdx.x == 0) {
    a.n_buf[s] = n;
    RowCut* cuts = static_cast<RowCut*>(a.cuts) + 2 * s;
    cuts[0] = t;
    cuts[1] = d;
  }
  double w[LogitRow<TT>::N], p[LogitRow<TT>::N], sw = 0., sp = 0.;
  v.weights(n, part * kVerifyThreads + int(threadIdx.x), t, d, w, p);
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
  const RowCut t = static_cast<const RowCut*>(a.cuts)[2 * s], d = static_cast<const RowCut*>(a.cuts)[2 * s + 1];
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
    note_first(mine > 0. && run > target, i, &pick);
    note_last(mine > 0., i, &last);
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
  v.weights(n, j, t, d, w, p);
  const int c = v.target(n).column(j);
  int end = -1;
#pragma unroll
  for (int e = 0; e < LogitRow<TT>::N; ++e) {
    w[e] = which == 0 ? w[e] : p[e];
    mine += w[e];
    end = w[e] > 0. ? c + e : end;
  }
  note_last(end >= 0, end, &last);
  const double upto = base + block_scan<kVerifyWaves>(mine, sh, all);
  note_first(!tail && mine > 0. && upto > target, tid, &pick);
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

// Parts of a target row: 256 vectors each, of its least vectors and one for a row that starts
// inside one.
static int verify_parts(bool bf16, int V) {
  const int N = bf16 ? 8 : 4;
  return ((V + 2 * N - 2) / N + kVerifyThreads - 1) / kVerifyThreads;
}

size_t accept_truncated_ws_bytes(bool bf16, int n_seq, int K, int V) {
  const size_t n = n_seq, rows = n * (K + 1), drafts = n * K;
  return cut_ws_bytes(bf16, int64_t(rows), V, false) + 2 * al256(rows * 8) + 4 * al256(rows * 4) + al256(drafts * 8) +
         al256(drafts * 4) + al256(n * 4) + al256(n * 2 * sizeof(RowCut)) + al256(n * verify_parts(bf16, V) * 16);
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
  const size_t rows = size_t(n_seq) * (a.K + 1), drafts = size_t(n_seq) * a.K;
  char* p = static_cast<char*>(ws);
  auto take = [&](size_t bytes) {
    char* q = p;
    p += al256(bytes);
    return q;
  };
  c.lse = reinterpret_cast<double*>(take(rows * 8));
  c.log_sum = reinterpret_cast<double*>(take(rows * 8));
  c.top = reinterpret_cast<float*>(take(rows * 4));
  c.cut_logit = reinterpret_cast<float*>(take(rows * 4));
  c.cut_index = reinterpret_cast<int32_t*>(take(rows * 4));
  c.kept = reinterpret_cast<int32_t*>(take(rows * 4));
  c.drafts = {a.dz, draft_bf16, a.ld, a.stride, a.K, int64_t(drafts), a.d_logit, a.d_index, a.d_lse,
              reinterpret_cast<float*>(take(drafts * 4)), reinterpret_cast<double*>(take(drafts * 8))};
  a.n_buf = reinterpret_cast<int32_t*>(take(size_t(n_seq) * 4));
  a.cuts = take(size_t(n_seq) * 2 * sizeof(RowCut));
  const int parts = verify_parts(target_bf16, a.V);
  a.sums = reinterpret_cast<double*>(take(size_t(n_seq) * parts * 16));
  a.t_logit = c.cut_logit;
  a.t_index = c.cut_index;
  a.t_lse = c.lse;
  a.t_top = c.top;
  a.t_log = c.log_sum;
  a.d_top = c.drafts.top;
  a.d_log = c.drafts.log_sum;
  const hipError_t e = launch_truncate(target_bf16, c, take(cut_ws_bytes(target_bf16, int64_t(rows), a.V, false)), s);
  if (e != hipSuccess) return e;
  if (draft_bf16)
    return target_bf16 ? launch_verify<bf16_t, bf16_t>(a, n_seq, parts, s)
                       : launch_verify<bf16_t, float>(a, n_seq, parts, s);
  return target_bf16 ? launch_verify<float, bf16_t>(a, n_seq, parts, s)
                     : launch_verify<float, float>(a, n_seq, parts, s);
}

}  // namespace hdf
