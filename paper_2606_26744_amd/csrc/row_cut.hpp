// Rows of logits cut to the head of their distribution: truncated draws (temperature, top-k,
// top-p, min-p) and a row's top logits.
//
// The entries of a row are ordered by value, ties to the lowest column; masked ones (-inf) have
// no place.  With m the greatest and w_v = e^((z_v - m) / T), the kept entries are the first
//     n = min(n_k, n_p, n_m):  n_k = top_k;  n_p = the fewest of those whose weights sum to top_p
//     of the first n_k entries' sum;  n_m = those with w_v >= min_p.
// The draw is the lowest column whose running sum of kept weights, in column order, passes
// u times their whole.  Sums are 64-bit throughout: a cut or a draw falls between neighbours that
// may be 1e-6 of the whole apart.
//
// First launch (row_head.hip): workgroup (row, chunk) keeps a chunk of a row in registers, lists
// its greatest entries and, where the cut is not a count of entries, sums the weights up in a
// histogram.  Second launch (row_cut.hip): a workgroup a row finds how far down the order the cut
// lies; a cut below the lists takes one more pass over the row.  (One workgroup a row for all of it,
// going over the row again and again: 128 rows of 129280 228 us where the two take 49.)
#pragma once

#include "kernels.hpp"
#include "rows.hpp"

namespace hdf {

constexpr int kHeadThreads = 512;
constexpr int kListMax = 2048;               // listed entries of a row; entries sorted at once
constexpr int kMaxChunks = 66;
constexpr float kLeast = -3.402823466e38f;   // the least finite value

// The histogram: bins of 1/16 octave of weight.  Entry z has t = 16 z log2(e) / T, bin n = rint(t)
// and within it the weight 2^((t - n) / 16), 0.978 .. 1.022, as a multiple of 2^-48; integers, so
// that the sums do not depend on their order.  Bins from the chunk's greatest entry down; entries
// of the last 40, more than 61 octaves below it, weigh nothing (all 2^20 of a row 2^-41 of the whole).
constexpr int kMassBins = 1024, kKeptBins = 984;
constexpr double kMassUnit = 1.0 / 281474976710656.0;   // 2^-48

struct HeadStat {
  float best;        // greatest value, its lowest column (of greedy rows)
  int32_t best_col;
  float floor;       // every entry >= floor is listed (-inf: all are)
  float near;        // a value that the chunk's share of the top_k entries reaches
  uint32_t valid;    // unmasked entries, listed ones
  uint32_t listed;
  int32_t top_bin;   // bin of the greatest value, and how many bins from it down are stored
  int32_t bins;      // (-1: values beyond the bins' range)
  double rest_ref;   // of top logits: rest = the sum of e^((z - rest_ref) / T) over the unlisted
  double rest;
};

// Between the phases of a row's cut: a nucleus' border bin, the weights above it and in the whole,
// the bin's values end <= z < over; the last key that min_p keeps.
struct CutNote {
  double whole, above;
  uint64_t cut_m;
  float end, over;
  int32_t border, by_p, left;
};

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
  bool greedy, binned;   // binned: the cut, or the draw, goes by weight and not by count
  bool open;             // nothing is cut
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
  // (A min_p below the bins' 61 octaves goes by the search.)
  s.binned = !s.greedy && s.top_k <= 0 && !(s.min_p > 0.f && s.min_p < 1e-18f);
  s.open = s.binned && !(s.top_p < 1.f) && !(s.min_p > 0.f);
  s.inv_t = s.greedy ? 1. : 1. / double(s.t);
  s.c2 = 1.4426950408889634074 * s.inv_t;
  return s;
}

// Bin of a value: the magic constant, 1.5 * 2^52, rounds to an integer in the low bits of the sum.
constexpr double kRound = 6755399441055744.;
__device__ __forceinline__ int weight_bin(float z, double k16) {
  return int(uint32_t(__builtin_bit_cast(uint64_t, fma_k(double(z), k16, kRound))));
}
// Bin and the weight within it: the series of 2^(g / 16), |g| <= 1/2, to the sixth power, with g^6
// replaced by 3/8 g^4 - 9/256 g^2 + 1/2048, from which it differs by T_6(2g) / 2048: 5e-15 of the
// weight at the most, and of alternating sign.  SCALE 2^(48 - 1074) makes the result subnormal and
// its bits the weight as a multiple of 2^-48.  c5: mass_coefficient(), kept in registers by the
// caller.
constexpr double kBits = 0x1p-1026;
constexpr double kLog16 = 0.69314718055994530942 / 16., kLog16_2 = kLog16 * kLog16;
constexpr double kMass6 = kLog16_2 * kLog16_2 * kLog16_2 / 720.;
__device__ __forceinline__ double mass_coefficient(double scale) {
  double c = kLog16_2 * kLog16_2 * kLog16 / 120. * scale;
  asm volatile("" : "+v"(c));   // not copied anew for every entry
  return c;
}
template <bool BITS>
__device__ __forceinline__ double bin_series(float z, double k16, double c5, int& n) {
  constexpr double S = BITS ? kBits : 1.;
  const double t = fma_k(double(z), k16, kRound);
  n = int(uint32_t(__builtin_bit_cast(uint64_t, t)));
  const double g = fma(double(z), k16, kRound - t);
  double p = fma_k(c5, g, (kLog16_2 * kLog16_2 / 24. + kMass6 * 0.375) * S);
  p = fma_k(p, g, kLog16_2 * kLog16 / 6. * S);
  p = fma_k(p, g, (kLog16_2 / 2. - kMass6 * 0.03515625) * S);
  p = fma_k(p, g, kLog16 * S);
  return fma_k(p, g, (1. + kMass6 / 2048.) * S);
}
__device__ __forceinline__ uint64_t weight_in_bin(float z, double k16, double c5, int& n) {
  return __builtin_bit_cast(uint64_t, bin_series<true>(z, k16, c5, n));
}

hipError_t launch_row_head(bool bf16, bool top, bool small, const CutArgs& a, const HeadArgs& h, hipStream_t s);

}  // namespace hdf
