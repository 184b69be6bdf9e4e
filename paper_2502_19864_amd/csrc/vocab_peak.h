// What the vocabulary head's kernels share: running maxima and sums, and which product a kernel makes.
#pragma once
#include "common.h"
#include "kernels.h"

namespace rg {

constexpr float LOG2E = 1.4426950408889634f;

// exp(x) of a difference to a maximum, x <= 0
__device__ __forceinline__ float exp_below(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

// (maximum, sum of exp(s - maximum)) of a run of columns, and the lowest column that has the maximum
struct Peak {
  float m, l;
  int at;
};
__device__ __forceinline__ Peak join(Peak a, Peak b) {
  const float m = fmaxf(a.m, b.m), z = m == -INFINITY ? 0.f : m;
  Peak r;
  r.m = m;
  r.l = a.l * exp_below(a.m - z) + b.l * exp_below(b.m - z);
  r.at = a.m > b.m ? a.at : b.m > a.m ? b.at : min(a.at, b.at);
  return r;
}

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

// rows of a piece that count
__device__ __forceinline__ int piece_rows(const VocabArgs& a) {
  return a.count ? max(0, min(*a.count - a.row0, a.R)) : a.rows;
}

// The unit of dloss: with bf16 tensors P holds dloss / unit, and dh and dw are multiplied by the unit in fp32.  Most
// often dloss is one number for all rows, so P's largest entries, -1 + p at the labels of unsure rows, are
// rounded as such: with the number in them they are all off by its rounding, up to 2^-9 of dw to the same side (900 x 4000, d 512: dw
// 0.0028 off float64, in units 0.0020, of which its own rounding is 0.0017).  A unit out of range is left out.
__device__ __forceinline__ float dloss_unit(const VocabArgs& a) {
  if (*a.n_counted == 0) return 1.f;
  const float g = fabsf(a.g_c[0]);
  return g >= 0x1p-40f && g <= 0x1p40f ? g : 1.f;
}

// A row of P sums to zero, so what all rows of w have in common reaches no dh.  With bf16 tensors P is rounded to bf16, after logits in fp16, and
// then it does: the largest rounding, the label's, stands alone, and of w = a common row + 0.1 of random ones (40 classes, d 64) it leaves a
// row of dh up to 0.05 off float64 (0.17 where 0.03 is random).  So what the stored P of a row falls short of zero, summed in fp32, goes
// to its label's row of w, in fp32 as well: dh = P w + left w[label], and an entry's error e meets w - w[label] alone.  The
// same rows are then 0.0027 off, dh's own rounding 0.0022.  Rows as sure of their label as 1 - 2^-24, whose own
// entry, from the loss, is zero where the others' are not, keep their dh too: 0.006 off at most, by the logits in fp16.
__device__ __forceinline__ float row_left(const VocabArgs& a, int m) {
  float v = 0.f;
#pragma unroll 8
  for (int i = 0; i < a.left_n; ++i) v += a.left[(long)m * a.left_n + i];
  return v;
}

// A row of dw takes the rounding of its label's entries as it is: 0.0020 off float64 in all, 0.0017 its own.  Of few rows one entry may
// be most of a class' sum, and of dh a row whose competitors lie around its label's w leaves little but P's roundings (4 rows, of which few
// count, 196 classes, d 8: the worst of 60 batches is 0.0038 off in dh and 0.0033 in dw, both 0.0028 in two parts).  So where at most 64 rows of a
// piece count, P is kept in two parts, the second in the 64 rows below, which the products' tiles have empty then: rows of A in dh, k in dw.
constexpr int TWO_PARTS = 64;
__device__ __forceinline__ bool two_parts(int cnt) { return cnt > 0 && cnt <= TWO_PARTS; }

// Workgroups that share the k of a tile: where the tiles of the rows that count leave CUs idle, at least `least` of k to each, and
// never more than `longest`, the chain of additions in the matrix unit that a sum's precision allows
__host__ __device__ inline int k_shares(int slots, int tiles, int K, int least, int longest) {
  const int by_slots = slots / tiles, by_k = K / least, s = by_slots < by_k ? by_slots : by_k, chains = (int)(((long)K + longest - 1) / longest);
  return s > chains ? s : chains > 1 ? chains : 1;
}

// The tile of C[m][n] = sum_k A(m, k) B(n, k) that a workgroup makes, by XCD: workgroups are dealt round-robin to the eight
// XCDs; each takes a contiguous run of a raster in bands of GROUP tile rows, so what its L2 holds is shared.
template <int GROUP>
__device__ __forceinline__ bool vocab_tile(int g, int ntm, int ntn, int& tm, int& tn) {
  const int n = ntm * ntn;
  if (g >= n) return false;
  const int x = g & 7, q = n >> 3, r = n & 7;
  g = x * q + min(x, r) + (g >> 3);
  const int band = g / (GROUP * ntn), first = band * GROUP, size = min(ntm - first, GROUP), in = g - band * GROUP * ntn;
  tm = first + in % size;
  tn = in / size;
  return true;
}

// the logits' statistics alone, with the logits, dh = P w, dw = P^T h
enum class Prod { Stats, Logits, Dh, Dw };

}  // namespace rg
