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

// rows of a piece that count
__device__ __forceinline__ int piece_rows(const VocabArgs& a) {
  return a.count ? max(0, min(*a.count - a.row0, a.R)) : a.rows;
}

// the logits' statistics alone, with the logits, dh = P w, dw = P^T h
enum class Prod { Stats, Logits, Dh, Dw };

}  // namespace rg
