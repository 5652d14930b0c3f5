// The statistics of a row of logits that one pass gives.
#pragma once

#include "tokens.h"

namespace gnnshap {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// m the largest of the logits x seen, s = sum e_j of e_j = exp(x_j - m).
struct Stats {
  float m, s, w;  // w = sum e_j log2(e_j)
};
__device__ __forceinline__ Stats no_stats() { return Stats{-INFINITY, 0.f, 0.f}; }

__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

// Moves a to the maximum m >= a.m.  Far below it f is 0, and what it multiplies
// has to stay finite: up to 2^30 logits times 1e4.
__device__ __forceinline__ void move_to(Stats& a, float m) {
  if (a.s != 0.f) {  // NaN too
    const float d = (a.m - finite_max(m)) * kLog2e, f = __builtin_amdgcn_exp2f(d);
    a.w = f * (a.w + a.s * fmaxf(d, -1e4f));
    a.s *= f;
  }
  a.m = m;
}

__device__ __forceinline__ void add(Stats& a, Stats b) {
  const float m = fmaxf(a.m, b.m);
  move_to(a, m);
  move_to(b, m);
  a.s += b.s;
  a.w += b.w;
}

__device__ __forceinline__ void wave_sum(Stats& a) {
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    Stats b;
    b.m = __shfl_xor(a.m, off);
    b.s = __shfl_xor(a.s, off);
    b.w = __shfl_xor(a.w, off);
    add(a, b);
  }
}

// Whole numbers in the order of the floats (-0 and 0 alike, NaN above all; none
// is all ones, so that every key is below the one that a search starts from).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  if (x != x) return 0xFFFFFFFEu;
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}

}  // namespace gnnshap
