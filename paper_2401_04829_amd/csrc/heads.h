// A head's elements spread over neighbouring lanes, as the operators that norm
// and rotate them hold them.
#pragma once

#include "tokens.h"

namespace gnnshap {

// Lanes that a head of `units` times 2 N elements is spread over.
inline int head_lanes(int units) {
  int x = 1;
  while (x < units && x < 64) x *= 2;
  return x;
}

// Calls f with the elements N of a pack, as a type: 16 bytes where the rotated
// half is whole packs, else the widest that fit.
template <class T, class F>
inline int with_pack(int head_dim, int rot, F f) {
  constexpr int kWide = 16 / sizeof(T);
  const auto fits = [&](int n) { return head_dim % (2 * n) == 0 && (rot / 2) % n == 0; };
  if (fits(kWide)) return f(std::integral_constant<int, kWide>());
  if (fits(4)) return f(std::integral_constant<int, 4>());
  if (fits(2)) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1>());
}

// The sum of x over the blockDim.x (a power of two) lanes of a head.
__device__ __forceinline__ float head_sum(float x) {
  for (unsigned off = 1; off < blockDim.x; off *= 2) x += __shfl_xor(x, static_cast<int>(off));
  return x;
}

// Two packs of N elements per unit, in fp32: the packs i and half + i on where
// pairs are of the rotated halves, else 2 N elements side by side.  The lane
// threadIdx.x has unit threadIdx.x (and, of packs of one element, that 64 on).
template <class T, int N>
struct HeadUnits {
  static constexpr int kUnits = N == 1 ? 2 : 1;
  float v[kUnits][2 * N];
  int at[kUnits][2];  // first elements of the packs; -1: the lane has no such unit
  int dim;
  __device__ __forceinline__ HeadUnits(int D, int rot, int interleaved) : dim(D) {
    const int half = rot / 2;
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      const int u = threadIdx.x + 64 * j;
      if (!interleaved && u < half / N) {
        at[j][0] = u * N;
        at[j][1] = half + u * N;
      } else {
        at[j][0] = interleaved ? 2 * N * u : rot + 2 * N * (u - half / N);
        at[j][1] = at[j][0] + N;
      }
      if (u >= D / (2 * N)) at[j][0] = at[j][1] = -1;
    }
  }
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int j = 0; j < kUnits; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Pack<T, N> x{};
        if (at[j][h] >= 0) x = load_pack<T, N>(p + at[j][h]);
#pragma unroll
        for (int e = 0; e < N; ++e) v[j][h * N + e] = static_cast<float>(x.v[e]);
      }
  }
  // (past the caches, few heads or many: 20,000 tokens into a cache 106 us by way of
  // them, 98 past them; 16,384 tokens forward and backward 198 and 186; without
  // what reads them next)
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int j = 0; j < kUnits; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (at[j][h] < 0) continue;
        Pack<T, N> x;
#pragma unroll
        for (int e = 0; e < N; ++e) x.v[e] = static_cast<T>(v[j][h * N + e]);
        stream_pack(p + at[j][h], x);
      }
  }
  // 1 / sqrt(mean square + eps) of the head, in all of its lanes.
  __device__ __forceinline__ float over_root(float eps) const {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < kUnits; ++j)
#pragma unroll
      for (int e = 0; e < 2 * N; ++e) s = fmaf(v[j][e], v[j][e], s);
    return 1.f / sqrtf(head_sum(s) / dim + eps);
  }
  __device__ __forceinline__ void times(float r) {
#pragma unroll
    for (int j = 0; j < kUnits; ++j)
#pragma unroll
      for (int e = 0; e < 2 * N; ++e) v[j][e] *= r;
  }
  // x r w; w NULL: all 1
  __device__ __forceinline__ void norm(const T* w, float eps) {
    times(over_root(eps));
    if (!w) return;
    HeadUnits u = *this;
    u.load(w);
#pragma unroll
    for (int j = 0; j < kUnits; ++j)
#pragma unroll
      for (int e = 0; e < 2 * N; ++e) v[j][e] *= u.v[j][e];
  }
  // The pairs of the first `rot` elements turned by cos and sin from these on; dir -1: back.
  __device__ __forceinline__ void turn(const float* cs, const float* sn, int rot, int interleaved, float dir) {
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      if (at[j][0] < 0) continue;
      if (!interleaved) {
        if (at[j][0] >= rot / 2) continue;
        const Pack<float, N> c = load_pack<float, N>(cs + at[j][0]), s = load_pack<float, N>(sn + at[j][0]);
#pragma unroll
        for (int e = 0; e < N; ++e) pair(v[j][e], v[j][N + e], c.v[e], dir * s.v[e]);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (at[j][0] + 2 * e < rot)
            pair(v[j][2 * e], v[j][2 * e + 1], cs[at[j][0] / 2 + e], dir * sn[at[j][0] / 2 + e]);
      }
    }
  }
  // (fused where it says so, so that all kernels round alike)
  static __device__ __forceinline__ void pair(float& x, float& y, float c, float s) {
    const float a = fmaf(x, c, -(y * s));
    y = fmaf(y, c, x * s);
    x = a;
  }
};

}  // namespace gnnshap
