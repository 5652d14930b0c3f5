// Log probabilities of given tokens with entropy, rank and the largest
// alternatives, and their gradient by the logits.
//
// With M the row's maximum, e_j = exp(x_j - M), s = sum e_j and
// w = sum e_j (x_j - M):
//     lse = M + log s,  log p_j = (x_j - M) - log s,  H = log s - w / s.
// A lane keeps (M, s, w) of the elements it has seen and moves them to a new
// maximum when a chunk brings one, so that one pass over the row gives them
// all; two such triples add up after both are moved to the larger maximum.
// The rank is a count of x_j > x_target.
//
// Alternatives: a wavefront keeps a falling list of 64 keys, lane i the i-th
// best; a key is (order-preserving image of x, ~token), so keys are unique
// and of equal logits the lowest token wins.  The list starts from a bound
// that the k-th best cannot be below: the k-th largest of the maxima that the
// lanes find in the row's first chunks.  A chunk, and of it what one load
// brought, is looked at again only if its maximum exceeds the bound, which
// rises to the list's k-th key once there is one.
//
// One wavefront reads chunks of 64 lanes x 4 x 16 bytes.  A row is one
// wavefront's, or one workgroup's, or (few rows) several workgroups', whose
// parts a second launch joins.  Bound by memory, and beside it by the vector
// instructions of the alternatives: 10,000 x 32,768 bf16 (656 MB) without them
// 137 us, 4.8 TB/s (from 127 to 160, by the clocks), with the top 5 152 us, 4.3
// TB/s.  One row of 131,072 with the top 20: 8.5 us, and 7.2 us to join its 16
// parts.
#include "stats.h"

namespace {

using gnnshap::bf16_t;
using gnnshap::f16_t;
using gnnshap::load_pack;
using gnnshap::Pack;
using gnnshap::store_pack;

using gnnshap::add;
using gnnshap::finite_max;
using gnnshap::kLn2;
using gnnshap::kLog2e;
using gnnshap::move_to;
using gnnshap::no_stats;
using gnnshap::ordered;
using gnnshap::Stats;
using gnnshap::wave_sum;

constexpr int kWaves = 4;      // wavefronts of a workgroup
constexpr int kMaxParts = 64;        // workgroups of a row
constexpr int kMaxPartKeys = 1024;  // of their alternatives

// The value of a lane of the same 16, `Turn` lanes on, moved within the vector unit.
template <int Turn>
__device__ __forceinline__ uint32_t turned(uint32_t x) {
  constexpr int kRowRor = 0x120;
  return __builtin_amdgcn_update_dpp(0, static_cast<int>(x), kRowRor + Turn, 0xF, 0xF, false);
}
template <int Turn>
__device__ __forceinline__ float turned(float x) {
  return __uint_as_float(turned<Turn>(__float_as_uint(x)));
}
template <int Turn>
__device__ __forceinline__ uint64_t turned(uint64_t x) {
  return static_cast<uint64_t>(turned<Turn>(static_cast<uint32_t>(x >> 32))) << 32 | turned<Turn>(static_cast<uint32_t>(x));
}
// x of LANES lanes (16 or 64) put together by `f`, in all of them.
template <int LANES, class X, class F>
__device__ __forceinline__ X together(X x, F f) {
  x = f(x, turned<8>(x));
  x = f(x, turned<4>(x));
  x = f(x, turned<2>(x));
  x = f(x, turned<1>(x));
  if constexpr (LANES == 64) {
    x = f(x, static_cast<X>(__shfl_xor(x, 16)));
    x = f(x, static_cast<X>(__shfl_xor(x, 32)));
  }
  return x;
}

// The float whose image is o.
__device__ __forceinline__ float unordered(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

// (image of the logit, ~token); 0 is below every logit's key.
typedef uint64_t Key;
__device__ __forceinline__ Key key_of(float x, int64_t token) {
  return static_cast<uint64_t>(ordered(x)) << 32 | static_cast<uint32_t>(~token);
}
__device__ __forceinline__ float logit_of(Key k) { return unordered(static_cast<uint32_t>(k >> 32)); }
__device__ __forceinline__ int32_t token_of(Key k) { return static_cast<int32_t>(~static_cast<uint32_t>(k)); }
__device__ __forceinline__ Key of_lane(Key k, int lane) {
  return static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(k >> 32), lane))) << 32 |
         static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(k), lane));
}
// The key of the lane below, moved within the vector unit.
__device__ __forceinline__ Key from_below(Key k) {
  constexpr int kWaveShr1 = 0x138;
  const int hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(k >> 32), kWaveShr1, 0xF, 0xF, false);
  const int lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(k), kWaveShr1, 0xF, 0xF, false);
  return static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo);
}

// The 64 best keys of a wavefront, lane i the i-th, of which the first k are wanted.
struct TopList {
  Key mine = 0, kth = 0;
  int k;
  __device__ __forceinline__ explicit TopList(int top) : k(top) {}
  // The keys of the lanes in `is`, the lowest lane first.
  __device__ __forceinline__ void offer(Key c, uint64_t is) {
    const int lane = threadIdx.x & 63;
    while (is) {
      const int src = __builtin_ctzll(is);
      is &= is - 1;
      const Key in = of_lane(c, src);
      if (in <= kth) continue;
      const int pos = __popcll(__ballot(mine > in));
      const Key up = from_below(mine);
      mine = lane > pos ? up : lane == pos ? in : mine;
      kth = of_lane(mine, k - 1);
    }
  }
};

// A lower bound of the k-th largest of the lanes' values (the upper half of its bits).
__device__ __forceinline__ uint32_t kth_of_lanes(uint32_t v, int k) {
  uint32_t t = 0;
#pragma unroll
  for (int b = 31; b >= 16; --b) {
    const uint32_t u = t | (1u << b);
    if (__popcll(__ballot(v >= u)) >= k) t = u;
  }
  return t;
}

// The largest float below those whose image is `from` or more; NaN if -inf is among them.
__device__ __forceinline__ float below(uint32_t from) {
  constexpr uint32_t kLowest = 0x007FFFFFu, kZero = 0x80000000u;  // of -inf, of 0 (whose image below is -0)
  return from <= kLowest ? NAN : unordered(from - (from == kZero ? 2u : 1u));
}

template <class T>
struct Chunk {
  static constexpr int kVec = 16 / sizeof(T);
  static constexpr int kLoads = 4;
  static constexpr int kElems = kVec * kLoads;  // per lane
  static constexpr int kSize = 64 * kElems;     // per wavefront
  typedef float Floats __attribute__((ext_vector_type(kElems)));
  Pack<T, kVec> p[kLoads];
  // Elements `base` on of a row of n; behind the row -inf.
  __device__ __forceinline__ void load(const T* row, int64_t base, int64_t n) {
    const int lane = threadIdx.x & 63;
    if (base + kSize <= n) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) p[u] = load_pack<T, kVec>(row + base + (u * 64 + lane) * kVec);
      return;
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int64_t i = base + (u * 64 + lane) * kVec;
      if (i + kVec <= n) {
        p[u] = load_pack<T, kVec>(row + i);
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) p[u].v[j] = i + j < n ? row[i + j] : static_cast<T>(-INFINITY);
      }
    }
  }
};

struct LogprobArgs {
  gnnshap_logits l;
  int32_t* info;
  int parts;         // workgroups of a row
  Stats* part_stats; // [rows][parts], with the rank's count beside them
  int32_t* part_rank;
  Key* part_keys;    // [rows][parts][top]
};

// What a row's statistics give the caller; logs = log st.s.
__device__ __forceinline__ void write_stats(const LogprobArgs& a, int64_t row, const Stats& st, float logs, int rank,
                                            bool has, float xt) {
  const bool none = st.s == 0.f;  // every logit is -inf
  if (a.l.lse) a.l.lse[row] = none ? -INFINITY : st.m + logs;
  if (a.l.maximum) a.l.maximum[row] = st.m;
  if (a.l.log_sum) a.l.log_sum[row] = none ? 0.f : logs;
  if (a.l.entropy) a.l.entropy[row] = none ? 0.f : logs - kLn2 * (st.w / st.s);
  if (a.l.logprob) a.l.logprob[row] = !has ? 0.f : none ? -INFINITY : (xt - st.m) - logs;
  if (a.l.rank) a.l.rank[row] = has ? rank : -1;
}

// The same and the alternatives, of which lane i holds the i-th; the whole wavefront calls it.
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t row, const Stats& st, int rank, Key mine,
                                          bool has, float xt) {
  const int lane = threadIdx.x & 63;
  const float logs = logf(st.s);
  if (lane == 0) write_stats(a, row, st, logs, rank, has, xt);
  if (lane < a.l.top) {
    const int64_t at = row * a.l.top + lane;
    if (a.l.top_logprob) a.l.top_logprob[at] = st.s == 0.f ? -INFINITY : (logit_of(mine) - st.m) - logs;
    if (a.l.top_id) a.l.top_id[at] = token_of(mine);
  }
}

// The k best of `lists` falling lists of k keys, into `best` (all in LDS;
// threads tid = 0 .. n - 1 call it, behind a barrier, and all threads of the
// workgroup together; it ends with one).  Keys below any list's last one are
// not among them; the place of one of the others (which go to `left`) is the
// number of those above it.  Keys are unique but for 0; where there are fewer
// than k others, `best` ends with 0.
__device__ __forceinline__ void join_lists(const Key* keys, int lists, int k, Key* left, int* n_left, Key* best, int tid,
                                           int n) {
  if (tid == 0) *n_left = 0;
  if (tid < k) best[tid] = 0;
  Key from = 1;
  for (int j = 0; j < lists; ++j) from = max(from, keys[j * k + k - 1]);
  __syncthreads();
  for (int i = tid; i < lists * k; i += n)
    if (keys[i] >= from) left[atomicAdd(n_left, 1)] = keys[i];
  __syncthreads();
  const int m = *n_left;
  for (int i = tid; i < m; i += n) {
    const Key mine = left[i];
    int place = 0;
#pragma unroll 8
    for (int j = 0; j < m; ++j) place += left[j] > mine;
    if (place < k) best[place] = mine;
  }
  __syncthreads();
}

// The row's given token and its logit; `has` false if there is none.
template <class T>
__device__ __forceinline__ float given(const LogprobArgs& a, const T* x, int64_t row, bool& has) {
  const int64_t t = a.l.targets ? a.l.targets[row] : -1;
  has = t >= 0 && t < a.l.vocab;
  if (t >= a.l.vocab && a.info) *a.info = 1;
  return has ? static_cast<float>(x[t]) : INFINITY;
}

// PER_ROW wavefronts of a workgroup read a row's chunks in turn (of one part
// of it, where a row has several workgroups).
template <class T, int PER_ROW>
__global__ __launch_bounds__(64 * kWaves) void k_token_logprobs(LogprobArgs a) {
  constexpr int kRows = kWaves / PER_ROW;
  using C = Chunk<T>;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t block = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts, way = wave % PER_ROW;
  const int64_t row = block * kRows + wave / PER_ROW;
  const bool in = row < a.l.num_rows;
  const int64_t V = a.l.vocab;
  const T* x = static_cast<const T*>(a.l.logits) + (in ? row : 0) * a.l.row_stride;

  Stats st = no_stats();
  TopList list(a.l.top);
  int rank = 0;
  bool has = false;
  float xt = 0.f;
  int64_t base = in ? (static_cast<int64_t>(part) * PER_ROW + way) * C::kSize : V;
  const int64_t step = static_cast<int64_t>(a.parts) * PER_ROW * C::kSize;
  C next;
  if (base < V) next.load(x, base, V);
  float bound = NAN;  // no logit up to it is wanted
  if (a.l.top > 0) {
    // at least top logits are no smaller than the top-th largest of the
    // maxima of as many sets of logits: a lane's, in all of the row's wavefronts
    uint32_t most = 0u;
    if (base < V) {
      float f = -INFINITY;
#pragma unroll
      for (int i = 0; i < C::kElems; ++i) f = fmaxf(f, static_cast<float>(next.p[i / C::kVec].v[i % C::kVec]));
      most = ordered(f);
    }
    if constexpr (PER_ROW > 1) {
      __shared__ uint32_t all[kWaves][64];
      all[wave][lane] = most;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PER_ROW; ++i) most = max(most, all[wave - way + i][lane]);
    }
    bound = below(kth_of_lanes(most, a.l.top));
  }
  if (in) {
    xt = given(a, x, row, has);
    for (; base < V; base += step) {
      const C c = next;
      if (base + step < V) next.load(x, base + step, V);
      typename C::Floats f;
      float of_load[C::kLoads], most = -INFINITY;
#pragma unroll
      for (int u = 0; u < C::kLoads; ++u) {
        of_load[u] = -INFINITY;
#pragma unroll
        for (int j = 0; j < C::kVec; ++j) {
          f[u * C::kVec + j] = static_cast<float>(c.p[u].v[j]);
          of_load[u] = fmaxf(of_load[u], f[u * C::kVec + j]);
        }
        most = fmaxf(most, of_load[u]);
      }
      if (most > st.m) move_to(st, most);
      const float m = finite_max(st.m);
      float s = 0.f, w = 0.f;
#pragma unroll
      for (int i = 0; i < C::kElems; ++i) {
        const float d = (f[i] - m) * kLog2e, e = __builtin_amdgcn_exp2f(d);
        s += e;
        w += e * fmaxf(d, -200.f);
        rank += __popcll(__ballot(f[i] > xt));
      }
      st.s += s;
      st.w += w;
      if (a.l.top > 0) {
        if (__ballot(!(most <= bound))) {
#pragma unroll
          for (int u = 0; u < C::kLoads; ++u) {
            if (!__ballot(!(of_load[u] <= bound))) continue;
            uint32_t any = 0u;  // elements of which some lane's may enter
#pragma unroll
            for (int j = 0; j < C::kVec; ++j) any |= __ballot(!(f[u * C::kVec + j] <= bound)) ? 1u << j : 0u;
            while (any) {
              const int j = __builtin_ctz(any);
              any &= any - 1u;
              const int64_t at = base + (u * 64 + lane) * C::kVec + j;
              const float x = f[u * C::kVec + j];
              list.offer(key_of(x, at), __ballot(!(x <= bound) && at < V));
            }
          }
          if (list.kth) bound = logit_of(list.kth);
        }
      }
    }
    wave_sum(st);
  }

  if constexpr (PER_ROW > 1) {
    __shared__ Stats stats[kWaves];
    __shared__ int ranks[kWaves], n_left[kRows];
    __shared__ Key keys[kWaves * GNNSHAP_MAX_TOP], left[kWaves * GNNSHAP_MAX_TOP], best[kRows * GNNSHAP_MAX_TOP];
    const int k = a.l.top, r = wave / PER_ROW;
    if (lane == 0) {
      stats[wave] = st;
      ranks[wave] = rank;
    }
    if (lane < k) keys[wave * k + lane] = list.mine;
    __syncthreads();
    if (k > 0)
      join_lists(keys + r * PER_ROW * k, PER_ROW, k, left + r * PER_ROW * GNNSHAP_MAX_TOP, n_left + r,
                 best + r * GNNSHAP_MAX_TOP, threadIdx.x % (64 * PER_ROW), 64 * PER_ROW);
    if (way != 0 || !in) return;
    for (int i = 1; i < PER_ROW; ++i) {
      add(st, stats[wave + i]);
      rank += ranks[wave + i];
    }
    if (lane < k) list.mine = best[r * GNNSHAP_MAX_TOP + lane];
    if (a.parts > 1) {
      const int64_t at = row * a.parts + part;
      if (lane == 0) {
        a.part_stats[at] = st;
        a.part_rank[at] = rank;
      }
      if (lane < k) a.part_keys[at * k + lane] = list.mine;
      return;
    }
  }
  if (in) write_row(a, row, st, rank, list.mine, has, xt);
}

// Joins the parts of a row that several workgroups read, a workgroup per row.
template <class T>
__global__ __launch_bounds__(64 * kWaves) void k_token_logprobs_join(LogprobArgs a) {
  __shared__ Key keys[kMaxPartKeys], left[kMaxPartKeys], best[GNNSHAP_MAX_TOP];
  __shared__ int n_left;
  const int lane = threadIdx.x & 63, k = a.l.top, n = a.parts * k;
  const int64_t row = blockIdx.x;
  for (int i = threadIdx.x; i < n; i += 64 * kWaves) keys[i] = a.part_keys[row * n + i];
  __syncthreads();
  if (k > 0) join_lists(keys, a.parts, k, left, &n_left, best, threadIdx.x, blockDim.x);
  if (threadIdx.x >= 64) return;
  Stats st = no_stats();
  int rank = 0;
  if (lane < a.parts) {
    st = a.part_stats[row * a.parts + lane];
    rank = a.part_rank[row * a.parts + lane];
  }
  bool has;
  const float xt = given(a, static_cast<const T*>(a.l.logits) + row * a.l.row_stride, row, has);
  wave_sum(st);
#pragma unroll
  for (int off = 1; off < 64; off *= 2) rank += __shfl_xor(rank, off);
  write_row(a, row, st, rank, lane < k ? best[lane] : 0, has, xt);
}

// Rows of up to LANES x N logits, LANES lanes per row: a row is in registers,
// so its maximum comes first and the alternatives are taken off one by one.
// Lanes of 16 are put together by moves within the vector unit: 100,000 x 41
// fp32 with the top 3 14.5 us, 0.9 less than by way of LDS; bf16 without
// alternatives 8.4.
template <class T, int LANES, int N>
__global__ __launch_bounds__(256) void k_token_logprobs_short(LogprobArgs a) {
  const int lane = threadIdx.x % LANES, V = static_cast<int>(a.l.vocab);
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  const bool in = row < a.l.num_rows;
  const T* x = static_cast<const T*>(a.l.logits) + (in ? row : 0) * a.l.row_stride;
  float f[N], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = in && lane + LANES * i < V ? static_cast<float>(x[lane + LANES * i]) : -INFINITY;
  bool has = false;
  const float xt = in ? given(a, x, row, has) : 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, f[i]);
  m = together<LANES>(m, [](float x, float y) { return fmaxf(x, y); });
  const float use = finite_max(m);
  float s = 0.f, w = 0.f;
  uint32_t rank = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float d = (f[i] - use) * kLog2e, e = __builtin_amdgcn_exp2f(d);
    s += e;
    w += e * fmaxf(d, -200.f);
    rank += f[i] > xt;
  }
  const auto plus = [](auto x, auto y) { return x + y; };
  s = together<LANES>(s, plus);
  w = together<LANES>(w, plus);
  rank = together<LANES>(rank, plus);
  const bool none = s == 0.f;
  const float logs = logf(s);
  if (in && lane == 0) write_stats(a, row, Stats{m, s, w}, logs, static_cast<int>(rank), has, xt);

  Key last = ~0ull;
  for (int k = 0; k < a.l.top; ++k) {
    Key best = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const Key key = key_of(f[i], lane + LANES * i);
      if (lane + LANES * i < V && key < last) best = max(best, key);
    }
    best = together<LANES>(best, [](Key x, Key y) { return max(x, y); });
    last = best;
    if (in && lane == k % LANES) {
      const int64_t at = row * a.l.top + k;
      if (a.l.top_logprob) a.l.top_logprob[at] = none ? -INFINITY : (logit_of(best) - m) - logs;
      if (a.l.top_id) a.l.top_id[at] = token_of(best);
    }
  }
}

struct GradArgs {
  gnnshap_logits l;
  const float* gl;
  const float* ge;
  void* grad;
  int64_t stride;
  int32_t* info;
};

constexpr int kGradPacks = 4;

// blockDim.x threads take a row's elements in packs of 16 bytes, four in
// flight, blockDim.y rows per workgroup; every element is read once and
// written once.  2,000 x 50,021 bf16 (400 MB, rows at odd addresses): 88 us,
// 4.5 TB/s (74 where other work runs between the calls); 115 us with one pack in
// flight.
template <class T>
__global__ __launch_bounds__(256) void k_token_logprobs_grad(GradArgs a) {
  constexpr int kVec = 16 / sizeof(T);
  const int64_t row = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  if (row >= a.l.num_rows) return;
  const T* x = static_cast<const T*>(a.l.logits) + row * a.l.row_stride;
  T* out = static_cast<T*>(a.grad) + row * a.stride;
  const int64_t V = a.l.vocab;
  int64_t t = a.l.targets ? a.l.targets[row] : -1;
  if (t >= V) {
    if (a.info) *a.info = 1;
    t = -1;
  }
  // log p = (x - top) - logs; by lse alone p is off by its rounding
  const float top = a.l.maximum ? a.l.maximum[row] : a.l.lse[row], logs = a.l.maximum ? a.l.log_sum[row] : 0.f;
  const float gl = a.gl && t >= 0 ? a.gl[row] : 0.f;
  const float ge = a.ge ? a.ge[row] : 0.f, ent = a.ge ? a.l.entropy[row] : 0.f;
  const bool none = top == -INFINITY && logs == 0.f;  // (a row of NaN alone has log_sum NaN)
  const auto d = [&](T xi, int64_t i) {
    const float logp = (static_cast<float>(xi) - top) - logs, p = __builtin_amdgcn_exp2f(logp * kLog2e);
    const float own = i == t ? gl : 0.f;
    const float r = own - p * (gl + ge * ((p == 0.f ? 0.f : logp) + ent));
    return static_cast<T>(none ? 0.f : r);
  };
  const int64_t turn = static_cast<int64_t>(blockDim.x) * kVec, step = gridDim.y * turn * kGradPacks;
  for (int64_t i = blockIdx.y * turn * kGradPacks + threadIdx.x * kVec; i < V; i += step) {
    if (i + (kGradPacks - 1) * turn + kVec <= V) {
      Pack<T, kVec> p[kGradPacks];
#pragma unroll
      for (int u = 0; u < kGradPacks; ++u) p[u] = load_pack<T, kVec>(x + i + u * turn);
#pragma unroll
      for (int u = 0; u < kGradPacks; ++u) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) p[u].v[e] = d(p[u].v[e], i + u * turn + e);
        store_pack(out + i + u * turn, p[u]);
      }
      continue;
    }
    for (int u = 0; u < kGradPacks; ++u) {
      const int64_t from = i + u * turn;
      if (from + kVec <= V) {
        Pack<T, kVec> p = load_pack<T, kVec>(x + from);
#pragma unroll
        for (int e = 0; e < kVec; ++e) p.v[e] = d(p.v[e], from + e);
        store_pack(out + from, p);
      } else {
        for (int64_t j = from; j < V; ++j) out[j] = d(x[j], j);
      }
    }
  }
}

int check_logits(const gnnshap_logits* l) {
  using gnnshap::fail;
  if (!l) return fail(GNNSHAP_EINVAL, "logits is NULL");
  if (l->dtype < GNNSHAP_F32 || l->dtype > GNNSHAP_BF16)
    return fail(GNNSHAP_EUNSUPPORTED, "dtype %d is not one of f32, f16, bf16", static_cast<int>(l->dtype));
  if (l->num_rows < 0 || l->vocab < 1)
    return fail(GNNSHAP_EINVAL, "%lld rows of %lld logits", static_cast<long long>(l->num_rows),
                static_cast<long long>(l->vocab));
  if (l->num_rows > INT32_MAX || l->vocab > (int64_t(1) << 30))
    return fail(GNNSHAP_EUNSUPPORTED, "%lld rows of %lld logits", static_cast<long long>(l->num_rows),
                static_cast<long long>(l->vocab));
  if (l->row_stride < 0) return fail(GNNSHAP_EINVAL, "negative row stride");
  if (l->top < 0 || l->top > l->vocab || l->top > GNNSHAP_MAX_TOP)
    return fail(GNNSHAP_EINVAL, "top %d of %lld logits (at most %d)", static_cast<int>(l->top),
                static_cast<long long>(l->vocab), GNNSHAP_MAX_TOP);
  return GNNSHAP_OK;
}

// How a row is read.  Up to 64 logits in registers of 16 lanes, up to 256 (and
// 1,024 where no alternatives are wanted) of a wavefront; longer rows by one
// wavefront, two or four with their lists, fewer where there are rows for all
// of the chip's wavefronts several times; few rows by several workgroups.
// Measured in bf16: 100,000 x 41, top 5: in registers 20 us, from lists 181;
// 10,000 x 500: without alternatives 7.6 against 14.7, with 5 22.0 against
// 20.8; 40,000 x 5,000: one wavefront 150, four 202; 10,000 x 32,768, top 5:
// two wavefronts 154, four 165.
enum Way { kShort64, kShort256, kShort1024, kWavefront, kTwoWavefronts, kWorkgroup };
struct Shape {
  Way way;
  int parts;
  int64_t workgroups(int64_t rows) const {
    switch (way) {
      case kShort64: return gnnshap::ceil_div(rows, 16);
      case kTwoWavefronts: return gnnshap::ceil_div(rows, kWaves / 2);
      case kWorkgroup: return rows * parts;
      default: return gnnshap::ceil_div(rows, kWaves);
    }
  }
};
Shape shape_of(const gnnshap_logits& l) {
  if (l.vocab <= 64) return {kShort64, 1};
  if (l.vocab <= (l.top ? 256 : 1024)) return {l.vocab <= 256 ? kShort256 : kShort1024, 1};
  const int64_t chunk = 64 * 4 * (l.dtype == GNNSHAP_F32 ? 4 : 8), chunks = gnnshap::ceil_div(l.vocab, chunk);
  if (chunks == 1 || (l.num_rows >= 4096 && chunks < 16)) return {kWavefront, 1};
  if (l.num_rows >= 4096 && chunks < 32) return {kTwoWavefronts, 1};
  const int64_t want = gnnshap::ceil_div(1024, std::max<int64_t>(l.num_rows, 1));
  return {kWorkgroup, static_cast<int>(std::min<int64_t>({gnnshap::ceil_div(chunks, kWaves), want, kMaxParts,
                                                          l.top ? kMaxPartKeys / l.top : kMaxParts}))};
}

size_t carve(LogprobArgs& a, void* ws) {
  gnnshap::Carver c(ws);
  if (a.parts == 1) return 0;
  const size_t n = static_cast<size_t>(a.l.num_rows) * a.parts;
  a.part_stats = c.take<Stats>(n);
  a.part_rank = c.take<int32_t>(n);
  a.part_keys = c.take<Key>(n * a.l.top);
  return c.bytes();
}

}  // namespace

extern "C" int gnnshap_token_logprobs_workspace(const gnnshap_logits* l, size_t* bytes) {
  GS_TRY_BEGIN
  gnnshap::clear_error();
  if (!bytes) return gnnshap::fail(GNNSHAP_EINVAL, "bytes is NULL");
  if (const int st = check_logits(l)) return st;
  LogprobArgs a{};
  a.l = *l;
  const Shape shape = shape_of(*l);
  if (const int st = gnnshap::check_launch(shape.workgroups(l->num_rows), 64 * kWaves)) return st;
  a.parts = shape.parts;
  *bytes = carve(a, nullptr);
  return GNNSHAP_OK;
  GS_TRY_END
}

extern "C" int gnnshap_token_logprobs(const gnnshap_logits* l, int32_t* info, void* ws, size_t ws_bytes,
                                      void* stream) {
  using gnnshap::fail;
  GS_TRY_BEGIN
  gnnshap::clear_error();
  if (const int st = check_logits(l)) return st;
  if (l->num_rows == 0) return GNNSHAP_OK;
  if (!l->logits) return fail(GNNSHAP_EINVAL, "logits array is NULL");
  LogprobArgs a{};
  a.l = *l;
  a.info = info;
  const Shape shape = shape_of(*l);
  if (const int st = gnnshap::check_launch(shape.workgroups(l->num_rows), 64 * kWaves)) return st;
  a.parts = shape.parts;
  const size_t need = carve(a, ws);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(GNNSHAP_ECAPACITY, "token_logprobs workspace needs %zu bytes, has %zu", need, ws ? ws_bytes : 0);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return gnnshap::with_dtype(l->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    const unsigned grid = static_cast<unsigned>(shape.workgroups(l->num_rows));
    {
      GS_TIMED("k_token_logprobs", s);
      switch (shape.way) {
        case kShort64: k_token_logprobs_short<T, 16, 4><<<grid, 256, 0, s>>>(a); break;
        case kShort256: k_token_logprobs_short<T, 64, 4><<<grid, 256, 0, s>>>(a); break;
        case kShort1024: k_token_logprobs_short<T, 64, 16><<<grid, 256, 0, s>>>(a); break;
        case kWavefront: k_token_logprobs<T, 1><<<grid, 64 * kWaves, 0, s>>>(a); break;
        case kTwoWavefronts: k_token_logprobs<T, 2><<<grid, 64 * kWaves, 0, s>>>(a); break;
        case kWorkgroup: k_token_logprobs<T, kWaves><<<grid, 64 * kWaves, 0, s>>>(a);
      }
    }
    GS_LAUNCHED();
    if (a.parts > 1) {
      GS_TIMED("k_token_logprobs_join", s);
      k_token_logprobs_join<T><<<static_cast<unsigned>(l->num_rows), 64 * kWaves, 0, s>>>(a);
      GS_LAUNCHED();
    }
    return static_cast<int>(GNNSHAP_OK);
  });
  GS_TRY_END
}

extern "C" int gnnshap_token_logprobs_backward(const gnnshap_logits* l, const float* g_logprob,
                                               const float* g_entropy, void* grad, int64_t grad_stride, int32_t* info,
                                               void* stream) {
  using gnnshap::fail;
  GS_TRY_BEGIN
  gnnshap::clear_error();
  if (const int st = check_logits(l)) return st;
  if (grad_stride < 0) return fail(GNNSHAP_EINVAL, "negative stride of the gradient");
  if (l->num_rows == 0) return GNNSHAP_OK;
  if (!l->maximum != !l->log_sum) return fail(GNNSHAP_EINVAL, "maximum and log_sum: both are needed, or neither");
  if (!l->logits || (!l->lse && !l->maximum) || !grad || (g_entropy && !l->entropy))
    return fail(GNNSHAP_EINVAL, "NULL logits, lse, grad or (with g_entropy) entropy");
  GradArgs a{*l, g_logprob, g_entropy, grad, grad_stride, info};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return gnnshap::with_dtype(l->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    const int64_t packs = gnnshap::ceil_div(l->vocab, 16 / sizeof(T));
    int x = 8;
    while (x < 256 && x < packs) x *= 2;
    const int64_t groups = gnnshap::ceil_div(l->num_rows, 256 / x);
    if (const int st = gnnshap::check_launch(groups, x)) return st;
    const dim3 grid(static_cast<unsigned>(groups),
                    static_cast<unsigned>(std::min<int64_t>(gnnshap::ceil_div(packs, x * kGradPacks), 1024)));
    {
      GS_TIMED("k_token_logprobs_grad", s);
      k_token_logprobs_grad<T><<<grid, dim3(x, 256 / x), 0, s>>>(a);
    }
    GS_LAUNCHED();
    return static_cast<int>(GNNSHAP_OK);
  });
  GS_TRY_END
}
