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
// and of equal logits the lowest token wins.  A chunk of a row is looked at
// again only if its maximum exceeds the list's k-th key; of the wavefront's
// first chunk only the logits from the k-th largest of the lanes' maxima on
// (at least k logits are no smaller).
//
// One wavefront reads chunks of 64 lanes x 4 x 16 bytes.  A row is one
// wavefront's, or one workgroup's, or (few rows) several workgroups', whose
// parts a second launch joins.
#include "tokens.h"

namespace {

using gnnshap::bf16_t;
using gnnshap::f16_t;
using gnnshap::load_pack;
using gnnshap::Pack;
using gnnshap::store_pack;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kWaves = 4;      // wavefronts of a workgroup
constexpr int kMaxParts = 64;  // workgroups of a row

struct Stats {
  float m, s, w;  // w = sum e_j log2(e_j)
};
__device__ __forceinline__ Stats no_stats() { return Stats{-INFINITY, 0.f, 0.f}; }

__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

// Moves a to the maximum m >= a.m.
__device__ __forceinline__ void move_to(Stats& a, float m) {
  if (a.s != 0.f) {  // NaN too
    const float d = (a.m - finite_max(m)) * kLog2e, f = __builtin_amdgcn_exp2f(d);
    a.w = f * (a.w + a.s * fmaxf(d, -1e30f));
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

// Whole numbers in the order of the floats (-0 and 0 alike, NaN above all).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  if (x != x) return 0xFFFFFFFFu;
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

struct Key {
  uint32_t v, i;  // i = ~token; (0, 0) is below every logit's key
};
__device__ __forceinline__ bool above(Key a, Key b) { return a.v > b.v || (a.v == b.v && a.i > b.i); }
__device__ __forceinline__ Key lane_key(Key a, int lane) {
  Key r;
  r.v = __builtin_amdgcn_readlane(a.v, lane);
  r.i = __builtin_amdgcn_readlane(a.i, lane);
  return r;
}

// The 64 best keys of a wavefront, of which the first k are wanted.
struct TopList {
  Key mine{0u, 0u}, kth{0u, 0u};
  int k;
  __device__ __forceinline__ explicit TopList(int top) : k(top) {}
  __device__ __forceinline__ void insert(Key c) {
    const int lane = threadIdx.x & 63;
    const int pos = __popcll(__ballot(above(mine, c)));
    Key up;
    up.v = __shfl_up(mine.v, 1);
    up.i = __shfl_up(mine.i, 1);
    if (lane > pos) mine = up;
    if (lane == pos) mine = c;
    kth = lane_key(mine, k - 1);
  }
  // Every lane's key; ends after at most 64 insertions.
  __device__ __forceinline__ void offer(Key c, bool is) {
    const int lane = threadIdx.x & 63;
    uint64_t b = __ballot(is && above(c, kth));
    while (b) {
      const int src = __builtin_ctzll(b);
      insert(lane_key(c, src));
      is = is && lane != src;
      b = __ballot(is && above(c, kth));
    }
  }
};

// The k-th largest of the lanes' values.
__device__ __forceinline__ uint32_t kth_of_lanes(uint32_t v, int k) {
  uint32_t t = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t u = t | (1u << b);
    if (__popcll(__ballot(v >= u)) >= k) t = u;
  }
  return t;
}

template <class T>
struct Chunk {
  static constexpr int kVec = 16 / sizeof(T);
  static constexpr int kLoads = 4;
  static constexpr int kElems = kVec * kLoads;  // per lane
  static constexpr int kSize = 64 * kElems;     // per wavefront
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

// What a row's statistics and list give the caller; the whole wavefront calls it.
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t row, const Stats& st, int rank,
                                          const TopList& list, bool has, float xt) {
  const int lane = threadIdx.x & 63;
  const bool none = st.s == 0.f;  // every logit is -inf
  const float logs = logf(st.s);
  if (lane == 0) {
    if (a.l.lse) a.l.lse[row] = none ? -INFINITY : st.m + logs;
    if (a.l.entropy) a.l.entropy[row] = none ? 0.f : logs - kLn2 * (st.w / st.s);
    if (a.l.logprob) a.l.logprob[row] = !has ? 0.f : none ? -INFINITY : (xt - st.m) - logs;
    if (a.l.rank) a.l.rank[row] = has ? rank : -1;
  }
  if (lane < a.l.top) {
    const int64_t at = row * a.l.top + lane;
    if (a.l.top_logprob) a.l.top_logprob[at] = none ? -INFINITY : (unordered(list.mine.v) - st.m) - logs;
    if (a.l.top_id) a.l.top_id[at] = static_cast<int32_t>(~list.mine.i);
  }
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
  if (in) {
    int64_t base = (static_cast<int64_t>(part) * PER_ROW + way) * C::kSize;
    const int64_t step = static_cast<int64_t>(a.parts) * PER_ROW * C::kSize;
    C next;
    if (base < V) next.load(x, base, V);
    xt = given(a, x, row, has);
    bool first = true;
    for (; base < V; base += step) {
      const C c = next;
      if (base + step < V) next.load(x, base + step, V);
      float f[C::kElems], most = -INFINITY;
#pragma unroll
      for (int i = 0; i < C::kElems; ++i) {
        f[i] = static_cast<float>(c.p[i / C::kVec].v[i % C::kVec]);
        most = fmaxf(most, f[i]);
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
        const uint32_t o = ordered(most);
        if (__ballot(o > list.kth.v)) {
          const uint32_t from = first ? kth_of_lanes(o, a.l.top) : 0u;
#pragma unroll
          for (int i = 0; i < C::kElems; ++i) {
            const int64_t at = base + ((i / C::kVec) * 64 + lane) * C::kVec + i % C::kVec;
            Key key;
            key.v = ordered(f[i]);
            key.i = ~static_cast<uint32_t>(at);
            list.offer(key, at < V && key.v >= from);
          }
        }
        first = false;
      }
    }
    wave_sum(st);
  }

  if constexpr (PER_ROW > 1) {
    __shared__ Stats stats[kWaves];
    __shared__ int ranks[kWaves];
    __shared__ Key keys[kWaves][64];
    if (lane == 0) {
      stats[wave] = st;
      ranks[wave] = rank;
    }
    keys[wave][lane] = list.mine;
    __syncthreads();
    if (wave != 0 || !in) return;
    for (int i = 1; i < PER_ROW; ++i) {
      add(st, stats[i]);
      rank += ranks[i];
      if (a.l.top > 0) list.offer(keys[i][lane], lane < a.l.top);
    }
    if (a.parts > 1) {
      const int64_t at = row * a.parts + part;
      if (lane == 0) {
        a.part_stats[at] = st;
        a.part_rank[at] = rank;
      }
      if (lane < a.l.top) a.part_keys[at * a.l.top + lane] = list.mine;
      return;
    }
  }
  if (in) write_row(a, row, st, rank, list, has, xt);
}

// Joins the parts of rows that several workgroups read, a wavefront per row.
template <class T>
__global__ __launch_bounds__(64 * kWaves) void k_token_logprobs_join(LogprobArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (row >= a.l.num_rows) return;
  Stats st = no_stats();
  int rank = 0;
  if (lane < a.parts) {
    st = a.part_stats[row * a.parts + lane];
    rank = a.part_rank[row * a.parts + lane];
  }
  wave_sum(st);
#pragma unroll
  for (int off = 1; off < 64; off *= 2) rank += __shfl_xor(rank, off);
  TopList list(a.l.top);
  const int keys = a.parts * a.l.top;
  for (int i = 0; i < keys; i += 64) {
    const bool is = i + lane < keys;
    Key key{0u, 0u};
    if (is) key = a.part_keys[row * keys + i + lane];
    list.offer(key, is);
  }
  bool has;
  const float xt = given(a, static_cast<const T*>(a.l.logits) + row * a.l.row_stride, row, has);
  write_row(a, row, st, rank, list, has, xt);
}

struct GradArgs {
  gnnshap_logits l;
  const float* gl;
  const float* ge;
  void* grad;
  int64_t stride;
  int32_t* info;
};

// blockDim.x threads take a row's elements in packs of 16 bytes, blockDim.y
// rows per workgroup; every element is read once and written once.
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
  const float lse = a.l.lse[row];
  const float gl = a.gl && t >= 0 ? a.gl[row] : 0.f;
  const float ge = a.ge ? a.ge[row] : 0.f, ent = a.ge ? a.l.entropy[row] : 0.f;
  const bool none = lse == -INFINITY;
  const auto d = [&](T xi, int64_t i) {
    const float logp = static_cast<float>(xi) - lse, p = __builtin_amdgcn_exp2f(logp * kLog2e);
    const float own = i == t ? gl : 0.f;
    const float r = own - p * (gl + ge * ((p == 0.f ? 0.f : logp) + ent));
    return static_cast<T>(none ? 0.f : r);
  };
  const int64_t step = static_cast<int64_t>(gridDim.y) * blockDim.x * kVec;
  for (int64_t i = (static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x) * kVec; i < V; i += step) {
    if (i + kVec <= V) {
      Pack<T, kVec> p = load_pack<T, kVec>(x + i);
#pragma unroll
      for (int e = 0; e < kVec; ++e) p.v[e] = d(p.v[e], i + e);
      store_pack(out + i, p);
    } else {
      for (int64_t j = i; j < V; ++j) out[j] = d(x[j], j);
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

// Wavefronts per row: one where there are rows for all of the chip's
// wavefronts several times, else four, and with few rows several workgroups.
struct Shape {
  int per_row, parts;
};
Shape shape_of(const gnnshap_logits& l) {
  const int64_t chunk = 64 * 4 * (l.dtype == GNNSHAP_F32 ? 4 : 8), chunks = gnnshap::ceil_div(l.vocab, chunk);
  if (l.num_rows >= 4096 || chunks == 1) return {1, 1};
  const int64_t want = gnnshap::ceil_div(1024, std::max<int64_t>(l.num_rows, 1));
  return {kWaves, static_cast<int>(std::min<int64_t>({gnnshap::ceil_div(chunks, kWaves), want, kMaxParts}))};
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
  a.parts = shape_of(*l).parts;
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
  a.parts = shape.parts;
  const size_t need = carve(a, ws);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(GNNSHAP_ECAPACITY, "token_logprobs workspace needs %zu bytes, has %zu", need, ws ? ws_bytes : 0);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return gnnshap::with_dtype(l->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    const unsigned groups = static_cast<unsigned>(gnnshap::ceil_div(l->num_rows, kWaves));
    {
      GS_TIMED("k_token_logprobs", s);
      if (shape.per_row == 1)
        k_token_logprobs<T, 1><<<groups, 64 * kWaves, 0, s>>>(a);
      else
        k_token_logprobs<T, kWaves><<<static_cast<unsigned>(l->num_rows * a.parts), 64 * kWaves, 0, s>>>(a);
    }
    GS_LAUNCHED();
    if (a.parts > 1) {
      GS_TIMED("k_token_logprobs_join", s);
      k_token_logprobs_join<T><<<groups, 64 * kWaves, 0, s>>>(a);
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
  if (!l->logits || !l->lse || !grad || (g_entropy && !l->entropy))
    return fail(GNNSHAP_EINVAL, "NULL logits, lse, grad or (with g_entropy) entropy");
  GradArgs a{*l, g_logprob, g_entropy, grad, grad_stride, info};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return gnnshap::with_dtype(l->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    const int64_t packs = gnnshap::ceil_div(l->vocab, 16 / sizeof(T));
    int x = 8;
    while (x < 256 && x < packs) x *= 2;
    const dim3 grid(static_cast<unsigned>(gnnshap::ceil_div(l->num_rows, 256 / x)),
                    static_cast<unsigned>(std::min<int64_t>(gnnshap::ceil_div(packs, x), 1024)));
    {
      GS_TIMED("k_token_logprobs_grad", s);
      k_token_logprobs_grad<T><<<grid, dim3(x, 256 / x), 0, s>>>(a);
    }
    GS_LAUNCHED();
    return static_cast<int>(GNNSHAP_OK);
  });
  GS_TRY_END
}
