// Attention of one new token per row over a paged cache of keys and values,
// a part of which rows may share, under coalition masks.
//
// For the query q of a row's head over its visible positions j:
//     s_j = scale q . k_j,  out = sum_j e^{s_j} v_j / sum_j e^{s_j}.
// One pass over the keys with a running maximum m, in powers of two:
// p_j = 2^(s_j log2 e - m), l = sum p_j, O = sum p_j v_j; where m rises, l and
// O are scaled down.  Two such triples (m, l, O) of parts of the context add
// up after scaling both to the larger m, so that a long context is split over
// wavefronts and workgroups and joined.
//
// The products run on matrix instructions, transposed: S^T = K Q^T has the
// query in the lane's column and the keys in its registers, which is how the
// right operand of O^T = V^T P^T wants P once the keys are counted in the
// registers' order; so the weights never leave their lane.  Keys are read by
// rows (lane = key), values by rows too and their 16-bit elements swapped in
// pairs of keys in registers.
//
// Rows that do not see a position must not be reached by what it holds.  Its
// score is replaced by -inf, and 0 times a finite value is 0; where a result
// comes out non-finite, the workgroup's queries are done again by a slow path
// that skips the positions each row does not see.
#include "tokens.h"

namespace {

using gnnshap::bf16_t;
using gnnshap::f16_t;
using gnnshap::load_pack;
using gnnshap::Pack;

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef unsigned u4_t __attribute__((ext_vector_type(4)));

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kWaves = 4;
constexpr int kChunk = 32;  // keys of a wavefront's step

// One part of the rows' contexts: `r` consecutive rows share each row of its
// table.  A group's rows times the query heads of a kv head are its queries,
// in tiles; a workgroup takes a tile over split_keys keys.
struct Part {
  const int32_t* table;
  const int32_t* lengths;
  int64_t width;
  int max_len;
  int r;
  int tiles;
  int splits;
  int split_keys;
  int slot0;  // first of the part's slots of partial results
};

struct AttendArgs {
  gnnshap_cache c;
  gnnshap_queries q;
  int share;       // query heads per kv head
  int page_shift;  // log2 of the page size, or -1
  float scale2;    // scale log2 e
  Part shared, own;
  bool direct;     // one part of one split: results go straight to the caller
  float* part_o;   // [slot][row][head][head_dim], not divided by l
  float2* part_ml; // [slot][row][head]: m, l
  int32_t* info;
};

__device__ __forceinline__ int page_of(const AttendArgs& a, int key, int& slot) {
  if (a.page_shift >= 0) {
    slot = key & ((1 << a.page_shift) - 1);
    return key >> a.page_shift;
  }
  const int p = key / a.c.page_size;
  slot = key - p * a.c.page_size;
  return p;
}

// The length of sequence `g` of a part, at most what its arrays hold.
__device__ __forceinline__ int length_of(const AttendArgs& a, const Part& part, int64_t g) {
  const int n = part.lengths[g];
  if (n < 0 || n > part.max_len) {
    if (a.info) *a.info = 1;
    return n < 0 ? 0 : part.max_len;
  }
  return n;
}

// Which of the positions at .. at + 31 a row sees; `at` counts from the first player.
__device__ __forceinline__ uint32_t seen(const uint64_t* row, int64_t at, int64_t players) {
  if (at + 32 <= 0 || at >= players) return ~0u;
  const uint32_t* w = reinterpret_cast<const uint32_t*>(row);
  const int64_t words = (players + 31) >> 5, i = at >> 5;
  const int sh = static_cast<int>(at & 31);
  const uint32_t lo = i >= 0 ? w[i] : 0u, hi = sh && i + 1 < words ? w[i + 1] : 0u;
  uint32_t bits = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
  if (at < 0) bits |= (1u << -at) - 1u;
  if (at + 32 > players) bits |= ~0u << (players - at);
  return bits;
}

// Where a query's results go.
__device__ __forceinline__ int64_t part_index(const AttendArgs& a, int slot, int64_t row, int head) {
  return (static_cast<int64_t>(slot) * a.q.num_rows + row) * a.q.heads + head;
}

template <class T>
__device__ __forceinline__ T* out_of(const AttendArgs& a, int64_t row, int head) {
  return static_cast<T*>(a.q.out) + row * a.q.out_row_stride + head * a.q.out_head_stride;
}

__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : m * kLn2 + logf(l); }

// The matrix instructions and operand layouts of an element type.  DP: the
// head_dim rounded up; kOwn: consecutive elements of a value row that a lane
// holds; kGroups: runs of 16 lanes of them.
template <class T, int DP>
struct Ops {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  static constexpr int kOwn = DP >= 128 ? 8 : 4, kGroups = DP / (16 * kOwn), kSteps = DP / 32;
  struct Row {  // 16 keys or queries, this lane's quarter of their elements
    u4_t s[kSteps];
    __device__ __forceinline__ void load(const T* p, int D) {
      const int g = (threadIdx.x >> 4) & 3;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int d = 32 * i + 8 * g;
        s[i] = u4_t{0u, 0u, 0u, 0u};
        if (d < D) __builtin_memcpy(&s[i], p + d, 16);
      }
    }
  };
  static __device__ __forceinline__ f4_t mfma(u4_t a, u4_t b, f4_t c) {
    if constexpr (std::is_same_v<T, bf16_t>)
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(vec8, a), __builtin_bit_cast(vec8, b), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec8, a), __builtin_bit_cast(vec8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f4_t scores(const Row& k, const Row& q) {
    f4_t c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) c = mfma(k.s[i], q.s[i], c);
    return c;
  }
  struct Values {  // 8 keys, kOwn elements of each in kGroups places
    unsigned v[8][kGroups][kOwn / 2];
    __device__ __forceinline__ void load(int j, const T* p, int D) {
      const int r = threadIdx.x & 15;
#pragma unroll
      for (int b = 0; b < kGroups; ++b) {
        const int d = (16 * b + r) * kOwn;
#pragma unroll
        for (int e = 0; e < kOwn / 2; ++e) v[j][b][e] = 0u;
        if (d < D) __builtin_memcpy(&v[j][b][0], p + d, 2 * kOwn);
      }
    }
    __device__ __forceinline__ u4_t operand(int b, int e) const {
      u4_t r;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        r[j] = __builtin_amdgcn_perm(v[2 * j + 1][b][e / 2], v[2 * j][b][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
      return r;
    }
  };
  // O^T += V^T P^T; the weights are rounded to the values' type here
  static __device__ __forceinline__ void add(f4_t (&o)[kGroups][kOwn], const Values& v, const float (&p)[8]) {
    vec8 w;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = static_cast<T>(p[j]);
#pragma unroll
    for (int b = 0; b < kGroups; ++b)
#pragma unroll
      for (int e = 0; e < kOwn; ++e) o[b][e] = mfma(v.operand(b, e), __builtin_bit_cast(u4_t, w), o[b][e]);
  }
};

template <int DP>
struct Ops<float, DP> {
  static constexpr int kOwn = 4, kGroups = DP / 64, kSteps = DP / 16;
  struct Row {
    f4_t s[kSteps];
    __device__ __forceinline__ void load(const float* p, int D) {
      const int g = (threadIdx.x >> 4) & 3;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int d = 16 * i + 4 * g;
        s[i] = f4_t{0.f, 0.f, 0.f, 0.f};
        if (d < D) __builtin_memcpy(&s[i], p + d, 16);
      }
    }
  };
  static __device__ __forceinline__ f4_t scores(const Row& k, const Row& q) {
    f4_t c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(k.s[i][e], q.s[i][e], c, 0, 0, 0);
    return c;
  }
  struct Values {
    f4_t v[8][kGroups];
    __device__ __forceinline__ void load(int j, const float* p, int D) {
      const int r = threadIdx.x & 15;
#pragma unroll
      for (int b = 0; b < kGroups; ++b) {
        const int d = (16 * b + r) * 4;
        v[j][b] = f4_t{0.f, 0.f, 0.f, 0.f};
        if (d < D) __builtin_memcpy(&v[j][b], p + d, 16);
      }
    }
  };
  static __device__ __forceinline__ void add(f4_t (&o)[kGroups][kOwn], const Values& v, const float (&p)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int b = 0; b < kGroups; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[b][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.v[j][b][e], p[j], o[b][e], 0, 0, 0);
  }
};

struct Place {  // what a workgroup works on
  int64_t group;
  int kv_head, tile, split;
  int64_t first;  // context position of the part's position 0, counted from the first player
  int k0, k1;     // keys of the split
};

// The slow path: queries one after the other, a thread per key and then per
// element; a position that the row does not see enters no product.
template <class T>
__device__ void attend_slowly(const AttendArgs& a, const Part& part, Place at, int queries, const int* pages,
                                           float* lds) {
  const int tid = threadIdx.x, D = a.c.head_dim, wave = tid >> 6, lane = tid & 63;
  float* weight = lds;       // 256
  float* red = lds + 256;    // 2 x kWaves
  const int page0 = at.k0 / a.c.page_size;
  const int64_t head_at = static_cast<int64_t>(at.kv_head) * a.c.head_stride;
  for (int i = 0; i < queries; ++i) {
    const int qi = at.tile * queries + i;
    if (qi >= part.r * a.share) break;
    const int64_t row = at.group * part.r + qi / a.share;
    const int head = at.kv_head * a.share + qi % a.share;
    const T* q = static_cast<const T*>(a.q.q) + row * a.q.q_row_stride + head * a.q.q_head_stride;
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int c = at.k0; c < at.k1; c += 256) {
      const int key = c + tid;
      bool sees = key < at.k1;
      if (sees && a.q.num_players > 0)
        sees = seen(a.q.masks + row * a.q.mask_words, at.first + key, a.q.num_players) & 1u;
      float s = -INFINITY;
      if (sees) {
        int slot;
        const int pg = page_of(a, key, slot);
        const T* k = static_cast<const T*>(a.c.k) + pages[pg - page0] * a.c.page_stride + slot * a.c.slot_stride + head_at;
        s = 0.f;
        for (int d = 0; d < D; ++d) s += static_cast<float>(q[d]) * static_cast<float>(k[d]);
        s *= a.scale2;
      }
      float top = s;
      for (int off = 1; off < 64; off *= 2) top = fmaxf(top, __shfl_xor(top, off));
      if (lane == 0) red[wave] = top;
      __syncthreads();
      top = m;
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, red[w]);
      const float use = top == -INFINITY ? 0.f : top;
      const float p = sees ? __builtin_amdgcn_exp2f(s - use) : -1.f;
      weight[tid] = p;
      float sum = sees ? p : 0.f;
      for (int off = 1; off < 64; off *= 2) sum += __shfl_xor(sum, off);
      if (lane == 0) red[kWaves + wave] = sum;
      __syncthreads();
      const float down = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - use);
      l *= down;
      for (int w = 0; w < kWaves; ++w) l += red[kWaves + w];
      m = top;
      if (tid < D) {
        o = m == -INFINITY ? 0.f : o * down;
        const int n = at.k1 - c < 256 ? at.k1 - c : 256;
        for (int j = 0; j < n; ++j) {
          const float pj = weight[j];
          if (pj < 0.f) continue;
          int slot;
          const int pg = page_of(a, c + j, slot);
          o += pj * static_cast<float>(static_cast<const T*>(a.c.v)[pages[pg - page0] * a.c.page_stride +
                                                                    slot * a.c.slot_stride + head_at + tid]);
        }
      }
      __syncthreads();
    }
    if (l == 0.f) o = 0.f;
    if (a.direct) {
      if (tid < D) out_of<T>(a, row, head)[tid] = static_cast<T>(l == 0.f ? 0.f : o / l);
      if (tid == 0 && a.q.lse) a.q.lse[row * a.q.heads + head] = lse_of(m, l);
    } else {
      const int64_t p = part_index(a, part.slot0 + at.split, row, head);
      if (tid < D) a.part_o[p * D + tid] = o;
      if (tid == 0) a.part_ml[p] = make_float2(m, l);
    }
  }
}

// A workgroup: 16 RT queries over one split of keys.  Its four wavefronts
// take the split's chunks of 32 keys in turn and are joined through LDS.
template <class T, int DP, int RT>
__global__ __launch_bounds__(64 * kWaves) void k_cache_attend(AttendArgs a, Part part, bool is_own) {
  using O = Ops<T, DP>;
  constexpr int kStride = DP + 4;
  extern __shared__ int lds[];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int D = a.c.head_dim;
  Place at;
  int64_t b = blockIdx.x;
  at.kv_head = b % a.c.kv_heads;
  b /= a.c.kv_heads;
  at.split = b % part.splits;
  b /= part.splits;
  at.tile = b % part.tiles;
  at.group = b / part.tiles;
  const int len = length_of(a, part, at.group);
  at.k0 = at.split * part.split_keys;
  at.k1 = len - at.k0 < part.split_keys ? len : at.k0 + part.split_keys;
  if (at.k0 >= at.k1) {
    if (!a.direct) return;
    at.k1 = at.k0;
  }
  at.first = -a.q.first_player;
  if (is_own && a.shared.table) at.first += length_of(a, a.shared, at.group / a.shared.r);

  // the pages of the split
  const int page0 = at.k0 / a.c.page_size;
  int* pages = lds;
  const int n_pages = at.k1 > at.k0 ? (at.k1 - 1) / a.c.page_size - page0 + 1 : 0;
  for (int i = tid; i < n_pages; i += 64 * kWaves) {
    int p = part.table[at.group * part.width + page0 + i];
    if (p < 0 || p >= a.c.num_pages) {
      if (a.info) *a.info = 1;
      p = 0;
    }
    pages[i] = p;
  }
  float* merge = reinterpret_cast<float*>(lds + ((part.split_keys / a.c.page_size + 2 + 3) & ~3));

  typename O::Row q[RT];
  int64_t row[RT];
  int head[RT];
  bool valid[RT];
  float m[RT], l[RT];
  f4_t o[RT][O::kGroups][O::kOwn];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int qi = (at.tile * RT + t) * 16 + r;
    valid[t] = qi < part.r * a.share;
    const int qs = valid[t] ? qi : 0;
    row[t] = at.group * part.r + qs / a.share;
    head[t] = at.kv_head * a.share + qs % a.share;
    q[t].load(static_cast<const T*>(a.q.q) + row[t] * a.q.q_row_stride + head[t] * a.q.q_head_stride, D);
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < O::kGroups; ++i)
#pragma unroll
      for (int e = 0; e < O::kOwn; ++e) o[t][i][e] = f4_t{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();

  const int64_t head_at = static_cast<int64_t>(at.kv_head) * a.c.head_stride;
  const auto offset = [&](int key) {
    key = key < at.k1 ? key : at.k1 - 1;
    int slot;
    const int pg = page_of(a, key, slot);
    return pages[pg - page0] * a.c.page_stride + slot * a.c.slot_stride + head_at;
  };
  for (int k = at.k0 + wave * kChunk; k < at.k1; k += kWaves * kChunk) {
    typename O::Row key[2];
    typename O::Values val;
#pragma unroll
    for (int i = 0; i < 2; ++i) key[i].load(static_cast<const T*>(a.c.k) + offset(k + 16 * i + r), D);
#pragma unroll
    for (int j = 0; j < 8; ++j) val.load(j, static_cast<const T*>(a.c.v) + offset(k + 16 * (j >> 2) + 4 * g + (j & 3)), D);
    const uint32_t there = at.k1 - k >= 32 ? ~0u : (1u << (at.k1 - k)) - 1u;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      uint32_t bits = there;
      if (a.q.num_players > 0) bits &= seen(a.q.masks + row[t] * a.q.mask_words, at.first + k, a.q.num_players);
      bits >>= 4 * g;
      float s[8], top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f4_t c = O::scores(key[i], q[t]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[4 * i + e] = bits >> (16 * i + e) & 1u ? c[e] * a.scale2 : -INFINITY;
          top = fmaxf(top, s[4 * i + e]);
        }
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      top = fmaxf(top, m[t]);
      const float use = top == -INFINITY ? 0.f : top, down = __builtin_amdgcn_exp2f(m[t] - use);
      m[t] = top;
      l[t] *= down;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[j] = __builtin_amdgcn_exp2f(s[j] - use);
        l[t] += s[j];
      }
#pragma unroll
      for (int i = 0; i < O::kGroups; ++i)
#pragma unroll
        for (int e = 0; e < O::kOwn; ++e) o[t][i][e] *= down;
      O::add(o[t], val, s);
    }
  }

  // join the wavefronts
  bool bad = false;
  float* ml = merge + kWaves * 16 * kStride;  // [wave][query]: m, then l
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] += __shfl_xor(l[t], 16);
    l[t] += __shfl_xor(l[t], 32);
    if (t > 0) __syncthreads();
    float* mine = merge + (wave * 16 + r) * kStride;
#pragma unroll
    for (int i = 0; i < O::kGroups; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < O::kOwn; ++e) mine[(16 * i + 4 * g + x) * O::kOwn + e] = o[t][i][e][x];
    if (g == 0) {
      ml[wave * 16 + r] = m[t];
      ml[kWaves * 16 + wave * 16 + r] = l[t];
    }
    __syncthreads();
    const int qi = (at.tile * RT + t) * 16 + (tid >> 4), d0 = (tid & 15) * (DP / 16);
    if (qi < part.r * a.share) {
      float top = -INFINITY, sum = 0.f, f[kWaves];
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w * 16 + (tid >> 4)]);
      const float use = top == -INFINITY ? 0.f : top;
      for (int w = 0; w < kWaves; ++w) {
        f[w] = __builtin_amdgcn_exp2f(ml[w * 16 + (tid >> 4)] - use);
        sum += f[w] * ml[kWaves * 16 + w * 16 + (tid >> 4)];
      }
      const int64_t row_t = at.group * part.r + qi / a.share;
      const int head_t = at.kv_head * a.share + qi % a.share;
      const int64_t p = part_index(a, part.slot0 + at.split, row_t, head_t);
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      bad |= !isfinite(sum);
#pragma unroll
      for (int e = 0; e < DP / 16; ++e) {
        const int d = d0 + e;
        float x = 0.f;
        for (int w = 0; w < kWaves; ++w) x += f[w] * merge[(w * 16 + (tid >> 4)) * kStride + d];
        if (d >= D) continue;
        bad |= !isfinite(x);
        if (a.direct)
          out_of<T>(a, row_t, head_t)[d] = static_cast<T>(x * inv);
        else
          a.part_o[p * D + d] = x;
      }
      if ((tid & 15) == 0) {
        if (!a.direct)
          a.part_ml[p] = make_float2(top, sum);
        else if (a.q.lse)
          a.q.lse[row_t * a.q.heads + head_t] = lse_of(top, sum);
      }
    }
  }
  if (__syncthreads_or(bad)) attend_slowly<T>(a, part, at, 16 * RT, pages, merge);
}

// Joins the parts of each query, a wavefront per row and head.
template <class T>
__global__ __launch_bounds__(256) void k_cache_attend_join(AttendArgs a) {
  const int lane = threadIdx.x & 63, D = a.c.head_dim;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (i >= a.q.num_rows * a.q.heads) return;
  const int64_t row = i / a.q.heads;
  const int head = static_cast<int>(i % a.q.heads);
  int ns = 0, no = 0;
  if (a.shared.table) ns = (length_of(a, a.shared, row / a.shared.r) + a.shared.split_keys - 1) / a.shared.split_keys;
  if (a.own.table) no = (length_of(a, a.own, row) + a.own.split_keys - 1) / a.own.split_keys;
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int n = 0; n < ns + no; ++n) {
    const int slot = n < ns ? a.shared.slot0 + n : a.own.slot0 + n - ns;
    const int64_t p = part_index(a, slot, row, head);
    const float2 ml = a.part_ml[p];
    if (ml.y == 0.f) continue;
    const float top = fmaxf(m, ml.x), use = top == -INFINITY ? 0.f : top;
    const float down = __builtin_amdgcn_exp2f(m - use), up = __builtin_amdgcn_exp2f(ml.x - use);
    m = top;
    l = l * down + ml.y * up;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (4 * lane + e < D) o[e] = o[e] * down + a.part_o[p * D + 4 * lane + e] * up;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (4 * lane + e < D) out_of<T>(a, row, head)[4 * lane + e] = static_cast<T>(o[e] * inv);
  if (lane == 0 && a.q.lse) a.q.lse[row * a.q.heads + head] = lse_of(m, l);
}

int check_queries(const gnnshap_cache* c, const gnnshap_queries* q) {
  using gnnshap::fail;
  if (const int st = gnnshap::check_cache(c)) return st;
  if (!q || q->num_rows < 0) return fail(GNNSHAP_EINVAL, "queries: NULL or a negative number of rows");
  if (q->heads < 1 || q->heads % c->kv_heads != 0)
    return fail(GNNSHAP_EINVAL, "%d query heads over %d kv heads", static_cast<int>(q->heads),
                static_cast<int>(c->kv_heads));
  if (!(q->scale != 0.0) || !std::isfinite(q->scale)) return fail(GNNSHAP_EINVAL, "scale is 0 or not finite");
  if (q->num_rows > INT32_MAX || q->num_rows * q->heads > (int64_t(1) << 40))
    return fail(GNNSHAP_EUNSUPPORTED, "%lld rows in one call", static_cast<long long>(q->num_rows));
  const struct {
    const char* name;
    const int32_t *table, *lengths;
    int64_t width, longest;
  } parts[2] = {{"shared", q->shared_table, q->shared_lengths, q->shared_width, q->max_shared},
                {"own", q->table, q->lengths, q->table_width, q->max_length}};
  for (const auto& p : parts) {
    if (!p.table) continue;
    if (!p.lengths) return fail(GNNSHAP_EINVAL, "%s table without lengths", p.name);
    if (p.longest < 0 || p.width < 0) return fail(GNNSHAP_EINVAL, "%s part: negative width or length", p.name);
    if (p.longest > INT32_MAX - 65536)
      return fail(GNNSHAP_EUNSUPPORTED, "%s part of up to %lld tokens", p.name, static_cast<long long>(p.longest));
    if (gnnshap::ceil_div(p.longest, c->page_size) > p.width)
      return fail(GNNSHAP_EINVAL, "%s part: %lld tokens do not fit %lld pages of %d", p.name,
                  static_cast<long long>(p.longest), static_cast<long long>(p.width), static_cast<int>(c->page_size));
  }
  if (q->shared_table && (q->rows_per_group < 1 || q->num_rows % q->rows_per_group != 0))
    return fail(GNNSHAP_EINVAL, "groups of %lld of %lld rows", static_cast<long long>(q->rows_per_group),
                static_cast<long long>(q->num_rows));
  if (q->num_players < 0 || q->num_players > INT32_MAX || q->first_player < 0 || q->first_player > INT32_MAX)
    return fail(GNNSHAP_EINVAL, "%lld players from position %lld", static_cast<long long>(q->num_players),
                static_cast<long long>(q->first_player));
  if (q->num_players > 0 && (!q->masks || q->mask_words < gnnshap::ceil_div(q->num_players, 64)))
    return fail(GNNSHAP_EINVAL, "%lld players without masks, or with %lld words", static_cast<long long>(q->num_players),
                static_cast<long long>(q->mask_words));
  return GNNSHAP_OK;
}

int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

// Tiles of 16 queries that a workgroup takes: more where many queries read the
// same keys, as far as the registers of a lane go.
int tile_of(int64_t queries, int head_dim) {
  return std::min(queries > 32 ? 4 : queries > 16 ? 2 : 1, 256 / padded_dim(head_dim));
}

// How the work is laid out over workgroups.
int lay_out(AttendArgs& a, const gnnshap_cache* c, const gnnshap_queries* q) {
  using gnnshap::ceil_div;
  a.c = *c;
  a.q = *q;
  a.share = q->heads / c->kv_heads;
  a.scale2 = static_cast<float>(q->scale * 1.4426950408889634074);
  a.page_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (c->page_size == 1 << i) a.page_shift = i;
  Part* parts[2] = {&a.shared, &a.own};
  int slots = 0;
  for (int i = 0; i < 2; ++i) {
    Part& p = *parts[i];
    p = Part{};
    p.table = i ? q->table : q->shared_table;
    if (!p.table) continue;
    p.lengths = i ? q->lengths : q->shared_lengths;
    p.width = i ? q->table_width : q->shared_width;
    p.max_len = static_cast<int>(i ? q->max_length : q->max_shared);
    p.r = static_cast<int>(i ? 1 : q->rows_per_group);
    const int64_t queries = static_cast<int64_t>(p.r) * a.share;
    if (queries > INT32_MAX) return gnnshap::fail(GNNSHAP_EUNSUPPORTED, "%lld queries of a group", static_cast<long long>(queries));
    p.tiles = static_cast<int>(ceil_div(queries, 16 * tile_of(queries, c->head_dim)));
    // enough workgroups for the chip, at least 256 keys each, at most 4096
    const int64_t base = q->num_rows / p.r * c->kv_heads * p.tiles;
    int64_t keys = ceil_div(std::max(p.max_len, 1), std::max<int64_t>(1, 1024 / std::max<int64_t>(base, 1)));
    keys = std::min<int64_t>(std::max<int64_t>(ceil_div(keys, 128) * 128, 256), i ? 1024 : 4096);
    p.split_keys = static_cast<int>(keys);
    p.splits = static_cast<int>(std::max<int64_t>(1, ceil_div(p.max_len, keys)));
    p.slot0 = slots;
    slots += p.splits;
    if (base * p.splits > INT32_MAX) return gnnshap::fail(GNNSHAP_EUNSUPPORTED, "too many workgroups");
  }
  a.direct = slots <= 1;
  return GNNSHAP_OK;
}

size_t carve(AttendArgs& a, void* ws) {
  if (a.direct) return 0;
  gnnshap::Carver c(ws);
  const size_t n = static_cast<size_t>(a.shared.splits + a.own.splits) * a.q.num_rows * a.q.heads;
  a.part_o = c.take<float>(n * a.c.head_dim);
  a.part_ml = c.take<float2>(n);
  return c.bytes();
}

template <class T, int DP, int RT>
int launch_part(const AttendArgs& a, const Part& p, bool is_own, hipStream_t s) {
  const int pages = p.split_keys / a.c.page_size + 2;
  const size_t bytes = sizeof(int) * ((pages + 3) & ~3) + sizeof(float) * (kWaves * 16 * (DP + 4) + 2 * kWaves * 16);
  const unsigned grid = static_cast<unsigned>(a.q.num_rows / p.r * a.c.kv_heads * p.tiles * p.splits);
  if (bytes > 65536)
    GS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&k_cache_attend<T, DP, RT>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)));
  {
    GS_TIMED("k_cache_attend", s);
    k_cache_attend<T, DP, RT><<<grid, 64 * kWaves, bytes, s>>>(a, p, is_own);
  }
  GS_LAUNCHED();
  return GNNSHAP_OK;
}

template <class T, int DP>
int launch_all(const AttendArgs& a, hipStream_t s) {
  for (int i = 0; i < 2; ++i) {
    const Part& p = i ? a.own : a.shared;
    if (!p.table) continue;
    const int tiles = tile_of(static_cast<int64_t>(p.r) * a.share, a.c.head_dim);
    int st = GNNSHAP_OK;
    if constexpr (DP <= 64)
      if (tiles == 4) st = launch_part<T, DP, 4>(a, p, i, s);
    if constexpr (DP <= 128)
      if (tiles == 2) st = launch_part<T, DP, 2>(a, p, i, s);
    if (tiles == 1) st = launch_part<T, DP, 1>(a, p, i, s);
    if (st) return st;
  }
  if (!a.direct || (!a.shared.table && !a.own.table)) {
    GS_TIMED("k_cache_attend_join", s);
    k_cache_attend_join<T><<<static_cast<unsigned>(gnnshap::ceil_div(a.q.num_rows * a.q.heads, 4)), 256, 0, s>>>(a);
    GS_LAUNCHED();
  }
  return GNNSHAP_OK;
}

}  // namespace

extern "C" int gnnshap_cache_attend_workspace(const gnnshap_cache* cache, const gnnshap_queries* q, size_t* bytes) {
  GS_TRY_BEGIN
  gnnshap::clear_error();
  if (!bytes) return gnnshap::fail(GNNSHAP_EINVAL, "bytes is NULL");
  if (const int st = check_queries(cache, q)) return st;
  AttendArgs a{};
  if (const int st = lay_out(a, cache, q)) return st;
  *bytes = carve(a, nullptr);
  return GNNSHAP_OK;
  GS_TRY_END
}

extern "C" int gnnshap_cache_attend(const gnnshap_cache* cache, const gnnshap_queries* q, int32_t* info, void* ws,
                                    size_t ws_bytes, void* stream) {
  using gnnshap::fail;
  GS_TRY_BEGIN
  gnnshap::clear_error();
  if (const int st = check_queries(cache, q)) return st;
  if (q->num_rows == 0) return GNNSHAP_OK;
  if (!q->q || !q->out) return fail(GNNSHAP_EINVAL, "NULL q or out");
  AttendArgs a{};
  if (const int st = lay_out(a, cache, q)) return st;
  a.info = info;
  const size_t need = carve(a, ws);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(GNNSHAP_ECAPACITY, "cache_attend workspace needs %zu bytes, has %zu", need, ws ? ws_bytes : 0);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return gnnshap::with_dtype(cache->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    switch (padded_dim(cache->head_dim)) {
      case 64: return launch_all<T, 64>(a, s);
      case 128: return launch_all<T, 128>(a, s);
      default: return launch_all<T, 256>(a, s);
    }
  });
  GS_TRY_END
}
