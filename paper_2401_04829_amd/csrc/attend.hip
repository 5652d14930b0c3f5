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
// comes out non-finite, the queries beside it are done again by a slow path
// that skips the positions each row does not see.
#include "attend.h"

namespace {

using namespace gnnshap;

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

// One query tile's state: running maximum, sum (this lane's part) and O^T.
template <class T, int DP>
struct State {
  using O = Ops<T, DP>;
  float m = -INFINITY, l = 0.f;
  f4_t o[O::kGroups][O::kOwn];
  __device__ __forceinline__ State() {
#pragma unroll
    for (int i = 0; i < O::kGroups; ++i)
#pragma unroll
      for (int e = 0; e < O::kOwn; ++e) o[i][e] = f4_t{0.f, 0.f, 0.f, 0.f};
  }
  // 32 keys, of which the lane's query sees those whose bit is set.
  __device__ __forceinline__ void step(const typename O::Row (&key)[2], const typename O::Values& val,
                                       const typename O::Row& q, uint32_t bits, float scale2) {
    bits >>= 4 * ((threadIdx.x >> 4) & 3);
    float s[8], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f4_t c = O::scores(key[i], q);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[4 * i + e] = bits >> (16 * i + e) & 1u ? c[e] * scale2 : -INFINITY;
        top = fmaxf(top, s[4 * i + e]);
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    top = fmaxf(top - kUp<T>, m);
    const float use = top == -INFINITY ? 0.f : top, down = __builtin_amdgcn_exp2f(m - use);
    m = top;
    l *= down;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[j] = __builtin_amdgcn_exp2f(s[j] - use);
      l += s[j];
    }
#pragma unroll
    for (int i = 0; i < O::kGroups; ++i)
#pragma unroll
      for (int e = 0; e < O::kOwn; ++e) o[i][e] *= down;
    O::add(o, val, s);
  }
};

// A wavefront: RT tiles of 16 queries of one kv head over its splits of the
// keys, 32 at a time, the next ones on their way while these are multiplied
// (where the registers hold both).  A wavefront of its own per split and kv
// head, because a split's keys are read once whatever its queries are, and
// wavefronts that do not wait for each other keep more loads in flight.  Bound
// by memory where the keys are many: 64 rows of 2,000 tokens, 32 fp16 heads
// over 8 of 128: 112 us, 4.7 TB/s, of 8,000 431 us, 4.9 TB/s (a large copy: 4.7);
// 64 rows of 1 to 20,000 tokens (530 MB): 139 us, 3.8 TB/s; in fp32 318 us, 3.3
// TB/s (heads of 128 leave registers for one wavefront per SIMD there).  One row
// of 4,000 waits for dependent loads (length, page, key): 9.6 us for 16 MB.  In
// fp32, 2,000 rows x 8 heads of 64 over 59 shared keys and up to 3 own: 21 us.
// (Calls in a row; with other work between, which takes the caches, 158 us for
// the unlike rows and 31 us for the last.)
template <class T, int DP, int RT, bool IS_OWN>
__global__ __launch_bounds__(64 * kWaves, DP * sizeof(T) <= 256 && RT == 1 ? 2 : 1) void k_cache_attend(AttendArgs a,
                                                                                                     Part part,
                                                                                                     unsigned places) {
  using O = Ops<T, DP>;
  constexpr int kQueries = 16 * RT;
  constexpr bool kPrefetch = DP * sizeof(T) <= 256;
  extern __shared__ int lds[];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int D = a.c.head_dim, n_queries = part.r * a.share;
  const unsigned number = blockIdx.x * kWaves + wave;
  if (number >= places) return;
  Place at = place_of(a, part, number);
  const int len = length_of(a, part, at.group);
  if (at.k0 >= len && !a.direct && !at.with_own) return;
  int* const pages = lds + wave * (part.split_keys / a.c.page_size + 2);
  at.first = -a.q.first_player;
  if (IS_OWN && a.shared.table) at.first += length_of(a, a.shared, at.group / a.shared.r);

  typename O::Row q[RT];
  int64_t row[RT];
  State<T, DP> st[RT];
  const int q0 = at.tile * kQueries;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int qi = q0 + t * 16 + r, qs = qi < n_queries ? qi : 0;
    row[t] = at.group * part.r + qs / a.share;
    const int head = at.kv_head * a.share + qs % a.share;
    q[t].load(static_cast<const T*>(a.q.q) + row[t] * a.q.q_row_stride + head * a.q.q_head_stride, D);
  }

  const int64_t head_at = static_cast<int64_t>(at.kv_head) * a.c.head_stride;
  const T* const kbase = static_cast<const T*>(a.c.k);
  const T* const vbase = static_cast<const T*>(a.c.v);
  struct Chunk {
    typename O::Row key[2];
    typename O::Values val;
  };
  Chunk now;
#pragma unroll 1
  for (int from = at.k0; from < len; from += part.splits * part.split_keys) {
    const int upto = min(from + part.split_keys, len), page0 = from / a.c.page_size;
    const int n = (upto - 1) / a.c.page_size - page0 + 1;
    for (int i = lane; i < n; i += 64) {
      int p = part.table[at.group * part.width + page0 + i];
      if (p < 0 || p >= a.c.num_pages) {
        if (a.info) *a.info = 1;
        p = 0;
      }
      pages[i] = p;
    }
    __builtin_amdgcn_wave_barrier();
    const auto offset = [&](int key) {
      key = key < upto ? key : upto - 1;
      int slot;
      const int pg = page_of(a, key, slot);
      return pages[pg - page0] * a.c.page_stride + slot * a.c.slot_stride + head_at;
    };
    const auto load = [&](Chunk& c, int k) {
#pragma unroll
      for (int i = 0; i < 2; ++i) c.key[i].load(kbase + offset(k + 16 * i + r), D);
#pragma unroll
      for (int j = 0; j < 8; ++j) c.val.load(j, vbase + offset(k + 16 * (j >> 2) + 4 * g + (j & 3)), D);
    };
    const auto add = [&](const Chunk& c, int k) {
      const uint32_t there = upto - k >= 32 ? ~0u : (1u << (upto - k)) - 1u;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        uint32_t bits = there;
        if (a.q.num_players > 0) bits &= seen(a.q.masks + row[t] * a.q.mask_words, at.first + k, a.q.num_players);
        st[t].step(c.key, c.val, q[t], bits, a.scale2);
      }
    };
    if constexpr (kPrefetch) {
      Chunk next;
      load(now, from);
#pragma unroll 1
      for (int k = from; k < upto; k += 2 * kChunk) {
        if (k + kChunk < upto) load(next, k + kChunk);
        add(now, k);
        if (k + 2 * kChunk < upto) load(now, k + 2 * kChunk);
        if (k + kChunk < upto) add(next, k + kChunk);
      }
    } else {
#pragma unroll 1
      for (int k = from; k < upto; k += kChunk) {
        load(now, k);
        add(now, k);
      }
    }
  }

  if (!IS_OWN && at.with_own) {
    const int64_t first = len - a.q.first_player;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int own_len = length_of(a, a.own, row[t]);
      const OwnTile own(a, part, at, q0 + t * 16, 16);
      const int passes = own.passes(own_len);
      for (int p = 0; p < passes; ++p) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int64_t x = own.at(a, p, 16 * i + r, at.kv_head);
          now.key[i].load(kbase + (x < 0 ? 0 : x), x < 0 ? 0 : D);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int64_t x = own.at(a, p, 16 * (j >> 2) + 4 * g + (j & 3), at.kv_head);
          now.val.load(j, vbase + (x < 0 ? 0 : x), x < 0 ? 0 : D);
        }
        st[t].step(now.key, now.val, q[t], own.bits(a, p, row[t], own_len, first), a.scale2);
      }
    }
  }

  bool bad = false;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float l = st[t].l;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const int qi = q0 + t * 16 + r;
    if (qi >= n_queries) continue;
    const int head = at.kv_head * a.share + qi % a.share;
    const int64_t p = part_index(a, part.slot0 + at.split, row[t], head);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bad |= !isfinite(l);
#pragma unroll
    for (int i = 0; i < O::kGroups; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int d = (16 * i + 4 * g + x) * O::kOwn;
        if (d >= D) continue;
        Pack<T, O::kOwn> done;
        Pack<float, O::kOwn> part_done;
#pragma unroll
        for (int e = 0; e < O::kOwn; ++e) {
          bad |= !isfinite(st[t].o[i][e][x]);
          done.v[e] = static_cast<T>(st[t].o[i][e][x] * inv);
          part_done.v[e] = st[t].o[i][e][x];
        }
        if (a.direct)
          store_pack(out_of<T>(a, row[t], head) + d, done);
        else
          store_pack(a.part_o + p * D + d, part_done);
      }
    if (g == 0) {
      if (!a.direct)
        a.part_ml[p] = make_float2(st[t].m, l);
      else if (a.q.lse)
        a.q.lse[row[t] * a.q.heads + head] = lse_of<T>(st[t].m, l);
    }
  }
  if (__ballot(bad)) attend_slowly<T>(a, part, at, q0, kQueries);
}

// Joins the parts of each query, a wavefront per row and head, or the four of a
// workgroup where there may be many parts: the lanes weigh 64 parts at a time,
// then add up the parts' elements, eight loads in flight.  Four wavefronts
// from 9 parts on: one row of 4,000 tokens in 63 parts 6 us (4 us less than with
// one wavefront each).
template <class T, int PER_QUERY>
__global__ __launch_bounds__(64 * kWaves) void k_cache_attend_join(AttendArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.c.head_dim;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * (kWaves / PER_QUERY) + wave / PER_QUERY;
  if (i >= a.q.num_rows * a.q.heads) return;
  const int64_t row = i / a.q.heads;
  const int head = static_cast<int>(i % a.q.heads);
  // the splits that have keys
  const auto splits_of = [&](const Part& part, int64_t seq) {
    return min(part.splits, (length_of(a, part, seq) + part.split_keys - 1) / part.split_keys);
  };
  int ns = 0, no = 0;
  if (a.shared.table) ns = splits_of(a.shared, row / a.shared.r);
  if (a.fused) ns = max(ns, 1);
  if (a.own.table && !a.fused) no = splits_of(a.own, row);
  const auto slot_of = [&](int n) { return n < ns ? a.shared.slot0 + n : a.own.slot0 + n - ns; };
  const int d = 4 * lane < D ? 4 * lane : 0;
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  // this wavefront's parts: wave % PER_QUERY, then PER_QUERY further
  const int first = wave % PER_QUERY, count = (ns + no - first + PER_QUERY - 1) / PER_QUERY;
  for (int n0 = 0; n0 < count; n0 += 64) {
    const int n = min(64, count - n0);
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < n) ml = a.part_ml[part_index(a, slot_of(first + (n0 + lane) * PER_QUERY), row, head)];
    float top = fmaxf(m, ml.x);
#pragma unroll
    for (int off = 1; off < 64; off *= 2) top = fmaxf(top, __shfl_xor(top, off));
    const float use = top == -INFINITY ? 0.f : top, down = __builtin_amdgcn_exp2f(m - use);
    const float up = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - use);
    float sum = ml.y == 0.f ? 0.f : ml.y * up;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) sum += __shfl_xor(sum, off);
    m = top;
    l = l * down + sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= down;
    // all lanes take part, so that every lane's weight is there to be read
    for (int j0 = 0; j0 < n; j0 += 8) {
      Pack<float, 4> x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        x[j] = load_pack<float, 4>(
            a.part_o + part_index(a, slot_of(first + (n0 + min(j0 + j, n - 1)) * PER_QUERY), row, head) * D + d);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w = j0 + j < n ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(up), j0 + j)) : 0.f;
        if (w != 0.f)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += x[j].v[e] * w;
      }
    }
  }
  if constexpr (PER_QUERY > 1) {
    __shared__ float parts[PER_QUERY][64 * 4], stats[PER_QUERY][2];
#pragma unroll
    for (int e = 0; e < 4; ++e) parts[wave][4 * lane + e] = o[e];
    if (lane == 0) {
      stats[wave][0] = m;
      stats[wave][1] = l;
    }
    __syncthreads();
    if (wave > 0) return;
    float top = -INFINITY;
    for (int w = 0; w < PER_QUERY; ++w) top = fmaxf(top, stats[w][0]);
    const float use = top == -INFINITY ? 0.f : top;
    m = top;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = 0.f;
    for (int w = 0; w < PER_QUERY; ++w) {
      if (stats[w][1] == 0.f) continue;
      const float up = __builtin_amdgcn_exp2f(stats[w][0] - use);
      l += stats[w][1] * up;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += parts[w][4 * lane + e] * up;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (4 * lane < D) {
    Pack<T, 4> done;
#pragma unroll
    for (int e = 0; e < 4; ++e) done.v[e] = static_cast<T>(o[e] * inv);
    store_pack(out_of<T>(a, row, head) + 4 * lane, done);
  }
  if (lane == 0 && a.q.lse) a.q.lse[row * a.q.heads + head] = lse_of<T>(m, l);
}

// The scale of scores in powers of two.
float scale2_of(const gnnshap_queries& q) { return static_cast<float>(q.scale * 1.4426950408889634074); }

int check_queries(const gnnshap_cache* c, const gnnshap_queries* q) {
  using gnnshap::fail;
  if (const int st = gnnshap::check_cache(c)) return st;
  if (!q || q->num_rows < 0) return fail(GNNSHAP_EINVAL, "queries: NULL or a negative number of rows");
  if (q->heads < 1 || q->heads % c->kv_heads != 0)
    return fail(GNNSHAP_EINVAL, "%d query heads over %d kv heads", static_cast<int>(q->heads),
                static_cast<int>(c->kv_heads));
  if (!(q->scale != 0.0) || !std::isfinite(scale2_of(*q)))
    return fail(GNNSHAP_EINVAL, "scale %g is 0 or not finite in fp32", q->scale);
  if (q->num_rows > INT32_MAX || q->num_rows * q->heads > INT32_MAX)
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
    if (p.longest > (int64_t(1) << 30))
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

// Whether results come from the join (also where there is no context), and its
// workgroups: one for each query's parts, or for kWaves queries'.
bool joined(const AttendArgs& a) { return !a.direct || (!a.shared.table && !a.own.table); }
bool many_parts(const AttendArgs& a) { return a.shared.splits + a.own.splits > 8; }
int64_t join_workgroups(const AttendArgs& a) {
  return gnnshap::ceil_div(a.q.num_rows * a.q.heads, many_parts(a) ? 1 : kWaves);
}

// How the work is laid out over workgroups.
int lay_out(AttendArgs& a, const gnnshap_cache* c, const gnnshap_queries* q) {
  using gnnshap::ceil_div;
  a.c = *c;
  a.q = *q;
  a.share = q->heads / c->kv_heads;
  a.scale2 = scale2_of(*q);
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
    if (i && a.fused) continue;
    const int64_t queries = static_cast<int64_t>(p.r) * a.share;
    if (queries > INT32_MAX - 1024)
      return gnnshap::fail(GNNSHAP_EUNSUPPORTED, "%lld queries of a group", static_cast<long long>(queries));
    // The wide kernel leaves part of its 128 queries empty where there are
    // fewer, and is still ahead from 32 on; where heads are wider than 128,
    // from 128 (bf16, 4,000 shared keys: 32 queries 22 us against 34, 128
    // queries 28 against 37; 512 keys and 16 queries 20.4 against 18.2; heads of
    // 256: 64 queries 35 against 25, 128 queries 38.4 against 38.3).
    p.wide = !i && queries >= (c->head_dim <= 128 ? 32 : 128) && c->dtype != GNNSHAP_F32;
    // Tiles of 16 queries that a wavefront takes: two for heads of 65 to 128
    // elements where there are wavefronts enough (64 heads over one, bf16: 512
    // rows of 1,000 keys 146 us with two against 157 with one, one row of 4,000
    // 16.8 against 14.2; 10,000 rows x 8 heads over 4 on 1,000 shared keys in
    // fp32 736 against 925, x 4 heads over 4 380 against 467, but with heads of 64
    // elements 226 against 166 at 2,000 rows).
    const bool two = padded_dim(c->head_dim) == 128 && queries > 16 &&
                     q->num_rows / p.r * c->kv_heads * ceil_div(queries, 32) *
                             ceil_div(std::max(p.max_len, 1), 256) >= 2048;
    // Own parts of few tokens ride along with the shared part: a wavefront
    // takes its rows' tokens 32 at a time, one such pass after the other at
    // about 3 us, where a launch for them costs about 4 us and their parts,
    // written and joined, about 1 us for each 1,200 heads (bf16, 32 heads over
    // 8, 512 shared keys, own tokens with the shared part against apart: 32
    // rows with 4 each 21.6 us against 25.5, with 16 30.1 against 25.5; 1,000
    // rows with 16 67 against 88, with 64 134 against 126).
    if (!i && q->table && q->max_length <= 64) {
      const int64_t rows = ceil_div(p.wide ? 32 : 16, a.share);
      const int64_t passes = ceil_div(q->max_length, std::max<int64_t>(kChunk / rows, 1));
      a.fused = 3 * passes <= 4 + q->num_rows * q->heads / 1200;
    }
    p.tile = p.wide ? 128 : two ? 32 : 16;
    p.tiles = static_cast<int>(ceil_div(queries, p.tile));
    // Splits.  The wide kernel: as many as give the chip two workgroups per
    // compute unit, of 256 keys at least.  The other: splits of 256 keys, 128
    // where there are few, and 64 where there are fewer still and the join has
    // not too many parts (bf16, 32 heads over 8 of 128 elements, 64 against
    // 128: one row of 500 keys 11.3 us against 14.6, of 4,000 13.2 against
    // 15.5, of 16,000 26.8 against 22.9; 8 rows of 1,000 14.6 against 16.5).
    // Up to 32 times the wavefronts that the chip holds, which come back for
    // further splits where the keys are more.  So many, because the lengths may
    // be unlike: a wavefront without keys ends at once, and one with many would
    // end last (64 rows of 1 to 20,000 tokens: 146 us; with 8,192 wavefronts
    // 192 us).
    const int64_t base = q->num_rows / p.r * c->kv_heads * p.tiles;
    const auto at_most = [&](int64_t n) { return std::max<int64_t>(1, n / std::max<int64_t>(base, 1)); };
    const int64_t longest = std::max(p.max_len, 1);
    if (p.wide) {
      p.split_keys = static_cast<int>(
          std::min<int64_t>(std::max<int64_t>(ceil_div(ceil_div(longest, at_most(512)), 128) * 128, 256), INT32_MAX / 2));
      p.splits = static_cast<int>(ceil_div(longest, p.split_keys));
    } else {
      p.split_keys = ceil_div(longest, 128) * base < 1024 && longest <= 8192 ? 64
                     : ceil_div(longest, 256) * base < 4096                  ? 128
                                                                             : 256;
      p.splits = static_cast<int>(std::min(ceil_div(longest, p.split_keys), at_most(65536)));
    }
    // a workgroup of the wide kernel per place, of the other one per kWaves
    if (const int st = check_launch(p.wide ? base * p.splits : ceil_div(base * p.splits, kWaves), 64 * kWaves)) return st;
    p.slot0 = slots;
    slots += p.splits;
  }
  a.direct = slots <= 1;
  return joined(a) ? check_launch(join_workgroups(a), 64 * kWaves) : GNNSHAP_OK;
}

size_t carve(AttendArgs& a, void* ws) {
  if (a.direct) return 0;
  gnnshap::Carver c(ws);
  const size_t n = static_cast<size_t>(a.shared.splits + a.own.splits) * a.q.num_rows * a.q.heads;
  a.part_o = c.take<float>(n * a.c.head_dim);
  a.part_ml = c.take<float2>(n);
  return c.bytes();
}

template <class T, int DP, int RT, bool IS_OWN>
int launch_part(const AttendArgs& a, const Part& p, hipStream_t s) {
  const int64_t places = a.q.num_rows / p.r * a.c.kv_heads * p.tiles * p.splits;
  const size_t bytes = sizeof(int) * kWaves * (p.split_keys / a.c.page_size + 2);
  {
    GS_TIMED("k_cache_attend", s);
    k_cache_attend<T, DP, RT, IS_OWN><<<static_cast<unsigned>(ceil_div(places, kWaves)), 64 * kWaves, bytes, s>>>(
        a, p, static_cast<unsigned>(places));
  }
  GS_LAUNCHED();
  return GNNSHAP_OK;
}

template <class T, int DP, bool IS_OWN>
int launch_tiles(const AttendArgs& a, const Part& p, hipStream_t s) {
  if constexpr (DP == 128)
    if (p.tile == 32) return launch_part<T, DP, 2, IS_OWN>(a, p, s);
  return launch_part<T, DP, 1, IS_OWN>(a, p, s);
}

template <class T, int DP>
int launch_all(const AttendArgs& a, hipStream_t s) {
  int st = GNNSHAP_OK;
  if (a.shared.table) st = a.shared.wide ? launch_attend_wide(a, s) : launch_tiles<T, DP, false>(a, a.shared, s);
  if (!st && a.own.table && !a.fused) st = launch_tiles<T, DP, true>(a, a.own, s);
  if (st) return st;
  if (joined(a)) {
    GS_TIMED("k_cache_attend_join", s);
    const unsigned grid = static_cast<unsigned>(join_workgroups(a));
    if (many_parts(a))
      k_cache_attend_join<T, kWaves><<<grid, 64 * kWaves, 0, s>>>(a);
    else
      k_cache_attend_join<T, 1><<<grid, 64 * kWaves, 0, s>>>(a);
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
  if (q->q == q->out) return fail(GNNSHAP_EINVAL, "out is q: a query may be read again after its output is written");
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
