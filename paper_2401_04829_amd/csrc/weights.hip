// What attention's queries looked at: each cached token's weight, summed over
// rows and heads.
//
// With a row's lse known, a weight is e^{scale q.k - lse} by itself: no maximum
// runs along, nothing is scaled again, values are not read.  A wavefront keeps 32
// keys of a kv head in registers as the left operand of the matrix
// instructions and takes the queries 16 at a time; the weights that come out (query in
// the lane's column, keys in its registers) are added up in the lane, and over
// the 16 columns at the end.
//
// Few queries (a new token of each sequence) are bound by reading the keys
// once, or by the call; the kv heads' sums meet in LDS.  Many (coalitions, a
// prompt's rows) are bound by the vector instructions of a weight (the
// exponential, its argument, the mask, the sum: 10 per query and key) and the
// matrix instructions beside them; their range is split so that the chip is
// full, and a second launch adds up the parts in order.  bf16, 32 heads over 8 of
// 128: 10,000 coalitions on 417 tokens 88 us and 5 to join (queries three tiles
// ahead instead of two: 91); one row on 4,000 tokens 7 us.
#include "attend.h"

namespace {

using namespace gnnshap;

constexpr float kLog2eF = 1.4426950408889634f;

struct WeightsArgs {
  gnnshap_cache c;
  gnnshap_observed o;
  int share, page_shift;
  int64_t queries;   // of a sequence and kv head
  float scale2;      // scale log2 e
  int splits;        // of the queries; 0: the kernel of few
  int64_t split;     // tiles of 16 queries of a split
  float* part;       // [sequence][kv head][split][max_length]
  int32_t* info;
};

// 16 keys or queries, this lane's quarter of their elements.  Behind the head's
// D elements keys are 0 and queries others of their own, so that loading them
// takes no branch, behind which the compiler would wait for all loads.
template <class T, int DP>
struct Vectors {
  static constexpr int kVec = 16 / sizeof(T), kSteps = DP / (4 * kVec);
  u4_t s[kSteps];
  __device__ __forceinline__ void load(const T* p, int D, bool keys) {
    const int g = (threadIdx.x >> 4) & 3;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int d = (4 * i + g) * kVec;
      __builtin_memcpy(&s[i], p + (d < D ? d : 0), 16);
      if (keys && d >= D) s[i] = u4_t{0u, 0u, 0u, 0u};
    }
  }
  typedef T vec8 __attribute__((ext_vector_type(8)));
  // c[n] = products of the N tiles of keys with the queries: steps outside, so that
  // an instruction does not wait for the one before it.
  template <int N>
  static __device__ __forceinline__ void products(const Vectors (&k)[N], const Vectors& q, f4_t (&c)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) c[n] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if constexpr (std::is_same_v<T, float>) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int n = 0; n < N; ++n)
            c[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[n].s[i][e]), __uint_as_float(q.s[i][e]), c[n], 0, 0, 0);
      } else {
#pragma unroll
        for (int n = 0; n < N; ++n) c[n] = mfma(k[n].s[i], q.s[i], c[n]);
      }
    }
  }
  static __device__ __forceinline__ f4_t mfma(u4_t a, u4_t b, f4_t c) {
    if constexpr (std::is_same_v<T, bf16_t>)
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(vec8, a), __builtin_bit_cast(vec8, b), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec8, a), __builtin_bit_cast(vec8, b), c, 0, 0, 0);
  }
};

// A wavefront's 16 NK keys, NK 2 or 4: where they are, and their part of the sums.
template <class T, int DP, int NK>
struct KeyTile {
  using V = Vectors<T, DP>;
  int64_t where;            // lane i: of key i
  uint64_t lost;            // keys whose page is out of range
  V key[NK];
  float sum[4 * NK];        // of keys 16 (i / 4) + 4 g + i % 4, this lane's queries

  __device__ __forceinline__ void find(const WeightsArgs& a, int64_t seq, int64_t k0) {
    const int64_t k = k0 + (threadIdx.x & (16 * NK - 1));
    int slot = 0, page = -1;
    if (k < a.o.max_length) {
      int pg;
      if (a.page_shift >= 0) {
        pg = static_cast<int>(k >> a.page_shift);
        slot = static_cast<int>(k) & ((1 << a.page_shift) - 1);
      } else {
        pg = static_cast<int>(k) / a.c.page_size;
        slot = static_cast<int>(k) - pg * a.c.page_size;
      }
      page = a.o.table[seq * a.o.table_width + pg];
    }
    const bool bad = page < 0 || page >= a.c.num_pages;
    lost = __ballot(bad);
    where = bad ? 0 : page * a.c.page_stride + slot * a.c.slot_stride;
#pragma unroll
    for (int i = 0; i < 4 * NK; ++i) sum[i] = 0.f;
  }
  __device__ __forceinline__ void load(const WeightsArgs& a, int kv_head) {
    const T* const k = static_cast<const T*>(a.c.k) + kv_head * a.c.head_stride;
#pragma unroll
    for (int i = 0; i < NK; ++i) key[i].load(k + __shfl(where, 16 * i + (threadIdx.x & 15)), a.c.head_dim, true);
  }
};

// Which of a wavefront's keys are players, and where their bits lie in a row's mask: the same for all rows.
template <int NK>
struct Players {
  uint32_t always[NK / 2];   // no players: seen by every row
  int at[NK / 2 + 1], shift;   // 32-bit words of a row, the first key's bit in the first
  __device__ __forceinline__ Players(const WeightsArgs& a, int64_t k0) {
    const bool any = a.o.num_players > 0;
    const int64_t first = k0 - a.o.first_player;   // the first key among the players
    const int words = any ? static_cast<int>((a.o.num_players + 31) >> 5) : 1;
    shift = static_cast<int>(first & 31);
#pragma unroll
    for (int w = 0; w <= NK / 2; ++w) {
      const int64_t word = (first >> 5) + w;
      at[w] = static_cast<int>(word < 0 ? 0 : word < words ? word : words - 1);
    }
#pragma unroll
    for (int w = 0; w < NK / 2; ++w) {
      const int64_t p = first + 32 * w;
      always[w] = 0u;
      if (p < 0) always[w] |= p <= -32 ? ~0u : (1u << -p) - 1u;
      if (p + 32 > a.o.num_players) always[w] |= p >= a.o.num_players ? ~0u : ~0u << (a.o.num_players - p);
    }
  }
};

// Where a sequence's queries of a kv head lie, and what goes with its rows;
// offsets from there are of type I, in bytes: 32 bits spare the kernel of many a
// quarter of its instructions.
template <class I>
struct Rows {
  const char *q, *lse, *len, *masks;
  I q_row, q_head, lse_row, mask_row;
  __device__ __forceinline__ Rows(const WeightsArgs& a, int64_t seq, int kv_head, int element) {
    const int64_t row = seq * a.o.rows_per_seq, head = static_cast<int64_t>(kv_head) * a.share;
    const bool any = a.o.num_players > 0;   // without players words are read that do not matter
    q = static_cast<const char*>(a.o.q) + (row * a.o.q_row_stride + head * a.o.q_head_stride) * element;
    lse = reinterpret_cast<const char*>(a.o.lse + row * a.o.heads + head);
    len = reinterpret_cast<const char*>(a.o.lengths + row);
    masks = any ? reinterpret_cast<const char*>(a.o.masks + row * a.o.mask_words) : lse;
    q_row = static_cast<I>(a.o.q_row_stride * element);
    q_head = static_cast<I>(a.o.q_head_stride * element);
    lse_row = static_cast<I>(a.o.heads) * 4;
    mask_row = any ? static_cast<I>(a.o.mask_words) * 8 : 0;
  }
};

// 16 queries of a sequence and kv head, this lane's among them: row `row` of the
// sequence, query head `of` of the kv head.  load() only asks memory, so that the
// next queries can be on their way while these are multiplied.
template <class T, int DP, int NK>
struct QueryTile {
  Vectors<T, DP> q;
  float lse;
  int len;
  uint32_t word[NK / 2 + 1];
  bool in;
  template <class I>
  __device__ __forceinline__ void load(const WeightsArgs& a, const Players<NK>& p, const Rows<I>& rows, int row, int of,
                                       bool there) {
    in = there;
    const I b = in ? row : 0, h = in ? of : 0;
    q.load(reinterpret_cast<const T*>(rows.q + (b * rows.q_row + h * rows.q_head)), a.c.head_dim, false);
    lse = *reinterpret_cast<const float*>(rows.lse + (b * rows.lse_row + h * 4));
    len = *reinterpret_cast<const int*>(rows.len + b * 4);
    const I m = b * rows.mask_row;
#pragma unroll
    for (int w = 0; w <= NK / 2; ++w)
      word[w] = *reinterpret_cast<const uint32_t*>(rows.masks + (m + static_cast<I>(4 * p.at[w])));
  }
  // The keys that the lane's query sees, of those from 32 w on.
  __device__ __forceinline__ uint32_t sees(const WeightsArgs& a, const Players<NK>& p, int64_t k0, int w, bool& bad) const {
    const int most = static_cast<int>(a.o.max_length), n = min(max(len, 0), most);
    bad |= n != len;
    const int left = min(n - static_cast<int>(k0) - 32 * w, 32);
    const uint32_t there = !in || lse == -INFINITY || left <= 0 ? 0u : ~0u >> (32 - left);
    return there & (__builtin_amdgcn_alignbit(word[w + 1], word[w], p.shift) | p.always[w]);
  }
};

// With n the whole number next to lse log2 e, a weight is 2^(s log2 e - n) times
// f = e^(n ln 2 - lse): one multiplication and addition makes the exponent, whose
// rounding is that of the score, and f, which is the row's, rides on the sum.  f's
// argument is reduced by ln 2 in two parts (the method of Cody and Waite): the
// first has 15 bits, so that n times it less lse is exact up to n = 2^9 and rounded
// once beyond (fused), the second is what is left of ln 2.  n itself has 24 bits:
// below 2^30 it is 65 off at most and f finite, so that what a row does not see, 0
// times f, adds nothing; from there on lse has no bits to make up for, and f is 1.
template <class T, int DP, int NK>
__device__ __forceinline__ void add(const WeightsArgs& a, const Players<NK>& p, KeyTile<T, DP, NK>& t,
                                    const QueryTile<T, DP, NK>& q, int64_t k0, bool& bad) {
  constexpr float kLn2High = 0.693145752f, kLn2Low = 1.42860677e-6f;   // their sum is ln 2
  const float n = rintf(q.lse * kLog2eF);
  float f = __builtin_amdgcn_exp2f(fmaf(n, kLn2Low, fmaf(n, kLn2High, -q.lse)) * kLog2eF);
  f = fabsf(n) < 0x1p30f ? f : 1.f;
  uint32_t bits[NK / 2], any = 0u;
#pragma unroll
  for (int w = 0; w < NK / 2; ++w) {
    const uint32_t lost = static_cast<uint32_t>(t.lost >> (32 * w)), all = q.sees(a, p, k0, w, bad);
    bad |= (all & lost) != 0u;
    bits[w] = (all & ~lost) >> (4 * ((threadIdx.x >> 4) & 3));
    any |= bits[w];
  }
  if (!__ballot(any)) return;
  f4_t c[NK];
  Vectors<T, DP>::products(t.key, q.q, c);
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // what is not seen may be NaN: its bits are cleared
      const float x = __builtin_amdgcn_exp2f(fmaf(c[i][e], a.scale2, -n));
      const uint32_t seen_too = static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(bits[i / 2]), 16 * (i % 2) + e, 1));
      t.sum[4 * i + e] = fmaf(__uint_as_float(__float_as_uint(x) & seen_too), f, t.sum[4 * i + e]);
    }
}

// Adds up the 16 columns; all lanes get the sums of their keys.
template <int N>
__device__ __forceinline__ void columns(float (&sum)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int off = 1; off < 16; off *= 2) sum[i] += __shfl_xor(sum[i], off);
}

// Few queries: a workgroup's wavefronts share 32 keys, each with its kv heads
// (or, where there are fewer kv heads, have 32 keys of their own).
template <class T, int DP>
__global__ __launch_bounds__(256) void k_cache_weights(WeightsArgs a, int by_heads, unsigned tiles) {
  __shared__ float sums[4][32];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int64_t seq = blockIdx.x / tiles;
  const int own = wave % by_heads, tile = wave / by_heads;   // wavefront of the keys, which keys
  const int64_t k0 = (static_cast<int64_t>(blockIdx.x % tiles) * (4 / by_heads) + tile) * 32;
  KeyTile<T, DP, 2> t;
  t.find(a, seq, k0);
  const Players<2> players(a, k0);
  bool bad = false;
  // a wavefront whose keys no row sees has nothing to read
  bool any = false;
  for (int64_t b = lane; b < a.o.rows_per_seq; b += 64) {
    const int len = a.o.lengths[seq * a.o.rows_per_seq + b];
    any |= len > k0;
    bad |= len < 0;
  }
  if (__ballot(any)) {
    for (int h = own; h < a.c.kv_heads; h += by_heads) {
      t.load(a, h);
      const Rows<int64_t> rows(a, seq, h, sizeof(T));
      for (int q0 = 0; q0 < a.queries; q0 += 16) {
        QueryTile<T, DP, 2> q;
        const int n = q0 + r, row = n / a.share;
        q.load(a, players, rows, row, n - row * a.share, n < a.queries);
        add(a, players, t, q, k0, bad);
      }
    }
  }
  if (bad && a.info) *a.info = 1;
  columns(t.sum);
  if (r == 0)
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave][16 * (i / 4) + 4 * g + i % 4] = t.sum[i];
  __syncthreads();
  if (own == 0 && lane < 32 && k0 + lane < a.o.max_length) {
    float s = 0.f;
    for (int i = 0; i < by_heads; ++i) s += sums[wave + i][lane];
    float* const w = a.o.weights + seq * a.o.weights_stride + k0 + lane;
    if (s != 0.f) *w += s;
  }
}

// Many queries: each wavefront has 16 NK keys and a split of the queries.  The
// wavefronts that share queries follow each other, the workgroups of an XCD (every
// eighth) too, so that the queries come through one cache.
template <class T, int DP, int NK>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 512 ? 2 : 1) void k_cache_weights_many(WeightsArgs a, unsigned tiles, unsigned places) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const unsigned xcd = blockIdx.x % 8, each = gridDim.x / 8, more = gridDim.x % 8;
  unsigned b = __builtin_amdgcn_readfirstlane((xcd * each + (xcd < more ? xcd : more) + blockIdx.x / 8) * 4 + wave);
  if (b >= places) return;
  const int64_t k0 = static_cast<int64_t>(b % tiles) * (16 * NK);
  b /= tiles;
  const int split = b % a.splits;
  b /= a.splits;
  const int kv_head = b % a.c.kv_heads;
  const int64_t seq = b / a.c.kv_heads;
  KeyTile<T, DP, NK> t;
  t.find(a, seq, k0);
  const int q0 = static_cast<int>(split * a.split * 16);
  const int q1 = static_cast<int>(q0 + a.split * 16 < a.queries ? q0 + a.split * 16 : a.queries);
  if (q0 < q1) {
    t.load(a, kv_head);
    const Players<NK> players(a, k0);
    const Rows<uint32_t> rows(a, seq, kv_head, sizeof(T));
    QueryTile<T, DP, NK> now, next;
    // this lane's query goes on by 16, the rows by 16 / share
    int n = q0 + r, row = n / a.share, of = n - row * a.share;
    const int rows_on = 16 / a.share, heads_on = 16 - rows_on * a.share;
    const auto load = [&](QueryTile<T, DP, NK>& q) {
      q.load(a, players, rows, row, of, n < q1);
      n += 16;
      row += rows_on;
      of += heads_on;
      if (of >= a.share) {
        of -= a.share;
        ++row;
      }
    };
    bool bad = false;
    load(now);
#pragma unroll 1
    for (int q = q0; q < q1; q += 32) {  // (behind the last queries others are loaded that see nothing)
      load(next);
      __builtin_amdgcn_sched_barrier(0);  // asked for before the products, not where they are wanted
      add(a, players, t, now, k0, bad);
      load(now);
      __builtin_amdgcn_sched_barrier(0);
      add(a, players, t, next, k0, bad);
    }
    if (bad && a.info) *a.info = 1;
  }
  columns(t.sum);
  float* const part = a.part + ((seq * a.c.kv_heads + kv_head) * a.splits + split) * a.o.max_length;
  if (r == 0)
#pragma unroll
    for (int i = 0; i < 4 * NK; ++i) {
      const int64_t k = k0 + 16 * (i / 4) + 4 * g + i % 4;
      if (k < a.o.max_length) part[k] = t.sum[i];
    }
}

// Tiles of 16 keys of a wavefront: four where they and two tiles of queries fit
// its registers (10,000 rows x 32 heads of 128 on 417 tokens: 138 us with four, 148
// with two).
constexpr int key_tiles_of(int padded_bytes) { return padded_bytes <= 256 ? 4 : 2; }

// Adds the parts up, a thread per token of a sequence.
__global__ __launch_bounds__(256) void k_cache_weights_join(WeightsArgs a) {
  __shared__ float sums[4][64];
  const int64_t tiles = (a.o.max_length + 63) / 64, seq = blockIdx.x / tiles, k = blockIdx.x % tiles * 64 + (threadIdx.x & 63);
  const int64_t parts = static_cast<int64_t>(a.c.kv_heads) * a.splits;
  const int way = threadIdx.x >> 6;
  float s = 0.f;
  if (k < a.o.max_length) {
    const float* const p = a.part + seq * parts * a.o.max_length + k;
#pragma unroll 8
    for (int64_t i = way; i < parts; i += 4) s += p[i * a.o.max_length];
  }
  sums[way][threadIdx.x & 63] = s;
  __syncthreads();
  if (way > 0 || k >= a.o.max_length) return;
  for (int i = 1; i < 4; ++i) s += sums[i][threadIdx.x];
  if (s != 0.f) a.o.weights[seq * a.o.weights_stride + k] += s;
}

int check_observed(const gnnshap_cache* c, const gnnshap_observed* o) {
  if (const int st = check_cache(c)) return st;
  if (!o || o->num_rows < 0) return fail(GNNSHAP_EINVAL, "observed queries: NULL or a negative number of rows");
  if (o->heads < 1 || o->heads % c->kv_heads != 0)
    return fail(GNNSHAP_EINVAL, "%d query heads over %d kv heads", static_cast<int>(o->heads),
                static_cast<int>(c->kv_heads));
  if (!(o->scale != 0.0) || !std::isfinite(static_cast<float>(o->scale * 1.4426950408889634074)))
    return fail(GNNSHAP_EINVAL, "scale %g is 0 or not finite in fp32", o->scale);
  if (o->num_rows > INT32_MAX || o->num_rows * o->heads > INT32_MAX)
    return fail(GNNSHAP_EUNSUPPORTED, "%lld rows in one call", static_cast<long long>(o->num_rows));
  if (o->rows_per_seq < 1 || o->num_rows % o->rows_per_seq != 0)
    return fail(GNNSHAP_EINVAL, "sequences of %lld of %lld rows", static_cast<long long>(o->rows_per_seq),
                static_cast<long long>(o->num_rows));
  if (o->table_width < 0 || o->max_length < 0) return fail(GNNSHAP_EINVAL, "negative width or length");
  if (o->max_length > (int64_t(1) << 30))
    return fail(GNNSHAP_EUNSUPPORTED, "up to %lld tokens", static_cast<long long>(o->max_length));
  if (ceil_div(o->max_length, c->page_size) > o->table_width)
    return fail(GNNSHAP_EINVAL, "%lld tokens do not fit %lld pages of %d", static_cast<long long>(o->max_length),
                static_cast<long long>(o->table_width), static_cast<int>(c->page_size));
  if (o->num_players < 0 || o->num_players > INT32_MAX || o->first_player < 0 || o->first_player > INT32_MAX)
    return fail(GNNSHAP_EINVAL, "%lld players from position %lld", static_cast<long long>(o->num_players),
                static_cast<long long>(o->first_player));
  if (o->num_players > 0 && (!o->masks || o->mask_words < ceil_div(o->num_players, 64)))
    return fail(GNNSHAP_EINVAL, "%lld players without masks, or with %lld words", static_cast<long long>(o->num_players),
                static_cast<long long>(o->mask_words));
  if (o->weights_stride < 0 || (o->weights_stride < o->max_length && o->num_rows > o->rows_per_seq))
    return fail(GNNSHAP_EINVAL, "the weights' rows, %lld apart, overlap", static_cast<long long>(o->weights_stride));
  return GNNSHAP_OK;
}

int64_t sequences(const WeightsArgs& a) { return a.o.num_rows / a.o.rows_per_seq; }
int64_t key_tiles(const WeightsArgs& a, int keys) { return ceil_div(std::max<int64_t>(a.o.max_length, 1), keys); }

// Keys of a wavefront of the kernel of many.
int keys_of_many(const WeightsArgs& a) {
  const int padded = a.c.head_dim <= 64 ? 64 : a.c.head_dim <= 128 ? 128 : 256;
  return 16 * key_tiles_of(padded * (a.c.dtype == GNNSHAP_F32 ? 4 : 2));
}

int by_heads(const WeightsArgs& a) { return a.c.kv_heads >= 4 ? 4 : a.c.kv_heads >= 2 ? 2 : 1; }

int lay_out(WeightsArgs& a, const gnnshap_cache* c, const gnnshap_observed* o) {
  a.c = *c;
  a.o = *o;
  a.share = o->heads / c->kv_heads;
  a.queries = o->rows_per_seq * a.share;
  a.scale2 = static_cast<float>(o->scale * 1.4426950408889634074);
  a.page_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (c->page_size == 1 << i) a.page_shift = i;
  if (a.queries > INT32_MAX - 1024)
    return fail(GNNSHAP_EUNSUPPORTED, "%lld queries of a sequence", static_cast<long long>(a.queries));
  const int64_t seqs = sequences(a), tiles = ceil_div(a.queries, 16);
  // the kernel of many counts a sequence's bytes in 32 bits
  const int element = c->dtype == GNNSHAP_F32 ? 4 : 2;
  const int64_t limit = int64_t(1) << 31, rows = o->rows_per_seq;
  const bool near = o->q_row_stride >= 0 && o->q_head_stride >= 0 && o->q_row_stride <= limit / element / rows && o->q_head_stride <= limit / element / o->heads &&
                    rows * o->heads * 4 < limit && rows * std::max<int64_t>(o->mask_words, 1) * 8 < limit;
  if (a.queries <= 64 || !near) return check_launch(seqs * key_tiles(a, 128 / by_heads(a)), 256);
  const int64_t base = seqs * c->kv_heads * key_tiles(a, keys_of_many(a));
  // two wavefronts per SIMD, in one round (10,000 rows x 32 heads on 417 tokens,
  // in wavefronts: 2,048 83 us, 3,072 93, both with one key tile in eight empty)
  const int64_t want = std::max<int64_t>(1, std::min(2048 / std::max<int64_t>(base, 1), ceil_div(tiles, 8)));
  a.split = ceil_div(tiles, want);
  a.splits = static_cast<int>(ceil_div(tiles, a.split));
  if (const int st = check_launch(ceil_div(base * a.splits, 4), 256)) return st;
  return check_launch(seqs * key_tiles(a, 64), 256);
}

size_t carve(WeightsArgs& a, void* ws) {
  if (a.splits == 0) return 0;
  Carver c(ws);
  a.part = c.take<float>(static_cast<size_t>(sequences(a)) * a.c.kv_heads * a.splits * a.o.max_length);
  return c.bytes();
}

template <class T, int DP>
int launch(const WeightsArgs& a, hipStream_t s) {
  if (a.splits == 0) {
    const int64_t tiles = key_tiles(a, 128 / by_heads(a));
    GS_TIMED("k_cache_weights", s);
    k_cache_weights<T, DP><<<static_cast<unsigned>(sequences(a) * tiles), 256, 0, s>>>(a, by_heads(a),
                                                                                       static_cast<unsigned>(tiles));
    GS_LAUNCHED();
    return GNNSHAP_OK;
  }
  constexpr int NK = key_tiles_of(DP * static_cast<int>(sizeof(T)));
  const int64_t tiles = key_tiles(a, 16 * NK), places = sequences(a) * a.c.kv_heads * a.splits * tiles;
  {
    GS_TIMED("k_cache_weights_many", s);
    k_cache_weights_many<T, DP, NK><<<static_cast<unsigned>(ceil_div(places, 4)), 256, 0, s>>>(
        a, static_cast<unsigned>(tiles), static_cast<unsigned>(places));
  }
  GS_LAUNCHED();
  {
    GS_TIMED("k_cache_weights_join", s);
    k_cache_weights_join<<<static_cast<unsigned>(sequences(a) * key_tiles(a, 64)), 256, 0, s>>>(a);
  }
  GS_LAUNCHED();
  return GNNSHAP_OK;
}

}  // namespace

extern "C" int gnnshap_cache_weights_workspace(const gnnshap_cache* cache, const gnnshap_observed* o, size_t* bytes) {
  GS_TRY_BEGIN
  clear_error();
  if (!bytes) return fail(GNNSHAP_EINVAL, "bytes is NULL");
  if (const int st = check_observed(cache, o)) return st;
  WeightsArgs a{};
  if (const int st = lay_out(a, cache, o)) return st;
  *bytes = carve(a, nullptr);
  return GNNSHAP_OK;
  GS_TRY_END
}

extern "C" int gnnshap_cache_weights(const gnnshap_cache* cache, const gnnshap_observed* o, int32_t* info, void* ws,
                                     size_t ws_bytes, void* stream) {
  GS_TRY_BEGIN
  clear_error();
  if (const int st = check_observed(cache, o)) return st;
  if (o->num_rows == 0 || o->max_length == 0) return GNNSHAP_OK;
  if (!o->q || !o->lse || !o->table || !o->lengths || !o->weights)
    return fail(GNNSHAP_EINVAL, "NULL q, lse, table, lengths or weights");
  WeightsArgs a{};
  if (const int st = lay_out(a, cache, o)) return st;
  a.info = info;
  const size_t need = carve(a, ws);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(GNNSHAP_ECAPACITY, "cache_weights workspace needs %zu bytes, has %zu", need, ws ? ws_bytes : 0);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return with_dtype(cache->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    if (cache->head_dim <= 64) return launch<T, 64>(a, s);
    if (cache->head_dim <= 128) return launch<T, 128>(a, s);
    return launch<T, 256>(a, s);
  });
  GS_TRY_END
}
