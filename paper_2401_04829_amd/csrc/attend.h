// What the attention kernels share: the layout of the work, where tokens are,
// which of them a row sees, and the slow path.
#pragma once

#include "tokens.h"

namespace gnnshap {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef unsigned u4_t __attribute__((ext_vector_type(4)));

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kWaves = 4;
constexpr int kChunk = 32;  // keys of a wavefront's step

// The exponent of the largest weight.  Weights enter the product with the
// values in the values' type; fp16 has no numbers below 2^-24, so a weight of 1
// or less would be off by 2^-25 and many small ones would be lost (2,048 keys,
// of which one weighs 1 and the others 2^-25.5 each: 12 % of those).  Carried
// 2^14 larger, of which fp16 holds 65,504, they keep 11 bits down to 2^-28 of the
// largest, at no cost: the running maximum m that scores are taken from is kept
// that much lower, so that l and O belong to it as they always do.
template <class T>
constexpr float kUp = std::is_same_v<T, f16_t> ? 14.f : 0.f;

// One part of the rows' contexts: `r` consecutive rows share each row of its
// table.  A group's rows times the query heads of a kv head are its queries,
// in tiles; a wavefront (a workgroup of the wide kernel) takes a tile over
// split_keys keys, and over those `splits` times as far on, and so on.
struct Part {
  const int32_t* table;
  const int32_t* lengths;
  int64_t width;
  int max_len;
  int r;
  int tile;       // queries
  int tiles;
  bool wide;      // the kernel of many 16-bit queries takes it
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
  bool fused;      // the shared part's kernel takes the own parts too
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

// A length as the caller's arrays can hold it.
__device__ __forceinline__ int bounded(const AttendArgs& a, const Part& part, int n) {
  if (n < 0 || n > part.max_len) {
    if (a.info) *a.info = 1;
    return n < 0 ? 0 : part.max_len;
  }
  return n;
}

// The length of sequence `g` of a part.
__device__ __forceinline__ int length_of(const AttendArgs& a, const Part& part, int64_t g) {
  return bounded(a, part, part.lengths[g]);
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

template <class T>
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : (m + kUp<T>) * kLn2 + logf(l * __builtin_exp2f(-kUp<T>));
}

struct Place {  // what a wavefront or workgroup works on
  int64_t group;
  int kv_head, tile, split;
  int64_t first;  // context position of the part's position 0, counted from the first player
  int k0, k1;     // keys of the split (its first ones)
  bool with_own;  // the rows' own parts too
};

// Decodes the number of a workgroup or wavefront.  Consecutive ones take
// consecutive kv heads: workgroups of one head, which read the same keys, then
// meet in an XCD's cache, and the wavefronts of a workgroup read neighbouring
// parts of the same tokens.  Splits change last, and each turns the rows by
// one: where lengths are unlike, neither the first splits, which all rows have,
// nor those of one long row may meet in one XCD.
__device__ __forceinline__ Place place_of(const AttendArgs& a, const Part& part, uint32_t number) {
  Place at;
  uint32_t b = number;
  at.kv_head = b % static_cast<uint32_t>(a.c.kv_heads);
  b /= static_cast<uint32_t>(a.c.kv_heads);
  at.tile = b % static_cast<uint32_t>(part.tiles);
  b /= static_cast<uint32_t>(part.tiles);
  const uint32_t groups = static_cast<uint32_t>(a.q.num_rows / part.r);
  at.split = b / groups;
  at.group = (b % groups + static_cast<uint32_t>(at.split)) % groups;
  at.k0 = at.split * part.split_keys;
  at.with_own = a.fused && at.split == 0;
  return at;
}

// The rest of it, which depends on the sequence's length.
__device__ __forceinline__ void bound(const AttendArgs& a, const Part& part, Place& at, int len, bool is_own) {
  at.k1 = len - at.k0 < part.split_keys ? len : at.k0 + part.split_keys;
  if (at.k1 < at.k0) at.k1 = at.k0;
  at.first = -a.q.first_player;
  if (is_own && a.shared.table) at.first += length_of(a, a.shared, at.group / a.shared.r);
}

// Where token `key` of sequence `seq` of a part is, straight from the table; -1 if its page is out of range.
__device__ __forceinline__ int64_t token_at(const AttendArgs& a, const Part& part, int64_t seq, int key, int kv_head) {
  int slot;
  const int pg = page_of(a, key, slot);
  const int p = part.table[seq * part.width + pg];
  if (p < 0 || p >= a.c.num_pages) {
    if (a.info) *a.info = 1;
    return -1;
  }
  return p * a.c.page_stride + slot * a.c.slot_stride + static_cast<int64_t>(kv_head) * a.c.head_stride;
}

// The own tokens of the rows of a tile of queries, as tiles of 32 keys of which
// each query sees its own row's: `per` tokens of each of the rows at a time.
struct OwnTile {
  int64_t row0;  // first row
  int rows, per;
  // q0: the tile's first query; size: how many it has
  __device__ __forceinline__ OwnTile(const AttendArgs& a, const Part& part, const Place& at, int q0, int size) {
    const int n = part.r * a.share, q1 = q0 + size - 1 < n - 1 ? q0 + size - 1 : n - 1;
    const int r0 = q0 / a.share;
    row0 = at.group * part.r + r0;
    rows = q0 < n ? q1 / a.share - r0 + 1 : 0;
    per = rows > 0 ? kChunk / rows : 1;
  }
  // Passes that the lanes' rows take, of `len` own tokens.
  __device__ __forceinline__ int passes(int len) const {
    int most = rows > 0 ? len : 0;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) most = max(most, __shfl_xor(most, off));
    return (most + per - 1) / per;
  }
  // Where the key in slot s of a pass is; -1: there is none.
  __device__ __forceinline__ int64_t at(const AttendArgs& a, int pass, int s, int kv_head) const {
    const int r = s / per, key = pass * per + s - r * per;
    if (r >= rows || key >= length_of(a, a.own, row0 + r)) return -1;
    return token_at(a, a.own, row0 + r, key, kv_head);
  }
  // The slots of a pass that a query of row `row` with `len` own tokens sees.
  __device__ __forceinline__ uint32_t bits(const AttendArgs& a, int pass, int64_t row, int len, int64_t first) const {
    const int left = len - pass * per, n = left < per ? left : per;
    if (n <= 0) return 0u;
    uint32_t b = n >= 32 ? ~0u : (1u << n) - 1u;
    if (a.q.num_players > 0) b &= seen(a.q.masks + row * a.q.mask_words, first + pass * per, a.q.num_players);
    return b << ((static_cast<int>(row - row0) * per) & 31);  // (a lane without a query: anything)
  }
};

// The slow path, by a wavefront for n of a group's queries from q0 on, one
// after the other: a lane per key, then per four elements; a position that the
// row does not see enters no product.
template <class T>
__device__ void attend_slowly(const AttendArgs& a, const Part& part, const Place& at, int q0, int n) {
  const int lane = threadIdx.x & 63, D = a.c.head_dim;
  for (int i = q0; i < q0 + n && i < part.r * a.share; ++i) {
    const int64_t row = at.group * part.r + i / a.share;
    const int head = at.kv_head * a.share + i % a.share;
    const T* q = static_cast<const T*>(a.q.q) + row * a.q.q_row_stride + head * a.q.q_head_stride;
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int own = 0; own < 2; ++own) {
      if (own && !at.with_own) break;
      const Part& p = own ? a.own : part;
      const int64_t seq = own ? row : at.group;
      const int len = length_of(a, p, seq), k0 = own ? 0 : at.k0;
      const int64_t first = own ? length_of(a, part, at.group) - a.q.first_player : at.first;
      for (int c = k0; c < len; c += 64) {
        // the splits between this one's turns
        if (!own && (c - k0) % p.split_keys == 0 && c > k0) c += (p.splits - 1) * p.split_keys;
        const int k1 = own ? len : min(len, c + p.split_keys - (c - k0) % p.split_keys);
        bool sees = c + lane < k1;
        if (sees && a.q.num_players > 0)
          sees = seen(a.q.masks + row * a.q.mask_words, first + c + lane, a.q.num_players) & 1u;
        const int64_t where = sees ? token_at(a, p, seq, c + lane, at.kv_head) : -1;
        sees = where >= 0;
        float s = -INFINITY;
        if (sees) {
          const T* k = static_cast<const T*>(a.c.k) + where;
          s = 0.f;
          for (int d = 0; d < D; ++d) s += static_cast<float>(q[d]) * static_cast<float>(k[d]);
          s *= a.scale2;
        }
        float top = fmaxf(m, s);
        for (int off = 1; off < 64; off *= 2) top = fmaxf(top, __shfl_xor(top, off));
        const float use = top == -INFINITY ? 0.f : top;
        const float down = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - use);
        const float e = sees ? __builtin_amdgcn_exp2f(s - use) : 0.f;
        float sum = e;
        for (int off = 1; off < 64; off *= 2) sum += __shfl_xor(sum, off);
        l = l * down + sum;
        for (int x = 0; x < 4; ++x) o[x] = m == -INFINITY ? 0.f : o[x] * down;
        m = top;
        for (uint64_t left = __ballot(sees); left; left &= left - 1) {
          const int j = __builtin_ctzll(left);
          const float w = __shfl(e, j);
          const T* v = static_cast<const T*>(a.c.v) + __shfl(where, j) + 4 * lane;
          if (4 * lane < D)
            for (int x = 0; x < 4; ++x) o[x] += w * static_cast<float>(v[x]);
        }
      }
    }
    const int64_t p = part_index(a, part.slot0 + at.split, row, head);
    if (4 * lane < D)
      for (int x = 0; x < 4; ++x) {
        if (a.direct)
          out_of<T>(a, row, head)[4 * lane + x] = static_cast<T>(l == 0.f ? 0.f : o[x] / l);
        else
          a.part_o[p * D + 4 * lane + x] = l == 0.f ? 0.f : o[x];
      }
    if (lane == 0) {
      if (!a.direct)
        a.part_ml[p] = make_float2(m, l);
      else if (a.q.lse)
        a.q.lse[row * a.q.heads + head] = lse_of<T>(m, l);
    }
  }
}

// Launches the kernel of many 16-bit queries of a group over the shared part (attend_wide.hip).
int launch_attend_wide(const AttendArgs& a, hipStream_t s);

}  // namespace gnnshap
