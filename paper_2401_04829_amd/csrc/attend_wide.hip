// Attention over the shared part for many 16-bit queries of a group: every
// coalition's new token, times the query heads of a kv head, against the same
// keys.
//
// It is a matrix product with a softmax inside, bound by the vector
// instructions of the softmax (one exponential per query and key among them)
// and, beside them, by the matrix instructions.  A workgroup takes 128
// queries, a wavefront 32 of them, over all keys of a split, 32 at a time.
// While it weighs the scores of 32 keys it multiplies the next 32 keys, so
// that the two kinds of instructions run side by side, then it adds up the
// values of the 32 that it has weighed.  Keys and values come from the cache
// to registers and from there to LDS in tiles of 64 (32 where a head is wider
// than 128), one barrier per tile; keys are half a tile (a tile) further than
// values.  32 bf16 heads over 8 of 128: 10,000 rows on 417 shared and up to 4 own
// tokens 167 us, 2,002 rows on 3,851 shared ones 172 us (126 GFLOP with the
// hidden pairs, 730 TFLOP/s; 900 per further key); by the kernel of 16 queries
// to a wavefront 1,000 rows on 512 take 112 us, here 58.  In the longer of the two
// the matrix units are busy in 34 % of the SIMDs' cycles and the vector units in
// 53 %.  At two wavefronts per SIMD heads of 128 spill 12 of 256 registers.
//
// The layout is the transposed one of the other kernels on 32 x 32 x 16
// instructions: S^T = K Q^T leaves query = lane % 32 and keys in registers,
// register i of a lane in the upper half (h = 1) or lower half key
// 8 (i / 4) + 4 h + i % 4; eight registers on end are the right operand of
// 16 keys of O^T = V^T P^T.  Values are turned over on the way to LDS: a row
// holds one element of the 64 keys, in the order of those registers.  Row r of
// the product's tile t is element NT r + t of the NT tiles, so that a lane's
// results (and the values that it reads for own tokens) are NT elements on
// end.  The 16-byte pieces of an LDS row are swapped by the row's number, so
// that the 16 lanes that are served at a time meet 16 different columns.
//
// Where a tile's keys are is found out two tiles ahead: one wavefront turns
// 64 page table entries into byte offsets in LDS, having asked for the next
// tile's entries a step before.
#include "attend.h"

namespace {

using namespace gnnshap;

typedef float f16v_t __attribute__((ext_vector_type(16)));
typedef unsigned u2_t __attribute__((ext_vector_type(2)));

constexpr int kQueries = 128;  // queries of a workgroup
constexpr int kAhead = 4;      // tiles whose keys' offsets are in LDS

template <class T, int DP>
struct Wide {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  static constexpr int kTile = DP <= 128 ? 64 : 32;  // keys of a step
  static constexpr int NK = kTile / 32;       // tiles of S^T
  static constexpr int NT = DP / 32;          // tiles of O^T, elements on end of a lane
  static constexpr int KS = DP / 16;          // steps of K Q^T
  static constexpr int kPieces = DP / 8;      // 16-byte pieces of a key's row
  static constexpr int kKeyLoads = kTile * kPieces / 256;  // of a thread, per tile
  static constexpr int kValElems = DP >= 128 ? 8 : 4;   // elements on end that a thread turns over, of four keys
  static constexpr int kValPieces = DP / kValElems;
  static constexpr int kValLoads = kTile / 4 * kValPieces / 256;  // times four keys
  static constexpr int kBytes = kTile * DP * 2;  // of a tile's keys or values: LDS holds two of each

  static __device__ __forceinline__ f16v_t mfma(u4_t a, u4_t b, f16v_t c) {
    if constexpr (std::is_same_v<T, bf16_t>)
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(vec8, a), __builtin_bit_cast(vec8, b), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(vec8, a), __builtin_bit_cast(vec8, b), c, 0, 0, 0);
  }
  // Byte of 16-byte piece p of key row r (of two tiles' keys), and of the values' row r of product tile t.
  static __device__ __forceinline__ int key_at(int r, int p) {
    return r * DP * 2 + ((p ^ (DP >= 128 ? r & 15 : (r >> 1) & 7)) << 4);
  }
  static __device__ __forceinline__ int val_at(int r, int t, int p) {
    return 2 * kBytes + (32 * t + r) * kTile * 2 + ((p ^ (kTile == 64 ? (r >> 1) & 7 : (r >> 2) & 3)) << 4);
  }
  // 8-byte place of the four keys 4 c on in a values' row: the order of the weights' registers.
  static __device__ __forceinline__ int quad_place(int c) {
    const int in = c & 7;  // of 32 keys
    return (c >> 3) * 8 + (in >> 2) * 4 + (in & 1) * 2 + ((in >> 1) & 1);
  }

  u4_t key[kKeyLoads];
  unsigned val[kValLoads][4][kValElems / 2];

  // kTile keys from `from` on, or a tile's values, on their way to registers
  // and then to LDS; offsets: the byte of each one's first element, for keys in
  // a ring.  Elements behind head_dim are read as others of the row: the
  // queries hold 0 there, and the results are not written.
  // Each in kMoves moves, to go between other instructions.
  static constexpr int kMoves = kKeyLoads + kValLoads * 4;
  __device__ __forceinline__ void load(int move, const AttendArgs& a, const int64_t* offsets, int keys_from, int tile) {
    const int tid = threadIdx.x;
    if (move < kKeyLoads) {
      const char* const k = static_cast<const char*>(a.c.k) + (8 * (tid % kPieces) < a.c.head_dim ? 16 * (tid % kPieces) : 0);
      const int r = keys_from + tid / kPieces + move * (256 / kPieces);
      __builtin_memcpy(&key[move], k + offsets[r & (kAhead * kTile - 1)], 16);
    } else {
      const int i = (move - kKeyLoads) / 4, j = (move - kKeyLoads) % 4, d = tid % kValPieces * kValElems;
      const char* const v = static_cast<const char*>(a.c.v) + (d < a.c.head_dim ? 2 * d : 0);
      const int r = 4 * (tid / kValPieces + i * (256 / kValPieces)) + j;
      __builtin_memcpy(&val[i][j][0], v + offsets[(tile & (kAhead - 1)) * kTile + r], 2 * kValElems);
    }
  }
  __device__ __forceinline__ void store(int move, char* room, int keys_from, int tile) const {
    const int tid = threadIdx.x;
    if (move < kKeyLoads) {
      const int r = keys_from + tid / kPieces + move * (256 / kPieces);
      *reinterpret_cast<u4_t*>(room + key_at(r & (2 * kTile - 1), tid % kPieces)) = key[move];
    } else {
      const int i = (move - kKeyLoads) / 4, part = (move - kKeyLoads) % 4;
      const int c = tid / kValPieces + i * (256 / kValPieces), d = tid % kValPieces * kValElems, at = quad_place(c);
#pragma unroll
      for (int e = part * (kValElems / 4); e < (part + 1) * (kValElems / 4); ++e) {
        const unsigned sel = e & 1 ? 0x07060302u : 0x05040100u;
        const u2_t x = {__builtin_amdgcn_perm(val[i][1][e / 2], val[i][0][e / 2], sel),
                        __builtin_amdgcn_perm(val[i][3][e / 2], val[i][2][e / 2], sel)};
        *reinterpret_cast<u2_t*>(room + (tile & 1) * kBytes + val_at((d + e) / NT, (d + e) % NT, at >> 1) + (at & 1) * 8) = x;
      }
    }
  }
};

// The value that the lane 32 on or back has.
__device__ __forceinline__ float other_half(float x) {
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(threadIdx.x & 32 ? both[0] : both[1]);
}

// A query's running maximum and sum (this lane's half of it) and its column of O^T.
template <class T, int DP>
struct WideState {
  using W = Wide<T, DP>;
  float m = -INFINITY, l = 0.f;
  f16v_t o[W::NT];
  __device__ __forceinline__ WideState() {
#pragma unroll
    for (int t = 0; t < W::NT; ++t) o[t] = f16v_t{};
  }
  // The starting value of a lane's i-th score: -inf where the query does not
  // see the key; off: the unseen keys' bits, from the lane's first key on.
  static __device__ __forceinline__ float unseen(uint32_t off, int i) {
    const int bit = 8 * (i / 4) + i % 4;
    return __uint_as_float(static_cast<uint32_t>(static_cast<int32_t>(off << (31 - bit)) >> 31) & 0xFF800000u);
  }
  static __device__ __forceinline__ uint32_t off_bits(uint32_t bits) { return ~bits >> (4 * (threadIdx.x >> 5 & 1)); }
  // Raises the running maximum (2^kUp below it) to `top`, this lane's largest score.  O is
  // scaled down whenever a query of the wavefront has a new maximum: leaving m
  // up to 2^8 below it saves 6 % of the time, but then the largest weights are
  // no longer rounded exactly, and the error of 16-bit outputs grows from 1.2
  // to 1.4 times that of their own rounding.
  __device__ __forceinline__ void raise(float top, float scale) {
    top = fmaf(fmaxf(top, other_half(top)), scale, -kUp<T>);
    if (__ballot(top > m)) {
      const float up = fmaxf(top, m), use = up == -INFINITY ? 0.f : up, down = __builtin_amdgcn_exp2f(m - use);
      m = up;
      l *= down;
#pragma unroll
      for (int t = 0; t < W::NT; ++t) o[t] *= down;
    }
  }
  // A score's weight.
  __device__ __forceinline__ float weight(float s, float scale, float use) {
    const float w = __builtin_amdgcn_exp2f(fmaf(s, scale, -use));
    l += w;
    return w;
  }
  __device__ __forceinline__ float maximum() const { return m == -INFINITY ? 0.f : m; }
  // Eight weights, rounded to the values' type: an operand of 16 keys.
  static __device__ __forceinline__ u4_t operand(const f16v_t& s, int u) {
    typename W::vec8 w;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = static_cast<T>(s[8 * u + j]);
    return __builtin_bit_cast(u4_t, w);
  }
};

template <class T, int DP>
__global__ __launch_bounds__(64 * kWaves, DP <= 128 ? 2 : 1) void k_cache_attend_wide(AttendArgs a, Part part) {
  using W = Wide<T, DP>;
  constexpr int kTile = W::kTile, NK = W::NK;
  extern __shared__ char room[];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r = lane & 31, h = lane >> 5;
  const int D = a.c.head_dim;
  // The first loads of all chains (queries; lengths, pages, then keys and
  // values, of the shared part and of the rows' own) before anything waits.
  Place at = place_of(a, part, blockIdx.x);
  const int raw_len = part.lengths[at.group];
  int64_t* const offsets = reinterpret_cast<int64_t*>(room + 4 * W::kBytes);  // of kAhead tiles

  const int n_queries = part.r * a.share, q0 = at.tile * kQueries + wave * 32, qi = q0 + r, qs = qi < n_queries ? qi : 0;
  const int64_t row = at.group * part.r + qs / a.share;
  const int head = at.kv_head * a.share + qs % a.share;
  const float scale = fabsf(a.scale2);
  u4_t q[W::KS];
#pragma unroll
  for (int i = 0; i < W::KS; ++i) {
    const int d = 16 * i + 8 * h;
    q[i] = u4_t{0u, 0u, 0u, 0u};
    if (d < D)
      __builtin_memcpy(&q[i], static_cast<const T*>(a.q.q) + row * a.q.q_row_stride + head * a.q.q_head_stride + d, 16);
  }
  // The page of this lane's key of a tile (behind the part's last one some page of the row).
  const int key_lane = lane & (kTile - 1);
  const auto page_id = [&](int k) {
    int slot;
    const int pg = page_of(a, min(k + key_lane, part.max_len - 1), slot);
    return part.max_len > 0 ? part.table[at.group * part.width + pg] : 0;
  };
  const int page0 = page_id(at.k0 + wave * kTile);
  int page = page_id(at.k0 + (wave + kAhead) * kTile);
  // The own token of this lane's slot in the first pass.
  const OwnTile own(a, part, at, q0, 32);
  const int own_r = r / own.per, own_key = r - own_r * own.per;
  const int64_t own_row = own.row0 + (own_r < own.rows ? own_r : 0);
  int own_slot, own_page = -1, raw_own = 0, raw_slot = 0;
  const int own_pg = page_of(a, own_key, own_slot);
  if (at.with_own && own.rows > 0) {
    raw_own = a.own.lengths[row];
    raw_slot = a.own.lengths[own_row];
    if (own_pg < a.own.width) own_page = a.own.table[own_row * a.own.width + own_pg];
  }
  bound(a, part, at, bounded(a, part, raw_len), false);
  if (at.k0 >= at.k1 && !a.direct && !at.with_own) return;
  if (a.scale2 < 0.f)
#pragma unroll
    for (int i = 0; i < W::KS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) q[i][e] ^= 0x80008000u;
  WideState<T, DP> st;

  // The offset of this lane's key of a tile; behind the last key that of the
  // tile's first one (in a tile of none any: nothing of it is used).
  const auto put_offset = [&](int k, int id, int64_t* to) {
    int slot;
    page_of(a, min(k + key_lane, part.max_len - 1), slot);
    if (k + key_lane < at.k1 && (id < 0 || id >= a.c.num_pages) && a.info) *a.info = 1;
    if (id < 0 || id >= a.c.num_pages) id = 0;
    const bool in = k + key_lane < at.k1;
    const int first_id = __builtin_amdgcn_readfirstlane(id), first_slot = __builtin_amdgcn_readfirstlane(slot);
    id = in ? id : first_id;
    slot = in ? slot : first_slot;
    to[key_lane] = 2 * (id * a.c.page_stride + slot * a.c.slot_stride + static_cast<int64_t>(at.kv_head) * a.c.head_stride);
  };
  // The mask bits of a tile's positions.  For 64 of them, two words of the row
  // are shifted together, of which the second is the next tile's first.
  const uint64_t* const mask = a.q.masks + row * a.q.mask_words;
  const bool masked = a.q.num_players > 0;
  int64_t at_word = (at.first + at.k0) >> 6;
  const int shift = static_cast<int>((at.first + at.k0) & 63);
  const auto word = [&]() {
    const int64_t i = at_word++;
    return masked && i >= 0 && i < (a.q.num_players + 63) >> 6 ? mask[i] : 0ull;
  };
  uint64_t lo = 0, hi = 0;
  const auto bits_of = [&](int k) {
    const int left = at.k1 - k;
    uint64_t bits = ~0ull;
    if (masked) {
      const int64_t p = at.first + k, n = a.q.num_players - p;  // p < 0: before the players; n: players from here on
      if constexpr (NK == 2) {
        bits = shift ? lo >> shift | hi << (64 - shift) : lo;
        if (p < 0) bits |= p <= -64 ? ~0ull : (1ull << -p) - 1;
        if (n < 64) bits |= n <= 0 ? ~0ull : ~0ull << n;
      } else {
        bits = seen(mask, p, a.q.num_players);
      }
    }
    return left >= 64 ? bits : left <= 0 ? 0ull : bits & ((1ull << left) - 1);
  };

  // One pass over own tokens: `mine` is where that of this lane's slot is, or -1.
  const auto own_pass = [&](int pass, int64_t mine, int len) {
    const int64_t first = bounded(a, part, raw_len) - a.q.first_player;
    f16v_t s;
    const uint32_t off = WideState<T, DP>::off_bits(own.bits(a, pass, row, len, first));
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = WideState<T, DP>::unseen(off, i);
#pragma unroll
    for (int i = 0; i < W::KS; ++i) {
      u4_t k = {0u, 0u, 0u, 0u};
      if (mine >= 0 && 16 * i + 8 * h < D)
        __builtin_memcpy(&k, static_cast<const T*>(a.c.k) + mine + 16 * i + 8 * h, 16);
      s = W::mfma(k, q[i], s);
    }
    unsigned v[2][8][W::NT / 2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int64_t x = __shfl(mine, 16 * u + 8 * (j / 4) + 4 * h + j % 4);
#pragma unroll
        for (int e = 0; e < W::NT / 2; ++e) v[u][j][e] = 0u;
        const int d = W::NT * r;
        if (x >= 0 && d < D) __builtin_memcpy(&v[u][j][0], static_cast<const T*>(a.c.v) + x + d, 2 * W::NT);
      }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
    st.raise(top, scale);
    const float use = st.maximum();
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = st.weight(s[i], scale, use);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const u4_t p = st.operand(s, u);
#pragma unroll
      for (int t = 0; t < W::NT; ++t) {
        u4_t x;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[j] = __builtin_amdgcn_perm(v[u][2 * j + 1][t / 2], v[u][2 * j][t / 2], t & 1 ? 0x07060302u : 0x05040100u);
        st.o[t] = W::mfma(x, p, st.o[t]);
      }
    }
  };
  const auto own_passes = [&]() {
    if (!at.with_own || own.rows == 0) return;
    const int len = bounded(a, a.own, raw_own);
    int64_t mine = -1;
    if (own_r < own.rows && own_key < bounded(a, a.own, raw_slot)) {
      if (own_page >= 0 && own_page < a.c.num_pages)
        mine = own_page * a.c.page_stride + own_slot * a.c.slot_stride + static_cast<int64_t>(at.kv_head) * a.c.head_stride;
      else if (a.info)
        *a.info = 1;
    }
    const int passes = own.passes(len);
    for (int pass = 0; pass < passes; ++pass) {
      if (pass > 0) mine = own.at(a, pass, r, at.kv_head);
      own_pass(pass, mine, len);
    }
  };

  if (at.k0 < at.k1) {
    const int steps = (at.k1 - at.k0 + kTile - 1) / kTile;
    // wavefront w finds out where the keys of tiles w, w + 4, ... are
    put_offset(at.k0 + wave * kTile, page0, offsets + wave * kTile);
    lo = word();
    hi = word();
    const auto cover = [&](f16v_t& to, int first, int n, uint32_t which) {
      const uint32_t off = WideState<T, DP>::off_bits(which);
#pragma unroll
      for (int i = first; i < first + n; ++i) to[i] = WideState<T, DP>::unseen(off, i);
    };
    __syncthreads();
    W next;
#pragma unroll
    for (int x = 0; x < W::kMoves; ++x) next.load(x, a, offsets, 0, 0);
    own_passes();
#pragma unroll
    for (int x = 0; x < W::kMoves; ++x) next.store(x, room, 0, 0);
#pragma unroll
    for (int x = 0; x < W::kKeyLoads; ++x) next.load(x, a, offsets, 32, 0);
#pragma unroll
    for (int x = 0; x < W::kKeyLoads; ++x) next.store(x, room, 32, 0);
    __syncthreads();
    f16v_t s[2];  // scores of 32 keys, and of the next 32: unseen ones -inf before the others are there
    const uint64_t bits = bits_of(at.k0);
    cover(s[0], 0, 16, static_cast<uint32_t>(bits));
    cover(s[1], 0, 16, static_cast<uint32_t>(NK == 2 ? bits >> 32 : bits_of(at.k0 + kTile)));
#pragma unroll
    for (int j = 0; j < W::KS; ++j) s[0] = W::mfma(*reinterpret_cast<const u4_t*>(room + W::key_at(r, 2 * j + h)), q[j], s[0]);
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < 16; ++x) top = fmaxf(top, s[0][x]);
    st.raise(top, scale);

    // A step: NK times KS products of the keys after, beside which the scores
    // are weighed, and 2 NT of the values, beside which the scores after are
    // looked through and those after them begun.  Their LDS operands are one
    // sequence, read kLead products ahead; the scheduler may move no vector
    // instruction, read or product out of its turn.
    constexpr int kHalf = W::KS + 2 * W::NT, kProducts = NK * kHalf, kLead = 6, kMayCross = 0x274;
    const auto step = [&](int i, auto odd) {
      constexpr int kOdd = decltype(odd)::value;
      const auto operand = [&](int x) {
        const int n = x / kHalf, j = x % kHalf;
        const char* at_x = room + (j < W::KS ? W::key_at((kTile * kOdd + 32 * (n + 1) + r) & (2 * kTile - 1), 2 * j + h)
                                             : kOdd * W::kBytes + W::val_at(r, (j - W::KS) % W::NT,
                                                                            4 * n + 2 * ((j - W::KS) / W::NT) + h));
        return *reinterpret_cast<const u4_t*>(at_x);
      };
      u4_t lead[kLead];
#pragma unroll
      for (int x = 0; x < kLead; ++x) lead[x] = operand(x);
      lo = hi;
      hi = word();
      if (wave == (i & (kAhead - 1))) {  // tile i's offsets have been read
        put_offset(at.k0 + (i + kAhead) * kTile, page, offsets + wave * kTile);
        page = page_id(at.k0 + (i + 2 * kAhead) * kTile);
      }
      const uint64_t later = bits_of(at.k0 + i * kTile + 64);  // behind the last key: none
      float use = st.maximum();
      u4_t p[2];
#pragma unroll
      for (int x = 0; x < kProducts; ++x) {
        const int n = x / kHalf, j = x % kHalf;
        f16v_t& now = s[NK == 2 ? n : kOdd];
        f16v_t& then = s[NK == 2 ? 1 - n : 1 - kOdd];
        __builtin_amdgcn_sched_barrier(kMayCross);
        if (j < W::KS) {
          then = W::mfma(lead[x % kLead], q[j], then);
        } else {
          if (j == W::KS) {
            p[0] = WideState<T, DP>::operand(now, 0);
            p[1] = WideState<T, DP>::operand(now, 1);
            top = -INFINITY;
          }
          const int v = j - W::KS;
          st.o[v % W::NT] = W::mfma(lead[x % kLead], p[v / W::NT], st.o[v % W::NT]);
        }
        if (x + kLead < kProducts) lead[x % kLead] = operand(x + kLead);
        // the tile after (behind the last one: the last key again) from the
        // cache in the first products, to LDS in the last ones
        if (x < W::kMoves) next.load(x, a, offsets, i * kTile + kTile + 32, i + 1);
        if (x >= kProducts - W::kMoves) next.store(x - (kProducts - W::kMoves), room, kTile * kOdd + kTile + 32, kOdd + 1);
        if (j < W::KS) {
          constexpr int kPart = 16 / W::KS;
#pragma unroll
          for (int e = 0; e < kPart; ++e) now[kPart * j + e] = st.weight(now[kPart * j + e], scale, use);
        } else {
          constexpr int kPart = 16 / W::NT;
          const int v = j - W::KS;
          if (v < W::NT) {
            cover(now, v * kPart, kPart, static_cast<uint32_t>(n ? later >> 32 : later));  // for the keys after the next
          } else {
#pragma unroll
            for (int e = 0; e < kPart; ++e) top = fmaxf(top, then[(v - W::NT) * kPart + e]);
          }
        }
        if (j == kHalf - 1) {
          __builtin_amdgcn_sched_barrier(kMayCross);
          st.raise(top, scale);
          use = st.maximum();
        }
      }
      __syncthreads();
    };
    int i = 0;
    for (; i + 1 < steps; i += 2) {
      step(i, std::integral_constant<int, 0>{});
      step(i + 1, std::integral_constant<int, 1>{});
    }
    if (i < steps) step(i, std::integral_constant<int, 0>{});
  } else {
    own_passes();
  }

  const float l = st.l + other_half(st.l);
  bool bad = false;
  if (qi < n_queries) {
    const int64_t p = part_index(a, part.slot0 + at.split, row, head);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bad = !isfinite(l);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int d = W::NT * (8 * (i / 4) + 4 * h + i % 4);
      if (d >= D) continue;
      Pack<T, W::NT> done;
      Pack<float, W::NT> part_done;
#pragma unroll
      for (int t = 0; t < W::NT; ++t) {
        bad |= !isfinite(st.o[t][i]);
        done.v[t] = static_cast<T>(st.o[t][i] * inv);
        part_done.v[t] = st.o[t][i];
      }
      if (a.direct)
        store_pack(out_of<T>(a, row, head) + d, done);
      else
        store_pack(a.part_o + p * D + d, part_done);
    }
    if (h == 0) {
      if (!a.direct)
        a.part_ml[p] = make_float2(st.m, l);
      else if (a.q.lse)
        a.q.lse[row * a.q.heads + head] = lse_of<T>(st.m, l);
    }
  }
  if (__ballot(bad)) attend_slowly<T>(a, part, at, q0, 32);
}

template <class T, int DP>
int launch(const AttendArgs& a, hipStream_t s) {
  const Part& p = a.shared;
  const size_t bytes = 4 * Wide<T, DP>::kBytes + kAhead * Wide<T, DP>::kTile * sizeof(int64_t);
  const unsigned grid = static_cast<unsigned>(a.q.num_rows / p.r * a.c.kv_heads * p.tiles * p.splits);
  GS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&k_cache_attend_wide<T, DP>),
                             hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)));
  {
    GS_TIMED("k_cache_attend_wide", s);
    k_cache_attend_wide<T, DP><<<grid, 64 * kWaves, bytes, s>>>(a, p);
  }
  GS_LAUNCHED();
  return GNNSHAP_OK;
}

template <class T>
int launch_type(const AttendArgs& a, hipStream_t s) {
  if (a.c.head_dim <= 64) return launch<T, 64>(a, s);
  if (a.c.head_dim <= 128) return launch<T, 128>(a, s);
  return launch<T, 256>(a, s);
}

}  // namespace

int gnnshap::launch_attend_wide(const AttendArgs& a, hipStream_t s) {
  return a.c.dtype == GNNSHAP_BF16 ? launch_type<bf16_t>(a, s) : launch_type<f16_t>(a, s);
}
