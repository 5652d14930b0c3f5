// Tokens that leave a paged cache: those that attention gave the least weight.
//
// One launch finds a sequence's kept tokens: the weights' order-preserving
// images are counted by digits of 11, 11 and 10 bits from the highest down,
// until the lowest kept image is known; then one pass in order hands out the
// places.  A second launch moves keys and values up.  The kept tokens stay in their
// order, so token i of them comes from a place p_i >= i, and p rises: a
// workgroup that has a slice of the elements of all of a sequence's tokens takes
// them in order, many at a time, and writes some only after all of these are
// read; no token further on can be overwritten by then.  Tokens in front of the
// first dropped one are not touched.
#include "stats.h"

namespace {

using namespace gnnshap;

constexpr int kSelect = 1024;  // threads that select
constexpr int kSlots = 4;      // elements of a thread at a time, 64 apart
constexpr int kBins = 2048;
constexpr int kCopies = 4;     // of the bins, by lanes: what adds to one place waits for each other

struct EvictArgs {
  gnnshap_cache c;
  gnnshap_eviction e;
  int page_shift;
  int32_t* begin;   // [sequence] first token that moves
  int32_t* info;
  int pieces, packs;  // slices of a head's elements, of so many packs of 16 bytes
};

// The sum of x over the threads before this one, and over all (1,024 threads).
__device__ __forceinline__ int before(int x, int* room, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int up = x;
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const int y = __shfl_up(up, off);
    if (lane >= off) up += y;
  }
  if (lane == 63) room[wave] = up;
  __syncthreads();
  int base = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kSelect / 64; ++w) {
    if (w < wave) base += room[w];
    all += room[w];
  }
  __syncthreads();
  return base + up - x;
}

// A token's image, by which it stays or goes: the first and the last ones' above
// all others, those behind the sequence below all (ordered() gives neither).
struct Images {
  int first, last, len;   // first <= place < last: the weight decides
  __device__ __forceinline__ uint32_t operator()(float w, int at) const {
    return at >= len ? 0u : at >= first && at < last ? ordered(w) : 0xFFFFFFFFu;
  }
};

// The images of up to 4,096 HELD tokens stay in registers, so that memory is
// waited for twice; HELD = 0: of any number, read for each digit and once more.
// One workgroup's instructions bound it: 30,000 tokens, of which 4,000 stay, 29 us
// (38 when an image was found anew for each digit, 47 when the weights were
// read for each); 64 x 2,001 tokens 10 us.
template <int HELD>
__global__ __launch_bounds__(kSelect) void k_evict_select(EvictArgs a) {
  constexpr int kWaves = kSelect / 64, kBlocks = kWaves * (HELD ? HELD : 1);
  constexpr int kTurn = kSelect * kSlots;   // tokens of a turn: a wavefront has kSlots times 64 on end
  __shared__ int bins[kBins * kCopies], room[kWaves], found[2], first_gap;
  __shared__ int block_sure[kBlocks], block_ties[kBlocks];
  const int64_t seq = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int keep = static_cast<int>(a.e.keep);
  const float* const w = a.e.weights + seq * a.e.weights_stride;
  const auto place_in = [&](int turn, int s) { return turn * kTurn + (wave * kSlots + s) * 64 + lane; };
  uint32_t held[HELD ? HELD : 1][kSlots];
  if constexpr (HELD > 0) {  // before the length is known
#pragma unroll
    for (int j = 0; j < HELD; ++j)
#pragma unroll
      for (int s = 0; s < kSlots; ++s)
        held[j][s] = place_in(j, s) < a.e.max_length ? __float_as_uint(w[place_in(j, s)]) : 0u;
  }
  int len = a.e.lengths[seq];
  if (len < 0 || len > a.e.max_length) {
    if (tid == 0 && a.info) *a.info = 1;
    len = len < 0 ? 0 : static_cast<int>(a.e.max_length);
  }
  __syncthreads();  // (new_lengths may be lengths)
  float* const out = a.e.new_weights + seq * a.e.new_weights_stride;
  int32_t* const kept = a.e.kept + seq * a.e.keep;
  const int now = len < keep ? len : keep;
  if (len <= keep) {
    for (int i = tid; i < len; i += kSelect) {
      kept[i] = i;
      if (out != w) out[i] = w[i];
    }
    if (tid == 0) a.begin[seq] = now;
  } else {
    const Images image{static_cast<int>(a.e.first), len - static_cast<int>(a.e.recent), len};
    if constexpr (HELD > 0) {
#pragma unroll
      for (int j = 0; j < HELD; ++j)
#pragma unroll
        for (int s = 0; s < kSlots; ++s) held[j][s] = image(__uint_as_float(held[j][s]), place_in(j, s));
    }
    // the lowest image that stays; of those with it, so many do as are not above it
    uint32_t low = 0xFFFFFFFFu, mask = 0;
    int ties = keep;
    const int want = keep - static_cast<int>(a.e.first) - static_cast<int>(a.e.recent);
    if (want > 0) {
      low = 0;
      ties = want;   // (the first and the last ones are not counted: many of one image wait for each other)
    }
#pragma unroll 1
    for (int digit = 0; digit < 3 && want > 0; ++digit) {
      const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
      for (int i = tid; i < kBins * kCopies; i += kSelect) bins[i] = 0;
      __syncthreads();
      const auto count = [&](uint32_t x) {
        if ((x & mask) == low && x - 1u < 0xFFFFFFFEu)
          atomicAdd(&bins[__builtin_amdgcn_ubfe(x, shift, bits) * kCopies + lane % kCopies], 1);
      };
      if constexpr (HELD > 0) {
#pragma unroll
        for (int j = 0; j < HELD; ++j)
          if (j * kTurn < len)
#pragma unroll
            for (int s = 0; s < kSlots; ++s) count(held[j][s]);
      } else {
#pragma unroll 4
        for (int i = tid; i < len; i += kSelect) count(image(w[i], i));
      }
      __syncthreads();
      // from the highest bin down: two of a thread
      int hi = 0, lo = 0, all;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        hi += bins[(kBins - 1 - 2 * tid) * kCopies + i];
        lo += bins[(kBins - 2 - 2 * tid) * kCopies + i];
      }
      const int above = before(hi + lo, room, all);
      if (above < ties && ties <= above + hi + lo) {
        const bool in_hi = ties <= above + hi;
        found[0] = kBins - 1 - 2 * tid - (in_hi ? 0 : 1);
        found[1] = in_hi ? above : above + hi;
      }
      __syncthreads();
      low |= static_cast<uint32_t>(found[0]) << shift;
      mask |= ((1u << bits) - 1u) << shift;
      ties -= found[1];
      __syncthreads();
    }
    if (tid == 0) first_gap = len;
    const uint64_t under = (1ull << lane) - 1ull;
    // Which of a turn's tokens stay (a bit per slot), behind `tied` ties, and their
    // places in `kept` from `placed` on.
    const auto choose = [&](const uint32_t (&x)[kSlots], int turn, int placed, int tied) {
      uint32_t stays = 0;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int at = place_in(turn, s);
        const uint64_t tie = __ballot(x[s] == low);
        const bool enters = x[s] > low || (x[s] == low && tied + __popcll(tie & under) < ties);
        const uint64_t in = __ballot(enters);
        const int to = placed + __popcll(in & under);
        stays |= enters ? 1u << s : 0u;
        if (enters)
          kept[to] = at;
        else if (to == at)   // (not behind the sequence, where there are fewer kept)
          atomicMin(&first_gap, to);
        placed += __popcll(in);
        tied += __popcll(tie);
      }
      return stays;
    };
    // Writes their weights, which have been read.
    const auto write = [&](const uint32_t (&x)[kSlots], uint32_t stays, int placed) {
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const uint64_t in = __ballot(stays >> s & 1u);
        if (stays >> s & 1u) out[placed + __popcll(in & under)] = __uint_as_float(x[s]);
        placed += __popcll(in);
      }
    };
    const auto totals = [&](const uint32_t (&x)[kSlots], int& sure, int& tied) {
      sure = tied = 0;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        sure += __popcll(__ballot(x[s] > low));
        tied += __popcll(__ballot(x[s] == low));
      }
    };
    if constexpr (HELD > 0) {
#pragma unroll
      for (int j = 0; j < HELD; ++j) {
        int sure, tied;
        totals(held[j], sure, tied);
        if (lane == 0) {
          block_sure[j * kWaves + wave] = sure;
          block_ties[j * kWaves + wave] = tied;
        }
      }
      __syncthreads();
      if (wave == 0) {  // of the blocks before each
        constexpr int kEach = (kBlocks + 63) / 64;
        int n_sure[kEach], n_ties[kEach], s = 0, t = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int b = lane * kEach + i;
          n_sure[i] = b < kBlocks ? block_sure[b] : 0;
          n_ties[i] = b < kBlocks ? block_ties[b] : 0;
          s += n_sure[i];
          t += n_ties[i];
        }
        int up_s = s, up_t = t;
#pragma unroll
        for (int off = 1; off < 64; off *= 2) {
          const int x = __shfl_up(up_s, off), y = __shfl_up(up_t, off);
          if (lane >= off) {
            up_s += x;
            up_t += y;
          }
        }
        s = up_s - s;
        t = up_t - t;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int b = lane * kEach + i;
          if (b < kBlocks) {
            block_sure[b] = s + min(t, ties);
            block_ties[b] = t;
          }
          s += n_sure[i];
          t += n_ties[i];
        }
      }
      __syncthreads();
      uint32_t stays[HELD];
#pragma unroll
      for (int j = 0; j < HELD; ++j) {
        stays[j] = 0;
        if (j * kTurn < len) {
          stays[j] = choose(held[j], j, block_sure[j * kWaves + wave], block_ties[j * kWaves + wave]);
#pragma unroll
          for (int s = 0; s < kSlots; ++s)
            if (stays[j] >> s & 1u) held[j][s] = __float_as_uint(w[place_in(j, s)]);
        }
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();  // all are read: new_weights may be weights
#pragma unroll
      for (int j = 0; j < HELD; ++j)
        if (j * kTurn < len) write(held[j], stays[j], block_sure[j * kWaves + wave]);
    } else {
      __syncthreads();
      int placed = 0, tied = 0;   // in the turns before, `placed` without ties
#pragma unroll 1
      for (int turn = 0; turn * kTurn < len; ++turn) {
        uint32_t x[kSlots], weight[kSlots];
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
          weight[s] = place_in(turn, s) < len ? __float_as_uint(w[place_in(turn, s)]) : 0u;
          x[s] = image(__uint_as_float(weight[s]), place_in(turn, s));
        }
        int n_sure, n_ties, all_sure, all_ties;
        totals(x, n_sure, n_ties);
        // (barriers: the turn is read before any of its places is written)
        const int s = __shfl(before(lane == 0 ? n_sure : 0, room, all_sure), 0);
        const int t = __shfl(before(lane == 0 ? n_ties : 0, room, all_ties), 0);
        const int from = placed + s + min(tied + t, ties);
        write(weight, choose(x, turn, from, tied + t), from);
        placed += all_sure;
        tied += all_ties;
      }
    }
    __syncthreads();
    if (tid == 0) a.begin[seq] = first_gap;
  }
  if (tid == 0) a.e.new_lengths[seq] = now;
  for (int i = now + tid; i < keep; i += kSelect) kept[i] = -1;
  for (int64_t i = now + tid; i < a.e.max_length; i += kSelect) out[i] = 0.f;
}

constexpr int kMove = 1024;    // threads that move
constexpr int kInFlight = 4;   // tokens of a thread

// Where token i of a sequence is; -1 if its page is out of range.
__device__ __forceinline__ int64_t place_of(const EvictArgs& a, int64_t seq, int i) {
  int page, slot;
  if (a.page_shift >= 0) {
    page = i >> a.page_shift;
    slot = i & ((1 << a.page_shift) - 1);
  } else {
    page = i / a.c.page_size;
    slot = i - page * a.c.page_size;
  }
  const int p = a.e.table[seq * a.e.table_width + page];
  if (p < 0 || p >= a.c.num_pages) {
    if (a.info) *a.info = 1;
    return -1;
  }
  return p * a.c.page_stride + slot * a.c.slot_stride;
}

// A workgroup: a.packs packs of 16 bytes of one head's keys or values, of all of a
// sequence's tokens.  Bound by memory where sequences are many (64 of 2,001 tokens,
// of which one goes and the last 200 to 220 of each move up, 120 MB: 24 us, 5
// TB/s), else by three dependent loads of each turn (kept place, page, element): 4,000
// tokens of one sequence 17 us.
template <class T>
__global__ __launch_bounds__(kMove) void k_evict_move(EvictArgs a) {
  unsigned b = blockIdx.x;
  // slices of the same head mostly meet in one XCD, whose cache holds the lines that they share
  const unsigned heads = gridDim.x / a.pieces;
  const int piece = b / heads;
  b -= piece * heads;
  const int head = b % a.c.kv_heads;
  b /= a.c.kv_heads;
  T* const pages = static_cast<T*>(b & 1 ? a.c.v : a.c.k);
  const int64_t seq = b >> 1;
  const int n = a.e.new_lengths[seq], begin = a.begin[seq];
  const int32_t* const kept = a.e.kept + seq * a.e.keep;
  const int per = kMove / a.packs, mine = threadIdx.x / a.packs, pack = threadIdx.x - mine * a.packs;
  const int64_t in_token = head * a.c.head_stride + (piece * a.packs + pack) * (16 / static_cast<int>(sizeof(T)));
#pragma unroll 1
  for (int base = begin; base < n; base += per * kInFlight) {
    Pack<unsigned, 4> x[kInFlight];
    int64_t from[kInFlight], to[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int i = base + u * per + mine;
      const bool in = mine < per && i < n;
      from[u] = in ? place_of(a, seq, kept[i]) : -1;
      to[u] = in ? place_of(a, seq, i) : -1;
    }
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      if (from[u] < 0) to[u] = -1;
      x[u] = load_pack<unsigned, 4>(reinterpret_cast<const unsigned*>(pages + (to[u] < 0 ? 0 : from[u]) + in_token));
    }
    // all of the workgroup's tokens are read
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
      if (to[u] >= 0) store_pack(reinterpret_cast<unsigned*>(pages + to[u] + in_token), x[u]);
  }
}

int check_eviction(const gnnshap_cache* c, const gnnshap_eviction* e) {
  if (const int st = check_cache(c)) return st;
  if (!e || e->num_seqs < 0) return fail(GNNSHAP_EINVAL, "eviction: NULL or a negative number of sequences");
  if (e->num_seqs > INT32_MAX)
    return fail(GNNSHAP_EUNSUPPORTED, "%lld sequences in one call", static_cast<long long>(e->num_seqs));
  if (e->table_width < 0 || e->max_length < 0) return fail(GNNSHAP_EINVAL, "negative width or length");
  if (e->max_length > (int64_t(1) << 30) || e->keep > (int64_t(1) << 30))
    return fail(GNNSHAP_EUNSUPPORTED, "%lld of up to %lld tokens", static_cast<long long>(e->keep),
                static_cast<long long>(e->max_length));
  if (ceil_div(e->max_length, c->page_size) > e->table_width)
    return fail(GNNSHAP_EINVAL, "%lld tokens do not fit %lld pages of %d", static_cast<long long>(e->max_length),
                static_cast<long long>(e->table_width), static_cast<int>(c->page_size));
  if (e->keep < 1 || e->first < 0 || e->recent < 0 || e->first > e->keep || e->recent > e->keep - e->first)
    return fail(GNNSHAP_EINVAL, "the first %lld and the last %lld of %lld kept tokens", static_cast<long long>(e->first),
                static_cast<long long>(e->recent), static_cast<long long>(e->keep));
  if (e->weights_stride < 0 || e->new_weights_stride < 0) return fail(GNNSHAP_EINVAL, "negative stride of the weights");
  if (e->new_weights_stride < e->max_length && e->num_seqs > 1)
    return fail(GNNSHAP_EINVAL, "the new weights' rows, %lld apart, overlap", static_cast<long long>(e->new_weights_stride));
  if (e->weights && e->weights == e->new_weights && e->weights_stride != e->new_weights_stride)
    return fail(GNNSHAP_EINVAL, "new_weights are weights with another stride");
  return GNNSHAP_OK;
}

// Slices of a head's elements: no more than give the chip two workgroups per
// compute unit, and not below 32 bytes.
int lay_out(EvictArgs& a, const gnnshap_cache* c, const gnnshap_eviction* e) {
  a.c = *c;
  a.e = *e;
  a.page_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (c->page_size == 1 << i) a.page_shift = i;
  const int packs = c->head_dim * (c->dtype == GNNSHAP_F32 ? 4 : 2) / 16;
  const int64_t base = e->num_seqs * 2 * c->kv_heads;
  a.pieces = 1;
  while (base * a.pieces < 512 && packs / a.pieces % 2 == 0 && packs / a.pieces > 2) a.pieces *= 2;
  a.packs = packs / a.pieces;
  if (const int st = check_launch(base * a.pieces, kMove)) return st;
  return check_launch(e->num_seqs, kSelect);
}

size_t carve(EvictArgs& a, void* ws) {
  Carver c(ws);
  a.begin = c.take<int32_t>(static_cast<size_t>(a.e.num_seqs));
  return c.bytes();
}

}  // namespace

extern "C" int gnnshap_cache_evict_workspace(const gnnshap_cache* cache, const gnnshap_eviction* e, size_t* bytes) {
  GS_TRY_BEGIN
  clear_error();
  if (!bytes) return fail(GNNSHAP_EINVAL, "bytes is NULL");
  if (const int st = check_eviction(cache, e)) return st;
  EvictArgs a{};
  if (const int st = lay_out(a, cache, e)) return st;
  *bytes = carve(a, nullptr);
  return GNNSHAP_OK;
  GS_TRY_END
}

extern "C" int gnnshap_cache_evict(const gnnshap_cache* cache, const gnnshap_eviction* e, int32_t* info, void* ws,
                                   size_t ws_bytes, void* stream) {
  GS_TRY_BEGIN
  clear_error();
  if (const int st = check_eviction(cache, e)) return st;
  if (e->num_seqs == 0) return GNNSHAP_OK;
  if (!e->table || !e->lengths || !e->weights || !e->kept || !e->new_lengths || !e->new_weights)
    return fail(GNNSHAP_EINVAL, "NULL table, lengths, weights, kept, new_lengths or new_weights");
  EvictArgs a{};
  if (const int st = lay_out(a, cache, e)) return st;
  a.info = info;
  const size_t need = carve(a, ws);
  if (!ws || ws_bytes < need)
    return fail(GNNSHAP_ECAPACITY, "cache_evict workspace needs %zu bytes, has %zu", need, ws ? ws_bytes : 0);
  hipStream_t s = static_cast<hipStream_t>(stream);
  {
    GS_TIMED("k_evict_select", s);
    const unsigned grid = static_cast<unsigned>(e->num_seqs);
    if (e->max_length <= 4096)
      k_evict_select<1><<<grid, kSelect, 0, s>>>(a);
    else if (e->max_length <= 8 * 4096)
      k_evict_select<8><<<grid, kSelect, 0, s>>>(a);
    else
      k_evict_select<0><<<grid, kSelect, 0, s>>>(a);
  }
  GS_LAUNCHED();
  return with_dtype(cache->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    {
      GS_TIMED("k_evict_move", s);
      k_evict_move<T><<<static_cast<unsigned>(e->num_seqs * 2 * cache->kv_heads * a.pieces), kMove, 0, s>>>(a);
    }
    GS_LAUNCHED();
    return static_cast<int>(GNNSHAP_OK);
  });
  GS_TRY_END
}
