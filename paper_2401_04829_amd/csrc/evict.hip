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

__global__ __launch_bounds__(kSelect) void k_evict_select(EvictArgs a) {
  __shared__ int bins[kBins], room[kSelect / 64], found[2], first_gap;
  const int64_t seq = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int keep = static_cast<int>(a.e.keep), first = static_cast<int>(a.e.first);
  int len = a.e.lengths[seq];
  if (len < 0 || len > a.e.max_length) {
    if (tid == 0 && a.info) *a.info = 1;
    len = len < 0 ? 0 : static_cast<int>(a.e.max_length);
  }
  __syncthreads();  // (new_lengths may be lengths)
  const float* const w = a.e.weights + seq * a.e.weights_stride;
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
    const int last = len - static_cast<int>(a.e.recent);   // first <= place < last: the weights decide
    int want = keep - first - static_cast<int>(a.e.recent);
    uint32_t low = 0xFFFFFFFFu;  // image of the last one that enters (none does if it stays so: images are below)
    int ties = 0;                // of those with this image, so many enter
    if (want > 0) {
      uint32_t prefix = 0, mask = 0;
#pragma unroll 1
      for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
        for (int i = tid; i < kBins; i += kSelect) bins[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (int i = first + tid; i < last; i += kSelect) {
          const uint32_t x = ordered(w[i]);
          if ((x & mask) == prefix) atomicAdd(&bins[x >> shift & ((1u << bits) - 1u)], 1);
        }
        __syncthreads();
        // from the highest bin down: two of a thread
        const int hi = bins[kBins - 1 - 2 * tid], lo = bins[kBins - 2 - 2 * tid];
        int all;
        const int above = before(hi + lo, room, all);
        if (above < want && want <= above + hi + lo) {
          const bool in_hi = want <= above + hi;
          found[0] = kBins - 1 - 2 * tid - (in_hi ? 0 : 1);
          found[1] = in_hi ? above : above + hi;
        }
        __syncthreads();
        prefix |= static_cast<uint32_t>(found[0]) << shift;
        mask |= ((1u << bits) - 1u) << shift;
        want -= found[1];
        __syncthreads();
      }
      low = prefix;
      ties = want;
    }
    if (tid == 0) first_gap = len;
    __syncthreads();
    int placed = 0, tied = 0;
#pragma unroll 1
    for (int base = 0; base < len; base += kSelect * kSlots) {
      float x[kSlots];
      bool sure[kSlots], tie[kSlots];
      int at[kSlots], n_tie = 0, all;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        at[s] = base + (wave * kSlots + s) * 64 + lane;
        x[s] = at[s] < len ? w[at[s]] : 0.f;
        const uint32_t image = ordered(x[s]);
        const bool middle = at[s] >= first && at[s] < last;
        sure[s] = at[s] < len && (!middle || image > low);
        tie[s] = middle && image == low;
        n_tie += tie[s];
      }
      // ties in the order of their places: the wavefront's first, then by slots
      const uint64_t under = (1ull << lane) - 1ull;
      int ties_before = 0, mine = 0;
      {
        int total = 0;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) total += __popcll(__ballot(tie[s]));
        const int b = before(lane == 0 ? total : 0, room, all);
        ties_before = tied + __shfl(b, 0);
        tied += all;
      }
      uint64_t in[kSlots];
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const uint64_t t = __ballot(tie[s]);
        const bool enters = sure[s] || (tie[s] && ties_before + __popcll(t & under) < ties);
        ties_before += __popcll(t);
        in[s] = __ballot(enters);
        mine += __popcll(in[s]);
      }
      int place = placed + __shfl(before(lane == 0 ? mine : 0, room, all), 0);
      placed += all;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int to = place + __popcll(in[s] & under);
        if (in[s] >> lane & 1ull) {
          kept[to] = at[s];
          out[to] = x[s];   // (all of these places have been read)
        } else if (at[s] < len && to == at[s]) {
          atomicMin(&first_gap, to);
        }
        place += __popcll(in[s]);
      }
    }
    __syncthreads();
    if (tid == 0) a.begin[seq] = first_gap;
  }
  if (tid == 0) a.e.new_lengths[seq] = now;
  for (int i = now + tid; i < keep; i += kSelect) kept[i] = -1;
  for (int64_t i = now + tid; i < a.e.max_length; i += kSelect) out[i] = 0.f;
}

constexpr int kMove = 512;     // threads that move
constexpr int kInFlight = 8;   // tokens of a thread

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

// A workgroup: a.packs packs of 16 bytes of one head's keys or values, of all of a sequence's tokens.
template <class T>
__global__ __launch_bounds__(kMove) void k_evict_move(EvictArgs a) {
  unsigned b = blockIdx.x;
  const int piece = b % a.pieces;
  b /= a.pieces;
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
    k_evict_select<<<static_cast<unsigned>(e->num_seqs), kSelect, 0, s>>>(a);
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
