// New tokens' keys and values into a paged cache, with the rotation of keys
// and queries on the way.
//
// A pair (x, y) of a head's elements at position t becomes
//     (x cos - y sin, y cos + x sin)
// with the angle's cosine and sine read from tables (so that long positions
// lose nothing to fp32 arguments), in fp32, rounded once to the element type.
// Every element is read once and written once: the call is bound by the
// copy, or by the launch when there are few tokens.  20,000 bf16 tokens of
// 32 query and 2 x 8 key and value heads of 128: 89 us in the kernel, 5.6 TB/s
// (a large copy reaches 4.7 to 5.1); one token: 3 us.  The norm of a head is a sum
// over the lanes that hold it (heads.h); with it 98 us and 4.
#include "heads.h"

namespace {

using gnnshap::bf16_t;
using gnnshap::f16_t;
using gnnshap::load_pack;
using gnnshap::Pack;
using gnnshap::store_pack;

struct AppendArgs {
  gnnshap_cache c;
  gnnshap_new_tokens t;
  int32_t* info;
  int q_heads;   // 0 without queries
};

// One workgroup: the heads y, y + blockDim.y, ... of one token; the thread x
// takes two packs of N elements of a head, which are rotated against each
// other where the pairs are N apart or more, each in itself where they are
// interleaved, and else are copied.  So the two halves of a pair meet in one
// thread's registers, and a head's threads read and write on end.
template <class T, int N, bool NORM>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
  const int64_t t = blockIdx.x;
  const int head = blockIdx.y * blockDim.y + threadIdx.y;
  const int heads = a.q_heads + 2 * a.c.kv_heads;
  if (head >= heads) return;
  const int D = a.c.head_dim, rot = a.t.cos ? a.t.rot_dim : 0, half = rot / 2;
  const int32_t index = a.t.index[t];
  const bool is_q = head < a.q_heads, is_v = head >= a.q_heads + a.c.kv_heads;

  const T* src;
  T* dst;
  if (is_q) {
    src = static_cast<const T*>(a.t.q) + t * a.t.q_token_stride + head * a.t.q_head_stride;
    dst = static_cast<T*>(a.t.q_out) + t * a.t.q_out_token_stride + head * a.t.q_out_head_stride;
  } else {
    if (index < 0) return;
    const int64_t row = a.t.rows ? a.t.rows[t] : t;
    const int64_t pg = index / a.c.page_size, slot = index % a.c.page_size;
    const bool in = row >= 0 && row < a.t.num_rows && pg < a.t.table_width;
    const int64_t page = in ? a.t.table[row * a.t.table_width + pg] : -1;
    if (page < 0 || page >= a.c.num_pages) {
      if (a.info) *a.info = 1;
      return;
    }
    const int h = head - a.q_heads - (is_v ? a.c.kv_heads : 0);
    const int64_t at = page * a.c.page_stride + slot * a.c.slot_stride + h * a.c.head_stride;
    if (is_v) {
      src = static_cast<const T*>(a.t.v) + t * a.t.v_token_stride + h * a.t.v_head_stride;
      dst = static_cast<T*>(a.c.v) + at;
    } else {
      src = static_cast<const T*>(a.t.k) + t * a.t.k_token_stride + h * a.t.k_head_stride;
      dst = static_cast<T*>(a.c.k) + at;
    }
  }

  bool turn = !is_v && rot > 0;
  int64_t pos = 0;
  if (turn) {
    pos = a.t.positions ? a.t.positions[t] : index;
    if (pos < 0) {
      turn = false;
    } else if (pos >= a.t.num_positions) {
      if (a.info) *a.info = 1;
      turn = false;
    }
  }
  const float* cs = turn ? a.t.cos + pos * half : nullptr;
  const float* sn = turn ? a.t.sin + pos * half : nullptr;

  const void* const weight = is_v ? nullptr : is_q ? a.t.q_norm : a.t.k_norm;
  if (NORM && weight) {
    gnnshap::HeadUnits<T, N> x(D, rot, a.t.interleaved);
    x.load(src);
    x.norm(static_cast<const T*>(weight), static_cast<float>(a.t.norm_eps));
    if (turn) x.turn(cs, sn, rot, a.t.interleaved, 1.f);
    x.store(dst);
    return;
  }
  for (int u = threadIdx.x; u < D / (2 * N); u += blockDim.x) {
    if (turn && !a.t.interleaved && u < half / N) {
      const int i = u * N;
      Pack<T, N> x = load_pack<T, N>(src + i), y = load_pack<T, N>(src + half + i);
      const Pack<float, N> c = load_pack<float, N>(cs + i), s = load_pack<float, N>(sn + i);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float xe = static_cast<float>(x.v[e]), ye = static_cast<float>(y.v[e]);
        x.v[e] = static_cast<T>(xe * c.v[e] - ye * s.v[e]);
        y.v[e] = static_cast<T>(ye * c.v[e] + xe * s.v[e]);
      }
      store_pack(dst + i, x);
      store_pack(dst + half + i, y);
      continue;
    }
    // 2 N elements side by side: from 2 N u on, or behind the rotated ones
    const int i = turn && !a.t.interleaved ? rot + 2 * N * (u - half / N) : 2 * N * u;
    Pack<T, 2 * N> x = load_pack<T, 2 * N>(src + i);
    if (turn && a.t.interleaved) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (i + 2 * e < rot) {
          const float c = cs[i / 2 + e], s = sn[i / 2 + e];
          const float xe = static_cast<float>(x.v[2 * e]), ye = static_cast<float>(x.v[2 * e + 1]);
          x.v[2 * e] = static_cast<T>(xe * c - ye * s);
          x.v[2 * e + 1] = static_cast<T>(ye * c + xe * s);
        }
      }
    }
    store_pack(dst + i, x);
  }
}

template <class T, int N>
int launch(const AppendArgs& a, hipStream_t s) {
  const int units = a.c.head_dim / (2 * N);
  const int x = gnnshap::head_lanes(units);
  if (const int st = gnnshap::check_launch(a.t.num_tokens, x)) return st;
  const int heads = a.q_heads + 2 * a.c.kv_heads, y = std::min(256 / x, heads);
  dim3 grid(static_cast<unsigned>(a.t.num_tokens), static_cast<unsigned>(gnnshap::ceil_div(heads, y)));
  {
    GS_TIMED("k_cache_append", s);
    if (a.t.q_norm || a.t.k_norm)
      k_cache_append<T, N, true><<<grid, dim3(x, y), 0, s>>>(a);
    else
      k_cache_append<T, N, false><<<grid, dim3(x, y), 0, s>>>(a);
  }
  GS_LAUNCHED();
  return GNNSHAP_OK;
}

}  // namespace

extern "C" int gnnshap_cache_append(const gnnshap_cache* cache, const gnnshap_new_tokens* t, int32_t* info,
                                    void* stream) {
  using gnnshap::fail;
  GS_TRY_BEGIN
  gnnshap::clear_error();
  if (const int st = gnnshap::check_cache(cache)) return st;
  if (!t || t->num_tokens < 0) return fail(GNNSHAP_EINVAL, "tokens: NULL or a negative number");
  if (t->num_tokens > INT32_MAX)
    return fail(GNNSHAP_EUNSUPPORTED, "%lld tokens in one call", static_cast<long long>(t->num_tokens));
  if (t->cos) {
    if (!t->sin || t->num_positions < 1) return fail(GNNSHAP_EINVAL, "cos without sin or positions");
    if (t->rot_dim < 0 || t->rot_dim % 2 != 0 || t->rot_dim > cache->head_dim)
      return fail(GNNSHAP_EINVAL, "rot_dim %d of head_dim %d", static_cast<int>(t->rot_dim),
                  static_cast<int>(cache->head_dim));
  }
  if ((t->q_norm || t->k_norm) && !(t->norm_eps >= 0.0 && std::isfinite(static_cast<float>(t->norm_eps))))
    return fail(GNNSHAP_EINVAL, "norm_eps %g is negative or not finite in fp32", t->norm_eps);
  if (t->q && (!t->q_out || t->heads < 1)) return fail(GNNSHAP_EINVAL, "queries without heads or q_out");
  if (t->num_rows < 1 || t->table_width < 1) return fail(GNNSHAP_EINVAL, "page table without rows or pages");
  if (t->num_tokens == 0) return GNNSHAP_OK;
  if (!t->k || !t->v || !t->index || !t->table) return fail(GNNSHAP_EINVAL, "NULL array of tokens");
  AppendArgs a;
  a.c = *cache;
  a.t = *t;
  a.info = info;
  a.q_heads = t->q ? t->heads : 0;
  if (gnnshap::ceil_div(a.q_heads + 2 * static_cast<int64_t>(cache->kv_heads), 4) > 65535)
    return fail(GNNSHAP_EUNSUPPORTED, "%d + 2 x %d heads", a.q_heads, static_cast<int>(cache->kv_heads));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int rot = t->cos ? t->rot_dim : 0;
  // 16-byte packs where the rotated half is whole packs, else the widest that fit
  return gnnshap::with_dtype(cache->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    return gnnshap::with_pack<T>(cache->head_dim, rot, [&](auto n) { return launch<T, decltype(n)::value>(a, s); });
  });
  GS_TRY_END
}
