// Gradients of the log probabilities from hidden states, by these and by the
// vocabulary's weights.
//
// With p = e^{x - lse} of the logits x = h w^T, H the entropy and g, g_H the
// incoming gradients of a row,
//     d_j = g (1[j = t] - p_j) - g_H p_j (log p_j + H),
//     dh = d w,  dw = d^T h.
// The logits are not kept by the forward pass: they are computed again (of 16-bit
// elements the same sums; in fp32 a piece's tiles may sum in another order than
// the forward's, by whose rounding their logits then differ), for a piece of the
// vocabulary at a time, whose d is written in the elements' type
// (of 16 bits in two parts, linear.h) and read by the two other products; w and h
// are turned over on the way from LDS to the matrix instructions.  So are three
// products of 2 rows vocabulary width operations each, in 16 bits five, where many
// rows make them bound by the matrix instructions; few rows are bound by reading
// the weights twice and writing their gradient once.
//
// dh sums over the vocabulary, of which several workgroups take parts where the
// tiles are few: each keeps its part of the sum in fp32 over all pieces, and a
// last launch adds the parts up in order.  So do dw's workgroups with the rows,
// where a small vocabulary leaves few tiles (100,000 rows x 41 tokens x 256
// in bf16: 35 us before the join; written at once, with d in one part, 880).
//
// In fp16 d is carried 2^k larger, k from the largest incoming gradient, so that
// its largest elements are below 2^15 and those down to 2^-28 of them keep 11
// bits; of bf16 and fp32 the exponent's range needs none of it.
#include "linear.h"

namespace {

using namespace gnnshap;

template <class P>
__global__ __launch_bounds__(P::kThreads) void k_linear_d(LinearArgs a) {
  using T = typename P::T;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const TileAt tile = tile_at(blockIdx.x, a.tiles_m, a.tiles_n);
  const int64_t v0 = static_cast<int64_t>(tile.m) * P::TM, b0 = static_cast<int64_t>(tile.n) * P::TN;
  P p;
  p.run(lds, Operand{static_cast<const T*>(a.l.weight) + a.v0 * a.l.weight_stride, a.l.weight_stride, a.tokens},
        Operand{a.l.hidden, a.l.hidden_stride, a.l.num_rows}, v0, b0, a.l.width);
  const float scale = a.scale ? a.scale[0] : 1.f;
#pragma unroll
  for (int t = 0; t < P::NT; ++t) {
    const int64_t row = b0 + p.col_of(t), b = row < a.l.num_rows ? row : 0;
    int64_t given = a.l.targets ? a.l.targets[b] : -1;
    if (given >= a.l.vocab) {
      if (a.info) *a.info = 1;
      given = -1;
    }
    const float top = a.l.maximum[b], logs = a.l.log_sum[b];
    const float gl = a.gl && given >= 0 ? a.gl[b] : 0.f;
    const float ge = a.ge ? a.ge[b] : 0.f, ent = a.ge ? a.l.entropy[b] : 0.f;
    const bool none = top == -INFINITY && logs == 0.f;
    given = given < 0 ? -1 : given - a.v0 - v0;
    float d[P::kRuns][P::kRun];
#pragma unroll
    for (int j = 0; j < P::kRuns; ++j)
#pragma unroll
      for (int i = 0; i < P::kRun; ++i) {
        const int at = p.run_of(j) + i;
        const float logp = (p.at(j, i, t) - top) - logs, e = __builtin_amdgcn_exp2f(logp * kLog2e);
        const float own = at == given ? gl : 0.f;
        d[j][i] = own - e * (gl + ge * ((e == 0.f ? 0.f : logp) + ent));
        if (none || v0 + at >= a.tokens) d[j][i] = 0.f;  // behind the piece, to the tile's end: the products read it
        d[j][i] *= scale;
      }
    T* const out = static_cast<T*>(a.d) + a.d0 + v0;
    p.template rows_out<T>(lds, t, [&](int j, int i) { return static_cast<T>(d[j][i]); }, [&](int n, int m, const auto& x) {
      if (b0 + n < a.l.num_rows) store_pack(out + (b0 + n) * a.pitch + m, x);
    });
    if (a.two)
      p.template rows_out<T>(
          lds, t,
          [&](int j, int i) {
            const float rest = d[j][i] - static_cast<float>(static_cast<T>(d[j][i]));
            return static_cast<T>(rest == rest ? rest : 0.f);  // an infinite d stays one
          },
          [&](int n, int m, const auto& x) {
            if (b0 + n < a.l.num_rows) store_pack(out + (a.l.num_rows + b0 + n) * a.pitch + m, x);
          });
  }
}

// A product whose K is split: dh's always, dw's of few tiles and many rows.
struct SplitArgs {
  const void* a;        // turned over
  int64_t a_stride;
  const void* d;
  int64_t pitch;
  int64_t K, rows, width;  // rows of the result, elements of a row
  int segments;            // d's parts, of which each starts `d_part` bytes behind the one before
  int64_t d_part;
  unsigned tiles_m, tiles_n;
  int64_t split;        // of K, a workgroup
  float* sums;          // [split][row][width]
  bool first;           // or: add to what is there
};

// The parts of dh (d by rows) or dw (d turned over): a tile's rows are elements
// of the width, its columns rows of the result.
template <class P>
__global__ __launch_bounds__(P::kThreads) void k_linear_parts(SplitArgs a) {
  using T = typename P::T;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const unsigned tiles = a.tiles_m * a.tiles_n, part = blockIdx.x / tiles;
  const TileAt tile = tile_at(blockIdx.x - part * tiles, a.tiles_m, a.tiles_n);
  const int64_t m0 = static_cast<int64_t>(tile.m) * P::TM, n0 = static_cast<int64_t>(tile.n) * P::TN;
  const int64_t k0 = part * a.split, K = a.K - k0 < a.split ? a.K - k0 : a.split;
  P p;
  p.run(lds, Operand{static_cast<const T*>(a.a) + k0 * a.a_stride, a.a_stride, a.width},
        Operand{static_cast<const T*>(a.d) + (P::kTurnedB ? k0 * a.pitch : k0), a.pitch, a.rows}, m0, n0, K > 0 ? K : 0,
        a.segments, 0, a.d_part);
#pragma unroll
  for (int t = 0; t < P::NT; ++t)
    p.template rows_out<float>(lds, t, [&](int j, int i) { return p.at(j, i, t); }, [&](int n, int m, const auto& x) {
      const int64_t row = n0 + n, at = m0 + m;
      if (row >= a.rows || at >= a.width) return;
      float* const out = a.sums + (part * a.rows + row) * a.width + at;
      const int there = a.width - at < 4 ? static_cast<int>(a.width - at) : 4;
      if (there == 4) {
        Pack<float, 4> y = x;
        if (!a.first) {
          const Pack<float, 4> z = load_pack<float, 4>(out);
#pragma unroll
          for (int e = 0; e < 4; ++e) y.v[e] += z.v[e];
        }
        store_pack(out, y);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < there) out[e] = a.first ? x.v[e] : x.v[e] + out[e];
      }
    });
}

struct JoinArgs {
  const float* sums;
  int64_t parts, rows, width;
  bool two;             // row b's second part is row rows / 2 + b
  const float* scale;
  void* out;
  int64_t stride;
};

// Adds up the parts: four elements to a thread, and (few rows) WAYS threads to
// these, each with every WAYS-th part (16 rows of 1,024 in 32 parts: 12.7 us with one, 4.0 with eight).
template <class T, int WAYS>
__global__ __launch_bounds__(256) void k_linear_parts_join(JoinArgs a) {
  constexpr int kPacks = 256 / WAYS;
  __shared__ float sums[WAYS][kPacks][4];
  const int64_t packs = (a.width + 3) / 4, rows = a.two ? a.rows / 2 : a.rows;
  const int way = threadIdx.x / kPacks, mine = threadIdx.x % kPacks;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kPacks + mine;
  const bool in = i < rows * packs;
  const int64_t row = in ? i / packs : 0, m = in ? (i - row * packs) * 4 : 0;
  const int n = a.width - m < 4 ? static_cast<int>(a.width - m) : 4;
  // the second parts of d's rows are parts like others
  const int64_t all = a.two ? 2 * a.parts : a.parts;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  const auto part_at = [&](int64_t p) {
    return a.sums + (a.two ? (p >> 1) * a.rows + (p & 1) * rows + row : p * a.rows + row) * a.width + m;
  };
  if (in && n == 4) {
#pragma unroll 8
    for (int64_t p = way; p < all; p += WAYS) {
      const Pack<float, 4> x = load_pack<float, 4>(part_at(p));
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += x.v[e];
    }
  } else if (in) {
    for (int64_t p = way; p < all; p += WAYS)
      for (int e = 0; e < n; ++e) s[e] += part_at(p)[e];
  }
  if constexpr (WAYS > 1) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[way][mine][e] = s[e];
    __syncthreads();
    if (way > 0) return;
#pragma unroll
    for (int w = 1; w < WAYS; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += sums[w][mine][e];
  }
  if (!in) return;
  const float over = a.scale ? a.scale[1] : 1.f;
  T* const out = static_cast<T*>(a.out) + row * a.stride + m;
  if (n == 4) {
    Pack<T, 4> x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x.v[e] = static_cast<T>(s[e] * over);
    store_pack(out, x);
  } else {
    for (int e = 0; e < n; ++e) out[e] = static_cast<T>(s[e] * over);
  }
}

struct WeightArgs {
  const void* hidden;
  int64_t hidden_stride;
  const void* d;
  int64_t pitch;
  int64_t piece, rows, width;  // rows of the hidden states
  int segments;                // as in SplitArgs
  int64_t d_part;
  unsigned tiles_m, tiles_n;
  const float* scale;
  void* out;            // of the piece
  int64_t stride;
};

// dw: a tile's rows are elements of the width, its columns tokens.  Written past
// the caches (fp32, 16 rows x 32,768 tokens x 2,048: d and dw 171 us by way of
// them, 89 past them; bf16: 73 and 61).
template <class P>
__global__ __launch_bounds__(P::kThreads) void k_linear_dw(WeightArgs a) {
  using T = typename P::T;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const TileAt tile = tile_at(blockIdx.x, a.tiles_m, a.tiles_n);
  const int64_t m0 = static_cast<int64_t>(tile.m) * P::TM, n0 = static_cast<int64_t>(tile.n) * P::TN;
  P p;
  p.run(lds, Operand{a.hidden, a.hidden_stride, a.width}, Operand{a.d, a.pitch, a.piece}, m0, n0, a.rows, a.segments,
        0, a.d_part);
  const float over = a.scale ? a.scale[1] : 1.f;
  constexpr int kPack = 16 / sizeof(T);
  static_assert(P::kRun >= kPack, "a lane's run is whole packs");
#pragma unroll
  for (int t = 0; t < P::NT; ++t)
    p.template rows_out<T>(lds, t, [&](int j, int i) { return static_cast<T>(p.at(j, i, t) * over); },
                           [&](int n, int m, const auto& x) {
                             const int64_t token = n0 + n, at = m0 + m;
                             if (token >= a.piece || at >= a.width) return;
                             T* const out = static_cast<T*>(a.out) + token * a.stride + at;
                             if (at + kPack <= a.width) {
                               stream_pack(out, x);
                             } else {
#pragma unroll
                               for (int e = 0; e < kPack; ++e)
                                 if (at + e < a.width) out[e] = x.v[e];
                             }
                           });
}

// The power of two that d is carried larger by, and one over it: |d| is at most
// 2 |g| + |g_H| (H + 1), of which the largest comes to 2^14 .. 2^15.
__global__ __launch_bounds__(1024) void k_linear_scale(LinearArgs a, float* scale) {
  __shared__ float most[16];
  float m = 0.f;
  for (int64_t b = threadIdx.x; b < a.l.num_rows; b += 1024) {
    float x = a.gl ? 2.f * fabsf(a.gl[b]) : 0.f;
    if (a.ge) x += fabsf(a.ge[b]) * (fabsf(a.l.entropy[b]) + 1.f);
    if (x < INFINITY) m = fmaxf(m, x);
  }
  for (int off = 1; off < 64; off *= 2) m = fmaxf(m, __shfl_xor(m, off));
  if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int i = 1; i < 16; ++i) m = fmaxf(m, most[i]);
  int e = 0;
  if (m > 0.f) frexpf(m, &e);
  const int k = m > 0.f ? max(-100, min(100, 15 - e)) : 0;
  scale[0] = ldexpf(1.f, k);
  scale[1] = ldexpf(1.f, -k);
}

// The weights and the hidden states turned over: their packs lie along the width.
template <class T>
bool direct_weight(const gnnshap_linear& l) {
  return direct_operand<T>(l.weight, l.weight_stride, l.width, 256);
}
template <class T>
bool direct_hidden(const gnnshap_linear& l) {
  return direct_operand<T>(l.hidden, l.hidden_stride, l.width, 256);
}

size_t carve(Layout& y, const gnnshap_linear& l, void* ws) {
  Carver c(ws);
  y.scale = c.take<float>(2);
  y.d = c.take<char>(static_cast<size_t>(y.d_rows) * y.pitch * (l.dtype == GNNSHAP_F32 ? 4 : 2));
  y.sums = c.take<float>(static_cast<size_t>(y.parts) * y.hidden_rows * l.width);
  if (y.weight_parts > 1)
    y.weight_sums = c.take<float>(static_cast<size_t>(y.weight_parts) * std::min(y.piece, l.vocab) * l.width);
  return c.bytes();
}

template <class P, class A>
int launch(void (*kernel)(A), const char* name, const A& a, int64_t workgroups, int lds, hipStream_t s) {
  if (const int st = check_launch(workgroups, P::kThreads)) return st;
  GS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, P::kLds));
  {
    GS_TIMED(name, s);
    kernel<<<static_cast<unsigned>(workgroups), P::kThreads, lds, s>>>(a);
  }
  GS_LAUNCHED();
  return GNNSHAP_OK;
}

template <class T>
int join(const JoinArgs& j, hipStream_t s) {
  const int64_t packs = (j.two ? j.rows / 2 : j.rows) * ceil_div(j.width, 4);
  const bool few = j.parts > 8 && packs < 65536;
  const int64_t groups = ceil_div(packs, few ? 32 : 256);
  if (const int st = check_launch(groups, 256)) return st;
  {
    GS_TIMED("k_linear_parts_join", s);
    if (few)
      k_linear_parts_join<T, 8><<<static_cast<unsigned>(groups), 256, 0, s>>>(j);
    else
      k_linear_parts_join<T, 1><<<static_cast<unsigned>(groups), 256, 0, s>>>(j);
  }
  GS_LAUNCHED();
  return GNNSHAP_OK;
}

template <class T>
int run(const LinearArgs& given, void* grad_hidden, int64_t gh_stride, void* grad_weight, int64_t gw_stride,
        Layout y, hipStream_t s) {
  const gnnshap_linear& l = given.l;
  LinearArgs a = given;
  if (l.dtype == GNNSHAP_F16 && l.num_rows > 0) {
    {
      GS_TIMED("k_linear_scale", s);
      k_linear_scale<<<1, 1024, 0, s>>>(a, y.scale);
    }
    GS_LAUNCHED();
    a.scale = y.scale;
  }
  a.d = y.d;
  a.pitch = y.pitch;
  a.two = y.two;
  const bool direct_logits_too = direct_logits<T>(l);
  const bool direct_w = direct_weight<T>(l), direct_h = direct_hidden<T>(l);
  const int64_t d_part = l.num_rows * y.pitch * static_cast<int64_t>(sizeof(T));
  for (int64_t v0 = 0; v0 < l.vocab; v0 += y.piece) {
    const int64_t piece = std::min(y.piece, l.vocab - v0);
    int st = GNNSHAP_OK;
    Segment segment[2];
    if (l.num_rows > 0) {
      const int segments = logit_segments(piece, l, sizeof(T), direct_logits_too, segment);
      for (int i = 0; i < segments; ++i) {
        a.v0 = v0 + segment[i].begin;
        a.tokens = segment[i].tokens;
        a.d0 = segment[i].begin;
        st = with_logits<T>(segment[i].shape, direct_logits_too, [&](auto* p) {
          using P = std::remove_pointer_t<decltype(p)>;
          a.tiles_m = static_cast<unsigned>(ceil_div(a.tokens, P::TM));
          a.tiles_n = static_cast<unsigned>(ceil_div(l.num_rows, P::TN));
          return launch<P>(k_linear_d<P>, "k_linear_d", a, static_cast<int64_t>(a.tiles_m) * a.tiles_n,
                           P::lds_for(l.width, 1), s);
        });
        if (st) return st;
      }
    }
    if (grad_hidden && l.num_rows > 0) {
      st = with_shape<T, true, false, kHiddenShapes>(y.hidden_shape, direct_w, [&](auto* p) {
        using P = std::remove_pointer_t<decltype(p)>;
        SplitArgs h{static_cast<const T*>(l.weight) + v0 * l.weight_stride, l.weight_stride, y.d, y.pitch, piece, y.hidden_rows,
                    l.width, y.hidden_segments, d_part, static_cast<unsigned>(ceil_div(l.width, P::TM)),
                    static_cast<unsigned>(ceil_div(y.hidden_rows, P::TN)), y.split, y.sums, v0 == 0};
        return launch<P>(k_linear_parts<P>, "k_linear_dh", h, y.parts * h.tiles_m * h.tiles_n,
                         P::lds_for(y.split, y.hidden_segments), s);
      });
      if (st) return st;
    }
    if (grad_weight && y.weight_parts > 1) {
      st = with_shape<T, true, true, kWeightShapes>(y.weight_shape, direct_h, [&](auto* p) {
        using P = std::remove_pointer_t<decltype(p)>;
        SplitArgs w{l.hidden, l.hidden_stride, y.d, y.pitch, l.num_rows, piece, l.width, y.weight_segments, d_part,
                    static_cast<unsigned>(ceil_div(l.width, P::TM)), static_cast<unsigned>(ceil_div(piece, P::TN)),
                    y.weight_split, y.weight_sums, true};
        return launch<P>(k_linear_parts<P>, "k_linear_dw", w, y.weight_parts * w.tiles_m * w.tiles_n,
                         P::lds_for(y.weight_split, y.weight_segments), s);
      });
      if (!st)
        st = join<T>(JoinArgs{y.weight_sums, y.weight_parts, piece, l.width, false, a.scale,
                              static_cast<T*>(grad_weight) + v0 * gw_stride, gw_stride}, s);
      if (st) return st;
    } else if (grad_weight) {
      const int segments = weight_segments_for(piece, l, sizeof(T), y.weight_segments, direct_h, segment);
      for (int i = 0; i < segments && !st; ++i)
        st = with_shape<T, true, true, kWeightShapes>(segment[i].shape, direct_h, [&](auto* p) {
          using P = std::remove_pointer_t<decltype(p)>;
          WeightArgs w{l.hidden, l.hidden_stride, static_cast<const T*>(y.d) + segment[i].begin, y.pitch, segment[i].tokens,
                       l.num_rows, l.width, y.weight_segments, d_part, static_cast<unsigned>(ceil_div(l.width, P::TM)),
                       static_cast<unsigned>(ceil_div(segment[i].tokens, P::TN)), a.scale,
                       static_cast<T*>(grad_weight) + (v0 + segment[i].begin) * gw_stride, gw_stride};
          return launch<P>(k_linear_dw<P>, "k_linear_dw", w, static_cast<int64_t>(w.tiles_m) * w.tiles_n,
                           P::lds_for(l.num_rows, y.weight_segments), s);
        });
      if (st) return st;
    }
  }
  if (grad_hidden && l.num_rows > 0)
    return join<T>(JoinArgs{y.sums, y.parts, y.hidden_rows, l.width, y.beside, a.scale, grad_hidden, gh_stride}, s);
  return GNNSHAP_OK;
}

}  // namespace

extern "C" int gnnshap_linear_logprobs_backward_workspace(const gnnshap_linear* l, size_t* bytes) {
  GS_TRY_BEGIN
  clear_error();
  if (!bytes) return fail(GNNSHAP_EINVAL, "bytes is NULL");
  if (const int st = check_linear(l)) return st;
  return with_dtype(l->dtype, [&](auto* x) {
    *bytes = 0;
    for (const int direct : {0, 1, 2, 3}) {  // as the call's addresses will have it
      Layout y = lay_out(*l, sizeof(std::remove_pointer_t<decltype(x)>), direct & 1, direct & 2);
      *bytes = std::max(*bytes, carve(y, *l, nullptr));
    }
    return static_cast<int>(GNNSHAP_OK);
  });
  GS_TRY_END
}

extern "C" int gnnshap_linear_logprobs_backward(const gnnshap_linear* l, const float* g_logprob, const float* g_entropy,
                                                void* grad_hidden, int64_t grad_hidden_stride, void* grad_weight,
                                                int64_t grad_weight_stride, int32_t* info, void* ws, size_t ws_bytes,
                                                void* stream) {
  GS_TRY_BEGIN
  clear_error();
  if (const int st = check_linear(l)) return st;
  if (grad_hidden_stride < 0 || grad_weight_stride < 0) return fail(GNNSHAP_EINVAL, "negative stride of a gradient");
  if (l->num_rows > 0 &&
      (!l->hidden || !l->weight || !l->maximum || !l->log_sum || (g_entropy && !l->entropy)))
    return fail(GNNSHAP_EINVAL, "NULL hidden, weight, maximum, log_sum or (with g_entropy) entropy");
  if (!grad_hidden && !grad_weight) return GNNSHAP_OK;
  LinearArgs a{};
  a.l = *l;
  a.gl = g_logprob;
  a.ge = g_entropy;
  a.info = info;
  return with_dtype(l->dtype, [&](auto* x) {
    using T = std::remove_pointer_t<decltype(x)>;
    Layout y = lay_out(*l, sizeof(T), direct_weight<T>(*l), direct_hidden<T>(*l));
    const size_t need = carve(y, *l, ws);
    if (!ws || ws_bytes < need)
      return fail(GNNSHAP_ECAPACITY, "linear_logprobs_backward workspace needs %zu bytes, has %zu", need,
                  ws ? ws_bytes : 0);
    return run<T>(a, grad_hidden, grad_hidden_stride, grad_weight, grad_weight_stride, y,
                  static_cast<hipStream_t>(stream));
  });
  GS_TRY_END
}
