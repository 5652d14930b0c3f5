// Log probabilities of given tokens and entropies straight from hidden states
// and the vocabulary's weights.
//
// The logits are a product, hidden weight^T, of which a workgroup computes a
// tile; what it keeps of it are each row's statistics over the tile's tokens
// (the largest logit m, s = sum e^{x - m} and w = sum e^{x - m} (x - m), stats.h)
// and the given token's logit.  A second launch adds up a row's statistics:
//     lse = m + log s,  log p = (x_t - m) - log s,  H = log s - w / s.
// Many rows are bound by the matrix instructions, few by reading the weights.
#include "linear.h"

namespace {

using namespace gnnshap;

template <class P>
__global__ __launch_bounds__(P::kThreads) void k_linear_stats(LinearArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const TileAt tile = tile_at(blockIdx.x, a.tiles_m, a.tiles_n);
  const int64_t v0 = static_cast<int64_t>(tile.m) * P::TM, b0 = static_cast<int64_t>(tile.n) * P::TN;
  P p;
  p.run(lds, Operand{static_cast<const typename P::T*>(a.l.weight) + a.v0 * a.l.weight_stride, a.l.weight_stride, a.tokens},
        Operand{a.l.hidden, a.l.hidden_stride, a.l.num_rows}, v0, b0, a.l.width);
  const int lane = threadIdx.x & 63;
  const int64_t left = a.tokens - v0;
  Stats* const mine = reinterpret_cast<Stats*>(lds) + p.wave_m() / (16 * P::MT) * P::TN;
#pragma unroll
  for (int t = 0; t < P::NT; ++t) {
    const int64_t row = b0 + p.col_of(t);
    float f[P::kRuns][P::kRun], most = -INFINITY;
#pragma unroll
    for (int j = 0; j < P::kRuns; ++j)
#pragma unroll
      for (int i = 0; i < P::kRun; ++i) {
        f[j][i] = p.at(j, i, t);
        if (left < P::TM && p.run_of(j) + i >= left) f[j][i] = -INFINITY;
        most = fmaxf(most, f[j][i]);
      }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    const float use = finite_max(most);
    float s = 0.f, w = 0.f;
#pragma unroll
    for (int j = 0; j < P::kRuns; ++j)
#pragma unroll
      for (int i = 0; i < P::kRun; ++i) {
        const float d = (f[j][i] - use) * kLog2e, e = __builtin_amdgcn_exp2f(d);
        s += e;
        w += e * fmaxf(d, -200.f);
      }
    s += __shfl_xor(s, 16);
    w += __shfl_xor(w, 16);
    s += __shfl_xor(s, 32);
    w += __shfl_xor(w, 32);
    if (lane < 16) mine[p.col_of(t)] = Stats{most, s, w};
    int64_t given = a.l.targets && row < a.l.num_rows ? a.l.targets[row] : -1;
    given = given < 0 ? -1 : given - a.v0 - v0;
    if (__ballot(given >= p.wave_m() && given < p.wave_m() + 16 * P::MT)) {
#pragma unroll
      for (int j = 0; j < P::kRuns; ++j)
#pragma unroll
        for (int i = 0; i < P::kRun; ++i)
          if (given == p.run_of(j) + i) a.given[row] = f[j][i];
    }
  }
  __syncthreads();
  for (int n = threadIdx.x; n < P::TN; n += P::kThreads) {
    if (b0 + n >= a.l.num_rows) break;
    const Stats* const s = reinterpret_cast<const Stats*>(lds) + n;
    Stats st = s[0];
    for (int i = 1; i < P::TM / (16 * P::MT); ++i) add(st, s[i * P::TN]);
    a.parts[(b0 + n) * a.row_parts + a.part0 + tile.m] = st;
  }
}

// Adds up a row's statistics, PER_ROW wavefronts to a row.
template <int PER_ROW>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs a) {
  __shared__ Stats stats[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (4 / PER_ROW) + wave / PER_ROW;
  if (row >= a.l.num_rows) return;
  Stats st = no_stats();
  for (unsigned i = wave % PER_ROW * 64 + lane; i < a.row_parts; i += 64 * PER_ROW) add(st, a.parts[row * a.row_parts + i]);
  wave_sum(st);
  if constexpr (PER_ROW > 1) {
    if (lane == 0) stats[wave] = st;
    __syncthreads();
    st = stats[0];
    for (int i = 1; i < PER_ROW; ++i) add(st, stats[i]);
  }
  if (lane > 0 || wave % PER_ROW > 0) return;
  const int64_t t = a.l.targets ? a.l.targets[row] : -1;
  const bool has = t >= 0 && t < a.l.vocab, none = st.s == 0.f;
  if (t >= a.l.vocab && a.info) *a.info = 1;
  const float logs = logf(st.s);
  if (a.l.lse) a.l.lse[row] = none ? -INFINITY : st.m + logs;
  if (a.l.maximum) a.l.maximum[row] = st.m;
  if (a.l.log_sum) a.l.log_sum[row] = none ? 0.f : logs;
  if (a.l.entropy) a.l.entropy[row] = none ? 0.f : logs - kLn2 * (st.w / st.s);
  if (a.l.logprob) a.l.logprob[row] = !has ? 0.f : none ? -INFINITY : (a.given[row] - st.m) - logs;
}

size_t carve(LinearArgs& a, void* ws) {
  Carver c(ws);
  a.parts = c.take<Stats>(static_cast<size_t>(a.l.num_rows) * a.row_parts);
  a.given = c.take<float>(static_cast<size_t>(a.l.num_rows));
  return c.bytes();
}

// The call's segments and a row's parts; a refusal of more workgroups than a launch takes.
template <class T>
int lay_out(LinearArgs& a, bool direct, Segment (&s)[2], int& segments) {
  segments = logit_segments(a.l.vocab, a.l, sizeof(T), direct, s);
  int64_t parts = 0;
  for (int i = 0; i < segments; ++i) {
    const int64_t m = ceil_div(s[i].tokens, kTileM[s[i].shape]), n = ceil_div(a.l.num_rows, kTileN[s[i].shape]);
    if (const int st = check_launch(m * n, 512)) return st;
    parts += m;
  }
  a.row_parts = static_cast<unsigned>(parts);
  return check_launch(a.l.num_rows, 64);
}

template <class P>
int launch(const LinearArgs& a, hipStream_t s) {
  GS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(k_linear_stats<P>), hipFuncAttributeMaxDynamicSharedMemorySize,
                             P::kLds));
  {
    GS_TIMED("k_linear_stats", s);
    k_linear_stats<P><<<a.tiles_m * a.tiles_n, P::kThreads, P::kLds, s>>>(a);
  }
  GS_LAUNCHED();
  return GNNSHAP_OK;
}

template <class T>
int run(LinearArgs a, bool direct, const Segment (&segment)[2], int segments, hipStream_t s) {
  for (int i = 0; i < segments; ++i) {
    a.v0 = segment[i].begin;
    a.tokens = segment[i].tokens;
    const int st = with_logits<T>(segment[i].shape, direct, [&](auto* p) {
      using P = std::remove_pointer_t<decltype(p)>;
      a.tiles_m = static_cast<unsigned>(ceil_div(a.tokens, P::TM));
      a.tiles_n = static_cast<unsigned>(ceil_div(a.l.num_rows, P::TN));
      return launch<P>(a, s);
    });
    if (st) return st;
    a.part0 += a.tiles_m;
  }
  {
    GS_TIMED("k_linear_join", s);
    if (a.row_parts > 64 && a.l.num_rows < 1024)
      k_linear_join<4><<<static_cast<unsigned>(a.l.num_rows), 256, 0, s>>>(a);
    else
      k_linear_join<1><<<static_cast<unsigned>(ceil_div(a.l.num_rows, 4)), 256, 0, s>>>(a);
  }
  GS_LAUNCHED();
  return GNNSHAP_OK;
}

}  // namespace

int gnnshap::check_linear(const gnnshap_linear* l) {
  if (!l) return fail(GNNSHAP_EINVAL, "linear is NULL");
  if (l->dtype < GNNSHAP_F32 || l->dtype > GNNSHAP_BF16)
    return fail(GNNSHAP_EUNSUPPORTED, "dtype %d is not one of f32, f16, bf16", static_cast<int>(l->dtype));
  if (l->num_rows < 0 || l->vocab < 1 || l->width < 1)
    return fail(GNNSHAP_EINVAL, "%lld rows of width %lld over %lld tokens", static_cast<long long>(l->num_rows),
                static_cast<long long>(l->width), static_cast<long long>(l->vocab));
  if (l->num_rows > (int64_t(1) << 30) || l->vocab > (int64_t(1) << 30) || l->width > (int64_t(1) << 24))
    return fail(GNNSHAP_EUNSUPPORTED, "%lld rows of width %lld over %lld tokens", static_cast<long long>(l->num_rows),
                static_cast<long long>(l->width), static_cast<long long>(l->vocab));
  if (l->hidden_stride < 0 || l->weight_stride < 0) return fail(GNNSHAP_EINVAL, "negative row stride");
  return GNNSHAP_OK;
}

extern "C" int gnnshap_linear_logprobs_workspace(const gnnshap_linear* l, size_t* bytes) {
  GS_TRY_BEGIN
  clear_error();
  if (!bytes) return fail(GNNSHAP_EINVAL, "bytes is NULL");
  if (const int st = check_linear(l)) return st;
  *bytes = 0;
  if (l->num_rows == 0) return GNNSHAP_OK;
  return with_dtype(l->dtype, [&](auto* x) {
    using T = std::remove_pointer_t<decltype(x)>;
    for (const bool direct : {true, false}) {  // as the call's addresses will have it
      LinearArgs a{};
      a.l = *l;
      Segment segment[2];
      int segments;
      if (const int st = lay_out<T>(a, direct, segment, segments)) return st;
      *bytes = std::max(*bytes, carve(a, nullptr));
    }
    return static_cast<int>(GNNSHAP_OK);
  });
  GS_TRY_END
}

extern "C" int gnnshap_linear_logprobs(const gnnshap_linear* l, int32_t* info, void* ws, size_t ws_bytes,
                                       void* stream) {
  GS_TRY_BEGIN
  clear_error();
  if (const int st = check_linear(l)) return st;
  if (l->num_rows == 0) return GNNSHAP_OK;
  if (!l->hidden || !l->weight) return fail(GNNSHAP_EINVAL, "NULL hidden states or weights");
  return with_dtype(l->dtype, [&](auto* x) {
    using T = std::remove_pointer_t<decltype(x)>;
    const bool direct = direct_logits<T>(*l);
    LinearArgs a{};
    a.l = *l;
    a.info = info;
    Segment segment[2];
    int segments;
    if (const int st = lay_out<T>(a, direct, segment, segments)) return st;
    const size_t need = carve(a, ws);
    if (!ws || ws_bytes < need)
      return fail(GNNSHAP_ECAPACITY, "linear_logprobs workspace needs %zu bytes, has %zu", need, ws ? ws_bytes : 0);
    return run<T>(a, direct, segment, segments, static_cast<hipStream_t>(stream));
  });
  GS_TRY_END
}
