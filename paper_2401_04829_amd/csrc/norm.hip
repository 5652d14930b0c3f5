// Norm and rotation of queries' and keys' heads, and their gradients.
//
// Per head, with r = 1 / sqrt(mean x^2 + eps) and R(p) the rotation by the
// position's angles:
//     y = R(p) (x r w)
//     z = R(-p) dy,  dx = r (z w - x r mean(z w x r)),  dw = sum z x r.
// r is found again in the gradient: x is read there anyway.  A head is spread
// over the lanes of one wavefront (heads.h), which read and write on end;
// sums over a head are moves between these lanes.  Everything is read once
// and written once.  The weights' gradient stays in the lanes' registers over
// all of a workgroup's heads, is added up in LDS, then by a second launch over
// the workgroups, always in the same order; of fp32 heads in 64 bits, as every
// chain of 32 additions in 32 bits would leave about 1.4e-7 (500 tokens of 8 heads of 64:
// 2.2e-7 off with all three chains in 32 bits).  Bound by memory: 16,384 bf16 tokens
// of 32 + 8 heads of 128: 61 us forward (336 MB, 5.5 TB/s), 109 us backward (503 MB,
// 4.6 TB/s) and 4 to add up.
#include "heads.h"

namespace {

using namespace gnnshap;

// What the weights' gradients are summed in.
template <class T>
using Sum = std::conditional_t<std::is_same_v<T, float>, double, float>;

struct NormArgs {
  gnnshap_normed n;
  gnnshap_heads grad[2];  // of queries and keys
  void* part[2];          // [workgroup][head_dim] of the weights' gradients, of type Sum<T>
  int groups[2];          // workgroups that take the queries, the keys
  void* dw[2];
  int32_t* info;
};

// The angles of a token; NULL: it is not rotated.
__device__ __forceinline__ const float* angles_of(const NormArgs& a, int64_t t, const float*& sn) {
  if (!a.n.cos || a.n.rot_dim == 0) return nullptr;
  const int64_t pos = a.n.positions ? a.n.positions[t] : t;
  if (pos < 0) return nullptr;
  if (pos >= a.n.num_positions) {
    if (a.info) *a.info = 1;
    return nullptr;
  }
  sn = a.n.sin + pos * (a.n.rot_dim / 2);
  return a.n.cos + pos * (a.n.rot_dim / 2);
}

template <class T, int N>
__global__ __launch_bounds__(256) void k_norm_rotate(NormArgs a) {
  const int64_t t = blockIdx.x;
  const int i = blockIdx.y * blockDim.y + threadIdx.y, q_heads = a.n.q.heads;
  if (i >= q_heads + a.n.k.heads) return;
  const bool is_q = i < q_heads;
  const gnnshap_heads& h = is_q ? a.n.q : a.n.k;
  const int head = is_q ? i : i - q_heads, rot = a.n.cos ? a.n.rot_dim : 0;
  HeadUnits<T, N> x(a.n.head_dim, rot, a.n.interleaved);
  x.load(static_cast<const T*>(h.x) + t * h.token_stride + head * h.head_stride);
  const float *sn = nullptr, *const cs = angles_of(a, t, sn);
  x.norm(static_cast<const T*>(is_q ? a.n.q_norm : a.n.k_norm), static_cast<float>(a.n.eps));
  if (cs) x.turn(cs, sn, rot, a.n.interleaved, 1.f);
  x.store(static_cast<T*>(h.out) + t * h.out_token_stride + head * h.out_head_stride);
}

// The first groups[0] workgroups take the queries' heads, the others the keys'.
template <class T, int N>
__global__ __launch_bounds__(256) void k_norm_rotate_grad(NormArgs a) {
  using Units = HeadUnits<T, N>;
  __shared__ Sum<T> sums[256 * Units::kUnits * 2 * N];
  const bool is_k = static_cast<int>(blockIdx.x) >= a.groups[0];
  const int group = is_k ? blockIdx.x - a.groups[0] : blockIdx.x, groups = a.groups[is_k];
  const gnnshap_heads& h = is_k ? a.n.k : a.n.q;
  const gnnshap_heads& g = a.grad[is_k];
  const T* const weight = static_cast<const T*>(is_k ? a.n.k_norm : a.n.q_norm);
  const int D = a.n.head_dim, rot = a.n.cos ? a.n.rot_dim : 0;
  Units w(D, rot, a.n.interleaved);
  Sum<T> dw[Units::kUnits][2 * N];
  if (weight) w.load(weight);
#pragma unroll
  for (int j = 0; j < Units::kUnits; ++j)
#pragma unroll
    for (int e = 0; e < 2 * N; ++e) {
      if (!weight) w.v[j][e] = 1.f;
      dw[j][e] = 0;
    }
  // the workgroups' heads in turn; from one to the next `on` tokens and `heads_on` heads further
  const int64_t first = static_cast<int64_t>(group) * blockDim.y + threadIdx.y;
  const int64_t step = static_cast<int64_t>(groups) * blockDim.y, on = step / h.heads;
  const int heads_on = static_cast<int>(step - on * h.heads);
  int64_t t = first / h.heads;
  int head = static_cast<int>(first - t * h.heads);
  for (; t < a.n.num_tokens; t += on, head += heads_on) {
    if (head >= h.heads) {
      head -= h.heads;
      if (++t >= a.n.num_tokens) break;
    }
    Units x = w, z = w;
    x.load(static_cast<const T*>(h.x) + t * h.token_stride + head * h.head_stride);
    z.load(static_cast<const T*>(g.x) + t * g.token_stride + head * g.head_stride);
    const float *sn = nullptr, *const cs = angles_of(a, t, sn);
    const float r = x.over_root(static_cast<float>(a.n.eps));
    if (cs) z.turn(cs, sn, rot, a.n.interleaved, -1.f);
    float along = 0.f;
#pragma unroll
    for (int j = 0; j < Units::kUnits; ++j)
#pragma unroll
      for (int e = 0; e < 2 * N; ++e) {
        x.v[j][e] *= r;
        dw[j][e] += static_cast<Sum<T>>(z.v[j][e]) * x.v[j][e];
        z.v[j][e] *= w.v[j][e];
        along += z.v[j][e] * x.v[j][e];
      }
    along = head_sum(along) / D;
#pragma unroll
    for (int j = 0; j < Units::kUnits; ++j)
#pragma unroll
      for (int e = 0; e < 2 * N; ++e) z.v[j][e] = r * (z.v[j][e] - x.v[j][e] * along);
    z.store(static_cast<T*>(g.out) + t * g.out_token_stride + head * g.out_head_stride);
  }
  if (!a.dw[is_k]) return;
#pragma unroll
  for (int j = 0; j < Units::kUnits; ++j)
#pragma unroll
    for (int e = 0; e < 2 * N; ++e)
      if (w.at[j][0] >= 0) sums[threadIdx.y * D + w.at[j][e / N] + e % N] = dw[j][e];
  __syncthreads();
  for (int d = threadIdx.y * blockDim.x + threadIdx.x; d < D; d += blockDim.x * blockDim.y) {
    Sum<T> s = 0;
    for (unsigned y = 0; y < blockDim.y; ++y) s += sums[y * D + d];
    static_cast<Sum<T>*>(a.part[is_k])[static_cast<int64_t>(group) * D + d] = s;
  }
}

constexpr int kColumns = 8;  // of a workgroup that adds up parts

// Adds up the workgroups' parts of the weights' gradients.
template <class T>
__global__ __launch_bounds__(256) void k_norm_weights_join(NormArgs a) {
  __shared__ Sum<T> sums[256 / kColumns][kColumns];
  const int is_k = blockIdx.y, c = threadIdx.x % kColumns, y = threadIdx.x / kColumns, D = a.n.head_dim;
  const int d = blockIdx.x * kColumns + c;
  if (!a.dw[is_k]) return;
  Sum<T> s = 0;
  const Sum<T>* const part = static_cast<const Sum<T>*>(a.part[is_k]);
#pragma unroll 8
  for (int i = y; i < a.groups[is_k]; i += 256 / kColumns) s += part[static_cast<int64_t>(i) * D + d];
  sums[y][c] = s;
  __syncthreads();
  if (y > 0) return;
  s = 0;
  for (int i = 0; i < 256 / kColumns; ++i) s += sums[i][c];
  static_cast<T*>(a.dw[is_k])[d] = static_cast<T>(s);
}

int check_heads(const gnnshap_heads& h, const char* name, int64_t tokens) {
  if (h.heads < 0) return fail(GNNSHAP_EINVAL, "%s: %d heads", name, static_cast<int>(h.heads));
  if (h.heads > 0 && tokens > 0 && (!h.x || !h.out)) return fail(GNNSHAP_EINVAL, "%s: NULL x or out", name);
  return GNNSHAP_OK;
}

int check_normed(const gnnshap_normed* n) {
  if (!n || n->num_tokens < 0) return fail(GNNSHAP_EINVAL, "heads to norm: NULL or a negative number of tokens");
  if (n->dtype < GNNSHAP_F32 || n->dtype > GNNSHAP_BF16)
    return fail(GNNSHAP_EUNSUPPORTED, "dtype %d is not one of f32, f16, bf16", static_cast<int>(n->dtype));
  if (n->head_dim < 8 || n->head_dim % 8 != 0 || n->head_dim > GNNSHAP_MAX_HEAD_DIM)
    return fail(n->head_dim < 1 ? GNNSHAP_EINVAL : GNNSHAP_EUNSUPPORTED,
                "head_dim %d is not a multiple of 8 from 8 to %d", static_cast<int>(n->head_dim), GNNSHAP_MAX_HEAD_DIM);
  if (n->num_tokens > INT32_MAX)
    return fail(GNNSHAP_EUNSUPPORTED, "%lld tokens in one call", static_cast<long long>(n->num_tokens));
  if (n->q.heads < 0 || n->k.heads < 0 || static_cast<int64_t>(n->q.heads) + n->k.heads > 4 * 65535)
    return fail(n->q.heads < 0 || n->k.heads < 0 ? GNNSHAP_EINVAL : GNNSHAP_EUNSUPPORTED, "%d and %d heads",
                static_cast<int>(n->q.heads), static_cast<int>(n->k.heads));
  if (n->cos) {
    if (!n->sin || n->num_positions < 1) return fail(GNNSHAP_EINVAL, "cos without sin or positions");
    if (n->rot_dim < 0 || n->rot_dim % 2 != 0 || n->rot_dim > n->head_dim)
      return fail(GNNSHAP_EINVAL, "rot_dim %d of head_dim %d", static_cast<int>(n->rot_dim),
                  static_cast<int>(n->head_dim));
  }
  if (!(n->eps >= 0.0 && std::isfinite(static_cast<float>(n->eps))))
    return fail(GNNSHAP_EINVAL, "eps %g is negative or not finite in fp32", n->eps);
  return GNNSHAP_OK;
}

int rot_of(const gnnshap_normed& n) { return n.cos ? n.rot_dim : 0; }

// Workgroups of the gradient's kernel: each kind's heads by its share of four
// per compute unit, no more than there are heads for.
int lay_out(NormArgs& a) {
  int lanes = 1;
  with_dtype(a.n.dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    return with_pack<T>(a.n.head_dim, rot_of(a.n), [&](auto n) {
      lanes = head_lanes(a.n.head_dim / (2 * decltype(n)::value));
      return 0;
    });
  });
  const int64_t all = a.n.num_tokens * (static_cast<int64_t>(a.n.q.heads) + a.n.k.heads), y = 256 / lanes;
  const gnnshap_heads* kinds[2] = {&a.n.q, &a.n.k};
  for (int i = 0; i < 2; ++i) {
    const int64_t items = a.n.num_tokens * kinds[i]->heads;
    a.groups[i] = items == 0 ? 0
                             : static_cast<int>(std::max<int64_t>(
                                   1, std::min<int64_t>(1024 * (items / 64 + 1) / (all / 64 + 1), ceil_div(items, y))));
  }
  return lanes;
}

size_t carve(NormArgs& a, void* ws) {
  Carver c(ws);
  const size_t sum = a.n.dtype == GNNSHAP_F32 ? sizeof(Sum<float>) : sizeof(Sum<bf16_t>);
  for (int i = 0; i < 2; ++i) a.part[i] = c.take<char>(static_cast<size_t>(a.groups[i]) * a.n.head_dim * sum);
  return c.bytes();
}

}  // namespace

extern "C" int gnnshap_norm_rotate(const gnnshap_normed* n, int32_t* info, void* stream) {
  GS_TRY_BEGIN
  clear_error();
  if (const int st = check_normed(n)) return st;
  if (const int st = check_heads(n->q, "queries", n->num_tokens)) return st;
  if (const int st = check_heads(n->k, "keys", n->num_tokens)) return st;
  const int heads = n->q.heads + n->k.heads;
  if (n->num_tokens == 0 || heads == 0) return GNNSHAP_OK;
  NormArgs a{};
  a.n = *n;
  a.info = info;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return with_dtype(n->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    return with_pack<T>(n->head_dim, rot_of(*n), [&](auto pack) {
      constexpr int N = decltype(pack)::value;
      const int x = head_lanes(n->head_dim / (2 * N)), y = std::min(256 / x, heads);
      if (const int st = check_launch(n->num_tokens, x)) return st;
      const dim3 grid(static_cast<unsigned>(n->num_tokens), static_cast<unsigned>(ceil_div(heads, y)));
      {
        GS_TIMED("k_norm_rotate", s);
        k_norm_rotate<T, N><<<grid, dim3(x, y), 0, s>>>(a);
      }
      GS_LAUNCHED();
      return static_cast<int>(GNNSHAP_OK);
    });
  });
  GS_TRY_END
}

extern "C" int gnnshap_norm_rotate_backward_workspace(const gnnshap_normed* n, size_t* bytes) {
  GS_TRY_BEGIN
  clear_error();
  if (!bytes) return fail(GNNSHAP_EINVAL, "bytes is NULL");
  if (const int st = check_normed(n)) return st;
  NormArgs a{};
  a.n = *n;
  lay_out(a);
  *bytes = carve(a, nullptr);
  return GNNSHAP_OK;
  GS_TRY_END
}

extern "C" int gnnshap_norm_rotate_backward(const gnnshap_normed* n, const gnnshap_heads* grad_q,
                                            const gnnshap_heads* grad_k, void* dq_norm, void* dk_norm, int32_t* info,
                                            void* ws, size_t ws_bytes, void* stream) {
  GS_TRY_BEGIN
  clear_error();
  if (const int st = check_normed(n)) return st;
  NormArgs a{};
  a.n = *n;
  a.info = info;
  const gnnshap_heads* grads[2] = {grad_q, grad_k};
  const gnnshap_heads* kinds[2] = {&n->q, &n->k};
  for (int i = 0; i < 2; ++i) {
    const char* const name = i ? "keys" : "queries";
    a.dw[i] = i ? dk_norm : dq_norm;
    if (kinds[i]->heads == 0) continue;
    if (!grads[i] || grads[i]->heads != kinds[i]->heads)
      return fail(GNNSHAP_EINVAL, "%s: no gradient, or one of other heads", name);
    if (n->num_tokens > 0 && !kinds[i]->x) return fail(GNNSHAP_EINVAL, "%s: NULL x", name);
    if (const int st = check_heads(*grads[i], name, n->num_tokens)) return st;
    a.grad[i] = *grads[i];
  }
  const int lanes = lay_out(a);
  const size_t need = carve(a, ws);
  const bool weights = a.dw[0] || a.dw[1];
  if (need > 0 && weights && (!ws || ws_bytes < need))
    return fail(GNNSHAP_ECAPACITY, "norm_rotate_backward workspace needs %zu bytes, has %zu", need, ws ? ws_bytes : 0);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return with_dtype(n->dtype, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    if (const unsigned grid = a.groups[0] + a.groups[1]) {
      const int st = with_pack<T>(n->head_dim, rot_of(*n), [&](auto pack) {
        {
          GS_TIMED("k_norm_rotate_grad", s);
          k_norm_rotate_grad<T, decltype(pack)::value><<<grid, dim3(lanes, 256 / lanes), 0, s>>>(a);
        }
        GS_LAUNCHED();
        return static_cast<int>(GNNSHAP_OK);
      });
      if (st) return st;
    }
    if (weights) {  // of no tokens or heads too: they are 0
      GS_TIMED("k_norm_weights_join", s);
      k_norm_weights_join<T><<<dim3(n->head_dim / kColumns, 2), 256, 0, s>>>(a);
      GS_LAUNCHED();
    }
    return static_cast<int>(GNNSHAP_OK);
  });
  GS_TRY_END
}
