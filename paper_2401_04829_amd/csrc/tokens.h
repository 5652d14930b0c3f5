// Element types, loads and argument checks of the token operators.
#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"

namespace gnnshap {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef unsigned u4_t __attribute__((ext_vector_type(4)));

// N elements that are loaded and stored at any element's address (gfx950
// takes wide accesses at any address).
template <class T, int N>
struct Pack {
  T v[N];
};

template <class T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
  Pack<T, N> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}

template <class T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& r) {
  __builtin_memcpy(p, &r, sizeof(r));
}

// The same past the caches' usual order, so that what is written once does not push
// out what is read: for results of a pass over memory.
template <class T, int N>
__device__ __forceinline__ void stream_pack(T* p, const Pack<T, N>& r) {
  if constexpr (sizeof(r) >= 4) {
    typedef unsigned words __attribute__((ext_vector_type(sizeof(r) / 4), aligned(alignof(T))));
    __builtin_nontemporal_store(__builtin_bit_cast(words, r), reinterpret_cast<words*>(p));
  } else {
    store_pack(p, r);
  }
}

// Calls f with a null pointer of the element type that `dtype` names.
template <class F>
inline int with_dtype(int32_t dtype, F f) {
  switch (dtype) {
    case GNNSHAP_F32: return f(static_cast<float*>(nullptr));
    case GNNSHAP_F16: return f(static_cast<f16_t*>(nullptr));
    case GNNSHAP_BF16: return f(static_cast<bf16_t*>(nullptr));
    default: return fail(GNNSHAP_EUNSUPPORTED, "dtype %d is not one of f32, f16, bf16", static_cast<int>(dtype));
  }
}

// GNNSHAP_OK, or the refusal of more threads along an axis than a launch takes.
inline int check_launch(int64_t workgroups, int64_t threads) {
  if (workgroups <= INT32_MAX && workgroups * threads < int64_t(1) << 32) return GNNSHAP_OK;
  return fail(GNNSHAP_EUNSUPPORTED, "%lld workgroups of %lld threads in one launch", static_cast<long long>(workgroups),
              static_cast<long long>(threads));
}

// GNNSHAP_OK, or the failure that a cache's description is.
inline int check_cache(const gnnshap_cache* c) {
  if (!c) return fail(GNNSHAP_EINVAL, "cache is NULL");
  if (c->dtype < GNNSHAP_F32 || c->dtype > GNNSHAP_BF16)
    return fail(GNNSHAP_EUNSUPPORTED, "dtype %d is not one of f32, f16, bf16", static_cast<int>(c->dtype));
  if (c->kv_heads < 1 || c->page_size < 1 || c->num_pages < 1 || c->num_pages > INT32_MAX)
    return fail(GNNSHAP_EINVAL, "cache of %d heads, %lld pages of %d tokens", static_cast<int>(c->kv_heads),
                static_cast<long long>(c->num_pages), static_cast<int>(c->page_size));
  if (c->head_dim < 8 || c->head_dim % 8 != 0 || c->head_dim > GNNSHAP_MAX_HEAD_DIM)
    return fail(c->head_dim < 1 ? GNNSHAP_EINVAL : GNNSHAP_EUNSUPPORTED,
                "head_dim %d is not a multiple of 8 from 8 to %d", static_cast<int>(c->head_dim), GNNSHAP_MAX_HEAD_DIM);
  if (!c->k || !c->v) return fail(GNNSHAP_EINVAL, "cache without keys or values");
  if (c->page_stride < 0 || c->slot_stride < 0 || c->head_stride < 0)
    return fail(GNNSHAP_EINVAL, "negative stride of the cache");
  return GNNSHAP_OK;
}

}  // namespace gnnshap
