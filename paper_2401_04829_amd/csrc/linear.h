// What the log probabilities from hidden states and their gradient share.
#pragma once

#include "linear_layout.h"
#include "product.h"
#include "stats.h"

namespace gnnshap {

struct LinearArgs {
  gnnshap_linear l;
  int32_t* info;
  unsigned tiles_m, tiles_n;  // of the segment of the vocabulary, of the rows
  Stats* parts;               // [row][tile of the vocabulary]
  unsigned part0, row_parts;  // the segment's first part of a row's, and all of them
  float* given;               // [row] logit of the given token
  // the gradient's
  const float* gl;
  const float* ge;
  const float* scale;         // of d in fp16, and one over it; NULL: 1
  void* d;                    // [row, then (two parts) what rounding left of row][pitch]
  int64_t pitch;
  bool two;                   // d in two parts
  int64_t v0, tokens;         // the segment: its first token and how many
  int64_t d0;                 // the segment's first column of d
};

// The products of the shapes: their tiles are kTileM x kTileN.
template <class T, int SHAPE, bool A_TURNED, bool B_TURNED, bool DIRECT>
struct ShapeOf;
#define GS_SHAPE(N, ...)                                              \
  template <class T, bool A_TURNED, bool B_TURNED, bool DIRECT>       \
  struct ShapeOf<T, N, A_TURNED, B_TURNED, DIRECT> {                  \
    using P = Product<T, __VA_ARGS__, A_TURNED, B_TURNED, DIRECT>;    \
  };
GS_SHAPE(0, 8, 4, 2, 4, 128, 2)  // 256 x 256
GS_SHAPE(1, 4, 4, 2, 2, 128, 2)  // 128 x 128
GS_SHAPE(2, 4, 2, 2, 2, 128, 3)  // 128 x 64
GS_SHAPE(3, 2, 2, 2, 2, 128, 4)  // 64 x 64
GS_SHAPE(4, 2, 1, 2, 2, 128, 4)  // 64 x 32
GS_SHAPE(5, 1, 1, 4, 1, 128, 4)  // 64 x 16
#undef GS_SHAPE

// Calls f with a null pointer of the product of a shape.
template <class T, bool A_TURNED, bool B_TURNED, unsigned WHICH, class F>
inline int with_shape(int shape, bool direct, F f) {
#define GS_CASE(N, D) f(static_cast<typename ShapeOf<T, N, A_TURNED, B_TURNED, D>::P*>(nullptr))
#define GS_SHAPE(N)                                                     \
  case N:                                                               \
    if constexpr ((WHICH >> N & 1u) != 0) {                             \
      if (direct) return GS_CASE(N, true);                              \
      if constexpr ((kThroughRegisters >> N & 1u) != 0) return GS_CASE(N, false); \
    }                                                                   \
    break;
  switch (shape) {
    GS_SHAPE(0)
    GS_SHAPE(1)
    GS_SHAPE(2)
    GS_SHAPE(3)
    GS_SHAPE(4)
    GS_SHAPE(5)
  }
#undef GS_SHAPE
#undef GS_CASE
  return fail(GNNSHAP_EUNSUPPORTED, "no product of shape %d", shape);
}

template <class T, class F>
inline int with_logits(int shape, bool direct, F f) {
  return with_shape<T, false, false, kLogitShapes>(shape, direct, f);
}

template <class T>
inline bool direct_logits(const gnnshap_linear& l) {
  return direct_operand<T>(l.hidden, l.hidden_stride, l.width, 256) &&
         direct_operand<T>(l.weight, l.weight_stride, l.width, 256);
}

int check_linear(const gnnshap_linear* l);

}  // namespace gnnshap
