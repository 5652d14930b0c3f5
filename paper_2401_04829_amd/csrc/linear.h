// What the log probabilities from hidden states and their gradient share.
#pragma once

#include "product.h"
#include "stats.h"

namespace gnnshap {

// Of up to this many rows the gradient by the logits is given in two parts,
// rounded and what that left: a few rows' gradients hang on few of its
// elements, so that one rounding would show (up to 2^-8 in bf16, where the
// result's own is 2^-9 on average), and cost nothing beside the weights.
constexpr int64_t kTwoParts = 128;

struct LinearArgs {
  gnnshap_linear l;
  int32_t* info;
  unsigned tiles_m, tiles_n;  // of the vocabulary (or piece), of the rows
  Stats* parts;               // [row][tile of the vocabulary]
  float* given;               // [row] logit of the given token
  // the gradient's
  const float* gl;
  const float* ge;
  const float* scale;         // of d in fp16, and one over it; NULL: 1
  void* d;                    // [row, then what rounding left of row][pitch]
  int64_t pitch;
  bool two;                   // d in two parts
  int64_t v0, piece;          // the piece of the vocabulary
};

// The product of logits: a tile's rows are tokens, its columns hidden states'
// rows, so that a lane has tokens on end.  256 x 256 for many rows; where they
// are fewer the weights' rows are read once, and a workgroup takes fewer of
// them so that all compute units have some.
template <class T, bool DIRECT>
using LogitsMany = Product<T, 8, 4, 2, 4, 64, 4, false, false, DIRECT>;
template <class T, bool DIRECT>
using LogitsSome = Product<T, 4, 2, 2, 2, 128, 3, false, false, DIRECT>;
template <class T, bool DIRECT>
using LogitsFew = Product<T, 1, 1, 4, 1, 128, 4, false, false, DIRECT>;

// Calls f with the product for `rows` rows.
template <class T, class F>
inline int with_logits(int64_t rows, bool direct, F f) {
  const auto pick = [&](auto d) {
    constexpr bool D = decltype(d)::value;
    if (rows <= 16) return f(static_cast<LogitsFew<T, D>*>(nullptr));
    if (rows <= 128) return f(static_cast<LogitsSome<T, D>*>(nullptr));
    return f(static_cast<LogitsMany<T, D>*>(nullptr));
  };
  return direct ? pick(std::true_type()) : pick(std::false_type());
}

template <class T>
inline bool direct_logits(const gnnshap_linear& l) {
  return direct_operand<T>(l.hidden, l.hidden_stride, l.width, 256) &&
         direct_operand<T>(l.weight, l.weight_stride, l.width, 256);
}

int check_linear(const gnnshap_linear* l);

}  // namespace gnnshap
