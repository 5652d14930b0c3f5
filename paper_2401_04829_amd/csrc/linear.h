// What the log probabilities from hidden states and their gradient share.
#pragma once

#include "product.h"
#include "stats.h"

namespace gnnshap {

// The gradient by the logits, d, enters the products of 16-bit types in two parts,
// rounded and what that left: rounded once, each of d's elements is off by up to u
// of itself (2^-8 in bf16), which the sums over the vocabulary and the rows keep
// even where the terms themselves cancel, as those of a vector that all weights
// share do (sum_j d_j = 0): up to 10 times the result's own rounding instead of
// none.  Two parts leave u^2, at the price of a product more for dh and for dw.
// (2,000 rows x 50,021 tokens of 2,048 in bf16: 1,230 us with one part, 2,000 with
// two; 200 rows: 258 and 355.)
// Of up to this many rows dh takes the second parts as rows of their own, so that
// the weights are read once; of more as a second sum over the vocabulary, so that
// no more results are written and added up (50,021 x 2,048, bf16, rows of their
// own and second sums: 200 rows 355 and 376 us, 256 rows 374 and 394, 400 rows 577 and 566).
constexpr int64_t kBeside = 256;

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

// The shapes of a product's tiles, from the largest on.  A large one reads less
// per product, a small one gives more compute units work.
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
constexpr int kShapes = 6;
constexpr int kTileM[kShapes] = {256, 128, 128, 64, 64, 64}, kTileN[kShapes] = {256, 128, 64, 64, 32, 16};

// The time of a tile's chunk (128 bytes of K) in us: of one workgroup alone,
// and of one of very many times a 256th (the chip's), in 16 and in 32 bits.
// Measured with the logits' kernel: bf16, 10,000 x 32,768 x 2,048: 1,162 us at
// 256 x 256, 1,331 at 128 x 128; 300 x 5,000 x 2,048: 65, 31, 25 (128 x 64), 21
// (64 x 64); 1,534 x 3 x 1,304: 46, 24, 20, 15, 12.5 (64 x 16); fp32, 2,000 x
// 32,768 x 1,024: 999 and 1,055; 1,534 x 3 x 1,304: 325, 97, 59, 37, 22.
struct Pace {
  float alone, full;
};
constexpr Pace kPace[2][kShapes] = {{{1.7f, 1.8f}, {.71f, .53f}, {.53f, .42f}, {.34f, .33f}, {.28f, .29f}, {.21f, .26f}},
                                    {{7.7f, 8.0f}, {2.2f, 2.1f}, {1.25f, 1.3f}, {.65f, .68f}, {.48f, .42f}, {.34f, .24f}}};
// Time of a chunk of `tiles` tiles that read `rows` rows of A.
inline float pace(int shape, bool wide, int64_t tiles, int64_t rows) {
  const Pace& p = kPace[wide][shape];
  // one workgroup of the largest shape, and in fp32 of each, fills a compute unit:
  // rounds are whole (87 rows x 17,374 tokens x 2,328, fp32: 182 us by parts of
  // rounds, 132 by whole ones; of many rounds the last one matters less)
  const bool whole = shape == 0 || (wide && tiles < 4 * 256);
  const float rounds = whole ? static_cast<float>(ceil_div(tiles, 256)) : static_cast<float>(tiles) / 256.f;
  // A, the larger operand, comes from memory at 5.2 TB/s at most
  return std::max({p.alone, p.full * rounds, static_cast<float>(rows) * 128.f / 5.2e6f});
}

// The fastest of the shapes in `which` (bits) for M x N; of equally fast ones
// (bound by memory) the smallest, of which more are resident (one row of 131,072
// x 2,048 in bf16: 64 x 16 102 us, 128 x 64 117).
inline int shape_for(int64_t M, int64_t N, bool wide, unsigned which) {
  int best = -1;
  float least = 0.f;
  for (int i = 0; i < kShapes; ++i) {
    if (!(which >> i & 1u)) continue;
    const float t = pace(i, wide, ceil_div(M, kTileM[i]) * ceil_div(std::max<int64_t>(N, 1), kTileN[i]), M);
    if (best < 0 || t <= least) {
      best = i;
      least = t;
    }
  }
  return best;
}

// Part of the tokens, and the shape that takes them.
struct Segment {
  int shape;
  int64_t begin, tokens;
};
// The tokens' segments, one or two: the largest shape's last round of
// workgroups may have little to do, which smaller tiles then do faster (2,000
// rows x 50,021 tokens of 2,048 are 6.1 rounds: 445 us, 403 and 24 as two).  The tokens are A's rows of the
// logits' product (ROWS) or B's of dw's, `across` the other operand's, K in bytes.
template <bool ROWS>
inline int segments_for(int64_t tokens, int64_t across, int64_t k_bytes, bool wide, unsigned which, Segment (&s)[2]) {
  const auto best = [&](int64_t n) { return ROWS ? shape_for(n, across, wide, which) : shape_for(across, n, wide, which); };
  const auto time = [&](int shape, int64_t n) {
    const int64_t m_rows = ROWS ? n : across, n_rows = ROWS ? across : n;
    return pace(shape, wide, ceil_div(m_rows, kTileM[shape]) * ceil_div(std::max<int64_t>(n_rows, 1), kTileN[shape]), m_rows);
  };
  s[0] = Segment{best(tokens), 0, tokens};
  if (s[0].shape != 0) return 1;
  const int64_t side = ceil_div(std::max<int64_t>(across, 1), 256), tiles = ceil_div(tokens, 256);
  const int64_t whole = tiles * side / 256 * 256 / side * 256;   // tokens of whole rounds
  if (whole == 0 || whole >= tokens) return 1;
  const int rest = best(tokens - whole);
  const float launch = 4.f * 128.f / static_cast<float>(k_bytes);  // us, a chunk's share
  if (time(0, whole) + time(rest, tokens - whole) + launch >= time(0, tokens)) return 1;
  s[0].tokens = whole;
  s[1] = Segment{rest, whole, tokens - whole};
  return 2;
}

// Calls f with a null pointer of the product of a shape; of operands that have
// to go through registers there are fewer shapes.
constexpr unsigned kThroughRegisters = 1u << 1 | 1u << 3 | 1u << 5;
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

// The logits' product: a tile's rows are tokens, its columns hidden states'
// rows, so that a lane has tokens on end.
constexpr unsigned kLogitShapes = 0x2F;  // (64 x 32 is no faster than its neighbours)
template <class T>
inline int logit_segments(int64_t tokens, const gnnshap_linear& l, bool direct, Segment (&s)[2]) {
  return segments_for<true>(tokens, l.num_rows, l.width * static_cast<int64_t>(sizeof(T)), sizeof(T) == 4,
                            direct ? kLogitShapes : kLogitShapes & kThroughRegisters, s);
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
