// How the products of the log probabilities from hidden states and of their
// gradient are laid out: which tiles take them, in how many parts.  Rules of sizes
// alone, without device code.
#pragma once

#include <algorithm>

#include "common.h"

namespace gnnshap {

// The shapes of a product's tiles, from the largest on.  A large one reads less
// per product, a small one gives more compute units work.
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
// rows x 50,021 tokens of 2,048 are 6.1 rounds: 445 us, 403 and 24 as two).  The
// tokens are A's rows of the logits' product (ROWS) or B's of dw's, `across` the
// other operand's, K in bytes.
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

// Of operands that have to go through registers there are fewer shapes.
constexpr unsigned kThroughRegisters = 1u << 1 | 1u << 3 | 1u << 5;

// The logits' product: a tile's rows are tokens, its columns hidden states'
// rows, so that a lane has tokens on end.
constexpr unsigned kLogitShapes = 0x2F;  // (64 x 32 is no faster than its neighbours)
inline int logit_segments(int64_t tokens, const gnnshap_linear& l, int64_t element, bool direct, Segment (&s)[2]) {
  return segments_for<true>(tokens, l.num_rows, l.width * element, element == 4,
                            direct ? kLogitShapes : kLogitShapes & kThroughRegisters, s);
}

// The gradient by the logits, d, enters the products of 16-bit types in two parts,
// rounded and what that left: rounded once, each of d's elements is off by up to u
// of itself (2^-8 in bf16), which the sums over the vocabulary and the rows keep
// even where the terms themselves cancel, as those of a vector that all weights
// share do (sum_j d_j = 0): up to 10 times the result's own rounding instead of
// none.  Two parts leave u^2, at the price of a product more for dh and for dw.
// (2,000 rows x 50,021 tokens of 2,048 in bf16: 1,230 us with one part, 2,000 with
// two; 200 rows: 258 and 355.)
//
// Of up to this many rows dh takes the second parts as rows of their own, so that
// the weights are read once; of more as a second sum over the vocabulary, so that
// no more results are written and added up (50,021 x 2,048, bf16, rows of their
// own and second sums: 200 rows 355 and 376 us, 256 rows 374 and 394, 400 rows 577 and 566).
constexpr int64_t kBeside = 256;

// Of d, all of it: each piece is another round of launches, whose last workgroups
// leave compute units without work, and another reading and writing of dh's sums
// (10,000 rows x 32,768 tokens of 2,048 in bf16: 9,220 us with 192 MB, 7,080 with 384,
// 6,260 with 768, 6,150 with 1,536).
constexpr int64_t kPieceBytes = int64_t(768) << 20;
constexpr float kJoinTime = 6.f;                     // us, of a launch that adds up few parts

// dh's product: a tile's rows are elements of the width, its columns rows of d.
constexpr unsigned kHiddenShapes = 0x1B;   // all but 128 x 64 and those whose A would be read element by element
// dw's: the width by tokens.
constexpr unsigned kWeightShapes = 0x0F;

// A chunk by way of registers takes about so many times as long (1,000 rows x
// 100 tokens x 100 in bf16, dw in 128 x 128: 2.2 us instead of 0.7).
constexpr float kSlow = 3.f;

// How a product whose K is split is laid out: its shape and how many workgroups
// take parts of K.  Each part is a sum more to write and to read.
struct Split {
  int shape;
  int64_t parts;
  float time;   // us
};
inline Split split_of(int64_t M, int64_t N, int64_t K, int segments, bool wide, unsigned shapes, float slow,
                      int64_t least_parts) {
  Split best{-1, 1, 0.f};
  for (int i = 0; i < kShapes; ++i) {
    if (!(shapes >> i & 1u)) continue;
    const int64_t tiles = ceil_div(M, kTileM[i]) * ceil_div(N, kTileN[i]);
    for (int64_t parts = least_parts; parts <= 64; parts *= 2) {
      if (parts > 1 && K / parts < 256) break;
      const int64_t chunks = ceil_div(ceil_div(K, parts), wide ? 32 : 64) * segments;
      // a part's sum: written and read, 8 bytes an element, at 3 TB/s
      const float t = pace(i, wide, tiles * parts, M * parts) * slow * static_cast<float>(chunks) +
                      static_cast<float>(parts * M * N) * 8.f / 3e6f;
      if (best.shape < 0 || t < best.time) best = Split{i, parts, t};
    }
  }
  return best;
}

// dw's parts, 1 where its tiles are enough: then it is written at once.
inline Split weight_split(const gnnshap_linear& l, int64_t tokens, int segments, bool direct) {
  const bool wide = l.dtype == GNNSHAP_F32;
  const unsigned shapes = direct ? kWeightShapes : kWeightShapes & kThroughRegisters;
  const float slow = direct ? 1.f : kSlow;
  const int shape = shape_for(l.width, tokens, wide, shapes);
  const float whole = pace(shape, wide, ceil_div(l.width, kTileM[shape]) * ceil_div(tokens, kTileN[shape]), l.width) *
                      slow * static_cast<float>(ceil_div(l.num_rows, wide ? 32 : 64) * segments);
  const Split s = split_of(l.width, tokens, l.num_rows, segments, wide, shapes, slow, 2);
  return s.shape >= 0 && s.time + kJoinTime < whole ? s : Split{-1, 1, 0.f};
}

// dw's segments of a piece of the vocabulary, where it is written at once.
inline int weight_segments_for(int64_t piece, const gnnshap_linear& l, int64_t element, int parts, bool direct,
                               Segment (&s)[2]) {
  return segments_for<false>(piece, l.width, std::max<int64_t>(l.num_rows, 1) * parts * element, element == 4,
                             direct ? kWeightShapes : kWeightShapes & kThroughRegisters, s);
}

// How the backward pass is laid out.
struct Layout {
  bool two, beside;                      // d in two parts, dh with these as rows beside each other
  int hidden_segments, weight_segments;  // d's parts that dh and dw sum over
  int hidden_shape, weight_shape;
  int64_t d_rows, hidden_rows, piece, pitch;   // rows of d and of dh's product
  int64_t split, parts;                  // of dh
  int64_t weight_split, weight_parts;    // of dw; one part: written at once
  float* scale;
  void* d;
  float *sums, *weight_sums;
};

inline Layout lay_out(const gnnshap_linear& l, int64_t element, bool direct_w, bool direct_h) {
  Layout y{};
  y.two = element == 2;
  y.beside = y.two && l.num_rows <= kBeside;
  y.d_rows = y.two ? 2 * l.num_rows : l.num_rows;
  y.hidden_rows = y.beside ? 2 * l.num_rows : l.num_rows;
  y.hidden_segments = y.two && !y.beside ? 2 : 1;
  y.weight_segments = y.two ? 2 : 1;
  // pieces of like size, whole tiles of 256
  const int64_t most = std::max<int64_t>(kPieceBytes / (std::max<int64_t>(y.d_rows, 1) * element) / 256 * 256, 256);
  const int64_t pieces = ceil_div(l.vocab, most);
  y.piece = ceil_div(ceil_div(l.vocab, pieces), 256) * 256;
  y.pitch = y.piece;
  const int64_t tokens = std::min(y.piece, l.vocab);
  const Split h = split_of(l.width, std::max<int64_t>(y.hidden_rows, 1), tokens, y.hidden_segments, !y.two,
                           direct_w ? kHiddenShapes : kHiddenShapes & kThroughRegisters, direct_w ? 1.f : kSlow, 1);
  y.hidden_shape = h.shape;
  y.split = ceil_div(ceil_div(y.piece, h.parts), 64) * 64;
  y.parts = ceil_div(y.piece, y.split);
  const Split w = weight_split(l, tokens, y.weight_segments, direct_h);
  y.weight_shape = w.shape;
  y.weight_split = ceil_div(ceil_div(std::max<int64_t>(l.num_rows, 1), w.parts), 64) * 64;
  y.weight_parts = ceil_div(std::max<int64_t>(l.num_rows, 1), y.weight_split);
  return y;
}

}  // namespace gnnshap
