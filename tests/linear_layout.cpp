// Prints how the products of the log probabilities from hidden states are laid
// out: for each line "bytes of an element, rows, vocabulary, width, direct" on
// standard input a line of words, which of the kernels' shapes run.
//   logits<shape>     one segment of the vocabulary's logits (forward)
//   logits<shape>+<shape>  two
//   d...              likewise, of a piece of the vocabulary in the gradient
//   dh<shape>[s]      dh's product; s: sums over both of d's parts
//   dw<shape>[+<shape>]    dw's product, written at once
//   dwparts<shape>    in parts of the rows
//   pieces            more than one piece of the vocabulary
#include <cstdio>

#include "linear_layout.h"

using namespace gnnshap;

static void show(const char* name, const Segment (&s)[2], int n) {
  printf("%s%d", name, s[0].shape);
  if (n == 2) printf("+%d", s[1].shape);
  printf(" ");
}

int main() {
  long long element, rows, vocab, width, direct;
  while (scanf("%lld %lld %lld %lld %lld", &element, &rows, &vocab, &width, &direct) == 5) {
    gnnshap_linear l{};
    l.dtype = element == 4 ? GNNSHAP_F32 : GNNSHAP_BF16;
    l.num_rows = rows;
    l.vocab = vocab;
    l.width = width;
    Segment s[2];
    show("logits", s, logit_segments(vocab, l, element, direct, s));
    const Layout y = lay_out(l, element, direct, direct);
    printf("dh%d%s ", y.hidden_shape, y.hidden_segments == 2 ? "s" : "");
    if (vocab > y.piece) printf("pieces ");
    for (int64_t v0 = 0; v0 < vocab; v0 += y.piece) {
      const int64_t piece = std::min<int64_t>(y.piece, vocab - v0);
      show("d", s, logit_segments(piece, l, element, direct, s));
      if (y.weight_parts > 1)
        printf("dwparts%d ", y.weight_shape);
      else
        show("dw", s, weight_segments_for(piece, l, element, y.weight_segments, direct, s));
    }
    printf("\n");
  }
}
