// Prints how the 8-bit linear layer cuts the products given on standard input (csrc/linear_e4m3_cut.h), a line each:
// rows, columns, inner, CTA pairs of the device, fp32 outputs (0 or 1) -> subs, tokens of a tile, CTAs that share a sum, whole sums.
#include <cstdio>

#include "linear_e4m3_cut.h"

int main() {
  int rows, cols, inner, pairs, f32;
  while (std::scanf("%d %d %d %d %d", &rows, &cols, &inner, &pairs, &f32) == 5) {
    const int k_iters = (inner + linear8::kTileK - 1) / linear8::kTileK;
    const bool whole = linear8::whole_sums(k_iters, f32 != 0);
    const linear8::Cut c = linear8::choose_cut(rows, cols, k_iters, pairs, !whole);
    std::printf("%d %d %d %d\n", c.subs, c.tile_t, c.split, (int)whole);
  }
}
