// How the 8-bit linear layer cuts a product into tiles: which of its two kernels, tile sizes, the split of a sum and its chunks.
// Plain C++ (no CUDA types), so that the host can ask it alone too.
#pragma once

#include <algorithm>

namespace linear8 {

constexpr int kTileFeatures = 128;                       // of a CTA's tile: the instruction's M
constexpr int kTileK = 128;                          // elements of `inner` per stage: one 128-byte swizzled row, one scale
constexpr int kScaleSlots = 4;                       // words of scales on their way
constexpr int kTileSlotBytes = 1024;                 // small tiles: a word of scales of the tile's features, and of its tokens
constexpr int kMaxTileFew = 64;                      // tokens per small tile, at most
constexpr int kMaxSplit = 8;                         // portable cluster size
constexpr int kMaxTileT = 240;                       // tokens per tile of the pairs, at most
constexpr int kPairRows = kMaxTileFew;               // up to so many tokens pairs are not considered

// As many stages as leave room for two CTAs on an SM: five up to 32 tokens (3% faster than four), four beyond.
constexpr int tile_stages(int tile_t) { return tile_t <= 32 ? 5 : 4; }
constexpr int tile_dynamic(int tile_t) {
  return tile_stages(tile_t) * (kTileFeatures + tile_t) * 128 + kScaleSlots * kTileSlotBytes + 1024;
}

// CTAs per tile: as many as it takes to give every SM work, while all of them run at once and each keeps four stages of the sum,
// or eight where the SMs have more than one CTA then.
inline int tile_split(long long tiles, int k_iters, int tile_t, int sms) {
  const int per_sm = 228 * 1024 / (tile_dynamic(tile_t) + 2 * 1024);
  int split = 1;
  while (split < kMaxSplit && tiles * split < sms && tiles * 2 * split <= (long long)sms * per_sm &&
         k_iters >= (tiles * 2 * split <= sms ? 8 : 16) * split)
    split *= 2;
  return split;
}

// fp32 outputs: the tensor core adds products to the accumulator by truncation, so a long sum drifts; there it is cut into chunks
// that are added with round-to-nearest, as in linear.cu.  A step of the 8-bit kind adds 32 products, twice those of the 16-bit
// kind, and drifts half as much.  Relative errors at inner = 5120, and in brackets the worst case, where all terms are positive: in chunks
// of 1280 0.8e-7 (2.5e-7), 1792 1.0e-7 (3.3e-7), 2048 1.1e-7 (4.3e-7), 2560 1.4e-7 (7.1e-7), in one go 2.8e-7 (2.0e-6); fp32 sums of a
// library product 1e-7 (2.4e-7).  Longer chunks than 1792 gain little time and lose digits; no chunks at all gain more, since a chunked sum's
// total is kept in registers, which hold a tile of 256 features and not one of 512: 4680 x 5120 x 5120 with gate and residual 145 us in
// chunks of 1792, 149 of 1280, 141 of 2560, 129 in one go (20 launches from cold); 4680 x 20480 x 5120 495, 504 and 486 in chunks (400 launches).
// So only what is one chunk goes in one: the drafter's inner axis of 1536, 4680 x 1536 x 1536 26 us (34 in chunks of 1280).  Small tiles have the room: chunks of 512.
constexpr int kPairChunkIters = 1792 / kTileK;
constexpr int kWholeIters = kPairChunkIters;
constexpr int kTileChunkIters = 512 / kTileK;
constexpr bool whole_sums(int k_iters, bool fp32) { return !fp32 || k_iters <= kWholeIters; }          // of the pairs

// How a product is cut: tiles of 128 features x tile_t tokens by clusters of `split` CTAs, or (subs > 0) tiles of subs x 256 features x tile_t
// tokens by pairs.  The cheapest by these estimates, in clocks, whose constants were fitted to times of both kinds at 45 sizes:
// a stage costs the bytes it brings to an SM, 56 of them a clock where CTAs come one or two to an SM, 36 and 43 for pairs, but not
// less than its barriers and instructions; a split sum is joined; pairs take longer to begin and end.  Pairs against small
// tiles, in us: 100 x 5120 x 1536 17.4 and 9.4, 333 x 5120 x 776 16.8 and 9.7, 1500 x 1536 x 1536 10.1 and 8.2, 300 x 5120 x 4000 18.3
// and 15.2, 512 x 4096 x 5120 17.3 and 23.9.
struct Cut {
  int subs, tile_t, split;
  double cost;
};
// chunked: the pairs' sum in several chunks
inline Cut choose_cut(int rows, int cols, int k_iters, int pairs, bool chunked) {
  auto ceil_div = [](long long a, long long b) { return (a + b - 1) / b; };
  const int sms = 2 * pairs;
  Cut best{0, 0, 0, 0};
  auto offer = [&](const Cut& c) {
    if (!best.tile_t || c.cost < best.cost) best = c;
  };
  const int most = (std::min(rows, kMaxTileFew) + 15) / 16 * 16;
  for (int nt = most; nt >= std::min(most, 32); nt -= 16) {
    const long long tiles = ceil_div(cols, kTileFeatures) * ceil_div(rows, nt);
    const int split = tile_split(tiles, k_iters, nt, sms);
    const long long on_sm = std::min(2ll, ceil_div(tiles * split, sms)), waves = ceil_div(tiles * split, 2 * sms);
    const double stage = std::max(250.0, on_sm * (kTileFeatures + nt) * 128 / 56.0);
    offer({0, nt, split, waves * ceil_div(k_iters, split) * stage + (split > 1 ? 1000 + 300 * split + 45 * nt : 0)});
  }
  if (rows <= kPairRows) return best;
  for (int subs = 1; subs <= (chunked ? 1 : 2); ++subs)
    for (int nt = kMaxTileT; nt >= 64; nt -= 16) {
      const long long waves = ceil_div(ceil_div(cols, 2 * kTileFeatures * subs) * ceil_div(rows, nt), pairs);
      const double stage = std::max(470.0, (kTileFeatures * subs + nt / 2) * 128 / (subs == 2 ? 43.0 : 36.0));
      offer({subs, nt, 1, 4500 + waves * (k_iters * stage + 2500 * subs)});
    }
  return best;
}

}  // namespace linear8
