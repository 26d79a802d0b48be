// fp8_choice.h — tiles of the 8-bit products and thread blocks that share one, from sizes
// alone, on the host. The order of a product's sums follows from them.
#pragma once

#include <cstdint>

namespace awsrc {
namespace fp8 {

constexpr int kSms = 152, kPairs = kSms / 2;
constexpr int kTileRows = 128;   // rows of w a thread block holds at most
constexpr int kFewSplit = 8;     // thread blocks that share a tile's columns (few rows of x)
constexpr int kPairSplit = 4;    // pairs of them that do (more rows)
constexpr int kPairLeast = 4;    // blocks of 128 columns that such a pair has at least
constexpr int kPairMaxN = 256;   // rows of x in a pair's tile

// Clusters of up to 8 thread blocks, by their size, that run at a time; 0: none of that size.
struct Clusters {
  int of[9];
};
struct Choice {
  int n, split;
};

// Few rows of x: rows of w in a tile and thread blocks per tile, the least time by a model
// of a thread block's stages, each 350 ns (its products) or its bytes at 50 GB/s, and 1.8 us
// where parts are joined.
inline Choice choose_few(int rows, int blocks, int x_rows, const Clusters& most_of) {
  Choice best{8, 1};
  const double x_bytes = 512.0 * x_rows;  // as if bf16: the choice, and so the sums, are the same for x and for its codes
  double least = 0;
  const int twos = (blocks + 1) / 2;
  for (int split = 1; split <= kFewSplit && split <= twos; ++split) {
    const int64_t most = split > 1 ? most_of.of[split] : kSms;  // tiles at a time
    if (most < 1) continue;
    int64_t waves = 1, r;
    for (;; ++waves) {
      r = (rows + most * waves - 1) / (most * waves);
      r = (r + 7) / 8 * 8;
      if (r <= kTileRows || split > 1) break;
    }
    if (r > kTileRows) continue;  // parts are joined in one wave
    const double bytes = (256.0 * r + x_bytes) / 50.0, stage = bytes > 350.0 ? bytes : 350.0;
    const double all = (double)waves * ((twos + split - 1) / split) * stage + (split > 1 ? 1800.0 : 0.0);
    if (least == 0 || all < least) least = all, best = Choice{(int)r, split};
  }
  return best;
}

// More rows: rows of x in a pair's tile and pairs per tile, the fewest cycles by a model of
// both. A block costs a pair what its bytes take at 52 bytes per cycle and SM, or its
// products at 2 cycles per row of x, the larger; a tile 2500 more, and 8 per row of x and
// further pair where pairs join their parts.
inline Choice choose_pairs(int rows, int blocks, int x_rows, const Clusters& most_of) {
  Choice best{64, 1};
  const int64_t tiles_w = ((int64_t)rows + 2 * kTileRows - 1) / (2 * kTileRows);
  double least = 0;
  for (int n = 64; n <= kPairMaxN; n += 64)
    for (int split = 1; split <= kPairSplit && (split == 1 || split * kPairLeast <= blocks); ++split) {
      const int64_t tiles = tiles_w * (((int64_t)x_rows + n - 1) / n);
      if (split > 1 && tiles > most_of.of[2 * split]) continue;
      const double load = (16384.0 + 64.0 * n) / 52.0, mma = 2.0 * n;
      const double tile = (double)((blocks + split - 1) / split) * (load > mma ? load : mma) + 2500.0 + 8.0 * n * (split - 1);
      const double all = (split > 1 ? 1.0 : (double)((tiles + kPairs - 1) / kPairs)) * tile;
      if (least == 0 || all < least) least = all, best = Choice{n, split};
    }
  return best;
}

}  // namespace fp8
}  // namespace awsrc
