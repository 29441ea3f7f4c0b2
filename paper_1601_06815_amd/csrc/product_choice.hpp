// Which tile a product of gated.hpp runs on, and how its sum is cut. Plain host code.
#pragma once

#include <algorithm>
#include <cstdlib>

#include "gated.hpp"

namespace oaa {

inline bool pair_on_i(ProductKind kind) { return kind == kUnitLast || kind == kUnitLastAgain; }
inline bool pair_on_j(ProductKind kind) { return kind == kUnitPlanes || kind == kUnitPlanesAgain; }

inline long product_tiles(ProductKind kind, int tile, long ni, long nj, long images, long halves) {
  const long fi = pair_on_i(kind) ? tile / 2 : tile, fj = pair_on_j(kind) ? tile / 2 : tile;
  return (ni + fi - 1) / fi * ((nj + fj - 1) / fj) * images * halves;
}

// Waves along i and j of a tile: each has at least 32 rows of i, or 32 of each of a pair's.
struct ProductWaves {
  int i, j;
};
constexpr ProductWaves product_waves(int tile, bool pair_i) {
  return tile == 256 ? ProductWaves{2, 4} : pair_i ? ProductWaves{1, 4} : ProductWaves{2, 2};
}

constexpr int kMostSplits = 128;
constexpr int kTilesAtOnce[] = {1280, 512, 256};  // of side 64, 128, 256 that the device holds

// Parts that the sum of a product on tiles of a side is cut into, where too few tiles
// would leave the device idle.
inline int splits_on(int size, ProductKind kind, int tile, long ni, long nj, long images, long halves, long K,
                     long segs) {
  if (pair_on_i(kind) || pair_on_j(kind)) return 1;
  const long tiles = product_tiles(kind, tile, ni, nj, images, halves);
  const long step = 128 / size, steps = (K + step - 1) / step * segs;
  return int(std::max(1l, std::min({512 / tiles, steps / 3, long(kMostSplits)})));
}

// Side of the tile: the least of the rounds of tiles that the device holds at once, times
// what a round takes (a tile's products at a rate that larger tiles come nearer to, and
// the wait for its first operands).
inline int product_tile(int size, ProductKind kind, long ni, long nj, long images, long halves, long K, long segs) {
  const bool again = kind == kUnitLastAgain || kind == kUnitPlanesAgain;
  if (const char* e = getenv("TILE")) return (size == 2 && !again) || atoi(e) < 256 ? atoi(e) : 128;
  int best = 64;
  double least = 0;
  for (int i = 0; i < (size == 2 && !again ? 3 : 2); ++i) {
    const int tile = 64 << i;
    const int splits = splits_on(size, kind, tile, ni, nj, images, halves, K, segs);
    const double tiles = double(product_tiles(kind, tile, ni, nj, images, halves)) * splits;
    const double step = 128.0 / size, steps = ((K + step - 1) / step * segs + splits - 1) / splits;
    const double rounds = std::max(1.0, tiles / kTilesAtOnce[i]);
    const double slow[] = {1.7, 1.3, 1.0};
    // ns: a step of a tile to itself; tiles that share a compute unit share its rate
    const double products = (size == 2 ? 1.0 : 14.0) * slow[i] * tile * tile * 0.0135 * std::min(tiles / 256, kTilesAtOnce[i] / 256.0);
    const double time = rounds * (3000 + steps * std::max(products, 400.0));
    if (i == 0 || time < least) {
      best = tile;
      least = time;
    }
  }
  return best;
}

inline int product_splits(int size, ProductKind kind, long ni, long nj, long images, long halves, long K, long segs) {
  return splits_on(size, kind, product_tile(size, kind, ni, nj, images, halves, K, segs), ni, nj, images, halves, K,
                   segs);
}

// Parts that the unit, in the backward pass, leaves the sums over the positions in:
// one for each wave's positions.
inline long product_sum_parts(int size, ProductKind kind, long ni, long nj, long images, long K) {
  const int tile = product_tile(size, kind, ni, nj, images, 1, K, 1);
  const ProductWaves w = product_waves(tile, pair_on_i(kind));
  return images * (((pair_on_i(kind) ? nj : ni) + tile - 1) / tile) * (pair_on_i(kind) ? w.j : w.i);
}

// Positions up to which the forward unit reads its weights without tiles.
constexpr long kFewPositions = 32;

// Whether the backward pass makes g and u again from x rather than having them stored.
inline bool product_remakes(int size, long C) { return size == 2 ? C <= 1024 : C <= 64; }

}  // namespace oaa
