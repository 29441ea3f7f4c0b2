// Which tile a product of gated.hpp runs on, and how its sum is cut. Plain host code.
#pragma once

#include <algorithm>
#include <cstdlib>

#include "gated.hpp"

namespace oaa {

inline long product_tiles(ProductKind kind, int tile, long ni, long nj, long images, long halves) {
  const long fi = kind == kUnitLast ? tile / 2 : tile, fj = kind == kUnitPlanes ? tile / 2 : tile;
  return (ni + fi - 1) / fi * ((nj + fj - 1) / fj) * images * halves;
}

// Waves along i and j of a tile: each has at least 64 rows of i, or 64 of each of a pair's.
struct ProductWaves {
  int i, j;
};
constexpr ProductWaves product_waves(int tile, bool pair_on_i) {
  return tile == 256 ? ProductWaves{2, 4} : pair_on_i ? ProductWaves{1, 4} : ProductWaves{2, 2};
}

// Side of the tile.
inline int product_tile(int size, ProductKind kind, long ni, long nj, long images, long halves, long splits) {
  if (const char* e = getenv("TILE")) return size == 2 ? atoi(e) : 128;
  return size == 2 && product_tiles(kind, 256, ni, nj, images, halves) * splits >= 256 ? 256 : 128;
}

// Parts that the unit, in the backward pass, leaves the sums over the positions in:
// one for each wave's positions.
inline long product_sum_parts(int size, ProductKind kind, long ni, long nj, long images) {
  const int tile = product_tile(size, kind, ni, nj, images, 1, 1);
  const ProductWaves w = product_waves(tile, kind == kUnitLast);
  return images * (((kind == kUnitLast ? nj : ni) + tile - 1) / tile) * (kind == kUnitLast ? w.j : w.i);
}

// Parts that the sum of a product is cut into, where too few tiles would leave the
// device idle.
inline int product_splits(int size, ProductKind kind, long ni, long nj, long images, long halves, long K, long segs) {
  const long tiles = product_tiles(kind, 128, ni, nj, images, halves);
  const long step = 128 / size, steps = (K + step - 1) / step * segs;
  return int(std::max(1l, std::min({(512 + tiles - 1) / tiles, steps / 4, 64l})));
}

// Whether the backward pass makes g and u again from x rather than having them stored.
inline bool product_remakes(int size, long C) { return size == 2 ? C <= 1024 : C <= 64; }

}  // namespace oaa
