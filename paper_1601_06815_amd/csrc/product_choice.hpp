// Which tile a product of gated.hpp runs on, and how its sum is cut. Plain host code.
#pragma once

#include <algorithm>

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

// The side of a product's tiles, and the parts that its sum is cut into.
struct ProductChoice {
  int tile, splits;
};

// The least of: the rounds of tiles that the device holds at once, times what a round takes
// (the wait for a tile's first operands, its results, and its steps), and the parts' way
// through memory. Large tiles read least, but take longest alone, and their last round may
// be nearly empty. Measured, us by side 64, 128, 256 (bfloat16 unit forward): 512 positions 512 ->
// 2048 7.4, 9.2, 17.8; 2048 positions 1024 -> 4096 66, 39, 34; 16 images of 64 x 64 planes,
// 256 -> 512 92, 57, 46. What passes through memory is not estimated, nor what a tile of few steps
// waits for: there the estimate may be half of what is measured. (A unit has to have its whole sums: it is not cut. In the backward pass
// it has no tile of 256: its registers do not hold what it needs besides the sums.)
inline ProductChoice product_choice(int size, ProductKind kind, long ni, long nj, long images, long halves, long K,
                                    long segs) {
  // ns of a step: of a tile that has a compute unit to itself, and at the full rate
  static constexpr double alone[2][3] = {{400, 500, 1000}, {1100, 2100, 4400}};
  static constexpr double full[2][3] = {{200, 450, 1600}, {660, 1830, 5600}};
  // around a tile's steps; small tiles' results in planes, many short pieces, take longer (bfloat16,
  // us without the 1500 ns and with: 128 planes of 54 x 54, 128 -> 512 252 and 238, 64 of 54 x 54,
  // 32 -> 128 40 and 31, 4 of 112 x 112, 64 -> 128 10.9 and 9.6; but 2 of 218 x 218, 64 -> 192 24 and
  // 30, in float32 43 and 49; ten other sizes the same)
  const double planes = kind == kUnitPlanes ? 1500 : 0, around[] = {3000 + planes, 3000 + planes, 6000};
  const bool again = kind == kUnitLastAgain || kind == kUnitPlanesAgain, pair = pair_on_i(kind) || pair_on_j(kind);
  const long step = 128 / size, steps = (K + step - 1) / step * segs;
  const long most = pair ? 1 : std::max(1l, std::min(steps / 3, long(kMostSplits)));
  ProductChoice best{64, 1};
  double least = 0;
  for (int i = 0; i < (again ? 2 : 3); ++i) {
    const long tiles = product_tiles(kind, 64 << i, ni, nj, images, halves);
    for (long splits = 1; splits <= most; splits *= 2) {
      const double all = double(tiles) * splits, each = double((steps + splits - 1) / splits);
      const double rounds = std::max(1.0, all / kTilesAtOnce[i]);
      const double shared = std::min(all, double(kTilesAtOnce[i])) / 256;
      double time = rounds * (around[i] + each * std::max(alone[size > 2][i], shared * full[size > 2][i]));
      // parts are written and read at 4 TB/s by one launch more
      if (splits > 1) time += 4000 + double(ni) * nj * images * halves * splits * 8 / 4000;
      if (least == 0 || time < least) {
        best = {64 << i, int(splits)};
        least = time;
      }
    }
  }
  return best;
}

// Parts that the unit, in the backward pass, leaves the sums over the positions in:
// one for each wave's positions.
inline long product_sum_parts(int size, ProductKind kind, long ni, long nj, long images, long K) {
  const int tile = product_choice(size, kind, ni, nj, images, 1, K, 1).tile;
  const ProductWaves w = product_waves(tile, pair_on_i(kind));
  return images * (((pair_on_i(kind) ? nj : ni) + tile - 1) / tile) * (pair_on_i(kind) ? w.j : w.i);
}

// Positions up to which the forward unit reads its weights without tiles.
constexpr long kFewPositions = 32;

// Whether the backward pass makes g and u again from x rather than having them stored: the
// product grows with C, what storing them moves (16 bytes a hidden value and position) does
// not. us of both passes, stored and made again: float32, 8 planes of 56 x 56, 64 -> 256 103 and
// 102, 16384 positions 32 -> 128 59 and 49, 256 -> 1024 412 and 446; bfloat16, 16384 positions, 256
// -> 1024 189 and 148, 512 -> 2048 486 and 412, 1024 -> 4096 1158 and 1233 (and 512 positions 87
// and 80), 2048 -> 8192 3300 and 4160; float16, 512 -> 2048 495 and 441. Of equals the one that
// needs no memory.
inline bool product_remakes(int size, long C) { return size == 2 ? C <= 1024 : C <= 64; }

}  // namespace oaa
