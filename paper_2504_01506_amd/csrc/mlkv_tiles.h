// Which tile a product of the orthogonalised updates (mlkv_orth.hip) takes.
// Host code only, apart so that a check can ask it on the CPU.
#pragma once

#include <stdint.h>

namespace mlkv {

constexpr int kOrthPad = 64;  // sides of X and A are padded to multiples of it, with zeros
constexpr int kOrthUnits = 256;

// k64K: a tile of 64 whose four waves each take pieces of the sum.
enum class OrthTile { k64K, k64, k128, k192, k256 };

// That of the least time by a fit to what the kernels measured, us a tile on a
// unit of its own, for 32 of k and beside that (symmetric results, and X with
// X^T).
//
// Large tiles read less for a product, 4096 x 4096 B X 370 us with 256,
// 430 with 128, 630 with 64; but tiles come in rounds of one a unit: the 253 tiles
// of 192 of a symmetric result of 4096 take 220 us, its 136 of 256 264, its 528
// of 128 287. Two of 128 or 64 fit a unit, so that a last round that is not full
// takes less, beside the one before: 276 of 128 take 1.6 times what 256 do (2944 x
// 3968, X X^T and A A 348 us, with 136 of 192 394).
// At most one round of 64 and sums of kOrthLongSum or more: four waves by
// pieces of k (1024 x 4096 X X^T 36 us, 41 in quarters; sums of 300 8.1 and 6.5).
constexpr int kOrthLongSum = 1024;
struct OrthTileTime {
  int side;
  OrthTile tile;
  float depth, rest[2];
};
constexpr OrthTileTime kOrthTimes[] = {{64, OrthTile::k64, 0.34f, {2.5f, 2.7f}},
                                       {128, OrthTile::k128, 0.9f, {5.0f, 11.0f}},
                                       {192, OrthTile::k192, 1.75f, {8.0f, 20.0f}},
                                       {256, OrthTile::k256, 3.2f, {10.0f, 16.0f}}};

// mp x np: the padded matrix (symmetric: the result is mp x mp), k: length of the sum.
inline OrthTile orth_tile(int64_t mp, int64_t np, int64_t batch, bool symmetric, int64_t k) {
  const OrthTileTime* best = nullptr;
  float least = 0.0f;
  bool one_round = false;
  for (const OrthTileTime& t : kOrthTimes) {
    const int64_t ti = (mp + t.side - 1) / t.side, tj = (np + t.side - 1) / t.side;
    const int64_t tiles = batch * (symmetric ? ti * (ti + 1) / 2 : ti * tj);
    const int64_t rounds = (tiles + kOrthUnits - 1) / kOrthUnits;
    const float part = (float)(tiles % kOrthUnits) / kOrthUnits;
    const bool beside = rounds > 1 && part > 0.0f && t.side <= 128;
    const float taken = beside ? (float)(rounds - 1) + 0.6f + 0.4f * part : (float)rounds;
    const float time = taken * (t.depth * (float)(k / 32) + t.rest[symmetric ? 0 : 1]);
    if (best == nullptr || time < least) {
      best = &t;
      least = time;
      one_round = rounds == 1;
    }
  }
  return best->tile == OrthTile::k64 && one_round && k >= kOrthLongSum ? OrthTile::k64K : best->tile;
}

}  // namespace mlkv
