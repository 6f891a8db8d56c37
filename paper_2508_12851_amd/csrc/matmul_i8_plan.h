// How prism_matmul_i8 cuts a product, by its sizes (no HIP in here: the rule runs and is tested on the CPU).
#ifndef PRISM_MATMUL_I8_PLAN_H_
#define PRISM_MATMUL_I8_PLAN_H_

#include <algorithm>
#include <cmath>

#include "ffn_paths.h"

namespace prism {
namespace mm8 {

constexpr int kMaxSplits = 8;
constexpr int kWorkgroups = 256;      // one per CU
constexpr size_t kMaxPartialBytes = (size_t)64 << 20;

enum class Tile { k64x64, k64x128, k128x128, k256x256, kShort };
struct Plan {
  Tile tile;
  int splits;
};

// The tile and the splits of a product, by an estimate of its time in us.  A round of items takes a fixed time and so much
// per k-tile of 128 bytes, more as more workgroups share the L2: fitted to 20 products from 1 x 1024 x 4096 to 4096 x 4096 x
// 14336, weights from HBM, of which each was run with all tiles and 1 to 8 splits.  Two 64 x 64 items share a CU, each then 1.5
// times as long.  A split costs the kernel that adds the parts and their traffic; more workgroups than CUs by splits were
// slower everywhere.  Measured, us, 64 x 64 / 64 x 128 / 128 x 128 (best number of splits of each): 1 x 4096 x 14336 16.9 / 18.0;
// 64 x 14336 x 4096 15.8 / 20.2; 128 x 14336 x 4096 23.7 / 19.8 / 23.9; 300 x 11008 x 4096 34.2 / 28.2 / 33.5; 600 x 4096 x 8192
// 59.5 / 49.5 / 36.5; 1000 x 4096 x 4096 32.8 / 28.2 / 22.1 (256 x 256 39.7); 2000 x 4096 x 4096 64.1 / 52.0 / 40.0 (45.8).
struct TileCost {
  Tile tile;
  int bm, bn, resident;     // resident: workgroups of a CU
  float fixed, per_kt, per_kt_load;
};
constexpr TileCost kTiles[] = {{Tile::k64x64, 64, 64, 2, 3.6f, 0.27f, 0.01f},
                               {Tile::k64x128, 64, 128, 1, 4.5f, 0.27f, 0.03f},
                               {Tile::k128x128, 128, 128, 1, 4.5f, 0.34f, 0.18f},
                               {Tile::k256x256, 256, 256, 1, 8.6f, 0.85f, 0.65f}};
constexpr float kSplitFixed = 3.7f, kBytesPerUs = 5e6f, kStreamBytesPerUs = 6e6f;
constexpr int kMinSplitKt = 3;        // k-tiles of a split, at least: the depth of the rings

static inline Plan plan_of(int M, int N, int K) {
  const int kt = (int)(align_up((size_t)K, kI8RowAlign) / 128);
  if (kt < kMinSplitKt) return Plan{Tile::kShort, 1};
  Plan best{Tile::k128x128, 1};
  float least = INFINITY;
  const float stream = (float)N * (float)K / kStreamBytesPerUs;
  for (const TileCost& t : kTiles) {
    const long long items = (long long)ceil_div(M, t.bm) * ceil_div(N, t.bn);
    for (int s = 1; s <= kMaxSplits && (s == 1 || kt / s >= kMinSplitKt); ++s) {
      const long long n = items * s;
      if (s > 1 && (n > kWorkgroups || t.tile == Tile::k256x256 || (size_t)s * M * align_up(N, 4) * 4 > kMaxPartialBytes)) break;
      float rounds = (float)((n + kWorkgroups - 1) / kWorkgroups);
      if (t.resident == 2 && n > kWorkgroups) rounds = 1.5f * (float)((n + 2 * kWorkgroups - 1) / (2 * kWorkgroups));
      const float load = std::min(1.f, (float)n / kWorkgroups);
      const float loop = rounds * (t.fixed + (float)ceil_div(kt, s) * (t.per_kt + t.per_kt_load * load));
      float us = std::max(loop, t.fixed + stream);
      if (s > 1) us += kSplitFixed + 8.f * (float)s * (float)M * (float)N / kBytesPerUs;
      if (us < least) {
        least = us;
        best = Plan{t.tile, s};
      }
    }
  }
  return best;
}

}  // namespace mm8
}  // namespace prism
#endif  // PRISM_MATMUL_I8_PLAN_H_
