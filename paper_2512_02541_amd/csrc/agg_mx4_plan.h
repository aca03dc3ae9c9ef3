// Which kernel computes which rows of a product of 4-bit floats: plain host code, so that a test can
// check it without a GPU.
#pragma once

#include <stdint.h>

#include "agg_linear_plan.h"

namespace agg {

// kernels, by their tile of tokens x channels
enum Mx4Kernel {
  kMx4Few,     // 16 x 16, k shared by eight wavefronts
  kMx4Tile64,  // 64 x 64, up to four workgroups on a CU
  kMx4Tile128, // 128 x 128, two on a CU, the next step's copies under way during a step
  kMx4Tile128Many,  // 128 x 128, four on a CU, whose copies run beside each other's products
  kMx4Tile256, // 256 x 256, one on a CU
  kMx4Panel    // 512 tokens in registers, passes of 64 channels
};

// The first `split` rows take 256 x 256 tiles, the rest `kernel` (split = 0: all).
struct Mx4Plan {
  int64_t split;
  Mx4Kernel kernel;
};

static inline int64_t mx4_tiles(int64_t rows, int64_t N, int count, int edge) {
  return (rows + edge - 1) / edge * ((N + edge - 1) / edge) * count;
}

constexpr int kPanelRows = 512;
constexpr int kPassChannels = 64;
constexpr int kPanelMostK = 1024;

static inline int64_t mx4_passes(int64_t rows, int64_t N, int count) {
  return (rows + kPanelRows - 1) / kPanelRows * ((N + kPassChannels - 1) / kPassChannels) * count;
}

// Measured in us, each side of a border by both kernels (N, K, matrices: rows: this side / the other).  The first border
// was measured with 32 rows and more; of few rows it sends wide or deep products to tiles that walk all of k in
// one workgroup: 1 row 11008 -> 4096 12.8 us, where its weights' bytes take 4.9.
//   few        1024, 1024, 3: 32: 4.1 / 4.6 with tiles of 64, 64: 5.0 / 4.6; 1024, 1024, 1: 128: 4.2 / 4.6,
//              261: 7.3 / 4.6; 1024, 4096, 1: 64: 5.8 / 7.8, 128: 9.3 / 8.0
//   tiles 64   1024, 1024, 3: 1044: 7.4 / 8.2 with 128, 1374: 9.5 / 9.4; 1024, 4096, 1: 2748: 14.4 / 15.2,
//              5496: 26.4 / 21.1
//   tiles 128, two or four on a CU   1024, 1024, 1: 5496: 9.2 / 9.6, 10992: 14.7 / 12.1;
//              1024, 4096, 1: 5496: 21.1 / 24.3, 10992: 38.5 / 32.0
//   panel      1024, 1024, 3: 21984: 53 / 56, 137400: 232 / 315, 10992: 36.6 / 31.0; 512, 512, 3:
//              21984: 23.6 / 23.4, 54960: 42.9 / 47.6
//   tiles 256  1024, 4096, 1: 10992: 30.7 / 32.0, 54960: 129 / 135; 4096, 4096, 1: 21984: 199 / 241;
//              for K up to 1024 their few steps do not pay for their start and end: 1024, 1024, 1: 21984: 26.0 / 22.1
static inline Mx4Plan plan_mx4(int64_t rows, int64_t N, int64_t K, int count, bool residual) {
  const int64_t few = mx4_tiles(rows, N, count, 16);
  if (few <= 2 * kGemmCus && few * K <= (int64_t)kGemmCus * 4096) return {0, kMx4Few};
  if (mx4_tiles(rows, N, count, 64) <= 4 * kGemmCus) return {0, kMx4Tile64};
  if (K <= kPanelMostK && !residual && mx4_passes(rows, N, count) >= 8 * kGemmCus) return {0, kMx4Panel};
  if (K > kPanelMostK) {
    // whole rounds of large tiles; a last round that is more than six tenths full counts as one
    const int64_t per_m = (N + 255) / 256 * count, tiles = mx4_tiles(rows, N, count, 256);
    const int64_t rounds = tiles / kGemmCus;
    if (tiles - rounds * kGemmCus > kGemmCus * 6 / 10 || tiles == rounds * kGemmCus) return {0, kMx4Tile256};
    const int64_t split = rounds * kGemmCus / per_m * 256;
    if (split > 0 && split < rows)
      return {split, mx4_tiles(rows - split, N, count, 64) <= 4 * kGemmCus    ? kMx4Tile64
                     : mx4_tiles(rows - split, N, count, 128) <= 2 * kGemmCus ? kMx4Tile128
                                                                               : kMx4Tile128Many};
  }
  return {0, mx4_tiles(rows, N, count, 128) <= 2 * kGemmCus ? kMx4Tile128 : kMx4Tile128Many};
}

}  // namespace agg
