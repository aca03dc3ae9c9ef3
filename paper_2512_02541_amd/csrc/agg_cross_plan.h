// How a call of attention to keys of another length is shared out over workgroups: plain host code, so that a test can compile
// it by itself.
#pragma once

#include <stdint.h>

namespace agg {

// A pair is a (batch element, key head); its rows are its queries by the heads that share the key head.
struct CrossPlan {
  int tiles;          // 16-row tiles of a wavefront
  int64_t row_tiles;  // workgroups along a pair's rows
  int splits;         // ... along its keys; more than one: partial results, joined by a second launch
};

constexpr int kFewWaves = 8;   // wavefronts of a workgroup, each with keys of its own (four of 64 rows)
constexpr int kKeyBlock = 32;  // keys of a wavefront's step

inline int few_waves(int tiles) { return tiles == 4 ? 4 : kFewWaves; }

inline CrossPlan plan_cross(int64_t pairs, int64_t rows, int64_t keys) {
  CrossPlan p;
  p.tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  p.row_tiles = (rows + 16 * p.tiles - 1) / (16 * p.tiles);
  const int64_t groups = pairs * p.row_tiles, steps = (keys + kKeyBlock - 1) / kKeyBlock / few_waves(p.tiles);
  int64_t splits = 512 / (groups < 1 ? 1 : groups);
  if (splits > steps / 2) splits = steps / 2;
  p.splits = splits < 1 ? 1 : (int)splits;
  return p;
}

}  // namespace agg
