// How a call of attention to keys of another length is shared out over workgroups: plain host code, so that a test can compile
// it by itself.
#pragma once

#include <stdint.h>

namespace agg {

// A pair is a (batch element, key head); its rows are its queries by the heads that share the key head.
struct CrossPlan {
  int wide;           // the kernel of many rows (cross_wide_kernel), else that of few (cross_few_kernel)
  int tiles;          // few: 16-row tiles of a wavefront
  int width;          // wide: rows of a workgroup, 256 or 128
  int tail;           // wide: rows of a pair's last workgroup where they are fewer, 0: it is as wide as the others
  int halves;         // wide, of width 128: eight wavefronts, four for each half of a workgroup's keys
  int64_t row_tiles;  // workgroups along a pair's rows
  int splits;         // ... along its keys; more than one: partial results, joined by a second launch
};

constexpr int kFewWaves = 8;    // wavefronts of a workgroup, each with keys of its own
constexpr int kKeyBlock = 32;   // keys of a wavefront's step
constexpr int kFewRows = 32;    // most rows of such a workgroup
constexpr int kWideRows = 256;  // rows of a wide workgroup
constexpr int kMostSplits = 64;
constexpr int kMostShared = 4096;  // most workgroups of a call that is shared out along the keys

// wide_fits: the distances between rows are what the wide kernel can address; ragged: the sequences may have different lengths
inline CrossPlan plan_cross(int64_t pairs, int64_t rows, int64_t keys, bool ragged, bool wide_fits) {
  CrossPlan p;
  p.width = p.tail = p.halves = 0;
  p.tiles = rows <= 16 ? 1 : 2;
  p.row_tiles = (rows + 16 * p.tiles - 1) / (16 * p.tiles);
  // Up to 32 rows the kernel of few rows.  Up to 64 while its two workgroups of a pair all run at once: us, few / wide, paged, 16 heads, 64 queries
  // to 262 keys 5.4 / 6.7, to 5496 12.6 / 19.4, to 137400 106 / 105; with 384 pairs to 1374 keys 45.7 / 26.1.
  p.wide = wide_fits && rows > kFewRows && (rows > 2 * kFewRows || pairs * p.row_tiles > 256);
  if (!p.wide) {
    // Splits by predicted time: a start, a wavefront's steps one after another, and a second launch.  More workgroups than run at once
    // (two on a CU of up to 16 rows, one of more) gain nothing: the memory is busy with them.
    const int64_t groups = pairs * p.row_tiles, steps = (keys + kKeyBlock * kFewWaves - 1) / (kKeyBlock * kFewWaves);
    const int64_t at_once = p.tiles == 1 ? 512 : 256;
    const double step = p.tiles == 1 ? 0.55 : 0.85;
    double best = 0;
    p.splits = 1;
    for (int64_t s = 1; s <= kMostSplits && (s == 1 || (groups * s <= at_once && steps / s >= 1)); ++s) {
      const double us = (double)((steps + s - 1) / s) * step + (s > 1 ? 3.0 + 0.03 * s : 0.0);
      if (s == 1 || us < best) {
        best = us;
        p.splits = (int)s;
      }
    }
    return p;
  }
  // Width and splits by predicted time: rounds of 512 workgroups (two on a CU; alone on it one takes little more than half as
  // long), each with its start, its end and its share of the key tiles; a second launch and the partial results' way to
  // memory and back.  Workgroups of 128 rows that all run alone on their CUs have eight wavefronts, four for each half of their keys, where
  // that is tiles enough.  Of sequences of different lengths half the workgroups are taken to be there.
  const int64_t tiles = (keys + 63) / 64;
  double best = -1;
  p.splits = 0;
  for (int width = kWideRows; width >= 128; width -= 128) {
    const int64_t row_tiles = (rows + width - 1) / width;
    const int rest = (int)(rows % width);
    const int tail = width == 128 || rest == 0 ? 0 : rest <= 128 ? 128 : rest <= 192 ? 192 : 0;
    const double pair = width == 128 ? 0.565 : 1.0;
    const double saved = tail ? (tail == 128 ? 0.435 : 0.21) / (double)row_tiles : 0.0;  // by narrow last workgroups
    for (int s = 1; s <= kMostSplits && (s == 1 || (tiles / s >= 4 && pairs * row_tiles * s <= kMostShared)); ++s) {
      const int64_t groups = pairs * row_tiles * s, there = ragged ? (groups + 1) / 2 : groups, rest_groups = there % 512;
      const int halves = width == 128 && groups <= 256 && tiles / s >= 8;
      const double alone = halves ? 0.285 : width == 128 ? 0.34 : 0.535;
      const double rounds = (double)(there / 512) * pair + (rest_groups == 0 ? 0.0 : rest_groups <= 256 ? alone : pair);
      double us = rounds * (there > 512 ? 1.0 - saved : 1.0) * 1.65 * (double)((tiles + s - 1) / s) + 4.0 + halves;
      if (s > 1) us += 6.0 + (double)pairs * (double)rows * s * 66 * 8 / 4.4e6;
      if (best < 0 || us < best) {
        best = us;
        p.width = width;
        p.tail = tail;
        p.halves = halves;
        p.row_tiles = row_tiles;
        p.splits = s;
      }
    }
  }
  return p;
}

}  // namespace agg
