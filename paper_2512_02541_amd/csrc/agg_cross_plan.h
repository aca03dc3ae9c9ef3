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
constexpr int kMostShared = 4096;       // most workgroups of a call that is shared out along the keys
constexpr int64_t kUncached = 1 << 20;  // keys of all pairs, 256 bytes each with their values, that fill the cache behind the L2s

// wide_fits: the distances between rows are what the wide kernel can address; ragged: the sequences may have different lengths, 2: of
// queries and of keys; paged: keys and values in a cache
inline CrossPlan plan_cross(int64_t pairs, int64_t rows, int64_t keys, int ragged, bool wide_fits, bool paged) {
  CrossPlan p;
  p.wide = p.width = p.tail = p.halves = 0;
  p.tiles = rows <= 16 ? 1 : 2;
  p.row_tiles = (rows + 16 * p.tiles - 1) / (16 * p.tiles);
  if (rows <= kFewRows || !wide_fits) {
    // Splits by predicted time: a wavefront's steps one after another, and a second launch.  More workgroups than run at once
    // (two on a CU of up to 16 rows, one of more) gain nothing where the sequences are alike: the memory is busy with them.  Where they
    // are not, the long ones would end alone: there more rounds are taken, of 2 us each (us, one token each over up to 10000
    // keys of 24 sequences, 16 heads: 124 unsplit, 103 / 95 / 91 / 106 with 2 / 4 / 16 / 32 splits; over 250 calls with random lengths
    // the choice is 4 % behind the fastest in the mean).
    const int64_t groups = pairs * p.row_tiles, steps = (keys + kKeyBlock * kFewWaves - 1) / (kKeyBlock * kFewWaves);
    const int64_t at_once = p.tiles == 1 ? 512 : 256, most = !ragged ? at_once : p.tiles == 1 ? 4096 : 1024;
    const double step = p.tiles == 1 ? 0.55 : 0.85;
    double best = 0;
    p.splits = 1;
    for (int64_t s = 1; s <= kMostSplits && (s == 1 || (groups * s <= most && steps / s >= 1)); ++s) {
      const double us = (double)((steps + s - 1) / s) * step + (s > 1 ? 3.0 + 0.03 * s : 0.0) +
                        (ragged ? 2.0 * (double)(groups * s) / (double)at_once : 0.0);
      if (s == 1 || us < best) {
        best = us;
        p.splits = (int)s;
      }
    }
    return p;
  }
  // Kernel, width and splits by predicted time.  A tile of keys takes 256 rows 1.65 us, two workgroups on a CU, and 0.535 of that alone on it;
  // 128 rows 0.565 and 0.34 of it; 128 rows and eight wavefronts, four for each half of the keys, 0.285, always alone; 32 rows of the
  // kernel of few rows 0.22 us out of pages and 0.33 in place, always alone.  To that come starts and ends, and for splits a second
  // launch and the partial results' way to memory and back.  (us, few / wide, out of pages, 16 heads: 261 queries to 1374 keys 9.0 / 13.0,
  // 512 to 512 6.3 / 8.9, 64 to 137400 106 / 105, 64 of 24 sequences to 1374 45.7 / 26.1; in place 261 to 1374 11.9 / 13.3, 522 to 522
  // 13.8 / 9.6.)
  // Like sequences: rounds of as many workgroups as run at once, eight wavefronts where that is one round.  Sequences of different
  // lengths, which the host does not know: their throughput, and a longest piece behind it, by constants fitted to 693 calls of 33 to 8000
  // rows a pair with random lengths, every kernel with up to 64 splits.  (Their choice is 4 % behind the fastest in the mean and 14 % at the
  // ninth decile; 0.4 of the full work at the rates above 8 % and 29 %: 36 queries of 8 sequences to 13740 cached keys, 16 heads, 64.1 us
  // against 48.0, 56 to 2878, 20 / 4 heads, 26.6 against 19.5.)  Where queries end early too there is less work: 0.8 of the first
  // term (349 such calls: 4 % behind with 0.8 as with 1, 8 % with 0.5).
  struct Ragged {
    double tile, ends;            // of a workgroup among as many as run at once
    double last_tile, last_ends;  // of the last ones
    double join, bytes;           // of the second launch
  };
  static constexpr Ragged kRagged[] = {{0.53, 5.3, 1.65, 14.2, 6.0, 0.67}, {0.37, 6.4, 0.84, 5.6, 6.0, 0.67}, {0.25, 7.1, 0.48, 6.2, 6.0, 0.67},
                                       {0.31, 6.1, 0.37, 1.0, 1.25, 1.29}, {0.34, 5.7, 0.21, 1.5, 1.25, 1.29}};  // kinds 0 to 3; 3 out of pages
  const int64_t tiles = (keys + 63) / 64;
  double best = -1;
  p.splits = 0;
  for (int kind = 0; kind < 4; ++kind) {
    const int width = kind == 0 ? kWideRows : kind == 3 ? kFewRows : 128, halves = kind == 2, few = kind == 3;
    const int64_t row_tiles = (rows + width - 1) / width, unsplit = pairs * row_tiles;
    const int log_at_once = halves || few ? 8 : 9;
    const int64_t at_once = (int64_t)1 << log_at_once;
    const int rest = (int)(rows % width);
    const int tail = width != kWideRows || rest == 0 ? 0 : rest <= 128 ? 128 : rest <= 192 ? 192 : 0;
    const double pair = few ? (paged ? 0.22 : 0.33) : (halves ? 0.285 : width == 128 ? 0.565 : 1.0) * 1.65;
    const double alone = few || halves ? pair : (width == 128 ? 0.34 : 0.535) * 1.65;
    // keys that no cache holds come from memory for each 32 rows again (us, 48 rows of 48 pairs to 32099 keys: 135, 128 rows wide 81)
    const double reads = few && pairs * keys >= kUncached ? (double)unsplit * (double)keys * 256 / 5.2e6 : 0.0;
    const double saved = tail ? (tail == 128 ? 0.435 : 0.21) / (double)row_tiles : 0.0;  // by narrow last workgroups
    // (few divisions: a call plans up to four times, once for each place that keys may lie in)
    int64_t most = tiles / (halves ? 8 : 4);
    if (most > kMostSplits) most = kMostSplits;
    const int64_t room = (halves && !ragged ? at_once : kMostShared) / unsplit;
    if (most > room) most = room;
    if (most < 1) {
      if (halves && (tiles < 8 || (!ragged && room < 1))) continue;
      most = 1;
    }
    for (int s = 1; s <= (int)most; ++s) {
      const int64_t groups = unsplit * s, last = groups & (at_once - 1);
      const double here = (double)((tiles + s - 1) / s);
      const double bytes = (double)pairs * (double)rows * s * 66 * 8 / 4.4e6;  // us of the partial results' way
      const double join = s > 1 ? (few ? 4.0 : 6.0) + bytes : 0.0;
      double us;
      if (ragged) {
        const Ragged& r = kRagged[few && paged ? 4 : kind];
        us = (ragged == 2 ? 0.8 : 1.0) * (double)groups / (double)at_once * (r.tile * here + r.ends) + r.last_tile * here +
             r.last_ends + (s > 1 ? r.join + r.bytes * bytes : 0.0);
      } else if (few) {
        us = (double)((groups + at_once - 1) >> log_at_once) * (3.8 + pair * here);
        if (us < reads) us = reads;
        us += join;
      } else {
        const double rounds = (double)(groups >> log_at_once) * pair + (last == 0 ? 0.0 : last <= 256 ? alone : pair);
        us = rounds * (groups > at_once ? 1.0 - saved : 1.0) * here + 4.0 + halves + join;
      }
      if (best < 0 || us < best) {
        best = us;
        p.wide = !few;
        p.width = few ? 0 : width;
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
