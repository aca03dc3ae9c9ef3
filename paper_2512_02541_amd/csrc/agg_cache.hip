// New tokens of a paged key/value cache: norm and rotary positions of keys (and queries) on the way, keys and values into
// the fragment order of their pages.
#include "agg_internal.h"
#include "agg_lds_copy.h"
#include "agg_rows.h"

namespace agg {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// A workgroup takes 32 (few rows: 16) consecutive rows of a sequence, half or a quarter of a page, and the tokens that become them:
// keys, values and queries.  It works out their cosines and signed sines once, a pair of channels a thread, and its wavefronts take
// the heads in turn, eight lanes a row of a head, a head's rows requested while the one before is worked on.  A key's 16-byte chunk
// goes to the page from the registers it was turned in: eight consecutive rows make a whole 128-byte line of one chunk number.
// Values turn through LDS with the transposing read, which leaves a lane with the eight rows of one channel that make a chunk of the
// page; a chunk that the new rows fill only in part is stored element by element, so that its other rows stay.
// Many rows are bound by HBM: 137400 of 16 heads, keys and values, 225 us = 5.0 TB/s; 21984 with their queries 57 us.  Few are one
// chain of latencies (lengths, page, rows, sines, exchange): a frame of 1374 tokens 7.8 to 8.8 us (12 in pieces of 32), one token
// 4.9.  Partners fetched through LDS took 21984 rows 68 us, with eight-way bank conflicts; queries and keys in workgroups of
// their own, each with a table, 3 x 8328 tokens of 12 and 4 heads 41 us instead of 30.
// ---------------------------------------------------------------------------
constexpr int kAppendThreads = 256;
constexpr int kAppendWaves = kAppendThreads / 64;

namespace {

// Where a channel's partner is: nowhere (nothing turns), beside it in the same lane's registers, in another lane's register of the
// same number, or anywhere.
enum { kNoPairs, kPairsInLane, kPairsAcrossLanes, kPairsAnywhere };

// What a lane knows of its eight channels of any row.
struct Channels {
  uint32_t other[2];    // a byte each: the channel's other one, bit 7: it turns at all
  int lane_at;          // kPairsAcrossLanes: 4 * the lane that holds the others
};

// a row's table of cosines and signed sines: 16-byte chunk q of lane j (channels 8 j + 2 q, + 1) lies at this place, so that the
// sixteen lanes served together, of two rows, read from different banks
__device__ __forceinline__ int turn_chunk(int row, int q, int j) { return row * 32 + ((q * 8 + j) ^ (8 * (row & 1))); }

// norm of a row's eight channels.  affine: what the norm multiplies by (from the lane's first channel on) and, kHeadDim behind, adds
__device__ __forceinline__ void norm8(float (&x)[8], int kind, float eps, const float* affine) {
  float mean = 0.f;
  if (kind == AGG_NORM_LAYER) {
#pragma unroll
    for (int i = 0; i < 8; ++i) mean += x[i];
    mean = sum_of_8(mean) * (1.f / kHeadDim);
  }
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] -= mean;
    sq += x[i] * x[i];
  }
  const float r = rsqrtf(sum_of_8(sq) * (1.f / kHeadDim) + eps);
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const f32x4 g = *reinterpret_cast<const f32x4*>(affine + i);
    const f32x4 b = *reinterpret_cast<const f32x4*>(affine + kHeadDim + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i + e] = x[i + e] * r * g[e] + b[e];
  }
}

// rotation of a row's eight channels; scratch: 512 floats of this wavefront
template <int kPairs>
__device__ __forceinline__ void turn8(float (&x)[8], const Channels& ch, int lane, int row, const f32x4* turns, float* scratch) {
  if constexpr (kPairs == kNoPairs) return;
  const int j = lane & 7;
  float y[8];
  if constexpr (kPairs == kPairsInLane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
  } else if constexpr (kPairs == kPairsAcrossLanes) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __int_as_float(__builtin_amdgcn_ds_bpermute(ch.lane_at, __float_as_int(x[i])));
  } else {
    // register i of all lanes in a row of 64 floats: every access of a lane group falls on as many banks as it has lanes, save where
    // a section ends inside a lane
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < 8; ++i) scratch[i * 64 + lane] = x[i];
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t other = ch.other[i / 4] >> (8 * (i % 4));
      y[i] = scratch[(other & 7u) * 64 + (lane & 56) + ((other >> 3) & 7u)];
    }
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const f32x4 cs = turns[turn_chunk(row, q, j)];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = 2 * q + e;
      const float turned = turn_channel(x[i], y[i], cs[2 * e], cs[2 * e + 1]);
      // by selection: an infinity times 0 is none of the other channels' business
      y[i] = (ch.other[i / 4] >> (8 * (i % 4))) & 0x80u ? turned : x[i];
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = y[i];
}

}  // namespace

template <int kPairs, int kRows>
__global__ __launch_bounds__(kAppendThreads, kPairs == kPairsAnywhere && kRows == 32 ? 3 : 4) void append_kernel(AppendArgs a) {
  __shared__ __align__(16) f32x4 turns[kRows * 32];
  // of a wavefront: eight rows of a head while they are turned, then a head's values while they are transposed
  __shared__ __align__(16) uint16_t space[kAppendWaves][kRows == 32 ? kRows * kHeadDim : 1024];
  __shared__ __align__(16) float affine[2][2 * kHeadDim];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, G = lane >> 4;
  const int row8 = lane >> 3, j = lane & 7, c0 = j * 8;  // this lane's row of eight, chunk of a head, first channel
  const RopeArgs& r = a.r;
  const int T = (int)r.NQ;

  Channels ch;
  const uint64_t others = *reinterpret_cast<const uint64_t*>(r.other + c0);
  ch.other[0] = (uint32_t)others;
  ch.other[1] = (uint32_t)(others >> 32);
  ch.lane_at = ((lane & 56) + (int)((others >> 3) & 7)) * 4;
  // this thread's pair of every eighth row's (requested here: the arguments lie far away)
  const int p = threadIdx.x % (kHeadDim / 2);
  const int axis = r.axis[p], lo = r.first[p], hi = r.second[p];
  const uint64_t freq = r.freq[p];
  if (threadIdx.x < 2 * kHeadDim) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float* const of = threadIdx.x < kHeadDim ? r.norm[t].gamma : r.norm[t].beta;
      affine[t][threadIdx.x] = of ? of[threadIdx.x % kHeadDim] : threadIdx.x < kHeadDim ? 1.f : 0.f;
    }
  }
  // channel c's cosine and signed sine in a row's table
  f32x2* const table = reinterpret_cast<f32x2*>(turns);
  auto table_at = [](int row, int c) { return turn_chunk(row, (c & 7) >> 1, c >> 3) * 2 + (c & 1); };

  for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
    const uint32_t it = (uint32_t)item;  // fewer than 2^32 (launch_append)
    const int part = (int)(it % (uint32_t)a.parts), unit = (int)(it / (uint32_t)a.parts % (uint32_t)a.units),
              b = (int)(it / (uint32_t)a.parts / (uint32_t)a.units);
    const int64_t start = a.start ? ((ScalarInts)a.start)[b] : 0;
    const int count = a.counts ? min(max(((ScalarInts)a.counts)[b], 0), T) : T;
    const int64_t cap = (int64_t)a.max_pages * kTileRows;
    if (unit == 0 && part == 0 && threadIdx.x == 0 && a.lens) a.lens[b] = (int32_t)min(max(start + count, (int64_t)0), cap);
    // the unit's first row of the cache, and the token that becomes it
    const int64_t row0 = (start >> (kRows == 32 ? 5 : 4)) * kRows + (int64_t)unit * kRows;
    const int64_t tok0 = row0 - start;
    // its rows whose tokens exist: from .. to - 1; all of them are rows of the cache or none: a cache begins and ends with a unit
    const int from = (int)min(max(-tok0, (int64_t)0), (int64_t)kRows);
    const int to = (int)min(max(count - tok0, (int64_t)0), (int64_t)kRows);
    if (from >= to) continue;
    int page = -1;
    if (row0 >= 0 && row0 < cap) page = ((ScalarInts)a.pages)[(int64_t)b * a.max_pages + row0 / kTileRows];
    const int k_heads = a.H_kv, heads = a.H_kv + a.q_heads;
    const bool stored = page >= 0 && page < a.n_pages;

    // heads: those of the keys, then those of the queries
    const int64_t tok_first = (int64_t)b * T + tok0;
    u32x4 raw[kRows / 8], val[kRows / 8];
    auto exists = [&](int i) { return 8 * i + row8 >= from && 8 * i + row8 < to; };
    auto request = [&](int h, int i) {
      const int t = h < k_heads ? 1 : 0;
      const int64_t stride = r.stride[t];
      if (exists(i))
        raw[i] = *reinterpret_cast<const u32x4*>(r.in[t] + (tok_first + 8 * i) * stride + (t ? h : h - k_heads) * kHeadDim +
                                                 (row8 * stride + c0));
    };
    auto request_v = [&](int h, int i) {
      if (h < k_heads && exists(i))
        val[i] = *reinterpret_cast<const u32x4*>(a.V + (tok_first + 8 * i) * a.v_stride + h * kHeadDim + (row8 * a.v_stride + c0));
    };
    // this lane's place behind a uniform one, of keys, of queries and of values
    const uint32_t k_lane = (uint32_t)(j * 32 + row8) * 8, q_lane = (uint32_t)row8 * (uint32_t)a.q_heads * kHeadDim + c0,
                   v_lane = (uint32_t)(kRows == 32 ? G * 64 + c : (G & 1) * 64 + (G >> 1) * 32 + c) * 8;
    const int in_page = (int)(row0 & (kTileRows - 1));
    const int step = a.parts * kAppendWaves;
    int h = part * kAppendWaves + wave;
    if (!stored)  // nothing of the keys is kept
      while (h < k_heads) h += step;
#pragma unroll
    for (int i = 0; i < kRows / 8; ++i) {
      raw[i] = val[i] = u32x4{0u, 0u, 0u, 0u};
      if (h < heads) request(h, i);
      if (h < heads) request_v(h, i);
    }

    lds_barrier();  // the last unit's reads are done; rows stay on their way
    if constexpr (kPairs != kNoPairs) {
      if (p < r.pairs) {
        for (int row = from + threadIdx.x / (kHeadDim / 2); row < to; row += kAppendThreads / (kHeadDim / 2)) {
          const uint32_t tok = (uint32_t)(tok0 + row);
          int32_t pos;
          if (r.pos) {
            pos = r.pos[((int64_t)b * T + tok) * 3 + axis];
          } else {
            const uint32_t frame = tok / (uint32_t)r.L;
            const int32_t patch = (int32_t)(tok % (uint32_t)r.L) - r.P;
            if (axis == 0) pos = r.t0 + (int32_t)frame;
            else if (patch < 0) pos = 0;
            else pos = r.patch0 + (axis == 1 ? patch / r.n_w : patch % r.n_w);
          }
          const uint64_t phase = (uint64_t)(int64_t)pos * freq;
          float sine, cosine;
          sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &sine, &cosine);
          table[table_at(row, lo)] = f32x2{cosine, -sine};
          table[table_at(row, hi)] = f32x2{cosine, sine};
        }
      }
    }
    lds_barrier();

    for (; h < heads; h += step) {
      const bool key = h < k_heads;
      const SeamNorm& norm = r.norm[key ? 1 : 0];
      const int64_t tile = ((int64_t)page * a.H_kv + h) * kTileElems;
#pragma unroll
      for (int i = 0; i < kRows / 8; ++i) {
        if (8 * i >= to || 8 * i + 8 <= from) continue;
        const int row = 8 * i + row8;
        float x[8];
        unpack8(raw[i], x);
        if (h + step < heads) request(h + step, i);
        if (norm.kind != AGG_NORM_NONE) norm8(x, norm.kind, norm.eps, affine[key ? 1 : 0] + c0);
        turn8<kPairs>(x, ch, lane, row, turns, (float*)space[wave]);
        if (exists(i)) {
          uint16_t* const at = key ? a.Kc + tile + (in_page / 32 * 256 + in_page % 32 + 8 * i) * 8 : r.out[0] + ((tok_first + 8 * i) * a.q_heads + (h - k_heads)) * kHeadDim;
          *reinterpret_cast<u32x4*>(at + (key ? k_lane : q_lane)) = pack8(x);
        }
      }
      if (!key) continue;
      // values, row-major with the upper half of a row's chunks exchanged with the lower on rows 2 and 3 mod 4 (the
      // transposing read's four rows then lie on different banks)
      lds_char* const v = (lds_char*)space[wave];
      wave_lds_fence();
#pragma unroll
      for (int i = 0; i < kRows / 8; ++i) {
        const int row = 8 * i + row8;
        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(v + row * 128 + (j ^ (4 * ((row >> 1) & 1))) * 16) = val[i];
        if (h + step < heads) request_v(h + step, i);
      }
      wave_lds_fence();
      // 32 rows: the lanes' groups of sixteen take the chunks of 16 rows and of four in them; 16 rows: halves of the channels
      const int k0 = (kRows == 32 ? 16 * (G >> 1) : 0) + 4 * (G & 1);  // first row of this lane's chunks: k0 .. + 3, k0 + 8 .. + 11
      const int row = k0 + (c >> 2);                                  // its row of the four that the read transposes
#pragma unroll
      for (int d = 0; d < kRows / 8; ++d) {
        const int dt = kRows == 32 ? d : 2 * (G >> 1) + d;
        lds_char* const at = v + row * 128 + ((2 * dt + ((c & 3) >> 1)) ^ (4 * ((row >> 1) & 1))) * 16 + (c & 1) * 8;
        const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
        const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * 128));
        uint16_t* const to_page = a.Vc + tile + in_page * kHeadDim + d * 128 + v_lane;
        if (k0 >= from && k0 + 11 < to) {
          const u32x2 l2 = __builtin_bit_cast(u32x2, x0), h2 = __builtin_bit_cast(u32x2, x1);
          *reinterpret_cast<u32x4*>(to_page) = u32x4{l2[0], l2[1], h2[0], h2[1]};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (k0 + e >= from && k0 + e < to) to_page[e] = (uint16_t)x0[e];
            if (k0 + 8 + e >= from && k0 + 8 + e < to) to_page[4 + e] = (uint16_t)x1[e];
          }
        }
      }
      wave_lds_fence();  // the reads are done before the next rows come
    }
  }
}

// Where the pairs of a rotation lie, seen from a lane of eight channels.
static int pairs_kind(const RopeArgs& r) {
  if (!r.pairs) return kNoPairs;
  bool in_lane = true, across = true;
  for (int c = 0; c < kHeadDim; ++c) {
    if (!(r.other[c] & 0x80)) continue;
    const int other = r.other[c] & 63;
    in_lane = in_lane && other == (c ^ 1);
    // all eight channels of a lane turn, with those of one lane in the same order
    across = across && other % 8 == c % 8 && (r.other[c & ~7] & 0x80) && (r.other[c & ~7] & 63) / 8 == other / 8;
  }
  return in_lane ? kPairsInLane : across ? kPairsAcrossLanes : kPairsAnywhere;
}

template <int kRows>
static void launch_rows(const AppendArgs& a, hipStream_t st) {
  constexpr int64_t kMost = 1 << 20;
  const dim3 grid((unsigned)(a.items < kMost ? a.items : kMost)), block(kAppendThreads);
  switch (pairs_kind(a.r)) {
    case kNoPairs: hipLaunchKernelGGL((append_kernel<kNoPairs, kRows>), grid, block, 0, st, a); break;
    case kPairsInLane: hipLaunchKernelGGL((append_kernel<kPairsInLane, kRows>), grid, block, 0, st, a); break;
    case kPairsAcrossLanes: hipLaunchKernelGGL((append_kernel<kPairsAcrossLanes, kRows>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((append_kernel<kPairsAnywhere, kRows>), grid, block, 0, st, a);
  }
}

hipError_t launch_append(const AppendArgs& args, hipStream_t st) {
  AppendArgs a = args;
  const int64_t T = a.r.NQ;
  a.q_heads = a.r.in[0] ? a.r.H : 0;
  const int most = (int)(((int64_t)a.H_kv + a.q_heads + kAppendWaves - 1) / kAppendWaves);
  // a sequence's tokens lie in one more piece than they fill where they begin inside one
  auto units = [&](int rows) { return (T + rows - 1) / rows + 1; };
  // Pieces of 16 rows while all of a call's wavefronts' turns at a head are no more than nine rounds (us, pieces of 32 / 16: clips of
  // three ragged streams 20.3 / 17.0, 4 frames 19.2 / 16.7, 8 29.1 / 28.3, 16 55.8 / 57.9), and heads shared out while all workgroups
  // still run at once.
  constexpr int64_t kAtOnce = 256 * 4;
  const bool few = a.B * units(16) * most <= 9 * kAtOnce;
  a.units = (int32_t)units(few ? 16 : 32);
  a.parts = 1;
  while (a.parts < most && (int64_t)a.B * a.units * (a.parts + 1) <= kAtOnce) ++a.parts;
  a.items = (int64_t)a.B * a.units * a.parts;
  if (a.items > 0xFFFFFFFFll) return kTooManyGroups;
  (void)hipGetLastError();
  if (few) launch_rows<16>(a, st);
  else launch_rows<32>(a, st);
  return hipGetLastError();
}

}  // namespace agg
