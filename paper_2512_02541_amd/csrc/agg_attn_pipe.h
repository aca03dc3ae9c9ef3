// The key loop that the attention kernels share: what a wavefront keeps in registers, where key/value tiles come from, their
// asynchronous copies into LDS, and the software pipeline over them.  agg_attn.hip describes it.
#pragma once

#include "agg_attn_plan.h"
#include "agg_internal.h"
#include "agg_lds_copy.h"

namespace agg {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kAttnThreads = 64 * kWaves;
constexpr int kBlocksPerCu = 2;         // two wavefronts per SIMD
constexpr int kXcds = 8;
constexpr int kLdsTiles = 3;
constexpr int kEpiStride = kHeadDim + 8;  // bf16 per query row of the epilogue's LDS tile (padded)
constexpr int kChunks = kTileElems / 8;  // 16-byte chunks per K or V tile (512)
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSumHi = 1.2379400392853803e27f;   // 2^90
constexpr float kSumLo = 8.077935669463161e-28f;   // 2^-90
constexpr float kLazy = 60.0f;  // general path: a unit may exceed the row's reference by 2^60
constexpr float kUnitHi = 1.2676506002282294e30f;  // 2^100: a unit's row sum that forces a look
// exact_logits: a look at 2^10, so that sums with values of up to 2^100 stay in float32's range, and references 20 above (base 2) the
// largest logit so far, so that it is not taken for every rise.  (Redone calls, us, logits of +-20 / 40 / 100, 512 queries to each of 24
// frames: 191 / 195 / 199 without the 20, 177 / 183 / 192 with it; 168 / 166 / 175 with a look at 2^100, which overflows with values of 2^50.)
constexpr float kUnitHiExact = 1024.0f;
constexpr float kAboveExact = 20.0f;

union Frag {
  u32x4 u;
  bf16x8 h;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  f32x2 p = {lo, hi};
  bf16x2 h = __builtin_convertvector(p, bf16x2);  // round to nearest even
  return __builtin_bit_cast(uint32_t, h);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Exchange between lanes l and l ^ 32.  v_permlane32_swap exchanges the upper 32 lanes of its
// first operand with the lower 32 of its second; fed the same value twice it returns
// (own, partner) in one order or the other, and both uses below are symmetric.
__device__ __forceinline__ float pair_max(float x) {
  const uint32_t b = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const uint32_t b = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

#define AGG_MFMA16(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_bf16((a).h, (b).h, (c), 0, 0, 0)

// Lane geometry of v_mfma_f32_16x16x32_bf16: c = lane & 15 is the row of the A operand, the
// column of the B operand and of the result; G = lane >> 4 selects eight of the 32 contraction
// elements (8 G .. 8 G + 7) in A and B, and result rows 4 G .. 4 G + 3.
//
// A 32-key block is scored as two 16-key tiles.  Tile kt takes the block's keys
//     row i  ->  key (i & 7) + 16 (i >> 3) + 8 kt          (tile 0: 0-7, 16-23; tile 1: 8-15, 24-31)
// so that the eight probabilities a lane holds after both tiles (rows 4 G .. 4 G + 3 of each) are
// exactly the eight keys of ONE 16-byte chunk of the compacted V tile (agg.h: chunk (t, g) holds
// keys 16 t + 4 g + {0..3, 8..11}; here t = 2 kb + (G >> 1), g = G & 1): the exponentiated scores
// are the B operand of O^T += V^T P^T as they stand, and V fragments are plain 16-byte reads.
__device__ __forceinline__ int row_key(int i) { return (i & 7) + 16 * (i >> 3); }

// sum / maximum over the four lanes c, c + 16, c + 32, c + 48 that share a query
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor(x, 16);
  return pair_sum(x);
}
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return pair_max(x);
}

// LDS words through which wavefronts tell each other of rows that the fast path cannot handle: four
// for the check inside the key loop, four for the one behind it.
constexpr int kVoteWords = 2 * kWaves;

// Whether x holds in any lane of the workgroup's first kWaves wavefronts (`mine`: this is one of them).
// Passes one barrier.  (The library's workgroup-wide "or" passes three and reduces through LDS: a layer
// of two frames of 16x16 14.55 us with it and 14.3 without, its block 43.5 / 43.1, index-driven, 40
// frames, 2700 / 2684; longer calls alike.)
__device__ __forceinline__ bool vote(bool x, uint32_t* words, int wave, int lane, bool mine) {
  const bool any = __builtin_amdgcn_ballot_w64(x) != 0;
  if (mine && lane == 0) words[wave] = any ? 1u : 0u;
  __syncthreads();
  const u32x4 all = *reinterpret_cast<const u32x4*>(words);
  return __builtin_amdgcn_readfirstlane(all[0] | all[1] | all[2] | all[3]) != 0;
}

// zero-padded rows of the last tile: key index inside the tile >= valid -> -inf
template <int kJ>
__device__ __forceinline__ void mask_unit(f32x4 (&S)[2 * kJ], int kb, int valid, int G) {
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int km = 32 * kb + 8 * kt + row_key(4 * G + r);
      if (km >= valid) {
#pragma unroll
        for (int j = 0; j < kJ; ++j) S[kJ * kt + j][r] = -INFINITY;
      }
    }
}

// Everything a wavefront keeps in registers across the key loop.  qb = query block, j = its
// 16-query tile, kt = 16-key tile of a key block, h = half of the channel range, dt = 16-channel
// tile of the output.
template <int kQB, int kJ>
struct Wave {
  Frag Qf[kQB][2 * kJ];    // [qb][2 j + h]: B operand of S^T = K Q^T, pre-multiplied by scale*log2(e) (exact_logits: as it is)
  f32x4 O[kQB][kJ][4];     // [qb][j][dt]: O^T accumulator; channel = 16 dt + 4 G + r, query = c
  f32x4 S[kQB][2 * kJ];    // [qb][kJ kt + j]: score tiles in flight; key = row_key(4 G + r) + 8 kt
  f32x4 L[kQB][kJ];        // [qb][j]: fast path: element 0 of the lanes G = 0 is the row sum, kept by the matrix core
  float la[kQB][kJ];       // [qb][j]: general path: this lane's part of the row sum
  float mref[kQB][kJ];     // general path: the row's reference (base-2 logit; exact_logits: plain product, -infinity where there is none yet)
  Frag a[4];               // [2 kt + h]: K fragments of the block whose scores are being computed
  Frag v[4];               // [dt]: V fragments of the block whose P V is being accumulated
  Frag P[kJ];              // [j]: probabilities of the previous unit
  float l2;                // exact_logits: scale*log2(e)
  Frag ones;               // A operand of the row sums: row 0 ones, the others zeros
};

// Probabilities of the 8 kJ base-2 logits a lane holds for a unit, packed as the B operands of
// the PV MFMAs: for query tile j, contraction elements 8 G .. 8 G + 7 are key tile 0's rows, then
// key tile 1's.  The query tiles alternate in the instruction stream.
// kScaled: the scores are plain products and take the factor l2 = scale*log2(e) here (exact_logits).
template <int kJ, bool kScaled = false>
__device__ __forceinline__ void exp_unit(const f32x4 (&S)[2 * kJ], Frag (&P)[kJ], float l2 = 1.f) {
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j)
        {
          const float s0 = S[kJ * kt + j][2 * i], s1 = S[kJ * kt + j][2 * i + 1];
          P[j].u[2 * kt + i] = pack_bf16(fast_exp2(kScaled ? s0 * l2 : s0), fast_exp2(kScaled ? s1 * l2 : s1));
        }
}

// General path: the same, and the sums of each query tile's part (there the vector ALU keeps
// the sums: the unit's own sum is what tells that a score has run away from the row's reference,
// and it is needed before the probabilities reach the matrix core)
template <int kJ>
__device__ __forceinline__ void exp_unit_sum(const f32x4 (&S)[2 * kJ], Frag (&P)[kJ], float (&l)[kJ]) {
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        const float e0 = fast_exp2(S[kJ * kt + j][2 * i]);
        const float e1 = fast_exp2(S[kJ * kt + j][2 * i + 1]);
        P[j].u[2 * kt + i] = pack_bf16(e0, e1);
        l[j] += e0;
        l[j] += e1;
      }
}

// General path of exact_logits: the scores and each row's reference are plain products, whose difference becomes a base-2 logit.  A
// reference far above or far below the scores costs them no digits, and one of their own is never below them: of references that are
// rounded products with l2, 10^10 is 512 off, and a multiply-add with it makes 2^512 of the row's largest probability.
template <int kJ>
__device__ __forceinline__ void exp_unit_relative(const f32x4 (&S)[2 * kJ], Frag (&P)[kJ], float (&l)[kJ], float l2, const float (&ref)[kJ]) {
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        const float e0 = fast_exp2((S[kJ * kt + j][2 * i] - ref[j]) * l2);
        const float e1 = fast_exp2((S[kJ * kt + j][2 * i + 1] - ref[j]) * l2);
        P[j].u[2 * kt + i] = pack_bf16(e0, e1);
        l[j] += e0;
        l[j] += e1;
      }
}

// Where the key/value tiles come from.
//   kSrcCompact: the fragment-order compacted tensors of agg_kv_subsample: a tile is a linear
//                8 KiB copy and already in MFMA operand order.
//   kSrcRows:    consecutive rows of the token-major K and V themselves (ordinary and per-frame
//                attention: every token is a key), no compacted copy.
//   kSrcIndexed: rows of K and V picked through a list of token ids (Sec. 4.3 restricts keys
//                and values to a subset of the tokens; here the subset is read in place).
// In the two row modes a tile lies in LDS row-major, 128 bytes per key, with the 16-byte chunk
// number XOR-ed by a function of the row so that the fragment reads spread over all 64 banks:
// K fragments (eight channels of one key per lane) are plain 16-byte reads; V fragments (eight
// keys of one channel per lane) come from the transposing read ds_read_b64_tr_b16, which hands
// lane i of a 16-lane group the i-th 16-bit column of the four 8-byte rows the group's lanes
// 4j .. 4j+3 point at.
//   kSrcStrided: consecutive rows of K and V, each with a distance of its own, whose number is a device's value (attention
//                to keys of another length).
//   kSrcPaged:   fragment-order tiles again, each found through a page table.
// The last two may end anywhere in memory that holds something else: their values are masked behind the last key, since 0
// times what lies there may be no number.
enum { kSrcCompact = 0, kSrcRows = 1, kSrcIndexed = 2, kSrcStrided = 3, kSrcPaged = 4 };
// Whose scores are products of the query as it is, multiplied by scale*log2(e) in float32 in front of the exponential, rather than
// of the query times that rounded to bf16.  The vector ALU, as loaded as the matrix core without it, has one instruction more
// per score, 7 to 15 % of a call by box (8 frames over 40 1874 -> 2043 us, 24 frames x 512 queries 62.5 -> 66.9, a frame over 13740 keys
// 81 -> 88 on one); the result's error against 64 bits is 0.0023 of it instead of 0.0034, 0.0017 of which are its own rounding.
constexpr bool exact_logits(int src) { return src == kSrcStrided || src == kSrcPaged; }
constexpr bool fragment_order(int src) { return src == kSrcCompact || src == kSrcPaged; }

typedef short s16x4 __attribute__((ext_vector_type(4)));

// chunk swizzle of a K row in the row modes: the 16 rows a lane group reads (i, i + 16 for eight
// consecutive i) must fall on 16 different 16-byte slots of the 256-byte bank period
__device__ __forceinline__ uint32_t k_swizzle(uint32_t row) {
  return ((row >> 1) & 3u) | (((row >> 4) & 1u) << 2);
}

// per-lane LDS byte offsets of the fragment reads (row modes) or chunk numbers (compact mode)
struct FragAddr {
  int lane;
  int kc[2];             // compact: chunk of tile kt inside a (key block, channel half) run
  int vc;                // compact: chunk inside a key block's V run (plus 16 dt)
  uint32_t k[4];         // rows: K fragment [2 kt + h]
  uint32_t v[4];         // rows: V fragment of channel tile dt (first four keys; +8 rows: the others)
};

__device__ __forceinline__ FragAddr frag_addr(int lane) {
  FragAddr f;
  const int c = lane & 15, G = lane >> 4;
  f.lane = lane;
  // compact K tile in LDS: [kb][h][G][32 keys], a key at position (key with bits 3 and 4
  // exchanged): tile kt's sixteen keys are then consecutive
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) f.kc[kt] = G * 32 + 16 * kt + c;
  f.vc = G * 64 + c;
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t row = (uint32_t)(row_key(c) + 8 * kt);
      f.k[2 * kt + h] = row * 128u + (((uint32_t)(4 * h + G) ^ k_swizzle(row)) * 16u);
    }
  // V: the lanes 4 i' .. 4 i' + 3 of a 16-lane group point at row i' of the group's first four
  // keys (16 (G >> 1) + 4 (G & 1) + i'), each at 8 of the 32 bytes of channels 16 dt .. 16 dt + 15;
  // chunk bit 2 is flipped on rows 2, 3 mod 4
  const int row = 16 * (G >> 1) + 4 * (G & 1) + (c >> 2);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) {
    const int chunk = (2 * dt + ((c & 3) >> 1)) ^ (4 * ((row >> 1) & 1));
    f.v[dt] = (uint32_t)(row * 128 + chunk * 16 + (c & 1) * 8);
  }
  return f;
}

template <int kSrc>
__device__ __forceinline__ void load_k_frags(const u32x4* __restrict__ lds, int buf, int kb,
                                             const FragAddr& f, Frag (&a)[4]) {
  if (fragment_order(kSrc)) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        a[2 * kt + h].u = lds[buf * kChunks + kb * 256 + h * 128 + f.kc[kt]];
  } else {
    const lds_char* base = (const lds_char*)lds + buf * (kChunks * 16) + kb * (32 * 128);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      a[i].u = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(base + f.k[i]);
  }
}
template <int kSrc>
__device__ __forceinline__ void load_v_frags(const u32x4* __restrict__ lds, int buf, int kb,
                                             const FragAddr& f, Frag (&v)[4]) {
  if (fragment_order(kSrc)) {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
      v[dt].u = lds[(kLdsTiles + buf) * kChunks + kb * 256 + dt * 16 + f.vc];
  } else {
    lds_char* base = (lds_char*)lds + (kLdsTiles + buf) * (kChunks * 16) + kb * (32 * 128);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      // the group's first four keys, then the four that lie eight rows further on: the order
      // the P operand has
      lds_char* at = base + f.v[dt];
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)(at + 8 * 128));
      const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
      v[dt].u = u32x4{l2[0], l2[1], h2[0], h2[1]};
    }
  }
}

// Values of keys behind the last one, of 32 whose first `left` exist, become zero.
__device__ __forceinline__ void mask_values(Frag (&v)[4], int left, int G) {
  const int k0 = 16 * (G >> 1) + 4 * (G & 1);  // a lane's eight keys: k0 .. + 3, k0 + 8 .. + 11
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = k0 + (i >> 1) * 8 + (i & 1) * 2;
    const uint32_t mask = (key < left ? 0xFFFFu : 0u) | (key + 1 < left ? 0xFFFF0000u : 0u);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) v[dt].u[i] &= mask;
  }
}

// What a workgroup needs to know about its key/value source.
struct KvSource {
  const uint16_t *k, *v;   // compact: tile 0 of this (batch, head); rows: token 0's row of this head
  const int32_t* list;     // indexed: the batch element's token ids
  int64_t rows;            // number of keys (M, or the sequence length)
  uint32_t row_bytes;      // rows: distance between consecutive tokens' rows (H * 128)
  uint32_t max_token;      // indexed: largest valid token id (N*L - 1)
  uint32_t v_row_bytes;    // strided: row_bytes of V
  ScalarInts pages;        // paged: the page numbers of this workgroup's tiles; k, v: head 0's tile of page 0
  int32_t tiles, last_page;  // paged: how many, the largest page number
  int64_t page_elems, head_elems;  // paged: from a page to the next, from head 0 to this one
};

// Issues the asynchronous copy of tile t into LDS buffer `buf`.  Every wavefront lands 64
// consecutive 16-byte LDS slots per instruction; which global chunk a lane fetches for its slot
// is what differs between the modes.
template <int kSrc>
struct TileCopier {
  KvSource src;
  const uint16_t *knext, *vnext;  // compact, rows: where the next tile to be copied starts
  int64_t tnext;                  // its number (tiles are copied in order)
  uint32_t wbase;          // LDS byte address of this wavefront's first slot in buffer 0
  // byte offset of this lane's first chunk from the tile's (rows, compact) or the row's (indexed)
  // start, for K and for V; the second lies half a tile (32 rows, whose swizzle is that of the first 32)
  // further on
  uint32_t vk, vv;
  uint32_t row;            // row of the tile this lane's first slot belongs to (rows)
  // Indexed: an instruction's eight rows and a tile's two instructions make 16 ids per wavefront.
  // Lane l holds the id of row l % 16 of them; byte offsets are worked out once per row and handed
  // to the eight lanes that fetch it, a tile ahead of their use.  (Every lane reading and scaling
  // its own two ids cost 17 vector instructions a tile instead of 8, in a loop that the vector ALU
  // bounds: 40 frames 2768 us against 2658, 100 frames 32.4 ms against 31.7, 8 frames 158 against 143.)
  uint32_t lane;           // of the wavefront
  uint32_t list_at;        // byte offset of this lane's id for the tile after the next
  uint32_t id;             // its id for the tile after the next to be copied
  uint32_t from[2];        // next tile to be copied: byte offset of the rows this lane fetches
  int32_t page;            // paged: page of the next tile to be copied

  __device__ __forceinline__ void init(const KvSource& s, const u32x4* lds, int tid, int wave) {
    src = s;
    knext = s.k;
    vnext = s.v;
    tnext = 0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_char*)lds);
    wbase = __builtin_amdgcn_readfirstlane(lds0 + (uint32_t)wave * 1024u);
    const uint32_t slot = (uint32_t)tid;  // 0 .. 255, and 256 more
    row = slot >> 3;
    const uint32_t c = slot & 7;
    const uint32_t ck = (c ^ k_swizzle(row)) * 16u;
    const uint32_t cv = (c ^ (4u * ((row >> 1) & 1))) * 16u;
    if (fragment_order(kSrc)) {
      // K: the LDS slot of a key has bits 3 and 4 of the key number exchanged (frag_addr)
      const uint32_t key = slot & 31u;
      const uint32_t swapped = (key & 7u) | ((key & 8u) << 1) | ((key & 16u) >> 1);
      vk = ((slot & ~31u) | swapped) * 16u;
      vv = slot * 16u;
    } else if (kSrc == kSrcRows) {
      vk = row * s.row_bytes + ck;
      vv = row * s.row_bytes + cv;
    } else if (kSrc == kSrcStrided) {
      vk = row * s.row_bytes + ck;
      vv = row * s.v_row_bytes + cv;
    } else {
      vk = ck;
      vv = cv;
    }
    if (kSrc == kSrcIndexed) {
      lane = tid & 63;
      const uint32_t l = lane & 15;
      list_at = ((l & 8) * 4u + wave * 8u + (l & 7)) * 4u;
      fetch_ids();
      spread_ids();
      fetch_ids();
    }
    if (kSrc == kSrcPaged) page = s.pages[0];
  }
  __device__ __forceinline__ void fetch_ids() {  // rows past the end repeat the last one; masked later
    const uint32_t at = min(list_at, ((uint32_t)src.rows - 1u) * 4u);
    id = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(src.list) + at);
    list_at += kTileRows * 4u;
  }
  __device__ __forceinline__ void spread_ids() {
    // an id outside the sequence cannot leave it
    const int base = (int)__umul24(min(id, src.max_token), src.row_bytes);
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
      from[hh] = (uint32_t)__builtin_amdgcn_ds_bpermute((int)((lane >> 3) + 8 * hh) * 4, base);
  }
  // copies tile tnext into LDS buffer `buf`
  __device__ __forceinline__ void issue(int buf) {
    const uint32_t mk = wbase + (uint32_t)buf * (kChunks * 16);
    const uint32_t mv = wbase + (uint32_t)(kLdsTiles + buf) * (kChunks * 16);
    static_assert(2 * kAttnThreads == kChunks, "two copies per thread and tile");
    if (kSrc == kSrcCompact) {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        dma16(knext + hh * (kTileElems / 2), vk, mk + hh * kAttnThreads * 16);
        dma16(vnext + hh * (kTileElems / 2), vv, mv + hh * kAttnThreads * 16);
      }
      knext += kTileElems;
      vnext += kTileElems;
    } else if (kSrc == kSrcRows) {
      // the tile's rows follow each other in memory
      const size_t half = (size_t)(kTileRows / 2) * (src.row_bytes / 2);
      if ((tnext + 1) * kTileRows <= src.rows) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          dma16(knext + hh * half, vk, mk + hh * kAttnThreads * 16);
          dma16(vnext + hh * half, vv, mv + hh * kAttnThreads * 16);
        }
      } else {  // last, partial tile: rows past the end repeat the last one; masked later
        const uint32_t last = (uint32_t)(src.rows - 1 - tnext * kTileRows);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const uint32_t r = row + hh * (kTileRows / 2);
          const uint32_t at = (min(r, last) - row) * src.row_bytes;  // (wraps where the row is before this lane's)
          dma16(knext, vk + at, mk + hh * kAttnThreads * 16);
          dma16(vnext, vv + at, mv + hh * kAttnThreads * 16);
        }
      }
      knext += 2 * half;
      vnext += 2 * half;
    } else if (kSrc == kSrcStrided) {
      const size_t k_half = (size_t)(kTileRows / 2) * (src.row_bytes / 2), v_half = (size_t)(kTileRows / 2) * (src.v_row_bytes / 2);
      if ((tnext + 1) * kTileRows <= src.rows) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          dma16(knext + hh * k_half, vk, mk + hh * kAttnThreads * 16);
          dma16(vnext + hh * v_half, vv, mv + hh * kAttnThreads * 16);
        }
      } else {  // last, partial tile: rows past the end repeat the last one; masked later
        const uint32_t last = (uint32_t)(src.rows - 1 - tnext * kTileRows);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const uint32_t r = row + hh * (kTileRows / 2);
          const uint32_t beyond = min(r, last) - row;  // (wraps where the row is before this lane's)
          dma16(knext, vk + beyond * src.row_bytes, mk + hh * kAttnThreads * 16);
          dma16(vnext, vv + beyond * src.v_row_bytes, mv + hh * kAttnThreads * 16);
        }
      }
      knext += 2 * k_half;
      vnext += 2 * v_half;
    } else if (kSrc == kSrcPaged) {
      // the page's number came a tile ahead; one outside the pool is read as the first or the last page
      const int64_t at = min(max(page, 0), src.last_page) * src.page_elems + src.head_elems;
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        dma16(src.k + at + hh * (kTileElems / 2), vk, mk + hh * kAttnThreads * 16);
        dma16(src.v + at + hh * (kTileElems / 2), vv, mv + hh * kAttnThreads * 16);
      }
      page = src.pages[min((int32_t)tnext + 1, src.tiles - 1)];
    } else {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        dma16(src.k, from[hh] + vk, mk + hh * kAttnThreads * 16);
        dma16(src.v, from[hh] + vv, mv + hh * kAttnThreads * 16);
      }
      spread_ids();  // the next tile's offsets; its ids came with the last wait
      fetch_ids();                   // and the ids after those
    }
    ++tnext;
  }
};

// Query tile of product i: 0 .. kJ-1, then back, so that consecutive products always have an operand
// in common.  Measured pass by pass against plain order on two boxes: layers of 100 and 800 frames take 0.1 to
// 0.3 % less (29.05 ms instead of 29.13), calls under 6 ms the same.  With the row of ones (pv_unit) it is 0.8 to
// 1.0 %; of 0.9 % under the counters 0.5 +- 0.2 were cycles and 0.4 +- 0.2 the clock, so less power is a part of it
// at most.
template <int kJ>
constexpr int there_and_back(int i) {
  return (i / kJ) % 2 ? kJ - 1 - i % kJ : i % kJ;
}

// Scores of one unit: the 32 keys of block fragments `a` against the 16 kJ queries of block tq.
// General path: the accumulator starts at minus the row's reference instead of zero, so the
// scores come out relative to it at no cost (the reference is a float, nothing is split).
// (Not with exact_logits, whose callers leave it out by kGen = false: it would round the scores to the reference's digits.)
template <bool kGen, int kQB, int kJ>
__device__ __forceinline__ void score_unit(const Wave<kQB, kJ>& w, int tq, f32x4 (&Sn)[2 * kJ]) {
  f32x4 init[kJ];
#pragma unroll
  for (int j = 0; j < kJ; ++j) {
    const float m = kGen ? -w.mref[tq][j] : 0.f;
    init[j] = f32x4{m, m, m, m};
  }
#pragma unroll
  for (int i = 0; i < 2 * kJ; ++i) {
    const int kt = i / kJ, j = there_and_back<kJ>(i);
    Sn[kJ * kt + j] = AGG_MFMA16(w.a[2 * kt], w.Qf[tq][2 * j], init[j]);
  }
#pragma unroll
  for (int i = 0; i < 2 * kJ; ++i) {
    const int kt = i / kJ, j = there_and_back<kJ>(i);
    Sn[kJ * kt + j] = AGG_MFMA16(w.a[2 * kt + 1], w.Qf[tq][2 * j + 1], Sn[kJ * kt + j]);
  }
}
// O^T += V^T P^T for the unit whose probabilities are in w.P.  Fast path: the row sums are one
// more product, a row of ones and fifteen of zeros against P^T: row 0 of that 16 x 16 result, in
// the lanes G = 0, is the sum of the unit's 32 probabilities of a query, and the vector ALU adds
// nothing.  (Sixteen rows of ones leave the sum in every lane but take 0.7 % longer: the layer of 100
// frames 29.25 ms instead of 29.05, ordinary attention, 24 frames, 1448 us instead of 1440; 0.3 to 0.7 % elsewhere.)
template <bool kGen, int kQB, int kJ>
__device__ __forceinline__ void pv_unit(Wave<kQB, kJ>& w, int pq) {
#pragma unroll
  for (int i = 0; i < 4 * kJ; ++i) {
    const int dt = i / kJ, j = there_and_back<kJ>(i);
    w.O[pq][j][dt] = AGG_MFMA16(w.v[dt], w.P[j], w.O[pq][j][dt]);
  }
  if (!kGen) {
#pragma unroll
    for (int j = 0; j < kJ; ++j) w.L[pq][j] = AGG_MFMA16(w.ones, w.P[j], w.L[pq][j]);
  }
}

// One step of the pipeline inside tile `cur` (see the file header).  kLast: the tile is the
// last one (`valid` of its 64 rows exist, nothing follows).  kGen: general path.
template <int kSrc, bool kLast, bool kGen, int kQB, int kJ>
__device__ __forceinline__ void tile_steps(Wave<kQB, kJ>& w, const u32x4* __restrict__ lds, int cur, int nxt,
                                           int valid, const FragAddr& fa, int G) {
#pragma unroll
  for (int sg = 0; sg < 2 * kQB; ++sg) {
    // A last tile of up to 32 keys: its second block is padding throughout.  (Left out from here on; a
    // separate body for such tiles spilled 80 registers.  Per-frame attention over 1374 keys, 90 frames, 663 /
    // 651 us; layer of 2 frames of 16x16 14.3 / 14.0; 9.5 ms calls alike.)
    if (kLast && sg == kQB && valid <= kTileRows / 2) break;
    const int kb = sg / kQB, qb = sg % kQB;
    const int un = sg + kQB - 1;              // unit whose scores start now
    const int tq = un % kQB;                  // its query block
    const bool beyond = un >= 2 * kQB;        // it belongs to the next tile
    const int pq = (qb + kQB - 1) % kQB;      // query block of the previous unit

    // ---- matrix core, part 1: scores of unit `un` ----
    const bool do_qk = !(kLast && beyond);
    f32x4 Sn[2 * kJ];
    if (do_qk) score_unit<kGen && !exact_logits(kSrc), kQB, kJ>(w, tq, Sn);
    if (tq == kQB - 1) {  // that was the block's last unit: fragments of the following block
      if (un / kQB == 0) load_k_frags<kSrc>(lds, cur, 1, fa, w.a);
      else if (!kLast) load_k_frags<kSrc>(lds, nxt, 0, fa, w.a);
    }

    // ---- vector ALU: probabilities of unit sg ----
    Frag Pn[kJ];
    float unit_sum[kJ];  // general path: the unit's own row sums
#pragma unroll
    for (int j = 0; j < kJ; ++j) unit_sum[j] = 0.f;
    {
      f32x4 (&S)[2 * kJ] = w.S[qb];
      if (kLast && valid < kTileRows) mask_unit<kJ>(S, kb, valid, G);
      if (!kGen) {
        exp_unit<kJ, exact_logits(kSrc)>(S, Pn, w.l2);
      } else if (exact_logits(kSrc)) {
        exp_unit_relative<kJ>(S, Pn, unit_sum, w.l2, w.mref[qb]);
      } else {
        // the scores are already relative to the row's reference; whether it still holds is
        // looked at below, behind the step's last MFMA
        exp_unit_sum<kJ>(S, Pn, unit_sum);
      }
    }
    if (do_qk) {
#pragma unroll
      for (int i = 0; i < 2 * kJ; ++i) w.S[tq][i] = Sn[i];
    }

    // ---- matrix core, part 2: P V of unit sg - 1 ----
    pv_unit<kGen, kQB, kJ>(w, pq);
    if (qb == 0) {  // the previous block is done with them
      load_v_frags<kSrc>(lds, cur, kb, fa, w.v);
      if (kSrc >= kSrcStrided && kLast && valid < kTileRows) mask_values(w.v, valid - 32 * kb, G);
    }
#pragma unroll
    for (int j = 0; j < kJ; ++j) w.P[j] = Pn[j];
    // Issue order inside the step: MFMAs and exponentials alternate one by one, a conversion
    // after every second pair (general path: pairs of MFMAs, then their share of the vector work,
    // which there includes the additions).  Left to itself the scheduler bunches the MFMAs, and
    // the wavefront then stalls on the matrix pipe with vector work still to issue.
    if (!kGen) {
      __builtin_amdgcn_sched_group_barrier(0x008, kJ, 0);  // the row-sum products of the last unit
#pragma unroll
      for (int i = 0; i < 4 * kJ; ++i) {
        // (orders with the multiplications one by one, behind the MFMAs or all at the end: 0 to 3 % slower)
        if (exact_logits(kSrc)) __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);  // transcendental
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
        __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 1, 0);  // the pair's conversion
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4 * kJ; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);  // conversion and two additions
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (kGen) {
      // The unit's sums tell whether the reference still holds: a score more than 2^100 (exact_logits: 2^10) above it
      // cannot hide in them.  Rare, wavefront-uniform: raise the reference of the rows that need
      // it (the others keep theirs: shift 0, factor 1), scale what they have accumulated, and
      // redo the unit's probabilities (its scores are untouched until the next step).
      float all = unit_sum[0];
#pragma unroll
      for (int j = 1; j < kJ; ++j) all += unit_sum[j];
      if (__builtin_amdgcn_ballot_w64(!(all < (exact_logits(kSrc) ? kUnitHiExact : kUnitHi))) != 0) {
        f32x4 (&S)[2 * kJ] = w.S[qb];
        float ref[kJ];  // exact_logits: what the unit is taken relative to
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          float mx = S[j][0];
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, S[kJ * kt + j][r]);
          mx = quad_max(mx);  // the four lanes of a row agree
          const float old = w.mref[qb][j];
          float f;
          if (exact_logits(kSrc)) {
            // A row without a reference gets here by itself: relative to -infinity its sum is infinite or no number.  It has none
            // as long as all its logits are -infinity, whose probabilities are 0 relative to anything.
            w.mref[qb][j] = fmaxf(old, mx + fminf(kAboveExact * __builtin_amdgcn_rcpf(w.l2), 1e30f));
            ref[j] = w.mref[qb][j] == -INFINITY ? 0.f : w.mref[qb][j];
            f = fast_exp2((old - ref[j]) * w.l2);
          } else {
            if (mx > kLazy) w.mref[qb][j] = old + mx;
            const float d = w.mref[qb][j] - old;
            f = fast_exp2(-d);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
              for (int r = 0; r < 4; ++r) S[kJ * kt + j][r] -= d;
          }
#pragma unroll
          for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) w.O[qb][j][dt][r] *= f;
          w.la[qb][j] *= f;
        }
#pragma unroll
        for (int j = 0; j < kJ; ++j) unit_sum[j] = 0.f;
        if (exact_logits(kSrc)) exp_unit_relative<kJ>(S, w.P, unit_sum, w.l2, ref);
        else exp_unit_sum<kJ>(S, w.P, unit_sum);
      }
#pragma unroll
      for (int j = 0; j < kJ; ++j) w.la[qb][j] += unit_sum[j];
    }
  }
}

// The key loop of one path.  `first_tile` runs once tile 0 is resident and its first K fragments
// are loaded (the general path takes its reference there).  Returns false when the fast path
// found a row sum it cannot trust.
// kSplit: the workgroup's other wavefronts walk other tiles, perhaps one fewer: no early check, whose
// barriers would not match (the sums are looked at when the loops are done).
template <int kSrc, bool kGen, bool kSplit, int kQB, int kJ, class FirstTile>
__device__ __forceinline__ bool key_loop(Wave<kQB, kJ>& w, u32x4* __restrict__ lds, uint32_t* votes,
                                         const KvSource& src, int ntiles, int last_valid, int tid, int wave,
                                         const FragAddr& fa, int G, FirstTile&& first_tile) {
  TileCopier<kSrc> copy;
  copy.init(src, lds, tid, wave);
  copy.issue(0);
  if (ntiles > 1) copy.issue(1);
  wait_vm0();
  lds_barrier();

  // fill: scores of units 0 .. kQB-2; nothing to multiply by V yet
  load_k_frags<kSrc>(lds, 0, 0, fa, w.a);
  first_tile();
#pragma unroll
  for (int i = 0; i < 4; ++i) w.v[i].u = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < kJ; ++j) w.P[j].u = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int qb = 0; qb + 1 < kQB; ++qb) score_unit<kGen && !exact_logits(kSrc), kQB, kJ>(w, qb, w.S[qb]);

  int t = 0, cur = 0;
  bool ok = true;
  // one iteration = three tiles, so that the LDS buffer of every access is a constant
  for (int round = 0;; ++round) {
#define AGG_TILE(CUR)                                                                       \
  if (t + 1 >= ntiles) {                                                                    \
    cur = CUR;                                                                              \
    break;                                                                                  \
  }                                                                                         \
  if (t + 2 < ntiles) copy.issue((CUR + 2) % kLdsTiles);                                    \
  tile_steps<kSrc, false, kGen, kQB, kJ>(w, lds, CUR, (CUR + 1) % kLdsTiles, kTileRows, fa, G);      \
  wait_vm0();                                                                               \
  lds_barrier();                                                                            \
  ++t;
    AGG_TILE(0)
    AGG_TILE(1)
    AGG_TILE(2)
#undef AGG_TILE
    if (!kGen && !kSplit && (round & 7) == 7) {  // an overflowing row ends the fast pass early
      bool bad = false;
#pragma unroll
      for (int qb = 0; qb < kQB; ++qb)
#pragma unroll
        for (int j = 0; j < kJ; ++j) bad = bad || !(w.L[qb][j][0] < kSumHi);
      if (vote(bad, votes, wave, tid & 63, true)) {
        ok = false;
        break;
      }
    }
  }
  if (!ok) return false;
  // last tile (runtime buffer number), then the P V of its last unit
  tile_steps<kSrc, true, kGen, kQB, kJ>(w, lds, cur, 0, last_valid, fa, G);
  pv_unit<kGen, kQB, kJ>(w, kQB - 1);
  return true;
}

constexpr int kTileLds = 2 * kLdsTiles * kTileElems;  // elements: K tiles, then V tiles

// Wavefronts of a workgroup: four; eight, of which four take the first half of the keys and four the second; eight that all do the
// same, so that their barriers match, the first four of which store.
enum { kAlone, kSplitKeys, kTwin };

// position in a launch list of n tiles per pair -> (pair, tile of the pair).  Consecutive ids go
// to consecutive XCDs.  Whole pairs are dealt out one per XCD, so that an XCD streams one
// key/value set at a time through its own L2; the npairs % 8 pairs that are left share the XCDs
// between them, each XCD taking an equal, contiguous run of their tiles.  (Dealing those out whole
// as well left XCDs idle: ordinary attention over 24 frames of 28x37 patches with 12 heads took
// 2.12 ms, with the shared run 1.52.)
struct TileList {
  int n;         // tiles per pair
  int whole;     // tiles of an XCD's whole pairs
  int rest;      // tiles of an XCD's run over the remaining pairs
  int groups;    // workgroups of the list
};
__host__ __device__ inline TileList tile_list(int npairs, int n) {
  TileList l;
  l.n = n;
  l.whole = npairs / kXcds * n;
  l.rest = (npairs % kXcds * n + kXcds - 1) / kXcds;
  l.groups = kXcds * (l.whole + l.rest);
  return l;
}
__device__ __forceinline__ bool list_tile(const TileList& l, int npairs, int bid, int& pair, int& i) {
  const int xcd = bid % kXcds;
  const int seq = bid / kXcds;
  if (seq < l.whole) {
    pair = (seq / l.n) * kXcds + xcd;
    i = seq % l.n;
  } else {
    const int u = seq - l.whole + xcd * l.rest;
    if (u >= npairs % kXcds * l.n) return false;  // uniform for the whole workgroup
    pair = npairs / kXcds * kXcds + u / l.n;
    i = u % l.n;
  }
  return true;
}

}  // namespace agg
