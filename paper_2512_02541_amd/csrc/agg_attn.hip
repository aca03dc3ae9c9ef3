// Flash-style forward kernel for subsampled global attention (AVGGT Sec. 4.3):
// every query attends to the compacted key/value set, plus -- inside the same
// softmax -- its own key/value when its token was dropped and the mean pair of
// all dropped patches.  With an un-subsampled compacted set and no extras the
// same kernel is ordinary global attention (Sec. 4.2).
//
// Mapping to gfx950
//   * One workgroup = 4 wavefronts; a wavefront owns kQB blocks of 16 kJ queries (2 x 32 at full
//     width) for the whole key loop and keeps Q and the output accumulator in registers.  The
//     last workgroups of a launch may be narrower (plan_tiles).
//   * Both products run on v_mfma_f32_16x16x32_bf16, which accumulates 32 products per pass
//     through its four accumulator registers: half the accumulator traffic per flop of the
//     32x32x16 shape, and the part is power-limited on this kernel (measured on hashed
//     operands, MFMAs alone: 1.94 against 1.74 PFLOP/s).
//   * The score tile is computed transposed, S^T = K * Q^T: a lane then holds keys of ONE
//     query (four per 16-key tile), so row sums are in-register plus a reduction over the four
//     lanes c, c+16, c+32, c+48, and the exponentiated tiles are already the B operand of the
//     second product O^T += V^T * P^T.  P never touches LDS.  A 32-key block is scored as two
//     16-key tiles whose rows are assigned to the block's keys such that the eight probabilities
//     of a lane belong to exactly one 16-byte chunk of the compacted V tile (row_key below).
//     On the fast path the row sums are a ninth product of the same shape per query tile, a
//     row of ones against P^T (+12.5 % MFMAs): the vector ALU, which has to issue twice as
//     many MFMAs as with the larger shape, then does nothing per score but exponentiate and
//     convert.
//   * K/V arrive in "fragment order" (agg.h): a 64-key tile is a linear 8 KiB
//     copy into LDS and every MFMA A operand is one conflict-free 16-byte read.
//     Three tiles are resident: the one in use, the next one and the one being
//     filled.  Tiles go global -> LDS without passing through registers
//     (global_load_lds_dwordx4 with a scalar base, so advancing a tile costs two
//     scalar adds); a wavefront waits for its own copies before the barrier that
//     ends an iteration.  The tile loop is unrolled over the three buffers, so every
//     LDS read uses an immediate offset: the loop spends no vector instruction on
//     addresses.
//   * At head dimension 64 the vector ALU is as loaded as the matrix core (one
//     exponential per 256 MFMA flops) and a wavefront issues in order, so the key
//     loop is a software pipeline over "units" (32 keys x 16 kJ queries).  Step u
//     exponentiates unit u on the vector ALU while the matrix core computes the
//     scores of unit u + kQB - 1 and then P V of unit u - 1.  K fragments of a
//     32-key block are fetched from LDS once per kQB units, V fragments likewise.
//   * Fast path: Q is pre-multiplied by scale*log2(e) and the probabilities are
//     exp2 of the raw base-2 logits, with NO reference subtracted: softmax is
//     invariant to the reference, float/bf16 exponents cover 2^+-126, and the
//     per-score work shrinks to exp + convert.  A row whose sum leaves
//     [2^-90, 2^90] (logits beyond about +-60 nats) makes the whole workgroup
//     redo its rows in the general path (in place, or by a second kernel behind this
//     one, see redo_in_place); ordinary attention logits never get there.  The
//     sums are checked every few tiles, so an overflow ends the fast pass early.
//   * General path: the same pipeline with a per-row reference.  The score MFMAs start from
//     an accumulator holding minus the reference instead of zero, so the scores come out
//     relative to it and the vector ALU does no more per score than on the fast path.  The
//     reference starts at the largest of the extras and the first 32 keys and is raised
//     lazily: a unit's row sums show when a score exceeds it by more than 2^100; only then
//     (a rare, wavefront-uniform branch) is the unit's maximum taken, the accumulator
//     rescaled and the unit redone.  No running maximum is computed otherwise.
//   * A launch with at most one workgroup per CU runs eight wavefronts in each: two groups of four
//     that take half the key tiles each and add their sums and accumulators at the end (attend).
//   * The zero-padded rows of the last tile are masked there (the last tile is
//     peeled), nowhere else.
//   * The extras enter as the initial state (sum, accumulator) of either path, so
//     the three parts share one normalisation by construction.
//   * Workgroups are numbered so that the 8 XCDs each stream a different
//     (batch, head): all workgroups resident on one XCD read the same K/V
//     stream and share it through that XCD's L2.
#include "agg_attn_pipe.h"

namespace agg {

// Kernel arguments.
struct AttnArgs {
  Geom g;
  uint32_t flags;
  float qscale, mean_bias2;  // scale*log2(e), mean_logit_bias*log2(e)
  const uint16_t *Q, *K, *V, *Kc, *Vc;
  const float *kmean, *vmean;
  uint16_t* O;
  float* lse;
  int npairs;
  TilePlan plan;
  const uint32_t* kept_bits;
  const int32_t* nd_dev;
  const int32_t* list;   // kSrcIndexed: token ids of the keys, [list_stride] per batch element
  int64_t list_stride;   // 0 when every batch element uses the same list
};

// One workgroup's queries q_begin .. q_end - 1 (at most what four wavefronts hold) by one of the
// two paths.  Returns false, without storing anything, when the fast path met a row it cannot
// handle.
// tiles: kTileLds elements of LDS per four wavefronts; votes: kVoteWords words.
// kMode:
//   kAlone      four wavefronts.
//   kSplitKeys  (fast path) eight: the first four take the extras and the first half of the key
//               tiles, the others the second half.  Without a reference the two halves' sums and
//               accumulators just add: the second group's go through LDS to the first, which
//               finishes the rows.
//   kTwin       eight: both groups do the same (so that their barriers match), the first stores.
template <int kSrc, bool kGen, int kQB, int kJ, int kMode = kAlone>
__device__ __forceinline__ bool attend(const AttnArgs& p, uint16_t* tiles, uint32_t* votes, int b, int h,
                                       int64_t q_begin, int64_t q_end) {
  constexpr bool kSplit = kMode == kSplitKeys;
  static_assert(!(kGen && kSplit), "the general path's halves would need a common reference");
  constexpr int kWaveQ = wave_queries(kQB, kJ);
  const Geom& g = p.g;
  // The general path starts from an opaque thread number, so that the addresses it has in common
  // with a fast pass ahead of it in the same kernel are worked out again: held across the fast
  // key loop they spilled (sga_attn_kernel).
  int thread = threadIdx.x;
  if (kGen) asm volatile("" : "+v"(thread));
  const int group = kMode != kAlone ? __builtin_amdgcn_readfirstlane(thread / kAttnThreads) : 0;
  uint16_t* smem = tiles + group * kTileLds;
  u32x4* lds = reinterpret_cast<u32x4*>(smem);
  const int tid = thread - group * kAttnThreads;
  const int lane = tid & 63;
  const int wave = tid >> 6;
  const int c = lane & 15;
  const int G = lane >> 4;
  const FragAddr fa = frag_addr(lane);

  // this group's key tiles: first_tile_no .. first_tile_no + ntiles - 1
  const int all_tiles = (int)(g.M_pad / kTileRows);
  const int half = kSplit ? (all_tiles + 1) / 2 : all_tiles;
  const int skip = kSplit && group ? half : 0;
  const int ntiles = kSplit && group ? all_tiles - half : half;
  const int64_t rows_here = min(g.M - (int64_t)skip * kTileRows, (int64_t)ntiles * kTileRows);
  const int last_valid = (int)(rows_here - (int64_t)(ntiles - 1) * kTileRows);  // 1..64
  KvSource src;
  src.rows = rows_here;
  src.row_bytes = (uint32_t)g.H * (kHeadDim * 2);
  src.max_token = (uint32_t)(g.NQ - 1);
  if (kSrc == kSrcCompact) {
    const int64_t bh_off = (((int64_t)b * g.H + h) * g.M_pad + (int64_t)skip * kTileRows) * kHeadDim;
    src.k = uniform_ptr(p.Kc + bh_off);
    src.v = uniform_ptr(p.Vc + bh_off);
    src.list = nullptr;
  } else {
    const int64_t first_row = (int64_t)b * g.NQ + (kSrc == kSrcRows ? (int64_t)skip * kTileRows : 0);
    const int64_t bh_off = (first_row * g.H + h) * kHeadDim;
    src.k = uniform_ptr(p.K + bh_off);
    src.v = uniform_ptr(p.V + bh_off);
    src.list = kSrc == kSrcIndexed
                   ? p.list + (int64_t)b * p.list_stride + (int64_t)skip * kTileRows
                   : nullptr;
  }

  Wave<kQB, kJ> w;
  const uint32_t one = c == 0 ? 0x3F803F80u : 0u;
  w.ones.u = u32x4{one, one, one, one};
  bool dropped[kQB][kJ];
  float l_self[kQB][kJ], l_mean[kQB][kJ];  // base-2 logits of the extras (-inf when absent)
  // caller's list: membership comes from a bitmap, the dropped count from device memory
  const int64_t n_drop = p.nd_dev ? (int64_t)p.nd_dev[b] : g.n_dropped;
  // ordinary and per-frame attention have no extras; where that is known at compile time the fast
  // path's code is a third shorter (the general path's would spill: 363 to 532 registers instead of 9
  // or 10 in the second launch, 64 to 271 instead of none where rows are redone in place)
  constexpr bool kExtras = kSrc != kSrcRows || kGen;
  const bool takes = kExtras && !(kSplit && group);
  const bool use_mean = takes && (p.flags & AGG_MEAN) && n_drop > 0;
  const bool use_diag = takes && (p.flags & AGG_DIAG) && (p.kept_bits != nullptr || n_drop > 0);
  const uint32_t* kbits = p.kept_bits ? p.kept_bits + (int64_t)b * ((g.NQ + 31) / 32) : nullptr;
  const int64_t q_wave = q_begin + wave * kWaveQ;
  // first element of query (qb, j, c)'s row of this head in Q, K, V and O
  auto row_base = [&](int qb, int j) {
    const int64_t q = q_wave + (qb * kJ + j) * 16 + c;
    const int64_t qc = q < q_end ? q : q_end - 1;  // tail rows recompute the last query, never stored
    return (((int64_t)b * g.NQ + qc) * g.H + h) * kHeadDim;
  };
  // this lane's channels 16 dt + 4 G .. + 3 of the query's own value and of the mean value
  auto load_own_v = [&](int qb, int j, int dt) {
    return *reinterpret_cast<const u32x2*>(p.V + row_base(qb, j) + 16 * dt + 4 * G);
  };
  auto load_mean_v = [&](int dt) {
    const float* vm = p.vmean + ((int64_t)b * g.H + h) * kHeadDim;
    return *reinterpret_cast<const f32x4*>(vm + 16 * dt + 4 * G);
  };

  // ---- Q fragments and the logits of the extras ----
  // A lane holds channels 32 h + 8 G .. + 7 (h = 0, 1) of its query: the four lanes c + 16 G
  // share the channel range.  Everything is requested before anything is used, and one lane per
  // query works out whether that was dropped: with a tile's loads behind the previous tile's
  // arithmetic, and every lane dividing for each of its tiles, a workgroup spent 14 us here before its
  // first key in a layer of 10 frames (now 8.5; 363 us a call instead of 370), 3.8 in one of two frames of
  // 16x16 (2.6; 14.5 instead of 15.1).
#pragma unroll
  for (int qb = 0; qb < kQB; ++qb)
#pragma unroll
    for (int j = 0; j < kJ; ++j)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
        w.Qf[qb][2 * j + hh].u = *reinterpret_cast<const u32x4*>(p.Q + row_base(qb, j) + hh * 32 + G * 8);
  uint64_t drop_mask = 0;  // bit i: query q_wave + i was dropped
  if (use_diag) {
    const int64_t q = q_wave + lane;
    bool d = false;
    if (lane < kWaveQ && q < q_end)
      d = kbits ? ((kbits[q >> 5] >> (q & 31)) & 1u) == 0u : (bool)token_is_dropped(g, q);
    drop_mask = __builtin_amdgcn_ballot_w64(d);
  }
  // the query's own key and value, the mean pair (general path: the values only once the row's
  // reference is known, its registers being scarcer)
  u32x4 own_k[kQB][kJ][2];
  u32x2 own_v[kQB][kJ][4];
  f32x4 mean_k[4], mean_v[4];
#pragma unroll
  for (int qb = 0; qb < kQB; ++qb)
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      dropped[qb][j] = (drop_mask >> (16 * (qb * kJ + j) + c)) & 1u;
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) own_k[qb][j][hh] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) own_v[qb][j][dt] = u32x2{0u, 0u};
      if (kExtras && dropped[qb][j]) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
          own_k[qb][j][hh] = *reinterpret_cast<const u32x4*>(p.K + row_base(qb, j) + hh * 32 + G * 8);
        if (!kGen) {
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) own_v[qb][j][dt] = load_own_v(qb, j, dt);
        }
      }
    }
  if (kExtras && use_mean) {
    const float* km = p.kmean + ((int64_t)b * g.H + h) * kHeadDim;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mean_k[i] = *reinterpret_cast<const f32x4*>(km + (i >> 1) * 32 + G * 8 + 4 * (i & 1));
      if (!kGen) mean_v[i] = load_mean_v(i);
    }
  }
#pragma unroll
  for (int qb = 0; qb < kQB; ++qb)
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const u32x4 raw = w.Qf[qb][2 * j + hh].u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w.Qf[qb][2 * j + hh].u[i] =
              pack_bf16(bf16_lo(raw[i]) * p.qscale, bf16_hi(raw[i]) * p.qscale);
      }
      float dot_self = 0.f, dot_mean = 0.f;
      if (use_mean || use_diag) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          float qv[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            qv[2 * i] = bf16_lo(w.Qf[qb][2 * j + hh].u[i]);
            qv[2 * i + 1] = bf16_hi(w.Qf[qb][2 * j + hh].u[i]);
          }
          if (use_mean) {
#pragma unroll
            for (int i = 0; i < 4; ++i) dot_mean += qv[i] * mean_k[2 * hh][i] + qv[4 + i] * mean_k[2 * hh + 1][i];
          }
          if (use_diag) {
            const u32x4 kr = own_k[qb][j][hh];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              dot_self += qv[2 * i] * bf16_lo(kr[i]) + qv[2 * i + 1] * bf16_hi(kr[i]);
          }
        }
      }
      dot_self = quad_sum(dot_self);
      dot_mean = quad_sum(dot_mean);
      l_self[qb][j] = dropped[qb][j] ? dot_self : -INFINITY;
      l_mean[qb][j] = use_mean ? dot_mean + p.mean_bias2 : -INFINITY;
    }

  // Initial state = extras weighted by exp2(logit - m0):  O0[d] = w_self v_i[d] + w_mean vmean[d]
  auto init_extras = [&](int qb, int j, float m0) {
    const float w_self = dropped[qb][j] ? fast_exp2(l_self[qb][j] - m0) : 0.f;
    const float w_mean = use_mean ? fast_exp2(l_mean[qb][j] - m0) : 0.f;
    const float l0 = w_self + w_mean;
    if (kGen) w.la[qb][j] = (G == 0) ? l0 : 0.f;  // four lanes split a row's sum
    else w.L[qb][j] = f32x4{l0, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      if (use_mean) acc = (kGen ? load_mean_v(dt) : mean_v[dt]) * w_mean;
      if (dropped[qb][j]) {
        const u32x2 vr = kGen ? load_own_v(qb, j, dt) : own_v[qb][j][dt];
        acc[0] += w_self * bf16_lo(vr[0]);
        acc[1] += w_self * bf16_hi(vr[0]);
        acc[2] += w_self * bf16_lo(vr[1]);
        acc[3] += w_self * bf16_hi(vr[1]);
      }
      w.O[qb][j][dt] = acc;
    }
  };

  if (!kGen) {
#pragma unroll
    for (int qb = 0; qb < kQB; ++qb)
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        w.mref[qb][j] = 0.f;
        init_extras(qb, j, 0.f);
      }
  }
  // general path: the reference is the largest of the extras and of the first 32 keys (row 0
  // always exists); taken when the first tile's K fragments are in registers
  auto first_tile = [&]() {
    if (!kGen) return;
    const int valid0 = ntiles == 1 ? last_valid : kTileRows;
#pragma unroll
    for (int qb = 0; qb < kQB; ++qb) {
#pragma unroll
      for (int j = 0; j < kJ; ++j) w.mref[qb][j] = 0.f;
      f32x4 s[2 * kJ];
      score_unit<kGen, kQB, kJ>(w, qb, s);
      if (valid0 < 32) mask_unit<kJ>(s, 0, valid0, G);
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        float mx = s[j][0];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[kJ * kt + j][r]);
        mx = quad_max(mx);
        mx = fmaxf(mx, fmaxf(l_self[qb][j], l_mean[qb][j]));
        // a NaN or infinite score cannot serve as reference; the row's result is NaN anyway
        if (!(fabsf(mx) < 3.0e38f)) mx = 0.f;
        w.mref[qb][j] = mx;
        init_extras(qb, j, mx);
      }
    }
  };

  const bool done = key_loop<kSrc, kGen, kSplit, kQB, kJ>(w, lds, votes, src, ntiles, last_valid, tid,
                                                          wave, fa, G, first_tile);
  if (kSplit) {
    // a loop passes one barrier per tile: the shorter one makes up for its missing tile
    if (ntiles < half) lds_barrier();
    __syncthreads();  // both groups are done with their tiles
    // [register][wavefront][lane], over the second group's tiles
    f32x4* over = reinterpret_cast<f32x4*>(tiles + kTileLds) + tid;
    float* over_l = reinterpret_cast<float*>(tiles + kTileLds) + kQB * kJ * 4 * 4 * kAttnThreads + tid;
    static_assert(!kSplit || kQB * kJ * (4 * 16 + 4) * kAttnThreads <= kTileLds * 2, "fits the group's LDS");
    if (group) {
#pragma unroll
      for (int i = 0; i < kQB * kJ; ++i) {
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) over[(4 * i + dt) * kAttnThreads] = w.O[i / kJ][i % kJ][dt];
        over_l[i * kAttnThreads] = w.L[i / kJ][i % kJ][0];
      }
    }
    __syncthreads();
    if (!group) {
#pragma unroll
      for (int i = 0; i < kQB * kJ; ++i) {
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) w.O[i / kJ][i % kJ][dt] += over[(4 * i + dt) * kAttnThreads];
        w.L[i / kJ][i % kJ][0] += over_l[i * kAttnThreads];
      }
    }
  }
  float l_fin[kQB][kJ];
  bool unsafe = false;
#pragma unroll
  for (int qb = 0; qb < kQB; ++qb)
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      l_fin[qb][j] = kGen ? quad_sum(w.la[qb][j]) : __shfl(w.L[qb][j][0], c);  // every lane knows its query's
      // a sum outside [2^-90, 2^90] (or NaN): the unreferenced exponentials were not safe
      unsafe = unsafe || (group == 0 && (!(l_fin[qb][j] < kSumHi) || !(l_fin[qb][j] > kSumLo)));
    }
  if (!kGen) {
    if (!done) return false;  // uniform: decided by a workgroup-wide vote inside the loop
    if (vote(unsafe, votes + kWaves, wave, lane, group == 0)) return false;
  }

  // ---- normalise and store ----
  // A lane holds four consecutive channels of one query per accumulator tile: stored from there,
  // every instruction would scatter 8-byte pieces over 16 rows that lie 2*H*64 bytes apart.
  // Each wavefront instead turns its tile, a query block at a time, through a private part of the
  // (now idle) K/V LDS and writes whole 128-byte (query, head) rows, eight per instruction.
  // every wavefront is done with the K/V tiles (fast path: the vote's barrier has seen to that)
  if (kGen) __syncthreads();
  if (group) return true;
  // (The thread number is made opaque here, so that this part's lane numbers and addresses are worked
  // out again: held across the key loop they take 6 to 14 registers more, and the narrow index-driven
  // kernels have none left.)
  int here = tid;
  asm volatile("" : "+v"(here));
  const int elane = here & 63, ec = here & 15, eG = elane >> 4;
  uint16_t* epi = smem + wave * (16 * kJ * kEpiStride);
#pragma unroll
  for (int qb = 0; qb < kQB; ++qb) {
    const int64_t q0 = q_wave + qb * kJ * 16;
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      const float l = l_fin[qb][j];
      const float inv = 1.0f / l;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        const int d0 = 16 * dt + 4 * eG;
        u32x2 o2;
        o2[0] = pack_bf16(w.O[qb][j][dt][0] * inv, w.O[qb][j][dt][1] * inv);
        o2[1] = pack_bf16(w.O[qb][j][dt][2] * inv, w.O[qb][j][dt][3] * inv);
        *reinterpret_cast<u32x2*>(epi + (16 * j + ec) * kEpiStride + d0) = o2;
      }
      if (p.lse && eG == 0 && q0 + 16 * j + ec < q_end)
        p.lse[((int64_t)b * g.H + h) * g.NQ + q0 + 16 * j + ec] =
            ((kGen ? w.mref[qb][j] : 0.f) + log2f(l)) * kLn2;
    }
    // the wavefront's own writes, read back by other lanes of the same wavefront
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
#pragma unroll
    for (int i = 0; i < 2 * kJ; ++i) {
      const int row = i * 8 + (elane >> 3);
      const int64_t q = q0 + row;
      const u32x4 o4 = *reinterpret_cast<const u32x4*>(epi + row * kEpiStride + (elane & 7) * 8);
      if (q < q_end)
        *reinterpret_cast<u32x4*>(p.O + (((int64_t)b * g.NQ + q) * g.H + h) * kHeadDim +
                                  (elane & 7) * 8) = o4;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  }
  return true;
}

__host__ __device__ inline TileList first_list(const TilePlan& t, int npairs) {
  return tile_list(npairs, t.n_full + (t.tails_last ? 0 : t.n_tail));
}
__host__ __device__ inline TileList second_list(const TilePlan& t, int npairs) {
  return tile_list(npairs, t.tails_last ? t.n_tail : 0);
}

// What a workgroup does: queries q_begin .. q_end - 1 of batch element b, head h.
struct Work {
  int b, h;
  int64_t q_begin, q_end;
  bool tail;
};
__device__ __forceinline__ bool workgroup_work(const AttnArgs& p, Work& w) {
  const TilePlan& t = p.plan;
  const TileList first = first_list(t, p.npairs);
  int pair, i;
  if ((int)blockIdx.x < first.groups) {
    if (!list_tile(first, p.npairs, blockIdx.x, pair, i)) return false;
  } else {
    if (!list_tile(second_list(t, p.npairs), p.npairs, blockIdx.x - first.groups, pair, i)) return false;
    i += t.n_full;
  }
  w.b = pair / p.g.H;
  w.h = pair % p.g.H;
  w.tail = i >= t.n_full;
  w.q_begin = w.tail ? (int64_t)t.n_full * kQTile + (int64_t)(i - t.n_full) * t.tail_q
                     : (int64_t)i * kQTile;
  w.q_end = min(p.g.NQ, w.q_begin + (w.tail ? t.tail_q : kQTile));
  return true;
}

// A workgroup whose fast pass failed leaves this pattern (four bf16 NaNs with distinct payloads)
// in the first four channels of its first output row and stores nothing else; the second kernel
// redoes exactly the workgroups that carry it.  Should a correct result ever equal the pattern,
// the second kernel recomputes that workgroup, which is harmless.
constexpr uint64_t kRedoMark = 0x7F997FC37FA57FC1ull;

__device__ __forceinline__ uint64_t* redo_slot(const AttnArgs& p, const Work& w) {
  return reinterpret_cast<uint64_t*>(p.O + (((int64_t)w.b * p.g.NQ + w.q_begin) * p.g.H + w.h) * kHeadDim);
}

// The kernel's arguments (its only parameter, at the start of its argument memory), to be read again
// from here on: what one path derives from them is then not held for another.
__device__ __forceinline__ const AttnArgs& args_again() {
  typedef const __attribute__((address_space(4))) AttnArgs* KernelArgs;
  KernelArgs args = (KernelArgs)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(args));
  return *(const AttnArgs*)args;
}

// blocks (of one 16-query tile) of a narrow workgroup's wavefront
constexpr int tail_blocks(int tail_q) { return tail_q == 192 ? 3 : 2; }

// kTailQ: queries of the launch's narrow workgroups (0: it has none).
// kRedo: a workgroup redoes its own rows by the general path, 128 queries at a time, instead of
// leaving the mark for a second launch.  At that width the general path needs no more registers
// than the fast one, provided that nothing is held for it meanwhile: it starts from an opaque
// thread number (attend) and reads the kernel's arguments again.  So no instance spills, which a
// build test checks, and each uses within 2 registers what it uses without kRedo (234 to 248).  Sharing
// both with the fast path spills 4 registers (compacted), 14 (rows) and 25 (indexed) at full width.
template <int kSrc, int kTailQ, bool kRedo>
__global__ __launch_bounds__(kAttnThreads, kBlocksPerCu) void sga_attn_kernel(AttnArgs p) {
  __shared__ __align__(16) uint16_t tiles[kTileLds];
  __shared__ __align__(16) uint32_t votes[kVoteWords];
  Work w;
  if (!workgroup_work(p, w)) return;
  bool done;
  if (kTailQ != 0 && w.tail)
    done = attend<kSrc, false, tail_blocks(kTailQ), 1>(p, tiles, votes, w.b, w.h, w.q_begin, w.q_end);
  else
    done = attend<kSrc, false, 2, 2>(p, tiles, votes, w.b, w.h, w.q_begin, w.q_end);
  if (done) return;
  if (!kRedo) {
    if (threadIdx.x == 0) *redo_slot(p, w) = kRedoMark;
    return;
  }
  const AttnArgs& again = args_again();
#pragma unroll 1
  for (int64_t q = w.q_begin; q < w.q_end; q += kWaves * wave_queries(2, 1)) {
    __syncthreads();  // the LDS is free
    attend<kSrc, true, 2, 1>(again, tiles, votes, w.b, w.h, q, min(w.q_end, q + kWaves * wave_queries(2, 1)));
  }
}

// A launch of few workgroups: 128 queries each, eight wavefronts.  Rows that leave the fast path's
// range are redone here by the general path, which at this width needs no more registers: an idle
// second launch would be a fifth of a small call's time.
template <int kSrc>
__global__ __launch_bounds__(2 * kAttnThreads, 2) void sga_attn_split_kernel(AttnArgs p) {
  __shared__ __align__(16) uint16_t tiles[2 * kTileLds];
  __shared__ __align__(16) uint32_t votes[kVoteWords];
  Work w;
  if (!workgroup_work(p, w)) return;
  if (attend<kSrc, false, 2, 1, kSplitKeys>(p, tiles, votes, w.b, w.h, w.q_begin, w.q_end)) return;
  __syncthreads();
  attend<kSrc, true, 2, 1, kTwin>(p, tiles, votes, w.b, w.h, w.q_begin, w.q_end);
}

// The general path is a kernel of its own, launched behind the first on the same stream: it is
// rarely needed, starts over from the workgroup's inputs, and this way does not weigh on the
// register allocation of the fast path.  Workgroups without the mark leave at once; narrow ones are
// redone at their own width.  (At full width, with the queries beyond their own left out, calls of
// which every workgroup is redone took, us, then / now, and with full-width workgroups alone in both
// launches: ordinary attention, 12 frames of 37x37 2013 / 1610, 1835; 10 frames of 28x37, 8 heads
// 398 / 301, 398; compacted, 25 frames 2927 / 2739, 2990.)
template <int kSrc, int kTailQ>
__global__ __launch_bounds__(kAttnThreads, kBlocksPerCu) void sga_attn_general_kernel(AttnArgs p) {
  __shared__ __align__(16) uint16_t tiles[kTileLds];
  __shared__ __align__(16) uint32_t votes[kVoteWords];
  Work w;
  if (!workgroup_work(p, w)) return;
  if (*redo_slot(p, w) != kRedoMark) return;  // same value in every lane
  __syncthreads();  // every wavefront has read the mark before any of them overwrites it
  if (kTailQ != 0 && w.tail)
    attend<kSrc, true, tail_blocks(kTailQ), 1>(args_again(), tiles, votes, w.b, w.h, w.q_begin, w.q_end);
  else
    attend<kSrc, true, 2, 2>(p, tiles, votes, w.b, w.h, w.q_begin, w.q_end);
}

template <int kSrc, int kTailQ>
static void launch_both(const AttnArgs& p, dim3 grid, hipStream_t st) {
  const dim3 block(kAttnThreads);
  if (redo_in_place(p.g.M_pad / kTileRows)) {
    hipLaunchKernelGGL((sga_attn_kernel<kSrc, kTailQ, true>), grid, block, 0, st, p);
  } else {
    hipLaunchKernelGGL((sga_attn_kernel<kSrc, kTailQ, false>), grid, block, 0, st, p);
    hipLaunchKernelGGL((sga_attn_general_kernel<kSrc, kTailQ>), grid, block, 0, st, p);
  }
}

static int64_t plan_groups(const TilePlan& t, int npairs) {
  return (int64_t)first_list(t, npairs).groups + second_list(t, npairs).groups;
}

template <int kSrc>
static void launch_source(const AttnArgs& p, hipStream_t st) {
  const dim3 grid((unsigned)plan_groups(p.plan, p.npairs));
  const int tail_q = p.plan.n_tail ? p.plan.tail_q : 0;
  if (p.plan.split) hipLaunchKernelGGL(sga_attn_split_kernel<kSrc>, grid, dim3(2 * kAttnThreads), 0, st, p);
  else if (tail_q == 0) launch_both<kSrc, 0>(p, grid, st);
  else if (tail_q == 192) launch_both<kSrc, 192>(p, grid, st);
  else launch_both<kSrc, 128>(p, grid, st);
}

hipError_t launch_attn(const Geom& g, uint32_t flags, float scale, float mean_bias, const void* Q,
                       const void* K, const void* V, const void* Kc, const void* Vc,
                       const float* kmean, const float* vmean, void* O, float* lse, hipStream_t st,
                       const uint32_t* kept_bits, const int32_t* nd_dev, int src_mode,
                       const int32_t* list, int64_t list_stride) {
  const int64_t pairs = (int64_t)g.B * g.H;
  // the bound on the grid, with whole pairs per XCD throughout (narrow workgroups: plan_tiles)
  if (pairs > 0x7FFFFFFF - kXcds ||
      (pairs + kXcds - 1) / kXcds * kXcds * ((g.NQ + kQTile - 1) / kQTile) > 0x7FFFFFFF)
    return hipErrorInvalidConfiguration;
  const int npairs = (int)pairs;
  const TilePlan plan = plan_tiles(g.NQ, npairs, g.M_pad / kTileRows);
  // A launch has fewer than 2^32 threads (kLaunchRows): beyond that each half of the batch is a call of its own.
  // Per-frame attention, whose frames are the batch here, gets there with 2^24 frames and heads of a few tokens.
  if (plan_groups(plan, npairs) > 0xFFFFFFFFll / kAttnThreads) {
    if (g.B < 2) return hipErrorInvalidConfiguration;
    Geom half[2] = {g, g};
    half[0].B = g.B / 2;
    half[1].B = g.B - half[0].B;
    int64_t b = 0;
    for (const Geom& h : half) {
      const int64_t rows = b * g.NQ * g.H * kHeadDim, kept = b * g.H * g.M_pad * kHeadDim, means = b * g.H * kHeadDim;
      auto at = [](const void* t, int64_t elements) { return t ? (const uint16_t*)t + elements : nullptr; };
      const hipError_t e = launch_attn(
          h, flags, scale, mean_bias, at(Q, rows), at(K, rows), at(V, rows), at(Kc, kept), at(Vc, kept),
          kmean ? kmean + means : nullptr, vmean ? vmean + means : nullptr, (uint16_t*)O + rows,
          lse ? lse + b * g.H * g.NQ : nullptr, st, kept_bits ? kept_bits + b * ((g.NQ + 31) / 32) : nullptr,
          nd_dev ? nd_dev + b : nullptr, src_mode, list ? list + b * list_stride : nullptr, list_stride);
      if (e != hipSuccess) return e;
      b += h.B;
    }
    return hipSuccess;
  }
  // indexed rows are addressed with 32-bit byte offsets from the (batch, head) base, formed by
  // a 24-bit multiplication of token id and row length
  if (src_mode == kSrcIndexed && ((uint64_t)g.NQ * g.H * (kHeadDim * 2) > 0xFFFFFFFFull ||
                                  g.NQ > 0xFFFFFF || (uint64_t)g.H * (kHeadDim * 2) > 0xFFFFFF))
    return hipErrorInvalidValue;
  (void)hipGetLastError();  // drop any stale error so the check below is this launch's
  AttnArgs p;
  p.g = g;
  p.flags = flags;
  p.qscale = scale * kLog2e;
  p.mean_bias2 = mean_bias * kLog2e;
  p.Q = (const uint16_t*)Q;
  p.K = (const uint16_t*)K;
  p.V = (const uint16_t*)V;
  p.Kc = (const uint16_t*)Kc;
  p.Vc = (const uint16_t*)Vc;
  p.kmean = kmean;
  p.vmean = vmean;
  p.O = (uint16_t*)O;
  p.lse = lse;
  p.npairs = npairs;
  p.plan = plan;
  p.kept_bits = kept_bits;
  p.nd_dev = nd_dev;
  p.list = list;
  p.list_stride = list_stride;
  if (src_mode == kSrcCompact) launch_source<kSrcCompact>(p, st);
  else if (src_mode == kSrcRows) launch_source<kSrcRows>(p, st);
  else launch_source<kSrcIndexed>(p, st);
  return hipGetLastError();
}

}  // namespace agg
