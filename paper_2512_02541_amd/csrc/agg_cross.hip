// Attention of queries to keys and values of another length, lying where they are or in the pages of a cache.
#include "agg_attn_pipe.h"
#include "agg_cross_plan.h"

namespace agg {

namespace {

// keys and queries of batch element b, whatever the caller's lengths hold
__device__ __forceinline__ int cross_keys(const CrossArgs& a, int b) {
  return a.k_lens ? min(max(((ScalarInts)a.k_lens)[b], 0), a.NK) : a.NK;
}
__device__ __forceinline__ int cross_queries(const CrossArgs& a, int b) {
  return a.q_lens ? min(max(((ScalarInts)a.q_lens)[b], 0), a.NQ) : a.NQ;
}

// row of a pair -> its query and its head
struct RowPlace {
  int q, head;
};
__device__ __forceinline__ RowPlace row_place(const CrossArgs& a, int hk, uint32_t row) {
  if (a.group == 1) return {(int)row, hk};
  const uint32_t q = row / (uint32_t)a.group;
  return {(int)q, hk * a.group + (int)(row - q * (uint32_t)a.group)};
}

// where a split's results of a pair's row lie in the workspace: 64 floats of a row, behind them all {reference, sum} of each.
// (Keys are shared out among at most kMostShared workgroups: fewer than 2^20 rows.)
__device__ __forceinline__ uint32_t partial_row(const CrossArgs& a, uint32_t pairs, uint32_t split, uint32_t pair, uint32_t row) {
  return (split * pairs + pair) * (uint32_t)(a.NQ * a.group) + row;
}

__device__ __forceinline__ float* partial_sums(const CrossArgs& a, uint32_t pairs, uint32_t splits) {
  return a.partial + (size_t)splits * pairs * (uint32_t)(a.NQ * a.group) * kHeadDim;
}

// part i of n units of work that are shared out in `parts`, fewer than 2^32 / 64 units and at most 64 parts: where it begins
__device__ __forceinline__ int part_begin(uint32_t n, uint32_t i, uint32_t parts) { return (int)(n * i / parts); }

__device__ __forceinline__ u32x2 pack4(f32x4 v) { return u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; }

// A finished row: four channels a thread.  m: the reference in base 2, l: the sum, o: sum of exp2(logit - m) v.
__device__ __forceinline__ void store_row(const CrossArgs& a, int b, int hk, uint32_t row, int quad, float m, float l, f32x4 o,
                                          bool no_keys) {
  const RowPlace at = row_place(a, hk, row);
  const float inv = no_keys ? 0.f : 1.f / l;
  *reinterpret_cast<u32x2*>(a.O + (((int64_t)b * a.NQ + at.q) * a.H + at.head) * kHeadDim + 4 * quad) = pack4(o * inv);
  if (a.lse && quad == 0)
    a.lse[((int64_t)b * a.H + at.head) * a.NQ + at.q] = no_keys ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

// ---------------------------------------------------------------------------
// Few rows a pair, and calls of more that fit on the card at once: bound by the keys and values, which are read once for every 16
// or 32 rows.  Every wavefront takes 32-key blocks of its own, straight into registers (a page's fragment order is the order of the
// matrix instruction's operands; rows read in place need one turn of the values through LDS), a block ahead of the one it works on,
// with the running maximum and sum of an online softmax; the wavefronts of a workgroup, and the workgroups that share a pair's keys,
// are joined at the end by their references.
// Measured (16 heads): one query over 137400 keys in pages 97 us = 5.8 TB/s, in place 112 = 5.0 (a device copy: 4.9); 32 rows the
// same within 5 %; over 262 keys 4.1 to 4.4, nearly all of it latencies one after another.  Four wavefronts of 64 rows: 15.8 us where two
// workgroups of 32 rows take 9.0 (64 rows, 1374 keys).
// ---------------------------------------------------------------------------
constexpr int kFewThreads = 64 * kFewWaves;
constexpr int kRowFloats = kHeadDim + 4;  // of a row in LDS, padded
constexpr uint32_t kRunsFrom = 768;       // workgroups from which each XCD takes a run of them

template <bool kPaged, int kJ>
__global__ __launch_bounds__(kFewThreads, kJ == 1 ? 4 : 2) void cross_few_kernel(CrossArgs a, CrossPlan plan, uint32_t pairs,
                                                                                    uint32_t first, uint32_t count) {
  constexpr int kW = kFewWaves;
  __shared__ __align__(16) float lds[kW * 16 * kJ * (kRowFloats + 2)];
  static_assert(sizeof(lds) >= kW * 4096, "a block of values for each wavefront");
  const int lane = threadIdx.x & 63, c = lane & 15, G = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (32-bit divisions: with 64 bits each a call of one query over 262 keys took 4.3 us instead of 4.1)
  // Many workgroups over rows in place: each XCD takes a run of them, so that the heads of a token, whose rows lie beside each other, are
  // read by one (us, 20 queries to 1374 keys of each of 100 and 48 frames, 16 heads: 135 -> 114, 50.8 -> 48.8; one query 118 -> 103; fewer
  // workgroups, and pages, are 0 to 6 % slower so).
  uint32_t number = blockIdx.x;
  if (!kPaged && count >= kRunsFrom) {
    number = (number % kXcds) * (gridDim.x / kXcds) + number / kXcds;
    if (number >= count) return;
  }
  const uint32_t id = first + number, pair = id % pairs;
  const uint32_t row_tile = id / pairs / (uint32_t)plan.splits;
  const int split = (int)(id / pairs % (uint32_t)plan.splits);
  const int b = (int)(pair / (uint32_t)a.H_kv), hk = (int)(pair % (uint32_t)a.H_kv);
  const int n = cross_keys(a, b);
  const uint32_t rows = (uint32_t)cross_queries(a, b) * (uint32_t)a.group;
  const uint32_t r0 = row_tile * (16 * kJ);
  if (r0 >= rows) return;
  const uint32_t blocks = ((uint32_t)n + kKeyBlock - 1) / kKeyBlock;
  const int lo = part_begin(blocks, split, plan.splits), hi = part_begin(blocks, split + 1, plan.splits);

  Frag Q[kJ][2];
#pragma unroll
  for (int j = 0; j < kJ; ++j) {
    const RowPlace at = row_place(a, hk, min(r0 + 16 * j + c, rows - 1));
    const uint16_t* q = a.Q + ((int64_t)b * a.NQ + at.q) * a.q_stride + at.head * kHeadDim;
#pragma unroll
    for (int h = 0; h < 2; ++h) Q[j][h].u = *reinterpret_cast<const u32x4*>(q + 32 * h + 8 * G);
  }

  struct Block {
    u32x4 k[4], v[4];
  };
  lds_char* const vbuf = (lds_char*)lds + wave * 4096;
  const FragAddr fa = frag_addr(lane);
  auto load = [&](int blk, Block& x) {
    if constexpr (kPaged) {
      const int page = min(max(((ScalarInts)a.pages)[(int64_t)b * a.max_pages + (blk >> 1)], 0), a.n_pages - 1);
      const int64_t base = ((int64_t)page * a.H_kv + hk) * kTileElems + (blk & 1) * (kTileElems / 2);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          x.k[2 * kt + h] = *reinterpret_cast<const u32x4*>(a.Kc + base + ((4 * h + G) * 32 + row_key(c) + 8 * kt) * 8);
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) x.v[dt] = *reinterpret_cast<const u32x4*>(a.Vc + base + (G * 64 + 16 * dt + c) * 8);
    } else {
      const int64_t first_row = (int64_t)b * a.NK;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {  // rows past the end repeat the last one; masked later
        const int row = min(blk * kKeyBlock + row_key(c) + 8 * kt, n - 1);
        const uint16_t* k = a.K + (first_row + row) * a.k_stride + hk * kHeadDim;
#pragma unroll
        for (int h = 0; h < 2; ++h) x.k[2 * kt + h] = *reinterpret_cast<const u32x4*>(k + 32 * h + 8 * G);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = blk * kKeyBlock + 8 * i + (lane >> 3);
        x.v[i] = u32x4{0u, 0u, 0u, 0u};
        if (row < n)
          x.v[i] = *reinterpret_cast<const u32x4*>(a.V + (first_row + row) * a.v_stride + hk * kHeadDim + (lane & 7) * 8);
      }
    }
  };

  f32x4 O[kJ][4];
  float m[kJ], l[kJ];  // m: largest score so far, a plain product (exp_unit_relative); l: this lane's part of the sum
#pragma unroll
  for (int j = 0; j < kJ; ++j) {
    m[j] = -INFINITY;
    l[j] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) O[j][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto step = [&](int blk, const Block& x) {
    const int left = n - blk * kKeyBlock;  // keys of the block that exist, if fewer than all
    Frag K[4], V[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) K[i].u = x.k[i];
    if constexpr (kPaged) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) V[dt].u = x.v[dt];
      if (left < kKeyBlock) mask_values(V, left, G);
    } else {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 8 * i + (lane >> 3), chunk = (lane & 7) ^ (4 * ((row >> 1) & 1));
        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(vbuf + row * 128 + chunk * 16) = x.v[i];
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        lds_char* at = vbuf + fa.v[dt];
        const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
        const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * 128));
        const u32x2 l2 = __builtin_bit_cast(u32x2, x0), h2 = __builtin_bit_cast(u32x2, x1);
        V[dt].u = u32x4{l2[0], l2[1], h2[0], h2[1]};
      }
    }
    f32x4 S[2 * kJ];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        S[kJ * kt + j] = AGG_MFMA16(K[2 * kt], Q[j][0], (f32x4{0.f, 0.f, 0.f, 0.f}));
        S[kJ * kt + j] = AGG_MFMA16(K[2 * kt + 1], Q[j][1], S[kJ * kt + j]);
      }
    if (left < kKeyBlock) mask_unit<kJ>(S, 0, left, G);
    Frag P[kJ];
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      float top = S[j][0];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, S[kJ * kt + j][r]);
      const float now = fmaxf(m[j], quad_max(top));
      const float ref = now == -INFINITY ? 0.f : now;  // (logits may be -infinity)
      const float f = fast_exp2((m[j] - ref) * a.scale2);
      m[j] = now;
      l[j] *= f;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) O[j][dt] *= f;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float e0 = fast_exp2((S[kJ * kt + j][2 * i] - ref) * a.scale2);
          const float e1 = fast_exp2((S[kJ * kt + j][2 * i + 1] - ref) * a.scale2);
          P[j].u[2 * kt + i] = pack_bf16(e0, e1);
          l[j] += e0 + e1;
        }
    }
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int j = 0; j < kJ; ++j) O[j][dt] = AGG_MFMA16(V[dt], P[j], O[j][dt]);
  };

  int blk = lo + wave;
  if (blk < hi) {
    Block x, ahead;
    load(blk, x);
    for (;;) {
      const int next = blk + kW;
      if (next < hi) load(next, ahead);
      step(blk, x);
      if (next >= hi) break;
      blk = next;
      x = ahead;
    }
  }

  // ---- join the wavefronts ----
  float* const sums = lds + kW * 16 * kJ * kRowFloats;  // {reference, sum} of each wavefront's rows
  __syncthreads();                                      // (the values' blocks lie here)
#pragma unroll
  for (int j = 0; j < kJ; ++j) {
    const float total = quad_sum(l[j]);
    float* const row = lds + (wave * 16 * kJ + 16 * j + c) * kRowFloats;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) *reinterpret_cast<f32x4*>(row + 16 * dt + 4 * G) = O[j][dt];
    if (G == 0) *reinterpret_cast<f32x2*>(sums + (wave * 16 * kJ + 16 * j + c) * 2) = f32x2{m[j], total};
  }
  __syncthreads();
  for (int item = threadIdx.x; item < 16 * kJ * 16; item += 64 * kW) {
    const int row = item >> 4, quad = item & 15;
    if (r0 + row >= rows) continue;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kW; ++w) top = fmaxf(top, sums[(w * 16 * kJ + row) * 2]);
    const float ref = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      const f32x2 s = *reinterpret_cast<const f32x2*>(sums + (w * 16 * kJ + row) * 2);
      const float f = fast_exp2((s[0] - ref) * a.scale2);
      total += s[1] * f;
      o += *reinterpret_cast<const f32x4*>(lds + (w * 16 * kJ + row) * kRowFloats + 4 * quad) * f;
    }
    if (plan.splits == 1) {
      store_row(a, b, hk, r0 + row, quad, ref * a.scale2, total, o, n == 0);
    } else {
      const size_t at = partial_row(a, pairs, split, pair, r0 + row);
      *reinterpret_cast<f32x4*>(a.partial + at * kHeadDim + 4 * quad) = o;
      // (-infinity: no keys, or none that weighs anything)
      if (quad == 0) *reinterpret_cast<f32x2*>(partial_sums(a, pairs, plan.splits) + at * 2) = f32x2{top * a.scale2, total};
    }
  }
}

// ---------------------------------------------------------------------------
// Many rows a pair: the pipeline of agg_attn.hip over keys that end where the sequence's do, bound like it by the matrix core
// and the vector ALU together, and by power.  256 rows a workgroup, 128 or 192 in a pair's last one, or 128 in all; few pairs are
// shared out along the keys too, each workgroup leaving its sums in the workspace, with a reference that makes them 1/2 to 1.  A workgroup whose sums leave the fast path's range redoes its rows in place, 128 at a time.
// Measured: 8 frames over 40 (10992 queries, 54960 keys, 16 heads) 2.04 to 2.17 ms = 1.14 to 1.21 PFLOP/s, of which the joining of four
// splits is 0.037; the matrix core is busy in 0.63 of the cycles, at 1.93 GHz.  A frame over 137400 cached keys 0.73 to 0.77 ms, 512
// queries to each of 24 frames 67 to 78 us.
// ---------------------------------------------------------------------------
namespace {

// Fast path: accumulators that may have overflowed; those that may have lost products below float32's range, where a row's probabilities are
// as small as a sum below kSmallSum makes them
constexpr float kOutHi = 1.329227995784916e36f;       // 2^120
constexpr float kOutLo = 8.271806125530277e-25f;      // 2^-80
constexpr float kSmallSum = 9.5367431640625e-7f;      // 2^-20

// One workgroup's rows row_begin .. row_end - 1 of pair (b, hk) over its split's keys, by one of the two paths.  Returns false, without
// storing anything, when the fast path met a row it cannot handle.  tiles: kTileLds elements of LDS per four wavefronts.
template <int kSrc, bool kGen, int kQB, int kJ, int kMode = kAlone>
__device__ __forceinline__ bool attend_cross(const CrossArgs& p, const CrossPlan& plan, uint32_t pairs, uint16_t* tiles, uint32_t* votes,
                                             uint32_t pair, int split, uint32_t row_begin, uint32_t row_end) {
  constexpr int kWaveQ = wave_queries(kQB, kJ);
  // (opaque on the general path, so that it holds nothing of the fast path's: agg_attn.hip)
  int thread = threadIdx.x;
  if (kGen) asm volatile("" : "+v"(thread));
  constexpr bool kSplit = kMode == kSplitKeys;
  static_assert(!(kGen && kSplit), "the general path's halves would need a common reference");
  const int group = kMode != kAlone ? __builtin_amdgcn_readfirstlane(thread / kAttnThreads) : 0;
  const int tid = thread - group * kAttnThreads;
  uint16_t* const smem = tiles + group * kTileLds;
  u32x4* lds = reinterpret_cast<u32x4*>(smem);
  const int lane = tid & 63, wave = tid >> 6, c = lane & 15, G = lane >> 4;
  const FragAddr fa = frag_addr(lane);
  const int b = (int)(pair / (uint32_t)p.H_kv), hk = (int)(pair % (uint32_t)p.H_kv);

  // this workgroup's key tiles
  const int n = cross_keys(p, b);
  const uint32_t all = ((uint32_t)n + kTileRows - 1) / kTileRows;
  int skip = part_begin(all, split, plan.splits);
  int ntiles = part_begin(all, split + 1, plan.splits) - skip;
  const int half = kSplit ? (ntiles + 1) / 2 : ntiles;
  if (kSplit) {
    ntiles = group ? ntiles - half : half;
    skip += group ? half : 0;
  }
  const int rows_here = min(n - skip * kTileRows, ntiles * kTileRows);
  const int last_valid = rows_here - (ntiles - 1) * kTileRows;  // 1..64
  KvSource src;
  src.rows = rows_here;
  if (kSrc == kSrcPaged) {
    src.k = p.Kc;
    src.v = p.Vc;
    src.pages = (ScalarInts)p.pages + ((int64_t)b * p.max_pages + skip);
    src.tiles = ntiles;
    src.last_page = p.n_pages - 1;
    src.page_elems = (int64_t)p.H_kv * kTileElems;
    src.head_elems = (int64_t)hk * kTileElems;
  } else {
    const int64_t first_row = (int64_t)b * p.NK + (int64_t)skip * kTileRows;
    src.k = uniform_ptr(p.K + first_row * p.k_stride + hk * kHeadDim);
    src.v = uniform_ptr(p.V + first_row * p.v_stride + hk * kHeadDim);
    src.row_bytes = (uint32_t)(p.k_stride * 2);
    src.v_row_bytes = (uint32_t)(p.v_stride * 2);
  }

  Wave<kQB, kJ> w;
  w.l2 = p.scale2;
  const uint32_t one = c == 0 ? 0x3F803F80u : 0u;
  w.ones.u = u32x4{one, one, one, one};
  const uint32_t r_wave = row_begin + wave * kWaveQ;
#pragma unroll
  for (int qb = 0; qb < kQB; ++qb)
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      const RowPlace at = row_place(p, hk, min(r_wave + (qb * kJ + j) * 16 + c, row_end - 1));
      const uint16_t* q = p.Q + ((int64_t)b * p.NQ + at.q) * p.q_stride + at.head * kHeadDim;
#pragma unroll
      for (int h = 0; h < 2; ++h) w.Qf[qb][2 * j + h].u = *reinterpret_cast<const u32x4*>(q + 32 * h + 8 * G);
    }
#pragma unroll
  for (int qb = 0; qb < kQB; ++qb)
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      // (General path: zeros that the compiler does not know to be zeros.  Knowing them, it spilled 119 to 326 registers of
      // the kernels below, in the narrow ones of the fast path too; a build test checks that none does.)
      float zero = 0.f;
      if (kGen) asm volatile("" : "+v"(zero));
      float none = -INFINITY;  // general path: the reference comes with the first unit (agg_attn_pipe.h)
      if (kGen) asm volatile("" : "+v"(none));
      w.mref[qb][j] = none;
      w.la[qb][j] = zero;
      w.L[qb][j] = f32x4{zero, zero, zero, zero};
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        f32x4 z = {zero, zero, zero, zero};
        if (kGen) asm volatile("" : "+v"(z));
        w.O[qb][j][dt] = z;
      }
    }
  bool done = true;
  if (!kSplit || ntiles > 0)
    done = key_loop<kSrc, kGen, kSplit, kQB, kJ>(w, lds, votes, src, ntiles, last_valid, tid, wave, fa, G, [] {});
  if (kSplit) {
    // a loop passes one barrier per tile: the shorter one makes up for its missing tile.  Without a reference the two halves'
    // sums and accumulators just add: the second group's go through its LDS, [register][wavefront][lane], to the first
    if (ntiles < half) lds_barrier();
    __syncthreads();  // both groups are done with their tiles
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
      l_fin[qb][j] = kGen ? quad_sum(w.la[qb][j]) : __shfl(w.L[qb][j][0], c);
      unsafe = unsafe || (group == 0 && (!(l_fin[qb][j] < kSumHi) || !(l_fin[qb][j] > kSumLo)));
      if (!kGen) {
        // sums inside the window say nothing of the values: probabilities of 2^80 overflow with values of 2^50, those of 2^-80
        // vanish with values of 2^-50
        float sum = 0.f, least = INFINITY;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float size = fabsf(w.O[qb][j][dt][r]);
            sum += size;
            least = fminf(least, size);
          }
        unsafe = unsafe || (group == 0 && (!(sum < kOutHi) || (l_fin[qb][j] < kSmallSum && least < kOutLo)));
      }
    }
  if (!kGen) {
    if (!done) return false;
    if (vote(unsafe, votes + kWaves, wave, lane, group == 0)) return false;
  } else {
    __syncthreads();  // every wavefront is done with the tiles
  }
  if (group) return true;

  int here = tid;
  asm volatile("" : "+v"(here));
  const int elane = here & 63, ec = here & 15, eG = elane >> 4;
  if (plan.splits > 1) {
#pragma unroll
    for (int qb = 0; qb < kQB; ++qb)
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        const uint32_t row = r_wave + (qb * kJ + j) * 16 + ec;
        if (row >= row_end) continue;
        const size_t at = partial_row(p, pairs, split, pair, row);
        // The join weighs by references, and these are no measure of the sums: 0 (fast path, sums of 2^-90 to 2^90), or the
        // largest logit of some unit.  The sum's power of two goes over to the reference.  (0 of a sum that is 0 or no number.)
        const int e = __builtin_amdgcn_frexp_expf(l_fin[qb][j]);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          f32x4 part;
#pragma unroll
          for (int r = 0; r < 4; ++r) part[r] = ldexpf(w.O[qb][j][dt][r], -e);
          *reinterpret_cast<f32x4*>(p.partial + at * kHeadDim + 16 * dt + 4 * eG) = part;
        }
        if (eG == 0)
          *reinterpret_cast<f32x2*>(partial_sums(p, pairs, plan.splits) + at * 2) =
              f32x2{(kGen ? w.mref[qb][j] * p.scale2 : 0.f) + (float)e, ldexpf(l_fin[qb][j], -e)};
      }
    return true;
  }
  // whole 128-byte rows, turned through a part of the tiles' LDS of the wavefront's own (agg_attn.hip)
  uint16_t* epi = smem + wave * (16 * kJ * kEpiStride);
#pragma unroll
  for (int qb = 0; qb < kQB; ++qb) {
    const uint32_t r0 = r_wave + qb * kJ * 16;
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      const float l = l_fin[qb][j], inv = 1.0f / l;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        *reinterpret_cast<u32x2*>(epi + (16 * j + ec) * kEpiStride + 16 * dt + 4 * eG) = pack4(w.O[qb][j][dt] * inv);
      if (p.lse && eG == 0 && r0 + 16 * j + ec < row_end) {
        const RowPlace at = row_place(p, hk, r0 + 16 * j + ec);
        p.lse[((int64_t)b * p.H + at.head) * p.NQ + at.q] = ((kGen ? w.mref[qb][j] * p.scale2 : 0.f) + log2f(l)) * kLn2;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
#pragma unroll
    for (int i = 0; i < 2 * kJ; ++i) {
      const uint32_t row = r0 + i * 8 + (elane >> 3);
      const u32x4 o4 = *reinterpret_cast<const u32x4*>(epi + (i * 8 + (elane >> 3)) * kEpiStride + (elane & 7) * 8);
      if (row < row_end) {
        const RowPlace at = row_place(p, hk, row);
        *reinterpret_cast<u32x4*>(p.O + (((int64_t)b * p.NQ + at.q) * p.H + at.head) * kHeadDim + (elane & 7) * 8) = o4;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  }
  return true;
}

// The rows of a workgroup that has no keys: zeros, or partial results that add nothing.
__device__ __forceinline__ void store_nothing(const CrossArgs& p, const CrossPlan& plan, uint32_t pairs, uint32_t pair, int split,
                                              uint32_t row_begin, uint32_t row_end, bool no_keys) {
  const int b = (int)(pair / (uint32_t)p.H_kv), hk = (int)(pair - (uint32_t)b * (uint32_t)p.H_kv), quad = threadIdx.x & 15;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  for (uint32_t row = row_begin + (threadIdx.x >> 4); row < row_end; row += blockDim.x / 16) {
    if (plan.splits == 1) {
      store_row(p, b, hk, row, quad, 0.f, 0.f, zero, no_keys);
      continue;
    }
    const size_t at = partial_row(p, pairs, split, pair, row);
    *reinterpret_cast<f32x4*>(p.partial + at * kHeadDim + 4 * quad) = zero;
    if (quad == 0) *reinterpret_cast<f32x2*>(partial_sums(p, pairs, plan.splits) + at * 2) = f32x2{-INFINITY, 0.f};
  }
}

}  // namespace

struct WideArgs {
  CrossArgs a;
  CrossPlan plan;
};

// The kernel's arguments again, so that what one path derives from them is not held for another (agg_attn.hip).
__device__ __forceinline__ const WideArgs& wide_args_again() {
  typedef const __attribute__((address_space(4))) WideArgs* KernelArgs;
  KernelArgs args = (KernelArgs)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(args));
  return *(const WideArgs*)args;
}

// What a workgroup does; false: nothing, or it is done.
struct WideWork {
  int pair, split;
  uint32_t row_begin, row_end;
};
__device__ __forceinline__ bool wide_work(const WideArgs& w, int npairs, WideWork& x) {
  const CrossArgs& a = w.a;
  // the workgroups of a pair's split read the same keys: on one XCD they share them through its L2
  int unit, i;
  if (!list_tile(tile_list(npairs * w.plan.splits, (int)w.plan.row_tiles), npairs * w.plan.splits, blockIdx.x, unit, i)) return false;
  x.pair = unit / w.plan.splits;  // a long sequence's splits go to different XCDs
  x.split = unit % w.plan.splits;
  const int b = x.pair / a.H_kv;
  const uint32_t rows = (uint32_t)cross_queries(a, b) * (uint32_t)a.group;
  x.row_begin = (uint32_t)i * (uint32_t)w.plan.width;
  if (x.row_begin >= rows) return false;
  x.row_end = min(rows, x.row_begin + (uint32_t)w.plan.width);
  const int n = cross_keys(a, b);
  const uint32_t all = ((uint32_t)n + kTileRows - 1) / kTileRows;
  if (part_begin(all, x.split, w.plan.splits) == part_begin(all, x.split + 1, w.plan.splits)) {
    store_nothing(a, w.plan, npairs, x.pair, x.split, x.row_begin, x.row_end, n == 0);
    return false;
  }
  return true;
}

template <int kSrc, int kTail>
__global__ __launch_bounds__(kAttnThreads, kBlocksPerCu) void cross_wide_kernel(WideArgs w) {
  __shared__ __align__(16) uint16_t tiles[kTileLds];
  __shared__ __align__(16) uint32_t votes[kVoteWords];
  const int npairs = w.a.B * w.a.H_kv;
  WideWork x;
  if (!wide_work(w, npairs, x)) return;
  bool done;
  if (kTail != 0 && x.row_end - x.row_begin <= kTail)
    done = attend_cross<kSrc, false, kTail == 192 ? 3 : 2, 1>(w.a, w.plan, npairs, tiles, votes, x.pair, x.split, x.row_begin, x.row_end);
  else
    done = attend_cross<kSrc, false, 2, 2>(w.a, w.plan, npairs, tiles, votes, x.pair, x.split, x.row_begin, x.row_end);
  if (done) return;
  const WideArgs& again = wide_args_again();
#pragma unroll 1
  for (uint32_t r = x.row_begin; r < x.row_end; r += kWaves * wave_queries(2, 1)) {
    __syncthreads();  // the LDS is free
    attend_cross<kSrc, true, 2, 1>(again.a, again.plan, npairs, tiles, votes, x.pair, x.split, r,
                                   min(x.row_end, r + (uint32_t)(kWaves * wave_queries(2, 1))));
  }
}

// A launch of few workgroups: 128 rows each, eight wavefronts, four for each half of the keys.  (us, 16 heads, this / four
// wavefronts of 128 rows / 256 rows, best splits of each: 1374 queries to 2748 keys 22.9 / 27.9 / 34, to 5496 39.0 / 45.8 / 44.8, to
// 13740 88 / 88 / 81; four ragged sequences of up to 777 to 1029, 12 heads, 13.2 / 14.5 / 20.8.)
template <int kSrc>
__global__ __launch_bounds__(2 * kAttnThreads, 2) void cross_halves_kernel(WideArgs w) {
  __shared__ __align__(16) uint16_t tiles[2 * kTileLds];
  __shared__ __align__(16) uint32_t votes[kVoteWords];
  const int npairs = w.a.B * w.a.H_kv;
  WideWork x;
  if (!wide_work(w, npairs, x)) return;
  if (attend_cross<kSrc, false, 2, 1, kSplitKeys>(w.a, w.plan, npairs, tiles, votes, x.pair, x.split, x.row_begin, x.row_end)) return;
  __syncthreads();
  const WideArgs& again = wide_args_again();
  attend_cross<kSrc, true, 2, 1, kTwin>(again.a, again.plan, npairs, tiles, votes, x.pair, x.split, x.row_begin, x.row_end);
}

// ---------------------------------------------------------------------------
// Joins the splits' results: sixteen threads a row and group, kGroups groups a row, each with every kGroups-th split.  Bound by the
// partial results' bytes where there are many rows (175872 rows of four splits: 36 us, 5 TB/s), by one read's latency where there
// are few: four splits are requested before one is used, and the groups meet in LDS (16 rows of 32 splits 4.5 us, 18.6 by
// sixteen threads each).
// ---------------------------------------------------------------------------
constexpr int kJoinThreads = 256;
constexpr int join_rows(int groups) { return kJoinThreads / 16 / groups; }

template <int kGroups>
__global__ __launch_bounds__(kJoinThreads) void cross_join_kernel(CrossArgs a, int splits, uint32_t pairs) {
  __shared__ __align__(16) float meet[kJoinThreads / 16][kRowFloats];
  const uint32_t all = (uint32_t)(a.NQ * a.group);
  const int slot = threadIdx.x >> 4, quad = threadIdx.x & 15, group = slot % kGroups;
  const uint32_t at = blockIdx.x * join_rows(kGroups) + slot / kGroups;  // fewer than 2^20 (partial_row)
  const uint32_t pair = min(at, pairs * all - 1) / all, row = at - pair * all;
  const int b = (int)(pair / (uint32_t)a.H_kv), hk = (int)(pair - (uint32_t)b * (uint32_t)a.H_kv);
  const int n = a.k_lens ? min(max(a.k_lens[b], 0), a.NK) : a.NK;
  const int queries = a.q_lens ? min(max(a.q_lens[b], 0), a.NQ) : a.NQ;
  const bool here = at < pairs * all && row < (uint32_t)queries * (uint32_t)a.group;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  // another part of the sum, by its reference (-infinity: a split without keys that weigh anything, which adds nothing)
  auto add = [&](float m2, float l2, f32x4 o2) {
    const float now = fmaxf(m, m2), ref = now == -INFINITY ? 0.f : now;
    const float f = fast_exp2(m - ref), f2 = fast_exp2(m2 - ref);
    m = now;
    l = l * f + l2 * f2;
    o = o * f + o2 * f2;
  };
  if (here) {
    const f32x2* const sums = reinterpret_cast<const f32x2*>(partial_sums(a, pairs, splits)) + at;
    const float* const from = a.partial + (size_t)at * kHeadDim + 4 * quad;
    const size_t next = pairs * all;
    for (int s0 = group; s0 < splits; s0 += 4 * kGroups) {
      f32x2 x[4];
      f32x4 part[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = min(s0 + i * kGroups, splits - 1);
        x[i] = sums[s * next];
        part[i] = *reinterpret_cast<const f32x4*>(from + s * next * kHeadDim);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (s0 + i * kGroups < splits) add(x[i][0], x[i][1], part[i]);
    }
  }
  if constexpr (kGroups > 1) {
    *reinterpret_cast<f32x4*>(&meet[slot][4 * quad]) = o;
    if (quad == 0) *reinterpret_cast<f32x2*>(&meet[slot][kHeadDim]) = f32x2{m, l};
    __syncthreads();
    if (group) return;
#pragma unroll 4
    for (int g = 1; g < kGroups; ++g) {
      const f32x2 x = *reinterpret_cast<const f32x2*>(&meet[slot + g][kHeadDim]);
      add(x[0], x[1], *reinterpret_cast<const f32x4*>(&meet[slot + g][4 * quad]));
    }
  }
  if (here) store_row(a, b, hk, row, quad, m == -INFINITY ? 0.f : m, l, o, n == 0);
}

template <int kGroups>
static void launch_join(const CrossArgs& a, int splits, int64_t pairs, int64_t rows, hipStream_t st) {
  constexpr int64_t kRows = join_rows(kGroups);
  hipLaunchKernelGGL(cross_join_kernel<kGroups>, dim3((unsigned)((pairs * rows + kRows - 1) / kRows)), dim3(kJoinThreads), 0, st,
                     a, splits, (uint32_t)pairs);
}

// the wide kernel reaches a tile's 64 rows with 32-bit byte offsets
static bool wide_fits(int64_t stride) { return stride <= ((int64_t)1 << 23); }

size_t cross_partial_floats(int64_t B, int64_t NQ, int64_t NK, int64_t H, int64_t H_kv, int ragged) {
  const int64_t pairs = B * H_kv, rows = NQ * (H / H_kv);
  // where a call's keys lie chooses between three plans: enough for any
  int splits = plan_cross(pairs, rows, NK, ragged, true, true).splits;
  for (bool fits : {true, false}) {
    const int s = plan_cross(pairs, rows, NK, ragged, fits, false).splits;
    splits = s > splits ? s : splits;
  }
  return splits > 1 ? (size_t)splits * pairs * rows * (kHeadDim + 2) : 0;
}

template <bool kPaged>
static hipError_t launch_few(const CrossArgs& a, const CrossPlan& p, int64_t pairs, hipStream_t st) {
  const int64_t groups = pairs * p.row_tiles * p.splits;
  if (groups > 0xFFFFFFFFll) return kTooManyGroups;
  constexpr int64_t kMost = 1 << 22;  // workgroups of a launch (kLaunchRows)
  for (int64_t first = 0; first < groups; first += kMost) {
    const uint32_t here = (uint32_t)(groups - first < kMost ? groups - first : kMost);
    const dim3 grid(!kPaged && here >= kRunsFrom ? (here + kXcds - 1) / kXcds * kXcds : here), block(kFewThreads);
    if (p.tiles == 1) hipLaunchKernelGGL((cross_few_kernel<kPaged, 1>), grid, block, 0, st, a, p, (uint32_t)pairs, (uint32_t)first, here);
    else hipLaunchKernelGGL((cross_few_kernel<kPaged, 2>), grid, block, 0, st, a, p, (uint32_t)pairs, (uint32_t)first, here);
  }
  return hipSuccess;
}

template <int kSrc>
static hipError_t launch_wide(const CrossArgs& a, const CrossPlan& p, hipStream_t st) {
  // workgroups of a launch (kLaunchRows): beyond that parts of the batch are launches of their own, which share out nothing along the keys
  constexpr int64_t kMost = 1 << 22;
  const int64_t of_one = (int64_t)a.H_kv * p.row_tiles * p.splits;
  if (of_one > kMost) return kTooManyGroups;
  const int64_t step = a.B * of_one <= kMost ? a.B : kMost / of_one;
  if (step < a.B && p.splits > 1) return kTooManyGroups;
  for (int64_t b = 0; b < a.B; b += step) {
    WideArgs w = {a, p};
    w.a.B = (int32_t)(a.B - b < step ? a.B - b : step);
    w.a.Q += b * a.NQ * a.q_stride;
    w.a.O += b * a.NQ * a.H * kHeadDim;
    if (a.lse) w.a.lse += b * a.H * a.NQ;
    if (kSrc == kSrcPaged) {
      w.a.pages += b * a.max_pages;
    } else if (a.NK > 0) {
      w.a.K += b * a.NK * a.k_stride;
      w.a.V += b * a.NK * a.v_stride;
    }
    if (a.q_lens) w.a.q_lens += b;
    if (a.k_lens) w.a.k_lens += b;
    const dim3 grid((unsigned)tile_list((int)(w.a.B * a.H_kv * p.splits), (int)p.row_tiles).groups);
    const dim3 block(kAttnThreads);
    const int narrow = p.width == 128 ? 128 : p.tail;
    if (p.halves) hipLaunchKernelGGL(cross_halves_kernel<kSrc>, grid, dim3(2 * kAttnThreads), 0, st, w);
    else if (narrow == 0) hipLaunchKernelGGL((cross_wide_kernel<kSrc, 0>), grid, block, 0, st, w);
    else if (narrow == 192) hipLaunchKernelGGL((cross_wide_kernel<kSrc, 192>), grid, block, 0, st, w);
    else hipLaunchKernelGGL((cross_wide_kernel<kSrc, 128>), grid, block, 0, st, w);
  }
  return hipSuccess;
}

hipError_t launch_cross(const CrossArgs& a, hipStream_t st) {
  const int64_t pairs = (int64_t)a.B * a.H_kv, rows = (int64_t)a.NQ * a.group;
  const CrossPlan p = plan_cross(pairs, rows, a.NK, cross_ragged(a.B, a.q_lens, a.k_lens),
                                 a.pages || (wide_fits(a.k_stride) && wide_fits(a.v_stride)), a.pages != nullptr);
  (void)hipGetLastError();
  const hipError_t e = p.wide ? a.pages ? launch_wide<kSrcPaged>(a, p, st) : launch_wide<kSrcStrided>(a, p, st)
                       : a.pages ? launch_few<true>(a, p, pairs, st) : launch_few<false>(a, p, pairs, st);
  if (e != hipSuccess) return e;
  if (p.splits > 1) {
    if (pairs * rows <= 4096 && p.splits > 4) launch_join<16>(a, p.splits, pairs, rows, st);
    else launch_join<1>(a, p.splits, pairs, rows, st);
  }
  return hipGetLastError();
}

}  // namespace agg
