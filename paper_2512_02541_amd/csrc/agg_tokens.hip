// The token-wise parts of a model's block: query/key normalisation with rotary positions, and the
// seam between one branch and the next (norm, gate, residual scale, sum, norm).  Both are single passes
// whose bound is HBM: every row is read once, held in registers in float32 and written once.
#include "agg_internal.h"
#include "agg_lds_copy.h"
#include "agg_stream.h"

namespace agg {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

__device__ inline uint32_t pack2(float lo, float hi) {
  f32x2 p = {lo, hi};
  bf16x2 h = __builtin_convertvector(p, bf16x2);
  return __builtin_bit_cast(uint32_t, h);
}
__device__ inline u32x4 pack8(const float (&v)[8]) {
  return u32x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
}
__device__ inline void unpack8(u32x4 w, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
// eight float parameters of the channels from `at` on, `other` where there are none
__device__ inline void load8(const float* p, int at, float other, float (&v)[8]) {
  f32x4 a = {other, other, other, other}, b = a;
  if (p) {
    a = *reinterpret_cast<const f32x4*>(p + at);
    b = *reinterpret_cast<const f32x4*>(p + at + 4);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}

// the sum over eight neighbouring lanes, in all of them: two exchanges within four lanes, one between them
__device__ inline float sum_of_8(float v) {
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, true));   // lane ^ 1
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, true));   // lane ^ 2
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xF, 0xF, true));  // 7 - lane
  return v;
}

// ... over the wavefront
__device__ inline float sum_of_wave(float v) {
  v = sum_of_8(v);
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xF, 0xF, true));  // 15 - lane
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// orders a wavefront's LDS writes before its own later reads
__device__ inline void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

}  // namespace

// ---------------------------------------------------------------------------
// Rotary positions behind an optional norm, per head.  Eight lanes hold a head, eight channels each;
// a wavefront takes `tokens` tokens at a time, its eight groups of lanes their heads in turn, queries
// and keys together.  The cosines and sines of a token are worked out once per wavefront, a pair of channels a lane, and
// passed to all heads through LDS.  The angle of a pair in turns is position * frequency
// modulo 1: a 64-bit product of the position and the frequency in units of 2^-64 turns wraps to
// exactly that.  A pair's other channel comes out of LDS too, which serves every pairing alike.
// Bound by HBM once enough is under way: a round's rows are requested before the one in hand is worked on, and awaited at
// its end together with its stores (the accesses are conditional, so the compiler counts none of them apart); four
// wavefronts on a SIMD cover that.
// Measured (16 frames of 16 heads with a LayerNorm, 180 MB / 100 frames with RMS and given positions, 1.13 GB): 49 / 323 us
// when rows were requested in their own round and sums went through LDS; 38 / 223 without that; 34 / 207 (5.4 TB/s) with a
// table of cosine and signed sine per channel, whose reads stand in front of their uses.  One frame of 261 tokens of 8 heads
// 4.1 us each of many in a graph, 5.1 to 5.4 alone; a copy in this form takes 2.9: the parameters' loads, the rows' and
// the positions' wait for each other in front of the first round.
// Outputs are stored past the caches at every size: 2 frames of 16 heads 7.9 us, 8.9 through them, 100 frames 210 and 217;
// with the per-frame attention behind it 33.0 and 34.6 (1 frame of 8 heads 12.0 and 11.6, 8 frames 82 and 80), blocks of
// 1 to 16 frames the same within 1 %.
// ---------------------------------------------------------------------------
constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / 64;
constexpr int kRopeMaxTokens = 8;            // of a wavefront's turn
constexpr int kRopePairs = kHeadDim / 2;
constexpr int kHeadStride = kHeadDim + 4;    // floats of a head in LDS: 16-byte aligned rows

template <bool kShared>
__global__ __launch_bounds__(kRopeThreads, 4) void rope_kernel(RopeArgs a) {
  __shared__ __align__(16) float heads[kRopeWaves][8][kHeadStride];
  __shared__ __align__(16) f32x2 turns[kRopeWaves][kRopeMaxTokens][kHeadDim];  // of a channel: cosine, signed sine
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int group = lane >> 3, c0 = (lane & 7) * 8;  // this lane's head among eight, its first channel
  const int H = a.H;

  // each channel's other one, and whether it turns at all
  int other[8];
  uint32_t turned = 0;
  const bool all_turn = a.pairs == kRopePairs;
  if (a.pairs) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      other[i] = a.other[c0 + i] & 63;
      if (a.other[c0 + i] & 0x80) turned |= 1u << i;
    }
    // channels that no pair writes
    for (int i = 0; i < a.tokens; ++i) turns[wave][i][lane] = f32x2{1.f, 0.f};
  }
  float g[2][8], b[2][8];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    load8(a.norm[t].gamma, c0, 1.f, g[t]);
    load8(a.norm[t].beta, c0, 0.f, b[t]);
  }
  float* const head = heads[wave][group];

  // kShared: several wavefronts share a turn's heads, or one takes the queries and one the keys; one turn each
  int64_t first = (int64_t)blockIdx.x * kRopeWaves + wave;
  int h0 = group % H, sub0 = group / H;
  int skip = -1;  // the tensor that is another wavefront's
  if constexpr (kShared) {
    const uint32_t sharing = a.parts * a.ways, item = (uint32_t)first;
    first = item / sharing;
    const int part = (int)(item % sharing) / a.ways;
    if (a.ways == 2) skip = ~item & 1;
    h0 = (part * 8 + group) % H;
    sub0 = (part * 8 + group) / H;
  }
  const int next = kShared ? 8 * a.parts : 8;
  const int64_t step = (int64_t)gridDim.x * kRopeWaves * a.tokens;
  for (int64_t t0 = first * a.tokens; t0 < a.total; t0 += step) {
    const int here = (int)min((int64_t)a.tokens, a.total - t0);
    // a turn's heads, eight at a time; a round's rows are requested while the one before is worked on
    int h = h0, sub = sub0;
    u32x4 ahead[2];
    auto request = [&]() {
      if (sub < here)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (a.in[t] && (!kShared || t != skip))
            ahead[t] = *reinterpret_cast<const u32x4*>(a.in[t] + (t0 + sub) * a.stride[t] + h * kHeadDim + c0);
    };
    request();
    if (a.pairs) {
      wave_lds_fence();  // the last turn's reads are done
      for (int i = lane; i < here * kRopePairs; i += 64) {
        const int p = i % kRopePairs, of = i / kRopePairs;
        if (p < a.pairs) {
          const int64_t tok = t0 + of;
          const int axis = a.axis[p];
          int32_t pos;
          if (a.pos) {
            pos = a.pos[tok * 3 + axis];
          } else {
            // < 2^31; a 64-bit division only where the token's number needs it
            const uint32_t in_seq = a.total >> 32 ? (uint32_t)(tok % a.NQ) : (uint32_t)tok % (uint32_t)a.NQ;
            const uint32_t frame = in_seq / (uint32_t)a.L;
            const int32_t patch = (int32_t)(in_seq % (uint32_t)a.L) - a.P;
            if (axis == 0) pos = a.t0 + (int32_t)frame;
            else if (patch < 0) pos = 0;
            else pos = a.patch0 + (axis == 1 ? patch / a.n_w : patch % a.n_w);
          }
          const uint64_t phase = (uint64_t)(int64_t)pos * a.freq[p];
          // the signed high half: a turn is 2^32, half a turn 2^31
          float s, c;
          sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &s, &c);
          turns[wave][of][a.first[p]] = f32x2{c, -s};
          turns[wave][of][a.second[p]] = f32x2{c, s};
        }
      }
      wave_lds_fence();
    }
    while (sub < here) {
      u32x4 raw[2] = {ahead[0], ahead[1]};
      const int at_h = h, at_sub = sub;
      h += next;
      while (h >= H) {
        h -= H;
        ++sub;
      }
      request();
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (!a.in[t] || (kShared && t == skip)) continue;
        float x[8];
        unpack8(raw[t], x);
        const int kind = a.norm[t].kind;
        if (kind != AGG_NORM_NONE) {
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
          const float r = rsqrtf(sum_of_8(sq) * (1.f / kHeadDim) + a.norm[t].eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = x[i] * r * g[t][i] + b[t][i];
        }
        if (a.pairs) {
          wave_lds_fence();
          *reinterpret_cast<f32x4*>(head + c0) = f32x4{x[0], x[1], x[2], x[3]};
          *reinterpret_cast<f32x4*>(head + c0 + 4) = f32x4{x[4], x[5], x[6], x[7]};
          wave_lds_fence();
          float y[8];
          f32x4 cs[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) cs[i] = *reinterpret_cast<const f32x4*>(&turns[wave][at_sub][c0 + 2 * i]);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = head[other[i]];
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = x[i] * cs[i / 2][i % 2 * 2] + y[i] * cs[i / 2][i % 2 * 2 + 1];
          if (all_turn) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = y[i];
          } else {  // by selection: an infinity times 0 is none of the other channels' business
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (turned >> i) & 1 ? y[i] : x[i];
          }
        }
        __builtin_nontemporal_store(
            pack8(x), reinterpret_cast<u32x4*>(a.out[t] + ((t0 + at_sub) * H + at_h) * kHeadDim + c0));
      }
    }
  }
}

hipError_t launch_rope(const RopeArgs& args, hipStream_t st) {
  RopeArgs a = args;
  // two tokens a turn fill the lanes that work out the angles; few tokens are spread over more wavefronts
  a.tokens = a.H < 4 ? kRopeMaxTokens / a.H : a.total <= 4096 ? 1 : 2;
  const int64_t turns = (a.total + a.tokens - 1) / a.tokens;
  // Few turns: a round costs a wavefront 0.6 to 1 us whatever runs beside it, so its heads are shared out, then queries and
  // keys too, while all wavefronts still run at once (four on a SIMD).  us with a LayerNorm, shared / not: 1 token of 16
  // heads 3.9 / 5.3, 261 of 8 4.0 / 4.4, of 16 4.3 / 5.7, 1374 of 16 6.5 / 6.9; beyond: 2748 of 16 8.8 / 7.9, 5496 12.0 / 11.5
  constexpr int kAtOnce = 256 * 4 * 4;
  a.parts = a.ways = 1;
  while (a.parts * 8 < a.tokens * a.H && turns * a.parts * 2 <= kAtOnce) a.parts *= 2;
  if (a.in[0] && a.in[1] && turns * a.parts * 2 <= kAtOnce) a.ways = 2;
  const int64_t groups = (turns * a.parts * a.ways + kRopeWaves - 1) / kRopeWaves;
  const dim3 grid((unsigned)(groups < 4096 ? groups : 4096));
  (void)hipGetLastError();
  const auto kernel = a.parts * a.ways > 1 ? rope_kernel<true> : rope_kernel<false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kRopeThreads), 0, st, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// h = x + gate * scale * post(branch),  n = pre(h).  A row is in registers in float32, statistics as in
// layernorm_kernel (mean, then variance of the centred values); norms' parameters stay in registers
// from row to row, and the next row is requested before the present one is worked on (and awaited behind that one's stores,
// as in rope_kernel).
// Rows of up to 1024 channels: one wavefront each, kPer 16-byte chunks a lane.  Few longer ones: the
// whole workgroup, of as many wavefronts as the row fills, whose sums meet in LDS.
// HBM-bound: 21 984 rows of 1024 with layer scale and LayerNorm 28 to 29 us (180 MB, much of it in the cache where a loop
// repeats the call; 35 on other tensors each time), 137 400 rows 200 (5.6 TB/s); one row 2.5 us alone, 3.3 each of many in a graph.
// ---------------------------------------------------------------------------
namespace {

// what a norm multiplies by and adds, of this thread's channels
template <int kPer>
struct SeamParams {
  float gamma[kPer][8], beta[kPer][8];
};

template <int kPer, bool kAcross>
struct SeamRow {
  float v[kPer][8];
  // the sum over the row; kAcross: over the workgroup's wavefronts too (`turn` alternates the slots, so that one
  // barrier a sum is enough: a slot is written again only behind the next sum's barrier)
  __device__ static inline float total(float x, float (*slots)[8], int& turn, int waves) {
    x = sum_of_wave(x);
    if constexpr (kAcross) {
      if ((threadIdx.x & 63) == 0) slots[turn][threadIdx.x >> 6] = x;
      lds_barrier();  // (of LDS alone: the next row's loads stay under way)
      float all = 0.f;
      for (int w = 0; w < waves; ++w) all += slots[turn][w];
      x = all;
      turn ^= 1;
    }
    return x;
  }
  __device__ inline void norm(const SeamNorm& n, const SeamParams<kPer>& p, const bool (&has)[kPer], float inv_c,
                              float (*slots)[8], int& turn, int waves) {
    float mean = 0.f;
    if (n.kind == AGG_NORM_LAYER) {
#pragma unroll
      for (int c = 0; c < kPer; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) mean += v[c][i];
      mean = total(mean, slots, turn, waves) * inv_c;
    }
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < kPer; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[c][i] = has[c] ? v[c][i] - mean : 0.f;
        sq += v[c][i] * v[c][i];
      }
    const float r = rsqrtf(total(sq, slots, turn, waves) * inv_c + n.eps);
#pragma unroll
    for (int c = 0; c < kPer; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * r * p.gamma[c][i] + p.beta[c][i];
  }
};

}  // namespace

template <int kPer, bool kAcross, bool kStream>
__global__ __launch_bounds__(kAcross ? 512 : 256) void seam_kernel(SeamArgs a) {
  __shared__ float slots[2][8];
  const int waves = blockDim.x >> 6;
  const int at = kAcross ? threadIdx.x : threadIdx.x & 63;  // this thread among those of a row
  const int nchunk = a.C / 8;
  const float inv_c = 1.f / (float)a.C;
  bool has[kPer];
  int off[kPer];  // of this thread's chunks; the missing ones read the row's first
#pragma unroll
  for (int c = 0; c < kPer; ++c) {
    const int ch = at + c * (kAcross ? (int)blockDim.x : 64);
    has[c] = ch < nchunk;
    off[c] = has[c] ? ch * 8 : 0;
  }
  SeamParams<kPer> post, pre;
  float scale[kPer][8];
#pragma unroll
  for (int c = 0; c < kPer; ++c) {
    load8(a.post.gamma, off[c], 1.f, post.gamma[c]);
    load8(a.post.beta, off[c], 0.f, post.beta[c]);
    load8(a.pre.gamma, off[c], 1.f, pre.gamma[c]);
    load8(a.pre.beta, off[c], 0.f, pre.beta[c]);
    load8(a.scale, off[c], 1.f, scale[c]);
  }
  const int64_t first = kAcross ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t step = kAcross ? (int64_t)gridDim.x : (int64_t)gridDim.x * 4;
  u32x4 xr[kPer], br[kPer], gr[kPer];
  auto request = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < kPer; ++c) {
      xr[c] = load16<kStream>(a.x + row * a.C + off[c]);
      if (a.branch) br[c] = load16<kStream>(a.branch + row * a.C + off[c]);
      if (a.gate)  // rows < 2^31 and gate_rows <= 2^31
        gr[c] = *reinterpret_cast<const u32x4*>(a.gate + (int64_t)((uint32_t)row / (uint32_t)a.gate_rows) * a.C + off[c]);
    }
  };
  int turn = 0;
  if (first < a.rows) request(first);
  for (int64_t row = first; row < a.rows; row += step) {
    SeamRow<kPer, kAcross> r;
    float x[kPer][8], g[kPer][8];
#pragma unroll
    for (int c = 0; c < kPer; ++c) {
      unpack8(xr[c], x[c]);
      if (a.branch) unpack8(br[c], r.v[c]);
      if (a.gate) unpack8(gr[c], g[c]);
    }
    if (row + step < a.rows) request(row + step);
#pragma unroll
    for (int c = 0; c < kPer; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[c][i] = has[c] ? x[c][i] : 0.f;
        r.v[c][i] = has[c] && a.branch ? r.v[c][i] : 0.f;
      }
    if (a.branch) {
      if (a.post.kind != AGG_NORM_NONE) r.norm(a.post, post, has, inv_c, slots, turn, waves);
#pragma unroll
      for (int c = 0; c < kPer; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          r.v[c][i] *= scale[c][i];
          if (a.gate) r.v[c][i] *= g[c][i];
          r.v[c][i] += x[c][i];
        }
#pragma unroll
      for (int c = 0; c < kPer; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[c][i] = has[c] ? r.v[c][i] : 0.f;
    } else {
#pragma unroll
      for (int c = 0; c < kPer; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[c][i] = x[c][i];
    }
    if (a.h) {
#pragma unroll
      for (int c = 0; c < kPer; ++c)
        if (has[c]) store16<true>(a.h + row * a.C + off[c], pack8(r.v[c]));
    }
    if (a.pre.kind != AGG_NORM_NONE) {
      r.norm(a.pre, pre, has, inv_c, slots, turn, waves);
#pragma unroll
      for (int c = 0; c < kPer; ++c)
        if (has[c]) store16<kStream>(a.n + row * a.C + off[c], pack8(r.v[c]));
    }
  }
}

// ---------------------------------------------------------------------------
// The same for many long rows: one wavefront a row again, kChunks chunks a lane, the parameters of all
// channels in LDS (registers would hold too few wavefronts, and a row shared by a workgroup's
// wavefronts fills the SIMDs unevenly unless they are a multiple of four).  kChunks is exact, so that all addresses but
// the last chunk's are a constant apart: with limits on every chunk it took 164 to 256 registers instead of 103 to 189.
// Measured: 8191 rows of 2112 channels, RMS before and behind, gate and scale, 26 us (5.3 TB/s) against 55 with a
// workgroup a row; 30 000 rows of 4096 with every part 204 (4.8 TB/s) against 251.
// ---------------------------------------------------------------------------
constexpr int kLongThreads = 256;

template <int kChunks, bool kStream>
__global__ __launch_bounds__(kLongThreads, kChunks <= 4 ? 4 : kChunks <= 6 ? 3 : 2) void seam_long_kernel(SeamArgs a) {
  extern __shared__ __align__(16) float params[];
  const int lane = threadIdx.x & 63;
  // kChunks is the row's number of 64-chunk runs: only the last one may be partial
  const int nchunk = a.C / 8;
  const bool in_last = lane + 64 * (kChunks - 1) < nchunk;
  const int last_at = (in_last ? lane + 64 * (kChunks - 1) : 0) * 8;
  auto at = [&](int c) { return c + 1 < kChunks ? lane * 8 + 512 * c : last_at; };
  auto has = [&](int c) { return c + 1 < kChunks || in_last; };
  const float inv_c = 1.f / (float)a.C;
  const float* const from[5] = {a.post.gamma, a.post.beta, a.scale, a.pre.gamma, a.pre.beta};
  int place[5], held = 0;  // of each parameter that is there
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    place[k] = -1;
    if (!from[k]) continue;
    place[k] = held * a.C;
    ++held;
    for (int c = threadIdx.x; c < a.C / 4; c += kLongThreads)
      *reinterpret_cast<f32x4*>(params + place[k] + 4 * c) = *reinterpret_cast<const f32x4*>(from[k] + 4 * c);
  }
  __syncthreads();

  auto norm = [&](float (&v)[kChunks][8], const SeamNorm& n, int gamma, int beta) {
    float mean = 0.f;
    if (n.kind == AGG_NORM_LAYER) {
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) mean += v[c][i];
      mean = sum_of_wave(mean) * inv_c;
    }
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[c][i] = has(c) ? v[c][i] - mean : 0.f;
        sq += v[c][i] * v[c][i];
      }
    const float r = rsqrtf(sum_of_wave(sq) * inv_c + n.eps);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] *= r;
      if (gamma >= 0) {
        float g[8];
        load8(params + gamma, at(c), 1.f, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= g[i];
      }
      if (beta >= 0) {
        float b[8];
        load8(params + beta, at(c), 0.f, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] += b[i];
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * (kLongThreads / 64);
  for (int64_t row = (int64_t)blockIdx.x * (kLongThreads / 64) + (threadIdx.x >> 6); row < a.rows; row += step) {
    u32x4 xr[kChunks], gr[kChunks];
    float v[kChunks][8];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      xr[c] = load16<kStream>(a.x + row * a.C + at(c));
      u32x4 br = {0u, 0u, 0u, 0u};
      if (a.branch) br = load16<kStream>(a.branch + row * a.C + at(c));
      if (a.gate)  // rows < 2^31 and gate_rows <= 2^31
        gr[c] = *reinterpret_cast<const u32x4*>(a.gate + (int64_t)((uint32_t)row / (uint32_t)a.gate_rows) * a.C + at(c));
      unpack8(br, v[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = has(c) ? v[c][i] : 0.f;
    }
    if (a.branch && a.post.kind != AGG_NORM_NONE) norm(v, a.post, place[0], place[1]);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      float f[8];
      if (place[2] >= 0) {
        load8(params + place[2], at(c), 1.f, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= f[i];
      }
      if (a.gate) {
        unpack8(gr[c], f);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= f[i];
      }
      unpack8(xr[c], f);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = has(c) ? v[c][i] + f[i] : 0.f;
      if (a.h && has(c)) store16<true>(a.h + row * a.C + at(c), pack8(v[c]));
    }
    if (a.pre.kind != AGG_NORM_NONE) {
      norm(v, a.pre, place[3], place[4]);
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
        if (has(c)) store16<kStream>(a.n + row * a.C + at(c), pack8(v[c]));
    }
  }
}

template <int kPer, bool kAcross, bool kStream>
static hipError_t launch_seam_rows(const SeamArgs& a, int threads, hipStream_t st) {
  const int64_t groups = kAcross ? a.rows : (a.rows + 3) / 4;
  // as many wavefronts as run at once: each keeps its parameters and requests ahead over the rows that are left.  us with
  // post norm, gate and pre norm against four times as many: 5496 rows of 1024 11.4 / 13.3, of 512 6.9 / 7.4; 1500 of
  // 4104 21.8 / 25.3; 54 960 of 1024 83.9 / 82.7
  const int64_t most = 256 * 4 * (kPer == 1 ? 4 : 2) / (threads / 64);
  hipLaunchKernelGGL((seam_kernel<kPer, kAcross, kStream>), dim3((unsigned)(groups < most ? groups : most)), dim3(threads), 0, st, a);
  return hipGetLastError();
}

template <int kChunks, bool kStream>
static hipError_t launch_seam_long(const SeamArgs& a, hipStream_t st) {
  const float* const from[5] = {a.post.gamma, a.post.beta, a.scale, a.pre.gamma, a.pre.beta};
  int held = 0;
  for (const float* f : from) held += f != nullptr;
  const int bytes = held * a.C * (int)sizeof(float);  // at most 80 KiB
  const int64_t groups = (a.rows + kLongThreads / 64 - 1) / (kLongThreads / 64);
  const int fit = bytes ? 160 * 1024 / bytes : 8;
  const int64_t most = 256 * (kChunks <= 4 ? min(fit, 4) : kChunks <= 6 ? min(fit, 3) : 2);
  if (bytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)seam_long_kernel<kChunks, kStream>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, 80 * 1024);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((seam_long_kernel<kChunks, kStream>), dim3((unsigned)(groups < most ? groups : most)), dim3(kLongThreads),
                     bytes, st, a);
  return hipGetLastError();
}

template <bool kStream>
static hipError_t launch_seam_many(const SeamArgs& a, int waves, hipStream_t st) {
  switch (waves) {
    case 1: return launch_seam_rows<1, false, kStream>(a, 256, st);
    case 2: return launch_seam_rows<2, false, kStream>(a, 256, st);
    case 3: return launch_seam_long<3, kStream>(a, st);
    case 4: return launch_seam_long<4, kStream>(a, st);
    case 5: return launch_seam_long<5, kStream>(a, st);
    case 6: return launch_seam_long<6, kStream>(a, st);
    case 7: return launch_seam_long<7, kStream>(a, st);
    case 8: return launch_seam_long<8, kStream>(a, st);
  }
  return launch_seam_rows<2, true, kStream>(a, 512, st);
}

hipError_t launch_seam(const SeamArgs& args, hipStream_t st) {
  SeamArgs a = args;
  if (a.gate_rows > a.rows) a.gate_rows = a.rows;
  if (a.post.kind == AGG_NORM_NONE) a.post.gamma = a.post.beta = nullptr;
  if (a.pre.kind == AGG_NORM_NONE) a.pre.gamma = a.pre.beta = nullptr;
  const int waves = (a.C / 8 + 63) / 64;  // one chunk a thread
  (void)hipGetLastError();
  // Few rows: the whole workgroup on one of them. us for 1, 512, 1000 rows of 2112 channels with every part:
  // 3.8, 5.1, 10.0 against 5.7, 7.0, 8.0 a wavefront each; 1, 768 rows of 4096: 3.7, 7.9 against 7.5, 10.4
  if (waves > 2 && waves <= 8 && a.rows <= 896) return launch_seam_rows<1, true, false>(a, 64 * waves, st);
  return streams(a.rows * a.C * 2) ? launch_seam_many<true>(a, waves, st) : launch_seam_many<false>(a, waves, st);
}

}  // namespace agg
