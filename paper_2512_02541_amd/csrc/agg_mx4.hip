// Microscaled 4-bit floats: quantisation, reading back, and the product of two matrices held so.
#include <type_traits>
#include <utility>

#include "agg_internal.h"
#include "agg_lds_copy.h"
#include "agg_mx4_block.h"
#include "agg_mx4_plan.h"
#include "agg_stream.h"

namespace agg {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

namespace {

__device__ inline uint32_t pack2(float lo, float hi) {
  f32x2 p = {lo, hi};
  bf16x2 h = __builtin_convertvector(p, bf16x2);
  return __builtin_bit_cast(uint32_t, h);
}
__device__ inline const uint8_t* uniform_ptr8(const uint8_t* q) { return (const uint8_t*)uniform_ptr((const uint16_t*)q); }
// f(0), f(1), ... with numbers that the compiler knows
template <class F, int... i>
__device__ __forceinline__ void for_each_of(F&& f, std::integer_sequence<int, i...>) {
  (f(std::integral_constant<int, i>{}), ...);
}
template <int n, class F>
__device__ __forceinline__ void for_each(F&& f) {
  for_each_of(f, std::make_integer_sequence<int, n>{});
}
// The lane's number, worked out where it stands: what follows from it is not held in registers from
// one place of a kernel to another.
__device__ __forceinline__ int lane_again() {
  uint32_t none = 0;
  asm volatile("" : "+v"(none));
  return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
}
// 16 x 16 += 16 x 128 times 128 x 16, both in 4 bits; kByte: which byte of sa and sw is the scale
template <int kByte>
__device__ __forceinline__ f32x4 mfma4(u32x4 a, u32x4 w, f32x4 acc, int sa, int sw) {
  const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8 y = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 4, 4, kByte, sa, kByte, sw);
}
__device__ inline float bf16_of(uint32_t bits) { return __uint_as_float(bits << 16); }

}  // namespace

// ---------------------------------------------------------------------------
// Quantisation: a lane holds eight channels, four lanes a block of 32, one wavefront a row; HBM-bound: 137 400 rows of
// 1024 and back 109 us (712 MB, the codes counted twice), 134 with ordinary accesses to the bf16 tensors.
// ---------------------------------------------------------------------------
constexpr int kQuantThreads = 256;

template <bool kStream>
__global__ __launch_bounds__(kQuantThreads) void mx4_quantize_kernel(
    const uint16_t* __restrict__ x, int64_t x_stride, uint32_t* __restrict__ codes,
    uint8_t* __restrict__ scales, int64_t rows, int K, int words, int scale_stride) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (kQuantThreads / 64) + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int nchunk = K / 8;
  // words: a multiple of 32, so four lanes leave together
  for (int w = blockIdx.y * 64 + lane; w < words; w += gridDim.y * 64) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (w < nchunk) v = load16<kStream>(x + row * x_stride + w * 8);
    uint32_t s;
    const uint32_t code = mx4_codes(v, s);
    codes[row * words + w] = code;
    if ((w & 3) == 0) scales[row * scale_stride + w / 4] = (uint8_t)s;
  }
  // the scales behind the row's last whole run of codes
  if (blockIdx.y == 0)
    for (int i = words / 4 + lane; i < scale_stride; i += 64) scales[row * scale_stride + i] = 0;
}

template <bool kStream>
__global__ __launch_bounds__(kQuantThreads) void mx4_dequantize_kernel(
    const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, uint16_t* __restrict__ x,
    int64_t rows, int K, int words, int scale_stride) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (kQuantThreads / 64) + (threadIdx.x >> 6);
  if (row >= rows) return;
  for (int w = blockIdx.y * 64 + lane; w < K / 8; w += gridDim.y * 64) {
    const uint32_t code = codes[row * words + w];
    const uint32_t s = scales[row * scale_stride + w / 4];
    const float scale = __uint_as_float(s << 23);
    u32x4 v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
    if (s == 255) v = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
    store16<kStream>(x + row * K + w * 8, v);
  }
}

// ---------------------------------------------------------------------------
// Product  Y[m, n] = sum_k A[m, k] W[n, k] + bias[n]  on v_mfma_scale_f32_16x16x128_f8f6f4 with both operands in 4
// bits: a lane holds the 32 channels of one scale (16 bytes) of one row, group G = lane / 16 of the
// lanes the G-th block of the 128.  The padding behind K is zeros, so no product needs a limit in k.
//
// For few rows: 16 tokens x 16 channels a workgroup, whose eight wavefronts share k; their sums meet
// in LDS, in a fixed order.  What counts is one chain of latencies: fragments come straight from memory,
// up to four steps of 128 channels under way at once.  Measured, each of many in a graph: 1 row of 1024 -> 1024 2.7 to
// 3.1 us (3.3 to 3.6 alone), of 4096 -> 1024 4.1 to 4.4 (7.2 and 15.7 in a 32 x 64 tile a wavefront); 64 rows of
// 4096 -> 1024 5.8 to 6.1.
// ---------------------------------------------------------------------------
constexpr int kFewWaves = 8;

__global__ __launch_bounds__(64 * kFewWaves) void mx4_few_kernel(Mx4LinearArgs p) {
  __shared__ f32x4 sums[kFewWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane & 15, G = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.y * 16;
  const int which = blockIdx.x / p.gn, n0 = (blockIdx.x - which * p.gn) * 16;
  const int64_t m = min(m0 + c, p.rows - 1);
  const int wn = min(n0 + c, p.N - 1);
  const uint8_t* a = p.a.codes + m * p.code_stride + G * 16;
  const uint8_t* as = p.a.scales + m * p.scale_stride + G;
  const uint8_t* w = p.w[which].codes + (int64_t)wn * p.code_stride + G * 16;
  const uint8_t* ws = p.w[which].scales + (int64_t)wn * p.scale_stride + G;

  // what the output's thread adds, requested first
  const int row = threadIdx.x >> 4 & 15, n = n0 + c;
  const bool mine = threadIdx.x < 256 && m0 + row < p.rows && n < p.N;
  float bias = 0.f, scale = 1.f, x = 0.f;
  if (mine) {
    if (p.bias[which]) bias = p.bias[which][n];
    if (p.res_scale) scale = p.res_scale[n];
    if (p.residual) x = bf16_of(p.residual[(m0 + row) * p.N + n]);
  }

  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const int steps = p.code_stride / 64;  // of 128 channels
  constexpr int kDeep = 4;
  for (int s0 = wave; s0 < steps; s0 += kFewWaves * kDeep) {
    u32x4 fa[kDeep], fw[kDeep];
    int sa[kDeep], sw[kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const int s = s0 + i * kFewWaves;
      if (s < steps) {
        fa[i] = *reinterpret_cast<const u32x4*>(a + s * 64);
        fw[i] = *reinterpret_cast<const u32x4*>(w + s * 64);
        sa[i] = as[s * 4];
        sw[i] = ws[s * 4];
      }
    }
#pragma unroll
    for (int i = 0; i < kDeep; ++i)
      if (s0 + i * kFewWaves < steps) acc = mfma4<0>(fa[i], fw[i], acc, sa[i], sw[i]);
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (!mine) return;
  // element (row, c) is register row % 4 of lane 16 (row / 4) + c
  float y = 0.f;
#pragma unroll
  for (int i = 0; i < kFewWaves; ++i) y += reinterpret_cast<const float*>(&sums[i][(row >> 2) * 16 + c])[row & 3];
  y += bias;
  if (p.residual) y = x + scale * y;
  p.y[which][(m0 + row) * p.N + n] = (uint16_t)pack2(y, 0.f);
}

// ---------------------------------------------------------------------------
// The same product in tiles of kTM tokens x kTN channels, shared out to kWM x kWN wavefronts.
// k advances 256 at a time, whole 128-byte lines of codes, copied global -> LDS without passing through
// registers into one or two stages; the scales of two steps, 16 bytes of a row, come with the
// first of them into slots of their own.  LDS rows are 128 bytes with the 16-byte chunk number
// XOR-ed by bits 1..3 of the row, which spreads the 16 rows of a fragment read over all banks.
// Which 32 of a step's 256 channels a group of lanes multiplies in which of the two MFMAs is free as
// long as both operands agree: group G takes blocks 2 G and 2 G + 1, so that both scales come with
// one two-byte read and the MFMA's own byte selection tells them apart; block 2 G + h lies at position
// 4 h + G of its row (with the blocks in order the reads conflicted two-way).
//
// With one stage nothing hides inside a workgroup: four of them share a CU, and one's copies and stores run beside
// another's products; with fewer tiles two stages are faster (the plan has both sides).  Outputs are stored past
// the caches, whose lines the operands need: Q/K/V of 137 400 x 1024 in tiles of 128, four on a CU,
// 451 us through them, 326 past them.  For few rows it makes no difference: blocks of 1 to 16 frames, whose attention
// reads Q, K and V at once, the same within 1 %.
// Some hundred rows are a chain of copies with one step under way: Q/K/V of 522 x 1024 5.6 us (6.3 alone) where their
// bytes take 1.1, 1374 x 4096 -> 1024 10.1 against 1.8, 2748 rows 14.1 against 3.5.
// Measured: 21 984 x 4096 -> 1024 60 us without a residual, 64 with one (184 GFLOP: 3.1 PFLOP/s); 21 984 x 4096 -> 4096
// 197 us (3.7 PFLOP/s, tiles of 256; MFMAs alone on random codes reach 6.3 to 6.8, limited by power: 9.6 on zeros).  A step of
// a 256-wide tile takes 1.5 us, of which its products are 0.9; its copies alone and its products with their fragment
// reads alone take 1.0 to 1.1 each.  No faster: a third stage; the next half's fragments read during a half's products;
// one group of wavefronts half a step behind the other; tiles of 192 tokens; tiles that begin at different k.
// ---------------------------------------------------------------------------
constexpr int kStepBytes = 128;   // of a row of codes: 256 channels
constexpr int kScaleBytes = 16;   // of a row of scales: two steps

template <int kTM, int kTN, int kWM, int kWN, int kStages, int kPerSimd>
__global__ __launch_bounds__(64 * kWM * kWN, kPerSimd) void mx4_tile_kernel(Mx4LinearArgs p) {
  constexpr int kWaves = kWM * kWN;
  constexpr int kMT = kTM / kWM / 16, kNT = kTN / kWN / 16;  // 16-token and 16-channel tiles of a wavefront
  constexpr int kWTM = kTM / kWM, kWTN = kTN / kWN;
  static_assert(8 % kNT == 0, "a lane's channels of a token all exist or none: N is a multiple of 8");
  constexpr int kStepA = kTM * kStepBytes, kStepW = kTN * kStepBytes;  // a step's rows
  constexpr int kCopiesA = kTM / 8 / kWaves, kCopiesW = kTN / 8 / kWaves;  // copies of a wavefront per step
  constexpr int kScaleSlots = (kStages + 2) / 2;
  constexpr int kScaleSlot = (kTM + kTN) * kScaleBytes;
  constexpr int kScalesAt = kStages * (kStepA + kStepW);
  constexpr int kScaleInstr = (kTM + kTN) / 64, kScaleCopies = (kScaleInstr + kWaves - 1) / kWaves;
  __shared__ __align__(16) char sm[kScalesAt + kScaleSlots * kScaleSlot];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, G = lane >> 4;
  const int wm = wave % kWM * kWTM, wn = wave / kWM * kWTN;

  // every XCD takes an equal run of the tiles: all of one token tile, then of the next, or the other way round
  // (32 bits: the tiles are fewer than 2^31)
  const uint32_t per_m = p.gn * p.count, gm = (uint32_t)p.gm;
  const uint64_t total = (uint64_t)gm * per_m;
  const uint32_t xcd = blockIdx.x % kGemmXcds;
  const uint32_t at = (uint32_t)(total * xcd / kGemmXcds) + blockIdx.x / kGemmXcds;
  if (at >= (uint32_t)(total * (xcd + 1) / kGemmXcds)) return;  // uniform for the workgroup, before any barrier
  const uint32_t high = at / (p.by_channels ? gm : per_m), low = at - high * (p.by_channels ? gm : per_m);
  const int nt = (int)(p.by_channels ? high : low);
  const int which = nt / p.gn;
  const int64_t m0 = (int64_t)(p.by_channels ? low : high) * kTM;
  const int n0 = (nt - which * p.gn) * kTN;
  const int nk = p.code_stride / kStepBytes;

  // Copies: an instruction lands 8 LDS rows of codes or 64 of scales.  LDS row 16 ct + i of a
  // wavefront's channels is channel kNT i + ct: a lane ends with kNT consecutive ones of a token.
  // Rows past the end repeat the last one; never stored.
  auto channel_of = [&](int row) {
    const int in = row % kWTN;
    return min(n0 + row - in + kNT * (in % 16) + in / 16, p.N - 1) - n0;
  };
  auto block_at = [](int at) { return (uint32_t)((at & 3) << 1 | at >> 2); };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)sm;
  const int64_t last = p.rows - 1 - m0;  // >= 0
  uint32_t aoff[kCopiesA], woff[kCopiesW], soff[kScaleCopies];
  const uint8_t* sbase[kScaleCopies];
#pragma unroll
  for (int i = 0; i < kCopiesA; ++i) {
    const int row = (wave * kCopiesA + i) * 8 + (lane >> 3);
    aoff[i] = (uint32_t)min((int64_t)row, last) * (uint32_t)p.code_stride + block_at((lane & 7) ^ ((row >> 1) & 7)) * 16u;
  }
#pragma unroll
  for (int i = 0; i < kCopiesW; ++i) {
    const int row = (wave * kCopiesW + i) * 8 + (lane >> 3);
    woff[i] = (uint32_t)channel_of(row) * (uint32_t)p.code_stride + block_at((lane & 7) ^ ((row >> 1) & 7)) * 16u;
  }
  // instruction i of the scales: 64 rows of A's, then of W's; where there are fewer than wavefronts some
  // copy the same, so that all wait for equally many
#pragma unroll
  for (int i = 0; i < kScaleCopies; ++i) {
    const int at = (wave + i * kWaves) % kScaleInstr;
    const bool of_a = at < kTM / 64;
    const int row = (of_a ? at : at - kTM / 64) * 64 + lane;
    soff[i] = (of_a ? (uint32_t)min((int64_t)row, last) : (uint32_t)channel_of(row)) * (uint32_t)p.scale_stride;
    sbase[i] = uniform_ptr8(of_a ? p.a.scales + m0 * p.scale_stride : p.w[which].scales + (int64_t)n0 * p.scale_stride);
  }
  const uint8_t* abase = uniform_ptr8(p.a.codes + m0 * p.code_stride);
  const uint8_t* wbase = uniform_ptr8(p.w[which].codes + (int64_t)n0 * p.code_stride);
  int c_stage = 0, c_slot = 0;  // where the next step's codes and the next two steps' scales go
  auto copy = [&](bool with_scales) {
    const uint32_t to = lds0 + c_stage * (kStepA + kStepW);
#pragma unroll
    for (int i = 0; i < kCopiesA; ++i) dma16(abase, aoff[i], to + (wave * kCopiesA + i) * 1024);
#pragma unroll
    for (int i = 0; i < kCopiesW; ++i) dma16(wbase, woff[i], to + kStepA + (wave * kCopiesW + i) * 1024);
    abase += kStepBytes;
    wbase += kStepBytes;
    c_stage = c_stage + 1 == kStages ? 0 : c_stage + 1;
    if (with_scales) {
#pragma unroll
      for (int i = 0; i < kScaleCopies; ++i) {
        dma16(sbase[i], soff[i], lds0 + kScalesAt + c_slot * kScaleSlot + (wave + i * kWaves) % kScaleInstr * 1024);
        sbase[i] += kScaleBytes;
      }
      c_slot = c_slot + 1 == kScaleSlots ? 0 : c_slot + 1;
    }
  };

  f32x4 acc[kMT][kNT];
#pragma unroll
  for (int t = 0; t < kMT; ++t)
#pragma unroll
    for (int u = 0; u < kNT; ++u) acc[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
  const lds_char* lds = (const lds_char*)sm;
  const int f0 = c * kStepBytes + ((G ^ ((c >> 1) & 7)) * 16);
  int stage = 0, slot = 0;
  int sa[kMT], sw[kNT];
  u32x4 fa[kMT], fw[kNT];
  auto mul = [&](auto which_half) {
    constexpr int h = decltype(which_half)::value;
#pragma unroll
    for (int t = 0; t < kMT; ++t)
#pragma unroll
      for (int u = 0; u < kNT; ++u) acc[t][u] = mfma4<h>(fa[t], fw[u], acc[t][u], sa[t], sw[u]);
  };
  // kOdd: the second of the two steps that share a row's scales
  auto step = [&](int k, auto odd) {
    constexpr int kOdd = decltype(odd)::value;
    if constexpr (kStages == 1) {
      if (k > 0) lds_barrier();
      copy(kOdd == 0);
    }
    wait_vm0();
    lds_barrier();  // everybody's copies of this step are in, and with two stages the last step's is free
    if (kStages == 2 && k + 1 < nk) copy(kOdd == 1);
    const lds_char* at_a = lds + stage * (kStepA + kStepW) + wm * kStepBytes;
    const lds_char* at_w = lds + stage * (kStepA + kStepW) + kStepA + wn * kStepBytes;
    const lds_char* sc = lds + kScalesAt + slot * kScaleSlot + c * kScaleBytes + 8 * kOdd + 2 * G;
    auto read_scales = [&]() {
#pragma unroll
      for (int t = 0; t < kMT; ++t)
        sa[t] = *reinterpret_cast<const __attribute__((address_space(3))) uint16_t*>(sc + (wm + 16 * t) * kScaleBytes);
#pragma unroll
      for (int u = 0; u < kNT; ++u)
        sw[u] = *reinterpret_cast<const __attribute__((address_space(3))) uint16_t*>(sc + (kTM + wn + 16 * u) * kScaleBytes);
    };
    auto read = [&](int h) {
#pragma unroll
      for (int u = 0; u < kNT; ++u)
        fw[u] = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(at_w + (f0 ^ (64 * h)) + u * 16 * kStepBytes);
#pragma unroll
      for (int t = 0; t < kMT; ++t)
        fa[t] = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(at_a + (f0 ^ (64 * h)) + t * 16 * kStepBytes);
    };
    read_scales();
    read(0);
    mul(std::integral_constant<int, 0>{});
    read(1);
    mul(std::integral_constant<int, 1>{});
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (kOdd) slot = slot + 1 == kScaleSlots ? 0 : slot + 1;
  };

  if (kStages == 2) copy(true);
  for (int k = 0; k < nk; k += 2) {
    step(k, std::integral_constant<int, 0>{});
    if (k + 1 >= nk) break;
    step(k + 1, std::integral_constant<int, 1>{});
  }

  const int place = lane_again(), ec = place & 15, eg = place >> 4 << 2;
  const int n = n0 + wn + kNT * ec;
  if (n >= p.N) return;  // N is a multiple of 8: all kNT channels exist or none
  float bias[kNT], scale[kNT];
#pragma unroll
  for (int u = 0; u < kNT; ++u) {
    bias[u] = p.bias[which] ? p.bias[which][n + u] : 0.f;
    scale[u] = p.res_scale ? p.res_scale[n + u] : 1.f;
  }
  typedef uint32_t Run __attribute__((ext_vector_type(kNT / 2)));  // kNT channels of a token
  const int64_t corner = (m0 + wm + eg) * p.N + n;
  const int64_t left = p.rows - (m0 + wm + eg);
  Run x[kMT][4];  // of the residual, requested at once
  if (p.residual)
#pragma unroll
    for (int t = 0; t < kMT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * t + r < left)
          x[t][r] = *reinterpret_cast<const Run*>(p.residual + corner + (int64_t)(16 * t + r) * p.N);
#pragma unroll
  for (int t = 0; t < kMT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (16 * t + r >= left) continue;
      float y[kNT];
#pragma unroll
      for (int u = 0; u < kNT; ++u) y[u] = acc[t][u][r] + bias[u];
      if (p.residual)
#pragma unroll
        for (int u = 0; u < kNT; ++u) {
          const uint32_t w = x[t][r][u / 2];
          y[u] = (u % 2 ? __uint_as_float(w & 0xFFFF0000u) : bf16_of(w)) + scale[u] * y[u];
        }
      Run out;
#pragma unroll
      for (int u = 0; u < kNT / 2; ++u) out[u] = pack2(y[2 * u], y[2 * u + 1]);
      __builtin_nontemporal_store(out, reinterpret_cast<Run*>(p.y[which] + corner + (int64_t)(16 * t + r) * p.N));
    }
}

template <int kTM, int kTN, int kWM, int kWN, int kStages, int kPerSimd>
static hipError_t launch_mx4_tiles(Mx4LinearArgs p, hipStream_t st) {
  p.gm = (p.rows + kTM - 1) / kTM;
  p.gn = (p.N + kTN - 1) / kTN;
  p.by_channels = p.rows < (int64_t)p.N * p.count;  // the operand of more rows is the one that is read once
  const int64_t groups = (p.gm * p.gn * p.count + kGemmXcds - 1) / kGemmXcds * kGemmXcds;
  if (groups > 0xFFFFFFFFll / (64 * kWM * kWN)) return hipErrorInvalidConfiguration;  // 2^32 threads (kLaunchRows)
  hipLaunchKernelGGL((mx4_tile_kernel<kTM, kTN, kWM, kWN, kStages, kPerSimd>), dim3((unsigned)groups),
                     dim3(64 * kWM * kWN), 0, st, p);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The same product for many rows and K up to 128 kKS: a wavefront keeps 64 tokens' codes and scales,
// all of k, in registers and multiplies them with 64 channels after another that all eight
// wavefronts read from a ring in LDS: a fragment read feeds four MFMAs, nothing of A is read twice, and the
// outputs leave evenly instead of a tile at a time.
// A pass over 64 channels is awaited three passes after it was requested, with the stores of those
// passes still on their way behind it.
// Workgroup: 512 tokens.  The list of (512 tokens, 64 channels) is shared out evenly.
//
// Measured: Q/K/V of 137 400 x 1024 (864 GFLOP, 844 MB of outputs) 232 us, 3.7 PFLOP/s; 250 with all wavefronts
// storing at a pass's end, 315 in tiles.  Without its stores 186, without its products 192, products and fragment
// reads alone 173: products (power) and stores (a kernel that does nothing else writes this pattern in 165 us) bound it
// together.  With few passes a workgroup its start and end count: 21 984 rows 52 us, 12 of them outside the nine passes.  K = 512, 3 x 512 channels: 93 us against 113.  With a residual, read like the stores are written and two
// 16-token tiles a wavefront for the registers, it was no faster than tiles (163 to 181 us against 173).
// ---------------------------------------------------------------------------
constexpr int kPanelThreads = 512;
constexpr int kPassSlots = 4;

template <int kKS>
__global__ __launch_bounds__(kPanelThreads, 2) void mx4_panel_kernel(Mx4LinearArgs p) {
  constexpr int kMT = 4;  // 16-token tiles of a wavefront
  constexpr int kRow = kKS * 64, kSRow = kKS * 4;  // bytes of an LDS row of codes, of scales
  constexpr int kScalesAt = kPassChannels * kRow, kBiasAt = kScalesAt + kPassChannels * kSRow;
  constexpr int kSlot = (kBiasAt + kPassChannels * 4 + kRow - 1) / kRow * kRow;
  constexpr int kCodeCopies = kPassChannels * kRow / 1024 / 8;
  constexpr int kGroup = kCodeCopies + 2;  // copies of a wavefront per pass
  constexpr int kStores = kMT * 4;         // its stores
  static_assert(kKS == 4 || kKS == 8, "rows of 16 or 32 chunks, four or eight scales in a row to a lane");
  __shared__ __align__(kRow) char sm[kPassSlots * kSlot];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // (32 bits: the passes are fewer than 2^31); consecutive runs of the list go to one XCD
  const uint32_t per_panel = p.gn * p.count;
  const uint64_t total = (uint64_t)p.gm * per_panel;
  const uint32_t mine = blockIdx.x % kGemmXcds * (kGemmCus / kGemmXcds) + blockIdx.x / kGemmXcds;
  const uint32_t first = (uint32_t)(total * mine / kGemmCus);
  const int passes = (int)((uint32_t)(total * (mine + 1) / kGemmCus) - first);
  if (passes <= 0) return;  // uniform for the workgroup, before any barrier

  // A pass in the list: its matrix, first channel and what belongs to it.
  struct Place {
    int which, n0;
  };
  auto next = [&](Place& a) {  // true at the end of the channels
    a.n0 += kPassChannels;
    if (a.n0 < p.N) return false;
    a.n0 = 0;
    if (++a.which < p.count) return false;
    a.which = 0;
    return true;
  };
  int panel = first / per_panel;
  const int in_panel = first % per_panel;
  Place now = {in_panel / p.gn, in_panel % p.gn * kPassChannels}, ahead = now;

  // Copies.  LDS row 16 ct + i of a pass is channel 4 i + ct; the 16-byte chunk at position q of a row
  // (before the XOR with the row's last four bits) is block kKS (q mod 4) + q / 4 of 32 channels: group G
  // of the lanes multiplies blocks kKS G + s in step s, whose scales are kKS bytes in a row.
  const int chunks = p.code_stride / 16;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)sm;
  int c_slot = 0;
  const uint8_t *codes, *scales, *bias_at;
  auto aim = [&]() {
    codes = uniform_ptr8(p.w[ahead.which].codes + (int64_t)ahead.n0 * p.code_stride);
    scales = uniform_ptr8(p.w[ahead.which].scales + (int64_t)ahead.n0 * p.scale_stride);
    // without a bias something else is copied and not looked at
    bias_at = uniform_ptr8(p.bias[ahead.which] ? (const uint8_t*)(p.bias[ahead.which] + ahead.n0) : codes);
  };
  auto copy = [&]() {
    const int most = p.N - 1 - ahead.n0;
    const uint32_t to = lds0 + c_slot * kSlot;
    const int place = lane_again();
#pragma unroll
    for (int i = 0; i < kCodeCopies; ++i) {
      const int at = (wave * kCodeCopies + i) * 64 + place;
      const int row = at / (kKS * 4), q = (at % (kKS * 4)) ^ (row & 15);
      dma16(codes, (uint32_t)min(4 * (row & 15) + (row >> 4), most) * (uint32_t)p.code_stride +
                       (uint32_t)min(kKS * (q & 3) + (q >> 2), chunks - 1) * 16u,
            to + (wave * kCodeCopies + i) * 1024);
    }
    const int at = (wave % kKS) * 64 + place, row = at / kKS;
    dma4(scales, (uint32_t)min(4 * (row & 15) + (row >> 4), most) * (uint32_t)p.scale_stride + (at % kKS) * 4u,
         to + kScalesAt + (wave % kKS) * 256);
    dma4(bias_at, (uint32_t)min(place, most) * 4u, to + kBiasAt);
    c_slot = c_slot + 1 == kPassSlots ? 0 : c_slot + 1;
    next(ahead);
    if (ahead.n0 == 0) {
      aim();
    } else {
      codes += (int64_t)kPassChannels * p.code_stride;
      scales += kPassChannels * p.scale_stride;
      bias_at += kPassChannels * 4;  // (of codes, where there is no bias: N rows of at least 128 bytes)
    }
  };

  aim();
  for (int i = 0; i < kPassSlots - 1; ++i)
    if (i < passes) copy();

  u32x4 fa[kMT][kKS];
  uint32_t sa[kMT][kKS / 4];
  int64_t m0 = 0;
  bool load = true;        // a panel begins
  int counted = 0;         // passes in a row whose stores all went out
  int slot = 0;

  // what a pass leaves: the first two of a lane's four channels packed, the other two as sums
  uint32_t first_two[kMT][4];
  f32x4 acc[kMT][2];
  char* y = nullptr;       // the wavefront's part of the output, its extent
  int y_rows = 0, y_channels = 0;
  auto store = [&]() {
    const int place = lane_again();
    const int ec = place & 15, eg = place >> 4 << 2;
    const uint32_t lane_at = (uint32_t)(eg * p.N + 4 * ec) * 2u;
    auto put = [&](int t, int r) {
      __builtin_nontemporal_store(u32x2{first_two[t][r], pack2(acc[t][0][r], acc[t][1][r])},
                                  reinterpret_cast<u32x2*>(y + (int64_t)(16 * t + r) * p.N * 2 + lane_at));
    };
    if (y_rows >= 64 && y_channels >= kPassChannels) {
#pragma unroll
      for (int t = 0; t < kMT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) put(t, r);
      ++counted;
    } else {
      if (4 * ec < y_channels) {
#pragma unroll
        for (int t = 0; t < kMT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * t + eg + r < y_rows) put(t, r);
      }
      counted = 0;
    }
  };

  // The two wavefronts of a SIMD take turns: one stores a pass at its end, the other one at the
  // beginning of the next, so that one's conversions and stores run beside the other's products.
  const bool late = wave >= kPanelThreads / 128;
  for (int j = 0; j < passes; ++j) {
    // this pass's copies are in; the next two passes' and the last three's stores need not be
    if (j + 2 >= passes) wait_vm0();
    else if (counted >= 3) wait_vm<2 * kGroup + 3 * kStores>();
    else wait_vm<2 * kGroup>();
    lds_barrier();  // everybody's copies of this pass are in, and the last pass's slot is free
    if (j + kPassSlots - 1 < passes) copy();
    if (late && j > 0) store();

    if (load) {
      m0 = (int64_t)panel * kPanelRows + wave * 64;
      const int place = lane_again(), c = place & 15, G = place >> 4;
#pragma unroll
      for (int t = 0; t < kMT; ++t) {
        const int64_t m = min(m0 + 16 * t + c, p.rows - 1);
#pragma unroll
        for (int s = 0; s < kKS; ++s)
          fa[t][s] = *reinterpret_cast<const u32x4*>(p.a.codes + m * p.code_stride + min(kKS * G + s, chunks - 1) * 16);
#pragma unroll
        for (int s = 0; s < kKS / 4; ++s)
          sa[t][s] = *reinterpret_cast<const uint32_t*>(p.a.scales + m * p.scale_stride + kKS * G + 4 * s);
      }
      // awaited here: a wait at their first use would be one in every pass, for the copies and stores too
#pragma unroll
      for (int t = 0; t < kMT; ++t) {
#pragma unroll
        for (int s = 0; s < kKS; ++s) asm volatile("" : "+v"(fa[t][s]));
#pragma unroll
        for (int s = 0; s < kKS / 4; ++s) asm volatile("" : "+v"(sa[t][s]));
      }
      y_rows = (int)max(min(p.rows - m0, (int64_t)64), (int64_t)0);
    }
    if (load || now.n0 == 0) {
      y = reinterpret_cast<char*>(p.y[now.which] + m0 * p.N + now.n0);
    } else {
      y += kPassChannels * 2;
    }
    y_channels = p.N - now.n0;
    const bool has_bias = p.bias[now.which] != nullptr;
    load = next(now);
    if (load) ++panel;

    // slots and rows begin at multiples of kRow: a step's chunk is an XOR away from the first one's
    const lds_char* const w = (const lds_char*)sm + slot * kSlot;
    slot = slot + 1 == kPassSlots ? 0 : slot + 1;
    const int place = lane_again(), c = place & 15, G = place >> 4;
    const uint32_t w0 = (uint32_t)(uintptr_t)w + c * kRow + (G ^ c) * 16;
    const lds_char* const ws = w + kScalesAt + c * kSRow + kKS * G;
    auto half = [&](auto which_half) {
      constexpr int h = decltype(which_half)::value;
      uint32_t sw[2][kKS / 4];
      f32x4 start[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int s = 0; s < kKS / 4; ++s)
          sw[u][s] = *reinterpret_cast<const __attribute__((address_space(3))) uint32_t*>(
              ws + 16 * (2 * h + u) * kSRow + 4 * s);
        float b = *reinterpret_cast<const __attribute__((address_space(3))) float*>(w + kBiasAt + 16 * c + 4 * (2 * h + u));
        b = has_bias ? b : 0.f;
        start[u] = f32x4{b, b, b, b};
      }
      // a step's fragments are read while the one before is multiplied
      auto read = [&](u32x4 (&fw)[2], int s) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          fw[u] = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(
              (const lds_char*)(uintptr_t)(w0 ^ (64 * s)) + 16 * (2 * h + u) * kRow);
      };
      u32x4 fw[2][2];
      read(fw[0], 0);
      auto step = [&](auto which_step) {
        constexpr int s = decltype(which_step)::value;
        if constexpr (s + 1 < kKS) read(fw[(s + 1) % 2], s + 1);
#pragma unroll
        for (int t = 0; t < kMT; ++t)
#pragma unroll
          for (int u = 0; u < 2; ++u)
            acc[t][u] = mfma4<s % 4>(fa[t][s], fw[s % 2][u], s == 0 ? start[u] : acc[t][u], sa[t][s / 4], sw[u][s / 4]);
        __builtin_amdgcn_sched_barrier(0);
      };
      for_each<kKS>(step);
      if constexpr (h == 0) {
#pragma unroll
        for (int t = 0; t < kMT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) first_two[t][r] = pack2(acc[t][0][r], acc[t][1][r]);
      }
    };
    half(std::integral_constant<int, 0>{});
    half(std::integral_constant<int, 1>{});
    if (!late) store();
  }
  if (late) store();
}

template <int kKS>
static hipError_t launch_mx4_panels(Mx4LinearArgs p, hipStream_t st) {
  p.gm = (p.rows + kPanelRows - 1) / kPanelRows;
  p.gn = (p.N + kPassChannels - 1) / kPassChannels;
  if (mx4_passes(p.rows, p.N, p.count) > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(mx4_panel_kernel<kKS>, dim3(kGemmCus), dim3(kPanelThreads), 0, st, p);
  return hipGetLastError();
}

static hipError_t launch_mx4_few(Mx4LinearArgs p, hipStream_t st) {
  p.gm = (p.rows + 15) / 16;
  p.gn = (p.N + 15) / 16;
  if (p.gm > 65535) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(mx4_few_kernel, dim3((unsigned)(p.gn * p.count), (unsigned)p.gm), dim3(64 * kFewWaves), 0, st, p);
  return hipGetLastError();
}

// Few rows are shared out by runs of 512 channels too: 1, 1374 rows of 4096 4.1, 5.1 us by whole rows, 2.5, 4.1 shared
// out; 21 984 rows 34.3 by whole rows, 39.7 shared out.
static dim3 quant_grid(int64_t rows, int words) {
  const int64_t runs = rows < 2048 ? (words + 63) / 64 : 1;
  return dim3((unsigned)((rows + kQuantThreads / 64 - 1) / (kQuantThreads / 64)), (unsigned)(runs < 65535 ? runs : 65535));
}
hipError_t launch_mx4_quantize(const void* x, int64_t x_stride, void* codes, void* scales, int64_t rows, int K,
                               hipStream_t st) {
  const int words = (int)(mx4_code_stride(K) / 4), scale_stride = (int)mx4_scale_stride(K);
  const auto kernel = streams(rows * K * 2) ? mx4_quantize_kernel<true> : mx4_quantize_kernel<false>;
  (void)hipGetLastError();
  for (int64_t first = 0; first < rows; first += kLaunchRows) {
    const int64_t here = rows - first < kLaunchRows ? rows - first : kLaunchRows;
    hipLaunchKernelGGL(kernel, quant_grid(here, words), dim3(kQuantThreads), 0, st,
                       (const uint16_t*)x + first * x_stride, x_stride, (uint32_t*)codes + first * words,
                       (uint8_t*)scales + first * scale_stride, here, K, words, scale_stride);
  }
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const void* codes, const void* scales, void* x, int64_t rows, int K, hipStream_t st) {
  const int words = (int)(mx4_code_stride(K) / 4), scale_stride = (int)mx4_scale_stride(K);
  const auto kernel = streams(rows * K * 2) ? mx4_dequantize_kernel<true> : mx4_dequantize_kernel<false>;
  (void)hipGetLastError();
  for (int64_t first = 0; first < rows; first += kLaunchRows) {
    const int64_t here = rows - first < kLaunchRows ? rows - first : kLaunchRows;
    hipLaunchKernelGGL(kernel, quant_grid(here, words), dim3(kQuantThreads), 0, st,
                       (const uint32_t*)codes + first * words, (const uint8_t*)scales + first * scale_stride,
                       (uint16_t*)x + first * K, here, K, words, scale_stride);
  }
  return hipGetLastError();
}

static hipError_t launch_mx4_kernel(Mx4Kernel kernel, const Mx4LinearArgs& p, hipStream_t st) {
  switch (kernel) {
    case kMx4Few: return launch_mx4_few(p, st);
    case kMx4Tile64: return launch_mx4_tiles<64, 64, 2, 2, 2, 4>(p, st);
    case kMx4Tile128: return launch_mx4_tiles<128, 128, 2, 2, 2, 2>(p, st);
    case kMx4Tile128Many: return launch_mx4_tiles<128, 128, 2, 2, 1, 4>(p, st);
    case kMx4Tile256: return launch_mx4_tiles<256, 256, 4, 2, 2, 2>(p, st);
    case kMx4Panel: return p.K <= 512 ? launch_mx4_panels<4>(p, st) : launch_mx4_panels<8>(p, st);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_mx4_linear(const Mx4LinearArgs& p, hipStream_t st) {
  (void)hipGetLastError();
  const Mx4Plan plan = plan_mx4(p.rows, p.N, p.K, p.count, p.residual != nullptr);
  if (plan.split == 0) return launch_mx4_kernel(plan.kernel, p, st);
  Mx4LinearArgs part = p;
  part.rows = plan.split;
  const hipError_t e = launch_mx4_kernel(kMx4Tile256, part, st);
  if (e != hipSuccess) return e;
  part = p;
  part.rows -= plan.split;
  part.a.codes += plan.split * p.code_stride;
  part.a.scales += plan.split * p.scale_stride;
  for (int i = 0; i < p.count; ++i) part.y[i] += plan.split * p.N;
  if (p.residual) part.residual += plan.split * p.N;
  return launch_mx4_kernel(plan.kernel, part, st);
}

}  // namespace agg
