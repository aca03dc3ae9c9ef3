// The token-wise parts of a model's block: query/key normalisation with rotary positions, and the
// seam between one branch and the next (norm, gate, residual scale, sum, norm).  Both are single passes
// whose bound is HBM: every row is read once, held in registers in float32 and written once.
#include "agg_internal.h"

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
// ---------------------------------------------------------------------------
constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / 64;
constexpr int kRopeMaxTokens = 8;            // of a wavefront's turn
constexpr int kRopePairs = kHeadDim / 2;
constexpr int kHeadStride = kHeadDim + 4;    // floats of a head in LDS: 16-byte aligned rows

__global__ __launch_bounds__(kRopeThreads, 4) void rope_kernel(RopeArgs a) {
  __shared__ __align__(16) float heads[kRopeWaves][8][kHeadStride];
  __shared__ __align__(16) f32x2 turns[kRopeWaves][kRopeMaxTokens][kRopePairs];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int group = lane >> 3, c0 = (lane & 7) * 8;  // this lane's head among eight, its first channel
  const int H = a.H;

  // each channel's other one, its pair and the sign of the other's share; unturned: itself, none
  int other[8], pair[8];
  float sign[8];
  uint32_t turned = 0;
  if (a.pairs) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t m = a.channel[c0 + i];
      other[i] = m & 63;
      pair[i] = (m >> 6) & 31;
      sign[i] = (m & 0x800) ? 1.f : -1.f;
      if (m & 0x1000) turned |= 1u << i;
    }
  }
  float g[2][8], b[2][8];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    load8(a.norm[t].gamma, c0, 1.f, g[t]);
    load8(a.norm[t].beta, c0, 0.f, b[t]);
  }
  float* const head = heads[wave][group];

  const int64_t step = (int64_t)gridDim.x * kRopeWaves * a.tokens;
  for (int64_t t0 = ((int64_t)blockIdx.x * kRopeWaves + wave) * a.tokens; t0 < a.total; t0 += step) {
    const int here = (int)min((int64_t)a.tokens, a.total - t0);
    if (a.pairs) {
      wave_lds_fence();  // the last turn's reads are done
      for (int i = lane; i < here * kRopePairs; i += 64) {
        const int p = i % kRopePairs, sub = i / kRopePairs;
        if (p < a.pairs) {
          const int64_t tok = t0 + sub;
          const int axis = a.axis[p];
          int32_t pos;
          if (a.pos) {
            pos = a.pos[tok * 3 + axis];
          } else {
            const uint32_t in_seq = (uint32_t)(tok % a.NQ);  // < 2^31
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
          turns[wave][sub][p] = f32x2{c, s};
        }
      }
      wave_lds_fence();
    }
    for (int item = group; item < here * H; item += 8) {
      const int sub = item / H, h = item - sub * H;
      const int64_t tok = t0 + sub;
      u32x4 raw[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (a.in[t])
          raw[t] = *reinterpret_cast<const u32x4*>(a.in[t] + tok * a.stride[t] + h * kHeadDim + c0);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (!a.in[t]) continue;
        float x[8];
        unpack8(raw[t], x);
        const int kind = a.norm[t].kind;
        if (kind != AGG_NORM_NONE) {
          float mean = 0.f;
          if (kind == AGG_NORM_LAYER) {
#pragma unroll
            for (int i = 0; i < 8; ++i) mean += x[i];
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) mean += __shfl_xor(mean, o);
            mean *= 1.f / kHeadDim;
          }
          float sq = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[i] -= mean;
            sq += x[i] * x[i];
          }
#pragma unroll
          for (int o = 1; o < 8; o <<= 1) sq += __shfl_xor(sq, o);
          const float r = rsqrtf(sq * (1.f / kHeadDim) + a.norm[t].eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = x[i] * r * g[t][i] + b[t][i];
        }
        if (a.pairs) {
          wave_lds_fence();
          *reinterpret_cast<f32x4*>(head + c0) = f32x4{x[0], x[1], x[2], x[3]};
          *reinterpret_cast<f32x4*>(head + c0 + 4) = f32x4{x[4], x[5], x[6], x[7]};
          wave_lds_fence();
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const f32x2 cs = turns[wave][sub][pair[i]];
            const float y = x[i] * cs[0] + sign[i] * head[other[i]] * cs[1];
            x[i] = (turned >> i) & 1 ? y : x[i];
          }
        }
        *reinterpret_cast<u32x4*>(a.out[t] + (tok * H + h) * kHeadDim + c0) = pack8(x);
      }
    }
  }
}

hipError_t launch_rope(const RopeArgs& args, hipStream_t st) {
  RopeArgs a = args;
  a.tokens = a.H >= 4 ? 2 : kRopeMaxTokens / a.H;
  const int64_t turns = (a.total + a.tokens - 1) / a.tokens;
  const int64_t groups = (turns + kRopeWaves - 1) / kRopeWaves;
  (void)hipGetLastError();
  hipLaunchKernelGGL(rope_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(kRopeThreads), 0, st, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// h = x + gate * scale * post(branch),  n = pre(h): one wavefront per row, the row in registers in
// float32, statistics as in layernorm_kernel (mean, then variance of the centred values).
// kChunks = 16-byte chunks per lane.
// ---------------------------------------------------------------------------
constexpr int kSeamThreads = 256;

namespace {

template <int kChunks>
__device__ inline void norm_row(float (&v)[kChunks][8], const SeamNorm& n, int lane, int nchunk, float inv_c) {
  float mean = 0.f;
  if (n.kind == AGG_NORM_LAYER) {
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      if (lane + 64 * c < nchunk)
#pragma unroll
        for (int i = 0; i < 8; ++i) mean += v[c][i];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) mean += __shfl_xor(mean, o);
    mean *= inv_c;
  }
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < kChunks; ++c)
    if (lane + 64 * c < nchunk)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[c][i] -= mean;
        sq += v[c][i] * v[c][i];
      }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) sq += __shfl_xor(sq, o);
  const float r = rsqrtf(sq * inv_c + n.eps);
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int ch = lane + 64 * c;
    if (ch < nchunk) {
      float g[8], b[8];
      load8(n.gamma, ch * 8, 1.f, g);
      load8(n.beta, ch * 8, 0.f, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * r * g[i] + b[i];
    }
  }
}

}  // namespace

template <int kChunks>
__global__ __launch_bounds__(kSeamThreads) void seam_kernel(SeamArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (kSeamThreads / 64) + (threadIdx.x >> 6);
  if (row >= a.rows) return;
  const int nchunk = a.C / 8;
  const float inv_c = 1.f / (float)a.C;
  float v[kChunks][8];
  u32x4 xr[kChunks];
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int ch = lane + 64 * c;
    if (ch < nchunk) {
      xr[c] = *reinterpret_cast<const u32x4*>(a.x + row * a.C + ch * 8);
      if (a.branch) unpack8(*reinterpret_cast<const u32x4*>(a.branch + row * a.C + ch * 8), v[c]);
    }
  }
  if (a.branch) {
    if (a.post.kind != AGG_NORM_NONE) norm_row<kChunks>(v, a.post, lane, nchunk, inv_c);
    const uint16_t* gate = a.gate ? a.gate + row / a.gate_rows * a.C : nullptr;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int ch = lane + 64 * c;
      if (ch < nchunk) {
        float s[8], x[8];
        load8(a.scale, ch * 8, 1.f, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= s[i];
        if (gate) {
          unpack8(*reinterpret_cast<const u32x4*>(gate + ch * 8), s);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[c][i] *= s[i];
        }
        unpack8(xr[c], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] += x[i];
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      if (lane + 64 * c < nchunk) unpack8(xr[c], v[c]);
  }
  if (a.h) {
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      if (lane + 64 * c < nchunk)
        *reinterpret_cast<u32x4*>(a.h + row * a.C + (lane + 64 * c) * 8) = pack8(v[c]);
  }
  if (a.pre.kind != AGG_NORM_NONE) {
    norm_row<kChunks>(v, a.pre, lane, nchunk, inv_c);
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      if (lane + 64 * c < nchunk)
        *reinterpret_cast<u32x4*>(a.n + row * a.C + (lane + 64 * c) * 8) = pack8(v[c]);
  }
}

hipError_t launch_seam(const SeamArgs& a, hipStream_t st) {
  const int64_t groups = (a.rows + kSeamThreads / 64 - 1) / (kSeamThreads / 64);
  if (groups > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)groups), block(kSeamThreads);
  (void)hipGetLastError();
  if (a.C <= 512 * 2) hipLaunchKernelGGL(seam_kernel<2>, grid, block, 0, st, a);
  else if (a.C <= 512 * 4) hipLaunchKernelGGL(seam_kernel<4>, grid, block, 0, st, a);
  else if (a.C <= 512 * 8) hipLaunchKernelGGL(seam_kernel<8>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(seam_kernel<16>, grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace agg
