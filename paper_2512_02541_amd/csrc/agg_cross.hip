// Attention of queries to keys and values of another length, lying where they are or in the pages of a cache.
#include "agg_attn_pipe.h"
#include "agg_cross_plan.h"

namespace agg {

namespace {

typedef const __attribute__((address_space(4))) int32_t* ScalarInts;

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

// where a split's results of a pair's row lie in the workspace: 64 floats of a row, behind them all {reference, sum} of each
__device__ __forceinline__ int64_t partial_row(const CrossArgs& a, int64_t pairs, int split, int64_t pair, uint32_t row) {
  return ((int64_t)split * pairs + pair) * ((int64_t)a.NQ * a.group) + row;
}

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
// Few rows a pair: bound by the keys and values, which are read once.  Every wavefront takes 32-key blocks of its own, straight into
// registers (a page's fragment order is the order of the matrix instruction's operands; rows read in place need one turn of the
// values through LDS), with the running maximum and sum of an online softmax; the wavefronts of a workgroup, and the
// workgroups that share a pair's keys, are joined at the end by their references.
// ---------------------------------------------------------------------------
constexpr int few_threads(int tiles) { return 64 * (tiles == 4 ? 4 : kFewWaves); }
constexpr int kRowFloats = kHeadDim + 4;  // of a row in LDS, padded

template <bool kPaged, int kJ>
__global__ __launch_bounds__(few_threads(kJ), kJ == 1 ? 4 : 2) void cross_few_kernel(CrossArgs a, CrossPlan plan, int64_t pairs,
                                                                                    int64_t first) {
  constexpr int kW = few_threads(kJ) / 64;
  __shared__ __align__(16) float lds[kW * 16 * kJ * (kRowFloats + 2)];
  static_assert(sizeof(lds) >= kW * 4096, "a block of values for each wavefront");
  const int lane = threadIdx.x & 63, c = lane & 15, G = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = first + blockIdx.x;
  const int64_t pair = id % pairs;
  const int split = (int)(id / pairs % plan.splits);
  const int b = (int)(pair / a.H_kv), hk = (int)(pair % a.H_kv);
  const int n = cross_keys(a, b);
  const uint32_t rows = (uint32_t)cross_queries(a, b) * (uint32_t)a.group;
  const uint32_t r0 = (uint32_t)(id / pairs / plan.splits) * (16 * kJ);
  if (r0 >= rows) return;
  const int64_t blocks = ((int64_t)n + kKeyBlock - 1) / kKeyBlock;
  const int lo = (int)(blocks * split / plan.splits), hi = (int)(blocks * (split + 1) / plan.splits);

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
  float m[kJ], l[kJ];  // m: largest logit so far, base 2; l: this lane's part of the sum
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
      if (left < kKeyBlock) {  // what lies behind the last key may be anything: 0 times it may be no number
        const int k0 = 16 * (G >> 1) + 4 * (G & 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = k0 + (i >> 1) * 8 + (i & 1) * 2;
          const uint32_t mask = (key < left ? 0xFFFFu : 0u) | (key + 1 < left ? 0xFFFF0000u : 0u);
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) V[dt].u[i] &= mask;
        }
      }
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
      const float now = fmaxf(m[j], quad_max(top) * a.scale2);
      const float ref = now == -INFINITY ? 0.f : now;  // (logits may be -infinity)
      const float f = fast_exp2(m[j] - ref);
      m[j] = now;
      l[j] *= f;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) O[j][dt] *= f;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float e0 = fast_exp2(fmaf(S[kJ * kt + j][2 * i], a.scale2, -ref));
          const float e1 = fast_exp2(fmaf(S[kJ * kt + j][2 * i + 1], a.scale2, -ref));
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
      const float f = fast_exp2(s[0] - ref);
      total += s[1] * f;
      o += *reinterpret_cast<const f32x4*>(lds + (w * 16 * kJ + row) * kRowFloats + 4 * quad) * f;
    }
    if (plan.splits == 1) {
      store_row(a, b, hk, r0 + row, quad, ref, total, o, n == 0);
    } else {
      const int64_t at = partial_row(a, pairs, split, pair, r0 + row);
      *reinterpret_cast<f32x4*>(a.partial + at * kHeadDim + 4 * quad) = o;
      if (quad == 0) {
        float* const s = a.partial + (int64_t)plan.splits * pairs * a.NQ * a.group * kHeadDim + at * 2;
        *reinterpret_cast<f32x2*>(s) = f32x2{hi > lo ? ref : -INFINITY, total};
      }
    }
  }
}

// Joins the splits' results: sixteen threads a row.
constexpr int kJoinThreads = 256;
__global__ __launch_bounds__(kJoinThreads) void cross_join_kernel(CrossArgs a, int splits, int64_t pairs, int64_t first) {
  const int64_t all = (int64_t)a.NQ * a.group;
  const int64_t at = first + (int64_t)blockIdx.x * (kJoinThreads / 16) + (threadIdx.x >> 4);
  const int quad = threadIdx.x & 15;
  if (at >= pairs * all) return;
  const int64_t pair = at / all;
  const uint32_t row = (uint32_t)(at - pair * all);
  const int b = (int)(pair / a.H_kv), hk = (int)(pair % a.H_kv);
  if (row >= (uint32_t)cross_queries(a, b) * (uint32_t)a.group) return;
  const f32x2* const sums = reinterpret_cast<const f32x2*>(a.partial + (int64_t)splits * pairs * all * kHeadDim);
  float top = -INFINITY;
  for (int s = 0; s < splits; ++s) top = fmaxf(top, sums[at + (int64_t)s * pairs * all][0]);
  const float ref = top == -INFINITY ? 0.f : top;
  float total = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    const int64_t p = at + (int64_t)s * pairs * all;
    const f32x2 x = sums[p];
    const float f = fast_exp2(x[0] - ref);  // 0 for a split without keys
    total += x[1] * f;
    o += *reinterpret_cast<const f32x4*>(a.partial + p * kHeadDim + 4 * quad) * f;
  }
  store_row(a, b, hk, row, quad, ref, total, o, cross_keys(a, b) == 0);
}

size_t cross_partial_floats(int64_t B, int64_t NQ, int64_t NK, int64_t H, int64_t H_kv) {
  const int64_t pairs = B * H_kv, rows = NQ * (H / H_kv);
  const CrossPlan p = plan_cross(pairs, rows, NK);
  return p.splits > 1 ? (size_t)p.splits * pairs * rows * (kHeadDim + 2) : 0;
}

template <bool kPaged>
static void launch_few(const CrossArgs& a, const CrossPlan& p, int64_t pairs, hipStream_t st) {
  const int64_t groups = pairs * p.row_tiles * p.splits;
  constexpr int64_t kMost = 1 << 22;  // workgroups of a launch (kLaunchRows)
  for (int64_t first = 0; first < groups; first += kMost) {
    const dim3 grid((unsigned)(groups - first < kMost ? groups - first : kMost));
    if (p.tiles == 1) hipLaunchKernelGGL((cross_few_kernel<kPaged, 1>), grid, dim3(few_threads(1)), 0, st, a, p, pairs, first);
    else if (p.tiles == 2) hipLaunchKernelGGL((cross_few_kernel<kPaged, 2>), grid, dim3(few_threads(2)), 0, st, a, p, pairs, first);
    else hipLaunchKernelGGL((cross_few_kernel<kPaged, 4>), grid, dim3(few_threads(4)), 0, st, a, p, pairs, first);
  }
}

hipError_t launch_cross(const CrossArgs& a, hipStream_t st) {
  const int64_t pairs = (int64_t)a.B * a.H_kv, rows = (int64_t)a.NQ * a.group;
  const CrossPlan p = plan_cross(pairs, rows, a.NK);
  (void)hipGetLastError();
  if (a.pages) launch_few<true>(a, p, pairs, st);
  else launch_few<false>(a, p, pairs, st);
  if (p.splits > 1) {
    constexpr int64_t kRows = kJoinThreads / 16, kMost = kRows << 22;
    for (int64_t first = 0; first < pairs * rows; first += kMost) {
      const int64_t here = pairs * rows - first < kMost ? pairs * rows - first : kMost;
      hipLaunchKernelGGL(cross_join_kernel, dim3((unsigned)((here + kRows - 1) / kRows)), dim3(kJoinThreads), 0, st, a, p.splits,
                         pairs, first);
    }
  }
  return hipGetLastError();
}

}  // namespace agg
