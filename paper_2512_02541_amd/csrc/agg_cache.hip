// New tokens of a paged key/value cache: norm and rotary positions of keys (and queries) on the way, keys and values into
// the fragment order of their pages.
#include "agg_internal.h"
#include "agg_lds_copy.h"
#include "agg_rows.h"

namespace agg {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// A workgroup takes 32 consecutive rows: half a page of a sequence (keys and values) or 32 tokens (queries).  It works out
// their cosines and signed sines once, a pair of channels a thread, and its wavefronts take the heads in turn, eight lanes a
// row of a head.  A key's 16-byte chunk goes to the page from the registers it was turned in: eight consecutive rows make a
// whole 128-byte line of one chunk number.  Values turn through LDS with the transposing read, which leaves a lane with
// the eight rows of one channel that make a chunk of the page; a chunk that the new rows fill only in part is
// stored element by element, so that its other rows stay.
// ---------------------------------------------------------------------------
constexpr int kAppendThreads = 256;
constexpr int kAppendWaves = kAppendThreads / 64;
constexpr int kAppendRows = 32;
constexpr int kHeadStride = kHeadDim + 4;  // floats of a head in LDS: 16-byte aligned rows

namespace {

// What a lane knows of its eight channels of any row.
struct Channels {
  int other[8];     // each channel's other one
  uint32_t turned;  // whether it turns at all
  float gamma[8], beta[8];
  int kind;
  float eps;
};

// norm and rotation of a row's eight channels; head: floats of this group of eight lanes, turns: the row's table
__device__ __forceinline__ void turn8(float (&x)[8], const Channels& ch, bool turns_any, int c0, float* head, const f32x2* turns) {
  if (ch.kind != AGG_NORM_NONE) {
    float mean = 0.f;
    if (ch.kind == AGG_NORM_LAYER) {
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
    const float r = rsqrtf(sum_of_8(sq) * (1.f / kHeadDim) + ch.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * ch.gamma[i] + ch.beta[i];
  }
  if (!turns_any) return;
  wave_lds_fence();
  *reinterpret_cast<f32x4*>(head + c0) = f32x4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4*>(head + c0 + 4) = f32x4{x[4], x[5], x[6], x[7]};
  wave_lds_fence();
  f32x4 cs[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) cs[i] = *reinterpret_cast<const f32x4*>(turns + c0 + 2 * i);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = x[i] * cs[i / 2][i % 2 * 2] + head[ch.other[i]] * cs[i / 2][i % 2 * 2 + 1];
    x[i] = (ch.turned >> i) & 1 ? y : x[i];  // by selection: an infinity times 0 is none of the other channels' business
  }
}

}  // namespace

__global__ __launch_bounds__(kAppendThreads, 3) void append_kernel(AppendArgs a) {
  __shared__ __align__(16) f32x2 turns[kAppendRows][kHeadDim];
  __shared__ __align__(16) float heads[kAppendWaves][8][kHeadStride];
  __shared__ __align__(16) uint16_t values[kAppendWaves][kAppendRows * kHeadDim];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row8 = lane >> 3, j = lane & 7, c0 = j * 8;  // this lane's row of eight, chunk of a head, first channel
  const RopeArgs& r = a.r;
  const int T = (int)r.NQ;

  Channels ch;
  const uint64_t others = *reinterpret_cast<const uint64_t*>(r.other + c0);
  ch.turned = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    ch.other[i] = (int)(others >> (8 * i)) & 63;
    if ((others >> (8 * i)) & 0x80) ch.turned |= 1u << i;
  }
  // this thread's pair of every eighth row's
  const int p = threadIdx.x % (kHeadDim / 2);
  const int axis = r.axis[p], lo = r.first[p], hi = r.second[p];
  const uint64_t freq = r.freq[p];
  float* const head = heads[wave][row8];
  if (r.pairs && r.pairs < kHeadDim / 2)  // channels that no pair writes
    for (int i = threadIdx.x; i < kAppendRows * kHeadDim; i += kAppendThreads)
      if (!(r.other[i % kHeadDim] & 0x80)) turns[i / kHeadDim][i % kHeadDim] = f32x2{1.f, 0.f};

  for (int64_t item = blockIdx.x; item < a.k_items + a.q_items; item += gridDim.x) {
    const bool keys = item < a.k_items;
    const uint32_t it = (uint32_t)(keys ? item : item - a.k_items);  // fewer than 2^32 of either (launch_append)
    const uint32_t parts = keys ? a.k_parts : a.q_parts, units = keys ? a.k_units : a.q_units;
    const int part = (int)(it % parts), unit = (int)(it / parts % units), b = (int)(it / parts / units);
    // rows of the unit: key rows of the cache, which are tokens from start on; or tokens
    const int64_t start = keys && a.start ? ((ScalarInts)a.start)[b] : 0;
    const int count = a.counts ? min(max(((ScalarInts)a.counts)[b], 0), T) : T;
    const int64_t cap = (int64_t)a.max_pages * kTileRows;
    const int64_t row0 = (keys ? max(start, (int64_t)0) / kAppendRows : 0) * kAppendRows + (int64_t)unit * kAppendRows;
    const int64_t tok0 = row0 - start;  // the unit's first row is this token
    if (keys && unit == 0 && part == 0 && threadIdx.x == 0 && a.lens)
      a.lens[b] = (int32_t)min(max(start + count, (int64_t)0), cap);
    // the unit's rows that exist: from .. to - 1
    const int from = (int)min(max(-tok0, (int64_t)0), (int64_t)kAppendRows);
    int64_t end = count - tok0;
    if (keys) end = min(end, cap - row0);
    const int to = (int)min(max(end, (int64_t)0), (int64_t)kAppendRows);
    if (from >= to) continue;
    const int page = keys ? ((ScalarInts)a.pages)[(int64_t)b * a.max_pages + row0 / kTileRows] : 0;
    if (keys && (page < 0 || page >= a.n_pages)) continue;

    // a head's rows are requested a head ahead, the first ones before the table of turns is worked out
    const int which = keys ? 1 : 0;
    const int H = keys ? a.H_kv : r.H;
    const int64_t tok_first = (int64_t)b * T + tok0;
    const uint16_t* const in = r.in[which] + (tok_first + row8) * r.stride[which] + c0;
    const uint16_t* const in_v = a.V + (tok_first + row8) * a.v_stride + c0;
    u32x4 raw[4], val[4];
    auto exists = [&](int i) { return 8 * i + row8 >= from && 8 * i + row8 < to; };
    auto request = [&](int h, int i) {
      raw[i] = u32x4{0u, 0u, 0u, 0u};
      if (exists(i)) raw[i] = *reinterpret_cast<const u32x4*>(in + 8 * i * r.stride[which] + h * kHeadDim);
    };
    auto request_v = [&](int h, int i) {
      val[i] = u32x4{0u, 0u, 0u, 0u};
      if (exists(i)) val[i] = *reinterpret_cast<const u32x4*>(in_v + 8 * i * a.v_stride + h * kHeadDim);
    };
    const int step = (int)parts * kAppendWaves;
    int h = part * kAppendWaves + wave;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (h < H) request(h, i);
      if (keys && h < H) request_v(h, i);
    }
    ch.kind = r.norm[which].kind;
    ch.eps = r.norm[which].eps;
    load8(r.norm[which].gamma, c0, 1.f, ch.gamma);
    load8(r.norm[which].beta, c0, 0.f, ch.beta);

    if (r.pairs) {
      __syncthreads();  // the last unit's reads are done
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
          float s, c;
          sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &s, &c);
          turns[row][lo] = f32x2{c, -s};
          turns[row][hi] = f32x2{c, s};
        }
      }
      __syncthreads();
    }

    for (; h < H; h += step) {
      const int64_t tile = ((int64_t)page * a.H_kv + h) * kTileElems + (row0 % kTileRows) * kHeadDim;
      // values, row-major with the upper half of a row's chunks exchanged with the lower on rows 2 and 3 mod 4 (the
      // transposing read's four rows then lie on different banks)
      lds_char* const v = (lds_char*)values[wave];
      if (keys) {
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = 8 * i + row8;
          *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(v + row * 128 + (j ^ (4 * ((row >> 1) & 1))) * 16) = val[i];
          if (h + step < H) request_v(h + step, i);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (8 * i >= to || 8 * i + 8 <= from) continue;
        const int row = 8 * i + row8;
        float x[8];
        unpack8(raw[i], x);
        if (h + step < H) request(h + step, i);
        turn8(x, ch, r.pairs != 0, c0, head, turns[row]);
        if (exists(i)) {
          uint16_t* const at = keys ? a.Kc + tile + (j * 32 + row) * 8 : r.out[0] + ((tok_first + row) * H + h) * kHeadDim + c0;
          *reinterpret_cast<u32x4*>(at) = pack8(x);
        }
      }
      if (!keys) continue;
      wave_lds_fence();
      const int c = lane & 15, G = lane >> 4;
      const int k0 = 16 * (G >> 1) + 4 * (G & 1);  // first row of this lane's chunks: k0 .. + 3, k0 + 8 .. + 11
      const int row = k0 + (c >> 2);               // its row of the four that the read transposes
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        lds_char* const at = v + row * 128 + ((2 * dt + ((c & 3) >> 1)) ^ (4 * ((row >> 1) & 1))) * 16 + (c & 1) * 8;
        const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
        const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * 128));
        uint16_t* const to_page = a.Vc + tile + (G * 64 + 16 * dt + c) * 8;
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
    }
  }
}

hipError_t launch_append(const AppendArgs& args, hipStream_t st) {
  AppendArgs a = args;
  const int64_t T = a.r.NQ;
  // a sequence's tokens lie in one more half page than they fill where they begin inside one
  a.k_units = (int32_t)((T + kAppendRows - 1) / kAppendRows + 1);
  a.q_units = a.r.in[0] ? (int32_t)((T + kAppendRows - 1) / kAppendRows) : 0;
  // few rows: their heads are shared out while all workgroups still run at once
  constexpr int64_t kAtOnce = 256 * 3;
  auto share = [&](int64_t units, int heads) {
    int parts = 1;
    const int most = (heads + kAppendWaves - 1) / kAppendWaves;
    while (parts < most && units * (parts + 1) <= kAtOnce) ++parts;
    return parts;
  };
  a.k_parts = share((int64_t)a.B * (a.k_units + a.q_units), a.H_kv);
  a.q_parts = share((int64_t)a.B * (a.k_units + a.q_units), a.r.H);
  a.k_items = (int64_t)a.B * a.k_units * a.k_parts;
  a.q_items = (int64_t)a.B * a.q_units * a.q_parts;
  if (a.k_items > 0xFFFFFFFFll || a.q_items > 0xFFFFFFFFll) return hipErrorInvalidConfiguration;
  const int64_t items = a.k_items + a.q_items;
  constexpr int64_t kMost = 1 << 20;
  (void)hipGetLastError();
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)(items < kMost ? items : kMost)), dim3(kAppendThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace agg
