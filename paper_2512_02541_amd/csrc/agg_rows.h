// Rows of bf16 channels in registers as floats, and sums over the lanes that hold one: what the token-wise kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

// a channel turned with its other one; which product is rounded is said here, so that every kernel rounds the same
__device__ inline float turn_channel(float x, float other, float cosine, float sine) { return fmaf(x, cosine, other * sine); }

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

}  // namespace agg
