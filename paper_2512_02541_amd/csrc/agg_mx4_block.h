// A lane's eight channels in 4 bits, where four neighbouring lanes hold a block of 32: the largest magnitude of a
// block is the largest of the bf16 patterns without their signs (their order is that of the values,
// NaN and infinity last), and its exponent field minus 2 is the scale's byte; the conversion
// instruction divides by the scale and rounds to the nearest, ties to even, saturating.  (For a
// scale byte of 0 the float with exponent field 0 stands for 2^-127: all 255 scales and all finite bf16
// values were compared with the definition.)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace agg {

typedef __bf16 mx4_pair __attribute__((ext_vector_type(2)));
typedef uint32_t mx4_chunk __attribute__((ext_vector_type(4)));
// (by value: a cast of a vector's element itself takes the vector's first)
__device__ inline mx4_pair as_pair(uint32_t w) { return __builtin_bit_cast(mx4_pair, w); }

// Codes of v's channels, lowest first; s: their block's scale, 255 (and codes 0) with a NaN or an infinity in the block.
__device__ __forceinline__ uint32_t mx4_codes(mx4_chunk v, uint32_t& s) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) most = max(most, max(v[i] & 0x7FFFu, (v[i] >> 16) & 0x7FFFu));
  most = max(most, (uint32_t)__shfl_xor((int)most, 1));
  most = max(most, (uint32_t)__shfl_xor((int)most, 2));
  const uint32_t e = most >> 7;
  s = e == 255 ? 255u : (e > 2 ? e - 2 : 0u);
  uint32_t code = 0;
  if (s != 255) {
    const float scale = __uint_as_float(s << 23);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(v[0]), scale, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(v[1]), scale, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(v[2]), scale, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(v[3]), scale, 3);
  }
  return code;
}

}  // namespace agg
