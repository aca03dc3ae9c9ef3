// Loads and stores of 16 bytes through the caches or past them, for passes that touch a tensor once.
//
// Past them (nontemporal) where a call's tensors are larger than what stays in the caches until the next call
// reads them: 64 MiB each, a few of which fill the 256 MiB behind the L2s.  Measured at 137 400 rows of 1024 channels (281 MB):
// quantisation and reading back 134 -> 109 us, a seam 215 -> 200, a block in 4 bits 1567 -> 1534.  Below that the next call
// finds its input in the caches: with the norm of 21 984 rows stored past them a block in bf16 takes 360 us instead
// of 351, and loads past them are slower from there (5496 rows: 13.3 instead of 11.7 us).  What is read again only much later (the
// residual sum, until the next seam) is always stored past them: 21 984 rows 36.6 -> 35.1 us, blocks the same or 1 % faster.
// So are, by their own measurements, the rotary calls' queries and keys and the 4-bit products' results (rope_kernel,
// mx4_tile_kernel).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace agg {

inline bool streams(int64_t tensor_bytes) { return tensor_bytes > ((int64_t)64 << 20); }

// A template's parameter, not an argument: of two sides that differ in nothing else the compiler makes one
// ordinary access.
typedef uint32_t stream16 __attribute__((ext_vector_type(4)));
template <bool kStream>
__device__ __forceinline__ stream16 load16(const void* p) {
  const stream16* q = reinterpret_cast<const stream16*>(p);
  if constexpr (kStream) return __builtin_nontemporal_load(q);
  else return *q;
}
template <bool kStream>
__device__ __forceinline__ void store16(void* p, stream16 v) {
  stream16* q = reinterpret_cast<stream16*>(p);
  if constexpr (kStream) __builtin_nontemporal_store(v, q);
  else *q = v;
}

}  // namespace agg
