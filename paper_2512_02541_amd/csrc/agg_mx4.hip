// Microscaled 4-bit floats: quantisation, reading back, and the product of two matrices held so.
#include "agg_internal.h"

namespace agg {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

namespace {

__device__ inline uint32_t pack2(float lo, float hi) {
  f32x2 p = {lo, hi};
  bf16x2 h = __builtin_convertvector(p, bf16x2);
  return __builtin_bit_cast(uint32_t, h);
}
// (by value: a cast of a vector's element itself takes the vector's first)
__device__ inline bf16x2 as_pair(uint32_t w) { return __builtin_bit_cast(bf16x2, w); }
__device__ inline float bf16_of(uint32_t bits) { return __uint_as_float(bits << 16); }

}  // namespace

// ---------------------------------------------------------------------------
// Quantisation: a lane holds eight channels, four lanes a block of 32.  The largest magnitude of a
// block is the largest of the bf16 patterns without their signs (their order is that of the values,
// NaN and infinity last), and its exponent field minus 2 is the scale's byte; the conversion
// instruction divides by the scale and rounds to the nearest, ties to even, saturating.  (For a
// scale byte of 0 the float with exponent field 0 stands for 2^-127: all 255 scales and all finite bf16
// values were compared with the definition.)  One wavefront per row; HBM-bound.
// ---------------------------------------------------------------------------
constexpr int kQuantThreads = 256;

__global__ __launch_bounds__(kQuantThreads) void mx4_quantize_kernel(
    const uint16_t* __restrict__ x, int64_t x_stride, uint32_t* __restrict__ codes,
    uint8_t* __restrict__ scales, int64_t rows, int K, int words, int scale_stride) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (kQuantThreads / 64) + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int nchunk = K / 8;
  for (int w = lane; w < words; w += 64) {  // words: a multiple of 32, so four lanes leave together
    u32x4 v = {0u, 0u, 0u, 0u};
    if (w < nchunk) v = *reinterpret_cast<const u32x4*>(x + row * x_stride + w * 8);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, max(v[i] & 0x7FFFu, (v[i] >> 16) & 0x7FFFu));
    most = max(most, (uint32_t)__shfl_xor((int)most, 1));
    most = max(most, (uint32_t)__shfl_xor((int)most, 2));
    const uint32_t e = most >> 7;  // 255: NaN or infinity in the block
    const uint32_t s = e == 255 ? 255u : (e > 2 ? e - 2 : 0u);
    uint32_t code = 0;
    if (s != 255) {
      const float scale = __uint_as_float(s << 23);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(v[0]), scale, 0);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(v[1]), scale, 1);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(v[2]), scale, 2);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, as_pair(v[3]), scale, 3);
    }
    codes[row * words + w] = code;
    if ((w & 3) == 0) scales[row * scale_stride + w / 4] = (uint8_t)s;
  }
  // the scales behind the row's last whole run of codes
  for (int i = words / 4 + lane; i < scale_stride; i += 64) scales[row * scale_stride + i] = 0;
}

__global__ __launch_bounds__(kQuantThreads) void mx4_dequantize_kernel(
    const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, uint16_t* __restrict__ x,
    int64_t rows, int K, int words, int scale_stride) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (kQuantThreads / 64) + (threadIdx.x >> 6);
  if (row >= rows) return;
  for (int w = lane; w < K / 8; w += 64) {
    const uint32_t code = codes[row * words + w];
    const uint32_t s = scales[row * scale_stride + w / 4];
    const float scale = __uint_as_float(s << 23);
    u32x4 v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
    if (s == 255) v = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
    *reinterpret_cast<u32x4*>(x + row * K + w * 8) = v;
  }
}

// ---------------------------------------------------------------------------
// Product  Y[m, n] = sum_k A[m, k] W[n, k] + bias[n]  on v_mfma_scale_f32_16x16x128_f8f6f4 with both operands in 4
// bits: a lane holds the 32 channels of one scale (16 bytes) of one row, group G = lane / 16 of the
// lanes the G-th block of the 128.  The padding behind K is zeros, so no product needs a limit in k.
// A wavefront owns 32 tokens x 64 channels and reads its fragments straight from memory; W's rows are taken in an order
// that leaves a lane with four consecutive channels of a token.
// ---------------------------------------------------------------------------
constexpr int kMxThreads = 256;

__global__ __launch_bounds__(kMxThreads) void mx4_linear_kernel(Mx4LinearArgs p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane & 15, G = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.x * 64 + (wave & 1) * 32;
  const int which = blockIdx.y / p.gn;
  const int n0 = (blockIdx.y % p.gn) * 128 + (wave >> 1) * 64;
  if (m0 >= p.rows || n0 >= p.N) return;
  const uint8_t *a[2], *as[2], *w[4], *ws[4];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int64_t m = min(m0 + 16 * t + c, p.rows - 1);
    a[t] = p.a.codes + m * p.code_stride + G * 16;
    as[t] = p.a.scales + m * p.scale_stride + G;
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int n = min(n0 + 4 * c + t, p.N - 1);
    w[t] = p.w[which].codes + (int64_t)n * p.code_stride + G * 16;
    ws[t] = p.w[which].scales + (int64_t)n * p.scale_stride + G;
  }
  f32x4 acc[2][4];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = p.code_stride / 64;  // of 128 channels
  for (int s = 0; s < steps; ++s) {
    i32x8 fa[2], fw[4];
    int sa[2], sw[4];
    auto frag = [](const uint8_t* q) {
      const u32x4 u = *reinterpret_cast<const u32x4*>(q);
      return i32x8{(int)u[0], (int)u[1], (int)u[2], (int)u[3], 0, 0, 0, 0};
    };
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      fa[t] = frag(a[t] + s * 64);
      sa[t] = as[t][s * 4];
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      fw[t] = frag(w[t] + s * 64);
      sw[t] = ws[t][s * 4];
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        acc[t][u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[t], fw[u], acc[t][u], 4, 4, 0, sa[t], 0, sw[u]);
  }
  const int n = n0 + 4 * c;
  if (n >= p.N) return;  // N is a multiple of 8: all four channels exist or none
  float bias[4] = {0.f, 0.f, 0.f, 0.f}, scale[4] = {1.f, 1.f, 1.f, 1.f};
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (p.bias[which]) bias[u] = p.bias[which][n + u];
    if (p.res_scale) scale[u] = p.res_scale[n + u];
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t m = m0 + 16 * t + 4 * G + r;
      if (m >= p.rows) continue;
      float y[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) y[u] = acc[t][u][r] + bias[u];
      if (p.residual) {
        const uint2 x = *reinterpret_cast<const uint2*>(p.residual + m * p.N + n);
        y[0] = bf16_of(x.x & 0xFFFFu) + scale[0] * y[0];
        y[1] = bf16_of(x.x >> 16) + scale[1] * y[1];
        y[2] = bf16_of(x.y & 0xFFFFu) + scale[2] * y[2];
        y[3] = bf16_of(x.y >> 16) + scale[3] * y[3];
      }
      *reinterpret_cast<uint2*>(p.y[which] + m * p.N + n) = uint2{pack2(y[0], y[1]), pack2(y[2], y[3])};
    }
}

static inline int64_t row_groups(int64_t rows) { return (rows + kQuantThreads / 64 - 1) / (kQuantThreads / 64); }

hipError_t launch_mx4_quantize(const void* x, int64_t x_stride, void* codes, void* scales, int64_t rows, int K,
                               hipStream_t st) {
  if (row_groups(rows) > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
  (void)hipGetLastError();
  hipLaunchKernelGGL(mx4_quantize_kernel, dim3((unsigned)row_groups(rows)), dim3(kQuantThreads), 0, st,
                     (const uint16_t*)x, x_stride, (uint32_t*)codes, (uint8_t*)scales, rows, K,
                     (int)(mx4_code_stride(K) / 4), (int)mx4_scale_stride(K));
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const void* codes, const void* scales, void* x, int64_t rows, int K, hipStream_t st) {
  if (row_groups(rows) > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
  (void)hipGetLastError();
  hipLaunchKernelGGL(mx4_dequantize_kernel, dim3((unsigned)row_groups(rows)), dim3(kQuantThreads), 0, st,
                     (const uint32_t*)codes, (const uint8_t*)scales, (uint16_t*)x, rows, K,
                     (int)(mx4_code_stride(K) / 4), (int)mx4_scale_stride(K));
  return hipGetLastError();
}

hipError_t launch_mx4_linear(const Mx4LinearArgs& args, hipStream_t st) {
  Mx4LinearArgs p = args;
  p.gn = (p.N + 127) / 128;
  const int64_t gm = (p.rows + 63) / 64;
  if (gm > 0x7FFFFFFF || (int64_t)p.gn * p.count > 65535) return hipErrorInvalidConfiguration;
  (void)hipGetLastError();
  hipLaunchKernelGGL(mx4_linear_kernel, dim3((unsigned)gm, (unsigned)(p.gn * p.count)), dim3(kMxThreads), 0, st, p);
  return hipGetLastError();
}

}  // namespace agg
