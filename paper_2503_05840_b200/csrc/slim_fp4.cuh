// The 4-bit K-cache format (SLIM_FP4), shared by the kernels that write, read and attend over such a cache.
//
// A key is an E2M1 code (sign, then 0, 0.5, 1, 1.5, 2, 3, 4 or 6) times the scale of its group of 32 columns of the row.
// The scale is a byte: the upper bits of a float16 without its sign (five exponent bits, three of the mantissa), so
// byte << 7 are the bits of the scale as a float16.  The smallest scale s with 6 s >= max |k| is taken, so that no key of
// a group saturates (above 6 * 10240 all do).  Code times scale has six significant bits and lies in [2^-18, 61440]: it is
// exact in float16 and in bfloat16.  A group that holds a number that is not finite has the scale byte 0xff, a NaN.
#pragma once
#include <cuda_fp16.h>

#include "slim_internal.h"

constexpr int FP4_GROUP = 32;                  // columns of a row that share a scale
constexpr int FP4_SCALE_MAX = 0xe2;            // 10240: 6 * 10240 is still finite in float16
constexpr int FP4_SCALE_NAN = 0xff;

__host__ __device__ inline int slim_fp4_code_pitch(int d) { return (d / 2 + 15) & ~15; }                                  // bytes of a row's codes
__host__ __device__ inline int slim_fp4_scale_pitch(int d) { return ((d + FP4_GROUP - 1) / FP4_GROUP + 15) & ~15; }      // and of its scales

#ifdef __CUDACC__
__device__ __forceinline__ float slim_fp4_scale(unsigned char byte) {
  return __half2float(__ushort_as_half((unsigned short)((unsigned)byte << 7)));
}
// magnitude of a code, times two: 0 1 2 3 4 6 8 12
__device__ __forceinline__ float slim_fp4_value(unsigned code) {
  const unsigned m = code & 7u;
  const float v = 0.5f * (float)((0xc8643210u >> (4 * m)) & 15u);
  return code & 8u ? -v : v;
}
// column `col` of the row whose codes and scales start at c and s
__device__ __forceinline__ float slim_fp4_at(const unsigned char* c, const unsigned char* s, int col) {
  const unsigned byte = __ldg(c + (col >> 1));
  return slim_fp4_value(col & 1 ? byte >> 4 : byte & 15u) * slim_fp4_scale(__ldg(s + col / FP4_GROUP));
}

// Scale byte of a group whose largest magnitude is amax (bad: it holds a number that is not finite): the smallest s with
// 6 s >= amax.  6 s has at most six significant bits, so the comparison is exact.
__device__ __forceinline__ int slim_fp4_scale_byte(float amax, bool bad) {
  if (bad) return FP4_SCALE_NAN;
  const float want = fminf(amax, 61440.f) * (1.f / 6.f);
  int b = (int)(__half_as_ushort(__float2half_rz(want)) >> 7);     // at most one step off, either way
  if (b > 0 && 6.f * slim_fp4_scale((unsigned char)(b - 1)) >= amax) --b;
  if (b < FP4_SCALE_MAX && 6.f * slim_fp4_scale((unsigned char)b) < amax) ++b;
  return b;
}
// Code of k under the scale s: the nearest of the eight magnitudes times s, on a border the even code.  The borders
// (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5) s are exact in float32, so no division and no rounding of a quotient is needed.
__device__ __forceinline__ unsigned slim_fp4_code(float k, float s) {
  const float a = fabsf(k);
  const bool upper = a >= 1.75f * s;                               // codes 4 .. 7
  const float b1 = upper ? 3.5f * s : 0.75f * s;                   // on it: up to the even code 6 or 2
  const bool u1 = a >= b1;
  const float b0 = upper ? (u1 ? 5.f * s : 2.5f * s) : (u1 ? 1.25f * s : 0.25f * s);      // on it: down, to 6, 4, 2 or 0
  const unsigned m = (upper ? 4u : 0u) + (u1 ? 2u : 0u) + (a > b0 ? 1u : 0u);
  return m && a > 0.f ? m | (k < 0.f ? 8u : 0u) : 0u;           // (all borders are 0 in a group of zeros)
}
#endif

cudaError_t slim_launch_fp4_decode(const slim_ctx* ctx, const SlimDecodeParams& p, float* scores, cudaStream_t st);
// tensor cores (slim_fp4_tc.cu): pairs of CTAs that fit the device, 0 = not this shape; umax: [units][H] scratch
int slim_fp4_tc_workers(const slim_ctx* ctx);
cudaError_t slim_fp4_tc_make_tmaps(const slim_ctx* ctx, slim_cache* c);       // codes in tmap[0], scales in tmap[1]
cudaError_t slim_launch_fp4_tc(const slim_ctx* ctx, const slim_cache* c, const SlimDecodeParams& p, float* umax, cudaStream_t st);
