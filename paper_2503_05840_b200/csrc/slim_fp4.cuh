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
// 6 s >= amax.  6 s has at most six significant bits, so the comparison is exact.  amax / 6 is rounded down, both times; it
// cannot fall behind a scale that lies below amax / 6 itself, because amax (a bf16 number, of eight bits) is 6 s or
// further than 2^-8 of it away.
__device__ __forceinline__ int slim_fp4_scale_byte(float amax, bool bad) {
  if (bad) return FP4_SCALE_NAN;
  const float want = __fmul_rz(fminf(amax, 61440.f), 0x1.555554p-3f);      // (the float32 below 1/6)
  int b = (int)(__half_as_ushort(__float2half_rz(want)) >> 7);     // the scale or the one before it
  if (b < FP4_SCALE_MAX && 6.f * slim_fp4_scale((unsigned char)b) < amax) ++b;
  return b;
}
// eight codes -> four float16 pairs
__device__ __forceinline__ void slim_fp4_decode8(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// eight numbers -> codes, to nearest, on a border to the even code
__device__ __forceinline__ uint32_t slim_fp4_encode8(const float (&y)[8]) {
  uint32_t d;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tcvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\tmov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(d) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return d;
}
#endif

cudaError_t slim_launch_fp4_decode(const slim_ctx* ctx, const SlimDecodeParams& p, float* scores, cudaStream_t st);
// tensor cores (slim_fp4_tc.cu): pairs of CTAs that fit the device, 0 = not this shape; umax: [units][H] scratch
int slim_fp4_tc_workers(const slim_ctx* ctx);
cudaError_t slim_fp4_tc_make_tmaps(const slim_ctx* ctx, slim_cache* c);       // codes in tmap[0], scales in tmap[1]
cudaError_t slim_launch_fp4_tc(const slim_ctx* ctx, const slim_cache* c, const SlimDecodeParams& p, float* umax, cudaStream_t st);
