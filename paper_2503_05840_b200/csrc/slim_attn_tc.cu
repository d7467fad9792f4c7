// Attention over packed prompts on the tensor cores (bf16, d_k up to 128; heads of other widths than 64, 96 and 128 are widened
// with zeros on their way into the workspace).
//
// attn_tc_values_kernel   float32 values as float16 in the workspace, and the largest of each column.
// attn_tc_prepare_kernel  rotated queries and keys as float16 (11 bits: bf16's 8 would cost as much accuracy as the rounding of P;
//                         without rotation they are read where they lie), the list of query tiles, the columns of values that
//                         need another factor.
// attn_tc_kernel          one CTA a (tile of 2 x 128 query rows, head).  Per key tile of 128 rows and query tile i:
//                           S_i = Q_i K^T       float16 (bf16 without rotation), both operands from shared memory, S in tensor memory
//                           P_i = 2^(S_i - m)   a thread a row: S to registers, maximum, exponentials, P as bf16 over S's
//                                               columns in tensor memory
//                           O_i += P_i V        P from tensor memory, V as it lies (MN-major); bf16 where the values are, float16
//                                               where they were float32 (a second rounding to 8 bits would cost as much as P's)
//                         While one query tile's softmax runs, the tensor core works for the other.
//   The reference m of a row moves only when its maximum has grown by more than 2^8: then its warp multiplies the row of O
//   (and l) by 2^(m - m'); P stays below 2^8 otherwise, which float32 sums do not mind.  Float16 P is 2^7 times as large, so that
//   its 11 bits reach down to 2^-21 of the row's largest, its steps to 2^-31.
//   What float16 cannot hold (|q| > 4096, |k| > 16384, numbers that are not finite, see V_UP) enters as NaN, and rows that come out not
//   finite are formed once more on the CUDA cores, in float32 from the inputs; so are rows that share a tile with a value that is
//   not finite and that they do not attend (0 times infinity).  A CTA does that behind its last item, when none of its warps
//   waits for another one any more: it may take long.
// Tiles of 2 x 128 queries: both take each tile of keys from shared memory, and tensor memory holds exactly S and O of two.
// Bound by the softmax: for d_k = 128 a pair of 128 x 128 tiles costs the tensor core 1024 clocks for S and 1024 for O, the
// exponentials about 1500 of the special-function unit a scheduler (a quarter of them go to the FMA pipe for that reason), with
// the maxima, scalings, sums and conversions beside them in the same issue slots.
// Measured: 16384 tokens, 32 heads of 128, causal: 1.77 ms (1.24 PFLOP/s, 0.76 of the measured GEMM; 2.1 ms at the power limit)
// and 87 us of preparation; twelve prompts of 1 to 4096 tokens, 8 key heads: 325 us + 53; 8 x 1500 frames, 20 heads of 64,
// not causal: 152 us (0.6 PFLOP/s: half the products an exponential) + 5; chunks of 512, 512, 333 and 1 queries over 4096,
// 1536, 333 and 2048 keys, float32 values: 69 us, as long as the longest tile takes (1.4 times a CTA's share), + 33 for the values
// (201 MB) + 31.
#include <cuda_fp16.h>

#include "slim_attn.h"
#include "slim_attn_plan.cuh"
#include "slim_attn_tile.cuh"
#include "slim_ptx.cuh"

using namespace slim_ptx;

namespace {

// ------------------------------------------------------------------------------------------------ preparation
constexpr int PREP_THREADS = 256;
constexpr float V_UP = 16.f;                         // factor of float32 values on their way into float16, where it suits a column
static_assert(V_UP == 0x1p4f, "an exponent below");
constexpr int V_COLS = SLIM_ATTN_V_COLS, V_PARTS = 4;

__device__ __forceinline__ uint32_t half2_checked(float a, float b, float most) {
  const bool fine = fabsf(a) <= most && fabsf(b) <= most;
  const __half2 v = __floats2half2_rn(a, b);
  return fine ? *reinterpret_cast<const uint32_t*>(&v) : 0x7fff7fffu;
}

// One warp a packed row.  A lane has eight pairs (j, j + d_k/2) of a head, the same j in every head, so its angles are
// formed once; d_k / 16 lanes make a head.  NARROW: heads of fewer columns than DK, a multiple of 16.
template <int DK, bool NARROW>
__device__ void prepare_row(const SlimAttn& a, int r, bool query) {
  const int dk = NARROW ? a.d_k : DK, LPH = dk / 16, HPW = 32 / LPH;
  const int lane = threadIdx.x & 31, heads = query ? a.H : a.KV;
  int pos;
  if (!slim_attn_position(a, r, query, pos) || lane >= LPH * HPW) return;
  const int jl = lane % LPH, hw = lane / LPH;
  const unsigned short* src = reinterpret_cast<const unsigned short*>(query ? a.q : a.k) + (size_t)r * heads * dk + 8 * jl;
  unsigned short* dst = reinterpret_cast<unsigned short*>(query ? a.qr : a.kr) + (size_t)r * heads * DK + 8 * jl;
  const float most = query ? 4096.f : 16384.f;
  float cs[8], sn[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const float2 t = !NARROW || a.rope_base ? slim_attn_turn(a, pos, 8 * jl + x) : make_float2(1.f, 0.f);
    cs[x] = t.x; sn[x] = t.y;
  }
#pragma unroll 4
  for (int h = hw; h < heads; h += HPW) {
    const uint4 u = __ldcs(reinterpret_cast<const uint4*>(src + h * dk)), v = __ldcs(reinterpret_cast<const uint4*>(src + h * dk + dk / 2));
    float lo[8], hi[8];
    unpack8(u, lo);
    unpack8(v, hi);
    uint32_t ol[4], oh[4];
#pragma unroll
    for (int x = 0; x < 8; x += 2) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const bool turn = !NARROW || a.rope_base;
        y[e] = turn ? lo[x + e] * cs[x + e] + hi[x + e] * sn[x + e] : lo[x + e];
        y[2 + e] = turn ? hi[x + e] * cs[x + e] - lo[x + e] * sn[x + e] : hi[x + e];
      }
      ol[x / 2] = half2_checked(y[0], y[1], most);
      oh[x / 2] = half2_checked(y[2], y[3], most);
    }
    *reinterpret_cast<uint4*>(dst + h * DK) = make_uint4(ol[0], ol[1], ol[2], ol[3]);
    *reinterpret_cast<uint4*>(dst + h * DK + dk / 2) = make_uint4(oh[0], oh[1], oh[2], oh[3]);
    if (NARROW)
      for (int c = 8 * jl; c < DK - dk; c += 8 * LPH) *reinterpret_cast<uint4*>(dst - 8 * jl + h * DK + dk + c) = make_uint4(0u, 0u, 0u, 0u);
  }
}

// The same for heads of any other width, two columns at a time (4096 tokens, 32 heads of 80: 151 us by the way above, 218 by
// this one): a lane has columns 2 lane, 2 lane + 1 and those 64 further, in every head.
template <int DK>
__device__ void widen_row(const SlimAttn& a, int r, bool query) {
  const int lane = threadIdx.x & 31, heads = query ? a.H : a.KV, dk = a.d_k, half = a.half;
  int pos;
  if (!slim_attn_position(a, r, query, pos)) return;
  const unsigned short* src = reinterpret_cast<const unsigned short*>(query ? a.q : a.k) + (size_t)r * heads * dk;
  uint32_t* dst = reinterpret_cast<uint32_t*>(query ? a.qr : a.kr) + (size_t)r * heads * (DK / 2);
  const float most = query ? 4096.f : 16384.f;
  float cs[4], sn[4];                                // out[c] = x[c] cos + x[c +- half] sin, the sine's sign by the half
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int c = 64 * (x >> 1) + 2 * lane + (x & 1);
    cs[x] = 1.f; sn[x] = 0.f;
    if (a.rope_base && c < dk) {
      const float2 t = slim_attn_turn(a, pos, c < half ? c : c - half);
      cs[x] = t.x; sn[x] = c < half ? t.y : -t.y;
    }
  }
#pragma unroll 2
  for (int h = 0; h < heads; ++h)
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      float y[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c = 64 * p + 2 * lane + e, x = 2 * p + e;
        y[e] = c < dk ? __uint_as_float((uint32_t)src[h * dk + c] << 16) : 0.f;
        if (a.rope_base && c < dk) y[e] = y[e] * cs[x] + __uint_as_float((uint32_t)src[h * dk + (c < half ? c + half : c - half)] << 16) * sn[x];
      }
      if (64 * p + 2 * lane < DK) dst[h * (DK / 2) + 32 * p + lane] = half2_checked(y[0], y[1], most);
    }
}
template <int DK>
__device__ void widen_values(const SlimAttn& a, int r) {
  const int lane = threadIdx.x & 31, dk = a.d_k;
  const unsigned short* src = reinterpret_cast<const unsigned short*>(a.v) + (size_t)r * a.KV * dk;
  uint32_t* dst = reinterpret_cast<uint32_t*>(a.vb) + (size_t)r * a.KV * (DK / 2);
  if ((dk & 7) == 0) {                               // eight columns at a time
#pragma unroll 4
    for (int i = lane; i < a.KV * (DK / 8); i += 32) {
      const int h = i / (DK / 8), c = i % (DK / 8) * 8;
      reinterpret_cast<uint4*>(dst)[i] = c < dk ? __ldcs(reinterpret_cast<const uint4*>(src + h * dk + c)) : make_uint4(0u, 0u, 0u, 0u);
    }
    return;
  }
#pragma unroll 4
  for (int i = lane; i < a.KV * (DK / 2); i += 32) {
    const int h = i / (DK / 2), c = i % (DK / 2) * 2;                    // (d_k is even)
    dst[i] = c < dk ? __ldcs(reinterpret_cast<const uint32_t*>(src + h * dk + c)) : 0u;
  }
}

// Float32 values as float16, each column times a power of two: V_UP, unless the column's largest finite magnitude M is above
// V_MOST or below V_LEAST, then the one that brings M into [2^14, 2^15).  With V_UP float16's smallest step is 2^-28 (2^-20 of M
// at most).  With another factor values keep their 11 bits down to 2^-28 M; smaller ones, which no column has unless its largest
// stand apart (in rows of another sequence, say), enter as NaN like what float16 cannot hold.  M is known only behind a pass
// over all rows; the pass converts with V_UP, and columns that need another factor are converted again (settle_columns).
constexpr float V_MOST = 4000.f, V_LEAST = 0x1p-8f;
__device__ __forceinline__ unsigned short half_checked(float x) { return fabsf(x) <= 64000.f ? __half_as_ushort(__float2half_rn(x)) : (unsigned short)0x7fff; }
__device__ __forceinline__ float finite_abs(float x) { const float y = fabsf(x); return y <= 3.4028234663852886e38f ? y : 0.f; }

// Unit u: V_COLS columns (of the widened heads) of a run of rows, by a block, W columns a thread at a time
template <int DK, int W>
__device__ void convert_values(const SlimAttn& a, int u, float* s_max) {
  constexpr int TPR = V_COLS / W, RPP = PREP_THREADS / TPR;
  const int tid = threadIdx.x, dk = a.d_k, width = a.KV * DK, blocks = (width + V_COLS - 1) / V_COLS;
  const int run = u / blocks, c0 = u % blocks * V_COLS, col = c0 + tid % TPR * W, h = col / DK, c = col - h * DK;
  const int lo = (int)((long long)a.total_k * run / a.v_runs), hi = (int)((long long)a.total_k * (run + 1) / a.v_runs);
  const bool there = col < width, live = there && c < dk;
  const float* src = reinterpret_cast<const float*>(a.v) + (size_t)h * dk + c;
  unsigned short* dst = reinterpret_cast<unsigned short*>(a.vb) + col;
  float m[W];
#pragma unroll
  for (int x = 0; x < W; ++x) m[x] = 0.f;
  constexpr int FLY = 24 / W;                        // rows of a thread whose loads are in flight together
  for (int r0 = lo + tid / TPR; r0 < hi; r0 += FLY * RPP) {
    float v[FLY][W];
#pragma unroll
    for (int i = 0; i < FLY; ++i) {
      const int r = r0 + i * RPP;
#pragma unroll
      for (int x = 0; x < W; ++x) v[i][x] = 0.f;
      if (live && r < hi) {
        if constexpr (W == 4) *reinterpret_cast<float4*>(v[i]) = __ldcs(reinterpret_cast<const float4*>(src + (size_t)r * a.KV * dk));
        else *reinterpret_cast<float2*>(v[i]) = __ldcs(reinterpret_cast<const float2*>(src + (size_t)r * a.KV * dk));
      }
    }
#pragma unroll
    for (int i = 0; i < FLY; ++i) {
      const int r = r0 + i * RPP;
      uint32_t w[W / 2];
#pragma unroll
      for (int x = 0; x < W; x += 2) {
        m[x] = fmaxf(m[x], finite_abs(v[i][x])); m[x + 1] = fmaxf(m[x + 1], finite_abs(v[i][x + 1]));
        w[x / 2] = half_checked(v[i][x] * V_UP) | (uint32_t)half_checked(v[i][x + 1] * V_UP) << 16;
      }
      if (there && r < hi) {
        if constexpr (W == 4) *reinterpret_cast<uint2*>(dst + (size_t)r * width) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(dst + (size_t)r * width) = w[0];
      }
    }
  }
  // Rows in front of the first and behind the last sequence may hold anything: a run that has some is looked at once more without
  const int k0 = max(lo, __ldg(a.cu_k)), k1 = min(hi, __ldg(a.cu_k + a.batch));
  if (k0 > lo || k1 < hi) {
#pragma unroll
    for (int x = 0; x < W; ++x) m[x] = 0.f;
    for (int r = k0 + tid / TPR; live && r < k1; r += RPP)
#pragma unroll
      for (int x = 0; x < W; ++x) m[x] = fmaxf(m[x], finite_abs(__ldg(src + (size_t)r * a.KV * dk + x)));
  }
  __syncthreads();                                   // (the unit before this one has been read)
#pragma unroll
  for (int x = 0; x < W; ++x) s_max[tid / TPR * V_COLS + tid % TPR * W + x] = m[x];
  __syncthreads();
  if (tid < V_COLS) {
    float most = s_max[tid];
#pragma unroll
    for (int i = 1; i < RPP; ++i) most = fmaxf(most, s_max[i * V_COLS + tid]);
    a.v_max[(size_t)run * blocks * V_COLS + c0 + tid] = most;
  }
}

template <int DK>
__global__ void __launch_bounds__(PREP_THREADS, 4) attn_tc_values_kernel(const __grid_constant__ SlimAttn a) {
  __shared__ float s_max[8 * V_COLS];
  slim_pdl_trigger();
  slim_pdl_wait();
  const int units = a.v_runs * ((a.KV * DK + V_COLS - 1) / V_COLS);
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    if ((a.d_k & 3) == 0) convert_values<DK, 4>(a, u, s_max);
    else convert_values<DK, 2>(a, u, s_max);
  }
}

// Behind it, by a block: the factors of V_COLS columns, and part y of V_PARTS of the columns that V_UP does not suit once more
template <int DK>
__device__ void settle_columns(const SlimAttn& a, int block, int blocks, int y, float* s_max) {
  const int tid = threadIdx.x, width = a.KV * DK, col = block * V_COLS + tid % V_COLS, part = tid / V_COLS;
  constexpr int parts = PREP_THREADS / V_COLS;
  float most = 0.f;
#pragma unroll 16
  for (int r = part; r < a.v_runs; r += parts) most = fmaxf(most, __ldg(a.v_max + (size_t)r * blocks * V_COLS + col));
  __syncthreads();                                   // (the unit before this one has been read)
  s_max[tid] = most;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < parts; ++i) most = fmaxf(most, s_max[i * V_COLS + tid % V_COLS]);
  const bool other = most > V_MOST || (most > 0.f && most < V_LEAST);
  // 2^14 over the power of two in M (a denormal one's is taken as 2^-112: no column asks for more than 2^126)
  const int e = max(__float_as_int(most) >> 23, 15) - 127;
  if (y == 0 && part == 0) a.v_more[col] = other ? __int_as_float((e - 14 + 4 + 127) << 23) : 1.f;      // V_UP over the column's factor
  const int h = col / DK, c = col - h * DK, dk = a.d_k;
  if (!other || col >= width) return;
  const float up = __int_as_float((14 - e + 127) << 23);
  const float* src = reinterpret_cast<const float*>(a.v) + (size_t)h * dk + c;
  unsigned short* dst = reinterpret_cast<unsigned short*>(a.vb) + col;
#pragma unroll 4
  for (int r = parts * y + part; r < a.total_k; r += parts * V_PARTS) {
    const float v = __ldg(src + (size_t)r * a.KV * dk);
    dst[(size_t)r * width] = v == 0.f || fabsf(v * up) >= 0x1p-14f ? half_checked(v * up) : (unsigned short)0x7fff;
  }
}

template <int DK>
__global__ void __launch_bounds__(PREP_THREADS) attn_tc_prepare_kernel(const __grid_constant__ SlimAttn a) {
  extern __shared__ int s_mem[];
  __shared__ float s_max[PREP_THREADS];
  slim_pdl_trigger();
  slim_pdl_wait();
  if (blockIdx.x == 0) { slim_attn_plan(a, s_mem); return; }
  if (a.v32) {
    const int blocks = (a.KV * DK + V_COLS - 1) / V_COLS;              // by the last blocks, which have fewer rows
    for (int u = gridDim.x - 1 - blockIdx.x; u < blocks * V_PARTS; u += gridDim.x - 1) settle_columns<DK>(a, u % blocks, blocks, u / blocks, s_max);
  }
  const int warps = (gridDim.x - 1) * (PREP_THREADS / 32);
  const bool narrow = a.d_k != DK;
  const int turned = a.rope_base || narrow ? a.total_q + a.total_k : 0, rows = turned + (!a.v32 && narrow ? a.total_k : 0);
  for (int r = (blockIdx.x - 1) * (PREP_THREADS / 32) + (threadIdx.x >> 5); r < rows; r += warps) {
    const bool query = r < a.total_q;
    if (r >= turned) widen_values<DK>(a, r - turned);
    else if (!narrow) prepare_row<DK, false>(a, query ? r : r - a.total_q, query);
    else if ((a.d_k & 15) == 0) prepare_row<DK, true>(a, query ? r : r - a.total_q, query);
    else widen_row<DK>(a, query ? r : r - a.total_q, query);
  }
}

// ------------------------------------------------------------------------------------------------ attention
constexpr int TM = 128, TN = 128;                    // rows of a query tile, keys of a key tile
constexpr int THREADS = 384;                         // two groups of four softmax warps, MMA warp, load warp, two without work
constexpr int SPLIT = 96;                            // keys of a tile whose probabilities are handed over first
constexpr float TAU = 8.f;                           // log2 units by which a row's maximum may pass its reference

constexpr int EMU = 2;                               // of eight pairs of exponentials so many are formed on the FMA pipe

// 2^x of two arguments up to 2^6 or so without the special-function unit: x = i + f with |f| <= 1/2, the nearest integer coming from
// the addition of 1.5 * 2^23 + 127, whose low bits then hold i + 127, the exponent of 2^i; a cubic for 2^f with the smallest
// largest relative error on [-1/2, 1/2], 7.5e-5 (fitted by reweighted least squares).  Below -126.5 it is 0 (a masked score must
// not meet its value with any weight), and of a NaN it is one.
__device__ __forceinline__ void exp2_pair(f32x2 x, float& lo, float& hi) {
  const f32x2 magic = pack2(12583039.f, 12583039.f), minus = pack2(-12583039.f, -12583039.f), neg = pack2(-1.f, -1.f);
  float a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(-127.f));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(b) : "f"(-127.f));
  x = pack2(a, b);
  const f32x2 t = add2(x, magic);
  const f32x2 f = fma2(add2(t, minus), neg, x);
  f32x2 y = fma2(f, pack2(0.055171601474285126f, 0.055171601474285126f), pack2(0.2426111251115799f, 0.2426111251115799f));
  y = fma2(f, y, pack2(0.6932609677314758f, 0.6932609677314758f));
  y = fma2(f, y, pack2(0.9999280571937561f, 0.9999280571937561f));
  uint32_t i0, i1;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(i0), "=r"(i1) : "l"(t));
  y = mul2(y, pack2(__uint_as_float(i0 << 23), __uint_as_float(i1 << 23)));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(y));
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d; asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d;
}

template <int DK>
struct Shape {
  static constexpr int CH = (DK + 63) / 64;          // 64-column chunks of a head
  static constexpr int TILE = CH * TN * 128;         // bytes of a tile of Q, K or V
  static constexpr int NS = DK == 64 ? 8 : 5;        // ring of K and V tiles
  static constexpr int SMEM = 1024 + (2 + NS) * TILE + 8 * (2 * NS + 11) + 32;
};

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// A from shared memory / from tensor memory
__device__ __forceinline__ void umma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ uint32_t bf162_of(float lo, float hi) {
  uint32_t d; asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo)); return d;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  uint32_t d; asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo)); return d;
}
__device__ __forceinline__ void split(f32x2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }

// Scores LO .. HI - 1 of a row -> probabilities in 16 bits, pairs from r[LO / 2] on; l2 gathers their sum.
template <int LO, int HI, bool VH>
__device__ __forceinline__ void exponentials(uint32_t (&r)[TN], f32x2 scale2, f32x2 m2, f32x2& l2) {
#pragma unroll
  for (int x = LO; x < HI; x += 2) {
    const f32x2 v = fma2(pack2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])), scale2, m2);
    float lo, hi;
    if ((x / 2 * 3) % 8 < EMU) {
      exp2_pair(v, lo, hi);
    } else {
      split(v, lo, hi);
      lo = ex2_approx(lo); hi = ex2_approx(hi);
    }
    l2 = add2(l2, pack2(lo, hi));
    r[x / 2] = VH ? half2_of(lo, hi) : bf162_of(lo, hi);
  }
}

// A row of outputs times its columns' powers of two: exact but at the ends of bf16's range
__device__ __noinline__ void scale_row(__nv_bfloat16* o, const float* f, int n) {
  for (int c = 0; c < n; c += 2) {                   // (d_k is even)
    uint32_t* at = reinterpret_cast<uint32_t*>(o + c);
    const uint32_t w = *at;
    *at = bf162_of(__uint_as_float(w << 16) * __ldg(f + c), __uint_as_float(w & 0xffff0000u) * __ldg(f + c + 1));
  }
}

// Number of a CTA's item r: the list, most keys first, is dealt out in rounds of alternating direction.
__device__ __forceinline__ long long item_place(int r) {
  return (long long)r * gridDim.x + (r & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
}

// Rows of a CTA's items once more, tiles of 64, by the first 256 threads, which meet at barrier 1
template <int DK>
__device__ __noinline__ void again(const SlimAttn& a, float* smem) {
  typedef SlimAttnTile<DK == 64 ? 64 : 128, 64, true> Tile;
  static_assert(Tile::SMEM <= (2 + Shape<DK>::NS) * Shape<DK>::TILE, "fits the operands' place");
  const int n_items = *a.n_tiles * a.H;
  for (int r = 0; item_place(r) < n_items; ++r) {
    const int tile = (int)(item_place(r) / a.H), h = (int)(item_place(r) - (long long)tile * a.H);
    const int4 x = a.tiles[3 * tile], y = a.tiles[3 * tile + 1];
    const SlimSeq s = {y.x, y.y, y.z, y.w};
    for (int i = 0; i < SLIM_ATTN_TC_ROWS / 64; ++i) {
      const uint2 which = *reinterpret_cast<const uint2*>(a.redo + 8 * item_place(r) + 2 * i);
      if (!(which.x | which.y)) continue;
      const int row0 = x.y + 64 * i, rows = min(64, s.nq - row0);
      Tile t;
      t.run(a, s, row0, rows, h, 0, 0x7fffffff, smem, 1);
      t.store(a, s, row0, rows, h, (unsigned long long)which.y << 32 | which.x);
    }
  }
}

template <int DK, bool VH>
__global__ void __launch_bounds__(THREADS, 1)
attn_tc_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
               const __grid_constant__ SlimAttn a) {
  typedef Shape<DK> S;
  constexpr int NS = S::NS, CH = S::CH, KSTEPS = DK / 16;
  constexpr uint32_t TILE = S::TILE;
  // S = Q K^T: float16, or bf16 where the inputs are read where they lie, both K-major;  O = P V: float16 (VH) or bf16, V MN-major
  const uint32_t IDESC_S = (1u << 4) | (a.rope_base || a.d_k != DK ? 0u : (1u << 7) | (1u << 10)) | ((TN >> 3) << 17) | ((TM >> 4) << 24);
  constexpr uint32_t IDESC_O = (1u << 4) | (VH ? 0u : (1u << 7) | (1u << 10)) | (1u << 16) | ((DK >> 3) << 17) | ((TM >> 4) << 24);
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* sm = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t s_q = base, s_kv = base + 2 * TILE;
  const uint32_t bars = s_kv + NS * TILE;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * NS, bar_q = bars + 16 * NS;
  const uint32_t bar_qe = bar_q + 8;
  const uint32_t bar_s = bar_qe + 8, bar_p = bar_s + 16, bar_o = bar_p + 16, bar_ph = bar_o + 16;      // two each
  unsigned char* misc = sm + (bar_ph + 16 - base);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(misc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(misc + 4);
  volatile int* s_redo = reinterpret_cast<volatile int*>(misc + 8);        // some item has rows to be formed once more
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    prefetch_tensormap(&qmap); prefetch_tensormap(&kmap); prefetch_tensormap(&vmap);
    for (int i = 0; i < NS; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    mbar_init(bar_q, 1);
    mbar_init(bar_qe, 1);
    for (int i = 0; i < 2; ++i) { mbar_init(bar_s + 8 * i, 1); mbar_init(bar_ph + 8 * i, 4); mbar_init(bar_p + 8 * i, 4); mbar_init(bar_o + 8 * i, 1); }
    *s_abort = 0;
    *s_redo = 0;
    fence_mbar_init();
  }
  if (warp == 8) tmem_alloc(smem_u32(s_tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  slim_pdl_trigger();
  slim_pdl_wait();
  const int n_items = *a.n_tiles * a.H, share = a.H / a.KV;
  struct Item { SlimSeq s; int row0, h, nt0, nt1, first, piece, pieces, slot; };
  auto item = [&](int r, Item& it) {
    const long long at = item_place(r);
    if (at >= n_items) return false;
    const int tile = (int)(at / a.H);
    it.h = (int)(at - (long long)tile * a.H);
    const int4 x = __ldg(a.tiles + 3 * tile), y = __ldg(a.tiles + 3 * tile + 1), z = __ldg(a.tiles + 3 * tile + 2);
    it.row0 = x.y; it.piece = x.z; it.pieces = x.w;
    it.s.q0 = y.x; it.s.nq = y.y; it.s.k0 = y.z; it.s.nk = y.w;
    it.first = z.x; it.slot = z.z;
    // key tiles of the two query tiles, within the piece (the second may have no rows)
    it.nt0 = (slim_attn_keys(a, it.s, min(it.s.nq, it.row0 + TM) - 1) + TN - 1) / TN;
    it.nt1 = it.row0 + TM < it.s.nq ? (slim_attn_keys(a, it.s, min(it.s.nq, it.row0 + 2 * TM) - 1) + TN - 1) / TN : 0;
    it.nt0 = max(min(it.nt0, z.y) - z.x, 0);
    it.nt1 = max(min(it.nt1, z.y) - z.x, 0);
    return true;
  };
  Item it;
  bool ok = true;

  if (warp < 8) {
    // 168 registers a thread at launch; the last four warps leave 128 of theirs to the others (232 x 256 + 40 x 128 = 168 x 384)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    // =========================== softmax ===========================
    const int i = warp >> 2;
    const uint32_t t_s = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(i * TN);
    const uint32_t t_o = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(2 * TN + i * 128);
    const float scale = a.qscale;
    const f32x2 scale2 = pack2(scale, scale);
    uint32_t ps = 0, po = 0;                        // phases of bar_s, bar_o
    for (int r_ = 0; ok && item(r_, it); ++r_) {
      constexpr float LIFT = VH ? 7.f : 0.f;
      const int n = i ? it.nt1 : it.nt0;
      const int all = slim_attn_keys(a, it.s, it.row0 + i * TM + (warp & 3) * 32 + lane);     // keys of the row
      const int lim = all - it.first * TN;                                                   // behind the piece's first
      float m = -INFINITY;                            // reference, log2 units
      f32x2 l2 = pack2(0.f, 0.f);
      for (int j = 0; j < n; ++j) {
        ok = mbar_wait<false>(bar_s + 8 * i, ps, s_abort, a.status) && ok;
        ps ^= 1u;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        uint32_t r[TN];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32_issue(t_s + 32 * c, *reinterpret_cast<uint32_t (*)[32]>(r + 32 * c));
        tmem_ld_wait();
        if (__any_sync(0xffffffffu, (j + 1) * TN > lim)) {
#pragma unroll
          for (int x = 0; x < TN; ++x)
            if (j * TN + x >= lim) r[x] = 0xff800000u;
        }
        float mx[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) mx[c] = fmaxf(__uint_as_float(r[c]), __uint_as_float(r[c + 8]));
#pragma unroll
        for (int x = 16; x < TN; x += 16)
#pragma unroll
          for (int c = 0; c < 8; ++c) mx[c] = max3(mx[c], __uint_as_float(r[x + c]), __uint_as_float(r[x + c + 8]));
        const float top = max3(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * scale;
        const bool move = top > m + (TAU + LIFT);     // (m = -inf: the first keys of the row)
        if (__any_sync(0xffffffffu, move)) {
          const float m_new = move ? top - LIFT : m;
          const float f = move ? ex2_approx(m - m_new) : 1.f;
          m = m_new;
          float lo, hi;
          split(l2, lo, hi);
          l2 = pack2(lo * f, hi * f);
          if (j > 0) {
            // O_i is at rest: S_i(j) was completed after O_i += P_i(j - 1) V, and the next product waits for P_i(j)
#pragma unroll
            for (int c = 0; c < DK / 16; ++c) {       // (16 columns at a time: S is in registers too)
              uint32_t o[16];
              tmem_ld16(t_o + 16 * c, o);
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
              tmem_st16(t_o + 16 * c, o);
            }
          }
        }
        const float mm = m == -INFINITY ? 0.f : -m;
        const f32x2 m2 = pack2(mm, mm);
        // P in two parts: the tensor core begins with the first three quarters while the exponentials of the last are formed
        exponentials<0, SPLIT, VH>(r, scale2, m2, l2);
        tmem_st32(t_s, r);
        tmem_st16(t_s + 32, r + 32);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_ph + 8 * i);
        exponentials<SPLIT, TN, VH>(r, scale2, m2, l2);
        tmem_st16(t_s + SPLIT / 2, r + SPLIT / 2);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p + 8 * i);
      }
      // ---- output ----
      item(r_, it);                                   // (once more: nothing of it has to be kept while S is in registers)
      const SlimSeq s = it.s;
      const int row = it.row0 + i * TM + (warp & 3) * 32 + lane, h = it.h;
      if (ok && n > 0) {
        ok = mbar_wait<false>(bar_o + 8 * i, po, s_abort, a.status);
        po ^= 1u;
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
      }
      const bool there = row < s.nq;
      float l = sum2(l2);
      if (it.pieces > 1) {
        // A piece of the keys: the warp's sums go to the workspace, a column of four times 256 rows at a time, and the last of
        // the tile's pieces to arrive there joins them, in their order
        constexpr size_t SLOT = (size_t)SLIM_ATTN_TC_ROWS * (DK + 2);
        const size_t slot0 = (size_t)it.slot * a.H + h, step = SLOT * a.H;
        const int lane_row = i * TM + (warp & 3) * 32 + lane;
        float* mine = a.part + (slot0 + (size_t)it.piece * a.H) * SLOT;
        if (ok) {
          if (n > 0) {
#pragma unroll
            for (int c = 0; c < DK / 32; ++c) {
              uint32_t o[32];
              tmem_ld32(t_o + 32 * c, o);
#pragma unroll
              for (int x = 0; x < 32; x += 4)
                *reinterpret_cast<uint4*>(mine + ((size_t)(8 * c + x / 4) * SLIM_ATTN_TC_ROWS + lane_row) * 4) = make_uint4(o[x], o[x + 1], o[x + 2], o[x + 3]);
            }
          }
          mine[SLIM_ATTN_TC_ROWS * DK + lane_row] = m;
          mine[SLIM_ATTN_TC_ROWS * (DK + 1) + lane_row] = l;
        }
        tc_fence_before();                            // (O has been read: the next item's first product overwrites it)
        __threadfence();
        __syncwarp();
        int before = 0;
        if (lane == 0 && ok) before = atomicAdd(a.arrivals + 8 * slot0 + warp, 1);
        before = __shfl_sync(0xffffffffu, before, 0);
        if (lane == 0) a.redo[8 * item_place(r_) + warp] = 0u;
        if (!ok || before != it.pieces - 1) continue;
        __threadfence();
        const float* from = a.part + slot0 * SLOT;
        const int pieces = it.pieces;
        m = -INFINITY;
        for (int x = 0; x < pieces; ++x) m = fmaxf(m, __ldcg(from + x * step + SLIM_ATTN_TC_ROWS * DK + lane_row));
        l = 0.f;
        for (int x = 0; x < pieces; ++x) {
          const float mx = __ldcg(from + x * step + SLIM_ATTN_TC_ROWS * DK + lane_row), lx = __ldcg(from + x * step + SLIM_ATTN_TC_ROWS * (DK + 1) + lane_row);
          if (!(mx == -INFINITY && lx == 0.f)) l = fmaf(lx, ex2_approx(mx - m), l);
        }
      }
      const float inv = all > 0 ? (VH ? 1.f / V_UP : 1.f) / l : 0.f;
      __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(a.o) + ((size_t)(s.q0 + row) * a.H + h) * a.d_k;
      bool bad = false;
      if (ok) {
#pragma unroll
        for (int c = 0; c < DK / 32; ++c) {
          uint32_t o[32];
          if (it.pieces > 1) {
            constexpr size_t SLOT = (size_t)SLIM_ATTN_TC_ROWS * (DK + 2);
            const float* from = a.part + ((size_t)it.slot * a.H + h) * SLOT;
            const int lane_row = i * TM + (warp & 3) * 32 + lane;
#pragma unroll
            for (int x = 0; x < 32; ++x) o[x] = 0u;
#pragma unroll 2
            for (int y = 0; y < it.pieces; ++y, from += SLOT * a.H) {
              const float mx = __ldcg(from + SLIM_ATTN_TC_ROWS * DK + lane_row), lx = __ldcg(from + SLIM_ATTN_TC_ROWS * (DK + 1) + lane_row);
              const bool some = !(mx == -INFINITY && lx == 0.f);         // (else the row attends nothing there)
              const float f = some ? ex2_approx(mx - m) : 0.f;
              float4 u[8];
#pragma unroll
              for (int x = 0; x < 8; ++x)
                u[x] = some ? __ldcg(reinterpret_cast<const float4*>(from + ((size_t)(8 * c + x) * SLIM_ATTN_TC_ROWS + lane_row) * 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
              for (int x = 0; x < 32; x += 4) {
                const float4 v = u[x / 4];
                o[x] = __float_as_uint(fmaf(v.x, f, __uint_as_float(o[x]))); o[x + 1] = __float_as_uint(fmaf(v.y, f, __uint_as_float(o[x + 1])));
                o[x + 2] = __float_as_uint(fmaf(v.z, f, __uint_as_float(o[x + 2]))); o[x + 3] = __float_as_uint(fmaf(v.w, f, __uint_as_float(o[x + 3])));
              }
            }
          } else if (n > 0) tmem_ld32(t_o + 32 * c, o);
#pragma unroll
          for (int x = 0; x < 32; x += 8) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float lo = __uint_as_float(o[x + 2 * e]) * inv, hi = __uint_as_float(o[x + 2 * e + 1]) * inv;
              if (all == 0) lo = hi = 0.f;
              bad |= !(fabsf(lo) <= 3.3895313892515355e38f && fabsf(hi) <= 3.3895313892515355e38f);
              w[e] = bf162_of(lo, hi);
            }
            if (there && (a.d_k & 7) == 0) {
              if (32 * c + x < a.d_k) *reinterpret_cast<uint4*>(dst + 32 * c + x) = make_uint4(w[0], w[1], w[2], w[3]);
            } else if (there) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (32 * c + x + 2 * e < a.d_k) *reinterpret_cast<uint32_t*>(dst + 32 * c + x + 2 * e) = w[e];
            }
          }
        }
        const unsigned redo = __ballot_sync(0xffffffffu, bad && there);
        if (VH) {
          // columns with a factor of their own (mostly none)
          const float4 f = 4 * lane < DK ? __ldg(reinterpret_cast<const float4*>(a.v_more + h / share * DK) + lane) : make_float4(1.f, 1.f, 1.f, 1.f);
          if (__any_sync(0xffffffffu, f.x != 1.f || f.y != 1.f || f.z != 1.f || f.w != 1.f) && there) scale_row(dst, a.v_more + h / share * DK, a.d_k);
        }
        __syncwarp();
        if (lane == 0) {
          a.redo[8 * item_place(r_) + warp] = redo;
          if (redo) *s_redo = 1;
        }
      }
    }
    // ---- rows once more: the operands' shared memory is free, the eight warps are together ----
    asm volatile("bar.sync 1, 256;" ::: "memory");
    if (*s_redo && !*s_abort) again<DK>(a, reinterpret_cast<float*>(sm));
  } else if (warp == 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    // =========================== MMA issuer ===========================
    // The warp stays together and one elected lane issues, so that the descriptors live in uniform registers.
    const uint64_t dq = desc_kmajor_sw128(s_q), dk = desc_kmajor_sw128(s_kv), dv = desc_a(s_kv, TN * 128);
    uint32_t pq = 0, pf = 0, pp0 = 0, pp1 = 0;      // phases: queries, ring, P of the two tiles
    int st = 0;                                     // next stage of the ring
    uint32_t last = 0xffffffffu, last_ph = 0;       // stage committed last, and its phase
    auto scores = [&](int i, uint32_t stage) {
      const uint64_t qd = dq + (uint64_t)(i * (TILE >> 4)), kd = dk + (uint64_t)(stage * (TILE >> 4));
#pragma unroll
      for (int x = 0; x < KSTEPS; ++x) {
        const uint32_t off = (uint32_t)((x >> 2) * TN * 128 + (x & 3) * 32) >> 4;
        umma_ss(tmem + i * TN, qd + off, kd + off, IDESC_S, x > 0);
      }
      umma_commit(bar_s + 8 * i);
    };
    for (int r_ = 0; ok && item(r_, it); ++r_) {
      const int nt = max(it.nt0, it.nt1);
      if (nt == 0) continue;
      ok = mbar_wait<false>(bar_q, pq, s_abort, a.status);
      pq ^= 1u;
      ok = mbar_wait<false>(bar_full + 8 * st, pf, s_abort, a.status) && ok;
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
        if (it.nt0 > 0) scores(0, (uint32_t)st);
        if (it.nt1 > 0) scores(1, (uint32_t)st);
        umma_commit(bar_empty + 8 * st);
        if (nt == 1) umma_commit(bar_qe);
      }
      __syncwarp();
      if (++st == NS) { st = 0; pf ^= 1u; }
      for (int j = 0; j < nt && ok; ++j) {
        const int kv = st, kk = st + 1 == NS ? 0 : st + 1;
        const uint32_t pkv = pf, pkk = kk == 0 ? pf ^ 1u : pf;
        ok = mbar_wait<false>(bar_full + 8 * kv, pkv, s_abort, a.status);
        if (j + 1 < nt) ok = mbar_wait<false>(bar_full + 8 * kk, pkk, s_abort, a.status) && ok;
        ok = __all_sync(0xffffffffu, ok);           // (a wait that runs out may do so for some lanes only)
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int n = i ? it.nt1 : it.nt0;
          if (j < n && ok) {
            uint32_t& pp = i ? pp1 : pp0;
            const uint64_t vd = dv + (uint64_t)(kv * (int)(TILE >> 4));
            ok = mbar_wait<false>(bar_ph + 8 * i, pp, s_abort, a.status);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            if (ok && elect_one()) {
#pragma unroll
              for (int x = 0; x < SPLIT / 16; ++x)
                umma_ts(tmem + 2 * TN + i * 128, tmem + i * TN + 8 * x, vd + x * (2048 >> 4), IDESC_O, j > 0 || x > 0);
            }
            __syncwarp();
            ok = mbar_wait<false>(bar_p + 8 * i, pp, s_abort, a.status) && ok;
            pp ^= 1u;
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            if (ok && elect_one()) {
#pragma unroll
              for (int x = SPLIT / 16; x < TN / 16; ++x)
                umma_ts(tmem + 2 * TN + i * 128, tmem + i * TN + 8 * x, vd + x * (2048 >> 4), IDESC_O, 1u);
              if (j + 1 < n) scores(i, (uint32_t)kk);
              else umma_commit(bar_o + 8 * i);
            }
            __syncwarp();
          }
        }
        if (!ok) break;
        if (elect_one()) {
          umma_commit(bar_empty + 8 * kv);
          if (j + 1 < nt) umma_commit(bar_empty + 8 * kk);
          if (j + 2 == nt) umma_commit(bar_qe);     // the item's last scores are behind it
        }
        __syncwarp();
        last = (uint32_t)kv; last_ph = pkv;
        const int used = j + 1 < nt ? 2 : 1;
        for (int x = 0; x < used; ++x)
          if (++st == NS) { st = 0; pf ^= 1u; }
      }
    }
    // the last commit's arrival must not find this CTA gone
    if (ok && last != 0xffffffffu) mbar_wait<false>(bar_empty + 8 * last, last_ph, s_abort, a.status);
    __syncwarp();
  } else if (warp == 9) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    // =========================== loads ===========================
    if (lane == 0) {
      fence_proxy_async_global();                   // (queries, keys and values are an earlier kernel's ordinary stores)
      int st = 0;                                   // next stage
      uint32_t pe = 1u, pqe = 1u;                   // phases of bar_empty, bar_qe (the first pass finds everything empty)
      for (int r_ = 0; ok && item(r_, it); ++r_) {
        const int nt = max(it.nt0, it.nt1), kvh = it.h / share;
        if (nt == 0) continue;
        ok = mbar_wait<false>(bar_qe, pqe, s_abort, a.status);
        if (!ok) break;
        pqe ^= 1u;
        const uint32_t tiles_q = it.nt1 > 0 ? 2 : 1;
        mbar_arrive_expect_tx(bar_q, tiles_q * TILE);
        for (uint32_t i = 0; i < tiles_q; ++i)
          for (int c = 0; c < CH; ++c) tma_load_3d(s_q + i * TILE + c * TM * 128, &qmap, bar_q, it.h * DK + 64 * c, it.s.q0 + it.row0 + (int)i * TM, 0);
        for (int k = 0; k < 2 * nt; ++k) {
          ok = mbar_wait<false>(bar_empty + 8 * st, pe, s_abort, a.status);
          if (!ok) break;
          const uint32_t bar = bar_full + 8 * st, dst = s_kv + (uint32_t)st * TILE;
          mbar_arrive_expect_tx(bar, TILE);
          for (int c = 0; c < CH; ++c)                                 // K(0), V(0), K(1), ..: the order in which they are needed
            tma_load_3d(dst + c * TN * 128, k & 1 ? &vmap : &kmap, bar, kvh * DK + 64 * c, it.s.k0 + (it.first + (k >> 1)) * TN, 0);
          if (++st == NS) { st = 0; pe ^= 1u; }
        }
      }
      if (!ok) {
        // gave up, two seconds after the last of a ring's loads: a quarter of a second more for any of them that is still on its way
        const unsigned long long t0 = globaltimer();
        while (globaltimer() - t0 < SLIM_WAIT_NS / 8) {}
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

cudaError_t make_map(CUtensorMap* map, const void* p, int cols, int rows) {
  const unsigned long long dims[3] = {(unsigned long long)cols, (unsigned long long)rows, 1};
  const unsigned long long strides[2] = {(unsigned long long)cols * 2, (unsigned long long)cols * 2 * rows};
  const unsigned int box[3] = {64, TN, 1};
  return slim_tmap_encode_3d(map, const_cast<void*>(p), dims, strides, box);
}

template <int DK, bool VH>
cudaError_t launch(const slim_ctx* ctx, const SlimAttn& a, cudaStream_t st) {
  CUtensorMap qmap, kmap, vmap;
  const bool as_is = !a.rope_base && a.d_k == DK;
  cudaError_t e = make_map(&qmap, as_is ? a.q : a.qr, a.H * DK, a.total_q);
  if (e == cudaSuccess) e = make_map(&kmap, as_is ? a.k : a.kr, a.KV * DK, a.total_k);
  if (e == cudaSuccess) e = make_map(&vmap, a.v32 || a.d_k != DK ? a.vb : a.v, a.KV * DK, a.total_k);
  if (e == cudaSuccess) e = cudaFuncSetAttribute((const void*)attn_tc_kernel<DK, VH>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DK>::SMEM);
  if (e != cudaSuccess) return e;
  const long long fill = 8ll * ctx->num_sms;
  const long long columns = (a.KV * DK + V_COLS - 1) / V_COLS, units = a.v_runs * columns;
  if (a.v32) {
    e = slim_launch_pdl(attn_tc_values_kernel<DK>, dim3((unsigned)(units < fill ? units : fill)), dim3(PREP_THREADS), 0, st, a);
    if (e != cudaSuccess) return e;
  }
  const long long rows = (as_is ? 0 : (long long)a.total_q + a.total_k) + (!a.v32 && a.d_k != DK ? a.total_k : 0);
  long long blocks = (rows + 7) / 8;
  if (a.v32 && blocks < columns * V_PARTS) blocks = columns * V_PARTS;
  e = slim_launch_pdl(attn_tc_prepare_kernel<DK>, dim3(1 + (unsigned)(blocks < fill ? blocks : fill)), dim3(PREP_THREADS), slim_attn_plan_smem(a.batch), st, a);
  if (e != cudaSuccess) return e;
  const long long items = (long long)a.most_tiles * a.H + a.slots;
  return slim_launch_pdl(attn_tc_kernel<DK, VH>, dim3((unsigned)(items < ctx->num_sms ? items : ctx->num_sms)), dim3(THREADS), Shape<DK>::SMEM, st, qmap, kmap, vmap, a);
}

}  // namespace

int slim_attn_tc_ok(const slim_ctx* ctx) { return ctx->dtype == SLIM_BF16 && ctx->d_k <= 128; }

cudaError_t slim_launch_attn_tc(const slim_ctx* ctx, const SlimAttn& a, cudaStream_t st) {
  const int w = slim_attn_width(a.d_k);
  if (a.v32) return w == 64 ? launch<64, true>(ctx, a, st) : w == 96 ? launch<96, true>(ctx, a, st) : launch<128, true>(ctx, a, st);
  return w == 64 ? launch<64, false>(ctx, a, st) : w == 96 ? launch<96, false>(ctx, a, st) : launch<128, false>(ctx, a, st);
}
