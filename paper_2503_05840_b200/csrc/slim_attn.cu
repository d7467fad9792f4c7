// Attention over packed prompts (slim_prompt_attention): preparation and the CUDA-core kernel.
//
//   o_i = sum_j p_ij v_j,  p_ij = softmax_j(R(i) q_i . R(j) k_j / sqrt(d_k)),  j <= i + nk - nq where causal
//
// Preparation (one kernel): rotated queries and keys into the workspace, each once instead of once a tile that reads them,
// and the list of query tiles, most keys first, so that the last tiles to start are the short ones.
// attn_kernel: one CTA a (tile of 64 or 32 query rows, piece of the keys, head); online softmax over tiles of 64 keys,
// everything float32.  Bound by the latency of its chain (products, maximum, exponentials, products) for few tiles, by
// the FMA pipe and shared memory's reads for many.  448 tokens, 6 heads of 64, causal: 20 us and 8 of preparation (the plan
// alone); 256 queries over 8192 keys, 8 heads: 222 us (19 TFLOP/s).
#include <cuda_fp16.h>

#include "slim_attn.h"
#include "slim_attn_plan.cuh"
#include "slim_ptx.cuh"

namespace {
using namespace slim_ptx;

constexpr int THREADS = 256;

// ------------------------------------------------------------------------------------------------ preparation
// One warp a packed row: all its heads, rotated.
template <bool F32>
__device__ void rotate_row(const SlimAttn& a, int r, bool query) {
  const int lane = threadIdx.x & 31, heads = query ? a.H : a.KV;
  int pos;
  if (!slim_attn_position(a, r, query, pos)) return;
  const size_t at = (size_t)r * heads * a.d_k;
  const void* src = query ? a.q : a.k;
  void* dst = query ? a.qr : a.kr;
  for (int j = lane; j < a.half; j += 32) {
    const float2 cs = a.rope_base ? slim_attn_turn(a, pos, j) : make_float2(1.f, 0.f);      // (bf16 rows are widened all the same)
    for (int h = 0; h < heads; ++h) {
      const size_t i = at + (size_t)h * a.d_k + j;
      const float x1 = slim_attn_ld(src, i, F32), x2 = slim_attn_ld(src, i + a.half, F32);
      reinterpret_cast<float*>(dst)[i] = a.rope_base ? x1 * cs.x + x2 * cs.y : x1;
      reinterpret_cast<float*>(dst)[i + a.half] = a.rope_base ? x2 * cs.x - x1 * cs.y : x2;
    }
  }
}

template <bool F32>
__global__ void __launch_bounds__(THREADS) attn_prepare_kernel(const __grid_constant__ SlimAttn a) {
  extern __shared__ int s_mem[];
  slim_pdl_trigger();
  slim_pdl_wait();
  if (blockIdx.x == 0) { slim_attn_plan(a, s_mem); return; }
  const int warps = (gridDim.x - 1) * (THREADS / 32);                  // (none where the inputs are read where they lie)
  for (int r = (blockIdx.x - 1) * (THREADS / 32) + (threadIdx.x >> 5); r < a.total_q + a.total_k; r += warps)
    rotate_row<F32>(a, r < a.total_q ? r : r - a.total_q, r < a.total_q);
}

// ------------------------------------------------------------------------------------------------ CUDA cores
constexpr int TK = 64;
// TR: query rows of a tile, 64 or 32; DKP: the head width rounded up to a multiple of 64, columns behind d_k are zero.
// Thread (ty, tx) = (tid / 16, tid % 16) has RT = TR / 16 rows, RT ty and the next; scores of keys tx, tx + 16, ..; outputs 4 tx + 64 c.
// Products in packed float32: even and odd columns of a score, neighbouring outputs.
__host__ __device__ constexpr int attn_stages(int dkp) { return dkp <= 128 ? 2 : 1; }      // (two of wider ones do not fit)
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool in) {          // zeros where `in` does not hold
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
template <int DKP, int TR, bool F32>
__global__ void __launch_bounds__(THREADS) attn_kernel(const __grid_constant__ SlimAttn a) {
  constexpr int PQ = DKP + 4, PP = TK + 4;                       // pitches that spread rows over the banks
  constexpr int NC = DKP / 64, NT = THREADS, RT = 16 * TR / NT;
  extern __shared__ __align__(16) float smem[];
  constexpr int ST = attn_stages(DKP), KS = TK * PQ, VS = TK * DKP;      // key tiles in shared memory
  float* s_q = smem;                                             // [TR][PQ]
  float* s_k0 = s_q + TR * PQ;                                   // [ST][TK][PQ]
  float* s_v0 = s_k0 + ST * KS;                                  // [ST][TK][DKP]
  float* s_p = s_v0 + ST * VS;                                   // [TR][PP]
  slim_pdl_trigger();
  slim_pdl_wait();
  const int item = blockIdx.x / a.H, h = blockIdx.x % a.H;
  if (item >= *a.n_tiles) return;
  const int4 tile = a.tiles[3 * item], range = a.tiles[3 * item + 1], piece = a.tiles[3 * item + 2];
  const SlimSeq s = {range.x, range.y, range.z, range.w};
  const int row0 = tile.y, rows = min(TR, s.nq - row0), dk = a.d_k, kvh = h / (a.H / a.KV);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const float* qr = reinterpret_cast<const float*>(a.qr) + ((size_t)(s.q0 + row0) * a.H + h) * dk;
  const float* kr = reinterpret_cast<const float*>(a.kr) + ((size_t)s.k0 * a.KV + kvh) * dk;
#pragma unroll 8
  for (int e = tid; e < TR * DKP; e += NT) {
    const int r = e / DKP, c = e % DKP;
    s_q[r * PQ + c] = r < rows && c < dk ? qr[(size_t)r * a.H * dk + c] * a.qscale : 0.f;
  }
  int lim[RT];
  float m[RT], l[RT];
  f32x2 acc[RT][NC][2];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    lim[i] = slim_attn_keys(a, s, row0 + ty * RT + i);
    m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[i][c][0] = acc[i][c][1] = pack2(0.f, 0.f);
  }
  const int first = piece.x * TK, keys = min(slim_attn_keys(a, s, row0 + rows - 1), (int)min((long long)piece.y * TK, 0x7fffffffll));
  // Key tile t0 into stage st: 16 bytes at a time behind the products of the tile before it, or element by element (d_k not a
  // multiple of four, bf16 values)
  const bool vec = (dk & 3) == 0 && a.v32;
  const float* vr = reinterpret_cast<const float*>(a.v) + ((size_t)s.k0 * a.KV + kvh) * dk;
  auto load = [&](int t0, int st) {
    float* s_k = s_k0 + st * KS;
    float* s_v = s_v0 + st * VS;
    if (vec) {
#pragma unroll 8
      for (int e = tid; e < TK * DKP / 4; e += NT) {
        const int r = e / (DKP / 4), c = e % (DKP / 4) * 4;
        const bool in = t0 + r < keys && c < dk;
        const size_t at = in ? (size_t)(t0 + r) * a.KV * dk + c : 0;
        cp_async16(smem_u32(s_k + r * PQ + c), kr + at, in);
        cp_async16(smem_u32(s_v + r * DKP + c), vr + at, in);
      }
    } else {
#pragma unroll 8
      for (int e = tid; e < TK * DKP; e += NT) {
        const int r = e / DKP, c = e % DKP;
        const bool in = t0 + r < keys && c < dk;
        s_k[r * PQ + c] = in ? kr[(size_t)(t0 + r) * a.KV * dk + c] : 0.f;
        s_v[r * DKP + c] = in ? slim_attn_ld(a.v, ((size_t)(s.k0 + t0 + r) * a.KV + kvh) * dk + c, a.v32) : 0.f;
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (first < keys) load(first, 0);
  int st = 0;
  for (int t0 = first; t0 < keys; t0 += TK) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();                                             // this tile is there, and nobody reads the one before it any more
    const float* s_k = s_k0 + st * KS;
    const float* s_v = s_v0 + st * VS;
    if (ST == 2 && t0 + TK < keys) load(t0 + TK, st ^ 1);
    f32x2 sv2[RT][4];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) sv2[i][j] = pack2(0.f, 0.f);
#pragma unroll 4
    for (int c = 0; c < DKP; c += 4) {
      ulonglong2 qv[RT], kv[4];
#pragma unroll
      for (int i = 0; i < RT; ++i) qv[i] = *reinterpret_cast<const ulonglong2*>(s_q + (ty * RT + i) * PQ + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const ulonglong2*>(s_k + (tx + 16 * j) * PQ + c);
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sv2[i][j] = fma2(qv[i].y, kv[j].y, fma2(qv[i].x, kv[j].x, sv2[i][j]));
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float mx = m[i], sv[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sv[j] = t0 + tx + 16 * j >= lim[i] ? -INFINITY : sum2(sv2[i][j]);
        mx = fmaxf(mx, sv[j]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float alpha = mx == m[i] ? 1.f : exp2f(m[i] - mx);
      float ps = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = t0 + tx + 16 * j >= lim[i] ? 0.f : exp2f(sv[j] - mx);
        s_p[(ty * RT + i) * PP + tx + 16 * j] = p;
        ps += p;
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, o);
      l[i] = l[i] * alpha + ps;
      m[i] = mx;
      const f32x2 al = pack2(alpha, alpha);
#pragma unroll
      for (int c = 0; c < NC; ++c) { acc[i][c][0] = mul2(acc[i][c][0], al); acc[i][c][1] = mul2(acc[i][c][1], al); }
    }
    __syncwarp();                                                // a row's probabilities come from its own half warp
#pragma unroll 2
    for (int t = 0; t < TK; t += 4) {
      float pv[RT][4];
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const float4 v = *reinterpret_cast<const float4*>(s_p + (ty * RT + i) * PP + t);
        pv[i][0] = v.x; pv[i][1] = v.y; pv[i][2] = v.z; pv[i][3] = v.w;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(s_v + (t + u) * DKP + c * 64 + tx * 4);
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            const f32x2 pp = pack2(pv[i][u], pv[i][u]);
            acc[i][c][0] = fma2(pp, v.x, acc[i][c][0]);
            acc[i][c][1] = fma2(pp, v.y, acc[i][c][1]);
          }
        }
    }
    if (ST == 2) {
      st ^= 1;
    } else if (t0 + TK < keys) {
      __syncthreads();
      load(t0 + TK, 0);
    }
  }
  if (tile.w > 1) {
    // A piece of the keys: its sums go to the workspace, and the last piece of the tile to arrive joins them, in their order
    constexpr int WIDE = DKP + 2;
    const size_t slot0 = (size_t)piece.z * a.H + h;              // of the tile's piece i: slot0 + i H
    float* mine = a.part + (slot0 + (size_t)tile.z * a.H) * (TR * WIDE);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int r = ty * RT + i;
#pragma unroll
      for (int c = 0; c < NC; ++c) *reinterpret_cast<ulonglong2*>(mine + r * DKP + c * 64 + tx * 4) = make_ulonglong2(acc[i][c][0], acc[i][c][1]);
      if (tx == 0) *reinterpret_cast<float2*>(mine + TR * DKP + 2 * r) = make_float2(m[i], l[i]);
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) s_p[0] = __int_as_float(atomicAdd(a.arrivals + 8 * slot0, 1));
    __syncthreads();
    if (__float_as_int(s_p[0]) != tile.w - 1) return;
    __threadfence();
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int r = ty * RT + i;
      const float* from = a.part + slot0 * (TR * WIDE);
      const size_t step = (size_t)a.H * (TR * WIDE);
      m[i] = -INFINITY; l[i] = 0.f;
      for (int x = 0; x < tile.w; ++x) m[i] = fmaxf(m[i], __ldcg(from + x * step + TR * DKP + 2 * r));
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[i][c][0] = acc[i][c][1] = pack2(0.f, 0.f);
      for (int x = 0; x < tile.w; ++x) {
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(from + x * step + TR * DKP + 2 * r));
        if (ml.x == -INFINITY && ml.y == 0.f) continue;          // the row attends nothing there
        const float f = exp2f(ml.x - m[i]);
        const f32x2 f2 = pack2(f, f);
        l[i] = fmaf(ml.y, f, l[i]);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const ulonglong2 v = __ldcg(reinterpret_cast<const ulonglong2*>(from + x * step + r * DKP + c * 64 + tx * 4));
          acc[i][c][0] = fma2(f2, v.x, acc[i][c][0]);
          acc[i][c][1] = fma2(f2, v.y, acc[i][c][1]);
        }
      }
    }
  }
  bool bad[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int r = ty * RT + i;
    const float inv = lim[i] > 0 ? 1.f / l[i] : 0.f;
    bad[i] = false;
    if (r >= rows) continue;
    const size_t at = ((size_t)(s.q0 + row0 + r) * a.H + h) * dk;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int col = c * 64 + tx * 4 + x;
        float lo, hi;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(acc[i][c][x >> 1]));
        const float y = lim[i] > 0 ? (x & 1 ? hi : lo) * inv : 0.f;
        if (col < dk) {
          bad[i] |= !(fabsf(y) <= 3.4028234663852886e38f);
          if (F32) reinterpret_cast<float*>(a.o)[at + col] = y;
          else reinterpret_cast<__nv_bfloat16*>(a.o)[at + col] = __float2bfloat16_rn(y);
        }
      }
  }
  // rows with a number that is not finite: once more, from what they attend alone
  __syncwarp();
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const unsigned any = __ballot_sync(0xffffffffu, bad[i]);
    const int r = (ty & ~1) * RT + i;                            // the warp's rows: RT of its lower half, RT of its upper
    if (any & 0x0000ffffu) slim_attn_row(a, tile.x, row0 + r, h);
    if (any & 0xffff0000u) slim_attn_row(a, tile.x, row0 + r + RT, h);
  }
}

template <int DKP, int TR>
cudaError_t launch_attn(const SlimAttn& a, cudaStream_t st) {
  const size_t smem = sizeof(float) * (TR * (DKP + 4) + attn_stages(DKP) * (TK * (DKP + 4) + TK * DKP) + TR * (TK + 4));
  auto kern = a.f32 ? attn_kernel<DKP, TR, true> : attn_kernel<DKP, TR, false>;
  cudaError_t e = cudaFuncSetAttribute((const void*)kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return slim_launch_pdl(kern, dim3((unsigned)((a.most_tiles + (a.slots + a.H - 1) / a.H) * a.H)), dim3(THREADS), smem, st, a);
}
template <int DKP>
cudaError_t launch_attn(const SlimAttn& a, cudaStream_t st) { return a.tile_rows == 32 ? launch_attn<DKP, 32>(a, st) : launch_attn<DKP, 64>(a, st); }

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Tiles of one path, and the pieces that they may be split into
void shape_of(const slim_ctx* ctx, SlimAttn& a, bool tc) {
  // Tiles of 32 query rows where those of 64 would not give every SM one (one sequence of 448 tokens, 6 heads, float32:
  // the call 34 us instead of 38).
  a.tile_rows = tc ? SLIM_ATTN_TC_ROWS : (long long)(a.total_q / 64 + a.batch) * a.H < ctx->num_sms ? 32 : 64;
  a.most_tiles = a.total_q / a.tile_rows + a.batch;
  a.key_rows = tc ? 128 : TK;
  a.least = tc ? 4 : 2;
  a.beside = tc ? 4 : 1;
  a.share_of = ctx->num_sms * (!tc && ctx->d_k <= 64 ? 2 : 1);          // (two CTAs of the narrow CUDA-core kernel fit an SM)
  const long long run = (long long)a.key_rows * a.least, pieces = (a.total_k + run - 1) / run;
  // (two query tiles for every SM or more: nothing is split)
  const long long all = pieces > 1 && (long long)(a.total_q / a.tile_rows) * a.H < 2ll * ctx->num_sms ? (long long)a.most_tiles * a.H * pieces : 0;
  a.slots = (int)(all < 2ll * a.share_of ? all : 2ll * a.share_of);
}
size_t part_bytes(const SlimAttn& a, int columns) { return sizeof(float) * (size_t)a.slots * a.tile_rows * (columns + 2); }

}  // namespace

SlimAttnLayout slim_attn_layout(const slim_ctx* ctx, int kv_heads, int batch, int total_q, int total_k) {
  SlimAttnLayout L;
  SlimAttn a = {};
  a.H = ctx->H; a.batch = batch; a.total_q = total_q; a.total_k = total_k;
  shape_of(ctx, a, false);
  size_t part = part_bytes(a, (ctx->d_k + 63) / 64 * 64), tiles = (size_t)a.most_tiles + a.slots;
  if (slim_attn_tc_ok(ctx)) {
    shape_of(ctx, a, true);
    if (part_bytes(a, slim_attn_width(ctx->d_k)) > part) part = part_bytes(a, slim_attn_width(ctx->d_k));
    if ((size_t)a.most_tiles + a.slots > tiles) tiles = (size_t)a.most_tiles + a.slots;
  }
  size_t off = 0;
  // bytes of a head: float32, or 16 bits and widened
  const size_t wide = slim_attn_tc_ok(ctx) ? 2 * (size_t)slim_attn_width(ctx->d_k) : 0, head = wide > 4 * (size_t)ctx->d_k ? wide : 4 * (size_t)ctx->d_k;
  L.qr = off; off = align256(off + head * total_q * ctx->H);
  L.kr = off; off = align256(off + head * total_k * kv_heads);
  L.vb = off; off = align256(off + wide * total_k * kv_heads);
  L.tiles = off; off = align256(off + 3 * sizeof(int4) * tiles);
  L.n_tiles = off; off = align256(off + sizeof(int));
  L.part = off; off = align256(off + part);
  L.arrivals = off; off = align256(off + sizeof(int) * 8 * 4 * (size_t)ctx->num_sms);
  L.total = off;
  return L;
}

cudaError_t slim_launch_attn(const slim_ctx* ctx, SlimAttn a, char* ws, int tc, cudaStream_t st) {
  const SlimAttnLayout L = slim_attn_layout(ctx, a.KV, a.batch, a.total_q, a.total_k);
  a.qr = ws + L.qr; a.kr = ws + L.kr; a.vb = ws + L.vb;
  a.tiles = reinterpret_cast<int4*>(ws + L.tiles);
  a.n_tiles = reinterpret_cast<int*>(ws + L.n_tiles);
  a.part = reinterpret_cast<float*>(ws + L.part);
  a.arrivals = reinterpret_cast<int*>(ws + L.arrivals);
  tc = tc && a.total_k > 0;                              // (a tensor map needs a row)
  shape_of(ctx, a, tc);
  if (tc) return slim_launch_attn_tc(ctx, a, st);
  const bool as_is = a.f32 && !a.rope_base;              // nothing to rotate, nothing to widen
  if (as_is) { a.qr = const_cast<void*>(a.q); a.kr = const_cast<void*>(a.k); }
  const int rows = as_is ? 0 : a.total_q + a.total_k;
  const int blocks = 1 + (int)((rows + 7ll) / 8 < 8ll * ctx->num_sms ? (rows + 7ll) / 8 : 8ll * ctx->num_sms);
  const size_t smem = slim_attn_plan_smem(a.batch);
  cudaError_t e = a.f32 ? slim_launch_pdl(attn_prepare_kernel<true>, dim3(blocks), dim3(THREADS), smem, st, a)
                        : slim_launch_pdl(attn_prepare_kernel<false>, dim3(blocks), dim3(THREADS), smem, st, a);
  if (e != cudaSuccess) return e;
  return a.d_k <= 64 ? launch_attn<64>(a, st) : a.d_k <= 128 ? launch_attn<128>(a, st) : a.d_k <= 192 ? launch_attn<192>(a, st) : launch_attn<256>(a, st);
}
