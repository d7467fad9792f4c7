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
#include "slim_attn_tile.cuh"
#include "slim_ptx.cuh"

namespace {
using namespace slim_ptx;

constexpr int THREADS = SLIM_ATTN_THREADS;

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
constexpr int TK = SLIM_ATTN_TK;
template <int DKP, int TR>
__global__ void __launch_bounds__(THREADS) attn_kernel(const __grid_constant__ SlimAttn a) {
  typedef SlimAttnTile<DKP, TR, false> Tile;
  constexpr int RT = Tile::RT, NC = Tile::NC;
  extern __shared__ __align__(16) float smem[];
  slim_pdl_trigger();
  slim_pdl_wait();
  const int item = blockIdx.x / a.H, h = blockIdx.x % a.H;
  if (item >= *a.n_tiles) return;
  const int4 tile = a.tiles[3 * item], range = a.tiles[3 * item + 1], piece = a.tiles[3 * item + 2];
  const SlimSeq s = {range.x, range.y, range.z, range.w};
  const int row0 = tile.y, rows = min(TR, s.nq - row0);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  Tile t;
  t.run(a, s, row0, rows, h, piece.x * TK, (int)min((long long)piece.y * TK, 0x7fffffffll), smem, 0);
  if (tile.w > 1) {
    // A piece of the keys: its sums go to the workspace, and the last piece of the tile to arrive joins them, in their order
    constexpr int WIDE = DKP + 2;
    const size_t slot0 = (size_t)piece.z * a.H + h;              // of the tile's piece i: slot0 + i H
    float* mine = a.part + (slot0 + (size_t)tile.z * a.H) * (TR * WIDE);
    float* s_p = smem;                                           // (a word of it; nobody reads the tiles any more)
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int r = ty * RT + i;
#pragma unroll
      for (int c = 0; c < NC; ++c) *reinterpret_cast<ulonglong2*>(mine + r * DKP + c * 64 + tx * 4) = make_ulonglong2(t.acc[i][c][0], t.acc[i][c][1]);
      if (tx == 0) *reinterpret_cast<float2*>(mine + TR * DKP + 2 * r) = make_float2(t.m[i], t.l[i]);
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
      float m = -INFINITY;
      for (int x = 0; x < tile.w; ++x) m = fmaxf(m, __ldcg(from + x * step + TR * DKP + 2 * r));
      t.l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) t.acc[i][c][0] = t.acc[i][c][1] = pack2(0.f, 0.f);
      for (int x = 0; x < tile.w; ++x) {
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(from + x * step + TR * DKP + 2 * r));
        if (ml.x == -INFINITY && ml.y == 0.f) continue;          // the row attends nothing there
        const float f = exp2f(ml.x - m);
        const f32x2 f2 = pack2(f, f);
        t.l[i] = fmaf(ml.y, f, t.l[i]);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const ulonglong2 v = __ldcg(reinterpret_cast<const ulonglong2*>(from + x * step + r * DKP + c * 64 + tx * 4));
          t.acc[i][c][0] = fma2(f2, v.x, t.acc[i][c][0]);
          t.acc[i][c][1] = fma2(f2, v.y, t.acc[i][c][1]);
        }
      }
    }
  }
  t.store(a, s, row0, rows, h, ~0ull);
}

template <int DKP, int TR>
cudaError_t launch_attn(const SlimAttn& a, cudaStream_t st) {
  constexpr int smem = SlimAttnTile<DKP, TR, false>::SMEM;
  cudaError_t e = cudaFuncSetAttribute((const void*)attn_kernel<DKP, TR>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return slim_launch_pdl(attn_kernel<DKP, TR>, dim3((unsigned)((a.most_tiles + (a.slots + a.H - 1) / a.H) * a.H)), dim3(THREADS), smem, st, a);
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
// Blocks of columns of the widened heads; runs of rows whose values are converted together: 64 rows at least, and two pieces of
// work for each block of the preparation, or 64 runs
int v_blocks(const slim_ctx* ctx, int kv_heads) { return (kv_heads * slim_attn_width(ctx->d_k) + SLIM_ATTN_V_COLS - 1) / SLIM_ATTN_V_COLS; }
int v_runs(const slim_ctx* ctx, int kv_heads, int total_k) {
  const int all = 16 * ctx->num_sms / v_blocks(ctx, kv_heads), most = all > 64 ? all : 64, runs = (total_k + 63) / 64;
  return runs < most ? runs : most;
}
size_t part_bytes(const SlimAttn& a, int columns) { return sizeof(float) * (size_t)a.slots * a.tile_rows * (columns + 2); }

}  // namespace

SlimAttnLayout slim_attn_layout(const slim_ctx* ctx, int kv_heads, int batch, int total_q, int total_k) {
  SlimAttnLayout L;
  SlimAttn a = {};
  a.H = ctx->H; a.batch = batch; a.total_q = total_q; a.total_k = total_k;
  shape_of(ctx, a, false);
  size_t part = part_bytes(a, (ctx->d_k + 63) / 64 * 64), tiles = (size_t)a.most_tiles + a.slots, redo = 0;
  if (slim_attn_tc_ok(ctx)) {
    shape_of(ctx, a, true);
    redo = 8 * sizeof(uint32_t) * ((size_t)a.most_tiles * a.H + a.slots);
    if (part_bytes(a, slim_attn_width(ctx->d_k)) > part) part = part_bytes(a, slim_attn_width(ctx->d_k));
    if ((size_t)a.most_tiles + a.slots > tiles) tiles = (size_t)a.most_tiles + a.slots;
  }
  size_t off = 0;
  // bytes of a head: float32, or 16 bits and widened
  const size_t wide = slim_attn_tc_ok(ctx) ? 2 * (size_t)slim_attn_width(ctx->d_k) : 0, head = wide > 4 * (size_t)ctx->d_k ? wide : 4 * (size_t)ctx->d_k;
  L.qr = off; off = align256(off + head * total_q * ctx->H);
  L.kr = off; off = align256(off + head * total_k * kv_heads);
  L.vb = off; off = align256(off + wide * total_k * kv_heads);
  const size_t columns = wide ? (size_t)v_blocks(ctx, kv_heads) * SLIM_ATTN_V_COLS : 0;
  L.v_max = off; off = align256(off + sizeof(float) * columns * v_runs(ctx, kv_heads, total_k));
  L.v_more = off; off = align256(off + sizeof(float) * columns);
  L.tiles = off; off = align256(off + 3 * sizeof(int4) * tiles);
  L.n_tiles = off; off = align256(off + sizeof(int));
  L.part = off; off = align256(off + part);
  L.arrivals = off; off = align256(off + sizeof(int) * 8 * 4 * (size_t)ctx->num_sms);
  L.redo = off; off = align256(off + redo);
  L.total = off;
  return L;
}

cudaError_t slim_launch_attn(const slim_ctx* ctx, SlimAttn a, char* ws, int tc, cudaStream_t st) {
  const SlimAttnLayout L = slim_attn_layout(ctx, a.KV, a.batch, a.total_q, a.total_k);
  a.qr = ws + L.qr; a.kr = ws + L.kr; a.vb = ws + L.vb;
  a.v_max = reinterpret_cast<float*>(ws + L.v_max); a.v_more = reinterpret_cast<float*>(ws + L.v_more);
  a.v_runs = v_runs(ctx, a.KV, a.total_k);
  a.tiles = reinterpret_cast<int4*>(ws + L.tiles);
  a.n_tiles = reinterpret_cast<int*>(ws + L.n_tiles);
  a.part = reinterpret_cast<float*>(ws + L.part);
  a.arrivals = reinterpret_cast<int*>(ws + L.arrivals);
  a.redo = reinterpret_cast<uint32_t*>(ws + L.redo);
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
