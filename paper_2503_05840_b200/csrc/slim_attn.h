// Attention over packed prompts (slim_prompt_attention): what its kernels share.
#pragma once
#include "slim_internal.h"

// Arguments and scratch of one call.
struct SlimAttn {
  int H, KV, d_k, half;          // query heads, key heads (H / KV query heads share one), head width and half of it
  int batch, total_q, total_k, max_k, causal;
  int f32, v32;                  // types of q, k and o (else bf16), and of v
  float qscale;                  // log2(e) / sqrt(d_k)
  const void* q;                 // [total_q][H][d_k]
  const void* k;                 // [total_k][KV][d_k]
  const void* v;                 // [total_k][KV][d_k]
  void* o;                       // [total_q][H][d_k]
  const int32_t* cu_q;           // [batch + 1]
  const int32_t* cu_k;           // [batch + 1]
  const float2* rope_base;       // position tables; NULL without rotation
  const float2* rope_off;
  int rope_rows;                 // positions that the tables cover
  int* status;
  // workspace
  void* qr;                      // rotated queries and keys, layout of q and k: float32 (CUDA cores) or float16 (tensor cores, heads
  void* kr;                      // widened to slim_attn_width with zeros)
  void* vb;                      // tensor cores: float32 values as float16, or bf16 values of widened heads
  float* v_max;                  // float32 values on the tensor cores: [v_runs][columns] largest finite magnitudes of a run of rows
  float* v_more;                 // [columns] what outputs are to be multiplied by, where a column has a factor of its own
  int v_runs;
  int4* tiles;                   // items, longest first, three entries each: (sequence, first query row, piece, pieces of the tile),
                                 // (q0, nq, k0, nk), (first key tile, key tile behind the last, slot of the tile's first piece, -)
  int* n_tiles;
  int tile_rows, most_tiles;     // query rows of a tile; tiles at most
  int key_rows, least, beside;   // keys of a key tile; key tiles of a piece at least; key tiles that a piece costs beside its own
  int share_of;                  // CTAs that run at a time
  int slots;                     // pieces times heads whose sums fit the workspace (0: nothing is split)
  float* part;                   // [slots][tile_rows][columns + 2]: sums of the pieces (a kernel's own order)
  int* arrivals;                 // [slots][8]
  uint32_t* redo;                // tensor cores: rows to be formed once more, a bit each, 8 words an item and head
};

struct SlimAttnLayout { size_t qr, kr, vb, v_max, v_more, tiles, n_tiles, part, arrivals, redo, total; };

// Columns that a head has on the tensor cores
__host__ __device__ inline int slim_attn_width(int d_k) { return d_k <= 64 ? 64 : d_k <= 96 ? 96 : 128; }
constexpr int SLIM_ATTN_V_COLS = 128;    // columns whose float32 values a block converts
constexpr int SLIM_ATTN_TC_ROWS = 256;   // query rows of an item on the tensor cores: two tiles of 128

int slim_attn_tc_ok(const slim_ctx* ctx);
cudaError_t slim_launch_attn_tc(const slim_ctx* ctx, const SlimAttn& a, cudaStream_t st);
SlimAttnLayout slim_attn_layout(const slim_ctx* ctx, int kv_heads, int batch, int total_q, int total_k);
cudaError_t slim_launch_attn(const slim_ctx* ctx, SlimAttn a, char* ws, int tc, cudaStream_t st);

#ifdef __CUDACC__
struct SlimSeq { int q0, nq, k0, nk; };
// Sequence b; none (nq = 0) where its starts do not ascend within the arrays or it has more than max_k keys.
__device__ __forceinline__ SlimSeq slim_attn_seq(const SlimAttn& a, int b) {
  SlimSeq s;
  s.q0 = a.cu_q[b]; s.k0 = a.cu_k[b];
  const int q1 = a.cu_q[b + 1], k1 = a.cu_k[b + 1];
  if (s.q0 < 0 || q1 < s.q0 || q1 > a.total_q || s.k0 < 0 || k1 < s.k0 || k1 > a.total_k || k1 - s.k0 > a.max_k) {
    atomicMax(a.status, (int)SLIM_ERR_CAPACITY);
    s.nq = s.nk = 0;
    return s;
  }
  s.nq = q1 - s.q0; s.nk = k1 - s.k0;
  return s;
}
// Pieces of a query tile with so many key tiles, where a piece is to have `most` at most
__device__ __forceinline__ int slim_attn_pieces(int tiles, int most) { return tiles > most ? (tiles + most - 1) / most : 1; }
// Keys that query row i of a sequence attends: the first so many.
__device__ __forceinline__ int slim_attn_keys(const SlimAttn& a, const SlimSeq& s, int i) {
  return a.causal ? max(0, min(s.nk, i + 1 + s.nk - s.nq)) : s.nk;
}
// (cos, sin) of a position's angle; a query in front of the first key has a negative one
__device__ __forceinline__ float2 slim_attn_turn(const SlimAttn& a, int pos, int j) {
  const int at = min(abs(pos), a.rope_rows - 1);
  const float2 cb = __ldg(a.rope_base + (size_t)(at / SLIM_TT) * a.half + j), co = __ldg(a.rope_off + (at % SLIM_TT) * a.half + j);
  const float s = cb.y * co.x + cb.x * co.y;
  return make_float2(cb.x * co.x - cb.y * co.y, pos < 0 ? -s : s);
}
__device__ __forceinline__ float slim_attn_ld(const void* p, size_t i, int f32) {
  return f32 ? __ldg(reinterpret_cast<const float*>(p) + i) : __bfloat162float(__ldg(reinterpret_cast<const __nv_bfloat16*>(p) + i));
}
#endif
