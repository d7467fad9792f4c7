// Shared by the kernels of slim_tree_decode.
#pragma once
#include "slim_internal.h"

// What the kernels of one slim_tree_decode call share: the tree's layout and the scratch arrays of the workspace.
struct SlimTreeView {
  int n;                             // drafted tokens of a sequence (padding included)
  const void* k_tree;                // [batch][n][d]
  int* depth;                        // [batch][n]  number of proper ancestors, -1 = padding
  int* len;                          // [batch]     cached rows, clamped into [0, t_cap]
  float* m;                          // [batch][H n] reference exponent of a row (log2 units)
  float* inv_l;                      // [batch][H n] 1 / softmax denominator, 0 = empty row
  float* s;                          // [batch][H n][s_ld] softmax arguments; drafted keys from column s_draft on
  int s_ld, s_draft;
  float* u;                          // [parts][batch][H n][d]
  int parts;
  // tensor-core path
  __nv_bfloat16* p;                  // [batch][H n][p_ld] probabilities relative to their block's reference; drafted keys from s_draft on
  int p_ld;
  float2* stat;                      // [batch][blocks of 128 keys + 1 (drafted)][H n] (reference, sum)
  __nv_bfloat16* tail;               // [batch][128][d] partial last block of cached rows, drafted keys
  __nv_bfloat16* uh;                 // [2][H][batch n][d] weighted sums as (bf16, bf16 of what that leaves)
  float* part;                       // [slots][mt 256][256] sums of pieces that are not whole tiles
  long long* sched;                  // [batch + 1 + pairs + 1 + 1] the product's schedule
  int g_tiles, g_ncol, g_split, g_pairs, g_whole;      // schedule of the product (slim_tree_tc.cu)
};

#ifdef __CUDACC__
// Ancestor mask and depth of token i from the parents of its sequence (shared memory; a parent that is not an earlier
// token has been replaced by -3).  Padding, and what hangs on it, has mask 0 and depth -1; `broken`: the tree is not one there.
__device__ __forceinline__ void slim_tree_chain(const int* s_par, int i, unsigned long long& mask, int& depth, bool& broken) {
  mask = 0; depth = -1;
  bool live = s_par[i] >= -1;
  broken = s_par[i] == -3;
  for (int at = i; live;) {                          // at most n steps: a parent is an earlier token
    mask |= 1ull << at;
    ++depth;
    const int p = s_par[at];
    if (p == -1) break;
    if (p < -1) { live = false; broken = true; }
    at = p;
  }
  if (!live) { mask = 0; depth = -1; }
}
#endif

struct SlimTreeLayout {
  size_t depth, len, inv_l, shared_end;
  size_t m, s, u;                    // CUDA-core kernels
  size_t p, stat, tail, uh, part, sched;    // tensor-core kernels (their scratch and the other kernels' share the same memory)
  size_t total;
  int parts, s_ld, s_draft;
  int mt, p_ld, p_s_draft, g_tiles, g_ncol, g_split, g_pairs, g_whole;
};

int  slim_tree_tc_ok(const slim_ctx* ctx);
void slim_tree_tc_layout(const slim_ctx* ctx, int batch, int t_cap, int n, SlimTreeLayout& L);
cudaError_t slim_launch_tree_tc(const slim_ctx* ctx, const SlimDecodeParams& p, const SlimTreeView& t, const SlimTreeLayout& L,
                                const int32_t* parents, long long total_rows, void* o, cudaStream_t st);
SlimTreeLayout slim_tree_ws_layout(const slim_ctx* ctx, int batch, int t_cap, int n);
