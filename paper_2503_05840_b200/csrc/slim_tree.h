// Shared by the kernels of slim_tree_decode.
#pragma once
#include "slim_internal.h"

// What the kernels of one slim_tree_decode call share: the tree's layout and the scratch arrays of the workspace.
struct SlimTreeView {
  int n;                             // drafted tokens of a sequence (padding included)
  const void* k_tree;                // [batch][n][d]
  unsigned long long* mask;          // [batch][n]  bit j: token i attends drafted key j (0 = padding)
  int* depth;                        // [batch][n]  number of proper ancestors, -1 = padding
  int* len;                          // [batch]     cached rows, clamped into [0, t_cap]
  float* m;                          // [batch][H n] reference exponent of a row (log2 units)
  float* inv_l;                      // [batch][H n] 1 / softmax denominator, 0 = empty row
  float* s;                          // [batch][H n][s_ld] softmax arguments; drafted keys from column s_draft on
  int s_ld, s_draft;
  float* u;                          // [parts][batch][H n][d]
  int parts;
};

struct SlimTreeLayout {
  size_t mask, depth, len, m, inv_l, s, u, total;
  int parts, s_ld, s_draft;
};

SlimTreeLayout slim_tree_ws_layout(const slim_ctx* ctx, int batch, int t_cap, int n);
