// Preparation steps that both paths of slim_prompt_attention share.
#pragma once
#include "slim_attn.h"

constexpr int SLIM_ATTN_BINS = 64;
inline size_t slim_attn_plan_smem(int batch) { return sizeof(int) * ((size_t)batch + 1 + SLIM_ATTN_BINS) + 64; }

// The list of items, by one CTA: a counting sort on the number of keys.
// Where the longest query tile has more than twice the key tiles that are a CTA's share of the whole work, query tiles are split
// along their keys into pieces of a share or somewhat more (`least` key tiles at least), whose sums are joined by the last of
// them to finish: else a few long tiles keep their CTAs while the others have nothing left (512 queries over 8192 keys, 16
// heads: the attention kernel 113 us in one piece, 50 in pieces).  Below that the pieces' sums cost more than they give (512
// queries over 4096 keys and 512 over 1536, 32 heads, 1.4 shares: the call 145 us in one piece and 164 in pieces).
// With c key tiles in a tile, H heads, n CTAs and L tiles a piece, a split tile (c > L) has less than c / L + 1 < 2 c / L pieces, and
// L is at least H sum(c) / n, so H times all their pieces stay below 2 n.
static __device__ void slim_attn_plan(const SlimAttn& a, int* s_mem) {
  int* s_prefix = s_mem;                            // [batch + 1] tiles before a sequence
  int* s_bin = s_mem + a.batch + 1;                 // [SLIM_ATTN_BINS]
  int* s_slot = s_bin + SLIM_ATTN_BINS;             // slots given out
  int* s_high = s_slot + 1;                         // key tiles of the longest query tile, of all
  int* s_count = s_high + 1;                        // [9]
  unsigned long long* s_work = reinterpret_cast<unsigned long long*>((reinterpret_cast<uintptr_t>(s_count + 9) + 7) & ~(uintptr_t)7);
  const int tid = threadIdx.x;
  for (int b = tid; b < a.batch; b += blockDim.x) s_prefix[b + 1] = (slim_attn_seq(a, b).nq + a.tile_rows - 1) / a.tile_rows;
  if (tid == 0) { s_prefix[0] = 0; *s_slot = 0; *s_high = 0; *s_work = 0; }
  if (tid < SLIM_ATTN_BINS) s_bin[tid] = 0;
  if (tid < 9) s_count[tid] = 0;
  __syncthreads();
  if (tid < 32) {
    const int chunk = (a.batch + 31) / 32, lo = tid * chunk, hi = min(a.batch, lo + chunk);
    int sum = 0;
    for (int b = lo; b < hi; ++b) sum += s_prefix[b + 1];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (tid >= o) incl += v;
    }
    int run = incl - sum;
    for (int b = lo; b < hi; ++b) { run += s_prefix[b + 1]; s_prefix[b + 1] = run; }
  }
  __syncthreads();
  const int n = min(s_prefix[a.batch], a.most_tiles);         // (more only where sequences overlap)
  if (tid == 0 && n < s_prefix[a.batch]) atomicMax(a.status, (int)SLIM_ERR_CAPACITY);
  // Query tile g's sequence and first row; its key tiles.  A thread keeps those of its first tile, mostly its only one.
  int kept_b = 0, kept_row = 0, kept = -1;
  SlimSeq kept_s = {};
  auto tile_of = [&](int g, int& b, int& row, SlimSeq& s) {
    if (g == tid && kept >= 0) { b = kept_b; row = kept_row; s = kept_s; return kept; }
    int lo = 0, hi = a.batch;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_prefix[mid] <= g) lo = mid; else hi = mid;
    }
    b = lo;
    s = slim_attn_seq(a, lo);
    row = (g - s_prefix[lo]) * a.tile_rows;
    const int tiles = (slim_attn_keys(a, s, min(s.nq, row + a.tile_rows) - 1) + a.key_rows - 1) / a.key_rows;
    if (g == tid) { kept_b = b; kept_row = row; kept_s = s; kept = tiles; }
    return tiles;
  };
  int b, row;
  SlimSeq s;
  int most = 0x7fffffff;                                       // key tiles of a piece
  if (a.slots > 0) {
    unsigned long long mine = 0;
    int high = 0;
    for (int g = tid; g < n; g += blockDim.x) {
      const int tiles = tile_of(g, b, row, s);
      mine += (unsigned)tiles;
      high = max(high, tiles);
    }
    if (mine) { atomicAdd(s_work, mine); atomicMax(s_high, high); }
    __syncthreads();
    const unsigned long long share = (*s_work * a.H + a.share_of - 1) / a.share_of;
    if ((unsigned long long)*s_high > 2 * share) {
      // Of nine lengths from one to two shares the one that takes least: rounds of all CTAs times the length and what a
      // piece costs beside
      const int base = max((int)share, a.least);
      int count[9] = {};
      for (int g = tid; g < n; g += blockDim.x) {
        const int tiles = tile_of(g, b, row, s);
#pragma unroll
        for (int i = 0; i < 9; ++i) count[i] += slim_attn_pieces(tiles, base + (int)((long long)base * i / 8));
      }
#pragma unroll
      for (int i = 0; i < 9; ++i)
        if (count[i]) atomicAdd(&s_count[i], count[i]);
      __syncthreads();
      float best = INFINITY;
#pragma unroll
      for (int i = 0; i < 9; ++i) {
        const int len = base + (int)((long long)base * i / 8);
        const float cost = ceilf((float)s_count[i] * (float)a.H / (float)a.share_of) * (float)(len + a.beside);
        if (cost < best) { best = cost; most = len; }
      }
    }
    for (int i = tid; i < a.slots * 8; i += blockDim.x) a.arrivals[i] = 0;
  }
  // bins: by the length of a piece
  const float per_bin = (float)(SLIM_ATTN_BINS - 1) / (float)max(1, min(most, (int)(((long long)a.max_k + a.key_rows - 1) / a.key_rows)));
  for (int pass = 0; pass < 2; ++pass) {
    for (int g = tid; g < n; g += blockDim.x) {
      const int tiles = tile_of(g, b, row, s), pieces = slim_attn_pieces(tiles, most);
      const int each = tiles / pieces, more = tiles - each * pieces;      // the first `more` pieces have a key tile more
      const int slot = pass == 1 && pieces > 1 ? atomicAdd(s_slot, pieces) : 0;
      for (int i = 0; i < pieces; ++i) {
        const int first = i * each + min(i, more), end = first + each + (i < more);
        const int bin = max(0, SLIM_ATTN_BINS - 1 - (int)((float)(end - first) * per_bin));
        if (pass == 0) atomicAdd(&s_bin[bin], 1);
        else {
          int4* to = a.tiles + 3 * (size_t)atomicAdd(&s_bin[bin], 1);
          to[0] = make_int4(b, row, i, pieces);
          to[1] = make_int4(s.q0, s.nq, s.k0, s.nk);
          to[2] = make_int4(first, end, slot, 0);
        }
      }
    }
    __syncthreads();
    if (pass == 0 && tid < 32) {
      static_assert(SLIM_ATTN_BINS == 64, "two bins a lane");
      const int c0 = s_bin[2 * tid], c1 = s_bin[2 * tid + 1];
      int incl = c0 + c1;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (tid >= o) incl += v;
      }
      s_bin[2 * tid] = incl - c0 - c1;
      s_bin[2 * tid + 1] = incl - c1;
      if (tid == 31) *a.n_tiles = incl;
    }
    __syncthreads();
  }
}

// Position of packed row r among the queries (keys); false: nothing needs the row (it belongs to no sequence, or attends nothing).
static __device__ bool slim_attn_position(const SlimAttn& a, int r, bool query, int& pos) {
  const int32_t* cu = query ? a.cu_q : a.cu_k;
  const SlimSeq s = slim_attn_seq(a, slim_warp_find(cu, a.batch, r));
  pos = query ? r - s.q0 + s.nk - s.nq : r - s.k0;
  if (query ? r < s.q0 || r >= s.q0 + s.nq || (a.causal && pos < 0) : r < s.k0 || r >= s.k0 + s.nk) return false;
  if (a.rope_base && pos <= -a.rope_rows) atomicMax(a.status, (int)SLIM_ERR_CAPACITY);       // (taken as the last covered one)
  return true;
}
