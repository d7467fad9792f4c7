// Preparation steps that both paths of slim_prompt_attention share.
#pragma once
#include "slim_attn.h"

constexpr int SLIM_ATTN_BINS = 64;
inline size_t slim_attn_plan_smem(int batch) { return sizeof(int) * ((size_t)batch + 1 + SLIM_ATTN_BINS); }

// The list of query tiles, by one CTA: a counting sort on the number of keys.
static __device__ void slim_attn_plan(const SlimAttn& a, int* s_mem) {
  int* s_prefix = s_mem;                            // [batch + 1] tiles before a sequence
  int* s_bin = s_mem + a.batch + 1;                 // [SLIM_ATTN_BINS]
  const int tid = threadIdx.x;
  for (int b = tid; b < a.batch; b += blockDim.x) s_prefix[b + 1] = (slim_attn_seq(a, b).nq + a.tile_rows - 1) / a.tile_rows;
  if (tid == 0) s_prefix[0] = 0;
  if (tid < SLIM_ATTN_BINS) s_bin[tid] = 0;
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
  for (int pass = 0; pass < 2; ++pass) {
    for (int g = tid; g < n; g += blockDim.x) {
      int lo = 0, hi = a.batch;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_prefix[mid] <= g) lo = mid; else hi = mid;
      }
      const SlimSeq s = slim_attn_seq(a, lo);
      const int row = (g - s_prefix[lo]) * a.tile_rows;
      const int keys = slim_attn_keys(a, s, min(s.nq, row + a.tile_rows) - 1);
      const int bin = SLIM_ATTN_BINS - 1 - (int)((long long)keys * (SLIM_ATTN_BINS - 1) / max(a.max_k, 1));
      if (pass == 0) atomicAdd(&s_bin[bin], 1);
      else {
        int4* to = a.tiles + 2 * atomicAdd(&s_bin[bin], 1);
        to[0] = make_int4(lo, row, 0, 0);
        to[1] = make_int4(s.q0, s.nq, s.k0, s.nk);
      }
    }
    __syncthreads();
    if (pass == 0 && tid == 0) {
      int run = 0;
      for (int i = 0; i < SLIM_ATTN_BINS; ++i) { const int c = s_bin[i]; s_bin[i] = run; run += c; }
      *a.n_tiles = n;
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
