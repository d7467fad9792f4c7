// Drafted tokens: verification against the target's probabilities (slim_tree_verify) and commit of the accepted
// tokens' keys into the K-cache (slim_tree_commit).
#include <cooperative_groups.h>

#include "slim_internal.h"

namespace cg = cooperative_groups;

namespace {

// Verification of one sequence by a cluster of VC CTAs; each warp of the cluster owns one contiguous range of the
// vocabulary.  The walk (which child is tested next, what it is tested against) is the same in every thread: the
// numbers it needs of a child -- target and draft probability of its token after its parent -- are fetched for all
// nodes at once before it starts, so an accepted child costs no trip to memory.  A rejected child costs one pass over
// the vocabulary for the mass S' of the residual W' = max(W - S q, 0), whose elements are recomputed from p and q
// through the chain of masses (a stage holds one double, not a vocabulary); the final draw costs one pass more, or
// none where the last rejection's masses are still there, and a scan of the one warp range that holds the drawn token.
// Everything is float64: a test next to its border and a draw next to a token's edge must not depend on the order of
// a sum.  Bound: latency of the passes (V = 131072: 128 KB of p and q a CTA); a cluster of eight keeps a pass near a
// microsecond where one CTA would take eight.  One sequence of 5 nodes, V = 32000: 9.6 us; 64 sequences of 16 nodes,
// V = 131072: 37 to 47 us, by box and clock (1.4 to 1.8 TB/s of the rows that a walk without rejections reads, about three
// times that with them).
constexpr int VC = 8;

template <int VW>
struct VerifyShared {
  int par[SLIM_MAX_TREE], tok[SLIM_MAX_TREE], path[SLIM_MAX_TREE];
  double r[SLIM_MAX_TREE], px[SLIM_MAX_TREE], qx[SLIM_MAX_TREE];
  double stage[SLIM_MAX_TREE];       // masses S of the rejections at the current node
  double warp_sum[VW];               // this CTA's ranges, last pass
  double cta_sum[2][VC];             // every CTA's sum of a pass (written by its owner into all; double-buffered)
  double piece[VW];                  // the final draw: sums of the warps' pieces
  int first, last, next;
};

// max(x, 0), and NaN for a NaN (fmax would return the 0): a row with a NaN has no mass, before a rejection as behind it
__device__ __forceinline__ double positive(double x) { return x < 0.0 ? 0.0 : x; }

// W(x) after the rejections whose masses are in `stage`: the products and differences are rounded one by one, so a stage
// is a function of its inputs alone.  NS >= 0: that many, in registers; NS < 0: ns of them, in shared memory.
template <int NS>
__device__ __forceinline__ double residual(float p, float q, const double* stage, int ns) {
  double w = (double)p;
  if (NS == 0) return w;
  const double qd = (double)q;
  if (NS > 0) {
#pragma unroll
    for (int k = 0; k < (NS > 0 ? NS : 1); ++k) w = positive(__dsub_rn(w, __dmul_rn(stage[k], qd)));
  } else {
    for (int k = 0; k < ns; ++k) w = positive(__dsub_rn(w, __dmul_rn(stage[k], qd)));
  }
  return w;
}

// This lane's share of sum W over [lo, hi) of a row: two 16-byte loads of p and q each in flight.
template <int NS>
__device__ __forceinline__ double range_sum(const float* __restrict__ pu, const float* __restrict__ qu, int lo, int hi, int lane, bool vec,
                                            const double* s_stage, int ns) {
  double stage[NS > 0 ? NS : 1];
  if (NS > 0)
#pragma unroll
    for (int k = 0; k < (NS > 0 ? NS : 1); ++k) stage[k] = s_stage[k];
  const double* st = NS > 0 ? stage : s_stage;
  double a = 0.0;
  if (vec) {
    for (int x0 = lo + 4 * lane; x0 < hi; x0 += 256) {
      float4 p4[2], q4[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int x = x0 + 128 * y;
        p4[y] = q4[y] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (x < hi) {
          p4[y] = __ldg(reinterpret_cast<const float4*>(pu + x));
          if (NS != 0) q4[y] = __ldg(reinterpret_cast<const float4*>(qu + x));
        }
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        a += residual<NS>(p4[y].x, q4[y].x, st, ns) + residual<NS>(p4[y].y, q4[y].y, st, ns);
        a += residual<NS>(p4[y].z, q4[y].z, st, ns) + residual<NS>(p4[y].w, q4[y].w, st, ns);
      }
    }
  } else {
#pragma unroll 4
    for (int x = lo + lane; x < hi; x += 32) a += residual<NS>(pu[x], NS != 0 ? qu[x] : 0.f, st, ns);
  }
  return a;
}

// VT threads a CTA: 512 while all CTAs fit the SMs twice over, 256 above (64 registers a thread: four of them an SM).
template <int VT>
__global__ void __cluster_dims__(VC, 1, 1) __launch_bounds__(VT, 1024 / VT)
slim_tree_verify_kernel(const float* __restrict__ P, const float* __restrict__ Q, const int32_t* __restrict__ tokens,
                        const int32_t* __restrict__ parents, const float* __restrict__ rnd, int n, int V, int32_t* __restrict__ path,
                        int32_t* __restrict__ count, int32_t* __restrict__ next_token, int* status) {
  constexpr int VW = VT / 32;
  __shared__ VerifyShared<VW> sh;
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = (int)cluster.block_rank(), b = blockIdx.x / VC;
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // (waited for before anything is written into a peer)
  slim_pdl_trigger();
  slim_pdl_wait();
  const float* Pb = P + (size_t)b * n * V;
  const float* Qb = Q + (size_t)b * n * V;
  if (tid < n) {
    const int par = parents[(size_t)b * n + tid], tok = tokens[(size_t)b * n + tid];
    bool child = tid > 0 && par >= 0;
    // (node 0 is the root whatever its parent says, so a parent that is padding is another node below -1)
    if (child && (par >= tid || tok < 0 || tok >= V || (par > 0 && parents[(size_t)b * n + par] < -1))) {
      child = false;
      if (rank == 0) atomicMax(status, (int)SLIM_ERR_TREE);
    }
    sh.par[tid] = child ? par : -2;
    sh.tok[tid] = child ? tok : 0;
    sh.r[tid] = (double)rnd[(size_t)b * n + tid];
    sh.px[tid] = child ? (double)Pb[(size_t)par * V + tok] : 0.0;
    sh.qx[tid] = child ? (double)Qb[(size_t)par * V + tok] : 0.0;
  }
  if (tid == 0) sh.next = -1;
  __syncthreads();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");

  // warp ranges: multiples of 4 elements, so that rows of a vocabulary that is one are read 16 bytes at a time
  const int range = ((V + VC * VW - 1) / (VC * VW) + 3) & ~3;
  const int lo = min(V, (rank * VW + warp) * range), hi = min(V, lo + range);
  const bool vec = (V & 3) == 0 && (((uintptr_t)P | (uintptr_t)Q) & 15) == 0;
  int pass = 0;
  double total = 0.0;
  // sum of W over the vocabulary after ns rejections at node u
  auto sum_pass = [&](int u, int ns) {
    const float* pu = Pb + (size_t)u * V;
    const float* qu = Qb + (size_t)u * V;
    double a;
    switch (ns) {
      case 0: a = range_sum<0>(pu, qu, lo, hi, lane, vec, sh.stage, 0); break;
      case 1: a = range_sum<1>(pu, qu, lo, hi, lane, vec, sh.stage, 1); break;
      case 2: a = range_sum<2>(pu, qu, lo, hi, lane, vec, sh.stage, 2); break;
      case 3: a = range_sum<3>(pu, qu, lo, hi, lane, vec, sh.stage, 3); break;
      default: a = range_sum<-1>(pu, qu, lo, hi, lane, vec, sh.stage, ns);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    if (lane == 0) sh.warp_sum[warp] = a;
    __syncthreads();
    if (tid < VC) {
      double s = 0.0;
      for (int w = 0; w < VW; ++w) s += sh.warp_sum[w];
      cluster.map_shared_rank(&sh, tid)->cta_sum[pass & 1][rank] = s;
    }
    cluster.sync();
    double s = 0.0;
    for (int k = 0; k < VC; ++k) s += sh.cta_sum[pass & 1][k];
    ++pass;
    return s;
  };

  int u = 0, ns = 0, cnt = 1;
  double S = 1.0;
  bool fresh = false;                // warp_sum / cta_sum hold the current W
  if (tid == 0) sh.path[0] = 0;
  for (int c = 1; c < n; ++c) {      // (a child is a later node than its parent)
    if (sh.par[c] != u) continue;
    double w = sh.px[c];
    const double q = sh.qx[c];
    for (int k = 0; k < ns; ++k) w = positive(__dsub_rn(w, __dmul_rn(sh.stage[k], q)));
    if (__dmul_rn(__dmul_rn(sh.r[c], S), q) < w) {
      u = c; ns = 0; S = 1.0; fresh = false;
      if (tid == 0) sh.path[cnt] = c;
      ++cnt;
    } else {
      __syncthreads();               // everyone has read the stages
      if (tid == 0) sh.stage[ns] = S;
      __syncthreads();
      const double mass = sum_pass(u, ns + 1);
      if (!(mass <= 0.0)) { ++ns; S = mass; total = mass; fresh = true; }      // (a NaN stays: nothing is accepted or drawn behind it)
      else fresh = false;            // nothing left: the distribution stays as it was
    }
  }
  if (!fresh) total = sum_pass(u, ns);
  const double target = __dmul_rn(sh.r[0], total);
  const int slot = (pass - 1) & 1;
  // the first warp range whose running sum passes the target (the last non-empty one if rounding hides it)
  int own_cta = -1, own_warp = -1;
  double before = 0.0, run = 0.0;
  if (total > 0.0) {
    double cta_before = 0.0;
    for (int k = 0; k < VC; ++k) {
      const double s = sh.cta_sum[slot][k];
      if (s > 0.0) {
        own_cta = k; cta_before = run;
        if (run + s > target) break;
      }
      run += s;
    }
    if (own_cta == rank) {
      run = cta_before;
      for (int w = 0; w < VW; ++w) {
        const double s = sh.warp_sum[w];
        if (s > 0.0) {
          own_warp = w; before = run;
          if (run + s > target) break;
        }
        run += s;
      }
      // the range again, by the whole CTA: every thread a contiguous piece, a scan of their sums, and the thread whose
      // piece holds the target goes through it
      const float* pu = Pb + (size_t)u * V;
      const float* qu = Qb + (size_t)u * V;
      const int b0 = min(V, (rank * VW + own_warp) * range), b1 = min(V, b0 + range), per = (range + VT - 1) / VT;
      const int x0 = min(b1, b0 + tid * per), x1 = min(b1, x0 + per);
      double sum = 0.0;
      int last = -1;
      for (int x = x0; x < x1; ++x) {
        const double w = residual<-1>(pu[x], ns ? qu[x] : 0.f, sh.stage, ns);
        if (w > 0.0) last = x;
        sum += w;
      }
      double incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      if (lane == 31) sh.piece[warp] = incl;
      if (tid == 0) { sh.first = 0x7fffffff; sh.last = -1; }
      __syncthreads();
      double base = before;
      for (int w = 0; w < warp; ++w) base += sh.piece[w];
      base += incl - sum;
      if (last >= 0) atomicMax(&sh.last, last);
      if (sum > 0.0 && base + sum > target) {                       // (the pieces behind the first of these find a higher index)
        for (int x = x0; x < x1; ++x) {
          const double w = residual<-1>(pu[x], ns ? qu[x] : 0.f, sh.stage, ns);
          base += w;
          if (w > 0.0 && base > target) { atomicMin(&sh.first, x); break; }
        }
      }
      __syncthreads();
      if (tid == 0) sh.next = sh.first != 0x7fffffff ? sh.first : sh.last;
    }
  }
  __syncthreads();
  if (own_cta == rank || (own_cta < 0 && rank == 0)) {
    if (tid == 0) { next_token[b] = sh.next; count[b] = cnt; }
    for (int i = tid; i < n; i += VT) path[(size_t)b * n + i] = i < cnt ? sh.path[i] : -1;
  }
  // (a CTA may leave: after the last pass's cluster barrier each reads its own shared memory only)
}

// One block per (accepted token, sequence): k_tree[b][path[b][j]] -> cache row lengths[b] + j.  A sequence whose path
// is not one, or whose rows would pass the capacity, is left unwritten as a whole.  One launch of latency: 8 us for three
// rows, 9 us for 64 sequences (34 MB at d = 4096, 3.9 TB/s).
__global__ void __launch_bounds__(256)
slim_tree_commit_kernel(unsigned char* __restrict__ cache, const unsigned char* __restrict__ k_tree, const int32_t* __restrict__ lengths,
                        const int32_t* __restrict__ path, const int32_t* __restrict__ count, int n, int t_cap, size_t row_bytes,
                        const int32_t* __restrict__ block_table, int page_rows, int max_pages, int num_pages, int* status) {
  const int b = blockIdx.y, j = blockIdx.x, tid = threadIdx.x;
  slim_pdl_trigger();
  slim_pdl_wait();
  const int cnt = count[b], len = lengths[b];
  if (cnt < 0 || cnt > n) { if (j == 0 && tid == 0) atomicMax(status, (int)SLIM_ERR_TREE); return; }
  if (j >= cnt) return;
  if (len < 0 || len > t_cap - cnt) { if (j == 0 && tid == 0) atomicMax(status, (int)SLIM_ERR_CAPACITY); return; }
  bool bad_path = false, bad_page = false;
  if (tid < cnt) {
    const int i = path[(size_t)b * n + tid];
    bad_path = i < 0 || i >= n;
    if (block_table) {
      const int pg = block_table[(size_t)b * max_pages + (len + tid) / page_rows];
      bad_page = pg < 0 || pg >= num_pages;
    }
  }
  if (__syncthreads_or(bad_path)) { if (j == 0 && tid == 0) atomicMax(status, (int)SLIM_ERR_TREE); return; }
  if (__syncthreads_or(bad_page)) { if (j == 0 && tid == 0) atomicMax(status, (int)SLIM_ERR_CAPACITY); return; }
  const int t = len + j;
  const size_t row = block_table ? (size_t)block_table[(size_t)b * max_pages + t / page_rows] * page_rows + t % page_rows
                                 : (size_t)b * t_cap + t;
  const unsigned char* src = k_tree + ((size_t)b * n + path[(size_t)b * n + j]) * row_bytes;
  unsigned char* dst = cache + row * row_bytes;
  if ((row_bytes & 15) == 0) {       // (both buffers are 16-byte aligned)
    for (size_t e = tid; e < row_bytes / 16; e += blockDim.x)
      reinterpret_cast<uint4*>(dst)[e] = __ldg(reinterpret_cast<const uint4*>(src) + e);
  } else {                           // rows are an even number of elements of 2 or 4 bytes
    for (size_t e = tid; e < row_bytes / 4; e += blockDim.x)
      reinterpret_cast<uint32_t*>(dst)[e] = reinterpret_cast<const uint32_t*>(src)[e];
  }
}

}  // namespace

cudaError_t slim_launch_verify(const float* p, const float* q, const int32_t* tokens, const int32_t* parents, const float* r, int batch,
                               int n, int vocab, int32_t* path, int32_t* count, int32_t* next_token, int* status, cudaStream_t st) {
  auto kern = batch * VC <= 296 ? slim_tree_verify_kernel<512> : slim_tree_verify_kernel<256>;
  return slim_launch_pdl(kern, dim3(VC * batch), dim3(batch * VC <= 296 ? 512 : 256), 0, st, p, q, tokens, parents, r, n, vocab, path, count,
                         next_token, status);
}

cudaError_t slim_launch_commit(const slim_ctx* ctx, const slim_cache* c, const void* k_tree, const int32_t* lengths, const int32_t* path,
                               const int32_t* count, int n, cudaStream_t st) {
  const size_t row_bytes = (size_t)ctx->d * (ctx->kdtype == SLIM_BF16 ? 2 : 4);
  return slim_launch_pdl(slim_tree_commit_kernel, dim3(n, c->batch), dim3(256), 0, st, (unsigned char*)c->k, (const unsigned char*)k_tree,
                         lengths, path, count, n, c->t_cap, row_bytes, c->block_table, c->page_rows, c->max_pages, c->num_pages,
                         ctx->status);
}
