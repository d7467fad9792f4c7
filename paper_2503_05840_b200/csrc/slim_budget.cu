// A long cache kept inside a budget: attention weights accumulated per cache row (slim_accumulate_weights) and
// eviction of the rows with the least of it (slim_evict).
#include "slim_internal.h"
#include "slim_sched.cuh"

namespace {

// ---------------------------------------------------------------- accumulated weights
// Reference exponent and denominator of every (sequence, head) from the softmax arguments [b][h][t_cap].
__global__ void __launch_bounds__(256) slim_weights_stat_kernel(const SlimDecodeParams p, const float* __restrict__ scores,
                                                                float* __restrict__ m_out, float* __restrict__ inv_out) {
  __shared__ float s_m[8], s_l[8];
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  slim_pdl_trigger();
  slim_pdl_wait();
  const int len = min(max(p.lengths[b], 0), p.t_cap);
  const float* S = scores + ((size_t)b * p.H + h) * p.t_cap;
  float m = -INFINITY, l = 0.f;
  for (int t = tid; t < len; t += 256) {
    const float s = S[t], top = fmaxf(m, s);
    if (top != -INFINITY) l = l * exp2f(m - top) + exp2f(s - top);
    m = top;
  }
  auto join = [](float& m0, float& l0, float m1, float l1) {
    const float top = fmaxf(m0, m1);
    if (top == -INFINITY) return;
    l0 = l0 * exp2f(m0 - top) + l1 * exp2f(m1 - top);
    m0 = top;
  };
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) join(m, l, __shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, l, o));
  if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 8; ++w) join(m, l, s_m[w], s_l[w]);
    m_out[(size_t)b * p.H + h] = m == -INFINITY ? 0.f : m;
    inv_out[(size_t)b * p.H + h] = l != 0.f ? 1.f / l : 0.f;
  }
}

__global__ void __launch_bounds__(256) slim_weights_add_kernel(const SlimDecodeParams p, const float* __restrict__ scores,
                                                               const float* __restrict__ m_in, const float* __restrict__ inv_in,
                                                               float* __restrict__ acc) {
  const int b = blockIdx.y, t = blockIdx.x * 256 + threadIdx.x;
  slim_pdl_trigger();
  slim_pdl_wait();
  const int len = min(max(p.lengths[b], 0), p.t_cap);
  if (t >= len) return;
  float a = 0.f;
  for (int h = 0; h < p.H; ++h)
    a += exp2f(scores[((size_t)b * p.H + h) * p.t_cap + t] - m_in[(size_t)b * p.H + h]) * inv_in[(size_t)b * p.H + h];
  acc[(size_t)b * p.t_cap + t] += a;
}

// ---------------------------------------------------------------- eviction
// Which rows stay.  One block per sequence: the (budget - recent)-th largest weight of the candidate rows by a radix
// selection on the order-preserving integer form of the floats (four passes of eight bits), then one pass that counts
// per warp and one that writes the kept indices in order: every row above the threshold, and of the rows equal to it
// the first ones.
constexpr int SEL_THREADS = 1024, SEL_WARPS = SEL_THREADS / 32;

__device__ __forceinline__ uint32_t order_key(float f) {
  if (f != f) return 0u;                              // NaN: below every number
  const uint32_t u = __float_as_uint(f + 0.f);        // -0 and 0 are equal
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(SEL_THREADS)
slim_evict_select_kernel(const int32_t* __restrict__ lengths, const float* __restrict__ acc, int t_cap, int budget, int recent,
                         int32_t* __restrict__ kept, int* status) {
  __shared__ unsigned hist[256];
  __shared__ int s_gt[SEL_WARPS], s_eq[SEL_WARPS];
  __shared__ unsigned s_prefix, s_need;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  slim_pdl_trigger();
  slim_pdl_wait();
  int len = lengths[b];
  if (len > t_cap) { len = t_cap; if (tid == 0) atomicMax(status, (int)SLIM_ERR_CAPACITY); }
  if (len < 0) len = 0;
  int32_t* K = kept + (size_t)b * budget;
  if (len <= budget) {
    for (int j = tid; j < budget; j += SEL_THREADS) K[j] = j < len ? j : -1;
    return;
  }
  const int cand = len - recent, need = budget - recent;          // 0 <= need < cand
  const float* A = acc + (size_t)b * t_cap;
  unsigned prefix = 0, left = (unsigned)need;                      // the left-th largest among the keys that share the prefix
  if (need > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += SEL_THREADS) hist[i] = 0;
      __syncthreads();
      for (int t0 = 0; t0 < cand; t0 += SEL_THREADS) {
        const int t = t0 + tid;
        const uint32_t key = t < cand ? order_key(A[t]) : 0u;
        const bool in = t < cand && (shift == 24 || (key >> (shift + 8)) == prefix);
        const unsigned active = __ballot_sync(0xffffffffu, in);
        if (in) {                                                  // one atomic a distinct digit and warp
          const unsigned digit = (key >> shift) & 255u, same = __match_any_sync(active, digit);
          if (lane == __ffs(same) - 1) atomicAdd(&hist[digit], __popc(same));
        }
      }
      __syncthreads();
      if (warp == 0) {                                             // lane k: digits 255 - 8 k .. 248 - 8 k, from the top
        unsigned c[8], sum = 0;
        for (int i = 0; i < 8; ++i) { c[i] = hist[255 - 8 * lane - i]; sum += c[i]; }
        unsigned incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned y = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += y;
        }
        unsigned above = incl - sum;
        if (above < left && left <= incl)
          for (int i = 0; i < 8; ++i) {
            if (left <= above + c[i]) { s_prefix = (prefix << 8) | (255 - 8 * lane - i); s_need = left - above; break; }
            above += c[i];
          }
      }
      __syncthreads();
      prefix = s_prefix; left = s_need;
    }
  }
  // rows with key > prefix stay, and the first `left` of those equal to it (none of either when need = 0)
  const uint32_t thr = need > 0 ? prefix : 0xffffffffu;
  const int seg = ((len + SEL_WARPS - 1) / SEL_WARPS + 31) & ~31, lo = min(len, warp * seg), hi = min(len, lo + seg);
  int gt = 0, eq = 0;
  for (int t0 = lo; t0 < hi; t0 += 32) {
    const int t = t0 + lane;
    const uint32_t key = t < hi && t < cand ? order_key(A[t]) : 0u;
    gt += __popc(__ballot_sync(0xffffffffu, t < hi && (t >= cand || (need > 0 && key > thr))));
    eq += __popc(__ballot_sync(0xffffffffu, t < hi && t < cand && need > 0 && key == thr));
  }
  if (lane == 0) { s_gt[warp] = gt; s_eq[warp] = eq; }
  __syncthreads();
  int eq_before = 0, out = 0;
  for (int w = 0; w < warp; ++w) {
    out += s_gt[w] + min(s_eq[w], max((int)left - eq_before, 0));
    eq_before += s_eq[w];
  }
  for (int t0 = lo; t0 < hi; t0 += 32) {
    const int t = t0 + lane;
    const uint32_t key = t < hi && t < cand ? order_key(A[t]) : 0u;
    const bool is_eq = t < hi && t < cand && need > 0 && key == thr;
    const unsigned eqs = __ballot_sync(0xffffffffu, is_eq), below = (1u << lane) - 1u;
    const bool keep = t < hi && (t >= cand || (need > 0 && key > thr) || (is_eq && eq_before + __popc(eqs & below) < (int)left));
    const unsigned ks = __ballot_sync(0xffffffffu, keep);
    if (keep) {
      const int j = out + __popc(ks & below);
      if (j < budget) K[j] = t;
    }
    out += __popc(ks);
    eq_before += __popc(eqs);
  }
}

// The kept rows move to rows 0 .. budget - 1, in place.  Row j comes from row kept[j] >= j, so a block that owns a
// column slice and goes through the rows in order may write a chunk as soon as all sources up to that chunk have been
// read: sources of later chunks lie behind everything it overwrites.  The last block of a sequence moves the weights
// and clears those of the rows that became free.
constexpr int MV_THREADS = 256, MV_COLS = 8, MV_ROWS = MV_THREADS / MV_COLS, MV_UNROLL = 4;

__device__ __forceinline__ long long storage_row(const int32_t* table, int page_rows, int max_pages, int num_pages, int t_cap, int b, int t,
                                                 int* status) {
  if (!table) return (long long)b * t_cap + t;
  const int pg = table[(size_t)b * max_pages + t / page_rows];
  if (pg < 0 || pg >= num_pages) { atomicMax(status, (int)SLIM_ERR_CAPACITY); return -1; }
  return (long long)pg * page_rows + t % page_rows;
}

template <typename VT>
__global__ void __launch_bounds__(MV_THREADS)
slim_evict_move_kernel(unsigned char* __restrict__ base, int vecs, const int32_t* __restrict__ lengths, int t_cap, int budget,
                       const int32_t* __restrict__ kept, const int32_t* __restrict__ table, int page_rows, int max_pages, int num_pages,
                       float* __restrict__ acc, int* status) {
  const int b = blockIdx.y, tid = threadIdx.x;
  slim_pdl_trigger();
  slim_pdl_wait();
  const int len = min(max(lengths[b], 0), t_cap);
  if (len <= budget) return;
  const int32_t* K = kept + (size_t)b * budget;
  if (acc && blockIdx.x == gridDim.x - 1) {
    float* A = acc + (size_t)b * t_cap;
    for (int j0 = 0; j0 < budget; j0 += MV_THREADS) {
      const int j = j0 + tid;
      const float v = j < budget ? A[K[j]] : 0.f;
      __syncthreads();
      if (j < budget) A[j] = v;
      __syncthreads();
    }
    for (int t = budget + tid; t < len; t += MV_THREADS) A[t] = 0.f;
    return;
  }
  const int col = blockIdx.x * MV_COLS + tid % MV_COLS, r = tid / MV_COLS;
  VT* K0 = reinterpret_cast<VT*>(base);
  for (int j0 = 0; j0 < budget; j0 += MV_ROWS * MV_UNROLL) {
    VT v[MV_UNROLL];
    long long dst[MV_UNROLL];
#pragma unroll
    for (int x = 0; x < MV_UNROLL; ++x) {
      const int j = j0 + x * MV_ROWS + r;
      dst[x] = -1;
      if (j < budget && col < vecs) {
        const int t = K[j];
        if (t != j) {
          const long long from = storage_row(table, page_rows, max_pages, num_pages, t_cap, b, t, status);
          const long long to = storage_row(table, page_rows, max_pages, num_pages, t_cap, b, j, status);
          if (from >= 0 && to >= 0) { dst[x] = to * vecs + col; v[x] = K0[from * vecs + col]; }
        }
      }
    }
    __syncthreads();                 // all sources up to here have been read
#pragma unroll
    for (int x = 0; x < MV_UNROLL; ++x)
      if (dst[x] >= 0) K0[dst[x]] = v[x];
  }
}

template <typename VT>
cudaError_t launch_move(const slim_ctx* ctx, const slim_cache* c, void* base, size_t row_bytes, const int32_t* lengths, int budget,
                        const int32_t* kept, float* acc, cudaStream_t st) {
  const int vecs = (int)(row_bytes / sizeof(VT));
  return slim_launch_pdl(slim_evict_move_kernel<VT>, dim3((vecs + MV_COLS - 1) / MV_COLS + (acc ? 1 : 0), c->batch), dim3(MV_THREADS), 0, st,
                         (unsigned char*)base, vecs, lengths, c->t_cap, budget, kept, c->block_table, c->page_rows, c->max_pages,
                         c->num_pages, acc, ctx->status);
}

}  // namespace

cudaError_t slim_launch_weights(const slim_ctx* ctx, const SlimDecodeParams& p, float* scores, float* m, float* inv_l, float* acc,
                                cudaStream_t st) {
  cudaError_t e = slim_launch_scores(ctx, p, scores, st);
  if (e == cudaSuccess) e = slim_launch_pdl(slim_weights_stat_kernel, dim3(p.H, p.batch), dim3(256), 0, st, p, (const float*)scores, m, inv_l);
  if (e == cudaSuccess)
    e = slim_launch_pdl(slim_weights_add_kernel, dim3((p.t_cap + 255) / 256, p.batch), dim3(256), 0, st, p, (const float*)scores,
                        (const float*)m, (const float*)inv_l, acc);
  return e;
}

cudaError_t slim_launch_evict(const slim_ctx* ctx, const slim_cache* c, const int32_t* lengths, float* acc, int budget, int recent,
                              int32_t* kept, cudaStream_t st) {
  cudaError_t e = slim_launch_pdl(slim_evict_select_kernel, dim3(c->batch), dim3(SEL_THREADS), 0, st, lengths, (const float*)acc, c->t_cap,
                                  budget, recent, kept, ctx->status);
  if (e != cudaSuccess) return e;
  if (ctx->kdtype == SLIM_FP8) {     // codes, then the exponents of the same rows
    const size_t row = (size_t)ctx->d;
    e = (row & 15) == 0 ? launch_move<uint4>(ctx, c, c->k, row, lengths, budget, kept, acc, st)
                        : launch_move<unsigned short>(ctx, c, c->k, row, lengths, budget, kept, acc, st);
    if (e == cudaSuccess) e = launch_move<unsigned char>(ctx, c, c->k_exp, ctx->H, lengths, budget, kept, nullptr, st);
    return e;
  }
  const size_t row = (size_t)ctx->d * (ctx->kdtype == SLIM_BF16 ? 2 : 4);
  if ((row & 15) == 0) return launch_move<uint4>(ctx, c, c->k, row, lengths, budget, kept, acc, st);
  return launch_move<unsigned short>(ctx, c, c->k, row, lengths, budget, kept, acc, st);
}
