// A long cache kept inside a budget: attention weights accumulated per cache row (slim_accumulate_weights) and
// eviction of the rows with the least of it (slim_evict).
#include "slim_internal.h"
#include "slim_ptx.cuh"
#include "slim_sched.cuh"

using namespace slim_ptx;

namespace {

__device__ __forceinline__ f32x2 sub2(f32x2 a, f32x2 b) { f32x2 d; asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }

// ---------------------------------------------------------------- accumulated weights
// Softmax arguments of one query per sequence, all heads, and the running (maximum, sum) of every head over a worker's
// rows.  The context is cut into tiles of 16 rows dealt out evenly over the ragged batch (slim_sched.cuh).  A thread owns
// a unit: VEC rotation pairs (16 bytes of the low half of a head, 16 of the high half) of one head, so that a warp reads
// whole contiguous rows.  The rotation is moved onto the query, q^ . R_t k = (R_(pos - t) q) . k, which is seeded from the
// tables at a tile's first row (float32 products of entries made in float64) and turned by one position a row with a
// packed complex product: at most 16 steps, so that its error stays below 2^-20.  Where a row has fewer units than a block
// has threads, groups of threads take different rows of the tile.  Everything is float32: sums of a unit's products in a
// register, of a head's units in order through shared memory.
// Bound by HBM: every key byte is read once, about 50 instructions a thread and row against the 340 clocks that an
// 8 KB row costs an SM at the copy rate.
constexpr int WT = 256;

template <typename KT> struct KeyVec;
template <> struct KeyVec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, f32x2 (&f)[2]) {
    f[0] = pack2(__uint_as_float(v.x), __uint_as_float(v.y)); f[1] = pack2(__uint_as_float(v.z), __uint_as_float(v.w));
  }
};
template <> struct KeyVec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, f32x2 (&f)[4]) {
    f[0] = unpack2(v.x); f[1] = unpack2(v.y); f[2] = unpack2(v.z); f[3] = unpack2(v.w);
  }
};

template <typename KT, bool ROPE>
__global__ void __launch_bounds__(WT, 2)
slim_weights_scores_kernel(const SlimDecodeParams p, float* __restrict__ scores, float2* __restrict__ part) {
  constexpr int VEC = KeyVec<KT>::N, NP = VEC / 2;
  extern __shared__ __align__(16) float s_part[];                  // [2][16][units + 4]
  const int d = p.d, H = p.H, dk = p.d_k, half = p.half, tid = threadIdx.x;
  const int units = d / (2 * VEC), per_head = half / VEC, ld = units + 4;
  int* s_prefix = reinterpret_cast<int*>(s_part + 2 * SLIM_TT * ld);
  slim_pdl_trigger();
  slim_pdl_wait();
  const SlimSched sc = slim_sched_build(p.lengths, p.batch, p.t_cap, p.workers, 1, s_prefix, p.status, 0);
  const int w = blockIdx.x;
  if (sc.total_tiles == 0 || w >= sc.workers_eff) return;
  const int g_begin = slim_worker_start(sc, w), g_end = slim_worker_start(sc, w + 1);
  int groups = 1;                                                  // row groups of a tile
  while (groups < SLIM_TT && 2 * groups * units <= WT) groups *= 2;
  const int rpg = SLIM_TT / groups, stride = groups > 1 ? units : WT;
  const int rg = groups > 1 ? min(tid / units, groups) : 0, u0 = groups > 1 ? tid % units : tid;      // rg == groups: no unit
  const KT* Kc = reinterpret_cast<const KT*>(p.k);

  int buf = 0;
  for (int g = g_begin; g < g_end;) {
    const int b = slim_seq_of_tile(s_prefix, p.batch, g);
    const int seg_end = min(g_end, s_prefix[b + 1]);
    const int len = min(max(p.lengths[b], 0), p.t_cap), pos = len - 1;
    const KT* q = reinterpret_cast<const KT*>(p.q) + (size_t)b * d;
    float run_m[4], run_l[4];                                      // of (head, row of the tile) number tid + 256 x
#pragma unroll
    for (int x = 0; x < 4; ++x) { run_m[x] = -INFINITY; run_l[x] = 0.f; }
    for (; g < seg_end; ++g, buf ^= 1) {
      const int t0 = (g - s_prefix[b]) * SLIM_TT;
      const KT* rows = Kc + (size_t)slim_cache_row(p, b, t0) * d;
      const int last = min(SLIM_TT - 1, len - 1 - t0);             // rows behind it are read as it, and not used
      float* out = s_part + buf * SLIM_TT * ld;
      for (int u = u0; u < units && rg < groups; u += stride) {
        const int h = u / per_head, j0 = (u - h * per_head) * VEC, at = h * dk + j0, r0 = rg * rpg;
        // the query, scaled and turned to the distance of this thread's first row
        f32x2 z1[NP], z2[NP], co[NP], si[NP];
        KeyVec<KT>::unpack(__ldg(reinterpret_cast<const uint4*>(q + at)), z1);
        KeyVec<KT>::unpack(__ldg(reinterpret_cast<const uint4*>(q + at + half)), z2);
        const int dist = max(pos - t0 - r0, 0);
#pragma unroll
        for (int x = 0; x < NP; ++x) {
          const f32x2 sc2 = pack2(p.qscale, p.qscale);
          z1[x] = mul2(z1[x], sc2); z2[x] = mul2(z2[x], sc2);
          if (ROPE) {
            const float4 cb = __ldg(reinterpret_cast<const float4*>(p.rope_base + (size_t)(dist / SLIM_TT) * half + j0) + x);
            const float4 cf = __ldg(reinterpret_cast<const float4*>(p.rope_off + (dist % SLIM_TT) * half + j0) + x);
            const float4 st = __ldg(reinterpret_cast<const float4*>(p.rope_off + half + j0) + x);      // one position
            const f32x2 c = pack2(cb.x * cf.x - cb.y * cf.y, cb.z * cf.z - cb.w * cf.w), s = pack2(cb.y * cf.x + cb.x * cf.y, cb.w * cf.z + cb.z * cf.w);
            const f32x2 a = fma2(z2[x], s, mul2(z1[x], c));
            z2[x] = sub2(mul2(z2[x], c), mul2(z1[x], s));
            z1[x] = a;
            co[x] = pack2(st.x, st.z); si[x] = pack2(st.y, st.w);
          }
        }
        for (int r = 0; r < rpg; r += 4) {
          uint4 k1[4], k2[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const KT* row = rows + (size_t)min(r0 + min(r + x, rpg - 1), last) * d + at;
            k1[x] = __ldg(reinterpret_cast<const uint4*>(row));
            k2[x] = __ldg(reinterpret_cast<const uint4*>(row + half));
          }
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            f32x2 f1[NP], f2[NP];
            KeyVec<KT>::unpack(k1[x], f1);
            KeyVec<KT>::unpack(k2[x], f2);
            f32x2 a = mul2(f1[0], z1[0]), c = mul2(f2[0], z2[0]);
#pragma unroll
            for (int y = 1; y < NP; ++y) { a = fma2(f1[y], z1[y], a); c = fma2(f2[y], z2[y], c); }
            if (r + x < rpg) out[(r0 + r + x) * ld + u] = sum2(add2(a, c));
            if (ROPE)
#pragma unroll
              for (int y = 0; y < NP; ++y) {                       // one position nearer: times e^{i theta}
                const f32x2 n1 = sub2(mul2(z1[y], co[y]), mul2(z2[y], si[y]));
                z2[y] = fma2(z1[y], si[y], mul2(z2[y], co[y]));
                z1[y] = n1;
              }
          }
        }
      }
      __syncthreads();                                             // (two buffers: the next tile may be written while this one is read)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int e = tid + WT * x, h = e / SLIM_TT, r = e % SLIM_TT;
        if (h >= H || t0 + r >= len) continue;
        const float* a = out + r * ld + h * per_head;
        float s = 0.f;
        for (int y = 0; y < per_head; ++y) s += a[y];
        scores[((size_t)b * H + h) * p.t_cap + t0 + r] = s;
        const float top = fmaxf(run_m[x], s);
        if (top != -INFINITY) run_l[x] = run_l[x] * exp2f(run_m[x] - top) + exp2f(s - top);
        run_m[x] = top;
      }
    }
    // the unit's (maximum, sum) of every head: over the 16 threads that share it
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float m = run_m[x], l = run_l[x];
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) {
        const float m1 = __shfl_xor_sync(0xffffffffu, m, o), l1 = __shfl_xor_sync(0xffffffffu, l, o), top = fmaxf(m, m1);
        if (top != -INFINITY) l = l * exp2f(m - top) + l1 * exp2f(m1 - top);
        m = top;
      }
      const int e = tid + WT * x, h = e / SLIM_TT;
      if (e % SLIM_TT == 0 && h < H) part[(size_t)(w + b) * H + h] = make_float2(m, l);
    }
  }
}

// Reference exponent and 1 / denominator of every (sequence, head) from its units' parts: a warp each.
__global__ void __launch_bounds__(256) slim_weights_join_kernel(const SlimDecodeParams p, const float2* __restrict__ part, float* __restrict__ m_out,
                                                                float* __restrict__ inv_out) {
  extern __shared__ int s_prefix2[];
  slim_pdl_trigger();
  slim_pdl_wait();
  const SlimSched sc = slim_sched_build(p.lengths, p.batch, p.t_cap, p.workers, 1, s_prefix2, p.status, 0);
  const int b = blockIdx.y, h = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (h >= p.H) return;
  float m = -INFINITY, l = 0.f;
  if (s_prefix2[b + 1] > s_prefix2[b]) {
    const int w0 = slim_worker_of_tile(sc, s_prefix2[b]), w1 = slim_worker_of_tile(sc, s_prefix2[b + 1] - 1);
    for (int w = w0 + lane; w <= w1; w += 32) {
      const float2 v = part[(size_t)(w + b) * p.H + h];
      const float top = fmaxf(m, v.x);
      if (top != -INFINITY) l = l * exp2f(m - top) + v.y * exp2f(v.x - top);
      m = top;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m1 = __shfl_xor_sync(0xffffffffu, m, o), l1 = __shfl_xor_sync(0xffffffffu, l, o), top = fmaxf(m, m1);
    if (top != -INFINITY) l = l * exp2f(m - top) + l1 * exp2f(m1 - top);
    m = top;
  }
  if (lane == 0) {
    m_out[(size_t)b * p.H + h] = m == -INFINITY ? 0.f : m;
    inv_out[(size_t)b * p.H + h] = l != 0.f ? 1.f / l : 0.f;
  }
}

// The same from the softmax arguments [b][h][t_cap] themselves (8-bit caches and shapes whose arguments come from
// slim_scores_kernel).
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

// Workers of the score kernel: two CTAs an SM.
int slim_weights_workers(const slim_ctx* ctx) { return 2 * ctx->num_sms; }

cudaError_t slim_launch_weights(const slim_ctx* ctx, const SlimDecodeParams& p_in, float* scores, float2* part, float* m, float* inv_l,
                                float* acc, cudaStream_t st) {
  SlimDecodeParams p = p_in;
  // whole 16-byte vectors of a head's halves (rows are then 16-byte aligned too); 8-bit codes and other widths take the
  // score kernel of slim_decode's CUDA-core path
  const int vec = p.kdtype == SLIM_BF16 ? 8 : 4;
  const size_t smem = sizeof(float) * 2 * SLIM_TT * (size_t)(p.d / (2 * vec) + 4) + sizeof(int) * (p.batch + 1);
  cudaError_t e;
  if (p.kdtype != SLIM_FP8 && p.half % vec == 0 && smem <= 200 * 1024) {
    p.workers = slim_weights_workers(ctx);
    auto kern = p.kdtype == SLIM_BF16 ? (p.rope ? slim_weights_scores_kernel<__nv_bfloat16, true> : slim_weights_scores_kernel<__nv_bfloat16, false>)
                                      : (p.rope ? slim_weights_scores_kernel<float, true> : slim_weights_scores_kernel<float, false>);
    if (smem > 48 * 1024 && (e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return e;
    e = slim_launch_pdl(kern, dim3(p.workers), dim3(WT), smem, st, p, scores, part);
    if (e == cudaSuccess)
      e = slim_launch_pdl(slim_weights_join_kernel, dim3((p.H + 7) / 8, p.batch), dim3(256), sizeof(int) * (p.batch + 1), st, p,
                          (const float2*)part, m, inv_l);
  } else {
    e = slim_launch_scores(ctx, p, scores, st);
    if (e == cudaSuccess) e = slim_launch_pdl(slim_weights_stat_kernel, dim3(p.H, p.batch), dim3(256), 0, st, p, (const float*)scores, m, inv_l);
  }
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
