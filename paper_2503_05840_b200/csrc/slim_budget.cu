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
// rows.  The context is cut into tiles of 16 rows dealt out evenly over the ragged batch (slim_sched.cuh), one CTA per
// SM; a producer warp brings whole rows (a tile is contiguous, in a page too) into a ring in shared memory with bulk
// copies.  LPH neighbouring lanes share a head, each with VEC rotation pairs (16 bytes of its low half, 16 of its high
// half); enough warps for all heads make a row group, and the groups take different rows of a tile.  A warp keeps
// (maximum, sum) of its heads and rows to itself, so nothing waits but for the ring.
// The rotation is moved onto the query, q^ . R_t k = (R_(pos - t) q) . k, which is seeded from the tables at the group's
// first row of a tile (float32 products of entries made in float64) and turned by one position a row with a packed
// complex product: at most 16 steps, so that its error stays below 2^-20.  Everything is float32.
// A maximum passes over NaN, so the sums carry it: one NaN makes its whole softmax NaN, wherever it stands.
// Bound by HBM: every key byte is read once.  16 ragged sequences, 196 k rows of 8 KB: 289 us, 5.6 TB/s, 0.86 of a copy's rate
// (305 us with the two kernels behind it, 20 us for 1500 float32 rows of 1.5 KB, three launches).  A rotation seeded per row,
// sums through shared memory, and four rows a round instead of two were slower.
constexpr int WC = 512, WT = WC + 32;                              // consumers; and the producer warp

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

struct WeightsRing { int rows, stages, groups, warps; };           // rows of a stage (a power of two up to 16); row groups and warps of one

template <typename KT, bool ROPE, int LPH>
__global__ void __launch_bounds__(WT, 1)
slim_weights_scores_kernel(const SlimDecodeParams p, float* __restrict__ scores, float2* __restrict__ part, const WeightsRing ring) {
  constexpr int VEC = KeyVec<KT>::N, NP = VEC / 2, HPW = 32 / LPH;
  extern __shared__ __align__(128) unsigned char sm[];
  const int d = p.d, H = p.H, dk = p.d_k, half = p.half, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t row_bytes = (uint32_t)(d * sizeof(KT)), stage_bytes = row_bytes * ring.rows;
  unsigned char* keys = sm;                                        // [stages][rows][row_bytes]
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + (size_t)ring.stages * stage_bytes);  // [stages] full, [stages] empty
  volatile int* s_abort = reinterpret_cast<volatile int*>(bars + 2 * ring.stages);
  int* s_prefix = const_cast<int*>(s_abort) + 2;
  const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8u * ring.stages;
  const int used = ring.groups * ring.warps;                       // consumer warps that have work
  if (tid == 0) {
    for (int i = 0; i < ring.stages; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, used); }
    *s_abort = 0;
    fence_mbar_init();
  }
  slim_pdl_trigger();
  slim_pdl_wait();
  const SlimSched sc = slim_sched_build(p.lengths, p.batch, p.t_cap, p.workers, 1, s_prefix, p.status, 0);      // (has block barriers)
  const int w = blockIdx.x;
  if (sc.total_tiles == 0 || w >= sc.workers_eff) return;
  const int g_begin = slim_worker_start(sc, w), g_end = slim_worker_start(sc, w + 1);
  const int per_tile = SLIM_TT / ring.rows;                        // stages of a tile

  if (tid >= WC) {
    // ---- producer ----
    if (tid == WC) {
      fence_proxy_async_global();                                  // (the keys may be an earlier kernel's ordinary stores)
      const unsigned char* Kc = reinterpret_cast<const unsigned char*>(p.k);
      int st = 0;
      uint32_t ph = 1;                                             // parity of a stage's "empty" that means free
      bool ok = true;
      for (int g = g_begin; g < g_end && ok; ++g) {
        const int b = slim_seq_of_tile(s_prefix, p.batch, g), t0 = (g - s_prefix[b]) * SLIM_TT;
        const int rows = min(SLIM_TT, min(p.lengths[b], p.t_cap) - t0);
        const unsigned char* src = Kc + (size_t)slim_cache_row(p, b, t0) * row_bytes;
        for (int x = 0; x < per_tile; ++x) {                       // (rows behind the last one are not fetched: their sums are not used)
          const int n = min(ring.rows, rows - x * ring.rows);
          ok = mbar_wait<false>(bar_empty + 8 * st, ph, s_abort, p.status);
          if (!ok) break;
          if (n <= 0) mbar_arrive(bar_full + 8 * st);
          else {
            mbar_arrive_expect_tx(bar_full + 8 * st, (uint32_t)n * row_bytes);
            bulk_load(smem_u32(keys) + (uint32_t)st * stage_bytes, src + (size_t)x * stage_bytes, (uint32_t)n * row_bytes, bar_full + 8 * st);
          }
          if (++st == ring.stages) { st = 0; ph ^= 1; }
        }
      }
      // (the consumers wait for every stage; after a time-out what was issued has landed long since)
    }
    return;
  }
  if (warp >= used) return;
  const int rpg = SLIM_TT / ring.groups, rg = warp / ring.warps, r0 = rg * rpg;
  const int li = lane % LPH, h = (warp - rg * ring.warps) * HPW + lane / LPH;
  const bool mine = h < H && li * VEC < half;                      // (lanes without pairs add zero)
  const int j0 = mine ? li * VEC : 0, at = (mine ? h : 0) * dk + j0;
  f32x2 co[NP], si[NP];                                            // one position
  if (ROPE)
#pragma unroll
    for (int x = 0; x < NP; ++x) {
      const float4 st = __ldg(reinterpret_cast<const float4*>(p.rope_off + half + j0) + x);
      co[x] = pack2(st.x, st.z); si[x] = pack2(st.y, st.w);
    }
  int st = 0;
  uint32_t ph = 0;                                                 // stage and parity of "full"
  for (int g = g_begin; g < g_end;) {
    const int b = slim_seq_of_tile(s_prefix, p.batch, g);
    const int seg_end = min(g_end, s_prefix[b + 1]);
    const int len = min(max(p.lengths[b], 0), p.t_cap), pos = len - 1;
    f32x2 q1[NP], q2[NP];                                          // the query, scaled; zero in lanes without pairs
    {
      const KT* q = reinterpret_cast<const KT*>(p.q) + (size_t)b * d + at;
      KeyVec<KT>::unpack(__ldg(reinterpret_cast<const uint4*>(q)), q1);
      KeyVec<KT>::unpack(__ldg(reinterpret_cast<const uint4*>(q + half)), q2);
      const float f = mine ? p.qscale : 0.f;
#pragma unroll
      for (int x = 0; x < NP; ++x) {
        q1[x] = mine ? mul2(q1[x], pack2(f, f)) : pack2(0.f, 0.f);
        q2[x] = mine ? mul2(q2[x], pack2(f, f)) : pack2(0.f, 0.f);
      }
    }
    float* out = scores + ((size_t)b * H + (h < H ? h : 0)) * p.t_cap;
    float run_m = -INFINITY, run_l = 0.f;
    for (; g < seg_end; ++g) {
      const int t0 = (g - s_prefix[b]) * SLIM_TT;
      // turned to the distance of this group's first row
      f32x2 z1[NP], z2[NP];
      const int dist = max(pos - t0 - r0, 0);
#pragma unroll
      for (int x = 0; x < NP; ++x) {
        z1[x] = q1[x]; z2[x] = q2[x];
        if (ROPE) {
          const float4 cb = __ldg(reinterpret_cast<const float4*>(p.rope_base + (size_t)(dist / SLIM_TT) * half + j0) + x);
          const float4 cf = __ldg(reinterpret_cast<const float4*>(p.rope_off + (dist % SLIM_TT) * half + j0) + x);
          const f32x2 fx = pack2(cf.x, cf.z), fy = pack2(cf.y, cf.w), bx = pack2(cb.x, cb.z), by = pack2(cb.y, cb.w);
          const f32x2 cs = sub2(mul2(bx, fx), mul2(by, fy)), sn = fma2(by, fx, mul2(bx, fy));
          z1[x] = fma2(q2[x], sn, mul2(q1[x], cs));
          z2[x] = sub2(mul2(q2[x], cs), mul2(q1[x], sn));
        }
      }
      float keep = -INFINITY;                                      // this lane's row of the last LPH ones
      for (int y = 0; y < per_tile; ++y) {
        const int a0 = max(r0, y * ring.rows), a1 = min(r0 + rpg, (y + 1) * ring.rows);
        // (also for stages of other groups' rows: a warp must not arrive twice on a barrier before the others have once.
        // Gave up: reported, and the loop runs on)
        mbar_wait<false>(bar_full + 8 * st, ph, s_abort, p.status);
        if (a0 < a1) {
          const unsigned char* row = keys + (size_t)st * stage_bytes + (size_t)(a0 - y * ring.rows) * row_bytes + (size_t)at * sizeof(KT);
          // this lane's product with a row, and the query turned one position nearer (times e^{i theta})
          auto row_sum = [&]() {
            f32x2 f1[NP], f2[NP];
            KeyVec<KT>::unpack(*reinterpret_cast<const uint4*>(row), f1);
            KeyVec<KT>::unpack(*reinterpret_cast<const uint4*>(row + half * sizeof(KT)), f2);
            row += row_bytes;
            f32x2 a = mul2(f1[0], z1[0]), e = mul2(f2[0], z2[0]);
#pragma unroll
            for (int x = 1; x < NP; ++x) { a = fma2(f1[x], z1[x], a); e = fma2(f2[x], z2[x], e); }
            const float v = sum2(add2(a, e));
            if (ROPE)
#pragma unroll
              for (int x = 0; x < NP; ++x) {
                const f32x2 n1 = sub2(mul2(z1[x], co[x]), mul2(z2[x], si[x]));
                z2[x] = fma2(z1[x], si[x], mul2(z2[x], co[x]));
                z1[x] = n1;
              }
            return mine ? v : 0.f;                                 // (a key element times zero could be NaN)
          };
          // rows r - r % LPH + li, up to r, lie in the lanes that keep them
          auto take = [&](int r) {
            const int t = t0 + r - r % LPH + li;
            if (li <= r % LPH && li >= r0 % LPH && t < len && h < H) {
              out[t] = keep;
              const float top = fmaxf(run_m, keep);
              if (top != -INFINITY) run_l = run_l * ex2_approx(run_m - top) + ex2_approx(keep - top);
              else if (keep != keep) run_l = keep;
              run_m = top;
            }
          };
          if (((a0 | a1) & 3) == 0) {
            // four rows at a time: the sums over the lanes of a head turn the rows around, lane li ends with row li % 4
            for (int r = a0; r < a1; r += 4) {
              const float v0 = row_sum(), v1 = row_sum(), v2 = row_sum(), v3 = row_sum();
              const bool b0 = li & 1, b1 = li & 2;
              const float x0 = (b0 ? v1 : v0) + __shfl_xor_sync(0xffffffffu, b0 ? v0 : v1, 1);
              const float x1 = (b0 ? v3 : v2) + __shfl_xor_sync(0xffffffffu, b0 ? v2 : v3, 1);
              float y4 = (b1 ? x1 : x0) + __shfl_xor_sync(0xffffffffu, b1 ? x0 : x1, 2);
#pragma unroll
              for (int o = 4; o < LPH; o <<= 1) y4 += __shfl_xor_sync(0xffffffffu, y4, o);
              if (li / 4 == r / 4 % (LPH / 4)) keep = y4;
              if ((r + 4) % LPH == 0 || r + 4 == r0 + rpg) take(r + 3);
            }
          } else {
            for (int r = a0; r < a1; ++r) {
              float v = row_sum();
#pragma unroll
              for (int o = 1; o < LPH; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
              if (r % LPH == li) keep = v;
              if ((r + 1) % LPH == 0 || r + 1 == r0 + rpg) take(r);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_empty + 8 * st);
        if (++st == ring.stages) { st = 0; ph ^= 1; }
      }
    }
    // (maximum, sum) of the head over this group's rows
#pragma unroll
    for (int o = 1; o < LPH; o <<= 1) {
      const float m1 = __shfl_xor_sync(0xffffffffu, run_m, o), l1 = __shfl_xor_sync(0xffffffffu, run_l, o), top = fmaxf(run_m, m1);
      run_l = top != -INFINITY ? run_l * ex2_approx(run_m - top) + l1 * ex2_approx(m1 - top) : run_l + l1;
      run_m = top;
    }
    if (li == 0 && h < H) part[((size_t)(w + b) * ring.groups + rg) * H + h] = make_float2(run_m, run_l);
  }
}

// 1 / denominator; of an empty sequence nobody reads it, so what is no positive number comes of arguments that are NaN or infinite.
__device__ __forceinline__ float inverse_sum(float l) { return l > 0.f && l < INFINITY ? 1.f / l : NAN; }

// Reference exponent and 1 / denominator of every (sequence, head) from its units' parts: a warp each.
__global__ void __launch_bounds__(256) slim_weights_join_kernel(const SlimDecodeParams p, const float2* __restrict__ part, int groups,
                                                                float* __restrict__ m_out, float* __restrict__ inv_out) {
  extern __shared__ int s_prefix2[];
  slim_pdl_trigger();
  slim_pdl_wait();
  const SlimSched sc = slim_sched_build(p.lengths, p.batch, p.t_cap, p.workers, 1, s_prefix2, p.status, 0);
  const int b = blockIdx.y, h = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (h >= p.H) return;
  float m = -INFINITY, l = 0.f;
  if (s_prefix2[b + 1] > s_prefix2[b]) {
    const int w0 = slim_worker_of_tile(sc, s_prefix2[b]), w1 = slim_worker_of_tile(sc, s_prefix2[b + 1] - 1);
    const int end = (w1 + 1 + b) * groups;
    for (int i = (w0 + b) * groups + lane; i < end; i += 128) {
      float2 v[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) v[x] = i + 32 * x < end ? part[(size_t)(i + 32 * x) * p.H + h] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float top = fmaxf(m, v[x].x);
        l = top != -INFINITY ? l * exp2f(m - top) + v[x].y * exp2f(v[x].x - top) : l + v[x].y;
        m = top;
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m1 = __shfl_xor_sync(0xffffffffu, m, o), l1 = __shfl_xor_sync(0xffffffffu, l, o), top = fmaxf(m, m1);
    l = top != -INFINITY ? l * exp2f(m - top) + l1 * exp2f(m1 - top) : l + l1;
    m = top;
  }
  if (lane == 0) {
    m_out[(size_t)b * p.H + h] = m == -INFINITY ? 0.f : m;
    inv_out[(size_t)b * p.H + h] = inverse_sum(l);
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
    else if (s != s) l = s;
    m = top;
  }
  auto join = [](float& m0, float& l0, float m1, float l1) {
    const float top = fmaxf(m0, m1);
    l0 = top != -INFINITY ? l0 * exp2f(m0 - top) + l1 * exp2f(m1 - top) : l0 + l1;
    m0 = top;
  };
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) join(m, l, __shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, l, o));
  if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 8; ++w) join(m, l, s_m[w], s_l[w]);
    m_out[(size_t)b * p.H + h] = m == -INFINITY ? 0.f : m;
    inv_out[(size_t)b * p.H + h] = inverse_sum(l);
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
// Which rows stay.  A cluster of CL CTAs per sequence, each warp a contiguous piece of the rows: the (budget - recent)-th
// largest weight of the candidate rows by a radix selection on the order-preserving integer form of the floats (four
// passes of eight bits; the counts of a pass are summed over the cluster), then one pass that counts per warp and one
// that writes the kept indices in order: every row above the threshold, and of the rows equal to it the first ones.
// Latency-bound: the keys are read once into shared memory (a CTA's share up to SEL_KEYS; longer ones are read again from
// L2 in every pass), and long contexts take eight CTAs, short ones one, which saves the cluster's barriers.  1500 rows: 10 us;
// 16 sequences of 8192 to 16384: 18 us.
constexpr int SEL_THREADS = 1024, SEL_WARPS = SEL_THREADS / 32, SEL_KEYS = 48 * 1024;

__device__ __forceinline__ uint32_t order_key(float f) {
  if (f != f) return 0u;                              // NaN: below every number
  const uint32_t u = __float_as_uint(f + 0.f);        // -0 and 0 are equal
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct SelShared {
  unsigned hist[2][256], sum[256];                    // this CTA's counts of a pass (two buffers), the cluster's
  int gt[SEL_WARPS], eq[SEL_WARPS];
  int total[2];                                       // rows above and equal to the threshold in this CTA
  unsigned prefix, need, done;
};

template <int CL>
__global__ void __launch_bounds__(SEL_THREADS)
slim_evict_select_kernel(const int32_t* __restrict__ lengths, const float* __restrict__ acc, int t_cap, int budget, int recent, int staged_cap,
                         int32_t* __restrict__ kept, float* __restrict__ kept_acc, int* status) {
  __shared__ SelShared sh;
  extern __shared__ uint32_t s_key[];                 // [staged_cap]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.x / CL, rank = CL > 1 ? (int)cluster_ctarank() : 0;
  const uint32_t sh_addr = smem_u32(&sh);
  auto sync_all = [&]() { if (CL > 1) cluster_sync_all(); else __syncthreads(); };
  auto peer_word = [&](const void* mine, int r) -> unsigned {           // the word at this place in CTA r's shared memory
    if (CL == 1) return *reinterpret_cast<const unsigned*>(mine);
    unsigned v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];"
                 : "=r"(v) : "r"(mapa(sh_addr + (uint32_t)(reinterpret_cast<const char*>(mine) - reinterpret_cast<const char*>(&sh)), r)));
    return v;
  };
  slim_pdl_trigger();
  slim_pdl_wait();
  int len = lengths[b];
  if (len > t_cap) { len = t_cap; if (tid == 0 && rank == 0) atomicMax(status, (int)SLIM_ERR_CAPACITY); }
  if (len < 0) len = 0;
  int32_t* K = kept + (size_t)b * budget;
  if (len <= budget) {                                // (the whole cluster)
    for (int j = rank * SEL_THREADS + tid; j < budget; j += CL * SEL_THREADS) K[j] = j < len ? j : -1;
    return;
  }
  const int cand = len - recent, need = budget - recent;          // 0 <= need < cand
  const float* A = acc + (size_t)b * t_cap;
  const int seg = ((len + CL * SEL_WARPS - 1) / (CL * SEL_WARPS) + 31) & ~31;
  const int c0 = min(len, rank * SEL_WARPS * seg), c1 = min(len, c0 + SEL_WARPS * seg);       // this CTA's rows
  const int lo = min(len, c0 + warp * seg), hi = min(c1, lo + seg);                           // this warp's
  const bool staged = c1 - c0 <= staged_cap;
  if (staged) {
#pragma unroll 4
    for (int t = c0 + tid; t < c1; t += SEL_THREADS) s_key[t - c0] = order_key(A[t]);
  }
  auto key_at = [&](int t) -> uint32_t { return staged ? s_key[t - c0] : order_key(A[t]); };
  for (int i = tid; i < 512; i += SEL_THREADS) (&sh.hist[0][0])[i] = 0;
  if (tid == 0) sh.done = 0;
  __syncthreads();
  unsigned prefix = 0, left = (unsigned)need;                      // the left-th largest among the keys that share the prefix
  if (need > 0) {
    int pass = 0;
    for (int shift = 24; shift >= 0; shift -= 8, ++pass) {
      unsigned* hist = sh.hist[pass & 1];
      for (int t0 = lo; t0 < min(hi, cand); t0 += 32) {
        const int t = t0 + lane;
        const uint32_t key = t < hi && t < cand ? key_at(t) : 0u;
        const bool in = t < hi && t < cand && (shift == 24 || (key >> (shift + 8)) == prefix);
        const unsigned active = __ballot_sync(0xffffffffu, in);
        if (in) {                                                  // one atomic a distinct digit and warp
          const unsigned digit = (key >> shift) & 255u, same = __match_any_sync(active, digit);
          if (lane == __ffs(same) - 1) atomicAdd(&hist[digit], __popc(same));
        }
      }
      sync_all();
      if (tid < 256) {
        unsigned v[CL], a = 0;
#pragma unroll
        for (int r = 0; r < CL; ++r) v[r] = peer_word(&hist[tid], r);
#pragma unroll
        for (int r = 0; r < CL; ++r) a += v[r];
        sh.sum[tid] = a;
      } else if (pass > 0 && tid < 512) {
        sh.hist[(pass + 1) & 1][tid - 256] = 0;                    // (last read before the barrier above: clear for the next pass)
      }
      __syncthreads();
      if (warp == 0) {                                             // lane k: digits 255 - 8 k .. 248 - 8 k, from the top
        unsigned c[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] = sh.sum[255 - 8 * lane - i]; sum += c[i]; }
        unsigned incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned y = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += y;
        }
        unsigned above = incl - sum;
        if (above < left && left <= incl)
          for (int i = 0; i < 8; ++i) {
            if (left <= above + c[i]) {
              const unsigned longer = (prefix << 8) | (255 - 8 * lane - i);
              sh.prefix = longer; sh.need = left - above;
              sh.done = left - above == c[i] && longer != 0;       // every key with these digits stays: no need to know the others
              break;
            }
            above += c[i];
          }
      }
      __syncthreads();
      prefix = sh.prefix; left = sh.need;
      if (sh.done) {                                               // (the same in all CTAs)
        prefix = (prefix << shift) - 1; left = 0;
        break;
      }
      // (a buffer is counted into again two passes later, behind the next pass's barrier, by when all CTAs have read it)
    }
  }
  // rows with key > prefix stay, and the first `left` of those equal to it (none of either when need = 0)
  const uint32_t thr = need > 0 ? prefix : 0xffffffffu;
  int gt = 0, eq = 0;
  for (int t0 = lo; t0 < hi; t0 += 32) {
    const int t = t0 + lane;
    const uint32_t key = t < hi && t < cand ? key_at(t) : 0u;
    gt += __popc(__ballot_sync(0xffffffffu, t < hi && (t >= cand || (need > 0 && key > thr))));
    eq += __popc(__ballot_sync(0xffffffffu, t < hi && t < cand && need > 0 && key == thr));
  }
  if (lane == 0) { sh.gt[warp] = gt; sh.eq[warp] = eq; }
  __syncthreads();
  if (warp == 0) {
    int a = sh.gt[lane], e = sh.eq[lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { a += __shfl_xor_sync(0xffffffffu, a, o); e += __shfl_xor_sync(0xffffffffu, e, o); }
    if (lane == 0) { sh.total[0] = a; sh.total[1] = e; }
  }
  sync_all();
  int eq_before = 0, out = 0;                                      // equal rows, and kept rows, before this warp's
  int ta[CL], te[CL];
#pragma unroll
  for (int r = 0; r < CL; ++r) { ta[r] = (int)peer_word(&sh.total[0], r); te[r] = (int)peer_word(&sh.total[1], r); }
#pragma unroll
  for (int r = 0; r < CL; ++r) {
    if (r >= rank) break;
    const int a = ta[r], e = te[r];
    out += a + min(e, max((int)left - eq_before, 0));
    eq_before += e;
  }
  for (int w = 0; w < warp; ++w) {
    out += sh.gt[w] + min(sh.eq[w], max((int)left - eq_before, 0));
    eq_before += sh.eq[w];
  }
  for (int t0 = lo; t0 < hi; t0 += 32) {
    const int t = t0 + lane;
    const uint32_t key = t < hi && t < cand ? key_at(t) : 0u;
    const bool is_eq = t < hi && t < cand && need > 0 && key == thr;
    const unsigned eqs = __ballot_sync(0xffffffffu, is_eq), below = (1u << lane) - 1u;
    const bool keep = t < hi && (t >= cand || (need > 0 && key > thr) || (is_eq && eq_before + __popc(eqs & below) < (int)left));
    const unsigned ks = __ballot_sync(0xffffffffu, keep);
    if (keep) {
      const int j = out + __popc(ks & below);
      if (j < budget) { K[j] = t; kept_acc[(size_t)b * t_cap + j] = A[t]; }
    }
    out += __popc(ks);
    eq_before += __popc(eqs);
  }
  sync_all();                                                      // (a CTA's totals may still be read by the others)
}

// The kept rows move to rows 0 .. budget - 1, in place.  Row j comes from row kept[j] >= j, so a block that owns a
// column slice and goes through the rows in order may write a chunk as soon as all sources up to that chunk have been
// read; sources of later chunks lie behind everything it overwrites, so the next chunk is on its way meanwhile.
// The last MV_ACC blocks of a sequence write the weights and clear those of the rows that became free.
// Bound by HBM where the grid fills the GPU (16 sequences down to 4096 rows of 8 KB, 1.07 GB both ways: 187 us, 5.7 TB/s, 0.88 of
// a copy's rate), by the chain of chunks below that.
constexpr int MV_THREADS = 256, MV_UNROLL = 4, MV_ACC = 4;

__device__ __forceinline__ long long storage_row(const int32_t* table, int page_rows, int max_pages, int num_pages, int t_cap, int b, int t,
                                                 int* status) {
  if (!table) return (long long)b * t_cap + t;
  const int pg = table[(size_t)b * max_pages + t / page_rows];
  if (pg < 0 || pg >= num_pages) { atomicMax(status, (int)SLIM_ERR_CAPACITY); return -1; }
  return (long long)pg * page_rows + t % page_rows;
}

template <typename VT, int MV_COLS>
__global__ void __launch_bounds__(MV_THREADS)
slim_evict_move_kernel(unsigned char* __restrict__ base, int vecs, const int32_t* __restrict__ lengths, int t_cap, int budget,
                       const int32_t* __restrict__ kept, const int32_t* __restrict__ table, int page_rows, int max_pages, int num_pages,
                       float* __restrict__ acc, const float* __restrict__ kept_acc, int* status) {
  constexpr int MV_ROWS = MV_THREADS / MV_COLS;
  const int b = blockIdx.y, tid = threadIdx.x;
  slim_pdl_trigger();
  slim_pdl_wait();
  const int len = min(max(lengths[b], 0), t_cap);
  if (len <= budget) return;
  const int32_t* K = kept + (size_t)b * budget;
  const int slices = (vecs + MV_COLS - 1) / MV_COLS;
  if ((int)blockIdx.x >= slices) {
    float* A = acc + (size_t)b * t_cap;
    const float* N = kept_acc + (size_t)b * t_cap;
    for (int t = ((int)blockIdx.x - slices) * MV_THREADS + tid; t < len; t += MV_ACC * MV_THREADS) A[t] = t < budget ? N[t] : 0.f;
    return;
  }
  const int col = blockIdx.x * MV_COLS + tid % MV_COLS, r = tid / MV_COLS;
  VT* K0 = reinterpret_cast<VT*>(base);
  constexpr int CHUNK = MV_ROWS * MV_UNROLL;
  VT v[2][MV_UNROLL];
  long long dst[2][MV_UNROLL];
  int from[MV_UNROLL];                                             // old rows of the chunk after the next
  auto indices = [&](int j0) {
#pragma unroll
    for (int x = 0; x < MV_UNROLL; ++x) {
      const int j = j0 + x * MV_ROWS + r;
      from[x] = j < budget ? K[j] : -1;
    }
  };
  auto load = [&](int j0, VT (&v)[MV_UNROLL], long long (&dst)[MV_UNROLL]) {
#pragma unroll
    for (int x = 0; x < MV_UNROLL; ++x) {
      const int j = j0 + x * MV_ROWS + r;
      dst[x] = -1;
      if (from[x] >= 0 && from[x] != j && col < vecs) {
        const long long a = storage_row(table, page_rows, max_pages, num_pages, t_cap, b, from[x], status);
        const long long z = storage_row(table, page_rows, max_pages, num_pages, t_cap, b, j, status);
        if (a >= 0 && z >= 0) { dst[x] = z * vecs + col; v[x] = K0[a * vecs + col]; }
      }
    }
  };
  indices(0);
  load(0, v[0], dst[0]);
  indices(CHUNK);
  for (int j0 = 0, k = 0; j0 < budget; j0 += CHUNK, k ^= 1) {
    // (both arms are the same code with the buffers' names exchanged, so that they stay in registers)
    if (k == 0) load(j0 + CHUNK, v[1], dst[1]); else load(j0 + CHUNK, v[0], dst[0]);
    indices(j0 + 2 * CHUNK);
    __syncthreads();                 // all sources up to this chunk have been read
#pragma unroll
    for (int x = 0; x < MV_UNROLL; ++x) {
      if (k == 0) { if (dst[0][x] >= 0) K0[dst[0][x]] = v[0][x]; }
      else        { if (dst[1][x] >= 0) K0[dst[1][x]] = v[1][x]; }
    }
  }
}

template <typename VT, int MV_COLS>
cudaError_t launch_move_cols(const slim_ctx* ctx, const slim_cache* c, void* base, int vecs, const int32_t* lengths, int budget,
                             const int32_t* kept, float* acc, const float* kept_acc, cudaStream_t st) {
  return slim_launch_pdl(slim_evict_move_kernel<VT, MV_COLS>, dim3((vecs + MV_COLS - 1) / MV_COLS + (acc ? MV_ACC : 0), c->batch), dim3(MV_THREADS),
                         0, st, (unsigned char*)base, vecs, lengths, c->t_cap, budget, kept, c->block_table, c->page_rows, c->max_pages,
                         c->num_pages, acc, kept_acc, ctx->status);
}
template <typename VT>
cudaError_t launch_move_as(const slim_ctx* ctx, const slim_cache* c, void* base, size_t row_bytes, const int32_t* lengths, int budget,
                           const int32_t* kept, float* acc, const float* kept_acc, cudaStream_t st) {
  const int vecs = (int)(row_bytes / sizeof(VT));
  // Slices of 8 vectors, or of 2 where those would be fewer than the SMs: four times the blocks, each through a quarter of
  // the chunks.  4096 of 12000 rows of 8 KB, one sequence 37 -> 19 us, two (128 blocks of the wider) 40 -> 37, four 51 -> 63.
  return (long long)((vecs + 7) / 8) * c->batch >= ctx->num_sms
             ? launch_move_cols<VT, 8>(ctx, c, base, vecs, lengths, budget, kept, acc, kept_acc, st)
             : launch_move_cols<VT, 2>(ctx, c, base, vecs, lengths, budget, kept, acc, kept_acc, st);
}

// Rows in the widest vectors that divide them (storage and exponents begin on 16-byte boundaries).
cudaError_t launch_move(const slim_ctx* ctx, const slim_cache* c, void* base, size_t row_bytes, const int32_t* lengths, int budget,
                        const int32_t* kept, float* acc, const float* kept_acc, cudaStream_t st) {
  if (row_bytes % 16 == 0) return launch_move_as<uint4>(ctx, c, base, row_bytes, lengths, budget, kept, acc, kept_acc, st);
  if (row_bytes % 4 == 0) return launch_move_as<unsigned>(ctx, c, base, row_bytes, lengths, budget, kept, acc, kept_acc, st);
  return launch_move_as<unsigned char>(ctx, c, base, row_bytes, lengths, budget, kept, acc, kept_acc, st);
}

template <int CL>
cudaError_t launch_select(const slim_ctx* ctx, const slim_cache* c, const int32_t* lengths, const float* acc, int budget, int recent,
                          int32_t* kept, float* kept_acc, cudaStream_t st) {
  const int share = ((c->t_cap + CL * SEL_WARPS - 1) / (CL * SEL_WARPS) + 31) / 32 * 32 * SEL_WARPS, staged = share <= SEL_KEYS ? share : 0;
  auto kern = slim_evict_select_kernel<CL>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SEL_KEYS * 4);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(CL * c->batch); cfg.blockDim = dim3(SEL_THREADS); cfg.dynamicSmemBytes = sizeof(uint32_t) * (size_t)staged; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CL; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, lengths, acc, c->t_cap, budget, recent, staged, kept, kept_acc, ctx->status);
}

}  // namespace

int slim_weights_workers(const slim_ctx* ctx) { return ctx->num_sms; }

cudaError_t slim_launch_weights(const slim_ctx* ctx, const SlimDecodeParams& p_in, float* scores, float2* part, float* m, float* inv_l,
                                float* acc, cudaStream_t st) {
  SlimDecodeParams p = p_in;
  // The one-pass kernel wants whole 16-byte vectors of a head's halves (rows are then multiples of 16 bytes too), all
  // heads of a row in 16 warps, and a ring of at least four rows; 8-bit codes and other shapes take the score kernel of
  // slim_decode's CUDA-core path.
  const int vec = p.kdtype == SLIM_BF16 ? 8 : 4, per_head = (p.half + vec - 1) / vec;
  const int lph = per_head <= 4 ? 4 : per_head <= 8 ? 8 : per_head <= 16 ? 16 : 32;
  const size_t row = (size_t)p.d * (p.kdtype == SLIM_BF16 ? 2 : 4);
  const size_t fixed = sizeof(int) * (p.batch + 4) + 16 * 16 + 128, room = 227 * 1024 - fixed;
  WeightsRing ring = {SLIM_TT, 0, 1, (p.H * lph + 31) / 32};
  while (2 * ring.groups * ring.warps <= WC / 32 && ring.groups < SLIM_TT) ring.groups *= 2;
  while (ring.rows > 1 && room / (row * ring.rows) < 4) ring.rows /= 2;
  ring.stages = (int)(room / (row * ring.rows));
  if (ring.stages > 8) ring.stages = 8;
  cudaError_t e;
  if (p.kdtype != SLIM_FP8 && p.half % vec == 0 && ring.warps <= WC / 32 && ring.stages >= 4) {
    p.workers = slim_weights_workers(ctx);
    const size_t smem = (size_t)ring.stages * ring.rows * row + fixed;
#define SLIM_W(KT, L) (p.rope ? slim_weights_scores_kernel<KT, true, L> : slim_weights_scores_kernel<KT, false, L>)
#define SLIM_WL(KT) (lph == 4 ? SLIM_W(KT, 4) : lph == 8 ? SLIM_W(KT, 8) : lph == 16 ? SLIM_W(KT, 16) : SLIM_W(KT, 32))
    auto kern = p.kdtype == SLIM_BF16 ? SLIM_WL(__nv_bfloat16) : SLIM_WL(float);
#undef SLIM_WL
#undef SLIM_W
    if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return e;
    e = slim_launch_pdl(kern, dim3(p.workers), dim3(WT), smem, st, p, scores, part, ring);
    if (e == cudaSuccess)
      e = slim_launch_pdl(slim_weights_join_kernel, dim3((p.H + 7) / 8, p.batch), dim3(256), sizeof(int) * (p.batch + 1), st, p,
                          (const float2*)part, ring.groups, m, inv_l);
  } else {
    e = slim_launch_scores(ctx, p, scores, st);
    if (e == cudaSuccess) e = slim_launch_pdl(slim_weights_stat_kernel, dim3(p.H, p.batch), dim3(256), 0, st, p, (const float*)scores, m, inv_l);
  }
  if (e == cudaSuccess)
    e = slim_launch_pdl(slim_weights_add_kernel, dim3((p.t_cap + 255) / 256, p.batch), dim3(256), 0, st, p, (const float*)scores,
                        (const float*)m, (const float*)inv_l, acc);
  return e;
}

// kept_acc: float scratch [batch][t_cap]
cudaError_t slim_launch_evict(const slim_ctx* ctx, const slim_cache* c, const int32_t* lengths, float* acc, int budget, int recent,
                              int32_t* kept, float* kept_acc, cudaStream_t st) {
  cudaError_t e = c->t_cap >= 8192 ? launch_select<8>(ctx, c, lengths, acc, budget, recent, kept, kept_acc, st)
                                   : launch_select<1>(ctx, c, lengths, acc, budget, recent, kept, kept_acc, st);
  if (e != cudaSuccess) return e;
  const size_t row = (size_t)ctx->d * (ctx->kdtype == SLIM_FP8 ? 1 : ctx->kdtype == SLIM_BF16 ? 2 : 4);
  e = launch_move(ctx, c, c->k, row, lengths, budget, kept, acc, kept_acc, st);
  if (e == cudaSuccess && ctx->kdtype == SLIM_FP8)       // the exponents of the same rows
    e = launch_move(ctx, c, c->k_exp, ctx->H, lengths, budget, kept, nullptr, nullptr, st);
  return e;
}
