// Attention for a tree of drafted tokens over the K-cache (slim_tree_decode): the CUDA-core kernels, which take every
// shape (f32 caches, head widths and model widths outside the tensor-core kernels).
//
// For token i of sequence b (L cached rows, position L + depth(i)) and head h, over the rows t < L and the drafted
// keys j that are i itself or one of its ancestors:
//   s_t = R_{pos(i)} q . R_{pos(t)} k_t log2(e) / sqrt(d_k),   p_t = 2^(s_t - m),   l = sum p_t,
//   u_{i,h} = sum_t (p_t / l) k_t    (the whole d-wide un-rotated row, Eq. 7 Option 2),   o_{i,h} = u_{i,h} W_KV,h.
// One sequence has R = H n rows u of d numbers each, far more than on-chip memory holds, so the arguments are laid
// down once ([b][h n + i][t], float) and the weighted sum is a matrix product P [R x T] K [T x d] cut into tiles;
// where there are few tiles, T is cut too and the parts are added in a fixed order.
//
// Short contexts are bound by latency: 1500 float32 rows, d = 384, 6 heads, 8 drafts 27 us in four launches (scores 9.5,
// statistics 5.5, sums 10, projection 6.5, overlapping); loads of the next step run under a step's products throughout.
// Long ones are bound by the shared-memory reads of the weighted sum's 64 x 64 tile: 4 x 16384 float32 rows, d = 2048, 16 heads,
// 8 drafts 1.99 ms (18.5 TFLOP/s; elementary torch operations 4.08 ms); 16 x 8192 bf16 rows, d = 2560, head width 80,
// 16 drafts 15.2 ms (23.6 TFLOP/s, as elementary torch operations).
#include <cstring>

#include "slim_internal.h"
#include "slim_ptx.cuh"
#include "slim_sched.cuh"
#include "slim_tree.h"

using namespace slim_ptx;

namespace {

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }   // the one rounding of a bf16 context's output

__device__ __forceinline__ float2 rope_at(const SlimDecodeParams& p, int pos, int j) {
  const float2 cb = __ldg(p.rope_base + (size_t)(pos / SLIM_TT) * p.half + j), co = __ldg(p.rope_off + (pos % SLIM_TT) * p.half + j);
  return make_float2(cb.x * co.x - cb.y * co.y, cb.y * co.x + cb.x * co.y);
}

__device__ __forceinline__ void turn_pair(float& u, float& v, float2 cs) {
  const float a = u * cs.x + v * cs.y;
  v = v * cs.x - u * cs.y;
  u = a;
}

// Softmax arguments (log2 units): block = 64 keys of one (sequence, head) against all its tokens; the last block
// of the row is the drafted keys, and that of head 0 leaves the length and the depths for the kernels behind.  A parent
// that is not an earlier token of the tree makes the token padding and raises SLIM_ERR_TREE; parents below -1 are padding.
constexpr int TS_KEYS = 64;
template <typename KT>
__global__ void __launch_bounds__(256) slim_tree_scores_kernel(const SlimDecodeParams p, const SlimTreeView t, const int32_t* __restrict__ parents) {
  extern __shared__ float sm[];
  __shared__ int s_par[SLIM_MAX_TREE], dep[SLIM_MAX_TREE];
  __shared__ unsigned long long mask[SLIM_MAX_TREE];
  const int dk = p.d_k, half = p.half, dk4 = (dk + 3) & ~3, ld = dk4 + 1, n = t.n, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float* Qs = sm;                                    // [n][dk4], zeros behind dk: four elements a read, the same ones in a warp
  float* Ks = Qs + n * dk4;                          // [TS_KEYS][dk4 + 1], an odd stride: the lanes' keys in different banks
  const int b = blockIdx.z, h = blockIdx.y;
  const bool draft = blockIdx.x == gridDim.x - 1;
  slim_pdl_trigger();
  slim_pdl_wait();
  const int stored = p.lengths[b], len = min(max(stored, 0), p.t_cap), t0 = draft ? 0 : blockIdx.x * TS_KEYS;
  if (!draft && t0 >= len) return;
  const int keys = draft ? n : min(TS_KEYS, len - t0);
  const bool opens = draft && h == 0;
  const KT* Kc = reinterpret_cast<const KT*>(p.k);
  const KT* Kt = reinterpret_cast<const KT*>(t.k_tree) + (size_t)b * n * p.d;
  auto load_keys = [&]() {                           // a warp's eight rows at a time
    const KT* row[8];
    int pos[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const int r = min(warp + 8 * x, keys - 1);
      row[x] = draft ? Kt + (size_t)r * p.d : Kc + (size_t)(slim_cache_row(p, b, (t0 + r) & ~(SLIM_TT - 1)) + (r & (SLIM_TT - 1))) * p.d;
      pos[x] = draft ? len + max(dep[r], 0) : t0 + r;
    }
    for (int j = lane; j < half; j += 32) {
      KT k1[8], k2[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) { k1[x] = row[x][h * dk + j]; k2[x] = row[x][h * dk + half + j]; }
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int r = warp + 8 * x;
        const bool live = r < keys && !(draft && dep[r] < 0);
        float u = live ? to_f(k1[x]) : 0.f, v = live ? to_f(k2[x]) : 0.f;
        if (p.rope) turn_pair(u, v, rope_at(p, pos[x], j));
        Ks[r * ld + j] = u; Ks[r * ld + half + j] = v;
      }
    }
  };
  if (tid < n) {
    const int q = parents[(size_t)b * n + tid];
    s_par[tid] = q >= tid ? -3 : q < -1 ? -2 : q;
  }
  if (!draft) load_keys();                           // (cached keys need not wait for the tree)
  __syncthreads();
  if (tid < n) {
    bool broken;
    slim_tree_chain(s_par, tid, mask[tid], dep[tid], broken);
    if (opens) {
      t.depth[(size_t)b * n + tid] = dep[tid];
      if (broken) atomicMax(p.status, (int)SLIM_ERR_TREE);
    }
  }
  if (opens && tid == 0) {
    t.len[b] = len;
    if (stored > p.t_cap) atomicMax(p.status, (int)SLIM_ERR_CAPACITY);
  }
  __syncthreads();
  if (draft) load_keys();
  if (dk4 != dk) {                                   // (an even width: two zeros)
    if (tid < TS_KEYS) Ks[tid * ld + dk] = Ks[tid * ld + dk + 1] = 0.f;
    if (tid < n) Qs[tid * dk4 + dk] = Qs[tid * dk4 + dk + 1] = 0.f;
  }
  const KT* Q = reinterpret_cast<const KT*>(p.q) + (size_t)b * n * p.d;
  for (int j = lane; j < half; j += 32) {            // all of a warp's tokens at a time
    KT q1[SLIM_MAX_TREE / 8], q2[SLIM_MAX_TREE / 8];
#pragma unroll
    for (int x = 0; x < SLIM_MAX_TREE / 8; ++x) {
      const size_t at = (size_t)(warp + 8 * x) * p.d + h * dk + j;
      if (warp + 8 * x < n) { q1[x] = Q[at]; q2[x] = Q[at + half]; }
    }
#pragma unroll
    for (int x = 0; x < SLIM_MAX_TREE / 8; ++x) {
      const int i = warp + 8 * x;
      if (i >= n) break;
      const bool live = dep[i] >= 0;
      float u = live ? to_f(q1[x]) * p.qscale : 0.f, v = live ? to_f(q2[x]) * p.qscale : 0.f;
      if (p.rope && live) turn_pair(u, v, rope_at(p, len + dep[i], j));
      Qs[i * dk4 + j] = u; Qs[i * dk4 + half + j] = v;
    }
  }
  __syncthreads();
  const int r = tid & (TS_KEYS - 1);
  if (r >= keys) return;
  float* S = t.s + ((size_t)b * p.H + h) * n * t.s_ld + (draft ? t.s_draft : t0) + r;
  for (int i0 = tid / TS_KEYS; i0 < n; i0 += 16) {   // four tokens at a time: i0, i0 + 4, i0 + 8, i0 + 12
    float a[4] = {0.f, 0.f, 0.f, 0.f};
    const int i1 = min(i0 + 4, n - 1), i2 = min(i0 + 8, n - 1), i3 = min(i0 + 12, n - 1);
    const float4* q0 = reinterpret_cast<const float4*>(Qs + i0 * dk4);
    const float4* q1 = reinterpret_cast<const float4*>(Qs + i1 * dk4);
    const float4* q2 = reinterpret_cast<const float4*>(Qs + i2 * dk4);
    const float4* q3 = reinterpret_cast<const float4*>(Qs + i3 * dk4);
    const float* kr = Ks + r * ld;
#pragma unroll 4
    for (int j = 0; j < dk4; j += 4) {
      const float4 u[4] = {q0[j / 4], q1[j / 4], q2[j / 4], q3[j / 4]};
      const float k0 = kr[j], k1 = kr[j + 1], k2 = kr[j + 2], k3 = kr[j + 3];
#pragma unroll
      for (int x = 0; x < 4; ++x) a[x] = fmaf(k3, u[x].w, fmaf(k2, u[x].z, fmaf(k1, u[x].y, fmaf(k0, u[x].x, a[x]))));
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int i = i0 + 4 * x;
      if (i < n) S[(size_t)i * t.s_ld] = (draft && !((mask[i] >> r) & 1)) ? -INFINITY : a[x];
    }
  }
}

// m and 1 / l of every row (one block a row); padding gets 1 / l = 0.  A token that is there attends itself at least, so a
// sum that is not a positive number (arguments that are NaN or infinite) is no empty row: its 1 / l is NaN.
__global__ void __launch_bounds__(256) slim_tree_stat_kernel(const SlimDecodeParams p, const SlimTreeView t) {
  __shared__ float s_m[8], s_l[8];
  slim_pdl_trigger();
  slim_pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, R = p.H * t.n, row = blockIdx.x, b = blockIdx.y;
  const int i = row % t.n, len = t.len[b];
  float m = -INFINITY, l = 0.f;
  auto join = [&](float m1, float l1) {
    const float top = fmaxf(m, m1);
    l = top != -INFINITY ? l * exp2f(m - top) + l1 * exp2f(m1 - top) : l + l1;       // (the maximum passes over NaN, the sum keeps it)
    m = top;
  };
  auto one = [](float v) { return v == -INFINITY ? 0.f : v == v ? 1.f : v; };
  const bool there = t.depth[(size_t)b * t.n + i] >= 0;
  if (there) {
    const float* S = t.s + ((size_t)b * R + row) * t.s_ld;
    for (int x = tid; x < len; x += 1024) {
      float v[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) v[y] = x + 256 * y < len ? S[x + 256 * y] : -INFINITY;
#pragma unroll
      for (int y = 0; y < 4; ++y) join(v[y], one(v[y]));
    }
    if (tid < t.n) {
      const float v = S[t.s_draft + tid];
      join(v, one(v));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float m1 = __shfl_xor_sync(0xffffffffu, m, o), l1 = __shfl_xor_sync(0xffffffffu, l, o);
      join(m1, l1);
    }
  }
  if (lane == 0) { s_m[tid >> 5] = m; s_l[tid >> 5] = l; }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 8; ++w) join(s_m[w], s_l[w]);
    t.m[(size_t)b * R + row] = m == -INFINITY ? 0.f : m;
    t.inv_l[(size_t)b * R + row] = !there ? 0.f : l > 0.f && l < INFINITY ? 1.f / l : NAN;
  }
}

// U = P K, 64 rows x 64 columns a block, 16 keys a step; blockIdx.z = sequence x part of the keys.
template <typename KT>
__global__ void __launch_bounds__(256) slim_tree_sum_kernel(const SlimDecodeParams p, const SlimTreeView t) {
  __shared__ float Ps[16][68], Bs[16][64], s_m[64], s_il[64];
  slim_pdl_trigger();
  slim_pdl_wait();
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, R = p.H * t.n;
  const int b = blockIdx.z / t.parts, part = blockIdx.z % t.parts;
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, len = t.len[b];
  const int nb = (len + 15) / 16, nd = (t.n + 15) / 16;            // 16-key steps: cached, drafted
  const int s0 = (int)((long long)(nb + nd) * part / t.parts), s1 = (int)((long long)(nb + nd) * (part + 1) / t.parts);
  const KT* Kc = reinterpret_cast<const KT*>(p.k);
  const KT* Kt = reinterpret_cast<const KT*>(t.k_tree) + (size_t)b * t.n * p.d;
  if (tid < 64) {
    const bool in = r0 + tid < R;
    s_m[tid] = in ? t.m[(size_t)b * R + r0 + tid] : 0.f;
    s_il[tid] = in ? t.inv_l[(size_t)b * R + r0 + tid] : 0.f;
  }
  float acc[4][4];
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < 4; ++y) acc[x][y] = 0.f;
  // arguments and keys of a step, used only after the step before; the page of the step after it is looked up meanwhile
  float sv[4];
  KT kv[4];
  long long row = s0 < min(s1, nb) ? slim_cache_row(p, b, s0 * 16) : 0;
  auto load = [&](int s) {
    const bool draft = s >= nb;
    const int t0 = (draft ? s - nb : s) * 16, keys = min(16, (draft ? t.n : len) - t0);
    const KT* K0 = draft ? Kt + (size_t)t0 * p.d : Kc + (size_t)row * p.d;
    if (s + 1 < min(s1, nb)) row = slim_cache_row(p, b, (s + 1) * 16);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int e = tid + 256 * x, r = e >> 4, k = e & 15;
      sv[x] = r0 + r < R && k < keys ? t.s[((size_t)b * R + r0 + r) * t.s_ld + (draft ? t.s_draft : 0) + t0 + k] : -INFINITY;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int e = tid + 256 * x, k = e >> 6, c = e & 63;
      const bool live = k < keys && c0 + c < p.d && !(draft && t.depth[(size_t)b * t.n + t0 + k] < 0);
      kv[x] = live ? K0[(size_t)k * p.d + c0 + c] : KT(0.f);
    }
  };
  if (s0 < s1) load(s0);
  for (int s = s0; s < s1; ++s) {
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int e = tid + 256 * x, r = e >> 4;
      const float il = s_il[r];
      Ps[e & 15][r] = il != 0.f ? exp2f(sv[x] - s_m[r]) * il : 0.f;
      Bs[e >> 6][e & 63] = to_f(kv[x]);
    }
    __syncthreads();
    if (s + 1 < s1) load(s + 1);                                   // on their way while this step's are used
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const float4 a = *reinterpret_cast<const float4*>(&Ps[k][4 * ty]), w = *reinterpret_cast<const float4*>(&Bs[k][4 * tx]);
      const float av[4] = {a.x, a.y, a.z, a.w}, wv[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[x][y] = fmaf(av[x], wv[y], acc[x][y]);
    }
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int r = r0 + 4 * ty + x;
    if (r >= R) continue;
    float* U = t.u + (((size_t)part * p.batch + b) * R + r) * p.d + c0 + 4 * tx;
    const bool none = s_il[4 * ty + x] == 0.f;                     // (padding: 0 whatever the keys hold)
#pragma unroll
    for (int y = 0; y < 4; ++y)
      if (c0 + 4 * tx + y < p.d) U[y] = none ? 0.f : acc[x][y];
  }
}

// o = u W_KV,h, the parts of u added in order: 8 (sequence, token) rows x 32 columns of one head a cluster, whose CTAs
// share the d rows of W_KV,h and add their sums through distributed shared memory, in order.  In a CTA eight threads share
// a column's j, eight rows of W_KV each, the next ones on their way meanwhile.  (The bound on the blocks an SM holds
// gives the loads their registers: without it the compiler allows 32, and the loads wait for one another, 34 us for 8.)
constexpr int TP_ROWS = 8, TP_J = 64, TP_MAX = 8;
template <int N>
__device__ __forceinline__ void add_parts(const float* const (&src)[2], size_t un, int s0, float (&u)[2]) {
  float v[N][2];
#pragma unroll
  for (int s = 0; s < N; ++s)
#pragma unroll
    for (int x = 0; x < 2; ++x) v[s][x] = src[x][(size_t)(s0 + s) * un];
#pragma unroll
  for (int s = 0; s < N; ++s)
#pragma unroll
    for (int x = 0; x < 2; ++x) u[x] += v[s][x];
}
template <typename KT>
__global__ void __launch_bounds__(256, 3) slim_tree_project_kernel(const SlimDecodeParams p, const SlimTreeView t, KT* __restrict__ o, int share) {
  __shared__ __align__(16) float Us[TP_ROWS][TP_J + 4];
  __shared__ float Rs[8][TP_ROWS][32], s_out[TP_ROWS][32];
  const int tid = threadIdx.x, c = tid & 31, g = tid >> 5, n = t.n, d = p.d, dk = p.d_k, h = blockIdx.z;
  const int rank = blockIdx.x % share, m0 = blockIdx.y * TP_ROWS, M = p.batch * n, col = blockIdx.x / share * 32 + c;
  const int ns = (d + TP_J - 1) / TP_J, j_end = ns * (rank + 1) / share * TP_J;
  const size_t un = (size_t)p.batch * p.H * n * d;
  const KT* W = reinterpret_cast<const KT*>(p.wkv) + (size_t)h * d * dk;
  slim_pdl_trigger();
  slim_pdl_wait();
  float acc[TP_ROWS];
#pragma unroll
  for (int r = 0; r < TP_ROWS; ++r) acc[r] = 0.f;
  // what a step loads, used (and converted) only after the step before; addresses behind the end are clamped
  KT w[TP_J / 8];
  float u[2];
  const float* row[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int m = min(m0 + ((tid + 256 * x) >> 6), M - 1);
    row[x] = t.u + (((size_t)(m / n) * p.H + h) * n + m % n) * d;
  }
  const KT* wcol = W + min(col, dk - 1);
  auto load = [&](int j0) {
#pragma unroll
    for (int x = 0; x < TP_J / 8; ++x) w[x] = wcol[(size_t)min(j0 + 8 * g + x, d - 1) * dk];
    const float* src[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      src[x] = row[x] + min(j0 + (tid & 63), d - 1);
      u[x] = *src[x];
    }
    int s0 = 1;
    for (; s0 + 12 <= t.parts; s0 += 12) add_parts<12>(src, un, s0, u);      // 24 loads in flight
    for (; s0 + 4 <= t.parts; s0 += 4) add_parts<4>(src, un, s0, u);
    for (; s0 < t.parts; ++s0) add_parts<1>(src, un, s0, u);
  };
  const int j_begin = ns * rank / share * TP_J;
  if (j_begin < j_end) load(j_begin);
  for (int j0 = j_begin; j0 < j_end; j0 += TP_J) {
    float wc[TP_J / 8];
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 2; ++x) Us[(tid + 256 * x) >> 6][tid & 63] = j0 + (tid & 63) < d ? u[x] : 0.f;
#pragma unroll
    for (int x = 0; x < TP_J / 8; ++x) wc[x] = j0 + 8 * g + x < d ? to_f(w[x]) : 0.f;
    __syncthreads();
    if (j0 + TP_J < j_end) load(j0 + TP_J);                // on their way while this step's are used
#pragma unroll
    for (int r = 0; r < TP_ROWS; ++r) {
      const float4 a = *reinterpret_cast<const float4*>(&Us[r][8 * g]), z = *reinterpret_cast<const float4*>(&Us[r][8 * g + 4]);
      acc[r] = fmaf(a.w, wc[3], fmaf(a.z, wc[2], fmaf(a.y, wc[1], fmaf(a.x, wc[0], acc[r]))));
      acc[r] = fmaf(z.w, wc[7], fmaf(z.z, wc[6], fmaf(z.y, wc[5], fmaf(z.x, wc[4], acc[r]))));
    }
  }
#pragma unroll
  for (int r = 0; r < TP_ROWS; ++r) Rs[g][r][c] = acc[r];
  __syncthreads();
  float v = 0.f;
#pragma unroll
  for (int x = 0; x < 8; ++x) v += Rs[x][g][c];
  if (share > 1) {                                         // row g is written by CTA g % share
    s_out[g][c] = v;
    cluster_sync_all();
    if (g % share == rank) {
      v = 0.f;
      for (int k = 0; k < share; ++k) v += ld_cluster_f32(mapa(smem_u32(&s_out[g][c]), k));
    }
    cluster_sync_all();                                    // a CTA's shared memory is read by the others until here
    if (g % share != rank) return;
  }
  if (m0 + g < M && col < dk) put(o + (size_t)(m0 + g) * d + h * dk + col, v);
}

template <typename KT>
cudaError_t launch_generic(const slim_ctx* ctx, const SlimDecodeParams& p, const SlimTreeView& t, const int32_t* parents, void* o, cudaStream_t st) {
  const size_t dk4 = (p.d_k + 3) & ~3, smem = sizeof(float) * (TS_KEYS * (dk4 + 1) + t.n * dk4);
  auto ks = slim_tree_scores_kernel<KT>;
  cudaError_t e = slim_allow_smem((const void*)ks);
  if (e != cudaSuccess) return e;
  const int R = p.H * t.n;
  e = slim_launch_pdl(ks, dim3((p.t_cap + TS_KEYS - 1) / TS_KEYS + 1, p.H, p.batch), dim3(256), smem, st, p, t, parents);
  if (e == cudaSuccess) e = slim_launch_pdl(slim_tree_stat_kernel, dim3(R, p.batch), dim3(256), 0, st, p, t);
  if (e == cudaSuccess)
    e = slim_launch_pdl(slim_tree_sum_kernel<KT>, dim3((p.d + 63) / 64, (R + 63) / 64, p.batch * t.parts), dim3(256), 0, st, p, t);
  if (e != cudaSuccess) return e;
  const int col_blocks = (p.d_k + 31) / 32, row_blocks = (p.batch * t.n + TP_ROWS - 1) / TP_ROWS;
  const long long blocks = (long long)col_blocks * row_blocks * p.H, ns = (p.d + TP_J - 1) / TP_J;
  long long fit = 2LL * ctx->num_sms / blocks;             // CTAs of a cluster: as many as leave two an SM
  if (fit > TP_MAX) fit = TP_MAX;
  const int share = (int)(fit > ns ? ns : fit < 1 ? 1 : fit);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(col_blocks * share, row_blocks, p.H); cfg.blockDim = dim3(256); cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = share; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, slim_tree_project_kernel<KT>, p, t, (KT*)o, share);
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

// Parts the keys are cut into: enough blocks for two on every SM, never more than 32.
static int tree_parts(const slim_ctx* ctx, int batch, int t_cap, int n) {
  const long long tiles = (long long)((ctx->d + 63) / 64) * ((ctx->H * n + 63) / 64) * batch;
  long long parts = (2 * ctx->num_sms + tiles - 1) / tiles;
  const long long most = (t_cap + 63) / 64;
  if (parts > most) parts = most;
  if (parts > 32) parts = 32;
  return parts < 1 ? 1 : (int)parts;
}

SlimTreeLayout slim_tree_ws_layout(const slim_ctx* ctx, int batch, int t_cap, int n) {
  SlimTreeLayout L;
  const size_t rows = (size_t)batch * ctx->H * n;
  L.parts = tree_parts(ctx, batch, t_cap, n);
  L.s_draft = (t_cap + 63) / 64 * 64;
  L.s_ld = L.s_draft + 64;
  size_t off = 0;
  L.depth = off; off = align256(off + sizeof(int) * (size_t)batch * n);
  L.len = off; off = align256(off + sizeof(int) * (size_t)batch);
  L.inv_l = off; off = align256(off + sizeof(float) * rows);
  L.shared_end = off;
  L.m = off; off = align256(off + sizeof(float) * rows);
  L.s = off; off = align256(off + sizeof(float) * rows * L.s_ld);
  L.u = off; off = align256(off + sizeof(float) * (size_t)L.parts * rows * ctx->d);
  L.total = off;
  if (slim_tree_tc_ok(ctx)) slim_tree_tc_layout(ctx, batch, t_cap, n, L);
  return L;
}

// tc: run the tensor-core kernels (the caller has checked slim_tree_tc_ok); total_rows: rows of the key storage
cudaError_t slim_launch_tree(const slim_ctx* ctx, const SlimDecodeParams& p, const void* k_tree, const int32_t* parents, int n,
                             void* o, char* ws, int tc, long long total_rows, cudaStream_t st) {
  const SlimTreeLayout L = slim_tree_ws_layout(ctx, p.batch, p.t_cap, n);
  SlimTreeView t;
  memset(&t, 0, sizeof(t));
  t.n = n; t.k_tree = k_tree;
  t.depth = reinterpret_cast<int*>(ws + L.depth);
  t.len = reinterpret_cast<int*>(ws + L.len);
  t.inv_l = reinterpret_cast<float*>(ws + L.inv_l);
  if (tc) {
    t.p = reinterpret_cast<__nv_bfloat16*>(ws + L.p); t.p_ld = L.p_ld; t.s_draft = L.p_s_draft;
    t.stat = reinterpret_cast<float2*>(ws + L.stat);
    t.tail = reinterpret_cast<__nv_bfloat16*>(ws + L.tail);
    t.uh = reinterpret_cast<__nv_bfloat16*>(ws + L.uh);
    t.part = reinterpret_cast<float*>(ws + L.part);
    t.sched = reinterpret_cast<long long*>(ws + L.sched);
    t.g_tiles = L.g_tiles; t.g_ncol = L.g_ncol; t.g_split = L.g_split; t.g_pairs = L.g_pairs; t.g_whole = L.g_whole;
    return slim_launch_tree_tc(ctx, p, t, L, parents, total_rows, o, st);
  }
  t.parts = L.parts; t.s_ld = L.s_ld; t.s_draft = L.s_draft;
  t.m = reinterpret_cast<float*>(ws + L.m);
  t.s = reinterpret_cast<float*>(ws + L.s);
  t.u = reinterpret_cast<float*>(ws + L.u);
  return p.dtype == SLIM_BF16 ? launch_generic<__nv_bfloat16>(ctx, p, t, parents, o, st) : launch_generic<float>(ctx, p, t, parents, o, st);
}
