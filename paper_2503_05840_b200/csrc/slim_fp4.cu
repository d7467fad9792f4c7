// Decode over a 4-bit K-cache on CUDA cores: every shape (head widths that the tensor-core kernel does not take, odd numbers
// of heads), float32 arithmetic.  Two passes over the keys, as for the other cache types: the softmax arguments of all
// heads (Eq. 2; keys rotated after the read), then the weighted sum of the full-width keys (Eq. 7 Option 2).
// Bound by its instructions, one code at a time: 16 contexts of 8-16k rows of 4096, 32 heads, 14.8 ms, where the tensor cores
// take 0.29; 64 contexts of 1500 rows of 1280 1.6 ms (0.07).
#include "slim_fp4.cuh"
#include "slim_sched.cuh"

namespace {

constexpr int THREADS = 256;

// One CTA walks tiles of 16 rows; a warp owns rows of the tile and goes over the heads, its lanes over the rotation pairs.
__global__ void __launch_bounds__(THREADS) fp4_scores_kernel(const SlimDecodeParams p, float* __restrict__ scores) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  float* s_q = reinterpret_cast<float*>(smem_raw);                    // [d] rotated, scaled query
  int* s_prefix = reinterpret_cast<int*>(s_q + p.d);
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int d = p.d, H = p.H, dk = p.d_k, half = p.half;
  const unsigned char* codes = reinterpret_cast<const unsigned char*>(p.k);
  const __nv_bfloat16* Q = reinterpret_cast<const __nv_bfloat16*>(p.q);
  const int pitch = slim_fp4_code_pitch(d), spitch = slim_fp4_scale_pitch(d);
  const SlimSched sc = slim_sched_build(p.lengths, p.batch, p.t_cap, p.workers, p.min_tiles, s_prefix, p.status, p.unit_cost);
  int cur_b = -1;
  for (int g = blockIdx.x; g < sc.total_tiles; g += gridDim.x) {
    const int b = slim_seq_of_tile(s_prefix, p.batch, g);
    const int tile = g - s_prefix[b], t0 = tile * SLIM_TT;
    const int len = min(max(p.lengths[b], 0), p.t_cap);
    if (b != cur_b) {
      cur_b = b;
      __syncthreads();
      const int m = len - 1, mt = m / SLIM_TT, mi = m % SLIM_TT;
      for (int e = tid; e < d; e += THREADS) {
        const int h = e / dk, jj = e - h * dk, j = jj < half ? jj : jj - half;
        const float q1 = __bfloat162float(Q[(size_t)b * d + h * dk + j]), q2 = __bfloat162float(Q[(size_t)b * d + h * dk + j + half]);
        float v = jj < half ? q1 : q2;
        if (p.rope) {
          const float2 cb = p.rope_base[(size_t)mt * half + j], co = p.rope_off[mi * half + j];
          const float c = cb.x * co.x - cb.y * co.y, s = cb.y * co.x + cb.x * co.y;
          v = jj < half ? (q1 * c + q2 * s) : (-q1 * s + q2 * c);
        }
        s_q[e] = v * p.qscale;
      }
      __syncthreads();
    }
    for (int t = wid; t < SLIM_TT; t += THREADS / 32) {
      if (t0 + t >= len) break;
      const long long row = slim_cache_row(p, b, t0) + t;
      const unsigned char* kc = codes + (size_t)row * pitch;
      const unsigned char* ks = p.k_sc4 + (size_t)row * spitch;
      for (int h = 0; h < H; ++h) {
        float a = 0.f;
        for (int j = lane; j < half; j += 32) {
          const float k1 = slim_fp4_at(kc, ks, h * dk + j), k2 = slim_fp4_at(kc, ks, h * dk + j + half);
          const float q1 = s_q[h * dk + j], q2 = s_q[h * dk + j + half];
          if (p.rope) {
            const float2 cb = __ldg(p.rope_base + (size_t)tile * half + j), co = __ldg(p.rope_off + t * half + j);
            const float c = cb.x * co.x - cb.y * co.y, s = cb.y * co.x + cb.x * co.y;
            a += c * (q1 * k1 + q2 * k2) + s * (q1 * k2 - q2 * k1);
          } else {
            a += q1 * k1 + q2 * k2;
          }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        if (lane == 0) scores[((size_t)b * H + h) * p.t_cap + t0 + t] = a;
      }
    }
  }
}

// CTA = (slice of 256 columns, worker): online softmax of every head over the worker's tiles, a column a thread.
template <int HP>
__global__ void __launch_bounds__(THREADS, 2) fp4_accum_kernel(const SlimDecodeParams p, const float* __restrict__ scores) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  float* s_P = reinterpret_cast<float*>(smem_raw);                  // [HP][TT]
  float* s_alpha = s_P + HP * SLIM_TT;                              // [HP]
  float* s_m = s_alpha + HP;                                        // [HP]
  float* s_l = s_m + HP;                                            // [HP]
  int* s_prefix = reinterpret_cast<int*>(s_l + HP);                 // [batch+1]
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int w = blockIdx.y, d = p.d, H = p.H;
  const int col = blockIdx.x * THREADS + tid;
  const unsigned char* codes = reinterpret_cast<const unsigned char*>(p.k);
  const int pitch = slim_fp4_code_pitch(d), spitch = slim_fp4_scale_pitch(d);
  const SlimSched sc = slim_sched_build(p.lengths, p.batch, p.t_cap, p.workers, p.min_tiles, s_prefix, p.status, p.unit_cost);
  if (sc.total_tiles == 0 || w >= sc.workers_eff) return;
  const int g_begin = slim_worker_start(sc, w), g_end = slim_worker_start(sc, w + 1);
  float acc[HP];
  for (int g = g_begin; g < g_end;) {
    const int b = slim_seq_of_tile(s_prefix, p.batch, g);
    const int seg_end = min(g_end, s_prefix[b + 1]);
    const int tile0 = g - s_prefix[b], tile1 = seg_end - s_prefix[b];
    const int unit = w + b;
    const int len = min(max(p.lengths[b], 0), p.t_cap);
    __syncthreads();
    if (tid < HP) { s_m[tid] = -INFINITY; s_l[tid] = 0.f; }
#pragma unroll
    for (int h = 0; h < HP; ++h) acc[h] = 0.f;
    __syncthreads();
    for (int tile = tile0; tile < tile1; ++tile) {
      const int t0 = tile * SLIM_TT;
      const long long row0 = slim_cache_row(p, b, t0);
      float kv[SLIM_TT];
#pragma unroll
      for (int t = 0; t < SLIM_TT; ++t)
        kv[t] = (col < d && t0 + t < len) ? slim_fp4_at(codes + (size_t)(row0 + t) * pitch, p.k_sc4 + (size_t)(row0 + t) * spitch, col) : 0.f;
      for (int h = wid; h < H; h += THREADS / 32) {
        const bool there = lane < SLIM_TT && t0 + lane < len;
        const float s = there ? __ldg(scores + ((size_t)b * H + h) * p.t_cap + t0 + lane) : -INFINITY;
        float mx = s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float m_old = s_m[h], m_new = fmaxf(m_old, mx);
        const float pr = s == -INFINITY ? 0.f : exp2f(s - m_new);
        float ps = pr;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, o);
        const float alpha = m_old == m_new ? 1.f : exp2f(m_old - m_new);
        if (lane < SLIM_TT) s_P[h * SLIM_TT + lane] = pr;
        if (lane == 0) { s_alpha[h] = alpha; s_m[h] = m_new; s_l[h] = s_l[h] * alpha + ps; }
      }
      __syncthreads();
#pragma unroll
      for (int h = 0; h < HP; ++h) {
        if (h < H) {
          const float4* P4 = reinterpret_cast<const float4*>(s_P + h * SLIM_TT);
          float a = acc[h] * s_alpha[h];
#pragma unroll
          for (int i = 0; i < SLIM_TT / 4; ++i) {
            const float4 v = P4[i];
            a = fmaf(v.x, kv[4 * i], a); a = fmaf(v.y, kv[4 * i + 1], a);
            a = fmaf(v.z, kv[4 * i + 2], a); a = fmaf(v.w, kv[4 * i + 3], a);
          }
          acc[h] = a;
        }
      }
      __syncthreads();
    }
    if (col < d) {
#pragma unroll
      for (int h = 0; h < HP; ++h)
        if (h < H) p.part_u[((size_t)unit * H + h) * d + col] = acc[h];
    }
    if (blockIdx.x == 0 && tid < H) {
      p.part_m[(size_t)unit * H + tid] = s_m[tid];
      p.part_l[(size_t)unit * H + tid] = s_l[tid];
    }
    g = seg_end;
  }
}

template <int HP>
cudaError_t launch_accum(const SlimDecodeParams& p, const float* scores, cudaStream_t st) {
  const size_t smem = sizeof(float) * (HP * SLIM_TT + 3 * HP) + sizeof(int) * (p.batch + 1);
  fp4_accum_kernel<HP><<<dim3((p.d + THREADS - 1) / THREADS, p.workers), THREADS, smem, st>>>(p, scores);
  return cudaGetLastError();
}

}  // namespace

cudaError_t slim_launch_fp4_decode(const slim_ctx* ctx, const SlimDecodeParams& p, float* scores, cudaStream_t st) {
  const size_t smem = sizeof(float) * p.d + sizeof(int) * (p.batch + 1);
  if (smem > 48 * 1024) {
    cudaError_t e = slim_allow_smem((const void*)fp4_scores_kernel);
    if (e != cudaSuccess) return e;
  }
  fp4_scores_kernel<<<4 * ctx->num_sms, THREADS, smem, st>>>(p, scores);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return p.H <= 8 ? launch_accum<8>(p, scores, st) : p.H <= 32 ? launch_accum<32>(p, scores, st) : launch_accum<64>(p, scores, st);
}
