// Decode over a 4-bit K-cache on the tensor cores (d_k in {64, 96, 128}, an even number of heads up to 32, d a multiple of
// 256 up to 4096).
//
// The work is split as in the bf16 kernel (slim_tc.cu): a worker is a pair of CTAs, each with half of the columns and the
// heads that live in them; both walk the worker's tiles of 16 rows; U^T[d x heads] stays in tensor memory; a unit's
// (reference, l, U) goes to the common combine and projection.  What differs is that a tile has to be decoded:
//   load warp    a tile's code and scale rows, one bulk copy a row, into a ring (a quarter of bf16's bytes)
//   score warps  one head each.  A thread (g, j) = (lane / 4, lane % 4) has rows g and g + 8 and a quarter of the head's
//                rotation pairs.  Codes become float16 pairs (exact: code times scale has six significant bits), which
//                  - are stored as the tile that the tensor core reads (MN-major, 128-byte swizzle), and
//                  - are rotated by g and fed to m16n8k16 products with the query.  Key row t0 + g (+ 8) rotated by g meets the
//                    query turned back to t0 (column 0) or t0 + 8 (column 1), so the rotation factors of a thread are
//                    the same for every tile and live in registers; half of each is taken, so that nothing leaves float16.
//                Then p = 2^(s - m) in float16, into the P tile.
//   query warp   turns the queries of all heads back by 16 positions a tile (float32, re-seeded from the tables every 64
//                tiles) and lays the two columns down in the order the products read them
//   MMA thread   of the even CTA: U^T[256 columns x 32 heads] += K^T[256 x 16] P^T[16 x 32] a pair of 128-column chunks, each
//                CTA supplying its own 128 columns and its own 16 heads' P (cta_group::2), so no probabilities travel
// float16 P: the reference is the first tile's maximum plus 8 (log2 units), so p reaches up to 2^15 for scores 23 above that
// maximum and keeps 11 bits down to 2^-14; smaller ones lose bits against terms 2^6 their size.  A score further up flags
// the unit; flagged units are walked again at the end, with the largest score as reference (known by then).
#include <cuda.h>

#include "slim_fp4.cuh"
#include "slim_ptx.cuh"
#include "slim_sched.cuh"

using namespace slim_ptx;

namespace {

constexpr int MAX_ST = 4, MAX_PK = 8;    // float16 stages, stages of packed tiles
constexpr int NQ = 2;                    // stages of query columns
constexpr int RESEED = 64;
constexpr float BIAS = 8.f, XMAX = 15.f;

// How a thread's pairs lie: pieces of PE consecutive columns of the first half of the head, and the same of the second
template <int DK>
struct Lane {
  static constexpr int HALF = DK / 2, PE = DK == 96 ? 4 : 8, NP = HALF / (4 * PE), KS = DK / 16;
  static constexpr int SB = KS * 8 % 32 == 16 ? KS * 8 : KS * 8 + 16;      // bytes of a thread's query words, an odd multiple of 16
  __host__ __device__ static constexpr int col(int j, int x) { return DK == 128 ? 16 * j + 8 * x : PE * (j + 4 * x); }
};

struct Geom {
  int dsl, hl, nch;                      // columns, heads, 128-column chunks of a CTA
  int sets, nsw, nswl;                   // score-warp sets, warps of a set (one head each), launched score / epilogue warps
  int nst, npk;
  int stage, pk;                         // bytes of a float16 stage and of a packed one
  int pp, spw, cb;                       // packed row pitches (codes, scales), bytes of a row's codes
  int pitch, spitch;                     // of the cache
  int tmem_cols;
  int off_p, off_pk, off_q, off_bar, smem;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// eight codes -> four float16 pairs
__device__ __forceinline__ void decode8(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) { uint32_t d; asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d; asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c)); return d;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  uint32_t d; asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo)); return d;
}
__device__ __forceinline__ uint32_t half2_of(f32x2 v) {
  uint32_t d;
  asm("{\n\t.reg .f32 lo, hi;\n\tmov.b64 {lo, hi}, %1;\n\tcvt.rn.f16x2.f32 %0, hi, lo;\n\t}" : "=r"(d) : "l"(v));
  return d;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t a) { uint32_t v; asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint32_t lds_u16(uint32_t a) { uint32_t v; asm volatile("ld.shared.u16 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint32_t lds32(uint32_t a) { uint32_t v; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint2 lds64(uint32_t a) { uint2 v; asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a)); return v; }
__device__ __forceinline__ void sts64(uint32_t a, uint32_t x, uint32_t y) { asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(a), "r"(x), "r"(y) : "memory"); }
// 2^e that brings x (> 0, finite) into [1, 2); 1 for anything else
__device__ __forceinline__ float pow2_to_one(float x) {
  if (!(x > 0.f) || !(x <= 3.4e38f)) return 1.f;
  const int e = min(max(127 - ((__float_as_int(x) >> 23) & 255), -120), 120);
  return __int_as_float((e + 127) << 23);
}

template <int DK, bool ROPE, int MAXT>
__global__ void __launch_bounds__(MAXT, 1) fp4_tc_kernel(const SlimDecodeParams p, const Geom g, float* __restrict__ umax) {
  typedef Lane<DK> L;
  constexpr int HALF = L::HALF, PE = L::PE, NP = L::NP, KS = L::KS, SB = L::SB, HB = 8 * SB;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* sm = smem_raw + (base - raw);
  const uint32_t s_p = base + g.off_p, s_pk = base + g.off_pk, s_qb = base + g.off_q;
  const uint32_t bars = base + g.off_bar;
  const uint32_t b_pkf = bars, b_pke = b_pkf + 8 * MAX_PK, b_pf = b_pke + 8 * MAX_PK, b_ke = b_pf + 8 * MAX_ST;
  const uint32_t b_qf = b_ke + 8 * MAX_ST, b_qe = b_qf + 8 * NQ, b_uf = b_qe + 8 * NQ, b_ue = b_uf + 8, b_xm = b_ue + 8, b_xl = b_xm + 8;
  unsigned char* misc = sm + (b_xl + 8 - base);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(misc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(misc + 4);
  float* s_qs = reinterpret_cast<float*>(misc + 8);           // [2][16] what a unit's query columns were divided by
  float* s_xm = s_qs + 32;                                    // [16] reference, from the set that has a unit's first tile
  float* s_xl = s_xm + 16;                                    // [16] the other set's share of l
  float* s_xx = s_xl + 16;                                    // [16] and its largest score
  int* s_prefix = reinterpret_cast<int*>(s_xx + 16);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_ctarank();
  const int w = blockIdx.x / 2;
  const int w_load = g.nswl, w_mma = g.nswl + 1, w_query = g.nswl + 2;
  const int nepi = (g.nswl / 4) * 4;

  if (tid == 0) {
    for (int i = 0; i < MAX_PK; ++i) { mbar_init(b_pkf + 8 * i, 1); mbar_init(b_pke + 8 * i, g.nsw); }
    for (int i = 0; i < MAX_ST; ++i) { mbar_init(b_pf + 8 * i, 2 * g.nsw); mbar_init(b_ke + 8 * i, 1); }
    for (int i = 0; i < NQ; ++i) { mbar_init(b_qf + 8 * i, 1); mbar_init(b_qe + 8 * i, ROPE ? g.nsw : g.nsw * g.sets); }
    mbar_init(b_uf, 1);
    mbar_init(b_ue, 2 * nepi);
    mbar_init(b_xm, g.nsw);
    mbar_init(b_xl, g.nsw);
    *s_abort = 0;
    fence_mbar_init();
  }
  for (int i = tid; i < g.nst * 512 / 16; i += blockDim.x) sts128_zero(s_p + 16 * i);       // rows of heads that are not there
  fence_proxy_async_smem();
  if (warp == w_mma) tmem_alloc2(smem_u32(s_tmem), (uint32_t)g.tmem_cols);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  slim_pdl_wait();
  const SlimSched sc = slim_sched_build(p.lengths, p.batch, p.t_cap, p.workers, p.min_tiles, s_prefix, p.status, p.unit_cost);
  const bool in_range = sc.total_tiles > 0 && w < sc.workers_eff;
  const int g_begin = in_range ? slim_worker_start(sc, w) : 0;
  const int g_end = in_range ? slim_worker_start(sc, w + 1) : 0;

  // Where a role stands, over both sweeps: tiles (it) and units (uc) so far.
  int it = 0, uc = 0;
  bool ok = true;
  for (int sweep = 0; sweep < 2; ++sweep) {
    // units of this sweep: all, then those flagged in either CTA
    auto wanted = [&](int unit) { return sweep == 0 || (__ldcg(p.unit_flags + 2 * unit) | __ldcg(p.unit_flags + 2 * unit + 1)) != 0; };
    if (warp < g.nswl) {
      // =========================== score / epilogue warps ===========================
      const bool scorer = warp < g.nsw * g.sets;
      const int set = warp >= g.nsw ? 1 : 0, hd = warp - set * g.nsw;       // a set takes every g.sets-th tile; head within the CTA
      const int gr = lane >> 2, j = lane & 3;
      const int head = (int)rank * g.hl + hd;
      uint32_t cs[NP * PE / 2], sn[NP * PE / 2];                 // half of cos and sin of gr theta, the thread's pairs
      if (ROPE && scorer) {
#pragma unroll
        for (int x = 0; x < NP; ++x)
#pragma unroll
          for (int e = 0; e < PE / 2; ++e) {
            const float2 a = __ldg(p.rope_off + gr * HALF + L::col(j, x) + 2 * e), b = __ldg(p.rope_off + gr * HALF + L::col(j, x) + 2 * e + 1);
            cs[x * (PE / 2) + e] = half2_of(0.5f * a.x, 0.5f * b.x);
            sn[x * (PE / 2) + e] = half2_of(0.5f * a.y, 0.5f * b.y);
          }
      }
      // byte offsets of the thread's pieces: codes in a packed row, scales, place in the float16 tile
      const uint32_t c_off = (uint32_t)(gr * g.pp + (hd * DK + L::col(j, 0)) / 2);
      const int s_shift = (int)((rank * (g.dsl / FP4_GROUP)) & 15);
      const uint32_t s_off = (uint32_t)(16 * g.pp + gr * g.spw + s_shift);
      auto tile_off = [&](int half, int x) {
        const int c = hd * DK + half * HALF + L::col(j, x);
        return (uint32_t)((c >> 6) * 2048 + gr * 128 + ((((c & 63) >> 3) ^ gr) << 4) + (c & 7) * 2);
      };
      uint32_t qb[2 * KS];
#pragma unroll
      for (int x = 0; x < 2 * KS; ++x) qb[x] = 0u;
      float qs = 1.f;
      for (int gg = g_begin; gg < g_end && ok;) {
        const int b = slim_seq_of_tile(s_prefix, p.batch, gg);
        const int seg_end = min(g_end, s_prefix[b + 1]);
        const int tile0 = gg - s_prefix[b], ntile = seg_end - gg, unit = w + b;
        gg = seg_end;
        if (!wanted(unit)) continue;
        const int len = min(max(p.lengths[b], 0), p.t_cap);
        const int kt0 = g.sets == 1 ? 0 : ((set - it) & 1);          // this set's first tile of the unit
        const bool owner = kt0 == 0;
        float mref = 0.f, lsum = 0.f, rmax = -INFINITY;
        if (scorer) {
          if (!ROPE) {
            ok = mbar_wait<false>(b_qf + 8 * (uc & 1), (uc >> 1) & 1, s_abort, p.status);
            if (gr < 2) {
#pragma unroll
              for (int x = 0; x < KS / 2; ++x) {
                const uint4 v = lds128(s_qb + (uint32_t)((uc & 1) * g.hl * HB + hd * HB + (gr * 4 + j) * SB + 16 * x));
                qb[4 * x] = v.x; qb[4 * x + 1] = v.y; qb[4 * x + 2] = v.z; qb[4 * x + 3] = v.w;
              }
            }
            qs = s_qs[(uc & 1) * 16 + hd];
            __syncwarp();
            if (lane == 0) mbar_arrive(b_qe + 8 * (uc & 1));
          }
          for (int kt = kt0; kt < ntile && ok; kt += g.sets) {
            const int n = it + kt, st = n % g.nst, ps = n % g.npk;
            const int t0 = (tile0 + kt) * SLIM_TT;
            ok = mbar_wait<false>(b_pkf + 8 * ps, (n / g.npk) & 1, s_abort, p.status);
            if (ROPE) ok = mbar_wait<false>(b_qf + 8 * (n & 1), (n >> 1) & 1, s_abort, p.status) && ok;
            ok = mbar_wait<false>(b_ke + 8 * st, ((n / g.nst) & 1) ^ 1, s_abort, p.status) && ok;
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (ROPE) {
              if (gr < 2) {
#pragma unroll
                for (int x = 0; x < KS / 2; ++x) {
                  const uint4 v = lds128(s_qb + (uint32_t)((n & 1) * g.hl * HB + hd * HB + (gr * 4 + j) * SB + 16 * x));
                  qb[4 * x] = v.x; qb[4 * x + 1] = v.y; qb[4 * x + 2] = v.z; qb[4 * x + 3] = v.w;
                }
              }
              if (kt == kt0) qs = s_qs[(uc & 1) * 16 + hd];
            }
            const uint32_t pk = s_pk + (uint32_t)(ps * g.pk), kh = base + (uint32_t)(st * g.stage);
            // codes of rows gr and gr + 8: first and second half of the head
            uint32_t cw[2][2][NP];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                const uint32_t at = pk + c_off + (uint32_t)(r * 8 * g.pp + half * HALF / 2);
                if constexpr (DK == 128) {
                  const uint2 v = lds64(at);
                  cw[r][half][0] = v.x; cw[r][half][1] = v.y;
                } else if constexpr (DK == 64) {
                  cw[r][half][0] = lds32(at);
                } else {
#pragma unroll
                  for (int x = 0; x < NP; ++x) cw[r][half][x] = lds_u16(at + 8 * x);
                }
              }
            const bool in0 = t0 + gr < len, in1 = t0 + gr + 8 < len;
            float acc[2][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[0][i] = acc[1][i] = 0.f;
            uint32_t sc2[2][2];
#pragma unroll
            for (int x = 0; x < NP; ++x) {
              uint32_t k[2][2][4];                                   // [row][half][pair of columns]
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                const uint32_t to = kh + tile_off(half, x);
                uint32_t both[4];                                    // pieces of four columns: the two rows side by side
                if (PE == 4) decode8(cw[0][half][x] | (cw[1][half][x] << 16), both);
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                  if (x == 0 || DK == 96) {                          // (a thread's pieces of a half share a group elsewhere)
                    const uint32_t byte = lds_u8(pk + s_off + (uint32_t)(r * 8 * g.spw + (hd * DK + half * HALF + L::col(j, x)) / FP4_GROUP));
                    sc2[r][half] = (r ? in1 : in0) ? byte * 0x00800080u : 0u;       // rows behind the sequence become zeros
                  }
                  if (PE == 8) decode8(cw[r][half][x], k[r][half]);
                  else { k[r][half][0] = both[2 * r]; k[r][half][1] = both[2 * r + 1]; }
#pragma unroll
                  for (int e = 0; e < PE / 2; ++e) k[r][half][e] = hmul2(k[r][half][e], sc2[r][half]);
                  if (PE == 8) sts128(to + r * 1024, make_uint4(k[r][half][0], k[r][half][1], k[r][half][2], k[r][half][3]));
                  else sts64(to + r * 1024, k[r][half][0], k[r][half][1]);
                }
              }
#pragma unroll
              for (int e = 0; e < PE / 2; ++e) {
                const int i = x * (PE / 2) + e;
                uint32_t a0 = k[0][0][e], a1 = k[1][0][e], a2 = k[0][1][e], a3 = k[1][1][e];
                if (ROPE) {
                  const uint32_t c = cs[i], s = sn[i], ns = s ^ 0x80008000u;
                  const uint32_t r0 = hfma2(a2, s, hmul2(a0, c)), r2 = hfma2(a0, ns, hmul2(a2, c));
                  const uint32_t r1 = hfma2(a3, s, hmul2(a1, c)), r3 = hfma2(a1, ns, hmul2(a3, c));
                  a0 = r0; a1 = r1; a2 = r2; a3 = r3;
                }
                mma_f16(acc[i & 1], a0, a1, a2, a3, qb[2 * i], qb[2 * i + 1]);
              }
            }
            // column 0 for row gr, column 1 for row gr + 8: both with thread j = 0
            const float s0 = (acc[0][0] + acc[1][0]) * qs, s1 = (acc[0][3] + acc[1][3]) * qs;
            const bool v0 = in0 && j == 0, v1 = in1 && j == 0;
            if (kt == kt0) {
              if (sweep == 1) {
                mref = __ldcg(umax + (size_t)unit * p.H + head);
              } else if (owner) {
                float mx = fmaxf(v0 ? s0 : -INFINITY, v1 ? s1 : -INFINITY);
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                mx = __shfl_sync(0xffffffffu, mx, 0);
                mref = mx + BIAS;
                if (g.sets == 2) {
                  if (lane == 0) s_xm[hd] = mref;
                  __syncwarp();
                  if (lane == 0) mbar_arrive(b_xm);
                }
              } else {
                ok = mbar_wait<false>(b_xm, uc & 1, s_abort, p.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                mref = s_xm[hd];
              }
              if (!(mref > -INFINITY)) mref = 0.f;                   // nothing but NaN so far
            }
            if (v0) rmax = fmaxf(rmax, s0);
            if (v1) rmax = fmaxf(rmax, s1);
            float x0 = s0 - mref, x1 = s1 - mref;
            if (((v0 && x0 > XMAX) || (v1 && x1 > XMAX)) && sweep == 0) p.unit_flags[2 * unit + (int)rank] = 1;
            x0 = x0 > XMAX ? XMAX : x0;
            x1 = x1 > XMAX ? XMAX : x1;
            const __half p0 = __float2half_rn(v0 ? ex2_approx(x0) : 0.f), p1 = __float2half_rn(v1 ? ex2_approx(x1) : 0.f);
            if (j == 0) {
              lsum += __half2float(p0) + __half2float(p1);
              sts_u16(s_p + (uint32_t)(st * 512) + p_offset(hd, gr), __half_as_ushort(p0));
              sts_u16(s_p + (uint32_t)(st * 512) + p_offset(hd, gr + 8), __half_as_ushort(p1));
            }
            fence_proxy_async_smem();            // keys and probabilities -> tensor core
            __syncwarp();
            if (lane == 0) {
              mbar_arrive_cluster(mapa(b_pf + 8 * st, 0));
              mbar_arrive(b_pke + 8 * ps);
              if (ROPE) mbar_arrive(b_qe + 8 * (n & 1));
            }
          }
          if (!ok) break;
          // ---- (reference, l) and the largest score of the unit ----
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) {
            lsum += __shfl_xor_sync(0xffffffffu, lsum, o);
            rmax = fmaxf(rmax, __shfl_xor_sync(0xffffffffu, rmax, o));
          }
          if (g.sets == 2) {
            // The set without the unit's first tile waits for the reference before it hands its share back, whether it had a
            // tile or not, and the other waits for that share: neither barrier can complete its next phase before both
            // sets have seen this one, and neither slot is written before it has been read.
            if (owner) {
              if (sweep == 1 && lane == 0) mbar_arrive(b_xm);        // (no reference to hand over)
              ok = mbar_wait<false>(b_xl, uc & 1, s_abort, p.status);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
              lsum += s_xl[hd];
              rmax = fmaxf(rmax, s_xx[hd]);
            } else {
              ok = mbar_wait<false>(b_xm, uc & 1, s_abort, p.status);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
              if (lane == 0) {
                s_xl[hd] = lsum; s_xx[hd] = rmax;
                mbar_arrive(b_xl);
              }
              __syncwarp();
            }
          }
          if (owner && lane == 0) {
            p.part_m[(size_t)unit * p.H + head] = mref;
            p.part_l[(size_t)unit * p.H + head] = lsum;
            if (sweep == 0) umax[(size_t)unit * p.H + head] = rmax;
          }
        }
        if (warp < nepi) {
          // warp w drains TMEM lanes 32 (w & 3) .. + 31 of chunks w >> 2, ..: a column is a head, CTA 0's heads then CTA 1's
          ok = mbar_wait<false>(b_uf, uc & 1, s_abort, p.status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          const int q = warp & 3, cstep = nepi >> 2;
          float* dst = p.part_u + (size_t)unit * p.H * p.d + (size_t)rank * g.dsl + q * 32 + lane;
          for (int c = warp >> 2; c < g.nch; c += cstep) {
            uint32_t r[32];
            tmem_ld32(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(c * 32), r);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const int h = i < 16 ? i : g.hl + i - 16;
              if ((i & 15) < g.hl) dst[(size_t)h * p.d + c * 128] = __uint_as_float(r[i]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(mapa(b_ue, 0));
        }
        it += ntile;
        ++uc;
      }
    } else if (warp == w_load) {
      // =========================== loads ===========================
      if (sweep == 0 && g_end > g_begin) {
        // No score warp can raise a flag before it has seen a tile that is loaded behind this.
        const int b_lo = slim_seq_of_tile(s_prefix, p.batch, g_begin), b_hi = slim_seq_of_tile(s_prefix, p.batch, g_end - 1);
        for (int b = b_lo + lane; b <= b_hi; b += 32) p.unit_flags[2 * (w + b) + (int)rank] = 0;
        __threadfence_block();
        __syncwarp();
      }
      const unsigned char* codes = reinterpret_cast<const unsigned char*>(p.k) + (size_t)rank * g.cb;
      const int s_lo = ((int)rank * (g.dsl / FP4_GROUP)) & ~15;
      const int s_bytes = (((int)(rank + 1) * (g.dsl / FP4_GROUP) + 15) & ~15) - s_lo;
      for (int gg = g_begin; gg < g_end && ok;) {
        const int b = slim_seq_of_tile(s_prefix, p.batch, gg);
        const int seg_end = min(g_end, s_prefix[b + 1]);
        const int tile0 = gg - s_prefix[b], ntile = seg_end - gg, unit = w + b;
        gg = seg_end;
        if (!wanted(unit)) continue;
        const int len = min(max(p.lengths[b], 0), p.t_cap);
        for (int kt = 0; kt < ntile; ++kt, ++it) {
          const int ps = it % g.npk, t0 = (tile0 + kt) * SLIM_TT;
          ok = mbar_wait<false>(b_pke + 8 * ps, ((it / g.npk) & 1) ^ 1, s_abort, p.status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const int rows = min(SLIM_TT, len - t0);                   // (rows behind the sequence may lie behind the storage)
          if (lane == 0) mbar_arrive_expect_tx(b_pkf + 8 * ps, (uint32_t)(rows * (g.cb + s_bytes)));
          const long long row = slim_cache_row(p, b, t0) + (lane & 15);
          __syncwarp();
          const uint32_t dst = s_pk + (uint32_t)(ps * g.pk);
          if ((lane & 15) < rows) {
            if (lane < 16) bulk_load(dst + (uint32_t)(lane * g.pp), codes + (size_t)row * g.pitch, (uint32_t)g.cb, b_pkf + 8 * ps);
            else bulk_load(dst + (uint32_t)(16 * g.pp + (lane & 15) * g.spw), p.k_sc4 + (size_t)row * g.spitch + s_lo, (uint32_t)s_bytes, b_pkf + 8 * ps);
          }
        }
        ++uc;
      }
      if (!ok && lane == 0) {
        // gave up: let the copies that were issued land before the CTA goes away
        const unsigned long long t = globaltimer();
        for (int n = max(0, it - g.npk); n < it; ++n)
          while (!mbar_try_wait(b_pkf + 8 * (n % g.npk), (n / g.npk) & 1) && globaltimer() - t < SLIM_WAIT_NS) {}
      }
      __syncwarp();
    } else if (warp == w_mma) {
      // =========================== MMA issuer (even CTA) ===========================
      if (lane == 0) {
        constexpr uint32_t IDESC = (1u << 4) | (1u << 15) | ((32u >> 3) << 17) | ((256u >> 4) << 24);      // float16, A MN-major, M = 256, N = 32
        const uint64_t ad = desc_a(base), bd = desc_b(s_p);
        const uint32_t a_lo = (uint32_t)ad, a_hi = (uint32_t)(ad >> 32), b_lo = (uint32_t)bd, b_hi = (uint32_t)(bd >> 32);
        for (int gg = g_begin; gg < g_end && ok;) {
          const int b = slim_seq_of_tile(s_prefix, p.batch, gg);
          const int seg_end = min(g_end, s_prefix[b + 1]);
          const int ntile = seg_end - gg, unit = w + b;
          gg = seg_end;
          if (!wanted(unit)) continue;
          if (rank == 0) {
            for (int kt = 0; kt < ntile; ++kt) {
              const int n = it + kt, st = n % g.nst;
              ok = mbar_wait<true>(b_pf + 8 * st, (n / g.nst) & 1, s_abort, p.status);
              if (ok && kt == 0 && uc > 0) ok = mbar_wait<true>(b_ue, (uc - 1) & 1, s_abort, p.status);
              if (!ok) break;
              fence_proxy_async_smem();
              tc_fence_after();
              uint32_t al = a_lo + (uint32_t)((st * g.stage) >> 4), dcol = tmem;
              const uint32_t bl = b_lo + (uint32_t)(st * (512 >> 4));
              for (int c = 0; c < g.nch; ++c, al += 4096u >> 4, dcol += 32u) umma2_bf16_words(dcol, al, a_hi, bl, b_hi, IDESC, kt > 0 ? 1u : 0u);
              umma2_commit_pair(b_ke + 8 * st);
            }
            if (ok) umma2_commit_pair(b_uf);
          }
          it += ntile;
          ++uc;
        }
        // the last commit's arrival must not find this CTA gone
        if (ok && it > 0) ok = mbar_wait<false>(b_ke + 8 * ((it - 1) % g.nst), ((it - 1) / g.nst) & 1, s_abort, p.status);
      }
      __syncwarp();
    } else if (warp == w_query) {
      // =========================== query columns ===========================
      // lane l: pairs 2 l, 2 l + 1 of every head
      const bool live = lane < HALF / 2;
      int jj, xx;                                                    // the thread and step that read them
      if (DK == 128) { jj = lane / 8; xx = lane % 8; }
      else if (DK == 64) { jj = (lane / 4) & 3; xx = lane % 4; }
      else { jj = (lane >> 1) & 3; xx = 2 * (lane >> 3) + (lane & 1); }
      const uint32_t at = s_qb + (uint32_t)(jj * SB + xx * 8);
      f32x2 c16 = 0, s16 = 0, n16 = 0, c8 = 0, s8 = 0, n8 = 0;       // cos and sin of 16 theta and of 8 theta
      if (ROPE && live) {
        const float2 a = p.rope_base[HALF + 2 * lane], b = p.rope_base[HALF + 2 * lane + 1];
        const float2 c = p.rope_off[8 * HALF + 2 * lane], d = p.rope_off[8 * HALF + 2 * lane + 1];
        c16 = pack2(a.x, b.x); s16 = pack2(a.y, b.y); n16 = pack2(-a.y, -b.y);
        c8 = pack2(c.x, d.x); s8 = pack2(c.y, d.y); n8 = pack2(-c.y, -d.y);
      }
      const uint32_t* Q = reinterpret_cast<const uint32_t*>(p.q);
      f32x2 q1[16], q2[16];
      for (int gg = g_begin; gg < g_end && ok;) {
        const int b = slim_seq_of_tile(s_prefix, p.batch, gg);
        const int seg_end = min(g_end, s_prefix[b + 1]);
        const int tile0 = gg - s_prefix[b], ntile = seg_end - gg, unit = w + b;
        gg = seg_end;
        if (!wanted(unit)) continue;
        const int len = min(max(p.lengths[b], 0), p.t_cap);
        // the queries at position pos, divided by a power of two a head; `say`: also leave that for the score warps
        auto seed = [&](int pos, bool say) {
          f32x2 c = pack2(1.f, 1.f), s = pack2(0.f, 0.f), ns = s;
          if (ROPE && live) {
            const float2 ba = __ldg(p.rope_base + (size_t)(pos / SLIM_TT) * HALF + 2 * lane), bb = __ldg(p.rope_base + (size_t)(pos / SLIM_TT) * HALF + 2 * lane + 1);
            const float2 oa = __ldg(p.rope_off + (pos % SLIM_TT) * HALF + 2 * lane), ob = __ldg(p.rope_off + (pos % SLIM_TT) * HALF + 2 * lane + 1);
            const float sa = ba.y * oa.x + ba.x * oa.y, sb = bb.y * ob.x + bb.x * ob.y;
            c = pack2(ba.x * oa.x - ba.y * oa.y, bb.x * ob.x - bb.y * ob.y);
            s = pack2(sa, sb); ns = pack2(-sa, -sb);
          }
#pragma unroll
          for (int h = 0; h < 16; ++h) {
            if (h >= g.hl) break;
            const size_t qi = (((size_t)b * p.d + (size_t)((int)rank * g.hl + h) * DK) >> 1) + lane;
            const f32x2 u = live ? unpack2(__ldg(Q + qi)) : 0, v = live ? unpack2(__ldg(Q + qi + HALF / 2)) : 0;
            float m0, m1, m2, m3;
            asm("mov.b64 {%0, %1}, %2;" : "=f"(m0), "=f"(m1) : "l"(u));
            asm("mov.b64 {%0, %1}, %2;" : "=f"(m2), "=f"(m3) : "l"(v));
            float mx = fmaxf(fmaxf(fabsf(m0), fabsf(m1)), fmaxf(fabsf(m2), fabsf(m3)));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float up = pow2_to_one(mx);
            const f32x2 f = pack2(up, up);
            const f32x2 x = mul2(u, f), y = mul2(v, f);
            q1[h] = fma2(y, s, mul2(x, c));
            q2[h] = fma2(x, ns, mul2(y, c));
            if (say && lane == 0) s_qs[(uc & 1) * 16 + h] = (ROPE ? 2.f : 1.f) * p.qscale / up;      // (the factors on the keys are halved)
          }
        };
        auto lay = [&](int stage) {
#pragma unroll
          for (int h = 0; h < 16; ++h) {
            if (h >= g.hl) break;
            const uint32_t to = at + (uint32_t)((stage * g.hl + h) * HB);
            if (live) {
              sts64(to, half2_of(q1[h]), half2_of(q2[h]));
              // turned back by 8 more: column 1
              if (ROPE) sts64(to + 4 * SB, half2_of(fma2(q2[h], n8, mul2(q1[h], c8))), half2_of(fma2(q1[h], s8, mul2(q2[h], c8))));
              else sts64(to + 4 * SB, half2_of(q1[h]), half2_of(q2[h]));
            }
            if (ROPE) {
              const f32x2 a = fma2(q2[h], n16, mul2(q1[h], c16));
              q2[h] = fma2(q1[h], s16, mul2(q2[h], c16));
              q1[h] = a;
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(b_qf + 8 * stage);
        };
        if (!ROPE) {
          ok = mbar_wait<false>(b_qe + 8 * (uc & 1), ((uc >> 1) & 1) ^ 1, s_abort, p.status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          seed(0, true);
          lay(uc & 1);
          it += ntile;
        } else {
          for (int kt = 0; kt < ntile; ++kt, ++it) {
            ok = mbar_wait<false>(b_qe + 8 * (it & 1), ((it >> 1) & 1) ^ 1, s_abort, p.status);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            // q(len - 1) against keys turned by t - t0: the query at len - 1 - t0 (not negative: t0 < len)
            if (kt % RESEED == 0) seed(len - 1 - (tile0 + kt) * SLIM_TT, kt == 0);
            lay(it & 1);
          }
          if (!ok) break;
        }
        ++uc;
      }
      __syncwarp();
    }
    if (sweep == 0) {
      // units that a score ran away in: known to both CTAs behind this
      ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
      it = __shfl_sync(0xffffffffu, it, 0);
      uc = __shfl_sync(0xffffffffu, uc, 0);
      __threadfence();
      __syncthreads();
      cluster_sync_all();
      bool any = false;
      if (g_end > g_begin) {
        const int b_lo = slim_seq_of_tile(s_prefix, p.batch, g_begin), b_hi = slim_seq_of_tile(s_prefix, p.batch, g_end - 1);
        for (int b = b_lo; b <= b_hi; ++b) any |= (__ldcg(p.unit_flags + 2 * (w + b)) | __ldcg(p.unit_flags + 2 * (w + b) + 1)) != 0;
      }
      if (!any) break;
    }
  }
  slim_pdl_trigger();
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == w_mma) {
    tc_fence_after();
    tmem_dealloc2(tmem, (uint32_t)g.tmem_cols);
  }
}

constexpr int SMEM_LIMIT = 227 * 1024;

template <int DK>
int query_bytes(int hl) { return NQ * hl * 8 * Lane<DK>::SB; }

// false: the shape does not fit
bool make_geom(int d, int H, int d_k, int batch, Geom& g) {
  if ((d_k != 64 && d_k != 96 && d_k != 128) || (H & 1) || H < 2 || H > 32 || d % 256 || d > 4096) return false;
  g.dsl = d / 2; g.hl = H / 2; g.nch = g.dsl / 128;
  g.nsw = g.hl;
  g.sets = 2 * g.nsw <= 20 ? 2 : 1;
  g.nswl = g.nsw * g.sets < 4 ? 4 : g.nsw * g.sets;
  g.stage = 32 * g.dsl;
  g.cb = g.dsl / 2;
  const int want = d_k == 128 ? 32 : 16;                       // rows of a warp's reads side by side in the banks
  g.pp = g.cb;
  while (g.pp % 128 != want) g.pp += 16;
  g.pitch = slim_fp4_code_pitch(d); g.spitch = slim_fp4_scale_pitch(d);
  const int per = g.dsl / FP4_GROUP, lo0 = 0, hi0 = (per + 15) & ~15, lo1 = per & ~15, hi1 = (2 * per + 15) & ~15;
  g.spw = hi0 - lo0 > hi1 - lo1 ? hi0 - lo0 : hi1 - lo1;
  g.pk = 16 * (g.pp + g.spw);
  int cols = 32;
  while (cols < 32 * g.nch) cols <<= 1;
  g.tmem_cols = cols;
  const int qbytes = d_k == 128 ? query_bytes<128>(g.hl) : d_k == 96 ? query_bytes<96>(g.hl) : query_bytes<64>(g.hl);
  const int fixed = 1024 + qbytes + 8 * (2 * MAX_PK + 2 * MAX_ST + 2 * NQ + 4) + 8 + 4 * (32 + 48) + 4 * (batch + 1) + 64;
  // two float16 stages at least; more of them, and of packed ones, while they fit
  g.nst = 2; g.npk = 2;
  auto total = [&](int st, int pk) { return fixed + st * (g.stage + 512) + pk * g.pk; };
  if (total(2, 2) > SMEM_LIMIT) return false;
  while (g.npk < 4 && total(g.nst, g.npk + 1) <= SMEM_LIMIT) ++g.npk;
  while (g.nst + 2 <= MAX_ST && total(g.nst + 2, g.npk) <= SMEM_LIMIT) g.nst += 2;
  while (g.npk < MAX_PK && total(g.nst, g.npk + 1) <= SMEM_LIMIT) ++g.npk;
  g.off_p = g.nst * g.stage;
  g.off_pk = g.off_p + g.nst * 512;
  g.off_q = g.off_pk + g.npk * g.pk;
  g.off_bar = g.off_q + qbytes;
  g.smem = total(g.nst, g.npk);
  if (g.smem < 120 * 1024) g.smem = 120 * 1024;                // one CTA an SM: tensor memory is not shared
  return true;
}

typedef void (*kernel_t)(const SlimDecodeParams, const Geom, float*);
template <int DK, bool ROPE>
kernel_t pick_threads(int threads) { return threads <= 640 ? fp4_tc_kernel<DK, ROPE, 640> : fp4_tc_kernel<DK, ROPE, 768>; }
kernel_t pick(int d_k, bool rope, int threads) {
  if (d_k == 64) return rope ? pick_threads<64, true>(threads) : pick_threads<64, false>(threads);
  if (d_k == 96) return rope ? pick_threads<96, true>(threads) : pick_threads<96, false>(threads);
  return rope ? pick_threads<128, true>(threads) : pick_threads<128, false>(threads);
}

int threads_of(const Geom& g) { return 32 * (g.nswl + 3); }

}  // namespace

int slim_fp4_tc_workers(const slim_ctx* ctx) {
  Geom g;
  if (!make_geom(ctx->d, ctx->H, ctx->d_k, SLIM_MAX_BATCH, g)) return 0;
  kernel_t kern = pick(ctx->d_k, ctx->rope_theta != 0.0, threads_of(g));
  if (cudaFuncSetAttribute((const void*)kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_LIMIT) != cudaSuccess) { cudaGetLastError(); return 0; }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * (ctx->num_sms / 2));
  cfg.blockDim = dim3(threads_of(g));
  cfg.dynamicSmemBytes = g.smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, (const void*)kern, &cfg) != cudaSuccess) { cudaGetLastError(); return 0; }
  return n < ctx->num_sms / 2 ? n : ctx->num_sms / 2;
}

cudaError_t slim_launch_fp4_tc(const slim_ctx* ctx, const SlimDecodeParams& p, float* umax, cudaStream_t st) {
  Geom g;
  if (!make_geom(ctx->d, ctx->H, ctx->d_k, p.batch, g)) return cudaErrorNotSupported;
  kernel_t kern = pick(ctx->d_k, ctx->rope_theta != 0.0, threads_of(g));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * p.workers);
  cfg.blockDim = dim3(threads_of(g));
  cfg.dynamicSmemBytes = g.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, p, g, umax);
}
