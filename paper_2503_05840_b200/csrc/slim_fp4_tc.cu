// Decode over a 4-bit K-cache on the tensor cores (d_k in {64, 96, 128}, an even number of heads up to 32, d a multiple of
// 256 up to 4096).
//
// The work is split as in the bf16 kernel (slim_tc.cu): a worker is a pair of CTAs, each with half of the columns and the
// heads that live in them; both walk the worker's tiles of 16 rows; U^T[d x heads] stays in tensor memory; a unit's
// (reference, l, U) goes to the common combine and projection.  What differs is that a tile has to be decoded:
//   load thread  a tile's codes and scales, one TMA load each, into a ring (a quarter of bf16's bytes)
//   score warps  one or two heads each.  A thread (g, j) = (lane / 4, lane % 4) has rows g and g + 8 and a quarter of the
//                head's rotation pairs.  Codes become float16 pairs (exact: code times scale has six significant bits), which
//                  - are stored as the tile that the tensor core reads (MN-major, 128-byte swizzle), and
//                  - are rotated by g and fed to m16n8k16 products with the query.  Key row t0 + g (+ 8) rotated by g meets the
//                    query turned back to t0 (column 0) or t0 + 8 (column 1), so the rotation factors of a thread are
//                    the same for every tile and live in registers; half of each is taken, so that nothing leaves float16.
//                The warp turns its heads' queries back by a tile (float32, re-seeded from the tables every 64 tiles) behind each
//                tile and lays the two columns down in the order the products read them.
//                Then p = 2^(s - m) in float16, into the P tile.
//   MMA thread   of the even CTA: U^T[256 columns x 32 heads] += K^T[256 x 16] P^T[16 x 32] a pair of 128-column chunks, each
//                CTA supplying its own 128 columns and its own 16 heads' P (cta_group::2), so no probabilities travel; the odd
//                CTA's passes on that its tile is complete
// float16 P keeps its 11 bits from 2^-14 up to 2^15, so the reference m of a unit has to leave room on both sides.  m is the mean of
// the first tile's scores plus 10 (log2 units), or that tile's maximum less 11 where that is more.  So scores may come out 25 above
// an ordinary first tile's mean, and 25 below a dominant key in it (the first token of a context often is one).  A unit is flagged by
// a score further up, or where what P's rounding below 2^-14 may lose (2^-25 a key, or the key) is more than 2^-16 of l.  Flagged
// units are walked again at the end, with the largest score, known by then, less 14 as reference.  For normal scores of up to 3
// nats' deviation, a first key 20 nats above them or not, one head of a unit in 10000 asks for that at most (3.5 nats: one in 500).
//
// Bound by the score warps.  A tile of 16 x 2048 keys takes a CTA 2650 clocks: a warp issues some 600 instructions for two
// heads (64 conversions of codes, 64 products with the scale, 128 of the rotation, 16 m16n8k16, 16 stores), two warps share a
// scheduler (registers: 168 a thread), the pipe that the float16 products need is half full, the issue slots 42 %; the tensor
// core works 560 clocks, HBM is at 18 %.  Measured: 131001 rows of 4096 in pages 187-196 us (285 MB, 1.5 TB/s), 16 contexts of
// 8-16k rows 288 us, 64 contexts of 1500 rows of 1280 54 us; the combine and the projection follow (32, 32 and 24 us).
// Tried without gain: fetching a tile's codes into registers behind the tile before (four warps' registers lent to the
// score warps, 304 -> 338 us), one head a warp and 16 warps (351 -> 455 us at the time).
#include <cuda.h>
#include <cstring>

#include "slim_fp4.cuh"
#include "slim_ptx.cuh"
#include "slim_sched.cuh"

using namespace slim_ptx;

namespace {

constexpr int MAX_ST = 4, MAX_PK = 8;    // float16 stages, stages of packed tiles
constexpr int RESEED = 64;
constexpr float XMAX = 15.f, XMIN = -14.f;            // log2 of the probabilities that float16 holds with all its bits
constexpr float ABOVE = 10.f, BELOW_MAX = 11.f, TOP = 14.f, STEP = 0x1p-25f, LOST = 0x1p-16f;

// How a thread's pairs lie: pieces of PE consecutive columns of the first half of the head, and the same of the second
template <int DK>
struct Lane {
  static constexpr int HALF = DK / 2, PE = DK == 96 ? 4 : 8, NP = HALF / (4 * PE), KS = DK / 16;
  static constexpr int SB = KS * 8 % 32 == 16 ? KS * 8 : KS * 8 + 16;      // bytes of a thread's query words, an odd multiple of 16
  __host__ __device__ static constexpr int col(int j, int x) { return DK == 128 ? 16 * j + 8 * x : PE * (j + 4 * x); }
};

struct Geom {
  int dsl, hl, nch, hpw;                 // columns, heads, 128-column chunks of a CTA; heads of a score warp
  int sets, nsw, nswl;                   // score-warp sets, warps of a set, launched score / epilogue warps
  int nst, npk;
  int stage, pk;                         // bytes of a float16 stage and of a packed one (codes in chunks of 64 bytes x 16 rows, scales)
  int win, s_lo[2], s_shift[2];          // bytes of a row's scales in a stage; where each CTA's begin, and its first among them
  int tmem_cols;
  int off_p, off_pk, off_q, off_bar, smem;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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
__device__ __forceinline__ uint32_t hneg2(uint32_t a) { uint32_t d; asm("neg.f16x2 %0, %1;" : "=r"(d) : "r"(a)); return d; }
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t sel) { uint32_t d; asm("prmt.b32 %0, %1, 0, %2;" : "=r"(d) : "r"(a), "r"(sel)); return d; }
__device__ __forceinline__ uint32_t lds_u8(uint32_t a) { uint32_t v; asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint32_t lds_u16(uint32_t a) { uint32_t v; asm volatile("ld.shared.u16 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint32_t lds32(uint32_t a) { uint32_t v; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint2 lds64(uint32_t a) { uint2 v; asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a)); return v; }
__device__ __forceinline__ void sts64(uint32_t a, uint32_t x, uint32_t y) { asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(a), "r"(x), "r"(y) : "memory"); }
// Arrival on a barrier of the other CTA behind what this CTA wrote to its own shared memory, and only that: a release of
// everything at cluster scope takes 1500 clocks a tile (16 contexts of 8-16k rows: the call 295 -> 310 us, 64 x 1500 rows of 1280
// 73 -> 98).
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_bar) {
  asm volatile("fence.release.sync_restrict::shared::cta.cluster;" ::: "memory");
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void umma2_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// 2^e that brings x (> 0, finite) into [1, 2); 1 for anything else
__device__ __forceinline__ float pow2_to_one(float x) {
  if (!(x > 0.f) || !(x <= 3.4e38f)) return 1.f;
  const int e = min(max(127 - ((__float_as_int(x) >> 23) & 255), -120), 120);
  return __int_as_float((e + 127) << 23);
}

// A ring's next stage and the phase of its barriers
struct Ring {
  int st;
  uint32_t ph;
  __device__ __forceinline__ void step(int by, int n) {
    st += by;
    if (st >= n) { st -= n; ph ^= 1u; }
  }
};

template <int DK, bool ROPE, int HPW, int MAXT>
__global__ void __launch_bounds__(MAXT, 1) fp4_tc_kernel(const __grid_constant__ CUtensorMap cmap, const __grid_constant__ CUtensorMap smap,
                                                         const SlimDecodeParams p, const Geom g, float* __restrict__ umax) {
  typedef Lane<DK> L;
  constexpr int HALF = L::HALF, PE = L::PE, NP = L::NP, KS = L::KS, SB = L::SB, HB = 8 * SB;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* sm = smem_raw + (base - raw);
  const uint32_t s_p = base + g.off_p, s_pk = base + g.off_pk, s_q = base + g.off_q;
  const uint32_t bars = base + g.off_bar;
  const uint32_t b_pkf = bars, b_pke = b_pkf + 8 * MAX_PK, b_pf = b_pke + 8 * MAX_PK, b_px = b_pf + 8 * MAX_ST, b_ke = b_px + 8 * MAX_ST;
  const uint32_t b_uf = b_ke + 8 * MAX_ST, b_ue = b_uf + 8, b_xm = b_ue + 8, b_xl = b_xm + 8;
  unsigned char* misc = sm + (b_xl + 8 - base);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(misc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(misc + 4);
  float* s_xm = reinterpret_cast<float*>(misc + 8);           // [16] reference, from the set that has a unit's first tile
  float* s_xl = s_xm + 16;                                    // [16] the other set's share of l
  float* s_xx = s_xl + 16;                                    // [16] its largest score
  float* s_xs = s_xx + 16;                                    // [16] and what it may have lost
  int* s_prefix = reinterpret_cast<int*>(s_xs + 16);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_ctarank();
  const int w = blockIdx.x / 2;
  const int w_load = g.nswl, w_mma = g.nswl + 1;
  const int nepi = (g.nswl / 4) * 4;

  if (tid == 0) {
    prefetch_tensormap(&cmap); prefetch_tensormap(&smap);
    for (int i = 0; i < MAX_PK; ++i) { mbar_init(b_pkf + 8 * i, 1); mbar_init(b_pke + 8 * i, g.nsw); }
    for (int i = 0; i < MAX_ST; ++i) { mbar_init(b_pf + 8 * i, g.nsw); mbar_init(b_px + 8 * i, 1); mbar_init(b_ke + 8 * i, 1); }
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
  const bool scorer = warp < g.nsw * g.sets;
  const int gr = lane >> 2, j = lane & 3;
  // Rotation factors, the same for every tile: half of cos and sin of gr theta for the thread's pairs (keys), cos and sin of a
  // set's step and of 8 theta for pairs 2 lane, 2 lane + 1 (queries).  No kernel before this one writes the tables.
  uint32_t cs[NP * PE / 2], sn[NP * PE / 2];
  f32x2 cst = 0, sst = 0, nst = 0, c8 = 0, s8 = 0, n8 = 0;
  if (ROPE && scorer) {
#pragma unroll
    for (int x = 0; x < NP; ++x)
#pragma unroll
      for (int e = 0; e < PE / 2; ++e) {
        const float2 a = __ldg(p.rope_off + gr * HALF + L::col(j, x) + 2 * e), b = __ldg(p.rope_off + gr * HALF + L::col(j, x) + 2 * e + 1);
        cs[x * (PE / 2) + e] = half2_of(0.5f * a.x, 0.5f * b.x);
        sn[x * (PE / 2) + e] = half2_of(0.5f * a.y, 0.5f * b.y);
      }
    if (lane < HALF / 2) {
      const float2 a = __ldg(p.rope_base + g.sets * HALF + 2 * lane), b = __ldg(p.rope_base + g.sets * HALF + 2 * lane + 1);
      const float2 c = __ldg(p.rope_off + 8 * HALF + 2 * lane), d = __ldg(p.rope_off + 8 * HALF + 2 * lane + 1);
      cst = pack2(a.x, b.x); sst = pack2(a.y, b.y); nst = pack2(-a.y, -b.y);
      c8 = pack2(c.x, d.x); s8 = pack2(c.y, d.y); n8 = pack2(-c.y, -d.y);
    }
  }
  slim_pdl_wait();
  const SlimSched sc = slim_sched_build(p.lengths, p.batch, p.t_cap, p.workers, p.min_tiles, s_prefix, p.status, p.unit_cost);
  const bool in_range = sc.total_tiles > 0 && w < sc.workers_eff;
  const int g_begin = in_range ? slim_worker_start(sc, w) : 0;
  const int g_end = in_range ? slim_worker_start(sc, w + 1) : 0;

  // Where a role stands, over both sweeps: tiles (it) and units (uc) so far, the next stage of each ring.
  int it = 0, uc = 0;
  const int set = warp < g.nswl && warp >= g.nsw ? 1 : 0;      // score warps: a set takes every g.sets-th tile
  Ring rp = {set, 0u}, rk = {set, 0u};
  bool ok = true;
  for (int sweep = 0; sweep < 2; ++sweep) {
    // units of this sweep: all, then those flagged in either CTA
    auto wanted = [&](int unit) { return sweep == 0 || (__ldcg(p.unit_flags + 2 * unit) | __ldcg(p.unit_flags + 2 * unit + 1)) != 0; };
    if (warp < g.nswl) {
      // =========================== score / epilogue warps ===========================
      const int hd0 = (warp - set * g.nsw) * HPW;                            // the warp's first head within the CTA
      // Offsets of the thread's pieces for its first head (the others follow at fixed distances; d_k = 96 goes piece by piece):
      // codes (64-byte chunks of 16 rows, 64-byte swizzle), scales, float16 tile (64-column chunks of 16 rows, 128-byte swizzle)
      const int sw = (gr >> 1) & 3;
      auto code_off = [&](int hd, int half, int x) {
        const int o = hd * (DK / 2) + half * (HALF / 2) + L::col(j, x) / 2;
        return (uint32_t)((o >> 6) * 1024 + gr * 64 + ((((o >> 4) & 3) ^ sw) << 4) + (o & 15));
      };
      auto tile_off = [&](int hd, int half, int x) {
        const int c = hd * DK + half * HALF + L::col(j, x);
        return (uint32_t)((c >> 6) * 2048 + gr * 128 + ((((c & 63) >> 3) ^ gr) << 4) + (c & 7) * 2);
      };
      const int s_at = rank ? g.s_shift[1] : g.s_shift[0];
      auto scale_off = [&](int i) { return (uint32_t)(8 * g.dsl + ((s_at + i) >> 4) * 256 + gr * 16 + ((s_at + i) & 15)); };       // of the CTA's group i
      const uint32_t c0 = code_off(hd0, 0, 0), t0_off = tile_off(hd0, 0, 0);
      uint32_t sc_off[HPW];
#pragma unroll
      for (int u = 0; u < HPW; ++u) sc_off[u] = scale_off((hd0 + u) * (DK / FP4_GROUP));
      // byte of a head's scale word -> the low byte of both halves of a register: first half of the head, second half
      const uint32_t sel0 = DK == 128 ? 0x4040u + 0x0101u * (uint32_t)(j >> 1) : 0x4040u, sel1 = sel0 + (DK == 128 ? 0x0202u : 0x0101u);
      const uint32_t q_own = s_q + (uint32_t)((set * g.hl + hd0) * HB);      // the warp's query columns
      // A product's column depends on its own column of the query operand only, so all eight are put to use: columns 0, 3 (and 4, 7)
      // are the first (second) head's two, and what the others hold does not matter.  Thread (gr, j) then finds in its own
      // sums the score of row gr + 8 (j & 1) under head hd0 + (j >> 1), and no score has to move.
      const uint32_t q_rd = q_own + (uint32_t)((HPW == 2 ? gr >> 2 : 0) * HB + (((gr & 3) >> 1) * 4 + j) * SB);
      const int mine = HPW == 2 ? j >> 1 : 0, odd = j & 1;                   // the thread's head and row half
      const bool scores = HPW == 2 || j < 2, speaks = scores && gr == 0 && odd == 0;      // (one thread a head)
      const uint32_t p_off = (uint32_t)(((hd0 + mine) & 7) * 16 + ((hd0 + mine) >> 3) * 256 + odd * 128 + gr * 2);
      // Queries: lane l has pairs 2 l, 2 l + 1 of a head, for the thread and step that read them
      const bool live = lane < HALF / 2;
      int jj, xx;
      if (DK == 128) { jj = lane / 8; xx = lane % 8; }
      else if (DK == 64) { jj = (lane / 4) & 3; xx = lane % 4; }
      else { jj = (lane >> 1) & 3; xx = 2 * (lane >> 3) + (lane & 1); }
      const uint32_t q_wr = q_own + (uint32_t)(jj * SB + xx * 8);
      f32x2 q1[HPW], q2[HPW];
#pragma unroll
      for (int u = 0; u < HPW; ++u) q1[u] = q2[u] = 0;
      for (int gg = g_begin; gg < g_end && ok;) {
        const int b = slim_seq_of_tile(s_prefix, p.batch, gg);
        const int seg_end = min(g_end, s_prefix[b + 1]);
        const int tile0 = gg - s_prefix[b], ntile = seg_end - gg, unit = w + b;
        gg = seg_end;
        if (!wanted(unit)) continue;
        const int len = min(max(p.lengths[b], 0), p.t_cap);
        const int kt0 = g.sets == 1 ? 0 : ((set - it) & 1);          // this set's first tile of the unit
        const bool owner = kt0 == 0;
        float qs = 1.f, mref = 0.f, lsum = 0.f, lsub = 0.f, rmax = -INFINITY;    // of the thread's head
        // The warp's queries at position pos, divided by a power of two a head
        auto seed = [&](int pos) {
          f32x2 c = pack2(1.f, 1.f), s = pack2(0.f, 0.f), ns = s;
          if (ROPE && live) {
            const float2 ba = __ldg(p.rope_base + (size_t)(pos / SLIM_TT) * HALF + 2 * lane), bb = __ldg(p.rope_base + (size_t)(pos / SLIM_TT) * HALF + 2 * lane + 1);
            const float2 oa = __ldg(p.rope_off + (pos % SLIM_TT) * HALF + 2 * lane), ob = __ldg(p.rope_off + (pos % SLIM_TT) * HALF + 2 * lane + 1);
            const float sa = ba.y * oa.x + ba.x * oa.y, sb = bb.y * ob.x + bb.x * ob.y;
            c = pack2(ba.x * oa.x - ba.y * oa.y, bb.x * ob.x - bb.y * ob.y);
            s = pack2(sa, sb); ns = pack2(-sa, -sb);
          }
          const uint32_t* Q = reinterpret_cast<const uint32_t*>(p.q);
#pragma unroll
          for (int u = 0; u < HPW; ++u) {
            const size_t qi = (((size_t)b * p.d + (size_t)((int)rank * g.hl + hd0 + u) * DK) >> 1) + lane;
            const f32x2 x = live ? unpack2(__ldg(Q + qi)) : 0, y = live ? unpack2(__ldg(Q + qi + HALF / 2)) : 0;
            float m0, m1, m2, m3;
            asm("mov.b64 {%0, %1}, %2;" : "=f"(m0), "=f"(m1) : "l"(x));
            asm("mov.b64 {%0, %1}, %2;" : "=f"(m2), "=f"(m3) : "l"(y));
            float mx = fmaxf(fmaxf(fabsf(m0), fabsf(m1)), fmaxf(fabsf(m2), fabsf(m3)));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float up = pow2_to_one(mx);                        // the largest element of a head into [1, 2)
            const f32x2 f = pack2(up, up), xf = mul2(x, f), yf = mul2(y, f);
            q1[u] = ROPE ? fma2(yf, s, mul2(xf, c)) : xf;
            q2[u] = ROPE ? fma2(xf, ns, mul2(yf, c)) : yf;
            if (u == mine) qs = (ROPE ? 2.f : 1.f) * p.qscale / up;  // what turns sums into scores (the factors on the keys are halved)
          }
        };
        auto lay = [&]() {                                           // the two columns of the next tile; the queries a step back
#pragma unroll
          for (int u = 0; u < HPW; ++u) {
            if (live) {
              sts64(q_wr + u * HB, half2_of(q1[u]), half2_of(q2[u]));
              if (ROPE) sts64(q_wr + u * HB + 4 * SB, half2_of(fma2(q2[u], n8, mul2(q1[u], c8))), half2_of(fma2(q1[u], s8, mul2(q2[u], c8))));
              else sts64(q_wr + u * HB + 4 * SB, half2_of(q1[u]), half2_of(q2[u]));
            }
            if (ROPE) {
              const f32x2 x = fma2(q2[u], nst, mul2(q1[u], cst));
              q2[u] = fma2(q1[u], sst, mul2(q2[u], cst));
              q1[u] = x;
            }
          }
        };
        if (scorer) {
          int fresh = 0;                                             // tiles since the queries came from the tables
          if (kt0 < ntile) {
            // q(len - 1) against keys turned by t - t0: the query at len - 1 - t0 (not negative: t0 < len)
            seed(len - 1 - (tile0 + kt0) * SLIM_TT);
            lay();
          }
          for (int kt = kt0; kt < ntile && ok; kt += g.sets, rp.step(g.sets, g.npk), rk.step(g.sets, g.nst)) {
            const int t0 = (tile0 + kt) * SLIM_TT;
            const uint32_t pk = s_pk + (uint32_t)(rp.st * g.pk), kh = base + (uint32_t)(rk.st * g.stage);
            // the keys are there (even lanes look) and the float16 stage is free (odd lanes)
            ok = mbar_wait<false>(lane & 1 ? b_ke + 8 * rk.st : b_pkf + 8 * rp.st, lane & 1 ? rk.ph ^ 1u : rp.ph, s_abort, p.status);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            __syncwarp();                                              // the query columns are down
            const bool in0 = t0 + gr < len, in1 = t0 + gr + 8 < len;
            // codes and scales of rows gr and gr + 8, first and second half of the heads
            uint32_t cw[HPW][2][2][NP], sc[HPW][2][2][DK == 96 ? NP : 1], qb[2 * KS];
            if constexpr (DK != 96) {
              const uint32_t ca = pk + c0, cb = ca ^ (DK == 128 ? 32u : 16u);
#pragma unroll
              for (int u = 0; u < HPW; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                  if constexpr (DK == 128) {
                    const uint2 v = lds64(ca + u * 1024 + r * 512), y = lds64(cb + u * 1024 + r * 512);
                    cw[u][r][0][0] = v.x; cw[u][r][0][1] = v.y;
                    cw[u][r][1][0] = y.x; cw[u][r][1][1] = y.y;
                  } else {
                    // heads two by two in a chunk: the second 32 bytes further, across the swizzle (hd0 is even where HPW is 2)
                    cw[u][r][0][0] = lds32((u ? ca ^ 32u : ca) + r * 512);
                    cw[u][r][1][0] = lds32((u ? cb ^ 32u : cb) + r * 512);
                  }
                  const uint32_t at = pk + sc_off[u] + r * 128;
                  uint32_t word = DK == 128 ? lds32(at) : lds_u16(at);
                  word = (r ? in1 : in0) ? word : 0u;                  // rows behind the sequence become zeros
                  sc[u][r][0][0] = prmt(word, sel0) << 7;
                  sc[u][r][1][0] = prmt(word, sel1) << 7;
                }
            } else {
#pragma unroll
              for (int u = 0; u < HPW; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                  for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int x = 0; x < NP; ++x) {
                      cw[u][r][half][x] = lds_u16(pk + code_off(hd0 + u, half, x) + r * 512);
                      const uint32_t byte = lds_u8(pk + scale_off(((hd0 + u) * DK + half * HALF + L::col(j, x)) / FP4_GROUP) + r * 128);
                      sc[u][r][half][x] = (r ? in1 : in0) ? byte * 0x00800080u : 0u;
                    }
            }
#pragma unroll
            for (int x = 0; x < KS / 2; ++x) {
              const uint4 v = lds128(q_rd + 16 * x);
              qb[4 * x] = v.x; qb[4 * x + 1] = v.y; qb[4 * x + 2] = v.z; qb[4 * x + 3] = v.w;
            }
            if (ROPE) {
              __syncwarp();
              lay();                                                   // of the next tile
            }
            const uint32_t ta = kh + t0_off;
            float acc[HPW][2][4];
#pragma unroll
            for (int u = 0; u < HPW; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[u][0][i] = acc[u][1][i] = 0.f;
#pragma unroll
            for (int x = 0; x < NP; ++x) {
#pragma unroll
              for (int u = 0; u < HPW; ++u) {
                uint32_t k[2][2][4];                                   // [row][half][pair of columns]
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                  uint32_t to;
                  if (DK == 128) to = (x ? ta ^ 16u : ta) + u * 4096 + half * 2048;
                  else if (DK == 64) to = (half ? ta ^ 64u : ta) + u * 2048;
                  else to = kh + tile_off(hd0 + u, half, x);
                  uint32_t both[4];                                    // pieces of four columns: the two rows side by side
                  if (PE == 4) slim_fp4_decode8(cw[u][0][half][x] | (cw[u][1][half][x] << 16), both);
#pragma unroll
                  for (int r = 0; r < 2; ++r) {
                    if (PE == 8) slim_fp4_decode8(cw[u][r][half][x], k[r][half]);
                    else { k[r][half][0] = both[2 * r]; k[r][half][1] = both[2 * r + 1]; }
#pragma unroll
                    for (int e = 0; e < PE / 2; ++e) k[r][half][e] = hmul2(k[r][half][e], sc[u][r][half][DK == 96 ? x : 0]);
                    if (PE == 8) sts128(to + r * 1024, make_uint4(k[r][half][0], k[r][half][1], k[r][half][2], k[r][half][3]));
                    else sts64(to + r * 1024, k[r][half][0], k[r][half][1]);
                  }
                }
#pragma unroll
                for (int e = 0; e < PE / 2; ++e) {
                  const int i = x * (PE / 2) + e;
                  uint32_t a0 = k[0][0][e], a1 = k[1][0][e], a2 = k[0][1][e], a3 = k[1][1][e];
                  if (ROPE) {
                    const uint32_t cc = cs[i], ss = sn[i], ns = hneg2(ss);
                    const uint32_t r0 = hfma2(a2, ss, hmul2(a0, cc)), r2 = hfma2(a0, ns, hmul2(a2, cc));
                    const uint32_t r1 = hfma2(a3, ss, hmul2(a1, cc)), r3 = hfma2(a1, ns, hmul2(a3, cc));
                    a0 = r0; a1 = r1; a2 = r2; a3 = r3;
                  }
                  mma_f16(acc[u][i & 1], a0, a1, a2, a3, qb[2 * i], qb[2 * i + 1]);
                }
              }
            }
            float s;
            {
              const float e0 = acc[0][0][0] + acc[0][1][0], e1 = acc[0][0][3] + acc[0][1][3];
              s = odd ? e1 : e0;
              if (HPW == 2) {
                const float f0 = acc[HPW - 1][0][0] + acc[HPW - 1][1][0], f1 = acc[HPW - 1][0][3] + acc[HPW - 1][1][3];
                s = mine ? (odd ? f1 : f0) : s;
              }
              s *= qs;
            }
            const bool v = scores && (odd ? in1 : in0);
            if (kt == kt0) {
              if (sweep == 1) {
                if (scores) mref = __ldcg(umax + (size_t)unit * p.H + (int)rank * g.hl + hd0 + mine) - TOP;
              } else if (owner) {
                float mx = v ? s : -INFINITY, sum = v ? s : 0.f;
#pragma unroll
                for (int o = 1; o < 32; o = o == 1 ? 4 : 2 * o) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                if constexpr (ROPE || DK != 128) {
#pragma unroll
                  for (int o = 1; o < 32; o = o == 1 ? 4 : 2 * o) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                } else {
                  // (lane by lane where a tree costs registers: 16 contexts of 12000 rows, d_k 128 without rotation, 258 us instead of 266)
                  const float own = sum;
                  sum = 0.f;
#pragma unroll 1
                  for (int i = 0; i < SLIM_TT; ++i) sum += __shfl_sync(0xffffffffu, own, (i >> 1) * 4 + (lane & 2) + (i & 1));
                }
                mref = fmaxf(sum / (float)min(SLIM_TT, len - t0) + ABOVE, mx - BELOW_MAX);      // (a NaN leaves the maximum)
                if (g.sets == 2) {
                  if (speaks) s_xm[hd0 + mine] = mref;
                  __syncwarp();
                  if (lane == 0) mbar_arrive(b_xm);
                }
              } else {
                ok = mbar_wait<false>(b_xm, uc & 1, s_abort, p.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                mref = s_xm[hd0 + mine];
              }
              if (!(mref > -INFINITY)) mref = 0.f;                     // nothing but NaN so far
            }
            if (v) rmax = fmaxf(rmax, s);
            float xv = s - mref;
            if (v && xv > XMAX && sweep == 0) p.unit_flags[2 * unit + (int)rank] = 1;
            xv = xv > XMAX ? XMAX : xv;
            const float pf = v ? ex2_approx(xv) : 0.f;
            if (xv < XMIN) lsub += fminf(pf, STEP);
            const __half pv = __float2half_rn(pf);
            if (scores) {
              lsum += __half2float(pv);
              sts_u16(s_p + (uint32_t)(rk.st * 512) + p_off, __half_as_ushort(pv));
            }
            fence_proxy_async_smem();            // keys and probabilities -> tensor core
            __syncwarp();
            if (lane < 2) mbar_arrive(lane ? b_pke + 8 * rp.st : b_pf + 8 * rk.st);
            if (ROPE && ++fresh == RESEED) {                           // (what was laid down for the next tile is replaced)
              fresh = 0;
              if (kt + g.sets < ntile) {
                seed(len - 1 - (tile0 + kt + g.sets) * SLIM_TT);
                lay();
              }
            }
          }
          if (!ok) break;
          // ---- (reference, l) and the largest score of the unit ----
#pragma unroll
          for (int o = 1; o < 32; o = o == 1 ? 4 : 2 * o) {
            lsum += __shfl_xor_sync(0xffffffffu, lsum, o);
            lsub += __shfl_xor_sync(0xffffffffu, lsub, o);
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
              lsum += s_xl[hd0 + mine];
              lsub += s_xs[hd0 + mine];
              rmax = fmaxf(rmax, s_xx[hd0 + mine]);
            } else {
              ok = mbar_wait<false>(b_xm, uc & 1, s_abort, p.status);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
              if (speaks) { s_xl[hd0 + mine] = lsum; s_xs[hd0 + mine] = lsub; s_xx[hd0 + mine] = rmax; }
              __syncwarp();
              if (lane == 0) mbar_arrive(b_xl);
            }
          }
          if (owner && speaks) {
            const size_t at = (size_t)unit * p.H + (int)rank * g.hl + hd0 + mine;
            p.part_m[at] = mref;
            p.part_l[at] = lsum;
            if (sweep == 0) {
              umax[at] = rmax;
              if (lsub > LOST * lsum) p.unit_flags[2 * unit + (int)rank] = 1;
            }
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
      if (lane == 0) {
        if (sweep == 0) fence_proxy_async_global();                    // (the rows may be an earlier kernel's ordinary stores)
        const uint64_t once = l2_policy_evict_first();
        for (int gg = g_begin; gg < g_end && ok;) {
          const int b = slim_seq_of_tile(s_prefix, p.batch, gg);
          const int seg_end = min(g_end, s_prefix[b + 1]);
          const int tile0 = gg - s_prefix[b], ntile = seg_end - gg, unit = w + b;
          gg = seg_end;
          if (!wanted(unit)) continue;
          for (int kt = 0; kt < ntile; ++kt, ++it, rp.step(1, g.npk)) {
            ok = mbar_wait<false>(b_pke + 8 * rp.st, rp.ph ^ 1u, s_abort, p.status);
            if (!ok) break;
            const int row = (int)slim_cache_row(p, b, (tile0 + kt) * SLIM_TT);       // (rows behind the storage come as zeros)
            const uint32_t dst = s_pk + (uint32_t)(rp.st * g.pk), bar = b_pkf + 8 * rp.st;
            mbar_arrive_expect_tx(bar, (uint32_t)(8 * g.dsl + 16 * g.win));
            tma_load_3d_hint(dst, &cmap, bar, 0, row, (int)rank * (g.dsl / 128), once);
            tma_load_3d_hint(dst + 8 * g.dsl, &smap, bar, 0, row, (rank ? g.s_lo[1] : g.s_lo[0]) / 16, once);
          }
          ++uc;
        }
        if (!ok) {
          // gave up: let the loads that were issued land before the CTA goes away
          const unsigned long long t = globaltimer();
          for (int n = max(0, it - g.npk); n < it; ++n)
            while (!mbar_try_wait(b_pkf + 8 * (n % g.npk), (n / g.npk) & 1) && globaltimer() - t < SLIM_WAIT_NS) {}
        }
      }
      __syncwarp();
    } else if (warp == w_mma) {
      // =========================== MMA issuer (even CTA), messenger (odd CTA) ===========================
      // The warp stays together and one elected lane issues: the operands then live in uniform registers, and an instruction costs
      // 39 clocks instead of the 74 that a lone lane needed to feed it (16 chunks; the operand reads alone are 32).
      constexpr uint32_t IDESC = (1u << 4) | (1u << 15) | ((32u >> 3) << 17) | ((256u >> 4) << 24);      // float16, A MN-major, M = 256, N = 32
      const uint64_t a0 = desc_a(base), b0 = desc_b(s_p);
      for (int gg = g_begin; gg < g_end && ok;) {
        const int b = slim_seq_of_tile(s_prefix, p.batch, gg);
        const int seg_end = min(g_end, s_prefix[b + 1]);
        const int ntile = seg_end - gg, unit = w + b;
        gg = seg_end;
        if (!wanted(unit)) continue;
        for (int kt = 0; kt < ntile; ++kt, ++it, rk.step(1, g.nst)) {
          ok = mbar_wait<false>(b_pf + 8 * rk.st, rk.ph, s_abort, p.status);
          if (rank != 0) {
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (elect_one()) mbar_arrive_remote(mapa(b_px + 8 * rk.st, 0));
            continue;
          }
          ok = mbar_wait<true>(b_px + 8 * rk.st, rk.ph, s_abort, p.status) && ok;
          if (kt == 0 && uc > 0) ok = mbar_wait<true>(b_ue, (uc - 1) & 1, s_abort, p.status) && ok;
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            uint64_t ad = a0 + (uint64_t)((uint32_t)(rk.st * g.stage) >> 4);
            const uint64_t bd = b0 + (uint64_t)(rk.st * (512 >> 4));
            uint32_t dcol = tmem;
            const uint32_t acc = kt > 0 ? 1u : 0u;
#pragma unroll 4
            for (int c = 0; c < g.nch; ++c, ad += 4096u >> 4, dcol += 32u) umma2_f16(dcol, ad, bd, IDESC, acc);
            umma2_commit_pair(b_ke + 8 * rk.st);
            if (kt + 1 == ntile) umma2_commit_pair(b_uf);
          }
          __syncwarp();
        }
        ++uc;
      }
      // the last commit's arrival must not find this CTA gone
      if (ok && it > 0) ok = mbar_wait<false>(b_ke + 8 * ((it - 1) % g.nst), ((it - 1) / g.nst) & 1, s_abort, p.status);
      __syncwarp();
    }
    if (sweep == 0) {
      // units that a score ran away in: known to both CTAs behind this
      ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
      it = __shfl_sync(0xffffffffu, it, 0);
      uc = __shfl_sync(0xffffffffu, uc, 0);
      rp.st = __shfl_sync(0xffffffffu, rp.st, 0);
      rp.ph = __shfl_sync(0xffffffffu, rp.ph, 0);
      rk.st = __shfl_sync(0xffffffffu, rk.st, 0);
      rk.ph = __shfl_sync(0xffffffffu, rk.ph, 0);
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

int threads_of(const Geom& g) { return 32 * (g.nswl + 2); }

// false: the shape does not fit
bool make_geom(int d, int H, int d_k, int batch, Geom& g) {
  if ((d_k != 64 && d_k != 96 && d_k != 128) || (H & 1) || H < 2 || H > 32 || d % 256 || d > 4096) return false;
  g.dsl = d / 2; g.hl = H / 2; g.nch = g.dsl / 128;
  // Two heads a warp where their number is even: a tile's fixed steps are shared by them.  Up to ten heads the warps come in two
  // sets that take the tiles in turn, since a small tile is bound by its chain of steps (more do not leave a thread the
  // registers for it).  64 x 1500 rows of 1280: the call 89 us with one head a warp, 81 with two.
  g.hpw = g.hl % 2 == 0 ? 2 : 1;
  g.nsw = g.hl / g.hpw;
  g.sets = g.hl > 10 ? 1 : 2;
  g.nswl = g.nsw * g.sets < 4 ? 4 : g.nsw * g.sets;
  g.stage = 32 * g.dsl;
  const int per = g.dsl / FP4_GROUP;
  int hi[2];
  for (int r = 0; r < 2; ++r) {
    g.s_lo[r] = (r * per) & ~15;
    g.s_shift[r] = (r * per) & 15;
    hi[r] = ((r + 1) * per + 15) & ~15;
  }
  g.win = hi[0] > hi[1] - g.s_lo[1] ? hi[0] : hi[1] - g.s_lo[1];
  int cols = 32;
  while (cols < 32 * g.nch) cols <<= 1;
  g.tmem_cols = cols;
  g.pk = (8 * g.dsl + 16 * g.win + 1023) & ~1023;
  const int qbytes = g.sets * g.hl * 8 * (d_k == 128 ? Lane<128>::SB : d_k == 96 ? Lane<96>::SB : Lane<64>::SB);
  const int fixed = 1024 + qbytes + 8 * (2 * MAX_PK + 3 * MAX_ST + 4) + 8 + 4 * 64 + 4 * (batch + 1) + 64;
  // two float16 stages at least; more of them, and of packed ones, while they fit
  g.nst = 2; g.npk = 2;
  auto total = [&](int st, int pk) { return fixed + st * (g.stage + 512) + pk * g.pk; };
  if (total(2, 2) > SMEM_LIMIT) return false;
  while (g.npk < 4 && total(g.nst, g.npk + 1) <= SMEM_LIMIT) ++g.npk;
  while (g.nst + 2 <= MAX_ST && total(g.nst + 2, g.npk) <= SMEM_LIMIT) g.nst += 2;
  while (g.npk < MAX_PK && total(g.nst, g.npk + 1) <= SMEM_LIMIT) ++g.npk;
  g.off_pk = g.nst * g.stage;
  g.off_p = g.off_pk + g.npk * g.pk;
  g.off_q = g.off_p + g.nst * 512;
  g.off_bar = g.off_q + qbytes;
  g.smem = total(g.nst, g.npk);
  if (g.smem < 120 * 1024) g.smem = 120 * 1024;                // one CTA an SM: tensor memory is not shared
  return true;
}

typedef void (*kernel_t)(const CUtensorMap, const CUtensorMap, const SlimDecodeParams, const Geom, float*);
template <int DK, bool ROPE>
kernel_t pick_heads(const Geom& g) {
  return g.hpw == 2 ? fp4_tc_kernel<DK, ROPE, 2, 384> : fp4_tc_kernel<DK, ROPE, 1, 640>;      // (most warps: 10 and 18, and two)
}
kernel_t pick(int d_k, bool rope, const Geom& g) {
  if (d_k == 64) return rope ? pick_heads<64, true>(g) : pick_heads<64, false>(g);
  if (d_k == 96) return rope ? pick_heads<96, true>(g) : pick_heads<96, false>(g);
  return rope ? pick_heads<128, true>(g) : pick_heads<128, false>(g);
}

}  // namespace

int slim_fp4_tc_workers(const slim_ctx* ctx) {
  Geom g;
  if (!make_geom(ctx->d, ctx->H, ctx->d_k, SLIM_MAX_BATCH, g)) return 0;
  kernel_t kern = pick(ctx->d_k, ctx->rope_theta != 0.0, g);
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

cudaError_t slim_fp4_tc_make_tmaps(const slim_ctx* ctx, slim_cache* c) {
  c->has_tmap[0] = c->has_tmap[1] = 0;
  Geom g;
  if (!make_geom(ctx->d, ctx->H, ctx->d_k, SLIM_MAX_BATCH, g)) return cudaErrorNotSupported;
  const unsigned long long rows = (unsigned long long)c->total_rows, pitch = (unsigned long long)slim_fp4_code_pitch(ctx->d), spitch = (unsigned long long)slim_fp4_scale_pitch(ctx->d);
  {
    // codes: 64-byte chunks of the rows; a box is the chunks of a CTA's half, 16 rows
    const unsigned long long dims[3] = {32, rows, pitch / 64}, strides[2] = {pitch, 64};
    const unsigned int box[3] = {32, SLIM_TT, (unsigned int)(g.dsl / 128)};
    const cudaError_t e = slim_tmap_encode_3d(c->tmap[0], c->k, dims, strides, box, 64);
    if (e != cudaSuccess) return e;
    c->has_tmap[0] = 1;
  }
  // scales: 16-byte chunks, so that the eight rows of a warp's load lie in different banks
  const unsigned long long dims[3] = {8, rows, spitch / 16}, strides[2] = {spitch, 16};
  const unsigned int box[3] = {8, SLIM_TT, (unsigned int)(g.win / 16)};
  const cudaError_t e = slim_tmap_encode_3d(c->tmap[1], c->k_sc4, dims, strides, box, 0);
  if (e == cudaSuccess) c->has_tmap[1] = 1;
  return e;
}

cudaError_t slim_launch_fp4_tc(const slim_ctx* ctx, const slim_cache* c, const SlimDecodeParams& p, float* umax, cudaStream_t st) {
  Geom g;
  if (!make_geom(ctx->d, ctx->H, ctx->d_k, p.batch, g)) return cudaErrorNotSupported;
  kernel_t kern = pick(ctx->d_k, ctx->rope_theta != 0.0, g);
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
  CUtensorMap cmap, smap;
  memcpy(&cmap, c->tmap[0], sizeof(cmap));
  memcpy(&smap, c->tmap[1], sizeof(smap));
  return cudaLaunchKernelEx(&cfg, kern, cmap, smap, p, g, umax);
}
