// Tensor-core path of slim_tree_decode (bf16 caches, d % 64 == 0, d_k in {64, 96, 128}).
//
// One sequence of L rows and n tokens has R = H n rows of probabilities and a weighted sum of R x d numbers (32 MB at
// n = 64, d = 4096): it cannot stay on chip as the one-token kernel's does, and its products, 2 L R d, are H times
// those of the scores.  So the step is a chain of kernels around one large matrix product:
//   scores      P = 2^(s - ref) in bf16, [b][h n + i][t], and (ref, sum) per row and block of 128 keys
//   finish      the row's reference and 1 / l; the last, partial block of 64 cached rows and the drafted keys, zero-padded,
//               in a scratch tail, so that the product only meets whole blocks of 64 finite rows; the product's schedule
//   sum         U = P K / l on tcgen05, CTA pairs (cta_group::2), bf16
//   join        adds the parts of tiles whose keys were cut
//   out         o = U W_KV,h on tcgen05
#include <cfloat>
#include <cmath>
#include <cstdlib>

#include "slim_ptx.cuh"
#include "slim_sched.cuh"
#include "slim_tree.h"

using namespace slim_ptx;

namespace {

__device__ __forceinline__ float2 turn(const SlimDecodeParams& p, int pos, int j) {      // (cos, sin) of pos theta_j
  const float2 cb = __ldg(p.rope_base + (size_t)(pos / SLIM_TT) * p.half + j), co = __ldg(p.rope_off + (pos % SLIM_TT) * p.half + j);
  return make_float2(cb.x * co.x - cb.y * co.y, cb.y * co.x + cb.x * co.y);
}

// ------------------------------------------------------------------------------------------------ scores
// The blocks of 128 keys of all heads of all sequences (a row's last block is its drafted keys) are dealt out evenly, one
// CTA per SM.  A CTA goes through its (sequence, head) rows one after another; its groups of eight warps share the tables and
// take a row's blocks in turn, with barriers of their own, so that one computes while the others wait.  Warp w of a group has keys
// 16 w .. 16 w + 15 of a block, rows g and g + 8 of m16n8k16 float16 tiles in each thread, and the tokens as the tiles'
// columns; its key tile comes by TMA into a buffer of its own, which nobody else reads.
//   - The contraction runs over rotation pairs: step (pc, x) puts the low elements of pairs j, j + 1 into the k-slots 2 c,
//     2 c + 1 and the high ones into 2 c + 8, 2 c + 9 (c = lane % 4), j = chunk(c, pc) VW + 2 x.  So a thread reads both
//     halves of its pairs as VW contiguous elements and rotates in registers (packed float32) on the way into the
//     instruction.
//   - R_pos(t) = R_(128 block) R_o: keys are turned by their offset o < 128 in the block only, whose (cos, sin) are
//     the same for every block (a table of the context, in the order the lanes read it); the queries, turned to
//     their positions once, are turned back by the block's angle, 64 complex factors a block.
//   - float16 keeps 11 bits of the rotated values (bf16's 8 would cost as much accuracy as the rounding of P does, for a
//     product that is 1 / H of the step's) at twice tf32's rate.  Its range: queries are scaled by a power of two per
//     token; keys go in as they are, and a warp whose sums overflow (those of attended keys), or whose queries are so large
//     that the smallest float16 steps of a key would show, repeats its tile with every key scaled by a power of two of its own.
//   - P is written relative to a reference that is a multiple of 64, kept from block to block while the arguments
//     stay below reference + 60 (the reference itself beside keys so large that P K could overflow): nearly always the
//     same for all blocks of a row, so that the blocks need no common maximum; `finish` shifts the exponents of the others,
//     exactly.  Sums l are taken from the rounded P, so the weights of a row add up to one.
// No unit is full (4 x 12000 rows, 16 drafts: issue slots 53 %, shared memory 48 %, DRAM 48 %, tensor pipe 11 %): with the
// four warps a scheduler that 128 registers allow, a warp issues every 7.5 cycles and spends 1.6 of them on fixed latencies,
// 1.3 on shared memory, 0.8 on the math pipes, 0.65 at barriers, 0.4 on loads.  d = 4096, d_k = 128: 16 ragged sequences,
// 196 k rows, 16 drafts 0.41 ms (3.9 TB/s of keys); 131001 rows, 64 drafts 0.56 ms; 8 x 12000 rows with 1, 8, 16, 32, 64
// drafts 0.16, 0.17, 0.20, 0.28, 0.43 ms (4.9 TB/s at one draft).
// Blocks dealt to CTAs as they come, not to (sequence, head) CTAs, and loads by the warp that uses them: a CTA per row left
// SMs idle at its end, block-wide tiles made every warp wait for the slowest load.
constexpr int SC_KEYS = 128, SC_GROUP = 256;

template <int DK, int NT>
struct ScoreShape {
  static constexpr int HALF = DK / 2, VW = DK == 96 ? 4 : 8, NPC = HALF / (4 * VW), STEPS = HALF / 8, PER = STEPS * 32;
  // a thread's (cos, sin) live in registers where they fit beside the sums (up to 16 tokens), else in shared memory
  static constexpr bool CSR = NT <= 2, QHALF = NT > 4;                   // QHALF: queries as float16 pairs (room; a second rounding to 11 bits)
  static constexpr int GROUPS = 2, THREADS = GROUPS * SC_GROUP, WARPS = THREADS / 32;
  static constexpr int KT = 16 * DK * 2, KS = CSR ? 2 : 1;               // bytes of a warp's key tile, buffers
  static constexpr size_t KR = (size_t)WARPS * KS * KT, CS = CSR ? 0 : (size_t)SC_KEYS * HALF * 8, QF = (size_t)NT * PER * 8;
  static constexpr size_t QS = (size_t)8 * NT * HALF * (QHALF ? 4 : 8);
  static constexpr size_t SR = (size_t)8 * NT * 8, MX = (size_t)8 * NT * 4, WS = (size_t)8 * NT * 8 * 4;
  static constexpr size_t OWN = 2 * QF + SR + MX + 2 * WS;               // of a group
  static constexpr size_t SMEM = 1024 + KR + CS + QS + GROUPS * OWN + 8 * (WARPS * KS + 1) + 16;
};
// which VW pairs of a head lane c takes in turn pc; for d_k = 128 even and odd key rows then meet different banks
__host__ __device__ constexpr int chunk_of(int dk, int c, int pc) { return dk == 128 ? 2 * c + pc : c + 4 * pc; }
// where a thread's VW low (hl = 0) or high elements of key r lie in a warp's tile of 16 keys: two 64-column atoms with
// 128-byte swizzle, one of them, or plain rows
template <int DK>
__device__ __forceinline__ uint32_t tile_off(int r, int c, int pc, int hl) {
  if (DK == 128) return (uint32_t)(hl * 2048 + r * 128 + (((2 * c + pc) ^ (r & 7)) << 4));
  if (DK == 64) return (uint32_t)(r * 128 + (((c + 4 * hl) ^ (r & 7)) << 4));
  return (uint32_t)(r * 192 + hl * 96 + (c + 4 * pc) * 8);
}

template <int VW> struct KVec;
template <> struct KVec<8> { typedef uint4 type; };
template <> struct KVec<4> { typedef uint2 type; };
__device__ __forceinline__ uint32_t word(const uint4& v, int x) { return x == 0 ? v.x : x == 1 ? v.y : x == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word(const uint2& v, int x) { return x == 0 ? v.x : v.y; }
__device__ __forceinline__ uint32_t& word_ref(uint4& v, int x) { return x == 0 ? v.x : x == 1 ? v.y : x == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t& word_ref(uint2& v, int x) { return x == 0 ? v.x : v.y; }
__device__ __forceinline__ uint32_t half2_of(f32x2 v) {                   // (low, high) -> float16 pair
  uint32_t d;
  asm("{\n\t.reg .f32 lo, hi;\n\tmov.b64 {lo, hi}, %1;\n\tcvt.rn.f16x2.f32 %0, hi, lo;\n\t}" : "=r"(d) : "l"(v));
  return d;
}
__device__ __forceinline__ uint32_t bf162_of(float lo, float hi) { uint32_t d; asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo)); return d; }
// two values as bf16 pairs hi + lo: what the first rounding leaves is kept in a second (16 bits in all)
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = bf162_of(a, b);
  lo = bf162_of(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
}
__device__ __forceinline__ f32x2 sub2(f32x2 a, f32x2 b) { f32x2 d; asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ int ordered(float f) { const int i = __float_as_int(f); return i ^ ((i >> 31) & 0x7fffffff); }
__device__ __forceinline__ float unordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }
// 2^e with the exponent that brings |x| near `top`; 1 for 0, infinities and NaN
__device__ __forceinline__ float pow2_to(float x, int top) {
  if (!(x > 0.f) || x > FLT_MAX) return 1.f;
  const int e = top - (((__float_as_int(x) >> 23) & 255) - 127);
  return __int_as_float((min(max(e, -120), 120) + 127) << 23);
}

// barriers of one group
__device__ __forceinline__ void group_sync(int group) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + group), "n"(SC_GROUP) : "memory"); }
__device__ __forceinline__ bool group_any(int group, bool v) {
  int r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"((int)v), "r"(1 + group), "n"(SC_GROUP) : "memory");
  return r != 0;
}

template <int DK, int NT, bool ROPE>
__global__ void __launch_bounds__((ScoreShape<DK, NT>::THREADS), 1)
slim_tree_p_kernel(const __grid_constant__ CUtensorMap cmap, const __grid_constant__ CUtensorMap dmap, const SlimDecodeParams p,
                   const SlimTreeView t, const int32_t* __restrict__ parents, const float4* __restrict__ table) {
  typedef ScoreShape<DK, NT> S;
  constexpr int HALF = S::HALF, VW = S::VW, NPC = S::NPC, TOK = 8 * NT;
  typedef typename KVec<VW>::type kvec;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* sm = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const int group = warp >> 3, hw = warp & 7, htid = tid & (SC_GROUP - 1);
  unsigned char* ring = sm + (size_t)warp * S::KS * S::KT;                // this warp's key tiles
  float4* cst = reinterpret_cast<float4*>(sm + S::KR);                    // [warp][row half][pc][VW / 2][lane] (cos, cos, sin, sin)
  unsigned char* qs = sm + S::KR + S::CS;                                 // [NT][STEPS][lane][2] the turned queries' pairs
  unsigned char* own = sm + S::KR + S::CS + S::QS + group * S::OWN;
  uint2* qf = reinterpret_cast<uint2*>(own);                              // [2][NT][STEPS][lane]
  float2* sr = reinterpret_cast<float2*>(own + 2 * S::QF);                // [TOK] (what a token's sums are multiplied by, its reference)
  int* smax = reinterpret_cast<int*>(own + 2 * S::QF + S::SR);            // [TOK] largest argument, where a reference has to move
  float* wsum = reinterpret_cast<float*>(own + 2 * S::QF + S::SR + S::MX);        // [2][warp][TOK] sums of a block's rows
  unsigned char* tail = sm + S::KR + S::CS + S::QS + S::GROUPS * S::OWN;
  const uint32_t bar_table = smem_u32(tail), bar = bar_table + 8u * (uint32_t)(1 + warp * S::KS);      // this warp's barriers
  volatile int* s_abort = reinterpret_cast<volatile int*>(tail + 8 * (S::WARPS * S::KS + 1));
  const int n = t.n, R = p.H * n;
  __shared__ int s_par[SLIM_MAX_TREE], s_dep[SLIM_MAX_TREE];              // the current sequence's tree
  __shared__ unsigned long long s_mask[SLIM_MAX_TREE];

  if (lane == 0) {
    for (int i = 0; i < S::KS; ++i) mbar_init(bar + 8 * i, 1);
    if (warp == 0) { mbar_init(bar_table, 1); prefetch_tensormap(&cmap); prefetch_tensormap(&dmap); *s_abort = 0; }
    fence_mbar_init();
  }
  if (ROPE && !S::CSR && tid == 0) {                                      // (a table of the context: no need to wait for it)
    mbar_arrive_expect_tx(bar_table, (uint32_t)S::CS);
    bulk_load(smem_u32(cst), table, (uint32_t)S::CS, bar_table);
  }
  // MMA rows g and g + 8 are keys key0 and key0 + 2 of the warp's tile: turned around, a thread then holds four
  // neighbouring keys of a token
  const int key0 = 4 * (g >> 1) + (g & 1);
  constexpr int NCS = S::CSR && ROPE ? NPC * (VW / 2) : 1;
  ulonglong2 csr[2][NCS];                                                 // (cos, cos), (sin, sin) of this thread's keys and pairs
  auto angles = [&](int rh, int o) {                                      // of key offset o
#pragma unroll
    for (int x = 0; x < NCS; ++x) csr[rh][x] = __ldg(reinterpret_cast<const ulonglong2*>(table) + ((o >> 3) * NCS + x) * 32 + ((o & 7) << 2) + c);
  };
  if (S::CSR && ROPE) { angles(0, 16 * hw + key0); angles(1, 16 * hw + key0 + 2); }
  __syncthreads();                                                        // (the abort flag is read from here on)
  slim_pdl_trigger();
  slim_pdl_wait();
  if (lane == 0) fence_proxy_async_global();                              // (keys and drafts may be an earlier kernel's ordinary stores)
  const int nb_cap = (p.t_cap + SC_KEYS - 1) / SC_KEYS;
  // this CTA's share of the line of blocks, and where it begins; the same in every warp
  int b = 0, h = 0, k0 = 0, remaining;
  {
    auto row_blocks = [&](int q) { return q < p.batch ? p.H * ((min(max(p.lengths[q], 0), p.t_cap) + SC_KEYS - 1) / SC_KEYS + 1) : 0; };
    int all = 0;
    const int first32 = row_blocks(lane);
    for (int q = lane + 32; q < p.batch; q += 32) all += row_blocks(q);
    all += first32;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    const int a0 = (int)((long long)all * blockIdx.x / gridDim.x);
    remaining = (int)((long long)all * (blockIdx.x + 1) / gridDim.x) - a0;
    if (remaining == 0) {                                                 // (not before the table has landed)
      if (ROPE && !S::CSR && tid == 0) mbar_wait<false>(bar_table, 0, s_abort, p.status);
      return;
    }
    for (int q0 = 0, before = 0; q0 < p.batch; q0 += 32) {
      const int mine = q0 ? row_blocks(q0 + lane) : first32;
      int incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
      const unsigned hit = __ballot_sync(0xffffffffu, before + incl > a0);
      if (hit) {
        const int l = __ffs(hit) - 1, row = __shfl_sync(0xffffffffu, mine, l), in = a0 - before - (__shfl_sync(0xffffffffu, incl, l) - row);
        const int nb = row / p.H;
        b = q0 + l;
        h = in / nb; k0 = in - h * nb;
        break;
      }
      before += __shfl_sync(0xffffffffu, incl, 31);
    }
  }
  int len = 0, nblk = 0, first = 0, mine = 0, total = 0, base = 0;        // of the current row; base: key tiles of the rows before
  constexpr int step = S::GROUPS;
  int tree = -1;                                                          // the sequence whose tree is in shared memory

  // this thread's part of the query fragments: pairs j0, j0 + 1 of token 8 nt + lane / 4, for nt = nt0, nt0 + NTS, ..
  constexpr int NTS = SC_GROUP / S::PER;
  const int nt0 = htid / S::PER, fi = htid % S::PER, fs = fi >> 5, j0 = chunk_of(DK, fi & 3, fs / (VW / 2)) * VW + 2 * (fs % (VW / 2));
  auto fetch = [&](int it) {                                              // (lane 0) rows that are not there are masked later
    const bool draft = it == mine;
    const int blk0 = draft ? 0 : (first + it * step) * SC_KEYS, st = (base + it) % S::KS;
    int t0 = blk0 + 16 * hw, row;
    if (!draft && blk0 + SC_KEYS <= len && !p.block_table) row = b * p.t_cap + t0;
    else {
      if (t0 >= (draft ? n : len)) t0 = blk0;
      row = draft ? b * n + t0 : (int)slim_cache_row(p, b, t0);
    }
    mbar_arrive_expect_tx(bar + 8 * st, S::KT);
    tma_load_3d(smem_u32(ring) + (uint32_t)(st * S::KT), draft ? &dmap : &cmap, bar + 8 * st, DK == 96 ? h * DK : 0, row,
                DK == 128 ? 2 * h : DK == 64 ? h : 0);
  };
  auto block_angle = [&](int it) {                                        // (cos, sin) of the block's angle, pairs j0, j0 + 1
    if (!ROPE) return make_float4(1.f, 0.f, 1.f, 0.f);
    if (it == mine) {
      const float2 a = turn(p, len, j0), z = turn(p, len, j0 + 1);
      return make_float4(a.x, a.y, z.x, z.y);
    }
    return __ldg(reinterpret_cast<const float4*>(p.rope_base + (size_t)(first + it * step) * (SC_KEYS / SLIM_TT) * HALF + j0));
  };
  auto fragments = [&](const float4& bc, int buf) {                       // queries turned back by the block's angle
    if (nt0 < NTS) {
#pragma unroll
      for (int nt = nt0; nt < NT; nt += NTS) {
        float4 q;
        if (S::QHALF) {
          const uint2 w = reinterpret_cast<const uint2*>(qs)[nt * S::PER + fi];
          const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&w.x)), v = __half22float2(*reinterpret_cast<const __half2*>(&w.y));
          q = make_float4(u.x, u.y, v.x, v.y);
        } else q = reinterpret_cast<const float4*>(qs)[nt * S::PER + fi];
        qf[(buf * NT + nt) * S::PER + fi] = make_uint2(half2_of(pack2(q.x * bc.x - q.y * bc.y, q.z * bc.z - q.w * bc.w)),
                                          half2_of(pack2(q.y * bc.x + q.x * bc.y, q.w * bc.z + q.z * bc.w)));
      }
    }
  };
  // sums and references of block `it`, once all warps have left theirs
  auto stats = [&](int it) {
    if (htid < n) {
      float l = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) l += wsum[((it & 1) * 8 + w) * TOK + htid];
      t.stat[((size_t)b * (nb_cap + 1) + (it == mine ? nb_cap : first + it * step)) * R + h * n + htid] = make_float2(sr[htid].y, l);
    }
  };

  __syncwarp();
  for (;;) {
    // ---- the next row: blocks k0 .. k1 - 1 of (b, h), the drafted keys' being number nblk
    const int stored = p.lengths[b];
    len = min(max(stored, 0), p.t_cap); nblk = (len + SC_KEYS - 1) / SC_KEYS;
    const int k1 = min(nblk + 1, k0 + remaining);
    first = k0 + group;
    total = k1 > first ? (k1 - 1 - first) / step + 1 : 0;
    mine = total > 0 && k1 == nblk + 1 && first + (total - 1) * step == nblk ? total - 1 : 0x7fffffff;      // which block is the drafted keys'
    const bool opens = h == 0 && k0 == 0;                                 // this CTA leaves the sequence's length and depths for the others
    if (lane == 0 && !*s_abort)
      for (int i = 0; i < S::KS && i < total; ++i) fetch(i);
    float4 bc = make_float4(1.f, 0.f, 1.f, 0.f);
    if (total > 0) bc = block_angle(0);
    if (b != tree) {
      if (tid < n) {
        const int q = parents[(size_t)b * n + tid];
        s_par[tid] = q >= tid ? -3 : q < -1 ? -2 : q;
      }
      __syncthreads();
      if (tid < n) {
        bool broken;
        slim_tree_chain(s_par, tid, s_mask[tid], s_dep[tid], broken);
        if (opens) {
          t.depth[(size_t)b * n + tid] = s_dep[tid];
          if (broken) atomicMax(p.status, (int)SLIM_ERR_TREE);
        }
      }
      __syncthreads();
      tree = b;
    }
    if (opens && tid == 0) {
      t.len[b] = len;
      if (stored > p.t_cap) atomicMax(p.status, (int)SLIM_ERR_CAPACITY);
    }
    // queries of this (sequence, head), scaled and turned to their positions; one warp a token
    bool large = false;
    {
      const __nv_bfloat16* Q = reinterpret_cast<const __nv_bfloat16*>(p.q) + (size_t)b * n * p.d + h * DK;
      for (int i = warp; i < TOK; i += S::WARPS) {
        const bool there = i < n && s_dep[i] >= 0;
        float2 v[(HALF + 31) / 32];
        float top = 0.f;
#pragma unroll
        for (int x = 0; x < (HALF + 31) / 32; ++x) {
          const int j = lane + 32 * x;
          v[x] = make_float2(0.f, 0.f);
          if (there && j < HALF) {
            const float q1 = __bfloat162float(Q[(size_t)i * p.d + j]) * p.qscale, q2 = __bfloat162float(Q[(size_t)i * p.d + HALF + j]) * p.qscale;
            if (ROPE) {
              const float2 cs = turn(p, len + s_dep[i], j);
              v[x] = make_float2(q1 * cs.x + q2 * cs.y, q2 * cs.x - q1 * cs.y);
            } else v[x] = make_float2(q1, q2);
          }
          top = fmaxf(top, fmaxf(fabsf(v[x].x), fabsf(v[x].y)));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float sc = pow2_to(top, 4);                                   // the largest element near 16
#pragma unroll
        for (int x = 0; x < (HALF + 31) / 32; ++x)
          if (lane + 32 * x < HALF) {
            const int j = lane + 32 * x, ch = j / VW, pc = DK == 128 ? ch & 1 : ch >> 2, cc = DK == 128 ? ch >> 1 : ch & 3;
            const int at = 2 * ((i >> 3) * S::PER + (pc * (VW / 2) + (j % VW) / 2) * 32 + (i & 7) * 4 + cc) + (j & 1);
            if (S::QHALF) reinterpret_cast<uint32_t*>(qs)[at] = half2_of(pack2(v[x].x * sc, v[x].y * sc));
            else reinterpret_cast<float2*>(qs)[at] = make_float2(v[x].x * sc, v[x].y * sc);
          }
        if (lane < S::GROUPS) {                                             // every group's copy; a token that is not there: P = 2^(s - inf) = 0
          unsigned char* o = sm + S::KR + S::CS + S::QS + lane * S::OWN + 2 * S::QF;
          reinterpret_cast<float2*>(o)[i] = make_float2(1.f / sc, there ? -INFINITY : INFINITY);
          reinterpret_cast<int*>(o + S::SR)[i] = ordered(-INFINITY);
        }
        // keys near 1 lose at most 2^-12 of themselves; steps of 2^-25 of smaller ones show where DK |q| 2^-25 does
        large = large || !(top <= 64.f);
      }
    }
    const bool careful = __syncthreads_or(large);
    if (ROPE && !S::CSR) mbar_wait<false>(bar_table, 0, s_abort, p.status);
    if (total > 0) fragments(bc, 0);
    if (total > 1) bc = block_angle(1);
    group_sync(group);
    __nv_bfloat16* p_base = t.p + ((size_t)b * R + (size_t)h * n + g) * t.p_ld + 16 * hw + 4 * c;      // of token g
    const size_t p_step = 8 * (size_t)t.p_ld;
    for (int it = 0; it < total; ++it) {
      const bool draft = it == mine;
      const int blk = first + it * step, t0 = draft ? 16 * hw : blk * SC_KEYS + 16 * hw;
      // ---- scores
      // a drafted key's offset in its block is its depth
      const ulonglong2* row_cs[2];
      if (ROPE) {
#pragma unroll
        for (int rh = 0; rh < 2; ++rh) {
          int o = 16 * hw + key0 + 2 * rh;
          if (draft) o = o < n ? max(s_dep[o], 0) : 0;
          if (S::CSR) { if (draft) angles(rh, o); }
          else row_cs[rh] = reinterpret_cast<const ulonglong2*>(cst) + (o >> 3) * (NPC * (VW / 2) * 32) + ((o & 7) << 2) + c;
        }
      }
      unsigned char* tile = ring + ((base + it) % S::KS) * S::KT;
      const uint2* qb = qf + (it & 1) * NT * S::PER;
      mbar_wait<false>(bar + 8 * ((base + it) % S::KS), ((base + it) / S::KS) & 1, s_abort, p.status);      // (gave up: reported, and the loop runs on to its end)
      float s[NT][4];
      float back = 1.f;                                                     // undoes the keys' scaling, but for the keys' own parts
      // Rows behind the sequence's last, padding and the next sequence's rows may hold anything; they must meet neither the
      // overflow test nor the scaling of others
      const bool edge = draft || t0 + 16 > len;
      auto attended = [&](int r) { return !edge || (draft ? r < n && s_dep[min(r, n - 1)] >= 0 : r < len); };
      for (int own2 = 0;;) {                                                // what is left of it for keys key0, key0 + 2: two exponents, above 0
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
        for (int pc = 0; pc < NPC; ++pc) {
          kvec k[2][2];                                                     // [row half][low / high elements of the pairs]
#pragma unroll
          for (int rh = 0; rh < 2; ++rh)
#pragma unroll
            for (int hl = 0; hl < 2; ++hl) k[rh][hl] = *reinterpret_cast<const kvec*>(tile + tile_off<DK>(key0 + 2 * rh, c, pc, hl));
#pragma unroll
          for (int xq = 0; xq < VW / 2; ++xq) {
            uint32_t a[4];
#pragma unroll
            for (int rh = 0; rh < 2; ++rh) {
              const f32x2 k1 = unpack2(word(k[rh][0], xq)), k2 = unpack2(word(k[rh][1], xq));
              if (ROPE) {
                const ulonglong2 cs = S::CSR ? csr[rh][(pc * (VW / 2) + xq) % NCS] : row_cs[rh][(pc * (VW / 2) + xq) * 32];
                a[rh] = half2_of(fma2(k2, cs.y, mul2(k1, cs.x)));
                a[2 + rh] = half2_of(sub2(mul2(k2, cs.x), mul2(k1, cs.y)));
              } else {
                a[rh] = half2_of(k1);
                a[2 + rh] = half2_of(k2);
              }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint2 f = qb[nt * S::PER + (pc * (VW / 2) + xq) * 32 + lane];
              mma_f16(s[nt], a, f.x, f.y);
            }
          }
        }
        if (own2) {
          const float f0 = ldexpf(1.f, (own2 & 0xffff) - 512), f1 = ldexpf(1.f, (own2 >> 16) - 512);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 4; ++x) s[nt][x] *= x < 2 ? f0 : f1;
          break;
        }
        if (edge)
#pragma unroll
          for (int rh = 0; rh < 2; ++rh)
            if (!attended(t0 + key0 + 2 * rh))
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) s[nt][2 * rh] = s[nt][2 * rh + 1] = 0.f;
        // an overflow shows as an infinity or a NaN, and 0 x it is a NaN
        float odd = 0.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 4; ++x) odd = fmaf(s[nt][x], 0.f, odd);
        if (!__any_sync(0xffffffffu, careful || odd != 0.f)) break;
        int most = -127, least = 127, all = -127;                           // exponents: the tokens' factors, the keys'
        // every key by its own largest element (its four lanes have it in common), so that none wipes out another; in place
#pragma unroll 1                                                            // (rare: no registers for it)
        for (int rh = 0; rh < 2; ++rh) {
          float top = 0.f;
#pragma unroll 1
          for (int e = 0; e < 2 * NPC; ++e) {
            const kvec v = *reinterpret_cast<const kvec*>(tile + tile_off<DK>(key0 + 2 * rh, c, e >> 1, e & 1));
#pragma unroll
            for (int x = 0; x < VW / 2; ++x)
              top = fmaxf(top, fmaxf(fabsf(__uint_as_float(word(v, x) << 16)), fabsf(__uint_as_float(word(v, x) & 0xffff0000u))));
          }
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const float ks = pow2_to(top, 10);
          const int e_back = 127 - (__float_as_int(ks) >> 23);
          own2 |= (e_back + 512) << (16 * rh);
          if (attended(t0 + key0 + 2 * rh)) all = max(all, e_back);
#pragma unroll 1
          for (int e = 0; e < 2 * NPC; ++e) {
            kvec* at = reinterpret_cast<kvec*>(tile + tile_off<DK>(key0 + 2 * rh, c, e >> 1, e & 1));
            kvec v = *at;
#pragma unroll
            for (int x = 0; x < VW / 2; ++x)                                // (a power of two: exact, but for what is 2^-100 of the largest)
              word_ref(v, x) = bf162_of(__uint_as_float(word(v, x) << 16) * ks, __uint_as_float(word(v, x) & 0xffff0000u) * ks);
            *at = v;
          }
        }
        // one factor for the warp, so that no token's factor times it overflows or vanishes: a sum far below the largest then
        // loses at most 2^-149 2^126 of its argument
        for (int i = lane; i < TOK; i += 32) {
          const int e = (__float_as_int(sr[i].x) >> 23) - 127;
          most = max(most, e); least = min(least, e);
        }
        most = __reduce_max_sync(0xffffffffu, most); least = __reduce_min_sync(0xffffffffu, least);
        all = min(max(__reduce_max_sync(0xffffffffu, all), -126 - least), 126 - most);
        back = __int_as_float((all + 127) << 23);
        own2 -= all * 0x10001;
        fence_proxy_async_smem();                                           // (the next tile comes by the async proxy)
      }
      __syncwarp();                                                         // all lanes have read the tile
      if (lane == 0 && it + S::KS < total && !*s_abort) fetch(it + S::KS);
      // ---- what is not attended
      if (edge) {
  #pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int r = t0 + key0 + (x & 2);
            const bool on = draft ? r < n && ((s_mask[min(8 * nt + 2 * c + (x & 1), n - 1)] >> (r & 63)) & 1) : r < len;
            if (!on) s[nt][x] = -INFINITY;
          }
      }
      // ---- arguments relative to the references; does one have to move?  (always in the first block: -inf)
      // P may reach 2^60, but only 1 beside keys that were scaled down (above 2^10, that is): P K must not overflow
      const float room = back > 1.f ? 0.f : 60.f;
      bool moves = false;
      float y[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float4 v = *reinterpret_cast<const float4*>(sr + 8 * nt + 2 * c);
        const float s0 = v.x * back, s1 = v.z * back;
        y[nt][0] = fmaf(s[nt][0], s0, -v.y); y[nt][1] = fmaf(s[nt][1], s1, -v.w);
        y[nt][2] = fmaf(s[nt][2], s0, -v.y); y[nt][3] = fmaf(s[nt][3], s1, -v.w);
        moves = moves || fmaxf(fmaxf(y[nt][0], y[nt][1]), fmaxf(y[nt][2], y[nt][3])) > room;
      }
      if (it + 1 < total) fragments(bc, (it + 1) & 1);
      if (it + 2 < total) bc = block_angle(it + 2);
      const bool any_moves = group_any(group, moves);
      if (it > 0) stats(it - 1);
      if (any_moves) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            float m = fmaf(fmaxf(s[nt][z], s[nt][2 + z]), sr[8 * nt + 2 * c + z].x * back, 60.f - room);
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (g == 0) atomicMax(smax + 8 * nt + 2 * c + z, ordered(m));
          }
        group_sync(group);
        if (htid < TOK) {
          const float m = unordered(smax[htid]);                            // (of the blocks that came here)
          if (m > sr[htid].y + 60.f) sr[htid].y = 64.f * rintf(fminf(m, FLT_MAX) * (1.f / 64.f));
        }
        group_sync(group);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float4 v = *reinterpret_cast<const float4*>(sr + 8 * nt + 2 * c);
          const float s0 = v.x * back, s1 = v.z * back;
          y[nt][0] = fmaf(s[nt][0], s0, -v.y); y[nt][1] = fmaf(s[nt][1], s1, -v.w);
          y[nt][2] = fmaf(s[nt][2], s0, -v.y); y[nt][3] = fmaf(s[nt][3], s1, -v.w);
        }
      }
      // ---- probabilities, turned around to [token][4 keys], out; their sums over this warp's keys
      __nv_bfloat16* Pout = p_base + (draft ? t.s_draft : blk * SC_KEYS);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint32_t d0 = movmatrix_trans(bf162_of(ex2_approx(y[nt][0]), ex2_approx(y[nt][1])));
        const uint32_t d1 = movmatrix_trans(bf162_of(ex2_approx(y[nt][2]), ex2_approx(y[nt][3])));
        const int i = 8 * nt + g;
        if (i < n && (!draft || hw < 4)) *reinterpret_cast<uint2*>(Pout + (size_t)nt * p_step) = make_uint2(d0, d1);
        float l = sum2(add2(unpack2(d0), unpack2(d1)));
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        if (c == 0) wsum[((it & 1) * 8 + hw) * TOK + i] = l;
      }
    }
    group_sync(group);
    if (total > 0) stats(total - 1);
    // ---- on to the next row
    if (S::CSR && ROPE && mine < total) { angles(0, 16 * hw + key0); angles(1, 16 * hw + key0 + 2); }      // (the drafted keys' took their place)
    base += total;
    remaining -= k1 - k0;
    if (remaining == 0) break;
    k0 = 0;
    if (++h == p.H) { h = 0; ++b; }
    __syncthreads();                                                      // (everyone is done with the queries, references and sums)
  }
}

// ------------------------------------------------------------------------------------------------ schedule of the product
// A tile is MT x 256 rows of P by 256 columns of K; its keys are walked in stages of 64 rows (the cached whole blocks,
// the partial one, the drafted keys).  Every tile of every sequence may be cut into S equal parts of its stages
// (subtiles; S > 1 where there are fewer tiles than CTA pairs).  The subtiles, in the order (sequence, part, tile), go
// to the pairs in turn, F of them as a whole, so that pairs in flight walk the same keys and the same rows of P at the
// same time and share them in L2; what is left over, about a round, is laid on a line and cut so that every pair ends
// up with the same number of stages.  A piece that is not a whole tile leaves float32 sums in a slot, and `join` adds
// the slots of a tile in the order of its keys: the schedule is a function of the lengths alone, so results are repeatable.
struct SumSched {
  int batch, tiles, S, P, F, TS;      // tiles of a sequence, parts, pairs, whole subtiles, subtiles in all
  const int* nk;                      // shared [batch]      stages of a sequence
  const long long* pre;               // shared [batch + 1]  tiles x stages before it
  const long long* cut;               // shared [P + 1]      the left-over line's cuts
  long long g0;                       // line position of subtile F
};
struct SumItem { int b, tile, k0, k1, slot; };       // slot -1: a whole tile

__host__ __device__ inline int stages_of(int len) { return len / 64 + (len % 64 ? 1 : 0) + 1; }

__device__ __forceinline__ int part_begin(int nk, int part, int S) {     // floor(nk part / S)
  if (S == 1) return part ? nk : 0;
  return nk < (1 << 21) ? (int)((unsigned)nk * (unsigned)part / (unsigned)S) : (int)((long long)nk * part / S);      // (S <= 1024)
}
__device__ __forceinline__ void subtile(const SumSched& s, int idx, int& b, int& tile, int& k0, int& k1) {
  const int per = s.S * s.tiles;
  b = idx / per;
  const int in = idx - b * per, part = in / s.tiles;
  tile = in - part * s.tiles;
  const int nk = s.nk[b];
  k0 = part_begin(nk, part, s.S); k1 = part_begin(nk, part + 1, s.S);
}
__device__ __forceinline__ long long line_pos(const SumSched& s, int idx) {       // stages before subtile idx
  if (idx >= s.TS) return s.pre[s.batch];
  int b, tile, k0, k1;
  subtile(s, idx, b, tile, k0, k1);
  return s.pre[b] + (long long)s.tiles * k0 + (long long)tile * (k1 - k0);
}
// the subtile that holds line position x < pre[batch]
__device__ __forceinline__ int at_pos(const SumSched& s, long long x) {
  int lo = 0, hi = s.batch;
  while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (s.pre[mid] <= x) lo = mid; else hi = mid; }
  const long long in = x - s.pre[lo];
  const int nk = s.nk[lo];
  const int k = in < (1ll << 31) ? (int)((unsigned)in / (unsigned)s.tiles) : (int)(in / s.tiles);   // in lies in the part whose [k0, k1) holds k
  int part = s.S == 1 ? 0 : (int)(((long long)(k + 1) * s.S - 1) / nk);
  while (part_begin(nk, part + 1, s.S) <= k) ++part;
  while (part_begin(nk, part, s.S) > k) --part;
  const int k0 = part_begin(nk, part, s.S), k1 = part_begin(nk, part + 1, s.S);
  const long long off = in - (long long)s.tiles * k0;
  return lo * s.S * s.tiles + part * s.tiles + (off < (1ll << 31) ? (int)((unsigned)off / (unsigned)(k1 - k0)) : (int)(off / (k1 - k0)));
}

// By all threads of a block; s_pre, s_cut, s_nk in shared memory.
__device__ __forceinline__ SumSched build_sum_sched(const SlimTreeView& t, int batch, int* s_nk, long long* s_pre, long long* s_cut) {
  SumSched s;
  s.batch = batch; s.tiles = t.g_tiles; s.S = t.g_split; s.P = t.g_pairs; s.F = t.g_whole; s.TS = batch * t.g_tiles * t.g_split;
  s.nk = s_nk; s.pre = s_pre; s.cut = s_cut;
  const int tid = threadIdx.x, nthr = blockDim.x;
  for (int b = tid; b < batch; b += nthr) s_nk[b] = stages_of(t.len[b]);
  __syncthreads();
  if (tid < 32) {
    const int chunk = (batch + 31) / 32, lo = min(batch, tid * chunk), hi = min(batch, lo + chunk);
    long long sum = 0;
    for (int b = lo; b < hi; ++b) sum += s_nk[b];
    long long incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const long long v = __shfl_up_sync(0xffffffffu, incl, o); if (tid >= o) incl += v; }
    long long run = incl - sum;
    for (int b = lo; b < hi; ++b) { s_pre[b] = run * s.tiles; run += s_nk[b]; }
    if (tid == 31) s_pre[batch] = incl * s.tiles;
  }
  __syncthreads();
  s.g0 = line_pos(s, s.F);
  const long long all = s_pre[batch], want = (all + s.P - 1) / s.P;
  for (int q = tid; q < s.P; q += nthr) {                               // what pair q has left to take
    long long load = 0;
    for (int idx = q; idx < s.F; idx += s.P) {
      int b, tile, k0, k1;
      subtile(s, idx, b, tile, k0, k1);
      load += k1 - k0;
    }
    s_cut[q + 1] = load < want ? want - load : 0;
  }
  __syncthreads();
  if (tid < 32) {                                                       // lane x: pairs x per .. x per + per - 1
    const int per = (s.P + 31) / 32, lo = min(s.P, tid * per), hi = min(s.P, lo + per);
    const long long rest = all - s.g0;
    long long mine = 0;
    for (int q = lo; q < hi; ++q) mine += s_cut[q + 1];
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const long long v = __shfl_up_sync(0xffffffffu, incl, o); if (tid >= o) incl += v; }
    const long long sum = __shfl_sync(0xffffffffu, incl, 31);
    const double scale = sum > 0 ? (double)rest / (double)sum : 0.0;
    long long run = incl - mine;
    if (tid == 0) s_cut[0] = 0;
    for (int q = lo; q < hi; ++q) {
      run += s_cut[q + 1];
      const long long cut = (long long)((double)run * scale);
      s_cut[q + 1] = (cut > rest || q == s.P - 1) ? rest : cut;
    }
  }
  __syncthreads();
  return s;
}

// The pieces of pair q, one after another.
struct SumWalk {
  int idx;
  long long at;
};
__device__ __forceinline__ SumWalk sum_begin(const SumSched& s, int q) { SumWalk w; w.idx = q; w.at = s.cut[q]; return w; }
__device__ __forceinline__ bool sum_next(const SumSched& s, int q, SumWalk& w, SumItem& it) {
  while (w.idx < s.F) {
    const int idx = w.idx;
    w.idx += s.P;
    subtile(s, idx, it.b, it.tile, it.k0, it.k1);
    if (it.k0 == it.k1) continue;
    it.slot = s.S == 1 ? -1 : 2 * s.P + idx;
    return true;
  }
  const long long end = s.cut[q + 1];
  if (w.at >= end) return false;
  const long long x = w.at + s.g0;
  const int idx = at_pos(s, x);
  const long long x0 = line_pos(s, idx);
  int k0, k1;
  subtile(s, idx, it.b, it.tile, k0, k1);
  const long long x1 = x0 + (k1 - k0), stop = min(x1, end + s.g0);
  it.k0 = k0 + (int)(x - x0); it.k1 = k0 + (int)(stop - x0);
  w.at = stop - s.g0;
  it.slot = (x == x0 && stop == x1) ? (s.S == 1 ? -1 : 2 * s.P + idx) : x > x0 ? 2 * q : 2 * q + 1;
  return true;
}

// ------------------------------------------------------------------------------------------------ finish
// 32 rows a block, 32 threads a row: M = the largest reference of the row's blocks that hold anything, 1 / l, and blocks of
// P whose reference is another (rare: a row whose block maxima are more than about 32 apart around a multiple of 64)
// multiplied by 2^(ref - M), a power of two: exact, down to values below 2^-94 of the row's largest, which become 0.
// A token that is there attends itself at least: a sum that is not a positive number (arguments that are NaN or infinite) is
// no empty row, its 1 / l is NaN.  FIN_TAIL blocks of a sequence behind these write its tail [128][d]: 0..63 the cached rows
// behind the last whole block of 64, 64..127 the drafted keys, everything else zero; one last block of the grid lays down the
// product's schedule.
constexpr int FIN_TAIL = 16;
__global__ void __launch_bounds__(1024) slim_tree_finish_kernel(const SlimDecodeParams p, const SlimTreeView t) {
  __shared__ float s_m[32][33], s_l[32][33];
  extern __shared__ __align__(16) unsigned char smem_raw[];
  slim_pdl_trigger();
  slim_pdl_wait();
  const int row_grid = (p.H * t.n + 31) / 32, tail_block = (int)blockIdx.x - row_grid;
  if (tail_block >= FIN_TAIL) {
    if (blockIdx.y != 0) return;
    long long* s_pre = reinterpret_cast<long long*>(smem_raw);
    long long* s_cut = s_pre + p.batch + 1;
    const SumSched sc = build_sum_sched(t, p.batch, reinterpret_cast<int*>(s_cut + t.g_pairs + 1), s_pre, s_cut);
    for (int i = threadIdx.x; i < p.batch + 1 + sc.P + 1; i += 1024) t.sched[i] = i <= p.batch ? s_pre[i] : s_cut[i - p.batch - 1];
    if (threadIdx.x == 0) t.sched[p.batch + sc.P + 2] = sc.g0;
    return;
  }
  if (tail_block >= 0) {
    const int b = blockIdx.y, r = tail_block * 8 + ((int)threadIdx.x >> 7), vecs = p.d / 8, len = t.len[b], row = (len & ~63) + r;
    const uint4* src = nullptr;
    if (r < 64) {
      if (row < len) src = reinterpret_cast<const uint4*>(p.k) + (size_t)(slim_cache_row(p, b, row & ~(SLIM_TT - 1)) + (row & (SLIM_TT - 1))) * vecs;
    } else if (r - 64 < t.n && t.depth[(size_t)b * t.n + r - 64] >= 0) {
      src = reinterpret_cast<const uint4*>(t.k_tree) + ((size_t)b * t.n + r - 64) * vecs;
    }
    uint4* dst = reinterpret_cast<uint4*>(t.tail) + ((size_t)b * 128 + r) * vecs;
    for (int e = threadIdx.x & 127; e < vecs; e += 128) dst[e] = src ? __ldg(src + e) : make_uint4(0, 0, 0, 0);
    return;
  }
  const int R = p.H * t.n, x = threadIdx.x & 31, y = threadIdx.x >> 5, b = blockIdx.y, row = blockIdx.x * 32 + x;
  const int nb_cap = (p.t_cap + SC_KEYS - 1) / SC_KEYS, nblk = (t.len[b] + SC_KEYS - 1) / SC_KEYS;
  const float2* stat = t.stat + (size_t)b * (nb_cap + 1) * R + row;
  float m = -INFINITY, l = 0.f;
  bool same = true;                                        // every block this thread saw has the same reference
  if (row < R)
    for (int k0 = y; k0 <= nblk; k0 += 128) {
      float2 v[4];
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        const int k = k0 + 32 * x4;
        v[x4] = k <= nblk ? stat[(size_t)(k == nblk ? nb_cap : k) * R] : make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        if (v[x4].y == 0.f) continue;
        if (v[x4].x == m) { l += v[x4].y; continue; }      // (also -inf: a sum without a reference is NaN, and stays)
        same = same && m == -INFINITY;
        const float top = fmaxf(m, v[x4].x);
        l = l * exp2f(m - top) + v[x4].y * exp2f(v[x4].x - top);
        m = top;
      }
    }
  s_m[y][x] = m; s_l[y][x] = l;
  __syncthreads();
  float M = -INFINITY, L = 0.f;
  for (int k = 0; k < 32; ++k) M = fmaxf(M, s_m[k][x]);
  for (int k = 0; k < 32; ++k) L += s_l[k][x] == 0.f ? 0.f : M == -INFINITY ? s_l[k][x] : s_l[k][x] * exp2f(s_m[k][x] - M);
  if (row >= R) return;
  const bool there = t.depth[(size_t)b * t.n + row % t.n] >= 0;
  if (y == 0) t.inv_l[(size_t)b * R + row] = !there ? 0.f : L > 0.f && L < INFINITY ? 1.f / L : NAN;
  if (same && (m == M || m == -INFINITY)) return;
  for (int k = y; k <= nblk; k += 32) {
    const float2 v = stat[(size_t)(k == nblk ? nb_cap : k) * R];
    if (v.y == 0.f || v.x == M) continue;
    const float f = exp2f(v.x - M);
    __nv_bfloat162* P = reinterpret_cast<__nv_bfloat162*>(t.p + ((size_t)b * R + row) * t.p_ld + (k == nblk ? t.s_draft : k * SC_KEYS));
    for (int e = 0; e < (k == nblk ? 32 : SC_KEYS / 2); ++e) {
      const float2 w = __bfloat1622float2(P[e]);
      P[e] = __floats2bfloat162_rn(w.x * f, w.y * f);
    }
  }
}

// ------------------------------------------------------------------------------------------------ U = P K
// Persistent, one CTA per SM in pairs.  A stage of 64 keys holds, per CTA, MT x 128 rows of P (K-major, 128-byte
// swizzle) and HALF of the tile's 256 columns of K (MN-major, as the cache rows come: two 64-column atoms); one
// tcgen05.mma.cta_group::2 has M = 256, N = 256, K = 16.  MT = 2 (more than 256 rows a sequence) runs two accumulators on
// one load of K: 48 KB of operands per 2 x 256 x 256 x 64 products instead of 64 KB, and half the trips of K through HBM;
// MT = 1 double-buffers the accumulator instead, so that a tile's epilogue runs under the next tile's products.
// Bound by the tensor cores: 64 drafts over 131001 rows (2.2 TFLOP) 1.40 ms, 1575 TFLOP/s, 0.95 of what a library product
// reaches in a burst; 16 ragged sequences, 196 k rows, 16 drafts (0.82 TFLOP) 0.567 ms, 1450 TFLOP/s, the power cap's rate.  With
// few drafts the 256 rows of an MMA are not all there, and it is bound by reading K: 8 x 12000 rows, one draft 0.15 ms
// (5.2 TB/s).
// Warp 0: TMA; warp 1 (even CTA): MMA issue; warps 2-5: epilogue.  A paged cache comes in pieces of 16 rows (a page
// holds whole ones), a contiguous one 64 rows at a time.
constexpr int SU_THREADS = 192, SU_ROWS = 128, SU_COLS = 256, SU_A = SU_ROWS * 128, SU_B = 64 * 256, SU_TURN = 4 * 2048;
template <int MT> struct SumShape {
  static constexpr int STAGE = MT * SU_A + SU_B, NS = MT == 1 ? 6 : 4;
  static size_t smem(int batch, int pairs) {
    return 1024 + (size_t)NS * STAGE + SU_TURN + 16 * NS + 32 + 64 + sizeof(long long) * (batch + 1 + pairs + 1) + sizeof(int) * batch + 16;
  }
};

template <int MT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(SU_THREADS, 1)
slim_tree_u_kernel(const __grid_constant__ CUtensorMap pmap, const __grid_constant__ CUtensorMap kmap,
                   const __grid_constant__ CUtensorMap tailmap, const SlimDecodeParams p, const SlimTreeView t) {
  constexpr int NS = SumShape<MT>::NS;
  constexpr uint32_t STAGE = SumShape<MT>::STAGE;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw_u32 = smem_u32(smem_raw);
  const uint32_t base = (raw_u32 + 1023u) & ~1023u;
  unsigned char* sm = smem_raw + (base - raw_u32);
  unsigned char* turn_buf = sm + NS * STAGE;               // 2 KB an epilogue warp
  const uint32_t bars = base + NS * STAGE + SU_TURN;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * NS, bar_accf = bars + 16 * NS, bar_acce = bar_accf + 16;
  unsigned char* misc = sm + NS * STAGE + SU_TURN + 16 * NS + 32;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(misc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(misc + 4);
  long long* s_pre = reinterpret_cast<long long*>(misc + 64);
  long long* s_cut = s_pre + p.batch + 1;
  int* s_nk = reinterpret_cast<int*>(s_cut + t.g_pairs + 1);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1;
  int* status = p.status;

  if (tid == 0) {
    prefetch_tensormap(&pmap); prefetch_tensormap(&kmap); prefetch_tensormap(&tailmap);
    for (int i = 0; i < NS; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(bar_accf + 8 * i, 1); mbar_init(bar_acce + 8 * i, 8); }
    *s_abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc2(smem_u32(s_tmem), 512);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *s_tmem;
  slim_pdl_trigger();
  slim_pdl_wait();
  // the schedule that `finish` laid down
  SumSched sc;
  sc.batch = p.batch; sc.tiles = t.g_tiles; sc.S = t.g_split; sc.P = t.g_pairs; sc.F = t.g_whole; sc.TS = p.batch * t.g_tiles * t.g_split;
  sc.nk = s_nk; sc.pre = s_pre; sc.cut = s_cut;
  for (int i = tid; i < p.batch + 1 + sc.P + 1; i += SU_THREADS) (i <= p.batch ? s_pre[i] : s_cut[i - p.batch - 1]) = t.sched[i];
  for (int i = tid; i < p.batch; i += SU_THREADS) s_nk[i] = stages_of(t.len[i]);
  sc.g0 = t.sched[p.batch + sc.P + 2];
  __syncthreads();
  const bool paged = p.block_table != nullptr;
  const int ntile = t.g_ncol;                              // column tiles; tile = row tile * ntile + column tile

  if (warp == 0) {
    // ---- producer ----
    fence_proxy_async_global();                            // (P and the tail were written by ordinary stores)
    int g = 0;
    bool ok = true;
    SumWalk w = sum_begin(sc, pair);
    SumItem it;
    while (ok && sum_next(sc, pair, w, it)) {
      const int len = t.len[it.b], whole = len / 64, nk = sc.nk[it.b];
      const int mt0 = it.tile / ntile, chunk = (it.tile % ntile) * 4 + 2 * (int)rank, row0 = mt0 * MT * 256 + (int)rank * SU_ROWS;
      int my_row = 0, have = -1;                           // lane x: storage row of the 16-key piece have + x
      for (int k = it.k0; k < it.k1; ++k, ++g) {
        if (paged && k < whole && (have < 0 || 4 * k >= have + 32)) {
          have = 4 * k;
          const int piece = have + lane;
          my_row = piece < 4 * whole ? (int)slim_cache_row(p, it.b, piece * 16) : 0;
        }
        int r4[4];
        if (paged && k < whole)
#pragma unroll
          for (int x = 0; x < 4; ++x) r4[x] = __shfl_sync(0xffffffffu, my_row, 4 * k - have + x);
        if (lane == 0) {
          const int st = g % NS;
          ok = mbar_wait<false>(bar_empty + 8 * st, ((g / NS) & 1) ^ 1, s_abort, status);
          if (ok) {
            const uint32_t dst = base + (uint32_t)st * STAGE, full0 = mapa(bar_full + 8 * st, 0);
            if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * st, 2 * STAGE);
            const int pcol = k < whole ? k * 64 : k == nk - 1 ? t.s_draft : whole * 64;
#pragma unroll
            for (int m = 0; m < MT; ++m) tma_load_3d_pair(dst + m * SU_A, &pmap, full0, pcol, row0 + m * 256, it.b);
            const CUtensorMap* map = k < whole ? &kmap : &tailmap;
            const int krow = it.b * (k < whole ? p.t_cap : 128) + (k < whole ? k * 64 : k == nk - 1 ? 64 : 0);
            if (!paged) tma_load_3d_pair(dst + MT * SU_A, map, full0, 0, krow, chunk);
            else
#pragma unroll
              for (int x = 0; x < 4; ++x)
                tma_load_3d_pair(dst + MT * SU_A + x * 4096, map, full0, 0, k < whole ? r4[x] : krow + 16 * x, chunk);
          }
        }
        ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
        if (!ok) break;
      }
    }
    if (!ok && lane == 0) {
      // gave up: what was issued has long landed; the even CTA still waits, bounded, on the barriers that count both
      // CTAs' bytes, the odd CTA lets a fixed time pass
      if (rank == 0) {
        const int issued = g < NS ? g : NS;
        for (int k = 0; k < issued; ++k) {
          const int j = g - 1 - k, st = j % NS;
          const unsigned long long tt = globaltimer();
          while (!mbar_try_wait(bar_full + 8 * st, (j / NS) & 1) && globaltimer() - tt < SLIM_WAIT_NS) {}
        }
      } else {
        const unsigned long long tt = globaltimer();
        while (globaltimer() - tt < 200000ull) {}
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      // ---- MMA issuer of the pair ----
      bool ok = true;
      int g = 0, i = 0;
      const uint64_t ad0 = desc_kmajor_sw128(base), bd0 = desc_a(base + MT * SU_A, paged ? 2048 : 8192);
      const uint32_t a_lo0 = (uint32_t)ad0, a_hi = (uint32_t)(ad0 >> 32), b_lo0 = (uint32_t)bd0, b_hi = (uint32_t)(bd0 >> 32);
      const uint32_t bstep = (paged ? 4096u : 2048u) >> 4;
      constexpr uint32_t idesc = umma_idesc_mn(256, SU_COLS, 0, 1);
      SumWalk w = sum_begin(sc, pair);
      SumItem it;
      for (; ok && sum_next(sc, pair, w, it); ++i) {
        const int acc0 = MT == 1 ? (i & 1) : 0;
        const uint32_t ph = MT == 1 ? (i >> 1) & 1 : i & 1;
        for (int k = it.k0; k < it.k1; ++k, ++g) {
          const int st = g % NS;
          ok = mbar_wait<true>(bar_full + 8 * st, (g / NS) & 1, s_abort, status);
          if (!ok) break;
          tc_fence_after();
          const uint32_t b_lo = b_lo0 + (uint32_t)st * (STAGE >> 4);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const int acc = acc0 + m;
            if (k == it.k0) {                              // both CTAs have read the accumulator out
              ok = mbar_wait<true>(bar_acce + 8 * acc, ph ^ 1, s_abort, status);
              if (!ok) break;
              tc_fence_after();
            }
            const uint32_t a_lo = a_lo0 + (uint32_t)st * (STAGE >> 4) + (uint32_t)m * (SU_A >> 4);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              umma2_bf16_words(tmem_base + (uint32_t)(acc * SU_COLS), a_lo + (uint32_t)kk * (32u >> 4), a_hi, b_lo + (uint32_t)kk * bstep, b_hi,
                               idesc, (k > it.k0 || kk) ? 1u : 0u);
          }
          if (!ok) break;
          umma2_commit_pair(bar_empty + 8 * st);
        }
        if (ok)
#pragma unroll
          for (int m = 0; m < MT; ++m) umma2_commit_pair(bar_accf + 8 * (acc0 + m));
      }
    }
  } else {
    // ---- epilogue ----
    // A lane holds a row of the accumulator; written like that, every 16 bytes of a warp's store lie in another row.  So
    // 64 bytes of each of the 32 rows are turned around in shared memory: four lanes then write 64 bytes of a row
    // together (the product of 16 ragged sequences with 16 drafts 600 -> 567 us, of 64 drafts over 131001 rows 1480 -> 1396,
    // of 15 two-row sequences with 54 drafts 270 -> 158).
    const int q = warp & 3, R = p.H * t.n;
    unsigned char* buf = turn_buf + q * 2048;
    auto turned = [&](const uint4 (&v)[4], uint4 (&o)[4]) {                // o[x]: chunk lane % 4 of row 8 x + lane / 4
      __syncwarp();
#pragma unroll
      for (int x = 0; x < 4; ++x) *reinterpret_cast<uint4*>(buf + lane * 64 + ((x ^ ((lane >> 1) & 3)) << 4)) = v[x];
      __syncwarp();
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int y = 8 * x + (lane >> 2);
        o[x] = *reinterpret_cast<const uint4*>(buf + y * 64 + (((lane & 3) ^ ((y >> 1) & 3)) << 4));
      }
    };
    bool ok = true;
    int i = 0;
    SumWalk w = sum_begin(sc, pair);
    SumItem it;
    for (; ok && sum_next(sc, pair, w, it); ++i) {
      const int mt0 = it.tile / ntile, col0 = (it.tile % ntile) * SU_COLS;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int acc = MT == 1 ? (i & 1) : m;
        const uint32_t ph = MT == 1 ? (i >> 1) & 1 : i & 1;
        ok = mbar_wait<false>(bar_accf + 8 * acc, ph, s_abort, status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const int in0 = m * 256 + (int)rank * SU_ROWS + q * 32, r = mt0 * MT * 256 + in0 + lane, mine = mt0 * MT * 256 + in0 + (lane >> 2);
        const uint32_t ta = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * SU_COLS);
        if (it.slot < 0) {
          const float il = r < R ? t.inv_l[(size_t)it.b * R + r] : 0.f;
          __nv_bfloat16* out[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int y = min(mine + 8 * x, R - 1), h = y / t.n, tok = y - h * t.n;
            out[x] = t.uh + (((size_t)h * p.batch + it.b) * t.n + tok) * p.d + col0 + 8 * (lane & 3);
          }
          const size_t to_lo = (size_t)p.H * p.batch * t.n * p.d;
          for (int c0 = 0; c0 < SU_COLS && col0 + c0 < p.d; c0 += 32) {
            uint32_t v[32];
            tmem_ld32(ta + (uint32_t)c0, v);
            uint4 hi[4], lo[4], o4[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
#pragma unroll
              for (int y = 0; y < 4; ++y)
                split2(__uint_as_float(v[8 * x + 2 * y]) * il, __uint_as_float(v[8 * x + 2 * y + 1]) * il, word_ref(hi[x], y), word_ref(lo[x], y));
              if (il == 0.f) hi[x] = lo[x] = make_uint4(0, 0, 0, 0);         // (padding is 0 whatever the keys hold)
            }
            turned(hi, o4);
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (mine + 8 * x < R) *reinterpret_cast<uint4*>(out[x] + c0) = o4[x];
            turned(lo, o4);
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (mine + 8 * x < R) *reinterpret_cast<uint4*>(out[x] + to_lo + c0) = o4[x];
          }
        } else {
          float* out = t.part + ((size_t)it.slot * MT * 256 + in0 + (lane >> 2)) * SU_COLS + 4 * (lane & 3);
          for (int c0 = 0; c0 < SU_COLS && col0 + c0 < p.d; c0 += 32) {
            uint32_t v[32];
            tmem_ld32(ta + (uint32_t)c0, v);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint4 c4[4], o4[4];
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const int e = 16 * half + 4 * x;
                c4[x] = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
              }
              turned(c4, o4);
#pragma unroll
              for (int x = 0; x < 4; ++x)
                if (mine + 8 * x < R) *reinterpret_cast<uint4*>(out + (size_t)8 * x * SU_COLS + c0 + 16 * half) = o4[x];
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(mapa(bar_acce + 8 * acc, 0));
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc2(tmem_base, 512);
  }
}

// ------------------------------------------------------------------------------------------------ join
// Block (tile of the batch, 4 RPT rows of it): sums of the tile's slots in the order of its keys, times 1 / l.  Bound by reading
// the slots (168 MB for 64 drafts over 131001 rows: 44 us, 3.8 TB/s, part of it from L2), by latency where they are few (12 us).
template <int RPT>
__global__ void __launch_bounds__(256, 2) slim_tree_join_kernel(const SlimDecodeParams p, const SlimTreeView t, int mt) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  long long* s_cut = reinterpret_cast<long long*>(smem_raw);       // [P + 1]
  int* s_slot = reinterpret_cast<int*>(s_cut + t.g_pairs + 1);     // [S + P]
  __shared__ int s_n;
  const int tid = threadIdx.x, R = p.H * t.n;
  slim_pdl_trigger();
  slim_pdl_wait();
  SumSched s;
  s.batch = p.batch; s.tiles = t.g_tiles; s.S = t.g_split; s.P = t.g_pairs; s.F = t.g_whole; s.TS = p.batch * t.g_tiles * t.g_split;
  const int at = blockIdx.x + (s.S == 1 ? s.F : 0), b = at / s.tiles, tile = at % s.tiles;
  const int row0 = (tile / t.g_ncol) * mt * 256 + blockIdx.y * 4 * RPT, col0 = (tile % t.g_ncol) * SU_COLS;
  if (row0 >= R) return;
  for (int q = tid; q <= s.P; q += 256) s_cut[q] = t.sched[p.batch + 1 + q];
  const int nk = stages_of(t.len[b]);
  const long long pre_b = t.sched[b], g0 = t.sched[p.batch + s.P + 2];
  __syncthreads();
  if (tid < 32) {
    int cnt = 0;
    for (int part = 0; part < s.S; ++part) {
      const int idx = (b * s.S + part) * s.tiles + tile;
      const int k0 = part_begin(nk, part, s.S), k1 = part_begin(nk, part + 1, s.S);
      if (k0 == k1) continue;
      if (idx < s.F) {
        if (s.S > 1) { if (tid == 0) s_slot[cnt] = 2 * s.P + idx; ++cnt; }
        continue;
      }
      const long long x0 = pre_b + (long long)s.tiles * k0 + (long long)tile * (k1 - k0) - g0, x1 = x0 + (k1 - k0);
      for (int q0 = 0; q0 < s.P; q0 += 32) {               // the pairs whose segments meet [x0, x1), in order
        const int q = q0 + tid;
        const long long a = q < s.P ? max(s_cut[q], x0) : 0, z = q < s.P ? min(s_cut[q + 1], x1) : 0;
        const bool whole = a == x0 && z == x1, in = a < z && !(whole && s.S == 1);
        const unsigned hit = __ballot_sync(0xffffffffu, in);
        if (in) s_slot[cnt + __popc(hit & ((1u << tid) - 1u))] = whole ? 2 * s.P + idx : a > x0 ? 2 * q : 2 * q + 1;
        cnt += __popc(hit);
      }
    }
    if (tid == 0) s_n = cnt;
  }
  __syncthreads();
  const int cnt = s_n;
  if (cnt == 0) return;                                    // written as a whole by one pair
  // RPT rows a thread (tid / 64 + 4 m), four columns each; the slots one after another, 16 loads in flight
  const int c = (tid % 64) * 4;
  if (col0 + c >= p.d) return;
  float4 a[RPT];
#pragma unroll
  for (int m = 0; m < RPT; ++m) a[m] = make_float4(0.f, 0.f, 0.f, 0.f);
  const float* src = t.part + (size_t)(blockIdx.y * 4 * RPT + tid / 64) * SU_COLS + c;
  for (int k0 = 0; k0 < cnt; k0 += 16 / RPT) {
    float4 v[16 / RPT][RPT];
#pragma unroll
    for (int k = 0; k < 16 / RPT; ++k) {
      const float* slot = src + (size_t)s_slot[min(k0 + k, cnt - 1)] * mt * 256 * SU_COLS;
#pragma unroll
      for (int m = 0; m < RPT; ++m) v[k][m] = *reinterpret_cast<const float4*>(slot + (size_t)4 * m * SU_COLS);      // (rows behind the last one are in the slot too, and not used)
    }
#pragma unroll
    for (int k = 0; k < 16 / RPT; ++k) {
      if (k0 + k >= cnt) break;
#pragma unroll
      for (int m = 0; m < RPT; ++m) { a[m].x += v[k][m].x; a[m].y += v[k][m].y; a[m].z += v[k][m].z; a[m].w += v[k][m].w; }
    }
  }
#pragma unroll
  for (int m = 0; m < RPT; ++m) {
    const int r = row0 + tid / 64 + 4 * m;
    if (r >= R) continue;
    const float il = t.inv_l[(size_t)b * R + r];
    if (il == 0.f) a[m] = make_float4(0.f, 0.f, 0.f, 0.f);    // (padding is 0 whatever the keys hold)
    const int h = r / t.n, tok = r - h * t.n;
    uint2 hi, lo;
    split2(a[m].x * il, a[m].y * il, hi.x, lo.x);
    split2(a[m].z * il, a[m].w * il, hi.y, lo.y);
    __nv_bfloat16* out = t.uh + (((size_t)h * p.batch + b) * t.n + tok) * p.d + col0 + c;
    *reinterpret_cast<uint2*>(out) = hi;
    *reinterpret_cast<uint2*>(out + (size_t)p.H * p.batch * t.n * p.d) = lo;
  }
}

// ------------------------------------------------------------------------------------------------ o = U W_KV,h
// CTA = (part of the d rows of W_KV,h, head, 128 (sequence, token) rows); the parts form a cluster and add their
// accumulators through distributed shared memory, in order, each the rows it writes.  U comes as two bf16 terms (one
// would cost as much accuracy as the rounding of the output does), both against the same tile of W_KV,h.  16 x 16 rows,
// d = 4096, 32 heads: 34 us for 168 MB of U and weights (4.9 TB/s), a third of it still in L2; a single sequence 9 us (latency).
constexpr int OU_NS = 4, OU_A = 128 * 128, OU_B = 64 * 256;
constexpr uint32_t OU_STAGE = 2 * OU_A + OU_B;
constexpr int OU_LD = 132;                                 // floats per accumulator row in shared memory
constexpr size_t OU_SMEM = 1024 + (size_t)OU_NS * OU_STAGE + 16 * OU_NS + 8 + 32;
static_assert(128 * OU_LD * 4 <= OU_NS * (int)OU_STAGE, "the accumulator is staged where the operands were");

__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}

__global__ void __launch_bounds__(128, 1) slim_tree_out_kernel(const __grid_constant__ CUtensorMap umap, const __grid_constant__ CUtensorMap wmap,
                                                            __nv_bfloat16* __restrict__ o, int rows, int d, int d_k, int H, int parts, int* status) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw_u32 = smem_u32(smem_raw), base = (raw_u32 + 1023u) & ~1023u;
  unsigned char* sm = smem_raw + (base - raw_u32);
  const uint32_t bar_full = base + OU_NS * OU_STAGE, bar_empty = bar_full + 8 * OU_NS, bar_done = bar_empty + 8 * OU_NS;
  unsigned char* misc = sm + OU_NS * OU_STAGE + 16 * OU_NS + 8;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(misc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(misc + 4);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int part = blockIdx.x, h = blockIdx.y, m0 = blockIdx.z * 128;
  const int ns = d / 64, s0 = ns * part / parts, s1 = ns * (part + 1) / parts;
  const uint32_t bytes = 2 * OU_A + (d_k == 64 ? OU_B / 2 : OU_B);
  if (tid == 0) {
    prefetch_tensormap(&umap); prefetch_tensormap(&wmap);
    for (int i = 0; i < OU_NS; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    mbar_init(bar_done, 1);
    *s_abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc(smem_u32(s_tmem), 128);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *s_tmem;
  slim_pdl_trigger();
  if (warp == 0 && lane == 0)                              // W_KV is no kernel's output: the first stages' tiles need not wait
    for (int j = 0; j < OU_NS && j < s1 - s0; ++j) {
      mbar_arrive_expect_tx(bar_full + 8 * j, bytes);
      tma_load_3d(base + (uint32_t)j * OU_STAGE + 2 * OU_A, &wmap, bar_full + 8 * j, 0, h * d + (s0 + j) * 64, 0);
    }
  slim_pdl_wait();
  if (warp == 0 && lane == 0) {
    fence_proxy_async_global();
    int s = s0;
    bool ok = true;
    for (; s < s1; ++s) {
      const int j = s - s0, st = j % OU_NS;
      ok = mbar_wait<false>(bar_empty + 8 * st, ((j / OU_NS) & 1) ^ 1, s_abort, status);
      if (!ok) break;
      const uint32_t dst = base + (uint32_t)st * OU_STAGE;
      if (j >= OU_NS) mbar_arrive_expect_tx(bar_full + 8 * st, bytes);
      tma_load_3d(dst, &umap, bar_full + 8 * st, s * 64, m0, h);
      tma_load_3d(dst + OU_A, &umap, bar_full + 8 * st, s * 64, m0, H + h);
      if (j >= OU_NS) tma_load_3d(dst + 2 * OU_A, &wmap, bar_full + 8 * st, 0, h * d + s * 64, 0);
    }
    if (!ok) {
      const int did = s - s0, issued = did < OU_NS ? did : OU_NS;
      for (int k = 0; k < issued; ++k) {
        const int j = did - 1 - k, st = j % OU_NS;
        const unsigned long long tt = globaltimer();
        while (!mbar_try_wait(bar_full + 8 * st, (j / OU_NS) & 1) && globaltimer() - tt < SLIM_WAIT_NS) {}
      }
    }
  } else if (warp == 1 && lane == 0) {
    bool ok = true;
    const uint64_t ad0 = desc_kmajor_sw128(base), bd0 = desc_a(base + 2 * OU_A, 8192);
    const uint32_t a_lo0 = (uint32_t)ad0, a_hi = (uint32_t)(ad0 >> 32), b_lo0 = (uint32_t)bd0, b_hi = (uint32_t)(bd0 >> 32);
    const uint32_t idesc = umma_idesc_major((uint32_t)d_k, 0, 1);
    for (int j = 0; j < s1 - s0; ++j) {
      const int st = j % OU_NS;
      ok = mbar_wait<false>(bar_full + 8 * st, (j / OU_NS) & 1, s_abort, status);
      if (!ok) break;
      tc_fence_after();
      const uint32_t a_lo = a_lo0 + (uint32_t)st * (OU_STAGE >> 4), b_lo = b_lo0 + (uint32_t)st * (OU_STAGE >> 4);
#pragma unroll
      for (int x = 0; x < 8; ++x)
        umma_bf16_words(tmem_base, a_lo + (uint32_t)(x >> 2) * (OU_A >> 4) + (uint32_t)(x & 3) * (32u >> 4), a_hi,
                        b_lo + (uint32_t)(x & 3) * (2048u >> 4), b_hi, idesc, (j | x) ? 1u : 0u);
      umma_commit(bar_empty + 8 * st);
    }
    if (ok) umma_commit(bar_done);
  }
  __syncwarp();
  bool ok = mbar_wait<false>(bar_done, 0, s_abort, status);
  ok = __all_sync(0xffffffffu, ok);
  float* acc = reinterpret_cast<float*>(sm);
  if (ok) {
    tc_fence_after();
    const int r = warp * 32 + lane;
    for (int c0 = 0; c0 < d_k; c0 += 32) {
      uint32_t v[32];
      tmem_ld32(tmem_base + ((uint32_t)(warp * 32) << 16) + (uint32_t)c0, v);
#pragma unroll
      for (int x = 0; x < 32; x += 4) *reinterpret_cast<uint4*>(acc + r * OU_LD + c0 + x) = make_uint4(v[x], v[x + 1], v[x + 2], v[x + 3]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (parts > 1) cluster_sync_all();
  if (ok) {
    const int per = 128 / parts, vecs = d_k / 8;
    for (int e = tid; e < per * vecs; e += 128) {
      const int r = part * per + e / vecs, c = (e % vecs) * 8;
      if (m0 + r >= rows) continue;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
      for (int k = 0; k < parts; ++k) {
        const uint32_t a = mapa(base + (uint32_t)(r * OU_LD + c) * 4u, k);
        const float4 u = ld_cluster_f32x4(a), v = ld_cluster_f32x4(a + 16);
        x.x += u.x; x.y += u.y; x.z += u.z; x.w += u.w;
        y.x += v.x; y.y += v.y; y.z += v.z; y.w += v.w;
      }
      const __nv_bfloat162 o0 = __floats2bfloat162_rn(x.x, x.y), o1 = __floats2bfloat162_rn(x.z, x.w), o2 = __floats2bfloat162_rn(y.x, y.y),
                           o3 = __floats2bfloat162_rn(y.z, y.w);
      *reinterpret_cast<uint4*>(o + (size_t)(m0 + r) * d + h * d_k + c) =
          make_uint4(*reinterpret_cast<const uint32_t*>(&o0), *reinterpret_cast<const uint32_t*>(&o1), *reinterpret_cast<const uint32_t*>(&o2),
                     *reinterpret_cast<const uint32_t*>(&o3));
    }
  }
  if (parts > 1) cluster_sync_all();                       // a CTA's shared memory is read by the others until here
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 128);
  }
}

// Tensor map of whole 16-row tiles of d_k = 96 elements of a head: 192 bytes, wider than a swizzle's rows, so plain ones.
cudaError_t encode_plain_rows(CUtensorMap* map, const void* base, unsigned long long cols, unsigned long long rows) {
  typedef CUresult (*encode_t)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                               const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static encode_t encode = nullptr;
  if (!encode) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (found != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
    encode = (encode_t)fn;
  }
  const cuuint64_t dims[3] = {cols, rows, 1}, strides[2] = {2 * cols, 2 * cols * rows};
  const cuuint32_t box[3] = {96, 16, 1}, step[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, step,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int DK, int NT, bool ROPE>
cudaError_t launch_p(const slim_ctx* ctx, const CUtensorMap& cmap, const CUtensorMap& dmap, const SlimDecodeParams& p, const SlimTreeView& t,
                     const int32_t* parents, cudaStream_t st) {
  constexpr size_t smem = ScoreShape<DK, NT>::SMEM;
  static_assert(smem <= 227 * 1024, "shared memory of an SM");
  auto kern = slim_tree_p_kernel<DK, NT, ROPE>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return slim_launch_pdl(kern, dim3(ctx->num_sms), dim3(ScoreShape<DK, NT>::THREADS), smem, st, cmap, dmap, p, t, parents,
                         reinterpret_cast<const float4*>(ctx->rope_frag));
}
template <int DK>
cudaError_t launch_p_tokens(const slim_ctx* ctx, const SlimDecodeParams& p, const SlimTreeView& t, const int32_t* parents, long long total_rows,
                            cudaStream_t st) {
  CUtensorMap map[2];                                      // cached rows, drafted keys: a warp's tile of 16 rows of one head
  for (int k = 0; k < 2; ++k) {
    const unsigned long long rows = k ? (unsigned long long)p.batch * t.n : (unsigned long long)total_rows;
    const unsigned long long dims[3] = {64, rows, (unsigned long long)(p.d / 64)}, str[2] = {2ull * p.d, 128};
    const unsigned int box[3] = {64, 16, DK == 128 ? 2u : 1u};
    void* base = k ? const_cast<void*>(t.k_tree) : const_cast<void*>(p.k);
    const cudaError_t e = DK == 96 ? encode_plain_rows(&map[k], base, (unsigned long long)p.d, rows) : slim_tmap_encode_3d(&map[k], base, dims, str, box);
    if (e != cudaSuccess) return e;
  }
#define SLIM_P(NT) (p.rope ? launch_p<DK, NT, true>(ctx, map[0], map[1], p, t, parents, st) : launch_p<DK, NT, false>(ctx, map[0], map[1], p, t, parents, st))
  return t.n <= 8 ? SLIM_P(1) : t.n <= 16 ? SLIM_P(2) : t.n <= 32 ? SLIM_P(4) : SLIM_P(8);
#undef SLIM_P
}

template <int MT>
cudaError_t launch_u(const slim_ctx* ctx, const SlimDecodeParams& p, const SlimTreeView& t, const CUtensorMap& pmap, const CUtensorMap& kmap,
                     const CUtensorMap& tailmap, cudaStream_t st) {
  auto kern = slim_tree_u_kernel<MT>;
  const size_t smem = SumShape<MT>::smem(p.batch, t.g_pairs);
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return slim_launch_pdl(kern, dim3(2 * t.g_pairs), dim3(SU_THREADS), smem, st, pmap, kmap, tailmap, p, t);
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

// (cos, sin) of the key offsets 0 .. 127 in the order the score kernel's lanes read them.
cudaError_t slim_tree_make_table(slim_ctx* ctx) {
  const int half = ctx->d_k / 2, vw = ctx->d_k == 96 ? 4 : 8, npc = half / (4 * vw);
  const size_t n = (size_t)SC_KEYS * half / 2;
  float4* host = static_cast<float4*>(malloc(sizeof(float4) * n));
  if (!host) return cudaErrorMemoryAllocation;
  for (size_t e = 0; e < n; ++e) {
    const int ln = e & 31, xq = (int)(e >> 5) % (vw / 2), rest = (int)(e >> 5) / (vw / 2), pc = rest % npc, rh = rest / npc % 2, w = rest / npc / 2;
    const int o = 16 * w + 8 * rh + (ln >> 2), j = chunk_of(ctx->d_k, ln & 3, pc) * vw + 2 * xq;
    const double a = o * std::pow(ctx->rope_theta, -2.0 * j / ctx->d_k), z = o * std::pow(ctx->rope_theta, -2.0 * (j + 1) / ctx->d_k);
    host[e] = make_float4((float)std::cos(a), (float)std::cos(z), (float)std::sin(a), (float)std::sin(z));
  }
  cudaError_t e = cudaMalloc(&ctx->rope_frag, sizeof(float4) * n);
  if (e == cudaSuccess) e = cudaMemcpy(ctx->rope_frag, host, sizeof(float4) * n, cudaMemcpyHostToDevice);
  free(host);
  return e;
}

int slim_tree_tc_ok(const slim_ctx* ctx) {
  return ctx->proj_ok && ctx->kdtype == SLIM_BF16 && ctx->e == ctx->d && ctx->d % 64 == 0;
}

void slim_tree_tc_layout(const slim_ctx* ctx, int batch, int t_cap, int n, SlimTreeLayout& L) {
  const size_t R = (size_t)ctx->H * n;
  const int nb = (t_cap + SC_KEYS - 1) / SC_KEYS;
  L.mt = R > 256 ? 2 : 1;
  L.g_ncol = (ctx->d + SU_COLS - 1) / SU_COLS;
  L.g_tiles = L.g_ncol * (int)((R + L.mt * 256 - 1) / (L.mt * 256));
  L.g_pairs = ctx->num_sms / 2;
  // Fewer tiles than pairs, and more probabilities than stay in L2 beside the keys: every tile is cut into parts of at
  // least eight stages, a part for every pair or more, so that the pairs in flight walk the same 100 MB of P, but no more
  // than five where that suffices: each drains its sums (product and join, 64 drafts over 131001 rows, 537 MB of P: 1.93 ms
  // whole, 1.55 in three parts, 1.50 in five, 1.52 in six; over 70000 rows, 287 MB: 0.79 in three, 0.80 in five; 16 drafts
  // over 4 x 50000 rows, 205 MB: 0.77 whole, 0.61 in three, 0.63 in five).  Otherwise parts only cost (16 drafts over
  // 8 x 12000 rows: 0.30 ms whole, 0.34 ms in three parts).
  const long long tiles = (long long)batch * L.g_tiles;
  const double p_bytes = 2.0 * batch * (double)R * t_cap;
  long long split = 1;
  if (tiles < L.g_pairs && p_bytes > 96e6) {
    const long long each = (L.g_pairs + tiles - 1) / tiles, fit = p_bytes < 5e8 ? (long long)(p_bytes / 1e8) + 1 : 5;
    split = each > fit ? each : fit;
  }
  const long long most = (t_cap / 64 + 2) / 8;
  if (split > most) split = most;
  L.g_split = split < 1 ? 1 : (int)split;
  if (tiles * L.g_split < L.g_pairs) L.g_split = 1;       // (no whole part for every pair: the tiles are cut where the pairs' shares end)
  // whole rounds of tiles; what is left over levels the pairs' loads, so a batch (ragged, perhaps) keeps a quarter of a
  // round for that
  const long long sub = tiles * L.g_split, waves = sub / L.g_pairs - (batch > 1 && sub % L.g_pairs < L.g_pairs / 4 ? 1 : 0);
  L.g_whole = waves > 0 ? (int)(waves * L.g_pairs) : 0;
  L.p_s_draft = nb * SC_KEYS;
  L.p_ld = L.p_s_draft + 64;
  const size_t slots = 2 * (size_t)L.g_pairs + (L.g_split > 1 ? (size_t)sub : 0);
  size_t off = L.shared_end;
  L.p = off; off = align256(off + 2 * (size_t)batch * R * L.p_ld);
  L.stat = off; off = align256(off + 8 * (size_t)batch * (nb + 1) * R);
  L.tail = off; off = align256(off + 2 * (size_t)batch * 128 * ctx->d);
  L.uh = off; off = align256(off + 2 * 2 * (size_t)batch * R * ctx->d);
  L.part = off; off = align256(off + sizeof(float) * slots * L.mt * 256 * SU_COLS);
  L.sched = off; off = align256(off + sizeof(long long) * ((size_t)batch + L.g_pairs + 3));
  if (off > L.total) L.total = off;
}

cudaError_t slim_launch_tree_tc(const slim_ctx* ctx, const SlimDecodeParams& p, const SlimTreeView& t, const SlimTreeLayout& L,
                                const int32_t* parents, long long total_rows, void* o, cudaStream_t st) {
  const int d = p.d, dk = p.d_k, H = p.H, R = H * t.n, M = p.batch * t.n;
  CUtensorMap pmap, kmap, tailmap, umap, wmap;
  cudaError_t e;
  {
    const unsigned long long dims[3] = {(unsigned long long)t.p_ld, (unsigned long long)R, (unsigned long long)p.batch};
    const unsigned long long str[2] = {2ull * t.p_ld, 2ull * t.p_ld * R};
    const unsigned int box[3] = {64, SU_ROWS, 1};
    if ((e = slim_tmap_encode_3d(&pmap, t.p, dims, str, box)) != cudaSuccess) return e;
  }
  for (int k = 0; k < 2; ++k) {
    const unsigned long long dims[3] = {64, k ? 128ull * p.batch : (unsigned long long)total_rows, (unsigned long long)(d / 64)};
    const unsigned long long str[2] = {2ull * d, 128};
    const unsigned int box[3] = {64, p.block_table ? 16u : 64u, 2};
    if ((e = slim_tmap_encode_3d(k ? &tailmap : &kmap, k ? t.tail : const_cast<void*>(p.k), dims, str, box)) != cudaSuccess) return e;
  }
  {
    const unsigned long long dims[3] = {(unsigned long long)d, (unsigned long long)M, 2ull * H};
    const unsigned long long str[2] = {2ull * d, 2ull * d * M};
    const unsigned int box[3] = {64, 128, 1};
    if ((e = slim_tmap_encode_3d(&umap, t.uh, dims, str, box)) != cudaSuccess) return e;
  }
  {   // (d_k = 96: the second half of a row runs into the next one, finite weights that N = 96 leaves out; the allocation is padded)
    const unsigned long long dims[3] = {64, (unsigned long long)H * d, dk == 64 ? 1ull : 2ull};
    const unsigned long long str[2] = {2ull * dk, 128};
    const unsigned int box[3] = {64, 64, dk == 64 ? 1u : 2u};
    if ((e = slim_tmap_encode_3d(&wmap, const_cast<void*>(p.wkv), dims, str, box)) != cudaSuccess) return e;
  }
  e = dk == 64 ? launch_p_tokens<64>(ctx, p, t, parents, total_rows, st) : dk == 96 ? launch_p_tokens<96>(ctx, p, t, parents, total_rows, st)
                                                                          : launch_p_tokens<128>(ctx, p, t, parents, total_rows, st);
  if (e != cudaSuccess) return e;
  const size_t fin_smem = sizeof(long long) * (p.batch + 1 + t.g_pairs + 1) + sizeof(int) * p.batch + 16;
  e = slim_launch_pdl(slim_tree_finish_kernel, dim3((R + 31) / 32 + FIN_TAIL + 1, p.batch), dim3(1024), fin_smem, st, p, t);
  if (e != cudaSuccess) return e;
  e = L.mt == 1 ? launch_u<1>(ctx, p, t, pmap, kmap, tailmap, st) : launch_u<2>(ctx, p, t, pmap, kmap, tailmap, st);
  if (e != cudaSuccess) return e;
  if (L.g_split > 1 || L.g_whole < p.batch * L.g_tiles) {
    const size_t smem = sizeof(long long) * (t.g_pairs + 1) + sizeof(int) * (L.g_split + t.g_pairs) + 16;
    const int tiles = p.batch * L.g_tiles - (L.g_split == 1 ? L.g_whole : 0);          // the others are written as a whole
    // four rows a thread, or one where that leaves SMs without a block (4093 rows, 5 drafts, 80 rows of U: 13.0 -> 11.5 us)
    const int tile_rows = R < L.mt * 256 ? R : L.mt * 256;
    e = (long long)tiles * ((R + 15) / 16) >= ctx->num_sms
            ? slim_launch_pdl(slim_tree_join_kernel<4>, dim3(tiles, (tile_rows + 15) / 16), dim3(256), smem, st, p, t, L.mt)
            : slim_launch_pdl(slim_tree_join_kernel<1>, dim3(tiles, (tile_rows + 3) / 4), dim3(256), smem, st, p, t, L.mt);
    if (e != cudaSuccess) return e;
  }
  // parts of the d rows: as many as leave one CTA an SM (a CTA fills an SM's shared memory), at most four
  const int ns = d / 64, ctas = H * ((M + 127) / 128);
  const int parts = ns >= 4 && 4 * ctas <= ctx->num_sms ? 4 : ns >= 2 && 2 * ctas <= ctx->num_sms ? 2 : 1;
  e = cudaFuncSetAttribute(slim_tree_out_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)OU_SMEM);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(parts, H, (M + 127) / 128); cfg.blockDim = dim3(128); cfg.dynamicSmemBytes = OU_SMEM; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, slim_tree_out_kernel, umap, wmap, (__nv_bfloat16*)o, M, d, dk, H, parts, p.status);
}
