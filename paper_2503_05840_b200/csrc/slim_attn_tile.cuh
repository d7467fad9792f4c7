// Tiles of query rows on CUDA cores: the attention kernel of shapes without tensor cores, and the rows that the tensor-core
// kernel cannot form.
#pragma once
#include "slim_attn.h"
#include "slim_ptx.cuh"

constexpr int SLIM_ATTN_TK = 64;             // keys of a key tile
constexpr int SLIM_ATTN_THREADS = 256;

// TR: query rows of a tile, 64 or 32; DKP: the head width rounded up to a multiple of 64, columns behind d_k are zero.
// Thread (ty, tx) = (tid / 16, tid % 16) has RT = TR / 16 rows, RT ty and the next; scores of keys tx, tx + 16, ..; outputs 4 tx + 64 c.
// Products in packed float32: even and odd columns of a score, neighbouring outputs.
// RAW: queries and keys come from the inputs and are rotated on the way (else from float32 rows, rotated before).
template <int DKP, int TR, bool RAW>
struct SlimAttnTile {
  static constexpr int TK = SLIM_ATTN_TK, NT = SLIM_ATTN_THREADS, PQ = DKP + 4, PP = TK + 4;      // pitches that spread rows over the banks
  static constexpr int NC = DKP / 64, RT = 16 * TR / NT, ST = RAW || DKP > 128 ? 1 : 2;           // key tiles in shared memory (two of wide ones do not fit)
  static constexpr int KS = TK * PQ, VS = TK * DKP;
  static constexpr int SMEM = (int)sizeof(float) * (TR * PQ + ST * (KS + VS) + TR * PP);
  int lim[RT];                               // keys that a row attends
  float m[RT], l[RT];
  slim_ptx::f32x2 acc[RT][NC][2];

  static __device__ __forceinline__ void sync(int bar) { asm volatile("bar.sync %0, %1;" ::"r"(bar), "n"(NT) : "memory"); }
  static __device__ __forceinline__ bool any(int bar, bool x) {
    int y;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbar.red.or.pred q, %2, %3, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
                 : "=r"(y) : "r"((int)x), "r"(bar), "n"(NT) : "memory");
    return y != 0;
  }
  static __device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool in) {          // zeros where `in` does not hold
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
  }
  // Heads of packed rows from `from` on (first element p), rotated to positions pos0 and the next, times f; zeros from row n on
  static __device__ __forceinline__ void rotated(const SlimAttn& a, const void* p, size_t from, int heads, int n, int rows, int pos0, float f, float* to) {
    const int tid = threadIdx.x, dk = a.d_k, half = a.half;
    for (int e = tid; e < rows * (DKP - 2 * half); e += NT) to[e / (DKP - 2 * half) * PQ + 2 * half + e % (DKP - 2 * half)] = 0.f;
#pragma unroll 4
    for (int e = tid; e < rows * half; e += NT) {
      const int r = e / half, j = e - r * half;
      float x1 = 0.f, x2 = 0.f;
      if (r < n) {
        const size_t at = from + (size_t)r * heads * dk + j;
        x1 = slim_attn_ld(p, at, a.f32); x2 = slim_attn_ld(p, at + half, a.f32);
        if (a.rope_base) {
          const float2 t = slim_attn_turn(a, pos0 + r, j);
          const float y = x1 * t.x + x2 * t.y;
          x2 = x2 * t.x - x1 * t.y; x1 = y;
        }
      }
      to[r * PQ + j] = x1 * f; to[r * PQ + half + j] = x2 * f;
    }
  }

  // Sums of query rows row0 .. row0 + rows - 1 of a sequence over its keys first .. end - 1 (first: a multiple of TK), by 256
  // threads that meet at barrier `bar`.
  __device__ __forceinline__ void run(const SlimAttn& a, const SlimSeq& s, int row0, int rows, int h, int first, int end, float* smem, int bar) {
    using namespace slim_ptx;
    float* s_q = smem;                                             // [TR][PQ]
    float* s_k0 = s_q + TR * PQ;                                   // [ST][TK][PQ]
    float* s_v0 = s_k0 + ST * KS;                                  // [ST][TK][DKP]
    float* s_p = s_v0 + ST * VS;                                   // [TR][PP]
    const int dk = a.d_k, kvh = h / (a.H / a.KV), tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const size_t q_at = ((size_t)(s.q0 + row0) * a.H + h) * dk, k_at = ((size_t)s.k0 * a.KV + kvh) * dk;
    const float* kr = reinterpret_cast<const float*>(a.kr) + k_at;
    if (RAW) {
      sync(bar);                                                   // (nobody reads an earlier tile any more)
      rotated(a, a.q, q_at, a.H, rows, TR, row0 + s.nk - s.nq, a.qscale, s_q);
    } else {
      const float* qr = reinterpret_cast<const float*>(a.qr) + q_at;
#pragma unroll 8
      for (int e = tid; e < TR * DKP; e += NT) {
        const int r = e / DKP, c = e % DKP;
        s_q[r * PQ + c] = r < rows && c < dk ? qr[(size_t)r * a.H * dk + c] * a.qscale : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      lim[i] = slim_attn_keys(a, s, row0 + ty * RT + i);
      m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[i][c][0] = acc[i][c][1] = pack2(0.f, 0.f);
    }
    const int keys = min(slim_attn_keys(a, s, row0 + rows - 1), end), least = slim_attn_keys(a, s, row0);
    // Key tile t0 into stage st: 16 bytes at a time behind the products of the tile before it, or element by element (d_k not a
    // multiple of four, bf16 values)
    const bool vec = !RAW && (dk & 3) == 0 && a.v32;
    const float* vr = reinterpret_cast<const float*>(a.v) + k_at;
    auto load = [&](int t0, int st) {
      float* s_k = s_k0 + st * KS;
      float* s_v = s_v0 + st * VS;
      if (vec) {
#pragma unroll 8
        for (int e = tid; e < TK * DKP / 4; e += NT) {
          const int r = e / (DKP / 4), c = e % (DKP / 4) * 4;
          const bool in = t0 + r < keys && c < dk;
          const size_t at = in ? (size_t)(t0 + r) * a.KV * dk + c : 0;
          cp_async16(smem_u32(s_k + r * PQ + c), kr + at, in);
          cp_async16(smem_u32(s_v + r * DKP + c), vr + at, in);
        }
      } else {
        if (RAW) rotated(a, a.k, k_at + (size_t)t0 * a.KV * dk, a.KV, keys - t0, TK, t0, 1.f, s_k);
#pragma unroll 8
        for (int e = tid; e < TK * DKP; e += NT) {
          const int r = e / DKP, c = e % DKP;
          const bool in = t0 + r < keys && c < dk;
          if (!RAW) s_k[r * PQ + c] = in ? kr[(size_t)(t0 + r) * a.KV * dk + c] : 0.f;
          s_v[r * DKP + c] = in ? slim_attn_ld(a.v, k_at + (size_t)(t0 + r) * a.KV * dk + c, a.v32) : 0.f;
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (first < keys) load(first, 0);
    int st = 0;
    for (int t0 = first; t0 < keys; t0 += TK) {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      sync(bar);                                                   // this tile is there, and nobody reads the one before it any more
      const float* s_k = s_k0 + st * KS;
      const float* s_v = s_v0 + st * VS;
      if (ST == 2 && t0 + TK < keys) load(t0 + TK, st ^ 1);
      // Keys that only some of the rows attend: is a value among them not finite?  (0 times it would not be 0.)
      bool apart = false;
      if (min(t0 + TK, keys) > least) {
        bool bad = false;
#pragma unroll 4
        for (int e = tid * 4; e < VS; e += NT * 4) {
          const float4 v = *reinterpret_cast<const float4*>(s_v + e);
          constexpr float most = 3.4028234663852886e38f;
          bad |= !(fabsf(v.x) <= most && fabsf(v.y) <= most && fabsf(v.z) <= most && fabsf(v.w) <= most);
        }
        apart = any(bar, bad);
      }
      f32x2 sv2[RT][4];
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sv2[i][j] = pack2(0.f, 0.f);
#pragma unroll 4
      for (int c = 0; c < DKP; c += 4) {
        ulonglong2 qv[RT], kv[4];
#pragma unroll
        for (int i = 0; i < RT; ++i) qv[i] = *reinterpret_cast<const ulonglong2*>(s_q + (ty * RT + i) * PQ + c);
#pragma unroll
        for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const ulonglong2*>(s_k + (tx + 16 * j) * PQ + c);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) sv2[i][j] = fma2(qv[i].y, kv[j].y, fma2(qv[i].x, kv[j].x, sv2[i][j]));
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        float mx = m[i], sv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sv[j] = t0 + tx + 16 * j >= lim[i] ? -INFINITY : sum2(sv2[i][j]);
          mx = fmaxf(mx, sv[j]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float alpha = mx == m[i] ? 1.f : exp2f(m[i] - mx);
        float ps = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = sv[j] == -INFINITY ? 0.f : exp2f(sv[j] - mx);      // (also where no score of the row was above -inf so far)
          s_p[(ty * RT + i) * PP + tx + 16 * j] = p;
          ps += p;
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, o);
        l[i] = l[i] * alpha + ps;
        m[i] = mx;
        const f32x2 al = pack2(alpha, alpha);
#pragma unroll
        for (int c = 0; c < NC; ++c) { acc[i][c][0] = mul2(acc[i][c][0], al); acc[i][c][1] = mul2(acc[i][c][1], al); }
      }
      __syncwarp();                                                // a row's probabilities come from its own half warp
      if (!apart) {
#pragma unroll 2
        for (int t = 0; t < TK; t += 4) {
          float pv[RT][4];
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(s_p + (ty * RT + i) * PP + t);
            pv[i][0] = v.x; pv[i][1] = v.y; pv[i][2] = v.z; pv[i][3] = v.w;
          }
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(s_v + (t + u) * DKP + c * 64 + tx * 4);
#pragma unroll
              for (int i = 0; i < RT; ++i) {
                const f32x2 pp = pack2(pv[i][u], pv[i][u]);
                acc[i][c][0] = fma2(pp, v.x, acc[i][c][0]);
                acc[i][c][1] = fma2(pp, v.y, acc[i][c][1]);
              }
            }
        }
      } else {                                                     // each row takes what it attends
#pragma unroll 1
        for (int t = 0; t < TK; ++t)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(s_v + t * DKP + c * 64 + tx * 4);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
              const float p = s_p[(ty * RT + i) * PP + t];
              if (t0 + t < lim[i]) {
                acc[i][c][0] = fma2(pack2(p, p), v.x, acc[i][c][0]);
                acc[i][c][1] = fma2(pack2(p, p), v.y, acc[i][c][1]);
              }
            }
          }
      }
      if (ST == 2) {
        st ^= 1;
      } else if (t0 + TK < keys) {
        sync(bar);
        load(t0 + TK, 0);
      }
    }
  }

  // Rows of the tile whose bit in `which` is set, from the sums of all their keys
  __device__ __forceinline__ void store(const SlimAttn& a, const SlimSeq& s, int row0, int rows, int h, unsigned long long which) const {
    const int dk = a.d_k, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int r = ty * RT + i;
      const float inv = lim[i] > 0 ? 1.f / l[i] : 0.f;
      if (r >= rows || !(which >> r & 1)) continue;
      const size_t at = ((size_t)(s.q0 + row0 + r) * a.H + h) * dk;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int col = c * 64 + tx * 4 + x;
          float lo, hi;
          asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(acc[i][c][x >> 1]));
          const float y = lim[i] > 0 ? (x & 1 ? hi : lo) * inv : 0.f;
          if (col < dk) {
            if (a.f32) reinterpret_cast<float*>(a.o)[at + col] = y;
            else reinterpret_cast<__nv_bfloat16*>(a.o)[at + col] = __float2bfloat16_rn(y);
          }
        }
    }
  }
};
