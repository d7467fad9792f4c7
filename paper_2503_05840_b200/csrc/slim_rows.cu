// Rows into and out of a K-cache: packed rows of several sequences (slim_append_rows, slim_read_rows) for float32, bf16
// and 4-bit caches, and the uniform append of a 4-bit cache (slim_append_k, slim_decode_step, slim_prefill).
//
// What HBM has to move: a row of d bf16 keys (2 d bytes) one way and d/2 + d/32 bytes the other.  A warp takes 256 columns of a
// row at a time, four such chunks in flight: 16 bytes a lane on the wide side, one 32-bit word of eight codes on the other; four
// lanes share a scale.
// Measured, rows of 4096: 37.5k rows written 92 us (389 MB, 4.2 TB/s: the issue slots are 77 % full, the rounding's steps; more
// warps an SM changed nothing) and read back 65 us (6.0 TB/s, 0.92 of a copy); 31k rows in pages read in 54 us; 16 rows 5 us
// either way (three dependent loads: start, position, page).  One prompt, 2000 rows: written in 7.6 us, read back in 5.0.  Rows of a bf16
// cache, both ways: 37.5k of 4096 101 us (6.1 TB/s), 2000 5.1 us, 9500 of 1280 6.4 us.
#include "slim_fp4.cuh"
#include "slim_ptx.cuh"

namespace {

struct RowsArgs {
  void* wide;                    // [total][d] packed rows (f32 or bf16): source of an append, destination of a read
  const int32_t* positions;      // [batch] first cache row of a sequence
  const int32_t* cu;             // [batch + 1] packed row where a sequence begins; NULL: n_new rows each
  int n_new, pos_is_length;      // uniform form; positions hold the lengths after the append
  int total, batch, d, t_cap;
  unsigned char* codes;          // cache rows (f32 and bf16 caches: the keys)
  unsigned char* scales;
  int pitch, spitch;             // bytes of a row
  const int32_t* block_table;
  int page_rows, max_pages, num_pages;
  int* status;
  int parts, chunks;             // a warp's share of a row: chunks of 256 columns (copies: of 512 bytes)
};

// Cache row of packed row r; -1 if it has none (outside every sequence, or not to be touched).  All lanes of a warp agree.
__device__ long long rows_target(const RowsArgs& a, int r) {
  int b, i, n;
  if (a.cu) {
    b = slim_warp_find(a.cu, a.batch, r);
    const int first = a.cu[b], end = a.cu[b + 1];
    if (first < 0 || r < first || r >= end || end > a.total) return -1;
    i = r - first; n = end - first;
  } else {
    b = r / a.n_new; i = r - b * a.n_new; n = a.n_new;
  }
  int pos = a.positions[b];
  if (a.pos_is_length) {
    if (pos <= 0) return -1;
    pos -= 1;
  }
  if (pos < 0 || n > a.t_cap || pos > a.t_cap - n) { atomicMax(a.status, (int)SLIM_ERR_CAPACITY); return -1; }
  const int t = pos + i;
  if (!a.block_table) return (long long)b * a.t_cap + t;
  const int pg = a.block_table[(size_t)b * a.max_pages + t / a.page_rows];
  if (pg < 0 || pg >= a.num_pages) { atomicMax(a.status, (int)SLIM_ERR_CAPACITY); return -1; }
  return (long long)pg * a.page_rows + t % a.page_rows;
}

// The warp's row and part of it (below 2^31 warps: at most 2^30 rows, and parts only where they are few)
__device__ __forceinline__ bool rows_share(const RowsArgs& a, int& r, int& part) {
  const unsigned w = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5), parts = (unsigned)a.parts;
  r = (int)(parts == 1 ? w : w / parts);
  part = (int)(w - (unsigned)r * parts);
  return r < a.total;
}

// Starts of packed sequences that do not ascend from 0 to at most `total` are reported (their rows are left out above).
// By the last block, which has no rows.
__device__ void rows_check(const RowsArgs& a) {
  if (!a.cu || blockIdx.x != gridDim.x - 1) return;
  for (int b = threadIdx.x; b < a.batch; b += blockDim.x)
    if (a.cu[b] < 0 || a.cu[b + 1] < a.cu[b] || a.cu[b + 1] > a.total) atomicMax(a.status, (int)SLIM_ERR_CAPACITY);
}

// 256 columns of a row: eight a lane, from bf16 rows of any alignment
__device__ __forceinline__ uint4 load8(const unsigned short* row, int col, int d, bool whole) {
  if (whole) return __ldcs(reinterpret_cast<const uint4*>(row + col));
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  for (int e = 0; e < 8 && col + e < d; ++e) w[e >> 1] |= (uint32_t)row[col + e] << (16 * (e & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Eight keys and the largest magnitude of their group -> codes and the scale byte.
// Codes are rounded by the conversion instruction, from k / s as k times the reciprocal of s.  That is off by some 2^-22,
// which only matters on a border between two codes (k is a bf16 number, of 8 bits, and border times scale has 7: k / s is the
// border itself or further than 2^-8 of it away).  Rounding to multiples of 2^-12 first brings the border's quotients
// back onto it and leaves the others on their side.
__device__ __forceinline__ uint32_t quantise8(const uint4& v, float amax, int& byte) {
  const bool bad = !(amax <= 3.4028234663852886e38f);
  byte = slim_fp4_scale_byte(amax, bad);
  const float s = slim_fp4_scale((unsigned char)byte);
  const float up = bad || !(amax > 0.f) ? 0.f : __fdividef(1.f, s);
  const slim_ptx::f32x2 up2 = slim_ptx::pack2(up, up), magic = slim_ptx::pack2(0x1.8p11f, 0x1.8p11f);      // float32 steps of 2^-12 around it
  const slim_ptx::f32x2 back = slim_ptx::pack2(-0x1.8p11f, -0x1.8p11f);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float y[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const slim_ptx::f32x2 k = slim_ptx::pack2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u));
    const slim_ptx::f32x2 z = slim_ptx::add2(slim_ptx::fma2(k, up2, magic), back);
    asm("mov.b64 {%0, %1}, %2;" : "=f"(y[2 * e]), "=f"(y[2 * e + 1]) : "l"(z));
  }
  const uint32_t out = slim_fp4_encode8(y);
  if (bad) return 0u;
  // codes of magnitude 0 have no sign
  const uint32_t some = (out | (out >> 1) | (out >> 2)) & 0x11111111u;
  return out & (0x77777777u | (some << 3));
}

// bf16 rows -> 4 bits; CH: chunks of 256 columns whose loads are in flight together; RAGGED: a warp's share is no multiple of it
// (37.5k rows of 4096: 82 us, 85 with the test for the end of the share between the chunks)
template <int CH, bool RAGGED>
__global__ void __launch_bounds__(256) rows_quantise_kernel(const RowsArgs a) {
  slim_pdl_trigger();
  slim_pdl_wait();
  rows_check(a);
  const int lane = threadIdx.x & 31;
  int rr, part;
  if (!rows_share(a, rr, part)) return;
  const unsigned short* src = reinterpret_cast<const unsigned short*>(a.wide) + (size_t)rr * a.d;
  const bool whole = (a.d & 7) == 0 && ((uintptr_t)a.wide & 15) == 0;
  const long long row = rows_target(a, rr);
  if (row < 0) return;
  unsigned char* dst = a.codes + (size_t)row * a.pitch;
  unsigned char* sdst = a.scales + (size_t)row * a.spitch;
  const int end = RAGGED ? min(a.d, (part + 1) * a.chunks * 256) : a.d;      // where the warp's share ends
  for (int c0 = 0; c0 < a.chunks; c0 += CH) {
    uint4 v[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (part * a.chunks + c0 + c) * 256 + lane * 8;
      v[c] = col < end ? load8(src, col, a.d, whole) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (RAGGED && c0 + c >= a.chunks) break;                         // (all lanes)
      const int col = (part * a.chunks + c0 + c) * 256 + lane * 8;
      // largest magnitude of the group's 32 columns, NaN if there is one: the sign cleared, the bits of bf16 numbers order as integers
      uint32_t m = __vmaxu2(__vmaxu2(v[c].x & 0x7fff7fffu, v[c].y & 0x7fff7fffu), __vmaxu2(v[c].z & 0x7fff7fffu, v[c].w & 0x7fff7fffu));
      m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 2));
      const float amax = __uint_as_float(max(m << 16, m & 0xffff0000u));
      int byte;
      const uint32_t out = quantise8(v[c], amax, byte);
      if (col < end) {
        if (col + 8 <= a.d) *reinterpret_cast<uint32_t*>(dst + (col >> 1)) = out;
        else
          for (int e = 0; 2 * e < a.d - col; ++e) dst[(col >> 1) + e] = (unsigned char)(out >> (8 * e));
        if ((lane & 3) == 0) sdst[col / FP4_GROUP] = (unsigned char)byte;
      }
    }
  }
}

// 4 bits -> bf16 rows (exact: a value has six significant bits)
template <int CH>
__global__ void __launch_bounds__(256) rows_expand_kernel(const RowsArgs a) {
  slim_pdl_trigger();
  slim_pdl_wait();
  rows_check(a);
  const int lane = threadIdx.x & 31;
  int rr, part;
  if (!rows_share(a, rr, part)) return;
  const long long row = rows_target(a, rr);
  if (row < 0) return;
  unsigned short* dst = reinterpret_cast<unsigned short*>(a.wide) + (size_t)rr * a.d;
  const unsigned char* src = a.codes + (size_t)row * a.pitch;
  const unsigned char* ssrc = a.scales + (size_t)row * a.spitch;
  const bool whole = (a.d & 7) == 0 && ((uintptr_t)a.wide & 15) == 0;
  const int end = min(a.d, (part + 1) * a.chunks * 256);               // where the warp's share ends
  for (int c0 = 0; c0 < a.chunks; c0 += CH) {
    uint32_t v[CH], s[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (part * a.chunks + c0 + c) * 256 + lane * 8;
      v[c] = col < end ? __ldcs(reinterpret_cast<const unsigned int*>(src + (col >> 1))) : 0u;      // (rows are padded to 16 bytes)
      s[c] = col < end ? __ldg(ssrc + col / FP4_GROUP) : 0u;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (c0 + c >= a.chunks) break;
      const int col = (part * a.chunks + c0 + c) * 256 + lane * 8;
      if (col >= end) continue;
      const uint32_t scale = s[c] * 0x00800080u;                       // a float16 pair
      uint32_t h[4], out[4];
      slim_fp4_decode8(v[c], h);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&h[e]), *reinterpret_cast<const __half2*>(&scale));
        const float2 f = __half22float2(x);
        const __nv_bfloat162 y = __floats2bfloat162_rn(f.x, f.y);
        out[e] = *reinterpret_cast<const uint32_t*>(&y);
      }
      if (whole) __stcs(reinterpret_cast<uint4*>(dst + col), make_uint4(out[0], out[1], out[2], out[3]));
      else
        for (int e = 0; e < 8 && col + e < a.d; ++e) dst[col + e] = (unsigned short)(out[e >> 1] >> (16 * (e & 1)));
    }
  }
}

// rows of a float32 or bf16 cache, to it or from it, in units of U bytes
template <typename U>
__global__ void __launch_bounds__(256) rows_copy_kernel(const RowsArgs a, int to_cache) {
  slim_pdl_trigger();
  slim_pdl_wait();
  rows_check(a);
  const int lane = threadIdx.x & 31;
  int rr, part;
  if (!rows_share(a, rr, part)) return;
  const long long row = rows_target(a, rr);
  if (row < 0) return;
  const int units = a.pitch / (int)sizeof(U);
  U* cache = reinterpret_cast<U*>(a.codes + (size_t)row * a.pitch);
  U* wide = reinterpret_cast<U*>(reinterpret_cast<unsigned char*>(a.wide) + (size_t)rr * a.pitch);
  U* dst = to_cache ? cache : wide;
  const U* src = to_cache ? wide : cache;
#pragma unroll 4
  for (int c = 0; c < a.chunks; ++c) {
    const int i = (part * a.chunks + c) * 32 + lane;
    if (i < units) dst[i] = src[i];
  }
}

cudaError_t launch_rows(const slim_ctx* ctx, RowsArgs a, int to_cache, cudaStream_t st) {
  if (a.total <= 0) return cudaSuccess;
  const bool fp4 = ctx->kdtype == SLIM_FP4;
  size_t unit = 16;
  if (!fp4) while ((a.pitch % unit) || (((uintptr_t)a.wide | (uintptr_t)a.codes) % unit)) unit >>= 1;
  const int span = fp4 ? 256 : 32;                                     // columns (units) a warp takes at a time
  const int n = ((fp4 ? a.d : a.pitch / (int)unit) + span - 1) / span;
  // A row a warp where the rows alone give every SM 64 warps (the row's place is then looked up once); with fewer rows they are
  // split, down to four chunks a warp, whose loads are in flight together, and to one where an SM has fewer than 96 of them
  // (2367 rows of 4096, 4 bits: written in 8.2 us by four, 10.2 by two; 900 rows 5.4 either way; 2367 rows of 1280 5.2 and 4.4).
  const int four = (n + 3) / 4, least = (n + four - 1) / four;
  a.chunks = n;
  while (a.chunks > least && (long long)a.total * ((n + a.chunks - 1) / a.chunks) < 64ll * ctx->num_sms) a.chunks = (a.chunks + 1) / 2 > least ? (a.chunks + 1) / 2 : least;
  if ((long long)a.total * n < 96ll * ctx->num_sms) a.chunks = 1;
  a.parts = (n + a.chunks - 1) / a.chunks;
  const long long warps = (long long)a.total * a.parts;
  const dim3 grid((unsigned)((warps + 7) / 8) + 1), block(256);
  if (fp4 && a.chunks == 1) return slim_launch_pdl(to_cache ? rows_quantise_kernel<1, false> : rows_expand_kernel<1>, grid, block, 0, st, a);
  if (fp4 && !to_cache) return slim_launch_pdl(rows_expand_kernel<4>, grid, block, 0, st, a);
  if (fp4) return slim_launch_pdl(a.chunks % 4 == 0 ? rows_quantise_kernel<4, false> : rows_quantise_kernel<4, true>, grid, block, 0, st, a);
  switch (unit) {
    case 16: return slim_launch_pdl(rows_copy_kernel<uint4>, grid, block, 0, st, a, to_cache);
    case 8: return slim_launch_pdl(rows_copy_kernel<uint2>, grid, block, 0, st, a, to_cache);
    case 4: return slim_launch_pdl(rows_copy_kernel<uint32_t>, grid, block, 0, st, a, to_cache);
    default: return slim_launch_pdl(rows_copy_kernel<unsigned short>, grid, block, 0, st, a, to_cache);
  }
}

RowsArgs rows_args(const slim_ctx* ctx, const slim_cache* c, void* wide, const int32_t* positions) {
  RowsArgs a = {};
  a.wide = wide; a.positions = positions;
  a.batch = c->batch; a.d = ctx->d; a.t_cap = c->t_cap;
  a.codes = reinterpret_cast<unsigned char*>(c->k); a.scales = c->k_sc4;
  a.pitch = ctx->kdtype == SLIM_FP4 ? slim_fp4_code_pitch(ctx->d) : ctx->d * (ctx->dtype == SLIM_BF16 ? 2 : 4);
  a.spitch = slim_fp4_scale_pitch(ctx->d);
  a.block_table = c->block_table; a.page_rows = c->page_rows; a.max_pages = c->max_pages; a.num_pages = c->num_pages;
  a.status = ctx->status;
  return a;
}

}  // namespace

cudaError_t slim_launch_rows(const slim_ctx* ctx, const slim_cache* c, void* wide, const int32_t* positions, const int32_t* cu, int total,
                             int to_cache, cudaStream_t st) {
  RowsArgs a = rows_args(ctx, c, wide, positions);
  a.cu = cu; a.total = total;
  return launch_rows(ctx, a, to_cache, st);
}

cudaError_t slim_launch_append_fp4(const slim_ctx* ctx, const slim_cache* c, const void* k_new, const int32_t* positions, int n_new,
                                   int pos_is_length, cudaStream_t st) {
  RowsArgs a = rows_args(ctx, c, const_cast<void*>(k_new), positions);
  a.n_new = n_new; a.pos_is_length = pos_is_length; a.total = c->batch * n_new;
  return launch_rows(ctx, a, 1, st);
}
