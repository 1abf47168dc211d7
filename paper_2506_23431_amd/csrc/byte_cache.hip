// A cache of keys and values in 8 bits: storing tokens, reading them back, attention over them.
//
// Per request and key head, tokens lie in blocks of 64.  A whole block holds signed codes of 8 bits and one fp32 scale for its
// keys, one for its values; the tokens behind the last whole block are halves in a tail of two slots (block b: slot b & 1).
// Everything lies in the order in which 16 lanes of a wave load 256 bytes that are operands of the matrix instruction (any order
// of a contraction is right that both operands share):
//   k       [block][hd / 16][64 tokens][16 dims]        k_tail  [2][hd / 8][64][8 dims] half
//   v       [block][4][hd][16 tokens]                   v_tail  [2][2][4][hd][8 tokens] half
// where place i of group g of a value's tokens is token 16 (i >> 2) + 4 g + (i & 3) of the block (tails: the first 8 places, then
// the others): the scores leave the matrix instruction in this order, and it is that of the operand for the outputs.
// Rows of [64][hd] and [hd][64] instead, where neighbouring lanes load pieces of different rows: 16384 tokens of one head of size
// 128 in one work-group of 8 waves 107 us against 73, 32 x 8 heads x 8192 tokens 76.8 against 71.0.
#include "byte_cache.h"

#include <algorithm>
#include <type_traits>

// ---------------------------------------------------------------------------
// store
// ---------------------------------------------------------------------------
struct StoreArgs {
  ByteCache c;
  const void *src[2];                 // new keys, new values
  int64_t s_req[2], s_tok[2], s_head[2];
  const int32_t *counts, *lens;
  int n_new, span;                    // most new tokens; blocks that they can touch
};

// Codes of N halves: the whole numbers nearest to x / s, ties to even, exactly.  The product with the reciprocal is at most one
// off, and the remainder, a whole multiple of the scale's last bit below 2^24 of them, is computed without rounding: below half
// a scale it proves the number; else (next to a border between two, about one in 10^5) the neighbours are compared.
template <int N>
__device__ __forceinline__ void codes_of(const f16_t *x, float s, float inv, int *c) {
  float worst = 0.f;
  const float h = 0.5f * s;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float q = rintf((float)x[j] * inv);
    worst = fmaxf(worst, fabsf(fmaf(-q, s, (float)x[j])));
    c[j] = (int)q;
  }
  if (worst >= h)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float r = fmaf(-(float)c[j], s, (float)x[j]);
      const bool odd = (c[j] & 1) != 0;
      c[j] += (r > h || (r == h && odd)) ? 1 : (r < -h || (r == -h && odd)) ? -1 : 0;
      c[j] = min(max(c[j], -127), 127);
    }
}
__device__ __forceinline__ uint32_t magnitude(f16_t x) { return __builtin_bit_cast(uint16_t, x) & 0x7fffu; }

__device__ __forceinline__ uint32_t bytes4(int a, int b, int c, int d) {
  const uint32_t lo = __builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x0c0c0400u), hi = __builtin_amdgcn_perm((uint32_t)d, (uint32_t)c, 0x04000c0cu);
  return lo | hi;
}

// A whole block, by tokens in LDS (P halves a row), and each thread's largest magnitude: codes and scale.
template <int HD, int P>
__device__ __forceinline__ void seal_block(const f16_t *tile, uint32_t *sm_top, uint32_t top, int kind, const ByteCache &cache, size_t block) {
  const int tid = threadIdx.x;
  // the largest magnitude by its bits, where NaN is above everything: then the scale is NaN, and so is the block
  for (int m = 32; m; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  if ((tid & 63) == 0) sm_top[tid >> 6] = top;
  __syncthreads();
  top = max(max(sm_top[0], sm_top[1]), max(sm_top[2], sm_top[3]));
  const float scale = __fdiv_rn((float)__builtin_bit_cast(f16_t, (uint16_t)top), 127.f);
  const float inv = 1.f / scale;
  if (tid == 0) (kind ? cache.v_scale : cache.k_scale)[block] = scale;
  int8_t *dst = (kind ? cache.v : cache.k) + block * BYTE_BLOCK * HD;
  if (!(scale > 0.f)) {                                // zeros, or a NaN among them: codes of zero
    for (int e = tid; e < BYTE_BLOCK * HD / 16; e += 256) ((uint4 *)dst)[e] = make_uint4(0, 0, 0, 0);
  } else if (!kind) {
    for (int e = tid; e < BYTE_BLOCK * HD / 16; e += 256) {        // 16 dims of a token
      union { uint4 q[2]; f16_t h[16]; } y;
      const f16_t *row = &tile[(e & 63) * P + (e >> 6) * 16];
      y.q[0] = *(const uint4 *)row; y.q[1] = *(const uint4 *)(row + 8);
      int c[16];
      codes_of<16>(y.h, scale, inv, c);
      ((uint4 *)dst)[e] = make_uint4(bytes4(c[0], c[1], c[2], c[3]), bytes4(c[4], c[5], c[6], c[7]),
                                     bytes4(c[8], c[9], c[10], c[11]), bytes4(c[12], c[13], c[14], c[15]));
    }
  } else {
    for (int e = tid; e < BYTE_BLOCK * HD / 32; e += 256) {        // 8 places of 4 dims
      const int half = e & 1, d = (e >> 1) % (HD / 4) * 4, g = (e >> 1) / (HD / 4);
      f16_t x4[4][8];
      int c[4][8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        union { uint2 q; f16_t h[4]; } z;
        z.q = *(const uint2 *)&tile[(16 * (2 * half + (j >> 2)) + 4 * g + (j & 3)) * P + d];
#pragma unroll
        for (int i = 0; i < 4; ++i) x4[i][j] = z.h[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) codes_of<8>(x4[i], scale, inv, c[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(uint2 *)(dst + (g * HD + d + i) * 16 + half * 8) =
            make_uint2(bytes4(c[i][0], c[i][1], c[i][2], c[i][3]), bytes4(c[i][4], c[i][5], c[i][6], c[i][7]));
    }
  }
}

// One work-group per (request, head, touched block, keys or values): the block's tokens go to LDS as halves, the old ones from
// the tail, the new ones from the caller (all requested before the first is used); a whole block leaves as codes, one that is not
// yet whole as halves of its new tokens.  Bound by the bytes: 8192 tokens of 16 fp32 heads of 128 in 42.5 us, 3.9 TB/s of the 4.9 that
// a copy reaches; 16 tokens of 4 x 32 bf16 heads of 128 5.8 us, one token of 12 heads of 64 3.3 us, which is a launch's least.
template <typename T, int HD, bool WIDE>
__global__ __launch_bounds__(256, 3) void k_byte_store(StoreArgs a) {
  constexpr int P = HD + 8;                              // halves per token row in LDS (16-byte rows)
  constexpr int IT = HD / 32;                            // pieces of 8 dims per thread
  __shared__ f16_t tile[BYTE_BLOCK * P];
  __shared__ uint32_t sm_top[4];
  const int tid = threadIdx.x;
  int u = blockIdx.x;                                    // heads first: their rows lie together
  const int h = u % a.c.n_kv_head; u /= a.c.n_kv_head;
  const int kind = u & 1, i0 = (u >> 1) % a.span, req = (u >> 1) / a.span;
  const int count = a.counts ? a.counts[req] : a.n_new, len = a.lens[req];
  if (!byte_append_fits(len, count, a.n_new, a.c.n_block)) return;
  const int before = len - count;
  const int first = before / BYTE_BLOCK, last = (len - 1) / BYTE_BLOCK;      // touched blocks
  const bool part = len % BYTE_BLOCK != 0;               // the last one stays in the tail
  // A last block with the first one's slot in the tail is stored by the work-group that has read that slot.
  const bool shared_slot = part && last > first && ((last - first) & 1) == 0;
  if (first + i0 > last || (shared_slot && i0 > 0 && first + i0 == last)) return;
  const size_t rhz = (size_t)req * a.c.n_kv_head + h;
  const T *src = (const T *)(kind ? a.src[1] : a.src[0]) + req * a.s_req[kind] + h * a.s_head[kind];
  const int64_t s_tok = a.s_tok[kind];
  f16_t *tail0 = (f16_t *)(kind ? a.c.v_tail : a.c.k_tail) + rhz * 2 * BYTE_BLOCK * HD;
  for (int pass = 0; pass < (i0 == 0 && shared_slot ? 2 : 1); ++pass) {
    const int b = pass ? last : first + i0, t0 = b * BYTE_BLOCK;
    const bool whole = t0 + BYTE_BLOCK <= len;
    const int n_old = min(max(before - t0, 0), BYTE_BLOCK), n_all = min(len - t0, BYTE_BLOCK);
    f16_t *tail = tail0 + (size_t)(b & 1) * BYTE_BLOCK * HD;
    if (pass) __syncthreads();
    float x[IT][8];
    uint4 old[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) {                    // new tokens (others: any new one's, not used)
      const int e = tid + it * 256, t = e / (HD / 8), d = e % (HD / 8) * 8;
      load8<T, WIDE>(src + (int64_t)min(max(t0 + t - before, 0), count - 1) * s_tok + d, x[it]);
    }
    const bool mixed = whole && n_old > 0;               // (the same for the whole work-group)
    if (mixed)
#pragma unroll
      for (int it = 0; it < IT; ++it) old[it] = ((const uint4 *)tail)[tid + it * 256];
    uint32_t top = 0;
    union Eight { f16_t h[8]; uint4 q; } y[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int t = (tid + it * 256) / (HD / 8);
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) { y[it].h[j] = (f16_t)x[it][j]; m = max(m, magnitude(y[it].h[j])); }
      top = max(top, t < n_old || t >= n_all ? 0u : m);
    }
    if (top >= 0x7c00u) {                                // beyond the halves: saturated; NaN stays
      top = 0;
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int t = (tid + it * 256) / (HD / 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (magnitude(y[it].h[j]) == 0x7c00u) y[it].h[j] = (f16_t)(x[it][j] > 0.f ? 65504.f : -65504.f);
          if (t >= n_old && t < n_all) top = max(top, magnitude(y[it].h[j]));
        }
      }
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + it * 256, t = e / (HD / 8), d = e % (HD / 8) * 8;
      if (t < n_old || t >= n_all) continue;
      if (whole) *(uint4 *)&tile[t * P + d] = y[it].q;
      else if (!kind) *(uint4 *)(tail + ((d >> 3) * BYTE_BLOCK + t) * 8) = y[it].q;
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) tail[(((t >> 5) * 4 + ((t >> 2) & 3)) * HD + d + j) * 8 + ((t >> 4) & 1) * 4 + (t & 3)] = y[it].h[j];
    }
    if (!whole) continue;
    if (mixed) {                                         // ... and the ones that were in the tail
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int e = tid + it * 256;
        union { uint4 q; f16_t h[8]; } y;
        y.q = old[it];
        if (!kind) {
          const int t = e & 63, d = (e >> 6) * 8;
          if (t >= n_old) continue;
          *(uint4 *)&tile[t * P + d] = y.q;
#pragma unroll
          for (int j = 0; j < 8; ++j) top = max(top, magnitude(y.h[j]));
        } else {
          const int d = e % HD, sg = e / HD;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int t = 16 * (2 * (sg >> 2) + (j >> 2)) + 4 * (sg & 3) + (j & 3);
            if (t >= n_old) continue;
            tile[t * P + d] = y.h[j];
            top = max(top, magnitude(y.h[j]));
          }
        }
      }
    }
    seal_block<HD, P>(tile, sm_top, top, kind, a.c, rhz * a.c.n_block + b);
  }
}

// ---------------------------------------------------------------------------
// read
// ---------------------------------------------------------------------------
struct ReadArgs {
  ByteCache c;
  void *out[2];                       // [req][n_tok][head][hd]
  const int32_t *first, *lens;
  int n_tok, span;
};

// One work-group per (request, head, block that the range can touch, keys or values): the block goes to LDS by tokens, a whole
// one as bytes, and leaves by rows of a token's dims.  Bound by the bytes: 4 requests of up to 4096 tokens of 32 heads of 128 to
// bf16 in 74 us, 4.9 TB/s, a copy's rate; 300 tokens of 2 x 12 heads of 64 3.7 us.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_byte_read(ReadArgs a) {
  constexpr int P = HD + 8, PB = HD + 16;                // halves, bytes per token row in LDS
  __shared__ uint4 mem[BYTE_BLOCK * P / 8];
  f16_t *tile = (f16_t *)mem;
  int8_t *codes = (int8_t *)mem;
  const int tid = threadIdx.x;
  int u = blockIdx.x;                                    // heads first: their rows lie together
  const int h = u % a.c.n_kv_head; u /= a.c.n_kv_head;
  const int kind = u & 1, i0 = (u >> 1) % a.span, req = (u >> 1) / a.span;
  const int64_t cap = (int64_t)a.c.n_block * BYTE_BLOCK;
  const int len = (int)min((int64_t)max(a.lens[req], 0), cap);
  const int from = a.first ? max(a.first[req], 0) : 0;
  const int64_t b = from / BYTE_BLOCK + i0, t0 = b * BYTE_BLOCK;
  if (t0 >= (int64_t)from + a.n_tok) return;
  const size_t rhz = (size_t)req * a.c.n_kv_head + h;
  const bool whole = t0 + BYTE_BLOCK <= len;
  const int n = (int)min(max((int64_t)len - t0, (int64_t)0), (int64_t)BYTE_BLOCK);
  float scale = 1.f;
  if (whole) {
    scale = (kind ? a.c.v_scale : a.c.k_scale)[rhz * a.c.n_block + b];
    const uint4 *src = (const uint4 *)((kind ? a.c.v : a.c.k) + (rhz * a.c.n_block + b) * BYTE_BLOCK * HD);
    if (!kind) {
#pragma unroll
      for (int it = 0; it < (HD + 63) / 64; ++it) {
        const int e = tid + it * 256;
        if (HD % 64 == 0 || e < HD * 4) *(uint4 *)&codes[(e & 63) * PB + (e >> 6) * 16] = src[e];
      }
    } else if (tid < HD) {                               // 16 places of 4 dims, turned
      const int d = tid % (HD / 4) * 4, g = tid / (HD / 4);
      uint4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = src[g * HD + d + i];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t p = (&x[0].x)[w], q = (&x[1].x)[w], r = (&x[2].x)[w], z = (&x[3].x)[w];
        const uint32_t pq0 = __builtin_amdgcn_perm(q, p, 0x05010400u), pq1 = __builtin_amdgcn_perm(q, p, 0x07030602u);
        const uint32_t rz0 = __builtin_amdgcn_perm(z, r, 0x05010400u), rz1 = __builtin_amdgcn_perm(z, r, 0x07030602u);
        int8_t *row = &codes[(16 * w + 4 * g) * PB + d];
        *(uint32_t *)row = __builtin_amdgcn_perm(rz0, pq0, 0x05040100u);
        *(uint32_t *)(row + PB) = __builtin_amdgcn_perm(rz0, pq0, 0x07060302u);
        *(uint32_t *)(row + 2 * PB) = __builtin_amdgcn_perm(rz1, pq1, 0x05040100u);
        *(uint32_t *)(row + 3 * PB) = __builtin_amdgcn_perm(rz1, pq1, 0x07060302u);
      }
    }
  } else if (n > 0) {
    const uint4 *src = (const uint4 *)((const f16_t *)(kind ? a.c.v_tail : a.c.k_tail) + (rhz * 2 + (b & 1)) * BYTE_BLOCK * HD);
#pragma unroll
    for (int it = 0; it < HD / 32; ++it) {
      const int e = tid + it * 256;
      union { uint4 q; f16_t h[8]; } y;
      y.q = src[e];
      if (!kind) *(uint4 *)&tile[(e & 63) * P + (e >> 6) * 8] = y.q;
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[(16 * (2 * (e / HD >> 2) + (j >> 2)) + 4 * (e / HD & 3) + (j & 3)) * P + e % HD] = y.h[j];
    }
  }
  __syncthreads();
  T *out = (T *)(kind ? a.out[1] : a.out[0]);
  for (int e = tid; e < BYTE_BLOCK * (HD / 8); e += 256) {
    const int t = e / (HD / 8), d = e % (HD / 8) * 8;
    const int64_t at = t0 + t - from;
    if (at < 0 || at >= a.n_tok) continue;
    float y[8];
    if (whole) {
      union { uint2 q; int8_t c[8]; } x;
      x.q = *(const uint2 *)&codes[t * PB + d];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = (float)x.c[j] * scale;
    } else {
      union { uint4 q; f16_t h[8]; } x;
      x.q = *(const uint4 *)&tile[t * P + d];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = t < n ? (float)x.h[j] : 0.f;
    }
    store8(out + (((size_t)req * a.n_tok + at) * a.c.n_kv_head + h) * HD + d, y);
  }
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
struct ByteAttnArgs {
  ByteCache c;
  const void *q;                      // [req][row][head][hd] by strides
  int64_t q_req, q_row, q_head;
  const int32_t *lens, *row_limit, *row_tag;
  const uint16_t *key_tag;            // [req][n_block * 64]
  void *out;                          // [req][row][head][hd]
  float *lse;                         // [req][row][head] or NULL
  float *part;
  int n_row, group, nqg, qt, nsplit, nblk; // group: query heads per key head; nqg: groups of 16 qt (row, query head) columns
  int q_wide;                              // queries lie at multiples of 16 bytes
  float scale_log2, scale_low;             // log2(e) times the scale, and what its rounding left
  // CTX: a decode step over a decoder's context.  Rows and queries are the step's (fragments of high and low halves), the first
  // nblk blocks of the context are codes, everything behind them lies in the decoder's own cache of halves.
  const f16_t *cq, *cq_lo; bf16_t *cout, *cout_lo;
  const int4 *qinfo; const uint16_t *gen_sub;
  const f16_t *hk, *hv;
  int gen_stride, kv_cap, L, req0;
};

// Four codes as four halves, exactly: a byte with its sign bit turned is code + 128, under 0x64 it is the half 1024 + 128 +
// code, and the subtraction leaves the code (conversion by instruction takes twice as many).
__device__ __forceinline__ void halves_of(uint32_t codes, uint32_t &lo, uint32_t &hi) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const uint32_t u = codes ^ 0x80808080u;
  const f16x2 off = {(f16_t)1152.f, (f16_t)1152.f};
  const uint32_t a = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u), b = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
  lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, a) - off);
  hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, b) - off);
}
__device__ __forceinline__ Frag frag_of(uint32_t c0, uint32_t c1) {
  Frag f;
  halves_of(c0, f.u.x, f.u.y);
  halves_of(c1, f.u.z, f.u.w);
  return f;
}

// Probabilities are held as 2^(15 - slack) p: halves then keep their full precision down to 2^-(29 - slack) instead of 2^-14, and
// the sums carry the same factor.  Their reference follows the running maximum only when that is more than the slack above it,
// so that after a wave's first blocks next to nothing is rescaled (128 products per block of 32 columns and 128 dims).  Where
// probabilities are pairs of halves the low one ends 11 bits sooner, and the slack is smaller.
constexpr float slack_of(bool pairs) { return pairs ? 4.f : 8.f; }

// (a condition that is the same for the whole wave, as a branch of the scalar unit)
__device__ __forceinline__ bool uniform(bool c) { return __builtin_amdgcn_readfirstlane(c ? 1 : 0) != 0; }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }

// Codes that a launch reads once (ONCE: one tile of columns per key head) are loaded with the non-temporal hint: us per launch with
// ordinary loads / with the hint, 4 requests x 32 heads x 5000 tokens of size 128 32.3 / 30.3, 32 x 8 x 8192 78.3 / 73.7, 16 x 8461
// 17.7 / 17.5, 12 x 1000 of size 64 8.1 / 8.1.  Groups of columns re-read them from L2: 1 x 16 heads, 2048 rows 133 / 143.
template <bool ONCE, typename U>
__device__ __forceinline__ U ld_code(const int8_t *p) {
  typedef unsigned words __attribute__((ext_vector_type(sizeof(U) / 4)));
  return __builtin_bit_cast(U, ONCE ? __builtin_nontemporal_load((const words *)p) : *(const words *)p);
}

typedef int intx4 __attribute__((ext_vector_type(4)));
// 16 x 16 sums of 64 products of bytes, exact
__device__ __forceinline__ intx4 mfma_codes(uint4 a, uint4 b, intx4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(intx4, a), __builtin_bit_cast(intx4, b), c, 0, 0, 0);
}

// grid: (split, group of 16 QT columns, key head, request), dealt by byte_attn_group; NW waves.  The blocks of 64 tokens of a (request, key head) are dealt
// round-robin to the waves of its splits.  A column is one query vector (row, query head of the key head's group).  Scores come
// out of the matrix instruction with a lane holding 16 tokens of one column, which are its operand for the outputs as they are:
// element e of step s of group g is token 32 s + 16 (e >> 2) + 4 g + (e & 3) of the block.
//  * Scores are products of bytes, exact in 32-bit integers: the keys' codes as they lie, queries as whole numbers of three bytes,
//    in steps of a power of two at most 2^-21 of the row's largest.  No key is converted.  (Two bytes would be enough for bf16
//    where a row's channels are alike, and 0.2-0.4 us less for a step, 10 % for a piece of a prompt; with one channel 1000 times the
//    others outputs were off by 6 times what all other roundings explain, and a decoder's logits by 4.5e-2 instead of 7e-4.)
//  * Values become halves in registers, exactly, once for QT tiles of 16 columns.
//  * A block's key scale multiplies its scores.  The reference of the exponentials is a whole number (a running maximum rounded
//    up), so that taking it off rounds nothing and rescaling by its change is exact.
//  * A block's value scale multiplies its probabilities, over a power of two (vref) within 4 times it: the outputs add up in
//    the matrix instruction, in units of vref, and are rescaled, exactly, where it moves (rare: scales of neighbouring blocks are alike).
//  * The sums of the probabilities are a product with ones: the same roundings as in the outputs, and no work for the vector
//    units.
// Measured: 32 requests, 4 query heads to each of 8 key heads, up to 8192 tokens of size 128 70 us, 4.9 TB/s (half queries); 16 rows of
// 4 x 32 heads, up to 5000 tokens 25 us and 4.1 for the merge (bf16).  Few short heads are a chain of trips to memory: 12 heads of
// 64, 1000 tokens 7 us, of which an empty launch is 2.3.  Pieces of a prompt are bound by what a SIMD issues: fp32, 2048 rows of 16 heads
// of 128 over 6144 tokens 177 us, 485 TFLOP/s.
// PP: probabilities as pairs of halves (22 bits): fp32 outputs need them, and half outputs are rounded as finely as single
// probabilities would be (error of the whole 1.3 times the output's rounding without).
// CTX: the columns are a decode step's rows, which see the context up to their limit and generated tokens by their tags.  32 tokens
// of halves are as many bytes as 64 of codes, and the two kinds of blocks are dealt round-robin as one sequence.
template <typename T, int HD, bool PP, int QT, int NW, bool CTX = false>
__global__ __launch_bounds__(64 * NW, 2) void k_byte_attn(ByteAttnArgs a) {
  static_assert(!CTX || (QT == 1 && !PP && sizeof(T) == 2), "decode steps: one tile of rows");
  constexpr int NS = HD / 32, NT = HD / 16;              // contraction steps of the scores, 16-dim tiles of the outputs
  constexpr int KW = HD / 64;                            // 16-byte loads per key and lane (8 bytes more where a step is left)
  constexpr int PSTR = HD + 2;
  constexpr int NP = 3, NC = (HD + 63) / 64;             // bytes of a query value; contraction steps of 64
  constexpr bool QP = sizeof(T) == 4 || CTX;
  constexpr float SLACK = slack_of(PP), P_BITS = 15.f - SLACK;
  __shared__ uint4 sm_qi[QT][NP][NC][64], sm_q[CTX ? 1 : QT][CTX ? 1 : (QP ? 2 : 1) * NS][64];
  __shared__ float sm_qf[QT][2][16];
  __shared__ uint32_t sm_top[QT][16][16];
  __shared__ float sm_m[QT][NW][16], sm_l[QT][NW][16];
  __shared__ floatx4 sm_o[NW][NT][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const ByteGroup me = byte_attn_group(blockIdx.x, a.c.n_req * a.c.n_kv_head, a.nqg, a.nsplit);
  const int unit = me.unit, split = me.split, qg = a.nqg - 1 - me.group;      // (the last rows of a causal piece have the most to do)
  const int h = unit % a.c.n_kv_head, reqi = unit / a.c.n_kv_head, req = CTX ? a.req0 + reqi : reqi;
  const int n_cols = a.n_row * a.group;
  const size_t rhz = CTX ? (size_t)req * a.c.n_kv_head + h : (size_t)unit;
  const int d_model = a.c.n_kv_head * HD;
  // CTX: the row of column n (clamped: loads stay in bounds) and what it is
  const int crow = CTX ? reqi * a.n_row + min(qg * 16 + n, a.n_row - 1) : 0;
  int4 qi = make_int4(0, 0, 0, 0);
  if constexpr (CTX) qi = a.qinfo[crow];

  // One block per wave is in flight while another is worked on: its keys are requested when the scores have taken the ones
  // before, its values when the outputs have.  The first is requested before anything else is read (a wave without one asks for
  // the last block that there is room for, and ignores it).  Scales come by vector loads, in order with the codes, so that
  // nothing waits for all that is under way.
  const int8_t *K = a.c.k + rhz * a.c.n_block * BYTE_BLOCK * HD + n * 16;
  const int8_t *V = a.c.v + rhz * a.c.n_block * BYTE_BLOCK * HD + (g * HD + n) * 16;
  int zero;
  asm("v_mov_b32 %0, 0" : "=v"(zero));
  const float *KS = a.c.k_scale + rhz * a.c.n_block + zero, *VS = a.c.v_scale + rhz * a.c.n_block + zero;
  const int stride = NW * a.nsplit;
  int kb = split * NW + wave;
  uint4 kw[4][KW ? KW : 1], vw[NT];
  uint2 kn[4];
  uint2 tg[4] = {make_uint2(0, 0), make_uint2(0, 0), make_uint2(0, 0), make_uint2(0, 0)};
  float ksc, vsc;
  const uint16_t *TG = a.key_tag ? a.key_tag + (size_t)req * a.c.n_block * BYTE_BLOCK + 4 * g : nullptr;
  auto load_tags = [&](int b) {
    if (TG) {
#pragma unroll
      for (int t = 0; t < 4; ++t) tg[t] = *(const uint2 *)(TG + (size_t)b * BYTE_BLOCK + 16 * t);
    }
  };
  auto load_k = [&](int b) {
    const int8_t *kp = K + (size_t)b * BYTE_BLOCK * HD;
    ksc = KS[b];
    load_tags(b);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int c = 0; c < KW; ++c) kw[t][c] = ld_code<QT == 1, uint4>(kp + ((c * 4 + g) * BYTE_BLOCK + 16 * t) * 16);
      if (NS & 1) kn[t] = ld_code<QT == 1, uint2>(kp + ((KW * 4 + (g >> 1)) * BYTE_BLOCK + 16 * t) * 16 + (g & 1) * 8);
    }
  };
  auto load_v = [&](int b) {
    const int8_t *vp = V + (size_t)b * BYTE_BLOCK * HD;
    vsc = VS[b];
#pragma unroll
    for (int i = 0; i < NT; ++i) vw[i] = ld_code<QT == 1, uint4>(vp + i * 256);
  };
  // ---- the queries of the columns: dims and columns dealt over all threads (columns beyond the last: that one's) ----
  // They are asked for first, so that they are not waited for behind the keys and values of the first block.
  constexpr int DP = HD / 16;                            // dims per (column, part)
  constexpr int IT = (QT * 256 + NW * 64 - 1) / (NW * 64);
  T xq[CTX ? 1 : IT][DP];
  f16_t xh[CTX ? IT : 1][2][DP];                         // CTX: high and low halves
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int e = threadIdx.x + it * NW * 64, qt = e >> 8, pt = e >> 4 & 15;
    const int col = min((qg * QT + min(qt, QT - 1)) * 16 + (e & 15), n_cols - 1);
    if constexpr (CTX) {
      const size_t at = act_off(reqi * a.n_row + col, h * HD + pt * DP, d_model);
      const f16_t *lo = a.cq_lo ? a.cq_lo : a.cq;
      if constexpr (HD != 96) {                          // (they lie in one granule of 8)
        typedef f16_t part_t __attribute__((ext_vector_type(DP)));
        union { part_t v; f16_t h[DP]; } u[2];
        u[0].v = *(const part_t *)(a.cq + at);
        u[1].v = *(const part_t *)(lo + at);
#pragma unroll
        for (int j = 0; j < DP; ++j) { xh[it][0][j] = u[0].h[j]; xh[it][1][j] = u[1].h[j]; }
      } else {
#pragma unroll
        for (int j = 0; j < DP; ++j) {
          const size_t one = act_off(reqi * a.n_row + col, h * HD + pt * DP + j, d_model);
          xh[it][0][j] = a.cq[one]; xh[it][1][j] = lo[one];
        }
      }
    } else {
      const int row = a.group == 1 ? col : col / a.group;
      const T *p = (const T *)a.q + req * a.q_req + row * a.q_row + (h * a.group + col - row * a.group) * a.q_head + pt * DP;
#pragma unroll
      for (int j = 0; j < DP; ++j) xq[CTX ? 0 : it][j] = p[j];
    }
  }
  __builtin_amdgcn_sched_barrier(0);
  load_k(min(kb, a.c.n_block - 1));
  load_v(min(kb, a.c.n_block - 1));
  __builtin_amdgcn_sched_barrier(0);

  // ... in operand order: whole numbers of NP bytes for the codes, halves for the tail
  {
    float x[IT][DP];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = threadIdx.x + it * NW * 64, qt = e >> 8, pt = e >> 4 & 15;
#pragma unroll
      for (int j = 0; j < DP; ++j)
        x[it][j] = CTX ? (float)xh[CTX ? it : 0][0][j] + (a.cq_lo ? (float)xh[CTX ? it : 0][1][j] : 0.f) : ld_f32(&xq[CTX ? 0 : it][j], 0);
      if (qt >= QT) continue;
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < DP; ++j) top = max(top, __float_as_uint(x[it][j]) & 0x7fffffffu);
      sm_top[qt][pt][e & 15] = top;
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = threadIdx.x + it * NW * 64, qt = e >> 8, pt = e >> 4 & 15, m = e & 15;
      if (qt >= QT) continue;
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) top = max(top, sm_top[qt][j][m]);
      // halves: divided by a power of two that brings the largest below 512, held where both powers are normal numbers
      const bool finite = top < 0x7f800000u;
      const int ex = finite ? max((int)(top >> 23) - 127, -100) : 8;
      const float down = __uint_as_float((uint32_t)(127 + 8 - ex) << 23);
      // whole numbers of up to 2^22, by a power of two, which rounds nothing; the factor of a row that is not finite is NaN, and so
      // are its scores
      const float sign = a.scale_log2 < 0.f ? -1.f : 1.f;          // (factors are not negative)
      const float up = finite ? __uint_as_float((uint32_t)(127 + 21 - ex) << 23) * sign : 0.f;
      if (pt == 0) {
        sm_qf[qt][0][m] = !finite ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(127 - 21 + ex) << 23);
        sm_qf[qt][1][m] = __uint_as_float((uint32_t)(127 - 8 + ex) << 23) * fabsf(a.scale_log2);
      }
#pragma unroll
      for (int j = 0; j < DP; ++j) {
        const int d = pt * DP + j;
        // dim -> (step of 64, group, byte) for the codes; 16 dims of a 16-byte load are 8 of two steps of 32 for the halves
        const bool wide = d < KW * 64;
        const int gg = wide ? (d & 63) >> 4 : (d & 31) >> 3, step = wide ? (d >> 6) * 2 + ((d >> 3) & 1) : 2 * KW;
        if constexpr (!CTX) {
          const float y = x[it][j] * down * sign;
          const f16_t hi = (f16_t)y;
          ((f16_t *)&sm_q[qt][step][gg * 16 + m])[d & 7] = hi;
          if (QP) ((f16_t *)&sm_q[qt][(QP ? NS : 0) + step][gg * 16 + m])[d & 7] = (f16_t)(y - (float)hi);
        }
        int w = finite ? (int)rintf(x[it][j] * up) : 0;
#pragma unroll
        for (int b = NP - 1; b >= 0; --b) {
          const int8_t c = (int8_t)w;
          ((int8_t *)&sm_qi[qt][b][wide ? d >> 6 : KW][gg * 16 + m])[wide ? d & 15 : d & 7] = c;
          w = (w - c) >> 8;
        }
      }
    }
  }
  // ---- what the columns see ----
  const int cap = a.c.n_block * BYTE_BLOCK;
  const int n_keys = CTX ? a.lens[req] : min(max(a.lens[req], 0), cap);
  int lim[QT], tag[QT], reach = 0, lim_all = 0x7fffffff, tag_all = 0x7fffffff;
  bool qvalid = true;
  if constexpr (CTX) {
    qvalid = qg * 16 + n < a.n_row && (qi.x & ROW_VALID);
    lim[0] = qvalid ? min(qi.z, n_keys) : 0;
    tag[0] = qvalid ? qi.y : -1;
    reach = qvalid ? (n_keys > a.L && qi.y >= 1 ? n_keys : lim[0]) : 0;
    if (qvalid) lim_all = lim[0];
  } else {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int col = (qg * QT + qt) * 16 + n, row = min(col, n_cols - 1) / a.group;
      lim[qt] = col < n_cols ? n_keys : 0;
      if (a.row_limit) lim[qt] = min(lim[qt], max(a.row_limit[(size_t)req * a.n_row + row], 0));
      tag[qt] = a.key_tag ? a.row_tag[(size_t)req * a.n_row + row] : 0;
      reach = max(reach, lim[qt]);
      if (col < n_cols) { lim_all = min(lim_all, lim[qt]); tag_all = min(tag_all, tag[qt]); }
    }
  }
  reach = __builtin_amdgcn_readfirstlane(fold_row(reach, Max()));
  lim_all = __builtin_amdgcn_readfirstlane(fold_row(lim_all, Min()));
  tag_all = __builtin_amdgcn_readfirstlane(fold_row(tag_all, Min()));
  const int whole = CTX ? a.nblk : n_keys / BYTE_BLOCK;  // blocks of codes; the next one is the tail (CTX: the first of halves)
  // (CTX: one sequence, 32 tokens of halves a block)
  const int end = CTX ? (reach <= a.nblk * BYTE_BLOCK ? (reach + BYTE_BLOCK - 1) / BYTE_BLOCK : (reach + 31) / 32 - a.nblk)
                      : min((reach + BYTE_BLOCK - 1) / BYTE_BLOCK, a.nblk);
  const int sealed_end = min(end, whole);
  __syncthreads();
  float qf[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) qf[qt] = sm_qf[qt][0][n];

  float m_run[QT], l_run[QT], vref = 0.f;
  floatx4 o[QT][NT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    m_run[qt] = -INFINITY; l_run[qt] = 0.f;
#pragma unroll
    for (int i = 0; i < NT; ++i) o[qt][i] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  Frag ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones.hh[e] = (f16_t)1.f;

  // CTX: blocks of 32 tokens of halves; place b of the sequence is block b + nblk of the decoder's cache (clamped: requested
  // unconditionally)
  uint4 hk[CTX ? 2 : 1][CTX ? NS : 1], hv[CTX ? NT : 1], htag;
  Frag hq[CTX ? 2 : 1][CTX ? NS : 1];                    // the step's queries as they are, high and low halves
  auto load_hq = [&]() {
    const size_t at = act_off(crow, h * HD + g * 8, d_model);
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      hq[0][CTX ? c : 0].u = *(const uint4 *)(a.cq + at + (size_t)c * 512);
      hq[CTX ? 1 : 0][CTX ? c : 0].u = *(const uint4 *)((a.cq_lo ? a.cq_lo : a.cq) + at + (size_t)c * 512);
    }
  };
  const uint4 *HK = (const uint4 *)(a.hk + ((size_t)req * a.c.n_kv_head + h) * a.kv_cap * HD) + lane;
  const uint4 *HV = (const uint4 *)(a.hv + ((size_t)req * a.c.n_kv_head + h) * a.kv_cap * HD) + lane;
  const int h_last = a.kv_cap / 32 - 1, L8 = a.L & ~7;
  auto load_hk = [&](int b) {
    const size_t hb = min(b + a.nblk, h_last);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < NS; ++c) hk[CTX ? t : 0][CTX ? c : 0] = HK[((hb * 2 + t) * NS + c) * 64];
    htag = *(const uint4 *)(a.gen_sub + (size_t)req * a.gen_stride + min(max((int)hb * 32 + 8 * g - L8, 0), a.gen_stride - 8));
  };
  auto load_hv = [&](int b) {
    const size_t hb = min(b + a.nblk, h_last);
#pragma unroll
    for (int i = 0; i < NT; ++i) hv[CTX ? i : 0] = HV[(hb * NT + i) * 64];
  };
  auto half_block = [&]() {
    floatx4 s[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int c = 0; c < NS; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        Frag f;
        f.u = hk[CTX ? t : 0][CTX ? c : 0];
        s[t] = mfma16h(f, hq[0][CTX ? c : 0], s[t]);
        if (a.cq_lo) s[t] = mfma16h(f, hq[CTX ? 1 : 0][CTX ? c : 0], s[t]);
      }
    union { uint4 u; uint16_t t[8]; } tags;
    tags.u = htag;
    load_hk(kb + stride);
    __builtin_amdgcn_sched_barrier(0);
    if (vref == 0.f) vref = 1.f;
    const int key0 = (kb + a.nblk) * 32 + 8 * g;          // element e: token key0 + e
    const float kf = a.scale_log2;
    float sv[8], mloc = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = key0 + e;
      const bool vis = (key < lim[0]) | ((key >= a.L) & (key < n_keys) & ((int)tags.t[e] <= tag[0]));
      sv[e] = vis ? s[e >> 2][e & 3] * kf : -INFINITY;
      mloc = fmaxf(mloc, sv[e]);
    }
    mloc = ceilf(fold32(fold16(mloc, Max()), Max()));
    const float m_new = mloc > m_run[0] + SLACK ? mloc : m_run[0], m_ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run[0] - m_ref);
    m_run[0] = m_new;
    Frag ph;
#pragma unroll
    for (int e = 0; e < 8; ++e) ph.hh[e] = (f16_t)__builtin_amdgcn_exp2f(sv[e] + (P_BITS - m_ref));
    const floatx4 t = mfma16h(ones, ph, floatx4{0.f, 0.f, 0.f, 0.f});
    l_run[0] = fmaf(l_run[0], alpha, t[0]);
    const float f = 1.f / vref;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      Frag v;
      v.u = hv[CTX ? i : 0];
      const floatx4 y = mfma16h(v, ph, floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int e = 0; e < 4; ++e) o[0][i][e] = fmaf(y[e], f, o[0][i][e] * alpha);
    }
    load_hv(kb + stride);
    kb += stride;
  };
  // KIND: 0 a block of codes with another one behind it, 1 the wave's last one, 2 the tail.  (Requests stand outside of all
  // branches: where a branch decides on one, waits count on its not having been made, and where two make it, what arrives is
  // waited for and copied.)
  auto block = [&](auto kind_) {
    constexpr int KIND = decltype(kind_)::value;
    constexpr bool TAIL = KIND == 2;
    const f16_t *kt = (const f16_t *)a.c.k_tail + (rhz * 2 + (kb & 1)) * BYTE_BLOCK * HD + n * 8;
    const f16_t *vt = (const f16_t *)a.c.v_tail + (rhz * 2 + (kb & 1)) * BYTE_BLOCK * HD + (g * HD + n) * 8;
    const int key0 = kb * BYTE_BLOCK + 4 * g;            // element e: token key0 + 16 (e >> 2) + (e & 3)
    auto key = [&](int e) { return key0 + 16 * (e >> 2) + (e & 3); };
    // the tail: everything that its scores need is requested before what its outputs need
    Frag vtail[TAIL ? NT : 1][2], ktail[TAIL && QT == 1 ? 4 : 1][TAIL && QT == 1 ? NS : 1];
    auto tail_k = [&](int c, int t) {
      return *(const uint4 *)(kt + ((c < 2 * KW ? (c >> 1) * 8 + g * 2 + (c & 1) : KW * 8 + g) * BYTE_BLOCK + 16 * t) * 8);
    };
    if (TAIL) {
      if (QT == 1)
#pragma unroll
        for (int c = 0; c < NS; ++c)
#pragma unroll
          for (int t = 0; t < 4; ++t) ktail[QT == 1 && TAIL ? t : 0][QT == 1 && TAIL ? c : 0].u = tail_k(c, t);
      load_tags(kb);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        vtail[TAIL ? i : 0][0].u = *(const uint4 *)(vt + i * 128);
        vtail[TAIL ? i : 0][1].u = *(const uint4 *)(vt + 4 * HD * 8 + i * 128);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    union { uint2 u[4]; uint16_t s[16]; uint32_t w[8]; } tags;
#pragma unroll
    for (int t = 0; t < 4; ++t) tags.u[t] = tg[t];
    const float ks = TAIL ? 1.f : ksc;
    // ---- scores: lane (n, g), element e  <->  token key(e) of column n ----
    float sv[QT][16];
    if (TAIL) {
      floatx4 s[QT][4];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int t = 0; t < 4; ++t) s[qt][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NS; ++c)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          Frag f, q;
          if (QT == 1) f = ktail[QT == 1 && TAIL ? t : 0][QT == 1 && TAIL ? c : 0];
          else f.u = tail_k(c, t);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) {
            q.u = sm_q[CTX ? 0 : qt][CTX ? 0 : c][lane];
            s[qt][t] = mfma16h(f, q, s[qt][t]);
            if (QP) { q.u = sm_q[CTX ? 0 : qt][CTX ? 0 : (QP ? NS : 0) + c][lane]; s[qt][t] = mfma16h(f, q, s[qt][t]); }
          }
        }
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int e = 0; e < 16; ++e) sv[qt][e] = s[qt][e >> 2][e & 3];
    } else {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        // the products of the highest byte, below 2^20, times 256 and those of the next one, added to them
        intx4 s[2][4];
#pragma unroll
        for (int b = 0; b < NP; ++b)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const uint4 q = sm_qi[qt][b][c][lane];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const intx4 from = c ? s[b >> 1][t] : b == 1 ? s[0][t] << 8 : intx4{0, 0, 0, 0};
              // (the last 32 dims: half of the bytes are zeros, and the query's beside them anything.  The instruction for 32
              // would do half the work, but its sums right behind those of the one for 64, whose results it adds to, came out
              // wrong.  Why is not known, and so the two never meet.)
              s[b >> 1][t] = mfma_codes(c < KW ? kw[t][c < KW ? c : 0] : make_uint4(kn[t].x, kn[t].y, 0, 0), q, from);
            }
          }
#pragma unroll
        for (int e = 0; e < 16; ++e) sv[qt][e] = fmaf((float)s[0][e >> 2][e & 3], 256.f, (float)s[1][e >> 2][e & 3]);
        if (QT > 1) __builtin_amdgcn_sched_barrier(0);
      }
    }
    // whether every column sees the whole block (the same for the whole wave)
    bool whole_seen = !TAIL && kb * BYTE_BLOCK + BYTE_BLOCK <= lim_all;
    if (!TAIL && TG) {
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, max(tags.w[e] >> 16, tags.w[e] & 0xffff));
      whole_seen = whole_seen && !__any((int)top > tag_all);
      whole_seen = uniform(whole_seen);
    }
    if (KIND == 0) load_k(kb + stride);
    if (KIND == 1 && CTX) { load_hq(); load_hk(kb + stride); }
    __builtin_amdgcn_sched_barrier(0);
    // ---- probabilities ----
    const float vs = TAIL ? 1.f : __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(vsc)));
    // vref, a power of two, is kept within 1 and 4 of the scales, so that the ratio takes at most 2 bits of the probabilities' room
    // (with a ratio of 2^-11.5, tokens of 2^-13 of the row's largest would be off by up to 2.8e-4 as pairs of halves and 4.5e-3 as
    // single ones, all alike, in the outputs and in the sums).  Moving it is exact: outputs stay below 2^15 127 2^30 (tokens) times
    // the largest vref there was over the present one, which is 2^64 at most as scales lie within 2^-32 and 2^32.
    float grow = 1.f;
    if (!TAIL && uniform(vs > vref || (vs * 4.f < vref && vs > 0.f))) {
      const float to = __uint_as_float((__float_as_uint(vs) + 0x7fffffu) & 0xff800000u);
      grow = vref / to;
      vref = to;
    }
    if (TAIL && vref == 0.f) vref = 1.f;
    // (a scale of zero goes with codes of zero)
    const float ratio = TAIL || vs == 0.f ? 1.f : vs * (1.f / vref), inv_ratio = __builtin_amdgcn_rcpf(ratio);
    Frag ph[QT][2], pl[QT][2];
    float take[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      // fp32: the factor with what its roundings leave, which would shift a block's probabilities together
      float kf = TAIL ? sm_qf[qt][1][n] : qf[qt] * ks, kf_low = 0.f;
      if (!TAIL) {
        const float f = qf[qt] * fabsf(a.scale_log2);
        kf = f * ks;
        if (sizeof(T) == 4) kf_low = fmaf(qf[qt] * a.scale_low, ks, fmaf(f, ks, -kf));
      }
      kf = kf == 0.f ? 1e-37f : kf;                      // (nothing but zeros comes of it, and -infinity stays what it is)
      if (!whole_seen)
#pragma unroll
        for (int e = 0; e < 16; ++e) sv[qt][e] = ((key(e) < lim[qt]) & ((int)tags.s[e] <= tag[qt])) ? sv[qt][e] : -INFINITY;
      float mloc = sv[qt][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mloc = fmaxf(mloc, sv[qt][e]);
      mloc = ceilf(fold32(fold16(mloc, Max()), Max()) * kf);
      const float m_new = mloc > m_run[qt] + SLACK ? mloc : m_run[qt], m_ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run[qt] - m_ref), down = alpha * grow;
      m_run[qt] = m_new;
      // (fp32 outputs: the scale's logarithm in the exponent would round it by up to 2^-19; NaN has to arrive all the same)
      const float off = P_BITS - m_ref + (sizeof(T) == 2 ? lg2(ratio) : 0.f * ratio);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = fmaf(sv[qt][e], kf, off);
        sv[qt][e] = sizeof(T) == 4 && !TAIL ? fmaf(fmaxf(sv[qt][e], -3e38f), kf_low, x) : x;
      }
      if (!whole_seen && __any(kf != kf || off != off))  // NaN takes the tokens that are seen only
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sv[qt][e] = ((key(e) < lim[qt]) & ((int)tags.s[e] <= tag[qt])) ? sv[qt][e] : -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float p = __builtin_amdgcn_exp2f(sv[qt][e]);
        if (sizeof(T) == 4) {
          p *= fminf(ratio, 1.f);
          // (one number for both halves: the compiler took the high one from the product as rounded and the low one from the product
          // and a conversion fused, and where the two differed, in one of a thousand, the pair was off by a whole step of a half)
          asm("" : "+v"(p));
        }
        ph[qt][e >> 3].hh[e & 7] = (f16_t)p;
        if (PP) pl[qt][e >> 3].hh[e & 7] = (f16_t)(p - (float)ph[qt][e >> 3].hh[e & 7]);
      }
      floatx4 t = mfma16h(ones, ph[qt][0], floatx4{0.f, 0.f, 0.f, 0.f});
      t = mfma16h(ones, ph[qt][1], t);
      if (PP) { t = mfma16h(ones, pl[qt][0], t); t = mfma16h(ones, pl[qt][1], t); }
      l_run[qt] = fmaf(t[0], inv_ratio == inv_ratio ? inv_ratio : 1.f, l_run[qt] * alpha);
      take[qt] = t[0];
      // (used here: sunk behind the branch below, the first use of the sums stood too close to the product for them to have
      // arrived, where the branch is taken.  tests/test_byte_cache_code.py walks every path of the built kernels for such uses.)
      asm volatile("" : "+v"(l_run[qt]), "+v"(take[qt]));
      if (__any(down != 1.f))
#pragma unroll
        for (int i = 0; i < NT; ++i) o[qt][i] *= down;
    }
    // ---- outputs ----
    __builtin_amdgcn_sched_barrier(0);
    if (TAIL) {
      const float f = 1.f / vref;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        // slots without a token hold anything: zeros instead, so that no product with a zero is NaN
        Frag v0, v1;
        v0 = vtail[TAIL ? i : 0][0];
        v1 = vtail[TAIL ? i : 0][1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (key(e) >= n_keys) v0.hh[e] = (f16_t)0.f;
          if (key(8 + e) >= n_keys) v1.hh[e] = (f16_t)0.f;
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          floatx4 t = mfma16h(v0, ph[qt][0], floatx4{0.f, 0.f, 0.f, 0.f});
          t = mfma16h(v1, ph[qt][1], t);
          if (PP) { t = mfma16h(v0, pl[qt][0], t); t = mfma16h(v1, pl[qt][1], t); }
          // a column that sees nothing of the tail takes nothing from it, NaN or not
#pragma unroll
          for (int e = 0; e < 4; ++e) o[qt][i][e] = take[qt] != 0.f ? fmaf(t[e], f, o[qt][i][e]) : o[qt][i][e];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const Frag v0 = frag_of(vw[i].x, vw[i].y), v1 = frag_of(vw[i].z, vw[i].w);
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          o[qt][i] = mfma16h(v0, ph[qt][0], o[qt][i]);
          o[qt][i] = mfma16h(v1, ph[qt][1], o[qt][i]);
          if (PP) { o[qt][i] = mfma16h(v0, pl[qt][0], o[qt][i]); o[qt][i] = mfma16h(v1, pl[qt][1], o[qt][i]); }
        }
      }
    }
    if (KIND == 0) load_v(kb + stride);
    if (KIND == 1 && CTX) load_hv(kb + stride);
    kb += stride;
  };
  while (kb + stride < sealed_end) block(std::integral_constant<int, 0>());
  if (kb < sealed_end) block(std::integral_constant<int, 1>());
  else if (CTX) { load_hq(); load_hk(kb); load_hv(kb); }
  if constexpr (CTX) {
    while (kb < end) half_block();
  } else if (kb < end) {
    block(std::integral_constant<int, 2>());                      // (end is at most one beyond)
  }

  // ---- the waves' states become one ----
#pragma unroll
  for (int qt = 0; qt < QT; ++qt)
    if (g == 0) { sm_m[qt][wave][n] = m_run[qt]; sm_l[qt][wave][n] = l_run[qt]; }
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    if (qt) __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) sm_o[wave][i][lane] = o[qt][i] * vref;
    __syncthreads();
    float fw[NW], M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) { fw[w] = sm_m[qt][w][n]; M = fmaxf(M, fw[w]); }
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      // (a wave whose keys are all NaN has no maximum but a sum)
      fw[w] = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(fw[w] - M);
      L += fw[w] * sm_l[qt][w][n];
    }
    const int col = (qg * QT + qt) * 16 + n;
    if (a.nsplit > 1) {
      const size_t pu = CTX ? ((size_t)reqi * a.nqg + qg) * a.c.n_kv_head + h : ((size_t)unit * a.nqg + qg) * QT + qt;
      float *pp = a.part + pu * a.nsplit * (size_t)(PSTR * 16) + split * (size_t)(PSTR * 16);
      if (wave == 0 && g == 0) { pp[n] = M; pp[16 + n] = L; }
      for (int i = wave; i < NT; i += NW) {
        floatx4 y = fw[0] * sm_o[0][i][lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) y += fw[w] * sm_o[w][i][lane];
        *(floatx4 *)(pp + 32 + ((i * 4 + g) * 16 + n) * 4) = y;
      }
      continue;
    }
    if (CTX ? !qvalid : col >= n_cols) continue;
    if constexpr (CTX) {
      const float inv = 1.f / L;
      for (int i = wave; i < NT; i += NW) {
        floatx4 y = fw[0] * sm_o[0][i][lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) y += fw[w] * sm_o[w][i][lane];
        const float r[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
        store4_split(a.cout, a.cout_lo, act_off(crow, h * HD + i * 16 + 4 * g, d_model), r);
      }
      continue;
    }
    const size_t at = ((size_t)req * a.n_row + col / a.group) * a.c.n_kv_head * a.group + h * a.group + col % a.group;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (a.lse && wave == 0 && g == 0) a.lse[at] = (M + (__builtin_amdgcn_logf(L) - P_BITS)) * 0.6931471805599453f;
    for (int i = wave; i < NT; i += NW) {
      floatx4 y = fw[0] * sm_o[0][i][lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) y += fw[w] * sm_o[w][i][lane];
      y *= inv;
      store4((T *)a.out + at * HD + i * 16 + 4 * g, y);
    }
  }
}

// Pieces of a prompt with bf16 or half queries.  A work-group of 8 waves takes 128 columns, 32 a wave; each half of its waves takes every
// other block.  A half's waves share the conversion of its blocks: codes become halves in LDS, in operand order, one step ahead (keys) or
// behind (values) of the scores.  As halves such queries are exact in steps of a power of two (what lies 2^-22 below the row's largest is
// rounded to 2^-33 of it), so that scores are one product of halves, added up in fp32, where the kernel above has three products of
// bytes and puts whole numbers together.  While one half of the waves multiplies and converts, the other one has its softmax: a
// barrier between the two keeps them apart.  Everything behind the scores is as above, the tail one more step of the first half.
// Bound by what a SIMD issues as well: bf16, 2048 rows of 16 heads of 128 over 6144 tokens 116 us, 745 TFLOP/s, vector instructions 58 %
// and matrix instructions 38 % of the time.  Halves with heads of 128 keep nine registers in scratch memory (150 us).
// us, the kernel above / this one, half (bf16): 16 heads of 128, 2048 rows, 6144 tokens 160 / 148 (129 / 116); 4 x 16 heads of 64, 512 rows,
// 2048 tokens without limits 51 / 41 (43 / 34); 28 x 8 heads of 128, 100 rows, 1000 tokens 45 / 41 (40 / 33), one block 19 / 12 (18 / 10).
template <typename T, int HD, bool PP>
__global__ __launch_bounds__(512, 2) void k_byte_piece(ByteAttnArgs a) {
  constexpr int NS = HD / 32, NT = HD / 16, ITEMS = HD * 4, IT = (ITEMS + 255) / 256;      // 16-byte loads of a block, per thread
  constexpr float SLACK = slack_of(PP), P_BITS = 15.f - SLACK;
  __shared__ uint4 sm[2][2][2][HD * 8];                  // [step & 1][half][keys, values][fragments of 64 lanes]
  __shared__ int sm_end[8];
  __shared__ float sm_m[4][2][16], sm_l[4][2][16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int cw = wave & 3, half = wave >> 2, tid = threadIdx.x & 255;
  const ByteGroup me = byte_attn_group(blockIdx.x, a.c.n_req * a.c.n_kv_head, a.nqg, 1);
  const int unit = me.unit, qg = a.nqg - 1 - me.group;   // (as above)
  const int h = unit % a.c.n_kv_head, req = unit / a.c.n_kv_head, n_cols = a.n_row * a.group, col0 = qg * 128 + cw * 32;
  const size_t rhz = unit;

  // ---- requests ----
  const uint4 *K = (const uint4 *)(a.c.k + rhz * a.c.n_block * BYTE_BLOCK * HD);
  const uint4 *V = (const uint4 *)(a.c.v + rhz * a.c.n_block * BYTE_BLOCK * HD);
  int zero;
  asm("v_mov_b32 %0, 0" : "=v"(zero));
  const float *KS = a.c.k_scale + rhz * a.c.n_block + zero, *VS = a.c.v_scale + rhz * a.c.n_block + zero;
  const uint16_t *TG = a.key_tag ? a.key_tag + (size_t)req * a.c.n_block * BYTE_BLOCK + 4 * g : nullptr;
  const int b_last = a.c.n_block - 1;
  uint4 rk[IT], rv[IT];
  auto load_keys = [&](int b) {                          // (blocks that are not there: the last one's place)
    const size_t at = (size_t)min(b, b_last) * ITEMS;
#pragma unroll
    for (int it = 0; it < IT; ++it) rk[it] = K[at + (ITEMS % 256 == 0 || tid + it * 256 < ITEMS ? tid + it * 256 : 0)];
  };
  auto load_values = [&](int b) {
    const size_t at = (size_t)min(b, b_last) * ITEMS;
#pragma unroll
    for (int it = 0; it < IT; ++it) rv[it] = V[at + (ITEMS % 256 == 0 || tid + it * 256 < ITEMS ? tid + it * 256 : 0)];
  };
  auto put_keys = [&](int buf) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + it * 256;
      if (ITEMS % 256 != 0 && e >= ITEMS) continue;
      uint4 *kp = &sm[buf][half][0][((e >> 7) * 4 + ((e >> 4) & 3)) * 64 + ((e >> 6) & 1) * 32 + (e & 15)];
      kp[0] = frag_of(rk[it].x, rk[it].y).u; kp[16] = frag_of(rk[it].z, rk[it].w).u;
    }
  };
  auto put_values = [&](int buf) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + it * 256, d = e % HD;
      if (ITEMS % 256 != 0 && e >= ITEMS) continue;
      uint4 *vp = &sm[buf][half][1][(d >> 4) * 128 + e / HD * 16 + (d & 15)];
      vp[0] = frag_of(rv[it].x, rv[it].y).u; vp[64] = frag_of(rv[it].z, rv[it].w).u;
    }
  };
  float ks_next, vs_next;
  uint2 tg[4] = {make_uint2(0, 0), make_uint2(0, 0), make_uint2(0, 0), make_uint2(0, 0)};
  auto load_scales = [&](int b) {
    b = min(b, b_last);
    ks_next = KS[b]; vs_next = VS[b];
    if (TG) {
#pragma unroll
      for (int t = 0; t < 4; ++t) tg[t] = *(const uint2 *)(TG + (size_t)b * BYTE_BLOCK + 16 * t);
    }
  };
  load_keys(half);
  load_values(half);
  load_scales(half);

  // ---- queries and what the columns see ----
  const int cap = a.c.n_block * BYTE_BLOCK, n_keys = min(max(a.lens[req], 0), cap);
  Frag q[2][NS];
  float qf[2];
  int lim[2], tag[2], reach = 0, lim_all = 0x7fffffff, tag_all = 0x7fffffff;
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const int col = min(col0 + qt * 16 + n, n_cols - 1), row = a.group == 1 ? col : col / a.group;
    const T *p = (const T *)a.q + req * a.q_req + row * a.q_row + (h * a.group + col - row * a.group) * a.q_head + 8 * g;
    float x[NS][8];
    if (a.q_wide)
#pragma unroll
      for (int c = 0; c < NS; ++c) load8<T, true>(p + c * 32, x[c]);
    else
#pragma unroll
      for (int c = 0; c < NS; ++c) load8<T, false>(p + c * 32, x[c]);
    int top = 0;
#pragma unroll
    for (int c = 0; c < NS; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, (int)(__float_as_uint(x[c][j]) & 0x7fffffffu));
    top = fold32(fold16(top, Max()), Max());
    const bool finite = top < 0x7f800000;
    const int ex = finite ? max((top >> 23) - 127, -100) : 8;
    const float down = __uint_as_float((uint32_t)(127 + 8 - ex) << 23) * (a.scale_log2 < 0.f ? -1.f : 1.f);
    qf[qt] = finite ? __uint_as_float((uint32_t)(127 - 8 + ex) << 23) * fabsf(a.scale_log2) : __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int c = 0; c < NS; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) q[qt][c].hh[j] = (f16_t)(x[c][j] * down);
    const bool there = col0 + qt * 16 + n < n_cols;
    lim[qt] = there ? n_keys : 0;
    if (a.row_limit) lim[qt] = min(lim[qt], max(a.row_limit[(size_t)req * a.n_row + row], 0));
    tag[qt] = a.key_tag ? a.row_tag[(size_t)req * a.n_row + row] : 0;
    reach = max(reach, lim[qt]);
    if (there) { lim_all = min(lim_all, lim[qt]); tag_all = min(tag_all, tag[qt]); }
  }
  reach = __builtin_amdgcn_readfirstlane(fold_row(reach, Max()));
  lim_all = __builtin_amdgcn_readfirstlane(fold_row(lim_all, Min()));
  tag_all = __builtin_amdgcn_readfirstlane(fold_row(tag_all, Min()));
  const int whole = n_keys / BYTE_BLOCK, end = min((reach + BYTE_BLOCK - 1) / BYTE_BLOCK, a.nblk), mine = min(end, whole);
  sm_end[wave] = end;
  put_keys(0);
  load_keys(half + 2);
  __syncthreads();
  const int end_all = __builtin_amdgcn_readfirstlane(max(max(sm_end[0], sm_end[1]), max(sm_end[2], sm_end[3])));
  const int steps = (min(end_all, whole) + 1) / 2;

  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f}, vref = 0.f;
  floatx4 o[2][NT];
#pragma unroll
  for (int qt = 0; qt < 2; ++qt)
#pragma unroll
    for (int i = 0; i < NT; ++i) o[qt][i] = floatx4{0.f, 0.f, 0.f, 0.f};
  Frag ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones.hh[e] = (f16_t)1.f;

  floatx4 s[2][4];
  Frag ph[2][2], pl[2][2];
  float alpha[2], inv_ratio;
  auto scores = [&](int buf) {
    const uint4 *kl = sm[buf][half][0] + lane;
#pragma unroll
    for (int c = 0; c < NS; ++c)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        Frag f;
        f.u = kl[(c * 4 + t) * 64];
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) s[qt][t] = mfma16h(f, q[qt][c], c ? s[qt][t] : floatx4{0.f, 0.f, 0.f, 0.f});
      }
  };
  auto probabilities = [&](auto tail_, int kb, float ks, float vs) {
    constexpr bool TAIL = decltype(tail_)::value;
    const int key0 = kb * BYTE_BLOCK + 4 * g;            // element e: token key0 + 16 (e >> 2) + (e & 3)
    auto key = [&](int e) { return key0 + 16 * (e >> 2) + (e & 3); };
    union { uint2 u[4]; uint16_t s[16]; uint32_t w[8]; } tags;
#pragma unroll
    for (int t = 0; t < 4; ++t) tags.u[t] = tg[t];
    bool whole_seen = !TAIL && kb * BYTE_BLOCK + BYTE_BLOCK <= lim_all;
    if (!TAIL && TG) {
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, max(tags.w[e] >> 16, tags.w[e] & 0xffff));
      whole_seen = uniform(whole_seen && !__any((int)top > tag_all));
    }
    float grow = 1.f;
    if (!TAIL && uniform(vs > vref || (vs * 4.f < vref && vs > 0.f))) {
      const float to = __uint_as_float((__float_as_uint(vs) + 0x7fffffu) & 0xff800000u);
      grow = vref / to;
      vref = to;
    }
    if (TAIL && vref == 0.f) vref = 1.f;
    // (the reciprocal of a power of two)
    const float ratio = TAIL || vs == 0.f ? 1.f : vs * __uint_as_float(0x7f000000u - __float_as_uint(vref)), inv = __builtin_amdgcn_rcpf(ratio);
    inv_ratio = inv == inv ? inv : 1.f;
    auto masked = [&]() {
#pragma unroll
      for (int qt = 0; qt < 2; ++qt)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[qt][e >> 2][e & 3] = ((key(e) < lim[qt]) & ((int)tags.s[e] <= tag[qt])) ? s[qt][e >> 2][e & 3] : -INFINITY;
    };
    if (!whole_seen) masked();
    float off[2], kf[2], down[2];
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      kf[qt] = qf[qt] * ks;
      kf[qt] = kf[qt] == 0.f ? 1e-37f : kf[qt];
      float mloc = s[qt][0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mloc = fmaxf(mloc, s[qt][e >> 2][e & 3]);
      mloc = ceilf(fold32(fold16(mloc, Max()), Max()) * kf[qt]);
      const float m_new = mloc > m_run[qt] + SLACK ? mloc : m_run[qt], m_ref = m_new == -INFINITY ? 0.f : m_new;
      alpha[qt] = __builtin_amdgcn_exp2f(m_run[qt] - m_ref);
      down[qt] = alpha[qt] * grow;
      m_run[qt] = m_new;
      off[qt] = P_BITS - m_ref + lg2(ratio);
    }
    if (uniform(__any(down[0] != 1.f || down[1] != 1.f)))
#pragma unroll
      for (int qt = 0; qt < 2; ++qt)
#pragma unroll
        for (int i = 0; i < NT; ++i) o[qt][i] *= down[qt];
#pragma unroll
    for (int qt = 0; qt < 2; ++qt)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[qt][e >> 2][e & 3] = fmaf(s[qt][e >> 2][e & 3], kf[qt], off[qt]);
    if (!whole_seen && __any(kf[0] != kf[0] || off[0] != off[0] || kf[1] != kf[1] || off[1] != off[1])) masked();
#pragma unroll
    for (int qt = 0; qt < 2; ++qt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(s[qt][e >> 2][e & 3]);
        ph[qt][e >> 3].hh[e & 7] = (f16_t)p;
        if (PP) pl[qt][e >> 3].hh[e & 7] = (f16_t)(p - (float)ph[qt][e >> 3].hh[e & 7]);
      }
  };
  auto outputs = [&](auto tail_, int buf) {
    constexpr bool TAIL = decltype(tail_)::value;
    const uint4 *vl = sm[buf][half][1] + lane;
    float take[2];
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      floatx4 t = mfma16h(ones, ph[qt][0], floatx4{0.f, 0.f, 0.f, 0.f});
      t = mfma16h(ones, ph[qt][1], t);
      if (PP) { t = mfma16h(ones, pl[qt][0], t); t = mfma16h(ones, pl[qt][1], t); }
      l_run[qt] = fmaf(t[0], inv_ratio, l_run[qt] * alpha[qt]);
      take[qt] = t[0];
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      Frag v0, v1;
      v0.u = vl[i * 128]; v1.u = vl[i * 128 + 64];
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        floatx4 t = mfma16h(v0, ph[qt][0], TAIL ? floatx4{0.f, 0.f, 0.f, 0.f} : o[qt][i]);
        t = mfma16h(v1, ph[qt][1], t);
        if (PP) { t = mfma16h(v0, pl[qt][0], t); t = mfma16h(v1, pl[qt][1], t); }
        if (!TAIL) o[qt][i] = t;
        else
#pragma unroll
          for (int e = 0; e < 4; ++e) o[qt][i][e] = take[qt] != 0.f ? fmaf(t[e], 1.f / vref, o[qt][i][e]) : o[qt][i][e];
      }
    }
  };
  // (one barrier more for one half here, for the other one at the end: both pass as many.  The branch is the wave's own, and nothing in
  // LDS waits for these two.)
  if (half == 1) __builtin_amdgcn_s_barrier();
  bool held = false;                                     // probabilities of the step before
  for (int step = 0; step < steps; ++step) {
    const int kb = 2 * step + half;
    if (held) outputs(std::false_type(), (step + 1) & 1);
    if (kb < mine) scores(step & 1);
    put_values(step & 1);
    put_keys((step + 1) & 1);
    load_values(kb + 2);
    load_keys(kb + 4);
    __syncthreads();
    if (kb < mine) probabilities(std::false_type(), kb, ks_next, __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(vs_next))));
    held = kb < mine;
    load_scales(kb + 2);
    __syncthreads();
  }
  if (held) outputs(std::false_type(), (steps + 1) & 1);
  if (half == 0) __builtin_amdgcn_s_barrier();
  if (end_all > whole) {                                 // the tail, by the waves of the first half
    __syncthreads();
    const uint4 *kt = (const uint4 *)a.c.k_tail + (rhz * 2 + (whole & 1)) * (HD * 8);
    const uint4 *vt = (const uint4 *)a.c.v_tail + (rhz * 2 + (whole & 1)) * (HD * 8);
    for (int e = threadIdx.x; e < HD * 8; e += 512) {
      sm[0][0][0][((e >> 8) * 4 + ((e >> 4) & 3)) * 64 + ((e >> 6) & 3) * 16 + (e & 15)] = kt[e];
      const int d = e % HD, sg = e / HD;                 // slots without a token hold anything: zeros instead
      Frag v;
      v.u = vt[e];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (whole * BYTE_BLOCK + 16 * (2 * (sg >> 2) + (j >> 2)) + 4 * (sg & 3) + (j & 3) >= n_keys) v.hh[j] = (f16_t)0.f;
      sm[0][0][1][(d >> 4) * 128 + (sg >> 2) * 64 + (sg & 3) * 16 + (d & 15)] = v.u;
    }
    __syncthreads();
    if (half == 0 && end > whole) {
      load_scales(whole);                                // (the tags)
      scores(0);
      probabilities(std::true_type(), whole, 1.f, 1.f);
      outputs(std::true_type(), 0);
    }
  }
  __syncthreads();

  // ---- the halves' states become one ----
  floatx4 *sm_o = (floatx4 *)sm;
  if (half == 1) {
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      if (g == 0) { sm_m[cw][qt][n] = m_run[qt]; sm_l[cw][qt][n] = l_run[qt]; }
#pragma unroll
      for (int i = 0; i < NT; ++i) sm_o[((cw * 2 + qt) * NT + i) * 64 + lane] = o[qt][i] * vref;
    }
  }
  __syncthreads();
  if (half == 1) return;
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const float m1 = sm_m[cw][qt][n], M = fmaxf(m_run[qt], m1);
    // (a half whose keys are all NaN has no maximum but a sum)
    const float f0 = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[qt] - M), f1 = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m1 - M);
    const float L = f0 * l_run[qt] + f1 * sm_l[cw][qt][n];
    const int col = col0 + qt * 16 + n;
    if (col >= n_cols) continue;
    const size_t at = ((size_t)req * a.n_row + col / a.group) * a.c.n_kv_head * a.group + h * a.group + col % a.group;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (a.lse && g == 0) a.lse[at] = (M + (__builtin_amdgcn_logf(L) - P_BITS)) * 0.6931471805599453f;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      floatx4 y = f0 * (o[qt][i] * vref) + f1 * sm_o[((cw * 2 + qt) * NT + i) * 64 + lane];
      y *= inv;
      store4((T *)a.out + at * HD + i * 16 + 4 * g, y);
    }
  }
}

// The splits of a unit become one: a block per (unit, 16-dim tile), wave w takes the splits w, w + 4, ...
template <typename T, int HD, bool PP>
__global__ __launch_bounds__(256) void k_byte_merge(ByteAttnArgs a) {
  constexpr int PSTR = HD + 2, NT = HD / 16;
  constexpr float P_BITS = 15.f - slack_of(PP);
  __shared__ float sm_m[4][64], sm_l[4][64];
  __shared__ floatx4 sm_o[4][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int i = blockIdx.x % NT;
  const size_t unit = blockIdx.x / NT;
  const int n16 = a.nqg * a.qt, qg = unit % n16, h = unit / n16 % a.c.n_kv_head, req = unit / n16 / a.c.n_kv_head;
  const float *pb = a.part + unit * a.nsplit * (size_t)(PSTR * 16);
  float M = -INFINITY, L = 0.f;
  floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int s = wave; s < a.nsplit; s += 4) {
    const float *p = pb + (size_t)s * (PSTR * 16);
    const float m = p[n], l = p[16 + n];
    const floatx4 x = *(const floatx4 *)(p + 32 + ((i * 4 + g) * 16 + n) * 4);
    const float Mn = fmaxf(M, m), ref = Mn == -INFINITY ? 0.f : Mn;
    const float fo = M == -INFINITY && Mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - ref);
    const float fx = m == -INFINITY && Mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - ref);
    L = L * fo + l * fx;
    o = o * fo + x * fx;
    M = Mn;
  }
  sm_m[wave][lane] = M; sm_l[wave][lane] = L; sm_o[wave][lane] = o;
  __syncthreads();
  const int col = qg * 16 + n;
  if (wave != 0 || col >= a.n_row * a.group) return;
  M = fmaxf(fmaxf(sm_m[0][lane], sm_m[1][lane]), fmaxf(sm_m[2][lane], sm_m[3][lane]));
  L = 0.f; o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(sm_m[w][lane] - M);
    L += f * sm_l[w][lane];
    o += f * sm_o[w][lane];
  }
  const size_t at = ((size_t)req * a.n_row + col / a.group) * a.c.n_kv_head * a.group + h * a.group + col % a.group;
  if (a.lse && i == 0 && g == 0) a.lse[at] = (M + (__builtin_amdgcn_logf(L) - P_BITS)) * 0.6931471805599453f;
  o *= L == 0.f ? 0.f : 1.f / L;
  store4((T *)a.out + at * HD + i * 16 + 4 * g, o);
}

// ---------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------
static int check_cache(const pd_byte_cache *c) {
  PD_REQUIRE(c, PD_EINVAL, "cache is NULL");
  PD_REQUIRE(c->n_req >= 1 && c->n_kv_head >= 1 && c->n_block >= 1, PD_EINVAL,
             "a byte cache has at least one request, head and block (got %d, %d, %d)", c->n_req, c->n_kv_head, c->n_block);
  PD_REQUIRE(c->head_dim == 32 || c->head_dim == 64 || c->head_dim == 96 || c->head_dim == 128, PD_EINVAL,
             "head_dim must be 32, 64, 96 or 128 (got %d)", c->head_dim);
  PD_REQUIRE(c->n_block <= (1 << 24), PD_EINVAL, "%d blocks per request: at most 2^24", c->n_block);
  PD_REQUIRE((int64_t)c->n_req * c->n_kv_head < (1ll << 26), PD_EINVAL, "too many requests and heads (%d x %d)", c->n_req,
             c->n_kv_head);
  PD_REQUIRE(c->k && c->v && c->k_scale && c->v_scale && c->k_tail && c->v_tail, PD_EINVAL, "a pointer of the cache is NULL");
  PD_REQUIRE((((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)c->k_tail | (uintptr_t)c->v_tail) & 15) == 0 &&
                 (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3) == 0,
             PD_EINVAL, "codes and tails must be 16-byte aligned, scales 4-byte aligned");
  return PD_OK;
}

static ByteCache view(const pd_byte_cache *c) {
  return ByteCache{(int8_t *)c->k, (int8_t *)c->v, c->k_scale, c->v_scale, c->k_tail, c->v_tail, c->n_req, c->n_kv_head, c->n_block};
}

static int type_bytes(int type) { return type == PD_TYPE_F32 ? 4 : 2; }
static int check_type(int type) {
  PD_REQUIRE(type == PD_TYPE_F32 || type == PD_TYPE_BF16 || type == PD_TYPE_F16, PD_EINVAL,
             "type must be PD_TYPE_F32, PD_TYPE_BF16 or PD_TYPE_F16 (got %d)", type);
  return PD_OK;
}
static int check_grid(int64_t blocks) {
  PD_REQUIRE(blocks < (1ll << 31), PD_EINVAL, "a launch of %lld work-groups is too large", (long long)blocks);
  return PD_OK;
}

// F(type, head_dim) for the run-time values
#define PD_BYTE_DIMS(T, HDV, F)                          \
  switch (HDV) {                                         \
    case 32: F(T, 32); break;                            \
    case 64: F(T, 64); break;                            \
    case 96: F(T, 96); break;                            \
    default: F(T, 128); break;                           \
  }
#define PD_BYTE_TYPES(TYPE, HDV, F)                      \
  switch (TYPE) {                                        \
    case PD_TYPE_F32: PD_BYTE_DIMS(float, HDV, F) break; \
    case PD_TYPE_BF16: PD_BYTE_DIMS(bf16_t, HDV, F) break; \
    default: PD_BYTE_DIMS(f16_t, HDV, F) break;          \
  }

extern "C" int pd_byte_append(const pd_byte_cache *cache, const void *k, const void *v, int type, const int64_t *k_strides,
                              const int64_t *v_strides, int n_new, const int32_t *counts, const int32_t *lens, void *hip_stream) {
  int rc;
  if ((rc = check_cache(cache)) || (rc = check_type(type))) return rc;
  PD_REQUIRE(n_new >= 0, PD_EINVAL, "n_new must be >= 0 (got %d)", n_new);
  if (n_new == 0) return PD_OK;
  PD_REQUIRE(k && v && k_strides && v_strides && lens, PD_EINVAL, "NULL argument");
  PD_REQUIRE((int64_t)n_new <= (int64_t)cache->n_block * BYTE_BLOCK, PD_EINVAL, "%d new tokens do not fit %d blocks", n_new,
             cache->n_block);
  const int es = type_bytes(type);
  PD_REQUIRE((((uintptr_t)k | (uintptr_t)v) & (es - 1)) == 0, PD_EINVAL, "keys and values must be aligned to their type");
  StoreArgs a;
  a.c = view(cache); a.src[0] = k; a.src[1] = v; a.counts = counts; a.lens = lens; a.n_new = n_new;
  a.span = (n_new + BYTE_BLOCK - 2) / BYTE_BLOCK + 1;
  uint64_t bits = (uintptr_t)k | (uintptr_t)v;
  for (int i = 0; i < 2; ++i) {
    const int64_t *st = i ? v_strides : k_strides;
    a.s_req[i] = st[0]; a.s_tok[i] = st[1]; a.s_head[i] = st[2];
    bits |= (uint64_t)((st[0] | st[1] | st[2]) * es);
  }
  const bool wide = (bits & 15) == 0;
  const int64_t blocks = (int64_t)cache->n_req * cache->n_kv_head * a.span * 2;
  if ((rc = check_grid(blocks))) return rc;
  hipStream_t s = (hipStream_t)hip_stream;
#define PD_STORE(T, HDV)                                                                                       \
  do {                                                                                                         \
    if (wide) hipLaunchKernelGGL((k_byte_store<T, HDV, true>), dim3((unsigned)blocks), dim3(256), 0, s, a);    \
    else hipLaunchKernelGGL((k_byte_store<T, HDV, false>), dim3((unsigned)blocks), dim3(256), 0, s, a);        \
  } while (0)
  PD_BYTE_TYPES(type, cache->head_dim, PD_STORE)
#undef PD_STORE
  PD_CHECK_HIP(hipGetLastError());
  return PD_OK;
}

extern "C" int pd_byte_read(const pd_byte_cache *cache, const int32_t *first, int n_tok, const int32_t *lens, void *out_k,
                            void *out_v, int type, void *hip_stream) {
  int rc;
  if ((rc = check_cache(cache)) || (rc = check_type(type))) return rc;
  PD_REQUIRE(n_tok >= 0, PD_EINVAL, "n_tok must be >= 0 (got %d)", n_tok);
  if (n_tok == 0) return PD_OK;
  PD_REQUIRE(lens && out_k && out_v, PD_EINVAL, "NULL argument");
  PD_REQUIRE((((uintptr_t)out_k | (uintptr_t)out_v) & 15) == 0, PD_EINVAL, "outputs must be 16-byte aligned");
  ReadArgs a;
  a.c = view(cache); a.out[0] = out_k; a.out[1] = out_v; a.first = first; a.lens = lens; a.n_tok = n_tok;
  a.span = first ? (n_tok - 1 + BYTE_BLOCK - 1) / BYTE_BLOCK + 1 : (n_tok + BYTE_BLOCK - 1) / BYTE_BLOCK;
  const int64_t blocks = (int64_t)cache->n_req * cache->n_kv_head * a.span * 2;
  if ((rc = check_grid(blocks))) return rc;
  hipStream_t s = (hipStream_t)hip_stream;
#define PD_READ(T, HDV) hipLaunchKernelGGL((k_byte_read<T, HDV>), dim3((unsigned)blocks), dim3(256), 0, s, a)
  PD_BYTE_TYPES(type, cache->head_dim, PD_READ)
#undef PD_READ
  PD_CHECK_HIP(hipGetLastError());
  return PD_OK;
}

struct ByteShape { int qt, nqg, nblk, nsplit, waves; int64_t units, grid; };

static int byte_shape(const pd_byte_cache *c, int n_head, int n_row, int max_len, ByteShape *out) {
  PD_REQUIRE(n_head >= 1 && n_head % c->n_kv_head == 0, PD_EINVAL, "n_head = %d is no multiple of %d key heads", n_head,
             c->n_kv_head);
  PD_REQUIRE(n_row >= 0 && max_len >= 0, PD_EINVAL, "n_row and max_len must be >= 0 (got %d, %d)", n_row, max_len);
  PD_REQUIRE((int64_t)n_row * (n_head / c->n_kv_head) < (1 << 30), PD_EINVAL, "too many rows and query heads (%d x %d)", n_row,
             n_head);
  const int64_t cap = (int64_t)c->n_block * BYTE_BLOCK;
  const int64_t most = max_len ? std::min<int64_t>(max_len, cap) : cap;
  const int64_t heads = (int64_t)c->n_req * c->n_kv_head;
  out->nblk = (int)((most + BYTE_BLOCK - 1) / BYTE_BLOCK);
  const ByteAttnShape sh = byte_attn_shape(n_row * (n_head / c->n_kv_head), heads, out->nblk, c->head_dim);
  out->qt = sh.tiles; out->waves = sh.waves; out->nsplit = sh.splits;
  out->nqg = sh.groups;
  out->units = heads * sh.groups;
  out->grid = out->units * out->nsplit;
  return check_grid(std::max(out->grid, out->units * out->qt * (c->head_dim / 16)));
}

extern "C" size_t pd_byte_attention_workspace_bytes(const pd_byte_cache *cache, int n_head, int n_row, int max_len) {
  ByteShape sh;
  if (check_cache(cache) || byte_shape(cache, n_head, n_row, max_len, &sh)) return 0;
  return sh.nsplit > 1 ? (size_t)sh.units * sh.qt * sh.nsplit * 16 * (cache->head_dim + 2) * sizeof(float) : 16;
}

extern "C" int pd_byte_attention(const pd_byte_cache *cache, const void *q, int type, const int64_t *q_strides, int n_head,
                                 int n_row, const int32_t *lens, const int32_t *row_limit, const uint16_t *key_tag,
                                 const int32_t *row_tag, float scale, int max_len, void *out, float *out_lse,
                                 void *workspace, size_t workspace_bytes, void *hip_stream) {
  int rc;
  ByteShape sh;
  if ((rc = check_cache(cache)) || (rc = check_type(type)) || (rc = byte_shape(cache, n_head, n_row, max_len, &sh))) return rc;
  if (n_row == 0) return PD_OK;
  PD_REQUIRE(q && q_strides && lens && out, PD_EINVAL, "NULL argument");
  PD_REQUIRE(!key_tag == !row_tag, PD_EINVAL, "key_tag and row_tag go together");
  PD_REQUIRE(((uintptr_t)key_tag & 15) == 0, PD_EINVAL, "key_tag must be 16-byte aligned");
  PD_REQUIRE(((uintptr_t)out & 15) == 0, PD_EINVAL, "out must be 16-byte aligned");
  const int es = type_bytes(type);
  PD_REQUIRE(((uintptr_t)q & (es - 1)) == 0, PD_EINVAL, "q must be aligned to its type");
  PD_REQUIRE(scale == scale && std::abs(scale) <= 2.0e38f, PD_EINVAL, "scale must be a number of magnitude up to 2e38");
  const size_t need = pd_byte_attention_workspace_bytes(cache, n_head, n_row, max_len);
  PD_REQUIRE(sh.nsplit == 1 || (workspace && workspace_bytes >= need), PD_ENOMEM, "workspace too small: %zu bytes given, %zu needed",
             workspace ? workspace_bytes : (size_t)0, need);
  PD_REQUIRE(sh.nsplit == 1 || ((uintptr_t)workspace & 15) == 0, PD_EINVAL, "workspace must be 16-byte aligned");
  ByteAttnArgs a;
  a.c = view(cache); a.q = q; a.q_req = q_strides[0]; a.q_row = q_strides[1]; a.q_head = q_strides[2];
  a.lens = lens; a.row_limit = row_limit; a.key_tag = key_tag; a.row_tag = row_tag; a.out = out; a.lse = out_lse;
  a.part = (float *)workspace; a.n_row = n_row; a.group = n_head / cache->n_kv_head;
  a.nqg = sh.nqg; a.qt = sh.qt; a.nsplit = sh.nsplit; a.nblk = sh.nblk;
  a.scale_log2 = (float)(scale * 1.4426950408889634);
  a.scale_low = (float)(std::abs(scale * 1.4426950408889634) - std::abs((double)a.scale_log2));
  a.q_wide = (((uintptr_t)q | (uint64_t)((q_strides[0] | q_strides[1] | q_strides[2]) * es)) & 15) == 0;
  hipStream_t s = (hipStream_t)hip_stream;
  if (type != PD_TYPE_F32 && byte_attn_pieces(n_row * a.group, (int64_t)cache->n_req * cache->n_kv_head)) {
    a.nqg = (n_row * a.group + 127) / 128;
    const int64_t work_groups = (int64_t)cache->n_req * cache->n_kv_head * a.nqg;
    if ((rc = check_grid(work_groups))) return rc;
#define PD_PIECE(T, HDV) \
  hipLaunchKernelGGL((k_byte_piece<T, HDV, std::is_same<T, f16_t>::value>), dim3((unsigned)work_groups), dim3(512), 0, s, a)
    if (type == PD_TYPE_BF16) PD_BYTE_DIMS(bf16_t, cache->head_dim, PD_PIECE)
    else PD_BYTE_DIMS(f16_t, cache->head_dim, PD_PIECE)
#undef PD_PIECE
    PD_CHECK_HIP(hipGetLastError());
    return PD_OK;
  }
  const unsigned grid = (unsigned)sh.grid, tiles = (unsigned)(sh.units * sh.qt * (cache->head_dim / 16));
#define PD_ATTEND_QT(T, HDV, QT, NW) \
  hipLaunchKernelGGL((k_byte_attn<T, HDV, !std::is_same<T, bf16_t>::value, QT, NW>), dim3(grid), dim3(64 * NW), 0, s, a)
#define PD_ATTEND(T, HDV)                                                                                    \
  do {                                                                                                       \
    if (sh.qt == 2 && sh.waves == 8) PD_ATTEND_QT(T, HDV, 2, 8);                                             \
    else if (sh.qt == 2) PD_ATTEND_QT(T, HDV, 2, 4);                                                         \
    else if (sh.waves == 8) PD_ATTEND_QT(T, HDV, 1, 8);                                                      \
    else PD_ATTEND_QT(T, HDV, 1, 4);                                                                         \
    if (sh.nsplit > 1) hipLaunchKernelGGL((k_byte_merge<T, HDV, !std::is_same<T, bf16_t>::value>), dim3(tiles), dim3(256), 0, s, a);          \
  } while (0)
  PD_BYTE_TYPES(type, cache->head_dim, PD_ATTEND)
#undef PD_ATTEND
#undef PD_ATTEND_QT
  PD_CHECK_HIP(hipGetLastError());
  return PD_OK;
}

// ---------------------------------------------------------------------------
// a decoder's context
// ---------------------------------------------------------------------------
// One work-group per (request, head, block of the context, keys or values): halves of the decoder's cache (two of its blocks of 32
// tokens), codes of this one.  Bound by the bytes: 4 x 4096 tokens of 32 heads of 128 in 88 us a layer, 4.6 TB/s of the 4.9 that a copy
// reaches; 8 x 2048 of 16 heads of 64 25 us, 1 x 8192 of 16 heads of 128 28, 1 x 1024 of 12 heads of 64 5.6.
template <int HD>
__global__ __launch_bounds__(256, 3) void k_byte_context(ByteCache c, const f16_t *kc, const f16_t *vc, int kv_cap, int n_whole) {
  constexpr int P = HD + 8;
  __shared__ f16_t tile[BYTE_BLOCK * P];
  __shared__ uint32_t sm_top[4];
  int u = blockIdx.x;
  const int h = u % c.n_kv_head; u /= c.n_kv_head;
  const int kind = u & 1, b = (u >> 1) % n_whole, req = (u >> 1) / n_whole;
  const size_t rhz = (size_t)req * c.n_kv_head + h;
  const uint4 *src = (const uint4 *)((kind ? vc : kc) + rhz * kv_cap * HD) + (size_t)b * BYTE_BLOCK * HD / 8;
  uint32_t top = 0;
#pragma unroll
  for (int it = 0; it < HD / 32; ++it) {
    const int e = threadIdx.x + it * 256, lane = e & 63, m = lane & 15, g = lane >> 4;
    union { uint4 q; f16_t h[8]; } y;
    y.q = src[e];
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, magnitude(y.h[j]));
    if (!kind) {                                         // fragment (32 tokens, tile, 32 dims): 8 dims of a token
      const int c32 = (e >> 6) % (HD / 32), t = (e >> 6) / (HD / 32);
      *(uint4 *)&tile[((t >> 1) * 32 + 8 * (m >> 2) + 4 * (t & 1) + (m & 3)) * P + c32 * 32 + g * 8] = y.q;
    } else {                                             // fragment (32 tokens, 16 dims): 8 tokens of a dim
      const int hb = (e >> 6) % (HD / 16), t32 = (e >> 6) / (HD / 16);
#pragma unroll
      for (int j = 0; j < 8; ++j) tile[(t32 * 32 + 8 * g + j) * P + hb * 16 + m] = y.h[j];
    }
  }
  seal_block<HD, P>(tile, sm_top, top, kind, c, rhz * c.n_block + b);
}

static ByteCache context_cache(const pd_ctx *c, const LayerPtrs &lp) {
  return ByteCache{lp.b_k, lp.b_v, lp.b_ks, lp.b_vs, nullptr, nullptr, c->B, c->cfg.n_head, c->byte_blocks_cap};
}

int byte_context_seal(pd_ctx *c, hipStream_t s) {
  const int n = c->L / BYTE_BLOCK, H = c->cfg.n_head;
  if (n == 0) return PD_OK;
  int rc = check_grid((int64_t)c->B * H * n * 2);
  if (rc) return rc;
  const dim3 grid((unsigned)(c->B * H * n * 2));
  for (const LayerPtrs &lp : c->layers) {
    if (!lp.b_k) continue;
    const ByteCache bc = context_cache(c, lp);
    const f16_t *kc = (const f16_t *)lp.kc, *vc = (const f16_t *)lp.vc;
    switch (c->cfg.head_dim) {
      case 32: hipLaunchKernelGGL(k_byte_context<32>, grid, dim3(256), 0, s, bc, kc, vc, c->kv_cap, n); break;
      case 64: hipLaunchKernelGGL(k_byte_context<64>, grid, dim3(256), 0, s, bc, kc, vc, c->kv_cap, n); break;
      case 96: hipLaunchKernelGGL(k_byte_context<96>, grid, dim3(256), 0, s, bc, kc, vc, c->kv_cap, n); break;
      default: hipLaunchKernelGGL(k_byte_context<128>, grid, dim3(256), 0, s, bc, kc, vc, c->kv_cap, n); break;
    }
  }
  PD_CHECK_HIP(hipGetLastError());
  return PD_OK;
}

int byte_context_attention(pd_ctx *c, const LayerPtrs &lw, int A, int nreq, int req0, hipStream_t s, int *splits) {
  const pd_config &g = c->cfg;
  ByteAttnArgs a;
  memset(&a, 0, sizeof(a));
  a.c = context_cache(c, lw);
  a.c.n_req = nreq;
  a.cq = (const f16_t *)c->q; a.cq_lo = (const f16_t *)mfma_lo(c, c->q, g.d_model);
  a.cout = (bf16_t *)c->att; a.cout_lo = mfma_lo(c, c->att, g.d_model);
  a.qinfo = c->rows.qinfo; a.gen_sub = c->sch.gen_sub; a.lens = c->sch.kv_len;
  a.hk = (const f16_t *)lw.kc; a.hv = (const f16_t *)lw.vc;
  a.gen_stride = c->gen_stride; a.kv_cap = c->kv_cap; a.L = c->L; a.req0 = req0;
  a.n_row = A; a.group = 1; a.nqg = (A + 15) / 16; a.qt = 1; a.nblk = c->L / BYTE_BLOCK;
  a.part = c->att_part;
  const double scale = 1.4426950408889634 / std::sqrt((double)g.head_dim);
  a.scale_log2 = (float)scale;
  // blocks of the middle of the run; the tokens behind the whole blocks are halves, 32 a block
  const int tail = c->L % BYTE_BLOCK + c->S * (c->M + 1) / 2;
  const int64_t units = (int64_t)nreq * a.nqg * g.n_head;
  PD_REQUIRE(units <= c->part_units, PD_EINVAL, "too many (request, head, query group) units: %lld", (long long)units);
  const ByteAttnShape shape = byte_attn_shape(16, units, a.nblk + (tail + 31) / 32, g.head_dim, 4.0);
  a.nsplit = c->opt_splits > 0 ? c->opt_splits : shape.splits;
  a.nsplit = (int)std::max<int64_t>(1, std::min<int64_t>(a.nsplit, c->part_units / units));
  *splits = a.nsplit;
  const int64_t grid = units * a.nsplit;
  int rc = check_grid(grid);
  if (rc) return rc;
#define PD_CONTEXT(HDV)                                                                                                       \
  do {                                                                                                                        \
    if (shape.waves == 8)                                                                                                     \
      hipLaunchKernelGGL((k_byte_attn<bf16_t, HDV, false, 1, 8, true>), dim3((unsigned)grid), dim3(512), 0, s, a);            \
    else                                                                                                                      \
      hipLaunchKernelGGL((k_byte_attn<bf16_t, HDV, false, 1, 4, true>), dim3((unsigned)grid), dim3(256), 0, s, a);            \
  } while (0)
  switch (g.head_dim) {
    case 32: PD_CONTEXT(32); break;
    case 64: PD_CONTEXT(64); break;
    case 96: PD_CONTEXT(96); break;
    default: PD_CONTEXT(128); break;
  }
#undef PD_CONTEXT
  PD_CHECK_HIP(hipGetLastError());
  return PD_OK;
}

static size_t context_layer_bytes(const pd_ctx *c) {
  const size_t units = (size_t)c->cfg.max_batch * c->cfg.n_head, blocks = (size_t)c->cfg.max_ctx / BYTE_BLOCK;
  const size_t codes = units * blocks * BYTE_BLOCK * c->cfg.head_dim, scales = (units * blocks * sizeof(float) + 255) / 256 * 256;
  return 2 * ((codes + 255) / 256 * 256 + scales);
}
static int context_layers(const pd_ctx *c) {
  int n = 0;
  for (const LayerPtrs &lp : c->layers) n += lp.kc_lo ? 0 : 1;
  return n;
}

extern "C" size_t pd_byte_context_bytes(const pd_ctx *c) {
  if (!c || c->arch == 1 || c->impl != 1) return 0;
  return std::max<size_t>(256, context_layers(c) * context_layer_bytes(c));
}

extern "C" int pd_byte_context(pd_ctx *c, void *dev_buffer, size_t bytes, void *hip_stream) {
  PD_REQUIRE(c, PD_EINVAL, "ctx is NULL");
  if (dev_buffer) {
    PD_REQUIRE(c->arch == 0 && c->impl == 1, PD_EINVAL,
               "an 8-bit context needs a decoder-only configuration on the matrix-core kernels");
    PD_REQUIRE(((uintptr_t)dev_buffer & 255) == 0, PD_EINVAL, "the buffer must be 256-byte aligned");
    const size_t need = pd_byte_context_bytes(c);
    PD_REQUIRE(bytes >= need, PD_ENOMEM, "buffer too small: %zu bytes given, %zu needed", bytes, need);
  }
  byte_context_drop_graph(c);
  const size_t units = (size_t)c->cfg.max_batch * c->cfg.n_head, blocks = (size_t)c->cfg.max_ctx / BYTE_BLOCK;
  const size_t codes = (units * blocks * BYTE_BLOCK * c->cfg.head_dim + 255) / 256 * 256;
  const size_t scales = (units * blocks * sizeof(float) + 255) / 256 * 256;
  c->byte_blocks_cap = (int)blocks;
  c->byte_context = dev_buffer != nullptr;
  char *p = (char *)dev_buffer;
  for (LayerPtrs &lp : c->layers) {
    const bool on = dev_buffer && !lp.kc_lo && blocks;
    lp.b_k = on ? (int8_t *)p : nullptr;
    lp.b_v = on ? (int8_t *)(p + codes) : nullptr;
    lp.b_ks = on ? (float *)(p + 2 * codes) : nullptr;
    lp.b_vs = on ? (float *)(p + 2 * codes + scales) : nullptr;
    if (on) p += 2 * (codes + scales);
  }
  if (!c->byte_context || !c->prefilled) return PD_OK;
  const int rc = byte_context_seal(c, (hipStream_t)hip_stream);
  if (rc) {                                              // without its codes the context stays in 16 bits
    c->byte_context = false;
    for (LayerPtrs &lp : c->layers) lp.b_k = lp.b_v = nullptr;
  }
  return rc;
}
