// A cache of keys and values in pages: storing tokens (keys and queries turned by their positions on the way), reading them back,
// attention of requests that may share a prefix.
//
// A page holds PD_PAGE = 64 tokens of every key head, in the order in which 16 lanes of a wave load 256 bytes that are operands of
// the 16x16x32 matrix instruction:
//   k  [page][head][hd / 8][64 tokens][8 dims]
//   v  [page][head][2][4][hd][8 tokens]            place i of (half s, group g): token 16 (2 s + (i >> 2)) + 4 g + (i & 3)
// where the order of a value's tokens is the one in which scores leave the instruction.
#include "paged_cache.h"

#include <algorithm>
#include <type_traits>

// ---------------------------------------------------------------------------
// store
// ---------------------------------------------------------------------------
struct PageStoreArgs {
  PageCache c;
  const void *src[3];                 // new keys, values, queries
  int64_t s_req[3], s_tok[3], s_head[3];
  int heads[3], groups[3];            // heads of each, and groups of STORE_HEADS of them
  const int32_t *counts, *lens, *pages, *places;
  const double *freqs;
  void *out_q;
  int n_freq, n_new, n_slot, span;    // most new tokens; blocks that they can touch
};

constexpr int STORE_HEADS = 8;

// 8 values that lie at a multiple of 16 bytes, as they are
template <typename T> __device__ __forceinline__ void fetch8(const T *p, T x[8]) {
  union { uint4 q[sizeof(T) / 2]; T h[8]; } y;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) y.q[i] = ((const uint4 *)p)[i];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = y.h[i];
}

// powers of two that hold n, as shifts
__device__ __forceinline__ int shift_for(int n) { return n <= 1 ? 0 : 32 - __clz(n - 1); }

// four tokens of eight dims each, as 16-bit values: the dims' four tokens, two to a register
__device__ __forceinline__ void dims_of(const uint4 t[4], uint2 d[8]) {
  const uint32_t w[4][4] = {{t[0].x, t[0].y, t[0].z, t[0].w}, {t[1].x, t[1].y, t[1].z, t[1].w},
                            {t[2].x, t[2].y, t[2].z, t[2].w}, {t[3].x, t[3].y, t[3].z, t[3].w}};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    d[2 * i] = make_uint2(__builtin_amdgcn_perm(w[1][i], w[0][i], 0x05040100u), __builtin_amdgcn_perm(w[3][i], w[2][i], 0x05040100u));
    d[2 * i + 1] = make_uint2(__builtin_amdgcn_perm(w[1][i], w[0][i], 0x07060302u), __builtin_amdgcn_perm(w[3][i], w[2][i], 0x07060302u));
  }
}
// and back
__device__ __forceinline__ void tokens_of(const uint2 d[8], uint4 t[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t sel = k & 1 ? 0x07060302u : 0x05040100u;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = k < 2 ? __builtin_amdgcn_perm(d[2 * i + 1].x, d[2 * i].x, sel) : __builtin_amdgcn_perm(d[2 * i + 1].y, d[2 * i].y, sel);
    t[k] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A work-group has up to 8 heads of keys, values or queries of the new tokens of one block.  The angles are taken once for all of
// them: place * freq in 64 bits as turns, less whole ones, so that far places lose nothing; sine and cosine of the rest by the
// instructions for them, whose errors of about 2^-20 vanish in the rounding to 16 bits (up to 2^-8, 2^-11 of the value).  A thread turns
// both halves of 8 pairs of dims; of values it takes 4 neighbouring tokens of 8 dims, which lie together in a page dim by dim (through
// rows of tokens in LDS, and every half of a pair with a load of its partner of its own: 69 us for 54).
// Bound by memory: 8192 tokens of 32 query, 8 key and 8 value heads of 128 (bf16, 201 MB in and out) 54 us, 3.7 TB/s of the 5.2 of a copy;
// few tokens by a chain of trips to memory (numbers, page, data): 32 x 16 tokens of 3 x 32 heads 11.4 us, one token of 3 x 12 3.8.
template <typename T, typename CT, int HD, bool WIDE>
__global__ __launch_bounds__(256) void k_page_store(PageStoreArgs a) {
  constexpr int NC = HD / 8;
  __shared__ __align__(16) float sm_cos[PD_PAGE * (HD / 2)], sm_sin[PD_PAGE * (HD / 2)];
  const int tid = threadIdx.x;
  int u = blockIdx.x;
  const int all = a.groups[0] + a.groups[1] + a.groups[2];
  int hg = u % all; u /= all;
  const int i0 = u % a.span, req = u / a.span;
  const int kind = hg < a.groups[0] ? 0 : hg < a.groups[0] + a.groups[1] ? 1 : 2;
  hg -= kind == 0 ? 0 : kind == 1 ? a.groups[0] : a.groups[0] + a.groups[1];
  const int h0 = hg * STORE_HEADS, nh = min(STORE_HEADS, a.heads[kind] - h0);
  const int count = a.counts ? a.counts[req] : a.n_new, len = a.lens[req];
  const bool fits = page_append_fits(len, count, a.n_new, a.n_slot);
  const int64_t s_tok = a.s_tok[kind], s_head = a.s_head[kind];
  const T *src = (const T *)a.src[kind] + req * a.s_req[kind] + h0 * s_head;
  CT *oq = (CT *)a.out_q + ((int64_t)req * a.n_new * a.heads[2] + h0) * HD;
  if (kind == 2) {                                       // queries of padding: zeros
    const int from = fits ? count : 0;
    const int64_t n = (int64_t)(a.n_new - from) * nh * NC;
    for (int64_t e = tid + i0 * 256; e < n; e += 256 * a.span) {
      const int c = e % NC, h = e / NC % nh;
      *(uint4 *)(oq + ((from + e / NC / nh) * a.heads[2] + h) * HD + c * 8) = make_uint4(0, 0, 0, 0);
    }
  }
  if (!fits) return;
  const int before = len - count, blk = before / PD_PAGE + i0;
  const int t0 = max(blk * PD_PAGE, before), t1 = min(blk * PD_PAGE + PD_PAGE, len), nt = t1 - t0, slot0 = t0 % PD_PAGE;
  if (nt <= 0) return;
  const int page = a.pages[(int64_t)req * a.n_slot + blk];
  if (kind < 2 && (unsigned)page >= (unsigned)a.c.n_page) return;
  src += (t0 - before) * s_tok;
  if (kind == 1) {
    // quads of tokens, of which all or some are new
    const int quad0 = slot0 >> 2, nq = ((slot0 + nt - 1) >> 2) - quad0 + 1, lg = shift_for(nq);
    uint16_t *dst = (uint16_t *)a.c.v + ((int64_t)page * a.c.n_kv_head + h0) * (PD_PAGE * HD);
    for (int e = tid; e < (nh << lg) * NC; e += 256) {
      const int c = e % NC, qd = e / NC & ((1 << lg) - 1), h = e / NC >> lg, first = (quad0 + qd) * 4 - slot0;
      if (qd >= nq) continue;
      float x[4][8];
#pragma unroll
      for (int k = 0; k < 4; ++k) load8<T, WIDE>(src + min(max(first + k, 0), nt - 1) * s_tok + h * s_head + c * 8, x[k]);
      uint4 y[4];
      uint2 d[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = cache8<CT>(x[k]);
      dims_of(y, d);
      uint16_t *p = dst + h * (PD_PAGE * HD) + value_place((quad0 + qd) * 4, HD) + c * 64;
      if (first >= 0 && first + 4 <= nt) {
#pragma unroll
        for (int i = 0; i < 8; ++i) *(uint2 *)(p + i * 8) = d[i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          union { uint2 q; uint16_t h[4]; } z;
          z.q = d[i];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (first + k >= 0 && first + k < nt) p[i * 8 + k] = z.h[k];
        }
      }
    }
    return;
  }
  const int n = a.n_freq;
  if (n) {
    const int lg = shift_for(n), j = tid & ((1 << lg) - 1);          // (a thread has one angle, of every so manieth token)
    if (j < n) {
      const double freq = a.freqs[j] * 0.15915494309189535;
      for (int t = tid >> lg; t < nt; t += 256 >> lg) {
        const int place = a.places ? a.places[(int64_t)req * a.n_new + t0 - before + t] : t0 + t;
        double turns = (double)place * freq;
        turns -= rint(turns);
        const float x = (float)turns;
        sm_cos[t * (HD / 2) + j] = __builtin_amdgcn_cosf(x);
        sm_sin[t * (HD / 2) + j] = __builtin_amdgcn_sinf(x);
      }
    }
    __syncthreads();
  }
  auto put = [&](int h, int t, int c, const float x[8]) {
    const uint4 y = cache8<CT>(x);
    if (kind == 0) ((uint4 *)a.c.k)[((int64_t)page * a.c.n_kv_head + h0 + h) * (PD_PAGE * NC) + c * PD_PAGE + slot0 + t] = y;
    else *(uint4 *)(oq + ((int64_t)(t0 - before + t) * a.heads[2] + h) * HD + c * 8) = y;
  };
  const int lt = shift_for(nt);
  if (WIDE && n % 8 == 0) {
    // 8 pairs of dims, or 8 dims behind the ones that turn; several such at a time, their values on their way together
    // (in the order in which they are written: queries head by head of a token, keys token by token of a head)
    const int np = n / 8, each = NC - np, lc = shift_for(each), lh = shift_for(nh), l0 = kind == 2 ? lh : lt, items = 1 << (lt + lc + lh);
    constexpr int U = sizeof(T) == 2 ? 4 : 2;
    for (int e0 = tid; e0 < items; e0 += 256 * U) {
      T x[U][2][8];
      int cc[U], tt[U], hh[U];
      bool ok[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int e = e0 + 256 * k;
        cc[k] = e & ((1 << lc) - 1);
        const int inner = e >> lc & ((1 << l0) - 1), outer = e >> (lc + l0);
        tt[k] = kind == 2 ? outer : inner; hh[k] = kind == 2 ? inner : outer;
        ok[k] = e < items && cc[k] < each && tt[k] < nt && hh[k] < nh;
        const T *p = src + (ok[k] ? tt[k] * s_tok + hh[k] * s_head + (cc[k] < np ? cc[k] : cc[k] + np) * 8 : 0);
        fetch8(p, x[k][0]);
        fetch8(ok[k] && cc[k] < np ? p + n : p, x[k][1]);
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (!ok[k]) continue;
        float lo[8], hi[8];
        if (cc[k] >= np) {
#pragma unroll
          for (int i = 0; i < 8; ++i) lo[i] = ld_f32(x[k][0], i);
          put(hh[k], tt[k], cc[k] + np, lo);
          continue;
        }
        const float *cs = sm_cos + tt[k] * (HD / 2) + cc[k] * 8, *sn = sm_sin + tt[k] * (HD / 2) + cc[k] * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x0 = ld_f32(x[k][0], i), x1 = ld_f32(x[k][1], i);
          lo[i] = x0 * cs[i] - x1 * sn[i];
          hi[i] = x1 * cs[i] + x0 * sn[i];
        }
        put(hh[k], tt[k], cc[k], lo);
        put(hh[k], tt[k], cc[k] + np, hi);
      }
    }
    return;
  }
  for (int e = tid; e < (nh << lt) * NC; e += 256) {
    const int c = e % NC, t = e / NC & ((1 << lt) - 1), h = e / NC >> lt;
    if (t >= nt) continue;
    const T *p = src + t * s_tok + h * s_head;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = c * 8 + i, j = d < n ? d : d - n;
      x[i] = ld_f32(p, d);
      if (d >= 2 * n) continue;
      const float y = ld_f32(p, d < n ? d + n : j), cs = sm_cos[t * (HD / 2) + j], sn = sm_sin[t * (HD / 2) + j];
      x[i] = d < n ? x[i] * cs - y * sn : x[i] * cs + y * sn;
    }
    put(h, t, c, x);
  }
}

// ---------------------------------------------------------------------------
// read
// ---------------------------------------------------------------------------
struct PageReadArgs {
  PageCache c;
  void *out[2];
  const int32_t *first, *lens, *pages;
  int n_tok, n_slot, span;
};

// A work-group has a block of tokens of 8 heads' keys or values; a thread 8 dims of 4 tokens (values: a quad, as they lie together; dim by
// dim with loads of 2 bytes 33 us for 19).  Bound by memory and its latency: 8192 tokens of 8 heads of 128 (67 MB in and out) 19 us, 3.5 TB/s.
template <typename T, typename CT, int HD>
__global__ __launch_bounds__(256) void k_page_read(PageReadArgs a) {
  constexpr int NC = HD / 8;
  int u = blockIdx.x;
  const int groups = (a.c.n_kv_head + STORE_HEADS - 1) / STORE_HEADS;
  const int h0 = u % groups * STORE_HEADS; u /= groups;
  const int kind = u & 1, i0 = (u >> 1) % a.span, req = (u >> 1) / a.span, nh = min(STORE_HEADS, a.c.n_kv_head - h0);
  const int len = min(a.lens[req], a.n_slot * PD_PAGE), first = a.first ? max(a.first[req], 0) : 0;
  const int64_t blk = first / PD_PAGE + i0, end = (int64_t)first + a.n_tok;
  const int64_t t0 = max(blk * PD_PAGE, (int64_t)first), t1 = min(blk * PD_PAGE + PD_PAGE, end);
  if (t0 >= t1) return;
  const int page = blk < a.n_slot ? a.pages[(int64_t)req * a.n_slot + blk] : -1;
  const int nt = (int)(t1 - t0), slot0 = (int)(t0 % PD_PAGE), quad0 = slot0 >> 2, nq = ((slot0 + nt - 1) >> 2) - quad0 + 1, lg = shift_for(nq);
  // tokens of the block that the request holds
  const int held = (unsigned)page < (unsigned)a.c.n_page ? (int)min(max((int64_t)len - t0, (int64_t)0), (int64_t)nt) : 0;
  const int64_t at = ((int64_t)(held ? page : 0) * a.c.n_kv_head + h0) * (PD_PAGE * HD);
  T *out = (T *)a.out[kind] + (((int64_t)req * a.n_tok + (t0 - first)) * a.c.n_kv_head + h0) * HD;
  for (int e = threadIdx.x; e < (nh << lg) * NC; e += 256) {
    const int c = e % NC, qd = e / NC & ((1 << lg) - 1), h = e / NC >> lg, slot = (quad0 + qd) * 4, t = slot - slot0;
    if (qd >= nq) continue;
    union { uint4 q; CT h[8]; } y[4];
    if (kind == 0) {
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k].q = *(const uint4 *)((const CT *)a.c.k + at + h * (PD_PAGE * HD) + (c * PD_PAGE + slot + k) * 8);
    } else {
      uint2 d[8];
      uint4 w[4];
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = *(const uint2 *)((const CT *)a.c.v + at + h * (PD_PAGE * HD) + value_place(slot, HD) + c * 64 + i * 8);
      tokens_of(d, w);
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k].q = w[k];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (t + k < 0 || t + k >= nt) continue;
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = t + k < held ? ld_f32(y[k].h, i) : 0.f;
      store8(out + ((int64_t)(t + k) * a.c.n_kv_head + h) * HD + c * 8, x);
    }
  }
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
// One row of one head by one wave, without matrix instructions: a lane per token for the scores, a lane per dim (or pair of
// them) for the outputs.  A token that is not seen is left out of every sum.
template <typename CT, int HD>
__device__ void page_row(const PageAttnArgs &a, int req, int row, int head) {
  constexpr int ND = (HD + 63) / 64;
  __shared__ float sm_p[4][PD_PAGE];
  __shared__ float sm_q[4][HD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = head / a.group;
  const CT *q = (const CT *)a.q + req * a.q_req + row * a.q_row + head * a.q_head;
  for (int d = lane; d < HD; d += 64) sm_q[wave][d] = ld_f32(q, d);
  wave_sync();
  const PageSpan sp = page_span(a, req);
  int lim = sp.len;
  if (a.row_limit) lim = min(lim, a.row_limit[(int64_t)req * a.n_row + row]);
  const int tag = a.key_tag ? a.row_tag[(int64_t)req * a.n_row + row] : 0;
  float m = -INFINITY, l = 0.f, o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) o[i] = 0.f;
  for (int part = 0; part < 2; ++part) {
    const int lo = part ? sp.shared : 0, hi = part ? lim : min(lim, sp.shared);
    const int32_t *pages = a.pages + (int64_t)(part ? req : sp.lead) * a.n_slot;
    for (int b = lo / PD_PAGE; b * PD_PAGE < hi; ++b) {
      const int page = pages[b];
      if ((unsigned)page >= (unsigned)a.c.n_page) continue;
      const int64_t at = ((int64_t)page * a.c.n_kv_head + h) * (PD_PAGE * HD);
      const int j = b * PD_PAGE + lane;
      bool sees = j >= lo && j < hi;
      if (part && a.key_tag) sees = sees && (int)a.key_tag[(int64_t)req * a.n_slot * PD_PAGE + j] <= tag;
      float s = 0.f;
#pragma unroll 1
      for (int c = 0; c < HD / 8; ++c) {
        float k[8];
        load8<CT, true>((const CT *)a.c.k + at + (c * PD_PAGE + lane) * 8, k);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(k[i], sm_q[wave][c * 8 + i], s);
      }
      const uint64_t seen = __ballot(sees);
      if (seen == 0) continue;
      s = sees ? s * a.scale_log2 : -INFINITY;
      const float top = fmaxf(m, fold_wave(s, Max())), ref = top == -INFINITY ? 0.f : top;
      const float down = __builtin_amdgcn_exp2f(m - ref), p = sees ? __builtin_amdgcn_exp2f(s - ref) : 0.f;
      m = top;
      l = l * down + fold_wave(p, Add());
      sm_p[wave][lane] = p;
      wave_sync();
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        const int d = lane + 64 * i;
        o[i] *= down;
        if (d >= HD) continue;
#pragma unroll 1
        for (int t = 0; t < PD_PAGE; ++t)
          if (seen >> t & 1) o[i] = fmaf(sm_p[wave][t], ld_f32((const CT *)a.c.v, at + value_place(t, HD) + d * 8), o[i]);
      }
      wave_sync();
    }
  }
  const int64_t out = ((int64_t)req * a.n_row + row) * a.n_head + head;
#pragma unroll
  for (int i = 0; i < ND; ++i)
    if (lane + 64 * i < HD) st_out((CT *)a.out, out * HD + lane + 64 * i, l == 0.f ? 0.f : o[i] / l);
  if (a.lse && lane == 0) a.lse[out] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}


template <typename CT> __device__ __forceinline__ floatx4 product(const Frag &a, const Frag &b, floatx4 c);
template <> __device__ __forceinline__ floatx4 product<bf16_t>(const Frag &a, const Frag &b, floatx4 c) { return mfma16(a, b, c); }
template <> __device__ __forceinline__ floatx4 product<f16_t>(const Frag &a, const Frag &b, floatx4 c) { return mfma16h(a, b, c); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// A number of the page table, the same for the whole wave, by the scalar path: as a vector load it would be waited for in order, behind
// all keys and values that are on their way.
__device__ __forceinline__ int page_number(const int32_t *pages, int b) {
  return ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)pages)[b];
}

// Probabilities meet the values in the cache's type, each up to 2^-8 off (halves 2^-11): the matrix instructions of 16 bits take 16-bit
// operands, and in two parts they would be half as many again.  Outputs are off by 2.0e-3 in the mean (2.5e-4), their own rounding 1.7e-3 (2.1e-4)
// of that.
// Probabilities are 2^PAGE_BITS times what the running maximum makes them (halves: further from the smallest half), and the maximum
// moves where it grows by more than 2^PAGE_SLACK, so that it is rarely looked for across lanes and the sums are rarely scaled: at most 2^14 of
// 65504.
template <typename CT> constexpr float PAGE_BITS = std::is_same<CT, f16_t>::value ? 8.f : 0.f;
constexpr float PAGE_SLACK = 6.f;

// 16 columns of a wave: their queries as operands, what they see, and their sums.
template <typename CT, int HD>
struct PageCols {
  static constexpr int NS = HD / 32, NT = HD / 16;
  Frag q[NS];
  int lim, tag;                       // tokens below lim, with tags up to tag; lim 0 where there is no column
  float m, l;                         // l: this lane's share
  floatx4 o[NT];

  __device__ __forceinline__ void start(const PageAttnArgs &a, const PageWork &w, bool shared, int unit, int col) {
    const int h = unit % a.c.n_kv_head, first = unit / a.c.n_kv_head * (shared ? a.per_group : 1), g = (threadIdx.x & 63) >> 4;
    const bool there = col < w.cols;
    const int cols = a.n_row * a.group, c = there ? col : 0, r = shared ? c / cols : 0, cc = c - r * cols, row = cc / a.group;
    const int req = first + r, head = h * a.group + cc - row * a.group;
    const CT *p = (const CT *)a.q + req * a.q_req + row * a.q_row + head * a.q_head + 8 * g;
    // (the sign of the scale is taken into the queries, which is exact; a scale of zero makes them zeros)
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u, keep = a.scale_log2 == 0.f || !there ? 0u : ~0u;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      if (a.q_wide) {
        q[s].u = *(const uint4 *)(p + s * 32);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[s].h[i] = ((const uint16_t *)p)[s * 32 + i];
      }
      q[s].u = make_uint4((q[s].u.x ^ flip) & keep, (q[s].u.y ^ flip) & keep, (q[s].u.z ^ flip) & keep, (q[s].u.w ^ flip) & keep);
    }
    const PageSpan sp = page_span(a, req);
    lim = sp.len;
    if (a.row_limit) lim = min(lim, max(a.row_limit[(int64_t)req * a.n_row + row], 0));
    if (shared) lim = min(lim, sp.shared);
    if (!there) lim = 0;
    tag = a.key_tag && !shared ? a.row_tag[(int64_t)req * a.n_row + row] : 0x7fffffff;
    m = -INFINITY; l = 0.f;
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // s: scores of a block, element e of tile t: token key0 + 16 t + e of this lane's column.  Their probabilities as operands.
  // whole: all columns of the wave see the whole block; else this one sees the tokens from lo on and below lim with tags up to tag
  __device__ __forceinline__ void weigh(floatx4 s[4], Frag p[2], float c, bool whole, int key0, int lo, int lim, int tag, const uint2 tags[4]) {
    if (!whole) {
      asm volatile("");                                 // (a branch, not 48 comparisons in every block)
      const int below = lim - key0, from = lo - key0;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t w[2] = {tags[t].x, tags[t].y};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = 16 * t + e, mark = (w[e >> 1] >> (16 * (e & 1))) & 0xffff;
          s[t][e] = ((at < below) & (at >= from) & (mark <= tag)) ? s[t][e] : -INFINITY;
        }
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e >> 2][e & 3]);
    // (a lane's own tokens are enough to see whether the maximum has to move: 302 us for 316, 1024 rows behind 16384 tokens)
    if (__any(top * c > m + PAGE_SLACK)) {
      asm volatile("");
      top = fold32(fold16(top, Max()), Max()) * c;
      const float m_new = top > m + PAGE_SLACK ? top : m, down = __builtin_amdgcn_exp2f(m - (m_new == -INFINITY ? 0.f : m_new));
      m = m_new;
      l *= down;
#pragma unroll
      for (int i = 0; i < NT; ++i) o[i] *= down;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
    const float off = PAGE_BITS<CT> - ref;
    // (the product is not rounded before the maximum, which was, is taken off: where a rounding of it is more than a small part of an
    // exponent, it has to be)
    if (__any(fabsf(ref) > 1048576.f)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e >> 2][e & 3] = __fmul_rn(s[e >> 2][e & 3], c);
      c = 1.f;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3], c, off));
      s[e >> 2][e & 3] = x;
      sum += x;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (std::is_same<CT, f16_t>::value) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[i].hh[e] = (f16_t)s[2 * i + (e >> 2)][e & 3];
      } else {
        p[i].u = make_uint4(pack2(s[2 * i][0], s[2 * i][1]), pack2(s[2 * i][2], s[2 * i][3]),
                            pack2(s[2 * i + 1][0], s[2 * i + 1][1]), pack2(s[2 * i + 1][2], s[2 * i + 1][3]));
      }
    }
    l += sum;
  }
};

// Where a column's results go: to the outputs, where this is all there is, else to the partial results.
template <typename CT, int HD>
__device__ __forceinline__ void page_result(const PageAttnArgs &a, const PageWork &w, bool shared, int unit, int split, int col, bool alone,
                                            float m, float l, const floatx4 *o) {
  constexpr int NT = HD / 16;
  const int g = (threadIdx.x & 63) >> 4;
  const bool there = col < w.cols;
  if (!alone) {
    if (!there) return;
    const int64_t at = w.first + ((int64_t)unit * w.splits + split) * w.cols + col;
    if (g == 0) *(float2 *)(a.sums + a.n_cols * HD + at * 2) = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < NT; ++i) *(floatx4 *)(a.sums + at * HD + i * 16 + 4 * g) = o[i];
    return;
  }
  const int row = col / a.group, head = unit % a.c.n_kv_head * a.group + col - row * a.group, req = unit / a.c.n_kv_head;
  const int64_t at = ((int64_t)req * a.n_row + row) * a.n_head + head;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bool fine = true;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const floatx4 y = o[i] * inv;
#pragma unroll
    for (int e = 0; e < 4; ++e) fine = fine && fabsf(y[e]) < INFINITY;
    if (there) store4((CT *)a.out + at * HD + i * 16 + 4 * g, y);
  }
  if (a.lse && there && g == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + (__builtin_amdgcn_logf(l) - PAGE_BITS<CT>)) * 0.6931471805599453f;
  uint64_t bad = __ballot(there && !fine);
  bad = (bad | bad >> 16 | bad >> 32 | bad >> 48) & 0xffff;
  for (; bad; bad &= bad - 1) {                          // (values that are not finite where a row sees them, or does not)
    const int n = __ffsll((unsigned long long)bad) - 1;
    page_row<CT, HD>(a, __builtin_amdgcn_readlane(req, n), __builtin_amdgcn_readlane(row, n), __builtin_amdgcn_readlane(head, n));
  }
}

// Attention by matrix instructions.  A work-group has some columns of a unit and a split of its blocks of 64 tokens.  Scores are S^T = K Q^T,
// outputs O^T = V^T P^T: the scores of a column leave the first product in the registers and the order in which the second one
// takes them.
//   width 16       the four waves have the same 16 columns and take the blocks in turn, keys and values straight into registers, the
//                  next block's on the way while one is multiplied
//   width 64, 128  every wave has 16 or 32 columns of its own, and the blocks come to LDS once for all four, the next one while one is
//                  multiplied
// What a group shares has work-groups of its own, for the columns of all its requests, or comes in front of every request's blocks where
// that costs less (PageAttnShape): 15 x 95 rows of 32 heads of 128, 32 shared tokens and up to 95 of their own, 20.3 us for 43.7.
// It is read once for all of its columns: 4 x 4096 tokens of 32 heads of 128 continued 8 times each, with up to 500 tokens
// of their own (403 MB), in 80 us, 5.0 of a copy's 5.2 TB/s.  With many columns a block of width 128 takes a compute unit about 4100 clocks,
// 1024 of them for matrix instructions on every SIMD: reads of LDS (128 KB for four waves) and the softmax (32 exponentials, a quarter of
// the rate of others, and 130 other instructions a lane) do not overlap with them in one wave.  Two work-groups to a compute unit
// take 2900 each: 1024 rows of 32 heads over 8 key heads, 16384 tokens 302 us, 910 TFLOP/s, one 475.  Values straight into every wave's
// registers instead of LDS spill and take 10 % more; LDS filled without registers in between, which has the first read of a block
// wait for the next one's, 54 us for 45 (64 rows).
template <typename CT, int HD>
__global__ __launch_bounds__(256, 2) void k_page_attn(PageAttnArgs a) {
  constexpr int NS = HD / 32, NT = HD / 16, BLOCK = PD_PAGE * HD / 8;       // granules of 16 bytes
  __shared__ uint4 sm[2][2][BLOCK];
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const bool shared = blockIdx.x < a.n_shared;
  const PageWork w = a.part[shared ? 0 : 1];
  const PagePiece me = page_piece(shared ? blockIdx.x : blockIdx.x - (int)a.n_shared, w.units * w.splits, w.tiles);
  const int unit = me.piece / w.splits, split = me.piece % w.splits, tile = me.tile, h = unit % a.c.n_kv_head;
  const int req = unit / a.c.n_kv_head * (shared ? a.per_group : 1);
  const PageSpan sp = page_span(a, req);
  const int lo = shared ? 0 : sp.shared, b0 = lo / PD_PAGE;
  const int32_t *pages = a.pages + (int64_t)req * a.n_slot;
  const uint16_t *tag_row = a.key_tag && !shared ? a.key_tag + (int64_t)req * a.n_slot * PD_PAGE : nullptr;
  const float c = fabsf(a.scale_log2) == 0.f ? 1.f : fabsf(a.scale_log2);
  const bool alone = !shared && a.n_shared == 0 && w.splits == 1;
  const uint4 *K = (const uint4 *)a.c.k + (int64_t)h * BLOCK, *V = (const uint4 *)a.c.v + (int64_t)h * BLOCK;
  const int64_t step = (int64_t)a.c.n_kv_head * BLOCK;

  auto run = [&](auto qt_) {
    constexpr int QT = decltype(qt_)::value;               // 0: all waves the same 16 columns
    constexpr int NQ = QT ? QT : 1;
    PageCols<CT, HD> x[NQ];
    int reach = 0, lim_all = 0x7fffffff, tag_all = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int col = tile * w.width + (QT ? (wave * QT + i) * 16 : 0) + n;
      x[i].start(a, w, shared, unit, col);
      reach = max(reach, x[i].lim);
      if (col < w.cols) { lim_all = min(lim_all, x[i].lim); tag_all = min(tag_all, x[i].tag); }
    }
    reach = uniform(fold_row(reach, Max()));
    lim_all = uniform(fold_row(lim_all, Min()));
    tag_all = uniform(fold_row(tag_all, Min()));
    // the blocks of this split: of those that any of the work-group's columns reaches
    int far = reach;
    if (QT) {
      int *ends = (int *)sm;
      if (lane == 0) ends[wave] = reach;
      __syncthreads();
      far = uniform(max(max(ends[0], ends[1]), max(ends[2], ends[3])));
      __syncthreads();
    }
    // (where what is shared has no work-groups of its own, its blocks come in front)
    const int front = !shared && a.n_shared == 0 ? (min(far, sp.shared) + PD_PAGE - 1) / PD_PAGE : 0;
    const int n_blocks = min(front + max((far + PD_PAGE - 1) / PD_PAGE - b0, 0), w.blocks);
    const int s0 = (int)((int64_t)n_blocks * split / w.splits), s1 = (int)((int64_t)n_blocks * (split + 1) / w.splits);
    auto good = [&](int page) { return (unsigned)page < (unsigned)a.c.n_page; };
    const int32_t *lead = a.pages + (int64_t)sp.lead * a.n_slot;
    auto block_of = [&](int i) { return i < front ? i : b0 + i - front; };
    auto find = [&](int i) { return i >= s1 ? -1 : i < front ? page_number(lead, i) : page_number(pages, b0 + i - front); };
    uint2 tags[4] = {make_uint2(0, 0), make_uint2(0, 0), make_uint2(0, 0), make_uint2(0, 0)};
    auto load_tags = [&](int b) {
      if (tag_row)
#pragma unroll
        for (int t = 0; t < 4; ++t) tags[t] = *(const uint2 *)(tag_row + b * PD_PAGE + 16 * t + 4 * g);
    };
    auto sees_all = [&](int b, int lo, int lim_all, bool tagged) {       // whether all columns of the wave see the whole block
      bool all = b * PD_PAGE >= lo && b * PD_PAGE + PD_PAGE <= lim_all;
      if (tagged) {
        uint32_t top = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t)
          top = max(max(top, max(tags[t].x & 0xffff, tags[t].x >> 16)), max(tags[t].y & 0xffff, tags[t].y >> 16));
        all = all && !__any((int)top > tag_all);
      }
      return (bool)uniform(all);
    };
    if constexpr (QT == 0) {
      Frag k[4][NS], v[NT][2];
      int page_k = 0, page_v = 0;
      auto load_k = [&](int page) {
        const uint4 *p = K + (good(page) ? page : 0) * step;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int t = 0; t < 4; ++t) k[t][s].u = p[(s * 4 + g) * PD_PAGE + t * 16 + n];
      };
      auto load_v = [&](int page) {
        const uint4 *p = V + (good(page) ? page : 0) * step;
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int s = 0; s < 2; ++s) v[i][s].u = p[(s * 4 + g) * HD + i * 16 + n];
      };
      int i = s0 + wave;
      if (i < s1) {
        page_k = find(i);
        load_k(page_k);
        load_tags(block_of(i));
        load_v(page_k);
      }
      for (; i < s1; i += 4) {
        page_v = page_k;
        page_k = find(i + 4);
        floatx4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < NS; ++d)
#pragma unroll
          for (int t = 0; t < 4; ++t) s[t] = product<CT>(k[t][d], x[0].q[d], s[t]);
        const bool ahead = i < front;                      // (of what is shared)
        const int b = block_of(i), from = ahead ? 0 : lo, lim = ahead ? min(x[0].lim, sp.shared) : x[0].lim;
        const bool whole = sees_all(b, from, ahead ? min(lim_all, sp.shared) : lim_all, tag_row && !ahead) && good(page_v);
        __builtin_amdgcn_sched_barrier(0);
        if (i + 4 < s1) load_k(page_k);
        __builtin_amdgcn_sched_barrier(0);
        Frag p[2];
        x[0].weigh(s, p, c, whole, good(page_v) ? b * PD_PAGE + 4 * g : 0x7fffff00, from, lim, ahead ? 0x7fffffff : x[0].tag, tags);
#pragma unroll
        for (int d = 0; d < NT; ++d) {
          x[0].o[d] = product<CT>(v[d][0], p[0], x[0].o[d]);
          x[0].o[d] = product<CT>(v[d][1], p[1], x[0].o[d]);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (i + 4 < s1) { load_tags(block_of(i + 4)); load_v(page_k); }
        __builtin_amdgcn_sched_barrier(0);
      }
      // the waves' sums become one
      x[0].l = fold32(fold16(x[0].l, Add()), Add());
      floatx4 *so = (floatx4 *)sm;                         // [wave][dims / 16][lane]
      float *sml = (float *)(so + 4 * NT * 64);            // [wave][16][2]
      static_assert(sizeof(sm) >= 4 * NT * 64 * 16 + 4 * 16 * 8, "");
#pragma unroll
      for (int i = 0; i < NT; ++i) so[(wave * NT + i) * 64 + lane] = x[0].o[i];
      if (g == 0) { sml[(wave * 16 + n) * 2] = x[0].m; sml[(wave * 16 + n) * 2 + 1] = x[0].l; }
      __syncthreads();
      if (wave != 0) return;
      float M = -INFINITY, L = 0.f, f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) M = fmaxf(M, sml[(j * 16 + n) * 2]);
      const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f[j] = __builtin_amdgcn_exp2f(sml[(j * 16 + n) * 2] - ref);
        L = fmaf(f[j], sml[(j * 16 + n) * 2 + 1], L);
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        x[0].o[i] *= f[0];
#pragma unroll
        for (int j = 1; j < 4; ++j) x[0].o[i] += f[j] * so[(j * NT + i) * 64 + lane];
      }
      wave_sync();
      page_result<CT, HD>(a, w, shared, unit, split, tile * w.width + n, alone, M, L, x[0].o);
    } else {
      // (a block comes through registers: behind loads that go straight to LDS, which any read of LDS may depend on, the compiler has
      // the first read wait for all of them, with nothing on the way while a block is multiplied)
      constexpr int PART = BLOCK / 256;
      typedef uint32_t Granule __attribute__((ext_vector_type(4)));
      Granule rk[PART], rv[PART];
      auto fetch = [&](int page) {
        const int64_t at = (unsigned)page < (unsigned)a.c.n_page ? page * step : 0;
#pragma unroll
        for (int i = 0; i < PART; ++i) rk[i] = ((const Granule *)K)[at + i * 256 + threadIdx.x];
#pragma unroll
        for (int i = 0; i < PART; ++i) rv[i] = ((const Granule *)V)[at + i * 256 + threadIdx.x];
      };
      auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < PART; ++i) ((Granule *)sm[buf][0])[i * 256 + threadIdx.x] = rk[i];
#pragma unroll
        for (int i = 0; i < PART; ++i) ((Granule *)sm[buf][1])[i * 256 + threadIdx.x] = rv[i];
      };
      int page = find(s0);
      if (s0 < s1) { load_tags(block_of(s0)); fetch(page); put(0); }
      int next = find(s0 + 1);
      __syncthreads();
      for (int i = s0, buf = 0; i < s1; ++i, buf ^= 1) {
        const int here = page, b = block_of(i);
        const bool ahead = i < front;                      // (of what is shared)
        page = next;
        fetch(i + 1 < s1 ? page : here);                    // (behind the last one: it again)
        next = find(i + 2);
        __builtin_amdgcn_sched_barrier(0);
        if (good(here) && b * PD_PAGE < reach) {
          const int from = ahead ? 0 : lo, most = ahead ? sp.shared : 0x7fffffff;
          const bool whole = sees_all(b, from, min(lim_all, most), tag_row && !ahead);
          const uint4 *kl = &sm[buf][0][g * PD_PAGE + n], *vl = &sm[buf][1][g * HD + n];
          floatx4 s[NQ][4];
          Frag f[2][4];
          // the next operands are read while some are multiplied
#pragma unroll
          for (int t = 0; t < 4; ++t) f[0][t].u = kl[t * 16];
#pragma unroll
          for (int d = 0; d < NS; ++d) {
            if (d + 1 < NS)
#pragma unroll
              for (int t = 0; t < 4; ++t) f[(d + 1) & 1][t].u = kl[(d + 1) * 4 * PD_PAGE + t * 16];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int j = 0; j < NQ; ++j) s[j][t] = product<CT>(f[d & 1][t], x[j].q[d], d ? s[j][t] : floatx4{0.f, 0.f, 0.f, 0.f});
            __builtin_amdgcn_sched_barrier(0);
          }
          // (two tiles of 16 dims, both halves of the tokens)
          auto values = [&](int d, Frag *to) {
#pragma unroll
            for (int j = 0; j < 4; ++j) to[j].u = vl[(j & 1) * 4 * HD + (d + (j >> 1)) * 16];
          };
          Frag p[NQ][2];
#pragma unroll
          for (int j = 0; j < NQ; ++j) {
            if (j == NQ - 1) values(0, f[0]);
            x[j].weigh(s[j], p[j], c, whole, b * PD_PAGE + 4 * g, from, min(x[j].lim, most), ahead ? 0x7fffffff : x[j].tag, tags);
            __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll
          for (int d = 0; d < NT; d += 2) {
            if (d + 2 < NT) values(d + 2, f[((d >> 1) + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int j = 0; j < NQ; ++j)
                x[j].o[d + (e >> 1)] = product<CT>(f[(d >> 1) & 1][e], p[j][e & 1], x[j].o[d + (e >> 1)]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (i + 1 < s1) {
          load_tags(block_of(i + 1));
          put(buf ^ 1);
          __syncthreads();
        }
      }
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        x[i].l = fold32(fold16(x[i].l, Add()), Add());
        page_result<CT, HD>(a, w, shared, unit, split, tile * w.width + (wave * QT + i) * 16 + n, alone, x[i].m, x[i].l, x[i].o);
      }
    }
  };
  if (w.width == 16) run(std::integral_constant<int, 0>());
  else if (w.width == 64) run(std::integral_constant<int, 1>());
  else run(std::integral_constant<int, 2>());
}

// The partial results of a row and head become one: a lane has four dims of them, 8 to 32 lanes a row and head, and all of these look
// at every part's maximum and sum themselves (a wave a row, with the parts' factors from lane to lane: 15 us for 5.8, 16384 rows of
// 64 dims in three parts; 6.0 for 5.3, 1024 rows of 128 in 17).  Bound by the trips to memory: 4 to 7 us.
constexpr int merge_lanes(int hd) { return hd == 96 ? 32 : hd / 4; }
constexpr int merge_rows(int hd) { return 256 / merge_lanes(hd); }
template <typename CT, int HD>
__global__ __launch_bounds__(256) void k_page_merge(PageAttnArgs a) {
  constexpr int LANES = merge_lanes(HD);
  const int d = threadIdx.x % LANES * 4;
  const int64_t rows = (int64_t)a.n_req * a.n_row * a.n_head, i = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const bool there = i < rows, mine = there && d < HD;
  const uint32_t at = there ? (uint32_t)i : 0, line = at / (uint32_t)a.n_head;               // (fewer than 2^31 of them)
  const int head = (int)(at - line * a.n_head), req = (int)(line / (uint32_t)a.n_row), row = (int)(line - (uint32_t)req * a.n_row);
  const int h = head / a.group, col = row * a.group + head - h * a.group;
  const float2 *ml[2];
  const float *x[2];
  float M = -INFINITY, L = 0.f;
  for (int part = a.n_shared ? 0 : 1; part < 2; ++part) {
    const PageWork &w = a.part[part];
    const int g = part ? req : req / a.per_group, c = part ? col : (req - g * a.per_group) * a.n_row * a.group + col;
    const int64_t first = w.first + (int64_t)(g * a.c.n_kv_head + h) * w.splits * w.cols + c;
    ml[part] = (const float2 *)(a.sums + a.n_cols * HD) + first;
    x[part] = a.sums + first * HD + (d < HD ? d : 0);
#pragma unroll 8
    for (int s = 0; s < w.splits; ++s) M = fmaxf(M, ml[part][(int64_t)s * w.cols].x);
  }
  const float ref = M == -INFINITY ? 0.f : M;
  floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int part = a.n_shared ? 0 : 1; part < 2; ++part) {
    const PageWork &w = a.part[part];
#pragma unroll 8
    for (int s = 0; s < w.splits; ++s) {
      const float2 own = ml[part][(int64_t)s * w.cols];
      const floatx4 y = *(const floatx4 *)(x[part] + (int64_t)s * w.cols * HD);
      const float f = own.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(own.x - ref);
      L = fmaf(f, own.y, L);
      o += f * y;
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  o *= inv;
  bool fine = true;
#pragma unroll
  for (int e = 0; e < 4; ++e) fine = fine && fabsf(o[e]) < INFINITY;
  if (mine) store4((CT *)a.out + i * HD + d, o);
  if (a.lse && there && d == 0) a.lse[i] = L == 0.f ? -INFINITY : (M + (__builtin_amdgcn_logf(L) - PAGE_BITS<CT>)) * 0.6931471805599453f;
  const uint64_t bad = __ballot(mine && !fine);
  if (bad == 0) return;
  wave_sync();
  for (int l = 0; l < 64; l += LANES)                    // (values that are not finite where a row sees them, or does not)
    if (bad >> l & ((1ull << LANES) - 1))
      page_row<CT, HD>(a, __builtin_amdgcn_readlane(req, l), __builtin_amdgcn_readlane(row, l), __builtin_amdgcn_readlane(head, l));
}

// ---------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------
static int check_pages(const pd_page_cache *c, const int32_t *pages, int n_req, int n_slot) {
  PD_REQUIRE(c, PD_EINVAL, "cache is NULL");
  PD_REQUIRE(c->type == PD_TYPE_BF16 || c->type == PD_TYPE_F16, PD_EINVAL, "a paged cache holds PD_TYPE_BF16 or PD_TYPE_F16 (got %d)", c->type);
  PD_REQUIRE(c->head_dim == 32 || c->head_dim == 64 || c->head_dim == 96 || c->head_dim == 128, PD_EINVAL,
             "head_dim must be 32, 64, 96 or 128 (got %d)", c->head_dim);
  PD_REQUIRE(c->n_page >= 1 && c->n_kv_head >= 1 && c->n_kv_head <= (1 << 20), PD_EINVAL,
             "a paged cache has at least one page and 1 to 2^20 heads (got %d, %d)", c->n_page, c->n_kv_head);
  PD_REQUIRE(c->k && c->v && pages, PD_EINVAL, "a pointer of the cache or its pages is NULL");
  PD_REQUIRE((((uintptr_t)c->k | (uintptr_t)c->v) & 15) == 0 && ((uintptr_t)pages & 3) == 0, PD_EINVAL,
             "keys and values must be 16-byte aligned, pages 4-byte aligned");
  PD_REQUIRE(n_req >= 1 && n_req <= (1 << 24), PD_EINVAL, "n_req must be within 1 and 2^24 (got %d)", n_req);
  PD_REQUIRE(n_slot >= 1 && n_slot <= (1 << 24), PD_EINVAL, "n_slot must be within 1 and 2^24 (got %d)", n_slot);
  return PD_OK;
}
static PageCache view(const pd_page_cache *c) { return PageCache{c->k, c->v, c->n_page, c->n_kv_head}; }
static int type_bytes(int type) { return type == PD_TYPE_F32 ? 4 : 2; }
static int check_type(int type) {
  PD_REQUIRE(type == PD_TYPE_F32 || type == PD_TYPE_BF16 || type == PD_TYPE_F16, PD_EINVAL,
             "type must be PD_TYPE_F32, PD_TYPE_BF16 or PD_TYPE_F16 (got %d)", type);
  return PD_OK;
}
// a launch of a * b work-groups of 256 threads, of which it may have fewer than 2^32
static int check_grid(int64_t a, int64_t b = 1) {
  PD_REQUIRE(a < (1 << 24) && b < (1 << 24) && a * b < (1 << 24), PD_EINVAL, "a launch of %lld x %lld work-groups is too large", (long long)a, (long long)b);
  return PD_OK;
}

// F(types..., head_dim) for the run-time values
#define PD_PAGE_DIMS(HDV, F, ...)                        \
  switch (HDV) {                                         \
    case 32: F(__VA_ARGS__, 32); break;                  \
    case 64: F(__VA_ARGS__, 64); break;                  \
    case 96: F(__VA_ARGS__, 96); break;                  \
    default: F(__VA_ARGS__, 128); break;                 \
  }
#define PD_PAGE_CACHE(CTYPE, HDV, F, ...)                            \
  if ((CTYPE) == PD_TYPE_BF16) PD_PAGE_DIMS(HDV, F, __VA_ARGS__, bf16_t) \
  else PD_PAGE_DIMS(HDV, F, __VA_ARGS__, f16_t)
#define PD_PAGE_TYPES(TYPE, CTYPE, HDV, F)                           \
  switch (TYPE) {                                                    \
    case PD_TYPE_F32: PD_PAGE_CACHE(CTYPE, HDV, F, float) break;     \
    case PD_TYPE_BF16: PD_PAGE_CACHE(CTYPE, HDV, F, bf16_t) break;   \
    default: PD_PAGE_CACHE(CTYPE, HDV, F, f16_t) break;              \
  }

extern "C" int pd_page_append(const pd_page_cache *cache, const int32_t *pages, int n_slot, int n_req, const void *k, const void *v,
                              const void *q, int type, const int64_t *k_strides, const int64_t *v_strides, const int64_t *q_strides,
                              int n_head, int n_new, const int32_t *counts, const int32_t *lens, const double *freqs, int n_freq,
                              const int32_t *places, void *out_q, void *hip_stream) {
  int rc;
  if ((rc = check_pages(cache, pages, n_req, n_slot)) || (rc = check_type(type))) return rc;
  PD_REQUIRE(n_new >= 0, PD_EINVAL, "n_new must be >= 0 (got %d)", n_new);
  if (n_new == 0) return PD_OK;
  PD_REQUIRE(k && v && k_strides && v_strides && lens, PD_EINVAL, "NULL argument");
  PD_REQUIRE((int64_t)n_new <= (int64_t)n_slot * PD_PAGE, PD_EINVAL, "%d new tokens do not fit %d pages", n_new, n_slot);
  PD_REQUIRE(!q == !out_q, PD_EINVAL, "q and out_q go together");
  PD_REQUIRE(!q || (q_strides && n_head >= 1 && n_head <= (1 << 20)), PD_EINVAL, "queries need strides and 1 to 2^20 heads (got %d)", n_head);
  PD_REQUIRE(((uintptr_t)out_q & 15) == 0, PD_EINVAL, "out_q must be 16-byte aligned");
  PD_REQUIRE(n_freq >= 0 && 2 * n_freq <= cache->head_dim, PD_EINVAL, "n_freq must be within 0 and half of head_dim (got %d)", n_freq);
  PD_REQUIRE(n_freq == 0 || (freqs && ((uintptr_t)freqs & 7) == 0), PD_EINVAL, "freqs must be given, and 8-byte aligned");
  const int es = type_bytes(type);
  PD_REQUIRE((((uintptr_t)k | (uintptr_t)v | (uintptr_t)q) & (es - 1)) == 0, PD_EINVAL, "keys, values and queries must be aligned to their type");
  PageStoreArgs a;
  a.c = view(cache); a.src[0] = k; a.src[1] = v; a.src[2] = q; a.counts = counts; a.lens = lens; a.pages = pages; a.places = places;
  a.freqs = freqs; a.out_q = out_q; a.n_freq = n_freq; a.n_new = n_new; a.n_slot = n_slot;
  a.span = (n_new + PD_PAGE - 2) / PD_PAGE + 1;
  uint64_t bits = 0;
  for (int i = 0; i < 3; ++i) {
    const int64_t *st = i == 0 ? k_strides : i == 1 ? v_strides : q_strides;
    a.heads[i] = i < 2 ? cache->n_kv_head : q ? n_head : 0;
    a.groups[i] = (a.heads[i] + STORE_HEADS - 1) / STORE_HEADS;
    a.s_req[i] = a.s_tok[i] = a.s_head[i] = 0;
    if (i == 2 && !q) continue;
    a.s_req[i] = st[0]; a.s_tok[i] = st[1]; a.s_head[i] = st[2];
    bits |= (uintptr_t)a.src[i] | (uint64_t)((st[0] | st[1] | st[2]) * es);
  }
  const bool wide = (bits & 15) == 0;
  const int64_t pieces = (int64_t)n_req * a.span, groups = a.groups[0] + a.groups[1] + a.groups[2], blocks = pieces * groups;
  if ((rc = check_grid(pieces, groups))) return rc;
  hipStream_t s = (hipStream_t)hip_stream;
#define PD_STORE(T, CT, HDV)                                                                                       \
  do {                                                                                                             \
    if (wide) hipLaunchKernelGGL((k_page_store<T, CT, HDV, true>), dim3((unsigned)blocks), dim3(256), 0, s, a);    \
    else hipLaunchKernelGGL((k_page_store<T, CT, HDV, false>), dim3((unsigned)blocks), dim3(256), 0, s, a);        \
  } while (0)
  PD_PAGE_TYPES(type, cache->type, cache->head_dim, PD_STORE)
#undef PD_STORE
  PD_CHECK_HIP(hipGetLastError());
  return PD_OK;
}

extern "C" int pd_page_read(const pd_page_cache *cache, const int32_t *pages, int n_slot, int n_req, const int32_t *first, int n_tok,
                            const int32_t *lens, void *out_k, void *out_v, int type, void *hip_stream) {
  int rc;
  if ((rc = check_pages(cache, pages, n_req, n_slot)) || (rc = check_type(type))) return rc;
  PD_REQUIRE(n_tok >= 0, PD_EINVAL, "n_tok must be >= 0 (got %d)", n_tok);
  if (n_tok == 0) return PD_OK;
  PD_REQUIRE(lens && out_k && out_v, PD_EINVAL, "NULL argument");
  PD_REQUIRE((((uintptr_t)out_k | (uintptr_t)out_v) & 15) == 0, PD_EINVAL, "outputs must be 16-byte aligned");
  PageReadArgs a;
  a.c = view(cache); a.out[0] = out_k; a.out[1] = out_v; a.first = first; a.lens = lens; a.pages = pages; a.n_tok = n_tok; a.n_slot = n_slot;
  a.span = (int)(first ? ((int64_t)n_tok - 1 + PD_PAGE - 1) / PD_PAGE + 1 : ((int64_t)n_tok + PD_PAGE - 1) / PD_PAGE);
  const int64_t pieces = (int64_t)n_req * a.span, groups = 2 * ((cache->n_kv_head + STORE_HEADS - 1) / STORE_HEADS), blocks = pieces * groups;
  if ((rc = check_grid(pieces, groups))) return rc;
  hipStream_t s = (hipStream_t)hip_stream;
#define PD_READ(T, CT, HDV) hipLaunchKernelGGL((k_page_read<T, CT, HDV>), dim3((unsigned)blocks), dim3(256), 0, s, a)
  PD_PAGE_TYPES(type, cache->type, cache->head_dim, PD_READ)
#undef PD_READ
  PD_CHECK_HIP(hipGetLastError());
  return PD_OK;
}

static int check_attention(const pd_page_cache *c, int n_req, int n_group, int n_head, int n_row, int max_shared, int max_behind) {
  PD_REQUIRE(n_head >= 1 && n_head % c->n_kv_head == 0, PD_EINVAL, "n_head = %d is no multiple of %d key heads", n_head, c->n_kv_head);
  PD_REQUIRE(n_group >= 0 && (n_group == 0 || n_req % n_group == 0), PD_EINVAL, "%d requests do not form %d groups of one size", n_req, n_group);
  PD_REQUIRE(n_row >= 0 && max_shared >= 0 && max_behind >= 0, PD_EINVAL, "n_row, max_shared and max_behind must be >= 0 (got %d, %d, %d)",
             n_row, max_shared, max_behind);
  PD_REQUIRE((int64_t)n_row * n_head < (1ll << 31) && (int64_t)n_row * n_head * n_req < (1ll << 31), PD_EINVAL, "too many rows (%d x %d x %d)", n_req,
             n_row, n_head);
  return PD_OK;
}

struct PageLaunch { PageWork part[2]; int64_t n_shared, n_own, n_cols, n_merge; size_t bytes; };

static int page_launch(const pd_page_cache *c, int n_slot, int n_req, int n_group, int n_head, int n_row, int max_shared, int max_behind,
                       PageLaunch *out) {
  int rc = check_attention(c, n_req, n_group, n_head, n_row, max_shared, max_behind);
  if (rc) return rc;
  if (n_row == 0) { *out = PageLaunch{}; return PD_OK; }
  const int cols = n_row * (n_head / c->n_kv_head);
  const PageAttnShape sh = page_attn_shape(c->n_kv_head, n_req, n_group, cols, n_slot, max_shared, max_behind, c->head_dim);
  for (int i = 0; i < 2; ++i) {
    PageWork &w = out->part[i];
    const PageAttnPart &p = sh.part[i];
    w.cols = (int)p.cols; w.width = p.width; w.tiles = (int)((p.cols + p.width - 1) / p.width);
    w.splits = p.splits; w.blocks = p.blocks; w.units = (int)p.units;
    w.first = i ? out->part[0].first + page_columns(sh.part[0]) : 0;
  }
  out->n_shared = page_work_groups(sh.part[0]);
  out->n_own = page_work_groups(sh.part[1]);
  const bool alone = out->n_shared == 0 && sh.part[1].splits == 1;
  out->n_cols = alone ? 0 : page_columns(sh.part[0]) + page_columns(sh.part[1]);
  out->bytes = alone ? 16 : (size_t)out->n_cols * (c->head_dim + 2) * sizeof(float);
  out->n_merge = alone ? 0 : ((int64_t)n_req * n_row * n_head + merge_rows(c->head_dim) - 1) / merge_rows(c->head_dim);
  if ((rc = check_grid(out->n_merge))) return rc;
  return check_grid(out->n_shared + out->n_own);
}

extern "C" size_t pd_page_attention_workspace_bytes(const pd_page_cache *cache, int n_slot, int n_req, int n_group, int n_head, int n_row,
                                                    int max_shared, int max_behind) {
  static const int32_t any = 0;
  PageLaunch l;
  if (check_pages(cache, &any, n_req, n_slot) || page_launch(cache, n_slot, n_req, n_group, n_head, n_row, max_shared, max_behind, &l)) return 0;
  return std::max<size_t>(l.bytes, 16);
}

extern "C" int pd_page_attention(const pd_page_cache *cache, const int32_t *pages, int n_slot, int n_req, const void *q,
                                 const int64_t *q_strides, int n_head, int n_row, const int32_t *lens, const int32_t *shared, int n_group,
                                 const int32_t *row_limit, const uint16_t *key_tag, const int32_t *row_tag, float scale, int max_shared,
                                 int max_behind, void *out, float *out_lse, void *workspace, size_t workspace_bytes, void *hip_stream) {
  int rc;
  PageLaunch l;
  if ((rc = check_pages(cache, pages, n_req, n_slot)) ||
      (rc = page_launch(cache, n_slot, n_req, n_group, n_head, n_row, max_shared, max_behind, &l)))
    return rc;
  if (n_row == 0) return PD_OK;
  PD_REQUIRE(q && q_strides && lens && out, PD_EINVAL, "NULL argument");
  PD_REQUIRE(!shared == !n_group, PD_EINVAL, "shared and n_group go together");
  PD_REQUIRE(!key_tag == !row_tag, PD_EINVAL, "key_tag and row_tag go together");
  PD_REQUIRE((((uintptr_t)key_tag | (uintptr_t)out) & 15) == 0, PD_EINVAL, "key_tag and out must be 16-byte aligned");
  PD_REQUIRE(((uintptr_t)q & 1) == 0, PD_EINVAL, "q must be aligned to its type");
  PD_REQUIRE(scale == scale && std::abs(scale) <= 2.0e38f, PD_EINVAL, "scale must be a number of magnitude up to 2e38");
  PD_REQUIRE(l.n_cols == 0 || (workspace && workspace_bytes >= l.bytes), PD_ENOMEM, "workspace too small: %zu bytes given, %zu needed",
             workspace ? workspace_bytes : (size_t)0, l.bytes);
  PD_REQUIRE(l.n_cols == 0 || ((uintptr_t)workspace & 15) == 0, PD_EINVAL, "workspace must be 16-byte aligned");
  PageAttnArgs a;
  a.c = view(cache); a.q = q; a.q_req = q_strides[0]; a.q_row = q_strides[1]; a.q_head = q_strides[2];
  a.pages = pages; a.lens = lens; a.shared = shared; a.row_limit = row_limit; a.key_tag = key_tag; a.row_tag = row_tag;
  a.out = out; a.lse = out_lse; a.n_req = n_req; a.n_row = n_row; a.n_head = n_head; a.group = n_head / cache->n_kv_head;
  a.n_slot = n_slot; a.per_group = n_group ? n_req / n_group : 1;
  a.scale_log2 = (float)(scale * 1.4426950408889634);
  a.q_wide = (((uintptr_t)q | (uint64_t)((q_strides[0] | q_strides[1] | q_strides[2]) * 2)) & 15) == 0;
  a.part[0] = l.part[0]; a.part[1] = l.part[1]; a.n_shared = l.n_shared; a.n_cols = l.n_cols; a.sums = (float *)workspace;
  hipStream_t s = (hipStream_t)hip_stream;
  const unsigned grid = (unsigned)(l.n_shared + l.n_own), merge = (unsigned)l.n_merge;
#define PD_ATTEND(CT, HDV)                                                                             \
  do {                                                                                                 \
    hipLaunchKernelGGL((k_page_attn<CT, HDV>), dim3(grid), dim3(256), 0, s, a);                        \
    if (merge) hipLaunchKernelGGL((k_page_merge<CT, HDV>), dim3(merge), dim3(256), 0, s, a);          \
  } while (0)
  if (cache->type == PD_TYPE_BF16) PD_PAGE_DIMS(cache->head_dim, PD_ATTEND, bf16_t)
  else PD_PAGE_DIMS(cache->head_dim, PD_ATTEND, f16_t)
#undef PD_ATTEND
  PD_CHECK_HIP(hipGetLastError());
  return PD_OK;
}
