// One token per row of logits for a given random number: temperature, top-k, top-p, min-p, then the inverse of the distribution.
//
// With e_i = exp((x_i - max x) / temperature) and the tokens in falling order of x, ties by rising index, every rule keeps a start of
// that order: the first k; those in front of which less than p of the sum of what k keeps has gone by; those with e_i >= min_p.  So a
// row is cut at one place of the order, (value, index), and what is kept is drawn from in the order of the indices: nothing is sorted but
// the few tokens around a cut.  A cut is found by histograms of numbers and sums of e over 2048 pieces of the range, in whole numbers of
// 64 bits of a unit for each piece, which come out the same in whatever order they are added.
// Which token a number falls on depends on sums next to borders: e and all sums have 64 bits (a multiply-add of 64 bits takes this
// chip 8 clocks a wave, twice one of 32).
//
// Bound by what one compute unit issues: a row is one work-group's.  Of the 26 us of a row of 32000 by top-p, loading and its largest
// value take 3, e with its additions in LDS 8 (18 instructions of 64 bits, and 34 clocks for 64 additions to random places), what lies around
// the cut 4, e once more and the running sums 8.  By rank nothing needs e but the few that stay: 13.9 us.  512 rows of 32128 by top-p (two
// rounds of the 256 compute units) 60 us, 64 rows of 50265 47.  fp32 rows of 50265, which are read again in every pass, 48 us, of 128000 105.
#include "pd_internal.h"

#include <type_traits>

constexpr int BINS = 2048, NEAR = 1024;                  // pieces of a range; tokens around a cut that are put in order at once

// bits whose order as whole numbers is that of the values (no NaN, no -0)
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return (int)b < 0 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }

// 2^(y + up) by n = the nearest whole number and the series of 2^f for f = y - n, |f| <= 1/2: the first term left out is below
// (ln 2 / 2)^11 / 11! = 2.2e-13.  y <= 0 or NaN; from -1023 on down, and for NaN, it is at most 2^(up - 1022), zero for up = 0 (so a
// product that is fused into the difference stays near n).  The nearest whole number is what adding 1.5 * 2^52 leaves in the last bits, and
// 2^n is its exponent's bits; up_bits: (up + 1023) * 2^20.
__device__ __forceinline__ double exp2_64(double y, uint32_t up_bits = 1023u << 20) {
  constexpr double WHOLE = 6755399441055744.0;
  y = fmax(y, -1023.0);
  const double t = y + WHOLE, f = y - (t - WHOLE);
  constexpr double L = 0.69314718055994530942, L2 = L * L / 2, L3 = L2 * L / 3, L4 = L3 * L / 4, L5 = L4 * L / 5, L6 = L5 * L / 6,
                   L7 = L6 * L / 7, L8 = L7 * L / 8, L9 = L8 * L / 9, L10 = L9 * L / 10;
  double p = L10;
  p = fma(p, f, L9); p = fma(p, f, L8); p = fma(p, f, L7); p = fma(p, f, L6); p = fma(p, f, L5);
  p = fma(p, f, L4); p = fma(p, f, L3); p = fma(p, f, L2); p = fma(p, f, L); p = fma(p, f, 1.0);
  const uint32_t n = ((uint32_t)__double_as_longlong(t) << 20) + up_bits;
  return p * __longlong_as_double((long long)((uint64_t)n << 32));
}

// A row's values in granules of 16 bytes.  KB: kilobytes of LDS in which they are kept, KB / 16 granules of every thread, next to each
// other in the row, so that sums in the order of the indices are sums in the order of the threads; 0: every pass reads the row again,
// granule j * 1024 + thread.  What is no value of the row, NaN, and -infinity are -infinity; there is no -0.
// (In registers they invite the compiler to keep what it computes of them from pass to pass: 800 bytes of scratch memory a thread.)
template <typename T, int KB>
struct Row {
  static constexpr int G = 16 / sizeof(T), C = KB / 16, STEP = 1025;       // (granules of a thread in LDS: 16 bytes beside whole banks)
  union Granule { uint4 u; T h[G]; };
  const T *p;
  uint4 *kept;
  int V, skip, chunks;                // skip: values in front of the row in its first granule
  bool endless;                       // there is +infinity: it alone counts, as 0

  __device__ __forceinline__ float clean(float x) const {
    x = fmaxf(x, -INFINITY) + 0.f;
    return endless ? (x == INFINITY ? 0.f : -INFINITY) : x;
  }
  __device__ __forceinline__ Granule granule(int q) const {
    const int i0 = q * G - skip;
    Granule w;
    if (i0 >= 0 && i0 + G <= V) {
      w.u = *(const uint4 *)(p + i0);
    } else {
#pragma unroll
      for (int e = 0; e < G; ++e) w.h[e] = i0 + e >= 0 && i0 + e < V ? p[i0 + e] : below();
    }
    return w;
  }
  __device__ __forceinline__ static T below() {
    if constexpr (sizeof(T) == 4) return -INFINITY;
    else if constexpr (std::is_same<T, bf16_t>::value) return 0xff80;
    else return (T)-INFINITY;
  }
  // (a barrier has to follow)
  __device__ __forceinline__ void start(const T *row, int vocab, uint4 *lds, float &top, float &low) {
    p = row; V = vocab; kept = lds; endless = false;
    skip = (int)(((uintptr_t)row & 15) / sizeof(T));
    chunks = KB ? C : (V + skip + 1024 * G - 1) / (1024 * G);
    auto take = [&](int j) {
      const int q = j * 1024 + threadIdx.x;
      Granule w = granule(q);
#pragma unroll
      for (int e = 0; e < G; ++e) {
        const float x = clean(ld_f32(w.h, e));
        top = fmaxf(top, x);
        low = x > -INFINITY ? fminf(low, x) : low;
        w.h[e] = as_kept(x);
      }
      if constexpr (KB > 0) kept[q % C * STEP + q / C] = w.u;
    };
    if constexpr (KB > 0) {
#pragma unroll
      for (int j = 0; j < C; ++j) take(j);
    } else {
      for (int j = 0; j < chunks; ++j) take(j);
    }
  }
  // (exact: it was one of the type's numbers)
  __device__ __forceinline__ static T as_kept(float x) {
    if constexpr (std::is_same<T, bf16_t>::value) return f32_to_bf16(x);
    else return (T)x;
  }
  __device__ __forceinline__ void only_endless() {
    endless = true;
    if constexpr (KB > 0)
      for (int j = 0; j < C; ++j) {
        Granule w;
        w.u = kept[j * STEP + threadIdx.x];
        for (int e = 0; e < G; ++e) w.h[e] = as_kept(clean(ld_f32(w.h, e)));
        kept[j * STEP + threadIdx.x] = w.u;
      }
  }
  // f(index of the first, values) of a granule of the thread's, and of all of them
  template <typename F> __device__ __forceinline__ void chunk(int j, F f) const {
    Granule w;
    if constexpr (KB > 0) w.u = kept[j * STEP + threadIdx.x];
    else w = granule(j * 1024 + threadIdx.x);
    float y[G];
#pragma unroll
    for (int e = 0; e < G; ++e) y[e] = KB ? ld_f32(w.h, e) : clean(ld_f32(w.h, e));
    f((KB ? (int)threadIdx.x * C + j : j * 1024 + (int)threadIdx.x) * G - skip, y);
  }
  template <typename F> __device__ __forceinline__ void chunk_by_chunk(F f) const {
    if constexpr (KB > 0) {
#pragma unroll 1
      for (int j = 0; j < C; ++j) chunk(j, f);
    } else {
      for (int j = 0; j < chunks; ++j) chunk(j, f);
    }
  }
  template <typename F> __device__ __forceinline__ void each(F f) const {
    chunk_by_chunk([&](int i, const float *y) {
#pragma unroll
      for (int e = 0; e < G; ++e) f(y[e], i + e);
    });
  }
  // what stands at index i counts no more (in LDS)
  __device__ __forceinline__ void erase(int i) {
    const int q = (i + skip) / G;
    ((T *)&kept[q % C * STEP + q / C])[(i + skip) % G] = below();
  }
  // place and value of value k of thread t, in LDS
  __device__ __forceinline__ int index(int t, int k) const { return t * C * G + k - skip; }
  __device__ __forceinline__ float at(int t, int k) const {
    return ld_f32((const T *)&kept[k / G * STEP + t], k % G);
  }
};

// exchanges of 64 bits between the lanes of a wave
template <typename V> __device__ __forceinline__ V from_lane(V v, int lane) {       // (the same lane for the whole wave)
  union { V v; int w[sizeof(V) / 4]; } u;
  u.v = v;
#pragma unroll
  for (int i = 0; i < (int)sizeof(V) / 4; ++i) u.w[i] = __builtin_amdgcn_readlane(u.w[i], lane);
  return u.v;
}
// the sum over the lanes up to this one: within rows of 16 by shifts, then the last lanes of rows are handed on
template <int CTRL, int ROWS, typename V> __device__ __forceinline__ V add_moved(V v) {
  if constexpr (sizeof(V) == 4) {
    return v + __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, true));
  } else {
    union { V v; int w[2]; } u, o;
    u.v = v;
    o.w[0] = __builtin_amdgcn_update_dpp(0, u.w[0], CTRL, ROWS, 0xf, true);
    o.w[1] = __builtin_amdgcn_update_dpp(0, u.w[1], CTRL, ROWS, 0xf, true);
    return v + o.v;
  }
}
template <typename V> __device__ __forceinline__ V wave_running(V v) {
  v = add_moved<0x111, 0xf>(v); v = add_moved<0x112, 0xf>(v); v = add_moved<0x114, 0xf>(v); v = add_moved<0x118, 0xf>(v);
  v = add_moved<0x142, 0xa>(v);
  return add_moved<0x143, 0xc>(v);
}

template <typename V> __device__ __forceinline__ V wave_total(V v) { return from_lane(wave_running(v), 63); }

template <int KB>
struct SampleShared {
  union {
    struct { unsigned long long mass[BINS]; uint32_t count[BINS]; };
    struct { unsigned long long near_[NEAR], sorted[NEAR]; double weight[NEAR]; };      // (when the histogram has been read)
  };
  uint32_t place[NEAR];
  double part[KB ? 1 : 16 * ((PD_SAMPLE_VOCAB + 3) / 4096 + 1)];                        // sums by chunk and wave
  unsigned long long wave_mass[16];
  double wave_sum[16];
  uint32_t wave_count[16];
  float top[16], low[16];
  double total, goal, before_d;
  int found, before, n_near, bin;
  uint32_t key_low, key_high;
};

// One work-group per row.
template <typename T, int KB>
__global__ __launch_bounds__(1024) void k_sample(SampleArgs a) {
  __shared__ SampleShared<KB> sm;
  __shared__ uint4 sm_row[KB ? KB / 16 * Row<T, KB>::STEP : 1];
  const int r = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, V = a.vocab;
  if (a.active && a.active[r] < 0) {
    if (tid == 0) { a.token[r] = -1; if (a.logprob) a.logprob[r] = 0.f; }
    return;
  }
  Row<T, KB> row;
  float top = -INFINITY, low = INFINITY;
  row.start((const T *)a.x + r * a.stride, V, sm_row, top, low);
  const float t = a.p.row_temperature ? a.p.row_temperature[r] : a.p.temperature;
  const float P = a.p.row_top_p ? a.p.row_top_p[r] : a.p.top_p, M = a.p.row_min_p ? a.p.row_min_p[r] : a.p.min_p;
  const int K = a.p.row_top_k ? a.p.row_top_k[r] : a.p.top_k;
  const float u = fminf(fmaxf(a.u[r], 0.f), 0x1.fffffep-1f);       // (within [0, 1); NaN is 0)

  // ---- the largest and the smallest value ----
  top = fold_wave(top, Max());
  low = -fold_wave(-low, Max());
  if (lane == 0) { sm.top[wave] = top; sm.low[wave] = low; }
  __syncthreads();
  top = fold_row(sm.top[lane & 15], Max());
  low = -fold_row(-sm.low[lane & 15], Max());
  if (top == INFINITY) { row.only_endless(); top = 0.f; low = 0.f; }
  const bool greedy = !(t > 0.f) || !(P > 0.f) || !(M <= 1.f) || K == 1;
  const double c = 1.4426950408889634074 / (double)t, mx = top;
  auto e_of = [&](float x) { return exp2_64(((double)x - mx) * c); };       // (0 for -infinity)

  // kept: above the cut, or equal to it and index up to last (in LDS: those behind are erased)
  float cut = -INFINITY;
  int last = 0x7fffffff;
  auto kept = [&](float x, int i) { return KB ? x >= cut : (x > cut) | ((x == cut) & (i <= last)); };

  constexpr int G = Row<T, KB>::G;
  // the sum over the threads up to this one, and over all
  auto running = [&](double v, double *all) {
    double upto = wave_running(v), sum = 0;
    if (lane == 63) sm.wave_sum[wave] = upto;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (k == wave) upto += sum;
      sum += sm.wave_sum[k];
    }
    *all = sum;
    __syncthreads();
    return upto;
  };
  // the lowest of the threads that say so, 1024 without any
  auto first_thread = [&](bool says) {
    const uint64_t some = __ballot(says);
    if (lane == 0) sm.wave_count[wave] = some ? wave * 64 + __ffsll((unsigned long long)some) - 1 : 1024;
    __syncthreads();
    uint32_t first = 1024;
#pragma unroll
    for (int k = 0; k < 16; ++k) first = min(first, sm.wave_count[k]);
    __syncthreads();
    return (int)first;
  };
  // The first index at which the running sum of w(value, index), which is 0 where it is not kept, passes goal(total), in the order of
  // the indices, with its weight; the last one that has a weight where rounding leaves none.
  struct Found { int index; double weight, total; };
  auto locate = [&](auto w, auto goal) {
    auto sum = [&](int i, const float *y) {
      double s = 0;
      bool any = false;
#pragma unroll
      for (int e = 0; e < G; ++e) any |= y[e] >= cut;
      if (__any(any))
#pragma unroll
        for (int e = 0; e < G; ++e) s += w(y[e], i + e);
      return s;
    };
    if constexpr (KB > 0) {
      double s = 0, total;
      row.chunk_by_chunk([&](int i, const float *y) { s += sum(i, y); });
      const double upto = running(s, &total), target = goal(total);
      int t = first_thread(s > 0 && upto > target);
      if (t == 1024) {
        const uint64_t some = __ballot(s > 0);
        if (lane == 0) sm.wave_count[wave] = some ? wave * 64 + 64 - __clzll(some) : 0;
        __syncthreads();
        uint32_t last_one = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) last_one = max(last_one, sm.wave_count[k]);
        t = max((int)last_one - 1, 0);
        __syncthreads();
      }
      if (tid == t) sm.before_d = upto - s;
      __syncthreads();
      if (wave == 0) {                                   // that thread's values, one to a lane
        const bool there = lane < Row<T, KB>::C * G;
        const float x = there ? row.at(t, lane) : -INFINITY;
        const int i = row.index(t, lane);
        const double own = there ? w(x, i) : 0.0, run = sm.before_d + wave_running(own);
        const uint64_t hit = __ballot(own > 0 && run > target), some = __ballot(own > 0);
        if (lane == (hit ? __ffsll((unsigned long long)hit) - 1 : some ? 63 - __clzll(some) : 0)) { sm.found = i; sm.goal = own; }
      }
      __syncthreads();
      return Found{sm.found, sm.goal, total};
    } else {
      row.chunk_by_chunk([&](int i, const float *y) {
        double s = sum(i, y);
        if (__any(s != 0)) s = wave_total(s);
        if (lane == 0) sm.part[(i + row.skip) / (1024 * G) * 16 + wave] = s;
      });
      __syncthreads();
      const int parts = row.chunks * 16;
      if (wave == 0) {
        double run = 0;
        for (int k = 0; k < parts; k += 64) run += wave_total(k + lane < parts ? sm.part[k + lane] : 0.0);
        const double total = run, target = goal(total);
        double before = 0, at_before = 0;
        int at = 0;
        for (int k = 0; k < parts; k += 64) {
          const double own = k + lane < parts ? sm.part[k + lane] : 0.0, upto = before + wave_running(own);
          const uint64_t hit = __ballot(own > 0 && upto > target), some = __ballot(own > 0);
          const int l = hit ? __ffsll((unsigned long long)hit) - 1 : some ? 63 - __clzll(some) : -1;
          if (l >= 0) { at = k + l; at_before = from_lane(upto - own, l); }
          if (hit) break;
          before = from_lane(upto, 63);
        }
        if (lane == 0) { sm.bin = at; sm.before_d = at_before; sm.goal = target; sm.total = total; }
      }
      __syncthreads();
      const int at = sm.bin;
      const double before = sm.before_d, target = sm.goal, total = sm.total;
      __syncthreads();
      if (wave == (at & 15)) {
        row.chunk(at >> 4, [&](int i, const float *y) {
          double own[G], s = 0;
#pragma unroll
          for (int e = 0; e < G; ++e) { own[e] = w(y[e], i + e); s += own[e]; }
          const double upto = before + wave_running(s);
          const uint64_t hit = __ballot(s > 0 && upto > target), some = __ballot(s > 0);
          if (lane == (hit ? __ffsll((unsigned long long)hit) - 1 : some ? 63 - __clzll(some) : 0)) {
            double run = upto - s;
            int found = i;
            double there = 0;
#pragma unroll
            for (int e = 0; e < G; ++e) {
              if (own[e] > 0 && (there == 0 || run <= target)) { found = i + e; there = own[e]; }
              run += own[e];
            }
            sm.found = found;
            sm.goal = there;
          }
        });
      }
      __syncthreads();
      return Found{sm.found, sm.goal, total};
    }
  };

  if (top == -INFINITY || greedy) {
    int first = 0x7fffffff;
    row.each([&](float x, int i) { first = x == top ? min(first, i) : first; });
    first = fold_wave(first, Min());
    if (lane == 0) sm.wave_count[wave] = first;
    __syncthreads();
    if (tid == 0) {
      for (int k = 1; k < 16; ++k) first = min(first, (int)sm.wave_count[k]);
      a.token[r] = top == -INFINITY ? -1 : first;
      if (a.logprob) a.logprob[r] = 0.f;
    }
    return;
  }

  // sm.near_[0 .. n) in falling order to sm.sorted.  Few: every entry counts those in front of it, with as many threads as there are for
  // it.  More: into 1024 places, of which a larger entry never has a later one, and every entry counts those in front of it in its place.
  // 64 rows of 8192, us, few / more: 70 tokens 13.9 / 15.5, 128 15.6 / 16.1, 180 17.2 / 16.5, 1000 73.5 / 18.7.
  auto put_in_order = [&](int n, auto place_of) {
    if (n <= 128) {
      const int lg = n <= 1 ? 0 : 32 - __clz(n - 1), i = tid & ((1 << lg) - 1), parts = 1024 >> lg;
      if (tid < n) sm.place[tid] = 0;
      __syncthreads();
      unsigned long long me = 0;
      if (i < n) {
        me = sm.near_[i];
        uint32_t ahead = 0;
#pragma unroll 4
        for (int k = tid >> lg; k < n; k += parts) ahead += sm.near_[k] > me;
        atomicAdd(&sm.place[i], ahead);
      }
      __syncthreads();
      if (tid < n) sm.sorted[sm.place[tid]] = me;
      __syncthreads();
      return;
    }
    const unsigned long long me = tid < n ? sm.near_[tid] : 0;
    const int b = tid < n ? place_of(me) : 0;
    sm.place[tid] = 0;
    __syncthreads();
    const uint32_t slot = tid < n ? atomicAdd(&sm.place[b], 1u) : 0;
    __syncthreads();
    const uint32_t own = sm.place[tid];
    uint32_t upto = wave_running(own), before = 0;
    if (lane == 63) sm.wave_count[wave] = upto;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) before += k < wave ? sm.wave_count[k] : 0;
    upto += before;
    sm.place[tid] = upto;
    __syncthreads();
    const uint32_t from = tid < n && b ? sm.place[b - 1] : 0, to = tid < n ? sm.place[b] : 0;
    if (tid < n) sm.sorted[from + slot] = me;
    __syncthreads();
    uint32_t at = from;
#pragma unroll 4
    for (uint32_t k = from; k < to; ++k) at += sm.sorted[k] > me;
    __syncthreads();
    if (tid < n) sm.sorted[at] = me;
    __syncthreads();
  };
  const float range = fminf(48.6f * t, top - low), per = range > 0.f && range < INFINITY ? BINS / range : 0.f;
  auto bin_of = [&](float x) { return min((int)((top - x) * per), BINS - 1); };
  // e in whole numbers of which one token has at most 2^51 (and what roundings of its piece leave above), and all together less than 2^63: times
  // 2^(bits + k), where the tokens of a piece are below 2^-k.  So a token is off by 2^-(bits + 1) of about itself, 2^-42 for the largest
  // vocabulary, however many there are and all of them to the same side.  (Of one unit for all pieces, 2^-bits: 700 tokens off, with 2^20 alike at
  // 2.8e-10 of the first.)
  const int bits = min(51, 62 - (32 - __clz(V)));
  const uint32_t fall = per > 0.f && per < INFINITY ? (uint32_t)(range * (float)c * (1048576.f / BINS)) : 0;     // (35900 at most)
  const uint32_t scale0 = (uint32_t)(bits + 1023) << 20;
  auto scale_of = [&](int b) { return (scale0 + __umul24(b, fall)) & 0xfff00000u; };                         // bits + k, as an exponent's bits
  auto pow2 = [](int n) { return __longlong_as_double((long long)(1023 + n) << 52); };
  // (added to 2^52, a number below it leaves itself, rounded, in the last bits)
  auto whole = [](double x) { return (unsigned long long)(__double_as_longlong(x + 4503599627370496.0) & 0xfffffffffffffll); };
  auto unit_of = [&](int b) { return pow2(1023 - (int)(scale_of(b) >> 20)); };

  // Moves the cut: by number (the first `most` of the tokens, MASS false) or by sum (those in front of which less than P of the sum of
  // the kept ones has gone by).  True: the tokens that are left, and perhaps some behind them, are sm.near_[0 .. *n_sorted), in no order, within the pieces in front of *deep.
  auto move_cut = [&](auto mass_, int most, int *n_sorted, float *deep) {
    constexpr bool MASS = decltype(mass_)::value;
    uint32_t from = 1, to = 0;                           // keys of the piece in question; none yet
    int bin = -1, shift = 0;
    uint32_t n_before = 0;
    double m_before = 0, target = 0;
    for (int level = 0;; ++level) {
      if (MASS) { sm.mass[tid] = 0; sm.mass[tid + 1024] = 0; }
      else { sm.count[tid] = 0; sm.count[tid + 1024] = 0; }
      if (tid == 0) { sm.n_near = 0; sm.key_low = 0xffffffffu; sm.key_high = 0; sm.bin = -1; }
      __syncthreads();
      // (what is far below the largest lies in the last piece, most of the row where the temperature is low, and 64 lanes that add to one
      // place take turns: there every thread counts by itself, and e that count as zero go to a place of each lane's)
      uint32_t n_last = 0;
      const float far = top - 48.6f * t;                   // (2^-70 and less of the largest)
      auto add = [&](float x, int b, bool counts) {
        if (MASS) {
          const float z = counts ? x : -INFINITY;
          const int at = level || z >= far ? b : lane;     // (of the first places' units what is far below the largest is zero)
          atomicAdd(&sm.mass[at], whole(exp2_64(((double)z - mx) * c, scale_of(level ? bin : at))));
        } else if (counts) {
          if (b == BINS - 1) ++n_last;
          else atomicAdd(&sm.count[b], 1u);
        }
      };
      if (level == 0) {
        if (!MASS || cut == -INFINITY) {                   // (-infinity has no e)
          row.each([&](float x, int) { add(x, bin_of(x), MASS | (x > -INFINITY)); });
        } else {
          row.chunk_by_chunk([&](int i, const float *y) {
            bool any = false;
#pragma unroll
            for (int e = 0; e < G; ++e) any |= y[e] >= cut;
            if (!__any(any)) return;
#pragma unroll
            for (int e = 0; e < G; ++e) add(y[e], bin_of(y[e]), kept(y[e], i + e));
          });
        }
      } else {
        row.each([&](float x, int i) {
          const uint32_t key = order_of(x);
          if (key >= from && key <= to && (!MASS || kept(x, i))) add(x, (to - key) >> shift, true);
        });
      }
      if (!MASS) {
        n_last = wave_total(n_last);
        if (lane == 0 && n_last) atomicAdd(&sm.count[BINS - 1], n_last);
      }
      __syncthreads();
      // running numbers over the pieces, two to a thread; the piece in which the cut lies: less than the goal in front of it, not less with it
      if constexpr (!MASS) {
        const uint32_t c0 = sm.count[2 * tid], c1 = sm.count[2 * tid + 1];
        uint32_t upto = wave_running(c0 + c1), all = 0;
        if (lane == 63) sm.wave_count[wave] = upto;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          if (k == wave) upto += all;
          all += sm.wave_count[k];
        }
        if (level == 0 && all <= (uint32_t)most) return false;       // all of them stay
        const uint32_t goal = (uint32_t)most - n_before, b1 = upto - c1, b0 = b1 - c0;
        if (b0 < goal && b1 >= goal) { sm.bin = 2 * tid; sm.before = b0; sm.found = c0; }
        if (b1 < goal && upto >= goal) { sm.bin = 2 * tid + 1; sm.before = b1; sm.found = c1; }
      } else {
        unsigned long long m0 = sm.mass[2 * tid], m1 = sm.mass[2 * tid + 1], all = 0;
        double per_unit = unit_of(max(bin, 0));
        if (level == 0) {                                  // in one unit, by what they come to: about 2^-50 of that
          const double d0 = (double)m0 * unit_of(2 * tid), d1 = (double)m1 * unit_of(2 * tid + 1);
          const float mine = fold_wave((float)(d0 + d1), Add());
          if (lane == 0) sm.top[wave] = mine;
          __syncthreads();
          const uint32_t sum = __builtin_amdgcn_readfirstlane(__float_as_uint(fold_row(sm.top[lane & 15], Add())));
          const int up = 50 + 127 - (int)(sum >> 23);     // (in which the sum is below 2^52)
          m0 = whole(d0 * pow2(up)); m1 = whole(d1 * pow2(up));
          per_unit = pow2(-up);
        }
        unsigned long long upto = wave_running(m0 + m1);
        if (lane == 63) sm.wave_mass[wave] = upto;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          if (k == wave) upto += all;
          all += sm.wave_mass[k];
        }
        if (level == 0) target = (double)P * ((double)all * per_unit);
        const double s0 = m_before + (double)(upto - m1 - m0) * per_unit, s1 = m_before + (double)(upto - m1) * per_unit,
                     s2 = m_before + (double)upto * per_unit;
        // (the last piece with anything in it, where roundings leave the sums of a piece's pieces a little short of its own)
        if (m0 && s0 < target && (s1 >= target || (m1 == 0 && upto == all))) { sm.bin = 2 * tid; sm.before_d = s0; }
        if (m1 && s1 < target && (s2 >= target || upto == all)) { sm.bin = 2 * tid + 1; sm.before_d = s1; }
      }
      __syncthreads();
      const int b = sm.bin;
      if (b < 0) return false;                           // (not reached: the largest has 1)
      if (MASS) m_before = sm.before_d;
      else n_before += sm.before;
      if (level == 0) bin = b;
      else { const uint32_t high = to - ((uint32_t)b << shift); from = max(from, high - ((1u << shift) - 1)); to = high; }
      // few in all: they are put in order, and there is nothing more to look for in the row
      const bool few = !MASS && level == 0 && n_before + sm.found <= NEAR;
      __syncthreads();
      // the tokens of that piece
      // (values that can be in it, by bounds of the piece with room for the roundings of bin_of; further levels: all)
      const float wide = per > 0.f ? (top - (float)(bin + 1) / per) - fabsf(top) * 4.8e-7f - range * 4.8e-7f : -INFINITY,
                  high = per > 0.f && !few ? (top - (float)bin / per) + fabsf(top) * 4.8e-7f + range * 4.8e-7f : INFINITY,
                  least_x = bin == BINS - 1 ? -INFINITY : wide;
      auto in_piece = [&](float x, int i) {
        const uint32_t key = order_of(x);
        const int b = bin_of(x);
        return x > -INFINITY && (level == 0 ? (few ? b <= bin : b == bin) : key >= from && key <= to) && (!MASS || kept(x, i));
      };
      auto take = [&](float x, int i) {
        if (!in_piece(x, i)) return;
        const uint32_t key = order_of(x);
        const int at = atomicAdd(&sm.n_near, 1);
        if (at < NEAR) sm.near_[at] = (unsigned long long)key << 32 | (uint32_t)~i;
      };
      row.chunk_by_chunk([&](int i, const float *y) {
        bool any = false;
#pragma unroll
        for (int e = 0; e < G; ++e) any |= (y[e] >= least_x) & (y[e] <= high);
        if (!__any(any)) return;
#pragma unroll
        for (int e = 0; e < G; ++e)
          if ((y[e] >= least_x) & (y[e] <= high)) take(y[e], i + e);
      });
      __syncthreads();
      const int n = sm.n_near;
      if (n > NEAR) {                                    // the keys that it has
        uint32_t kl = 0xffffffffu, kh = 0;
        row.each([&](float x, int i) {
          const uint32_t key = order_of(x);
          if (in_piece(x, i)) { kl = min(kl, key); kh = max(kh, key); }
        });
        if (kl <= kh) { atomicMin(&sm.key_low, kl); atomicMax(&sm.key_high, kh); }
        __syncthreads();
        from = sm.key_low; to = sm.key_high;
        if (from == to) {                                // ties: by index
          const double e = e_of(value_of(from));
          const int stay = MASS ? (int)fmin(fmax(ceil((target - m_before) / e), 1.0), (double)n) : most - (int)n_before;
          const float tie = value_of(from);
          const Found l = locate([&](float x, int i) { return (x == tie) & kept(x, i) ? 1.0 : 0.0; }, [&](double) { return stay - 0.5; });
          cut = tie; last = l.index;
          if constexpr (KB > 0) {
            row.each([&](float x, int i) { if ((x == tie) & (i > last)) row.erase(i); });
            __syncthreads();
          }
          return false;
        }
        shift = max(32 - __clz(to - from) - 11, 0);
        __syncthreads();
        continue;
      }
      if (few) { *n_sorted = n; *deep = (float)(bin + 1); return true; }
      // (level 0: parts of the piece's range; further ones: of its keys)
      put_in_order(n, [&](unsigned long long x) {
        const uint32_t key = (uint32_t)(x >> 32);
        const float part = level == 0 ? ((top - value_of(key)) * per - (float)bin) * 1024.f : (float)(to - key) * (1024.f / ((float)(to - from) + 1.f));
        return (int)fminf(fmaxf(part, 0.f), 1023.f);
      });
      int stay = most - (int)n_before;
      if (MASS) {
        double all;
        const double own = tid < n ? e_of(value_of((uint32_t)(sm.sorted[tid] >> 32))) : 0.0, upto = running(own, &all);
        const int number = __popcll(__ballot(tid < n && m_before + (upto - own) < target));
        if (lane == 0) sm.wave_count[wave] = number;
        __syncthreads();
        stay = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) stay += sm.wave_count[k];
        stay = max(stay, 1);
      }
      const unsigned long long at = sm.sorted[stay - 1];
      cut = value_of((uint32_t)(at >> 32));
      last = (int)~(uint32_t)at;
      if constexpr (KB > 0) {
        if (tid >= stay && tid < n && (uint32_t)(sm.sorted[tid] >> 32) == (uint32_t)(at >> 32)) row.erase((int)~(uint32_t)sm.sorted[tid]);
      }
      __syncthreads();
      return false;
    }
  };
  int n_sorted = 0;
  float deep = 1.f;
  if (K > 0 && move_cut(std::false_type(), K, &n_sorted, &deep)) {
    if (n_sorted <= 64) {                                // one wave does the rest by itself
      if (wave != 0) return;
      // entries to their places in falling order
      auto ordered = [&](unsigned long long me, int n) {
        uint32_t ahead = 0;
#pragma unroll 8
        for (int k = 0; k < n; ++k) ahead += sm.near_[k] > me;
        if (lane < n) sm.sorted[ahead] = me;
        wave_sync();
        return lane < n ? sm.sorted[lane] : 0;
      };
      const unsigned long long me = ordered(lane < n_sorted ? sm.near_[lane] : 0, n_sorted);
      double e = lane < K && lane < n_sorted ? e_of(value_of((uint32_t)(me >> 32))) : 0.0;
      const double upto = wave_running(e), all = from_lane(upto, 63);
      const bool stays = lane == 0 || (e > 0 && e >= (double)M && (P >= 1.f || upto - e < (double)P * all));
      const int n = __popcll(__ballot(stays));           // (the first ones)
      const unsigned long long by_index = (unsigned long long)~(uint32_t)me << 32 | (uint32_t)lane;
      sm.weight[lane] = e;
      sm.near_[lane] = by_index;
      wave_sync();
      ordered(by_index, n);
      const unsigned long long by = lane < n ? sm.sorted[n - 1 - lane] : 0;
      e = lane < n ? sm.weight[(uint32_t)by] : 0.0;
      const double passed = wave_running(e), total = from_lane(passed, 63), target = (double)u * total;
      const uint64_t hit = __ballot(lane < n && (passed > target || lane == n - 1));
      if (lane == __ffsll((unsigned long long)hit) - 1) {
        a.token[r] = (int)(by >> 32);
        if (a.logprob) a.logprob[r] = (float)log(e / total);
      }
      return;
    }
    const float parts = 1024.f / deep;
    put_in_order(n_sorted, [&](unsigned long long x) { return (int)fminf((top - value_of((uint32_t)(x >> 32))) * per * parts, 1023.f); });
    // the tokens in order: the other rules by running sums, then the ones that stay in the order of their indices
    const unsigned long long me = tid < K ? sm.sorted[tid] : 0;
    double e = tid < K ? e_of(value_of((uint32_t)(me >> 32))) : 0.0, all;
    const double upto = running(e, &all);
    const bool stays = tid == 0 || (e > 0 && e >= (double)M && (P >= 1.f || upto - e < (double)P * all));
    const uint64_t some = __ballot(stays);
    if (lane == 0) sm.wave_count[wave] = __popcll(some);
    sm.near_[tid] = (unsigned long long)~(uint32_t)me << 32 | (uint32_t)tid;      // (an earlier index is a later entry of falling ones)
    __syncthreads();
    int n = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) n += sm.wave_count[k];              // (those that stay are the first ones)
    sm.weight[tid] = e;
    const float across = 1024.f / (float)V;
    put_in_order(n, [&](unsigned long long x) { return 1023 - (int)fminf((float)(uint32_t)(x >> 32) * across, 1023.f); });
    const unsigned long long by = tid < n ? sm.sorted[n - 1 - tid] : 0;
    e = tid < n ? sm.weight[(uint32_t)by] : 0.0;
    double total;
    const double passed = running(e, &total), target = (double)u * total;
    // (the last one where rounding leaves none)
    const int first = first_thread(tid < n && (passed > target || tid == n - 1));
    if (tid == first) {
      a.token[r] = (int)(by >> 32);
      if (a.logprob) a.logprob[r] = (float)log(e / total);
    }
    return;
  }
  if (P < 1.f) move_cut(std::true_type(), 0, nullptr, nullptr);

  // ---- the draw ----
  auto goal = [&](double all) { return (double)u * all; };
  const double least = M;
  Found f;
  if (cut == -INFINITY && !(M > 0.f)) f = locate([&](float x, int) { return e_of(x); }, goal);
  else if (!(M > 0.f)) f = locate([&](float x, int i) { return e_of(kept(x, i) ? x : -INFINITY); }, goal);
  else f = locate([&](float x, int i) { const double e = e_of(kept(x, i) ? x : -INFINITY); return e >= least ? e : 0.0; }, goal);
  if (tid == 0) {
    a.token[r] = f.index;
    if (a.logprob) a.logprob[r] = (float)log(f.weight / f.total);
  }
}

template <typename T> static void run_sample(const SampleArgs &a, int n_row, hipStream_t s) {
  constexpr int G = 16 / sizeof(T);
  const dim3 grid((unsigned)n_row), threads(1024);
  const int granules = (a.vocab + 2 * G - 2) / G, chunks = (granules + 1023) / 1024;      // (a row may begin within one)
  if constexpr (sizeof(T) == 4)                          // (for 16-bit values that variant keeps registers in scratch memory)
    if (chunks <= 1) {
      hipLaunchKernelGGL((k_sample<T, 16>), grid, threads, 0, s, a);
      return;
    }
  if (chunks <= 2) hipLaunchKernelGGL((k_sample<T, 32>), grid, threads, 0, s, a);
  else if (chunks <= 4) hipLaunchKernelGGL((k_sample<T, 64>), grid, threads, 0, s, a);
  else if (chunks <= 6) hipLaunchKernelGGL((k_sample<T, 96>), grid, threads, 0, s, a);
  else if (chunks <= 8) hipLaunchKernelGGL((k_sample<T, 128>), grid, threads, 0, s, a);
  else hipLaunchKernelGGL((k_sample<T, 0>), grid, threads, 0, s, a);
}

int launch_sample(const SampleArgs &a, int type, int n_row, hipStream_t s) {
  PD_REQUIRE(n_row < (1 << 22), PD_EINVAL, "a launch of %d rows is too large", n_row);      // (of 1024 threads, of which it may have fewer than 2^32)
  if (type == PD_TYPE_F32) run_sample<float>(a, n_row, s);
  else if (type == PD_TYPE_BF16) run_sample<bf16_t>(a, n_row, s);
  else run_sample<f16_t>(a, n_row, s);
  PD_CHECK_HIP(hipGetLastError());
  return PD_OK;
}

extern "C" int pd_sample(const void *logits, int type, int64_t row_stride, int n_row, int vocab, const float *u,
                         const pd_sampling *params, int32_t *out_token, float *out_logprob, void *hip_stream) {
  PD_REQUIRE(type == PD_TYPE_F32 || type == PD_TYPE_BF16 || type == PD_TYPE_F16, PD_EINVAL,
             "type must be PD_TYPE_F32, PD_TYPE_BF16 or PD_TYPE_F16 (got %d)", type);
  PD_REQUIRE(n_row >= 0 && vocab >= 1 && vocab <= PD_SAMPLE_VOCAB, PD_EINVAL, "n_row must be >= 0 and vocab within 1 and %d (got %d, %d)",
             PD_SAMPLE_VOCAB, n_row, vocab);
  if (n_row == 0) return PD_OK;
  PD_REQUIRE(logits && u && params && out_token, PD_EINVAL, "NULL argument");
  PD_REQUIRE(((uintptr_t)logits & (type == PD_TYPE_F32 ? 3 : 1)) == 0, PD_EINVAL, "logits must be aligned to their type");
  SampleArgs a{logits, row_stride, vocab, u, *params, out_token, out_logprob, nullptr};
  return launch_sample(a, type, n_row, (hipStream_t)hip_stream);
}
