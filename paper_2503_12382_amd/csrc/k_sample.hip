// Symbols drawn from rows of logits (reno_head.h).
//
// Decisions next to borders have to be those of exact sums, so masses are
// integers: a symbol's weight 2^y, y = (z - max) log2(e) / T, is computed in 64
// bits and counted in units of 2^-S of the largest, 2^S V < 2^63.  Sums of them
// are exact in any order, that of LDS atomics among it.
//
// What is kept is a run of the row in descending order, ties by index: logits
// above a cut, and some of those that equal it.  The cut of a count or a mass is
// found without sorting: a histogram by value over the row, then among the few
// logits of the bin that holds it the sums of all pairs (more than fit a list:
// histograms over what the bin spans, until that is one value).  The symbol is
// found by sums along the row, of a lane or of a wave's turn, and in the one that
// holds it once more.
//
// Bound by instructions, not by the read of the logits: an exact weight is 21 of
// them, 17 in 64 bits, which run at the rate of 32.
//   k_sample_short  rows of up to 256: 16 lanes a row, so that one wave's
//                   instructions serve four rows, the row and its weights in
//                   registers.  233737 x 256 fp32, top_p 0.95, a mask: 119 us,
//                   2.0 TB/s, 1241 vector instructions of a wave, 469 of them
//                   the cut's (76 us and 772 without one)
//   k_sample_long   a block a row.  Small counts: the k-th largest of many
//                   groups' maxima bounds the k-th largest logit, and what lies
//                   above is cut, weighed and drawn from in a list (one row of
//                   131071 fp32, top_k 50: 30 us, one block's latency).  bf16
//                   by mass: values are counted first and weighed once each
//                   (4096 x 32768, top_p 0.9, min_p 0.001: 148 us, 33 vector
//                   instructions a logit).  Else by a histogram of weights
//                   (2048 x 32768 fp32, top_p 0.9: 157 us, 805 MB read)
// Times: of a call among many in a row on one input.  The first few after a
// pause, as a short trace has them, take up to a sixth longer (137 us for 119).

#include <algorithm>
#include <cmath>

#include "dev.h"
#include "head.h"
#include "head_dev.h"
#include "logits.h"

namespace reno {
namespace {

constexpr uint32_t FIRST_LIVE = 0x00800000u;   // ordered(-inf) + 1
constexpr uint32_t ALL = 0xffffffffu;

// a b + c with c from scalar registers: the compiler would copy a constant to the result's registers first, two moves
// for each step of a polynomial.
__device__ __forceinline__ double fma_s(double a, double b, double c) {
  double r;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(c));
  return r;
}

// 2^y for N values of y >= -900, below 2^52.  All steps of the values side by side: one chain would wait for itself.
template <int N>
__device__ __forceinline__ void exp2_all(const double (&y)[N], double (&w)[N]) {
  constexpr double ROUND = 0x1.8p52;
  double t[N], f[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    t[e] = y[e] + ROUND;
    f[e] = y[e] - (t[e] - ROUND);
    w[e] = 0x1.e5e9ef7b8cd7ap-28;
  }
  // (2^f - 1) / f on [-1/2, 1/2], interpolated at the zeros of a Chebyshev polynomial; 1 + f q is right to 2^-50
  constexpr double C[9] = {0x1.b6571e5ac5dabp-24, 0x1.62bfe465e6f1bp-20, 0x1.ffcb7678282dfp-17,
                           0x1.4309130375a29p-13, 0x1.5d87fe908fa7dp-10, 0x1.3b2ab6fba3871p-7,
                           0x1.c6b08d7044119p-5,  0x1.ebfbdff82c590p-3,  0x1.62e42fefa39f7p-1};
#pragma unroll
  for (int k = 0; k < 9; ++k)
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = fma_s(w[e], f[e], C[k]);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    // the whole part goes to the exponent
    const uint64_t b = __builtin_bit_cast(uint64_t, __builtin_fma(w[e], f[e], 1.0));
    const uint32_t n = (uint32_t)__builtin_bit_cast(uint64_t, t[e]) << 20;
    w[e] = __builtin_bit_cast(double, (uint64_t)((uint32_t)(b >> 32) + n) << 32 | (uint32_t)b);
  }
}

// 2^((x - m) c) in units of 2^-S, to the nearest; x <= m, c >= 0, S <= 51 a whole number.  -inf and NaN give 0.
template <int N>
__device__ __forceinline__ void units_all(const float* x, double m, double c, double S, uint64_t* u) {
  double y[N], w[N];
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] = fmax(__builtin_fma((double)x[e] - m, c, S), -900.0);
  exp2_all<N>(y, w);
  // the sum with 2^52 rounds to a whole number, which its fraction then is
#pragma unroll
  for (int e = 0; e < N; ++e) u[e] = __builtin_bit_cast(uint64_t, w[e] + 0x1p52) & 0xfffffffffffffull;
}
__device__ __forceinline__ uint64_t units(float x, double m, double c, double S) {
  uint64_t u;
  units_all<1>(&x, m, c, S, &u);
  return u;
}

// log2 of a whole number from 1, to 2^-42: fp32's logarithm, and what 2 to its power lacks.
__device__ __forceinline__ double log2_of(uint64_t n) {
  const int e = 63 - __builtin_clzll(n);
  const double f = __builtin_ldexp((double)n, -e);           // 1 .. 2
  const double l = (double)__builtin_amdgcn_logf((float)f);
  const double y[1] = {-l};
  double w[1];
  exp2_all<1>(y, w);
  return (double)e + l + __builtin_fma(f, w[0], -1.0) * 1.4426950408889634;
}

__device__ __forceinline__ void add(uint64_t* to, uint64_t v) {   // LDS
  atomicAdd(reinterpret_cast<unsigned long long*>(to), (unsigned long long)v);
}

// The units of a row of V: the sum of V of them stays below 2^63.
int unit_bits(int V) {
  int lg = 0;
  while ((int64_t(1) << lg) < V) ++lg;
  return std::min(51, 62 - lg);
}

// ceil(p m), 1 at least, for p < 1, and floor(u m) for 0 <= u < 1, the products as 64-bit floats: so that a share of
// equal weights is what it says (0.9 of 3000 is 2700, though the float next to 0.9 lies above it).
__device__ __forceinline__ uint64_t share_up(double p, uint64_t m) {
  return max(min((uint64_t)__builtin_ceil(fmax(p, 0.0) * (double)m), m), (uint64_t)1);
}
__device__ __forceinline__ uint64_t share_down(float u, uint64_t m) { return (uint64_t)((double)u * (double)m); }

// A row's settings.
struct Row {
  double T, c, p, least, log_least;   // c: log2(e) / T, 0 for a T of 0
  float octaves;                      // below the largest weight: the cut by p lies above
  int64_t k;                          // 0: all
  float u;
  bool valid;
};

struct SampleArgs {
  const void* z;
  int64_t stride;
  int V, S;
  double T, c, p, least, log_least;
  float octaves;
  int k;
  const float *T_rows, *p_rows, *least_rows;
  const int32_t* k_rows;
  const uint8_t* allowed;
  int64_t allowed_stride;
  const float* u;
  int32_t* symbol;
  float* bits;
};

constexpr double LOG2E_D = 1.4426950408889634;

// V weights below (1 - p) / V of the largest are together less than what a share of p may miss.
__host__ __device__ __forceinline__ float octaves_of(int V, double p) {
  return log2f((float)V) - log2f(fmaxf((float)(1.0 - p), 0x1p-60f)) + 1.0f;
}

__device__ __forceinline__ Row settings(const SampleArgs& a, int64_t r) {
  Row s;
  s.u = a.u[r];
  s.T = a.T;
  if (a.T_rows) {   // past the range: its end
    const double T = (double)a.T_rows[r];
    s.T = T > 0.0 && T < (double)INFINITY ? fmin(fmax(T, 0x1p-126), 0x1p126) : T;
  }
  s.p = a.p_rows ? (double)a.p_rows[r] : a.p;
  s.least = a.least_rows ? (double)a.least_rows[r] : a.least;
  s.k = max(a.k_rows ? a.k_rows[r] : a.k, 0);
  s.c = a.c;
  if (a.T_rows) s.c = s.T > 0.0 ? LOG2E_D / s.T : 0.0;
  s.octaves = a.octaves;
  if (a.p_rows) s.octaves = octaves_of(a.V, fmax(s.p, 0.0));
  s.valid = s.T >= 0.0 && s.T < (double)INFINITY && s.p == s.p && s.least == s.least;
  s.least = fmin(s.least, 1.0);
  s.log_least = a.log_least;
  if (a.least_rows) s.log_least = s.least > 0.0 ? log(s.least) : 0.0;
  if (s.T == 0.0) {   // the largest alone
    s.k = 1;
    s.p = 1.0;
    s.least = 0.0;
  }
  return s;
}

// The ordered value from which on logits have a weight of set.least of the largest, m.
__device__ __forceinline__ uint32_t least_key(const Row& set, float m) {
  if (!(set.least > 0.0)) return FIRST_LIVE;
  const double z = (double)m + set.T * set.log_least;
  float f = (float)z;
  if ((double)f < z) f = nextafterf(f, INFINITY);
  return max(ordered(f), FIRST_LIVE);
}

// ---------------------------------------------------------------------------
// Rows of up to 256 logits: 16 lanes a row.

constexpr int SHORT_LANE = 16;      // logits of a lane, lanes of a row
constexpr int SHORT_ROWS = 4;       // rows of a wave
constexpr int SHORT_BINS = 64;

template <int CTRL>
__device__ __forceinline__ uint64_t dpp64(uint64_t v) {   // lanes without a source: 0
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, 0xF, 0xF, true);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t row16_scan(uint64_t v) {   // inclusive
  v += dpp64<0x111>(v);
  v += dpp64<0x112>(v);
  v += dpp64<0x114>(v);
  return v + dpp64<0x118>(v);
}
__device__ __forceinline__ uint32_t row16_scan(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, true);
  return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
  v = max(v, dpp<0x128>(v));
  v = max(v, dpp<0x124>(v));
  v = max(v, dpp<0x122>(v));
  return max(v, dpp<0x121>(v));
}
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, __uint_as_float(dpp<0x128>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(dpp<0x124>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(dpp<0x122>(__float_as_uint(v))));
  return fmaxf(v, __uint_as_float(dpp<0x121>(__float_as_uint(v))));
}
__device__ __forceinline__ float row16_min(float v) {
  v = fminf(v, __uint_as_float(dpp<0x128>(__float_as_uint(v))));
  v = fminf(v, __uint_as_float(dpp<0x124>(__float_as_uint(v))));
  v = fminf(v, __uint_as_float(dpp<0x122>(__float_as_uint(v))));
  return fminf(v, __uint_as_float(dpp<0x121>(__float_as_uint(v))));
}
template <typename T>
__device__ __forceinline__ T row16_last(T v) { return __shfl(v, lane_id() | 15); }
// The lane of this row whose condition holds (one of them; 15 where none does).
__device__ __forceinline__ int row16_which(bool here) {
  const uint32_t b = (uint32_t)(__ballot(here) >> (lane_id() & 48)) & 0xffffu;
  return (lane_id() & 48) | (b ? __builtin_ctz(b) : 15);
}

// Shared memory of a wave.
struct ShortShared {
  uint64_t hist[SHORT_ROWS][SHORT_BINS + 16];   // 63 bins, then the last one, of each lane: most logits lie far below
  ulonglong2 cand[SHORT_ROWS][16];
  float x[SHORT_ROWS][16 * SHORT_LANE];   // the rows, for the turns that are rare: logit i of lane l at 16 i + l
};

// A row's logits in registers, -inf where there is none, with their weights.
template <int PL>
struct Short {
  float x[PL];
  uint64_t w[PL];
  int v0;             // the lane's first symbol
};

// The last logit of the row's order that is kept: logits above x, and those that equal it up to symbol v.  split: there
// are others that equal it behind v.
struct ShortCut {
  float x;
  int v;
  bool split;
};

// A search under way: `above` lies above the range that still holds the cut, `wanted` is what it has to reach.
struct ShortSearch {
  uint64_t above, wanted;
  bool active;
};

// A place in the row's order: the ordered value, then the index complemented.
__device__ __forceinline__ uint64_t place_of(float x, int v) { return (uint64_t)ordered(x) << 8 | (uint32_t)(255 - v); }

__device__ __forceinline__ float next_below(float x) { return __uint_as_float(__float_as_uint(x) - 1u); }   // x > 0
__device__ __forceinline__ float next_above(float x) {
  return x == 0.0f ? 0x1p-149f : __uint_as_float(__float_as_uint(x) + (x > 0.0f ? 1u : ~0u));
}

// The bin of a histogram at which what is wanted is reached; q.above becomes what lies above it.
__device__ __forceinline__ int short_bin(ShortSearch& q, uint64_t (&h)[SHORT_BINS / 16], uint64_t mine,
                                         uint64_t upto) {
  constexpr int PER = SHORT_BINS / 16;
  uint64_t a = q.above + upto - mine;
  const int owner = row16_which(a < q.wanted && a + mine >= q.wanted);
  int bin = (lane_id() & 15) * PER;
  bool past = false;
#pragma unroll
  for (int i = 0; i < PER - 1; ++i) {
    past |= a + h[i] >= q.wanted;
    bin += past ? 0 : 1;
    a += past ? 0 : h[i];
  }
  const uint64_t above = __shfl(a, owner);
  q.above = q.active ? above : q.above;
  return __shfl(bin, owner);
}

// The cut among the `n` <= 16 candidates that lie in LDS, for rows with `few`: ranks and sums of all pairs.
__device__ __forceinline__ void short_pairs(const ShortShared& s, ShortSearch& q, bool few, uint32_t n, ShortCut* cut) {
  const int lane = lane_id(), l15 = lane & 15, rw = lane >> 4;
  wave_lds_fence();
  const bool there = few && l15 < (int)n;
  const ulonglong2 me = s.cand[rw][l15];
  uint64_t sum = q.above;
  for (int j = 0; __any(few && j < (int)n); ++j) {
    const ulonglong2 o = s.cand[rw][j];
    sum += j < (int)n && o.x >= me.x ? o.y : 0;
  }
  const int who = row16_which(there && sum >= q.wanted && sum - me.y < q.wanted);
  const uint64_t last = __shfl((uint64_t)me.x, who);
  const bool behind = there && me.x < last && me.x >> 8 == last >> 8;
  cut->x = few ? from_ordered((uint32_t)(last >> 8)) : cut->x;
  cut->v = few ? 255 - (int)(last & 255) : cut->v;
  cut->split = few ? (__ballot(behind) >> (lane & 48) & 0xffffu) != 0 : cut->split;
  q.active = q.active && !few;
  wave_lds_fence();
}

// The rare turns, for rows whose bin holds more than 16 logits (from what `in` says first): a histogram over what the
// bin spans until few are left or all are equal.  One logit at a time from LDS.
template <bool MASS, int PL, typename In>
__device__ __forceinline__ void short_more(ShortShared& s, ShortSearch& q, int v0, float m, double c, double S,
                                           const In& in, ShortCut* cut) {
  constexpr int PER = SHORT_BINS / 16;
  const int lane = lane_id(), l15 = lane & 15, rw = lane >> 4;
  uint32_t lo = 0, top = ALL;   // the ordered values that are left
  int shift = 0;
  bool first = true;
  const auto measure = [&](float x) -> uint64_t { return MASS ? units(x, (double)m, c, S) : 1; };
  const auto left = [&](float x) {
    const uint32_t o = ordered(x);
    return q.active && (first ? in(x) : o >= lo && o <= top);
  };
  while (__any(q.active)) {
    uint32_t n = 0, kmax = 0, kmin = ALL;
#pragma unroll 1
    for (int i = 0; i < PL; ++i) {
      const float x = s.x[rw][i * 16 + l15];
      if (left(x)) {
        ++n;
        kmax = max(kmax, ordered(x));
        kmin = min(kmin, ordered(x));
      }
    }
    const uint32_t upto_n = row16_scan(n);
    const uint32_t all_n = row16_last(upto_n);
    kmax = row16_max(kmax);
    kmin = ~row16_max(~kmin);
    const bool few = q.active && all_n <= 16;
    if (__any(few)) {
      uint32_t at = upto_n - n;
#pragma unroll 1
      for (int i = 0; i < PL; ++i) {
        const float x = s.x[rw][i * 16 + l15];
        if (few && left(x)) s.cand[rw][at++] = make_ulonglong2(place_of(x, v0 + i), measure(x));
      }
      short_pairs(s, q, few, all_n, cut);
    }
    const bool same = q.active && kmin == kmax;
    if (__any(same)) {   // equal logits: the symbol by their number
      const uint64_t each = max(measure(from_ordered(kmax)), (uint64_t)1);
      const uint32_t ties = (uint32_t)((q.wanted - q.above + each - 1) / each);   // the cut's place among them
      uint32_t to_go = ties - (upto_n - n);                                       // ... among the lane's
      const int who = row16_which(upto_n >= ties && upto_n - n < ties);
      int v = 0;
#pragma unroll 1
      for (int i = 0; i < PL; ++i)
        if (same && left(s.x[rw][i * 16 + l15])) {
          v = to_go == 1 ? v0 + i : v;
          --to_go;
        }
      v = __shfl(v, who);
      cut->x = same ? from_ordered(kmax) : cut->x;
      cut->v = same ? v : cut->v;
      cut->split |= same;
      q.active = q.active && !same;
    }
    if (!__any(q.active)) break;
    lo = kmin;
    top = kmax;
    shift = max(0, 26 - (int)__builtin_clz((kmax - kmin) | 1u));
    first = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) s.hist[rw][l15 * PER + i] = 0;
    wave_lds_fence();
#pragma unroll 1
    for (int i = 0; i < PL; ++i) {
      const float x = s.x[rw][i * 16 + l15];
      if (left(x)) add(&s.hist[rw][(top - ordered(x)) >> shift], measure(x));
    }
    wave_lds_fence();
    uint64_t h[PER], mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine += h[i] = s.hist[rw][l15 * PER + i];
    const int bin = short_bin(q, h, mine, row16_scan(mine));
    top -= (uint32_t)bin << shift;
    lo = max(lo, top - min(top, (1u << shift) - 1u));
  }
}

// For rows that are `active`: the last logit at which `want` of the measure (logits, or with MASS their weights) is
// reached from the largest, m, on; want(total) is asked with the measure of all, and more than that changes no `cut`.
// range: how far below m the cut lies at most, or is worth bins.
template <bool MASS, int PL, typename F>
__device__ __forceinline__ void short_search(const Short<PL>& row, ShortShared& s, bool active, float m, float range,
                                             double c, double S, const F& want, ShortCut* cut) {
  constexpr int PER = SHORT_BINS / 16;
  const int lane = lane_id(), l15 = lane & 15, rw = lane >> 4;
  ShortSearch q;
  q.above = 0;
  // (a range of 0: all are equal, and any scale puts them first and what is not there last)
  const float scale = active ? (range > 0.0f ? fminf((float)SHORT_BINS / fminf(range, 3e38f), 3e38f) : 1.0f) : NAN;
  const auto bin_of = [&](float x) { return (m - x) * scale; };   // NaN where the row is not searched
#pragma unroll
  for (int i = 0; i < PER + 1; ++i) s.hist[rw][i * 16 + l15] = 0;
  wave_lds_fence();
  const float last = (float)(SHORT_BINS - 1 + l15);
#pragma unroll
  for (int i = 0; i < PL; ++i)
    add(&s.hist[rw][(uint32_t)fminf(bin_of(row.x[i]), last)], MASS ? row.w[i] : 1);
  wave_lds_fence();
  uint64_t h[PER], mine = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    h[i] = i < PER - 1 || l15 < 15 ? s.hist[rw][l15 * PER + i] : 0;
    mine += h[i];
  }
  uint64_t upto = row16_scan(mine);
  const uint64_t far = row16_last(row16_scan(s.hist[rw][SHORT_BINS - 1 + l15]));
  const uint64_t all = row16_last(upto) + far;
  if (l15 == 15) {
    h[PER - 1] += far;
    mine += far;
    upto += far;
  }
  q.wanted = want(all);
  q.active = active && q.wanted <= all;
  const int bin = short_bin(q, h, mine, upto);
  // the bin's logits
  const float b0 = q.active ? (float)bin : NAN;
  const float b1 = bin == SHORT_BINS - 1 ? INFINITY : next_below((float)(bin + 1));
  const auto in = [&](float x) {
    const float b = bin_of(x);
    return b >= b0 && b <= b1;
  };
  uint32_t which = 0;
#pragma unroll
  for (int i = PL - 1; i >= 0; --i) which = which + which + (in(row.x[i]) ? 1u : 0u);
  const uint32_t n = (uint32_t)__builtin_popcount(which);
  const uint32_t upto_n = row16_scan(n);
  const uint32_t all_n = row16_last(upto_n);
  const bool few = q.active && all_n <= 16;
  uint32_t* list = reinterpret_cast<uint32_t*>(s.hist[rw]);   // the bins are done with
  wave_lds_fence();
  which = few ? which : 0;
  for (uint32_t at = upto_n - n; __any(which != 0); ++at) {
    if (which) list[at] = (uint32_t)__builtin_ctz(which) * 16u + (uint32_t)l15;
    which &= which - 1u;
  }
  wave_lds_fence();
  if (few && l15 < (int)all_n) {
    const uint32_t p = list[l15];
    const float x = s.x[rw][p];
    s.cand[rw][l15] =
        make_ulonglong2(place_of(x, (int)(p & 15u) * PL + (int)(p >> 4)), MASS ? units(x, (double)m, c, S) : 1);
  }
  short_pairs(s, q, few, all_n, cut);
  if (__any(q.active)) short_more<MASS, PL>(s, q, row.v0, m, c, S, in, cut);
}

// Whether logit i of the lane is kept: `lim`, the last of the lane whose ties are, is cut.v - v0.
__device__ __forceinline__ bool is_kept(float x, int i, float cut, float above, int lim) {
  return x >= (i <= lim ? cut : above);
}

template <int TYPE, int PL>
__device__ __forceinline__ void short_load(const SampleArgs& a, int64_t at, int v0, float (&x)[PL]) {
  const int V = a.V;
  if (PL == SHORT_LANE && v0 + PL <= V) {
#pragma unroll
    for (int i = 0; i < PL; i += Vec<TYPE>::N) {
      Vec<TYPE> t;
      uint4 raw;   // one load, wherever the row starts
      __builtin_memcpy(&raw, static_cast<const char*>(a.z) + (at + v0 + i) * (16 / Vec<TYPE>::N), 16);
      t.from(raw);
#pragma unroll
      for (int e = 0; e < Vec<TYPE>::N && i + e < PL; ++e) x[i + e] = t.x[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      x[i] = logit<TYPE>(a.z, at + min(v0 + i, V - 1));
      x[i] = v0 + i < V ? x[i] : -INFINITY;
    }
  }
}
template <int PL>
__device__ __forceinline__ void short_mask(const uint8_t* allowed, int V, int v0, float (&x)[PL]) {
  if (PL == SHORT_LANE && v0 + PL <= V) {
    uint32_t there[(PL + 3) / 4];
    __builtin_memcpy(there, allowed + v0, PL);
#pragma unroll
    for (int i = 0; i < PL; ++i) x[i] = there[i / 4] & (0xffu << (8 * (i & 3))) ? x[i] : -INFINITY;
  } else {
#pragma unroll
    for (int i = 0; i < PL; ++i) x[i] = allowed[min(v0 + i, V - 1)] ? x[i] : -INFINITY;
  }
}

// (4 waves a SIMD leave 128 registers, which the row, its weights and four of those under way fill, three to scratch:
// 233737 x 256 takes 119 us, 136 with 2 waves and 250 with 5, which spill far more.)
template <int TYPE, int PL>
__global__ void __launch_bounds__(256, 4) k_sample_short(SampleArgs a, int64_t rows) {
  __shared__ ShortShared s_all[4];
  const int lane = lane_id(), wave = threadIdx.x >> 6, l15 = lane & 15, rw = lane >> 4;
  const int64_t r0 = ((int64_t)blockIdx.x * 4 + wave) * SHORT_ROWS;
  if (r0 >= rows) return;
  ShortShared& s = s_all[wave];
  const int64_t r = min(r0 + rw, rows - 1);
  const double S = (double)a.S;
  Short<PL> row;
  row.v0 = l15 * PL;
  short_load<TYPE, PL>(a, r * a.stride, row.v0, row.x);
  const Row set = settings(a, r);
  const bool taken = r0 + rw < rows && set.u >= 0.0f && set.u < 1.0f;
  if (a.allowed) short_mask<PL>(a.allowed + r * a.allowed_stride, a.V, row.v0, row.x);
  bool odd = false;
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    odd |= !(row.x[i] < INFINITY);
    m = fmaxf(m, row.x[i]);
    s.x[rw][i * 16 + l15] = row.x[i];
  }
  m = row16_max(m);
  const bool bad = taken && (!set.valid || (__ballot(odd) >> (lane & 48) & 0xffffu) != 0);
  const bool live = taken && !bad && m > -INFINITY;
  const double c = set.c;
#pragma unroll
  for (int i = 0; i < PL; i += PL < 4 ? 1 : 4) units_all<PL < 4 ? 1 : 4>(row.x + i, (double)m, c, S, row.w + i);
  ShortCut cut{-INFINITY, 255, false};
  const bool by_count = live && set.k > 0 && set.k < a.V;
  if (__any(by_count)) {
    float low = INFINITY;
#pragma unroll
    for (int i = 0; i < PL; ++i) low = fminf(low, row.x[i] > -INFINITY ? row.x[i] : INFINITY);
    short_search<false>(row, s, by_count, m, m - row16_min(low), c, S, [&](uint64_t) { return (uint64_t)set.k; }, &cut);
    // what is cut off has no part in the shares
    const float over = next_above(cut.x);
#pragma unroll
    for (int i = 0; i < PL; ++i)
      if (!is_kept(row.x[i], i, cut.x, over, cut.v - row.v0)) {
        row.x[i] = -INFINITY;
        row.w[i] = 0;
        s.x[rw][i * 16 + l15] = -INFINITY;
      }
  }
  const bool by_mass = live && set.p < 1.0;
  if (__any(by_mass))
    short_search<true>(row, s, by_mass, m, set.octaves * __builtin_amdgcn_rcpf((float)c), c, S,
                       [&](uint64_t t) { return share_up(set.p, t); }, &cut);
  if (__any(live && set.least > 0.0)) {
    const float least = from_ordered(least_key(set, m));
    if (live && set.least > 0.0 && least > cut.x) cut = ShortCut{least, 255, false};
  }
  uint64_t mine = 0;
  const float over = next_above(cut.x);
  if (__any(cut.split)) {   // among logits that equal the last one
#pragma unroll
    for (int i = 0; i < PL; ++i) row.w[i] = is_kept(row.x[i], i, cut.x, over, cut.v - row.v0) ? row.w[i] : 0;
  } else {
#pragma unroll
    for (int i = 0; i < PL; ++i) row.w[i] = row.x[i] >= cut.x ? row.w[i] : 0;
  }
#pragma unroll
  for (int i = 0; i < PL; ++i) mine += row.w[i];
  uint64_t upto = row16_scan(mine);
  const uint64_t total = row16_last(upto);
  const uint64_t want = share_down(set.u, total) + 1;
  if (__any(live && want == 1)) {   // a share of nothing: the first symbol of any weight, though it be less than a unit
    const bool any = live && want == 1;
    uint64_t ones = 0;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const bool some =
          is_kept(row.x[i], i, cut.x, over, cut.v - row.v0) && ((double)row.x[i] - (double)m) * c >= -1074.0;
      row.w[i] = any ? (some ? 1 : 0) : row.w[i];
      ones += row.w[i];
    }
    mine = any ? ones : mine;
    upto = row16_scan(mine);
  }
  // the lane that holds the symbol hands its weights to the row's lanes
  const int who = row16_which(upto - mine < want && upto >= want);
  uint64_t* wl = s.hist[rw];
  if (lane == who) {
#pragma unroll
    for (int i = 0; i < PL; ++i) wl[i] = row.w[i];
  }
  wave_lds_fence();
  const uint64_t w = l15 < PL ? wl[l15] : 0;
  const uint64_t before = __shfl(upto - mine, who);
  const uint64_t at = before + row16_scan(w);
  if (live && at >= want && at - w < want) {
    const int v = (who & 15) * PL + l15;
    a.symbol[r] = v;
    a.bits[r] = (float)(log2_of(total) - S - ((double)s.x[rw][l15 * 16 + (who & 15)] - (double)m) * c);
  }
  if (!live && l15 == 0 && r0 + rw < rows) {
    a.symbol[r] = -1;
    a.bits[r] = bad ? NAN : 0.0f;
  }
}

// ---------------------------------------------------------------------------
// A block a row.

constexpr int BINS = 1024;
constexpr int LIST = 512;       // logits that are compared with one another
constexpr int LIST_K = 256;     // counts up to this are cut in a list of what the maxima of groups bound from below

// Of each row of lanes in ROWS: the value of lane 15 of the row before (0x142), or of lane 31 (0x143); else 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_rows(uint64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, false);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {   // inclusive
  v = row16_scan(v);
  v += dpp_rows<0x142, 0xA>(v);
  return v + dpp_rows<0x143, 0xC>(v);
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {   // in every lane
  v = wave_scan(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), 63);
  return (uint64_t)hi << 32 | lo;
}

// bf16 logits of 2^-6 to 2^6 are counted by value, one of 12 times 128 values of either sign.
constexpr int ZONE = 12 * 128, ZONE_FIRST = (127 - 6) << 7, OTHERS = 512;

// What a row keeps: logits above x, and of those that equal it the first `ties` (ALL: all).
struct Cut {
  float x;
  uint32_t ties;
};

// A wave's turn: what its logits above the cut weigh, and how many equal it.
struct Turn {
  uint64_t above, equal;
};

// THREADS a row.  A wave's pieces of 16 bytes follow one another: the row's order is by wave, then by turn, then by
// lane.  KEEP: the first look leaves the row in LDS, where a thread reads what it wrote itself.  Else the row is read
// anew for each look: with rows for every CU LDS has no place for enough of them (4096 rows of 32768 bf16, with four
// looks a row: 210 us, and 247 with the row in LDS; two looks now).
template <int TYPE, int THREADS, bool KEEP>
struct Long {
  static constexpr int N = Vec<TYPE>::N, WAVES = THREADS / 64, SIZE = 16 / N;
  static constexpr uint32_t DEAD = TYPE == RENO_T_FP32 ? 0xff800000u : TYPE == RENO_T_BF16 ? 0xff80ff80u : 0xfc00fc00u;
  const char* z;
  const uint8_t* allowed;
  uint4* kept;
  int V, turns, first;      // first: this thread's first piece

  // a piece; -inf where there is no logit
  __device__ __forceinline__ uint4 read(int piece) const {
    uint32_t w[4] = {DEAD, DEAD, DEAD, DEAD};
    const int v = piece * N;
    if (v + N <= V) {
      __builtin_memcpy(w, z + (int64_t)v * SIZE, 16);   // one load, wherever the row starts
      if (allowed) {
        uint8_t a[N];
        __builtin_memcpy(a, allowed + v, N);
#pragma unroll
        for (int e = 0; e < N; ++e) put(w, e, a[e] != 0);
      }
    } else if (v < V) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (v + e < V) {
          if constexpr (N == 4) w[e] = reinterpret_cast<const uint32_t*>(z)[v + e];
          else w[e / 2] = (w[e / 2] & (e & 1 ? 0xffffu : 0xffff0000u)) |
                          (uint32_t)reinterpret_cast<const uint16_t*>(z)[v + e] << (16 * (e & 1));
          if (allowed) put(w, e, allowed[v + e] != 0);
        }
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static __forceinline__ void put(uint32_t (&w)[4], int e, bool there) {
    if constexpr (N == 4) w[e] = there ? w[e] : DEAD;
    else {
      const uint32_t mask = e & 1 ? 0xffff0000u : 0xffffu;
      w[e / 2] = there ? w[e / 2] : (w[e / 2] & ~mask) | (DEAD & mask);
    }
  }
  __device__ __forceinline__ Turn* sums() const {
    return reinterpret_cast<Turn*>(kept + (KEEP ? turns * THREADS : 0));
  }
  __device__ __forceinline__ int index(int turn, int e) const { return (first + turn * 64) * N + e; }
  __device__ __forceinline__ uint4 load(int turn) const {   // the first look
    const uint4 r = read(first + turn * 64);
    if constexpr (KEEP) kept[turn * THREADS + threadIdx.x] = r;
    return r;
  }
  __device__ __forceinline__ uint4 raw(int turn) const {
    if constexpr (KEEP) return kept[turn * THREADS + threadIdx.x];
    else return read(first + turn * 64);
  }
  __device__ __forceinline__ Vec<TYPE> at(int turn) const {
    Vec<TYPE> x;
    x.from(raw(turn));
    return x;
  }
  // f(turn, logits) for every turn of the thread
  template <typename F>
  __device__ __forceinline__ void each(const F& f) const {
    for (int t = 0; t < turns; ++t) {
      const Vec<TYPE> x = at(t);
      f(t, x.x);
    }
  }
};

// Shared memory of a row.
template <int WAVES>
struct Shared {
  uint64_t hist[BINS + 64];   // the last bin is one of each lane's: what lies far below meets there; then weights
  uint64_t list[LIST];        // places: the ordered value, then the index complemented, or the turn
  uint16_t other[OTHERS];     // bf16 values outside the table of counts, which lies over both of the above
  uint64_t part[WAVES];
  uint64_t above, total, before;
  uint32_t lo, hi, left;
  float top[WAVES], x;
  int odd[WAVES], count[2 * WAVES];
  int bin, n, wave, turn, index;
};

__device__ __forceinline__ uint64_t place64(float x, int v) { return (uint64_t)ordered(x) << 32 | (uint32_t)~v; }
__device__ __forceinline__ float x_of(uint64_t place) { return from_ordered((uint32_t)(place >> 32)); }
__device__ __forceinline__ int v_of(uint64_t place) { return (int)~(uint32_t)place; }

// The sum of a value a thread, in every thread.
template <int WAVES>
__device__ __forceinline__ uint64_t block_total(Shared<WAVES>& s, uint64_t v) {
  v = wave_sum(v);
  __syncthreads();
  if (lane_id() == 0) s.part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
  for (int i = 0; i < WAVES; ++i) v += s.part[i];
  return v;
}

// Wave 0: the first bin at whose end `want` of what `above` and the bins hold is reached, and what lies above it.
// want(total) is asked with what all bins hold; bin -1: more than there is.
template <int WAVES, typename F>
__device__ __forceinline__ void find_bin(Shared<WAVES>& s, uint64_t above, const F& want) {
  if (threadIdx.x < 64) {
    constexpr int PER = BINS / 64;
    const int lane = lane_id();
    const uint64_t far = wave_sum(s.hist[BINS - 1 + lane]);   // (slot BINS - 1 + 64 lies past the lanes')
    uint64_t mine = lane == 63 ? far : 0;
#pragma unroll
    for (int i = 0; i < PER - 1; ++i) mine += s.hist[lane * PER + i];
    if (lane < 63) mine += s.hist[lane * PER + PER - 1];
    const uint64_t upto = wave_scan(mine);
    const uint64_t total = __shfl(upto, 63);
    const uint64_t w = want(total);
    uint64_t a = above + upto - mine;
    if (lane == 0) {
      s.total = total;
      if (w > above + total) s.bin = -1;
    }
    if (a < w && a + mine >= w) {
      int i = lane * PER;
      while (i < BINS - 1 && a + s.hist[i] < w) a += s.hist[i++];
      s.bin = i;
      s.above = a;
    }
  }
}

// A search by mass that has found its bin, and leaves the cut in it to the next look at the row: what lies above the
// bin, and what the cut has to reach.
struct Pending {
  bool on;
  float b0, b1, m, scale, over;   // the bin's logits: b0 <= (m - x) scale <= b1 and x > over
  uint64_t above, wanted;
};

// The cut at x: as many of the logits that equal it, `equal` together and each of weight w, as it takes after what lies
// above.
__device__ __forceinline__ Cut cut_at(float x, uint64_t w, uint64_t wanted, uint64_t above, uint64_t equal) {
  const uint64_t ties = (wanted - above + w - 1) / w;
  return Cut{x, ties * w >= equal ? ALL : (uint32_t)ties};
}

// The cut among n listed logits (their ordered values in the upper halves) of the measures s.hist: sums of all pairs.
template <int WAVES>
__device__ __forceinline__ Cut pairs(Shared<WAVES>& s, int n, uint64_t wanted, uint64_t above) {
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += WAVES * 64) {
    const uint32_t me = (uint32_t)(s.list[i] >> 32);
    uint64_t more = above, equal = 0;
    for (int j = 0; j < n; ++j) {
      const uint32_t o = (uint32_t)(s.list[j] >> 32);
      more += o > me ? s.hist[j] : 0;
      equal += o == me ? s.hist[j] : 0;
    }
    if (more < wanted && more + equal >= wanted) {   // (all that are equal write the same)
      s.x = from_ordered(me);
      s.above = s.hist[i];
      s.before = more;
      s.total = equal;
    }
  }
  __syncthreads();
  return cut_at(s.x, s.above, wanted, s.before, s.total);
}

// The symbol at which the weights along the row of what the cut keeps reach want(total), at least 1, and its logit.
// PEND: a search is pending, and the cut found on the way (false: too many logits in its bin, nothing is done).
template <bool PEND, typename L, typename S, typename W>
__device__ __forceinline__ bool pick(const L& row, S& s, Cut& cut, const Pending& pend, double m, double c, double bits,
                                     const W& want, int* index, float* logit, uint64_t* total) {
  constexpr int N = L::N, WAVES = L::WAVES, PUSHED = (int)(sizeof(s.hist) + (PEND ? 0 : sizeof(s.list))) / 4 / WAVES;
  Turn* turns = row.sums();
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  float* pushed = reinterpret_cast<float*>(s.hist) + wave * PUSHED;   // a turn's logits, where histogram and list were
  bool whole = cut.ties == ALL;                // of those that equal the cut too
  float from = whole ? cut.x : next_above(cut.x);
  __syncthreads();
  for (int t = 0; t < row.turns; ++t) {
    const auto x = row.at(t);
    uint64_t mine = 0;
    int n = 0, equal = 0;
    // few are kept as a rule: they are pushed together first, so that a weight is computed by every lane
    const bool all = !PEND && from == -INFINITY;
    const auto push = [&](bool kept, float y) {
      const uint64_t which = __ballot(kept);
      const uint32_t at = __builtin_amdgcn_mbcnt_hi((uint32_t)(which >> 32),
                                                    __builtin_amdgcn_mbcnt_lo((uint32_t)which, (uint32_t)n));
      if (kept && (PUSHED >= 64 * N || at < PUSHED)) pushed[at] = y;
      n += (int)__popcll(which);
    };
    if constexpr (PEND) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float b = (pend.m - x.x[e]) * pend.scale;
        push(b < pend.b0, x.x[e]);
        if (b >= pend.b0 && b <= pend.b1 && x.x[e] > pend.over) {
          const int i = atomicAdd(&s.n, 1);
          if (i < LIST) s.list[i] = (uint64_t)ordered(x.x[e]) << 32 | (uint32_t)(wave * row.turns + t);
        }
      }
    } else if (!all) {
#pragma unroll
      for (int e = 0; e < N; ++e) push(x.x[e] >= from, x.x[e]);
    }
    if (!PEND && !whole) {
#pragma unroll
      for (int e = 0; e < N; ++e) equal += (int)__popcll(__ballot(x.x[e] == cut.x));
    }
    if (!all && (PUSHED >= 64 * N || n <= PUSHED)) {
      wave_lds_fence();
      for (int i = lane; i < n; i += 64) mine += units(pushed[i], m, c, bits);
      wave_lds_fence();
    } else {
#pragma unroll
      for (int e0 = 0; e0 < N; e0 += 4) {
        uint64_t w[4];
        units_all<4>(x.x + e0, m, c, bits, w);
#pragma unroll
        for (int e = 0; e < 4; ++e)   // (-inf weighs nothing)
          mine += (PEND ? (pend.m - x.x[e0 + e]) * pend.scale < pend.b0 : x.x[e0 + e] >= from) ? w[e] : 0;
      }
    }
    mine = wave_sum(mine);
    if (lane == 0) turns[wave * row.turns + t] = Turn{mine, (uint64_t)equal};
  }
  __syncthreads();
  if constexpr (PEND) {
    const int n = s.n;
    if (n > LIST) return false;
    for (int i = threadIdx.x; i < n; i += WAVES * 64) s.hist[i] = units(x_of(s.list[i]), m, c, bits);
    cut = pairs(s, n, pend.wanted, pend.above);
    whole = cut.ties == ALL;
    from = whole ? cut.x : next_above(cut.x);
    // the bin's part in the turns' sums
    for (int i = threadIdx.x; i < n; i += WAVES * 64) {
      Turn& to = turns[(uint32_t)s.list[i]];
      if (x_of(s.list[i]) >= from) add(&to.above, s.hist[i]);
      else if (x_of(s.list[i]) == cut.x) add(&to.equal, 1);
    }
    __syncthreads();
  }
  const uint64_t each = whole ? 0 : units(cut.x, m, c, bits);
  if (wave == 0) {
    const int n = WAVES * row.turns, per = (n + 63) / 64, first = lane * per, end = min(n, first + per);
    uint64_t mine = 0, equal = 0;
    for (int i = first; i < end; ++i) {
      mine += turns[i].above;
      equal += turns[i].equal;
    }
    // of what equals the cut, what is left to those from the lane's first turn on
    const uint64_t before = wave_scan(equal) - equal;
    uint64_t left = cut.ties > before ? cut.ties - before : 0;
    mine += min(left, equal) * each;
    const uint64_t upto = wave_scan(mine);
    const uint64_t all = __shfl(upto, 63);
    const uint64_t w = want(all);
    uint64_t a = upto - mine;
    if (lane == 0) s.total = all;
    if (a < w && a + mine >= w) {
      int i = first;
      for (; i < end; ++i) {
        const uint64_t here = turns[i].above + min(left, turns[i].equal) * each;
        if (a + here >= w) break;
        a += here;
        left -= min(left, turns[i].equal);
      }
      s.wave = i / row.turns;
      s.turn = i % row.turns;
      s.before = a;
      s.left = (uint32_t)left;
    }
  }
  __syncthreads();
  *total = s.total;
  const uint64_t w = want(s.total);
  if (wave == s.wave) {
    const int t = s.turn;
    const auto x = row.at(t);
    uint32_t equal = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) equal += !whole && x.x[e] == cut.x ? 1 : 0;
    uint32_t place = (uint32_t)wave_scan((uint64_t)equal) - equal;   // among the turn's that equal the cut
    uint64_t v[N], mine = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      bool kept = x.x[e] >= from;
      if (!whole && x.x[e] == cut.x) kept = place++ < s.left;
      v[e] = kept ? units(x.x[e], m, c, bits) : 0;
      mine += v[e];
    }
    uint64_t a = s.before + wave_scan(mine) - mine;
    if (a < w && a + mine >= w) {
      bool here = false;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        a += v[e];
        if (!here && a >= w) {
          here = true;
          s.index = row.index(t, e);
          s.x = x.x[e];
        }
      }
    }
  }
  __syncthreads();
  *index = s.index;
  *logit = s.x;
  return true;
}

// Where `want` of the measure (logits, or with MASS their weights) is reached in the row's order, of what `from` keeps;
// want(total) is asked with the measure of all of it, and more than that leaves `from`.
// range: how far below the largest, m, the cut lies at most, or is worth bins.  pend: NULL, or takes what is left to do
// once the bin is found.
template <bool MASS, typename L, typename S, typename F>
__device__ __forceinline__ Cut search(const L& row, S& s, const Cut from, float m, float range, double c, double bits,
                                      const F& want, Pending* pend) {
  constexpr int N = L::N, THREADS = L::WAVES * 64;
  const int tid = threadIdx.x;
  const float scale = range > 0.0f ? fminf((float)BINS / fminf(range, 3e38f), 3e38f) : 1.0f;
  const auto bin_of = [&](float x) { return (m - x) * scale; };
  const auto measure = [&](float x) -> uint64_t { return MASS ? units(x, (double)m, c, bits) : 1; };
  const auto clear = [&] {
    for (int i = tid; i < BINS + 64; i += THREADS) s.hist[i] = 0;
    __syncthreads();
  };
  const auto at = [&](float x, uint64_t wanted, uint64_t above) {   // (equal to x: as many as it takes)
    return cut_at(x, max(measure(x), (uint64_t)1), wanted, above, ~0ull);
  };
  clear();
  const float last = (float)(BINS - 1 + lane_id());
  row.each([&](int, const float (&x)[N]) {
#pragma unroll
    for (int e0 = 0; e0 < N; e0 += 4) {
      uint64_t w[4];
      if constexpr (MASS) units_all<4>(x + e0, (double)m, c, bits, w);
#pragma unroll
      for (int e = e0; e < e0 + 4; ++e)
        if (x[e] > from.x)
          add(&s.hist[(uint32_t)fminf(bin_of(x[e]), last)], MASS ? w[e - e0] : 1);
    }
  });
  if (tid == 0) s.n = 0;
  __syncthreads();
  const uint64_t tail = from.x > -INFINITY ? from.ties * measure(from.x) : 0;   // what equals from.x and is kept
  find_bin(s, 0, [&](uint64_t t) { return want(t + tail); });
  __syncthreads();
  const uint64_t wanted = want(s.total + tail);
  const int bin = s.bin;
  if (bin < 0) return tail && wanted < s.total + tail ? at(from.x, wanted, s.total) : from;
  uint64_t above = s.above;
  // the bin's logits
  const float b0 = (float)bin, b1 = bin == BINS - 1 ? INFINITY : next_below((float)(bin + 1));
  const auto in_bin = [&](float x) {
    const float b = bin_of(x);
    return b >= b0 && b <= b1 && x > from.x;
  };
  if (pend) {
    *pend = Pending{true, b0, b1, m, scale, from.x, above, wanted};
    return from;
  }
  row.each([&](int, const float (&x)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (in_bin(x[e])) {
        const int i = atomicAdd(&s.n, 1);
        if (i < LIST) s.list[i] = (uint64_t)ordered(x[e]) << 32;
      }
  });
  __syncthreads();
  const int n = s.n;
  if (n <= LIST) {
    for (int i = tid; i < n; i += THREADS) s.hist[i] = measure(x_of(s.list[i]));
    const Cut cut = pairs(s, n, wanted, above);
    // a search by mass asks a count for the number of its ties
    return MASS || cut.ties != ALL ? cut : Cut{cut.x, (uint32_t)(wanted - s.before)};
  }
  // too many: histograms of ordered values over what the bin spans, until one value is left
  if (tid == 0) {
    s.lo = ALL;
    s.hi = 0;
  }
  __syncthreads();
  uint32_t kmin = ALL, kmax = 0;
  row.each([&](int, const float (&x)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (in_bin(x[e])) {
        kmin = min(kmin, ordered(x[e]));
        kmax = max(kmax, ordered(x[e]));
      }
  });
  if (kmax) {
    atomicMin(&s.lo, kmin);
    atomicMax(&s.hi, kmax);
  }
  __syncthreads();
  uint32_t lo = s.lo, hi = s.hi;
  while (lo != hi) {
    const int shift = max(0, 22 - (int)__builtin_clz(hi - lo));   // hi - lo < BINS << shift
    clear();
    row.each([&](int, const float (&x)[N]) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint32_t o = ordered(x[e]), b = (hi - o) >> shift;
        if (o >= lo && o <= hi) add(&s.hist[b], measure(x[e]));
      }
    });
    __syncthreads();
    find_bin(s, above, [&](uint64_t) { return wanted; });
    __syncthreads();
    above = s.above;
    hi -= (uint32_t)s.bin << shift;
    lo = max(lo, hi - min(hi, (1u << shift) - 1u));
    __syncthreads();
  }
  return at(from_ordered(hi), wanted, above);
}

// The value at place i of the table.
__device__ __forceinline__ float zone_value(int i) {
  const uint32_t mag = (uint32_t)(i < ZONE ? ZONE - 1 - i : i - ZONE) + ZONE_FIRST;
  return __uint_as_float((mag | (i < ZONE ? 0x8000u : 0u)) << 16);
}

// A row of bf16 by how often each value occurs, for its first look: the largest logit, m, and the cut by mass, for which
// a weight is computed once for a value instead of for each logit.  Logits outside the table, of |x| below 2^-6 or from
// 2^6, are kept in a list.  *known: m and odd are set.  True: the cut too; else there are too many others, or the cut
// lies among them.
template <typename L, typename S, typename F>
__device__ __forceinline__ bool by_counts(const L& row, S& s, double c, double bits, const F& want, float* m, bool* odd,
                                          bool* known, Cut* cut) {
  constexpr int WAVES = L::WAVES, THREADS = WAVES * 64, PER = 8, RUNS = 2 * ZONE / PER;   // values of a thread's turn
  constexpr int TURNS = (RUNS + THREADS - 1) / THREADS;
  static_assert(sizeof(s.hist) + sizeof(s.list) >= 2 * ZONE * 4, "the table lies over hist and list");
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  uint32_t* table = reinterpret_cast<uint32_t*>(s.hist);   // from the lowest value up
  for (int i = tid; i < 2 * ZONE; i += THREADS) table[i] = 0;
  if (tid == 0) {
    s.n = 0;
    s.bin = -1;
    s.hi = 0;
    s.lo = 0;
  }
  __syncthreads();
  const auto count = [&](const uint4& r) {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t w = u[e / 2];
      const uint32_t d = (e & 1 ? w >> 16 & 0x7fffu : w & 0x7fffu) - ZONE_FIRST;
      const uint32_t sign = (uint32_t)(e & 1 ? (int32_t)w >> 31 : (int32_t)(w << 16) >> 31);
      if (d < ZONE) {
        atomicAdd(&table[(d ^ sign) + ZONE], 1u);
      } else {
        const uint32_t raw = e & 1 ? w >> 16 : w & 0xffffu;
        if (raw != 0xff80u) {
          const int i = atomicAdd(&s.n, 1);
          if (i < OTHERS) s.other[i] = (uint16_t)raw;
        }
      }
    }
  };
  for (int t0 = 0; t0 < row.turns; t0 += 4) {   // four loads under way
    uint4 raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t0 + i < row.turns) raw[i] = row.load(t0 + i);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t0 + i < row.turns) count(raw[i]);
  }
  __syncthreads();
  const int n = s.n;
  __syncthreads();   // (who goes on without this sets s.n anew)
  *known = n <= OTHERS;
  if (n > OTHERS) return false;
  // the largest: ordered values of the others, or the topmost count
  uint32_t top = 0;
  for (int i = tid; i < n; i += THREADS) top = max(top, ordered(__uint_as_float((uint32_t)s.other[i] << 16)));
  uint32_t k[TURNS][PER];
#pragma unroll
  for (int q = 0; q < TURNS; ++q) {
    const int run = q * THREADS + tid;
#pragma unroll
    for (int e = 0; e < PER; ++e) {   // from the top: a thread's values follow one another, threads take runs in turn
      const int i = 2 * ZONE - 1 - (run * PER + e);
      k[q][e] = run < RUNS ? table[i] : 0;
      if (k[q][e]) top = max(top, ordered(zone_value(i)));
    }
  }
  for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  if (lane == 0 && top) atomicMax(&s.hi, top);
  // NaN of a negative sign is ordered as any NaN; +inf and NaN: no distribution
  __syncthreads();
  top = s.hi;
  *odd = top >= 0xff800000u;
  *m = top ? from_ordered(top) : -INFINITY;
  if (*odd || !top) return true;
  const double dm = (double)*m;
  // what the others weigh: small ones, in the order between the table's halves, and large ones above or below all of it
  uint64_t small = 0, below = 0;
  for (int i = tid; i < n; i += THREADS) {
    const float x = __uint_as_float((uint32_t)s.other[i] << 16);
    const uint64_t w = units(x, dm, c, bits);
    if (x >= 0x1p6f) s.lo = 1;   // (any thread)
    if (x > -0x1p-6f) small += w;
    else below += w;
  }
  uint64_t mine[TURNS], all = 0;
#pragma unroll
  for (int q = 0; q < TURNS; ++q) {
    mine[q] = 0;
#pragma unroll
    for (int e0 = 0; e0 < PER; e0 += 4) {
      if (k[q][e0] | k[q][e0 + 1] | k[q][e0 + 2] | k[q][e0 + 3]) {
        float x[4];
        uint64_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = zone_value(2 * ZONE - 1 - ((q * THREADS + tid) * PER + e0 + e));
        units_all<4>(x, dm, c, bits, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[q] += k[q][e0 + e] ? k[q][e0 + e] * w[e] : 0;
      }
    }
    all += mine[q];
  }
  small = block_total(s, small);
  if (s.lo) return false;
  below = block_total(s, below);
  const uint64_t wanted = want(block_total(s, all) + small + below);
  uint64_t base = 0;
#pragma unroll
  for (int q = 0; q < TURNS; ++q) {
    const uint64_t upto = wave_scan(mine[q]);
    __syncthreads();
    if (lane == 63) s.part[wave] = upto;
    __syncthreads();
    uint64_t a = base + upto - mine[q];
    for (int i = 0; i < WAVES; ++i) {
      a += i < wave ? s.part[i] : 0;
      base += s.part[i];
    }
    const int run = q * THREADS + tid;
    if (run * PER >= ZONE) a += small;   // (a run lies on one side)
    if (run < RUNS && a < wanted && a + mine[q] >= wanted) {
      float x = 0.0f;
      uint64_t w = 0, times = 0;
#pragma unroll 1
      for (int e = 0; e < PER; ++e) {
        const int i = 2 * ZONE - 1 - (run * PER + e);
        x = zone_value(i);
        times = table[i];
        w = times ? units(x, dm, c, bits) : 0;
        if (a + times * w >= wanted) break;
        a += times * w;
      }
      s.x = x;
      s.bin = 1;
      const uint64_t ties = (wanted - a + w - 1) / w;
      s.left = ties < times ? (uint32_t)ties : ALL;
    }
  }
  __syncthreads();
  if (s.bin < 0) return false;
  *cut = Cut{s.x, s.left};
  return true;
}

template <int TYPE, int THREADS, bool KEEP>
__global__ void __launch_bounds__(THREADS) k_sample_long(SampleArgs a) {
  typedef Long<TYPE, THREADS, KEEP> L;
  constexpr int N = L::N, WAVES = L::WAVES, GROUPS = 4;
  __shared__ Shared<WAVES> s;
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const Row set = settings(a, r);
  const auto answer = [&](int symbol, float bits) {
    a.symbol[r] = symbol;
    a.bits[r] = bits;
  };
  if (!(set.u >= 0.0f && set.u < 1.0f) || !set.valid) {
    if (tid == 0) answer(-1, set.u >= 0.0f && set.u < 1.0f ? NAN : 0.0f);
    return;
  }
  L row;
  row.z = static_cast<const char*>(a.z) + r * a.stride * L::SIZE;
  row.allowed = a.allowed ? a.allowed + r * a.allowed_stride : nullptr;
  row.V = a.V;
  row.turns = (a.V + N * THREADS - 1) / (N * THREADS);
  row.first = wave * row.turns * 64 + lane;
  extern __shared__ uint4 s_row[];   // the row, where it is kept, then its turns' sums
  row.kept = s_row;
  const double c = set.c, S = (double)a.S;
  const bool by_count = set.k > 0 && set.k < a.V;
  const auto share = [&](uint64_t t) { return share_up(set.p, t); };
  float m = -INFINITY;
  bool odd = false, known = false, found = false;
  Cut cut{-INFINITY, ALL};   // nothing is cut off
  if constexpr (TYPE == RENO_T_BF16 && THREADS > 64)
    if (set.p < 1.0 && !by_count) found = by_counts(row, s, c, S, share, &m, &odd, &known, &cut);
  float group[GROUPS] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  if (!known) {
    // the largest logit, and the largest of the thread's groups
    const auto look = [&](const uint4& raw) {
      Vec<TYPE> x;
      x.from(raw);
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        odd |= !(x.x[e] < INFINITY);
        top = fmaxf(top, x.x[e]);
      }
      const float first = fmaxf(group[0], top);
#pragma unroll
      for (int g = 0; g + 1 < GROUPS; ++g) group[g] = group[g + 1];
      group[GROUPS - 1] = first;
    };
    for (int t0 = 0; t0 < row.turns; t0 += 4) {   // four loads under way
      uint4 raw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t0 + i < row.turns) raw[i] = row.load(t0 + i);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t0 + i < row.turns) look(raw[i]);
    }
    m = fmaxf(fmaxf(group[0], group[1]), fmaxf(group[2], group[3]));
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const bool any_odd = __ballot(odd) != 0;
    if (lane == 0) {
      s.top[wave] = m;
      s.odd[wave] = any_odd;
    }
    if (tid == 0) s.n = 0;
    __syncthreads();
    odd = false;
    for (int i = 0; i < WAVES; ++i) {
      m = fmaxf(m, s.top[i]);
      odd |= s.odd[i] != 0;
    }
  }
  if (odd || m == -INFINITY) {
    if (tid == 0) answer(-1, odd ? NAN : 0.0f);
    return;
  }
  const float least = from_ordered(least_key(set, m));

  if (set.k > 0 && set.k <= LIST_K && set.k < a.V) {
    // the largest 16-bit prefix that at least k groups' maxima reach bounds the k-th largest logit from below
    uint32_t bound = 0;
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t next = bound | 1u << bit;
      int n = 0;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) n += (int)__popcll(__ballot(ordered(group[g]) >= next));
      int* b = s.count + (bit & 1) * WAVES;   // two buffers: one barrier a turn
      if (lane == 0) b[wave] = n;
      __syncthreads();
      n = 0;
      for (int i = 0; i < WAVES; ++i) n += b[i];
      if (n >= (int)set.k) bound = next;
    }
    const float low = from_ordered(max(bound, FIRST_LIVE));
    row.each([&](int t, const float (&x)[N]) {
      float top = x[0];
#pragma unroll
      for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
      if (!__any(top >= low)) return;
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (x[e] >= low) {
          const int i = atomicAdd(&s.n, 1);
          if (i < LIST) s.list[i] = place64(x[e], row.index(t, e));
        }
    });
    __syncthreads();
    const int n = s.n;
    if (n <= LIST) {   // all that is left to do concerns the list: ranks and sums of all pairs
      for (int i = tid; i < n; i += THREADS) s.hist[i] = units(x_of(s.list[i]), (double)m, c, S);
      __syncthreads();
      // what each thread's logits weigh with all above them (LIST / THREADS of a thread, one at least)
      constexpr int PER = (LIST + THREADS - 1) / THREADS;
      uint64_t upto[PER], mine = 0;
      int rank[PER];
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        const int i = tid + q * THREADS;
        upto[q] = 0;
        rank[q] = 0;
        if (i < n) {
          const uint64_t me = s.list[i];
          for (int j = 0; j < n; ++j) {
            const bool up = s.list[j] >= me;
            upto[q] += up ? s.hist[j] : 0;
            rank[q] += up ? 1 : 0;
          }
          if (rank[q] <= set.k) mine += s.hist[i];
        }
      }
      const uint64_t mass = block_total(s, mine);
      const uint64_t wanted = set.p < 1.0 ? share_up(set.p, mass) : mass;
      mine = 0;
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        const int i = tid + q * THREADS;
        if (i < n) {
          const uint64_t w = s.hist[i];
          const bool kept = rank[q] <= set.k && (set.p >= 1.0 || upto[q] - w < wanted) &&
                            (x_of(s.list[i]) >= least || rank[q] == 1);
          rank[q] = kept;
          mine += kept ? w : 0;
        } else {
          rank[q] = 0;
        }
      }
      const uint64_t total = block_total(s, mine);   // (its barriers: everyone has read the weights)
      const uint64_t want = share_down(set.u, total) + 1;
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        const int i = tid + q * THREADS;
        if (i < n && !rank[q]) s.list[i] = 0;   // no place: what is not kept
      }
      if (tid == 0) s.index = a.V;
      __syncthreads();
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        const int i = tid + q * THREADS;
        if (i < n && rank[q]) {
          const uint64_t me = s.list[i];
          if (want == 1) {   // a share of nothing: the first symbol of any weight, though it be less than a unit
            if (((double)x_of(me) - (double)m) * c >= -1074.0) atomicMin(&s.index, v_of(me));
          } else {
            uint64_t sum = 0;
            for (int j = 0; j < n; ++j) sum += s.list[j] && v_of(s.list[j]) <= v_of(me) ? s.hist[j] : 0;
            if (sum >= want && sum - s.hist[i] < want) s.index = v_of(me);
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        const int i = tid + q * THREADS;
        if (i < n && rank[q] && v_of(s.list[i]) == s.index)
          answer(s.index, (float)(log2_of(total) - S - ((double)x_of(s.list[i]) - (double)m) * c));
      }
      return;
    }
  }
  if (by_count)
    cut = set.k == 1 ? Cut{m, 1}
                     : search<false>(row, s, cut, m, (float)fmin(40.0 / c, 3e38), c, S,
                                     [&](uint64_t) { return (uint64_t)set.k; }, nullptr);
  const bool by_least = set.least > 0.0;
  bool by_mass = set.p < 1.0 && !found;
  const float range = set.octaves * __builtin_amdgcn_rcpf((float)c);
  const auto drawn = [&](uint64_t all) { return share_down(set.u, all) + 1; };
  int index = 0;
  float z = 0.0f;
  uint64_t total = 0;
  Pending pend{};
  bool done = false;
  // the cut is found while the kept are weighed: a look less (2048 rows of 32768 fp32: 157 us, 177 without), but not where a
  // look is cheap or counts find it as a rule
  if constexpr (!KEEP && TYPE != RENO_T_BF16)
    if (by_mass && !by_least) {
      Cut last = search<true>(row, s, cut, m, range, c, S, share, &pend);
      if (pend.on) done = pick<true>(row, s, last, pend, (double)m, c, S, drawn, &index, &z, &total);
      if (done || !pend.on) cut = last;
      by_mass = pend.on && !done;
    }
  if (!done) {
    if (by_mass) cut = search<true>(row, s, cut, m, range, c, S, share, nullptr);
    if (by_least && least > cut.x) cut = Cut{least, ALL};
    pick<false>(row, s, cut, pend, (double)m, c, S, drawn, &index, &z, &total);
  }
  if (share_down(set.u, total) == 0) {   // a share of nothing: the first symbol of any weight, though it be less than a unit
    const bool whole = cut.ties == ALL;   // (the cut's own weight is a unit at least, or it is none by mass)
    int first = a.V;
    row.each([&](int t, const float (&x)[N]) {
#pragma unroll
      for (int e = N - 1; e >= 0; --e)
        if ((x[e] > cut.x || (whole && x[e] == cut.x)) && ((double)x[e] - (double)m) * c >= -1074.0)
          first = min(first, row.index(t, e));
    });
    if (!whole && ((double)cut.x - (double)m) * c >= -1074.0) {
      // the first that equals the cut is kept
      row.each([&](int t, const float (&x)[N]) {
#pragma unroll
        for (int e = N - 1; e >= 0; --e)
          if (x[e] == cut.x) first = min(first, row.index(t, e));
      });
    }
    __syncthreads();
    if (tid == 0) s.index = a.V;
    __syncthreads();
    atomicMin(&s.index, first);
    __syncthreads();
    index = s.index;
    z = logit<TYPE>(row.z, index);
  }
  if (tid == 0) answer(index, (float)(log2_of(total) - S - ((double)z - (double)m) * c));
}

template <int TYPE>
void run(const SampleArgs& a, int64_t rows, hipStream_t st) {
  if (a.V <= 16 * SHORT_LANE) {
    const dim3 grid((unsigned)((rows + 4 * SHORT_ROWS - 1) / (4 * SHORT_ROWS)));
    const auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a, rows); };
    if (a.V <= 16) go(k_sample_short<TYPE, 1>);
    else if (a.V <= 64) go(k_sample_short<TYPE, 4>);
    else go(k_sample_short<TYPE, 16>);
    return;
  }
  const int pieces = (a.V + Vec<TYPE>::N - 1) / Vec<TYPE>::N;
  const auto go = [&](auto kern, int threads, bool keep) {
    const int turns = (pieces + threads - 1) / threads;
    const unsigned lds = (unsigned)sizeof(Turn) * turns * (threads / 64) + (keep ? 16 * turns * threads : 0);
    hipLaunchKernelGGL(kern, dim3((unsigned)rows), dim3(threads), lds, st, a);
  };
  // Threads of a row.  With rows for every CU several blocks share one, and fewer threads wait less for one another
  // (2048 rows of 32768 fp32, top_p, with 128, 256, 512, 1024: 181, 170, 157, 233 us; 8192 of 4096: 105, 98, 144, 338);
  // else a row is as quick as its threads are many (64 rows of 50021 fp16: 113, 65, 46, 40), and is kept where it fits
  // (39; with a mask 40 against 46).
  int threads = pieces <= 128 ? 64 : pieces <= 512 ? 128 : pieces <= 4096 ? 256 : 512;
  if (rows <= 256)
    while (threads < 1024 && threads * 2 < pieces) threads *= 2;
  switch (threads) {
    case 64: go(k_sample_long<TYPE, 64, false>, 64, false); break;
    case 128: go(k_sample_long<TYPE, 128, false>, 128, false); break;
    case 256: go(k_sample_long<TYPE, 256, false>, 256, false); break;
    case 512: go(k_sample_long<TYPE, 512, false>, 512, false); break;
    default:
      if (pieces <= 8 * 1024) go(k_sample_long<TYPE, 1024, true>, 1024, true);   // 128 of 160 KB
      else go(k_sample_long<TYPE, 1024, false>, 1024, false);
  }
}

}  // namespace

hipError_t launch_sample(const reno_sample& p, const void* logits, const float* u, int32_t* symbol, float* bits,
                         hipStream_t st) {
  // a row is given up to 1024 threads
  for (int64_t r = 0; r < p.rows; r += LAUNCH_ROWS / 4) {
    const int64_t n = std::min(LAUNCH_ROWS / 4, p.rows - r);
    SampleArgs a;
    a.z = static_cast<const char*>(logits) + r * p.row_stride * (p.type == RENO_T_FP32 ? 4 : 2);
    a.stride = p.row_stride;
    a.V = p.symbols;
    a.S = unit_bits(p.symbols);
    a.T = p.temperature;
    a.c = a.T > 0.0 ? LOG2E_D / a.T : 0.0;
    a.octaves = octaves_of(a.V, p.top_p);
    a.log_least = p.min_p > 0.0 ? std::log(p.min_p) : 0.0;
    a.p = p.top_p;
    a.least = p.min_p;
    a.k = p.top_k;
    a.T_rows = p.temperature_rows ? p.temperature_rows + r : nullptr;
    a.p_rows = p.top_p_rows ? p.top_p_rows + r : nullptr;
    a.least_rows = p.min_p_rows ? p.min_p_rows + r : nullptr;
    a.k_rows = p.top_k_rows ? p.top_k_rows + r : nullptr;
    a.allowed = p.allowed ? p.allowed + r * p.allowed_stride : nullptr;
    a.allowed_stride = p.allowed_stride;
    a.u = u + r;
    a.symbol = symbol + r;
    a.bits = bits + r;
    switch (p.type) {
      case RENO_T_FP32: run<RENO_T_FP32>(a, n, st); break;
      case RENO_T_BF16: run<RENO_T_BF16>(a, n, st); break;
      default: run<RENO_T_FP16>(a, n, st);
    }
  }
  return hipGetLastError();
}

}  // namespace reno
