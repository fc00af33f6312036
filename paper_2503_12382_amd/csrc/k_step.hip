// The step that follows a gradient (reno_step.h): sums of squares over a list of
// tensors, gradients scaled down to a norm, AdamW.
//
// Every launch takes up to LIST tensors, by value (a captured graph keeps them),
// in chunks of equal length, a block a chunk; a block finds its tensor by one
// comparison a lane.  Loads and stores of 16 bytes wherever a tensor starts,
// several in flight a lane; bound by their bytes:
//   k_squares, k_norm  two launches.  2048 x 65536 + 65536 bf16: 48 and 5 us,
//                      5.6 TB/s in the first; 40 where the gradients lie in the
//                      memory side cache in part
//   k_clip             1000 x 50021 + 50021 fp16: 32 us, 6.3 TB/s (read from the
//                      memory side cache, where the norm left them); 8.3e6
//                      fp32: 10 us
//   k_adamw            1.3e8 bf16 weights with fp32 copies: 694 us, 5.4 TB/s;
//                      8.3e6 fp32: 41 us, 5.6 TB/s; 1e5 fp32: 7 us, latency
// Times: the mean of many calls in a row.

#include <algorithm>
#include <cmath>

#include "dev.h"
#include "step.h"

namespace reno {
namespace {

constexpr int LIST = 64;          // tensors of a launch: their places are compared by one wave
constexpr int THREADS = 256;

// Elements of a chunk for so many in all.
// (4096 blocks at most, as long as they are short: a list of 1.3e8 weights takes as long with 1024 and 8192.)
int64_t chunk_of(int64_t total) {
  int64_t c = 4096;
  while (total / c > 4096 && c < 1 << 24) c *= 2;
  return c;
}

// Where a block works: tensor i of the launch, its elements from `at`, `n` of them.
struct Place {
  int i, n;
  int64_t at;
};

struct Starts {
  uint32_t first[LIST];   // first block of each tensor; those past the list: past the grid
};

__device__ __forceinline__ Place place(const Starts& s, const int64_t* sizes, uint32_t chunk) {
  const uint32_t b = blockIdx.x;
  const int i = (int)__popcll(__ballot(s.first[lane_id()] <= b)) - 1;
  Place p;
  p.i = i;
  p.at = (int64_t)(b - s.first[i]) * chunk;
  p.n = (int)min((int64_t)chunk, sizes[i] - p.at);
  return p;
}

// N elements in memory, wherever they start, and as floats.
template <int TYPE, int N>
struct Piece {
  static constexpr int SIZE = TYPE == RENO_T_FP32 ? 4 : 2, WORDS = N * SIZE / 4;
  uint32_t u[WORDS];
  __device__ __forceinline__ void load(const void* p, int64_t i) {
    __builtin_memcpy(u, static_cast<const char*>(p) + i * SIZE, N * SIZE);
  }
  // past the caches: what is read or written once a step (1.3e8 bf16 weights with copies: 765 us through them, 694 so)
  typedef uint32_t Words __attribute__((ext_vector_type(WORDS), aligned(SIZE)));
  __device__ __forceinline__ void stream_in(const void* p, int64_t i) {
    const Words w = __builtin_nontemporal_load(reinterpret_cast<const Words*>(static_cast<const char*>(p) + i * SIZE));
#pragma unroll
    for (int k = 0; k < WORDS; ++k) u[k] = w[k];
  }
  __device__ __forceinline__ void stream_out(void* p, int64_t i) const {
    Words w;
#pragma unroll
    for (int k = 0; k < WORDS; ++k) w[k] = u[k];
    __builtin_nontemporal_store(w, reinterpret_cast<Words*>(static_cast<char*>(p) + i * SIZE));
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (TYPE == RENO_T_FP32) return __uint_as_float(u[e]);
    else if constexpr (TYPE == RENO_T_BF16) return __uint_as_float(e & 1 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)(u[e / 2] >> (16 * (e & 1))));
  }
};

__device__ __forceinline__ uint16_t to_bf16(float x) {
  const uint32_t u = __float_as_uint(x);
  return x != x ? (uint16_t)(u >> 16 | 0x40u) : (uint16_t)((u + 0x7fffu + (u >> 16 & 1u)) >> 16);
}
template <int TYPE, int N>
__device__ __forceinline__ Piece<TYPE, N> pack(const float (&x)[N]) {
  Piece<TYPE, N> p;
  if constexpr (TYPE == RENO_T_FP32) {
#pragma unroll
    for (int e = 0; e < N; ++e) p.u[e] = __float_as_uint(x[e]);
  } else {
    uint16_t h[N];
#pragma unroll
    for (int e = 0; e < N; ++e)
      h[e] = TYPE == RENO_T_BF16 ? to_bf16(x[e]) : __builtin_bit_cast(uint16_t, (_Float16)x[e]);
#pragma unroll
    for (int e = 0; e < N; e += 2) p.u[e / 2] = h[e] | (uint32_t)h[e + 1] << 16;
  }
  return p;
}
template <int TYPE>
__device__ __forceinline__ float get1(const void* p, int64_t i) {
  if constexpr (TYPE == RENO_T_FP32) return static_cast<const float*>(p)[i];
  else if constexpr (TYPE == RENO_T_BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
  else return (float)static_cast<const _Float16*>(p)[i];
}
template <int TYPE>
__device__ __forceinline__ void put1(void* p, int64_t i, float x) {
  if constexpr (TYPE == RENO_T_FP32) static_cast<float*>(p)[i] = x;
  else if constexpr (TYPE == RENO_T_BF16) static_cast<uint16_t*>(p)[i] = to_bf16(x);
  else static_cast<_Float16*>(p)[i] = (_Float16)x;
}

// ---------------------------------------------------------------------------
// Norm.  Squares in 64 bits: those of any fp32 value fit, so that neither large
// nor small gradients leave the range, and 2^40 of them lose nothing that fp32
// shows.  A chunk's sum a block, the chunks' sums in order by one block.

struct NormList {
  Starts s;
  int64_t n[LIST];
  const void* p[LIST];
  uint8_t type[LIST];
};

template <int TYPE>
__device__ __forceinline__ double squares(const void* p, int64_t at, int n) {
  constexpr int N = TYPE == RENO_T_FP32 ? 4 : 8, U = 4;
  double s[2] = {0.0, 0.0};
  const int whole = n / N;
  for (int i0 = threadIdx.x; i0 < whole; i0 += U * THREADS) {
    Piece<TYPE, N> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * THREADS < whole) x[u].load(p, at + (int64_t)(i0 + u * THREADS) * N);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * THREADS < whole)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const double v = (double)x[u].get(e);
          s[e & 1] = __builtin_fma(v, v, s[e & 1]);
        }
  }
  for (int i = whole * N + threadIdx.x; i < n; i += THREADS) {
    const double v = (double)get1<TYPE>(p, at + i);
    s[0] = __builtin_fma(v, v, s[0]);
  }
  return s[0] + s[1];
}

// Sum of a value a thread, in thread 0.
template <int T>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double s[T / 64];
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if (lane_id() == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
  if (threadIdx.x == 0)
    for (int i = 0; i < T / 64; ++i) t += s[i];
  return t;
}

__global__ void __launch_bounds__(THREADS) k_squares(NormList l, uint32_t chunk, double* __restrict__ parts) {
  const Place w = place(l.s, l.n, chunk);
  const void* p = l.p[w.i];
  const int type = l.type[w.i];
  double s;
  if (type == RENO_T_FP32) s = squares<RENO_T_FP32>(p, w.at, w.n);
  else if (type == RENO_T_BF16) s = squares<RENO_T_BF16>(p, w.at, w.n);
  else s = squares<RENO_T_FP16>(p, w.at, w.n);
  s = block_sum<THREADS>(s);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

__global__ void __launch_bounds__(1024) k_norm(const double* __restrict__ parts, int64_t n, double scale,
                                               float* __restrict__ norm) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += parts[i];
  s = block_sum<1024>(s);
  if (threadIdx.x == 0) *norm = (float)(scale * __builtin_sqrt(s));
}

// What gradients are multiplied by, scale min(1, max_norm / norm), as a float and a power of two for what passes the
// floats' range: the factor may lie outside it where the product does not.  The power goes first, which rounds nothing
// (what it makes subnormal the float, 2^-126 then, makes 0), so that the product is rounded once, subnormal or not.
// (In 64 bits its conversions bound clipping: 5e7 fp16 gradients took 56 us, 31 so.)
struct Factor {
  float f;
  int exp;
  __device__ __forceinline__ float of(float g) const { return __builtin_amdgcn_ldexpf(g, exp) * f; }
};
__device__ __forceinline__ Factor factor(const float* norm, double scale, double max_norm) {
  const double n = norm ? (double)*norm : 0.0;
  const double f = n <= max_norm ? scale : scale * (max_norm / n);
  const int e = __builtin_amdgcn_frexp_exp(f), in = min(max(e, -125), 127);
  return Factor{(float)__builtin_ldexp(__builtin_amdgcn_frexp_mant(f), in), e - in};
}

// ---------------------------------------------------------------------------
// Clipping.

struct ClipList {
  Starts s;
  int64_t n[LIST];
  const void* p[LIST];
  void* out[LIST];
  uint8_t type[LIST];
};

template <int TYPE>
__device__ __forceinline__ void scale_to(const void* p, void* out, int64_t at, int n, Factor f) {
  constexpr int N = TYPE == RENO_T_FP32 ? 4 : 8, U = 4;
  const int whole = n / N;
  for (int i0 = threadIdx.x; i0 < whole; i0 += U * THREADS) {
    Piece<TYPE, N> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * THREADS < whole) x[u].load(p, at + (int64_t)(i0 + u * THREADS) * N);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * THREADS < whole) {
        float y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = f.of(x[u].get(e));
        pack<TYPE, N>(y).stream_out(out, at + (int64_t)(i0 + u * THREADS) * N);
      }
  }
  for (int i = whole * N + threadIdx.x; i < n; i += THREADS)
    put1<TYPE>(out, at + i, f.of(get1<TYPE>(p, at + i)));
}

__global__ void __launch_bounds__(THREADS) k_clip(ClipList l, uint32_t chunk, const float* norm, double scale,
                                                  double max_norm) {
  const Place w = place(l.s, l.n, chunk);
  const Factor f = factor(norm, scale, max_norm);
  const void* p = l.p[w.i];
  void* out = l.out[w.i];
  const int type = l.type[w.i];
  if (type == RENO_T_FP32) scale_to<RENO_T_FP32>(p, out, w.at, w.n, f);
  else if (type == RENO_T_BF16) scale_to<RENO_T_BF16>(p, out, w.at, w.n, f);
  else scale_to<RENO_T_FP16>(p, out, w.at, w.n, f);
}

// ---------------------------------------------------------------------------
// AdamW.

struct AdamList {
  Starts s;
  int64_t n[LIST];
  const void* grad[LIST];
  void* param[LIST];
  float* master[LIST];
  float *m[LIST], *v[LIST];
};

struct AdamHow {
  double lr, beta1, beta2, scale, max_norm;
  float eps, decay;
  const float *lr_factor, *norm;
  int32_t* steps;
  int last;   // the call's last launch counts the step
};

// b^t for t >= 0, by squares (relative error below t 2^-52)
__device__ __forceinline__ double power(double b, uint32_t t) {
  double r = 1.0;
  for (; t; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

// beta in two floats, and 1 - beta: of beta's first 24 bits alone and 1 - beta the sum is not 1, and a moment settles beside
// the mean that it stands for (exp_avg_sq by 1.3e-5 of it at 0.999, by 1.4e-3 at 0.99999).
struct Decay {
  float hi, lo, gain;
};
__device__ __forceinline__ Decay decay_of(double beta) {
  Decay d;
  d.hi = (float)beta;
  d.lo = (float)(beta - (double)d.hi);
  d.gain = (float)(1.0 - beta);
  return d;
}

struct AdamTerms {
  Factor f;   // the gradients'
  Decay b1, b2;
  float inv1, inv2, lr, eps, decay;

  __device__ __forceinline__ void update(float g0, float& m, float& v, float& w) const {
    const float g = f.of(g0);
    m = fmaf(b1.hi, m, fmaf(b1.gain, g, b1.lo * m));
    // (infinite: it stays so, whatever b2 would make of it, and the step is none; m inv1 might be infinite too)
    v = v == INFINITY ? v : fmaf(b2.hi, v, fmaf(b2.gain * g, g, b2.lo * v));
    const float step = m / (__builtin_sqrtf(v) * inv2 + eps) * inv1;
    w = fmaf(-lr, fmaf(decay, w, step), w);   // decay inside: 1 - lr decay would be rounded
  }
};

// A weight of 16 bits is the rounding of its copy as stored: without this the last product and sum are rounded to 16
// bits in one instruction, which differs where the copy lies halfway between two of them.
__device__ __forceinline__ void rounded(float& x) { asm("" : "+v"(x)); }

template <int PT, int GT, bool MASTER>
__global__ void __launch_bounds__(THREADS) k_adamw(AdamList l, uint32_t chunk, AdamHow h) {
  constexpr int N = 4, U = 2;
  __shared__ AdamTerms s_terms;
  if (h.norm && !(*h.norm <= 0x1.fffffep127f)) return;   // inf or NaN: the step is not made
  // terms that all elements share: one thread's work, 64-bit quotients and powers
  uint32_t t = 0;
  if (threadIdx.x == 0) {
    t = (uint32_t)h.steps[0] + 1u;
    AdamTerms a;
    a.f = factor(h.norm, h.scale, h.max_norm);
    a.b1 = decay_of(h.beta1);
    a.b2 = decay_of(h.beta2);
    a.inv1 = (float)(1.0 / (1.0 - power(h.beta1, t)));
    a.inv2 = (float)(1.0 / __builtin_sqrt(1.0 - power(h.beta2, t)));
    a.lr = (float)(h.lr * (h.lr_factor ? (double)*h.lr_factor : 1.0));
    a.eps = h.eps;
    a.decay = h.decay;
    s_terms = a;
  }
  __syncthreads();
  if (l.s.first[0] == 0) {   // a list without elements has one block, to count
    const AdamTerms a = s_terms;
    const Place pl = place(l.s, l.n, chunk);
    const void* gp = l.grad[pl.i];
    void* wp = MASTER ? (void*)l.master[pl.i] : l.param[pl.i];
    void* out = l.param[pl.i];
    float *mp = l.m[pl.i], *vp = l.v[pl.i];
    constexpr int WT = MASTER ? RENO_T_FP32 : PT;
    const int whole = pl.n / N;
    for (int i0 = threadIdx.x; i0 < whole; i0 += U * THREADS) {
      Piece<GT, N> g[U];
      Piece<WT, N> w[U];
      Piece<RENO_T_FP32, N> m[U], v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * THREADS < whole) {
          const int64_t i = pl.at + (int64_t)(i0 + u * THREADS) * N;
          g[u].stream_in(gp, i);
          m[u].stream_in(mp, i);
          v[u].stream_in(vp, i);
          w[u].stream_in(wp, i);
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * THREADS < whole) {
          const int64_t i = pl.at + (int64_t)(i0 + u * THREADS) * N;
          float x[N], y[N], z[N];
#pragma unroll
          for (int e = 0; e < N; ++e) {
            x[e] = m[u].get(e);
            y[e] = v[u].get(e);
            z[e] = w[u].get(e);
            a.update(g[u].get(e), x[e], y[e], z[e]);
            if constexpr (MASTER) rounded(z[e]);
          }
          pack<RENO_T_FP32, N>(x).stream_out(mp, i);
          pack<RENO_T_FP32, N>(y).stream_out(vp, i);
          if constexpr (MASTER) pack<RENO_T_FP32, N>(z).stream_out(wp, i);
          pack<PT, N>(z).stream_out(out, i);
        }
    }
    for (int j = whole * N + threadIdx.x; j < pl.n; j += THREADS) {
      const int64_t i = pl.at + j;
      float m = mp[i], v = vp[i], w = get1<WT>(wp, i);
      a.update(get1<GT>(gp, i), m, v, w);
      if constexpr (MASTER) rounded(w);
      mp[i] = m;
      vp[i] = v;
      if constexpr (MASTER) put1<RENO_T_FP32>(wp, i, w);
      put1<PT>(out, i, w);
    }
  }
  // The last block to come here knows that every other has read the count.  (No fence: nothing else is handed over,
  // and one would write this XCD's L2 back, for each block.  8.3e6 fp32 weights: 108 us with it, 39 without.)
  if (h.last && threadIdx.x == 0) {
    if (atomicAdd(&h.steps[1], 1) == (int)gridDim.x - 1) {
      h.steps[0] = (int32_t)t;
      h.steps[1] = 0;
    }
  }
}

// f(first, last entry, blocks) for each launch of a list; chunk: elements of a block.  fill(j, i): entry i is the
// launch's j-th.  Entries without elements are left out.
template <typename List, typename Fill, typename Launch>
void in_launches(int64_t count, const int64_t chunk, List& l, const Fill& fill, const Launch& launch) {
  int j = 0;
  uint32_t blocks = 0;
  const auto flush = [&] {
    for (int k = j; k < LIST; ++k) l.s.first[k] = UINT32_MAX;
    if (j) launch(blocks);
    j = 0;
    blocks = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const int64_t n = fill(j, i);
    if (n == 0) continue;
    l.n[j] = n;
    l.s.first[j++] = blocks;
    blocks += (uint32_t)((n + chunk - 1) / chunk);
    if (j == LIST) flush();
  }
  flush();
}

template <typename T>
int64_t total_of(const T* x, int64_t count) {
  int64_t n = 0;
  for (int64_t i = 0; i < count; ++i) n += x[i].n;
  return n;
}

template <int PT, int GT, bool MASTER>
void adamw_kind(const reno_parameter* p, int64_t count, int64_t chunk, const AdamHow& how, hipStream_t st, bool last) {
  AdamList l;
  // the entries of this kind that are left, so that the call's last launch is known
  const auto mine = [&](const reno_parameter& x) {
    return x.n && x.type == PT && x.grad_type == GT && (x.master != nullptr) == MASTER;
  };
  int64_t left = 0;
  for (int64_t i = 0; i < count; ++i) left += mine(p[i]);
  in_launches(
      count, chunk, l,
      [&](int j, int64_t i) -> int64_t {
        const reno_parameter& x = p[i];
        if (!mine(x)) return 0;
        l.grad[j] = x.grad;
        l.param[j] = x.param;
        l.master[j] = x.master;
        l.m[j] = x.exp_avg;
        l.v[j] = x.exp_avg_sq;
        --left;
        return x.n;
      },
      [&](uint32_t blocks) {
        AdamHow h = how;
        h.last = last && left == 0;
        hipLaunchKernelGGL((k_adamw<PT, GT, MASTER>), dim3(blocks), dim3(THREADS), 0, st, l, (uint32_t)chunk, h);
      });
}

}  // namespace

int64_t norm_parts(const reno_gradient* g, int64_t count) {
  const int64_t chunk = chunk_of(total_of(g, count));
  int64_t parts = 0;
  for (int64_t i = 0; i < count; ++i) parts += (g[i].n + chunk - 1) / chunk;
  return parts;
}

hipError_t launch_norm(const reno_gradient* g, int64_t count, double scale, float* norm, double* parts, hipStream_t st) {
  const int64_t chunk = chunk_of(total_of(g, count));
  NormList l;
  int64_t at = 0;
  in_launches(
      count, chunk, l,
      [&](int j, int64_t i) {
        l.p[j] = g[i].grad;
        l.type[j] = (uint8_t)g[i].type;
        return g[i].n;
      },
      [&](uint32_t blocks) {
        hipLaunchKernelGGL(k_squares, dim3(blocks), dim3(THREADS), 0, st, l, (uint32_t)chunk, parts + at);
        at += blocks;
      });
  hipLaunchKernelGGL(k_norm, dim3(1), dim3(1024), 0, st, parts, at, scale, norm);
  return hipGetLastError();
}

hipError_t launch_clip(const reno_gradient* g, int64_t count, const float* norm, double scale, double max_norm,
                       hipStream_t st) {
  const int64_t chunk = chunk_of(total_of(g, count));
  ClipList l;
  in_launches(
      count, chunk, l,
      [&](int j, int64_t i) {
        l.p[j] = g[i].grad;
        l.out[j] = g[i].out;
        l.type[j] = (uint8_t)g[i].type;
        return g[i].n;
      },
      [&](uint32_t blocks) {
        hipLaunchKernelGGL(k_clip, dim3(blocks), dim3(THREADS), 0, st, l, (uint32_t)chunk, norm, scale, max_norm);
      });
  return hipGetLastError();
}

hipError_t launch_adamw(const reno_parameter* p, int64_t count, const reno_adamw& how, hipStream_t st) {
  const int64_t chunk = chunk_of(total_of(p, count));
  AdamHow h{how.lr, how.beta1, how.beta2, how.scale, how.max_norm, (float)how.eps, (float)how.weight_decay,
            how.lr_factor, how.norm, how.steps, 0};
  typedef void (*Kind)(const reno_parameter*, int64_t, int64_t, const AdamHow&, hipStream_t, bool);
  struct {
    int type, grad;
    bool master;
    Kind run;
    bool any;
  } kinds[] = {{RENO_T_FP32, RENO_T_FP32, false, adamw_kind<RENO_T_FP32, RENO_T_FP32, false>, false},
               {RENO_T_BF16, RENO_T_BF16, false, adamw_kind<RENO_T_BF16, RENO_T_BF16, false>, false},
               {RENO_T_BF16, RENO_T_BF16, true, adamw_kind<RENO_T_BF16, RENO_T_BF16, true>, false},
               {RENO_T_BF16, RENO_T_FP32, false, adamw_kind<RENO_T_BF16, RENO_T_FP32, false>, false},
               {RENO_T_BF16, RENO_T_FP32, true, adamw_kind<RENO_T_BF16, RENO_T_FP32, true>, false},
               {RENO_T_FP16, RENO_T_FP16, false, adamw_kind<RENO_T_FP16, RENO_T_FP16, false>, false},
               {RENO_T_FP16, RENO_T_FP16, true, adamw_kind<RENO_T_FP16, RENO_T_FP16, true>, false},
               {RENO_T_FP16, RENO_T_FP32, false, adamw_kind<RENO_T_FP16, RENO_T_FP32, false>, false},
               {RENO_T_FP16, RENO_T_FP32, true, adamw_kind<RENO_T_FP16, RENO_T_FP32, true>, false}};
  int last = -1;
  for (int64_t i = 0; i < count; ++i)
    for (int k = 0; k < 9; ++k)
      if (p[i].n && p[i].type == kinds[k].type && p[i].grad_type == kinds[k].grad &&
          (p[i].master != nullptr) == kinds[k].master) {
        kinds[k].any = true;
        last = std::max(last, k);
      }
  for (int k = 0; k <= last; ++k)
    if (kinds[k].any) kinds[k].run(p, count, chunk, h, st, k == last);
  if (last < 0) {   // no elements: one block counts the step
    AdamList l;
    for (int j = 0; j < LIST; ++j) l.s.first[j] = UINT32_MAX;
    h.last = 1;
    hipLaunchKernelGGL((k_adamw<RENO_T_FP32, RENO_T_FP32, false>), dim3(1), dim3(THREADS), 0, st, l, (uint32_t)chunk, h);
  }
  return hipGetLastError();
}

}  // namespace reno
