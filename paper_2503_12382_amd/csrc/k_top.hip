// The k largest logits of each row with the row's normaliser (reno_head.h).
//
// A logit's order and its index are one 64-bit key: the float's bits as an
// integer that sorts the same way (NaN above everything, -0 with +0), then the
// index complemented, so that the largest key is the largest logit of the
// lowest index and no two keys are equal.  Bound by the one read of the logits
// as long as a row's selection costs fewer instructions than its bytes take:
//   k_top_short  rows of up to 256: 16 lanes a row, so that one wave's
//                instructions serve four rows; every lane sorts its 16 logits
//                in registers, then the largest head of 16 sorted lists is
//                taken k times.  233737 x 256 fp32, k 16: 86 us, 3.1 TB/s; bound by its
//                some 650 instructions for four rows
//   k_top_long   a block a row.  The k-th largest of many groups' maxima bounds
//                the k-th largest logit from below, so a second look at the row
//                (from L2) keeps little more than k candidates, whose ranks are
//                counted; rows with too many equal logits for that are cut
//                exactly, by a radix selection.  Rows that fit the registers are
//                held there between the looks.  4096 x 32768 bf16, k 64: 72 us,
//                3.7 TB/s; one row of 131071 fp32: 23 us, the latency of one block

#include <algorithm>

#include "dev.h"
#include "head.h"
#include "head_dev.h"

namespace reno {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

template <int TYPE>
__device__ __forceinline__ float logit(const void* p, int64_t i) {
  if constexpr (TYPE == RENO_T_FP32) return static_cast<const float*>(p)[i];
  else if constexpr (TYPE == RENO_T_BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
  else return (float)static_cast<const _Float16*>(p)[i];
}

// logits of 16 bytes in memory
template <int TYPE>
struct Vec {
  static constexpr int N = TYPE == RENO_T_FP32 ? 4 : 8;
  typedef uint4 Raw;
  float x[N];
  __device__ static __forceinline__ uint4 raw(const void* p, int64_t i) {
    return *reinterpret_cast<const uint4*>(static_cast<const char*>(p) + i * (16 / N));
  }
  __device__ __forceinline__ void load(const void* p, int64_t i) { from(raw(p, i)); }
  __device__ __forceinline__ void from(uint4 v) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (TYPE == RENO_T_FP32) {
        x[e] = __uint_as_float(u[e]);
      } else if constexpr (TYPE == RENO_T_BF16) {
        x[2 * e] = __uint_as_float(u[e] << 16);
        x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
      } else {
        x[2 * e] = (float)__builtin_bit_cast(_Float16, (uint16_t)u[e]);
        x[2 * e + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(u[e] >> 16));
      }
    }
  }
};

// An unsigned integer in the order of the floats, from 1 (0: no logit).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  const uint32_t o = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return x != x ? 0xfffffffeu : o;
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
  if (o == 0xfffffffeu) return NAN;
  return o == 0 ? -INFINITY : __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t make_key(uint32_t o, uint32_t i) { return (uint64_t)o << 32 | (uint32_t)~i; }

// ---------------------------------------------------------------------------
// Rows of up to 256 logits.

constexpr int SHORT_LANE = 16;      // logits of a lane, lanes of a row
constexpr int SHORT_ROWS = 4;       // rows of a wave

__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
  v = max(v, dpp<0x128>(v));
  v = max(v, dpp<0x124>(v));
  v = max(v, dpp<0x122>(v));
  return max(v, dpp<0x121>(v));
}
__device__ __forceinline__ float row16_sum(float v) {
  v += __uint_as_float(dpp<0x128>(__float_as_uint(v)));
  v += __uint_as_float(dpp<0x124>(__float_as_uint(v)));
  v += __uint_as_float(dpp<0x122>(__float_as_uint(v)));
  return v + __uint_as_float(dpp<0x121>(__float_as_uint(v)));
}

// A lane sorts its logits as doubles from [1, 2), the ordered value over the index complemented in their
// fraction: a comparison of two is one maximum and one minimum instead of a 64-bit comparison and four selects.
__device__ __forceinline__ double sort_key(uint32_t o, int i) {
  return __builtin_bit_cast(double, 0x3ff0000000000000ull | (uint64_t)o << 20 | (uint32_t)(255 - i));
}
__device__ __forceinline__ uint32_t key_value(uint64_t k) { return (uint32_t)(k >> 20); }
__device__ __forceinline__ void sort_pair(double& a, double& b) {
  double hi, lo;
  asm("v_max_f64 %0, %1, %2" : "=v"(hi) : "v"(a), "v"(b));
  asm("v_min_f64 %0, %1, %2" : "=v"(lo) : "v"(a), "v"(b));
  a = hi;
  b = lo;
}

// PL: logits of a lane (a power of two, 16 PL >= V); a lane's are consecutive, so that of two lanes with
// equal heads the lower one holds the lower index.
template <int TYPE, int PL>
__global__ void __launch_bounds__(256) k_top_short(const void* __restrict__ z, int64_t rows, int V, int64_t stride, int k,
                                                   int32_t* __restrict__ index, float* __restrict__ value,
                                                   float* __restrict__ lse) {
  extern __shared__ uint64_t s_mem[];                      // for each wave: sorted lists, then the results
  const int lane = lane_id(), wave = threadIdx.x >> 6, l15 = lane & 15, rw = lane >> 4;
  const int64_t r0 = ((int64_t)blockIdx.x * 4 + wave) * SHORT_ROWS;
  if (r0 >= rows) return;
  const int64_t r = min(r0 + rw, rows - 1);
  const int64_t at = r * stride;
  const int v0 = l15 * PL;
  // a row of lanes for each of PL + 1 places, then [SHORT_ROWS][k] results
  const int lists = wave * ((PL + 1) * 64 + SHORT_ROWS * k), out = lists + (PL + 1) * 64;
  float x[PL];
  if (PL == SHORT_LANE && v0 + PL <= V) {
#pragma unroll
    for (int i = 0; i < PL; i += Vec<TYPE>::N) {
      Vec<TYPE> t;
      uint4 raw;   // one load, wherever the row starts (233737 x 255 fp32, k 16: 102 us; by elements 124)
      __builtin_memcpy(&raw, static_cast<const char*>(z) + (at + v0 + i) * (16 / Vec<TYPE>::N), 16);
      t.from(raw);
#pragma unroll
      for (int e = 0; e < Vec<TYPE>::N && i + e < PL; ++e) x[i + e] = t.x[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < PL; ++i) x[i] = logit<TYPE>(z, at + min(v0 + i, V - 1));   // past the row: not used
  }
  double key[PL];
#pragma unroll
  for (int i = 0; i < PL; ++i) key[i] = v0 + i < V ? sort_key(ordered(x[i]), v0 + i) : sort_key(0, 0);
  // a lane's list, largest first: odd-even merges of runs of p
#pragma unroll
  for (int p = 1; p < PL; p *= 2)
#pragma unroll
    for (int q = p; q >= 1; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < PL; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < PL && (i + j) / (2 * p) == (i + j + q) / (2 * p)) sort_pair(key[i + j], key[i + j + q]);
#pragma unroll
  for (int i = 0; i < PL; ++i) s_mem[lists + i * 64 + lane] = __builtin_bit_cast(uint64_t, key[i]);
  s_mem[lists + PL * 64 + lane] = __builtin_bit_cast(uint64_t, sort_key(0, 0));
  wave_lds_fence();
  if (lse) {
    const float m = from_ordered(row16_max(key_value(__builtin_bit_cast(uint64_t, key[0]))));
    const float base = exp_base(m);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < PL; ++i) s += v0 + i < V ? __builtin_amdgcn_exp2f((x[i] - base) * LOG2E) : 0.0f;
    s = row16_sum(s);
    if (l15 == 0 && r0 + rw < rows) lse[r] = m != m ? m : base + __builtin_amdgcn_logf(s) * LN2;
  }
  int place = 0;
  for (int j = 0; j < k; ++j) {
    const uint64_t head = s_mem[lists + place * 64 + lane];
    const uint32_t o = key_value(head);
    const uint32_t top = row16_max(o);
    const uint32_t tied = (uint32_t)(__ballot(o == top) >> (lane & 48)) & 0xffffu;
    const bool won = (tied & (0u - tied)) == 1u << l15;
    if (won) s_mem[out + rw * k + j] = head;
    place += won && place < PL ? 1 : 0;
  }
  wave_lds_fence();
  const int n = (int)min((int64_t)SHORT_ROWS, rows - r0) * k;
  for (int i = lane; i < n; i += 64) {
    const uint64_t h = s_mem[out + i];
    const uint32_t o = key_value(h);
    index[r0 * k + i] = o ? 255 - (int32_t)(h & 255) : -1;
    value[r0 * k + i] = from_ordered(o);
  }
}

// ---------------------------------------------------------------------------
// Longer rows: a block a row.

constexpr int LONG_CAP = 1024;      // candidates kept
constexpr int LONG_GROUPS = 4;      // groups of a thread

// A row as its 16-byte pieces and what lies before the first and after the last of them.
template <int TYPE, int THREADS>
struct LongRow {
  static constexpr int N = Vec<TYPE>::N;
  const void* z;
  int64_t at;
  int V, head, whole;   // logits before the pieces, pieces

  __device__ __forceinline__ LongRow(const void* z_, int64_t at_, int V_) : z(z_), at(at_), V(V_) {
    constexpr int SIZE = 16 / N;
    const uint32_t off = (uint32_t)((uintptr_t)z + (uint64_t)at * SIZE) & 15u;
    head = min(V, (int)((16u - off) & 15u) / SIZE);
    whole = (V - head) / N;
  }
  __device__ __forceinline__ Vec<TYPE> piece(int i) const {
    Vec<TYPE> t;
    t.load(z, at + head + (int64_t)i * N);
    return t;
  }
  // f(index, logit) for the logits outside the pieces (fewer than 2 N)
  template <typename F>
  __device__ __forceinline__ void rest(const F& f) const {
    const int tid = threadIdx.x, tail = head + whole * N;
    if (tid < head) f(tid, logit<TYPE>(z, at + tid));
    if (tid < V - tail) f(tail + tid, logit<TYPE>(z, at + tail + tid));
  }
  // f(index, logit) for every logit, in an order of its own
  template <typename F>
  __device__ __forceinline__ void each(const F& f) const {
    for (int i = threadIdx.x; i < whole; i += THREADS) {
      const Vec<TYPE> t = piece(i);
#pragma unroll
      for (int e = 0; e < N; ++e) f(head + i * N + e, t.x[e]);
    }
    rest(f);
  }
};

template <int THREADS>
__device__ __forceinline__ int block_count(int mine, int* s, int phase) {
  // sum of one value a wave; two buffers, so that one barrier a call is enough
  const int wave = threadIdx.x >> 6;
  int* b = s + (phase & 1) * (THREADS / 64);
  if (lane_id() == 0) b[wave] = mine;
  __syncthreads();
  int n = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) n += b[i];
  return n;
}

// Exact cut of a row: the k-th largest ordered value *cut and how many lie above it.
template <int TYPE, int THREADS>
__device__ void radix_cut(const LongRow<TYPE, THREADS>& row, int k, uint32_t* hist, uint32_t* found, uint32_t* cut,
                          int* above) {
  uint32_t prefix = 0;
  int want = k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += THREADS) hist[i] = 0;
    __syncthreads();
    row.each([&](int, float x) {
      const uint32_t o = ordered(x);
      if (shift == 24 || o >> (shift + 8) == prefix >> (shift + 8)) {
        const uint32_t bin = o >> shift & 255u;
        // equal logits fall into one bin: one add for all lanes that agree with the first
        const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane((int)bin);
        const uint64_t same = __ballot(bin == first);
        if (bin != first) atomicAdd(&hist[bin], 1u);
        else if (rank_below(same) == 0) atomicAdd(&hist[bin], (uint32_t)__popcll(same));
      }
    });
    __syncthreads();
    if (threadIdx.x == 0) {
      int left = want, b = 255;
      while (b > 0 && (int)hist[b] < left) left -= (int)hist[b--];
      found[0] = (uint32_t)b;
      found[1] = (uint32_t)left;
    }
    __syncthreads();
    prefix |= found[0] << shift;
    want = (int)found[1];
    __syncthreads();
  }
  *cut = prefix;
  *above = k - want;
}

// KEEP: pieces a thread holds between the two looks, where they fit (else 0: the row is read again).
template <int TYPE, int THREADS, int KEEP>
__global__ void __launch_bounds__(THREADS) k_top_long(const void* __restrict__ z, int V, int64_t stride, int k,
                                                      int32_t* __restrict__ index, float* __restrict__ value,
                                                      float* __restrict__ lse) {
  constexpr int WAVES = THREADS / 64, N = Vec<TYPE>::N;
  __shared__ uint64_t s_key[LONG_CAP];
  __shared__ uint32_t s_hist[256];
  __shared__ uint32_t s_found[2];
  __shared__ int s_sum[2 * WAVES];
  __shared__ float2 s_ms[WAVES];
  __shared__ int s_n;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const int64_t r = blockIdx.x;
  const LongRow<TYPE, THREADS> row(z, r * stride, V);
  if (tid == 0) s_n = 0;
  // one look: maxima of the thread's groups, running maximum and sum of exponentials
  uint32_t group[LONG_GROUPS] = {};
  float m = -INFINITY, s = 0.0f;
  const auto take = [&](const float (&x)[N], int n, uint32_t& g) {
    float top = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = e < n ? fmaxf(top, x[e]) : top;
    g = max(g, ordered(top));   // NaN beside a number does not count: it only lowers the bound
    const float next = fmaxf(m, top);
    const float base = exp_base(next);
    s *= __builtin_amdgcn_exp2f((m - base) * LOG2E);
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) s += __builtin_amdgcn_exp2f((x[e] - base) * LOG2E);
    m = next;
  };
  typename Vec<TYPE>::Raw kept[KEEP ? KEEP : 1];
  float piece_max[KEEP ? KEEP : 1];
  bool odd = false;   // the thread holds a NaN or +inf: its pieces' maxima do not tell
  if constexpr (KEEP > 0) {
#pragma unroll
    for (int u = 0; u < KEEP; ++u)
      if (tid + u * THREADS < row.whole) kept[u] = Vec<TYPE>::raw(z, row.at + row.head + (int64_t)(tid + u * THREADS) * N);
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
      piece_max[u] = -INFINITY;
      if (tid + u * THREADS < row.whole) {
        Vec<TYPE> t;
        t.from(kept[u]);
        float top = t.x[0];
#pragma unroll
        for (int e = 1; e < N; ++e) top = fmaxf(top, t.x[e]);
        piece_max[u] = top;
        group[u % LONG_GROUPS] = max(group[u % LONG_GROUPS], ordered(top));
        m = fmaxf(m, top);
      }
    }
    const float base = exp_base(m);
#pragma unroll
    for (int u = 0; u < KEEP; ++u)
      if (tid + u * THREADS < row.whole) {
        Vec<TYPE> t;
        t.from(kept[u]);
#pragma unroll
        for (int e = 0; e < N; ++e) s += __builtin_amdgcn_exp2f((t.x[e] - base) * LOG2E);
      }
    odd = !(s < INFINITY);
  } else {
    for (int i0 = tid; i0 < row.whole; i0 += LONG_GROUPS * THREADS) {
      Vec<TYPE> t[LONG_GROUPS];
#pragma unroll
      for (int u = 0; u < LONG_GROUPS; ++u)
        if (i0 + u * THREADS < row.whole) t[u] = row.piece(i0 + u * THREADS);
#pragma unroll
      for (int u = 0; u < LONG_GROUPS; ++u)
        if (i0 + u * THREADS < row.whole) take(t[u].x, N, group[u]);
    }
  }
  row.rest([&](int, float y) {
    float x[N];
    x[0] = y;
    take(x, 1, group[0]);
  });
  // the row's normaliser
  for (int o = 32; o > 0; o >>= 1) {
    const float om = __shfl_xor(m, o), os = __shfl_xor(s, o);
    const float next = fmaxf(m, om), base = exp_base(next);
    s = s * __builtin_amdgcn_exp2f((m - base) * LOG2E) + os * __builtin_amdgcn_exp2f((om - base) * LOG2E);
    m = next;
  }
  if (lane == 0) s_ms[wave] = make_float2(m, s);
  __syncthreads();
  if (tid == 0 && lse) {
    for (int i = 1; i < WAVES; ++i) {
      const float2 o = s_ms[i];
      const float next = fmaxf(m, o.x), base = exp_base(next);
      s = s * __builtin_amdgcn_exp2f((m - base) * LOG2E) + o.y * __builtin_amdgcn_exp2f((o.x - base) * LOG2E);
      m = next;
    }
    const float base = exp_base(m);
    lse[r] = base + __builtin_amdgcn_logf(s) * LN2;
  }
  // the largest 16-bit prefix that at least k groups' maxima reach (0 where there are fewer groups)
  uint32_t cut = 0;
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t next = cut | 1u << bit;
    int n = 0;
#pragma unroll
    for (int u = 0; u < LONG_GROUPS; ++u) n += (int)__popcll(__ballot(group[u] >= next));
    if (block_count<THREADS>(n, s_sum, bit) >= k) cut = next;
  }
  cut = max(cut, 1u);
  const float cut_x = from_ordered(cut);
  const auto collect = [&](int v, float x) {
    if (!(x < cut_x)) {   // NaN too
      const int i = atomicAdd(&s_n, 1);
      if (i < LONG_CAP) s_key[i] = make_key(ordered(x), (uint32_t)v);
    }
  };
  if constexpr (KEEP > 0) {
#pragma unroll
    for (int u = 0; u < KEEP; ++u)
      if (tid + u * THREADS < row.whole && (odd || !(piece_max[u] < cut_x))) {
        Vec<TYPE> t;
        t.from(kept[u]);
#pragma unroll
        for (int e = 0; e < N; ++e) collect(row.head + (tid + u * THREADS) * N + e, t.x[e]);
      }
    row.rest(collect);
  } else {
    row.each(collect);
  }
  __syncthreads();
  int n = s_n;
  if (n > LONG_CAP) {  // equal logits past the cut: what lies above the exact one, and the first that equal it
    __syncthreads();
    int above;
    radix_cut(row, k, s_hist, s_found, &cut, &above);
    if (tid == 0) s_n = 0;
    __syncthreads();
    row.each([&](int v, float x) {
      const uint32_t o = ordered(x);
      if (o > cut) s_key[atomicAdd(&s_n, 1)] = make_key(o, (uint32_t)v);
    });
    int have = above;
    for (int v0 = 0, phase = 0; v0 < V && have < k; v0 += THREADS, ++phase) {
      const int v = v0 + tid;
      const bool eq = v < V && ordered(logit<TYPE>(z, row.at + v)) == cut;
      const uint64_t b = __ballot(eq);
      const int before_all = block_count<THREADS>((int)__popcll(b), s_sum, phase);
      int before = 0;
      for (int i = 0; i < wave; ++i) before += s_sum[(phase & 1) * WAVES + i];
      const int at = have + before + (int)rank_below(b);
      if (eq && at < k) s_key[at] = make_key(cut, (uint32_t)v);
      have += before_all;
    }
    __syncthreads();
    n = k;
  }
  // ranks among the candidates
  for (int i = tid; i < n; i += THREADS) {
    const uint64_t mine = s_key[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += s_key[j] > mine ? 1 : 0;
    if (rank < k) {
      index[r * k + rank] = (int32_t)~(uint32_t)mine;
      value[r * k + rank] = from_ordered((uint32_t)(mine >> 32));
    }
  }
  for (int j = n + tid; j < k; j += THREADS) {
    index[r * k + j] = -1;
    value[r * k + j] = -INFINITY;
  }
}

template <int TYPE>
void run(const void* z, int64_t rows, int V, int64_t stride, int k, int32_t* index, float* value, float* lse,
         hipStream_t st) {
  if (V <= 16 * SHORT_LANE) {
    const dim3 grid((unsigned)((rows + 4 * SHORT_ROWS - 1) / (4 * SHORT_ROWS)));
    const auto args = [&](auto kern, int pl) {
      const unsigned lds = 4 * 8 * ((pl + 1) * 64 + SHORT_ROWS * k);   // 52 KB at most
      hipLaunchKernelGGL(kern, grid, dim3(256), lds, st, z, rows, V, stride, k, index, value, lse);
    };
    if (V <= 16) args(k_top_short<TYPE, 1>, 1);
    else if (V <= 64) args(k_top_short<TYPE, 4>, 4);
    else args(k_top_short<TYPE, 16>, 16);
    return;
  }
  const dim3 grid((unsigned)rows);
  const auto args = [&](auto kern, int threads) {
    hipLaunchKernelGGL(kern, grid, dim3(threads), 0, st, z, V, stride, k, index, value, lse);
  };
  // threads: about 32 logits each or more, so that the groups outnumber k; a row of up to 16 pieces a thread is kept
  const int whole = V / Vec<TYPE>::N;
  if (V <= 2048) args(k_top_long<TYPE, 64, 8>, 64);
  else if (whole <= 8 * 256) args(k_top_long<TYPE, 256, 8>, 256);
  else if (whole <= 16 * 256) args(k_top_long<TYPE, 256, 16>, 256);
  else if (whole <= 16 * 1024) args(k_top_long<TYPE, 1024, 16>, 1024);
  else args(k_top_long<TYPE, 1024, 0>, 1024);
}

}  // namespace

hipError_t launch_top(const void* z, int type, int64_t rows, int V, int64_t stride, int k, int32_t* index, float* value,
                      float* lse, hipStream_t st) {
  // a row is given up to 1024 threads
  for (int64_t r = 0; r < rows; r += LAUNCH_ROWS / 4) {
    const int64_t n = std::min(LAUNCH_ROWS / 4, rows - r);
    const char* x = static_cast<const char*>(z) + r * stride * (type == RENO_T_FP32 ? 4 : 2);
    int32_t* ix = index + r * k;
    float *v = value + r * k, *l = lse ? lse + r : nullptr;
    switch (type) {
      case RENO_T_FP32: run<RENO_T_FP32>(x, n, V, stride, k, ix, v, l, st); break;
      case RENO_T_BF16: run<RENO_T_BF16>(x, n, V, stride, k, ix, v, l, st); break;
      default: run<RENO_T_FP16>(x, n, V, stride, k, ix, v, l, st);
    }
  }
  return hipGetLastError();
}

}  // namespace reno
