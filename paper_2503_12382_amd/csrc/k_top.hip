// The k largest logits of each row with the row's normaliser (reno_head.h).
//
// A logit's order and its index are one 64-bit key: the float's bits as an
// integer that sorts the same way (NaN above everything), then the index
// complemented, so that the largest key is the largest logit of the lowest
// index and no two keys are equal.

#include <algorithm>

#include "dev.h"
#include "head.h"

namespace reno {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

template <int TYPE>
__device__ __forceinline__ float logit(const void* p, int64_t i) {
  if constexpr (TYPE == RENO_T_FP32) return static_cast<const float*>(p)[i];
  else if constexpr (TYPE == RENO_T_BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
  else return (float)static_cast<const _Float16*>(p)[i];
}

// An unsigned integer in the order of the floats: all NaN on top, -0 with +0.
__device__ __forceinline__ uint32_t ordered(float x) {
  if (x != x) return 0xfffffffeu;  // below the key of nothing, all ones
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t i) { return (uint64_t)ordered(x) << 32 | (uint32_t)~i; }

__device__ __forceinline__ uint64_t wave_max64(uint64_t v) {
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t w = __shfl_xor(v, o);
    v = w > v ? w : v;
  }
  return v;
}

// One wave a row: k times the largest key below the last one.
template <int TYPE>
__global__ void __launch_bounds__(256) k_top_scan(const void* __restrict__ z, int64_t rows, int V, int64_t stride, int k,
                                                  int32_t* __restrict__ index, float* __restrict__ value,
                                                  float* __restrict__ lse) {
  const int lane = lane_id();
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const int64_t at = r * stride;
  uint64_t below = ~uint64_t(0);
  float first = 0.0f;
  for (int j = 0; j < k; ++j) {
    uint64_t best = 0;
    for (int v = lane; v < V; v += 64) {
      const uint64_t key = key_of(logit<TYPE>(z, at + v), (uint32_t)v);
      if (key < below && key > best) best = key;
    }
    best = wave_max64(best);
    const uint32_t i = ~(uint32_t)best;
    const bool have = best != 0;
    const float x = have ? logit<TYPE>(z, at + i) : -INFINITY;
    if (lane == 0) {
      index[r * k + j] = have ? (int32_t)i : -1;
      value[r * k + j] = x;
    }
    if (j == 0) first = x;
    below = best;
  }
  if (!lse) return;
  const float base = first > -INFINITY ? first : 0.0f;
  float s = 0.0f;
  for (int v = lane; v < V; v += 64) s += __builtin_amdgcn_exp2f((logit<TYPE>(z, at + v) - base) * LOG2E);
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (lane == 0) lse[r] = base + __builtin_amdgcn_logf(s) * LN2;
}

template <int TYPE>
void run(const void* z, int64_t rows, int V, int64_t stride, int k, int32_t* index, float* value, float* lse,
         hipStream_t st) {
  hipLaunchKernelGGL(k_top_scan<TYPE>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, z, rows, V, stride, k, index,
                     value, lse);
}

}  // namespace

hipError_t launch_top(const void* z, int type, int64_t rows, int V, int64_t stride, int k, int32_t* index, float* value,
                      float* lse, hipStream_t st) {
  switch (type) {
    case RENO_T_FP32: run<RENO_T_FP32>(z, rows, V, stride, k, index, value, lse, st); break;
    case RENO_T_BF16: run<RENO_T_BF16>(z, rows, V, stride, k, index, value, lse, st); break;
    default: run<RENO_T_FP16>(z, rows, V, stride, k, index, value, lse, st);
  }
  return hipGetLastError();
}

}  // namespace reno
