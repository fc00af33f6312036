// Rows of logits as the kernels that select among them read them: elements of
// any reno_type, 16 bytes of them, and their order as integers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "head.h"

namespace reno {

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

}  // namespace reno
