// Device helpers that the kernels of the head's training operators share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "dev.h"
#include "gemm.h"

namespace reno {

constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_hw(float x) { return __builtin_amdgcn_logf(x); }

// What logits are taken off before their exponentials: the largest, where that is finite.  Without any logit the sum
// is 0 and the normaliser -inf; with one of +inf the sum is +inf, or NaN beside NaN.  (inf - inf would be NaN at
// once.  In this form k_narrow with gradients takes 119 us for 58711 x 128 x 256, as one median of three or as a
// comparison of |m| 123.5: the compiler then places the tiles' registers differently.)
__device__ __forceinline__ float exp_base(float m) { return m > -INFINITY ? fminf(m, 0x1.fffffep127f) : 0.0f; }

constexpr int GPARTS = 64;   // partial maxima of |g|, in the workspace

// e: the largest |g| of the rows that are taken is below 2^e and at least half of it (0 without weights, or with
// none but 0).  dz is carried over G = 2^e.
__device__ __forceinline__ int weight_exp(const float* gpart) {
  if (!gpart) return 0;
  float m = gpart[lane_id()];
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  return m == 0.0f ? 0 : __builtin_amdgcn_frexp_expf(m);
}

// What brings the sums of dz to gradients: 1 / (T ln 2), over 2^14 for fp16, as a number below 1 and a power of two.
// That power and G may each be past the floats where the gradient is not; they meet as integers.
struct OutScale {
  float mant;
  int exp;
};
inline OutScale out_scale(float temperature) {
  OutScale s;
  s.mant = (float)std::frexp(1.0 / (0.6931471805599453 * (double)temperature), &s.exp);
  return s;
}
__device__ __forceinline__ float scaled(float x, OutScale s) { return __builtin_amdgcn_ldexpf(x * s.mant, s.exp); }
__device__ __forceinline__ OutScale with_weights(OutScale s, const float* gpart) {
  s.exp += __builtin_amdgcn_readfirstlane(weight_exp(gpart));
  return s;
}

// The three bf16 planes of x: each takes the leading 8 bits of what is left, cut off, so that
// the parts add up to x exactly.  An infinity leaves NaN in the lower planes (inf - inf): products
// with it are NaN where fp32 might keep an infinity; NaN stays NaN.
__device__ __forceinline__ void split3(float x, uint16_t (&o)[3]) {
  const uint32_t u = __float_as_uint(x);
  const float r = x - __uint_as_float(u & 0xffff0000u);
  const uint32_t v = __float_as_uint(r);
  o[0] = (uint16_t)(u >> 16);
  o[1] = (uint16_t)(v >> 16);
  o[2] = (uint16_t)(__float_as_uint(r - __uint_as_float(v & 0xffff0000u)) >> 16);
}

// The planes of 8 values as three fragments.
__device__ __forceinline__ void split_any8(const float (&x)[8], s16x8 (&o)[3]) {
  uint32_t w[3][4];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    uint32_t p[3][2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const uint32_t u = __float_as_uint(x[e + q]);
      const float r = x[e + q] - __uint_as_float(u & 0xffff0000u);
      const uint32_t v = __float_as_uint(r);
      p[0][q] = u;
      p[1][q] = v;
      p[2][q] = __float_as_uint(r - __uint_as_float(v & 0xffff0000u));
    }
#pragma unroll
    for (int t = 0; t < 3; ++t) w[t][e / 2] = __builtin_amdgcn_perm(p[t][1], p[t][0], 0x07060302u);
  }
#pragma unroll
  for (int t = 0; t < 3; ++t) {
    const i32x4 v = {(int)w[t][0], (int)w[t][1], (int)w[t][2], (int)w[t][3]};
    o[t] = __builtin_bit_cast(s16x8, v);
  }
}

}  // namespace reno
