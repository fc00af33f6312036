// Narrow fp32 heads (C <= 128, V <= 256: the codec's own): code length and
// distillation with their gradients in one pass over the rows.
//
// A block takes 16 rows a wave at a time, all V logits of a row in the registers
// of 4 lanes: softmax statistics are two lane exchanges, and nothing of the
// logits goes to memory.  Every operand is three bf16 parts
// (24 bits), a product six terms of them (TERMS_FP32).
//   z   = W^T h     A: 16 symbols x 32 channels of W, B: 32 channels x 16 rows
//   dh  = W dz      the accumulator layout of z (row = lane & 15, symbols 4 (lane >> 4) + i
//                   of each 16) taken as it is for B: k runs over the symbols in that
//                   order, and W is read in the same one
//   dw  = h dz^T    k runs over rows, so dz crosses lanes through LDS, 32 symbols of
//                   all the block's rows at a time, and is read back transposed; each wave
//                   holds the sums of its own tiles of dw over all rows of the block
// W lies in LDS for C <= 32 (one copy serves both products: transposed reads
// for z, rows for dh); wider ones stream from L2, laid out as the lanes read them.
// The blocks' sums of dw and db are joined in a fixed order by k_narrow_join.
//
// Bound: matrix instructions (6 terms x 3 products: 35 % of the cycles at 233737 x
// 32 x 256) and the vector work of a logit (scaling, exponential, splitting:
// some 20 instructions, 45 %) overlap little, since the waves of a SIMD do the
// same at the same time; memory would allow several times the rate.  With all
// gradients 233737 x 32 x 256 takes 100 us, 58711 x 128 x 256 120 (of which the weights'
// way from L2 some 40; the matrix unit's share of either is 57), forward alone 37 and 38.  A distillation of 16 entries
// (58711 rows) takes 67 us at 32 channels, 102 at 64 and 232 at 128: its tiles of q and the logits that it keeps beside
// the sums do not fit the registers (71, 95 and 201 spilled; code length at 64 and 128 channels: 10 and 65).

#include <algorithm>

#include "dev.h"
#include "gemm.h"
#include "head.h"
#include "head_dev.h"

namespace reno {
namespace {

// Waves of a block.  C <= 32: two blocks of 4 waves a CU, so that one's products run during the other's
// vector work; wider heads, whose tiles of dw would not fit the registers of so few waves: one block of 8.
constexpr int waves_of(int ct) { return ct == 2 ? 4 : 8; }

struct NarrowArgs {
  int64_t N;
  int C, V, k;
  int64_t h_stride, w_stride;
  const float *h, *w, *b, *g;
  const int32_t* index;    // [N][k]
  const float* q;          // [N][k] joined probabilities, or null: one entry with 1
  const float* ent;
  const uint8_t* flag;
  float scale;             // log2(e) / T
  OutScale out_scale;      // 1 / (T ln 2)
  const float* gpart;      // partial maxima of |g| that dz is carried over, or null: as it is
  const uint16_t* wz;      // streamed W, in the order of use: fragments of 16 symbols x 32 channels for z,
  const uint16_t* wd;      // of 16 channels x 32 symbols for dh
  float *bits, *lse, *dh;
  float* part;             // [blocks][C + waves / 2][V]: dw, shares of db
};

// acc += the six terms of a b, the smallest first
__device__ __forceinline__ f32x4 mfma6(const s16x8 (&a)[3], const s16x8 (&b)[3], f32x4 acc) {
  acc = mfma<false>(a[2], b[0], acc);
  acc = mfma<false>(a[0], b[2], acc);
  acc = mfma<false>(a[1], b[1], acc);
  acc = mfma<false>(a[1], b[0], acc);
  acc = mfma<false>(a[0], b[1], acc);
  return mfma<false>(a[0], b[0], acc);
}

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ s16x8 read_tr(const char* lo, const char* hi) {
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)lo);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)hi);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ void store8(char* base, int lo, int hi, s16x8 x) {
  *reinterpret_cast<s16x4*>(base + lo) = __builtin_shufflevector(x, x, 0, 1, 2, 3);
  *reinterpret_cast<s16x4*>(base + hi) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
}

// Where the 8-byte piece p of row r lies, for rows of B bytes (64, or a multiple of 128): pieces change places
// by the row, so that neither a transposed read (4 pieces of 4 consecutive rows for each 16 lanes) nor one piece of
// 16 rows meets a bank twice.
// The low 4 (64-byte rows: 3) bits of p change with r mod 16 alone: 16 rows or 16 (8) pieces on are a constant away.
template <int B>
__device__ __forceinline__ int piece(int r, int p) {
  const int s = B == 64 ? (r >> 1 & 1) << 2 | (r >> 2 & 3) : (r & 3) << 2 | (r >> 2 & 3);
  return r * B + (p ^ s) * 8;
}

template <int CT, int VQ, bool GRAD, bool DENSE>
struct NarrowLds {
  static constexpr int NW = waves_of(CT), ROWS = 16 * NW, CP = 16 * CT;
  static constexpr bool W_HERE = CT == 2;
  static constexpr int W_PLANE = CP * VQ * 128, H_PLANE = ROWS * CP * 2, D_PLANE = ROWS * 64;
  static constexpr int W = 0, H = W + (W_HERE ? 3 * W_PLANE : 0), D = H + (GRAD ? 3 * H_PLANE : 0);
  // 32 symbols' dz; a block alone on its CU has two such buffers and half the barriers.  They also hold
  // the targets' probabilities while dz is made.
  static constexpr int D_BUF = 3 * D_PLANE, BUFS = GRAD && NW == 8 ? 2 : 1;
  static constexpr int B = D + (GRAD || DENSE ? BUFS * D_BUF : 0), BYTES = B + VQ * 64 * 4;
};

// DENSE: targets with probabilities (a distillation); the registers then keep the logits, whose
// exponentials are taken again for dz, so that no probability is too small for its bits.
template <int CT, int VQ, bool GRAD, bool DENSE>
__global__ void __launch_bounds__(64 * waves_of(CT), 2) k_narrow(NarrowArgs a) {
  using L = NarrowLds<CT, VQ, GRAD, DENSE>;
  constexpr int NB_WAVES = L::NW, NB_THREADS = 64 * NB_WAVES, NB_ROWS = L::ROWS;
  constexpr int CP = L::CP, KS = CP / 32, VT = 4 * VQ;
  __shared__ __attribute__((aligned(1024))) char lds[L::BYTES];
  const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float* s_bias = reinterpret_cast<float*>(lds + L::B);
  for (int i = tid; i < VQ * 64; i += NB_THREADS) s_bias[i] = i >= a.V ? -INFINITY : a.b ? a.b[i] * a.scale : 0.0f;
  if constexpr (L::W_HERE) {
    for (int i = tid; i < CP * VQ * 8; i += NB_THREADS) {  // 8 symbols of a channel
      const int c = i / (VQ * 8), v = i % (VQ * 8) * 8;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = c < a.C && v + e < a.V ? a.w[c * a.w_stride + v + e] : 0.0f;
      s16x8 p[3];
      split_any8(x, p);
#pragma unroll
      for (int t = 0; t < 3; ++t) store8(lds + L::W + t * L::W_PLANE, piece<VQ * 128>(c, v / 4), piece<VQ * 128>(c, v / 4 + 1), p[t]);
    }
  }
  __syncthreads();
  // What the loop over rows reads of W is the same every time, but does not fit the registers: with the lane and
  // the pointers opaque to the compiler it is not taken out of the loop (and spilled).
  // Streamed fragments come in the order of their use.
  int lane_w = lane;
  typedef const __attribute__((address_space(1))) s16x8* frag_ptr;   // stays a global pointer behind the asm
  frag_ptr pz = nullptr, pd = nullptr;
  const auto next = [](frag_ptr& p, s16x8 (&o)[3]) {
#pragma unroll
    for (int t = 0; t < 3; ++t) o[t] = p[t * 64];
    p += 192;
    asm volatile("" : "+v"(p));
  };
  // LDS places: W for z (4 symbol groups, channels c and c + 4) and for dh, dz and h as written and as read back
  int az[4][2], ad[2][2], dw_at[2], dr_at[2], hw_at[2], hr_at[2];
  const int my_v = wave & 1, my_c = wave >> 1;   // this wave's tiles of dw: 16 of 32 symbols, every (NW / 2)th 16 channels
  {
    const int c = 8 * g + (l15 >> 2), r = 16 * wave + l15;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int q = 0; q < 2; ++q) az[i][q] = L::W + piece<VQ * 128>(c + 4 * q, 4 * i + (l15 & 3));
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int q = 0; q < 2; ++q) ad[i][q] = L::W + piece<VQ * 128>(l15, 8 * i + 4 * q + g);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      dw_at[q] = L::D + piece<64>(r, 4 * q + g);
      dr_at[q] = L::D + piece<64>(c + 4 * q, 4 * my_v + (l15 & 3));
      hw_at[q] = L::H + piece<CP * 2>(r, 2 * g + q);
      hr_at[q] = L::H + piece<CP * 2>(c + 4 * q, 4 * my_c + (l15 & 3));
    }
  }
  // fragments of W: 16 symbols x 32 channels (z), and 16 channels x 32 symbols in the order of z's registers (dh)
  const auto frag_z = [&](int vt, int ks, s16x8 (&o)[3]) {
    if constexpr (L::W_HERE) {
      const char* p0 = lds + az[vt & 3][0] + (32 * ks * VQ * 128 + (vt >> 2) * 128);
      const char* p1 = lds + az[vt & 3][1] + (32 * ks * VQ * 128 + (vt >> 2) * 128);
#pragma unroll
      for (int t = 0; t < 3; ++t) o[t] = read_tr(p0 + t * L::W_PLANE, p1 + t * L::W_PLANE);
    } else {
      next(pz, o);
    }
  };
  const auto frag_d = [&](int u, int ct, s16x8 (&o)[3]) {
    if constexpr (L::W_HERE) {
      const char* p0 = lds + ad[u & 1][0] + (16 * ct * VQ * 128 + (u >> 1) * 128);
      const char* p1 = lds + ad[u & 1][1] + (16 * ct * VQ * 128 + (u >> 1) * 128);
#pragma unroll
      for (int t = 0; t < 3; ++t) {
        const s16x4 lo = *reinterpret_cast<const s16x4*>(p0 + t * L::W_PLANE);
        const s16x4 hi = *reinterpret_cast<const s16x4*>(p1 + t * L::W_PLANE);
        o[t] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    } else {
      next(pd, o);
    }
  };

  constexpr int DB = NB_WAVES / 2, DW_N = CT / DB, U = 2 * VQ;
  f32x4 dw[GRAD ? U : 1][DW_N], db[(U + 3) / 4];   // db of u: the lanes with lane >> 4 = u & 3
  if constexpr (GRAD) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      db[i / 4] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < DW_N; ++j) dw[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  const int g_exp = GRAD ? __builtin_amdgcn_readfirstlane(weight_exp(a.gpart)) : 0;
  const OutScale out_scale{a.out_scale.mant, a.out_scale.exp + g_exp};
  const int64_t steps = (a.N + NB_ROWS - 1) / NB_ROWS;
  // this lane's piece of its row: channels 32 ks + 8 g .. + 7
  float x[KS][8];
  const auto load_h = [&](int64_t step) {
    const int64_t r = step * NB_ROWS + 16 * wave + l15;
    const bool in = r < a.N;
    const float* p = a.h + r * a.h_stride;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int c = 32 * ks + 8 * g;
      if (in && c + 8 <= a.C) {
        __builtin_memcpy(x[ks], p + c, 32);   // two loads, wherever the row starts
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[ks][e] = in && c + e < a.C ? p[c + e] : 0.0f;
      }
    }
  };
  constexpr bool AHEAD = CT < 8;   // rows of the next step are loaded early where registers are left
  if (AHEAD && (int64_t)blockIdx.x < steps) load_h(blockIdx.x);
  for (int64_t step = blockIdx.x; step < steps; step += gridDim.x) {
    asm volatile("" : "+v"(lane_w));
    if constexpr (!L::W_HERE) {
      pz = (frag_ptr)a.wz + lane;
      pd = (frag_ptr)a.wd + lane;
    }
    const int64_t row = step * NB_ROWS + 16 * wave + l15;
    const bool in = row < a.N;
    int32_t target = -1;
    int flag = 0;
    if (in) {
      if constexpr (DENSE) {
        flag = a.flag[row];
      } else {
        target = max(a.index[row], -1);
        flag = target < 0 ? 0 : target < a.V ? 1 : 2;
      }
    }
    float weight = 1.0f;
    if (GRAD && a.g && flag) weight = __builtin_amdgcn_ldexpf(a.g[row], -g_exp);
    if (!AHEAD) load_h(step);
    // logits, 32 channels at a time.  Fragments of W on their way: one or two ahead
    constexpr int RING = L::W_HERE && DENSE ? 2 : 3;
    s16x8 w[RING][3];
    f32x4 z[VT];
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) frag_z(i % VT, i / VT, w[i]);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      s16x8 hf[3];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[ks][e] = flag ? x[ks][e] : 0.0f;
      split_any8(x[ks], hf);
      if constexpr (GRAD) {
#pragma unroll
        for (int t = 0; t < 3; ++t) {
          // 8 ks pieces on: past the 16 that the rows exchange, or (ks odd) the same with bit 3 of the place flipped
          const int far = t * L::H_PLANE + (ks >> 1) * 128, flip = ks & 1 ? 64 : 0;
          store8(lds + far, hw_at[0] ^ flip, hw_at[1] ^ flip, hf[t]);
        }
      }
#pragma unroll
      for (int vt = 0; vt < VT; ++vt) {
        const int i = ks * VT + vt, n = i + RING - 1;
        if (ks == 0) z[vt] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (n < VT * KS) frag_z(n % VT, n / VT, w[n % RING]);
        z[vt] = mfma6(w[i % RING], hf, z[vt]);
        __builtin_amdgcn_sched_barrier(0);   // no more of them than that
      }
    }
    if (AHEAD && step + gridDim.x < steps) load_h(step + gridDim.x);
    float m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) {
      const int v = 16 * vt + 4 * g;
      const f32x4 bs = *reinterpret_cast<const f32x4*>(s_bias + v);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        z[vt][e] = fmaf(z[vt][e], a.scale, bs[e]);   // W is zero and the bias -inf past the alphabet
        m = fmaxf(m, z[vt][e]);
      }
    }
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    const float base = exp_base(m);
    // the target is element sub of the 4 in register group tv, in the lane with its row and (target >> 2 & 3) = g
    f32x4 at_target = {0.f, 0.f, 0.f, 0.f};
    const int tv = DENSE || (target >> 2 & 3) != g ? -1 : target >> 4;
#pragma unroll
    for (int vt = 0; vt < VT; ++vt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float t = z[vt][e] - base, y = exp2_hw(t);
        if (!DENSE) at_target[e] = tv == vt ? t : at_target[e];
        z[vt][e] = DENSE ? t : y;
        s += y;
      }
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    const float lse = log2_hw(s);  // over base
    float bits = 0.0f;
    if constexpr (!DENSE) {
      const int e = target & 3;
      const float t = e == 0 ? at_target[0] : e == 1 ? at_target[1] : e == 2 ? at_target[2] : at_target[3];
      bits = flag == 1 && tv >= 0 ? lse - t : 0.0f;
    }
    if (lane < 16 && in && a.lse) a.lse[row] = flag ? (base + lse) * LN2 : 0.0f;
    const float w1 = flag == 2 ? NAN : flag ? weight : 0.0f;
    const float inv = flag ? w1 / s : 0.0f;
    f32x4 sub;
#pragma unroll
    for (int e = 0; e < 4; ++e) sub[e] = (target & 3) == e ? -w1 : 0.0f;
    int tq = tv;
    asm volatile("" : "+v"(tq));   // the comparisons are made again: kept, they fill the scalar registers
    // the first entries of the row lane >> 2, held by its four lanes; further ones are read for every 32 symbols
    constexpr int NEAR = 4;
    int near_id[DENSE ? NEAR : 1];
    float near_q[DENSE ? NEAR : 1];
    if constexpr (DENSE) {
      const int64_t r = step * NB_ROWS + 16 * wave + (lane >> 2);
#pragma unroll
      for (int i = 0; i < NEAR; ++i) {
        const int j = 4 * i + (lane & 3);
        const bool have = r < a.N && j < a.k;
        near_id[i] = have ? a.index[r * a.k + j] : -1;
        near_q[i] = have ? a.q[r * a.k + j] : 0.0f;
      }
    }
    f32x4 dh[GRAD ? CT : 1];
#pragma unroll
    for (int ct = 0; ct < (GRAD ? CT : 1); ++ct) dh[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int buf = (u % L::BUFS) * L::D_BUF;
      f32x4 q[2];
      if constexpr (DENSE) {  // the targets' probabilities of 16 rows and 32 symbols, dense: rows 0-7 in plane 0, 8-15 in 1
        char* mine = lds + L::D + buf + wave * 1024;
        const int rl = lane >> 2;
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4*>(mine + i * L::D_PLANE + lane * 16) = f32x4{0.f, 0.f, 0.f, 0.f};
        wave_lds_fence();
        const int64_t r = step * NB_ROWS + 16 * wave + rl;
        const auto put = [&](int id, float y) {
          if (id >> 5 == u) *reinterpret_cast<float*>(mine + (rl >> 3) * L::D_PLANE + (rl & 7) * 128 + (id & 31) * 4) = y;
        };
#pragma unroll
        for (int i = 0; i < NEAR; ++i) put(near_id[i], near_q[i]);
        if (a.k > 4 * NEAR && r < a.N) {
          const int32_t* ix = a.index + r * a.k;
          const float* qx = a.q + r * a.k;
          for (int j0 = 4 * NEAR + (lane & 3); j0 < a.k; j0 += 4 * 8) {   // 16 loads in flight
            int id[8];
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int j = j0 + 4 * i;
              id[i] = j < a.k ? ix[j] : -1;
              y[i] = j < a.k ? qx[j] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) put(id[i], y[i]);
          }
        }
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < 2; ++i)
          q[i] = *reinterpret_cast<const f32x4*>(mine + (l15 >> 3) * L::D_PLANE + (l15 & 7) * 128 + (16 * i + 4 * g) * 4);
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (q[i][e] != 0.0f) bits += q[i][e] * (lse - z[2 * u + i][e]);
      }
      if constexpr (GRAD) {
#pragma unroll
        for (int i = 0; i < RING - 1; ++i) frag_d(u, i, w[i]);
        __builtin_amdgcn_sched_barrier(0);
        float d[8];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int vt = 2 * u + i;
            const float one = DENSE ? -w1 * q[i][e] : tq == vt ? sub[e] : 0.0f;
            d[4 * i + e] = fmaf(DENSE ? exp2_hw(z[vt][e]) : z[vt][e], inv, one);
          }
        s16x8 p[3];
        split_any8(d, p);
#pragma unroll
        for (int t = 0; t < 3; ++t) store8(lds + buf + t * L::D_PLANE, dw_at[0], dw_at[1], p[t]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const int n = ct + RING - 1;
          if (n < CT) frag_d(u, n, w[n % RING]);
          dh[ct] = mfma6(w[ct % RING], p, dh[ct]);
          __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
        // products of these 32 symbols' dz with h for this wave's tiles, before the other block's vector work
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int ks = 0; ks < NB_ROWS / 32; ++ks) {
          s16x8 dz[3];
#pragma unroll
          for (int t = 0; t < 3; ++t)
            dz[t] = read_tr(lds + dr_at[0] + (buf + t * L::D_PLANE + 32 * ks * 64), lds + dr_at[1] + (buf + t * L::D_PLANE + 32 * ks * 64));
#pragma unroll
          for (int j = 0; j < DW_N; ++j) {
            // NW / 2 tiles of channels on: 8 or 16 pieces (NW = 8: past what the rows exchange)
            static_assert(DW_N == 1 || NB_WAVES == 8, "one tile of channels a wave, or 64 channels apart");
            s16x8 h[3];
#pragma unroll
            for (int t = 0; t < 3; ++t) {
              const int far = t * L::H_PLANE + 32 * ks * (CP * 2) + j * 128;
              h[t] = read_tr(lds + hr_at[0] + far, lds + hr_at[1] + far);
            }
            dw[u][j] = mfma6(h, dz, dw[u][j]);
          }
          if (ks == my_c) {  // db: ones for h, in four of the 16 output rows; the waves of other channels take other rows
            const int one = (lane_w >> 2 & 3) == (u & 3) ? 0x3f803f80 : 0;
            const s16x8 ones = __builtin_bit_cast(s16x8, i32x4{one, one, one, one});
#pragma unroll
            for (int t = 2; t >= 0; --t) db[u / 4] = mfma<false>(ones, dz[t], db[u / 4]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (L::BUFS == 1 || u + 1 == U) __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    bits += __shfl_xor(bits, 16);
    bits += __shfl_xor(bits, 32);
    if (DENSE && flag == 1) bits += a.ent[row];
    if (lane < 16 && in) a.bits[row] = flag == 2 ? NAN : flag ? bits : 0.0f;
    if constexpr (GRAD) {
      if (a.dh && in) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const int c = 16 * ct + 4 * g;
          float* o = a.dh + row * a.C + c;
          f32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = flag ? scaled(dh[ct][e], out_scale) : 0.0f;   // 0 also where weights that are NaN reach it
          if (a.C % 4 == 0 && (uintptr_t)a.dh % 16 == 0) {
            if (c < a.C) *reinterpret_cast<f32x4*>(o) = y;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (c + e < a.C) o[e] = y[e];
          }
        }
      }
    }
  }
  if constexpr (GRAD) {
    float* part = a.part + (int64_t)blockIdx.x * (a.C + DB) * a.V;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = 32 * u + 16 * my_v + l15;
      if (v >= a.V) continue;
#pragma unroll
      for (int j = 0; j < DW_N; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = 16 * (my_c + DB * j) + 4 * g + e;
          if (c < a.C) part[(int64_t)c * a.V + v] = dw[u][j][e];
        }
      if (g == (u & 3)) part[(int64_t)(a.C + my_c) * a.V + v] = db[u / 4][0];
    }
  }
}

// W as the lanes of k_narrow read it where it does not lie in LDS.
__global__ void __launch_bounds__(256) k_narrow_pack(NarrowArgs a, int KS, int CT, int VT, uint16_t* wz, uint16_t* wd) {
  const int nz = VT * KS * 64, nd = VT / 2 * CT * 64;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < nz + nd; i += gridDim.x * 256) {
    const bool z = i < nz;
    const int f = (z ? i : i - nz) / 64, lane = i % 64, l15 = lane & 15, g = lane >> 4;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int v = z ? 16 * (f % VT) + l15 : 32 * (f / CT) + 16 * (e >> 2) + 4 * g + (e & 3);
      const int c = z ? 32 * (f / VT) + 8 * g + e : 16 * (f % CT) + l15;
      x[e] = c < a.C && v < a.V ? a.w[c * a.w_stride + v] : 0.0f;
    }
    s16x8 p[3];
    split_any8(x, p);
    s16x8* o = reinterpret_cast<s16x8*>(z ? wz : wd) + (int64_t)f * 3 * 64 + lane;
#pragma unroll
    for (int t = 0; t < 3; ++t) o[t * 64] = p[t];
  }
}

// dw and db from the blocks' sums: 16 values a block, 16 shares of the blocks each.
__global__ void __launch_bounds__(256) k_narrow_join(const float* __restrict__ part, int blocks, int C, int V, int DB,
                                                     OutScale out_scale, const float* __restrict__ gpart,
                                                     float* __restrict__ dw, float* __restrict__ db) {
  __shared__ float s[16][17];
  const OutScale scale = with_weights(out_scale, gpart);
  const int i = threadIdx.x & 15, share = threadIdx.x >> 4;
  const int64_t n = (int64_t)C * V, all = n + (int64_t)DB * V, at = (int64_t)blockIdx.x * 16 + i;
  float x = 0.0f;
  if (at < n + V) {
    const int shares = at < n ? 1 : DB;   // db has DB rows, each a share of the block's rows
    for (int q = 0; q < shares; ++q) {
      const float* p = part + at + (int64_t)q * V;
#pragma unroll 16
      for (int b = share; b < blocks; b += 16) x += p[b * all];
    }
  }
  s[share][i] = x;
  __syncthreads();
  if (share != 0 || at >= n + V) return;
  x = 0.0f;
  for (int k = 0; k < 16; ++k) x += s[k][i];
  if (at < n) {
    if (dw) dw[at] = scaled(x, scale);
  } else if (db) db[at - n] = scaled(x, scale);
}

int width_of(int channels) { return channels <= 32 ? 2 : channels <= 64 ? 4 : 8; }
// as many as run at a time
int narrow_blocks(const reno_head& p) {
  const int nw = waves_of(width_of(p.channels));
  return (int)std::min<int64_t>(256 * (8 / nw), (p.rows + 16 * nw - 1) / (16 * nw));
}
int64_t part_bytes(const reno_head& p) {
  return (int64_t)narrow_blocks(p) * (p.channels + waves_of(width_of(p.channels)) / 2) * p.symbols * 4;
}
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

template <int CT, int VQ>
void run(const NarrowArgs& a, bool grad, int blocks, hipStream_t st) {
  const auto args = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(blocks), dim3(64 * waves_of(CT)), 0, st, a); };
  if (a.q) grad ? args(k_narrow<CT, VQ, true, true>) : args(k_narrow<CT, VQ, false, true>);
  else grad ? args(k_narrow<CT, VQ, true, false>) : args(k_narrow<CT, VQ, false, false>);
}

}  // namespace

bool head_is_narrow(const reno_head& p) { return p.type == RENO_T_FP32 && p.channels <= 128 && p.symbols <= 256; }

// workspace: the blocks' sums, then W as it is streamed
int64_t head_narrow_bytes(const reno_head& p, bool grad) {
  const int64_t cp = 16 * width_of(p.channels);
  int64_t n = grad ? up256(part_bytes(p)) : 0;
  if (cp > 32) n += 2 * up256(cp * 256 * 3 * 2);
  return n;
}

hipError_t launch_head_narrow(const HeadCall& c, const HeadTargets& t, const float* gpart, char* ws, hipStream_t st) {
  const reno_head& p = c.p;
  NarrowArgs a{};
  a.N = p.rows;
  a.C = p.channels;
  a.V = p.symbols;
  a.k = c.k;
  a.h_stride = p.h_stride;
  a.w_stride = p.w_stride;
  a.h = static_cast<const float*>(c.d.h);
  a.w = static_cast<const float*>(c.d.w);
  a.b = static_cast<const float*>(c.d.b);
  a.g = c.d.row_weight;
  a.index = t.index;
  a.q = t.q;
  a.ent = t.ent;
  a.flag = t.flag;
  a.scale = (float)(1.4426950408889634 / (double)c.temperature);
  a.out_scale = out_scale(c.temperature);
  a.gpart = gpart;
  a.bits = c.d.bits;
  a.lse = c.d.lse;
  a.dh = static_cast<float*>(c.d.dh);
  const int blocks = narrow_blocks(p);
  char* at = ws;
  if (c.grad) {
    a.part = reinterpret_cast<float*>(at);
    at += up256(part_bytes(p));
  }
  const int CT = width_of(p.channels), VQ = p.symbols <= 64 ? 1 : 4;
  if (CT > 2) {
    uint16_t* wz = reinterpret_cast<uint16_t*>(at);
    uint16_t* wd = reinterpret_cast<uint16_t*>(at + up256((int64_t)CT * 16 * 256 * 3 * 2));
    a.wz = wz;
    a.wd = wd;
    const int n = 4 * VQ * (CT / 2) * 64 + 2 * VQ * CT * 64;
    hipLaunchKernelGGL(k_narrow_pack, dim3((n + 255) / 256), dim3(256), 0, st, a, CT / 2, CT, 4 * VQ, wz, wd);
  }
  if (VQ == 1) {
    if (CT == 2) run<2, 1>(a, c.grad, blocks, st);
    else if (CT == 4) run<4, 1>(a, c.grad, blocks, st);
    else run<8, 1>(a, c.grad, blocks, st);
  } else {
    if (CT == 2) run<2, 4>(a, c.grad, blocks, st);
    else if (CT == 4) run<4, 4>(a, c.grad, blocks, st);
    else run<8, 4>(a, c.grad, blocks, st);
  }
  if (c.d.dw || c.d.db) {
    const int64_t n = (int64_t)(a.C + 1) * a.V;
    hipLaunchKernelGGL(k_narrow_join, dim3((unsigned)((n + 15) / 16)), dim3(256), 0, st, a.part, blocks, a.C, a.V,
                       waves_of(CT) / 2, a.out_scale, a.gpart, static_cast<float*>(c.d.dw), static_cast<float*>(c.d.db));
  }
  return hipGetLastError();
}

}  // namespace reno
