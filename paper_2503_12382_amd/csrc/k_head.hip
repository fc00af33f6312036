// Code length of a linear head with its gradient, and distillation from a
// teacher's top logits with its gradient (reno_head.h).
//
// With t = z log2(e) / T (logits at the temperature, in powers of two) a row's
// loss in bits is sum_j q_j (log2 q_j + lse2 - t_j), lse2 = log2 sum_v 2^t_v, over
// its target entries (one with q = 1: the code length), and its gradient for z
// is g / (T ln 2) (2^(t - lse2) - q).  Steps, over pieces of rows so that the logits
// are never kept whole:
//   k_head_targets  (distillation) q, entries of one index joined
//   k_head_setup    operands as 16-bit planes, padded; rows left out as zeros; the scaled bias
//   k_head_logits   z by MFMA; every wave leaves the maximum and the sum of 2^(t - max)
//                   of its part of the alphabet for each row, the t of the rows' targets, and
//                   (gradient) what dz needs of this piece: t, for bf16 2^(t - max) in 16 bits
//   k_head_rows     lse2 and the bits from the parts
//   k_head_dz       dz as 16-bit planes, and its sums over rows
//   k_head_product  dh = dz w^T and dw = h^T dz by MFMA, split over k where the
//                   outputs alone do not fill the chip
//   k_head_reduce   joins splits; k_head_db the sums of dz; both in a fixed order
// Up to 4 rows without gradients take k_head_few and k_head_rows instead; narrow
// fp32 heads k_head_narrow.hip.
//
// dz is carried over the largest |g| (a power of two, G) and put right in the
// products' results: fp16 and the low planes of fp32 lose nothing of it for small g.
//
// Bound: the three products.  8192 x 2048 x 65536 bf16 (6.6 TFLOP, two pieces) takes 6.6 ms, 1000 TFLOP/s, where
// one large product of the library's reaches 1207; of a piece of 4096 rows k_head_logits takes 1.13 ms, dh 1.10,
// dw 0.97 and (the second piece, which reads and writes the first one's sums) 1.27, k_head_dz 0.23.

#include <algorithm>

#include "dev.h"
#include "gemm.h"
#include "head.h"
#include "head_dev.h"

namespace reno {
namespace {

constexpr int DZ_COLS = 512;     // symbols of a wave of k_head_dz
constexpr int HALF_SHIFT = 14;   // dz in fp16 is scaled by 2^14

// ---- element types ----
template <int TYPE>
__device__ __forceinline__ float load_as_float(const void* p, int64_t i) {
  if constexpr (TYPE == RENO_T_FP32) return static_cast<const float*>(p)[i];
  else if constexpr (TYPE == RENO_T_BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
  else return (float)static_cast<const _Float16*>(p)[i];
}
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ uint16_t to_fp16(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }

// 8 values as they lie in memory (16 bytes, fp32: 32)
template <int TYPE>
__device__ __forceinline__ void widen8(const uint4 (&raw)[TYPE == RENO_T_FP32 ? 2 : 1], float (&x)[8]) {
#pragma unroll
  for (int q = 0; q < (TYPE == RENO_T_FP32 ? 2 : 1); ++q) {
    const uint32_t b[4] = {raw[q].x, raw[q].y, raw[q].z, raw[q].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (TYPE == RENO_T_FP32) x[4 * q + e] = __uint_as_float(b[e]);
      else if constexpr (TYPE == RENO_T_BF16) {
        x[2 * e] = __uint_as_float(b[e] << 16);
        x[2 * e + 1] = __uint_as_float(b[e] & 0xffff0000u);
      } else {
        x[2 * e] = (float)__builtin_bit_cast(_Float16, (uint16_t)b[e]);
        x[2 * e + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(b[e] >> 16));
      }
    }
  }
}

template <int TYPE, int PLANES>
__device__ __forceinline__ void to_planes(float x, uint16_t (&o)[PLANES]) {
  if constexpr (TYPE == RENO_T_FP32) {
    split3(x, o);
  } else if constexpr (TYPE == RENO_T_BF16) {
    o[0] = to_bf16(x);
    if constexpr (PLANES == 2) o[1] = to_bf16(x - __uint_as_float((uint32_t)o[0] << 16));
  } else {
    o[0] = to_fp16(x);
    if constexpr (PLANES == 2) o[1] = to_fp16(x - (float)__builtin_bit_cast(_Float16, o[0]));
  }
}
constexpr int planes_of(int type) { return type == RENO_T_FP32 ? 3 : 1; }

// What every kernel of one call needs.
struct HeadArgs {
  int64_t N;               // rows of the call
  int64_t r0, R;           // first row and rows of this piece
  int C, V, k;
  int64_t Cp, Vp;          // padded to BK
  int64_t h_stride, w_stride;
  const void *h, *w, *b;
  const float* g;
  const int32_t* index;    // targets as given (code length) or joined (distillation)
  const float* q;          // their probabilities, or null: 1
  const float* ent;        // sum q log2 q a row (distillation)
  const uint8_t* flag;     // row state (distillation)
  float scale;             // log2(e) / T
  float* bias;             // b * scale
  uint16_t* hp;            // planes of h [R][Cp]
  uint16_t* wp;            // planes of w [C][Vp], if they are made
  int64_t h_plane, w_plane, d_plane;
  float2* part;            // [parts][R] maximum and sum
  int parts;
  float* tt;               // [R][k] t of the targets
  float* t;                // [R][Vp], or (bf16)
  uint16_t* t16;           // [R][Vp]: 2^(t - the part's maximum + 15) in fp16; dz takes its place
  int part_width;          // symbols of a part
  float* lse2;             // [R]
  uint16_t* dz;            // planes [R][Vp]
  float* dbp;              // [ceil(R / dz_rows)][Vp]
  int dz_rows;             // rows of a wave of k_head_dz
  const float* gpart;      // [GPARTS]
  float *bits, *lse;       // of the call
};

// 0: left out, 1: taken, 2: a target outside the alphabet
__device__ __forceinline__ int row_flag(const HeadArgs& a, int64_t row) {
  if (a.flag) return a.flag[row];
  const int32_t s = a.index[row];
  return s < 0 ? 0 : s < a.V ? 1 : 2;
}

// ---- targets of a distillation ----
// LW lanes a row, PER entries a lane (k <= LW PER).
template <int LW, int PER>
__global__ void __launch_bounds__(256) k_head_targets(const int32_t* __restrict__ index, const float* __restrict__ logit,
                                                      int64_t n, int k, int V, float scale, int32_t* __restrict__ out,
                                                      float* __restrict__ q_out, float* __restrict__ ent,
                                                      uint8_t* __restrict__ flag) {
  __shared__ uint32_t s_seen[256 / LW][128];   // a bit for each of 4096 hashes of the row's indices
  const int lane = threadIdx.x % LW;
  const int64_t row = (int64_t)blockIdx.x * (256 / LW) + threadIdx.x / LW;
  uint32_t* seen = s_seen[threadIdx.x / LW];
#pragma unroll
  for (int i = 0; i < 128 / LW; ++i) seen[i * LW + lane] = 0;
  wave_lds_fence();
  const bool in = row < n;
  const auto top_of = [](float v) {
    for (int o = LW / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
  };
  const auto sum_of = [](float v) {
    for (int o = LW / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
  };
  int32_t id[PER];
  float t[PER], q[PER];
  float m = -INFINITY, bad = 0.0f;
#pragma unroll
  for (int c = 0; c < PER; ++c) {
    const int j = c * LW + lane;
    id[c] = in && j < k ? index[row * k + j] : -1;
    t[c] = id[c] >= 0 ? logit[row * k + j] : -INFINITY;
    if (id[c] >= V || t[c] != t[c]) bad = 1.0f;
    m = fmaxf(m, t[c]);
  }
  m = top_of(m);
  const bool any_bad = top_of(bad) != 0.0f || m == INFINITY;
  float sum = 0.0f;
#pragma unroll
  for (int c = 0; c < PER; ++c) {
    q[c] = m > -INFINITY ? exp2_hw((t[c] - m) * scale) : 0.0f;
    sum += q[c];
  }
  sum = sum_of(sum);
#pragma unroll
  for (int c = 0; c < PER; ++c) {
    q[c] = sum > 0.0f ? q[c] / sum : 0.0f;
    if (q[c] == 0.0f) id[c] = -1;
  }
  // entries of one index: the first takes the sum, in order, the others go.  Most rows have none: no two entries
  // then meet in a bit (up to 4096 symbols: exactly, beyond: of their hashes), and the walk over them is left out
  float joined[PER];
  bool later[PER] = {};
  bool met = false;
#pragma unroll
  for (int c = 0; c < PER; ++c) {
    joined[c] = q[c];
    if (id[c] >= 0) {
      const uint32_t hash = V <= 4096 ? (uint32_t)id[c] & 4095u : (uint32_t)id[c] * 0x9e3779b1u >> 20;
      met |= (atomicOr(&seen[hash >> 5], 1u << (hash & 31)) >> (hash & 31)) & 1;
    }
  }
  if (__ballot(met)) {
#pragma unroll
    for (int c = 0; c < PER; ++c) joined[c] = 0.0f;
#pragma unroll
    for (int s = 0; s < PER; ++s) {
      const int cnt = min(max(k - s * LW, 0), LW);
      for (int l = 0; l < cnt; ++l) {
        const int32_t oi = __shfl(id[s], l, LW);
        const float oq = __shfl(q[s], l, LW);
#pragma unroll
        for (int c = 0; c < PER; ++c)
          if (oi == id[c]) {
            joined[c] += oq;
            later[c] |= s * LW + l < c * LW + lane;
          }
      }
    }
  }
  float e = 0.0f;
#pragma unroll
  for (int c = 0; c < PER; ++c) {
    const int j = c * LW + lane;
    const bool keep = id[c] >= 0 && !later[c] && !any_bad;
    if (in && j < k) {
      out[row * k + j] = keep ? id[c] : -1;
      q_out[row * k + j] = keep ? joined[c] : 0.0f;
    }
    if (keep) e += joined[c] * log2_hw(joined[c]);
  }
  e = sum_of(e);
  if (lane == 0 && in) {
    ent[row] = e;
    flag[row] = any_bad ? 2 : m > -INFINITY ? 1 : 0;
  }
}

// ---- what the products need: operands as planes, the scaled bias, maxima of the weights ----
template <int TYPE>
__device__ __forceinline__ void pack8(const void* src, int64_t at, int n, uint16_t* dst, int64_t plane) {
  constexpr int P = planes_of(TYPE);
  uint16_t o[P][8];
  float x[8] = {};
  if (n >= 8) {   // whole loads, of any alignment
    uint4 raw[TYPE == RENO_T_FP32 ? 2 : 1];
    __builtin_memcpy(raw, static_cast<const char*>(src) + at * (TYPE == RENO_T_FP32 ? 4 : 2), sizeof raw);
    widen8<TYPE>(raw, x);
  } else if (n > 0) {   // what is there, no load waiting for another
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = load_as_float<TYPE>(src, at + min(e, n - 1));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint16_t v[P];
    to_planes<TYPE, P>(e < n ? x[e] : 0.0f, v);
#pragma unroll
    for (int p = 0; p < P; ++p) o[p][e] = v[p];
  }
#pragma unroll
  for (int p = 0; p < P; ++p) *reinterpret_cast<uint4*>(dst + p * plane) = *reinterpret_cast<const uint4*>(o[p]);
}

// Rows left out become zeros: nothing of them may reach dw.
template <int TYPE>
__device__ __forceinline__ void pack_h(const HeadArgs& a, int64_t block, int64_t blocks) {
  const int64_t per = a.Cp / 8, total = a.R * per;
  for (int64_t i = block * 256 + threadIdx.x; i < total; i += blocks * 256) {
    const int64_t r = i / per;
    const int c0 = (int)(i % per) * 8;
    const int n = row_flag(a, a.r0 + r) != 0 ? a.C - c0 : 0;
    pack8<TYPE>(a.h, (a.r0 + r) * a.h_stride + c0, n, a.hp + r * a.Cp + c0, a.h_plane);
  }
}

template <int TYPE>
__global__ void __launch_bounds__(256) k_head_pack_h(HeadArgs a) {
  pack_h<TYPE>(a, blockIdx.x, gridDim.x);
}

// Blocks of the first launch, by what they do: the first piece's rows of h, GPARTS partial maxima of the finite |g|
// of rows with a target (what the others weigh must not move the scale of dz), b * scale padded to whole tiles, the
// weights (where they cannot be read in place).
struct SetupBlocks {
  unsigned h, g, b, w;
};

template <int TYPE>
__global__ void __launch_bounds__(256) k_head_setup(HeadArgs a, SetupBlocks n, int64_t Vb, float* __restrict__ gpart) {
  __shared__ float s[4];
  unsigned x = blockIdx.x;
  if (x < n.h) return pack_h<TYPE>(a, x, n.h);
  x -= n.h;
  if (x < n.g) {
    float m = 0.0f;
#pragma unroll 4
    for (int64_t i = (int64_t)x * 256 + threadIdx.x; i < a.N; i += GPARTS * 256) {
      const bool taken = row_flag(a, i) == 1;
      const float y = fabsf(a.g[i]);
      if (taken && y < INFINITY) m = fmaxf(m, y);
    }
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    if (lane_id() == 0) s[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) gpart[x] = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    return;
  }
  x -= n.g;
  if (x < n.b) {
    const int64_t i = (int64_t)x * 256 + threadIdx.x;
    if (i < Vb) a.bias[i] = a.b && i < a.V ? load_as_float<TYPE>(a.b, i) * a.scale : 0.0f;
    return;
  }
  x -= n.b;
  const int64_t per = a.Vp / 8, total = a.C * per;
  for (int64_t i = (int64_t)x * 256 + threadIdx.x; i < total; i += (int64_t)n.w * 256) {
    const int64_t c = i / per, v0 = (i % per) * 8;
    pack8<TYPE>(a.w, c * a.w_stride + v0, (int)min((int64_t)8, a.V - v0), a.wp + c * a.Vp + v0, a.w_plane);
  }
}

// ---- logits ----
// 2048 x 2048 x 32768 bf16 forward: 232 us, 1185 TFLOP/s; fp32 (six products for one): 1.33 ms, 1237.
// The lookup of 64 entries a row adds 80 us to the 300 of 4096 x 1024 x 32768.
// m runs over symbols, n over rows: a lane holds one row and 4 consecutive
// symbols of each 16, so that a row's maximum and sum need two lane exchanges.
template <int BM, int BN, int WM, int WN, bool HALF>
__global__ void __launch_bounds__(WM* WN * 64) k_head_logits(HeadArgs a, Operand W, Operand H, TileOrder order, Terms terms) {
  using Tile = GemmTile<BM, BN, WM, WN, true, false, HALF>;
  __shared__ __attribute__((aligned(1024))) char lds[Tile::LDS];
  int tm, tn, split;
  order.at(blockIdx.x, gridDim.x, tm, tn, split);
  f32x4 acc[Tile::MF][Tile::NF];
  Tile::run(lds, W, H, (int64_t)tm * BM, (int64_t)tn * BN, 0, a.Cp, terms, acc);
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const int l15 = lane & 15, g = lane >> 4;
  const int v0 = tm * BM + (wave / WN) * (BM / WM);
  const int64_t n0 = (int64_t)tn * BN + (wave % WN) * (BN / WN);
#pragma unroll
  for (int i = 0; i < Tile::MF; ++i) {
    const int v = v0 + 16 * i + 4 * g;
    const f32x4 bs = *reinterpret_cast<const f32x4*>(a.bias + v);
#pragma unroll
    for (int j = 0; j < Tile::NF; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = v + e < a.V ? fmaf(acc[i][j][e], a.scale, bs[e]) : -INFINITY;
  }
  const int p = v0 / (BM / WM);
#pragma unroll
  for (int j = 0; j < Tile::NF; ++j) {
    const int64_t r = n0 + 16 * j + l15;
    float m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int i = 0; i < Tile::MF; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][j][e]);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    const float base = exp_base(m);
#pragma unroll
    for (int i = 0; i < Tile::MF; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s += exp2_hw(acc[i][j][e] - base);
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (g == 0 && r < a.R && p < a.parts) a.part[(int64_t)p * a.R + r] = make_float2(m, s);
    if (a.t16 && r < a.R) {
#pragma unroll
      for (int i = 0; i < Tile::MF; ++i) {
        const int v = v0 + 16 * i + 4 * g;
        uint16_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = to_fp16(exp2_hw(acc[i][j][e] - base + 15.0f));
        if (v < a.Vp) *reinterpret_cast<uint2*>(a.t16 + r * a.Vp + v) = *reinterpret_cast<const uint2*>(o);
      }
    }
    if (a.t && r < a.R) {
#pragma unroll
      for (int i = 0; i < Tile::MF; ++i) {
        const int v = v0 + 16 * i + 4 * g;
        if (v < a.Vp) *reinterpret_cast<f32x4*>(a.t + r * a.Vp + v) = acc[i][j];
      }
    }
  }
  // the targets' t
  if (a.k == 1) {
#pragma unroll
    for (int j = 0; j < Tile::NF; ++j) {
      const int64_t r = n0 + 16 * j + l15;
      const int id = r < a.R ? a.index[a.r0 + r] : -1;
      const int want = id < 0 ? -1 : id - v0 - 4 * g;
#pragma unroll
      for (int i = 0; i < Tile::MF; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (id >= 0 && want == 16 * i + e) a.tt[r] = acc[i][j][e];
    }
    return;
  }
  // several entries a row: 16 PR rows at a time pass through the wave's share of LDS, and every lane looks up
  // the entries of its own
  constexpr int MW = BM / WM, PR = 16384 / (MW * 4) / 16;   // symbols of the wave, groups of 16 rows in 16 KB
  static_assert(Tile::LDS >= WM * WN * 16384 && Tile::NF % PR == 0, "a wave's share of LDS holds 16 PR rows");
  constexpr int AHEAD = 16;
  char* mine = lds + wave * 16384;
#pragma unroll
  for (int j0 = 0; j0 < Tile::NF; j0 += PR) {
#pragma unroll
    for (int j = 0; j < PR; ++j)
#pragma unroll
      for (int i = 0; i < Tile::MF; ++i)   // pieces of 16 bytes, spread over the banks by the row
        *reinterpret_cast<f32x4*>(mine + (16 * j + l15) * (MW * 4) + (((4 * i + g) ^ l15) * 16)) = acc[i][j0 + j];
    wave_lds_fence();
    const int64_t r0 = n0 + 16 * j0;
    const int rows = (int)max((int64_t)0, min((int64_t)(16 * PR), a.R - r0));
    const int all = rows * a.k;
    const float inv_k = 1.0f / (float)a.k;
    const int32_t* ix = a.index + (a.r0 + r0) * a.k;
    for (int x0 = 0; x0 < all; x0 += 64 * AHEAD) {
      int id[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) id[u] = ix[min(x0 + 64 * u + lane, all - 1)];   // none waits for another
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int x = x0 + 64 * u + lane, v = id[u] - v0;
        if (x < all && id[u] >= v0 && v < MW) {
          const int rl = (int)(((float)x + 0.5f) * inv_k);   // x / k: x + 1/2 lies at least 1/2 off its multiples
          a.tt[r0 * a.k + x] = *reinterpret_cast<const float*>(mine + rl * (MW * 4) + (((v >> 2) ^ (rl & 15)) * 16) + (v & 3) * 4);
        }
      }
    }
    wave_lds_fence();
  }
}

// ---- few rows, no gradient: w is read once, by vector instructions ----
// A block takes CB symbols and all channels; a lane 8 consecutive symbols of every (512 / (CB / 8))th
// channel, so that a wave reads whole lines of w with 16-byte loads (fp32: two), FEW_AHEAD of them in
// flight, wherever the rows start (1 x 2048 x 50021: fp32 88 us, bf16 60; element by element 234 and 124).
// Bound by the read of w: 1 x 2048 x 65536 bf16 in 52 us, 5.1 TB/s.  FEW_ROWS: 4 rows take 55 us here
// and 70 by k_head_logits, 8 rows 114 and 70.
constexpr int FEW_ROWS = 4, FEW_AHEAD = 8;
constexpr int FEW_H = 16384;   // values of h that are held in LDS

template <int TYPE, int CB, int NR>
__global__ void __launch_bounds__(512) k_head_few(HeadArgs a) {
  constexpr int LANES = CB / 8, SHARES = 512 / LANES;
  __shared__ float s_h[FEW_H];
  __shared__ float s_sum[512 / 64][NR][CB];
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  for (int i = tid; i < NR * a.C; i += 512) {
    const int r = i / a.C, c = i % a.C;
    s_h[i] = r < a.R && row_flag(a, r) != 0 ? load_as_float<TYPE>(a.h, r * a.h_stride + c) : 0.0f;
  }
  __syncthreads();
  const int v0 = blockIdx.x * CB, v = v0 + tid % LANES * 8;
  float acc[NR][8] = {};
  const auto fma8 = [&](int c, const float (&x)[8]) {
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const float y = s_h[r * a.C + c];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[r][e] = fmaf(y, x[e], acc[r][e]);
    }
  };
  if (v + 8 <= a.V) {
    constexpr int Q = TYPE == RENO_T_FP32 ? 2 : 1;
    const char* p = static_cast<const char*>(a.w) + (int64_t)v * (TYPE == RENO_T_FP32 ? 4 : 2);
    const int64_t ld = a.w_stride * (TYPE == RENO_T_FP32 ? 4 : 2);
    for (int c0 = tid / LANES; c0 < a.C; c0 += SHARES * FEW_AHEAD) {
      uint4 raw[FEW_AHEAD][Q];
#pragma unroll
      for (int u = 0; u < FEW_AHEAD; ++u) {
        const int c = min(c0 + u * SHARES, a.C - 1);
#pragma unroll
        for (int q = 0; q < Q; ++q) __builtin_memcpy(&raw[u][q], p + c * ld + q * 16, 16);   // of any alignment
      }
#pragma unroll
      for (int u = 0; u < FEW_AHEAD; ++u) {
        if (c0 + u * SHARES >= a.C) break;
        float x[8];
        widen8<TYPE>(raw[u], x);
        fma8(c0 + u * SHARES, x);
      }
    }
  } else {
#pragma unroll 4
    for (int c = tid / LANES; c < a.C; c += SHARES) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)   // past the alphabet: its last symbol again, whose sums are not used
        x[e] = load_as_float<TYPE>(a.w, c * a.w_stride + min(v + e, a.V - 1));
      fma8(c, x);
    }
  }
  // channels' shares of a wave, then the waves'
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int o = LANES; o < 64; o *= 2) acc[r][e] += __shfl_xor(acc[r][e], o);
      if (lane < LANES) s_sum[wave][r][lane * 8 + e] = acc[r][e];
    }
  __syncthreads();
  // a wave a row: t, maximum and sum, the row's entries
  for (int r = wave; r < NR && r < a.R; r += 8) {
    float m = -INFINITY, s = 0.0f, t[CB / 64];
#pragma unroll
    for (int i = 0; i < CB / 64; ++i) {
      const int x = lane + 64 * i;
      float z = 0.0f;
#pragma unroll
      for (int w = 0; w < 8; ++w) z += s_sum[w][r][x];
      const float b = a.b && v0 + x < a.V ? load_as_float<TYPE>(a.b, v0 + x) : 0.0f;
      t[i] = v0 + x < a.V ? fmaf(z, a.scale, b * a.scale) : -INFINITY;
      m = fmaxf(m, t[i]);
    }
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float base = exp_base(m);
#pragma unroll
    for (int i = 0; i < CB / 64; ++i) {
      s += exp2_hw(t[i] - base);
      s_sum[0][r][lane + 64 * i] = t[i];   // a wave's own row from here on
    }
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) a.part[(int64_t)blockIdx.x * a.R + r] = make_float2(m, s);
    wave_lds_fence();
    for (int j = lane; j < a.k; j += 64) {
      const int id = a.index[r * a.k + j];
      if (id >= v0 && id < min(v0 + CB, a.V)) a.tt[r * a.k + j] = s_sum[0][r][id - v0];
    }
  }
}

// ---- rows: lse2 and bits from the parts; 16 rows a block, 16 lanes each ----
__global__ void __launch_bounds__(256) k_head_rows(HeadArgs a) {
  __shared__ float2 s_p[16][17];
  __shared__ float s_b[16][17];
  const int rl = threadIdx.x & 15, pl = threadIdx.x >> 4;
  const int64_t r = (int64_t)blockIdx.x * 16 + rl;
  const bool in = r < a.R;
  float m = -INFINITY, s = 0.0f;
  if (in)
    for (int p0 = pl; p0 < a.parts; p0 += 16 * 8) {   // 8 loads in flight
      float2 x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        x[u] = p0 + 16 * u < a.parts ? a.part[(int64_t)(p0 + 16 * u) * a.R + r] : make_float2(-INFINITY, 0.0f);
      float n = m;
#pragma unroll
      for (int u = 0; u < 8; ++u) n = fmaxf(n, x[u].x);
      const float base = exp_base(n);
      s *= exp2_hw(m - base);
#pragma unroll
      for (int u = 0; u < 8; ++u) s += x[u].y * exp2_hw(x[u].x - base);
      m = n;
    }
  s_p[rl][pl] = make_float2(m, s);
  __syncthreads();
  float top = -INFINITY;
  for (int p = 0; p < 16; ++p) top = fmaxf(top, s_p[rl][p].x);
  const float base = exp_base(top);
  float sum = 0.0f;
  for (int p = 0; p < 16; ++p) sum += s_p[rl][p].y * exp2_hw(s_p[rl][p].x - base);
  const float over = log2_hw(sum), lse2 = base + over;
  const int flag = in ? row_flag(a, a.r0 + r) : 0;
  float b = 0.0f;
  if (flag == 1) {
    for (int j = pl; j < a.k; j += 16) {
      const float q = a.q ? a.q[(a.r0 + r) * a.k + j] : 1.0f;
      if (q != 0.0f) b += q * ((base - a.tt[r * a.k + j]) + over);   // not from lse2: where p is near 1 that rounds more than the bits
    }
  }
  s_b[rl][pl] = b;
  __syncthreads();
  if (pl != 0 || !in) return;
  b = a.ent && flag == 1 ? a.ent[a.r0 + r] : 0.0f;
  for (int p = 0; p < 16; ++p) b += s_b[rl][p];
  a.lse2[r] = lse2;
  a.bits[a.r0 + r] = flag == 2 ? NAN : b;
  if (a.lse) a.lse[a.r0 + r] = flag ? lse2 * LN2 : 0.0f;
}

// ---- dz of a piece: a wave takes 512 symbols of dz_rows rows ----
// Bound by memory: t read, dz written (bf16 in its place: 4 bytes a logit in all).  4096 x 65536 bf16: 225 us,
// 4.8 TB/s.  bf16 keeps 2^(t - max + 15) in fp16 between the two: 2^-12 of itself down to 2^-29, an eighth of what
// rounding dz to bf16 takes; the targets' p - q come from their t in fp32.
template <int TYPE, int P>
__global__ void __launch_bounds__(256) k_head_dz(HeadArgs a) {
  constexpr bool T16 = TYPE == RENO_T_BF16;
  constexpr int U = 4;   // rows whose loads are in flight
  constexpr int S = DZ_COLS / 64;   // symbols of a lane
  constexpr float SHIFT = TYPE == RENO_T_FP16 ? (float)(1 << HALF_SHIFT) : 1.0f;
  const int lane = lane_id();
  const int ge = __builtin_amdgcn_readfirstlane(weight_exp(a.gpart));
  const int64_t groups = (a.Vp + 64 * S - 1) / (64 * S), blocks = (a.R + a.dz_rows - 1) / a.dz_rows;
  const int64_t task = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (task >= groups * blocks) return;
  const int v0 = (int)(task % groups) * (64 * S);
  const int64_t rb = task / groups;
  const int v = v0 + lane * S;
  const bool mine = v < a.Vp;
  const int vc = mine ? v : 0;
  float sum[S] = {};
  const int64_t end = min(a.R, (rb + 1) * a.dz_rows);
  for (int64_t r1 = rb * a.dz_rows; r1 < end; r1 += U) {
    f32x4 t[U][2];
    uint4 t16[U];
    float pm[U], lse2[U], w[U], tt[U], q[U];
    int id[U], flag[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = min(r1 + u, end - 1), row = a.r0 + r;
      if constexpr (T16) {
        t16[u] = *reinterpret_cast<const uint4*>(a.t16 + r * a.Vp + vc);
        pm[u] = a.part[(int64_t)min(vc / a.part_width, a.parts - 1) * a.R + r].x;
      } else {
        t[u][0] = *reinterpret_cast<const f32x4*>(a.t + r * a.Vp + vc);
        t[u][1] = *reinterpret_cast<const f32x4*>(a.t + r * a.Vp + vc + 4);
      }
      flag[u] = row_flag(a, row);
      lse2[u] = a.lse2[r];
      w[u] = a.g ? a.g[row] : 1.0f;
      if (a.q) {
        id[u] = lane < a.k ? a.index[row * a.k + lane] : -1;
        q[u] = lane < a.k ? a.q[row * a.k + lane] : 0.0f;
        tt[u] = T16 && lane < a.k ? a.tt[r * a.k + lane] : 0.0f;
      } else {
        id[u] = a.index[row];
        tt[u] = a.tt[r];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = r1 + u, row = a.r0 + r;
      if (r >= end) break;
      float d[S] = {};
      if (flag[u]) {
        const float wr = flag[u] == 2 ? NAN : a.g ? __builtin_amdgcn_ldexpf(w[u], -ge) : 1.0f;
        if constexpr (T16) {
          // a part without any logit adds nothing, however far below it the row's normaliser lies
          const float f = pm[u] > -INFINITY ? exp2_hw(pm[u] - lse2[u] - 15.0f) : lse2[u] > -INFINITY ? 0.0f : NAN;
          const uint32_t x[4] = {t16[u].x, t16[u].y, t16[u].z, t16[u].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            d[2 * e] = (float)__builtin_bit_cast(_Float16, (uint16_t)x[e]) * f;
            d[2 * e + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(x[e] >> 16)) * f;
          }
        } else {
#pragma unroll
          for (int e = 0; e < S; ++e) d[e] = exp2_hw(t[u][e >> 2][e & 3] - lse2[u]);
        }
        // targets: p - q from the t that was kept exactly
        if (!a.q) {
          const int want = id[u] - v;
          const float y = (T16 ? exp2_hw(tt[u] - lse2[u]) : 0.0f) - 1.0f;
#pragma unroll
          for (int e = 0; e < S; ++e)
            if (want == e) d[e] = T16 ? y : d[e] - 1.0f;
        } else {
          for (int k0 = 0; k0 < a.k; k0 += 64) {
            int32_t ids = id[u];
            float qs = q[u], ts = tt[u];
            if (k0) {
              const int at = k0 + lane;
              ids = at < a.k ? a.index[row * a.k + at] : -1;
              qs = at < a.k ? a.q[row * a.k + at] : 0.0f;
              ts = T16 && at < a.k ? a.tt[r * a.k + at] : 0.0f;
            }
            const float y = T16 ? exp2_hw(ts - lse2[u]) - qs : qs;
            uint64_t hits = __ballot(ids >= v0 && ids < v0 + 64 * S);
            while (hits) {
              const int l = __builtin_ctzll(hits);
              hits &= hits - 1;
              const int want = __builtin_amdgcn_readlane(ids, l) - v0;
              const float yy = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(y), l));
#pragma unroll
              for (int e = 0; e < S; ++e)
                if (want == lane * S + e) d[e] = T16 ? yy : d[e] - yy;
            }
          }
        }
#pragma unroll
        for (int e = 0; e < S; ++e) {
          d[e] = v + e < a.V ? d[e] * wr : 0.0f;
          sum[e] += d[e];
        }
      }
      if (mine) {
        uint16_t o[P][S];
#pragma unroll
        for (int e = 0; e < S; ++e) {
          uint16_t x[P];
          to_planes<TYPE, P>(d[e] * SHIFT, x);
#pragma unroll
          for (int p = 0; p < P; ++p) o[p][e] = x[p];
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
          *reinterpret_cast<uint4*>(a.dz + p * a.d_plane + r * a.Vp + v) = *reinterpret_cast<const uint4*>(o[p]);
      }
    }
  }
  if (!mine) return;
#pragma unroll
  for (int e = 0; e < S; e += 4)
    *reinterpret_cast<f32x4*>(a.dbp + rb * a.Vp + v + e) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
}

// ---- dh and dw ----
// Where a product's result goes: out [n][m] of the operands' type, times scale
// and G, or fp32 sums of one split (added to what an earlier piece left there).
struct ProductOut {
  void* out;
  int type;
  OutScale scale;
  const float* gpart;
  float* part;       // [splits][N][M], or null
  int add;           // part holds sums of earlier pieces
  int last;          // with one split: the result goes to out
  int64_t M, N;
};

__device__ __forceinline__ void store_typed(void* out, int type, int64_t i, float x) {
  if (type == RENO_T_FP32) static_cast<float*>(out)[i] = x;
  else static_cast<uint16_t*>(out)[i] = type == RENO_T_BF16 ? to_bf16(x) : to_fp16(x);
}

template <int BM, int BN, int WM, int WN, bool ACOL, bool BCOL, bool HALF>
__global__ void __launch_bounds__(WM* WN * 64) k_head_product(Operand A, Operand B, int64_t K, TileOrder order, Terms terms,
                                                              ProductOut o) {
  using Tile = GemmTile<BM, BN, WM, WN, ACOL, BCOL, HALF>;
  __shared__ __attribute__((aligned(1024))) char lds[Tile::LDS];
  int tm, tn, split;
  order.at(blockIdx.x, gridDim.x, tm, tn, split);
  const int64_t steps = (K + GEMM_BK - 1) / GEMM_BK;
  const int64_t each = (steps + order.splits - 1) / order.splits;
  const int64_t k0 = min(steps, split * each) * GEMM_BK, k1 = min(steps, (split + 1) * each) * GEMM_BK;
  f32x4 acc[Tile::MF][Tile::NF];
  Tile::run(lds, A, B, (int64_t)tm * BM, (int64_t)tn * BN, k0, k1, terms, acc);
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const int l15 = lane & 15, g = lane >> 4;
  const int64_t m0 = (int64_t)tm * BM + (wave / WN) * (BM / WM);
  const int64_t n0 = (int64_t)tn * BN + (wave % WN) * (BN / WN);
  const OutScale scale = with_weights(o.scale, o.gpart);
  float* part = o.part ? o.part + split * o.M * o.N : nullptr;
  const bool typed = !o.part || (o.last && order.splits == 1);
  const bool add = part && o.add;
  // pieces of 4 outputs a lane, where they are aligned
  const bool wide = o.M % 4 == 0 && (!typed || (uintptr_t)o.out % (o.type == RENO_T_FP32 ? 16 : 8) == 0);
  // 16 PR rows n at a time through the wave's share of LDS: lanes hold 16 rows of 4 outputs each, memory wants
  // whole lines of one row
  constexpr int MW = BM / WM, PR = 16384 / (MW * 4) / 16, LR = MW / 4;   // LR lanes a row
  static_assert(Tile::LDS >= WM * WN * 16384 && Tile::NF % PR == 0, "a wave's share of LDS holds 16 PR rows");
  char* mine = lds + wave * 16384;
#pragma unroll
  for (int j0 = 0; j0 < Tile::NF; j0 += PR) {
#pragma unroll
    for (int j = 0; j < PR; ++j)
#pragma unroll
      for (int i = 0; i < Tile::MF; ++i)   // pieces of 16 bytes, spread over the banks by the row
        *reinterpret_cast<f32x4*>(mine + (16 * j + l15) * (MW * 4) + (((4 * i + g) ^ l15) * 16)) = acc[i][j0 + j];
    wave_lds_fence();
    if (wide) {
#pragma unroll 4
      for (int r = lane / LR; r < 16 * PR; r += 64 / LR) {
        const int64_t n = n0 + 16 * j0 + r, m = m0 + 4 * (lane % LR), at = n * o.M + m;
        if (n >= o.N || m >= o.M) continue;
        f32x4 x = *reinterpret_cast<const f32x4*>(mine + r * (MW * 4) + (((lane % LR) ^ (r & 15)) * 16));
        if (add) x += *reinterpret_cast<const f32x4*>(part + at);
        if (!typed) {
          *reinterpret_cast<f32x4*>(part + at) = x;
        } else if (o.type == RENO_T_FP32) {
          f32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = scaled(x[e], scale);
          *reinterpret_cast<f32x4*>(static_cast<float*>(o.out) + at) = y;
        } else {
          uint16_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) h[e] = o.type == RENO_T_BF16 ? to_bf16(scaled(x[e], scale)) : to_fp16(scaled(x[e], scale));
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(o.out) + at) = *reinterpret_cast<const uint2*>(h);
        }
      }
    } else {
#pragma unroll 4
      for (int r = 0; r < 16 * PR; ++r)
#pragma unroll
        for (int i = 0; i < MW / 64; ++i) {
          const int c = lane + 64 * i;
          const int64_t n = n0 + 16 * j0 + r, m = m0 + c, at = n * o.M + m;
          if (n >= o.N || m >= o.M) continue;
          float x = *reinterpret_cast<const float*>(mine + r * (MW * 4) + (((c >> 2) ^ (r & 15)) * 16) + (c & 3) * 4);
          if (add) x += part[at];
          if (typed) store_typed(o.out, o.type, at, scaled(x, scale));
          else part[at] = x;
        }
    }
    wave_lds_fence();
  }
}

// out[i] = scale G (sum over s of part[s][i]), i < n; rows of `width` values of which `cols` are stored
__global__ void __launch_bounds__(256) k_head_reduce(const float* __restrict__ part, int64_t count, int64_t n, void* out,
                                                     int type, OutScale scale, const float* __restrict__ gpart) {
  const OutScale s = with_weights(scale, gpart);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float x = 0.0f;
    for (int64_t p = 0; p < count; ++p) x += part[p * n + i];
    store_typed(out, type, i, scaled(x, s));
  }
}

// Column sums of dz: acc[v] (+)= sum over the piece's row blocks, four lanes'
// worth of blocks at a time; the last piece stores db.
__global__ void __launch_bounds__(256) k_head_db(const float* __restrict__ dbp, int64_t blocks, int64_t Vp, int V,
                                                 float* __restrict__ acc, int add, int last, void* out, int type, OutScale scale,
                                                 const float* __restrict__ gpart) {
  __shared__ float s[4][64];
  const OutScale sc = with_weights(scale, gpart);
  const int lane = lane_id(), w = threadIdx.x >> 6;
  const int64_t v = (int64_t)blockIdx.x * 64 + lane;
  float x = 0.0f;
#pragma unroll 8
  for (int64_t b = w; b < blocks; b += 4) x += dbp[b * Vp + v];
  s[w][lane] = x;
  __syncthreads();
  if (w != 0) return;
  x = s[0][lane] + s[1][lane] + s[2][lane] + s[3][lane];
  if (add) x += acc[v];
  if (!last) acc[v] = x;
  else if (v < V) store_typed(out, type, v, scaled(x, sc));
}

__global__ void __launch_bounds__(256) k_head_zero(void* out, int64_t bytes) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < bytes / 2; i += (int64_t)gridDim.x * 256)
    static_cast<uint16_t*>(out)[i] = 0;
}

// ---------------------------------------------------------------------------
// Host: the sizes of a call and where its scratch lies.

int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

int64_t tiles_of(bool big, int64_t M, int64_t N) {
  const int64_t b = big ? 256 : 128;
  return ((M + b - 1) / b) * ((N + b - 1) / b);
}

// Tiles of 256 x 256 by 8 waves, one block a CU, or of 128 x 128 by 4 waves, two a CU: 512 of these are half the work
// of 256 of the others.  Both reach the same rate when all CUs are full, so that what counts is how much of
// the last turn is used (dw of 1021 x 1000 x 50021, 784 or 3128 tiles: 228 and 206 us); even, the large ones
// move less.
bool big_tiles(int64_t M, int64_t N) {
  return (tiles_of(true, M, N) + 255) / 256 * 2 <= (tiles_of(false, M, N) + 511) / 512;
}

// Splits of k where the outputs' tiles leave most of the chip idle, none shorter than 8 steps.  A split costs a
// write and a read of fp32 sums: not for tiles that fill more than half a turn (dw of 1024 x 512 x 50000,
// 392 tiles: 190 us in two splits, 80 in one).
int splits_for(bool big, int64_t tiles, int64_t K, int terms) {
  const int64_t steps = (K + GEMM_BK - 1) / GEMM_BK * terms;
  const int64_t s = std::min<int64_t>((big ? 256 : 512) / tiles, steps / 8);
  return (int)std::max<int64_t>(1, std::min<int64_t>(s, 256));
}

// Symbols a block of k_head_few takes; 0: not for this call.
int few_width(const reno_head& p, bool grad) {
  if (grad || p.rows > FEW_ROWS || (int64_t)(p.rows <= 1 ? 1 : 4) * p.channels > FEW_H) return 0;
  return p.symbols >= 32768 ? 128 : 64;
}

struct Plan {
  int planes, dz_planes;
  int64_t Cp, Vp, Vb;   // Vb: padded to whole tiles
  int64_t R;            // rows of a piece
  int64_t pieces;
  int part_width;       // symbols of one part
  int dz_rows;
  bool big1, big2, big3;
  int split2, split3;
  // offsets into the workspace
  int64_t idx, q, ent, flag, narrow, bias, wp, gpart, hp, part, tt, lse2, t, dz, dbp, dba, dhp, dwp, bytes;
};

// Whether the products read w where it lies.  Its rows must start on 16 bytes; what they read past V (k is taken in
// steps of BK) meets zeros of dz, and is the next row's start, whose NaN would be everywhere already: only
// without a gap between the rows, of which nothing is known.
bool w_in_place(const reno_head& p, const void* w) {
  return p.type != RENO_T_FP32 && (p.symbols % GEMM_BK == 0 || p.w_stride == p.symbols) && p.w_stride % 8 == 0 &&
         p.w_stride <= GEMM_MAX_LD && (uintptr_t)w % 16 == 0;
}

Plan make_plan(const reno_head& p, int k, bool grad) {
  Plan a{};
  const int64_t N = std::max<int64_t>(p.rows, 1);
  int64_t at = 0;
  const auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at += up(bytes, 256);
    return o;
  };
  a.idx = take(N * k * 4);
  a.q = take(N * k * 4);
  a.ent = take(N * 4);
  a.flag = take(N);
  if (head_is_narrow(p)) {
    a.gpart = take(GPARTS * 4);
    a.narrow = at;
    a.bytes = at + std::max<int64_t>(256, head_narrow_bytes(p, grad));
    return a;
  }
  if (const int few = few_width(p, grad)) {
    a.part_width = few;
    a.part = take((p.symbols + few - 1) / few * N * 8);
    a.tt = take(N * k * 4);
    a.lse2 = take(N * 4);
    a.bytes = at;
    return a;
  }
  a.planes = planes_of(p.type);
  // A second plane of dz for few rows: with many, the roundings of dz average out and leave as much as that of the
  // result; in one row that of the target's dz is the whole result's.  Up to 16 rows the products wait for w and dw
  // (1 x 2048 x 65536 bf16: 280 us; 17 rows, with one plane, 251).
  a.dz_planes = p.type == RENO_T_FP32 ? 3 : p.rows <= 16 ? 2 : 1;
  const int dz_terms = p.type == RENO_T_FP32 ? TERMS_FP32.n : a.dz_planes;
  a.Cp = up(p.channels, GEMM_BK);
  a.Vp = up(p.symbols, GEMM_BK);
  a.Vb = up(p.symbols, 256);
  // A piece: at most 2^28 logits (2^27 in fp32) where they are kept for the gradient, 2^32 where they are not, and
  // 2^31 bytes of what is copied of a row (h as planes, its targets' t): with few symbols h is the larger part.
  const int64_t most = !grad ? int64_t(1) << 32 : p.type == RENO_T_FP32 ? int64_t(1) << 27 : int64_t(1) << 28;
  const int64_t copied = a.planes * a.Cp * 2 + 4 * (int64_t)k;
  const int64_t R = std::max<int64_t>(256, std::min(most / a.Vp, (int64_t(1) << 31) / copied) / 256 * 256);
  a.pieces = (N + R - 1) / R;
  a.R = std::min(N, up((N + a.pieces - 1) / a.pieces, 256));
  a.pieces = (N + a.R - 1) / a.R;
  // Rows of a wave of k_head_dz: 64, so that the column sums it leaves are few, or fewer down to 4 where that would
  // leave less than 4 waves a SIMD (100 x 8000 bf16: 51 us with 64 rows)
  a.dz_rows = 64;
  while (a.dz_rows > 4 && (a.Vp + DZ_COLS - 1) / DZ_COLS * ((a.R + a.dz_rows - 1) / a.dz_rows) < 4096) a.dz_rows /= 2;
  a.big1 = big_tiles(p.symbols, a.R);
  a.big2 = big_tiles(p.channels, a.R);
  a.big3 = big_tiles(p.symbols, p.channels);
  a.part_width = a.big1 ? 128 : 64;
  const int64_t parts = (p.symbols + a.part_width - 1) / a.part_width;
  a.split2 = splits_for(a.big2, tiles_of(a.big2, p.channels, a.R), a.Vp, dz_terms);
  a.split3 = splits_for(a.big3, tiles_of(a.big3, p.symbols, p.channels), a.R, dz_terms);
  a.bias = take(a.Vb * 4);
  a.wp = take(a.planes * (int64_t)p.channels * a.Vp * 2);
  a.gpart = take(GPARTS * 4);
  a.hp = take(a.planes * a.R * a.Cp * 2);
  a.part = take(parts * a.R * 8);
  a.tt = take(a.R * k * 4);
  a.lse2 = take(a.R * 4);
  if (grad) {
    a.t = p.type == RENO_T_BF16 ? at : take(a.R * a.Vp * 4);
    a.dz = take(a.dz_planes * a.R * a.Vp * 2);
    a.dbp = take((a.R + a.dz_rows - 1) / a.dz_rows * a.Vp * 4);
    a.dba = take(a.Vp * 4);
    a.dhp = a.split2 > 1 ? take(a.split2 * a.R * p.channels * 4) : at;
    a.dwp = a.split3 > 1 || a.pieces > 1 ? take((int64_t)a.split3 * p.channels * p.symbols * 4) : at;
  }
  a.bytes = at;
  return a;
}

unsigned blocks_for(int64_t n, int64_t per, int64_t most = 8192) {
  return (unsigned)std::max<int64_t>(1, std::min(most, (n + per - 1) / per));
}

template <bool HALF>
void run_logits(const HeadArgs& a, const Operand& W, const Operand& H, bool big, Terms terms, hipStream_t st) {
  const int64_t b = big ? 256 : 128;
  const TileOrder o{(int)((a.V + b - 1) / b), (int)((a.R + b - 1) / b), 1};
  const dim3 grid((unsigned)((int64_t)o.tm * o.tn));
  if (big) hipLaunchKernelGGL((k_head_logits<256, 256, 2, 4, HALF>), grid, dim3(512), 0, st, a, W, H, o, terms);
  else hipLaunchKernelGGL((k_head_logits<128, 128, 2, 2, HALF>), grid, dim3(256), 0, st, a, W, H, o, terms);
}

template <bool ACOL, bool BCOL, bool HALF>
void run_product(const Operand& A, const Operand& B, int64_t K, bool big, int splits, Terms terms, const ProductOut& po,
                 hipStream_t st) {
  const int64_t b = big ? 256 : 128;
  const TileOrder o{(int)((po.M + b - 1) / b), (int)((po.N + b - 1) / b), splits};
  const dim3 grid((unsigned)((int64_t)o.tm * o.tn * splits));
  if (big)
    hipLaunchKernelGGL((k_head_product<256, 256, 2, 4, ACOL, BCOL, HALF>), grid, dim3(512), 0, st, A, B, K, o, terms, po);
  else
    hipLaunchKernelGGL((k_head_product<128, 128, 2, 2, ACOL, BCOL, HALF>), grid, dim3(256), 0, st, A, B, K, o, terms, po);
}

template <int TYPE>
hipError_t run_head(const HeadCall& c, hipStream_t st) {
  constexpr bool HALF = TYPE == RENO_T_FP16;
  const reno_head& p = c.p;
  const int64_t N = p.rows;
  const int size = TYPE == RENO_T_FP32 ? 4 : 2;
  if (N == 0) {  // nothing reaches the weights
    const auto zero = [&](void* out, int64_t n) {
      if (out) hipLaunchKernelGGL(k_head_zero, dim3(blocks_for(n * size / 2, 256)), dim3(256), 0, st, out, n * size);
    };
    zero(c.d.dw, (int64_t)p.channels * p.symbols);
    zero(c.d.db, p.symbols);
    return hipGetLastError();
  }
  const Plan pl = make_plan(p, c.k, c.grad);
  char* ws = c.ws;
  HeadTargets t{c.index, nullptr, nullptr, nullptr};
  if (c.logit) {
    int32_t* idx = reinterpret_cast<int32_t*>(ws + pl.idx);
    float* q = reinterpret_cast<float*>(ws + pl.q);
    float* ent = reinterpret_cast<float*>(ws + pl.ent);
    uint8_t* flag = reinterpret_cast<uint8_t*>(ws + pl.flag);
    const int per = c.k <= 16 ? 16 : c.k <= 32 ? 8 : 4;   // rows a block
    const auto args = [&](auto kern) {
      for (int64_t r = 0; r < N; r += LAUNCH_ROWS) {
        const int64_t n = std::min(LAUNCH_ROWS, N - r);
        hipLaunchKernelGGL(kern, dim3((unsigned)((n + per - 1) / per)), dim3(256), 0, st, c.index + r * c.k,
                           c.logit + r * c.k, n, c.k, p.symbols, (float)(1.4426950408889634 / (double)c.temperature),
                           idx + r * c.k, q + r * c.k, ent + r, flag + r);
      }
    };
    if (c.k <= 16) args(k_head_targets<16, 1>);
    else if (c.k <= 32) args(k_head_targets<32, 1>);
    else if (c.k <= 64) args(k_head_targets<64, 1>);
    else args(k_head_targets<64, 2>);
    t = HeadTargets{idx, q, ent, flag};
  }
  HeadArgs a{};
  a.N = N;
  a.C = p.channels;
  a.V = p.symbols;
  a.k = c.k;
  a.g = c.d.row_weight;
  a.index = t.index;
  a.q = t.q;
  a.ent = t.ent;
  a.flag = t.flag;
  if (head_is_narrow(p)) {
    // These carry dz as g (p - q), as long as 1 / T leaves that within 2^24 of the gradients' own size; beyond,
    // over the largest weight too (233737 x 32 x 256, 16 entries a row: 187 us for 180).
    const bool far = c.grad && c.d.row_weight && !(c.temperature >= 0x1p-24f && c.temperature <= 0x1p24f);
    float* gpart = far ? reinterpret_cast<float*>(ws + pl.gpart) : nullptr;
    if (far)
      hipLaunchKernelGGL(k_head_setup<TYPE>, dim3(GPARTS), dim3(256), 0, st, a, SetupBlocks{0, GPARTS, 0, 0}, int64_t(0), gpart);
    return launch_head_narrow(c, t, gpart, ws + pl.narrow, st);
  }
  a.Cp = pl.Cp;
  a.Vp = pl.Vp;
  a.h_stride = p.h_stride;
  a.w_stride = p.w_stride;
  a.h = c.d.h;
  a.w = c.d.w;
  a.b = c.d.b;
  a.scale = (float)(1.4426950408889634 / (double)c.temperature);
  a.bias = reinterpret_cast<float*>(ws + pl.bias);
  a.hp = reinterpret_cast<uint16_t*>(ws + pl.hp);
  a.wp = reinterpret_cast<uint16_t*>(ws + pl.wp);
  a.h_plane = pl.R * pl.Cp;
  a.w_plane = (int64_t)p.channels * pl.Vp;
  a.d_plane = pl.R * pl.Vp;
  a.part = reinterpret_cast<float2*>(ws + pl.part);
  a.parts = (p.symbols + pl.part_width - 1) / pl.part_width;
  a.part_width = pl.part_width;
  a.dz_rows = pl.dz_rows;
  a.tt = reinterpret_cast<float*>(ws + pl.tt);
  a.lse2 = reinterpret_cast<float*>(ws + pl.lse2);
  a.bits = c.d.bits;
  a.lse = c.d.lse;
  if (const int few = few_width(p, c.grad)) {
    const dim3 grid((unsigned)a.parts);
    a.R = N;
    const auto args = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(512), 0, st, a); };
    if (few == 128) N <= 1 ? args(k_head_few<TYPE, 128, 1>) : args(k_head_few<TYPE, 128, 4>);
    else N <= 1 ? args(k_head_few<TYPE, 64, 1>) : args(k_head_few<TYPE, 64, 4>);
    hipLaunchKernelGGL(k_head_rows, dim3((unsigned)((N + 15) / 16)), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  if (c.grad) {
    a.dz = reinterpret_cast<uint16_t*>(ws + pl.dz);
    if (TYPE == RENO_T_BF16) a.t16 = a.dz;
    else a.t = reinterpret_cast<float*>(ws + pl.t);
    a.dbp = reinterpret_cast<float*>(ws + pl.dbp);
    if (c.d.row_weight) a.gpart = reinterpret_cast<float*>(ws + pl.gpart);
  }
  const bool in_place = w_in_place(p, c.d.w);
  a.R = std::min(pl.R, N);
  const SetupBlocks sb{blocks_for(a.R * a.Cp / 8, 256, 2048), a.gpart ? (unsigned)GPARTS : 0u, (unsigned)(pl.Vb / 256),
                       in_place ? 0u : blocks_for(a.C * a.Vp / 8, 256)};
  hipLaunchKernelGGL(k_head_setup<TYPE>, dim3(sb.h + sb.g + sb.b + sb.w), dim3(256), 0, st, a, sb, pl.Vb,
                     a.gpart ? reinterpret_cast<float*>(ws + pl.gpart) : nullptr);
  const int64_t wl = in_place ? p.w_stride : pl.Vp;
  const Operand W{in_place ? static_cast<const uint16_t*>(c.d.w) : a.wp, wl, p.channels,
                  (p.channels - 1) * wl + (in_place ? p.symbols : pl.Vp), a.w_plane};
  const OutScale scale = out_scale(c.temperature);
  const OutScale scale_d{scale.mant, scale.exp - (HALF ? HALF_SHIFT : 0)};
  for (int64_t i = 0; i < pl.pieces; ++i) {
    a.r0 = i * pl.R;
    a.R = std::min(pl.R, N - a.r0);
    const bool last = i + 1 == pl.pieces;
    if (i > 0) hipLaunchKernelGGL(k_head_pack_h<TYPE>, dim3(blocks_for(a.R * a.Cp / 8, 256)), dim3(256), 0, st, a);
    const Operand H{a.hp, pl.Cp, a.R, a.R * pl.Cp, a.h_plane};
    run_logits<HALF>(a, W, H, pl.big1, TYPE == RENO_T_FP32 ? TERMS_FP32 : TERMS_ONE, st);
    hipLaunchKernelGGL(k_head_rows, dim3((unsigned)((a.R + 15) / 16)), dim3(256), 0, st, a);
    if (!c.grad) continue;
    const int64_t row_blocks = (a.R + a.dz_rows - 1) / a.dz_rows;
    const Terms dz_b = TYPE == RENO_T_FP32 ? TERMS_FP32 : pl.dz_planes == 2 ? TERMS_B2 : TERMS_ONE;   // dz the second operand
    const Terms dz_a = TYPE == RENO_T_FP32 ? TERMS_FP32 : pl.dz_planes == 2 ? TERMS_A2 : TERMS_ONE;   // the first
    constexpr bool F32 = TYPE == RENO_T_FP32;
    const auto make_dz = pl.dz_planes == 1 ? k_head_dz<TYPE, F32 ? 3 : 1> : k_head_dz<TYPE, F32 ? 3 : 2>;
    hipLaunchKernelGGL(make_dz, dim3((unsigned)(((a.Vp + DZ_COLS - 1) / DZ_COLS * row_blocks + 3) / 4)), dim3(256), 0, st, a);
    const Operand D{a.dz, pl.Vp, a.R, a.R * pl.Vp, a.d_plane};
    if (c.d.dh) {
      void* out = static_cast<char*>(c.d.dh) + a.r0 * p.channels * size;
      float* part = reinterpret_cast<float*>(ws + pl.dhp);
      const ProductOut po{out, TYPE, scale_d, a.gpart, pl.split2 > 1 ? part : nullptr, 0, 1, p.channels, a.R};
      run_product<false, false, HALF>(W, D, a.Vp, pl.big2, pl.split2, dz_b, po, st);
      if (pl.split2 > 1)
        hipLaunchKernelGGL(k_head_reduce, dim3(blocks_for(a.R * a.C, 256)), dim3(256), 0, st, part, (int64_t)pl.split2,
                           a.R * a.C, out, TYPE, scale_d, a.gpart);
    }
    if (c.d.dw) {
      float* part = reinterpret_cast<float*>(ws + pl.dwp);
      const bool keep = pl.split3 > 1 || pl.pieces > 1;
      const ProductOut po{c.d.dw, TYPE, scale_d, a.gpart, keep ? part : nullptr, i > 0, last, p.symbols, p.channels};
      run_product<true, true, HALF>(D, H, a.R, pl.big3, pl.split3, dz_a, po, st);
      if (last && pl.split3 > 1)
        hipLaunchKernelGGL(k_head_reduce, dim3(blocks_for((int64_t)a.C * a.V, 256)), dim3(256), 0, st, part,
                           (int64_t)pl.split3, (int64_t)a.C * a.V, c.d.dw, TYPE, scale_d, a.gpart);
    }
    if (c.d.db)
      hipLaunchKernelGGL(k_head_db, dim3((unsigned)(a.Vp / 64)), dim3(256), 0, st, a.dbp, row_blocks, a.Vp, a.V,
                         reinterpret_cast<float*>(ws + pl.dba), (int)(i > 0), (int)last, c.d.db, TYPE, scale, a.gpart);
  }
  return hipGetLastError();
}

}  // namespace

int64_t head_workspace(const reno_head& p, int k, bool grad) { return make_plan(p, k, grad).bytes; }

hipError_t launch_head(const HeadCall& c, hipStream_t st) {
  switch (c.p.type) {
    case RENO_T_FP32: return run_head<RENO_T_FP32>(c, st);
    case RENO_T_BF16: return run_head<RENO_T_BF16>(c, st);
    default: return run_head<RENO_T_FP16>(c, st);
  }
}

}  // namespace reno
