// Matrix product core of the head's training operators (gfx950): the tile of
// D[m][n] = sum_k A(m, k) B(n, k) that one block computes on bf16 or fp16 MFMA
// with fp32 sums.
//
// Either operand may lie with k contiguous (rows m, "by rows") or with m
// contiguous (rows k, "by columns"): the products of a head and its gradient
// (h w, dz w^T, h^T dz) need all of these, and a copy of a transposed operand
// would cost as much traffic as the product itself.  Tiles go from memory to
// LDS without passing registers (buffer loads to LDS, 16 bytes a lane), two
// stages of BK values of k deep; a tile by columns is read back transposed
// (ds_read_b64_tr_b16).
//
// LDS layouts.  The loads write a wave's 64 pieces of 16 bytes to consecutive
// LDS, so the order that avoids bank conflicts is made by which piece a lane
// loads:
//  by rows     row m of 128 bytes (BK = 64 values), piece c of it at place
//              c ^ (m & 7): the 8 lanes that read one piece each of 8 rows
//              (ds_read_b128) cover all banks;
//  by columns  row k of 2 BT bytes, its 32-byte slot s at place s ^ f(k),
//              f(k) = (k & 3) | (k >> 3 & 1) << 2: a transposed read takes one
//              slot of each of 16 rows k, which fall on 8 places.
//
// Rates (MI355X): 256 x 256 tiles of 8 waves and two blocks a CU of 128 x 128 tiles of 4 waves both reach
// 990 to 1220 TFLOP/s of bf16 where the grid fills the chip; a large product of the library's 1207.
//
// Bounds.  A buffer's size field ends at the operand's last row, so what a tile
// reaches past it reads as zero; rows of an operand by rows are clamped as well.
// Pieces past an operand's columns but inside its rows belong to outputs that
// are not stored (by columns) or are zero in memory (by rows: k is padded to a
// multiple of BK with zeros by whoever laid the operand out).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace reno {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int GEMM_BK = 64;

// An operand in memory: `rows` rows of 16-bit values `ld` apart (a multiple of
// 8, at most GEMM_MAX_LD), `size` values from its first to its last, and how
// far its planes are apart.
struct Operand {
  const uint16_t* p;
  int64_t ld;
  int64_t rows;
  int64_t size;
  int64_t plane;
};
constexpr int64_t GEMM_MAX_LD = int64_t(1) << 22;  // 256 rows inside 32-bit offsets

// The products of planes that make one product: plane a (b) of term t in bits 2 t, 2 t + 1.  They follow
// one another for each step of k, so that a plane read again is still in L2.
struct Terms {
  uint32_t a, b;
  int n;
};
// fp32 operands are three bf16 planes x = x0 + x1 + x2 (8 bits each, cut off: x1 below 2^-7 of x0, x2 below 2^-15), and
// six of the nine products are taken, smallest first.  x1 y2, x2 y1 and x2 y2, left out, are below 2^-21 of the whole
// together, 2^-24.6 on average, and of its sign; the heads measured err
// by 2e-7 to 6e-7 in all, plain float32 sums by 2e-7 to 2.3e-6.
constexpr Terms TERMS_FP32{0x052, 0x118, 6};   // 2 0 1 1 0 0 by 0 2 1 0 1 0
constexpr Terms TERMS_ONE{0, 0, 1};
constexpr Terms TERMS_A2{1, 0, 2}, TERMS_B2{0, 1, 2};   // two planes of one operand, the lower first

template <bool HALF>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (HALF)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// 16 bytes a lane from the buffer at voff + soff to LDS at lds + 16 lane.  The
// compiler does not count these loads: every use waits for them itself.
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t voff, i32x4 srd) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %1, %2, 0 offen lds"
      :
      : "s"(lds), "v"(voff), "s"(srd)
      : "memory");
}

// This wave's loads to LDS have landed and its LDS reads are done, and every
// other wave's too.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}

// Loads of one operand's tile of BT rows (of m or n) and BK values of k by NW waves.
template <int BT, bool COL, int NW>
struct TileLoad {
  static constexpr int NI = BT * GEMM_BK * 2 / 1024 / NW;  // loads of a wave
  static_assert(NI * NW * 1024 == BT * GEMM_BK * 2, "a tile is a whole number of loads");
  uint32_t voff[NI];
  int64_t left;         // bytes from the tile's first value to the operand's end
  const uint16_t* base;

  // first: first row of m (or n) of the tile
  __device__ __forceinline__ void init(const Operand& op, int64_t first, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int idx = wave * NI + i;
      if constexpr (COL) {
        constexpr int PIECES = BT / 8;  // 16-byte pieces of a row
        const int k = idx * (64 / PIECES) + lane / PIECES;
        const int pc = lane % PIECES;
        const int f = (k & 3) | ((k >> 3 & 1) << 2);
        const int c = (((pc >> 1) ^ f) << 1) | (pc & 1);
        voff[i] = (uint32_t)(k * (uint32_t)op.ld * 2u + c * 16u);
      } else {
        const int m = idx * 8 + (lane >> 3);
        const int64_t last = op.rows - 1 - first;
        const uint32_t row = (uint32_t)(m < last ? m : last);
        const int c = (lane & 7) ^ (m & 7);
        voff[i] = row * (uint32_t)op.ld * 2u + c * 16u;
      }
    }
    const int64_t off = COL ? first : first * op.ld;
    base = op.p + off;
    left = (op.size - off) * 2;
  }

  // the tile's values of k from k0 on, of the plane at `plane`
  __device__ __forceinline__ void issue(const Operand& op, int64_t plane, int64_t k0, uint32_t lds, int wave) const {
    const int64_t adv = COL ? k0 * op.ld : k0;
    const uint64_t a = (uint64_t)(base + plane + adv);
    int64_t size = left - adv * 2;
    size = size < 0 ? 0 : size > 0xfffffff0ll ? 0xfffffff0ll : size;
    i32x4 srd;
    srd[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    srd[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xffff);
    srd[2] = __builtin_amdgcn_readfirstlane((int)(uint32_t)size);
    srd[3] = 0x00020000;
#pragma unroll
    for (int i = 0; i < NI; ++i) load_to_lds(lds + (wave * NI + i) * 1024, voff[i], srd);
  }
};

// Reads the 16 x 32 fragments of NF consecutive groups of 16 rows (of m or n)
// from a tile in LDS: lane l holds row l & 15, values k = 8 (l >> 4) .. + 7.
template <int BT, bool COL, int NF>
struct TileRead {
  uint32_t off[COL ? NF : 2];
  __device__ __forceinline__ void init(int first, int lane) {
    const int l15 = lane & 15, g = lane >> 4;
    if constexpr (COL) {
      const int f = (l15 >> 2) | ((g & 1) << 2);
      const int k = 8 * g + (l15 >> 2);
#pragma unroll
      for (int i = 0; i < NF; ++i) off[i] = k * (BT * 2) + (((first >> 4) + i) ^ f) * 32 + (l15 & 3) * 8;
    } else {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) off[kk] = (first + l15) * 128 + ((kk * 4 + g) ^ (l15 & 7)) * 16;
    }
  }
  __device__ __forceinline__ s16x8 get(const char* tile, int i, int kk) const {
    if constexpr (COL) {
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const char* p = tile + off[i] + kk * 32 * (BT * 2);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + 4 * (BT * 2)));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *reinterpret_cast<const s16x8*>(tile + off[kk] + i * 16 * 128);
    }
  }
};

// One block's tile: acc[i][j] of the wave (wm, wn) holds rows m = 16 i + 4 (lane
// >> 4) + e, columns n = 16 j + (lane & 15) of its part.  k runs over [k0, k1) in steps
// of BK, for each the products of planes `terms`.
template <int BM, int BN, int WM, int WN, bool ACOL, bool BCOL, bool HALF>
struct GemmTile {
  static constexpr int NW = WM * WN, MF = BM / WM / 16, NF = BN / WN / 16;
  static constexpr int STAGE = (BM + BN) * GEMM_BK * 2;
  static constexpr int LDS = 2 * STAGE;

  __device__ static __forceinline__ void run(char* lds, const Operand& A, const Operand& B, int64_t m0, int64_t n0,
                                             int64_t k0, int64_t k1, Terms terms, f32x4 (&acc)[MF][NF]) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    TileLoad<BM, ACOL, NW> la;
    TileLoad<BN, BCOL, NW> lb;
    la.init(A, m0, wave, lane);
    lb.init(B, n0, wave, lane);
    TileRead<BM, ACOL, MF> ra;
    TileRead<BN, BCOL, NF> rb;
    ra.init(wm * (BM / WM), lane);
    rb.init(wn * (BN / WN), lane);
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const uint32_t lds0 = lds_offset(lds);
    const int steps = (int)((k1 - k0) / GEMM_BK) * terms.n;
    int term = 0;
    int64_t k = k0;
    auto issue = [&](int stage) {
      const uint32_t at = lds0 + stage * STAGE;
      la.issue(A, (terms.a >> 2 * term & 3) * A.plane, k, at, wave);
      lb.issue(B, (terms.b >> 2 * term & 3) * B.plane, k, at + BM * GEMM_BK * 2, wave);
      if (++term == terms.n) {
        term = 0;
        k += GEMM_BK;
      }
    };
    if (steps > 0) issue(0);
    for (int s = 0; s < steps; ++s) {
      stage_barrier();
      if (s + 1 < steps) issue((s + 1) & 1);
      const char* ta = lds + (s & 1) * STAGE;
      const char* tb = ta + BM * GEMM_BK * 2;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        s16x8 a[MF], b[NF];
#pragma unroll
        for (int i = 0; i < MF; ++i) a[i] = ra.get(ta, i, kk);
#pragma unroll
        for (int j = 0; j < NF; ++j) b[j] = rb.get(tb, j, kk);
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
          for (int j = 0; j < NF; ++j) acc[i][j] = mfma<HALF>(a[i], b[j], acc[i][j]);
      }
    }
    stage_barrier();
  }
};

// The tile (m, n, split) of a block.  Blocks are dealt to the 8 XCDs in turn, so
// each XCD gets a run of consecutive tiles; inside it 8 tiles of m are taken for
// each of n, so that the 32 blocks an XCD runs at a time share 8 + 4 operand tiles.
struct TileOrder {
  int tm, tn, splits;
  __device__ __forceinline__ void at(uint32_t block, uint32_t blocks, int& m, int& n, int& split) const {
    const uint32_t per = blocks / 8, rest = blocks % 8, x = block % 8;
    uint32_t id = x * per + (x < rest ? x : rest) + block / 8;
    const uint32_t each = (uint32_t)tm * tn;
    split = (int)(id / each);
    id %= each;
    const uint32_t group = id / (8u * tn), first = group * 8u;
    const uint32_t gm = min(8u, (uint32_t)tm - first);
    const uint32_t in = id - group * 8u * tn;
    m = (int)(first + in % gm);
    n = (int)(in / gm);
  }
};

}  // namespace reno
