// Matrix-instruction tiles of the grouped products: C = P Q^T on BM x BN tiles for float32, bfloat16 and float16.
//
// An operand is one of
//   KC  rows of the tile are rows of memory, the summed index consecutive      (x, y's A, dx's dy)
//   KR  rows of the tile are columns of memory, the summed index goes by rows  (dx's A, da's dy and x)
// and is moved to LDS 128 bytes of the summed index a slice (64 values of 16 bits, 32 of 32), 16 bytes a lane
// straight from memory to LDS, past the registers.  What lies outside the operand is fetched at an offset outside
// the buffer, which reads zero.  Rows start at multiples of 16 bytes and widths are multiples of 16 bytes: other
// operands are copied into such a layout first (group_pack_kernel).
//
// LDS: two stages.  KC tiles are [x][128 bytes], the 16-byte group q of row x at q ^ (x & 7); KR tiles are
// [k][x], 16 bits: 32-byte pairs at p ^ f(k) (pieces::kr_f), read four rows at a time by the transposing LDS read;
// 32 bits: 64-byte units at u ^ (k / 4), read a word a lane.  Either way the lanes of a read fall in distinct banks.
#pragma once

#include "operators_device.h"
#include "pieces.h"

namespace tile {

enum { KC = 0, KR = 1 };

template <int TYPE> struct Mfma;
template <> struct Mfma<OT_F32> {
  typedef v4f Frag;          // four k of one row: k = 4 (lane / 16) + 0..3 of 16
  static constexpr int STEPS = 2;
  __device__ __forceinline__ static v4f mul(const Frag& a, const Frag& b, v4f c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};
template <> struct Mfma<OT_BF16> {
  typedef v8bf Frag;         // eight k of one row: k = 8 (lane / 16) + 0..7 of 32
  __device__ __forceinline__ static v4f mul(const Frag& a, const Frag& b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Mfma<OT_F16> {
  typedef v8h Frag;
  __device__ __forceinline__ static v4f mul(const Frag& a, const Frag& b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

// One operand of a workgroup: BX rows of the tile, loaded by NW waves.
template <int TYPE, int MODE, int BX, int NW>
struct Operand {
  static constexpr int ES = TYPE == OT_F32 ? 4 : 2;
  static constexpr int KS = 128 / ES;            // summed index of a slice
  static constexpr int EV = 16 / ES;             // values of 16 bytes
  static constexpr int BYTES = BX * 128;
  static constexpr int MOVES = BX / 8 / NW;      // 1 KB each, a wave's share
  static constexpr int RS = BX * ES / 16;        // KR: 16-byte slots of a row
  static constexpr int UM = BX / 16 - 1 < 3 ? BX / 16 - 1 : 3;
  static constexpr int BL = BX / 64;             // KR, 16 bits: 128-byte blocks of a row
  static_assert(MODE == KC || TYPE == OT_F32 || BX >= 64, "a row of four pairs at least");
  static_assert(BX % (8 * NW) == 0, "whole moves");

  const char* base;
  int64_t step;        // bytes from a slice to the next
  uint32_t off[MOVES];
  uint32_t kat[MOVES]; // the summed index that a move's lane fetches, in its slice
  uint32_t kdim;
  int wave;

  __device__ __forceinline__ static int kr_swizzle(int row) {
    return TYPE == OT_F32 ? (row >> 2) & UM : pieces::kr_f<(BL < 1 ? 1 : BL)>(row);
  }

  // p: the tile's first row (KC: rows ld apart; KR: the first row of the summed index at the tile's first column);
  // xdim: rows that exist
  __device__ __forceinline__ void open(const void* p, int64_t ld, int xdim, int64_t kd, int w, int lane) {
    base = (const char*)p;
    wave = w;
    kdim = (uint32_t)kd;
    step = MODE == KC ? 128 : (int64_t)KS * ld * ES;
#pragma unroll
    for (int j = 0; j < MOVES; ++j) {
      const int inst = w + NW * j;
      if (MODE == KC) {
        const int x = 8 * inst + (lane >> 3), q = (lane & 7) ^ (x & 7);
        kat[j] = q * EV;
        off[j] = x < xdim ? (uint32_t)(x * (uint32_t)(ld * ES) + 16 * q) : pieces::kOob;
      } else {
        const int slot = inst * 64 + lane, row = slot / RS, s = slot % RS;
        const int col = TYPE == OT_F32 ? 16 * ((s >> 2) ^ kr_swizzle(row)) + 4 * (s & 3)
                                       : 16 * ((s >> 1) ^ kr_swizzle(row)) + 8 * (s & 1);
        kat[j] = row;
        off[j] = col < xdim ? (uint32_t)(row * (uint32_t)(ld * ES) + col * ES) : pieces::kOob;
      }
    }
  }

  // slice kt into the stage at lds
  __device__ __forceinline__ void fetch(char* lds, int kt) const {
    const rsrc_t rs = pieces::make_rsrc(base + kt * step);
#pragma unroll
    for (int j = 0; j < MOVES; ++j) {
      const uint32_t o = (uint32_t)kt * KS + kat[j] < kdim ? off[j] : pieces::kOob;
      pieces::dma16(rs, lds + (wave + NW * j) * 1024, o, 0);
    }
  }

  // the 16 rows from 16 blk on, summed indices of step s (half a slice)
  __device__ __forceinline__ static typename Mfma<TYPE>::Frag read(const char* lds, int blk, int s, int lane) {
    typedef typename Mfma<TYPE>::Frag Frag;
    const int l16 = lane & 15, g = lane >> 4;
    if constexpr (MODE == KC) {
      return *(const Frag*)(lds + (16 * blk + l16) * 128 + (((4 * s + g) ^ (l16 & 7)) << 4));
    } else if constexpr (TYPE == OT_F32) {
      Frag f;
      const char* p = lds + (16 * s + 4 * g) * (BX * 4) + ((blk ^ (g & UM)) << 6) + l16 * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = *(const float*)(p + j * BX * 4);
      return f;
    } else {
      const int row = 8 * g + (l16 >> 2);
      const uint32_t at = pieces::lds_offset(lds) + s * 32 * (BX * 2);
      const uint32_t a0 = (uint32_t)(row * BX * 2 + ((kr_swizzle(row) ^ blk) << 5) + (l16 & 3) * 8);
      const uint32_t a1 = (uint32_t)((row + 4) * BX * 2 + ((kr_swizzle(row + 4) ^ blk) << 5) + (l16 & 3) * 8);
      return __builtin_bit_cast(Frag, pieces::kr_fragment(at + a0, at + a1));
    }
  }
};

// A BM x BN tile by WM x WN waves, each (BM / WM) x (BN / WN) of it.
template <int TYPE, int MP, int MQ, int BM, int BN, int WM, int WN>
struct Tile {
  static constexpr int NW = WM * WN;
  static constexpr int IB = BM / WM / 16, JB = BN / WN / 16;   // 16 x 16 blocks of a wave
  typedef Operand<TYPE, MP, BM, NW> P;
  typedef Operand<TYPE, MQ, BN, NW> Q;
  static constexpr int STAGE = P::BYTES + Q::BYTES;
  static constexpr int LDS = 2 * STAGE;
  static constexpr int KS = P::KS;

  // acc[i][j][r]: row 16 i + lane % 16, column 16 j + 4 (lane / 16) + r of the wave's part (Q feeds the matrix
  // instruction's rows, so that a lane holds four consecutive columns of C)
  __device__ __forceinline__ static void run(char* lds, const void* p, int64_t ldp, int rows, const void* q, int64_t ldq,
                                             int cols, int64_t depth, v4f (&acc)[IB][JB]) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = w / WN, wn = w % WN;
    P op;
    Q oq;
    op.open(p, ldp, rows, depth, w, lane);
    oq.open(q, ldq, cols, depth, w, lane);
#pragma unroll
    for (int i = 0; i < IB; ++i)
#pragma unroll
      for (int j = 0; j < JB; ++j) acc[i][j] = (v4f){0.f, 0.f, 0.f, 0.f};
    const int nk = (int)((depth + KS - 1) / KS);
    if (nk == 0) return;
    op.fetch(lds, 0);
    oq.fetch(lds + P::BYTES, 0);
    typename Mfma<TYPE>::Frag fp[2][IB], fq[2][JB];
    auto read = [&](const char* stage, int s) {
#pragma unroll
      for (int j = 0; j < JB; ++j) fq[s][j] = Q::read(stage + P::BYTES, wn * JB + j, s, lane);
#pragma unroll
      for (int i = 0; i < IB; ++i) fp[s][i] = P::read(stage, wm * IB + i, s, lane);
    };
    auto multiply = [&](int s) {
#pragma unroll
      for (int i = 0; i < IB; ++i)
#pragma unroll
        for (int j = 0; j < JB; ++j) acc[i][j] = Mfma<TYPE>::mul(fq[s][j], fp[s][i], acc[i][j]);
    };
    pieces::wait_loads();      // this wave's part of the slice has landed,
    pieces::lds_barrier();     // and everyone's
    read(lds, 0);
    op.fetch(lds + STAGE, 1);
    oq.fetch(lds + STAGE + P::BYTES, 1);
    // Half a slice is multiplied while the next half is read and the slice behind it fetched: one barrier a slice.
    // The last two rounds fetch past the operands, which moves zeros, so that a round is one block of code.
    for (int kt = 0; kt < nk; ++kt) {
      char* now = lds + (kt & 1) * STAGE;
      char* next = lds + (~kt & 1) * STAGE;
      read(now, 1);
      multiply(0);
      interleave<0>();
      __builtin_amdgcn_sched_barrier(0);   // the products stay ahead of the wait
      pieces::wait_loads();    // the next slice has landed
      pieces::lds_barrier();   // everywhere, and `now` has been read
      __builtin_amdgcn_sched_barrier(0);
      read(next, 0);
      op.fetch(now, kt + 2);
      oq.fetch(now + P::BYTES, kt + 2);
      multiply(1);
      interleave<P::MOVES + Q::MOVES>();
      __builtin_amdgcn_sched_barrier(0);
    }
    pieces::wait_loads();      // nothing may still move into this workgroup's LDS
  }

  // spreads the LDS reads and fetches of half a slice between its products
  template <int FETCHES>
  __device__ __forceinline__ static void interleave() {
    constexpr int PRODUCTS = IB * JB * (TYPE == OT_F32 ? 4 : 1);
    constexpr int READS = (MP == KC ? IB : (TYPE == OT_F32 ? 4 : 2) * IB) + (MQ == KC ? JB : (TYPE == OT_F32 ? 4 : 2) * JB);
    constexpr int PER = PRODUCTS / (READS + FETCHES) < 1 ? 1 : PRODUCTS / (READS + FETCHES);
#pragma unroll
    for (int k = 0; k < READS; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);     // an LDS read
      __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);   // products
    }
#pragma unroll
    for (int k = 0; k < FETCHES; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);     // a fetch
      __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
    }
  }

  // rounds the tile to TO and stores it; vec: rows of C start at multiples of four values' bytes
  template <int TO>
  __device__ __forceinline__ static void store(const v4f (&acc)[IB][JB], void* c, int64_t ldc, int rows, int cols, bool vec) {
    typedef typename Elem<TO>::T T;
    typedef T T4 __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r0 = (w / WN) * IB * 16 + (lane & 15), c0 = (w % WN) * JB * 16 + 4 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < IB; ++i) {
      const int row = r0 + 16 * i;
      if (row >= rows) continue;
      T* out = (T*)c + row * ldc;
#pragma unroll
      for (int j = 0; j < JB; ++j) {
        const int col = c0 + 16 * j;
        const v4f v = acc[i][j];
        if (vec && col + 3 < cols) {
          *(T4*)(out + col) = (T4){(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (col + r < cols) out[col + r] = (T)v[r];
        }
      }
    }
  }
};

// Hardware hands workgroups to the eight XCDs in turn, each with an L2 of its own: the workgroup's place such that
// every XCD takes one run of consecutive places.
__device__ __forceinline__ uint32_t xcd_place(uint32_t id, uint32_t n) {
  const uint32_t q = n >> 3, r = n & 7, xcd = id & 7;
  return xcd * q + min(xcd, r) + (id >> 3);
}

}  // namespace tile
