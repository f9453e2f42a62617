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
// LDS: two stages, arrays of their own and named in the code (an LDS read behind a load to LDS otherwise waits for it,
// wherever the two go).  KC tiles are [x][128 bytes], the 16-byte group q of row x at q ^ (x & 7); KR tiles are
// [k][x], 16 bits: 32-byte pairs at p ^ f(k) (pieces::kr_f), read four rows at a time by the transposing LDS read;
// 32 bits: 64-byte units at u ^ (k / 4), read a word a lane.  Either way the lanes of a read fall in distinct banks.
#pragma once

#include "operators_device.h"
#include "pieces.h"

namespace tile {

enum { KC = 0, KR = 1 };

typedef __attribute__((address_space(3))) char lds_t;   // LDS by its own address space, so that an access names its array

template <int TYPE> struct Mfma;
template <> struct Mfma<OT_F32> {
  typedef v4f Frag;          // four k of one row: k = 4 (lane / 16) + 0..3 of 16
  static constexpr int SUB = 4;   // products of a step, one k each
  __device__ __forceinline__ static v4f mul(const Frag& a, const Frag& b, v4f c, int r) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
  }
};
template <> struct Mfma<OT_BF16> {
  typedef v8bf Frag;         // eight k of one row: k = 8 (lane / 16) + 0..7 of 32
  static constexpr int SUB = 1;
  __device__ __forceinline__ static v4f mul(const Frag& a, const Frag& b, v4f c, int) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Mfma<OT_F16> {
  typedef v8h Frag;
  static constexpr int SUB = 1;
  __device__ __forceinline__ static v4f mul(const Frag& a, const Frag& b, v4f c, int) {
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
  uint32_t ldb;        // bytes from a row to the next
  uint32_t off[MOVES]; // this lane's 16 bytes in each of the wave's moves
  uint32_t kat, kdim;  // KC: the summed index that they hold, in their slice; its end
  uint32_t bytes;      // KC: of the rows that exist
  int wave;

  __device__ __forceinline__ static int kr_swizzle(int row) {
    return TYPE == OT_F32 ? (row >> 2) & UM : pieces::kr_f<(BL < 1 ? 1 : BL)>(row);
  }

  // p: the tile's first row (KC: rows ld apart; KR: the first row of the summed index at the tile's first column);
  // xdim: rows that exist
  __device__ __forceinline__ void open(const void* p, int64_t ld, int xdim, int64_t kd, int w, int lane) {
    // scalars, though they come from offsets that were read by a vector load
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)(uint64_t)p);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)p >> 32));
    base = (const char*)(((uint64_t)hi << 32) | lo);
    wave = w;
    kdim = __builtin_amdgcn_readfirstlane((uint32_t)kd);
    ldb = (uint32_t)(ld * ES);
    step = MODE == KC ? 128 : (int64_t)KS * ldb;
    kat = 0;
    bytes = 0;
    if (MODE == KC) {
      bytes = __builtin_amdgcn_readfirstlane((uint32_t)min(xdim, BX) * ldb);
      const int q = (lane & 7) ^ (lane >> 3);   // row % 8 is lane / 8
      kat = q * EV;
#pragma unroll
      for (int j = 0; j < MOVES; ++j) off[j] = (uint32_t)(8 * (w + NW * j) + (lane >> 3)) * ldb + 16 * q;
    } else {
#pragma unroll
      for (int j = 0; j < MOVES; ++j) {
        const int slot = (w + NW * j) * 64 + lane, row = slot / RS, s = slot % RS;
        const int col = TYPE == OT_F32 ? 16 * ((s >> 2) ^ kr_swizzle(row)) + 4 * (s & 3)
                                       : 16 * ((s >> 1) ^ kr_swizzle(row)) + 8 * (s & 1);
        off[j] = col < xdim ? (uint32_t)row * ldb + col * ES : pieces::kOob;
      }
    }
  }

  // slice kt into the stage, `at` bytes in.  The buffer's size leaves out the rows past the operand (KC: past its
  // rows; KR: past the summed index).
  __device__ __forceinline__ void fetch(lds_t* lds, int at, int kt) const {
    const char* p = base + kt * step;
    uint32_t size = bytes;
    if (MODE == KR) {
      const uint32_t done = (uint32_t)kt * KS;
      size = __builtin_amdgcn_readfirstlane(min(max(kdim, done) - done, (uint32_t)KS) * ldb);
    }
    const rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)p, (short)0, size, 0x00020000);
    const bool in = MODE == KR || (uint32_t)kt * KS + kat < kdim;
#pragma unroll
    for (int j = 0; j < MOVES; ++j) {
      const uint32_t o = in ? off[j] : pieces::kOob;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (pieces::lds_void*)(lds + (at + (wave + NW * j) * 1024)), 16, o, 0, 0, 0);
    }
  }

  // Where this lane reads: places in the tile from which the constants of block and step lead on.  They are made
  // opaque so that an address stays its array, a place and a constant: from longer chains the compiler loses which
  // array it reads, and then waits for the loads to the other one too.
  int place[2];
  __device__ __forceinline__ void reader(int lane, int blk0) {
    const int l16 = lane & 15, g = lane >> 4;
    if (MODE == KC) {
      place[0] = (16 * blk0 + l16) * 128 + ((g ^ (l16 & 7)) << 4);
      place[1] = (16 * blk0 + l16) * 128 + (((4 + g) ^ (l16 & 7)) << 4);
    } else if (TYPE == OT_F32) {
      place[0] = 4 * g * (BX * 4) + (((g & UM) ^ blk0) << 6) + l16 * 4;
      place[1] = 0;
    } else {
      const int row = 8 * g + (l16 >> 2);
      place[0] = row * BX * 2 + ((kr_swizzle(row) ^ blk0) << 5) + (l16 & 3) * 8;
      place[1] = (row + 4) * BX * 2 + ((kr_swizzle(row + 4) ^ blk0) << 5) + (l16 & 3) * 8;
    }
    __asm__("" : "+v"(place[0]), "+v"(place[1]));
  }

  // the wave's 16 rows from 16 blk on, summed indices of step s (half a slice), of the operand `at` bytes into the stage
  __device__ __forceinline__ typename Mfma<TYPE>::Frag read(const lds_t* lds, int at, int blk, int s) const {
    typedef typename Mfma<TYPE>::Frag Frag;
    if constexpr (MODE == KC) {
      return *(const __attribute__((address_space(3))) Frag*)(lds + place[s] + (at + blk * 2048));
    } else if constexpr (TYPE == OT_F32) {
      Frag f;
      const int o = place[0] ^ (blk << 6);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f[j] = *(const __attribute__((address_space(3))) float*)(lds + o + (at + (16 * s + j) * BX * 4));
      return f;
    } else {
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((pieces::lds_v4s*)(lds + (place[0] ^ (blk << 5)) + (at + s * 64 * BX)));
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((pieces::lds_v4s*)(lds + (place[1] ^ (blk << 5)) + (at + s * 64 * BX)));
      typedef short v8s __attribute__((ext_vector_type(8)));
      return __builtin_bit_cast(Frag, (v8s)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// A workgroup barrier behind this wave's LDS reads and all but the last N of its loads to LDS.  (A fence for LDS
// contents in its place waits for every load to LDS: the next slice's too.)
template <int N>
__device__ __forceinline__ void stage_barrier() {
  static_assert(N < 64, "six bits");
  __builtin_amdgcn_sched_barrier(0);
  __asm__ volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));   // vmcnt(N) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  __asm__ volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// A BM x BN tile by WM x WN waves, each (BM / WM) x (BN / WN) of it.
template <int TYPE, int MP, int MQ, int BM, int BN, int WM, int WN>
struct Tile {
  static constexpr int NW = WM * WN;
  static constexpr int IB = BM / WM / 16, JB = BN / WN / 16;   // 16 x 16 blocks of a wave
  typedef Operand<TYPE, MP, BM, NW> P;
  typedef Operand<TYPE, MQ, BN, NW> Q;
  static constexpr int STAGE = P::BYTES + Q::BYTES;
  static constexpr int KS = P::KS;
  static constexpr int FETCHES = P::MOVES + Q::MOVES;

  // acc[i][j][r]: row 16 i + lane % 16, column 16 j + 4 (lane / 16) + r of the wave's part (Q feeds the matrix
  // instruction's rows, so that a lane holds four consecutive columns of C)
  __device__ __forceinline__ static void run(lds_t* lds0, lds_t* lds1, const void* p, int64_t ldp, int rows,
                                             const void* q, int64_t ldq, int cols, int64_t depth,
                                             v4f (&acc)[IB][JB]) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = w / WN, wn = w % WN;
    P op;
    Q oq;
    op.open(p, ldp, rows, depth, w, lane);
    op.reader(lane, wm * IB);
    oq.open(q, ldq, cols, depth, w, lane);
    oq.reader(lane, wn * JB);
#pragma unroll
    for (int i = 0; i < IB; ++i)
#pragma unroll
      for (int j = 0; j < JB; ++j) acc[i][j] = (v4f){0.f, 0.f, 0.f, 0.f};
    const int nk = (int)((depth + 2 * KS - 1) / (2 * KS)) * 2;   // an even number of slices
    if (nk == 0) return;
    if constexpr (NW == 8 && MP == KR) {
      fetch(lds0, op, oq, 0);
      if (wm * IB * 16 >= rows || wn * JB * 16 >= cols) turns<0>(lds0, lds1, op, oq, nk, w >= 4, acc);
      else turns<IB>(lds0, lds1, op, oq, nk, w >= 4, acc);
      pieces::wait_loads();
      return;
    }
    fetch(lds0, op, oq, 0);
    fetch(lds1, op, oq, 1);
    stage_barrier<FETCHES>();    // slice 0 has landed
    if (wm * IB * 16 >= rows || wn * JB * 16 >= cols) {
      // nothing of this wave's part is stored: it only moves its share, and leaves the matrix unit to the others
      for (int kt = 0; kt < nk; kt += 2) {
        stage_barrier<FETCHES>();
        fetch(lds0, op, oq, kt + 2);
        stage_barrier<FETCHES>();
        stage_barrier<FETCHES>();
        fetch(lds1, op, oq, kt + 3);
        stage_barrier<FETCHES>();
      }
      pieces::wait_loads();
      return;
    }
    // A part of whose blocks only the first half has rows multiplies those alone.
    if (IB > 1 && rows - wm * IB * 16 <= IB * 8) slices<(IB + 1) / 2>(lds0, lds1, op, oq, nk, acc);
    else slices<IB>(lds0, lds1, op, oq, nk, acc);
    pieces::wait_loads();      // nothing may still move into this workgroup's LDS
  }

  __device__ __forceinline__ static void fetch(lds_t* stage, const P& op, const Q& oq, int kt) {
    op.fetch(stage, 0, kt);
    oq.fetch(stage, P::BYTES, kt);
  }

  // The products by eight waves, two on each of the four units, which take turns: one reads half a slice while the
  // other multiplies its half; a slice is four turns, the second wave a turn behind.  Half as many registers hold what
  // was read, which two KR operands at 256 x 256 need.  (Where both fit, slices() is faster by 0 to 5 %: a fetch has a
  // slice and a half to arrive there, one here.)  IA 0: the wave only moves its share.
  template <int IA>
  __device__ __forceinline__ static void turns(lds_t* lds0, lds_t* lds1, const P& op, const Q& oq, int nk, bool second,
                                               v4f (&acc)[IB][JB]) {
    typename Mfma<TYPE>::Frag fp[IA < 1 ? 1 : IA], fq[JB];
    auto read = [&](const lds_t* stage, int s) {
      if (IA == 0) return;
#pragma unroll
      for (int j = 0; j < JB; ++j) fq[j] = oq.read(stage, P::BYTES, j, s);
#pragma unroll
      for (int i = 0; i < IA; ++i) fp[i] = op.read(stage, 0, i, s);
    };
    auto multiply = [&]() {
#pragma unroll
      for (int r = 0; r < Mfma<TYPE>::SUB; ++r)
#pragma unroll
        for (int i = 0; i < IA; ++i)
#pragma unroll
          for (int j = 0; j < JB; ++j) acc[i][j] = Mfma<TYPE>::mul(fq[j], fp[i], acc[i][j], r);
    };
    stage_barrier<0>();            // slice 0 has landed
    if (second) {
      fetch(lds1, op, oq, 1);
      stage_barrier<FETCHES>();
      auto slice = [&](lds_t* now, int kt) {
        read(now, 0);
        stage_barrier<FETCHES>();
        multiply();
        stage_barrier<FETCHES>();
        read(now, 1);
        stage_barrier<0>();        // slice kt + 1 has landed, and everyone has read this one
        fetch(now, op, oq, kt + 2);
        multiply();
        if (IA > 0) interleave<0, FETCHES, IA * JB>();
        stage_barrier<FETCHES>();
      };
      for (int kt = 0; kt < nk; kt += 2) {
        slice(lds0, kt);
        slice(lds1, kt + 1);
      }
    } else {
      auto slice = [&](lds_t* now, lds_t* next, int kt) {
        read(now, 0);
        stage_barrier<FETCHES>();
        fetch(next, op, oq, kt + 1);   // read by everyone before this slice
        multiply();
        if (IA > 0) interleave<0, FETCHES, IA * JB>();
        stage_barrier<FETCHES>();
        read(now, 1);
        stage_barrier<FETCHES>();
        multiply();
        stage_barrier<0>();        // slice kt + 1 has landed
      };
      for (int kt = 0; kt < nk; kt += 2) {
        slice(lds0, lds1, kt);
        slice(lds1, lds0, kt + 1);
      }
      stage_barrier<0>();
    }
  }

  // the wave's products over nk slices, of its first IA row blocks
  template <int IA>
  __device__ __forceinline__ static void slices(lds_t* lds0, lds_t* lds1, const P& op, const Q& oq, int nk,
                                                v4f (&acc)[IB][JB]) {
    typename Mfma<TYPE>::Frag fp[2][IA], fq[2][JB];
    auto read = [&](const lds_t* stage, int s) {
#pragma unroll
      for (int j = 0; j < JB; ++j) fq[s][j] = oq.read(stage, P::BYTES, j, s);
#pragma unroll
      for (int i = 0; i < IA; ++i) fp[s][i] = op.read(stage, 0, i, s);
    };
    auto multiply = [&](int s, int i0, int i1) {
#pragma unroll
      for (int r = 0; r < Mfma<TYPE>::SUB; ++r)   // products of one block apart: each waits for the one before
#pragma unroll
        for (int i = i0; i < i1; ++i)
#pragma unroll
          for (int j = 0; j < JB; ++j) acc[i][j] = Mfma<TYPE>::mul(fq[s][j], fp[s][i], acc[i][j], r);
    };
    // A slice's second half is read behind the first products of its first; then everyone has read the stage, and the
    // slice two further on is fetched into it, which has more than a slice and a half to arrive; the second half is
    // multiplied while the next slice's first is read.  (With one barrier, fetches issued behind the first half: 0.7
    // slices to arrive, and 41 % of the waves' time spent waiting.)  The last rounds fetch and read past the operands,
    // zeros, so that a round is one block of code.
    constexpr int IH = (IA + 3) / 4;
    constexpr int READS = (MP == KC ? IA : (TYPE == OT_F32 ? 4 : 2) * IA) + (MQ == KC ? JB : (TYPE == OT_F32 ? 4 : 2) * JB);
    auto round = [&](lds_t* now, const lds_t* next, int kt) {
      read(now, 1);
      multiply(0, 0, IH);
      interleave<READS, 0, IH * JB>();
      stage_barrier<FETCHES>();    // everyone has read the stage
      fetch(now, op, oq, kt + 2);
      multiply(0, IH, IA);
      interleave<0, FETCHES, (IA - IH) * JB>();
      stage_barrier<FETCHES>();    // slice kt + 1 has landed
      read(next, 0);
      multiply(1, 0, IA);
      interleave<READS, 0, IA * JB>();
      __builtin_amdgcn_sched_barrier(0);
    };
    read(lds0, 0);
    for (int kt = 0; kt < nk; kt += 2) {
      round(lds0, lds1, kt);
      round(lds1, lds0, kt + 1);
    }
  }

  // spreads LDS reads and fetches between the products of a part of a round
  template <int NR, int NF, int BLOCKS>
  __device__ __forceinline__ static void interleave() {
    constexpr int PRODUCTS = BLOCKS * Mfma<TYPE>::SUB;
    constexpr int PER = NR + NF == 0 || PRODUCTS / (NR + NF) < 1 ? 1 : PRODUCTS / (NR + NF);
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);     // an LDS read
      __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);   // products
    }
#pragma unroll
    for (int k = 0; k < NF; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);     // a fetch
      __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
    }
  }

  // rounds the tile to TO and stores it, four values at a time wherever a row starts
  template <int TO>
  __device__ __forceinline__ static void store(const v4f (&acc)[IB][JB], void* c, int64_t ldc, int rows, int cols) {
    typedef typename Elem<TO>::T T;
    typedef T T4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
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
        if (col + 3 < cols) {
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

}  // namespace tile
