// Products with one matrix per group of rows (include/pbg_operators.h, pbg_group_linear):
//   forward  y[t, :]  = A_g x[t, :]                over in_dim
//   dx       dx[t, :] = A_g^T dy[t, :]             over out_dim
//   da       dA_g     = sum_t dy[t, :] x[t, :]^T   over the group's rows
// The host does not know the groups' sizes, so it launches a workgroup for every slot of rows that there could be, and
// a kernel ahead of the products (which also checks the offsets) writes down which group and rows a slot is.  (Every
// workgroup searching the offsets itself: four loads one behind the other before its first fetch, 2.5 of the 10 us of
// a workgroup with 32 rows of 400.)  Offsets of up to 63 groups fit the lanes of a wave: there every wave reads and
// checks them all in one load, and small products need no kernel ahead of them.
//
// Measured and what bounds it (us; the product alone, without the call's 15):
//   float32, 1,345 groups of sizes as 1 / rank^1.2 (1,272 have rows), 40,000 rows, 400 x 400, y: 256.  942 MB at 3.7 TB/s
//     of 5.1 that a copy reaches; 50 TFLOP/s.  55 % of the slots' rows are filled, and of the 40,000 rows 28,500 lie in
//     groups of 128 and more, which read their matrix once every 32 rows.
//   bfloat16, 32 groups, 32,768 rows, 2,048 to 4,096, y: 560, 980 TFLOP/s; one group: 500, 1,100.  A large library
//     product reaches 1,370.  The slices' way from memory bounds it: the loads alone, nothing multiplied, take as long
//     (585; 389 where all operands lie in the cache beside the memory), while LDS reads are hidden and products alone
//     take 425.  Two slices of 64 KB are what the LDS holds, and a slice waits for its slowest row.  What did not help:
//     reading ahead into the L2 (4 or 16 bytes a line, a slice or four ahead), padded rows, a persistent workgroup
//     that fetches the next tile's slices before it stores (1 to 5 %).
//   bfloat16, 32 groups, 16,384 rows, 2,048 x 2,048: dx 188 (730 TFLOP/s), da 230 (600; 268 MB written).
//   float16, 24 rows in 16 groups, 2,048 x 2,048, y: 20, 134 MB of matrices read at 6.6 TB/s (partly from the cache).
#include <algorithm>

#include "operators_tile.h"

namespace {

using tile::KC;
using tile::KR;

struct Launch {
  const int4* slots;          // NULL: up to 63 groups, every wave finds its slot itself
  int shift;                  // rows of a slot: 2^shift
  int64_t first;              // this launch's first slot
  int row_tiles, col_tiles;   // da: tiles of one matrix; y, dx: slots of the launch, tiles of the columns
  uint32_t blocks, band, chunk;   // tiles; the order in which they are taken
  float* partial;             // da: partial sums of the groups of several slots
  const int4* join;
};

// Rows cut into slots of 2^shift that never straddle two groups: group g's slots start at
// floor(offsets[g] / 2^shift) + g.  A group of L rows needs ceil(L / 2^shift) of them and has
// floor(end / 2^shift) - floor(start / 2^shift) + 1, which is never less; n / 2^shift + groups slots hold every group.
// A group's places for partial sums start at floor(2 offsets[g] / 2^shift): one of L > 2^shift rows has at least
// ceil(L / 2^shift) of them, so that 2 n / 2^shift places are enough, however many groups there are.
__device__ __forceinline__ int64_t first_slot(int64_t offset, int g, int shift) { return (offset >> shift) + g; }
__device__ __forceinline__ int64_t first_place(int64_t offset, int shift) { return (2 * offset) >> shift; }

// slot v of slots of 2^shift rows, where group g holds rows [first, last) and slot v is at or behind its first slot
__device__ __forceinline__ int4 slot_in(int g, int64_t first, int64_t last, int shift, int64_t v, bool places) {
  const int64_t part = v - first_slot(first, g, shift), r0 = first + (part << shift);
  if (part > 0 && r0 >= last) return make_int4(0, 0, -1, -1);
  const int64_t rows = min((int64_t)1 << shift, last - r0);
  const bool several = places && last - first > (int64_t)1 << shift;
  return make_int4((int)r0, (int)rows, g, several ? (int)(first_place(first, shift) + part) : -1);
}

// the entry for a group's partial sums: {group or -1, number of sums, place of the first}
__device__ __forceinline__ int4 join_of(int g, int64_t first, int64_t last, int shift) {
  const int64_t rows = last - first;
  if (rows <= (int64_t)1 << shift) return make_int4(-1, 0, 0, 0);
  return make_int4(g, (int)((rows + ((int64_t)1 << shift) - 1) >> shift), (int)first_place(first, shift), 0);
}

// All offsets of up to 63 groups, one a lane.
struct FewGroups {
  int64_t mine;
  int lane, groups;

  // false: the offsets are not in order, which the first workgroup tells the host
  __device__ __forceinline__ bool load(const GroupArgs& g) {
    lane = threadIdx.x & 63;
    groups = g.groups;
    mine = g.offsets[min(lane, groups)];
    const int64_t next = __shfl(mine, min(lane + 1, 63), 64);
    const bool bad = mine < 0 || mine > g.n || next < mine;   // lanes past the last offset repeat it
    if (__ballot(bad) == 0) return true;
    if (blockIdx.x == 0 && threadIdx.x == 0) *(volatile uint32_t*)g.host_bad = OPS_BAD_OFFSETS;
    return false;
  }
  __device__ __forceinline__ int4 slot(int shift, int64_t v, bool places) const {
    const int g = __popcll(__ballot(lane < groups && first_slot(mine, lane, shift) <= v)) - 1;
    if (g < 0) return make_int4(0, 0, -1, -1);
    return slot_in(g, __shfl(mine, g, 64), __shfl(mine, g + 1, 64), shift, v, places);
  }
  __device__ __forceinline__ int4 join(int shift, int g) const {
    return join_of(g, __shfl(mine, g, 64), __shfl(mine, g + 1, 64), shift);
  }
};

// slot v of the launch; false: the arguments are not good
__device__ __forceinline__ bool find_slot(const GroupArgs& g, const Launch& L, int64_t v, bool places, int4& slot) {
  if (L.slots) {
    slot = L.slots[v];
    return args_good(g.bad, g.host_bad);
  }
  FewGroups f;
  if (!f.load(g)) return false;
  const int4 at = f.slot(L.shift, v, places);
  slot = make_int4(__builtin_amdgcn_readfirstlane(at.x), __builtin_amdgcn_readfirstlane(at.y),
                   __builtin_amdgcn_readfirstlane(at.z), __builtin_amdgcn_readfirstlane(at.w));
  return true;
}

// Tiles in bands of `band` slots, column by column: the workgroups that an XCD runs at a time share the rows of a few
// slots and the matrix rows of a few columns, which its L2 then fetches once.
__device__ __forceinline__ void band_tile(uint32_t at, uint32_t band, uint32_t slots, uint32_t cols, uint32_t& slot,
                                          uint32_t& col) {
  const uint32_t b = at / (band * cols), r = at - b * (band * cols);
  const uint32_t h = min(band, slots - band * b);
  col = r / h;
  slot = band * b + (r - col * h);
}

// Hardware hands workgroups to the eight XCDs in turn, each with an L2 of its own: the tile of this workgroup such that
// the XCDs take chunks of L.chunk tiles in turn.  Tiles in a chunk share operands; and every XCD gets its part of the
// long groups and of the short ones.  L.blocks and more: none.
__device__ __forceinline__ uint32_t chunk_tile(const Launch& L) {
  const uint32_t j = blockIdx.x >> 3, chunk = j / L.chunk;
  return (chunk * 8 + (blockIdx.x & 7)) * L.chunk + (j - chunk * L.chunk);
}

// y and dx: one slot of a group's rows, one tile of the output's columns
template <int TYPE, int WHICH, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void group_rows_kernel(GroupArgs g, Launch L) {
  typedef tile::Tile<TYPE, KC, WHICH == GP_FORWARD ? KC : KR, BM, BN, WM, WN> Tl;
  constexpr int ES = TYPE == OT_F32 ? 4 : 2;
  __shared__ __attribute__((aligned(1024))) char lds0[Tl::STAGE], lds1[Tl::STAGE];
  // Few rows a matrix: little is shared, and the XCDs are kept even by taking the tiles in turn.
  const uint32_t at = BM >= 128 ? chunk_tile(L) : blockIdx.x;
  if (at >= L.blocks) return;
  uint32_t slot, col;
  band_tile(at, L.band, L.row_tiles, L.col_tiles, slot, col);
  const int j0 = (int)col * BN;
  int4 at_slot;
  if (!find_slot(g, L, L.first + slot, false, at_slot)) return;
  const int64_t r0 = at_slot.x;
  const int rows = at_slot.y, grp = at_slot.z;
  if (rows <= 0) return;
  const char* a = (const char*)g.a + (g.a_by_row ? g.offsets[grp] : grp) * g.a_group * ES;
  v4f acc[Tl::IB][Tl::JB];
  const int width = WHICH == GP_FORWARD ? g.m : g.k;
  if (WHICH == GP_FORWARD)
    Tl::run((tile::lds_t*)lds0, (tile::lds_t*)lds1, (const char*)g.x + r0 * g.ldx * ES, g.ldx, rows,
            a + (int64_t)j0 * g.lda * ES, g.lda, g.m - j0, g.kd, acc);
  else
    Tl::run((tile::lds_t*)lds0, (tile::lds_t*)lds1, (const char*)g.dy + r0 * g.lddy * ES, g.lddy, rows,
            a + (int64_t)j0 * ES, g.lda, g.kd - j0, g.m, acc);
  Tl::template store<TYPE>(acc, (char*)g.out + (r0 * g.ldo + j0) * ES, g.ldo, rows, width - j0);
}

// da: one slot of a group's rows, one tile of its matrix.  A group of one slot is stored; the slots of a longer one
// leave float32 sums, which group_join_kernel adds in their order.
template <int TYPE, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void group_da_kernel(GroupArgs g, Launch L) {
  typedef tile::Tile<TYPE, KR, KR, BM, BN, WM, WN> Tl;
  constexpr int ES = TYPE == OT_F32 ? 4 : 2;
  __shared__ __attribute__((aligned(1024))) char lds0[Tl::STAGE], lds1[Tl::STAGE];
  const int tiles = L.row_tiles * L.col_tiles;
  const uint32_t at = chunk_tile(L);
  if (at >= L.blocks) return;
  int4 slot;
  if (!find_slot(g, L, L.first + at / tiles, true, slot)) return;
  const int t = (int)(at % tiles);
  const int i0 = t / L.col_tiles * BM, j0 = t % L.col_tiles * BN;
  if (slot.z < 0) return;   // the first slot of an empty group stores zeros
  const int64_t r0 = slot.x, depth = slot.y;
  const int grp = slot.z;
  v4f acc[Tl::IB][Tl::JB];
  Tl::run((tile::lds_t*)lds0, (tile::lds_t*)lds1, (const char*)g.dy + (r0 * g.lddy + i0) * ES, g.lddy, g.md - i0,
          (const char*)g.x + (r0 * g.ldx + j0) * ES, g.ldx, g.kd - j0, depth, acc);
  const int rows = min(BM, g.m - i0), cols = g.k - j0;
  if (slot.w < 0) {
    Tl::template store<TYPE>(acc, (char*)g.out + (((int64_t)grp * g.m + i0) * g.k + j0) * ES, g.k, rows, cols);
  } else {
    float* p = L.partial + (int64_t)slot.w * g.m * g.k;
    Tl::template store<OT_F32>(acc, p + (int64_t)i0 * g.k + j0, g.k, rows, cols);
  }
}

// Adds a group's partial sums: of more than 32, 64 elements a workgroup, each of its four waves a quarter of the slots
// in their order, then the waves in theirs.  (One thread an element over all slots: 65 us for 78 slots of 100 x 100,
// loads one behind the other; 4 us so.)
template <int TYPE>
__global__ __launch_bounds__(256) void group_join_kernel(GroupArgs g, Launch L) {
  typedef typename Elem<TYPE>::T T;
  __shared__ float sums[4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int4 at;
  if (L.slots) {
    if (!args_good(g.bad, g.host_bad)) return;
    at = L.join[blockIdx.y];
  } else {
    FewGroups f;
    if (!f.load(g)) return;
    at = f.join(L.shift, blockIdx.y);
  }
  if (at.x < 0) return;
  const int64_t grp = at.x, place = at.z;
  const int parts = at.y;
  const int per = (parts + 3) >> 2, i0 = w * per, i1 = min(parts, i0 + per);
  const int64_t mk = (int64_t)g.m * g.k;
  const float* p = L.partial + place * mk;
  T* out = (T*)g.out + grp * mk;
  if (parts <= 32) {   // few enough for one thread's loads, eight at a time
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < mk; e += (int64_t)gridDim.x * 256) {
      float sum = p[e];
      for (int i = 1; i < parts; i += 8) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = p[min(i + u, parts - 1) * mk + e];
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += i + u < parts ? v[u] : 0.0f;
      }
      out[e] = (T)sum;
    }
    return;
  }
  for (int64_t e0 = (int64_t)blockIdx.x * 64; e0 < mk; e0 += (int64_t)gridDim.x * 64) {
    const int64_t e = min(e0 + lane, mk - 1);
    float s = 0.0f;
    int i = i0;
    for (; i + 8 <= i1; i += 8) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = p[(i + u) * mk + e];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
    for (; i < i1; ++i) s += p[i * mk + e];
    sums[w][lane] = s;
    __syncthreads();
    if (w == 0 && e0 + lane < mk) out[e] = (T)(((sums[0][lane] + sums[1][lane]) + sums[2][lane]) + sums[3][lane]);
    __syncthreads();
  }
}

// Copies rows of `width` values into rows of `wp` >= width, a multiple of 16 bytes, with zeros behind them.  Only what
// the products read is copied: the rows between the first and the last offset, and the matrices of groups that have
// rows.  Where there are fewer rows than groups, a matrix's place is its group's first row, so that the copies take no
// more than a matrix a row, however many groups there are (float16, 24 rows in 400 groups, 501 x 333, y: 36 us; 76 with
// every matrix copied).  Offsets that are not in order only choose which of the groups' matrices are copied to which
// places: they have not been checked here.
struct PackArgs {
  GroupPack op[3];
  uint32_t first[4];   // first workgroup of each
  int64_t per;         // rows of a workgroup
  const int64_t* offsets;
  int groups;
};

// the group whose matrix has this place (the same in all lanes of a wave), or -1: none that has rows
__device__ __forceinline__ int group_at_place(const PackArgs& a, bool by_row, int64_t place) {
  if (by_row) {
    const int g = sequence_of_row(a.offsets, a.groups, place);
    return g >= 0 && a.offsets[g] == place ? g : -1;
  }
  return a.offsets[place] < a.offsets[place + 1] ? (int)place : -1;
}

template <int TYPE>
__global__ __launch_bounds__(256) void group_pack_kernel(PackArgs a) {
  typedef typename Elem<TYPE>::T T;
  typedef typename Vec<TYPE>::V V;
  constexpr int N = Vec<TYPE>::N;
  const int w = blockIdx.x >= a.first[2] ? 2 : (blockIdx.x >= a.first[1] ? 1 : 0);
  const GroupPack& op = a.op[w];
  int64_t r0 = (int64_t)(blockIdx.x - a.first[w]) * a.per, r1 = min(op.rows, r0 + a.per);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const bool by_row = op.matrix && op.rows < (int64_t)a.groups * op.matrix;
  if (!op.matrix) {
    r1 = min(r1, a.offsets[a.groups]);
    r0 = max(r0, min(r1, a.offsets[0]));
  }
  int64_t place = -1, shift = 0;   // a matrix's rows in src lie so many behind its place's
  int grp = 0;
  for (int64_t r = r0 + wave; r < r1; r += 4) {
    if (op.matrix && (place < 0 || r >= (place + 1) * op.matrix)) {
      place = r / op.matrix;
      grp = group_at_place(a, by_row, place);
      shift = (grp - place) * op.matrix;
    }
    if (grp < 0) continue;
    const T* s = (const T*)op.src + (r + shift) * op.ld;
    T* d = (T*)op.dst + r * op.wp;
    for (int c = lane * N; c < op.wp; c += 64 * N) {   // wp is a multiple of N
      if (c + N <= op.width) {
        *(V*)(d + c) = *(const V*)(s + c);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) d[c + j] = c + j < op.width ? s[c + j] : (T)0.0f;
      }
    }
  }
}

// ---- what is launched ------------------------------------------------------------------------------
int64_t tiles_of(int64_t v, int b) { return (v + b - 1) / b; }

// a launch takes so many workgroups; of more, the slots are launched in turn
constexpr int64_t kLaunch = 1 << 22;

// workgroups such that chunk_tile() gives every tile
unsigned chunk_grid(const Launch& L) { return (unsigned)(tiles_of(L.blocks, 8 * (int)L.chunk) * 8 * L.chunk); }

template <int TYPE, int WHICH, int BM, int BN, int WM, int WN>
void launch_rows(const GroupArgs& g, const GroupPlan& p, Launch L, hipStream_t s) {
  L.slots = p.rows.at;
  L.shift = p.rows.shift;
  L.col_tiles = (int)tiles_of(WHICH == GP_FORWARD ? g.m : g.k, BN);
  // A chunk is a band.  (XCDs with an eighth of all tiles in a row each: float16, one group of 32,768 rows, 2,048 to
  // 4,096, y 540 us for 501, dx 582 for 484; 1,024 groups, 65,536 rows, 512 to 1,024: 306 and 272 for 281 and 259.
  // Bands of two keep the XCDs even where there are few slots: 8 groups of 1,024 rows, 2,048 x 2,048: 112 for 102;
  // float32, 8 of 2,048, 1,024 to 2,048: 598 for 545.)
  L.band = BM < 128 ? 8 : p.rows.count >= 160 ? 4 : 2;
  L.chunk = L.band * L.col_tiles;
  const int64_t step = kLaunch / L.col_tiles;   // col_tiles <= 1024
  for (L.first = 0; L.first < p.rows.count; L.first += step) {
    L.row_tiles = (int)std::min(step, p.rows.count - L.first);
    L.blocks = (uint32_t)L.row_tiles * L.col_tiles;
    const unsigned grid = BM >= 128 ? chunk_grid(L) : L.blocks;
    group_rows_kernel<TYPE, WHICH, BM, BN, WM, WN><<<grid, 64 * WM * WN, 0, s>>>(g, L);
  }
}

template <int TYPE, int B>
void launch_da(const GroupArgs& g, const GroupPlan& p, Launch L, hipStream_t s) {
  L.slots = p.da.at;
  L.shift = p.da.shift;
  L.partial = p.partial;
  L.join = p.join;
  L.row_tiles = (int)tiles_of(g.m, B);
  L.col_tiles = (int)tiles_of(g.k, B);
  const int64_t tiles = (int64_t)L.row_tiles * L.col_tiles, step = kLaunch / tiles;   // 1,024 x 1,024 tiles at most
  for (L.first = 0; L.first < p.da.count; L.first += step) {
    L.blocks = (uint32_t)(std::min(step, p.da.count - L.first) * tiles);
    // An eighth of a slot, where that is tiles enough to share operands, else a slot.  (Eighths of all tiles in a row:
    // bfloat16, 32 groups, 65,536 rows, the longest group 3 times the average, 2,048 x 2,048: 817 us for 566; float32,
    // 1,345 groups, 40,000 rows, sizes as 1 / rank, 400 x 400: 860 for 500.)
    L.chunk = (uint32_t)(tiles >= 64 ? tiles / 8 : tiles);
    constexpr int WN = B == 256 ? 4 : 2;
    group_da_kernel<TYPE, B, B, 2, WN><<<chunk_grid(L), 128 * WN, 0, s>>>(g, L);
  }
  if (p.joins > 0) {
    // most entries are groups of one slot, whose workgroups end at once: 16,384 in all
    const int64_t chunks = std::max<int64_t>(64, 16384 / p.joins);
    const dim3 grid((unsigned)std::min(tiles_of((int64_t)g.m * g.k, 64), chunks), (unsigned)p.joins);
    group_join_kernel<TYPE><<<grid, 256, 0, s>>>(g, L);
  }
}

// Rows and columns of a tile of da: in float32 the matrix unit sets the time, and more, smaller workgroups keep it
// busier (8 groups, 40,000 rows, 100 x 100: both gradients 75 us by 128 x 128, 70 by 64 x 64); in 16 bits reading the
// operands does (128 x 128 / 256 x 256, of 2,048 x 2,048: 32 groups of 512 rows 267 / 248 us, of 2,048 rows 610 / 535,
// uneven ones 672 / 566; where groups have to be cut to give every compute unit a tile, 4 groups of 4,096 rows:
// 153 / 258).  On either side of the two lines, both gradients, us, even sizes, then sizes as 1 / rank^0.8: 32 groups of
// 2,048 x 2,048, of 256 rows 321 / 305, 329 / 334, of 384 rows 385 / 370, 394 / 394, of 576 rows 492 / 470, 494 / 475;
// 576 rows each, 64 groups of 512 x 512 (256 tiles) 101 / 188, 125 / 153, 8 of 2,048 x 2,048 (512 tiles) 136 / 132,
// 142 / 141, 32 of 1,024 x 1,024 (512 tiles) 150 / 151, 155 / 180, 128 of them (2,048 tiles) 541 / 510, 560 / 572.
int da_tile(int type, int64_t n, int64_t groups, int64_t m, int64_t k) {
  if (type == OT_F32) return 64;
  return n / groups >= 512 && groups * tiles_of(m, 256) * tiles_of(k, 256) >= 512 ? 256 : 128;
}

// Rows of a tile of y or dx, 2^shift, by the average group and the number of tiles.  Measured (us, 32 x 64 / 128 x 128 /
// 256 x 256 tiles):
//   float32, 256 groups of 32 rows of 400 x 400: 77 / 94; of 1,024 rows: 814 / 893; 8 groups of 2,048 of 4,096 x 4,096:
//     4,657 / 4,018.  The matrix unit sets the time, and many small workgroups keep it busiest until operands are
//     read over and over.
//   bfloat16, 32 groups of 16 rows of 1,024 x 1,024: 29 / 34; of 32: 35 / 34; one of 1,024 rows of 512: 22 / 26 (16
//     tiles); 4 groups of 128 rows of 2,048 x 2,048: 44 / 36 / 49; 32 of 512 rows: 569 / 194 / 191; 32 of 1,024 rows of
//     2,048 x 4,096: 2,292 / 646 / 560; one of 8,192: 590 / 152 / 163 (2 tiles of 256 a compute unit).
int row_shift(int type, int64_t n, int groups, int64_t cols) {
  const int64_t average = n / groups, tiles = n / 128 * tiles_of(cols, 128), wide = n / 256 * tiles_of(cols, 256);
  if (type == OT_F32) return average >= 1024 && tiles >= 1024 ? 7 : 5;
  if (average >= 256 && wide >= 1024) return 8;
  return average >= 32 && tiles >= 64 ? 7 : 5;
}

template <int TYPE, int WHICH>
void launch_rows_by_size(const GroupArgs& g, const GroupPlan& p, const Launch& L, hipStream_t s) {
  if constexpr (TYPE != OT_F32) {
    if (p.rows.shift == 8) return launch_rows<TYPE, WHICH, 256, 256, 2, 4>(g, p, L, s);
  }
  if (p.rows.shift == 7) return launch_rows<TYPE, WHICH, 128, 128, 2, 2>(g, p, L, s);
  return launch_rows<TYPE, WHICH, 32, 64, 1, 4>(g, p, L, s);
}

template <int TYPE>
void launch_typed(const GroupArgs& g, int which, const GroupPlan& p, hipStream_t s) {
  Launch L{};
  if (which == GP_DA) {
    if constexpr (TYPE == OT_F32) {
      return launch_da<TYPE, 64>(g, p, L, s);
    } else {
      if (p.da_tile == 256) return launch_da<TYPE, 256>(g, p, L, s);
      return launch_da<TYPE, 128>(g, p, L, s);
    }
  }
  if (which == GP_FORWARD) return launch_rows_by_size<TYPE, GP_FORWARD>(g, p, L, s);
  return launch_rows_by_size<TYPE, GP_DX>(g, p, L, s);
}

// ---- the tables of slots ---------------------------------------------------------------------------
// the last group whose first slot (PLACE: first place) is at most v, or -1
template <bool PLACE>
__device__ __forceinline__ int group_at(const int64_t* offsets, int groups, int shift, int64_t v) {
  int lo = -1, hi = groups;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    const int64_t o = offsets[mid];
    if ((PLACE ? first_place(o, shift) : first_slot(o, mid, shift)) <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int4 slot_of(const int64_t* offsets, int groups, int shift, int64_t v, bool places) {
  const int g = group_at<false>(offsets, groups, shift, v);
  if (g < 0) return make_int4(0, 0, -1, -1);
  return slot_in(g, offsets[g], offsets[g + 1], shift, v, places);
}

// Offsets that are not in order are found here; what the tables then hold is not used.
__global__ __launch_bounds__(256) void group_plan_kernel(GroupPlan p, const int64_t* offsets, int groups, int64_t n,
                                                         uint32_t* flag) {
  const int64_t total = p.rows.count + p.da.count + p.joins;
  const int64_t step = (int64_t)gridDim.x * 256;
  bool bad = false;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total || i <= groups; i += step) {
    if (i <= groups) {
      const int64_t v = offsets[i];
      bad |= v < 0 || v > n || (i < groups && offsets[i + 1] < v);
    }
    int64_t v = i;
    if (v < p.rows.count) {
      p.rows.at[v] = slot_of(offsets, groups, p.rows.shift, v, false);
      continue;
    }
    v -= p.rows.count;
    if (v < p.da.count) {
      p.da.at[v] = slot_of(offsets, groups, p.da.shift, v, true);
      continue;
    }
    v -= p.da.count;
    if (v < p.joins) {
      // by group; or by place: a group of several slots holds two places at least, so at its first one it is the last
      // group that starts there or before
      const bool by_group = p.joins == groups;
      const int g = by_group ? (int)v : group_at<true>(offsets, groups, p.da.shift, v);
      int4 at = make_int4(-1, 0, 0, 0);
      if (g >= 0 && (by_group || first_place(offsets[g], p.da.shift) == v))
        at = join_of(g, offsets[g], offsets[g + 1], p.da.shift);
      p.join[v] = at;
    }
  }
  if (__ballot(bad) && (threadIdx.x & 63) == 0) atomicOr(flag, (uint32_t)OPS_BAD_OFFSETS);
}

}  // namespace

void launch_group_plan(const GroupPlan& p, const int64_t* offsets, int groups, int64_t n, uint32_t* flag,
                       hipStream_t s) {
  if (!p.tables) return;
  const int64_t work = std::max<int64_t>(p.rows.count + p.da.count + p.joins, groups + 1);
  const unsigned blocks = (unsigned)std::min<int64_t>(tiles_of(work, 256), 65536);
  group_plan_kernel<<<blocks, 256, 0, s>>>(p, offsets, groups, n, flag);
}

GroupPlan plan_group(int type, int which, int64_t n, int groups, int64_t m, int64_t k, bool want_da) {
  GroupPlan p{};
  // Tables written ahead cost a launch (2 us), offsets read by every workgroup 0.5 us for each workgroup that follows
  // another on its compute unit.  Without / with tables, us: y in float32, 128 x 128, 32 groups, 8,192 rows 23 / 25,
  // 131,072 (2^24) 72 / 74, 524,288 204 / 199, 2^20 378 / 368; float16, 2,048 x 2,048, 8 rows 38 / 40, 8,192 (2^24)
  // 128 / 130, 32,768 327 / 322; bfloat16, 512 x 512, 2^15 rows 48 / 50, 2^18 234 / 236; both gradients in float16, 32 of
  // 2,048 x 2,048, 2,048 rows 238 / 227 (many tiles of da for few rows), 16,384 453 / 453.
  p.tables = groups > 63 || n * std::max(m, k) > 1 << 24;
  if (which != GP_DA) {
    p.rows.shift = row_shift(type, n, groups, which == GP_FORWARD ? m : k);
    p.rows.count = (n >> p.rows.shift) + groups;
  }
  if (!want_da) return p;
  // Rows of a slot of da: enough slots for a few workgroups on each of the 256 compute units, where the matrices' tiles
  // alone are not, but 256 rows (of 128: float16, 37 groups of 135 rows, 336 x 504: 59 us for 33, partial sums written
  // and read); with tiles enough, longer groups than four times the average in 16 bits (twice: 32 groups, 16,384 rows,
  // 2,048 x 2,048: 288 for 259), than the average in float32 (four times: 37 groups, 5,000 rows, sizes as 1 / rank^1.5,
  // 336 x 504: 106 for 71).
  p.da_tile = da_tile(type, n, groups, m, k);
  const int64_t tiles = tiles_of(m, p.da_tile) * tiles_of(k, p.da_tile);
  int64_t rows = std::max<int64_t>(256, n * tiles / 1024);
  if (groups * tiles >= 512) rows = std::max(rows, (type == OT_F32 ? 1 : 4) * n / groups);
  int shift = 7;
  while (shift < 31 && ((int64_t)1 << shift) < rows) ++shift;
  // the partial sums stay below 512 MB, and a grid has 65,535 of them
  while (shift < 31 && (((2 * n) >> shift) * m * k * 4 > (512ll << 20) || (2 * n) >> shift > 65535)) ++shift;
  p.da.shift = shift;
  p.da.count = (n >> shift) + groups;
  p.partial_slots = n > (int64_t)1 << shift ? (2 * n) >> shift : 0;
  p.joins = p.tables ? std::min<int64_t>(groups, p.partial_slots) : (p.partial_slots > 0 ? groups : 0);
  return p;
}

void launch_group_pack(int type, int count, const GroupPack* op, const int64_t* offsets, int groups, hipStream_t s) {
  PackArgs a{};
  a.offsets = offsets;
  a.groups = groups;
  int64_t total = 0;
  for (int i = 0; i < count; ++i) total += op[i].rows;
  a.per = 16;
  while (total / a.per > kLaunch) a.per *= 2;
  uint32_t at = 0;
  for (int i = 0; i < 3; ++i) {
    a.first[i] = at;
    if (i >= count) continue;
    a.op[i] = op[i];
    at += (uint32_t)((op[i].rows + a.per - 1) / a.per);
  }
  if (!at) return;
  if (type == OT_F32) group_pack_kernel<OT_F32><<<at, 256, 0, s>>>(a);
  else if (type == OT_BF16) group_pack_kernel<OT_BF16><<<at, 256, 0, s>>>(a);
  else group_pack_kernel<OT_F16><<<at, 256, 0, s>>>(a);
}

void launch_group_product(const GroupArgs& g, int type, int which, const GroupPlan& p, hipStream_t s) {
  switch (type) {
    case OT_F32: return launch_typed<OT_F32>(g, which, p, s);
    case OT_BF16: return launch_typed<OT_BF16>(g, which, p, s);
    default: return launch_typed<OT_F16>(g, which, p, s);
  }
}
