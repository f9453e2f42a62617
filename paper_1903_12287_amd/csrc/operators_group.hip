// Products with one matrix per group of rows (include/pbg_operators.h, pbg_group_linear):
//   forward  y[t, :]  = A_g x[t, :]            over in_dim
//   dx       dx[t, :] = A_g^T dy[t, :]         over out_dim
//   da       dA_g     = sum_t dy[t, :] x[t, :]^T   over the group's rows
#include "operators_device.h"

namespace {

constexpr int kTile = 64;     // rows and columns of a tile
constexpr int kShift = 6;
constexpr int kDepth = 16;

// One 64 x 64 tile of a product C = P Q^T, P[i][k] at p + i pi + k pk and Q[j][k] at q + j qi + k qk (elements).
template <int TYPE>
__device__ __forceinline__ void tile_product(const typename Elem<TYPE>::T* p, int64_t pi, int64_t pk, int rows,
                                             const typename Elem<TYPE>::T* q, int64_t qi, int64_t qk, int cols,
                                             int64_t depth, typename Elem<TYPE>::T* c, int64_t ldc) {
  typedef typename Elem<TYPE>::T T;
  __shared__ float ps[kDepth][kTile + 1], qs[kDepth][kTile + 1];
  const int tid = threadIdx.x, ti = tid >> 4, tj = tid & 15;
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < depth; k0 += kDepth) {
    __syncthreads();
    for (int f = tid; f < kDepth * kTile; f += 256) {
      const int i = f / kDepth, k = f % kDepth;
      const bool in = k0 + k < depth;
      ps[k][i] = in && i < rows ? (float)p[i * pi + (k0 + k) * pk] : 0.0f;
      qs[k][i] = in && i < cols ? (float)q[i * qi + (k0 + k) * qk] : 0.0f;
    }
    __syncthreads();
    for (int k = 0; k < kDepth; ++k) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[u][v] += ps[k][ti + 16 * u] * qs[k][tj + 16 * v];
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (ti + 16 * u < rows && tj + 16 * v < cols) c[(ti + 16 * u) * ldc + tj + 16 * v] = (T)acc[u][v];
}

template <int TYPE, int WHICH>
__global__ __launch_bounds__(256) void group_rows_kernel(GroupArgs g, int col_tiles) {
  typedef typename Elem<TYPE>::T T;
  if (!args_good(g.bad, g.host_bad)) return;
  const int64_t slot = blockIdx.x / col_tiles;
  const int j0 = (int)(blockIdx.x % col_tiles) * kTile;
  const int grp = group_of_slot(g.offsets, g.groups, kShift, slot);
  if (grp < 0) return;
  const int64_t r0 = g.offsets[grp] + ((slot - first_slot(g.offsets, grp, kShift)) << kShift);
  const int rows = (int)min((int64_t)kTile, g.offsets[grp + 1] - r0);
  if (rows <= 0) return;
  const T* a = (const T*)g.a + (int64_t)grp * g.m * g.k;
  T* out = (T*)g.out + r0 * g.ldo + j0;
  if (WHICH == GP_FORWARD)
    tile_product<TYPE>((const T*)g.x + r0 * g.ldx, g.ldx, 1, rows, a + (int64_t)j0 * g.k, g.k, 1, g.m - j0, g.k, out, g.ldo);
  else
    tile_product<TYPE>((const T*)g.dy + r0 * g.lddy, g.lddy, 1, rows, a + j0, 1, g.k, g.k - j0, g.m, out, g.ldo);
}

template <int TYPE>
__global__ __launch_bounds__(256) void group_da_kernel(GroupArgs g, int m_tiles, int k_tiles) {
  typedef typename Elem<TYPE>::T T;
  if (!args_good(g.bad, g.host_bad)) return;
  const int grp = blockIdx.x / (m_tiles * k_tiles), tile = blockIdx.x % (m_tiles * k_tiles);
  const int i0 = tile / k_tiles * kTile, j0 = tile % k_tiles * kTile;
  const int64_t r0 = g.offsets[grp], depth = g.offsets[grp + 1] - r0;
  tile_product<TYPE>((const T*)g.dy + r0 * g.lddy + i0, 1, g.lddy, g.m - i0, (const T*)g.x + r0 * g.ldx + j0, 1, g.ldx,
                     g.k - j0, depth, (T*)g.out + ((int64_t)grp * g.m + i0) * g.k + j0, g.k);
}

template <int TYPE>
bool launch_typed(const GroupArgs& g, int which, hipStream_t s) {
  const int mt = (g.m + kTile - 1) / kTile, kt = (g.k + kTile - 1) / kTile;
  const int64_t slots = (g.n >> kShift) + g.groups;
  const int64_t blocks = which == GP_DA ? (int64_t)g.groups * mt * kt : slots * (which == GP_FORWARD ? mt : kt);
  if (blocks > (1ll << 32) / 256 - 1) return false;
  const unsigned nb = (unsigned)blocks;
  if (which == GP_FORWARD) group_rows_kernel<TYPE, GP_FORWARD><<<nb, 256, 0, s>>>(g, mt);
  else if (which == GP_DX) group_rows_kernel<TYPE, GP_DX><<<nb, 256, 0, s>>>(g, kt);
  else group_da_kernel<TYPE><<<nb, 256, 0, s>>>(g, mt, kt);
  return true;
}

__global__ __launch_bounds__(256) void check_offsets_kernel(const int64_t* offsets, int groups, int64_t n,
                                                            uint32_t* flag) {
  bool bad = false;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i <= groups; i += (int64_t)gridDim.x * 256) {
    const int64_t v = offsets[i];
    bad |= v < 0 || v > n || (i < groups && offsets[i + 1] < v);
  }
  if (__ballot(bad) && (threadIdx.x & 63) == 0) atomicOr(flag, (uint32_t)OPS_BAD_OFFSETS);
}

}  // namespace

void launch_check_offsets(const int64_t* offsets, int groups, int64_t n, uint32_t* flag, hipStream_t s) {
  const int blocks = (groups + 256) / 256;
  check_offsets_kernel<<<blocks < 1024 ? blocks : 1024, 256, 0, s>>>(offsets, groups, n, flag);
}

bool launch_group_product(const GroupArgs& g, int type, int which, hipStream_t s) {
  switch (type) {
    case OT_F32: return launch_typed<OT_F32>(g, which, s);
    case OT_BF16: return launch_typed<OT_BF16>(g, which, s);
    default: return launch_typed<OT_F16>(g, which, s);
  }
}
