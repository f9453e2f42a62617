// The joint norm of many gradients and their scaling (include/pbg_operators.h, pbg_clip_gradients).
#include "operators_device.h"

namespace {

// the tensor of this workgroup and its first value
__device__ __forceinline__ int tensor_of_block(const ClipBatch& b, int64_t& at) {
  int t = 0;
  while (t + 1 < b.n && b.first[t + 1] <= blockIdx.x) ++t;
  at = (int64_t)(blockIdx.x - b.first[t]) * kClipBlock;
  return t;
}

template <int TYPE>
__device__ __forceinline__ double squares(const void* g, int64_t at, int64_t end) {
  const typename Elem<TYPE>::T* p = (const typename Elem<TYPE>::T*)g;
  double s = 0.0;
  for (int64_t i = at + threadIdx.x; i < end; i += 256) {
    const double v = (double)(float)p[i];
    s = fma(v, v, s);
  }
  return s;
}

template <int TYPE>
__device__ __forceinline__ void scaled(const void* g, void* o, int64_t at, int64_t end, double f) {
  typedef typename Elem<TYPE>::T T;
  for (int64_t i = at + threadIdx.x; i < end; i += 256) {
    const float v = (float)((const T*)g)[i];
    ((T*)o)[i] = (T)(f == 1.0 ? v : (float)((double)v * f));
  }
}

__global__ __launch_bounds__(256) void clip_squares_kernel(ClipBatch b, double* parts) {
  __shared__ double red[4];
  int64_t at;
  const int t = tensor_of_block(b, at);
  const int64_t end = min(b.count[t], at + kClipBlock);
  double s = b.type[t] == OT_F32 ? squares<OT_F32>(b.g[t], at, end)
                                 : (b.type[t] == OT_BF16 ? squares<OT_BF16>(b.g[t], at, end)
                                                         : squares<OT_F16>(b.g[t], at, end));
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(1024) void clip_factor_kernel(const double* parts, int64_t n, double max_norm,
                                                           double* scale, double* host_norm) {
  __shared__ double red[16];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += parts[i];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x) return;
  s = 0.0;
  for (int w = 0; w < 16; ++w) s += red[w];
  const double norm = sqrt(s);
  *(volatile double*)host_norm = norm;
  *scale = isfinite(norm) && norm > max_norm ? max_norm / norm : 1.0;
}

__global__ __launch_bounds__(256) void clip_scale_kernel(ClipBatch b, const double* scale) {
  int64_t at;
  const int t = tensor_of_block(b, at);
  const double f = *scale;
  if (f == 1.0 && b.o[t] == b.g[t]) return;
  const int64_t end = min(b.count[t], at + kClipBlock);
  if (b.type[t] == OT_F32) scaled<OT_F32>(b.g[t], b.o[t], at, end, f);
  else if (b.type[t] == OT_BF16) scaled<OT_BF16>(b.g[t], b.o[t], at, end, f);
  else scaled<OT_F16>(b.g[t], b.o[t], at, end, f);
}

}  // namespace

void launch_clip_squares(const ClipBatch& b, double* parts, hipStream_t s) {
  if (b.first[b.n]) clip_squares_kernel<<<b.first[b.n], 256, 0, s>>>(b, parts);
}

void launch_clip_factor(const double* parts, int64_t n, double max_norm, double* scale, double* host_norm, hipStream_t s) {
  clip_factor_kernel<<<1, 1024, 0, s>>>(parts, n, max_norm, scale, host_norm);
}

void launch_clip_scale(const ClipBatch& b, const double* scale, hipStream_t s) {
  if (b.first[b.n]) clip_scale_kernel<<<b.first[b.n], 256, 0, s>>>(b, scale);
}
