// The joint norm of many gradients and their scaling (include/pbg_operators.h, pbg_clip_gradients):
// norm = sqrt(sum of all squares), out = g min(1, max_norm / norm).
//
// Bound by memory: the gradients are read for the norm, read again and written.  A workgroup takes 8,192 values of one
// tensor at a time, 16 bytes a load, all of a thread's loads on their way at once; its sum of squares goes to a place of
// its own, so the norm does not depend on the order in which workgroups end.  The scaling walks the workgroups
// backwards: what the norm read last is still in the 256 MB cache beside the memory.  Squares and their sums are
// float64 (an instruction a value: the vector unit keeps up with memory), so the norm neither overflows nor loses small
// gradients, and a scaled value is rounded once, to its own type.
//
// Measured: 620 million float32 values (2.48 GB) 418 us for the squares (5.9 TB/s) and 907 for the scaling (5.5 TB/s
// read and written; a large copy reaches 5.1); 56 tensors of 50 million values of two types 21 and 41 us, the second
// read mostly from the cache, 4 for the factor between them.
#include "operators_device.h"

namespace {

// the tensor of this workgroup, and its first value in it
__device__ __forceinline__ int tensor_of_block(const ClipBatch& b, uint32_t block, int64_t& at) {
  const int lane = threadIdx.x & 63;
  int t = 0;
#pragma unroll
  for (int i = 0; i < kClipBatch; i += 64) {
    const int k = i + lane;
    t += __popcll(__ballot(k < b.n && b.first[k < kClipBatch ? k : 0] <= block));
  }
  t = __builtin_amdgcn_readfirstlane(t - 1);
  at = (int64_t)(block - b.first[t]) * b.span;
  return t;
}

template <int TYPE>
__device__ __forceinline__ void squares(const void* g, int64_t at, int64_t count, double (&s)[4]) {
  typedef typename Elem<TYPE>::T T;
  typedef typename Vec<TYPE>::V V;
  constexpr int N = Vec<TYPE>::N, LOADS = kClipBlock / 256 / N;
  const T* p = (const T*)g + at;
  if (count - at >= kClipBlock) {
    V v[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) v[i] = *(const V*)(p + (i * 256 + threadIdx.x) * N);
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const double x = (double)(float)v[i][j];
        s[j & 3] = fma(x, x, s[j & 3]);
      }
  } else {
    const int n = (int)(count - at);
    for (int i = threadIdx.x * N; i < n; i += 256 * N) {
      if (i + N <= n) {
        const V v = *(const V*)(p + i);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const double x = (double)(float)v[j];
          s[j & 3] = fma(x, x, s[j & 3]);
        }
      } else {
        for (int j = i; j < n; ++j) {
          const double x = (double)(float)p[j];
          s[0] = fma(x, x, s[0]);
        }
      }
    }
  }
}

template <int TYPE>
__device__ __forceinline__ typename Elem<TYPE>::T scaled(typename Elem<TYPE>::T v, double f) {
  return (typename Elem<TYPE>::T)(float)((double)(float)v * f);
}
// float64 to float32, to the neighbour with its last bit set where it lies between two: rounding that to 16 bits gives
// what rounding the float64 value itself would (through the nearest float32 it would be rounded twice)
__device__ __forceinline__ float to_odd(double x) {
  const float r = (float)x;
  const double d = x - (double)r;
  if (d == 0.0 || !(fabs(x) < 3.0e38)) return r;
  const uint32_t u = __float_as_uint(r);
  if (u & 1) return r;   // else the neighbour on x's other side
  const bool up = (d > 0.0) == (x > 0.0);
  return __uint_as_float(up ? u + 1 : u - 1);
}
template <>
__device__ __forceinline__ __bf16 scaled<OT_BF16>(__bf16 v, double f) { return (__bf16)to_odd((double)(float)v * f); }
template <>
__device__ __forceinline__ _Float16 scaled<OT_F16>(_Float16 v, double f) { return (_Float16)to_odd((double)(float)v * f); }

template <int TYPE>
__device__ __forceinline__ void scale_block(const void* g, void* o, int64_t at, int64_t count, double f) {
  typedef typename Elem<TYPE>::T T;
  typedef typename Vec<TYPE>::V V;
  constexpr int N = Vec<TYPE>::N, LOADS = kClipBlock / 256 / N;
  const T* p = (const T*)g + at;
  T* q = (T*)o + at;
  if (count - at >= kClipBlock) {
    V v[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) v[i] = *(const V*)(p + (i * 256 + threadIdx.x) * N);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] = f == 1.0 ? v[i][j] : scaled<TYPE>(v[i][j], f);
      *(V*)(q + (i * 256 + threadIdx.x) * N) = v[i];
    }
  } else {
    const int n = (int)(count - at);
    for (int i = threadIdx.x * N; i < n; i += 256 * N) {
      if (i + N <= n) {
        V v = *(const V*)(p + i);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = f == 1.0 ? v[j] : scaled<TYPE>(v[j], f);
        *(V*)(q + i) = v;
      } else {
        for (int j = i; j < n; ++j) q[j] = f == 1.0 ? p[j] : scaled<TYPE>(p[j], f);
      }
    }
  }
}

__global__ __launch_bounds__(256) void clip_squares_kernel(ClipBatch b, double* parts) {
  __shared__ double red[4];
  int64_t at;
  const int t = tensor_of_block(b, blockIdx.x, at);
  const int64_t end = min(b.count[t], at + b.span);
  double p[4] = {0.0, 0.0, 0.0, 0.0};
  for (; at < end; at += kClipBlock) {
    if (b.type[t] == OT_F32) squares<OT_F32>(b.g[t], at, end, p);
    else if (b.type[t] == OT_BF16) squares<OT_BF16>(b.g[t], at, end, p);
    else squares<OT_F16>(b.g[t], at, end, p);
  }
  double s = (p[0] + p[1]) + (p[2] + p[3]);
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// the sum of n parts, the same in every thread and, whatever the workgroup, in the same order
template <int THREADS>
__device__ __forceinline__ double sum_parts(const double* parts, int64_t n) {
  __shared__ double red[THREADS / 64];
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int64_t i = threadIdx.x; i < n; i += 4 * THREADS) {
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] += i + u * THREADS < n ? parts[i + u * THREADS] : 0.0;
  }
  const double w = wave_sum_d((s[0] + s[1]) + (s[2] + s[3]));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = w;
  __syncthreads();
  double all = red[0];
#pragma unroll
  for (int i = 1; i < THREADS / 64; ++i) all += red[i];
  return all;
}

__device__ __forceinline__ double clip_factor(double norm, double max_norm) {
  return isfinite(norm) && norm > max_norm ? max_norm / norm : 1.0;
}

__global__ __launch_bounds__(1024) void clip_factor_kernel(const double* parts, int64_t n, double max_norm,
                                                           double* scale, double* host_norm) {
  const double norm = sqrt(sum_parts<1024>(parts, n));
  if (threadIdx.x) return;
  *(volatile double*)host_norm = norm;
  *scale = clip_factor(norm, max_norm);
}

// OWN: every workgroup adds the parts itself
template <bool OWN>
__global__ __launch_bounds__(256) void clip_scale_kernel(ClipBatch b, const double* scale, const double* parts, int64_t n,
                                                         double max_norm, double* host_norm) {
  double f;
  if (OWN) {
    const double norm = sqrt(sum_parts<256>(parts, n));
    f = clip_factor(norm, max_norm);
    if (blockIdx.x == 0 && threadIdx.x == 0) *(volatile double*)host_norm = norm;
  } else {
    f = *scale;
  }
  int64_t at;
  const int t = tensor_of_block(b, gridDim.x - 1 - blockIdx.x, at);
  if (f == 1.0 && b.o[t] == b.g[t]) return;
  const int64_t end = min(b.count[t], at + b.span);
  for (; at < end; at += kClipBlock) {
    if (b.type[t] == OT_F32) scale_block<OT_F32>(b.g[t], b.o[t], at, end, f);
    else if (b.type[t] == OT_BF16) scale_block<OT_BF16>(b.g[t], b.o[t], at, end, f);
    else scale_block<OT_F16>(b.g[t], b.o[t], at, end, f);
  }
}

// Up to so many parts every workgroup of the scaling adds them itself, four loads a thread: a launch less (a small
// call's three launches ended 4 us later).
constexpr int64_t kOwnParts = 1024;

}  // namespace

void launch_clip(const ClipBatch* b, int batches, int64_t blocks, double max_norm, double* scale, double* parts,
                 double* host_norm, hipStream_t s) {
  int64_t at = 0;
  for (int i = 0; i < batches; ++i) {
    clip_squares_kernel<<<b[i].first[b[i].n], 256, 0, s>>>(b[i], parts + at);
    at += b[i].first[b[i].n];
  }
  const bool own = batches == 1 && blocks <= kOwnParts;
  if (!own) clip_factor_kernel<<<1, 1024, 0, s>>>(parts, blocks, max_norm, scale, host_norm);
  for (int i = batches - 1; i >= 0; --i) {
    const uint32_t n = b[i].first[b[i].n];
    if (own) clip_scale_kernel<true><<<n, 256, 0, s>>>(b[i], scale, parts, blocks, max_norm, host_norm);
    else clip_scale_kernel<false><<<n, 256, 0, s>>>(b[i], scale, parts, blocks, max_norm, host_norm);
  }
}
