// Preference loss on pairs of sequences of candidate scores (include/pbg_operators.h, pbg_preference_loss).
//
// A row's log probability is l = z[y] - m - log sum_v exp(z[v] - m) with its largest score m: one pass over the row
// keeps the running maximum and the sum relative to it.  The gradient of the row is
// dlogp (1[v = y] - exp(z[v] - m - log sum)), a second pass over the scores once the pairs' losses are known.
#include "operators_device.h"

namespace {

// (m, s) of the union of two sets of scores, s relative to m; an empty set is (-inf, 0)
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  if (top == -INFINITY) {
    s += s2;   // both empty, or a NaN
    return;
  }
  s = s * expf(m - top) + s2 * expf(m2 - top);
  m = top;
}

template <int TYPE>
__global__ __launch_bounds__(256) void row_stats_kernel(PrefArgs p) {
  typedef typename Elem<TYPE>::T T;
  __shared__ float sm[4], ss[4];
  if (!args_good(p.bad, p.host_bad)) return;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  if (t >= p.n) return;   // no rows: the launch only hands over the verdict
  if (sequence_of_row(p.offsets, 2 * p.pairs, t) < 0) return;
  const int label = p.labels[t];
  if (label < 0) {
    if (tid == 0) {
      p.stats[2 * t] = p.stats[2 * t + 1] = 0.0f;
      p.picked[t] = 0.0;
    }
    return;
  }
  const T* z = (const T*)p.logits + t * p.ld;
  float m = -INFINITY, s = 0.0f;
  for (int v = tid; v < p.V; v += 256) {
    const float x = (float)z[v];
    join(m, s, x, x == -INFINITY ? 0.0f : (x == x ? 1.0f : x));
  }
  for (int o = 32; o > 0; o >>= 1) {
    const float m2 = __shfl_xor(m, o, 64), s2 = __shfl_xor(s, o, 64);
    join(m, s, m2, s2);
  }
  if ((tid & 63) == 0) {
    sm[tid >> 6] = m;
    ss[tid >> 6] = s;
  }
  __syncthreads();
  if (tid) return;
  for (int w = 1; w < 4; ++w) join(m, s, sm[w], ss[w]);
  const bool none = m == -INFINITY && s == 0.0f;
  const float ls = none ? 0.0f : logf(s);
  p.stats[2 * t] = m;
  p.stats[2 * t + 1] = ls;
  p.picked[t] = none ? 0.0 : (double)((float)z[label] - m) - (double)ls;
}

// one workgroup per pair: each sequence's rows are added in a fixed order
__global__ __launch_bounds__(256) void pair_loss_kernel(PrefArgs p) {
  __shared__ double part[2][4];
  if (!args_good(p.bad, p.host_bad)) return;
  const int64_t pair = blockIdx.x;
  const int tid = threadIdx.x;
  for (int w = 0; w < 2; ++w) {
    double s = 0.0;
    const int64_t end = p.offsets[2 * pair + w + 1];
    for (int64_t t = p.offsets[2 * pair + w] + tid; t < end; t += 256) s += p.picked[t];
    s = wave_sum_d(s);
    if ((tid & 63) == 0) part[w][tid >> 6] = s;
  }
  __syncthreads();
  if (tid) return;
  double lp[2], ratio[2];
  for (int w = 0; w < 2; ++w) {
    lp[w] = part[w][0] + part[w][1] + part[w][2] + part[w][3];
    ratio[w] = lp[w] - (p.ref ? (double)p.ref[2 * pair + w] : 0.0);
    p.logp[2 * pair + w] = (float)lp[w];
  }
  const double b = p.beta, eps = p.smoothing, h = b * (ratio[0] - ratio[1]);
  const double soft = log1p(exp(-fabs(h)));
  if (p.loss) {
    double loss = (1.0 - eps) * (soft + (h < 0.0 ? -h : 0.0));
    if (eps > 0.0) loss += eps * (soft + (h > 0.0 ? h : 0.0));
    p.loss[pair] = h == h ? (float)loss : NAN;
  }
  if (p.dlogp) {
    const double d = b * (eps / (1.0 + exp(-h)) - (1.0 - eps) / (1.0 + exp(h)));
    p.dlogp[2 * pair] = (float)d;
    p.dlogp[2 * pair + 1] = (float)-d;
  }
}

template <int TYPE>
__global__ __launch_bounds__(256) void preference_backward_kernel(PrefArgs p) {
  typedef typename Elem<TYPE>::T T;
  if (!args_good(p.bad, p.host_bad)) return;
  const int64_t t = blockIdx.x;
  if (t >= p.n) return;
  const int q = sequence_of_row(p.offsets, 2 * p.pairs, t);
  if (q < 0) return;
  const int label = p.labels[t];
  const T* z = (const T*)p.logits + t * p.ld;
  T* dz = (T*)p.dlogits + t * p.lddl;
  const float m = p.stats[2 * t], ls = p.stats[2 * t + 1];
  const bool counts = label >= 0 && !(m == -INFINITY && ls == 0.0f);
  const float g = p.dlogp[q];
  for (int v = threadIdx.x; v < p.V; v += 256) {
    float d = 0.0f;
    if (counts) d = g * ((v == label ? 1.0f : 0.0f) - expf((float)z[v] - m - ls));
    dz[v] = (T)d;
  }
}

// labels of rows inside a sequence are below V (negative ones do not count)
__global__ __launch_bounds__(256) void check_labels_kernel(PrefArgs p) {
  const int64_t first = p.offsets[0], last = p.offsets[2 * p.pairs];
  bool bad = false;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < p.n; t += (int64_t)gridDim.x * 256)
    bad |= t >= first && t < last && p.labels[t] >= p.V;
  if (__ballot(bad) && (threadIdx.x & 63) == 0) atomicOr(p.bad, (uint32_t)OPS_BAD_LABEL);
}

}  // namespace

void launch_check_labels(const PrefArgs& p, hipStream_t s) {
  const int64_t blocks = (p.n + 255) / 256;
  check_labels_kernel<<<(unsigned)(blocks < 1 ? 1 : (blocks > 1024 ? 1024 : blocks)), 256, 0, s>>>(p);
}

void launch_preference_loss(const PrefArgs& p, int type, hipStream_t s) {
  const unsigned rows = p.n > 0 ? (unsigned)p.n : 1u;
  if (type == OT_F32) row_stats_kernel<OT_F32><<<rows, 256, 0, s>>>(p);
  else if (type == OT_BF16) row_stats_kernel<OT_BF16><<<rows, 256, 0, s>>>(p);
  else row_stats_kernel<OT_F16><<<rows, 256, 0, s>>>(p);
  pair_loss_kernel<<<p.pairs, 256, 0, s>>>(p);
}

void launch_preference_backward(const PrefArgs& p, int type, hipStream_t s) {
  const unsigned rows = p.n > 0 ? (unsigned)p.n : 1u;
  if (type == OT_F32) preference_backward_kernel<OT_F32><<<rows, 256, 0, s>>>(p);
  else if (type == OT_BF16) preference_backward_kernel<OT_BF16><<<rows, 256, 0, s>>>(p);
  else preference_backward_kernel<OT_F16><<<rows, 256, 0, s>>>(p);
}
