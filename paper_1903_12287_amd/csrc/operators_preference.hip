// Preference loss on pairs of sequences of candidate scores (include/pbg_operators.h, pbg_preference_loss).
//
// A row's log probability is l = z[y] - m - log sum_v exp(z[v] - m) with its largest score m: one pass over the row
// keeps the running maximum and the sum relative to it.  The gradient of the row is
// dlogp (1[v = y] - exp(z[v] - m - log sum)), a second pass over the scores once the pairs' losses are known (a pair's
// loss needs every row of both sequences).  m and log sum are kept apart, so that z - m stays exact however far from
// zero the scores lie.
//
// Bound by memory: the scores are read for the loss, read again and overwritten by the gradient.  Rows without a label
// are not read.  16 bytes a load wherever the row starts; a wave takes a short row, a workgroup a longer one, and few rows
// are cut into segments whose (m, sum) are joined afterwards.
//
// Measured, bfloat16, 16,384 rows of 15,000 candidates, a fifth of them without a label: 69 us for the sums by
// themselves (393 MB, 5.7 TB/s; an exponential a score), 108 right behind a gradient whose writes are still on their way
// to memory, as in a loop of both; 154 for the gradient (393 MB read, 492 written, 5.7 TB/s; a large copy reaches 5.1).
// float16, 96 rows of 131,001: 9 us for the parts, 8 to join them.
#include <algorithm>

#include "operators_device.h"

namespace {

// exp(d), d <= 0: base 2 through the hardware, whose argument d log2(e) is rounded.  Float32 results get the rest back;
// gradients of 16 bits do not hold it (|d| half steps of float32).
template <int TYPE>
__device__ __forceinline__ float exp_of(float d) {
  constexpr float L = 1.44269502f, LL = 1.92596299e-8f;   // log2(e) in two parts
  const float t = d * L;
  const float r = __builtin_amdgcn_exp2f(t);
  if (TYPE != OT_F32) return r;
  // what t leaves out; 0 where it is not a number (infinite d) or r has vanished
  const float e = fmaf(d, L, -t) + d * LL;
  return r > 0.0f && r < INFINITY ? fmaf(r, e * 0.693147181f, r) : r;
}

// the largest score and the sum relative to it, of a set of scores; an empty set is (-inf, 0)
struct Stats {
  float m, s;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

// a set's sum relative to `base`, its largest score or above: all of the sum is off by what this exp is, so it keeps
// float32 whatever the scores' type.  (Without: 2e-8 to 7e-8 of the sums to one side, growing with the row.)
__device__ __forceinline__ float sum_at(const Stats& a, float base) { return a.s * exp_of<OT_F32>(a.m - base); }

// Scores of 16 bits take exp(x - m) as 2^(x log2(e) - M), M = m log2(e) rounded: one multiply-add and its rounding.  What
// M's rounding left out is the same for every term and comes off the sum; what float32 leaves out of log2(e) stays and
// makes a term too large by 1.3e-8 |x - m| of itself.  (Log sums of 300 to 131,001 normal scores are off by 7e-8 to
// 1.0e-7, root mean square, their own rounding to float32 included, as with log2(e) in two parts.)  Far from zero (where
// M's rounding would no longer be small) and in float32 the difference is formed first.
template <int TYPE, int COUNT>
__device__ __forceinline__ void add_scores(Stats& a, const float (&x)[COUNT]) {
  float m = a.m;
#pragma unroll
  for (int i = 0; i < COUNT; ++i) m = fmaxf(m, x[i]);
  const float base = base_of(m);
  const float old = sum_at(a, base);
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (TYPE != OT_F32 && fabsf(base) < 65536.0f * 16.0f) {
    constexpr float L = 1.44269502f;
    const float M = base * L;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i & 3] += __builtin_amdgcn_exp2f(fmaf(x[i], L, -M));
    const float left = fmaf(base, L, -M);
    a.s = fmaf((s[0] + s[1]) + (s[2] + s[3]), __builtin_amdgcn_exp2f(-left), old);
  } else {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) s[i & 3] += exp_of<TYPE>(x[i] - base);
    a.s = old + ((s[0] + s[1]) + (s[2] + s[3]));
  }
  a.m = m;
}

// values [first, last) of a row by THREADS threads, U loads of 16 bytes on their way at a time, and the next U while
// they are added
template <int TYPE, int THREADS>
__device__ __forceinline__ Stats scan(const typename Elem<TYPE>::T* z, int first, int last, int tid) {
  typedef typename Vec<TYPE>::V V;
  constexpr int N = Vec<TYPE>::N, U = 4, STEP = THREADS * N * U;
  Stats a = {-INFINITY, 0.0f};
  if (last - first < N) {
    const float y[1] = {first + tid < last ? (float)z[first + tid] : -INFINITY};
    add_scores<TYPE>(a, y);
  } else {
    // 16 bytes that would reach past the end are taken from before it, so that no load is behind a branch; what they
    // hold twice counts for nothing
    auto load = [&](V (&w)[U], int v0) {
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = *(const V*)(z + min(v0 + (u * THREADS + tid) * N, last - N));
    };
    float x[U * N];
    V w[U], next[U];
    load(w, first);
    int v0 = first;
    for (; v0 + STEP < last; v0 += STEP) {   // every value of w counts, and more are left
      load(next, v0 + STEP);
#pragma unroll
      for (int i = 0; i < U * N; ++i) x[i] = (float)w[i / N][i % N];
      add_scores<TYPE>(a, x);
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = next[u];
    }
#pragma unroll
    for (int i = 0; i < U * N; ++i) {
      const int v = v0 + (i / N * THREADS + tid) * N;
      x[i] = v + N <= last || last - N + i % N >= v ? (float)w[i / N][i % N] : -INFINITY;
    }
    add_scores<TYPE>(a, x);
  }
  float m = a.m;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  float s = sum_at(a, base_of(m));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  return {m, s};
}

// a workgroup's stats from its waves'
__device__ __forceinline__ Stats join_waves(const Stats& a) {
  __shared__ Stats part[4];
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
  __syncthreads();
  const float m = fmaxf(fmaxf(part[0].m, part[1].m), fmaxf(part[2].m, part[3].m)), base = base_of(m);
  return {m, (sum_at(part[0], base) + sum_at(part[1], base)) + (sum_at(part[2], base) + sum_at(part[3], base))};
}

// a counted row's stats and log probability; a row without a distribution does not count.  The logarithm is taken in
// float64: rounded to float32, at a size of ten, it is what a sequence of many rows would be off by.  The stats that the
// gradient takes are the caller's float32 and hold it rounded: all probabilities of a row are off by that, up to 4.8e-7 of
// themselves (7e-8 to 8e-8, root mean square, beside 2.5e-7 to 3.5e-7 of float32 exponentials).
__device__ __forceinline__ void finish_row(const Stats& a, float z_label, float2& stats, double& picked) {
  const bool none = a.m == -INFINITY && a.s == 0.0f;
  const double ls = none ? 0.0 : log((double)a.s);
  stats = make_float2(a.m, (float)ls);
  picked = none ? 0.0 : ((double)z_label - (double)a.m) - ls;
}

// Many rows, whose labels and offsets have been checked: WAVE, a wave a row, else a workgroup.
template <int TYPE, bool WAVE>
__global__ __launch_bounds__(256) void row_stats_kernel(PrefArgs p) {
  typedef typename Elem<TYPE>::T T;
  if (!args_good(p.bad, p.host_bad)) return;
  const int64_t t = WAVE ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int tid = WAVE ? threadIdx.x & 63 : threadIdx.x;
  if (t >= p.n) return;
  const int label = p.labels[t];
  if (t < p.offsets[0] || t >= p.offsets[2 * p.pairs]) return;   // which sequence it is does not matter here
  if (label < 0) {
    if (tid == 0) {
      p.stats[2 * t] = p.stats[2 * t + 1] = 0.0f;
      p.picked[t] = 0.0;
    }
    return;
  }
  const T* z = (const T*)p.logits + t * p.ld;
  const float z_label = (float)z[label];
  Stats a;
  if (WAVE) a = scan<TYPE, 64>(z, 0, p.V, tid);
  else a = join_waves(scan<TYPE, 256>(z, 0, p.V, tid));
  if (tid) return;
  float2 st;
  finish_row(a, z_label, st, p.picked[t]);
  p.stats[2 * t] = st.x;
  p.stats[2 * t + 1] = st.y;
}

// Few rows: segment blockIdx.x % splits of row blockIdx.x / splits, and the checks of the call's labels and offsets on
// the way.  Nothing but the workspace is written.
template <int TYPE>
__global__ __launch_bounds__(256) void row_parts_kernel(PrefArgs p) {
  typedef typename Elem<TYPE>::T T;
  const int64_t t = blockIdx.x / p.splits;
  const int part = blockIdx.x % p.splits, tid = threadIdx.x;
  const int sequences = 2 * p.pairs;
  if (blockIdx.x == 0) {
    bool bad = false;
    for (int i = tid; i <= sequences; i += 256) {
      const int64_t v = p.offsets[i];
      bad |= v < 0 || v > p.n || (i < sequences && p.offsets[i + 1] < v);
    }
    if (__ballot(bad) && (tid & 63) == 0) atomicOr(p.bad, (uint32_t)OPS_BAD_OFFSETS);
  }
  if (t >= p.n) return;
  const int label = p.labels[t];
  if (t < p.offsets[0] || t >= p.offsets[sequences]) return;
  if (label >= p.V && tid == 0) atomicOr(p.bad, (uint32_t)OPS_BAD_LABEL);
  if (label < 0 || label >= p.V) return;
  const int per = ((p.V + p.splits - 1) / p.splits + 255) & ~255;
  const int first = min(p.V, part * per), last = min(p.V, first + per);
  const Stats a = join_waves(scan<TYPE, 256>((const T*)p.logits + t * p.ld, first, last, tid));
  if (tid == 0) ((Stats*)p.parts)[blockIdx.x] = a;
}

// One workgroup per pair: each sequence's rows are added in a fixed order.  FEW: their segments are joined first.
template <int TYPE, bool FEW>
__global__ __launch_bounds__(1024) void pair_loss_kernel(PrefArgs p) {
  typedef typename Elem<TYPE>::T T;
  __shared__ double part[2][16];
  if (!args_good(p.bad, p.host_bad)) return;
  const int64_t pair = blockIdx.x;
  const int tid = threadIdx.x, waves = blockDim.x >> 6;
  for (int w = 0; w < 2; ++w) {
    double s = 0.0;
    const int64_t end = p.offsets[2 * pair + w + 1];
    for (int64_t t = p.offsets[2 * pair + w] + tid; t < end; t += blockDim.x) {
      if (FEW) {
        const int label = p.labels[t];
        float2 st = make_float2(0.0f, 0.0f);
        double l = 0.0;
        if (label >= 0) {
          const Stats* q = (const Stats*)p.parts + t * p.splits;
          const float z_label = (float)((const T*)p.logits)[t * p.ld + label];
          Stats a = {-INFINITY, 0.0f};
          for (int i0 = 0; i0 < p.splits; i0 += 8) {   // eight loads on their way at a time
            Stats b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = q[min(i0 + i, p.splits - 1)];
            float m = a.m;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, b[i].m);
            const float base = base_of(m);
            a = {m, sum_at(a, base)};
#pragma unroll
            for (int i = 0; i < 8; ++i) a.s += i0 + i < p.splits ? sum_at(b[i], base) : 0.0f;
          }
          finish_row(a, z_label, st, l);
        }
        p.stats[2 * t] = st.x;
        p.stats[2 * t + 1] = st.y;
        s += l;
      } else {
        s += p.picked[t];
      }
    }
    s = wave_sum_d(s);
    if ((tid & 63) == 0) part[w][tid >> 6] = s;
  }
  __syncthreads();
  if (tid) return;
  double lp[2], ratio[2];
  for (int w = 0; w < 2; ++w) {
    lp[w] = part[w][0];
    for (int i = 1; i < waves; ++i) lp[w] += part[w][i];
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

// segment `part` of `splits` of a row's gradient
template <int TYPE, int THREADS>
__device__ __forceinline__ void row_gradient(const PrefArgs& p, int64_t t, int part, int tid) {
  typedef typename Elem<TYPE>::T T;
  typedef typename Vec<TYPE>::V V;
  constexpr int N = Vec<TYPE>::N, U = 4;
  const int label = p.labels[t];
  const int q = sequence_of_row(p.offsets, 2 * p.pairs, t);
  if (q < 0) return;
  const T* z = (const T*)p.logits + t * p.ld;
  T* dz = (T*)p.dlogits + t * p.lddl;
  const float m = p.stats[2 * t], ls = p.stats[2 * t + 1];
  const bool counts = label >= 0 && !(m == -INFINITY && ls == 0.0f);
  const float g = p.dlogp[q];
  const int per = ((p.V + p.splits - 1) / p.splits + 255) & ~255;
  const int first = min(p.V, part * per), last = min(p.V, first + per);
  if (!counts) {
    for (int v = first + tid * N; v < last; v += THREADS * N) {
      if (v + N <= last) {
        V w;
#pragma unroll
        for (int j = 0; j < N; ++j) w[j] = (T)0.0f;
        *(V*)(dz + v) = w;
      } else {
        for (int j = v; j < last; ++j) dz[j] = (T)0.0f;
      }
    }
    return;
  }
  // exp(x - m) times exp(-ls), not exp((x - m) - ls): a second difference of about ten would be rounded by what is more
  // than the whole error of the rest
  const float inverse = (float)exp(-(double)ls);
  auto slope = [&](float x, int v) {
    const float pr = exp_of<TYPE>(x - m) * inverse;
    return (T)(g * ((v == label ? 1.0f : 0.0f) - pr));
  };
  for (int v0 = first; v0 < last; v0 += THREADS * N * U) {
    V w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = v0 + (u * THREADS + tid) * N;
      if (v + N <= last) w[u] = *(const V*)(z + v);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = v0 + (u * THREADS + tid) * N;
      if (v + N <= last) {
#pragma unroll
        for (int j = 0; j < N; ++j) w[u][j] = slope((float)w[u][j], v + j);
        *(V*)(dz + v) = w[u];
      } else {
        for (int j = v; j < last; ++j) dz[j] = slope((float)z[j], j);
      }
    }
  }
}

// what is not in order of the call's offsets and labels, by thread i0 of `step`: offsets nondecreasing within [0, n];
// labels of rows inside a sequence below V (negative ones do not count)
__device__ __forceinline__ uint32_t bad_args(const PrefArgs& p, int64_t i0, int64_t step) {
  const int sequences = 2 * p.pairs;
  const int64_t first = p.offsets[0], last = p.offsets[sequences];
  uint32_t bad = 0;
  for (int64_t i = i0; i <= sequences; i += step) {
    const int64_t v = p.offsets[i];
    if (v < 0 || v > p.n || (i < sequences && p.offsets[i + 1] < v)) bad |= OPS_BAD_OFFSETS;
  }
  for (int64_t t = i0; t < p.n; t += step)
    if (t >= first && t < last && p.labels[t] >= p.V) bad |= OPS_BAD_LABEL;
  return bad;
}

// CHECK: every workgroup checks the call's labels and offsets itself
template <int TYPE, bool WAVE, bool CHECK>
__global__ __launch_bounds__(256) void preference_backward_kernel(PrefArgs p) {
  if (CHECK) {
    const uint32_t bad = bad_args(p, threadIdx.x, 256);
    const int offsets = __syncthreads_or(bad & OPS_BAD_OFFSETS), labels = __syncthreads_or(bad & OPS_BAD_LABEL);
    if (offsets || labels) {
      if (blockIdx.x == 0 && threadIdx.x == 0)
        *(volatile uint32_t*)p.host_bad = (offsets ? OPS_BAD_OFFSETS : 0u) | (labels ? OPS_BAD_LABEL : 0u);
      return;
    }
  } else {
    if (!args_good(p.bad, p.host_bad)) return;
  }
  if (WAVE) {
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t < p.n) row_gradient<TYPE, 64>(p, t, 0, threadIdx.x & 63);
  } else {
    const int64_t t = blockIdx.x / p.splits;
    if (t < p.n) row_gradient<TYPE, 256>(p, t, blockIdx.x % p.splits, threadIdx.x);
  }
}

__global__ __launch_bounds__(256) void check_preference_kernel(PrefArgs p) {
  uint32_t bad = bad_args(p, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) bad |= (uint32_t)__shfl_xor((int)bad, o, 64);
  if (bad && (threadIdx.x & 63) == 0) atomicOr(p.bad, bad);
}

void check(const PrefArgs& p, hipStream_t s) {
  const int64_t work = std::max<int64_t>(p.n, 2 * (int64_t)p.pairs + 1);
  check_preference_kernel<<<(unsigned)std::min<int64_t>((work + 255) / 256, 1024), 256, 0, s>>>(p);
}

// A wave takes a row of up to so many bytes, a workgroup a longer one: a workgroup's start and end are spread over four
// rows, a long row's own work over four waves.  Loss, us, wave / workgroup: bfloat16, 65,536 rows of 2,500 89 / 158,
// 20,000 of 7,000 62 / 67, 8,192 of 12,000 52 / 53, 16,384 of 15,000 99 / 93; float32, 16,384 of 5,000 66 / 79, of 8,000
// 103 / 98.  Gradient: bfloat16, 65,536 rows of 2,500 155 / 196, 40,000 of 4,096 134 / 136, 32,768 of 5,000 147 / 138;
// float32, 40,000 of 2,500 172 / 160.
constexpr int kWaveStats = 24576, kWaveGradient = 8192;

template <int TYPE>
void launch_loss_typed(const PrefArgs& p, hipStream_t s) {
  if (p.splits > 0) {
    row_parts_kernel<TYPE><<<(unsigned)(std::max<int64_t>(p.n, 1) * p.splits), 256, 0, s>>>(p);
    pair_loss_kernel<TYPE, true><<<p.pairs, 256, 0, s>>>(p);
    return;
  }
  check(p, s);
  if (p.V * (int)sizeof(typename Elem<TYPE>::T) <= kWaveStats) row_stats_kernel<TYPE, true><<<(unsigned)((p.n + 3) / 4), 256, 0, s>>>(p);
  else row_stats_kernel<TYPE, false><<<(unsigned)p.n, 256, 0, s>>>(p);
  pair_loss_kernel<TYPE, false><<<p.pairs, p.n / p.pairs > 8192 ? 1024 : 256, 0, s>>>(p);
}

// Up to so many rows and sequences every workgroup of the gradient checks them all, a few loads a thread, which saves
// the launch of a kernel ahead of it (2.5 of a small call's 20 us).
constexpr int64_t kCheckHere = 512;

template <int TYPE, bool WAVE>
void launch_gradient(const PrefArgs& p, int64_t blocks, hipStream_t s) {
  if (p.n <= kCheckHere && 2 * (int64_t)p.pairs <= kCheckHere) {
    preference_backward_kernel<TYPE, WAVE, true><<<(unsigned)blocks, 256, 0, s>>>(p);
  } else {
    check(p, s);
    preference_backward_kernel<TYPE, WAVE, false><<<(unsigned)blocks, 256, 0, s>>>(p);
  }
}

template <int TYPE>
void launch_backward_typed(PrefArgs p, hipStream_t s) {
  const int64_t rows = std::max<int64_t>(p.n, 1);
  if (p.V * (int)sizeof(typename Elem<TYPE>::T) <= kWaveGradient) {
    launch_gradient<TYPE, true>(p, (rows + 3) / 4, s);
  } else {
    // four workgroups and more on each of the 256 compute units where there are few rows
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(p.V / 2048, 2048 / rows));
    launch_gradient<TYPE, false>(p, rows * p.splits, s);
  }
}

}  // namespace

int preference_splits(int64_t n, int V) {
  // Few rows: their stats are finished by the pairs' workgroups, a thread a row, which saves a launch and lets long
  // rows be cut.  Up to 2,048 rows; segments of 4,096 candidates and more, as many as give the chip work.
  if (n > 2048) return 0;
  return (int)std::max<int64_t>(1, std::min<int64_t>(V / 4096, 2048 / std::max<int64_t>(n, 1)));
}

void launch_preference_loss(const PrefArgs& p, int type, hipStream_t s) {
  if (type == OT_F32) launch_loss_typed<OT_F32>(p, s);
  else if (type == OT_BF16) launch_loss_typed<OT_BF16>(p, s);
  else launch_loss_typed<OT_F16>(p, s);
}

void launch_preference_backward(const PrefArgs& p, int type, hipStream_t s) {
  if (type == OT_F32) launch_backward_typed<OT_F32>(p, s);
  else if (type == OT_BF16) launch_backward_typed<OT_BF16>(p, s);
  else launch_backward_typed<OT_F16>(p, s);
}
