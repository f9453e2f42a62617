// Device helpers shared by the operators on a caller's own tensors.
#pragma once

#include "device_common.h"
#include "operators.h"

template <int TYPE> struct Elem;
template <> struct Elem<OT_F32> { typedef float T; };
template <> struct Elem<OT_BF16> { typedef __bf16 T; };
template <> struct Elem<OT_F16> { typedef _Float16 T; };

// 16 bytes of values at any place that their type allows (the hardware reads and writes them so)
template <int TYPE> struct Vec;
template <> struct Vec<OT_F32> {
  static constexpr int N = 4;
  typedef float V __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct Vec<OT_BF16> {
  static constexpr int N = 8;
  typedef __bf16 V __attribute__((ext_vector_type(8), aligned(2)));
};
template <> struct Vec<OT_F16> {
  static constexpr int N = 8;
  typedef _Float16 V __attribute__((ext_vector_type(8), aligned(2)));
};

// A workgroup's verdict on the call's arguments: true where the checks ahead of it found nothing.  The first
// workgroup hands the word to the host otherwise.
__device__ __forceinline__ bool args_good(const uint32_t* bad, uint32_t* host_bad) {
  const uint32_t v = *bad;
  if (v && blockIdx.x == 0 && threadIdx.x == 0) *(volatile uint32_t*)host_bad = v;
  return v == 0;
}

// the sequence that holds row t: the last one with offsets[q] <= t < offsets[q + 1] (empty ones in front of it share
// its start), or -1
__device__ __forceinline__ int sequence_of_row(const int64_t* offsets, int sequences, int64_t t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = sequences;
  while (true) {
    const int step = (hi - lo + 63) >> 6;
    const int q = lo + lane * step;
    const bool in = q < hi && offsets[q] <= t;
    const int c = __popcll(__ballot(in));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    if (step == 1) break;
    hi = min(hi, lo + step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  return t < offsets[lo + 1] ? lo : -1;
}
