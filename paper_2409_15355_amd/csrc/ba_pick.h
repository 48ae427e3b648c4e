// The n largest of a list, by one workgroup: places of them in ascending order, of equal ones the first.
#pragma once

#include "ba_lds.h"

namespace ba {

// Order of floats as unsigned numbers above 0 (0: not in the list); -0 as 0, a NaN below everything, kPickAlways above it.
constexpr uint32_t kPickAlways = 0xffffffffu;
__device__ __forceinline__ uint32_t pick_key(float x) {
  if (x != x) return 1u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Digits of 11, 11 and 10 bits, from the highest: a histogram of those that share the digits found so far, in LDS, says in which bin the
// n-th largest lies; then every wave counts and writes a run of places of its own.
constexpr int kPickWaves = 16, kPickThreads = kPickWaves * 64, kPickBins = 2048;
struct PickLds {
  uint32_t hist[kPickBins];
  uint32_t wave_sum[kPickWaves], wave_equal[kPickWaves];
  uint32_t bin, left, total;
};
// key(i), i in [0, n): its order, 0: not in the list.  emit(position, i) for the `want` largest (all, if there are no more).  Returns their number.
template <typename Key, typename Emit>
__device__ __forceinline__ int pick_largest(PickLds &l, int n, int want, Key &&key, Emit &&emit) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t found = 0, left = (uint32_t)want, total = 0;
  int bits = 32;
  bool all = false;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int width = pass == 2 ? 10 : 11, shift = bits - width;
    for (int b = tid; b < kPickBins; b += kPickThreads) l.hist[b] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kPickThreads) {
      const uint32_t u = key(i);
      if (u != 0 && (bits == 32 || (u >> (bits & 31)) == found)) atomicAdd(&l.hist[(u >> shift) & ((1u << width) - 1)], 1u);
    }
    __syncthreads();
    // two bins a thread, from the highest down
    const int top = kPickBins - 1 - 2 * tid;
    const uint32_t a = l.hist[top], b = l.hist[top - 1];
    uint32_t upto = a + b;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const uint32_t o = __shfl_up(upto, m);
      if (lane >= m) upto += o;
    }
    if (lane == 63) l.wave_sum[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += l.wave_sum[w];
    if (pass == 0) {
      if (tid == kPickThreads - 1) l.total = upto;
      __syncthreads();
      total = l.total;
      if (total <= left) {
        all = true;
        break;
      }
    }
    const uint32_t before = upto - a - b;
    if (before < left && left <= upto) {
      const bool first = left <= before + a;
      l.bin = (uint32_t)(first ? top : top - 1);
      l.left = left - before - (first ? 0 : a);
    }
    __syncthreads();
    found = (pass == 0 ? 0 : found << width) | l.bin;
    left = l.left;
    bits = shift;
  }
  // those above the last one, and the first `left` of its equals
  if (all || want <= 0) found = all ? 0 : kPickAlways, left = 0;
  const int run = ((n + kPickThreads - 1) / kPickThreads) * 64, begin = wave * run, end = min(n, begin + run);
  uint32_t above = 0, equal = 0;
  for (int i = begin + lane; i < begin + run; i += 64) {
    const uint32_t u = i < end ? key(i) : 0;
    above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(u > found));
    equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(u == found && u != 0));
  }
  __syncthreads();
  if (lane == 0) l.wave_sum[wave] = above, l.wave_equal[wave] = equal;
  __syncthreads();
  above = equal = 0;
  for (int w = 0; w < wave; ++w) above += l.wave_sum[w], equal += l.wave_equal[w];
  const uint64_t below_me = (1ull << lane) - 1;
  for (int i = begin + lane; i < begin + run; i += 64) {
    const uint32_t u = i < end ? key(i) : 0;
    const uint64_t gt = __builtin_amdgcn_ballot_w64(u > found), eq = __builtin_amdgcn_ballot_w64(u == found && u != 0);
    const uint32_t g = above + __builtin_popcountll(gt & below_me), e = equal + __builtin_popcountll(eq & below_me);
    if (u > found || (u == found && u != 0 && e < left)) emit((int)(g + min(e, left)), i);
    above += __builtin_popcountll(gt);
    equal += __builtin_popcountll(eq);
  }
  return (int)min(total, (uint32_t)max(want, 0));
}

}  // namespace ba
