// The n largest of a list, by one workgroup: places of them in ascending order, of equal ones the first.
#pragma once

#include "ba_lds.h"
#include "ba_long.h"

namespace ba {

// Order of floats as unsigned numbers; -0 as 0, a NaN below everything.  0: not in the list, kPickAlways: taken ahead of all others.
constexpr uint32_t kPickAlways = 0xffffffffu;
__device__ __forceinline__ uint32_t pick_key(float x) {
  if (x != x) return 1u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

constexpr int kPickFew = 128;  // (no more than threads)
// W: waves of the workgroup, 4 or 16; two bins a thread
template <int W>
struct PickLds {
  uint32_t hist[W * 128];
  alignas(16) uint32_t a[W], b[W], least[W], most[W], above[W], equal[W];  // of each wave
  alignas(16) uint32_t few[kPickFew];
  uint32_t bin, left, in_bin, n_few;
};
// Across the 64 lanes without a trip through LDS: the smallest, the largest (in all of them), sums up to each lane.
template <typename Op>
__device__ __forceinline__ uint32_t pick_reduce(uint32_t x, Op &&op) {
  auto with = [&](auto ctrl) __attribute__((always_inline)) { x = op(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, decltype(ctrl)::value, 0xf, 0xf, true)); };
  with(std::integral_constant<int, 0xb1>{});   // (as sum_over_lanes)
  with(std::integral_constant<int, 0x4e>{});
  with(std::integral_constant<int, 0x141>{});
  with(std::integral_constant<int, 0x140>{});
  auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = op((uint32_t)r[0], (uint32_t)r[1]);
  r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return op((uint32_t)r[0], (uint32_t)r[1]);
}
__device__ __forceinline__ uint32_t pick_sums_upto(uint32_t x) {
  auto add = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
  };
  using std::integral_constant;
  add(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});  // one, two, four, eight lanes on within sixteen
  add(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  add(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  add(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  add(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});  // a sixteen's last lane to the next sixteen, the second and the fourth
  add(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});  // the first half's last lane to the other half
  return x;
}
// The sum of what the waves in front of this one have left in `of`.
template <int W>
__device__ __forceinline__ uint32_t pick_before(const uint32_t (&of)[W], int wave, int lane) {
  const uint32_t x = lane < wave ? of[lane & (W - 1)] : 0;
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)pick_reduce(x, [](uint32_t a, uint32_t b) { return a + b; }));
}

// value(i), i in [0, n): a number; key(i, number): its order.  emit(position, i, number) for the `want` largest (all that are in the list, if there
// are no more).  Returns their number.
// E > 0: n is at most E times the threads, and every thread keeps its numbers and keys; E = 0: they are looked up again by every pass.
//
// Every wave has a run of places of its own.  The smallest and the largest key say how many bits they differ in; a histogram by the highest
// nine or eleven of those says in which bin the last one that is taken lies, and so on with the next ones within it, until its bin is taken whole,
// holds equal keys only, or few enough to be ranked one against the other.  Bound by latency, and with a list a compute unit by the
// instructions of its waves, which share four SIMDs: what is the same in all waves is done by one of them.
template <int W, int E, typename Value, typename Key, typename Emit>
__device__ __forceinline__ int pick_largest(PickLds<W> &l, int n, int want, Value &&value, Key &&key, Emit &&emit) {
  constexpr int kPickThreads = W * 64, kPickBins = 2 * kPickThreads, kDigit = W == 16 ? 11 : 9;
  static_assert(1 << kDigit == kPickBins, "a bin for each digit");
  auto uniform = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
  const int tid = threadIdx.x, lane = tid & 63, wave = (int)uniform(tid >> 6);
  const int steps = (n + kPickThreads - 1) / kPickThreads, run = steps * 64, begin = wave * run;
  float number[E > 0 ? E : 1];
  uint32_t mine[E > 0 ? E : 1];
  if constexpr (E > 0) {
    constexpr int kTogether = E < 8 ? E : 8;  // (asked for together)
#pragma unroll
    for (int g = 0; g < E; g += kTogether) {
#pragma unroll
      for (int s = g; s < g + kTogether; ++s) mine[s] = 0, number[s] = 0.f;
      if (g >= steps) continue;
#pragma unroll
      for (int s = g; s < g + kTogether; ++s) number[s] = value(min(begin + s * 64 + lane, n - 1));
#pragma unroll
      for (int s = g; s < g + kTogether; ++s) {
        const int i = begin + s * 64 + lane;
        mine[s] = s < steps && i < n ? key(i, number[s]) : 0;
      }
    }
  }
  // f(step, key, number): this lane's of every step, the same steps in all lanes
  auto each = [&](auto &&f) __attribute__((always_inline)) {
    if constexpr (E > 0) {
      constexpr int kOnce = E < 4 ? E : 4;  // (behind the last step keys are 0; a branch a step: 14,085 tokens 13.4 us, not 12.3)
#pragma unroll
      for (int g = 0; g < E; g += kOnce)
        if (g < steps)
#pragma unroll
          for (int s = g; s < g + kOnce; ++s) f(s, mine[s], number[s]);
    } else {
      constexpr int kTogether = 8;  // (eight lists of 100,000, 4,096 kept: one by one 153 to 182 us, so 143)
#pragma unroll 1
      for (int s0 = 0; s0 < steps; s0 += kTogether) {
        float x[kTogether];
#pragma unroll
        for (int s = 0; s < kTogether; ++s) x[s] = value(min(begin + (s0 + s) * 64 + lane, n - 1));
#pragma unroll
        for (int s = 0; s < kTogether; ++s) {
          const int i = begin + (s0 + s) * 64 + lane;
          if (s0 + s < steps) f(s0 + s, i < n ? key(i, x[s]) : 0u, x[s]);
        }
      }
    }
  };
  auto ordinary = [](uint32_t u) { return u - 1 < kPickAlways - 1; };

  // ---- how many there are, and between what
  for (int b = tid; b < kPickBins; b += kPickThreads) l.hist[b] = 0;
  if (tid == 0) l.n_few = 0;
  if (tid < kPickFew) l.few[tid] = 0;
  uint32_t least = kPickAlways, most = 0, n_always = 0, n_ordinary = 0;
  each([&](int, uint32_t u, float) {
    n_always += __builtin_popcountll(__builtin_amdgcn_ballot_w64(u == kPickAlways));
    n_ordinary += __builtin_popcountll(__builtin_amdgcn_ballot_w64(ordinary(u)));
    least = min(least, u - 1);  // (0 comes out above all)
    most = max(most, u == kPickAlways ? 0 : u);
  });
  least = pick_reduce(least, [](uint32_t a, uint32_t b) { return min(a, b); });
  most = pick_reduce(most, [](uint32_t a, uint32_t b) { return max(a, b); });
  least += least != kPickAlways;  // (of the ordinary ones, if there is one)
  if (lane == 0) l.a[wave] = n_always, l.b[wave] = n_ordinary, l.least[wave] = least, l.most[wave] = most;
  __syncthreads();
  {  // a lane for each wave's
    const int w = lane & (W - 1);
    n_always = lane < W ? l.a[w] : 0, n_ordinary = lane < W ? l.b[w] : 0;
    least = uniform(pick_reduce(l.least[w], [](uint32_t a, uint32_t b) { return min(a, b); }));
    most = uniform(pick_reduce(l.most[w], [](uint32_t a, uint32_t b) { return max(a, b); }));
    const auto add = [](uint32_t a, uint32_t b) { return a + b; };
    n_always = uniform(pick_reduce(n_always, add)), n_ordinary = uniform(pick_reduce(n_ordinary, add));
  }
  const uint32_t total = min(n_always + n_ordinary, (uint32_t)max(want, 0));
  uint32_t left = total - min(total, n_always);  // ordinary ones that are taken

  // ---- the last one that is taken: those above `found`, and the first `left` of its equals
  uint32_t found = 0;
  if (left == 0) {
    found = kPickAlways - 1;  // (no ordinary key is above it)
  } else if (left == n_ordinary) {
    left = 0;
  } else {
    uint32_t base = least;
    int bits = 32 - __builtin_clz((most - least) | 1);
    while (true) {  // (the same in all threads)
      const int shift = max(0, bits - kDigit);
      const uint32_t reach = bits < 32 ? min((1u << bits) - 1, most - base) : most - base;  // (0 and kPickAlways lie further on)
      each([&](int, uint32_t u, float) {
        if (u - base <= reach) atomicAdd(&l.hist[(u - base) >> shift], 1u);
      });
      __syncthreads();
      // two bins a thread, from the highest down
      const int top = kPickBins - 1 - 2 * tid;
      const uint32_t first = l.hist[top], second = l.hist[top - 1];
      uint32_t upto = pick_sums_upto(first + second);
      if (lane == 63) l.a[wave] = upto;
      __syncthreads();
      upto += pick_before(l.a, wave, lane);
      const uint32_t before = upto - first - second;
      if (before < left && left <= upto) {
        const bool in_first = left <= before + first;
        l.bin = (uint32_t)(in_first ? top : top - 1);
        l.left = left - before - (in_first ? 0 : first);
        l.in_bin = in_first ? first : second;
      }
      __syncthreads();
      base += uniform(l.bin) << shift;
      left = uniform(l.left);
      bits = shift;
      const uint32_t in_bin = uniform(l.in_bin);
      if (left == in_bin) {  // all of them
        found = base - 1;
        left = 0;
        break;
      }
      if (shift == 0) {  // equal keys
        found = base;
        break;
      }
      if (in_bin <= kPickFew) {
        each([&](int, uint32_t u, float) {
          if (u - base <= min((1u << bits) - 1, most - base)) l.few[atomicAdd(&l.n_few, 1u)] = u;
        });
        __syncthreads();
        if (tid < (int)in_bin) {  // how many are above this thread's, and how many are its equals
          typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
          const uint32_t my = l.few[tid];
          uint32_t above = 0, equals = 0;
#pragma unroll 4
          for (int o = 0; o < (int)in_bin; o += 4) {  // (behind the last one there are zeros)
            const u32x4 u = *reinterpret_cast<const u32x4 *>(l.few + o);
#pragma unroll
            for (int c = 0; c < 4; ++c) above += u[c] > my, equals += u[c] == my;
          }
          if (above < left && left <= above + equals) l.bin = my, l.left = left - above;  // (its equals write the same)
        }
        __syncthreads();
        found = uniform(l.bin);
        left = uniform(l.left);
        break;
      }
      for (int b = tid; b < kPickBins; b += kPickThreads) l.hist[b] = 0;
      __syncthreads();
    }
  }

  // ---- their places, in order
  uint32_t above = 0, equal = 0;
  each([&](int, uint32_t u, float) { above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(u > found)); });
  if (left > 0) each([&](int, uint32_t u, float) { equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(u == found)); });
  if (lane == 0) l.above[wave] = above, l.equal[wave] = equal;
  __syncthreads();
  above = pick_before(l.above, wave, lane);
  if (left > 0) equal = pick_before(l.equal, wave, lane);
  auto lanes_before = [&](uint64_t mask, uint32_t from) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, from)); };
  each([&](int s, uint32_t u, float x) {
    const uint64_t gt = __builtin_amdgcn_ballot_w64(u > found);
    uint64_t eq = 0;
    if (left > 0) eq = __builtin_amdgcn_ballot_w64(u == found);
    if ((gt | eq) == 0) return;
    const uint32_t e = lanes_before(eq, equal), at = lanes_before(gt, above) + min(e, left);
    if (u > found || (u == found && e < left)) emit((int)at, begin + s * 64 + lane, x);
    above += __builtin_popcountll(gt);
    equal += __builtin_popcountll(eq);
  });
  return (int)total;
}
// Calls f with the waves and the number of keys that a thread has to keep for lists of up to n.
// us a call of eight lists, 4 / 8 / 16 waves: selection out of 2,000 pages 11.8 / 10.9 / 9.7, eviction out of 2,064 tokens (rows in a
// launch of their own) 11.6 / 12.0 / 11.5; of 512 lists: selection out of up to 1,000 pages, 4 / 16 waves 8 / 12 (the kernel alone).
template <typename F>
auto with_pick_shape(int64_t n, F &&f) {
  using std::integral_constant;
  constexpr integral_constant<int, 4> four{};
  constexpr integral_constant<int, 16> sixteen{};
  if (n <= kPickFourWaves) return f(four, integral_constant<int, 4>{});
  if (n <= 4 * 1024) return f(sixteen, integral_constant<int, 4>{});
  if (n <= 8 * 1024) return f(sixteen, integral_constant<int, 8>{});
  if (n <= 16 * 1024) return f(sixteen, integral_constant<int, 16>{});
  if (n <= 32 * 1024) return f(sixteen, integral_constant<int, 32>{});
  return f(sixteen, integral_constant<int, 0>{});
}

}  // namespace ba
