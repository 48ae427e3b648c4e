// Which pages of a long cache a step reads (arXiv 2409.15355, Section 2.5: the answer's tokens over a context whose keys are cached).
//   bounds: per page, KV head and dimension the largest and the smallest key, in 8 bits with a power of two of the page and head;
//   scores: max over the step's query rows (in 8 bits, too) of sum_d max(c hi, c lo) = <max(c, 0), hi> + <min(c, 0), lo>: one product of whole
//     numbers of length 2 D (v_mfma_i32_16x16x64_i8), exact, so that which page is larger does not depend on the order of the sum;
//   pick: the largest ones of every (sequence, KV head), ba_pick.h.
#include <algorithm>

#include "ba_long.h"
#include "ba_pick.h"

namespace ba {
namespace {

// the least e with top <= 127 * 2^e, within limits: top = m 2^x with m in [1/2, 1).  An infinity's is the largest: were it left out, the codes of
// rows that come later could not say any more that it was there.
__device__ __forceinline__ int bound_exponent(float top) {
  const int x = __builtin_amdgcn_frexp_expf(top);
  const int e = __builtin_amdgcn_frexp_mantf(top) <= 127.f / 128.f ? x - 7 : x - 6;
  return top == 0.f ? kBoundMinExp : top == INFINITY ? kBoundMaxExp : max(kBoundMinExp, min(kBoundMaxExp, e));
}
__device__ __forceinline__ int clamp_code(float x) { return (int)fminf(127.f, fmaxf(-127.f, x)); }
// (what is too small for 32 bits next to the largest is not nothing: rounding goes away from zero here)
__device__ __forceinline__ int code_up(float x, int e) { return max(clamp_code(ceilf(__builtin_ldexpf(x, -e))), x > 0.f ? 1 : -127); }
__device__ __forceinline__ int code_down(float x, int e) { return min(clamp_code(floorf(__builtin_ldexpf(x, -e))), x < 0.f ? -1 : 127); }

// pages that a sequence's tokens lie in
__device__ __forceinline__ int pages_held(const PagedTableParams &t, int len) {
  return len > 0 ? min(t.max_pages, (int)fast_div((uint32_t)(len - 1), t.page_div) + 1) : 0;
}

// Two bf16 numbers as two whole ones of the same order (and back: the map is its own inverse), and the larger, the smaller of each.
typedef short s16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t ordered(uint32_t x) {
  return x ^ (__builtin_bit_cast(uint32_t, __builtin_bit_cast(s16x2_t, x) >> 15) & 0x7fff7fffu);
}
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2_t, a), __builtin_bit_cast(s16x2_t, b)));
}
__device__ __forceinline__ uint32_t smaller(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2_t, a), __builtin_bit_cast(s16x2_t, b)));
}
constexpr uint32_t kOrderedLeast = 0x80008000u, kOrderedMost = 0x7fff7fffu;
// a NaN in either half: above +infinity or below -infinity in this order
__device__ __forceinline__ bool any_nan(uint32_t hi, uint32_t lo) {
  const s16x2_t h = __builtin_bit_cast(s16x2_t, hi), l = __builtin_bit_cast(s16x2_t, lo);
  return h[0] > 0x7f80 || h[1] > 0x7f80 || l[0] < (short)(0xff80 ^ 0x7fff) || l[1] < (short)(0xff80 ^ 0x7fff);
}
// x of both lanes i and i ^ M joined by op (M 8, 16, 32)
template <int M, typename Op>
__device__ __forceinline__ uint32_t join_lanes(uint32_t x, Op &&op) {
  if constexpr (M == 8) return op(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, true));  // (eight lanes on, within sixteen)
  else if constexpr (M == 16) {
    auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return op((uint32_t)r[0], (uint32_t)r[1]);
  } else {
    auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return op((uint32_t)r[0], (uint32_t)r[1]);
  }
}
// the largest of each run of N lanes (8 or 16), in every lane of the run (as sum_over_lanes)
template <int N>
__device__ __forceinline__ float max_over_lanes(float x) {
  auto with = [&](auto ctrl) __attribute__((always_inline)) {
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true)));
  };
  with(std::integral_constant<int, 0xb1>{});
  with(std::integral_constant<int, 0x4e>{});
  with(std::integral_constant<int, 0x141>{});
  if constexpr (N == 16) with(std::integral_constant<int, 0x140>{});
  return x;
}

// ---- bounds -----------------------------------------------------------------------------------------------------
// A wave a (page, KV head), D / 8 lanes a row; nothing is computed twice, each key is read once.  Bound by HBM where much is new (31,744 tokens, 8
// heads of 128: 16 us, 65 MB in and 4 out), by the launch in a decoding step (128 sequences 4.6 us).
// Waves of a launch.  us, 2,048 / 4,096 / 8,192: 128 sequences that take one token more 4.7 / 5.6 / 8.0, all of 31,744 tokens 16.0 / 15.3 / 15.4.
constexpr int kBoundTarget = 2048;
constexpr int kBoundThreads = 256, kBoundWaves = kBoundThreads / 64;
template <int D>
__global__ __launch_bounds__(kBoundThreads) void page_bounds_kernel(PageBoundsParams p, int parts) {
  constexpr int CPR = D / 8, RPI = 64 / CPR, kAhead = 4;
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kBoundWaves + (threadIdx.x >> 6));
  const int kvh = id % p.n_kv_heads, rest = id / p.n_kv_heads, part = rest % parts, seq = rest / parts;
  if (seq >= p.n_seqs) return;
  const int rows = p.pages.page_rows;
  const int len = max(0, min(p.seq_len[seq], p.cap)), since = p.from ? max(0, p.from[seq]) : 0;
  if (since >= len) return;
  const int c = lane % CPR, sub = lane / CPR;
  const int first = (int)fast_div((uint32_t)since, p.pages.page_div), last = min(p.pages.max_pages - 1, (int)fast_div((uint32_t)(len - 1), p.pages.page_div));
  // A run of rows at a time, of the page that the wave is at; the next one's are asked for ahead of its sums.  (Few waves with much on the way
  // each: a launch of many costs more than it reads where there is little new.)
  if (first + part > last) return;
  constexpr int RUN = RPI * kAhead;
  struct Run {
    int n, page, row0, row1, r;  // the wave's n-th page, its number; its new rows; the run's first row
  };
  const int n_pages = (last - first - part) / parts + 1;
  int ids = 0;  // entries of the table for 64 of the wave's pages, one a lane
  auto look_up = [&](int n) __attribute__((always_inline)) {
    ids = p.pages.table[seq * p.pages.stride + first + part + min(n + lane, n_pages - 1) * parts];
  };
  auto begin_page = [&](int n) __attribute__((always_inline)) {
    if ((n & 63) == 0) look_up(n);
    const int page = __builtin_amdgcn_readlane(ids, n & 63), at = first + part + n * parts;
    Run run = {n, page >= 0 && page < p.pages.n_pages ? page : -1, 0, 0, 0};
    run.row0 = run.r = max(0, since - at * rows);
    run.row1 = min(rows, len - at * rows);
    return run;
  };
  const char *const head = (const char *)(p.k.base + kvh * p.k.sh) + c * 16;
  auto fetch = [&](const Run &n, u32x4_t (&x)[kAhead]) __attribute__((always_inline)) {
    const char *const base = head + ((uint64_t)(uint32_t)max(n.page, 0) * p.k.page_b16 << 4);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)  // (the last row more than once changes nothing; a page that is not there: page 0, nothing is written)
      x[u] = *reinterpret_cast<const u32x4_t *>(base + (uint64_t)(uint32_t)min(n.r + u * RPI + sub, n.row1 - 1) * p.k.rb);
  };
  u32x4_t x[kAhead], next_x[kAhead];
  Run now = begin_page(0);
  fetch(now, x);
  // Largest and smallest as whole numbers in the order of the keys, two dimensions a register: half the instructions.  A NaN (0 by definition)
  // stands out among them at the end, and the page is gone through again.
  uint32_t hi[4], lo[4];
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int w = 0; w < 4; ++w) hi[w] = kOrderedLeast, lo[w] = kOrderedMost;
  };
  auto add = [&](uint32_t (&v)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int w = 0; w < 4; ++w) hi[w] = larger(hi[w], v[w]), lo[w] = smaller(lo[w], v[w]);
  };
  auto join_rows = [&]() __attribute__((always_inline)) {
    const auto up = [](uint32_t a, uint32_t b) { return larger(a, b); };
    const auto down = [](uint32_t a, uint32_t b) { return smaller(a, b); };
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (CPR == 8) hi[w] = join_lanes<8>(hi[w], up), lo[w] = join_lanes<8>(lo[w], down);
      hi[w] = join_lanes<32>(join_lanes<16>(hi[w], up), up);
      lo[w] = join_lanes<32>(join_lanes<16>(lo[w], down), down);
    }
  };
  clear();
  // (the two sets of rows take turns: to move one into the other would wait for it)
  auto take = [&](u32x4_t (&x)[kAhead], u32x4_t (&next_x)[kAhead]) __attribute__((always_inline)) {
    const bool ends = now.r + RUN >= now.row1;
    Run next = now;
    next.r += RUN;
    const bool more = !ends || now.n + 1 < n_pages;
    if (!more) next = now;  // (asked for all the same: the waits count what is on the way)
    else if (ends) next = begin_page(now.n + 1);
    fetch(next, next_x);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      uint32_t v[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) v[w] = ordered(x[u][w]);
      add(v);
    }
    if (ends) {
      join_rows();
      bool nan = false;
#pragma unroll
      for (int w = 0; w < 4; ++w) nan |= any_nan(hi[w], lo[w]);
      if (__builtin_amdgcn_ballot_w64(nan) != 0) {
        clear();
        const char *const base = head + ((uint64_t)(uint32_t)max(now.page, 0) * p.k.page_b16 << 4);
#pragma unroll 1
        for (int r = now.row0; r < now.row1; r += RPI) {
          u32x4_t y = *reinterpret_cast<const u32x4_t *>(base + (uint64_t)(uint32_t)min(r + sub, now.row1 - 1) * p.k.rb);
          uint32_t v[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            if (bf16_lo(y[w]) != bf16_lo(y[w])) y[w] &= 0xffff0000u;
            if (bf16_hi(y[w]) != bf16_hi(y[w])) y[w] &= 0xffffu;
            v[w] = ordered(y[w]);
          }
          add(v);
        }
        join_rows();
      }
      // every lane has all rows' of its eight dimensions now; of those, two are a lane's to write
      uint32_t my_hi = hi[0], my_lo = lo[0];
      float top = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        hi[w] = ordered(hi[w]), lo[w] = ordered(lo[w]);
        my_hi = sub == w ? hi[w] : my_hi, my_lo = sub == w ? lo[w] : my_lo;
        top = fmaxf(top, fmaxf(fmaxf(fabsf(bf16_lo(hi[w])), fabsf(bf16_hi(hi[w]))), fmaxf(fabsf(bf16_lo(lo[w])), fabsf(bf16_hi(lo[w])))));
      }
      top = max_over_lanes<CPR>(top);
      if (sub < 4 && now.page >= 0) {
        my_hi = sub == 0 ? hi[0] : my_hi, my_lo = sub == 0 ? lo[0] : my_lo;
        int e = bound_exponent(top);
        int8_t *const exp_at = p.exps + (int64_t)now.page * p.n_kv_heads + kvh;
        uint16_t *const hi_at = reinterpret_cast<uint16_t *>(p.codes + ((int64_t)now.page * p.n_kv_heads + kvh) * 2 * D + c * 8 + sub * 2), *const lo_at = hi_at + D / 2;
        int was[4], by = 0;  // the old codes, and how far they move
        if (now.row0 > 0) {
          const int old_e = *exp_at;
          const uint32_t was_hi = *hi_at, was_lo = *lo_at;
          was[0] = (int)(int8_t)was_hi, was[1] = (int)(int8_t)(was_hi >> 8), was[2] = (int)(int8_t)was_lo, was[3] = (int)(int8_t)(was_lo >> 8);
          e = max(e, old_e);
          by = min(e - old_e, 15);
        }
        int up0 = code_up(bf16_lo(my_hi), e), up1 = code_up(bf16_hi(my_hi), e), down0 = code_down(bf16_lo(my_lo), e), down1 = code_down(bf16_hi(my_lo), e);
        if (now.row0 > 0) {
          up0 = max(up0, -(-was[0] >> by)), up1 = max(up1, -(-was[1] >> by));
          down0 = min(down0, was[2] >> by), down1 = min(down1, was[3] >> by);
        }
        *hi_at = (uint16_t)((up0 & 0xff) | (up1 & 0xff) << 8);
        *lo_at = (uint16_t)((down0 & 0xff) | (down1 & 0xff) << 8);
        if (lane == 0) *exp_at = (int8_t)e;
      }
      clear();
    }
    now = next;
    return more;
  };
  while (take(x, next_x) && take(next_x, x)) {
  }
}

// ---- scores -----------------------------------------------------------------------------------------------------
typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i32x4_t lds_i32x4;
typedef __attribute__((address_space(3))) u32x2_t lds_u32x2;
typedef __attribute__((address_space(3))) int32_t lds_i;

// A wave takes 32 pages, 16 to a product (v_mfma_i32_16x16x64_i8), their codes in its registers.  The query rows lie in LDS, tiles of 16:
// max(c, 0), then min(c, 0).  Bound by the 256 bytes here and there that a page has of a head: 64 sequences of up to 1,000 pages, 8 rows, 66 MB, 17 us, of
// one of 2,000 pages 4.1.  The same: 32 pages to a product (lanes that take 32 bytes a row); fewer workgroups that walk on, the next pages' codes ahead.
constexpr int kScoreThreads = 256, kScoreRows = 16;
static_assert(kScorePages == kScoreThreads / 64 * 32, "32 pages a wave");
// A tile of query rows in 8 bits into LDS.
template <int D, int kThreads>
__device__ __forceinline__ void stage_queries(const PageSelectParams &p, int seq, int kvh, int row0, lds_char *smem, lds_i *exps) {
  constexpr int CPR = D / 8, RPP = kThreads / CPR, ROWB = 2 * D + 16;  // (off the last row's banks)
  const int n_rows = p.nq * p.group;
#pragma unroll 1
  for (int r = threadIdx.x / CPR; r < kScoreRows; r += RPP) {  // (the last row more than once changes nothing)
    const int of = min(row0 + r, n_rows - 1), i = (int)fast_div((uint32_t)of, p.group_div), c = threadIdx.x % CPR;
    const u32x4_t x = *reinterpret_cast<const u32x4_t *>(p.q + ((int64_t)seq * p.nq + i) * p.q_st + (kvh * p.group + of - i * p.group) * p.q_sh + c * 8);
    float f[8], top = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      f[d] = d & 1 ? bf16_hi(x[d / 2]) : bf16_lo(x[d / 2]);
      f[d] = f[d] != f[d] ? 0.f : f[d];
      top = fmaxf(top, fabsf(f[d]));
    }
    const int e = bound_exponent(max_over_lanes<CPR>(top));
    u32x2_t up = {0, 0}, down = {0, 0};
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const int code = clamp_code(__builtin_rintf(__builtin_ldexpf(f[d], -e)));
      up[d / 4] |= (uint32_t)(max(code, 0) & 0xff) << (d % 4 * 8);
      down[d / 4] |= (uint32_t)(min(code, 0) & 0xff) << (d % 4 * 8);
    }
    *(lds_u32x2 *)(smem + r * ROWB + c * 8) = up;
    *(lds_u32x2 *)(smem + r * ROWB + D + c * 8) = down;
    if (c == 0) exps[r] = e;
  }
}
// Pages of a wave, 16 to a lane's `col`: their codes, and their scores for a tile of query rows.
template <int D>
struct WavePages {
  static constexpr int K2 = 2 * D, CH = K2 / 64, ROWB = K2 + 16;
  int e[2];
  bool there[2];
  i32x4_t codes[2][CH];
  __device__ __forceinline__ void load(const PageSelectParams &p, int seq, int kvh, int first, int held, int lane) {
    int page[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) page[g] = p.pages.table[seq * p.pages.stride + min(first + g * 16 + (lane & 15), held - 1)];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      there[g] = page[g] >= 0 && page[g] < p.pages.n_pages;
      const int64_t where = (int64_t)(there[g] ? page[g] : 0) * p.n_kv_heads + kvh;
#pragma unroll
      for (int i = 0; i < CH; ++i) codes[g][i] = *reinterpret_cast<const i32x4_t *>(p.codes + where * K2 + i * 64 + (lane >> 4) * 16);
      e[g] = p.exps[where];
    }
  }
  __device__ __forceinline__ void score(lds_char *smem, lds_i *exps, int lane, float (&best)[2]) const {
    i32x4_t s[2] = {};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const i32x4_t qc = *(lds_i32x4 *)(smem + (lane & 15) * ROWB + i * 64 + (lane >> 4) * 16);
#pragma unroll
      for (int g = 0; g < 2; ++g) s[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(qc, codes[g][i], s[g], 0, 0, 0);
    }
    const i32x4_t qe = *(lds_i32x4 *)(exps + (lane >> 4) * 4);
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int v = 0; v < 4; ++v) best[g] = fmaxf(best[g], __builtin_ldexpf((float)s[g][v], qe[v]));
  }
  // the largest of all rows, in the page's own units; -infinity: it is not there
  __device__ __forceinline__ float result(int g, float best) const {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(best), __float_as_uint(best), false, false);
    best = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    best = fmaxf(best, other_half(best));
    return there[g] ? __builtin_ldexpf(best, e[g]) : -INFINITY;
  }
};
template <int D>
__global__ __launch_bounds__(kScoreThreads) void page_scores_kernel(PageSelectParams p, int chunks) {
  __shared__ __attribute__((aligned(16))) char smem_generic[kScoreRows * (2 * D + 16) + kScoreRows * 4];
  lds_char *const smem = (lds_char *)smem_generic;
  lds_i *const exps = (lds_i *)(smem + kScoreRows * (2 * D + 16));
  // The heads of a sequence's pages one after the other on one XCD (ids go round the eight): the exponents of a page are one piece of memory.
  const int kvh = blockIdx.x / 8 % p.n_kv_heads, unit = blockIdx.x / 8 / p.n_kv_heads * 8 + blockIdx.x % 8, seq = unit / chunks;
  const int first = (unit + seq) % chunks * kScorePages;  // (turned on from sequence to sequence, so that no XCD gets all the beginnings)
  if (seq >= p.n_seqs) return;
  const int len = max(0, min(p.seq_len[seq], p.cap)), held = pages_held(p.pages, len);
  if (first >= held) return;
  const int lane = threadIdx.x & 63, mine = first + (threadIdx.x >> 6) * 32;
  WavePages<D> pages;
  pages.load(p, seq, kvh, mine, held, lane);
  float best[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
  for (int row0 = 0; row0 < p.nq * p.group; row0 += kScoreRows) {
    if (row0 > 0) __syncthreads();
    stage_queries<D, kScoreThreads>(p, seq, kvh, row0, smem, exps);
    __syncthreads();
    pages.score(smem, exps, lane, best);
  }
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float x = pages.result(g, best[g]);
    const int at = mine + g * 16 + (lane & 15);
    if (lane >> 4 == g && at < held) p.scores[((int64_t)seq * p.n_kv_heads + kvh) * p.score_stride + at] = x;
  }
}

// ---- pick -------------------------------------------------------------------------------------------------------
// Latency (see ba_pick.h): eight lists of 2,000 pages 5.9 us, 512 of up to 1,000 5.6.
template <int W, int E, typename Value>
__device__ __forceinline__ void pick_pages(const PageSelectParams &p, PickLds<W> &lds, int seq, int kvh, int len, int held, Value &&value) {
  const int newest = len > p.nq ? (int)fast_div((uint32_t)(len - p.nq), p.pages.page_div) : 0;
  const int last0 = min(held - p.n_last, newest);
  const int64_t list = (int64_t)seq * p.n_kv_heads + kvh;
  int32_t *selected = p.selected + list * p.n_select;
  float *scores_out = p.scores_out ? p.scores_out + list * p.n_select : nullptr;
  const int n = pick_largest<W, E>(
      lds, held, p.n_select, value,
      [&](int i, float x) { return x == -INFINITY ? 0u : i < p.n_first || i >= last0 ? kPickAlways : pick_key(x); },  // (-infinity: not there)
      [&](int at, int i, float x) {
        selected[at] = i;
        if (scores_out) scores_out[at] = x;
      });
  for (int j = n + threadIdx.x; j < p.n_select; j += W * 64) {
    selected[j] = -1;
    if (scores_out) scores_out[j] = -INFINITY;
  }
}
template <int W, int E>
__global__ __launch_bounds__(W * 64) void page_pick_kernel(PageSelectParams p) {
  __shared__ PickLds<W> lds;
  const int kvh = blockIdx.x % p.n_kv_heads, seq = blockIdx.x / p.n_kv_heads;
  const int len = max(0, min(p.seq_len[seq], p.cap)), held = pages_held(p.pages, len);
  const float *scores = p.scores + ((int64_t)seq * p.n_kv_heads + kvh) * p.score_stride;
  pick_pages<W, E>(p, lds, seq, kvh, len, held, [&](int i) { return scores[i]; });
}
// Both in one launch, where a list's pages are few: scores stay in LDS.  Latency: table, codes, product, choice one behind the other, 63 pages 5.7 us.
constexpr int kSelectOneWaves = 4;
template <int D, int W>
__global__ __launch_bounds__(W * 64) void page_select_kernel(PageSelectParams p) {
  __shared__ PickLds<W> lds;
  __shared__ float scores[kSelectOneLaunch];
  __shared__ __attribute__((aligned(16))) char smem_generic[kScoreRows * (2 * D + 16) + kScoreRows * 4];
  lds_char *const smem = (lds_char *)smem_generic;
  lds_i *const exps = (lds_i *)(smem + kScoreRows * (2 * D + 16));
  const int kvh = blockIdx.x % p.n_kv_heads, seq = blockIdx.x / p.n_kv_heads;
  const int len = max(0, min(p.seq_len[seq], p.cap)), held = pages_held(p.pages, len);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_rows = p.nq * p.group;
  if (n_rows <= kScoreRows) {
    stage_queries<D, W * 64>(p, seq, kvh, 0, smem, exps);
    __syncthreads();
  }
#pragma unroll 1
  for (int first = 0; first < held; first += W * 32) {  // (the same in all waves)
    const int mine = first + wave * 32;
    WavePages<D> pages;
    pages.load(p, seq, kvh, mine, held, lane);
    float best[2] = {-INFINITY, -INFINITY};
    if (n_rows <= kScoreRows) {
      pages.score(smem, exps, lane, best);
    } else {
#pragma unroll 1
      for (int row0 = 0; row0 < n_rows; row0 += kScoreRows) {
        __syncthreads();
        stage_queries<D, W * 64>(p, seq, kvh, row0, smem, exps);
        __syncthreads();
        pages.score(smem, exps, lane, best);
      }
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const float x = pages.result(g, best[g]);
      const int at = mine + g * 16 + (lane & 15);
      if (lane >> 4 == g && at < held) scores[at] = x;
    }
  }
  __syncthreads();
  pick_pages<W, kSelectOneLaunch / (W * 64)>(p, lds, seq, kvh, len, held, [&](int i) { return scores[i]; });
}

}  // namespace

hipError_t launch_page_bounds(const PageBoundsParams &p, int head_dim, hipStream_t stream) {
  const int64_t lists = (int64_t)p.n_seqs * p.n_kv_heads, pages = ((int64_t)p.cap + p.pages.page_rows - 1) / p.pages.page_rows;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(pages, kBoundTarget / lists)), wgs = (lists * parts + kBoundWaves - 1) / kBoundWaves;
  if (wgs < 1 || wgs > kMaxWorkgroups) return hipErrorInvalidValue;
  if (head_dim == 128) page_bounds_kernel<128><<<(unsigned)wgs, kBoundThreads, 0, stream>>>(p, (int)parts);
  else page_bounds_kernel<64><<<(unsigned)wgs, kBoundThreads, 0, stream>>>(p, (int)parts);
  return hipGetLastError();
}
hipError_t launch_page_scores(const PageSelectParams &p, int head_dim, hipStream_t stream) {
  const int64_t pages = ((int64_t)p.cap + p.pages.page_rows - 1) / p.pages.page_rows, chunks = (pages + kScorePages - 1) / kScorePages;
  const int64_t wgs = ((int64_t)p.n_seqs * chunks + 7) / 8 * 8 * p.n_kv_heads;
  if (wgs < 1 || wgs > kMaxWorkgroups) return hipErrorInvalidValue;
  if (head_dim == 128) page_scores_kernel<128><<<(unsigned)wgs, kScoreThreads, 0, stream>>>(p, (int)chunks);
  else page_scores_kernel<64><<<(unsigned)wgs, kScoreThreads, 0, stream>>>(p, (int)chunks);
  return hipGetLastError();
}
hipError_t launch_page_select(const PageSelectParams &p, int head_dim, hipStream_t stream) {
  const int64_t wgs = (int64_t)p.n_seqs * p.n_kv_heads;
  if (wgs < 1 || wgs > kMaxPickWorkgroups || p.score_stride > kSelectOneLaunch) return hipErrorInvalidValue;
  if (head_dim == 128) page_select_kernel<128, kSelectOneWaves><<<(unsigned)wgs, kSelectOneWaves * 64, 0, stream>>>(p);
  else page_select_kernel<64, kSelectOneWaves><<<(unsigned)wgs, kSelectOneWaves * 64, 0, stream>>>(p);
  return hipGetLastError();
}
hipError_t launch_page_pick(const PageSelectParams &p, hipStream_t stream) {
  const int64_t wgs = (int64_t)p.n_seqs * p.n_kv_heads;
  if (wgs < 1 || wgs > kMaxPickWorkgroups) return hipErrorInvalidValue;
  return with_pick_shape(p.score_stride, [&](auto w, auto e) {
    page_pick_kernel<decltype(w)::value, decltype(e)::value><<<(unsigned)wgs, decltype(w)::value * 64, 0, stream>>>(p);
    return hipGetLastError();
  });
}

}  // namespace ba
