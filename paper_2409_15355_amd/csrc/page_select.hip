// Which pages of a long cache a step reads (arXiv 2409.15355, Section 2.5: the answer's tokens over a context whose keys are cached).
//   bounds: per page, KV head and dimension the largest and the smallest key, in 8 bits with a power of two of the page and head;
//   scores: max over the step's query rows (in 8 bits, too) of sum_d max(c hi, c lo) = <max(c, 0), hi> + <min(c, 0), lo>: one product of whole
//     numbers of length 2 D (v_mfma_i32_32x32x32_i8), exact, so that which page is larger does not depend on the order of the sum;
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

// ---- bounds -----------------------------------------------------------------------------------------------------
// A wave a (page, KV head), D / 8 lanes a row.
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
#pragma unroll 1
  for (int at = first + part; at <= last; at += parts) {
    const int page = p.pages.table[seq * p.pages.stride + at];
    if (page < 0 || page >= p.pages.n_pages) continue;
    const int row0 = max(0, since - at * rows), row1 = min(rows, len - at * rows);
    const char *base = (const char *)(p.k.base + kvh * p.k.sh) + ((uint64_t)(uint32_t)page * p.k.page_b16 << 4) + c * 16;
    float hi[8], lo[8], top = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d) hi[d] = -INFINITY, lo[d] = INFINITY;
#pragma unroll 1
    for (int r = row0 + sub; r - sub < row1; r += RPI * kAhead) {
      u32x4_t x[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)  // (the last row more than once changes nothing)
        x[u] = *reinterpret_cast<const u32x4_t *>(base + (uint64_t)(uint32_t)min(r + u * RPI, row1 - 1) * p.k.rb);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          float f = d & 1 ? bf16_hi(x[u][d / 2]) : bf16_lo(x[u][d / 2]);
          f = f != f ? 0.f : f;
          hi[d] = fmaxf(hi[d], f);
          lo[d] = fminf(lo[d], f);
          top = fmaxf(top, fabsf(f));
        }
    }
#pragma unroll
    for (int m = CPR; m < 64; m *= 2)
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        hi[d] = fmaxf(hi[d], __shfl_xor(hi[d], m));
        lo[d] = fminf(lo[d], __shfl_xor(lo[d], m));
      }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    if (sub != 0) continue;
    int e = bound_exponent(top), by = -1;  // by: how far the old codes move, -1: there are none
    int8_t *const exp_at = p.exps + (int64_t)page * p.n_kv_heads + kvh;
    u32x2_t *const hi_at = reinterpret_cast<u32x2_t *>(p.codes + ((int64_t)page * p.n_kv_heads + kvh) * 2 * D + c * 8), *const lo_at = hi_at + D / 8;
    u32x2_t old_hi = {0, 0}, old_lo = {0, 0};
    if (row0 > 0) {
      const int old_e = *exp_at;
      old_hi = *hi_at, old_lo = *lo_at;
      e = max(e, old_e);
      by = min(e - old_e, 15);
    }
    u32x2_t new_hi = {0, 0}, new_lo = {0, 0};
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      int up = code_up(hi[d], e), down = code_down(lo[d], e);
      if (by >= 0) {
        const int was_up = (int)(int8_t)(old_hi[d / 4] >> (d % 4 * 8)), was_down = (int)(int8_t)(old_lo[d / 4] >> (d % 4 * 8));
        up = max(up, -(-was_up >> by));
        down = min(down, was_down >> by);
      }
      new_hi[d / 4] |= (uint32_t)(up & 0xff) << (d % 4 * 8);
      new_lo[d / 4] |= (uint32_t)(down & 0xff) << (d % 4 * 8);
    }
    *hi_at = new_hi;
    *lo_at = new_lo;
    if (lane == 0) *exp_at = (int8_t)e;
  }
}

// ---- scores -----------------------------------------------------------------------------------------------------
typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef int32_t i32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) i32x4_t lds_i32x4;
typedef __attribute__((address_space(3))) u32x2_t lds_u32x2;
typedef __attribute__((address_space(3))) int32_t lds_i;

// A wave takes 32 pages, whose codes lie in its registers; the query rows go through LDS in tiles of 32: max(c, 0), then min(c, 0).
constexpr int kScoreThreads = 256;
static_assert(kScorePages == kScoreThreads / 64 * 32, "32 pages a wave");
template <int D>
__global__ __launch_bounds__(kScoreThreads) void page_scores_kernel(PageSelectParams p, int chunks) {
  constexpr int K2 = 2 * D, CH = K2 / 32, CPR = D / 8, RPP = kScoreThreads / CPR;
  constexpr int ROWB = K2 + 16;  // (off the last row's banks)
  __shared__ __attribute__((aligned(16))) char smem_generic[32 * ROWB + 32 * 4];
  lds_char *const smem = (lds_char *)smem_generic;
  lds_i *const exps = (lds_i *)(smem + 32 * ROWB);
  const int kvh = blockIdx.x % p.n_kv_heads, rest = blockIdx.x / p.n_kv_heads, chunk = rest % chunks, seq = rest / chunks;
  const int len = max(0, min(p.seq_len[seq], p.cap));
  const int held = pages_held(p.pages, len);
  if (chunk * kScorePages >= held) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, hf = lane >> 5;
  const int at = chunk * kScorePages + wave * 32 + col;
  int page = p.pages.table[seq * p.pages.stride + min(at, held - 1)];
  page = page >= 0 && page < p.pages.n_pages ? page : 0;  // (not there: left out by the pick)
  const int64_t where = (int64_t)page * p.n_kv_heads + kvh;
  i32x4_t kc[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) kc[i] = *reinterpret_cast<const i32x4_t *>(p.codes + where * K2 + i * 32 + hf * 16);
  const int page_e = p.exps[where];

  const int n_rows = p.nq * p.group;
  float best = -INFINITY;
#pragma unroll 1
  for (int row0 = 0; row0 < n_rows; row0 += 32) {
    if (row0 > 0) __syncthreads();
    const int here = min(32, (n_rows - row0 + 7) & ~7);  // (the last row more than once changes nothing)
    for (int r = threadIdx.x / CPR; r < here; r += RPP) {
      const int of = min(row0 + r, n_rows - 1), i = (int)fast_div((uint32_t)of, p.group_div), c = threadIdx.x % CPR;
      const u32x4_t x = *reinterpret_cast<const u32x4_t *>(p.q + ((int64_t)seq * p.nq + i) * p.q_st + (kvh * p.group + of - i * p.group) * p.q_sh + c * 8);
      float f[8], top = 0.f;
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        f[d] = d & 1 ? bf16_hi(x[d / 2]) : bf16_lo(x[d / 2]);
        f[d] = f[d] != f[d] ? 0.f : f[d];
        top = fmaxf(top, fabsf(f[d]));
      }
#pragma unroll
      for (int m = 1; m < CPR; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
      const int e = bound_exponent(top);
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
    __syncthreads();
    i32x16_t s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const i32x4_t qc = *(lds_i32x4 *)(smem + col * ROWB + i * 32 + hf * 16);
      s = __builtin_amdgcn_mfma_i32_32x32x32_i8(qc, kc[i], s, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i * 8 >= here) break;
      const i32x4_t e = *(lds_i32x4 *)(exps + i * 8 + hf * 4);
#pragma unroll
      for (int v = 0; v < 4; ++v) best = fmaxf(best, __builtin_ldexpf((float)s[i * 4 + v], e[v]));
    }
  }
  best = fmaxf(best, other_half(best));
  if (hf == 0 && at < held) p.scores[((int64_t)seq * p.n_kv_heads + kvh) * p.score_stride + at] = __builtin_ldexpf(best, page_e);
}

// ---- pick -------------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(kPickThreads) void page_pick_kernel(PageSelectParams p) {
  __shared__ PickLds lds;
  const int kvh = blockIdx.x % p.n_kv_heads, seq = blockIdx.x / p.n_kv_heads;
  const int len = max(0, min(p.seq_len[seq], p.cap));
  const int held = pages_held(p.pages, len);
  const int newest = len > p.nq ? (int)fast_div((uint32_t)(len - p.nq), p.pages.page_div) : 0;
  const int last0 = min(held - p.n_last, newest);
  const int64_t list = (int64_t)seq * p.n_kv_heads + kvh;
  const float *scores = p.scores + list * p.score_stride;
  const int32_t *table = p.pages.table + seq * p.pages.stride;
  int32_t *selected = p.selected + list * p.n_select;
  float *scores_out = p.scores_out ? p.scores_out + list * p.n_select : nullptr;
  const int n = pick_largest(
      lds, held, p.n_select,
      [&](int i) {
        const int page = table[i];
        const float x = scores[i];
        if (page < 0 || page >= p.pages.n_pages) return 0u;
        return i < p.n_first || i >= last0 ? kPickAlways : pick_key(x);
      },
      [&](int at, int i) {
        selected[at] = i;
        if (scores_out) scores_out[at] = scores[i];
      });
  for (int j = n + threadIdx.x; j < p.n_select; j += kPickThreads) {
    selected[j] = -1;
    if (scores_out) scores_out[j] = -INFINITY;
  }
}

}  // namespace

hipError_t launch_page_bounds(const PageBoundsParams &p, int head_dim, hipStream_t stream) {
  const int64_t lists = (int64_t)p.n_seqs * p.n_kv_heads, pages = ((int64_t)p.cap + p.pages.page_rows - 1) / p.pages.page_rows;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(pages, 32768 / lists)), wgs = (lists * parts + kBoundWaves - 1) / kBoundWaves;
  if (wgs < 1 || wgs > kMaxWorkgroups) return hipErrorInvalidValue;
  if (head_dim == 128) page_bounds_kernel<128><<<(unsigned)wgs, kBoundThreads, 0, stream>>>(p, (int)parts);
  else page_bounds_kernel<64><<<(unsigned)wgs, kBoundThreads, 0, stream>>>(p, (int)parts);
  return hipGetLastError();
}
hipError_t launch_page_scores(const PageSelectParams &p, int head_dim, hipStream_t stream) {
  const int64_t pages = ((int64_t)p.cap + p.pages.page_rows - 1) / p.pages.page_rows, chunks = (pages + kScorePages - 1) / kScorePages;
  const int64_t wgs = (int64_t)p.n_seqs * p.n_kv_heads * chunks;
  if (wgs < 1 || wgs > kMaxWorkgroups) return hipErrorInvalidValue;
  if (head_dim == 128) page_scores_kernel<128><<<(unsigned)wgs, kScoreThreads, 0, stream>>>(p, (int)chunks);
  else page_scores_kernel<64><<<(unsigned)wgs, kScoreThreads, 0, stream>>>(p, (int)chunks);
  return hipGetLastError();
}
hipError_t launch_page_pick(const PageSelectParams &p, hipStream_t stream) {
  const int64_t wgs = (int64_t)p.n_seqs * p.n_kv_heads;
  if (wgs < 1 || wgs > kMaxPickWorkgroups) return hipErrorInvalidValue;
  page_pick_kernel<<<(unsigned)wgs, kPickThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace ba
