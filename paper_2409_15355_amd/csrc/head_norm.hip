// Norms of queries and keys for each head with the rotation of Eq. 1 (arXiv 2409.15355, Section 2.3) in the same pass, the
// gradients of that, and the same on the way into the pages of a cache.
//
// A head vector x of D elements becomes y = R(pos) (w o x r), r = (mean x^2 + eps)^-1/2.  With the gradient dy of y:
// g = R(pos)^T dy, dw = sum over tokens and heads of g o (x r), b = w o g, dx = r (b - (x r) mean(b o x r)).
//
// One pass over memory, 10 to 25 operations an element: the stream bounds it in large calls, launch and the way to memory and
// back in small ones.  The 16-byte pieces c and c + CH / 2 of a vector belong to one lane, so that either pairing of the rotation
// stays inside a lane, and the sum of squares is three or four adds of neighbouring lanes.  A lane meets the heads of one token
// one after the other, so cos and sin (some 40 operations a pair) are worked out once for all of them.
// Measured, bf16, heads of 128: 32 over 8 heads, 32,000 tokens, 655 MB read and written in 112 us, 5.9 TB/s (a copy of 1 GiB: 5.2); their
// gradients, 32,513 tokens, 999 MB in 177 us and the gains' sums in 6; keys and values of 31,744 tokens into pages, 8 heads, 260 MB in
// 50 us, 5.2 TB/s.  fp32, 8 over 2 heads of 64, 2,077 tokens: 5.9 us.  64 tokens take 4.5 us, one into a page 4.3: launch, and to memory and back.
#include <algorithm>
#include <type_traits>

#include "ba_lds.h"
#include "ba_paged.h"
#include "ba_rotate.h"

namespace ba {
namespace {

constexpr int kFewSlots = 16;
// kSlots: heads of a token that a workgroup takes at a time
template <typename T, int D, int kSlots>
struct RowGeo {
  static constexpr int VEC = 16 / sizeof(T);
  static constexpr int CH = D / VEC;       // 16-byte pieces of a head vector
  static constexpr int TPV = CH / 2;       // lanes per head vector
  static constexpr int TPT = TPV * kSlots; // lanes per token
  static constexpr int TOK = kRotThreads / TPT;
  static_assert(TOK >= 1, "a token's lanes fit a workgroup");
};

// a lane's VEC pairs: in its two pieces one after the other (interleaved), or of its first with its second (half)
template <int VEC, int CH, int LAYOUT>
__device__ __forceinline__ int lane_pair(int c, int e) {
  return LAYOUT == 0 ? (e < VEC / 2 ? c * (VEC / 2) + e : (c + CH / 2) * (VEC / 2) + (e - VEC / 2)) : c * VEC + e;
}
template <int VEC, int CH, int LAYOUT>
__device__ __forceinline__ void lane_turns(const RopeTable &rt, int c, int pos, float (&cs)[VEC], float (&sn)[VEC]) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) sincos_phase(rope_phase(pos, rt.turns[lane_pair<VEC, CH, LAYOUT>(c, e)]), cs[e], sn[e]);
}
template <int VEC, int LAYOUT>
__device__ __forceinline__ void turn_pieces(float (&x)[VEC], float (&y)[VEC], const float (&cs)[VEC], const float (&sn)[VEC]) {
  if (LAYOUT == 0) {
#pragma unroll
    for (int e = 0; e < VEC / 2; ++e) {
      rotate(x[2 * e], x[2 * e + 1], cs[e], sn[e]);
      rotate(y[2 * e], y[2 * e + 1], cs[VEC / 2 + e], sn[VEC / 2 + e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) rotate(x[e], y[e], cs[e], sn[e]);
  }
}
// a lane's gains
template <int VEC, int CH>
__device__ __forceinline__ void lane_gains(const void *w, bool f32, int c, float (&wx)[VEC], float (&wy)[VEC]) {
  auto piece = [&](int at, float (&to)[VEC]) __attribute__((always_inline)) {
    if (!w) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) to[e] = 1.f;
    } else if (f32) {
#pragma unroll
      for (int e = 0; e < VEC; e += 4) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>((const float *)w + at + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) to[e + i] = x[i];
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; e += 4) {
        const u32x2_t x = *reinterpret_cast<const u32x2_t *>((const uint16_t *)w + at + e);
        to[e] = bf16_lo(x[0]), to[e + 1] = bf16_hi(x[0]), to[e + 2] = bf16_lo(x[1]), to[e + 3] = bf16_hi(x[1]);
      }
    }
  };
  piece(c * VEC, wx);
  piece((c + CH / 2) * VEC, wy);
}

// The row of the paged cache that a token's keys and values go to.
struct CacheRow {
  bool kept;  // there is one
  int64_t page;
  int row;
};
__device__ __forceinline__ CacheRow cache_row(const HeadRowsParams &p, int t) {
  CacheRow r = {false, 0, 0};
  const int seq = p.seq_of_token ? p.seq_of_token[t] : t, at = p.cache_pos[t];
  if (seq >= 0 && seq < p.n_seqs && at >= 0 && at < p.max_rows) {
    const uint32_t i = fast_div((uint32_t)at, p.page_div);
    r.row = at - (int)i * p.page_rows;
    r.page = p.page_table[seq * p.stride_table + i];
    r.kept = r.page >= 0 && r.page < p.n_pages;
  }
  return r;
}

// A few heads of one tensor and token on their way: kBatch of them in flight per lane.  kPast: see past_caches.
template <typename T, int D, int LAYOUT, bool kPaged, int kPast>
struct HeadRows {
  static constexpr int kBatch = 4;
  typedef Chunk<T, (kPast > 1), (kPast > 0)> Ch;
  static constexpr int VEC = Ch::VEC, CH = D / VEC, TPV = CH / 2;
  const HeadRowsParams &p;
  int kind, c, n;
  const T *src;
  bool norm, turn;
  float wx[VEC], wy[VEC];
  Ch x[kBatch], y[kBatch];
  __device__ __forceinline__ HeadRows(const HeadRowsParams &p_, int kind_, int c_, int t)
      : p(p_), kind(kind_), c(c_), n(p_.n_heads[kind_]), src((const T *)p_.src[kind_] + t * p_.src_st[kind_] + c_ * VEC),
        norm(kind_ != kRowsV && p_.eps >= 0.f), turn(kind_ != kRowsV && p_.rope) {}
  __device__ __forceinline__ void gains() {
    if (norm) lane_gains<VEC, CH>(p.weight[kind], p.weight_f32, c, wx, wy);
  }
  __device__ __forceinline__ void load(int h0, int step) {
    const int64_t sh = p.src_sh[kind];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int h = min(h0 + u * step, n - 1);
      x[u].load(src + h * sh);
      y[u].load(src + h * sh + (CH / 2) * VEC);
    }
  }
  __device__ __forceinline__ T *target(int t, const CacheRow &to) const {
    T *dst = (T *)p.dst[kind] + c * VEC;
    return dst + (kPaged && kind != kRowsQ ? to.page * p.dst_page[kind] + to.row * p.dst_st[kind] : t * p.dst_st[kind]);
  }
  __device__ __forceinline__ void store(T *dst, int h0, int step, const float (&cs)[VEC], const float (&sn)[VEC]) {
    const int64_t sh = p.dst_sh[kind];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int h = h0 + u * step;
      if (h >= n) break;
      if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) ss += x[u].f[e] * x[u].f[e] + y[u].f[e] * y[u].f[e];
        const float r = rsqrtf(sum_over_lanes<TPV>(ss) * (1.0f / D) + p.eps);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          x[u].f[e] *= r * wx[e];
          y[u].f[e] *= r * wy[e];
        }
      }
      if (turn) turn_pieces<VEC, LAYOUT>(x[u].f, y[u].f, cs, sn);
      x[u].store(dst + h * sh);
      y[u].store(dst + h * sh + (CH / 2) * VEC);
    }
  }
};

// Calls that fill the chip: a lane takes every fourth head of a token's tensors, one tensor after the other.
// kPaged: keys and values go to their rows of a paged cache.
template <typename T, int D, int LAYOUT, bool kPaged, int kPast>
__global__ __launch_bounds__(kRotThreads) void head_rows_kernel(HeadRowsParams p, RopeTable rt) {
  using G = RowGeo<T, D, kManySlots>;
  using Rows = HeadRows<T, D, LAYOUT, kPaged, kPast>;
  const int c = threadIdx.x % G::TPV, slot = threadIdx.x / G::TPV % kManySlots;
  const int t = blockIdx.x * G::TOK + threadIdx.x / G::TPT;
  if (t >= p.n_tokens) return;
  float cs[G::VEC], sn[G::VEC];
  if (p.rope) lane_turns<G::VEC, G::CH, LAYOUT>(rt, c, p.positions ? p.positions[t] : t, cs, sn);
  CacheRow to = {};
  if constexpr (kPaged) to = cache_row(p, t);
#pragma unroll 1
  for (int kind = 0; kind < (kPaged ? 3 : 2); ++kind) {
    if (!p.src[kind] || (kPaged && kind != kRowsQ && !to.kept)) continue;
    Rows rows(p, kind, c, t);
    rows.gains();
    T *dst = rows.target(t, to);
#pragma unroll 1
    for (int h0 = slot; h0 < rows.n; h0 += kManySlots * Rows::kBatch) {
      rows.load(h0, kManySlots);
      rows.store(dst, h0, kManySlots, cs, sn);
    }
  }
}

// Calls bound by the way to memory and back: a workgroup per tensor (blockIdx.y) and token or two, all of its loads ahead of
// everything else; cos and sin are worked out once for the token's heads, a pair or less to a lane.
template <typename T, int D, int LAYOUT, bool kPaged>
__global__ __launch_bounds__(kRotThreads) void head_rows_few_kernel(HeadRowsParams p, RopeTable rt) {
  using G = RowGeo<T, D, kFewSlots>;
  using Rows = HeadRows<T, D, LAYOUT, kPaged, 0>;
  constexpr int VEC = G::VEC;
  static_assert(G::TPT >= D / 2, "a lane for every pair");
  __shared__ float2 turns[G::TOK][D / 2];
  const int kind = blockIdx.y;
  const int c = threadIdx.x % G::TPV, slot = threadIdx.x / G::TPV % kFewSlots, tl = threadIdx.x / G::TPT, j = threadIdx.x % G::TPT;
  const int t = min((int)blockIdx.x * G::TOK + tl, p.n_tokens - 1);
  const bool mine = (int)blockIdx.x * G::TOK + tl < p.n_tokens;
  if (!p.src[kind]) return;
  Rows rows(p, kind, c, t);
  rows.load(slot, kFewSlots);
  rows.gains();
  CacheRow to = {};
  if (kPaged && kind != kRowsQ) to = cache_row(p, t);
  float cs[VEC], sn[VEC];
  if (rows.turn) {
    if (j < D / 2) {
      float cj, sj;
      sincos_phase(rope_phase(p.positions ? p.positions[t] : t, rt.turns[j]), cj, sj);
      turns[tl][j] = make_float2(cj, sj);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float2 f = turns[tl][lane_pair<VEC, G::CH, LAYOUT>(c, e)];
      cs[e] = f.x, sn[e] = f.y;
    }
  }
  if (!mine || (kPaged && kind != kRowsQ && !to.kept)) return;
  T *dst = rows.target(t, to);
#pragma unroll 1
  for (int h0 = slot; h0 < rows.n; h0 += kFewSlots * Rows::kBatch) {
    if (h0 != slot) rows.load(h0, kFewSlots);
    rows.store(dst, h0, kFewSlots, cs, sn);
  }
}

// The first wg_q workgroups take queries, the others keys, a chunk of tokens each and every wg_q-th (n_wg - wg_q-th) after it, and leave
// their sums of the gain's gradient (one workgroup for each tensor: the gradient itself).  A lane takes every kSlots-th head of its token,
// the next one's pieces on their way meanwhile.
template <typename T, int D, int LAYOUT, int kSlots, int kPast>
__global__ __launch_bounds__(kRotThreads, 4) void norm_backward_kernel(NormBackwardParams p, RopeTable rt) {
  using G = RowGeo<T, D, kSlots>;
  typedef Chunk<T, (kPast > 1), (kPast > 0)> Ch;
  constexpr int VEC = G::VEC, CH = G::CH, kVecs = kRotThreads / G::TPV;
  __shared__ float red[kVecs][D];
  const HeadRowsParams &r = p.rows;
  const int kind = (int)blockIdx.x >= p.wg_q, first = blockIdx.x - (kind ? p.wg_q : 0), step = kind ? p.n_wg - p.wg_q : p.wg_q;
  const int c = threadIdx.x % G::TPV, slot = threadIdx.x / G::TPV % kSlots, n = r.n_heads[kind];
  const T *src = (const T *)r.src[kind] + c * VEC, *grad = (const T *)p.grad[kind] + c * VEC;
  T *dst = (T *)r.dst[kind] + c * VEC;
  struct Pieces {
    u32x4_t x, y, gx, gy;  // as they lie in memory: half the registers that they take as floats
    int pos;
  };
  auto load = [&](Pieces &w, int64_t t, int h) __attribute__((always_inline)) {
    const T *s = src + t * r.src_st[kind] + h * r.src_sh[kind], *g = grad + t * p.grad_st[kind] + h * p.grad_sh[kind];
    w.x = load_row_piece<(kPast > 1)>((const char *)(s));
    w.y = load_row_piece<(kPast > 1)>((const char *)(s + (CH / 2) * VEC));
    w.gx = load_row_piece<(kPast > 1)>((const char *)(g));
    w.gy = load_row_piece<(kPast > 1)>((const char *)(g + (CH / 2) * VEC));
    w.pos = r.positions ? r.positions[t] : (int)t;
  };
  int64_t t = (int64_t)first * G::TOK + threadIdx.x / G::TPT;
  int h = slot;
  bool live = t < r.n_tokens && h < n;
  Pieces next;
  if (live) load(next, t, h);
  // (the gains wait in LDS: with them, too, a lane would hold more than the 128 registers that let four workgroups share a compute unit)
  __shared__ __attribute__((aligned(16))) float gains[D];
  if ((int)threadIdx.x < G::TPV) {
    float wx[VEC], wy[VEC];
    lane_gains<VEC, CH>(r.weight[kind], r.weight_f32, c, wx, wy);
#pragma unroll
    for (int e = 0; e < VEC; ++e) gains[c * VEC + e] = wx[e], gains[(c + CH / 2) * VEC + e] = wy[e];
  }
  __syncthreads();
  float dw[2 * VEC], cs[VEC], sn[VEC];
#pragma unroll
  for (int e = 0; e < 2 * VEC; ++e) dw[e] = 0.f;
#pragma unroll 1
  while (live) {
    int64_t t2 = t;
    int h2 = h + kSlots;
    if (h2 >= n) h2 = slot, t2 += (int64_t)step * G::TOK;
    live = t2 < r.n_tokens;
    struct {
      Ch x, y, gx, gy;
      int pos;
    } cur;
    cur.x.expand(next.x), cur.y.expand(next.y), cur.gx.expand(next.gx), cur.gy.expand(next.gy);
    cur.pos = next.pos;
    if (live) load(next, t2, h2);
    if (r.rope) {
      if (h == slot) {
        lane_turns<VEC, CH, LAYOUT>(rt, c, cur.pos, cs, sn);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sn[e] = -sn[e];  // the gradient turns back
      }
      turn_pieces<VEC, LAYOUT>(cur.gx.f, cur.gy.f, cs, sn);
    }
    int cw = c;
    asm volatile("" : "+v"(cw));  // (read anew each time)
    float ss = 0.f, dot = 0.f, wx[VEC], wy[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      wx[e] = gains[cw * VEC + e], wy[e] = gains[(cw + CH / 2) * VEC + e];
      ss += cur.x.f[e] * cur.x.f[e] + cur.y.f[e] * cur.y.f[e];
      dot += cur.x.f[e] * (cur.gx.f[e] * wx[e]) + cur.y.f[e] * (cur.gy.f[e] * wy[e]);
    }
    const float rs = rsqrtf(sum_over_lanes<G::TPV>(ss) * (1.0f / D) + r.eps);
    const float m = sum_over_lanes<G::TPV>(dot) * (1.0f / D) * rs * rs;  // mean(b o x r) r
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      dw[e] += cur.gx.f[e] * (cur.x.f[e] * rs);
      dw[VEC + e] += cur.gy.f[e] * (cur.y.f[e] * rs);
      cur.x.f[e] = rs * (cur.gx.f[e] * wx[e] - cur.x.f[e] * m);
      cur.y.f[e] = rs * (cur.gy.f[e] * wy[e] - cur.y.f[e] * m);
    }
    T *to = dst + t * r.dst_st[kind] + h * r.dst_sh[kind];
    cur.x.store(to);
    cur.y.store(to + (CH / 2) * VEC);
    t = t2, h = h2;
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    red[threadIdx.x / G::TPV][c * VEC + e] = dw[e];
    red[threadIdx.x / G::TPV][(c + CH / 2) * VEC + e] = dw[VEC + e];
  }
  __syncthreads();
  if (threadIdx.x < D) {
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) sum += red[v][threadIdx.x];
    if (!p.one_each) p.partial[(int64_t)blockIdx.x * D + threadIdx.x] = sum;
    else if (p.weight_grad[kind]) p.weight_grad[kind][threadIdx.x] = sum;
  }
}

// partial [n_wg][D] -> the gradients of the gains, in a fixed order (64-bit sums: they are few)
constexpr int kGainThreads = 1024, kGainCols = 16;
template <int D>
__global__ __launch_bounds__(kGainThreads) void gain_sums_kernel(NormBackwardParams p) {
  constexpr int kCols = kGainCols, kWays = kGainThreads / kCols;
  __shared__ double red[kWays][kCols];
  const int kind = blockIdx.x / (D / kCols), col = blockIdx.x % (D / kCols) * kCols + threadIdx.x % kCols, way = threadIdx.x / kCols;
  if (!p.weight_grad[kind]) return;
  const int first = kind ? p.wg_q : 0, n = kind ? p.n_wg - p.wg_q : p.wg_q;
  static_assert(kNormBwdMaxWg % kWays == 0, "as many rounds as fit the registers");
  float x[kNormBwdMaxWg / kWays];  // (all of a thread's loads go out together)
#pragma unroll
  for (int r = 0; r < kNormBwdMaxWg / kWays; ++r) {
    const int i = r * kWays + way;
    x[r] = i < n ? p.partial[(int64_t)(first + i) * D + col] : 0.f;
  }
  double sum = 0.0;
#pragma unroll
  for (int r = 0; r < kNormBwdMaxWg / kWays; ++r) sum += (double)x[r];
  red[way][threadIdx.x % kCols] = sum;
  __syncthreads();
  for (int half = kWays / 2; half > 0; half /= 2) {
    if (way < half) red[way][threadIdx.x % kCols] += red[way + half][threadIdx.x % kCols];
    __syncthreads();
  }
  if (way == 0) p.weight_grad[kind][col] = (float)red[0][threadIdx.x];
}

// Which of the two, us a call, many / few (Python face and all, without which none is made in less than 3.7).  32 over 8 heads of 128, norm and
// rotation, bf16: 64 tokens 7.6 / 5.2, 512 8.2 / 5.1, 1,024 9.5 / 7.0, 2,048 11.3 / 11.1, 3,000 13.9 / 15.1; fp32: 512 7.5 / 6.5, 1,024 9.7 / 9.7,
// 1,536 12.1 / 12.2, 2,048 16.1 / 15.1, 3,000 21.7 / 25.8; heads of 64, fp32: 1,024 7.6 / 6.3, 2,048 9.8 / 9.6.  16 over 8 of 128, bf16: 1,024
// 6.9 / 5.5, 2,048 8.9 / 9.5; fp32: 768 6.4 / 6.1, 1,024 7.4 / 8.1.  8 over 2 of 64, fp32: 1,024 4.7 / 4.4, 1,536 5.0 / 5.3.
// Keys and values of 8 heads into pages: 512 5.3 / 5.3, 2,048 6.5 / 7.8.  The first one's lanes wait for memory once for every sixteen heads.
inline bool few_tokens(const HeadRowsParams &p) {
  const int heads = std::max(p.src[kRowsQ] ? p.n_heads[kRowsQ] : 0, p.n_heads[kRowsK]);
  return p.n_tokens <= (heads > kManySlots * 4 ? 2048 : 1024);
}
// Which accesses go past the caches, by the bytes that a call reads and writes (`tensors` for each of its own): none, 1 the stores, 2 the
// loads as well.  us, none / stores / both, 32 over 8 heads of 128, bf16: forward 84 MB 17.0 / 17.5 / 18.5, 168 MB 36.1 / 29.9 / 32.1, 246 MB
// 50.7 / 47.7 / 45.2, 655 MB 123.5 / 118.1 / 111.8; backward 63 MB 20.2 / 20.4 / 21.6, 126 MB 33.8 / 29.5 / 31.7, 252 MB 58.0 / 56.1 /
// 53.8, 999 MB 196 / 190 / 184; keys and values into pages 67 MB 13.1 / 13.5 / 15.3, 131 MB 29.9 / 22.8 / 27.1, 260 MB 54.2 / 51.7 / 50.9.
inline int past_caches(const HeadRowsParams &p, int tensors) {
  int64_t rows = 0;
  for (int kind = 0; kind < 3; ++kind) rows += p.src[kind] ? p.n_heads[kind] : 0;
  const int64_t bytes = rows * p.n_tokens * p.head_dim * (p.dtype == 0 ? 2 : 4) * tensors;
  return bytes > kCacheBytes * 3 / 4 ? 2 : bytes > kCacheBytes * 3 / 8 ? 1 : 0;
}
template <typename T, int D, int LAYOUT, bool kPaged>
hipError_t launch_rows(const HeadRowsParams &p, const RopeTable &rt, hipStream_t stream) {
  if (few_tokens(p)) {
    constexpr int TOK = RowGeo<T, D, kFewSlots>::TOK;
    head_rows_few_kernel<T, D, LAYOUT, kPaged><<<dim3((unsigned)(p.n_tokens + TOK - 1) / TOK, kPaged ? 3 : 2), kRotThreads, 0, stream>>>(p, rt);
  } else {
    constexpr int TOK = RowGeo<T, D, kManySlots>::TOK;
    static_assert(kRotThreads == kRowsThreads && TOK == head_rows_tokens(D, sizeof(T)), "what the size of a call is checked with");
    const unsigned wgs = (unsigned)((p.n_tokens + (int64_t)TOK - 1) / TOK);
    const int past = past_caches(p, 2);
    if (past == 2) head_rows_kernel<T, D, LAYOUT, kPaged, 2><<<wgs, kRotThreads, 0, stream>>>(p, rt);
    else if (past == 1) head_rows_kernel<T, D, LAYOUT, kPaged, 1><<<wgs, kRotThreads, 0, stream>>>(p, rt);
    else head_rows_kernel<T, D, LAYOUT, kPaged, 0><<<wgs, kRotThreads, 0, stream>>>(p, rt);
  }
  return hipGetLastError();
}
template <typename T, int D, bool kPaged>
hipError_t launch_rows_d(const HeadRowsParams &p, const RopeTable &rt, hipStream_t stream) {
  return p.layout == 0 ? launch_rows<T, D, 0, kPaged>(p, rt, stream) : launch_rows<T, D, 1, kPaged>(p, rt, stream);
}
template <typename T, int D, int LAYOUT>
void launch_back_rows(const NormBackwardParams &p, const RopeTable &rt, hipStream_t stream) {
  // us a call, every fourth head / every sixteenth: 32 over 8 heads of 128, bf16, one token 13.1 / 9.6, 256 14.5 / 11.1, 512 15.7 / 13.4, 1,024
  // 18.4 / 18.4, 2,048 21.1 / 24.5; 16 over 8, fp32, 256 10.8 / 9.8, 1,024 15.2 / 16.6; 8 over 2 of 64, fp32, 64 9.0 / 9.0, 512 11.0 / 11.6.
  const int heads = p.heads, past = past_caches(p.rows, 3);
  if (p.one_each ? heads > 2 * kManySlots : p.rows.n_tokens <= (heads > kManySlots * 4 ? 512 : 256))
    norm_backward_kernel<T, D, LAYOUT, kFewSlots, 0><<<p.n_wg, kRotThreads, 0, stream>>>(p, rt);
  else if (past == 2)
    norm_backward_kernel<T, D, LAYOUT, kManySlots, 2><<<p.n_wg, kRotThreads, 0, stream>>>(p, rt);
  else if (past == 1)
    norm_backward_kernel<T, D, LAYOUT, kManySlots, 1><<<p.n_wg, kRotThreads, 0, stream>>>(p, rt);
  else
    norm_backward_kernel<T, D, LAYOUT, kManySlots, 0><<<p.n_wg, kRotThreads, 0, stream>>>(p, rt);
}
template <typename T, int D>
hipError_t launch_back(const NormBackwardParams &p, const RopeTable &rt, hipStream_t stream) {
  if (p.n_wg > 0) {
    if (p.rows.layout == 0) launch_back_rows<T, D, 0>(p, rt, stream);
    else launch_back_rows<T, D, 1>(p, rt, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.one_each || (!p.weight_grad[0] && !p.weight_grad[1])) return hipSuccess;
  gain_sums_kernel<D><<<2 * D / kGainCols, kGainThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rotate(const HeadRowsParams &p, const RopeTable &rt, hipStream_t stream) {
  if (p.dtype == 0) return p.head_dim == 128 ? launch_rows_d<uint16_t, 128, false>(p, rt, stream) : launch_rows_d<uint16_t, 64, false>(p, rt, stream);
  return p.head_dim == 128 ? launch_rows_d<float, 128, false>(p, rt, stream) : launch_rows_d<float, 64, false>(p, rt, stream);
}
hipError_t launch_paged_append(const HeadRowsParams &p, const RopeTable &rt, hipStream_t stream) {
  return p.head_dim == 128 ? launch_rows_d<uint16_t, 128, true>(p, rt, stream) : launch_rows_d<uint16_t, 64, true>(p, rt, stream);
}
hipError_t launch_norm_rotate_backward(const NormBackwardParams &p, const RopeTable &rt, hipStream_t stream) {
  const HeadRowsParams &r = p.rows;
  if (r.dtype == 0) return r.head_dim == 128 ? launch_back<uint16_t, 128>(p, rt, stream) : launch_back<uint16_t, 64>(p, rt, stream);
  return r.head_dim == 128 ? launch_back<float, 128>(p, rt, stream) : launch_back<float, 64>(p, rt, stream);
}

}  // namespace ba
