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
#include <type_traits>

#include "ba_lds.h"
#include "ba_paged.h"
#include "ba_rotate.h"

namespace ba {
namespace {

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

// cos and sin of a lane's VEC pairs: in its two pieces one after the other (interleaved), or of its first with its second (half)
template <int VEC, int CH, int LAYOUT>
__device__ __forceinline__ void lane_turns(const RopeTable &rt, int c, int pos, float (&cs)[VEC], float (&sn)[VEC]) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int j = LAYOUT == 0 ? (e < VEC / 2 ? c * (VEC / 2) + e : (c + CH / 2) * (VEC / 2) + (e - VEC / 2)) : c * VEC + e;
    sincos_phase(rope_phase(pos, rt.turns[j]), cs[e], sn[e]);
  }
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
template <int VEC, int CH>
__device__ __forceinline__ void lane_gains(const void *w, bool f32, int c, float (&wx)[VEC], float (&wy)[VEC]) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int a = c * VEC + e, b = (c + CH / 2) * VEC + e;
    if (!w) {
      wx[e] = wy[e] = 1.f;
    } else if (f32) {
      wx[e] = ((const float *)w)[a];
      wy[e] = ((const float *)w)[b];
    } else {
      wx[e] = bf16_lo(((const uint16_t *)w)[a]);
      wy[e] = bf16_lo(((const uint16_t *)w)[b]);
    }
  }
}

// kPaged: keys and values go to their rows of a paged cache.  gridDim.y: one workgroup for all of a token's tensors, or one each.
template <typename T, int D, int LAYOUT, int kSlots, bool kPaged>
__global__ __launch_bounds__(kRotThreads) void head_rows_kernel(HeadRowsParams p, RopeTable rt) {
  using G = RowGeo<T, D, kSlots>;
  typedef Chunk<T, false, false> Ch;
  constexpr int VEC = G::VEC, CH = G::CH;
  constexpr int kBatch = 4;  // heads in flight per lane
  const int c = threadIdx.x % G::TPV, slot = threadIdx.x / G::TPV % kSlots;
  const int t = blockIdx.x * G::TOK + threadIdx.x / G::TPT;
  if (t >= p.n_tokens) return;

  float cs[VEC], sn[VEC];
  if (p.rope) lane_turns<VEC, CH, LAYOUT>(rt, c, p.positions ? p.positions[t] : t, cs, sn);
  // the token's row of the cache; none: nothing is kept of it
  bool kept = true;
  int64_t page = 0;
  int row = 0;
  if constexpr (kPaged) {
    const int seq = p.seq_of_token ? p.seq_of_token[t] : t, at = p.cache_pos[t];
    kept = seq >= 0 && seq < p.n_seqs && at >= 0 && at < p.max_rows;
    if (kept) {
      const uint32_t i = fast_div((uint32_t)at, p.page_div);
      row = at - (int)i * p.page_rows;
      page = p.page_table[seq * p.stride_table + i];
      kept = page >= 0 && page < p.n_pages;
    }
  }
  const int first = gridDim.y == 1 ? 0 : blockIdx.y, last = gridDim.y == 1 ? 2 : blockIdx.y;
#pragma unroll 1
  for (int kind = first; kind <= last; ++kind) {
    if (!p.src[kind] || (kPaged && kind != kRowsQ && !kept)) continue;
    const T *src = (const T *)p.src[kind] + t * p.src_st[kind] + c * VEC;
    T *dst = (T *)p.dst[kind] + c * VEC;
    dst += kPaged && kind != kRowsQ ? page * p.dst_page[kind] + row * p.dst_st[kind] : t * p.dst_st[kind];
    const int64_t src_sh = p.src_sh[kind], dst_sh = p.dst_sh[kind];
    const int n = p.n_heads[kind];
    const bool norm = kind != kRowsV && p.eps >= 0.f, turn = kind != kRowsV && p.rope;
    float wx[VEC], wy[VEC];
    if (norm) lane_gains<VEC, CH>(p.weight[kind], p.weight_f32, c, wx, wy);
#pragma unroll 1
    for (int h0 = slot; h0 < n; h0 += kSlots * kBatch) {
      Ch x[kBatch], y[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int h = min(h0 + u * kSlots, n - 1);
        x[u].load(src + h * src_sh);
        y[u].load(src + h * src_sh + (CH / 2) * VEC);
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int h = h0 + u * kSlots;
        if (h >= n) break;
        if (norm) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < VEC; ++e) ss += x[u].f[e] * x[u].f[e] + y[u].f[e] * y[u].f[e];
          const float r = rsqrtf(sum_over_lanes<G::TPV>(ss) * (1.0f / D) + p.eps);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            x[u].f[e] *= r * wx[e];
            y[u].f[e] *= r * wy[e];
          }
        }
        if (turn) turn_pieces<VEC, LAYOUT>(x[u].f, y[u].f, cs, sn);
        x[u].store(dst + h * dst_sh);
        y[u].store(dst + h * dst_sh + (CH / 2) * VEC);
      }
    }
  }
}

// A workgroup takes token chunks blockIdx.x, + gridDim.x, ... and leaves its sums of the gains' gradients.
template <typename T, int D, int LAYOUT, int kSlots>
__global__ __launch_bounds__(kRotThreads) void norm_backward_kernel(NormBackwardParams p, RopeTable rt) {
  using G = RowGeo<T, D, kSlots>;
  typedef Chunk<T, false, false> Ch;
  constexpr int VEC = G::VEC, CH = G::CH, kVecs = kRotThreads / G::TPV;
  __shared__ float red[kVecs][D];
  const HeadRowsParams &r = p.rows;
  const int c = threadIdx.x % G::TPV, slot = threadIdx.x / G::TPV % kSlots;
  float dw[2][2 * VEC];
#pragma unroll
  for (int e = 0; e < 2 * VEC; ++e) dw[0][e] = dw[1][e] = 0.f;
#pragma unroll 1
  for (int64_t t = (int64_t)blockIdx.x * G::TOK + threadIdx.x / G::TPT; t < r.n_tokens; t += (int64_t)gridDim.x * G::TOK) {
    float cs[VEC], sn[VEC];
    if (r.rope) {
      lane_turns<VEC, CH, LAYOUT>(rt, c, r.positions ? r.positions[t] : (int)t, cs, sn);
#pragma unroll
      for (int e = 0; e < VEC; ++e) sn[e] = -sn[e];  // the gradient turns back
    }
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      if (!r.src[kind]) continue;
      float wx[VEC], wy[VEC];
      lane_gains<VEC, CH>(r.weight[kind], r.weight_f32, c, wx, wy);
      const T *src = (const T *)r.src[kind] + t * r.src_st[kind] + c * VEC;
      const T *grad = (const T *)p.grad[kind] + t * p.grad_st[kind] + c * VEC;
      T *dst = (T *)r.dst[kind] + t * r.dst_st[kind] + c * VEC;
#pragma unroll 1
      for (int h = slot; h < r.n_heads[kind]; h += kSlots) {
        Ch x, y, gx, gy;
        x.load(src + h * r.src_sh[kind]);
        y.load(src + h * r.src_sh[kind] + (CH / 2) * VEC);
        gx.load(grad + h * p.grad_sh[kind]);
        gy.load(grad + h * p.grad_sh[kind] + (CH / 2) * VEC);
        if (r.rope) turn_pieces<VEC, LAYOUT>(gx.f, gy.f, cs, sn);
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          ss += x.f[e] * x.f[e] + y.f[e] * y.f[e];
          dot += x.f[e] * (gx.f[e] * wx[e]) + y.f[e] * (gy.f[e] * wy[e]);
        }
        const float rs = rsqrtf(sum_over_lanes<G::TPV>(ss) * (1.0f / D) + r.eps);
        const float m = sum_over_lanes<G::TPV>(dot) * (1.0f / D) * rs * rs;  // mean(b o x r) r
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          dw[kind][e] += gx.f[e] * (x.f[e] * rs);
          dw[kind][VEC + e] += gy.f[e] * (y.f[e] * rs);
          x.f[e] = rs * (gx.f[e] * wx[e] - x.f[e] * m);
          y.f[e] = rs * (gy.f[e] * wy[e] - y.f[e] * m);
        }
        x.store(dst + h * r.dst_sh[kind]);
        y.store(dst + h * r.dst_sh[kind] + (CH / 2) * VEC);
      }
    }
  }
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      red[threadIdx.x / G::TPV][c * VEC + e] = dw[kind][e];
      red[threadIdx.x / G::TPV][(c + CH / 2) * VEC + e] = dw[kind][VEC + e];
    }
    __syncthreads();
    if (threadIdx.x < D) {
      float sum = 0.f;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) sum += red[v][threadIdx.x];
      p.partial[((int64_t)blockIdx.x * 2 + kind) * D + threadIdx.x] = sum;
    }
  }
}

// partial [n_wg][2][D] -> the gradients of the gains, in the order of the workgroups (64-bit sums: they are few)
template <int D>
__global__ __launch_bounds__(kRotThreads) void gain_sums_kernel(NormBackwardParams p) {
  constexpr int kCols = 32, kWays = kRotThreads / kCols;
  __shared__ double red[kWays][kCols];
  const int kind = blockIdx.x / (D / kCols), col = blockIdx.x % (D / kCols) * kCols + threadIdx.x % kCols, way = threadIdx.x / kCols;
  if (!p.weight_grad[kind]) return;
  double sum = 0.0;
#pragma unroll 8
  for (int i = way; i < p.n_wg; i += kWays) sum += (double)p.partial[((int64_t)i * 2 + kind) * D + col];
  red[way][threadIdx.x % kCols] = sum;
  __syncthreads();
  if (way == 0) {
#pragma unroll
    for (int w = 1; w < kWays; ++w) sum += red[w][threadIdx.x];
    p.weight_grad[kind][col] = (float)sum;
  }
}

template <typename T, int D, int kSlots, bool kPaged>
hipError_t launch_rows(const HeadRowsParams &p, const RopeTable &rt, bool split, hipStream_t stream) {
  const dim3 grid((unsigned)((p.n_tokens + RowGeo<T, D, kSlots>::TOK - 1) / RowGeo<T, D, kSlots>::TOK), split ? (kPaged ? 3 : 2) : 1);
  if (p.layout == 0)
    head_rows_kernel<T, D, 0, kSlots, kPaged><<<grid, kRotThreads, 0, stream>>>(p, rt);
  else
    head_rows_kernel<T, D, 1, kSlots, kPaged><<<grid, kRotThreads, 0, stream>>>(p, rt);
  return hipGetLastError();
}
template <typename T, int D, bool kPaged>
hipError_t launch_rows_d(const HeadRowsParams &p, const RopeTable &rt, hipStream_t stream) {
  if (p.n_tokens <= 2048) return launch_rows<T, D, 16, kPaged>(p, rt, true, stream);
  return launch_rows<T, D, 4, kPaged>(p, rt, false, stream);
}
template <typename T, int D>
hipError_t launch_back(const NormBackwardParams &p, const RopeTable &rt, hipStream_t stream) {
  if (p.n_wg > 0) {
    if (p.rows.layout == 0)
      norm_backward_kernel<T, D, 0, 4><<<p.n_wg, kRotThreads, 0, stream>>>(p, rt);
    else
      norm_backward_kernel<T, D, 1, 4><<<p.n_wg, kRotThreads, 0, stream>>>(p, rt);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  gain_sums_kernel<D><<<2 * D / 32, kRotThreads, 0, stream>>>(p);
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
