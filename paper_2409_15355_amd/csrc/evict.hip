// Eviction from a paged cache by the weights of its keys (arXiv 2409.15355, Section 2.5: a cache that answers go on from): of every sequence
// and KV head the first, the last and the heaviest tokens stay, in order, and move to other pages.
//   pick: a workgroup a (sequence, KV head) finds the n_keep largest weights (ba_pick.h) and writes their places, their weights and the new length;
//   copy: rows of keys and values by those places, sixteen bytes a lane.
#include "ba_long.h"
#include "ba_pick.h"

namespace ba {
namespace {

__global__ __launch_bounds__(kPickThreads) void evict_pick_kernel(EvictParams p) {
  __shared__ PickLds lds;
  const int kvh = blockIdx.x % p.n_kv_heads, seq = blockIdx.x / p.n_kv_heads;
  const int len = max(0, min(p.seq_len[seq], p.cap));
  const int64_t list = (int64_t)seq * p.n_kv_heads + kvh;
  const float *w = p.weights + list * p.w_stride;
  int32_t *kept = p.kept + list * p.n_keep;
  float *w_out = p.w_out ? p.w_out + list * p.w_out_stride : nullptr;
  const int last0 = len - p.n_last;
  const int n = pick_largest(
      lds, len, p.n_keep, [&](int i) { return i < p.n_first || i >= last0 ? kPickAlways : pick_key(w[i]); },
      [&](int at, int i) {
        kept[at] = i;
        if (w_out) w_out[at] = w[i];
      });
  for (int j = n + threadIdx.x; j < p.n_keep; j += kPickThreads) kept[j] = -1;
  if (kvh == 0 && threadIdx.x == 0 && p.len_out) p.len_out[seq] = n;
}

constexpr int kCopyThreads = 256, kCopyRows = kEvictCopyRows;
__device__ __forceinline__ int page_of(const PagedTableParams &t, int seq, int at, int &row) {
  const int i = (int)fast_div((uint32_t)at, t.page_div);
  row = at - i * t.page_rows;
  const int page = i < t.max_pages ? t.table[seq * t.stride + i] : -1;
  return page >= 0 && page < t.n_pages ? page : -1;
}
__device__ __forceinline__ const char *row_at(const PagedRowsParams &r, int kvh, int page, int row) {
  return (const char *)(r.base + kvh * r.sh) + ((uint64_t)(uint32_t)page * r.page_b16 << 4) + (uint64_t)(uint32_t)row * r.rb;
}
template <int D>
__global__ __launch_bounds__(kCopyThreads) void evict_copy_kernel(EvictParams p, int chunks) {
  constexpr int CPR = D / 8, RPP = kCopyThreads / CPR, N = kCopyRows / RPP;
  const int kvh = blockIdx.x % p.n_kv_heads, rest = blockIdx.x / p.n_kv_heads, chunk = rest % chunks, seq = rest / chunks;
  const int32_t *kept = p.kept + ((int64_t)seq * p.n_kv_heads + kvh) * p.n_keep;
  const int c = threadIdx.x % CPR * 16;
  u32x4_t x[N][2];
  char *to[N][2];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int j = chunk * kCopyRows + u * RPP + threadIdx.x / CPR;
    const int of = j < p.n_keep ? kept[j] : -1;
    to[u][0] = to[u][1] = nullptr;
    if (of < 0) continue;
    int row, to_row;
    const int page = page_of(p.from, seq, of, row), to_page = page_of(p.to, seq, j, to_row);
    if (page < 0 || to_page < 0) continue;
    x[u][0] = *reinterpret_cast<const u32x4_t *>(row_at(p.k, kvh, page, row) + c);
    x[u][1] = *reinterpret_cast<const u32x4_t *>(row_at(p.v, kvh, page, row) + c);
    to[u][0] = (char *)row_at(p.to_k, kvh, to_page, to_row) + c;
    to[u][1] = (char *)row_at(p.to_v, kvh, to_page, to_row) + c;
  }
#pragma unroll
  for (int u = 0; u < N; ++u)
    if (to[u][0]) {
      *reinterpret_cast<u32x4_t *>(to[u][0]) = x[u][0];
      *reinterpret_cast<u32x4_t *>(to[u][1]) = x[u][1];
    }
}

}  // namespace

hipError_t launch_evict_pick(const EvictParams &p, hipStream_t stream) {
  const int64_t wgs = (int64_t)p.n_seqs * p.n_kv_heads;
  if (wgs < 1 || wgs > kMaxPickWorkgroups) return hipErrorInvalidValue;
  evict_pick_kernel<<<(unsigned)wgs, kPickThreads, 0, stream>>>(p);
  return hipGetLastError();
}
hipError_t launch_evict_copy(const EvictParams &p, hipStream_t stream) {
  const int64_t chunks = (p.n_keep + kCopyRows - 1) / kCopyRows, wgs = (int64_t)p.n_seqs * p.n_kv_heads * chunks;
  if (wgs < 1 || wgs > kMaxWorkgroups) return hipErrorInvalidValue;
  if (p.head_dim == 128) evict_copy_kernel<128><<<(unsigned)wgs, kCopyThreads, 0, stream>>>(p, (int)chunks);
  else evict_copy_kernel<64><<<(unsigned)wgs, kCopyThreads, 0, stream>>>(p, (int)chunks);
  return hipGetLastError();
}

}  // namespace ba
