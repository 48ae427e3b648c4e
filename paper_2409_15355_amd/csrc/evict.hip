// Eviction from a paged cache by the weights of its keys (arXiv 2409.15355, Section 2.5: a cache that answers go on from): of every sequence
// and KV head the first, the last and the heaviest tokens stay, in order, and move to other pages.
//   pick: a workgroup a (sequence, KV head) finds the n_keep largest weights (ba_pick.h) and writes their places, their weights and the new
//     length; of few lists several workgroups each, which copy the rows as well;
//   copy: rows of keys and values by those places, sixteen bytes a lane.
#include <algorithm>

#include "ba_long.h"
#include "ba_pick.h"

namespace ba {
namespace {

__device__ __forceinline__ char *row_at(const PagedRowsParams &r, int kvh, int page, int row) {
  return (char *)(r.base + kvh * r.sh) + ((uint64_t)(uint32_t)page * r.page_b16 << 4) + (uint64_t)(uint32_t)row * r.rb;
}
// Rows of one sequence by what `which` says of the n-th: its head, its place among the kept ones, its token (-1: none).  A row's place comes out of three
// loads one behind the other; N rows' go together.
template <int D, int N, bool kPast, typename Which>
__device__ __forceinline__ void copy_rows(const EvictParams &p, int seq, int first, int apart, Which &&which) {
  const int c = threadIdx.x % (D / 8) * 16;
  int kvh[N], at[N], of[N], page[N], to_page[N];
#pragma unroll
  for (int u = 0; u < N; ++u) which(first + u * apart, kvh[u], at[u], of[u]);
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int i = (int)fast_div((uint32_t)max(of[u], 0), p.from.page_div), to_i = (int)fast_div((uint32_t)at[u], p.to.page_div);
    page[u] = p.from.table[seq * p.from.stride + min(i, p.from.max_pages - 1)];
    to_page[u] = p.to.table[seq * p.to.stride + min(to_i, p.to.max_pages - 1)];
    if (of[u] < 0 || i >= p.from.max_pages || to_i >= p.to.max_pages || page[u] < 0 || page[u] >= p.from.n_pages || to_page[u] < 0 || to_page[u] >= p.to.n_pages)
      page[u] = -1;  // (not copied)
    of[u] -= i * p.from.page_rows, at[u] -= to_i * p.to.page_rows;
  }
  u32x4_t x[N][2];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int row = page[u] < 0 ? 0 : of[u];
    x[u][0] = load_row_piece<kPast>(row_at(p.k, kvh[u], max(page[u], 0), row) + c);
    x[u][1] = load_row_piece<kPast>(row_at(p.v, kvh[u], max(page[u], 0), row) + c);
  }
#pragma unroll
  for (int u = 0; u < N; ++u)
    if (page[u] >= 0) {
      store_row_piece<kPast>(row_at(p.to_k, kvh[u], to_page[u], at[u]) + c, x[u][0]);
      store_row_piece<kPast>(row_at(p.to_v, kvh[u], to_page[u], at[u]) + c, x[u][1]);
    }
}

// Bound by latency for a few lists (eight of 2,064 tokens, 512 rows of 128 each copied: a call 7.4 us), by the instructions of sixteen waves a list
// for many (512 of up to 8,000 tokens 13.3 us: 49 % of the vector units' cycles; 9 MB).
// kRows: head_dim, and rows are copied, too.  Then a list may have several workgroups: each of them makes the same choice, and writes and copies its part
// of the rows, so nothing is handed on.  0: one workgroup a list, and no copies.
template <int W, int E, int kRows>
__global__ __launch_bounds__(W * 64) void evict_pick_kernel(EvictParams p) {
  __shared__ PickLds<W> lds;
  __shared__ int32_t place_of[kRows > 0 ? kEvictPartMost / kRows : 1];
  const int lists = p.n_seqs * p.n_kv_heads, part = kRows > 0 ? (int)blockIdx.x / lists : 0, of_list = kRows > 0 ? (int)blockIdx.x % lists : (int)blockIdx.x;
  const int kvh = of_list % p.n_kv_heads, seq = of_list / p.n_kv_heads;
  const int len = max(0, min(p.seq_len[seq], p.cap));
  const int64_t list = (int64_t)seq * p.n_kv_heads + kvh;
  const float *w = p.weights + list * p.w_stride;
  int32_t *kept = p.kept + list * p.n_keep;
  float *w_out = p.w_out ? p.w_out + list * p.w_out_stride : nullptr;
  const uint32_t between = (uint32_t)max(0, len - p.n_last - p.n_first);  // tokens that are neither of the first nor of the last
  const int lo = kRows > 0 ? part * p.part_rows : 0, hi = kRows > 0 && part + 1 < p.parts ? lo + p.part_rows : p.n_keep;
  const int n = pick_largest<W, E>(
      lds, len, p.n_keep, [&](int i) { return w[i]; }, [&](int i, float x) { return (uint32_t)(i - p.n_first) < between ? pick_key(x) : kPickAlways; },
      [&](int at, int i, float x) {
        if (kRows > 0 && (at < lo || at >= hi)) return;
        kept[at] = i;
        if (w_out) w_out[at] = x;
        if constexpr (kRows > 0) place_of[at - lo] = i;
      });
  for (int j = max(n, lo) + threadIdx.x; j < hi; j += W * 64) kept[j] = -1;
  if (kvh == 0 && part == 0 && threadIdx.x == 0 && p.len_out) p.len_out[seq] = n;
  if constexpr (kRows > 0) {
    constexpr int RPP = W * 64 / (kRows / 8);  // rows of a pass of the threads
    const int end = min(n, hi);
    auto which = [&](int j, int &head, int &at, int &of) __attribute__((always_inline)) {
      head = kvh, at = min(j, end - 1);
      of = j < end ? place_of[at - lo] : -1;
    };
    if (lo >= end) return;
    __syncthreads();
    const int first = lo + threadIdx.x / (kRows / 8);
    if (p.part_rows <= RPP) {
      copy_rows<kRows, 1, false>(p, seq, first, RPP, which);
    } else {
#pragma unroll 1
      for (int j0 = 0; lo + j0 < end; j0 += 4 * RPP) copy_rows<kRows, 4, false>(p, seq, first + j0, RPP, which);
    }
  }
}

// The copies apart from the lists: a workgroup takes kCopyRows new rows of heads, a token's heads one after the other, so what it writes lies together.
// Bound by HBM: 64 sequences, 1,024 rows of eight heads of 128, 271 MB in and 261 out, 104 us, 5.1 TB/s.
constexpr int kCopyThreads = 256, kCopyRows = kEvictCopyRows;
template <int D, bool kPast>
__global__ __launch_bounds__(kCopyThreads) void evict_copy_kernel(EvictParams p, int chunks) {
  constexpr int RPP = kCopyThreads / (D / 8);
  const int chunk = blockIdx.x % chunks, seq = blockIdx.x / chunks;
  copy_rows<D, kCopyRows / RPP, kPast>(p, seq, chunk * kCopyRows + threadIdx.x / (D / 8), RPP, [&](int r, int &head, int &at, int &of) {
    at = (int)fast_div((uint32_t)r, p.heads_div), head = r - at * p.n_kv_heads;
    of = p.kept[((int64_t)seq * p.n_kv_heads + head) * p.n_keep + min(at, p.n_keep - 1)];
    if (at >= p.n_keep) of = -1;
  });
}

}  // namespace

hipError_t launch_evict_pick(const EvictParams &p, hipStream_t stream) {
  const int64_t wgs = (int64_t)p.n_seqs * p.n_kv_heads * std::max(p.parts, 1);
  if (wgs < 1 || wgs > kMaxPickWorkgroups || (p.parts > 0 && (int64_t)p.part_rows * p.head_dim > kEvictPartMost)) return hipErrorInvalidValue;
  return with_pick_shape(p.cap, [&](auto w, auto e) {
    auto launch = [&](auto rows) {
      evict_pick_kernel<decltype(w)::value, decltype(e)::value, decltype(rows)::value><<<(unsigned)wgs, decltype(w)::value * 64, 0, stream>>>(p);
      return hipGetLastError();
    };
    using std::integral_constant;
    if (p.parts == 0) return launch(integral_constant<int, 0>{});
    return p.head_dim == 128 ? launch(integral_constant<int, 128>{}) : launch(integral_constant<int, 64>{});
  });
}
hipError_t launch_evict_copy(const EvictParams &p, hipStream_t stream) {
  const int64_t chunks = evict_copy_chunks(p.n_keep, p.cap, p.n_kv_heads), wgs = (int64_t)p.n_seqs * chunks;
  if (wgs > kMaxWorkgroups) return hipErrorInvalidValue;
  if (wgs == 0) return hipSuccess;
  auto launch = [&](auto d, auto past) {
    evict_copy_kernel<decltype(d)::value, decltype(past)::value><<<(unsigned)wgs, kCopyThreads, 0, stream>>>(p, (int)chunks);
    return hipGetLastError();
  };
  using D128 = std::integral_constant<int, 128>;
  using D64 = std::integral_constant<int, 64>;
  if (p.past_caches) return p.head_dim == 128 ? launch(D128{}, std::true_type{}) : launch(D64{}, std::true_type{});
  return p.head_dim == 128 ? launch(D128{}, std::false_type{}) : launch(D64{}, std::false_type{});
}

}  // namespace ba
