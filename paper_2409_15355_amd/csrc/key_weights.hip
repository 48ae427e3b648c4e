// Attention that cached keys have been given (arXiv 2409.15355, Section 2.5's final block, and the answer's tokens after it): for a
// sequence's query rows (token i, head h of the KV head) and its key t <= p(i)
//   w_t = decay w_t + sum_rows exp(scale <q_row, k_t> - lse_row).
//
// A work item is a range of keys of one KV head, of a group's prefix (for the rows of all its sequences, whose weights lie apart)
// or of what a sequence has behind it.  S = Q K^T by v_mfma_f32_32x32x16_bf16 with the keys as columns: a lane owns a key, its
// registers run over the rows, so the sum over rows is a lane's own and is stored as 128 consecutive bytes a half-wave.  A wave's
// keys come straight from the pages into its registers, once; the query rows go round through LDS in tiles of 32, for all waves.
// A sequence's rows begin at a multiple of 4 (of 8 if it has more than 4): a quad of accumulators is one sequence's.
#include "ba_device.h"
#include "ba_lds.h"
#include "ba_long.h"

namespace ba {
namespace {

constexpr int kWThreads = 256;
typedef __attribute__((address_space(3))) float lds_f;
typedef __attribute__((address_space(3))) int32_t lds_i;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4;
typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i32x4_t lds_i32x4;
typedef const __attribute__((address_space(3))) bf16x8_t lds_bf16x8;

__device__ __forceinline__ int clamped_length(const int32_t *seq_len, int cap, int seq) { return max(0, min(seq_len[seq], cap)); }

template <int D, int NT, typename Groups>
__global__ __launch_bounds__(kWThreads) void key_weights_kernel(KeyWeightsParams p, Groups groups) {
  constexpr int CPR = D / 8, KCH = D / 16, ROWB = D * 2, LPR = 256 / ROWB;
  constexpr uint32_t TB = 32 * ROWB;                       // a tile of query rows
  constexpr int RPP = kWThreads / CPR, PIECES = 32 / RPP;  // rows a pass of the threads stages, passes
  constexpr int kMeta = 3 * 32 * 4 + 16;
  __shared__ __attribute__((aligned(16))) char smem_generic[2 * (TB + kMeta)];
  lds_char *const smem = (lds_char *)smem_generic;

  int seq0, n_mem, kvh, key0, key_end;
  if ((int)blockIdx.x < p.prefix_items) {
    const int id = (int)blockIdx.x;
    int lo = 0, hi = groups.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (groups.item0[mid] <= id) lo = mid; else hi = mid;
    }
    const int rel = id - groups.item0[lo];
    seq0 = groups.seq0[lo];
    n_mem = groups.members[lo];
    kvh = rel % p.n_kv_heads;
    key0 = rel / p.n_kv_heads * key_weights_keys(NT);
    key_end = groups.prefix[lo];
  } else {
    int rel = (int)blockIdx.x - p.prefix_items;
    kvh = rel % p.n_kv_heads;
    rel /= p.n_kv_heads;
    const int chunk = rel % p.own_chunks;
    seq0 = rel / p.own_chunks;
    n_mem = 1;
    int lo = 0, hi = groups.n;  // its group
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (groups.seq0[mid] <= seq0) lo = mid; else hi = mid;
    }
    const bool in = groups.n > 0 && groups.seq0[lo] <= seq0 && seq0 < groups.seq0[lo] + groups.members[lo];
    key0 = (in ? groups.prefix[lo] : 0) + chunk * key_weights_keys(NT);
    key_end = clamped_length(p.seq_len, p.cap, seq0);
  }
  if (key0 >= key_end) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hf = lane >> 5;
  const int item_last = min(key_end, key0 + key_weights_keys(NT)) - 1;

  // ---- a wave's keys ------------------------------------------------------------------------------------------
  int key[NT];
  bool there[NT];
  bf16x8_t kf[NT][KCH];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    key[t] = key0 + (wave * NT + t) * 32 + col;
    const int k = min(key[t], key_end - 1), page_at = (int)fast_div((uint32_t)k, p.pages.page_div);
    int page = page_at < p.pages.max_pages ? p.pages.table[seq0 * p.pages.stride + page_at] : -1;
    there[t] = page >= 0 && page < p.pages.n_pages;
    page = there[t] ? page : 0;  // (some row that is there: its sums are dropped)
    const char *row = (const char *)(p.k.base + kvh * p.k.sh) + ((uint64_t)(uint32_t)page * p.k.page_b16 << 4) +
                      (uint64_t)(uint32_t)(k - page_at * p.pages.page_rows) * p.k.rb + hf * 16;
#pragma unroll
    for (int kk = 0; kk < KCH; ++kk) kf[t][kk] = *reinterpret_cast<const bf16x8_t *>(row + kk * 32);
  }

  // ---- query rows, a tile of 32 at a time ---------------------------------------------------------------------
  const int n_rows = n_mem * p.padded, n_tiles = (n_rows + 31) / 32;
  auto tok_of = [&](int r, int &head, int &i) __attribute__((always_inline)) {  // row -> its token, -1: padding
    const int j = (int)fast_div((uint32_t)r, p.padded_div), at = r - j * p.padded;
    i = (int)fast_div((uint32_t)at, p.group_div);
    head = kvh * p.group + at - i * p.group;
    return r < n_rows && at < p.rows ? (seq0 + j) * p.nq + i : -1;
  };
  u32x4_t piece[PIECES];
  float my_nl = 0.f;
  int my_limit = 0, my_len = 0;
  auto load_tile = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
      int head, i;
      const int tok = tok_of(tile * 32 + u * RPP + (int)threadIdx.x / CPR, head, i);
      piece[u] = u32x4_t{0, 0, 0, 0};
      if (tok >= 0) piece[u] = *reinterpret_cast<const u32x4_t *>(p.q + tok * p.q_st + head * p.q_sh + threadIdx.x % CPR * 8);
    }
    if (threadIdx.x < 32) {
      const int r = tile * 32 + (int)threadIdx.x;
      int head, i;
      const int tok = tok_of(r, head, i);
      my_len = clamped_length(p.seq_len, p.cap, min(seq0 + (int)fast_div((uint32_t)min(r, n_rows - 1), p.padded_div), p.n_seqs - 1));
      my_limit = 0;
      if (tok >= 0) {
        const float l = p.lse[(int64_t)tok * (p.n_kv_heads * p.group) + head];
        my_nl = -l * 1.4426950408889634f;
        my_limit = l == -INFINITY ? 0 : my_len - p.nq + i + 1;
      }
    }
  };
  auto store_tile = [&](int tile) __attribute__((always_inline)) {
    lds_char *const to = smem + (tile & 1) * (TB + kMeta);
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
      const int row = u * RPP + threadIdx.x / CPR, c = threadIdx.x % CPR;
      *(lds_u32x4 *)(to + row * ROWB + ((c ^ ((row / LPR) & (CPR - 1))) << 4)) = piece[u];
    }
    if (threadIdx.x < 32) {
      ((lds_f *)(to + TB))[threadIdx.x] = my_nl;
      ((lds_i *)(to + TB))[32 + threadIdx.x] = my_limit;
      ((lds_i *)(to + TB))[64 + threadIdx.x] = my_len;
      // whether every row of the tile sees all of the item's keys
      const bool all = (uint32_t)__builtin_amdgcn_ballot_w64(my_limit > item_last) == ~0u;
      if (threadIdx.x == 0) ((lds_i *)(to + TB))[96] = all;
    }
  };
  load_tile(0);
  store_tile(0);
  __syncthreads();

  float sum[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) sum[t] = 0.f;
  // the weights of sequence seq0 + j: what there was, and the new sum
  auto finish = [&](int t, int j, float total, int len) __attribute__((always_inline)) {
    if (key[t] > item_last || key[t] >= len) return;
    const int64_t at = ((int64_t)(seq0 + j) * p.n_kv_heads + kvh) * p.w_stride + key[t];
    float w = there[t] ? total : 0.f;
    if (p.w_in && key[t] < len - p.nq) w = __builtin_fmaf(p.decay, p.w_in[at], w);
    p.w_out[at] = w;
  };
#pragma unroll 1
  for (int tile = 0; tile < n_tiles; ++tile) {
    if (tile + 1 < n_tiles) load_tile(tile + 1);
    lds_char *const from = smem + (tile & 1) * (TB + kMeta);
    const bool all = ((lds_i *)(from + TB))[96] != 0;
    f32x16_t s[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[t][v] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KCH; ++kk) {
      const bf16x8_t qf = *(lds_bf16x8 *)(from + col * ROWB + (((2 * kk + hf) ^ ((col / LPR) & (CPR - 1))) << 4));
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[t][kk], s[t], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r0 = tile * 32 + i * 8;  // this lane's rows: r0 + hf * 4 + (0 .. 3)
      if (r0 >= n_rows) break;
      const f32x4_t nl = *(const lds_f32x4 *)(from + TB + (i * 8 + hf * 4) * 4);
      const i32x4_t limit = *(const lds_i32x4 *)(from + TB + (32 + i * 8 + hf * 4) * 4);
      const int len = ((const lds_i *)(from + TB))[64 + i * 8 + hf * 4];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float e[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          e[c] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i * 4 + c], p.scale_log2e, nl[c]));
          if (!all && key[t] >= limit[c]) e[c] = 0.f;
        }
        const float quad = (e[0] + e[1]) + (e[2] + e[3]);
        if (p.padded == 4) {
          if (r0 + hf * 4 < n_rows) finish(t, r0 / 4 + hf, quad, len);
        } else {
          sum[t] += quad;
        }
      }
      if (p.padded > 4) {
        const int j = (int)fast_div((uint32_t)r0, p.padded_div);
        if (r0 + 8 == (j + 1) * p.padded) {  // the sequence's last rows
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const float total = sum[t] + other_half(sum[t]);
            if (hf == 0) finish(t, j, total, len);
            sum[t] = 0.f;
          }
        }
      }
    }
    if (tile + 1 < n_tiles) store_tile(tile + 1);
    __syncthreads();
  }
}

template <int D, typename Groups>
hipError_t launch_d(const KeyWeightsParams &p, const Groups &g, int tiles, hipStream_t stream) {
  const int64_t items = p.prefix_items + (int64_t)p.n_seqs * p.n_kv_heads * p.own_chunks;
  if (items < 1 || items > kMaxWorkgroups) return hipErrorInvalidValue;
  if (tiles == 2) key_weights_kernel<D, 2, Groups><<<(unsigned)items, kWThreads, 0, stream>>>(p, g);
  else key_weights_kernel<D, 1, Groups><<<(unsigned)items, kWThreads, 0, stream>>>(p, g);
  return hipGetLastError();
}

}  // namespace

template <typename Groups>
hipError_t launch_key_weights(const KeyWeightsParams &p, const Groups &g, int head_dim, int tiles, hipStream_t stream) {
  return head_dim == 128 ? launch_d<128>(p, g, tiles, stream) : launch_d<64>(p, g, tiles, stream);
}
template hipError_t launch_key_weights(const KeyWeightsParams &, const PagedGroups &, int, int, hipStream_t);
template hipError_t launch_key_weights(const KeyWeightsParams &, const PagedGroupsSmall &, int, int, hipStream_t);

}  // namespace ba
