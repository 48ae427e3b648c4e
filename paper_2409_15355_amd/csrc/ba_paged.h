// Internal interface between the C boundary (ba_api_paged.hip) and the kernels of head norms (head_norm.hip) and
// of the paged cache's attention (paged_attention.hip).
#pragma once

#include "ba_internal.h"

namespace ba {

// Workgroups of 256 that a launch may have: the runtime counts its threads in 32 bits.
constexpr int64_t kMaxWorkgroups = 0xffffffffll / 256;

// ---------------------------------------------------------------- head norms, appending ----------
enum { kRowsQ = 0, kRowsK = 1, kRowsV = 2 };

// Rows of up to three tensors [tokens][heads][D] on their way through one pass: queries and keys normed (eps >= 0) and
// rotated, values copied.  A null src leaves a tensor out.
struct HeadRowsParams {
  const void *src[3];
  void *dst[3];
  int64_t src_st[3], src_sh[3], dst_st[3], dst_sh[3];  // token / head strides, elements
  int32_t n_heads[3];
  const void *weight[2];  // gains of the query and key norm, null: ones
  int32_t weight_f32;
  float eps;              // negative: no norm
  int32_t n_tokens, head_dim, dtype, layout, rope;
  const int32_t *positions;  // device, null: a token's number
  // keys and values into pages (dst of kRowsK, kRowsV: page 0, row 0)
  const int32_t *page_table, *seq_of_token, *cache_pos;
  int64_t stride_table, dst_page[3];
  int32_t n_seqs, n_pages, max_rows;  // max_rows: rows that a sequence's part of the table spans
  int32_t page_rows;
  FastDiv page_div;
};
// Tokens of a workgroup in calls of many tokens (a lane for two 16-byte pieces, four heads at a time).
constexpr int kRowsThreads = 256, kManySlots = 4;
constexpr int head_rows_tokens(int head_dim, int elt_bytes) { return kRowsThreads / (head_dim * elt_bytes / 16 / 2 * kManySlots); }
hipError_t launch_norm_rotate(const HeadRowsParams &p, const RopeTable &rt, hipStream_t stream);
hipError_t launch_paged_append(const HeadRowsParams &p, const RopeTable &rt, hipStream_t stream);

// src, dst, weight and positions as above (queries and keys only); grad: the gradient of dst's forward counterpart
struct NormBackwardParams {
  HeadRowsParams rows;
  const void *grad[2];
  int64_t grad_st[2], grad_sh[2];
  float *weight_grad[2];  // device [D], nullable
  float *partial;         // [workgroups][D]
  int32_t wg_q, n_wg;     // workgroups for the queries, and all of them
  int32_t heads;          // the most of a tensor, also of one that is not there
  int32_t one_each;       // one for each tensor: its sums are the gradient
};
constexpr int kNormBwdMaxWg = 1024;
// Queries of this many bytes at most: a workgroup for each tensor, and no second launch for the gains' gradients.  us a call, one each / many: 32
// heads of 128, bf16, 1 token 5.9 / 10.8, 4 (32 KB) 7.4 / 10.0, 6 9.1 / 10.1, 8 10.8 / 10.0; fp32, 2 (32 KB) 6.2 / 9.6; 4 heads of 64, bf16, 64 tokens
// (32 KB) 8.6 / 10.2.
constexpr int64_t kNormBwdOneWgBytes = 32768;
hipError_t launch_norm_rotate_backward(const NormBackwardParams &p, const RopeTable &rt, hipStream_t stream);

// ---------------------------------------------------------------- attention over pages ----------
constexpr int kPagedTileRows = 128;    // rows of a work item
// ... up to this many in a problem: all of them, and the walk for few rows.  us, that walk and the one for many, 8 key heads of 128:
// 16 sequences of 2,000 keys, 20 rows 34 / 35, 32 rows 36 / 37, 48 rows 41 / 39; 1 of 4,000, 20 rows 17.1 / 15.6, 32 rows 17.9 / 18.0, 48
// rows 22 / 19; 64 of 4,000, 32 rows 201 / 204, 48 rows 218 / 217.
constexpr int kPagedStreamRows = 32;
BA_HD int paged_tile_rows(int n_rows) { return n_rows > kPagedStreamRows ? kPagedTileRows : kPagedStreamRows; }
constexpr int kPagedMaxChunk = 2048;  // keys of a work item at most: its part of the page table lies in LDS
constexpr int kPagedMergeRows = 16;   // rows that a workgroup of the merge takes, at one way a row

struct PagedAttnParams {
  const uint16_t *q;
  int64_t q_st, q_sh;
  uint16_t *o;
  int64_t o_st, o_sh;
  float *lse;  // [tokens][query heads], nullable
  const uint16_t *k, *v;
  int64_t k_sh, v_sh;          // head strides, elements
  uint32_t k_page_b16, v_page_b16;  // from page to page, in units of 16 bytes
  uint32_t k_rb, v_rb;         // bytes from row to row
  const int32_t *page_table;
  int64_t stride_table;
  int32_t n_pages, page_rows;
  FastDiv page_div, group_div, nq_div;
  const int32_t *seq_len;
  int32_t cap;  // no sequence is taken to be longer
  int32_t n_seqs, nq, group, n_kv_heads;
  float scale_log2e;
  int32_t chunk, own_chunk;  // keys of a work item of a prefix, of a sequence's own
  int32_t prefix_items;
  int32_t own_splits, own_row_tiles;
  uint16_t *part_o;         // [part][token][query head][D], fp16
  float *part_ml;           // [part][token][query head][4]: reference in log2 units, sum, what part_o is to be multiplied by
  int64_t part_rows;        // tokens * query heads
  int32_t max_parts;        // of a row
  int32_t past_caches;      // keys and values are read past the caches
  int32_t direct;           // one part for every row: the result itself
};
// Groups of sequences that share a prefix, in the order of their sequences.
template <int N>
struct PagedGroupsT {
  static constexpr int kGroups = N;
  int32_t n;
  int32_t seq0[N], members[N], prefix[N], splits[N], item0[N + 1];
};
using PagedGroups = PagedGroupsT<96>;
using PagedGroupsSmall = PagedGroupsT<8>;

// In place of the groups: the pages that every sequence and KV head reads.
struct PagedSelection {
  const int32_t *pages;  // [sequences][KV heads][n], numbers within the sequence
  int32_t n, max_pages;
  int32_t keys;          // of the listed pages at most: min(n * page_rows, cap)
};
// Keys of a work item at most: its part of the list lies in LDS as well.
constexpr int kSelectedMaxPages = 1154;
inline int32_t selected_max_chunk(int32_t page_rows) {
  const int64_t keys = (int64_t)(kSelectedMaxPages - 2) * page_rows / 64 * 64;
  return keys < 4096 ? (int32_t)keys : 4096;
}

template <typename Groups>
hipError_t launch_paged_attention(const PagedAttnParams &p, const Groups &g, int head_dim, hipStream_t stream);
template <typename Groups>
hipError_t launch_paged_merge(const PagedAttnParams &p, const Groups &g, int head_dim, hipStream_t stream);

}  // namespace ba
