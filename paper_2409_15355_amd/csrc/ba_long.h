// Internal interface between the C boundary (ba_api_long.hip) and the kernels that keep long caches affordable: weights of cached keys
// (key_weights.hip), eviction by them (evict.hip), bounds of pages and selection by them (page_select.hip).
#pragma once

#include "ba_internal.h"
#include "ba_paged.h"

namespace ba {

// Keys (or values) in pages, as a kernel sees them.
struct PagedRowsParams {
  const uint16_t *base;      // page 0, row 0, head 0
  int64_t sh;                // head stride, elements
  uint32_t page_b16;         // from page to page, in units of 16 bytes
  uint32_t rb;               // bytes from row to row
};
struct PagedTableParams {
  const int32_t *table;
  int64_t stride;
  int32_t n_pages, page_rows, max_pages;
  FastDiv page_div;
};

// ---------------------------------------------------------------- weights of cached keys ----------
struct KeyWeightsParams {
  const uint16_t *q;
  int64_t q_st, q_sh;
  const float *lse;        // [tokens][query heads]
  PagedRowsParams k;
  PagedTableParams pages;
  const int32_t *seq_len;
  int32_t cap;             // no sequence is taken to be longer
  int32_t n_seqs, nq, group, n_kv_heads;
  int32_t rows, padded;    // query rows of a sequence and KV head; padded to 4, or to a multiple of 8
  FastDiv group_div, padded_div;
  float scale_log2e, decay;
  const float *w_in;       // null: nothing was given before
  float *w_out;
  int64_t w_stride;
  int32_t prefix_items, own_chunks;
  int32_t own_go_on;       // a sequence may have more than own_chunks ranges of keys of its own: their workgroups go on
  int32_t item_members;    // sequences of a group that a work item takes
  // many rows without groups, in parts: tiles of 32 rows of a part (0: one part), its sums [part][sequence][KV head][cap]
  int32_t part_tiles, row_parts;
  float *part;
};
hipError_t launch_key_weights_merge(const KeyWeightsParams &p, hipStream_t stream);
constexpr int kWeightsFewKeys = 128, kWeightsManyKeys = 256;  // keys of a work item of the kernels for few and for many rows a sequence
template <typename Groups>
hipError_t launch_key_weights(const KeyWeightsParams &p, const Groups &g, int head_dim, bool many, hipStream_t stream);

// ---------------------------------------------------------------- eviction ----------
struct EvictParams {
  const float *weights;
  int64_t w_stride;
  const int32_t *seq_len;
  int32_t cap, n_seqs, n_kv_heads, head_dim;
  int32_t n_keep, n_first, n_last;
  int32_t *kept;           // [sequences][KV heads][n_keep]
  float *w_out;            // nullable
  int64_t w_out_stride;
  int32_t *len_out;        // nullable
  PagedRowsParams k, v, to_k, to_v;
  PagedTableParams from, to;
  FastDiv heads_div;       // by n_kv_heads
  int32_t past_caches;     // rows are copied past the caches
  // workgroups of a list (0: one, and the rows go in a launch of their own), rows that each of them writes and copies
  int32_t parts, part_rows;
};
constexpr int64_t kMaxPickWorkgroups = 0xffffffffll / 1024;
constexpr int kPickFourWaves = 1024;  // of lists up to here a choice takes four waves, of longer ones sixteen
constexpr int kEvictPartLeast = 32 * 128, kEvictPartMost = 256 * 128;  // elements of the rows that a list's workgroup copies
constexpr int kEvictCopyRows = 64;  // rows of heads that a workgroup copies
inline int64_t evict_copy_chunks(int64_t n_keep, int64_t cap, int64_t n_kv_heads) {
  return ((n_keep < cap ? n_keep : cap) * n_kv_heads + kEvictCopyRows - 1) / kEvictCopyRows;
}
hipError_t launch_evict_pick(const EvictParams &p, hipStream_t stream);
hipError_t launch_evict_copy(const EvictParams &p, hipStream_t stream);

// ---------------------------------------------------------------- bounds of pages, selection ----------
constexpr int kBoundMinExp = -60, kBoundMaxExp = 40;
struct PageBoundsParams {
  PagedRowsParams k;
  PagedTableParams pages;
  int8_t *codes, *exps;
  const int32_t *from, *seq_len;
  int32_t cap, n_seqs, n_kv_heads;
};
hipError_t launch_page_bounds(const PageBoundsParams &p, int head_dim, hipStream_t stream);

constexpr int kScorePages = 128;  // pages that a workgroup scores
struct PageSelectParams {
  const uint16_t *q;
  int64_t q_st, q_sh;
  PagedTableParams pages;
  const int8_t *codes, *exps;
  const int32_t *seq_len;
  int32_t cap, n_seqs, n_kv_heads, nq, group;
  FastDiv group_div;
  int32_t n_select, n_first, n_last;
  int32_t *selected;
  float *scores_out;       // nullable
  float *scores;           // [sequences][KV heads][score_stride]
  int64_t score_stride;
};
hipError_t launch_page_scores(const PageSelectParams &p, int head_dim, hipStream_t stream);
// Pages of a sequence up to which one launch does both.  us, eight lists, in one launch (4 waves / 16) and in two: 63 pages 5.7 / 6.7 and 8.3, 500 pages
// 10.0 / 9.4 and 9.5, 1,000 pages 15 / 13 and 9.8; 512 lists of up to 1,000 pages 24.7 / 26 and 21.7.
constexpr int kSelectOneLaunch = 256;
hipError_t launch_page_select(const PageSelectParams &p, int head_dim, hipStream_t stream);
hipError_t launch_page_pick(const PageSelectParams &p, hipStream_t stream);

}  // namespace ba
