// C boundary of what surrounds the paged cache of answers: head norms with rotation and their backward, appending to the pages, attention
// over them.  Page tables, lengths and positions are device memory here (they change from step to step, a captured step reads the new
// ones), so the kernels check every index that comes from them; the host arrays are the groups that share a prefix.
// Nothing in this file touches device memory itself or synchronises.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "../../include/ba.h"
#include "ba_api_common.h"
#include "ba_internal.h"
#include "ba_paged.h"
#include "ba_plan.h"

namespace ba {
namespace api {
namespace {

// ---- where a tensor lies: its rows [0, tokens) -------------------------------------------------------
struct Extent {
  int64_t lo, hi;           // bytes
  int64_t period, width;    // bytes from row to row, bytes of a row from its first head to its last
  int64_t step, head;       // bytes from head to head, bytes of a head
  int64_t rows;
  int32_t heads;
};
Extent extent(const ba_tensor *t, int64_t tokens, int n_heads, int D) {
  const int64_t es = (int64_t)elt_size(t->dtype);
  Extent x;
  x.period = t->stride_tok * es;
  x.step = t->stride_head * es;
  x.head = D * es;
  x.width = (n_heads - 1) * x.step + x.head;
  x.rows = tokens;
  x.heads = n_heads;
  x.lo = (int64_t)(uintptr_t)t->ptr;
  x.hi = x.lo + (tokens - 1) * x.period + x.width;
  return x;
}
// Whether no element is in both: apart altogether, or among each other in rows of one period (query and key heads of one projection, side by
// side or one after the other).  Rows of different periods that lie among each other are taken to meet.
bool apart(const Extent &a, const Extent &b) {
  if (a.hi <= b.lo || b.hi <= a.lo) return true;
  if (a.period != b.period || a.period == 0) return false;
  const int64_t d = ((b.lo - a.lo) % a.period + a.period) % a.period;
  if (d >= a.width && d + b.width <= a.period) return true;
  // a head of b that begins `by` bytes behind one of a in the same row meets it, or that of another row
  auto meet = [&](int64_t by) {
    int64_t m = -by / a.period;  // (rows between them, and the next: a period is a head at least)
    if (m * a.period > -by) --m;
    for (int i = 0; i < 2; ++i) {
      const int64_t at = by + std::min(b.rows - 1, std::max(1 - a.rows, m + i)) * a.period;
      if (at < a.head && at > -b.head) return true;
    }
    return false;
  };
  if (a.step == b.step) {  // (pairs of heads as far from each other are one case)
    for (int32_t j = 1 - a.heads; j < b.heads; ++j)
      if (meet(b.lo - a.lo + j * a.step)) return false;
    return true;
  }
  for (int32_t i = 0; i < a.heads; ++i)
    for (int32_t j = 0; j < b.heads; ++j)
      if (meet(b.lo - a.lo + j * b.step - i * a.step)) return false;
  return true;
}
bool same_place(const ba_tensor *a, const ba_tensor *b) {
  return a->ptr == b->ptr && a->stride_tok == b->stride_tok && a->stride_head == b->stride_head;
}

int32_t check_norm(const ba_head_norm *n) {
  if (n->dtype != BA_DTYPE_BF16 && n->dtype != BA_DTYPE_F32) return fail(BA_ERR_UNSUPPORTED, "norm: dtype %d of the gains not supported", n->dtype);
  if (!(n->eps > 0.f) || !std::isfinite(n->eps)) return fail(BA_ERR_INVALID_ARG, "norm: eps must be positive");
  if (((uintptr_t)n->q_weight | (uintptr_t)n->k_weight) & 15) return fail(BA_ERR_ALIGNMENT, "norm: gains must be 16-byte aligned");
  return BA_OK;
}
int32_t check_rope_mode(int32_t rope_mode) {
  return rope_mode == BA_ROPE_NONE || rope_mode == BA_ROPE_APPLY ? BA_OK : fail(BA_ERR_INVALID_ARG, "rope_mode %d unknown", rope_mode);
}
int32_t check_int_array(const void *p, const char *name) {
  return (uintptr_t)p & 3 ? fail(BA_ERR_ALIGNMENT, "%s: not aligned to its type", name) : BA_OK;
}

void set_source(HeadRowsParams *p, int kind, const ba_tensor *t, int n_heads) {
  p->src[kind] = t->ptr;
  p->src_st[kind] = t->stride_tok;
  p->src_sh[kind] = t->stride_head;
  p->n_heads[kind] = n_heads;
}
void set_target(HeadRowsParams *p, int kind, const ba_tensor *t) {
  p->dst[kind] = t->ptr;
  p->dst_st[kind] = t->stride_tok;
  p->dst_sh[kind] = t->stride_head;
}
void set_pass(HeadRowsParams *p, const ba_heads *h, const ba_head_norm *norm, int32_t n_tokens, int32_t dtype, const int32_t *positions,
              int32_t rope_mode) {
  p->eps = -1.f;
  if (norm) {
    p->weight[0] = norm->q_weight;
    p->weight[1] = norm->k_weight;
    p->weight_f32 = norm->dtype == BA_DTYPE_F32;
    p->eps = norm->eps;
  }
  p->n_tokens = n_tokens;
  p->head_dim = h->head_dim;
  p->dtype = dtype;
  p->layout = h->rope_layout;
  p->rope = rope_mode == BA_ROPE_APPLY;
  p->positions = positions;
}

// As many tokens as a launch of the forward passes takes.
int32_t check_tokens(int32_t n_tokens, const ba_heads *h, int32_t dtype) {
  const int64_t per_wg = head_rows_tokens(h->head_dim, (int)elt_size(dtype));
  return n_tokens <= kMaxWorkgroups * per_wg ? BA_OK : fail(BA_ERR_UNSUPPORTED, "more than %lld tokens in one call", (long long)(kMaxWorkgroups * per_wg));
}

// One tensor and its output of the norm passes: types, and exactly in place or apart.
int32_t check_pair(const ba_tensor *x, const char *name, const ba_tensor *y, const char *y_name, const ba_heads *h, int n_heads, int64_t tokens) {
  int32_t rc;
  if ((rc = check_tensor(x, name, true, h->head_dim, n_heads))) return rc;
  if ((rc = check_tensor(y, y_name, true, h->head_dim, n_heads))) return rc;
  if (x->dtype != y->dtype) return fail(BA_ERR_UNSUPPORTED, "%s and %s must share a dtype", name, y_name);
  if (!same_place(x, y) && !apart(extent(x, tokens, n_heads, h->head_dim), extent(y, tokens, n_heads, h->head_dim)))
    return fail(BA_ERR_INVALID_ARG, "%s overlaps %s without being exactly in place", y_name, name);
  return BA_OK;
}
int32_t check_apart(const ba_tensor *a, const char *a_name, int a_heads, const ba_tensor *b, const char *b_name, int b_heads, int64_t tokens, int D) {
  if (!a || !b || apart(extent(a, tokens, a_heads, D), extent(b, tokens, b_heads, D))) return BA_OK;
  return fail(BA_ERR_INVALID_ARG, "%s overlaps %s", a_name, b_name);
}

// Workgroups of the backward pass: as many as the chip holds at a time, shared out by heads (each tensor's share is the same without the
// other: so are the bits of its gain's gradient).
void backward_wgs(int64_t tokens, const ba_heads *h, bool q, bool k, NormBackwardParams *p) {
  const int64_t hq = h->n_q_heads, all = hq + h->n_kv_heads;
  p->heads = h->n_q_heads;
  p->one_each = tokens * hq * h->head_dim * (p->rows.dtype == 0 ? 2 : 4) <= kNormBwdOneWgBytes;
  if (p->one_each) {
    p->wg_q = q;
    p->n_wg = (int)q + k;
    return;
  }
  p->wg_q = q ? (int32_t)std::min<int64_t>(tokens, kNormBwdMaxWg * hq / all) : 0;
  p->n_wg = p->wg_q + (k ? (int32_t)std::min<int64_t>(tokens, std::max<int64_t>(1, kNormBwdMaxWg * (all - hq) / all)) : 0);
}

// ---- the paged cache -----------------------------------------------------------------------------------
int32_t check_cache(const ba_paged_cache *c, const ba_heads *h) {
  int32_t rc;
  if (!c) return fail(BA_ERR_INVALID_ARG, "cache: null");
  if ((rc = check_tensor(&c->k, "cache k", false, h->head_dim, h->n_kv_heads))) return rc;
  if ((rc = check_tensor(&c->v, "cache v", false, h->head_dim, h->n_kv_heads))) return rc;
  if (c->n_pages < 1 || c->page_rows < 1) return fail(BA_ERR_INVALID_ARG, "cache: at least one page of at least one row");
  if (c->n_seqs < 0 || c->max_pages < 0) return fail(BA_ERR_INVALID_ARG, "cache: negative sequence or page count");
  if (((c->k_stride_page | c->v_stride_page) * 2) & 15) return fail(BA_ERR_ALIGNMENT, "cache: page strides must be 16-byte aligned");
  if (c->k_stride_page < 0 || c->v_stride_page < 0) return fail(BA_ERR_INVALID_ARG, "cache: negative page stride");
  if (std::max(c->k_stride_page, c->v_stride_page) >= (int64_t)1 << 35)  // (counted in 32-bit units of 16 bytes)
    return fail(BA_ERR_UNSUPPORTED, "cache: pages of 64 GB and more");
  if (c->n_seqs > 0 && c->max_pages > 0) {
    if (!c->page_table) return fail(BA_ERR_INVALID_ARG, "page_table: null");
    if (c->stride_table < 0 || (c->n_seqs > 1 && c->stride_table < c->max_pages))
      return fail(BA_ERR_INVALID_ARG, "page_table: rows of the table overlap");
    if ((rc = check_int_array(c->page_table, "page_table"))) return rc;
  }
  if ((int64_t)c->max_pages * c->page_rows > 0x7fffffff - 1024)
    return fail(BA_ERR_UNSUPPORTED, "cache: sequences of 2^31 rows and more");
  return BA_OK;
}
Extent pool_extent(const ba_tensor *t, int64_t stride_page, const ba_paged_cache *c, const ba_heads *h) {
  Extent x = extent(t, c->page_rows, h->n_kv_heads, h->head_dim);
  x.hi += (int64_t)(c->n_pages - 1) * stride_page * 2;
  x.period = 0;  // (nothing lies side by side with its rows)
  return x;
}

// ---- plan of an attention call ---------------------------------------------------------------------------
// Sequences [seq0, seq0 + n_seqs) with at most kMost groups that share something.
struct PagedPlan {
  int32_t seq0, n_seqs, group_end;  // (group_end: the first group that is left for the next plan)
  int32_t chunk, own_chunk, own_splits, own_row_tiles, prefix_items;
  int32_t parts;
  int64_t items;  // of the launch, all of them
  int64_t keys;   // of all prefixes, and as many as the sequences may have of their own
  PagedGroups groups;
};

int32_t check_groups(int32_t n_seqs, int32_t max_len, int32_t n_groups, const int32_t *cu_group, const int32_t *prefix_len) {
  if (n_groups < 0) return fail(BA_ERR_INVALID_ARG, "negative group count");
  if (n_groups == 0) return BA_OK;
  if (!cu_group || !prefix_len) return fail(BA_ERR_INVALID_ARG, "cu_group / prefix_len: null");
  if (cu_group[0] != 0) return fail(BA_ERR_INVALID_ARG, "cu_group[0] must be 0");
  for (int g = 0; g < n_groups; ++g) {
    if (cu_group[g + 1] < cu_group[g]) return fail(BA_ERR_INVALID_ARG, "group %d: cu_group decreases", g);
    if (prefix_len[g] < 0 || prefix_len[g] > max_len) return fail(BA_ERR_INVALID_ARG, "group %d: prefix_len outside 0 .. max_len", g);
  }
  if (cu_group[n_groups] != n_seqs) return fail(BA_ERR_INVALID_ARG, "cu_group ends at %d, the call has %d sequences", cu_group[n_groups], n_seqs);
  return BA_OK;
}

// The plan of the sequences from those of group g0 on.  Without groups: of all of them.
void plan_paged(const ba_heads *h, int32_t n_seqs, int32_t nq, int32_t max_len, int32_t n_groups, const int32_t *cu_group,
                const int32_t *prefix_len, int g0, int cus, PagedPlan *pl) {
  memset(pl, 0, sizeof(*pl));
  const int64_t G = h->n_q_heads / h->n_kv_heads, hkv = h->n_kv_heads;
  auto row_tiles = [](int64_t rows) { return (rows + paged_tile_rows((int)rows) - 1) / paged_tile_rows((int)rows); };
  pl->own_row_tiles = (int32_t)row_tiles(nq * G);
  int64_t prefix_work = 0, own_work = 0;  // keys of all items together
  int32_t least_prefix = max_len;
  if (n_groups == 0) {
    pl->n_seqs = n_seqs;
    least_prefix = 0;
    own_work = (int64_t)n_seqs * max_len * pl->own_row_tiles * hkv;
    pl->keys = (int64_t)n_seqs * max_len;
  } else {
    pl->seq0 = cu_group[g0];
    int g = g0;
    for (; g < n_groups; ++g) {
      const int32_t members = cu_group[g + 1] - cu_group[g];
      const bool shares = members > 1 && prefix_len[g] > 0;
      if (shares && pl->groups.n == PagedGroups::kGroups) break;
      const int32_t prefix = shares ? prefix_len[g] : 0;
      if (shares) {
        const int i = pl->groups.n++;
        pl->groups.seq0[i] = cu_group[g] - pl->seq0;
        pl->groups.members[i] = members;
        pl->groups.prefix[i] = prefix;
        prefix_work += prefix * row_tiles(members * nq * G) * hkv;
        pl->keys += prefix;
      }
      if (members > 0) least_prefix = std::min(least_prefix, prefix);
      own_work += (int64_t)members * (max_len - prefix) * pl->own_row_tiles * hkv;
      pl->keys += (int64_t)members * (max_len - prefix);
    }
    pl->group_end = g;
    pl->n_seqs = cu_group[g] - pl->seq0;
  }
  const int64_t slots = 2 * cus;
  auto chunk_of = [&](int64_t keys, int64_t least, int64_t most) {
    return (int32_t)std::min(most, std::max(least, (keys + 63) / 64 * 64));
  };
  // One item a slot: each costs about as much as 100 keys of its own, so where the least chunks together are more than one
  // round of the slots, they are doubled.  With that and without (us; calls of 8 key heads and 4 query heads each, one token a
  // sequence): 16 sequences of 1,000 keys 16.9 and 23.8, 4 of 4,000 16.8 and 25.4, 1 of 16,000 13.9 and 16.2; 4 groups of 32
  // after 6,000 keys (2 key heads of 64) 17 and 22.  A round of small ones is faster: 1 sequence of 2,000 keys 10.7 in 264 items, 11.1 in 136; 1
  // of 4,000 with 8 tokens 17.6 in 504, 18.1 in 128.  The many-row walk reads a chunk in tiles of 32 keys behind barriers
  // and writes more rows: 64 tokens of 4,000 keys 22.5 with 256 keys a chunk, 26.2 with 128.
  // A call of one part needs no merge (3 us and more).  In one part and in several: 1 sequence of 250 keys 8.2 and 9.7, of 380
  // 9.4 and 9.6, of 500 10.5 and 10.1; 16 of 500 11.4 and 14.5, of 1,020 16.4 and 19.2; with 32 tokens each 1 of 400
  // keys 25.5 and 17.4, 16 of 380 23.8 and 26.2, of 1,000 41.3 and 37.5.
  const int64_t rows = (int64_t)nq * G, walks = pl->n_seqs * hkv * pl->own_row_tiles;
  const bool one_part = prefix_work == 0 && ((max_len <= 384 && rows <= 16) ||
                                             (max_len <= (rows <= kPagedStreamRows ? 1024 : 512) && walks >= cus / 2));
  const bool one_round = prefix_work / 128 + own_work / 64 <= slots;
  const int64_t least_own = one_part ? max_len / 64 * 64 + 64 : one_round ? 64 : rows <= kPagedStreamRows ? 128 : 256;
  // (the keys of the sequences' own are mostly fewer than max_len bounds them to: they weigh less where prefixes are cut)
  pl->chunk = chunk_of((prefix_work + own_work / 4) / slots, one_round ? 128 : 256, kPagedMaxChunk);
  // Cut at 1,024 keys so that ragged lengths even out (32 sequences of up to 8,000 keys, 4 tokens each 97 us, at 2,048 103, 8 tokens 106 and
  // 113), at 2,048 where that still makes more than two rounds, and rows enough that an item's start and end count (128 of 500 to 3,000
  // keys, 8 tokens 196 and 188, 48 of 500 to 6,000, 16 tokens 167 and 162; 256 of up to 2,000, one token 182 and 179; 128 of up to 8,000 328 and 330).
  const int64_t most_own = rows > 16 && own_work > 2048 * 2 * slots ? 2048 : 1024;
  pl->own_chunk = chunk_of((prefix_work + own_work) / slots, least_own, most_own);
  auto splits = [&](int64_t keys, int64_t chunk) { return (int32_t)((keys + chunk - 1) / chunk); };
  pl->own_splits = splits(max_len - least_prefix / 16 * 16, pl->own_chunk);
  pl->parts = least_prefix == 0 ? pl->own_splits : 0;
  int64_t items = 0;
  for (int i = 0; i < pl->groups.n; ++i) {
    pl->groups.splits[i] = splits(pl->groups.prefix[i], pl->chunk);
    pl->groups.item0[i] = (int32_t)std::min<int64_t>(items, INT32_MAX);
    items += (int64_t)(pl->groups.splits[i] * row_tiles(pl->groups.members[i] * nq * G) * hkv);
    pl->parts = std::max(pl->parts, pl->groups.splits[i] + splits(max_len - pl->groups.prefix[i] / 16 * 16, pl->own_chunk));
  }
  pl->groups.item0[pl->groups.n] = (int32_t)std::min<int64_t>(items, INT32_MAX);
  pl->prefix_items = (int32_t)std::min<int64_t>(items, INT32_MAX);
  // (somebody has to write the rows of sequences that see nothing)
  if (pl->parts <= 1 && items == 0) pl->own_splits = 1;
  pl->items = items + (int64_t)pl->n_seqs * hkv * pl->own_row_tiles * pl->own_splits;
}
size_t plan_bytes(const PagedPlan &pl, const ba_heads *h, int32_t nq) {
  if (pl.parts <= 1 && pl.groups.n == 0) return 0;
  const size_t rows = (size_t)pl.n_seqs * nq * h->n_q_heads;
  return align256(rows * pl.parts * h->head_dim * 2) + align256(rows * pl.parts * 16);
}

// All plans of a call: whether they can be launched, and the workspace of the largest.
int32_t check_plans(const ba_heads *h, int32_t n_seqs, int32_t nq, int32_t max_len, int32_t n_groups, const int32_t *cu_group,
                    const int32_t *prefix_len, size_t *bytes) {
  *bytes = 0;
  PagedPlan pl;
  int g = 0;
  do {
    plan_paged(h, n_seqs, nq, max_len, n_groups, cu_group, prefix_len, g, num_cus(), &pl);
    if (pl.n_seqs > 0 && pl.items > kMaxWorkgroups) return fail(BA_ERR_UNSUPPORTED, "2^24 work items and more in one launch");
    const size_t need = plan_bytes(pl, h, nq);
    if (need > 0 && ((int64_t)pl.n_seqs * nq * h->n_q_heads + kPagedMergeRows - 1) / kPagedMergeRows > kMaxWorkgroups)
      return fail(BA_ERR_UNSUPPORTED, "2^28 query rows and more in one launch");
    *bytes = std::max(*bytes, need);
    g = pl.group_end;
  } while (g < n_groups);
  return BA_OK;
}

int32_t check_paged_sizes(const ba_heads *h, int32_t n_seqs, int32_t nq, int32_t max_len) {
  int32_t rc;
  if ((rc = check_heads(h, true))) return rc;
  if (n_seqs < 0) return fail(BA_ERR_INVALID_ARG, "negative sequence count");
  if (nq < 1) return fail(BA_ERR_INVALID_ARG, "q_per_seq must be positive");
  if (max_len < 0) return fail(BA_ERR_INVALID_ARG, "negative max_len");
  // (row, key and item numbers are 32-bit)
  if (max_len > (1 << 30)) return fail(BA_ERR_UNSUPPORTED, "max_len beyond 2^30");
  if ((int64_t)n_seqs * nq > (1 << 28) || (int64_t)n_seqs * nq * h->n_q_heads > (1 << 28))
    return fail(BA_ERR_UNSUPPORTED, "more than 2^28 query rows in one call");
  return BA_OK;
}

}  // namespace
}  // namespace api
}  // namespace ba

using namespace ba;
using namespace ba::api;

extern "C" {

int32_t ba_norm_rotate(const ba_heads *heads, const ba_head_norm *norm, const ba_tensor *q, const ba_tensor *k, const ba_tensor *q_out,
                       const ba_tensor *k_out, int32_t n_tokens, const int32_t *positions, int32_t rope_mode, void *stream) {
  int32_t rc;
  if ((rc = check_heads(heads, true))) return rc;
  if (!norm) return fail(BA_ERR_INVALID_ARG, "norm: null");
  if ((rc = check_norm(norm)) || (rc = check_rope_mode(rope_mode)) || (rc = check_int_array(positions, "positions"))) return rc;
  if (n_tokens < 0) return fail(BA_ERR_INVALID_ARG, "negative token count");
  if (n_tokens == 0) return BA_OK;  // (tensors without rows need not lie anywhere)
  if (!q && !k) return fail(BA_ERR_INVALID_ARG, "q and k: both null");
  const int hq = heads->n_q_heads, hkv = heads->n_kv_heads, D = heads->head_dim;
  if (q && (rc = check_pair(q, "q", q_out, "q_out", heads, hq, n_tokens))) return rc;
  if (k && (rc = check_pair(k, "k", k_out, "k_out", heads, hkv, n_tokens))) return rc;
  if (q && k) {
    if (q->dtype != k->dtype) return fail(BA_ERR_UNSUPPORTED, "q and k must share a dtype");
    if ((rc = check_apart(q_out, "q_out", hq, k, "k", hkv, n_tokens, D)) || (rc = check_apart(k_out, "k_out", hkv, q, "q", hq, n_tokens, D)) ||
        (rc = check_apart(q_out, "q_out", hq, k_out, "k_out", hkv, n_tokens, D)))
      return rc;
  }
  if ((rc = check_tokens(n_tokens, heads, q ? q->dtype : k->dtype))) return rc;
  HeadRowsParams p;
  memset(&p, 0, sizeof(p));
  if (q) set_source(&p, kRowsQ, q, hq), set_target(&p, kRowsQ, q_out);
  if (k) set_source(&p, kRowsK, k, hkv), set_target(&p, kRowsK, k_out);
  set_pass(&p, heads, norm, n_tokens, q ? q->dtype : k->dtype, positions, rope_mode);
  RopeTable rt;
  build_rope_table(heads, &rt);
  ProfileScope ps(BA_PROFILE_REENCODE, (hipStream_t)stream);
  const hipError_t e = launch_norm_rotate(p, rt, (hipStream_t)stream);
  return e == hipSuccess ? BA_OK : device_fail(e, "head norm launch");
}

size_t ba_norm_rotate_backward_workspace_bytes(const ba_heads *heads, int32_t n_tokens) {
  if (check_heads(heads, true) != BA_OK || n_tokens <= 0) return 0;
  return align256((size_t)std::min<int64_t>(2 * (int64_t)n_tokens, kNormBwdMaxWg) * heads->head_dim * 4);
}

int32_t ba_norm_rotate_backward(const ba_heads *heads, const ba_head_norm *norm, const ba_tensor *q, const ba_tensor *k,
                                const ba_tensor *d_q_out, const ba_tensor *d_k_out, const ba_tensor *dq, const ba_tensor *dk,
                                float *dq_weight, float *dk_weight, int32_t n_tokens, const int32_t *positions, int32_t rope_mode, void *ws,
                                size_t ws_bytes, void *stream) {
  int32_t rc;
  if ((rc = check_heads(heads, true))) return rc;
  if (!norm) return fail(BA_ERR_INVALID_ARG, "norm: null");
  if ((rc = check_norm(norm)) || (rc = check_rope_mode(rope_mode)) || (rc = check_int_array(positions, "positions")) ||
      (rc = check_int_array(dq_weight, "dq_weight")) || (rc = check_int_array(dk_weight, "dk_weight")))
    return rc;
  if (n_tokens < 0) return fail(BA_ERR_INVALID_ARG, "negative token count");
  NormBackwardParams p;
  memset(&p, 0, sizeof(p));
  p.weight_grad[0] = dq_weight;
  p.weight_grad[1] = dk_weight;
  RopeTable rt;
  build_rope_table(heads, &rt);
  auto launch = [&]() {
    ProfileScope ps(BA_PROFILE_REENCODE, (hipStream_t)stream);
    const hipError_t e = launch_norm_rotate_backward(p, rt, (hipStream_t)stream);
    return e == hipSuccess ? BA_OK : device_fail(e, "head norm backward launch");
  };
  if (n_tokens == 0) {  // (tensors without rows need not lie anywhere)
    p.rows.head_dim = heads->head_dim;
    return dq_weight || dk_weight ? launch() : BA_OK;
  }
  if (!q && !k) return fail(BA_ERR_INVALID_ARG, "q and k: both null");
  if (!q && dq_weight) return fail(BA_ERR_INVALID_ARG, "dq_weight without q");
  if (!k && dk_weight) return fail(BA_ERR_INVALID_ARG, "dk_weight without k");
  const int hq = heads->n_q_heads, hkv = heads->n_kv_heads, D = heads->head_dim;
  if (q && ((rc = check_pair(d_q_out, "d_q_out", dq, "dq", heads, hq, n_tokens)) || (rc = check_pair(q, "q", dq, "dq", heads, hq, n_tokens)))) return rc;
  if (k && ((rc = check_pair(d_k_out, "d_k_out", dk, "dk", heads, hkv, n_tokens)) || (rc = check_pair(k, "k", dk, "dk", heads, hkv, n_tokens)))) return rc;
  if (q && k) {
    if (q->dtype != k->dtype) return fail(BA_ERR_UNSUPPORTED, "q and k must share a dtype");
    if ((rc = check_apart(dq, "dq", hq, k, "k", hkv, n_tokens, D)) || (rc = check_apart(dq, "dq", hq, d_k_out, "d_k_out", hkv, n_tokens, D)) ||
        (rc = check_apart(dk, "dk", hkv, q, "q", hq, n_tokens, D)) || (rc = check_apart(dk, "dk", hkv, d_q_out, "d_q_out", hq, n_tokens, D)) ||
        (rc = check_apart(dq, "dq", hq, dk, "dk", hkv, n_tokens, D)))
      return rc;
  }
  const size_t need = ba_norm_rotate_backward_workspace_bytes(heads, n_tokens);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(BA_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than %zu bytes", need);
  HeadRowsParams &r = p.rows;
  if (q) {
    set_source(&r, kRowsQ, q, hq), set_target(&r, kRowsQ, dq);
    p.grad[0] = d_q_out->ptr, p.grad_st[0] = d_q_out->stride_tok, p.grad_sh[0] = d_q_out->stride_head;
  }
  if (k) {
    set_source(&r, kRowsK, k, hkv), set_target(&r, kRowsK, dk);
    p.grad[1] = d_k_out->ptr, p.grad_st[1] = d_k_out->stride_tok, p.grad_sh[1] = d_k_out->stride_head;
  }
  set_pass(&r, heads, norm, n_tokens, q ? q->dtype : k->dtype, positions, rope_mode);
  p.partial = (float *)ws;
  backward_wgs(n_tokens, heads, q != nullptr, k != nullptr, &p);
  return launch();
}

int32_t ba_paged_append(const ba_heads *heads, const ba_head_norm *norm, const ba_paged_cache *cache, const ba_tensor *q, const ba_tensor *k,
                        const ba_tensor *v, const ba_tensor *q_out, int32_t n_tokens, const int32_t *cache_pos, const int32_t *seq_of_token,
                        const int32_t *rope_pos, int32_t rope_mode, void *stream) {
  int32_t rc;
  if ((rc = check_heads(heads, q != nullptr))) return rc;
  if ((rc = check_cache(cache, heads))) return rc;
  if ((norm && (rc = check_norm(norm))) || (rc = check_rope_mode(rope_mode))) return rc;
  if (n_tokens < 0) return fail(BA_ERR_INVALID_ARG, "negative token count");
  if (n_tokens == 0) return BA_OK;  // (tensors without rows need not lie anywhere)
  const int hq = heads->n_q_heads, hkv = heads->n_kv_heads, D = heads->head_dim;
  if ((rc = check_tensor(k, "k", false, D, hkv)) || (rc = check_tensor(v, "v", false, D, hkv))) return rc;
  if (q && q->dtype != BA_DTYPE_BF16) return fail(BA_ERR_UNSUPPORTED, "q: dtype %d not supported here", q->dtype);
  if (q && (rc = check_pair(q, "q", q_out, "q_out", heads, hq, n_tokens))) return rc;
  if (!cache_pos) return fail(BA_ERR_INVALID_ARG, "cache_pos: null");
  if ((rc = check_int_array(cache_pos, "cache_pos")) || (rc = check_int_array(seq_of_token, "seq_of_token")) ||
      (rc = check_int_array(rope_pos, "rope_pos")))
    return rc;
  if (!apart(extent(&cache->k, cache->page_rows, hkv, D), extent(&cache->v, cache->page_rows, hkv, D)))
    return fail(BA_ERR_INVALID_ARG, "cache: keys and values of a page overlap");
  const Extent pools[2] = {pool_extent(&cache->k, cache->k_stride_page, cache, heads), pool_extent(&cache->v, cache->v_stride_page, cache, heads)};
  for (const Extent &pool : pools)
    if (!apart(pool, extent(k, n_tokens, hkv, D)) || !apart(pool, extent(v, n_tokens, hkv, D)) ||
        (q && (!apart(pool, extent(q, n_tokens, hq, D)) || !apart(pool, extent(q_out, n_tokens, hq, D)))))
      return fail(BA_ERR_INVALID_ARG, "q, k, v or q_out overlap the cache");
  if (q && ((rc = check_apart(q_out, "q_out", hq, k, "k", hkv, n_tokens, D)) || (rc = check_apart(q_out, "q_out", hq, v, "v", hkv, n_tokens, D)))) return rc;
  if ((rc = check_tokens(n_tokens, heads, BA_DTYPE_BF16))) return rc;
  HeadRowsParams p;
  memset(&p, 0, sizeof(p));
  if (q) set_source(&p, kRowsQ, q, hq), set_target(&p, kRowsQ, q_out);
  set_source(&p, kRowsK, k, hkv), set_target(&p, kRowsK, &cache->k);
  set_source(&p, kRowsV, v, hkv), set_target(&p, kRowsV, &cache->v);
  p.dst_page[kRowsK] = cache->k_stride_page;
  p.dst_page[kRowsV] = cache->v_stride_page;
  set_pass(&p, heads, norm, n_tokens, BA_DTYPE_BF16, rope_pos ? rope_pos : cache_pos, rope_mode);
  p.page_table = cache->page_table;
  p.stride_table = cache->stride_table;
  p.seq_of_token = seq_of_token;
  p.cache_pos = cache_pos;
  p.n_seqs = cache->n_seqs;
  p.n_pages = cache->n_pages;
  p.max_rows = cache->max_pages * cache->page_rows;
  p.page_rows = cache->page_rows;
  p.page_div = make_fast_div((uint32_t)cache->page_rows);
  RopeTable rt;
  build_rope_table(heads, &rt);
  ProfileScope ps(BA_PROFILE_REENCODE, (hipStream_t)stream);
  const hipError_t e = launch_paged_append(p, rt, (hipStream_t)stream);
  return e == hipSuccess ? BA_OK : device_fail(e, "append launch");
}

size_t ba_paged_attention_workspace_bytes(const ba_heads *heads, int32_t n_seqs, int32_t q_per_seq, int32_t max_len,
                                          int32_t n_groups, const int32_t *cu_group, const int32_t *prefix_len) {
  if (check_paged_sizes(heads, n_seqs, q_per_seq, max_len) != BA_OK ||
      check_groups(n_seqs, max_len, n_groups, cu_group, prefix_len) != BA_OK)
    return 0;
  size_t bytes;
  return check_plans(heads, n_seqs, q_per_seq, max_len, n_groups, cu_group, prefix_len, &bytes) == BA_OK ? bytes : 0;
}

int32_t ba_paged_attention(const ba_heads *heads, const ba_paged_cache *cache, const ba_tensor *q, const ba_tensor *o_out, float *lse_out,
                           int32_t q_per_seq, const int32_t *seq_len, int32_t max_len, int32_t n_groups, const int32_t *cu_group,
                           const int32_t *prefix_len, void *ws, size_t ws_bytes, void *stream_) {
  hipStream_t stream = (hipStream_t)stream_;
  int32_t rc;
  if ((rc = check_heads(heads, true)) || (rc = check_cache(cache, heads))) return rc;
  const int32_t n_seqs = cache->n_seqs;
  if ((rc = check_paged_sizes(heads, n_seqs, q_per_seq, max_len))) return rc;
  if (n_seqs == 0) return check_groups(0, max_len, n_groups, cu_group, prefix_len);  // (tensors without rows need not lie anywhere)
  if ((rc = check_tensor(q, "q", false, heads->head_dim, heads->n_q_heads)) || (rc = check_tensor(o_out, "o_out", false, heads->head_dim, heads->n_q_heads)))
    return rc;
  if (max_len > (int64_t)cache->max_pages * cache->page_rows) return fail(BA_ERR_INVALID_ARG, "max_len reaches beyond the page table");
  // (a work item reads the query rows that it writes and no others, but the pages are everybody's)
  const Extent out = extent(o_out, (int64_t)n_seqs * q_per_seq, heads->n_q_heads, heads->head_dim);
  if (!same_place(q, o_out) && !apart(out, extent(q, (int64_t)n_seqs * q_per_seq, heads->n_q_heads, heads->head_dim)))
    return fail(BA_ERR_INVALID_ARG, "o_out overlaps q without being exactly in place");
  if (!apart(pool_extent(&cache->k, cache->k_stride_page, cache, heads), out) || !apart(pool_extent(&cache->v, cache->v_stride_page, cache, heads), out))
    return fail(BA_ERR_INVALID_ARG, "o_out overlaps the cache");
  if ((rc = check_groups(n_seqs, max_len, n_groups, cu_group, prefix_len))) return rc;
  if (!seq_len) return fail(BA_ERR_INVALID_ARG, "seq_len: null");
  if ((rc = check_int_array(seq_len, "seq_len")) || (rc = check_int_array(lse_out, "lse_out"))) return rc;
  size_t need;
  if ((rc = check_plans(heads, n_seqs, q_per_seq, max_len, n_groups, cu_group, prefix_len, &need))) return rc;
  if (need > 0 && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need))
    return fail(BA_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than %zu bytes", need);

  PagedPlan pl;
  int g = 0;
  do {  // (a launch's table of groups is full now and then)
    plan_paged(heads, n_seqs, q_per_seq, max_len, n_groups, cu_group, prefix_len, g, num_cus(), &pl);
    g = pl.group_end;
    if (pl.n_seqs == 0) continue;
    const int64_t tok0 = (int64_t)pl.seq0 * q_per_seq;
    PagedAttnParams p;
    memset(&p, 0, sizeof(p));
    p.q = (const uint16_t *)q->ptr + tok0 * q->stride_tok;
    p.q_st = q->stride_tok, p.q_sh = q->stride_head;
    p.o = (uint16_t *)o_out->ptr + tok0 * o_out->stride_tok;
    p.o_st = o_out->stride_tok, p.o_sh = o_out->stride_head;
    p.lse = lse_out ? lse_out + tok0 * heads->n_q_heads : nullptr;
    p.k = (const uint16_t *)cache->k.ptr, p.v = (const uint16_t *)cache->v.ptr;
    p.k_sh = cache->k.stride_head, p.v_sh = cache->v.stride_head;
    p.k_page_b16 = (uint32_t)(cache->k_stride_page / 8), p.v_page_b16 = (uint32_t)(cache->v_stride_page / 8);
    p.k_rb = (uint32_t)cache->k.stride_tok * 2, p.v_rb = (uint32_t)cache->v.stride_tok * 2;
    p.page_table = cache->page_table + (int64_t)pl.seq0 * cache->stride_table;
    p.stride_table = cache->stride_table;
    p.n_pages = cache->n_pages, p.page_rows = cache->page_rows;
    p.group = heads->n_q_heads / heads->n_kv_heads;
    p.page_div = make_fast_div((uint32_t)cache->page_rows);
    p.group_div = make_fast_div((uint32_t)p.group);
    p.nq_div = make_fast_div((uint32_t)q_per_seq);
    p.seq_len = seq_len + pl.seq0;
    p.cap = max_len;
    p.n_seqs = pl.n_seqs, p.nq = q_per_seq, p.n_kv_heads = heads->n_kv_heads;
    p.scale_log2e = scale_log2e(heads);
    p.chunk = pl.chunk, p.own_chunk = pl.own_chunk, p.prefix_items = pl.prefix_items;
    p.own_splits = pl.own_splits, p.own_row_tiles = pl.own_row_tiles;
    p.part_rows = (int64_t)pl.n_seqs * q_per_seq * heads->n_q_heads;
    p.max_parts = pl.parts;
    // Keys and values are read once a step (twice by two row tiles, at the same time), the next step's after all other layers'.  us with / without
    // the hint, 32 over 8 heads of 128, sequences of their own: 65 MB 27.5 / 25.7 (found again in the cache in front of HBM when the
    // calls of a program have no more than that), 262 MB 52.3 / 58.8, 1.05 GB 177 / 193, 1.98 GB 340 / 370; 48 drafts of 4 tokens, 175 MB 46.4 / 51.3.
    p.past_caches = pl.keys * heads->n_kv_heads * heads->head_dim * 4 > kCacheBytes * 3 / 8;
    p.direct = pl.parts <= 1 && pl.groups.n == 0;
    p.part_o = (uint16_t *)ws;
    p.part_ml = (float *)((char *)ws + align256((size_t)p.part_rows * pl.parts * heads->head_dim * 2));
    auto run = [&](const auto &groups) {
      hipError_t e;
      {
        ProfileScope ps(BA_PROFILE_ATTENTION, stream);
        e = launch_paged_attention(p, groups, heads->head_dim, stream);
      }
      if (e != hipSuccess || p.direct) return e;
      ProfileScope ps(BA_PROFILE_COMBINE, stream);
      return launch_paged_merge(p, groups, heads->head_dim, stream);
    };
    hipError_t e;
    if (pl.groups.n <= PagedGroupsSmall::kGroups) {  // (a small table: many large argument blocks in flight hold up the queue)
      PagedGroupsSmall few;
      memset(&few, 0, sizeof(few));
      few.n = pl.groups.n;
      for (int i = 0; i < few.n; ++i) {
        few.seq0[i] = pl.groups.seq0[i], few.members[i] = pl.groups.members[i], few.prefix[i] = pl.groups.prefix[i];
        few.splits[i] = pl.groups.splits[i], few.item0[i] = pl.groups.item0[i];
      }
      few.item0[few.n] = pl.groups.item0[few.n];
      e = run(few);
    } else {
      e = run(pl.groups);
    }
    if (e != hipSuccess) return device_fail(e, "paged attention launch");
  } while (g < n_groups);
  return BA_OK;
}

}  // extern "C"
