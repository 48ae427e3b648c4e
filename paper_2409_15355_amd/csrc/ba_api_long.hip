// C boundary of what keeps long paged caches affordable: weights of cached keys and eviction by them, bounds of pages and selection by
// them.  As around the rest of the paged cache, page tables, lengths and numbers of pages are device memory, and the kernels check them.
// Nothing in this file touches device memory itself or synchronises.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "ba_api_paged.h"
#include "ba_long.h"
#include "ba_plan.h"

namespace ba {
namespace api {
namespace {

Extent flat(const void *p, int64_t bytes) {
  Extent x;
  memset(&x, 0, sizeof(x));
  x.lo = (int64_t)(uintptr_t)p;
  x.hi = x.lo + std::max<int64_t>(bytes, 0);
  return x;
}
// [lists] of `n` elements of four bytes, `stride` apart
Extent lists_extent(const void *p, int64_t lists, int64_t stride, int64_t n) { return flat(p, n > 0 ? ((lists - 1) * stride + n) * 4 : 0); }
Extent k_pool(const ba_paged_cache *c, const ba_heads *h) { return pool_extent(&c->k, c->k_stride_page, c, h); }
Extent v_pool(const ba_paged_cache *c, const ba_heads *h) { return pool_extent(&c->v, c->v_stride_page, c, h); }

int32_t check_max_len(const ba_paged_cache *c, int32_t max_len) {
  if (max_len < 0) return fail(BA_ERR_INVALID_ARG, "negative max_len");
  if (max_len > (1 << 30)) return fail(BA_ERR_UNSUPPORTED, "max_len beyond 2^30");
  if (c && max_len > (int64_t)c->max_pages * c->page_rows) return fail(BA_ERR_INVALID_ARG, "max_len reaches beyond the page table");
  return BA_OK;
}
int32_t check_lists(int64_t n_seqs, const ba_heads *h) {
  return n_seqs * h->n_kv_heads <= kMaxPickWorkgroups ? BA_OK : fail(BA_ERR_UNSUPPORTED, "2^22 sequences and KV heads and more in one launch");
}
int32_t check_bounds(const ba_page_bound_table *b) {
  if (!b || !b->codes || !b->exponents) return fail(BA_ERR_INVALID_ARG, "bounds: null");
  return (uintptr_t)b->codes & 15 ? fail(BA_ERR_ALIGNMENT, "bounds: codes must be 16-byte aligned") : BA_OK;
}
void set_rows(PagedRowsParams *p, const ba_tensor *t, int64_t stride_page) {
  p->base = (const uint16_t *)t->ptr;
  p->sh = t->stride_head;
  p->page_b16 = (uint32_t)(stride_page / 8);
  p->rb = (uint32_t)t->stride_tok * 2;  // (check_tensor: below 2^25)
}
void set_table(PagedTableParams *p, const ba_paged_cache *c) {
  p->table = c->page_table;
  p->stride = c->stride_table;
  p->n_pages = c->n_pages, p->page_rows = c->page_rows, p->max_pages = c->max_pages;
  p->page_div = make_fast_div((uint32_t)c->page_rows);
}

constexpr int64_t kWeightsSlots = 4, kWeightsOwn = 8;  // workgroups to a compute unit

// ---- weights of cached keys --------------------------------------------------------------------------------
struct WeightsPlan {
  int32_t seq0, n_seqs, group_end;
  int32_t prefix_items, own_chunks, item_members;
  int32_t part_tiles, row_parts;  // (see KeyWeightsParams)
  bool many, own_go_on;
  int64_t items;
  PagedGroups groups;
};
int32_t padded_rows(const ba_heads *h, int32_t nq) {
  const int32_t rows = nq * (h->n_q_heads / h->n_kv_heads);
  return rows <= 4 ? 4 : (rows + 7) & ~7;
}
// The sequences from those of group g0 on, with at most kGroups groups that share something.
void plan_weights(const ba_heads *h, int32_t n_seqs, int32_t nq, int32_t max_len, int32_t n_groups, const int32_t *cu_group, const int32_t *prefix_len,
                  int g0, WeightsPlan *pl) {
  memset(pl, 0, sizeof(*pl));
  int32_t least_prefix = 0, most_prefix = 0;
  if (n_groups == 0) {
    pl->n_seqs = n_seqs;
  } else {
    pl->seq0 = cu_group[g0];
    least_prefix = max_len;
    int g = g0;
    for (; g < n_groups; ++g) {
      const int32_t members = cu_group[g + 1] - cu_group[g];
      const bool shares = members > 1 && prefix_len[g] > 0;
      if (shares && pl->groups.n == PagedGroups::kGroups) break;
      if (shares) {
        const int i = pl->groups.n++;
        pl->groups.seq0[i] = cu_group[g] - pl->seq0;
        pl->groups.members[i] = members;
        pl->groups.prefix[i] = prefix_len[g];
      }
      if (members > 0) least_prefix = std::min(least_prefix, shares ? prefix_len[g] : 0);
      if (shares) most_prefix = std::max(most_prefix, prefix_len[g]);
    }
    pl->group_end = g;
    pl->n_seqs = cu_group[g] - pl->seq0;
  }
  // By rows alone.  us, the kernel for few rows and the one for many, 8 KV heads of 128: 1 sequence of 32,000 keys, 16 rows 14.6 / 16.9, 24 14.9 / 17.0,
  // 32 14.8 / 14.2, 48 16.9 / 19.3, 64 16.8 / 15.3, 128 22.9 / 18.7, 1,024 99 / 79; of 2,000, 16 rows 4.6 / 5.9, 32 5.1 / 6.0, 64 5.8 / 6.9, 128 7.7 / 8.5,
  // 256 12.2 / 10.7, 1,024 40 / 14; 16 sequences on a shared prefix of 2,000, 16 rows 7.1 / 10.3, 32 9.2 / 9.9, 64 12.3 / 15.2, 128 18.3 / 20.0, of 8,000 13.6 / 23.5,
  // 19.4 / 18.7, 30.6 / 25.4, 52 / 42; 64 on 30,000 111 / 216, 192 / 154, 356 / 274, 684 / 515.  So between 32 and 128 rows few keys cost 1 to 3 us more than
  // they would have to, and 48 rows, whose second tile is half empty, up to 2.4.
  pl->many = nq * (h->n_q_heads / h->n_kv_heads) >= 32;
  const int32_t keys = pl->many ? kWeightsManyKeys : kWeightsFewKeys;
  int64_t items = 0, most_members = 1;
  for (int i = 0; i < pl->groups.n; ++i) {
    items += ((int64_t)pl->groups.prefix[i] + keys - 1) / keys * h->n_kv_heads;
    most_members = std::max<int64_t>(most_members, pl->groups.members[i]);
  }
  // A group's sequences in parts (nothing has to be added up: their weights are their own) where its keys do not fill the chip, of 64 rows at least.
  // us, in one part and in several (of 32 / 64 / 128 rows at least): 46 answers of 4 rows on 1,141 keys 11.2 and 7.0 / 7.3 / 9.3; two groups of 28 of
  // 16 rows on 1,096 keys 19.5 and 13.1 / 13.1 / 11.5; 16 of 32 rows on 2,000 keys 24.4 and 14.4 / 11.1 / 11.2.
  constexpr int64_t kRowsLeast = 64;
  const int64_t parts = items > 0 ? std::max<int64_t>(1, kWeightsSlots * num_cus() / items) : 1, padded = padded_rows(h, nq);
  pl->item_members = (int32_t)std::min(most_members, std::max((kRowsLeast + padded - 1) / padded, (most_members + parts - 1) / parts));
  items = 0;
  for (int i = 0; i < pl->groups.n; ++i) {
    pl->groups.item0[i] = (int32_t)std::min<int64_t>(items, INT32_MAX);
    items += ((int64_t)pl->groups.prefix[i] + keys - 1) / keys * h->n_kv_heads * ((pl->groups.members[i] + pl->item_members - 1) / pl->item_members);
  }
  pl->groups.item0[pl->groups.n] = pl->prefix_items = (int32_t)std::min<int64_t>(items, INT32_MAX);
  pl->own_chunks = (int32_t)(((int64_t)max_len - least_prefix + keys - 1) / keys);
  const int64_t lists = (int64_t)pl->n_seqs * h->n_kv_heads;
  // What a sequence has of its own is max_len less the shortest prefix at most, and mostly no more than max_len less the longest: with few rows there
  // are workgroups for that, and they go on where there is more; a workgroup without keys costs its way to seq_len.  us, with workgroups for all and
  // so: eight groups of 25 on 1,796 to 3,590 keys, up to 12 of their own 41.9 / 25.2; five of 40, 16 rows, on 481 to 963, up to 124 37.2 / 21.7.
  // (Two workgroups a sequence where 39 are needed: 130 / 165.)
  if (!pl->many && pl->groups.n > 0 && lists > 0) {
    const int64_t mostly = std::max<int64_t>({((int64_t)max_len - most_prefix + keys - 1) / keys, 1, kWeightsOwn * num_cus() / lists});
    if (mostly < pl->own_chunks) pl->own_chunks = (int32_t)mostly, pl->own_go_on = true;
  }
  const int64_t own_items = lists * pl->own_chunks;
  // Many rows in up to eight parts: what costs least, in tenths of the time that a tile takes a compute unit's workgroups together: 12 for one of them, 20
  // for two, 10 each for more; the merge (a launch) 50 and its bytes.  us, in 1 / 2 / 4 / 8 parts, 8 heads of 128: 1 sequence, 1,024 rows over 500 keys
  // 36 / 23 / 16 / 13, over 8,000 38 / 31 / 31 / 35, over 20,000 63 / 58 / 58 / 72, 256 rows over 2,000 12.5 / 12.5 / 11.0 / 11.1, over 8,000
  // 14.8 / 15.6 / 18.1 / 24.5; 8 of 3,000 keys, 1,024 rows 66 / 73 / 71 / 83, 400 rows 36 / 39 / 49 / 54; 23 of 698, 920 rows 63 / 58 / 56 / 66.
  pl->row_parts = 1;
  if (pl->many && pl->groups.n == 0 && own_items > 0) {
    const int64_t tiles = ((int64_t)nq * (h->n_q_heads / h->n_kv_heads) + 31) / 32, cus = num_cus();
    int64_t least_cost = INT64_MAX;
    for (int64_t p = 1; p <= std::min<int64_t>(tiles, 8); ++p) {
      const int64_t taken = (tiles + p - 1) / p, parts = (tiles + taken - 1) / taken, together = (own_items * parts + cus - 1) / cus;
      const int64_t cost = taken * (together == 1 ? 12 : 10 * together) + (parts > 1 ? 50 + lists * max_len * parts / 10000 : 0);
      if (cost < least_cost) least_cost = cost, pl->part_tiles = parts > 1 ? (int32_t)taken : 0, pl->row_parts = (int32_t)parts;
    }
  }
  pl->items = items + own_items * pl->row_parts;
}
size_t weights_bytes(const WeightsPlan &pl, const ba_heads *h, int32_t max_len) {
  return pl.part_tiles ? align256((size_t)pl.row_parts * pl.n_seqs * h->n_kv_heads * max_len * 4) : 0;
}

}  // namespace
}  // namespace api
}  // namespace ba

using namespace ba;
using namespace ba::api;

extern "C" {

size_t ba_paged_key_weights_workspace_bytes(const ba_heads *heads, int32_t n_seqs, int32_t q_per_seq, int32_t max_len, int32_t n_groups,
                                            const int32_t *cu_group, const int32_t *prefix_len) {
  if (check_paged_sizes(heads, n_seqs, q_per_seq, max_len) != BA_OK || check_groups(n_seqs, max_len, n_groups, cu_group, prefix_len) != BA_OK) return 0;
  size_t bytes = 0;
  WeightsPlan pl;
  int g = 0;
  do {
    plan_weights(heads, n_seqs, q_per_seq, max_len, n_groups, cu_group, prefix_len, g, &pl);
    bytes = std::max(bytes, weights_bytes(pl, heads, max_len));
    g = pl.group_end;
  } while (g < n_groups);
  return bytes;
}

int32_t ba_paged_key_weights(const ba_heads *heads, const ba_paged_cache *cache, const ba_tensor *q, const float *lse, const float *weights_in,
                             float *weights_out, int64_t stride_weights, float decay, int32_t q_per_seq, const int32_t *seq_len, int32_t max_len,
                             int32_t n_groups, const int32_t *cu_group, const int32_t *prefix_len, void *ws, size_t ws_bytes, void *stream) {
  int32_t rc;
  if ((rc = check_heads(heads, true)) || (rc = check_cache(cache, heads))) return rc;
  const int32_t n_seqs = cache->n_seqs, hq = heads->n_q_heads, D = heads->head_dim;
  if ((rc = check_paged_sizes(heads, n_seqs, q_per_seq, max_len)) || (rc = check_groups(n_seqs, max_len, n_groups, cu_group, prefix_len))) return rc;
  if (!std::isfinite(decay)) return fail(BA_ERR_INVALID_ARG, "decay must be finite");
  if (n_seqs == 0 || max_len == 0) return BA_OK;  // (tensors without rows need not lie anywhere)
  if ((rc = check_tensor(q, "q", false, D, hq)) || (rc = check_max_len(cache, max_len))) return rc;
  if (!lse || !weights_out || !seq_len) return fail(BA_ERR_INVALID_ARG, "lse / weights_out / seq_len: null");
  if ((rc = check_int_array(lse, "lse")) || (rc = check_int_array(weights_in, "weights_in")) || (rc = check_int_array(weights_out, "weights_out")) ||
      (rc = check_int_array(seq_len, "seq_len")))
    return rc;
  if (stride_weights < max_len) return fail(BA_ERR_INVALID_ARG, "stride_weights smaller than max_len");
  const int64_t lists = (int64_t)n_seqs * heads->n_kv_heads, tokens = (int64_t)n_seqs * q_per_seq;
  const Extent out = lists_extent(weights_out, lists, stride_weights, max_len);
  if (weights_in && weights_in != weights_out && !apart(out, lists_extent(weights_in, lists, stride_weights, max_len)))
    return fail(BA_ERR_INVALID_ARG, "weights_out overlaps weights_in without being exactly in place");
  if (!apart(out, k_pool(cache, heads)) || !apart(out, v_pool(cache, heads)) || !apart(out, extent(q, tokens, hq, D)) || !apart(out, flat(lse, tokens * hq * 4)) ||
      !apart(out, flat(seq_len, (int64_t)n_seqs * 4)))
    return fail(BA_ERR_INVALID_ARG, "weights_out overlaps q, lse, seq_len or the cache");
  WeightsPlan pl;
  int g = 0;
  do {  // (whether every launch can be made, ahead of the first)
    plan_weights(heads, n_seqs, q_per_seq, max_len, n_groups, cu_group, prefix_len, g, &pl);
    if (pl.items > kMaxWorkgroups) return fail(BA_ERR_UNSUPPORTED, "2^24 work items and more in one launch");
    const size_t need = weights_bytes(pl, heads, max_len);
    if (need > 0 && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need))
      return fail(BA_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than %zu bytes", need);
    if (pl.groups.n > 0 && (int64_t)padded_rows(heads, q_per_seq) * pl.n_seqs > (1 << 30)) return fail(BA_ERR_UNSUPPORTED, "2^30 query rows and more");
    g = pl.group_end;
  } while (g < n_groups);
  g = 0;
  do {
    plan_weights(heads, n_seqs, q_per_seq, max_len, n_groups, cu_group, prefix_len, g, &pl);
    g = pl.group_end;
    if (pl.n_seqs == 0 || pl.items == 0) continue;
    KeyWeightsParams p;
    memset(&p, 0, sizeof(p));
    const int64_t tok0 = (int64_t)pl.seq0 * q_per_seq, at = (int64_t)pl.seq0 * heads->n_kv_heads * stride_weights;
    p.q = (const uint16_t *)q->ptr + tok0 * q->stride_tok;
    p.q_st = q->stride_tok, p.q_sh = q->stride_head;
    p.lse = lse + tok0 * hq;
    set_rows(&p.k, &cache->k, cache->k_stride_page);
    set_table(&p.pages, cache);
    p.pages.table += (int64_t)pl.seq0 * cache->stride_table;
    p.seq_len = seq_len + pl.seq0;
    p.cap = max_len;
    p.n_seqs = pl.n_seqs, p.nq = q_per_seq, p.n_kv_heads = heads->n_kv_heads;
    p.group = hq / heads->n_kv_heads;
    p.rows = q_per_seq * p.group, p.padded = padded_rows(heads, q_per_seq);
    p.group_div = make_fast_div((uint32_t)p.group);
    p.padded_div = make_fast_div((uint32_t)p.padded);
    p.scale_log2e = scale_log2e(heads);
    p.decay = decay;
    p.w_in = weights_in && decay != 0.f ? weights_in + at : nullptr;
    p.w_out = weights_out + at;
    p.w_stride = stride_weights;
    p.prefix_items = pl.prefix_items, p.own_chunks = pl.own_chunks, p.item_members = pl.item_members;
    p.own_go_on = pl.own_go_on;
    p.part_tiles = pl.part_tiles, p.row_parts = pl.row_parts;
    p.part = (float *)ws;
    ProfileScope ps(BA_PROFILE_ATTENTION, (hipStream_t)stream);
    hipError_t e;
    if (pl.groups.n <= PagedGroupsSmall::kGroups) {  // (a small table: many large argument blocks in flight hold up the queue)
      PagedGroupsSmall few;
      memset(&few, 0, sizeof(few));
      few.n = pl.groups.n;
      for (int i = 0; i < few.n; ++i)
        few.seq0[i] = pl.groups.seq0[i], few.members[i] = pl.groups.members[i], few.prefix[i] = pl.groups.prefix[i], few.item0[i] = pl.groups.item0[i];
      few.item0[few.n] = pl.groups.item0[few.n];
      e = launch_key_weights(p, few, D, pl.many, (hipStream_t)stream);
    } else {
      e = launch_key_weights(p, pl.groups, D, pl.many, (hipStream_t)stream);
    }
    if (e == hipSuccess && pl.part_tiles) e = launch_key_weights_merge(p, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "key weights launch");
  } while (g < n_groups);
  return BA_OK;
}

size_t ba_paged_evict_workspace_bytes(const ba_heads *heads, int32_t n_seqs, int32_t max_len, int32_t n_keep) { return 0; }

int32_t ba_paged_evict(const ba_heads *heads, const ba_paged_cache *cache, const ba_paged_cache *to, const float *weights, int64_t stride_weights,
                       const int32_t *seq_len, int32_t max_len, int32_t n_keep, int32_t n_first, int32_t n_last, int32_t *kept_out, float *weights_out,
                       int64_t stride_out, int32_t *len_out, void *ws, size_t ws_bytes, void *stream_) {
  hipStream_t stream = (hipStream_t)stream_;
  int32_t rc;
  if ((rc = check_heads(heads, false)) || (rc = check_cache(cache, heads)) || (rc = check_cache(to, heads)) || (rc = check_max_len(cache, max_len)))
    return rc;
  const int32_t n_seqs = cache->n_seqs, hkv = heads->n_kv_heads, D = heads->head_dim;
  if (to->n_seqs != n_seqs) return fail(BA_ERR_INVALID_ARG, "to has %d sequences, the cache %d", to->n_seqs, n_seqs);
  if (n_keep < 1 || n_keep > (1 << 30)) return fail(BA_ERR_INVALID_ARG, "n_keep outside 1 .. 2^30");
  if (n_first < 0 || n_last < 0 || (int64_t)n_first + n_last > n_keep) return fail(BA_ERR_INVALID_ARG, "n_first and n_last: more than n_keep, or negative");
  if ((int64_t)to->max_pages * to->page_rows < std::min(n_keep, max_len)) return fail(BA_ERR_INVALID_ARG, "n_keep reaches beyond the page table of to");
  if (n_seqs == 0) return BA_OK;
  if (!kept_out || !seq_len || (!weights && max_len > 0)) return fail(BA_ERR_INVALID_ARG, "kept_out / seq_len / weights: null");
  if ((rc = check_int_array(weights, "weights")) || (rc = check_int_array(weights_out, "weights_out")) || (rc = check_int_array(seq_len, "seq_len")) ||
      (rc = check_int_array(kept_out, "kept_out")) || (rc = check_int_array(len_out, "len_out")))
    return rc;
  if (stride_weights < max_len) return fail(BA_ERR_INVALID_ARG, "stride_weights smaller than max_len");
  if (weights_out && stride_out < n_keep) return fail(BA_ERR_INVALID_ARG, "stride_out smaller than n_keep");
  const int64_t lists = (int64_t)n_seqs * hkv;
  if ((rc = check_lists(n_seqs, heads))) return rc;
  if (n_seqs * evict_copy_chunks(n_keep, max_len, hkv) > kMaxWorkgroups || (int64_t)std::min(n_keep, max_len) * hkv > (1 << 30))
    return fail(BA_ERR_UNSUPPORTED, "2^24 work items and more in one launch");
  // ---- where everything lies
  if (!apart(extent(&to->k, to->page_rows, hkv, D), extent(&to->v, to->page_rows, hkv, D)))
    return fail(BA_ERR_INVALID_ARG, "to: keys and values of a page overlap");
  const Extent from[2] = {k_pool(cache, heads), v_pool(cache, heads)}, target[2] = {k_pool(to, heads), v_pool(to, heads)};
  const bool same = same_place(&cache->k, &to->k) && same_place(&cache->v, &to->v) && cache->k_stride_page == to->k_stride_page &&
                    cache->v_stride_page == to->v_stride_page;
  if (same) {
    if (cache->page_table == to->page_table) return fail(BA_ERR_INVALID_ARG, "to names the pages that the sequences read");
    if (!apart(extent(&cache->k, cache->page_rows, hkv, D), extent(&cache->v, cache->page_rows, hkv, D)))
      return fail(BA_ERR_INVALID_ARG, "cache: keys and values of a page overlap");
  } else {
    for (const Extent &a : from)
      for (const Extent &b : target)
        if (!apart(a, b)) return fail(BA_ERR_INVALID_ARG, "to overlaps the cache without being the same pool");
  }
  struct {
    Extent x;
    const char *name;
    bool written;
  } all[] = {{from[0], "the cache", false}, {from[1], "the cache", false}, {target[0], "to", true}, {target[1], "to", true},
             {lists_extent(weights, lists, stride_weights, max_len), "weights", false}, {flat(seq_len, (int64_t)n_seqs * 4), "seq_len", false},
             {flat(kept_out, lists * n_keep * 4), "kept_out", true},
             {weights_out ? lists_extent(weights_out, lists, stride_out, n_keep) : flat(nullptr, 0), "weights_out", true},
             {len_out ? flat(len_out, (int64_t)n_seqs * 4) : flat(nullptr, 0), "len_out", true}};
  for (int i = 4; i < 9; ++i)
    for (int j = 0; j < i; ++j)
      if ((all[i].written || all[j].written) && !apart(all[i].x, all[j].x)) return fail(BA_ERR_INVALID_ARG, "%s overlaps %s", all[i].name, all[j].name);
  EvictParams p;
  memset(&p, 0, sizeof(p));
  p.weights = weights, p.w_stride = stride_weights;
  p.seq_len = seq_len;
  p.cap = max_len, p.n_seqs = n_seqs, p.n_kv_heads = hkv, p.head_dim = D;
  p.n_keep = n_keep, p.n_first = n_first, p.n_last = n_last;
  p.kept = kept_out;
  p.w_out = weights_out, p.w_out_stride = stride_out;
  p.len_out = len_out;
  set_rows(&p.k, &cache->k, cache->k_stride_page), set_rows(&p.v, &cache->v, cache->v_stride_page);
  set_rows(&p.to_k, &to->k, to->k_stride_page), set_rows(&p.to_v, &to->v, to->v_stride_page);
  set_table(&p.from, cache), set_table(&p.to, to);
  p.heads_div = make_fast_div((uint32_t)hkv);
  // Rows go by once, and are read next after all other layers' have gone by, too.  us a call with / without the hint, 1,024 rows of eight heads of
  // 128 for 8 sequences (67 MB read and written) 22.3 / 21.5, 16 36.1 / 39.7, 24 50.0 / 54.0, 64 118 / 124.
  p.past_caches = lists * std::min(n_keep, max_len) * D * 8 > kCacheBytes * 3 / 8;
  // Up to a list a compute unit, and lists short enough for four waves: one launch, in which as many workgroups as there is room for make a list's
  // choice, each of them for 32 rows of 128 at least.  us, in one launch and in two, 8 lists of 2,064 tokens, 64 rows of 128 kept 7.1 / 10.7, 512 7.5 / 10.6
  // (for 16, 64, 128 rows at least 7.4, 7.6, 9.1); 64 lists, 512 12.3 / 14.5; 256 lists, 256 19.1 / 20.5; 8 lists of 8,000, 2,048 13.4 / 15.6; 512 lists of
  // 100 tokens, 50 8.8 / 12.0; of 1,000, 64 11.8 / 14.8; of 2,000, 128 23.6 / 22.3; of 8,000, 128 35 / 30.
  const int64_t rows = std::max<int64_t>(1, std::min(n_keep, max_len));
  if (lists <= num_cus() || max_len <= kPickFourWaves) {
    p.parts = (int32_t)std::min<int64_t>(std::max<int64_t>(1, num_cus() / lists), (rows * D + kEvictPartLeast - 1) / kEvictPartLeast);
    p.part_rows = (int32_t)((rows + p.parts - 1) / p.parts);
    p.parts = (int32_t)((rows + p.part_rows - 1) / p.part_rows);
    if ((int64_t)p.part_rows * D > kEvictPartMost) p.parts = p.part_rows = 0;
  }
  hipError_t e;
  {
    ProfileScope ps(BA_PROFILE_COMBINE, stream);
    e = launch_evict_pick(p, stream);
  }
  if (e == hipSuccess && p.parts == 0) {
    ProfileScope ps(BA_PROFILE_REENCODE, stream);
    e = launch_evict_copy(p, stream);
  }
  return e == hipSuccess ? BA_OK : device_fail(e, "evict launch");
}

int32_t ba_page_bounds(const ba_heads *heads, const ba_paged_cache *cache, const ba_page_bound_table *bounds, const int32_t *from_token,
                       const int32_t *seq_len, int32_t max_len, void *stream) {
  int32_t rc;
  if ((rc = check_heads(heads, false)) || (rc = check_cache(cache, heads)) || (rc = check_max_len(cache, max_len)) || (rc = check_bounds(bounds)))
    return rc;
  const int32_t n_seqs = cache->n_seqs, hkv = heads->n_kv_heads;
  if (n_seqs == 0 || max_len == 0) return BA_OK;
  if (!seq_len) return fail(BA_ERR_INVALID_ARG, "seq_len: null");
  if ((rc = check_int_array(seq_len, "seq_len")) || (rc = check_int_array(from_token, "from_token")) || (rc = check_lists(n_seqs, heads))) return rc;
  const int64_t per_page = (int64_t)hkv * 2 * heads->head_dim;
  const Extent codes = flat(bounds->codes, cache->n_pages * per_page), exps = flat(bounds->exponents, (int64_t)cache->n_pages * hkv);
  for (const Extent &pool : {k_pool(cache, heads), v_pool(cache, heads)})
    if (!apart(pool, codes) || !apart(pool, exps)) return fail(BA_ERR_INVALID_ARG, "bounds overlap the cache");
  if (!apart(codes, exps)) return fail(BA_ERR_INVALID_ARG, "bounds: codes and exponents overlap");
  PageBoundsParams p;
  memset(&p, 0, sizeof(p));
  set_rows(&p.k, &cache->k, cache->k_stride_page);
  set_table(&p.pages, cache);
  p.codes = bounds->codes, p.exps = bounds->exponents;
  p.from = from_token, p.seq_len = seq_len;
  p.cap = max_len, p.n_seqs = n_seqs, p.n_kv_heads = hkv;
  ProfileScope ps(BA_PROFILE_REENCODE, (hipStream_t)stream);
  const hipError_t e = launch_page_bounds(p, heads->head_dim, (hipStream_t)stream);
  return e == hipSuccess ? BA_OK : device_fail(e, "page bounds launch");
}

size_t ba_page_select_workspace_bytes(const ba_heads *heads, int32_t n_seqs, int32_t page_rows, int32_t max_len) {
  if (check_heads(heads, true) != BA_OK || n_seqs <= 0 || page_rows < 1 || check_max_len(nullptr, max_len) != BA_OK || check_lists(n_seqs, heads) != BA_OK) return 0;
  return align256((size_t)n_seqs * heads->n_kv_heads * (((size_t)max_len + page_rows - 1) / page_rows) * 4);
}

int32_t ba_page_select(const ba_heads *heads, const ba_paged_cache *cache, const ba_page_bound_table *bounds, const ba_tensor *q, int32_t q_per_seq,
                       const int32_t *seq_len, int32_t max_len, int32_t n_select, int32_t n_first, int32_t n_last, int32_t *selected_out,
                       float *scores_out, void *ws, size_t ws_bytes, void *stream_) {
  hipStream_t stream = (hipStream_t)stream_;
  int32_t rc;
  if ((rc = check_heads(heads, true)) || (rc = check_cache(cache, heads)) || (rc = check_bounds(bounds))) return rc;
  const int32_t n_seqs = cache->n_seqs, hkv = heads->n_kv_heads, hq = heads->n_q_heads, D = heads->head_dim;
  if ((rc = check_paged_sizes(heads, n_seqs, q_per_seq, max_len)) || (rc = check_max_len(cache, max_len))) return rc;
  const int64_t newest = ((int64_t)q_per_seq + cache->page_rows - 2) / cache->page_rows + 1;  // pages that a sequence's newest tokens may lie in
  if (n_first < 0 || n_last < 0 || n_select < 1 || n_first + std::max<int64_t>(n_last, newest) > n_select)
    return fail(BA_ERR_INVALID_ARG, "n_select has no room for the first, the last and the newest pages");
  if (n_select > (1 << 30)) return fail(BA_ERR_UNSUPPORTED, "n_select beyond 2^30");  // (places of a list are counted on in 32 bits)
  if (n_seqs == 0) return BA_OK;
  if ((rc = check_tensor(q, "q", false, D, hq)) || (rc = check_lists(n_seqs, heads))) return rc;
  if (!seq_len || !selected_out) return fail(BA_ERR_INVALID_ARG, "seq_len / selected_out: null");
  if ((rc = check_int_array(seq_len, "seq_len")) || (rc = check_int_array(selected_out, "selected_out")) || (rc = check_int_array(scores_out, "scores_out")))
    return rc;
  const int64_t lists = (int64_t)n_seqs * hkv, tokens = (int64_t)n_seqs * q_per_seq;
  const Extent out[2] = {flat(selected_out, lists * n_select * 4), scores_out ? flat(scores_out, lists * n_select * 4) : flat(nullptr, 0)};
  for (const Extent &x : out)
    if (!apart(x, extent(q, tokens, hq, D)) || !apart(x, flat(bounds->codes, (int64_t)cache->n_pages * hkv * 2 * D)) ||
        !apart(x, flat(bounds->exponents, (int64_t)cache->n_pages * hkv)) || !apart(x, flat(seq_len, (int64_t)n_seqs * 4)))
      return fail(BA_ERR_INVALID_ARG, "selected_out or scores_out overlap q, the bounds or seq_len");
  if (!apart(out[0], out[1])) return fail(BA_ERR_INVALID_ARG, "scores_out overlaps selected_out");
  const size_t need = ba_page_select_workspace_bytes(heads, n_seqs, cache->page_rows, max_len);
  if (need > 0 && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need))
    return fail(BA_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than %zu bytes", need);
  PageSelectParams p;
  memset(&p, 0, sizeof(p));
  p.q = (const uint16_t *)q->ptr;
  p.q_st = q->stride_tok, p.q_sh = q->stride_head;
  set_table(&p.pages, cache);
  p.codes = bounds->codes, p.exps = bounds->exponents;
  p.seq_len = seq_len;
  p.cap = max_len, p.n_seqs = n_seqs, p.n_kv_heads = hkv, p.nq = q_per_seq, p.group = hq / hkv;
  p.group_div = make_fast_div((uint32_t)p.group);
  p.n_select = n_select, p.n_first = n_first, p.n_last = n_last;
  p.selected = selected_out, p.scores_out = scores_out;
  p.scores = (float *)ws;
  p.score_stride = ((int64_t)max_len + cache->page_rows - 1) / cache->page_rows;
  if ((n_seqs * ((p.score_stride + kScorePages - 1) / kScorePages) + 8) * hkv > kMaxWorkgroups) return fail(BA_ERR_UNSUPPORTED, "2^24 work items and more in one launch");
  hipError_t e = hipSuccess;
  if (p.score_stride <= kSelectOneLaunch) {
    ProfileScope ps(BA_PROFILE_ATTENTION, stream);
    e = launch_page_select(p, D, stream);
    return e == hipSuccess ? BA_OK : device_fail(e, "page selection launch");
  }
  if (max_len > 0) {
    ProfileScope ps(BA_PROFILE_ATTENTION, stream);
    e = launch_page_scores(p, D, stream);
  }
  if (e == hipSuccess) {
    ProfileScope ps(BA_PROFILE_COMBINE, stream);
    e = launch_page_pick(p, stream);
  }
  return e == hipSuccess ? BA_OK : device_fail(e, "page selection launch");
}

}  // extern "C"
