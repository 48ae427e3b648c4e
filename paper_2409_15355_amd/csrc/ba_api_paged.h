// Checks that the entry points around the paged cache share (ba_api_paged.hip, ba_api_long.hip).  Defined in ba_api_paged.hip.
#pragma once

#include "../../include/ba.h"
#include "ba_api_common.h"

namespace ba {
namespace api {

// Where a tensor lies: its rows [0, tokens).
struct Extent {
  int64_t lo, hi;           // bytes
  int64_t period, width;    // bytes from row to row, bytes of a row from its first head to its last
  int64_t step, head;       // bytes from head to head, bytes of a head
  int64_t rows;
  int32_t heads;
};
Extent extent(const ba_tensor *t, int64_t tokens, int n_heads, int D);
Extent pool_extent(const ba_tensor *t, int64_t stride_page, const ba_paged_cache *c, const ba_heads *h);
bool apart(const Extent &a, const Extent &b);
bool same_place(const ba_tensor *a, const ba_tensor *b);

int32_t check_int_array(const void *p, const char *name);
int32_t check_apart(const ba_tensor *a, const char *a_name, int a_heads, const ba_tensor *b, const char *b_name, int b_heads, int64_t tokens, int D);
int32_t check_cache(const ba_paged_cache *c, const ba_heads *h);
int32_t check_groups(int32_t n_seqs, int32_t max_len, int32_t n_groups, const int32_t *cu_group, const int32_t *prefix_len);
int32_t check_paged_sizes(const ba_heads *h, int32_t n_seqs, int32_t nq, int32_t max_len);

}  // namespace api
}  // namespace ba
