// How the attention over pages cuts its work, and the workspace that the shares need: host arithmetic, as tree_plan.hpp.  Internal to the library.
#pragma once
#include "tree_plan.hpp"

namespace forge {

// The cut of the drafted trees' kernel of 16 query rows, whose frame this one has; more than 16 query heads of a cache head are further blocks of each share
inline TreePlan plan_paged(int batch, int q_heads, int kv_heads, int head_dim, int max_len, int element_bytes, int cus) {
  const int group = q_heads / kv_heads;
  TreePlan p = plan_tree(batch, kv_heads * (group < 16 ? group : 16), kv_heads, head_dim, 1, max_len, 1 << 30, element_bytes, true, cus);
  p.row_blocks = ceil_div(group, 16);
  return p;
}
// floats of the partials of one share: two slots of 16 rows for each block of query heads, an output row and two statistics each
inline int64_t paged_partials(int row_blocks, int head_dim) { return (int64_t)row_blocks * 2 * 16 * (head_dim + 2); }

// Room for the shares of any smaller batch and shorter request: their number only falls with either.
inline size_t paged_room(int batch, int q_heads, int kv_heads, int head_dim, int max_len, int cus) {
  const int most = kMaxPairs / kv_heads < MAX_DEALT ? kMaxPairs / kv_heads : MAX_DEALT;
  const int64_t pairs = (int64_t)(batch < most ? batch : most) * kv_heads;
  if (max_len <= MIN_CUT_ROWS) return 0;
  return (size_t)(tree_shares(pairs, max_len, 1, 2, cus) * paged_partials(ceil_div(q_heads / kv_heads, 16), head_dim)) * sizeof(float);
}

}  // namespace forge
