// How the attention of drafted trees cuts its work: host arithmetic without a device, so that a host build of it can be asked.  Internal
// to the library.  (ceil_div and ceil_div64 come before it, from common.hpp.)
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>

namespace forge {

constexpr int TILE = 32;                  // cache rows per step of a wave
constexpr int UNIT = 128;                 // cache rows that are dealt together
constexpr int MAX_DEALT = 256;            // sequences of a dealt batch (a larger one has blocks enough)
constexpr int kMaxPairs = 65535;          // (sequence, cache head) pairs of one: a grid dimension of the merge

// ---- how the work is cut ---------------------------------------------------------------------------------------
// The kernel by its query rows per block, whole pairs or shares (one or two per CU), by the least estimated time: a block alone on its CU walks
// over `alone` cache rows per us, the blocks of a full CU together over `full`, the memory gives 6.2 MB; to the largest of the three (a cubic
// mean: they add a little) comes 1 us for every block per CU, and for shares the merge launch of 3 us, the partials at 4.2 MB per us and
// 1.4 us for every pair a share has on the average.  The host does not know a ragged batch's lengths; 0.63 of the longest cache is taken for
// the mean, that of lengths spread evenly from a quarter to all, as in the calls that the other numbers were fitted to (1100 drawn ones of more than
// 16 query rows, heads of 64 and 128, 1 to 64 sequences, 3 to 64 tokens, timed at every choice).  What the choice costs over the best one, in the
// geometric mean and at most, 250 other calls of 1 to 64 tokens each: lengths like that 1.3 and 27 %, all alike 1.3 and 29 %, one long cache among
// short ones 4.3 and 62 %.  Anything from 0.4 in its place moves these by less than a point.  us, whole | 256 shares | 512:
// 7 sequences up to 4984 rows of 16 heads of 128, 5 tokens 56.8 | 39.7 | 40.4, 62 up to 137 of 8 x 4, 10 tokens, blocks of 128 rows
// 15.8 | 27.5 | 26.5, of 32 rows 25.4 | 35.9 | 29.2, 16 up to 8191 of 8 x 4, 64 tokens, of 256 rows 195 | 124 | -, of 128 rows 167 | 145 | 133,
// of 32 rows 181 | 221 | 181.
struct TreePlan { int block_rows, row_blocks, shares, dealt, each; };
struct TreeSpeed { int block_rows; float alone[2], full[2]; };      // rows per us, heads of 128: 8 bits, 16 bits
constexpr TreeSpeed kSpeeds[] = {{16, {160.f, 190.f}, {300.f, 200.f}}, {32, {150.f, 167.f}, {105.f, 86.f}},
                                 {128, {51.f, 60.f}, {54.f, 54.f}}, {256, {35.f, 40.f}, {133.f, 52.f}}};
constexpr int MIN_CUT_ROWS = 512;         // a shorter cache is never dealt, so its calls need no workspace

// whether a call may run on blocks of this many query rows (fp32 and few rows: the smallest; a cache of less than one tile: not on
// the kernel that reads whole tiles, unless it is fp32, where that clamps each row)
inline bool tree_rows_ok(int block_rows, int rows, int cap, bool f32) {
  if (f32) return block_rows == 16;
  if (cap < TILE) return block_rows == 128;
  if (rows <= 16) return block_rows == 16;
  return block_rows == 32 || block_rows == 128 || (block_rows == 256 && rows > 128);
}
inline int64_t tree_units(int64_t pairs, int len) { return pairs * ceil_div(len, UNIT); }
// the shares of a dealt call with `per_cu` blocks per CU: of two units at least
inline int tree_shares(int64_t pairs, int len, int row_blocks, int per_cu, int cus) {
  const int64_t most = (int64_t)per_cu * cus / row_blocks, least = ceil_div64(tree_units(pairs, len), 2);
  return (int)(most < 1 ? 1 : most < least ? most : least);
}
inline bool tree_may_deal(int batch, int64_t pairs, int len) {
  return batch <= MAX_DEALT && len > MIN_CUT_ROWS && tree_units(pairs, len) < (1ll << 31) && pairs <= kMaxPairs;
}
inline TreePlan plan_tree(int batch, int q_heads, int kv_heads, int head_dim, int n, int len, int cap, int element_bytes, bool ragged,
                          int cus) {
  const int rows = q_heads / kv_heads * n, wide = element_bytes > 1;
  const bool f32 = element_bytes == 4;
  const double pairs = (double)batch * kv_heads, mean = (ragged && batch > 1 ? 0.63 : 1.0) * len;
  const double mb = pairs * mean * 2.0 * (head_dim * element_bytes + (wide ? 0 : 4)) * 1e-6;
  TreePlan best = {};
  double least = 0.0;
  for (const TreeSpeed& v : kSpeeds) {
    if (!tree_rows_ok(v.block_rows, rows, cap, f32)) continue;
    const int rb = ceil_div(rows, v.block_rows);
    const double by = head_dim == 128 ? 1.0 : f32 ? 2.0 : v.block_rows == 16 ? 1.6 : v.block_rows == 32 ? 1.8 : 1.5;
    const double alone = v.alone[wide] * by * (f32 ? 0.32 : 1.0), full = v.full[wide] * by * (f32 ? 0.2 : 1.0);
    for (int per_cu = 0; per_cu <= (v.block_rows == 256 ? 1 : 2); ++per_cu) {      // 0: whole pairs
      if (per_cu > 0 && !tree_may_deal(batch, (int64_t)batch * kv_heads, len)) break;
      const int shares = per_cu > 0 ? tree_shares((int64_t)batch * kv_heads, len, rb, per_cu, cus) : batch * kv_heads;
      const double share = fmax(pairs * mean / shares, (double)UNIT);
      const double a = (per_cu > 0 ? share : len) / alone, b = pairs * mean * rb / (cus * full), c = mb / 6.2;
      double us = cbrt(a * a * a + b * b * b + c * c * c) + (double)shares * rb / cus;
      if (per_cu > 0)
        us += 3.0 + (shares + pairs) * rb * fmin(v.block_rows, rows) * head_dim * 8e-6 / 4.2 + 1.4 * pairs / shares;
      if (best.block_rows == 0 || us < least) {
        least = us;
        best = {v.block_rows, rb, shares, per_cu > 0, 0};
      }
    }
  }
  // A short cache has fewer tiles than a block waves; where blocks have to wait for others, a wave per pair instead (of 16 query rows, also of
  // the second 16 of up to 32).  us, a block | a wave a pair, one token: 55 x 12 pairs of 64 up to 22 rows 9.0 | 4.9, 64 x 8 of 128 up to 28 8.7 | 5.7,
  // 99 x 8 up to 82 14.0 | 10.2; time of the wave against the block's: 1 to 2 pairs a CU up to 96 rows 0.7 to 0.95, up to 256 1.0 to 1.2; more pairs
  // up to 192 rows 0.65 to 0.95, up to 400 1.0 to 1.1; 17 to 32 query rows up to 192 rows 0.6 to 0.9, up to 256 0.9 to 1.05 (62 x 16 up to 86, 17 tokens
  // 30.6 | 20.3); 33 query rows and more 0.8 to 1.3, so not there
  const int64_t blocks = (int64_t)best.shares * best.row_blocks;
  const bool two = best.block_rows > 16 && rows <= 32 && cap >= TILE;
  if (!best.dealt && blocks > cus &&
      (two ? len <= 192 : best.block_rows == 16 && len <= (blocks > 2 * cus ? 192 : 96))) {
    best.each = 1;
    best.block_rows = 16;
    best.row_blocks = ceil_div(rows, 16);
  }
  return best;
}

// room for the shares of any shorter cache too: for each kind of block their number only falls with the length
inline size_t tree_workspace_bytes(int batch, int q_heads, int kv_heads, int head_dim, int n, int len, int cap, bool f32, int cus) {
  const int64_t pairs = (int64_t)batch * kv_heads;
  const int rows = q_heads / kv_heads * n;
  if (batch > MAX_DEALT || pairs > kMaxPairs || len <= MIN_CUT_ROWS) return 0;
  size_t most = 0;
  for (const TreeSpeed& v : kSpeeds) {
    if (!tree_rows_ok(v.block_rows, rows, cap, f32)) continue;
    const int rb = ceil_div(rows, v.block_rows);
    const size_t b = (size_t)tree_shares(pairs, len, rb, v.block_rows == 256 ? 1 : 2, cus) * rb * 2 * v.block_rows * (head_dim + 2) * sizeof(float);
    most = b > most ? b : most;
  }
  return most;
}

}  // namespace forge
