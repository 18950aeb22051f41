// How the adapters of many requests cut their work: host arithmetic without a device, so that a host build of it can be asked.  Internal
// to the library.  (ceil_div and ceil_div64 come before it, from common.hpp.)
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace forge {

constexpr int JT = 4;          // 16-wide tiles of the inner index a block of the first launch works on

// groups: of 64 columns, a block of the second launch
struct Cut { int tiles, splits, chunks, lanes, groups; };

// Whether blocks take 64 rows, most of which share an adapter with their neighbours: where their tiles of 64 rows and 256 columns, and in the first launch
// 64 rows and 64 inner columns, are enough.  bf16, 64 rows | 16, us: 768 x 768, rank 64, 1500 rows (69 tiles) 14.2 | 14.0, 4096 (192) 15.5 | 18.7; 4096 x 4096,
// rank 64, 512 rows (128, 8 in the first launch) 18.6 | 17.0, 1000 20.9 | 22.4, 4096 36.6 | 50.4; beside q, k and v (192, 24) 24.5 | 28.0.  In fp32 a block's
// chain of matrix instructions is 8 times as long: 2304 x 768, rank 64, 1500 rows (207 tiles) 36.1 | 35.6, 4096 (576) 61.5 | 71.1; rank 8 17.9 | 16.3 and
// 30.1 | 31.4.
// The adapter numbers lie on the device, so the rule cannot see a batch whose neighbours have different adapters: a block then works through up to 64 of them in
// turn, with 16 rows at most 16, dealt over more blocks.  4096 x 4096, row m with adapter m mod n, us: 1024 rows, rank 8, n = 8 25.7 | 31.3, 16 43.7 | 56.0,
// 24 64.6 | 55.2, 64 159 | 56.7, 1024 160 | 63.4; rank 64, 16 63.6 | 136, 32 110 | 136, 64 204 | 137, 512 233 | 183; 2048 rows, rank 8, 2048 249 | 125, rank 64,
// 512 318 | 293; fp32, 1024 rows, rank 8, 16 100 | 117, 64 369 | 119.  In runs of 16 rows, 1024 rows, rank 8 17.0 | 12.1, rank 64 29.8 | 24.4.  So the larger
// tiles gain up to about 20 adapters that alternate, and decode batches of more than 900 requests with one each lose by them.
constexpr int MANY = 512;
inline bool adapters_many(int M, int N, int inner, bool f32) {
  const int64_t tiles = (int64_t)(M / 64) * ceil_div(N, 256);
  return M >= MANY && (int64_t)M * ceil_div(inner, 16 * JT) >= 900 && tiles >= (f32 ? 256 : 72);
}
// whether the columns are whole blocks of the second launch for many rows
inline bool adapters_whole(int ldy, int parts, const int* part_end) {
  bool whole = ldy % 4 == 0;
  for (int i = 0; i < parts; ++i) whole = whole && part_end[i] % 256 == 0;
  return whole;
}
// steps of 64 bytes of a row of b that the second launch's kernel holds: 1, 2, 4, in fp32 also 8
inline int adapters_steps(int rank, bool f32) {
  const int steps = ceil_div(rank, f32 ? 16 : 32);
  return steps <= 2 ? steps : steps <= 4 ? 4 : 8;
}

// Blocks beside one another that deal a tile's adapters, of which 16 rows have at most 16, where there are few tiles: as many as are resident at once (a
// tile of a prompt has one adapter, and what more there are pass over it in turn; 3 | 8 per CU in both launches, 4096 x 4096, us: 500 rows of 5 requests,
// rank 64, 16.9 | 19.6; 256 requests of rank 8 20.0 | 26.1)
inline int adapters_lanes(int64_t blocks, int rows, int cus) {
  const int64_t l = ceil_div64(3 * cus, blocks);
  const int most = rows < 16 ? rows : 16;
  return (int)(l < 1 ? 1 : l < most ? l : most);
}

// K in ranges until the blocks fill the chip twice (of many rows once: 4096 x 4096, rank 64, 4 | 8 ranges 15.2 | 15.6 us, and less to add up)
inline int adapters_units(int K, bool f32) { return ceil_div(K, f32 ? 128 : 256); }
inline Cut adapters_cut(int M, int K, int inner, bool many, bool f32, int cus) {
  const int units = adapters_units(K, f32);
  Cut c;
  c.tiles = ceil_div(M, many ? 64 : 16);
  c.chunks = ceil_div(inner, 16 * JT);
  const int64_t blocks = (int64_t)c.tiles * c.chunks;
  const int want = (int)ceil_div64((many ? 1 : 2) * cus, blocks);
  const int most = many ? units : ceil_div(units, 2);     // (two units a block: both are on their way at once)
  c.splits = want < most ? want : most;
  c.lanes = many ? 2 : adapters_lanes(blocks * c.splits, M, cus);
  c.groups = 1;
  return c;
}

// Room for the ranges' t of any smaller M too: of m rows in `tiles` tiles the ranges are at most the units of K, and at most 2 cus (1 of 64 rows) /
// (tiles chunks) + 1; times m rows, of which a tile has at most 16 or 64
inline size_t adapters_room(int M, int K, int inner, bool f32, int cus) {
  const int64_t most = (int64_t)adapters_units(K, f32) * M;
  const int64_t full = ceil_div((M >= MANY ? 64 : 32) * cus, ceil_div(inner, 16 * JT)) + (int64_t)M;
  return (size_t)(most < full ? most : full) * inner * sizeof(float);
}

}  // namespace forge
