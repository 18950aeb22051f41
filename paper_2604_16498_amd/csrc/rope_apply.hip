// Rotary positions of strided rows: both pairings, part of a head, any position.  Memory-bound: every row is read
// and written once, in 16-byte accesses.
//
// The angle of pair i at position p is p * inc_i in units of 2^-64 turns, modulo 2^64: one integer multiply that loses whole
// turns and nothing else, so that neither a table by position nor fp64 is needed and cos / sin are good to 1.2e-7 at any
// position.  A thread owns 16 elements of a token's rows that hold 8 whole pairs (two runs of 8: both halves of the pairs, or
// neighbours) and walks over a group of heads, whose angles are the same, two rows requested while two are turned.
// Measured: 4096 tokens x 40 heads of 128 in bf16 (84 MB) 17 us, 4.9 TB/s, where a copy of as many bytes takes 18; in
// fp32 (168 MB) 43 us, 3.9 TB/s at 3 waves per SIMD; 3 tokens x 24 heads of 64 in fp32 3.1 us, the time of a launch.  Stores that pass the caches by are faster alone (15 us) and slower with what reads the
// rows next (32 MB and a reader 29.7 against 33.0 us), so they are ordinary ones.
#include "tree.hpp"
#include "rope_rows.hpp"

namespace forge {
namespace {

template <typename T, bool HALF>
__global__ __launch_bounds__(256) void rope_apply_kernel(Turns t, Heads x, Heads y, const int* __restrict__ positions, int n,
                                                         int heads, int items, uint32_t total) {
  const uint32_t gid = blockIdx.x * 256u + threadIdx.x;
  if (gid >= total) return;
  const uint32_t item = gid % items, tok = gid / items, b = tok / n, i = tok % n;
  const int per = ceil_div(heads, gridDim.y), h0 = blockIdx.y * per, h1 = min(heads, h0 + per);
  PairTurns<HALF> w(t, item, items * 16);
  const T* xr = reinterpret_cast<const T*>(x.p) + b * x.bs + i * x.ts;
  T* yr = reinterpret_cast<T*>(y.p) + b * y.bs + i * y.ts;
  walk_heads<T>(h0, h1, w.e0, w.e1, [&](int h) { return xr + h * x.hs; }, [&] { w.at(t, positions[tok]); },
                [&](int h, float (&a)[8], float (&c)[8]) {
                  w.turn(a, c);
                  Vec8<T>::store(yr + h * y.hs + w.e0, a);
                  Vec8<T>::store(yr + h * y.hs + w.e1, c);
                });
}

}  // namespace

forge_status launch_rope_apply(const Turns& t, const Heads& x, const Heads& y, const int* positions, int batch, int n,
                               int heads, int head_dim, forge_dtype dt, hipStream_t s) {
  const int items = head_dim / 16;
  const int64_t total = (int64_t)batch * n * items;        // <= 2^24 * 64
  const unsigned blocks = (unsigned)ceil_div64(total, 256);
  const dim3 grid(blocks, row_head_groups(blocks, heads));
  auto go = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(t, x, y, positions, n, heads, items, (uint32_t)total); };
  if (dt == FORGE_BF16) t.half ? go(rope_apply_kernel<bf16, true>) : go(rope_apply_kernel<bf16, false>);
  else t.half ? go(rope_apply_kernel<float, true>) : go(rope_apply_kernel<float, false>);
  return launch_status();
}

}  // namespace forge
