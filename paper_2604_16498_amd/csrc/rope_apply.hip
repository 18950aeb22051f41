// Rotary positions of strided rows: both pairings, part of a head, any position.  Memory-bound: every row is read
// and written once, in 16-byte accesses.
//
// The angle of pair i at position p is p * inc_i in units of 2^-64 turns, modulo 2^64: one integer multiply that loses whole
// turns and nothing else, so that neither a table by position nor fp64 is needed and cos / sin are good to 1.2e-7 at any
// position.  A thread owns 16 elements of a row that hold 8 whole pairs (two runs of 8: both halves of the pairs, or neighbours)
// and walks over a group of heads of one token, whose angles are the same; few tokens are spread over one head per thread.
#include "tree.hpp"
#include "rope_rows.hpp"

namespace forge {
namespace {

template <typename T>
__global__ __launch_bounds__(256) void rope_apply_kernel(Turns t, Heads x, Heads y, const int* __restrict__ positions, int n,
                                                         int heads, int items, int head_groups, uint32_t total) {
  const uint32_t gid = blockIdx.x * 256u + threadIdx.x;
  if (gid >= total) return;
  const uint32_t item = gid % items, rest = gid / items;
  const uint32_t hg = rest % head_groups, tok = rest / head_groups;
  const uint32_t b = tok / n, i = tok % n;
  const int per = ceil_div(heads, head_groups), h0 = hg * per, h1 = min(heads, h0 + per);
  PairTurns w(t, item, positions[tok]);
  const T* xr = reinterpret_cast<const T*>(x.p) + b * x.bs + i * x.ts;
  T* yr = reinterpret_cast<T*>(y.p) + b * y.bs + i * y.ts;
  for (int h = h0; h < h1; ++h) {
    float a[8], c[8];
    Vec8<T>::load(xr + h * x.hs + w.e0, a);
    Vec8<T>::load(xr + h * x.hs + w.e1, c);
    w.turn(a, c);
    Vec8<T>::store(yr + h * y.hs + w.e0, a);
    Vec8<T>::store(yr + h * y.hs + w.e1, c);
  }
}

}  // namespace

forge_status launch_rope_apply(const Turns& t, const Heads& x, const Heads& y, const int* positions, int batch, int n,
                               int heads, int head_dim, forge_dtype dt, hipStream_t s) {
  const int items = head_dim / 16;
  const int64_t base = (int64_t)batch * n * items;         // <= 2^24 * 64
  const int head_groups = row_head_groups(base, heads);
  const int64_t total = base * head_groups;                // <= max(base, 2^18): 32 bits
  const unsigned blocks = (unsigned)ceil_div64(total, 256);
  if (dt == FORGE_BF16)
    rope_apply_kernel<bf16><<<blocks, 256, 0, s>>>(t, x, y, positions, n, heads, items, head_groups, (uint32_t)total);
  else
    rope_apply_kernel<float><<<blocks, 256, 0, s>>>(t, x, y, positions, n, heads, items, head_groups, (uint32_t)total);
  return launch_status();
}

}  // namespace forge
