// The rotation of 16 elements of a row, 8 whole pairs, shared by the kernels that rotate strided rows.
#pragma once
#include "tree.hpp"

namespace forge {

struct PairTurns {
  float cs[8], sn[8];
  int e0, e1;        // the two runs of 8 elements
  bool turns, half;

  // item: which 16 elements of the row.  HALF: those of the pairs 8 item .. 8 item + 7, rot / 2 apart
  __device__ inline PairTurns(const Turns& t, int item, int position) {
    half = t.half;
    turns = t.inc != nullptr && 16 * item < t.rot;
    e0 = turns && half ? 8 * item : 16 * item;
    e1 = turns && half ? e0 + t.rot / 2 : e0 + 8;
    if (turns) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        turn_cos_sin((uint64_t)(int64_t)position * t.inc[8 * item + i], cs[i], sn[i]);
        cs[i] *= t.factor;
        sn[i] *= t.factor;
      }
    }
  }
  __device__ inline void turn(float (&a)[8], float (&c)[8]) const {
    if (!turns) return;
    if (half) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = a[i], w = c[i];
        a[i] = u * cs[i] - w * sn[i];
        c[i] = w * cs[i] + u * sn[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float u = a[2 * i], w = a[2 * i + 1], u2 = c[2 * i], w2 = c[2 * i + 1];
        a[2 * i] = u * cs[i] - w * sn[i];
        a[2 * i + 1] = w * cs[i] + u * sn[i];
        c[2 * i] = u2 * cs[4 + i] - w2 * sn[4 + i];
        c[2 * i + 1] = w2 * cs[4 + i] + u2 * sn[4 + i];
      }
    }
  }
};

// Head groups: enough to reach 128k threads, at most one per head (long prompts share an angle among the heads of a token)
inline int row_head_groups(int64_t base_threads, int heads) {
  const int64_t g = ceil_div64(131072, base_threads);
  return (int)(g > heads ? heads : g);
}

}  // namespace forge
