// The rotation of 16 elements of a row, 8 whole pairs, shared by the kernels that rotate strided rows.
#pragma once
#include "tree.hpp"

namespace forge {

// 8 elements as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<bf16> {
  u32x4 w;
  __device__ inline void load(const bf16* p) { w = *reinterpret_cast<const u32x4*>(p); }
  __device__ inline void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf_lo(w[i]); v[2 * i + 1] = bf_hi(w[i]); }
  }
};
template <> struct Raw8<float> {
  floatx4 w[2];
  __device__ inline void load(const float* p) {
    w[0] = *reinterpret_cast<const floatx4*>(p);
    w[1] = *reinterpret_cast<const floatx4*>(p + 4);
  }
  __device__ inline void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = w[0][i]; v[4 + i] = w[1][i]; }
  }
};

// Which 16 elements of a row of dh an item owns: two runs of 8, those of neighbouring items side by side.
// HALF: of the turning part the pairs 8 item .. 8 item + 7, rot / 2 apart, of the rest its halves; otherwise the row's halves.
template <bool HALF>
struct PairTurns {
  float cs[8], sn[8];
  int e0, e1;        // the two runs of 8 elements
  bool turns[2];     // each of them (HALF: both or none)

  __device__ inline PairTurns(const Turns& t, int item, int dh) {
    const int rot = t.inc != nullptr ? t.rot : 0;
    if (HALF) {
      const bool in = 16 * item < rot;
      e0 = in ? 8 * item : rot + 8 * (item - rot / 16);
      e1 = e0 + (in ? rot : dh - rot) / 2;
      turns[0] = turns[1] = in;
    } else {
      e0 = 8 * item;
      e1 = e0 + dh / 2;
      turns[0] = e0 < rot;
      turns[1] = e1 < rot;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
  }
  __device__ inline void at(const Turns& t, int position) {
#pragma unroll
    for (int r = 0; r < 2; ++r)
      if (turns[r]) {
        // HALF: pairs e0 + i; otherwise those inside the run
        const uint64_t* inc = t.inc + (HALF ? e0 + 4 * r : (r ? e1 : e0) / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          turn_cos_sin(turned(position, inc[i]), cs[4 * r + i], sn[4 * r + i]);
          cs[4 * r + i] *= t.factor;
          sn[4 * r + i] *= t.factor;
        }
      }
  }
  // (elements that do not turn are left alone: 0 * infinity would be NaN)
  __device__ inline void turn(float (&a)[8], float (&c)[8]) const {
    auto pair = [&](float& u, float& w, int i) {
      const float x = u, y = w;
      u = x * cs[i] - y * sn[i];
      w = y * cs[i] + x * sn[i];
    };
    if constexpr (HALF) {
      if (turns[0])
#pragma unroll
        for (int i = 0; i < 8; ++i) pair(a[i], c[i], i);
    } else {
      if (turns[0])
#pragma unroll
        for (int i = 0; i < 4; ++i) pair(a[2 * i], a[2 * i + 1], i);
      if (turns[1])
#pragma unroll
        for (int i = 0; i < 4; ++i) pair(c[2 * i], c[2 * i + 1], 4 + i);
    }
  }
};

// Head groups (the grid's second axis): enough for 4 waves per SIMD, at most one per head; long prompts share the angles of a token
// among the heads of a group, a few tokens are spread over all heads.  As many as the registers let run, about: 92 to 110 of them, 4 or 5 waves, for
// 16-bit rotation and 8-bit append; 80 and up to 6 for 16-bit append, 110 to 132 and 3 or 4 in fp32, where more groups were not
// measured.  us for 2 | 4 | 8 | 16: rotation of 4096 tokens x 40 heads of 128 19.1 | 19.9 | 21.5 | 23.5, of 8192 x 32 36.8 | 30.6 | 32.8 | 35.8; append of
// 8192 x 48 to fp8 43.7 | 40.7 | 41.8 | 43.1, of 2048 x 48 to int8 11.7 | 12.0 | 12.8 | 15.0.
inline int row_head_groups(int64_t blocks, int heads) {
  const int64_t g = ceil_div64(4 * (int64_t)compute_units(), blocks);
  return (int)(g > heads ? heads : g);
}

// Rows h0 .. h1 - 1 in turn, two requested while two are worked on: row(h) gives one, finish(h, a, c) takes its two runs.
// first: called once the first are on their way (what does not depend on them).
template <typename T, typename Row, typename First, typename Finish>
__device__ inline void walk_heads(int h0, int h1, int e0, int e1, Row row, First first, Finish finish) {
  constexpr int N = 2;
  Raw8<T> a[2][N], c[2][N];
  auto request = [&](int h, int buf) {
#pragma unroll
    for (int u = 0; u < N; ++u)
      if (h + u < h1) {
        const T* r = row(h + u);
        a[buf][u].load(r + e0);
        c[buf][u].load(r + e1);
      }
  };
  request(h0, 0);
  first();
  for (int h = h0; h < h1; h += 2 * N) {
#pragma unroll
    for (int buf = 0; buf < 2; ++buf) {
      const int at = h + buf * N;
      request(at + N, buf ^ 1);
#pragma unroll
      for (int u = 0; u < N; ++u)
        if (at + u < h1) {
          float x[8], y[8];
          a[buf][u].values(x);
          c[buf][u].values(y);
          finish(at + u, x, y);
        }
    }
  }
}

}  // namespace forge
