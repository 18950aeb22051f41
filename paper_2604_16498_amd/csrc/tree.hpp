// What the operators of serving drafted trees share: arguments of their launchers, cache rows in 8 bits.
// Internal to the library.
#pragma once
#include "common.hpp"

namespace forge {

// device copy of a forge_heads (strides of axes with one entry are 0)
struct Heads {
  char* p;
  int64_t bs, ts, hs;    // elements
};

// device copy of a forge_rope_desc; increments NULL: no rotation
struct Turns {
  const uint64_t* inc;
  int rot;               // elements of a head that turn
  int half;              // pairs (i, i + rot / 2) instead of (2i, 2i + 1)
  float factor;
};

// one layer of a cache
struct CacheView {
  char *k, *v;
  float *ks, *vs;
  int64_t bs, hs;        // elements; of the scales these over head_dim
};

struct AppendArgs {
  CacheView c;
  Turns t;
  Heads k, v, q, qo;     // q.p NULL: none
  int batch, n, q_heads, kv_heads, head_dim, max_pos;
  const int* seq_pos;
  const int* positions;
  forge_kv_type type;
  forge_dtype dt;
};

struct TreeArgs {
  CacheView c;
  Heads q;
  void* out;
  const int* seq_pos;
  const uint64_t* visible;
  int batch, n, q_heads, kv_heads, head_dim, max_pos, cap;
  float scale;
  forge_kv_type type;
  forge_dtype dt;
  void* workspace;
};

forge_status launch_rope_apply(const Turns& t, const Heads& x, const Heads& y, const int* positions, int batch, int n,
                               int heads, int head_dim, forge_dtype dt, hipStream_t s);
forge_status launch_kv_append(const AppendArgs& a, hipStream_t s);
forge_status launch_kv_read(const CacheView& c, forge_kv_type type, forge_dtype dt, int batch, int kv_heads, int head_dim,
                            void* k_out, void* v_out, const int* seq_pos, int n, int max_pos, hipStream_t s);
forge_status launch_kv_commit(const CacheView& c, forge_kv_type type, forge_dtype dt, int n_layers, int64_t layer_stride,
                              int batch, int kv_heads, int head_dim, const int* path, const int* accepted,
                              const int* seq_pos, int n, int max_pos, hipStream_t s);
forge_status launch_attn_tree(const TreeArgs& a, hipStream_t s);
// serves every smaller max_pos too
size_t attn_tree_workspace_bytes(int batch, int q_heads, int kv_heads, int head_dim, int n, int max_pos, int cap, bool f32);

// codes <-> fp32.  The largest code of a row's type, and four codes a word.
template <forge_kv_type T> struct Codes;
template <> struct Codes<FORGE_KV_INT8> {
  static constexpr float top = 127.f;
  // of values up to 127 (1 + 2^-23) in magnitude: in x + 1.5 * 2^23 the sum is rounded to a whole number, ties to even, whose two's
  // complement is the low byte
  static __device__ inline uint32_t pack(float a, float b, float c, float d) {
    auto q = [](float x) { return __float_as_uint(x + 12582912.f); };
    const uint32_t lo = __builtin_amdgcn_perm(q(b), q(a), 0x0c0c0400), hi = __builtin_amdgcn_perm(q(d), q(c), 0x04000c0c);
    return lo | hi;
  }
  static __device__ inline void unpack(uint32_t w, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
  }
};
template <> struct Codes<FORGE_KV_FP8> {
  static constexpr float top = 448.f;
  // of values up to 448 (1 + 2^-23) in magnitude, which is rounded to 448
  static __device__ inline uint32_t pack(float a, float b, float c, float d) {
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
  }
  static __device__ inline void unpack(uint32_t w, float* f) {
    const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
  }
};

}  // namespace forge
