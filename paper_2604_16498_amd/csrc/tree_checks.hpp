// Argument checks of strided views and rotations, shared by the entry points that take them.  Internal to the library.
#pragma once
#include <cmath>
#include "api_internal.hpp"
#include "tree.hpp"

namespace forge {

inline bool int_ptr_ok(const void* p) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool bits_ok(const void* p) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

// the strides of axes with one entry are not looked at
inline bool stride_ok(int64_t stride, int entries, int64_t least) {
  return entries == 1 || (stride >= least && stride % 8 == 0 && stride <= (int64_t)1 << 40);
}
inline bool heads_ok(const forge_heads* x, int batch, int n, int heads, int head_dim, bool written) {
  const int64_t least = written ? head_dim : 0;
  return x != nullptr && req(x->ptr) && stride_ok(x->batch_stride, batch, least) && stride_ok(x->token_stride, n, least) &&
         stride_ok(x->head_stride, heads, least);
}
inline Heads view(const forge_heads* x, int batch, int n, int heads) {
  return {static_cast<char*>(x->ptr), batch == 1 ? 0 : x->batch_stride, n == 1 ? 0 : x->token_stride,
          heads == 1 ? 0 : x->head_stride};
}
inline bool same_view(const Heads& a, const Heads& b) { return a.bs == b.bs && a.ts == b.ts && a.hs == b.hs; }

inline forge_status check_rope(const forge_rope_desc* r, int head_dim) {
  if (r == nullptr || r->increments == nullptr || (reinterpret_cast<uintptr_t>(r->increments) & 7u) != 0)
    return FORGE_ERR_INVALID_ARG;
  if (r->style != FORGE_ROPE_HALF && r->style != FORGE_ROPE_INTERLEAVED) return FORGE_ERR_INVALID_ARG;
  if (r->rot_dim < 1 || r->rot_dim > head_dim || !std::isfinite(r->factor)) return FORGE_ERR_INVALID_ARG;
  return r->rot_dim % 16 == 0 ? FORGE_OK : FORGE_ERR_UNSUPPORTED;
}
inline Turns turns(const forge_rope_desc* r) {
  if (r == nullptr) return {nullptr, 0, 0, 1.0f};
  return {r->increments, r->rot_dim, r->style == FORGE_ROPE_HALF, r->factor};
}

}  // namespace forge
