// Entry points of serving drafted trees: argument checks on the host, then the launches on the caller's stream.  Nothing here
// allocates, frees or synchronises.
#include <cmath>
#include "api_internal.hpp"
#include "tree.hpp"
#include "tree_checks.hpp"

using namespace forge;

namespace {

constexpr int kMaxDrafts = 64;

forge_status check_cache(const forge_kv_cache* c) {
  if (c == nullptr || !dtype_ok(c->dt) || !req(c->k) || !req(c->v) || c->k == c->v) return FORGE_ERR_INVALID_ARG;
  if (c->type != FORGE_KV_SAME && c->type != FORGE_KV_INT8 && c->type != FORGE_KV_FP8) return FORGE_ERR_INVALID_ARG;
  if (c->n_layers < 1 || c->batch < 1 || c->kv_heads < 1 || c->cap < 1) return FORGE_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return FORGE_ERR_UNSUPPORTED;
  if (c->type != FORGE_KV_SAME) {
    if (c->dt != FORGE_BF16) return FORGE_ERR_UNSUPPORTED;
    if (c->k_scale == nullptr || c->v_scale == nullptr || c->k_scale == c->v_scale || !int_ptr_ok(c->k_scale) ||
        !int_ptr_ok(c->v_scale))
      return FORGE_ERR_INVALID_ARG;
  }
  if (c->n_layers > kMaxGridDim || c->batch > kMaxGridDim || c->kv_heads > kMaxGridDim / 2) return FORGE_ERR_UNSUPPORTED;
  const int64_t head = (int64_t)c->cap * c->head_dim;
  if (c->kv_heads > 1 && (c->head_stride < head || c->head_stride % c->head_dim != 0)) return FORGE_ERR_INVALID_ARG;
  if (c->batch > 1 && (c->batch_stride < head || c->batch_stride % c->head_dim != 0)) return FORGE_ERR_INVALID_ARG;
  if (c->n_layers > 1 && (c->layer_stride < head || c->layer_stride % c->head_dim != 0)) return FORGE_ERR_INVALID_ARG;
  return FORGE_OK;
}
CacheView layer_of(const forge_kv_cache* c, int layer) {
  const int64_t es = c->type != FORGE_KV_SAME ? 1 : (int64_t)esize(c->dt);
  const int64_t e = layer > 0 ? layer * c->layer_stride : 0;
  const bool scaled = c->type != FORGE_KV_SAME;
  return {static_cast<char*>(c->k) + e * es, static_cast<char*>(c->v) + e * es,
          scaled ? c->k_scale + e / c->head_dim : nullptr, scaled ? c->v_scale + e / c->head_dim : nullptr,
          c->batch > 1 ? c->batch_stride : 0, c->kv_heads > 1 ? c->head_stride : 0};
}

// the attention's blocks, a (sequence, cache head) and 16 query rows each, rounded up to whole turns of the XCDs, are a 32-bit grid
bool tree_sizes_ok(const forge_kv_cache* c, int q_heads, int n) {
  return q_heads <= kMaxGridDim && rows_ok(c->batch, n) &&
         ((int64_t)c->batch * c->kv_heads + 8) * ceil_div(q_heads / c->kv_heads * n, 16) < ((int64_t)1 << 24);
}

forge_status check_tree(const forge_kv_cache* c, int layer, int q_heads, int n, int max_pos) {
  if (layer < 0 || layer >= c->n_layers || q_heads < 1 || q_heads % c->kv_heads != 0) return FORGE_ERR_INVALID_ARG;
  if (n > kMaxDrafts) return FORGE_ERR_UNSUPPORTED;
  if (!span_ok(max_pos, n, c->cap)) return FORGE_ERR_INVALID_ARG;
  return tree_sizes_ok(c, q_heads, n) ? FORGE_OK : FORGE_ERR_UNSUPPORTED;
}

struct TreeBlockPlan {
  size_t y, qkv, o, u, attn, gemm, total;
};
TreeBlockPlan plan_tree_block(const forge_block_desc* d, int batch, int n, int max_pos, int cap) {
  const size_t es = esize(d->dt), T = (size_t)batch * n;
  const int hd = d->q_heads * d->head_dim, nqkv = (d->q_heads + 2 * d->kv_heads) * d->head_dim, rows = (int)T;
  const bool w8 = block_w8(d);
  TreeBlockPlan p;
  p.y = align_up(T * d->d_model * es, 256);
  p.qkv = align_up(T * nqkv * es, 256);
  p.o = align_up(T * hd * es, 256);
  p.u = block_mlp_bytes(d, T);
  p.attn = align_up(attn_tree_workspace_bytes(batch, d->q_heads, d->kv_heads, d->head_dim, n, max_pos, cap, d->dt == FORGE_F32), 256);
  p.gemm = 0;
  for (size_t v : {gemm_ws(rows, nqkv, d->d_model, FORGE_ACT_NONE, d->dt, w8, true),
                   gemm_ws(rows, d->d_model, hd, FORGE_ACT_NONE, d->dt, w8),
                   gemm_ws(rows, d->d_ff, d->d_model, d->mlp_act, d->dt, w8, true),
                   gemm_ws(rows, d->d_model, d->d_ff, FORGE_ACT_NONE, d->dt, w8)})
    p.gemm = v > p.gemm ? v : p.gemm;
  p.gemm = align_up(p.gemm, 256);
  p.total = p.y + p.qkv + p.o + p.u + p.attn + p.gemm;
  return p;
}
bool fits(const forge_block_desc* d, const forge_kv_cache* c) {
  return d->dt == c->dt && d->kv_heads == c->kv_heads && d->head_dim == c->head_dim;
}

}  // namespace

extern "C" {

forge_status forge_rope_increments(double base, int rot_dim, forge_rope_scaling scaling, double by, double context,
                                   double low, double high, uint64_t* increments, float* factor) {
  if (increments == nullptr || factor == nullptr || rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 1024 ||
      !std::isfinite(base) || !(base > 1.0))
    return FORGE_ERR_INVALID_ARG;
  if (scaling < FORGE_ROPE_SCALE_NONE || scaling > FORGE_ROPE_SCALE_RAMP) return FORGE_ERR_INVALID_ARG;
  if (scaling != FORGE_ROPE_SCALE_NONE && !(std::isfinite(by) && by >= 1.0)) return FORGE_ERR_INVALID_ARG;
  if (scaling == FORGE_ROPE_SCALE_BASE && rot_dim == 2) return FORGE_ERR_INVALID_ARG;      // the exponent's pole
  const bool banded = scaling == FORGE_ROPE_SCALE_BANDS || scaling == FORGE_ROPE_SCALE_RAMP;
  if (banded && !(std::isfinite(context) && context > 0.0 && std::isfinite(high) && low > 0.0 && high > low))
    return FORGE_ERR_INVALID_ARG;
  // long double has 64 significant bits on the host: in 53 a fast pair's increment is off by some hundred units, a few 1e-7 of its angle at the last positions
  typedef long double real;
  const real turn = 6.283185307179586476925286766559L;
  real grown = base;
  if (scaling == FORGE_ROPE_SCALE_BASE) grown *= std::pow((real)by, rot_dim / (rot_dim - (real)2.0));
  if (!std::isfinite((double)grown)) return FORGE_ERR_INVALID_ARG;
  real first = 0.0, last = 1.0;
  if (scaling == FORGE_ROPE_SCALE_RAMP) {
    auto pair = [&](real turns) { return rot_dim * std::log(context / (turns * turn)) / (2 * std::log(grown)); };
    first = std::fmax((real)0.0, std::floor(pair(high)));
    last = std::fmin((real)(rot_dim - 1), std::ceil(pair(low)));
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    real theta = std::pow(grown, (real)(-2 * i) / rot_dim), g = 1.0;
    if (scaling == FORGE_ROPE_SCALE_LINEAR) g = 0.0;
    if (scaling == FORGE_ROPE_SCALE_BANDS) g = (context * theta / turn - low) / ((real)high - low);
    // (bands that coincide: a step)
    if (scaling == FORGE_ROPE_SCALE_RAMP) g = 1 - (i - first) / std::fmax((real)1e-3, last - first);
    g = std::fmin((real)1.0, std::fmax((real)0.0, g));
    if (scaling != FORGE_ROPE_SCALE_NONE && scaling != FORGE_ROPE_SCALE_BASE) theta *= g + (1 - g) / by;
    increments[i] = (uint64_t)std::rint(theta / turn * 18446744073709551616.0L);
  }
  *factor = scaling == FORGE_ROPE_SCALE_RAMP ? (float)(0.1 * std::log(by) + 1.0) : 1.0f;
  return FORGE_OK;
}

forge_status forge_rope_apply(const forge_rope_desc* rope, const forge_heads* x, const forge_heads* y,
                              const int32_t* positions, int batch, int n, int heads, int head_dim, forge_dtype dt,
                              void* stream) {
  if (!dtype_ok(dt) || batch < 1 || n < 1 || heads < 1 || head_dim < 1) return FORGE_ERR_INVALID_ARG;
  if (positions == nullptr || !int_ptr_ok(positions)) return FORGE_ERR_INVALID_ARG;
  if (!heads_ok(x, batch, n, heads, head_dim, false) || !heads_ok(y, batch, n, heads, head_dim, true))
    return FORGE_ERR_INVALID_ARG;
  const forge_status st = check_rope(rope, head_dim);
  if (st != FORGE_OK) return st;
  if (head_dim % 16 != 0 || head_dim > 1024 || !grid_ok(batch, heads) || !rows_ok(batch, n)) return FORGE_ERR_UNSUPPORTED;
  const Heads xv = view(x, batch, n, heads), yv = view(y, batch, n, heads);
  if (xv.p == yv.p && !same_view(xv, yv)) return FORGE_ERR_INVALID_ARG;
  return launch_rope_apply(turns(rope), xv, yv, positions, batch, n, heads, head_dim, dt, static_cast<hipStream_t>(stream));
}

forge_status forge_kv_append(const forge_kv_cache* cache, int layer, const forge_rope_desc* rope, const forge_heads* k,
                             const forge_heads* v, const forge_heads* q, const forge_heads* q_out, int q_heads,
                             const int32_t* seq_pos, const int32_t* positions, int n, int max_pos, void* stream) {
  forge_status st = check_cache(cache);
  if (st != FORGE_OK) return st;
  const int B = cache->batch, dh = cache->head_dim;
  if (layer < 0 || layer >= cache->n_layers || !span_ok(max_pos, n, cache->cap)) return FORGE_ERR_INVALID_ARG;
  if (!int_ptr_ok(seq_pos) || !int_ptr_ok(positions)) return FORGE_ERR_INVALID_ARG;
  if (!heads_ok(k, B, n, cache->kv_heads, dh, false) || !heads_ok(v, B, n, cache->kv_heads, dh, false))
    return FORGE_ERR_INVALID_ARG;
  if (rope != nullptr && (st = check_rope(rope, dh)) != FORGE_OK) return st;
  AppendArgs a = {};
  if (q != nullptr) {
    if (q_heads < 1 || !heads_ok(q, B, n, q_heads, dh, false) || !heads_ok(q_out, B, n, q_heads, dh, true))
      return FORGE_ERR_INVALID_ARG;
    if (q_heads > kMaxGridDim) return FORGE_ERR_UNSUPPORTED;
    a.q = view(q, B, n, q_heads);
    a.qo = view(q_out, B, n, q_heads);
    if (a.q.p == a.qo.p && !same_view(a.q, a.qo)) return FORGE_ERR_INVALID_ARG;
  }
  if (!rows_ok(B, n)) return FORGE_ERR_UNSUPPORTED;
  a.c = layer_of(cache, layer);
  a.t = turns(rope);
  a.k = view(k, B, n, cache->kv_heads);
  a.v = view(v, B, n, cache->kv_heads);
  a.batch = B;
  a.n = n;
  a.q_heads = q_heads;
  a.kv_heads = cache->kv_heads;
  a.head_dim = dh;
  a.max_pos = max_pos;
  a.seq_pos = seq_pos;
  a.positions = positions;
  a.type = cache->type;
  a.dt = cache->dt;
  return launch_kv_append(a, static_cast<hipStream_t>(stream));
}

forge_status forge_kv_read(const forge_kv_cache* cache, int layer, void* k_out, void* v_out, const int32_t* seq_pos, int n,
                           int max_pos, void* stream) {
  const forge_status st = check_cache(cache);
  if (st != FORGE_OK) return st;
  if (layer < 0 || layer >= cache->n_layers || !span_ok(max_pos, n, cache->cap) || !int_ptr_ok(seq_pos))
    return FORGE_ERR_INVALID_ARG;
  if (!req(k_out) || !req(v_out) || k_out == v_out || k_out == cache->k || k_out == cache->v || v_out == cache->k ||
      v_out == cache->v)
    return FORGE_ERR_INVALID_ARG;
  if (!rows_ok(cache->batch, n)) return FORGE_ERR_UNSUPPORTED;
  return launch_kv_read(layer_of(cache, layer), cache->type, cache->dt, cache->batch, cache->kv_heads, cache->head_dim, k_out,
                        v_out, seq_pos, n, max_pos, static_cast<hipStream_t>(stream));
}

size_t forge_attn_tree_workspace_bytes(const forge_kv_cache* cache, int q_heads, int n, int max_pos) {
  if (check_cache(cache) != FORGE_OK || check_tree(cache, 0, q_heads, n, max_pos) != FORGE_OK) return 0;
  return attn_tree_workspace_bytes(cache->batch, q_heads, cache->kv_heads, cache->head_dim, n, max_pos, cache->cap, cache->dt == FORGE_F32);
}

forge_status forge_attn_tree(const forge_kv_cache* cache, int layer, const forge_heads* q, void* out, const int32_t* seq_pos,
                             const uint64_t* visible, int q_heads, int n, int max_pos, float scale, void* workspace,
                             size_t workspace_bytes, void* stream) {
  forge_status st = check_cache(cache);
  if (st == FORGE_OK) st = check_tree(cache, layer, q_heads, n, max_pos);
  if (st != FORGE_OK) return st;
  const int B = cache->batch;
  if (!heads_ok(q, B, n, q_heads, cache->head_dim, false) || !req(out) || !opt(workspace) || !int_ptr_ok(seq_pos) ||
      !bits_ok(visible) || !scale_ok(scale))
    return FORGE_ERR_INVALID_ARG;
  if (out == q->ptr || out == cache->k || out == cache->v) return FORGE_ERR_INVALID_ARG;
  const size_t need = attn_tree_workspace_bytes(B, q_heads, cache->kv_heads, cache->head_dim, n, max_pos, cache->cap, cache->dt == FORGE_F32);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return FORGE_ERR_WORKSPACE;
  TreeArgs a = {layer_of(cache, layer), view(q, B, n, q_heads), out, seq_pos, visible, B, n, q_heads, cache->kv_heads,
                cache->head_dim, max_pos, cache->cap, scale, cache->type, cache->dt, workspace};
  return launch_attn_tree(a, static_cast<hipStream_t>(stream));
}

forge_status forge_kv_commit(const forge_kv_cache* cache, const int32_t* path, const int32_t* accepted, const int32_t* seq_pos,
                             int n, int max_pos, void* stream) {
  const forge_status st = check_cache(cache);
  if (st != FORGE_OK) return st;
  if (path == nullptr || accepted == nullptr || !int_ptr_ok(path) || !int_ptr_ok(accepted) || !int_ptr_ok(seq_pos))
    return FORGE_ERR_INVALID_ARG;
  if (n > kMaxDrafts) return FORGE_ERR_UNSUPPORTED;
  if (!span_ok(max_pos, n, cache->cap)) return FORGE_ERR_INVALID_ARG;
  return launch_kv_commit(layer_of(cache, 0), cache->type, cache->dt, cache->n_layers,
                          cache->n_layers > 1 ? cache->layer_stride : 0, cache->batch, cache->kv_heads, cache->head_dim, path,
                          accepted, seq_pos, n, max_pos, static_cast<hipStream_t>(stream));
}

size_t forge_decoder_block_tree_workspace_bytes(const forge_block_desc* desc, const forge_kv_cache* cache, int n, int max_pos) {
  if (check_block_desc(desc) != FORGE_OK || check_cache(cache) != FORGE_OK || !fits(desc, cache) ||
      check_tree(cache, 0, desc->q_heads, n, max_pos) != FORGE_OK)
    return 0;
  return plan_tree_block(desc, cache->batch, n, max_pos, cache->cap).total;
}

forge_status forge_decoder_block_tree(const forge_block_desc* desc, const forge_rope_desc* rope, const forge_kv_cache* cache,
                                      int layer, const void* x_in, void* x_out, const int32_t* seq_pos,
                                      const int32_t* positions, const uint64_t* visible, int n, int max_pos, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  forge_status st = check_block_desc(desc);
  if (st == FORGE_OK) st = check_cache(cache);
  if (st != FORGE_OK) return st;
  if (!fits(desc, cache)) return FORGE_ERR_INVALID_ARG;
  if ((st = check_tree(cache, layer, desc->q_heads, n, max_pos)) != FORGE_OK) return st;
  if ((desc->use_rope != 0) != (rope != nullptr)) return FORGE_ERR_INVALID_ARG;
  if (rope != nullptr && (st = check_rope(rope, desc->head_dim)) != FORGE_OK) return st;
  if (!req(x_in) || !req(x_out) || !req(workspace) || !int_ptr_ok(seq_pos) || !int_ptr_ok(positions) || !bits_ok(visible))
    return FORGE_ERR_INVALID_ARG;
  const int B = cache->batch, T = B * n, dm = desc->d_model, dh = desc->head_dim, hq = desc->q_heads, hkv = desc->kv_heads;
  const TreeBlockPlan pl = plan_tree_block(desc, B, n, max_pos, cache->cap);
  if (workspace_bytes < pl.total) return FORGE_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const forge_dtype dt = desc->dt;
  const int64_t es = (int64_t)esize(dt), nqkv = (int64_t)(hq + 2 * hkv) * dh;
  Carver cv(workspace);
  void* y = cv.take(pl.y);
  char* qkv = static_cast<char*>(cv.take(pl.qkv));
  void* o = cv.take(pl.o);
  void* u = cv.take(pl.u);
  void* aws = cv.take(pl.attn);
  void* gws = cv.take(pl.gemm);

  st = launch_residual_norm(x_in, nullptr, desc->norm1_g, desc->norm1_b, nullptr, y, T, dm, desc->eps, desc->norm, dt, s);
  if (st != FORGE_OK) return st;
  GemmArgs g = {y, desc->w_qkv, desc->b_qkv, nullptr, qkv, T, (int)nqkv, dm, 0, FORGE_ACT_NONE, nullptr, nullptr, gws, pl.gemm, desc->s_qkv};
  st = gemm_dispatch(g, dt, s);
  if (st != FORGE_OK) return st;
  // q, k and v where the projection left them; q is rotated in place
  auto part = [&](int head) { return Heads{qkv + (int64_t)head * dh * es, n * nqkv, nqkv, dh}; };
  AppendArgs ap = {layer_of(cache, layer), turns(rope), part(hq), part(hq + hkv), part(0), part(0), B, n, hq, hkv, dh, max_pos,
                   seq_pos, positions, cache->type, dt};
  if (rope == nullptr) ap.q.p = nullptr;
  st = launch_kv_append(ap, s);
  if (st != FORGE_OK) return st;
  TreeArgs at = {ap.c, part(0), o, seq_pos, visible, B, n, hq, hkv, dh, max_pos, cache->cap, 1.0f / sqrtf((float)dh), cache->type, dt, aws};
  st = launch_attn_tree(at, s);
  if (st != FORGE_OK) return st;
  // (decode-sized: the reduce step of the projection also produces the second norm)
  const bool norm_in_gemm = gemm_fuses_tail(T, dm, dt);
  NormTail nt = {desc->norm2_g, desc->norm2_b, y, desc->eps, desc->norm};
  g = GemmArgs{o, desc->w_o, desc->b_o, x_in, x_out, T, dm, hq * dh, 0, FORGE_ACT_NONE, nullptr,
               norm_in_gemm ? &nt : nullptr, gws, pl.gemm, desc->s_o};
  st = gemm_dispatch(g, dt, s);
  if (st != FORGE_OK) return st;
  if (!norm_in_gemm) {
    st = launch_residual_norm(x_out, nullptr, desc->norm2_g, desc->norm2_b, nullptr, y, T, dm, desc->eps, desc->norm, dt, s);
    if (st != FORGE_OK) return st;
  }
  g = GemmArgs{y, desc->w_up, desc->b_up, nullptr, u, T, desc->d_ff, dm, 0, desc->mlp_act, nullptr, nullptr, gws, pl.gemm, desc->s_up};
  st = gemm_dispatch(g, dt, s);
  if (st != FORGE_OK) return st;
  g = GemmArgs{u, desc->w_down, desc->b_down, x_out, x_out, T, dm, desc->d_ff, 0, FORGE_ACT_NONE, nullptr, nullptr, gws, pl.gemm, desc->s_down};
  return gemm_dispatch(g, dt, s);
}

}  // extern "C"
