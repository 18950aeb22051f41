// Entry points of serving many requests over one pool of cache pages: argument checks on the host, then the launches on the
// caller's stream.  Nothing here allocates, frees or synchronises.
#include "api_internal.hpp"
#include "paged.hpp"
#include "tree_checks.hpp"

using namespace forge;

namespace {

// (a slot is a 32-bit number)
bool page_rows_ok(int rows) { return rows >= 16 && rows <= 1024 && (rows & (rows - 1)) == 0; }
bool fits_32_bits(int pages, int rows) { return (int64_t)pages * rows < ((int64_t)1 << 31); }
constexpr int kMaxPages = 1 << 25;      // of a pool, of a table's row: 64 requests' sums then stay in 32 bits
int shift_of(int rows) { return __builtin_ctz((unsigned)rows); }

forge_status check_pages(const forge_paged_cache* c) {
  if (c == nullptr || !dtype_ok(c->dt) || !req(c->k) || !req(c->v) || c->k == c->v) return FORGE_ERR_INVALID_ARG;
  if (c->type != FORGE_KV_SAME && c->type != FORGE_KV_INT8 && c->type != FORGE_KV_FP8) return FORGE_ERR_INVALID_ARG;
  if (c->n_layers < 1 || c->n_pages < 1 || c->page_rows < 1 || c->kv_heads < 1) return FORGE_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return FORGE_ERR_UNSUPPORTED;
  if (!page_rows_ok(c->page_rows) || !fits_32_bits(c->n_pages, c->page_rows)) return FORGE_ERR_UNSUPPORTED;
  if (c->type != FORGE_KV_SAME) {
    if (c->dt != FORGE_BF16) return FORGE_ERR_UNSUPPORTED;
    if (c->k_scale == nullptr || c->v_scale == nullptr || c->k_scale == c->v_scale || !int_ptr_ok(c->k_scale) ||
        !int_ptr_ok(c->v_scale))
      return FORGE_ERR_INVALID_ARG;
  }
  if (c->n_layers > kMaxGridDim || c->kv_heads > kMaxGridDim / 2) return FORGE_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)c->page_rows * c->head_dim, most = (int64_t)1 << 40;
  auto apart = [&](int entries, int64_t stride) {
    return entries == 1 || (stride >= rows && stride <= most && stride % c->head_dim == 0);
  };
  if (!apart(c->kv_heads, c->head_stride) || !apart(c->n_pages, c->page_stride) || !apart(c->n_layers, c->layer_stride))
    return FORGE_ERR_INVALID_ARG;
  return FORGE_OK;
}
PagedView layer_of(const forge_paged_cache* c, int layer) {
  const bool scaled = c->type != FORGE_KV_SAME;
  const int64_t es = scaled ? 1 : (int64_t)esize(c->dt), e = layer > 0 ? layer * c->layer_stride : 0;
  const CacheView v = {static_cast<char*>(c->k) + e * es, static_cast<char*>(c->v) + e * es,
                       scaled ? c->k_scale + e / c->head_dim : nullptr, scaled ? c->v_scale + e / c->head_dim : nullptr,
                       c->n_pages > 1 ? c->page_stride : 0, c->kv_heads > 1 ? c->head_stride : 0};
  return {v, c->n_pages, shift_of(c->page_rows)};
}
bool is_cache(const forge_paged_cache* c, const void* p) { return p == c->k || p == c->v; }

// the attention's blocks, a (request, cache head) and 16 query heads each, rounded up to whole turns of the XCDs, are a 32-bit grid
forge_status check_attn(const forge_paged_cache* c, int q_heads, int batch, int max_len) {
  if (q_heads < 1 || q_heads % c->kv_heads != 0 || batch < 1 || max_len < 1) return FORGE_ERR_INVALID_ARG;
  if (q_heads > kMaxGridDim || batch > kMaxGridDim || max_len > 1 << 30 ||
      ((int64_t)batch * c->kv_heads + 8) * ceil_div(q_heads / c->kv_heads, 16) >= ((int64_t)1 << 24))
    return FORGE_ERR_UNSUPPORTED;
  return FORGE_OK;
}

forge_status check_adapters(const forge_adapters* d) {
  if (d == nullptr || !dtype_ok(d->dt) || !req(d->a) || !req(d->b) || !int_ptr_ok(d->scale)) return FORGE_ERR_INVALID_ARG;
  if (d->n_adapters < 1 || d->rank < 1 || d->K < 1 || d->N < 1 || d->n_parts < 1) return FORGE_ERR_INVALID_ARG;
  if (d->n_parts > 4 || d->rank % 8 != 0 || d->rank > 128 || d->K % (d->dt == FORGE_BF16 ? 8 : 4) != 0) return FORGE_ERR_UNSUPPORTED;
  if (d->K > kMaxRows || d->N > kMaxRows) return FORGE_ERR_UNSUPPORTED;
  int at = 0;
  for (int p = 0; p < d->n_parts; ++p) {
    if (d->part_end[p] <= at) return FORGE_ERR_INVALID_ARG;
    at = d->part_end[p];
    if (p + 1 < d->n_parts && at % 16 != 0) return FORGE_ERR_UNSUPPORTED;
  }
  return at == d->N ? FORGE_OK : FORGE_ERR_INVALID_ARG;
}

}  // namespace

extern "C" {

forge_status forge_pages_assign(const forge_page_pool* pool, const int32_t* lengths, const int32_t* change, int32_t* lengths_out,
                                int32_t* granted, int32_t* starts, int32_t* slots, int32_t* positions, int32_t* owners,
                                int max_tokens, void* stream) {
  if (pool == nullptr || pool->n_pages < 1 || pool->page_rows < 1 || pool->batch < 1 || pool->table_cols < 1 || max_tokens < 0)
    return FORGE_ERR_INVALID_ARG;
  for (const void* p : {(const void*)pool->free_pages, (const void*)pool->free_count, (const void*)pool->table, (const void*)lengths,
                        (const void*)change, (const void*)lengths_out, (const void*)granted, (const void*)starts})
    if (p == nullptr || !int_ptr_ok(p)) return FORGE_ERR_INVALID_ARG;
  for (const void* p : {slots, positions, owners})
    if ((p == nullptr && max_tokens > 0) || !int_ptr_ok(p)) return FORGE_ERR_INVALID_ARG;
  // (what is written while it is still read elsewhere)
  const void* out[] = {lengths_out, granted, starts, pool->free_pages, pool->free_count, pool->table};
  for (const void* p : out) {
    if (p == change || (p == lengths && p != lengths_out)) return FORGE_ERR_INVALID_ARG;
    for (const void* q : {(const void*)slots, (const void*)positions, (const void*)owners})
      if (max_tokens > 0 && p == q) return FORGE_ERR_INVALID_ARG;
  }
  for (int i = 0; i < 6; ++i)
    for (int j = 0; j < i; ++j)
      if (out[i] == out[j]) return FORGE_ERR_INVALID_ARG;
  if (max_tokens > 0 && (slots == positions || slots == owners || positions == owners)) return FORGE_ERR_INVALID_ARG;
  for (const void* q : {slots, positions, owners})
    if (max_tokens > 0 && (q == lengths || q == change)) return FORGE_ERR_INVALID_ARG;
  if (!page_rows_ok(pool->page_rows) || pool->batch > kMaxGridDim || max_tokens > kMaxRows || pool->n_pages > kMaxPages ||
      pool->table_cols > kMaxPages ||
      !fits_32_bits(pool->n_pages, pool->page_rows) || !fits_32_bits(pool->table_cols, pool->page_rows))
    return FORGE_ERR_UNSUPPORTED;
  const PagesArgs a = {pool->n_pages, shift_of(pool->page_rows), pool->batch, pool->table_cols, max_tokens, pool->free_pages,
                       pool->free_count, pool->table, lengths, change, lengths_out, granted, starts, slots, positions, owners};
  return launch_pages_assign(a, static_cast<hipStream_t>(stream));
}

forge_status forge_paged_append(const forge_paged_cache* cache, int layer, const forge_rope_desc* rope, const forge_heads* k,
                                const forge_heads* v, const forge_heads* q, const forge_heads* q_out, int q_heads,
                                const int32_t* slots, const int32_t* positions, int tokens, void* stream) {
  forge_status st = check_pages(cache);
  if (st != FORGE_OK) return st;
  const int dh = cache->head_dim;
  if (layer < 0 || layer >= cache->n_layers || tokens < 1) return FORGE_ERR_INVALID_ARG;
  if (slots == nullptr || !int_ptr_ok(slots) || !int_ptr_ok(positions) || (rope != nullptr && positions == nullptr))
    return FORGE_ERR_INVALID_ARG;
  if (!heads_ok(k, 1, tokens, cache->kv_heads, dh, false) || !heads_ok(v, 1, tokens, cache->kv_heads, dh, false))
    return FORGE_ERR_INVALID_ARG;
  if (rope != nullptr && (st = check_rope(rope, dh)) != FORGE_OK) return st;
  AppendArgs a = {};
  if (q != nullptr) {
    if (q_heads < 1 || !heads_ok(q, 1, tokens, q_heads, dh, false) || !heads_ok(q_out, 1, tokens, q_heads, dh, true))
      return FORGE_ERR_INVALID_ARG;
    if (q_heads > kMaxGridDim) return FORGE_ERR_UNSUPPORTED;
    a.q = view(q, 1, tokens, q_heads);
    a.qo = view(q_out, 1, tokens, q_heads);
    if ((a.q.p == a.qo.p && !same_view(a.q, a.qo)) || is_cache(cache, q_out->ptr)) return FORGE_ERR_INVALID_ARG;
  }
  if (is_cache(cache, k->ptr) || is_cache(cache, v->ptr)) return FORGE_ERR_INVALID_ARG;
  if (tokens > kMaxRows) return FORGE_ERR_UNSUPPORTED;
  const PagedView pv = layer_of(cache, layer);
  a.c = pv.c;
  a.t = turns(rope);
  a.k = view(k, 1, tokens, cache->kv_heads);
  a.v = view(v, 1, tokens, cache->kv_heads);
  a.batch = 1;
  a.n = tokens;
  a.q_heads = q_heads;
  a.kv_heads = cache->kv_heads;
  a.head_dim = dh;
  a.positions = positions;
  a.slots = slots;
  a.n_slots = cache->n_pages * cache->page_rows;
  a.shift = pv.shift;
  a.type = cache->type;
  a.dt = cache->dt;
  return launch_kv_append(a, static_cast<hipStream_t>(stream));
}

forge_status forge_paged_read(const forge_paged_cache* cache, int layer, const forge_heads* k_out, const forge_heads* v_out,
                              const int32_t* slots, int tokens, void* stream) {
  const forge_status st = check_pages(cache);
  if (st != FORGE_OK) return st;
  if (layer < 0 || layer >= cache->n_layers || tokens < 1 || slots == nullptr || !int_ptr_ok(slots)) return FORGE_ERR_INVALID_ARG;
  const int dh = cache->head_dim, heads = cache->kv_heads;
  if (!heads_ok(k_out, 1, tokens, heads, dh, true) || !heads_ok(v_out, 1, tokens, heads, dh, true)) return FORGE_ERR_INVALID_ARG;
  if (k_out->ptr == v_out->ptr || is_cache(cache, k_out->ptr) || is_cache(cache, v_out->ptr)) return FORGE_ERR_INVALID_ARG;
  if (tokens > kMaxRows) return FORGE_ERR_UNSUPPORTED;
  const PagedRows a = {layer_of(cache, layer), view(k_out, 1, tokens, heads), view(v_out, 1, tokens, heads), slots, tokens, heads, dh,
                       cache->type, cache->dt};
  return launch_paged_read(a, static_cast<hipStream_t>(stream));
}

size_t forge_attn_paged_workspace_bytes(const forge_paged_cache* cache, int q_heads, int batch, int max_len) {
  if (check_pages(cache) != FORGE_OK || check_attn(cache, q_heads, batch, max_len) != FORGE_OK) return 0;
  return attn_paged_workspace_bytes(batch, q_heads, cache->kv_heads, cache->head_dim, max_len);
}

forge_status forge_attn_paged(const forge_paged_cache* cache, int layer, const forge_heads* q, void* out, const int32_t* lengths,
                              const int32_t* table, int table_cols, int q_heads, int batch, int max_len, float scale,
                              void* workspace, size_t workspace_bytes, void* stream) {
  forge_status st = check_pages(cache);
  if (st == FORGE_OK) st = check_attn(cache, q_heads, batch, max_len);
  if (st != FORGE_OK) return st;
  if (layer < 0 || layer >= cache->n_layers || table_cols < 1 || max_len > (int64_t)table_cols * cache->page_rows)
    return FORGE_ERR_INVALID_ARG;
  if (!heads_ok(q, batch, 1, q_heads, cache->head_dim, false) || !req(out) || !opt(workspace) || !scale_ok(scale))
    return FORGE_ERR_INVALID_ARG;
  if (lengths == nullptr || table == nullptr || !int_ptr_ok(lengths) || !int_ptr_ok(table)) return FORGE_ERR_INVALID_ARG;
  if (out == q->ptr || is_cache(cache, out)) return FORGE_ERR_INVALID_ARG;
  if (!fits_32_bits(table_cols, cache->page_rows)) return FORGE_ERR_UNSUPPORTED;
  const size_t need = attn_paged_workspace_bytes(batch, q_heads, cache->kv_heads, cache->head_dim, max_len);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return FORGE_ERR_WORKSPACE;
  const PagedAttnArgs a = {layer_of(cache, layer), view(q, batch, 1, q_heads), out, lengths, table, table_cols, batch, q_heads,
                           cache->kv_heads, cache->head_dim, max_len, scale, cache->type, cache->dt, workspace};
  return launch_attn_paged(a, static_cast<hipStream_t>(stream));
}

size_t forge_adapters_workspace_bytes(const forge_adapters* d, int M) {
  if (check_adapters(d) != FORGE_OK || M < 1 || !gemm_size_ok(M, d->N)) return 0;
  return adapters_workspace_bytes(M, d->K, d->rank, d->n_parts, d->dt);
}

forge_status forge_adapters_add(const forge_adapters* d, const void* x, const void* base, void* y, const int32_t* ids, int M,
                                int ldy, void* workspace, size_t workspace_bytes, void* stream) {
  const forge_status st = check_adapters(d);
  if (st != FORGE_OK) return st;
  if (M < 1 || !req(x) || !req(base) || !req(y) || !opt(workspace) || ids == nullptr || !int_ptr_ok(ids) || x == y)
    return FORGE_ERR_INVALID_ARG;
  if (ldy != 0 && ldy < d->N) return FORGE_ERR_INVALID_ARG;
  if (!gemm_size_ok(M, d->N) || ldy > kMaxRows) return FORGE_ERR_UNSUPPORTED;
  const size_t need = adapters_workspace_bytes(M, d->K, d->rank, d->n_parts, d->dt);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return FORGE_ERR_WORKSPACE;
  const AdapterArgs a = {d->a, d->b, d->scale, x, base, y, ids, M, d->N, d->K, d->n_adapters, d->rank, d->n_parts,
                         ldy == 0 ? d->N : ldy, {d->part_end[0], d->part_end[1], d->part_end[2], d->part_end[3]}, d->dt, workspace};
  return launch_adapters(a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
