// What the operators of a paged cache and of many requests' adapters share: arguments of their launchers.  Internal to the library.
#pragma once
#include "tree.hpp"

namespace forge {

struct PagesArgs {
  int n_pages, shift, batch, cols, max_tokens;      // a page has 1 << shift rows
  int *free_pages, *free_count, *table;
  const int *lengths, *change;
  int *lengths_out, *granted, *starts, *slots, *positions, *owners;
};
forge_status launch_pages_assign(const PagesArgs& a, hipStream_t s);

// one layer of a paged cache: c.bs is the stride of a page
struct PagedView {
  CacheView c;
  int n_pages, shift;
};

struct PagedRows {
  PagedView cache;
  Heads k, v;                                       // out (a read) or in
  const int* slots;
  int tokens, kv_heads, head_dim;
  forge_kv_type type;
  forge_dtype dt;
};
forge_status launch_paged_read(const PagedRows& a, hipStream_t s);

struct PagedAttnArgs {
  PagedView cache;
  Heads q;                                          // bs: of a request, hs: of a head
  void* out;
  const int *lengths, *table;
  int table_cols, batch, q_heads, kv_heads, head_dim, max_len;
  float scale;
  forge_kv_type type;
  forge_dtype dt;
  void* workspace;
};
forge_status launch_attn_paged(const PagedAttnArgs& a, hipStream_t s);
size_t attn_paged_workspace_bytes(int batch, int q_heads, int kv_heads, int head_dim, int max_len);

struct AdapterArgs {
  const void *a, *b;
  const float* scale;
  const void *x, *base;
  void* y;
  const int* ids;
  int M, N, K, n_adapters, rank, parts, ldy;
  int part_end[4];
  forge_dtype dt;
  void* workspace;
};
forge_status launch_adapters(const AdapterArgs& a, hipStream_t s);
size_t adapters_workspace_bytes(int M, int K, int rank, int parts, forge_dtype dt);

}  // namespace forge
