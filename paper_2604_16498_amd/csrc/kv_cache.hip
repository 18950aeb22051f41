// A cache that holds its rows in 8 bits: written with the rotation, read back, and its accepted rows moved together.
// Memory- and latency-bound; every row is touched once, in accesses of 8 and 16 bytes.  Rows of heads of 128, measured:
//   append  8192 tokens x (16 q + 32 k, v), bf16 to fp8 (169 MB): 38 to 41 us, 4.1 to 4.4 TB/s, kept as they are (201 MB) 47 us, 4.3 TB/s: latency at
//           4 waves per SIMD with two rows in flight (the vector ALU is half busy to 8 bits, 13 instructions an element);
//           24 x 13 tokens x (32 q + 16 k, v) to int8 (7 MB): 4.6 to 5.4 us, as they are 4.3
//   read    4 x 8191 rows x 16, int8 to bf16 (203 MB): 37 us, 5.5 TB/s
//   commit  8 layers x 24 sequences x 16 heads, up to 26 rows: 3.8 us; 12 x 1 x 24 of 64, up to 5: 2.0, a launch
#include "paged.hpp"
#include "rope_rows.hpp"

namespace forge {
namespace {

__device__ inline int first_row(const int* seq_pos, int b, int max_pos) {
  return seq_pos != nullptr ? min(max(seq_pos[b], 0), max_pos) : max_pos;
}

// the largest of 8 (DH 128) or 4 (DH 64) neighbouring lanes, on the vector ALU
template <int LANES>
__device__ inline uint32_t row_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));     // quad_perm:[1,0,3,2]
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));     // quad_perm:[2,3,0,1]
  if (LANES == 8) v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));   // row_half_mirror
  return v;
}

// x / scale from r = 1 / scale: the quotient by r is a few units in the last place off, a step on the exact
// remainder leaves it correctly rounded but for quotients that lie within 2^-23 units of the middle between two values; one that
// is a value itself, as the ties between codes are, comes out exactly.  Three instructions where the general division takes ten; the
// remainder needs room above the subnormals.
__device__ inline float divide(float x, float scale, float r) {
  const float q = x * r;
  return __builtin_fmaf(__builtin_fmaf(-q, scale, x), r, q);
}

// A thread per 16 elements of a token's rows and group of heads (blockIdx.y), as the rotation alone; the q heads come first, then
// those of k and v.  The row's maximum is taken over the bits of |x|: as integers they order like the values, infinities and
// NaN above all.
// PAGED: tokens go to slots of their own, one whose slot is outside the pool is left out.
template <typename T, forge_kv_type S, int DH, bool HALF, bool PAGED>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs p, uint32_t total) {
  constexpr int ITEMS = DH / 16;
  const uint32_t gid = blockIdx.x * 256u + threadIdx.x;
  if (gid >= total) return;            // (whole rows: total is a multiple of ITEMS)
  const uint32_t item = gid % ITEMS, tok = gid / ITEMS, b = tok / p.n, i = tok % p.n;
  const int nq = p.q.p != nullptr ? p.q_heads : 0, all = nq + 2 * p.kv_heads;
  const int per = ceil_div(all, gridDim.y), h0 = blockIdx.y * per, h1 = min(all, h0 + per);
  if (h0 >= h1) return;
  int64_t at_row = 0, at_scale = 0;      // of this sequence's and token's row in the first head
  Turns t = p.t;
  if (h0 >= nq + p.kv_heads) t.inc = nullptr;                 // rows of v only
  PairTurns<HALF> w(t, item, DH);
  auto source = [&](int h) {
    const Heads& x = h < nq ? p.q : h < nq + p.kv_heads ? p.k : p.v;
    const int hh = h < nq ? h : h < nq + p.kv_heads ? h - nq : h - nq - p.kv_heads;
    return reinterpret_cast<const T*>(x.p) + b * x.bs + i * x.ts + hh * x.hs;
  };
  bool live = true;                      // (the same for all lanes of a row)
  auto finish = [&](int h, float (&a)[8], float (&c)[8]) {
    if (PAGED && !live) return;
    const bool is_v = h >= nq + p.kv_heads;
    if (!is_v) w.turn(a, c);                                  // (rows of v are split as those of k: any 16 elements of the row do)
    if (h < nq) {
      T* yr = reinterpret_cast<T*>(p.qo.p) + b * p.qo.bs + i * p.qo.ts + h * p.qo.hs;
      Vec8<T>::store(yr + w.e0, a);
      Vec8<T>::store(yr + w.e1, c);
      return;
    }
    const int64_t head = (is_v ? h - nq - p.kv_heads : h - nq) * p.c.hs, e = head + at_row;
    char* cache = is_v ? p.c.v : p.c.k;
    if constexpr (S == FORGE_KV_SAME) {
      T* yr = reinterpret_cast<T*>(cache) + e;
      Vec8<T>::store(yr + w.e0, a);
      Vec8<T>::store(yr + w.e1, c);
    } else {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, max(__float_as_uint(a[j]) & 0x7fffffffu, __float_as_uint(c[j]) & 0x7fffffffu));
      m = row_max<ITEMS>(m);
      const bool finite = m < 0x7f800000u;
      float scale = divide(__uint_as_float(m), Codes<S>::top, 1.f / Codes<S>::top);      // (an infinity: NaN)
      if (scale < 1.17549435e-38f) scale = 1.f;
      if (!finite) scale = __uint_as_float(0x7fc00000u);
      float by = scale, r;
      if (__any(!finite || scale < 1e-30f)) {                 // (rare)
        const float k = !finite ? 0.f : scale < 1e-30f ? 18446744073709551616.f : 1.f;       // room below, by a power of two
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          a[j] = finite ? a[j] * k : 0.f;
          c[j] = finite ? c[j] * k : 0.f;
        }
        by = finite ? scale * k : 1.f;
      }
      r = __builtin_amdgcn_rcpf(by);
      r = __builtin_fmaf(__builtin_fmaf(-by, r, 1.f), r, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        a[j] = divide(a[j], by, r);
        c[j] = divide(c[j], by, r);
      }
      const u32x2 lo = {Codes<S>::pack(a[0], a[1], a[2], a[3]), Codes<S>::pack(a[4], a[5], a[6], a[7])};
      const u32x2 hi = {Codes<S>::pack(c[0], c[1], c[2], c[3]), Codes<S>::pack(c[4], c[5], c[6], c[7])};
      *reinterpret_cast<u32x2*>(cache + e + w.e0) = lo;
      *reinterpret_cast<u32x2*>(cache + e + w.e1) = hi;
      if (item == 0) (is_v ? p.c.vs : p.c.ks)[head / DH + at_scale] = scale;
    }
  };
  walk_heads<T>(h0, h1, w.e0, w.e1, source, [&] {
    if constexpr (PAGED) {
      const int slot = p.slots[tok];
      live = (uint32_t)slot < (uint32_t)p.n_slots;
      at_row = (slot >> p.shift) * p.c.bs + (int64_t)(slot & ((1 << p.shift) - 1)) * DH;
      at_scale = at_row / DH;
      w.at(t, p.positions != nullptr ? p.positions[tok] : 0);       // (none: no rotation)
    } else {
      const int row = first_row(p.seq_pos, b, p.max_pos) + i;
      at_row = b * p.c.bs + (int64_t)row * DH;
      at_scale = at_row / DH;
      w.at(t, p.positions != nullptr ? p.positions[tok] : row);
    }
  }, finish);
}

// Rows back as values: a thread per 8 elements; grid (rows of one head in blocks, heads of k and v, batch)
template <typename T, forge_kv_type S, int DH>
__global__ __launch_bounds__(256) void kv_read_kernel(CacheView c, T* k_out, T* v_out, int kv_heads, const int* seq_pos, int n,
                                                      int max_pos) {
  const int h = blockIdx.y >> 1, b = blockIdx.z;
  const bool is_v = blockIdx.y & 1;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;         // 8 elements of this head's rows
  if (at >= (int64_t)n * (DH / 8)) return;
  const int row = first_row(seq_pos, b, max_pos);
  const int64_t e = b * c.bs + h * c.hs + (int64_t)row * DH + at * 8;
  float x[8];
  if constexpr (S == FORGE_KV_SAME) {
    Vec8<T>::load(reinterpret_cast<const T*>(is_v ? c.v : c.k) + e, x);
  } else {
    const u32x2 w = *reinterpret_cast<const u32x2*>((is_v ? c.v : c.k) + e);
    const float scale = (is_v ? c.vs : c.ks)[e / DH];
    Codes<S>::unpack(w[0], x);
    Codes<S>::unpack(w[1], x + 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= scale;
  }
  Vec8<T>::store((is_v ? v_out : k_out) + ((int64_t)b * kv_heads + h) * n * DH + at * 8, x);
}

// Rows of any slots: a thread per 8 elements of k and v of two tokens, so that stores are whole lines; grid (tokens in blocks, heads).  30011 rows of 8
// heads of 128, int8 (186 MB): 34.3 us, 5.4 TB/s; the rows through the caches 36.6, a thread per 16 elements of one token, half lines a store, 40.8.
// Stores past the caches too take 28.0, but what reads the rows next then takes longer than they save: 30000 rows and the attention of 256 tokens over
// them 175 | 181 us, 8000 rows 63 | 64.
template <typename T, forge_kv_type S, int DH>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedRows p) {
  constexpr int ITEMS = DH / 8, ROWS = 256 / ITEMS;
  const int h = blockIdx.y, d = threadIdx.x % ITEMS * 8, shift = p.cache.shift;
  const CacheView& c = p.cache.c;
  int64_t e[2];
  int tok[2];
  bool live[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    tok[i] = blockIdx.x * (2 * ROWS) + i * ROWS + threadIdx.x / ITEMS;
    const int slot = tok[i] < p.tokens ? p.slots[tok[i]] : -1;
    live[i] = (uint32_t)slot < (uint32_t)p.cache.n_pages << shift;
    e[i] = live[i] ? (slot >> shift) * c.bs + h * c.hs + (int64_t)(slot & ((1 << shift) - 1)) * DH + d : 0;
  }
  if constexpr (S == FORGE_KV_SAME) {
    constexpr int N = sizeof(T) / 2;       // 16-byte words of 8 elements
    u32x4 k[2][N], v[2][N];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int w = 0; w < N; ++w) {
        k[i][w] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(reinterpret_cast<const T*>(c.k) + e[i]) + w);
        v[i][w] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(reinterpret_cast<const T*>(c.v) + e[i]) + w);
      }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!live[i]) continue;
#pragma unroll
      for (int w = 0; w < N; ++w) {
        reinterpret_cast<u32x4*>(reinterpret_cast<T*>(p.k.p) + tok[i] * p.k.ts + h * p.k.hs + d)[w] = k[i][w];
        reinterpret_cast<u32x4*>(reinterpret_cast<T*>(p.v.p) + tok[i] * p.v.ts + h * p.v.hs + d)[w] = v[i][w];
      }
    }
  } else {
    u32x2 k[2], v[2];
    float ks[2], vs[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(c.k + e[i]));
      v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(c.v + e[i]));
      ks[i] = c.ks[e[i] / DH];
      vs[i] = c.vs[e[i] / DH];
    }
    auto put = [](T* y, const u32x2& w, float scale) {
      float x[8];
      Codes<S>::unpack(w[0], x);
      Codes<S>::unpack(w[1], x + 4);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= scale;
      Vec8<T>::store(y, x);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!live[i]) continue;
      put(reinterpret_cast<T*>(p.k.p) + tok[i] * p.k.ts + h * p.k.hs + d, k[i], ks[i]);
      put(reinterpret_cast<T*>(p.v.p) + tok[i] * p.v.ts + h * p.v.hs + d, v[i], vs[i]);
    }
  }
}

// A wave per (layer, sequence, head, k or v) walks over the accepted rows in rising order, ROWS of them at a time.  In place: a
// row's source lies at or behind it, so a store never reaches a row that is still to be read (a group's loads return
// before its stores go out, and the groups follow one another).
template <int ROW_BYTES>
__global__ __launch_bounds__(64) void kv_commit_kernel(CacheView c, int64_t layer_bytes, int64_t layer_rows, int64_t bs_bytes,
                                                       int64_t hs_bytes, int64_t bs_rows, int64_t hs_rows, int kv_heads,
                                                       const int* path, const int* accepted, const int* seq_pos, int n,
                                                       int max_pos) {
  constexpr int LANES = ROW_BYTES / 16, ROWS = 64 / LANES;
  const int h = blockIdx.x >> 1, b = blockIdx.y, lane = threadIdx.x;
  const bool is_v = blockIdx.x & 1;
  const int take = min(max(accepted[b], 0), n), pos = first_row(seq_pos, b, max_pos);
  char* rows = (is_v ? c.v : c.k) + blockIdx.z * layer_bytes + b * bs_bytes + h * hs_bytes + (int64_t)pos * ROW_BYTES;
  float* scales = is_v ? c.vs : c.ks;
  if (scales != nullptr) scales += blockIdx.z * layer_rows + b * bs_rows + h * hs_rows + pos;
  const int mine = min(max(lane < n ? path[(int64_t)b * n + lane] : 0, 0), n - 1);      // n <= 64: an entry a lane
  for (int j0 = 0; j0 < take; j0 += ROWS) {
    const int j = j0 + lane / LANES, from = __shfl(mine, j & 63, 64);
    if (j >= take || from == j) continue;
    const u32x4 x = *reinterpret_cast<const u32x4*>(rows + (int64_t)from * ROW_BYTES + lane % LANES * 16);
    float s = 0.f;
    if (scales != nullptr && lane % LANES == 0) s = scales[from];
    *reinterpret_cast<u32x4*>(rows + (int64_t)j * ROW_BYTES + lane % LANES * 16) = x;
    if (scales != nullptr && lane % LANES == 0) scales[j] = s;
  }
}

template <typename T, forge_kv_type S>
void append_dh(const AppendArgs& a, const dim3& grid, uint32_t total, hipStream_t s) {
  auto go = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(a, total); };
  if (a.slots != nullptr) {
    if (a.head_dim == 64) a.t.half ? go(kv_append_kernel<T, S, 64, true, true>) : go(kv_append_kernel<T, S, 64, false, true>);
    else a.t.half ? go(kv_append_kernel<T, S, 128, true, true>) : go(kv_append_kernel<T, S, 128, false, true>);
    return;
  }
  if (a.head_dim == 64) a.t.half ? go(kv_append_kernel<T, S, 64, true, false>) : go(kv_append_kernel<T, S, 64, false, false>);
  else a.t.half ? go(kv_append_kernel<T, S, 128, true, false>) : go(kv_append_kernel<T, S, 128, false, false>);
}

template <typename T, forge_kv_type S>
void read_dh(const CacheView& c, int batch, int kv_heads, int head_dim, void* k_out, void* v_out, const int* seq_pos, int n,
             int max_pos, hipStream_t s) {
  const dim3 grid((unsigned)ceil_div64((int64_t)n * (head_dim / 8), 256), 2 * kv_heads, batch);
  if (head_dim == 64) kv_read_kernel<T, S, 64><<<grid, 256, 0, s>>>(c, (T*)k_out, (T*)v_out, kv_heads, seq_pos, n, max_pos);
  else kv_read_kernel<T, S, 128><<<grid, 256, 0, s>>>(c, (T*)k_out, (T*)v_out, kv_heads, seq_pos, n, max_pos);
}

template <typename T, forge_kv_type S>
void paged_read_dh(const PagedRows& a, hipStream_t s) {
  const dim3 grid((unsigned)ceil_div64((int64_t)a.tokens * (a.head_dim / 8), 512), a.kv_heads);
  if (a.head_dim == 64) paged_read_kernel<T, S, 64><<<grid, 256, 0, s>>>(a);
  else paged_read_kernel<T, S, 128><<<grid, 256, 0, s>>>(a);
}

}  // namespace

forge_status launch_kv_append(const AppendArgs& a, hipStream_t s) {
  const int heads = (a.q.p != nullptr ? a.q_heads : 0) + 2 * a.kv_heads;
  const int64_t total = (int64_t)a.batch * a.n * (a.head_dim / 16);
  const unsigned blocks = (unsigned)ceil_div64(total, 256);
  const dim3 grid(blocks, row_head_groups(blocks, heads));
  if (a.dt == FORGE_F32) append_dh<float, FORGE_KV_SAME>(a, grid, (uint32_t)total, s);
  else if (a.type == FORGE_KV_SAME) append_dh<bf16, FORGE_KV_SAME>(a, grid, (uint32_t)total, s);
  else if (a.type == FORGE_KV_INT8) append_dh<bf16, FORGE_KV_INT8>(a, grid, (uint32_t)total, s);
  else append_dh<bf16, FORGE_KV_FP8>(a, grid, (uint32_t)total, s);
  return launch_status();
}

forge_status launch_kv_read(const CacheView& c, forge_kv_type type, forge_dtype dt, int batch, int kv_heads, int head_dim,
                            void* k_out, void* v_out, const int* seq_pos, int n, int max_pos, hipStream_t s) {
  if (dt == FORGE_F32) read_dh<float, FORGE_KV_SAME>(c, batch, kv_heads, head_dim, k_out, v_out, seq_pos, n, max_pos, s);
  else if (type == FORGE_KV_SAME) read_dh<bf16, FORGE_KV_SAME>(c, batch, kv_heads, head_dim, k_out, v_out, seq_pos, n, max_pos, s);
  else if (type == FORGE_KV_INT8) read_dh<bf16, FORGE_KV_INT8>(c, batch, kv_heads, head_dim, k_out, v_out, seq_pos, n, max_pos, s);
  else read_dh<bf16, FORGE_KV_FP8>(c, batch, kv_heads, head_dim, k_out, v_out, seq_pos, n, max_pos, s);
  return launch_status();
}

forge_status launch_paged_read(const PagedRows& a, hipStream_t s) {
  if (a.dt == FORGE_F32) paged_read_dh<float, FORGE_KV_SAME>(a, s);
  else if (a.type == FORGE_KV_SAME) paged_read_dh<bf16, FORGE_KV_SAME>(a, s);
  else if (a.type == FORGE_KV_INT8) paged_read_dh<bf16, FORGE_KV_INT8>(a, s);
  else paged_read_dh<bf16, FORGE_KV_FP8>(a, s);
  return launch_status();
}

forge_status launch_kv_commit(const CacheView& c, forge_kv_type type, forge_dtype dt, int n_layers, int64_t layer_stride,
                              int batch, int kv_heads, int head_dim, const int* path, const int* accepted,
                              const int* seq_pos, int n, int max_pos, hipStream_t s) {
  const int es = type != FORGE_KV_SAME ? 1 : dt == FORGE_BF16 ? 2 : 4, row_bytes = head_dim * es;
  const dim3 grid(2 * kv_heads, batch, n_layers);
  const int64_t bs_rows = c.bs / head_dim, hs_rows = c.hs / head_dim, layer_rows = layer_stride / head_dim;
  auto go = [&](auto kernel) {
    kernel<<<grid, 64, 0, s>>>(c, layer_stride * es, layer_rows, c.bs * es, c.hs * es, bs_rows, hs_rows, kv_heads, path,
                               accepted, seq_pos, n, max_pos);
  };
  switch (row_bytes) {
    case 64: go(kv_commit_kernel<64>); break;
    case 128: go(kv_commit_kernel<128>); break;
    case 256: go(kv_commit_kernel<256>); break;
    case 512: go(kv_commit_kernel<512>); break;
    default: return FORGE_ERR_UNSUPPORTED;
  }
  return launch_status();
}

}  // namespace forge
