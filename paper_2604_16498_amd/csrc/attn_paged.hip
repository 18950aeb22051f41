// Attention of one new token per request over a cache in pages, in 16 or 32 bits, int8 or fp8.
//
// One pass over a pair's (request, cache head) rows with the running maximum and sum of the softmax:
//   s_j = scale q . k_j,  m = max s_j,  l = sum exp(s_j - m),  o = sum exp(s_j - m) v_j / l
// A block of 4 waves takes the 16 query heads (or fewer) of a cache head as the columns of one matrix operand, and its waves take the 32-row tiles of
// its range of rows in turn; the tile layouts, the products and the dealing of rows over blocks are those of the attention of drafted trees.
// Up to 8 query heads a cache head: the 16 columns hold each twice, and the second takes what the weights of the first lose in bf16, so that they count with
// 16 bits, for no further product (from 9 heads on they are rounded to bf16, 2^-9 each, as there).
// A weight is positive, however far its row lies below the maximum: an infinity in that row of v counts.  So weights, the running rescaling and the
// waves' and shares' parts do not become 0 where fp32 would round them to it; what that adds to a finite sum is 2^-133 of its rows of v.
// What is its own is where a tile lies: in two halves of 16 rows, each inside a page, whose numbers a wave keeps in a
// register, an entry a lane, for its next 32 tiles; a half's address is then scalar arithmetic.  Rows are asked for past the caches: up to 16 query heads a cache
// head they are read once.  (With more each block of 16 reads them, those of a share beside one another on one XCD; 40 over 1 of 128, 16 up to 8192 rows,
// bf16, 42 MB: 26.3 us, 1.6 TB/s.)
// Measured, 32 heads over 8 of 128: 64 requests up to 2049 rows, int8 (164 MB) 33.5 us, 4.9 TB/s (rows through the caches 37.0), two blocks a CU of uneven
// lengths; 7 up to 30011 rows, bf16 (430 MB) 67 to 69 us, 6.2 to 6.4 TB/s, and 4.6 for the merge (through the caches 77).  One of 334 rows of 12 heads of
// 64: 6.0 us, 5.2 in a graph, a chain of loads (length, pages, three tiles).  fp32, 12 heads of 64, 8 up to 1000 rows (31 MB) 16.4 us: in fp32 the cut's
// speeds are those of the drafted trees' kernel, not fitted here, and heads of 128 hold 134 KB of LDS, one block a CU where the cut counts on two.
// max_len far above the lengths, as a recorded step has it (the cut is then made for that): 64 up to 2048 rows, bf16, max_len 2048 54.6, 32768 55.1,
// 131072 60.0; int8 33.3, 36.6, 36.9; 64 up to 300 rows, int8, 300 11.5, 4096 11.8, 32768 14.6; 8 up to 4096, bf16, 4096 to 131072 20.2 to 21.0; one of 334
// 5.1, from 4096 on 7.9 (the merge's launch).
// Registers: 162 for 8-bit and 216 for 16-bit heads of 128, 117 to 140 for heads of 64; fp32 162, 251 and 40 accumulation registers.  Up to 9 scalar ones of
// the 8-bit kernels are spilled into vector registers, no others.
#include "cache_tiles.hpp"
#include "paged.hpp"
#include "paged_plan.hpp"

namespace forge {
namespace {

constexpr float LEAST = 9.183549615799121e-41f;      // 2^-133, the smallest positive number in bf16

struct PagedParams {
  CacheView c;             // bs: of a page
  Heads q;
  char* out;
  float* part;             // [shares, row_blocks, 2, 16, DH] unnormalised outputs, then [.., 2] (maximum, sum)
  float* stat;
  const int *lengths, *table;
  int table_cols, n_pages, shift;
  int batch, q_heads, kv_heads, group, n, rows, max_len;      // rows = group, n = 1
  int shares, dealt, by_length, row_blocks;
  float scale_log2e;
};

// The row of the new token, -1 where there is none
__device__ inline int position_of(const PagedParams& p, int b) { return min(max(p.lengths[b], 0), p.max_len) - 1; }
__device__ inline int units_of(const PagedParams&, int pos) { return (pos + UNIT) / UNIT; }
__device__ inline int next_sequence(const PagedParams& p, int& b) {
  for (++b;; b += 64) {                  // (a share with rows left has them in a later request)
    const int at = b + (int)(threadIdx.x & 63), pos = at < p.batch ? position_of(p, at) : -1;
    const uint64_t some = __ballot(pos >= 0);
    if (some == 0 && b + 64 < p.batch) continue;
    const int j = some != 0 ? __ffsll((unsigned long long)some) - 1 : 0;
    b = min(b + j, p.batch - 1);
    return __builtin_amdgcn_readlane(pos, j);
  }
}

// EACH: pairs are not cut, and every wave takes one by itself; nothing is added up between waves.
template <forge_kv_type S, typename T, int DH, bool EACH>
__global__ __launch_bounds__(NW * 64, sizeof(T) == 2 && (S != FORGE_KV_SAME || DH == 64) ? 3 : 2) void attn_paged_kernel(PagedParams p) {
  typedef Store<S, T> St;
  constexpr int BYTES = St::BYTES;
  constexpr bool F32 = sizeof(T) == 4, SCALED = S != FORGE_KV_SAME;
  constexpr int NJ = F32 ? DH / 4 : DH / 32;       // MFMAs of a score tile
  constexpr int NM = DH / 16;                      // 16-column tiles of the output
  constexpr int NQ = F32 ? DH / 16 : DH / 32;
  typedef Raw<BYTES, DH> R;
  typedef Patch<BYTES, DH> L;
  constexpr int PAD = DH + 4;
  constexpr int WAVE_LDS = L::BYTES_ALL > 16 * PAD * 4 ? L::BYTES_ALL : 16 * PAD * 4;
  __shared__ __attribute__((aligned(16))) char patch[NW][WAVE_LDS];      // the tile, and at the end 16 rows of the wave's outputs
  __shared__ float sml[NW][16][2];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  constexpr int SIDE = EACH ? 1 : NW;                          // waves side by side in a range of rows
  const int beside = EACH ? 0 : wave;
  Share<PagedParams> share;
  if (!share.start(p, EACH ? NW : 1, EACH ? wave : 0)) return;
  const int c = lane & 15, kg = lane >> 4;
  const bool twice = !F32 && p.rows <= 8;
  const int column = twice ? c & 7 : c;                        // the query head of this lane, counted in its block
  const uint32_t second = twice && c >= 8 ? ~0u : 0u;          // this lane's column holds what the weights lose
  char* const lds = patch[wave];
  const int in_page = (1 << p.shift) - 1;

  // ---- what a piece needs first, requested before its request's length has to be known -----------------------
  int64_t head;                                                // elements
  int begin = 0;
  int pages;                                                   // of half l % 2 of this wave's tile l / 2 of the next 32
  u32x4 qf[NQ];                                                // query head of this lane's column
  u32x4 rk[L::LOADS], rv[L::LOADS];                            // the tile in flight
  float rs = 0.f;
  auto tile_base = [&](int t) { return begin + (t * SIDE + beside) * TILE; };
  auto load_pages = [&](int b, int t0) {
    const uint32_t row = (uint32_t)tile_base(t0) + (uint32_t)(lane >> 1) * (SIDE * TILE) + 16 * (lane & 1);
    const uint32_t col = min(row >> p.shift, (uint32_t)p.table_cols - 1);
    pages = min(max(p.table[(int64_t)b * p.table_cols + col], 0), p.n_pages - 1);
  };
  // wanted: a tile of this wave's; otherwise the loads, which stay so that their number is known, ask for little.
  // (scheduled among its neighbours, a tile's loads go to second registers, and the copies back wait for them)
  auto load_tile = [&](int t, bool wanted) {
    __builtin_amdgcn_sched_barrier(0);
    const int base = tile_base(t), l = lane & (wanted ? -1 : 0);
    int64_t e[2];
#pragma unroll
    for (int f = 0; f < 2; ++f)
      e[f] = head + __builtin_amdgcn_readlane(pages, 2 * (t & 31) + f) * p.c.bs + (int64_t)((base + 16 * f) & in_page) * DH;
    auto piece = [&](const char* from, int i) {
      constexpr int HALF = 16 / L::PER;
      return from + e[i / HALF] * BYTES + i % HALF * 1024 + l * 16;
    };
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) rk[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(piece(p.c.k, i)));
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) rv[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(piece(p.c.v, i)));
    if constexpr (SCALED) rs = (lane < TILE ? p.c.ks : p.c.vs)[e[(lane >> 4) & 1] / DH + (l & 15)];
    __builtin_amdgcn_sched_barrier(0);
  };
  auto request = [&](int b, int g, int from) {
    head = g * p.c.hs;
    begin = from;
    load_pages(b, 0);
    const int row = share.rb * 16 + column;
    const T* qr = reinterpret_cast<const T*>(p.q.p) + b * p.q.bs + (g * p.group + (row < p.rows ? row : 0)) * p.q.hs;
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      u32x4 x = {0, 0, 0, 0};
      if constexpr (F32) { if (row < p.rows) x = *reinterpret_cast<const u32x4*>(qr + 16 * j + 4 * kg); }
      else { if (row < p.rows) x = *reinterpret_cast<const u32x4*>(qr + St::q_at(j, kg)); }
      qf[j] = x;
    }
    load_tile(0, tile_base(0) < p.max_len);
  };
  const int piece_row = lane / (L::ROW / 16), piece_at = lane % (L::ROW / 16) * 16;
  const int k_put = L::k_slot(piece_row) * L::STRIDE + piece_at, v_put = TILE * L::STRIDE + piece_row * L::STRIDE + piece_at;
  bool odd_scale = false;                  // a row of the tile has a scale of v that is not finite
  // behind: rows from this one of the tile on are not the request's: their weights are 0, and their V is cleared (0 * infinity would be NaN)
  auto put_tile = [&](int behind) {
    wave_lds_sync();                       // the tile before has been read
    if (S != FORGE_KV_INT8 && behind < TILE) {
#pragma unroll
      for (int i = 0; i < L::LOADS; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) rv[i][w] = i * L::PER + piece_row < behind ? rv[i][w] : 0u;
    }
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i)     // (k_slot is a permutation of bits: of a sum without carries the sum)
      *reinterpret_cast<u32x4*>(lds + k_put + L::k_slot(i * L::PER) * L::STRIDE) = rk[i];
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) *reinterpret_cast<u32x4*>(lds + v_put + i * L::PER * L::STRIDE) = rv[i];
    if constexpr (SCALED) {
      *reinterpret_cast<float*>(lds + L::SCALES + lane * 4) = rs;
      odd_scale = __any(lane >= TILE && !(fabsf(rs) < INFINITY));
    }
    wave_lds_sync();
  };
  request(share.b, share.g, share.unit * UNIT);

  for (;;) {
  const Piece at = share.next(p);
  const int len = at.pos + 1, stop = at.stop;
  const int ntile = stop > begin + beside * TILE ? ceil_div(stop - begin - beside * TILE, SIDE * TILE) : 0;
  float m_run = -FLT_MAX, l_run = 0.f;
  floatx4 acc[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) acc[m] = floatx4{0.f, 0.f, 0.f, 0.f};

  auto step = [&](int t) {
    R r;
    float ksr[8], vsr[8];
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int j = 0; j < R::KL; ++j)
        r.k[f][j] = *reinterpret_cast<const u32x4*>(lds + (16 * f + c) * L::STRIDE + 16 * kg + 64 * j);
    if constexpr (SCALED) {
      const float* sc = reinterpret_cast<const float*>(lds + L::SCALES) + 8 * kg;
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const floatx4 a = *reinterpret_cast<const floatx4*>(sc + i), b = *reinterpret_cast<const floatx4*>(sc + TILE + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) { ksr[i + e] = a[e]; vsr[i + e] = b[e]; }
      }
    }
    const int base = tile_base(t), mine = len - base - 8 * kg;      // of this lane's 8 cache rows the first `mine` are the request's
    const bool edge = base + TILE > len;
    // ---- scores --------------------------------------------------------------------------------------
    float s[8];
    {
      floatx4 sa[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if constexpr (F32)
            sa[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(r.k[f][j / 4][j & 3]), __uint_as_float(qf[j / 4][j & 3]), sa[f], 0, 0, 0);
          else
            sa[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(St::k(r, f, j), __builtin_bit_cast(bf16x8, qf[j]), sa[f], 0, 0, 0);
        }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[e] = sa[e >> 2][e & 3] * p.scale_log2e;
        if constexpr (SCALED) s[e] *= ksr[e];
      }
    }
    if (edge) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = e < mine ? s[e] : -INFINITY;
    }
    // ---- softmax -------------------------------------------------------------------------------------
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[e]);
    if (__any(mx > m_run + 8.f)) {                       // (wave-uniform)
      const float m_new = fmaxf(m_run, lanes_max(mx));
      const float alpha = share_weight(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int m = 0; m < NM; ++m) acc[m] *= alpha;
    }
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(s[e] - m_run);
    bool tiny = odd_scale;                               // (8-bit rows have an infinity by their scale alone, one a lane)
    if constexpr (!SCALED) {
      uint32_t least = __float_as_uint(w[0]);            // (as integers they order like the values, NaN above all)
#pragma unroll
      for (int e = 1; e < 8; ++e) least = min(least, __float_as_uint(w[e]));
      tiny = __any(least < 0x00800000u);
    }
    if (tiny) {                                          // (rare)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = s[e] > -INFINITY ? fmaxf(w[e], LEAST) : w[e];       // (NaN stays)
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      l_run += w[e];
      s[e] = SCALED ? w[e] * vsr[e] : w[e];
    }
    if (SCALED && edge) {                                // (a row behind the length may have any scale)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = e < mine ? s[e] : 0.f;
    }
    // ---- P . V ---------------------------------------------------------------------------------------
#pragma unroll
    for (int i = 0; i < 8; ++i) load_words<R::VW>(lds + (TILE + 8 * kg + i) * L::STRIDE + c * (R::VW * 4), r.v[i]);
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int m = 0; m < NM; ++m) acc[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(r.v[e][m]), s[e], acc[m], 0, 0, 0);
    } else {
      u32x4 words;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t hi = pack_bf2(s[2 * e], s[2 * e + 1]) & second;      // (masked: an infinite weight times 0 would be NaN)
        words[e] = pack_bf2(s[2 * e] - bf_lo(hi), s[2 * e + 1] - bf_hi(hi));
      }
      const bf16x8 pf = __builtin_bit_cast(bf16x8, words);
#pragma unroll
      for (int m = 0; m < NM; ++m)
        acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, St::v(r, m)), pf, acc[m], 0, 0, 0);
    }
  };

  for (int t = 0; t < ntile; ++t) {
    put_tile(len - tile_base(t));
    if (((t + 1) & 31) == 0) load_pages(at.b, t + 1);
    load_tile(t + 1, t + 1 < ntile);
    step(t);
  }
  const bool more = share.left > 0;
  if (more) request(share.b, share.g, 0);      // (on its way while this piece is finished)
  // ---- the waves' shares, added in wave order ----------------------------------------------------------------
  const int64_t slot = slot_of(p, share.i, share.rb, max(at.which, 0), 16);
  const float l = lanes_sum(l_run);
  wave_lds_sync();
#pragma unroll
  for (int v = 0; v < 4; ++v)
#pragma unroll
    for (int m = 0; m < NM; m += 4)
      *reinterpret_cast<floatx4*>(lds + c * (PAD * 4) + ((4 * kg + v) * NM + m) * 4) = floatx4{acc[m][v], acc[m + 1][v], acc[m + 2][v], acc[m + 3][v]};
  if (kg == 0) { sml[wave][c][0] = m_run; sml[wave][c][1] = l; }
  if constexpr (EACH) wave_lds_sync();
  else lds_barrier();
  for (int idx = EACH ? lane : tid; idx < 16 * (DH / 4); idx += SIDE * 64) {
    const int r = idx / (DH / 4), d = idx % (DH / 4) * 4, row = share.rb * 16 + r;
    if (row >= p.rows) continue;           // (so r < 8 where heads are there twice)
    const int w0 = EACH ? wave : 0;
    float mn = sml[w0][r][0];
#pragma unroll
    for (int w = 1; w < SIDE; ++w) mn = fmaxf(mn, sml[w][r][0]);
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    float lt = 0.f;
#pragma unroll
    for (int w = w0; w < w0 + SIDE; ++w) {
      const float a = share_weight(sml[w][r][0] - mn);
      floatx4 x = *reinterpret_cast<const floatx4*>(patch[w] + r * (PAD * 4) + d * 4);
      if (twice) {                         // (where a row has an infinity, the first part says which)
        const floatx4 y = *reinterpret_cast<const floatx4*>(patch[w] + (r + 8) * (PAD * 4) + d * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += fabsf(x[i]) < INFINITY ? y[i] : 0.f;
      }
      o += x * a;
      lt += sml[w][r][1] * a;
    }
    if (at.which < 0) {
      store4<T>(out_row<T>(p, at.b, at.g, row, DH) + d, o * (lt == 0.f ? 0.f : 1.f / lt));
    } else {
      *reinterpret_cast<floatx4*>(p.part + (slot + r) * DH + d) = o;
      if (d == 0) { p.stat[(slot + r) * 2] = mn; p.stat[(slot + r) * 2 + 1] = lt; }
    }
  }
  if (!more) break;
  if constexpr (!EACH) lds_barrier();
  }
}

template <forge_kv_type S, typename T>
void launch_dh(const PagedParams& p, unsigned blocks, bool each, int head_dim, hipStream_t s) {
  if (head_dim == 64) {
    if (each) attn_paged_kernel<S, T, 64, true><<<blocks, NW * 64, 0, s>>>(p);
    else attn_paged_kernel<S, T, 64, false><<<blocks, NW * 64, 0, s>>>(p);
  } else {
    if (each) attn_paged_kernel<S, T, 128, true><<<blocks, NW * 64, 0, s>>>(p);
    else attn_paged_kernel<S, T, 128, false><<<blocks, NW * 64, 0, s>>>(p);
  }
}
template <typename T>
void launch_merge(const PagedParams& p, int head_dim, hipStream_t s) {
  const int pairs = p.batch * p.kv_heads;
  const bool split = p.shares > 4 * pairs && (int64_t)p.rows * pairs <= 8 * compute_units();      // (as in the attention of drafted trees)
  const dim3 grid(split ? p.rows : ceil_div(p.rows, head_dim == 64 ? 16 : 8), pairs);
  if (head_dim == 64) split ? attn_merge_kernel<T, 64, true><<<grid, 256, 0, s>>>(p, 16) : attn_merge_kernel<T, 64, false><<<grid, 256, 0, s>>>(p, 16);
  else split ? attn_merge_kernel<T, 128, true><<<grid, 256, 0, s>>>(p, 16) : attn_merge_kernel<T, 128, false><<<grid, 256, 0, s>>>(p, 16);
}

}  // namespace

size_t attn_paged_workspace_bytes(int batch, int q_heads, int kv_heads, int head_dim, int max_len) {
  return paged_room(batch, q_heads, kv_heads, head_dim, max_len, compute_units());
}

forge_status launch_attn_paged(const PagedAttnArgs& a, hipStream_t s) {
  const bool f32 = a.dt == FORGE_F32;
  const int group = a.q_heads / a.kv_heads, cus = compute_units();
  const TreePlan pl = plan_paged(a.batch, a.q_heads, a.kv_heads, a.head_dim, a.max_len, a.type != FORGE_KV_SAME ? 1 : f32 ? 4 : 2, cus);
  PagedParams p;
  p.c = a.cache.c;
  p.q = a.q;
  p.out = (char*)a.out;
  p.lengths = a.lengths;
  p.table = a.table;
  p.table_cols = a.table_cols;
  p.n_pages = a.cache.n_pages;
  p.shift = a.cache.shift;
  p.batch = a.batch;
  p.q_heads = a.q_heads;
  p.kv_heads = a.kv_heads;
  p.group = group;
  p.n = 1;
  p.rows = group;
  p.max_len = a.max_len;
  p.shares = pl.shares;
  p.dealt = pl.dealt;
  p.row_blocks = pl.row_blocks;
  const int apart = pl.each ? NW : 1;
  const int64_t each_blocks = ceil_div(pl.shares, apart);
  p.by_length = !pl.dealt && a.batch > 1 && a.batch <= 64 && each_blocks * p.row_blocks > cus && p.row_blocks <= cus ? cus / p.row_blocks * apart : 0;
  p.scale_log2e = a.scale * 1.4426950408889634f;
  p.part = (float*)a.workspace;
  p.stat = p.part + (int64_t)pl.shares * p.row_blocks * 2 * 16 * a.head_dim;
  const unsigned blocks = p.row_blocks > 1 ? (unsigned)(ceil_div64(each_blocks, 8) * 8 * p.row_blocks) : (unsigned)each_blocks;
  if (f32) launch_dh<FORGE_KV_SAME, float>(p, blocks, pl.each, a.head_dim, s);
  else if (a.type == FORGE_KV_SAME) launch_dh<FORGE_KV_SAME, bf16>(p, blocks, pl.each, a.head_dim, s);
  else if (a.type == FORGE_KV_INT8) launch_dh<FORGE_KV_INT8, bf16>(p, blocks, pl.each, a.head_dim, s);
  else launch_dh<FORGE_KV_FP8, bf16>(p, blocks, pl.each, a.head_dim, s);
  if (!pl.dealt) return launch_status();
  if (hipGetLastError() != hipSuccess) return FORGE_ERR_HIP;
  if (f32) launch_merge<float>(p, a.head_dim, s);
  else launch_merge<bf16>(p, a.head_dim, s);
  return launch_status();
}

}  // namespace forge
