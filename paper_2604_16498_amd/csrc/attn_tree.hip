// Attention of 1 .. 64 new tokens per sequence over a cache in 16 or 32 bits, int8 or fp8, each of the new tokens seeing the
// cached rows and its own ancestors among the new ones.
//
// The G = Hq / Hkv query heads of a cache head and the n tokens are one set of G n query rows (row = token * G + head), taken in
// tiles of 16.  A block of 4 waves owns RT such tiles of one (sequence, cache head) and one range of cache rows; its waves take
// the 32-row tiles of the range in turn, each through a patch of LDS that no other wave touches, and meet only to add up:
//   scores   S^T = K . Q^T (v_mfma_f32_16x16x32_bf16): K rows are the A operand, 16 bytes a lane and read
//            (the order of the contraction is free, Q follows it).  Row r of the 16-row half f of a tile is cache row
//            8 (r / 4) + r % 4 + 4 f, so that a lane ends up with the scores of 8 consecutive cache rows for its query row ...
//   softmax  ... and with their weights as the B operand of the second product, without moving them.  Running maximum per
//            query row, held back until a tile exceeds it by 2^8 (fp32 sums have room for that, and rescaling becomes rare).
//   P . V    O^T = V^T . P^T: the lane that reads columns c (DH / 16) .. of its 8 cache rows
//            forms the transposed operand with the packing that the conversion needs anyway.
// Rows in 8 bits become bf16 exactly (int8 and e4m3 both fit its 8 significant bits); their scales multiply the scores
// and the weights in fp32.  fp32 caches run the same way on v_mfma_f32_16x16x4_f32, all operands in fp32.
// Many query rows: attn_tree_wide_kernel below, whose waves share the cache rows through LDS.
// The rows of all (sequence, cache head) pairs are dealt evenly over the blocks in units of 128 where that is estimated to pay, whatever the lengths,
// which only the device knows: every block finds its share from the positions.  A pair that one block holds whole is
// finished there; of the others fp32 partials go to the workspace and a second kernel merges them in order.  No atomics.
// Measured, 32 heads over 8 of 128: one token, 64 sequences up to 2049 rows, int8 (174 MB) 38 us, 4.6 TB/s: memory.  26 tokens, 5 up to 8217 rows, fp8
// 38 us, 6 of them the merge, 0.29 PFLOP/s; 64 tokens, 16 up to 8255, bf16 121 us, 12 of them the merge, 0.72 PFLOP/s (the launch alone 104 to
// 140 us by the clock that the card holds): a SIMD's matrix and vector cycles, which add up whichever of its waves they come from, then the
// partials.  One token, 334 rows of 12 heads of 64: 5.8 us, a chain of loads.  fp32, 12 heads of 64, 8 up to 1000 rows, one token 18, 32 tokens 21 us.
// Registers: of the kernel of 128 query rows for 16-bit heads of 128 14 are spilled (60 bytes a lane), the wide ones for 8-bit heads of 64 spill 50
// to 117 scalar ones into vector registers.
#include "cache_tiles.hpp"

namespace forge {
namespace {

struct TreeParams {
  CacheView c;
  Heads q;
  char* out;
  float* part;             // [shares, row_blocks, 2, rows of a block, DH] unnormalised outputs, then [.., 2] (maximum, sum)
  float* stat;
  const int* seq_pos;
  const uint64_t* visible;
  int batch, q_heads, kv_heads, group, n, rows, max_pos, cap; // rows = group * n
  int shares;              // blocks that the cache rows are dealt over
  int dealt;               // 0: a share is one (sequence, cache head), no partials
  int by_length;           // > 0: those, by length in rounds of this many
  int row_blocks;          // blocks that hold the query rows, each beside every share
  float scale_log2e;
};

// which of the cache rows first .. first + 31 a query row sees, a bit each: d0 = first - (cached rows), bits: the drafts it sees
__device__ inline uint32_t seen_rows(uint64_t bits, int d0) {
  if (d0 <= -32) return 0xffffffffu;
  if (d0 < 0) return (uint32_t)(bits << -d0) | ((1u << -d0) - 1u);
  return d0 < 64 ? (uint32_t)(bits >> d0) : 0u;
}
// of query row `row` of n drafted tokens
__device__ inline uint64_t bits_of(const TreeParams& p, int b, int tok) {
  const uint64_t all = ~0ull >> (64 - p.n);
  return (p.visible != nullptr ? p.visible[(int64_t)b * p.n + tok] : (2ull << tok) - 1) & all;
}

__device__ inline int position_of(const TreeParams& p, int b) {
  return p.seq_pos != nullptr ? min(max(p.seq_pos[b], 0), p.max_pos) : p.max_pos;
}
__device__ inline int units_of(const TreeParams& p, int pos) { return (pos + p.n + UNIT - 1) / UNIT; }
__device__ inline int next_sequence(const TreeParams& p, int& b) { return position_of(p, ++b); }      // (each has its new rows)

// An infinity or NaN in a row that only some query rows see would reach the others as 0 * NaN.  So among the new rows (and behind
// them) such elements of V are taken out as a tile is stored, and added at the end where they belong.
// row: of the piece, counted from the first new one; marks: new rows that had any
template <typename St>
__device__ inline void take_out(u32x4& piece, int row, int n, uint64_t& marks) {
  uint32_t any = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t m = row >= 0 ? St::odd(piece[w]) : 0u;
    any |= m;
    piece[w] &= ~m;
  }
  marks |= any != 0 && row < n ? 1ull << (row & 63) : 0ull;
}
// those of columns d .. d + 3 that query token `tok` sees, added to its sums (whatever the row's weight: one that rounds to 0 is positive)
template <typename St, int DH>
__device__ inline void put_back(const TreeParams& p, int b, int tok, uint64_t marks, const char* vb, int pos, int d, floatx4& o) {
  for (uint64_t m = marks & bits_of(p, b, tok); m != 0; m &= m - 1) {
    const int row = pos + __ffsll((unsigned long long)m) - 1;
    float f[4];
    St::values4(vb + (int64_t)row * (DH * St::BYTES) + d * St::BYTES, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += fabsf(f[i]) < INFINITY ? 0.f : f[i];
  }
}
// the marks of all lanes (few ever have any)
__device__ inline uint64_t wave_marks(uint64_t mine) {
  uint64_t all = 0;
  for (uint64_t who = __ballot(mine != 0); who != 0; who &= who - 1) {
    const int l = __ffsll((unsigned long long)who) - 1;
    all |= (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, l) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), l) << 32;
  }
  return all;
}

// EACH: pairs are not cut, and every wave takes one by itself; nothing is added up between waves.
template <forge_kv_type S, typename T, int DH, int RT, bool EACH>
__global__ __launch_bounds__(NW * 64, RT == 1 && sizeof(T) == 2 && (S != FORGE_KV_SAME || DH == 64) ? 3 : 2) void attn_tree_kernel(TreeParams p) {
  typedef Store<S, T> St;
  constexpr int BYTES = St::BYTES;
  constexpr bool F32 = sizeof(T) == 4, SCALED = S != FORGE_KV_SAME;
  constexpr int NJ = F32 ? DH / 4 : DH / 32;       // MFMAs of a score tile
  constexpr int NM = DH / 16;                      // 16-column tiles of the output
  typedef Raw<BYTES, DH> R;
  typedef Patch<BYTES, DH> L;
  constexpr int PAD = DH + 4;
  constexpr int WAVE_LDS = L::BYTES_ALL > 16 * PAD * 4 ? L::BYTES_ALL : 16 * PAD * 4;
  __shared__ __attribute__((aligned(16))) char patch[NW][WAVE_LDS];      // the tile, and at the end 16 rows of the wave's outputs
  __shared__ float sml[NW][16][2];
  __shared__ uint64_t oddbuf[NW];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  constexpr int SIDE = EACH ? 1 : NW;                          // waves side by side in a range of rows
  const int beside = EACH ? 0 : wave;
  Share<TreeParams> share;
  if (!share.start(p, EACH ? NW : 1, EACH ? wave : 0)) return;
  const int c = lane & 15, kg = lane >> 4;
  char* const lds = patch[wave];

  // ---- what a piece needs first, requested before its sequence's length has to be known -----------------------
  const char *kb, *vb;
  const float *ksb, *vsb;
  u32x4 qf[RT][F32 ? DH / 16 : DH / 32];                       // query rows of this lane's column ...
  uint64_t bits[RT];                                           // ... and the drafts they see
  u32x4 rk[L::LOADS], rv[L::LOADS];                            // the tile in flight
  float rs = 0.f;
  int begin = 0;
  auto tile_base = [&](int t) { return begin + (t * SIDE + beside) * TILE; };
  // Tiles are read whole: one that passes the end of the cache from the cache's last rows instead (those that belong to
  // the tile before are cut below), what lies between the end of the sequence and that is cut too.  So the addresses of a tile are one
  // scalar base and constant offsets.  (fp32: each piece clamped, so that a cache may be shorter than a tile)
  auto read_base = [&](int t) { return F32 ? tile_base(t) : min(tile_base(t), p.cap - TILE); };
  // wanted: a tile of this wave's; otherwise the loads, which stay so that their number is known, ask for little.
  // (scheduled among its neighbours, a tile's loads go to second registers, and the copies back wait for them)
  auto load_tile = [&](int t, bool wanted) {
    __builtin_amdgcn_sched_barrier(0);
    const int base = wanted ? read_base(t) : 0, l = lane & (wanted ? -1 : 0);
    const char *kf = kb + (int64_t)base * L::ROW, *vf = vb + (int64_t)base * L::ROW;
    auto piece = [&](const char* from, int i) {
      if constexpr (F32) return from + (int64_t)min(i * L::PER + l / (L::ROW / 16), p.cap - 1 - base) * L::ROW + l % (L::ROW / 16) * 16;
      else return from + l * 16 + i * 1024;
    };
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) rk[i] = *reinterpret_cast<const u32x4*>(piece(kf, i));
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) rv[i] = *reinterpret_cast<const u32x4*>(piece(vf, i));
    if constexpr (SCALED) rs = (lane < TILE ? ksb : vsb)[base + (l & (TILE - 1))];
    __builtin_amdgcn_sched_barrier(0);
  };
  auto request = [&](int b, int g, int from) {
    const int64_t head = b * p.c.bs + g * p.c.hs;              // elements
    kb = p.c.k + head * BYTES;
    vb = p.c.v + head * BYTES;
    ksb = SCALED ? p.c.ks + head / DH : nullptr;
    vsb = SCALED ? p.c.vs + head / DH : nullptr;
    begin = from;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int row = (share.rb * RT + i) * 16 + c;
      const bool real = row < p.rows;
      const int t = real ? row / p.group : 0, hh = g * p.group + (real ? row % p.group : 0);
      const T* qr = reinterpret_cast<const T*>(p.q.p) + b * p.q.bs + t * p.q.ts + hh * p.q.hs;
#pragma unroll
      for (int j = 0; j < (F32 ? DH / 16 : DH / 32); ++j) {
        u32x4 x = {0, 0, 0, 0};
        if constexpr (F32) { if (real) x = *reinterpret_cast<const u32x4*>(qr + 16 * j + 4 * kg); }
        else { if (real) x = *reinterpret_cast<const u32x4*>(qr + St::q_at(j, kg)); }
        qf[i][j] = x;
      }
      bits[i] = real ? bits_of(p, b, t) : 0;
    }
    load_tile(0, tile_base(0) < p.max_pos + p.n);
  };
  const int piece_row = lane / (L::ROW / 16), piece_at = lane % (L::ROW / 16) * 16;
  const int k_put = L::k_slot(piece_row) * L::STRIDE + piece_at, v_put = TILE * L::STRIDE + piece_row * L::STRIDE + piece_at;
  uint64_t marks = 0;
  // behind: the tile's first row less the new ones' first; again: rows that the tile before had too, of a tile moved back (so that behind +
  // TILE > 0).  Their weights are 0 here: an infinity in them would become NaN, so their V is cleared, by a loop that needs few registers;
  // and a draft among them is not marked, the share may not hold it (this wave's own tiles lie too far apart to have marked one of them;
  // EACH: all rows are this wave's).  fp8 has no infinities, and who sees the row of a NaN gets it either way.
  auto put_tile = [&](int behind, int again) {
    wave_lds_sync();                       // the tile before has been read
    if (S != FORGE_KV_INT8 && behind + TILE > 0) {
#pragma unroll
      for (int i = 0; i < L::LOADS; ++i) take_out<St>(rv[i], behind + i * L::PER + piece_row, p.n, marks);
    }
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i)     // (k_slot is a permutation of bits: of a sum without carries the sum)
      *reinterpret_cast<u32x4*>(lds + k_put + L::k_slot(i * L::PER) * L::STRIDE) = rk[i];
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) *reinterpret_cast<u32x4*>(lds + v_put + i * L::PER * L::STRIDE) = rv[i];
    if (S == FORGE_KV_SAME && again > 0) {
      if (!EACH && behind + again > 0) marks &= ~0ull << (behind + again);
#pragma unroll 1
      for (int o = lane * 4; o < again * L::STRIDE; o += 256) *reinterpret_cast<uint32_t*>(lds + TILE * L::STRIDE + o) = 0;
    }
    if constexpr (SCALED) *reinterpret_cast<float*>(lds + L::SCALES + lane * 4) = rs;
    wave_lds_sync();
  };
  request(share.b, share.g, share.unit * UNIT);

  for (;;) {
  const Piece at = share.next(p);
  const int pos = at.pos, stop = at.stop;
  const int ntile = stop > begin + beside * TILE ? ceil_div(stop - begin - beside * TILE, SIDE * TILE) : 0;
  marks = 0;
  float m_run[RT], l_run[RT];
  floatx4 acc[RT][NM];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    m_run[i] = -FLT_MAX;
    l_run[i] = 0.f;
#pragma unroll
    for (int m = 0; m < NM; ++m) acc[i][m] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

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
    const int base = read_base(t), first = base + 8 * kg;      // this lane's 8 cache rows
    const bool edge = base + TILE > pos;
    // ---- scores --------------------------------------------------------------------------------------
    float s[RT][8];
    {
      floatx4 sa[RT][2];
#pragma unroll
      for (int i = 0; i < RT; ++i) sa[i][0] = sa[i][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if constexpr (F32) {
            const float x = __uint_as_float(r.k[f][j / 4][j & 3]);
#pragma unroll
            for (int i = 0; i < RT; ++i)
              sa[i][f] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, __uint_as_float(qf[i][j / 4][j & 3]), sa[i][f], 0, 0, 0);
          } else {
            const bf16x8 x = St::k(r, f, j);
#pragma unroll
            for (int i = 0; i < RT; ++i)
              sa[i][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8, qf[i][j]), sa[i][f], 0, 0, 0);
          }
        }
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s[i][e] = sa[i][e >> 2][e & 3] * p.scale_log2e;
          if constexpr (SCALED) s[i][e] *= ksr[e];
        }
    }
    uint32_t seen[RT];                                   // bit e: query row i sees cache row first + e
    if (edge) {
      const uint32_t fresh = ~0u << min(max(tile_base(t) - first, 0), 8);
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        seen[i] = seen_rows(bits[i], first - pos) & fresh;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = seen[i] >> e & 1 ? s[i][e] : -INFINITY;
      }
    }
    // ---- softmax -------------------------------------------------------------------------------------
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float mx = s[i][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[i][e]);
      if (__any(mx > m_run[i] + 8.f)) {                  // (wave-uniform)
        const float m_new = fmaxf(m_run[i], lanes_max(mx));
        const float alpha = __builtin_amdgcn_exp2f(m_run[i] - m_new);
        m_run[i] = m_new;
        l_run[i] *= alpha;
#pragma unroll
        for (int m = 0; m < NM; ++m) acc[i][m] *= alpha;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = __builtin_amdgcn_exp2f(s[i][e] - m_run[i]);
        l_run[i] += w;
        s[i][e] = w;
        if constexpr (SCALED) s[i][e] = w * vsr[e];
      }
      if (SCALED && edge) {                              // (a row that is not seen may hold any scale)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = seen[i] >> e & 1 ? s[i][e] : 0.f;
      }
    }
    // ---- P . V ---------------------------------------------------------------------------------------
#pragma unroll
    for (int i = 0; i < 8; ++i) load_words<R::VW>(lds + (TILE + 8 * kg + i) * L::STRIDE + c * (R::VW * 4), r.v[i]);
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
          for (int i = 0; i < RT; ++i)
            acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(r.v[e][m]), s[i][e], acc[i][m], 0, 0, 0);
    } else {
      bf16x8 pf[RT];
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_bf2(s[i][2 * e], s[i][2 * e + 1]);
        pf[i] = __builtin_bit_cast(bf16x8, w);
      }
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        const bf16x8 x = __builtin_bit_cast(bf16x8, St::v(r, m));
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, pf[i], acc[i][m], 0, 0, 0);
      }
    }
  };

  for (int t = 0; t < ntile; ++t) {
    put_tile(read_base(t) - pos, tile_base(t) - read_base(t));
    load_tile(t + 1, t + 1 < ntile);
    step(t);
  }

  const char* const v_rows = vb;
  if constexpr (S != FORGE_KV_INT8) {
    const uint64_t m = wave_marks(marks);
    if (lane == 0) oddbuf[wave] = m;
  }
  const bool more = share.left > 0;
  if (more) request(share.b, share.g, 0);      // (on its way while this piece is finished)
  // ---- the waves' shares, added in wave order, 16 query rows at a time ---------------------------------------
  const int64_t slot = slot_of(p, share.i, share.rb, max(at.which, 0), RT * 16);
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const float l = lanes_sum(l_run[i]);
    wave_lds_sync();
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int m = 0; m < NM; m += 4)
        *reinterpret_cast<floatx4*>(lds + c * (PAD * 4) + ((4 * kg + v) * NM + m) * 4) =
            floatx4{acc[i][m][v], acc[i][m + 1][v], acc[i][m + 2][v], acc[i][m + 3][v]};
    if (kg == 0) { sml[wave][c][0] = m_run[i]; sml[wave][c][1] = l; }
    if constexpr (EACH) wave_lds_sync();
    else lds_barrier();
    for (int idx = EACH ? lane : tid; idx < 16 * (DH / 4); idx += SIDE * 64) {
      const int r = idx / (DH / 4), d = idx % (DH / 4) * 4, row = (share.rb * RT + i) * 16 + r;
      if (row >= p.rows) continue;
      const int w0 = EACH ? wave : 0;
      float mn = sml[w0][r][0];
#pragma unroll
      for (int w = 1; w < SIDE; ++w) mn = fmaxf(mn, sml[w][r][0]);
      floatx4 o = {0.f, 0.f, 0.f, 0.f};
      float lt = 0.f;
#pragma unroll
      for (int w = w0; w < w0 + SIDE; ++w) {
        const float a = __builtin_amdgcn_exp2f(sml[w][r][0] - mn);
        o += *reinterpret_cast<const floatx4*>(patch[w] + r * (PAD * 4) + d * 4) * a;
        lt += sml[w][r][1] * a;
      }
      if constexpr (S != FORGE_KV_INT8) {
        uint64_t odd = 0;
#pragma unroll
        for (int w = w0; w < w0 + SIDE; ++w) odd |= oddbuf[w];
        if (odd != 0) put_back<St, DH>(p, at.b, row / p.group, odd, v_rows, pos, d, o);
      }
      if (at.which < 0) {
        store4<T>(out_row<T>(p, at.b, at.g, row, DH) + d, o * (lt == 0.f ? 0.f : 1.f / lt));
      } else {
        *reinterpret_cast<floatx4*>(p.part + (slot + 16 * i + r) * DH + d) = o;
        if (d == 0) { p.stat[(slot + 16 * i + r) * 2] = mn; p.stat[(slot + 16 * i + r) * 2 + 1] = lt; }
      }
    }
    if constexpr (!EACH) lds_barrier();
  }
  if (!more) break;
  }
}

// ---- many query rows -------------------------------------------------------------------------------------------
// A block of WAVES waves owns 32 query rows a wave and walks over its cache rows in tiles of KT, which come from memory through
// registers into LDS as bf16 (8-bit rows are converted once per block there), two buffers each of K and V: a tile is stored
// while the one before it is multiplied, and requested a tile earlier still.  v_mfma_f32_32x32x16_bf16: S^T = K . Q^T with a query row
// per lane, whose weights are the B operand of O^T = V^T . P^T as they are; V^T is read by the transposing LDS read.
// Scales lie in LDS beside the tiles and multiply scores and weights in fp32.
template <forge_kv_type S> __device__ inline void codes_to_bf16(u32x4 w, u32x4& lo, u32x4& hi) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float f[4];
    Codes<S>::unpack(w[i], f);
    const uint32_t a = pack_bf2(f[0], f[1]), b = pack_bf2(f[2], f[3]);
    if (i < 2) { lo[2 * i] = a; lo[2 * i + 1] = b; }
    else { hi[2 * i - 4] = a; hi[2 * i - 3] = b; }
  }
}
template <> __device__ inline void codes_to_bf16<FORGE_KV_FP8>(u32x4 w, u32x4& lo, u32x4& hi) {
  typedef Store<FORGE_KV_FP8, bf16> St;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    lo[2 * i] = St::pair(w[i], false);
    lo[2 * i + 1] = St::pair(w[i], true);
    hi[2 * i] = St::pair(w[i + 2], false);
    hi[2 * i + 1] = St::pair(w[i + 2], true);
  }
}

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef short v8i16 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

template <forge_kv_type S, int DH, int WAVES, int KT>
__global__ __launch_bounds__(WAVES * 64, 2) void attn_tree_wide_kernel(TreeParams p) {
  constexpr bool SCALED = S != FORGE_KV_SAME;
  constexpr int BYTES = SCALED ? 1 : 2;
  constexpr int KS = DH * 2 + 16;                            // row strides in LDS, bytes
  constexpr int VS = DH * 2 + (DH == 64 ? 32 : 64);
  constexpr int THREADS = WAVES * 64, CPR = DH * BYTES / 16; // 16-byte pieces of a row in memory
  constexpr int LPT = KT * CPR / THREADS;                    // of K and of V, per thread and tile
  constexpr int NKB = KT / 32, NKS = DH / 16, NDT = DH / 32;
  static_assert(LPT >= 1 && LPT * THREADS == KT * CPR, "a tile is whole pieces of every thread");
  __shared__ __attribute__((aligned(16))) char kbuf[2][KT * KS];
  __shared__ __attribute__((aligned(16))) char vbuf[2][KT * VS];
  __shared__ __attribute__((aligned(16))) float sbuf[2][2][SCALED ? KT : 4];
  __shared__ uint64_t oddbuf[WAVES];

  Share<TreeParams> share;
  if (!share.start(p)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  const int row = (share.rb * WAVES + wave) * 32 + fr;       // this lane's query row
  const bool real = row < p.rows;
  const int tok = real ? row / p.group : 0, sub = real ? row % p.group : 0;
  const int vt_lane = (((lane & 15) >> 2) + 4 * fh) * VS + (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;

  // ---- what a piece needs first, requested before its sequence's length has to be known
  const char *kb, *vb;
  const float *ksb, *vsb;
  int begin, last;                                           // rows past `last` read it again
  u32x4 rk[LPT], rv[LPT];
  float rs = 0.f;
  bf16x8 qf[NKS];
  uint64_t bits;
  // (a tile is one run of memory; what lies past row `last` is its end again, cut below)
  auto load = [&](int t) {
    const int base = min(begin + t * KT, last), most = min(last - base, KT) * (DH * BYTES) + (DH * BYTES - 16);
    const char *kf = kb + (int64_t)base * (DH * BYTES), *vf = vb + (int64_t)base * (DH * BYTES);
#pragma unroll
    for (int i = 0; i < LPT; ++i) rk[i] = *reinterpret_cast<const u32x4*>(kf + (uint32_t)min((tid + i * THREADS) * 16, most));
    if constexpr (SCALED) {
      if (tid < 2 * KT) rs = (tid < KT ? ksb : vsb)[min(base + tid % KT, last)];
    }
#pragma unroll
    for (int i = 0; i < LPT; ++i) rv[i] = *reinterpret_cast<const u32x4*>(vf + (uint32_t)min((tid + i * THREADS) * 16, most));
  };
  auto request = [&](int b, int g, int from) {
    const int64_t head = b * p.c.bs + g * p.c.hs;
    kb = p.c.k + head * BYTES;
    vb = p.c.v + head * BYTES;
    ksb = SCALED ? p.c.ks + head / DH : nullptr;
    vsb = SCALED ? p.c.vs + head / DH : nullptr;
    begin = from;
    last = p.max_pos + p.n - 1;                              // (inside the cache)
    load(0);
    const bf16* qr = reinterpret_cast<const bf16*>(p.q.p) + b * p.q.bs + tok * p.q.ts + (g * p.group + sub) * p.q.hs;
#pragma unroll
    for (int j = 0; j < NKS; ++j) {
      u32x4 x = {0, 0, 0, 0};
      if (real) x = *reinterpret_cast<const u32x4*>(qr + (2 * j + fh) * 8);
      qf[j] = __builtin_bit_cast(bf16x8, x);
    }
    bits = real ? bits_of(p, b, tok) : 0;
  };
  request(share.b, share.g, share.unit * UNIT);

  for (;;) {
    const Piece at = share.next(p);
    const int pos = at.pos;
    last = pos + p.n - 1;
    uint64_t marks = 0;
    auto store = [&](int buf, int behind) {                  // behind: the tile's first row less the new ones' first
#pragma unroll
      for (int i = 0; i < LPT; ++i) {
        const int idx = tid + i * THREADS, r = idx / CPR, o = idx % CPR;
        if (S != FORGE_KV_INT8 && behind + KT > 0) take_out<Store<S, bf16>>(rv[i], behind + r, p.n, marks);
        char* kd = kbuf[buf] + r * KS;
        char* vd = vbuf[buf] + r * VS;
        if constexpr (SCALED) {
          u32x4 lo, hi;
          codes_to_bf16<S>(rk[i], lo, hi);
          *reinterpret_cast<u32x4*>(kd + o * 32) = lo;
          *reinterpret_cast<u32x4*>(kd + o * 32 + 16) = hi;
          codes_to_bf16<S>(rv[i], lo, hi);
          *reinterpret_cast<u32x4*>(vd + o * 32) = lo;
          *reinterpret_cast<u32x4*>(vd + o * 32 + 16) = hi;
        } else {
          *reinterpret_cast<u32x4*>(kd + o * 16) = rk[i];
          *reinterpret_cast<u32x4*>(vd + o * 16) = rv[i];
        }
      }
      if constexpr (SCALED) {
        if (tid < 2 * KT) sbuf[buf][tid / KT][tid % KT] = rs;
      }
    };
    const int ntile = ceil_div(at.stop - at.begin, KT);
    floatx16 acc[NDT];
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
    float m_run = -FLT_MAX, l_run = 0.f;
    store(0, begin - pos);
    load(1);
    lds_barrier();
    for (int t = 0; t < ntile; ++t) {
      const int buf = t & 1, base = at.begin + t * KT;
      if (t + 1 < ntile) store(buf ^ 1, base + KT - pos);       // its last readers finished tile t - 1 before the barrier
      load(t + 2);                             // (past the end: the last row again)
      const bool edge = base + KT > pos;
      // ---- scores: fragments are read AHEAD products before their use (the order pinned, or each product waits for its read)
      constexpr int AHEAD = 4;
      floatx16 sc[NKB];
      {
        constexpr int NF = NKB * NKS;
        bf16x8 kf[AHEAD];
        auto read = [&](int i) {       // (the row halves of a tile in turn: two chains)
          const int f = i % NKB, j = i / NKB;
          return *reinterpret_cast<const bf16x8*>(kbuf[buf] + (f * 32 + fr) * KS + (2 * j + fh) * 16);
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) kf[i] = read(i);
#pragma unroll
        for (int i = 0; i < NF; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          const int f = i % NKB, j = i / NKB;
          const floatx16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
          sc[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % AHEAD], qf[j], j == 0 ? zero : sc[f], 0, 0, 0);
          if (i + AHEAD < NF) kf[i % AHEAD] = read(i + AHEAD);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      // ---- softmax: register v of tile f is cache row 32 f + 8 (v / 4) + 4 fh + v % 4
      if constexpr (SCALED) {
#pragma unroll
        for (int f = 0; f < NKB; ++f)
#pragma unroll
          for (int v = 0; v < 16; v += 4) {
            const floatx4 k4 = *reinterpret_cast<const floatx4*>(&sbuf[buf][0][32 * f + 2 * v + 4 * fh]);
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[f][v + e] *= k4[e];
          }
      }
      uint32_t seen[NKB];                      // bit r: cache row base + 32 f + 4 fh + r
      if (edge) {
#pragma unroll
        for (int f = 0; f < NKB; ++f) {
          seen[f] = seen_rows(bits, base + 32 * f + 4 * fh - pos);
#pragma unroll
          for (int v = 0; v < 16; ++v) sc[f][v] = seen[f] >> (8 * (v >> 2) + (v & 3)) & 1 ? sc[f][v] : -INFINITY;
        }
      }
      float mx = sc[0][0];
#pragma unroll
      for (int f = 0; f < NKB; ++f)
#pragma unroll
        for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sc[f][v]);
      mx *= p.scale_log2e;
      if (__any(mx > m_run + 8.f)) {
        auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        const float m_new = fmaxf(m_run, fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int i = 0; i < NDT; ++i) acc[i] *= alpha;
      }
      bf16x8 pf[2 * NKB];
#pragma unroll
      for (int f = 0; f < NKB; ++f) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[f][v], p.scale_log2e, -m_run));
          l_run += w;
          sc[f][v] = w;
        }
        if constexpr (SCALED) {
#pragma unroll
          for (int v = 0; v < 16; v += 4) {
            const floatx4 v4 = *reinterpret_cast<const floatx4*>(&sbuf[buf][1][32 * f + 2 * v + 4 * fh]);
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[f][v + e] *= v4[e];
          }
          if (edge) {
#pragma unroll
            for (int v = 0; v < 16; ++v) sc[f][v] = seen[f] >> (8 * (v >> 2) + (v & 3)) & 1 ? sc[f][v] : 0.f;
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e) pf[2 * f + h][e] = (bf16)sc[f][8 * h + e];
      }
      // ---- O^T += V^T . P^T
      {
        constexpr int NF = 2 * NKB * NDT;
        v4i16 lo[AHEAD], hi[AHEAD];
        auto read = [&](int i) {
          const char* va = vbuf[buf] + vt_lane + 16 * (i / NDT) * VS + i % NDT * 64;
          lo[i % AHEAD] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)va);
          hi[i % AHEAD] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(va + 8 * VS));
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
        for (int i = 0; i < NF; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          const v4i16 l = lo[i % AHEAD], h = hi[i % AHEAD];
          const v8i16 both = {l[0], l[1], l[2], l[3], h[0], h[1], h[2], h[3]};
          acc[i % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, both), pf[i / NDT], acc[i % NDT], 0, 0, 0);
          if (i + AHEAD < NF) read(i + AHEAD);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      lds_barrier();
    }
    const char* const v_rows = vb;
    uint64_t odd = 0;
    if constexpr (S != FORGE_KV_INT8) {                      // (tiles are stored by all waves)
      const uint64_t m = wave_marks(marks);
      if (lane == 0) oddbuf[wave] = m;
      lds_barrier();
#pragma unroll
      for (int w = 0; w < WAVES; ++w) odd |= oddbuf[w];
    }
    const bool more = share.left > 0;
    if (more) request(share.b, share.g, 0);                  // (on its way while this piece is written)
    // ---- this lane's query row: columns 32 i + 8 q + 4 fh .. + 3 from registers 4 q .. 4 q + 3
    auto lr = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
    const float l = __uint_as_float(lr[0]) + __uint_as_float(lr[1]);
    if (real) {
      const int64_t slot = slot_of(p, share.i, share.rb, max(at.which, 0), WAVES * 32) + wave * 32 + fr;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16* out = out_row<bf16>(p, at.b, at.g, row, DH);
#pragma unroll
      for (int i = 0; i < NDT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          floatx4 o = {acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]};
          const int d = 32 * i + 8 * q + 4 * fh;
          if constexpr (S != FORGE_KV_INT8) {
            if (odd != 0) put_back<Store<S, bf16>, DH>(p, at.b, tok, odd, v_rows, pos, d, o);
          }
          if (at.which < 0) store4<bf16>(out + d, o * inv);
          else *reinterpret_cast<floatx4*>(p.part + slot * DH + d) = o;
        }
      if (at.which >= 0 && fh == 0) { p.stat[slot * 2] = m_run; p.stat[slot * 2 + 1] = l; }
    }
    if (!more) break;
  }
}

template <forge_kv_type S, typename T, int DH>
void launch_blocks(const TreeParams& p, const TreePlan& pl, hipStream_t s) {
  const int apart = pl.each ? ceil_div(pl.shares, NW) : pl.shares;
  const unsigned blocks = pl.row_blocks > 1 ? (unsigned)(ceil_div(apart, 8) * 8 * pl.row_blocks) : (unsigned)apart;
  if (pl.block_rows == 16 && pl.each) attn_tree_kernel<S, T, DH, 1, true><<<blocks, NW * 64, 0, s>>>(p);
  if (pl.block_rows == 16 && !pl.each) attn_tree_kernel<S, T, DH, 1, false><<<blocks, NW * 64, 0, s>>>(p);
  if constexpr (sizeof(T) == 2) {
    if (pl.block_rows == 32) attn_tree_kernel<S, T, DH, 2, false><<<blocks, NW * 64, 0, s>>>(p);
    // (8-bit rows of 64: a tile of 64 rows is less than a piece for each of 8 waves' threads)
    constexpr int KT8 = S != FORGE_KV_SAME && DH == 64 ? 128 : 64;
    if (pl.block_rows == 128) attn_tree_wide_kernel<S, DH, 4, 64><<<blocks, 4 * 64, 0, s>>>(p);
    if (pl.block_rows == 256) attn_tree_wide_kernel<S, DH, 8, KT8><<<blocks, 8 * 64, 0, s>>>(p);
  }
}
template <forge_kv_type S, typename T>
void launch_dh(const TreeParams& p, const TreePlan& pl, int head_dim, hipStream_t s) {
  if (head_dim == 64) launch_blocks<S, T, 64>(p, pl, s);
  else launch_blocks<S, T, 128>(p, pl, s);
}
template <typename T>
void launch_merge(const TreeParams& p, int block_rows, int head_dim, hipStream_t s) {
  // a row over a block where it has more shares than a round trip takes and the blocks fit the chip (us, attention and merge, 8 rows a block | a row:
  // one sequence of 8 x 4 heads, 8191 rows, one token 17.0 | 11.9, 16 21.2 | 19.6, 64 29.7 | 29.3, 3 of 7966, 4 tokens 19.4 | 16.6, 5 of 8191, 26 40.1 | 41.5)
  const int pairs = p.batch * p.kv_heads;
  const bool split = p.shares > 4 * pairs && (int64_t)p.rows * pairs <= 8 * compute_units();
  const dim3 grid(split ? p.rows : ceil_div(p.rows, head_dim == 64 ? 16 : 8), pairs);
  if (head_dim == 64) split ? attn_merge_kernel<T, 64, true><<<grid, 256, 0, s>>>(p, block_rows) : attn_merge_kernel<T, 64, false><<<grid, 256, 0, s>>>(p, block_rows);
  else split ? attn_merge_kernel<T, 128, true><<<grid, 256, 0, s>>>(p, block_rows) : attn_merge_kernel<T, 128, false><<<grid, 256, 0, s>>>(p, block_rows);
}

}  // namespace

size_t attn_tree_workspace_bytes(int batch, int q_heads, int kv_heads, int head_dim, int n, int max_pos, int cap, bool f32) {
  return tree_workspace_bytes(batch, q_heads, kv_heads, head_dim, n, max_pos + n, cap, f32, compute_units());
}

forge_status launch_attn_tree(const TreeArgs& a, hipStream_t s) {
  const bool f32 = a.dt == FORGE_F32;
  const TreePlan pl = plan_tree(a.batch, a.q_heads, a.kv_heads, a.head_dim, a.n, a.max_pos + a.n, a.cap,
                                a.type != FORGE_KV_SAME ? 1 : f32 ? 4 : 2, a.seq_pos != nullptr, compute_units());
  TreeParams p;
  p.c = a.c;
  p.q = a.q;
  p.out = (char*)a.out;
  p.seq_pos = a.seq_pos;
  p.visible = a.visible;
  p.batch = a.batch;
  p.q_heads = a.q_heads;
  p.kv_heads = a.kv_heads;
  p.group = a.q_heads / a.kv_heads;
  p.n = a.n;
  p.rows = p.group * a.n;
  p.max_pos = a.max_pos;
  p.cap = a.cap;
  p.shares = pl.shares;
  p.dealt = pl.dealt;
  // Whole pairs by length where some CU gets a second block (us, in batch order | by length, 64 sequences up to 2001 rows of 8 heads of 128: 8 tokens
  // 16 bits 72.3 | 70.0, int8 52.9 | 50.8, 48 of them 46.4 | 42.0, 21 up to 1401 of 16 heads, one token 36.8 | 32.4)
  const int apart = pl.each ? NW : 1;
  const int64_t blocks = (int64_t)ceil_div(pl.shares, apart) * pl.row_blocks;
  p.by_length = !pl.dealt && a.seq_pos != nullptr && a.batch > 1 && a.batch <= 64 && blocks > compute_units() && pl.row_blocks <= compute_units()
                    ? compute_units() / pl.row_blocks * apart : 0;
  p.row_blocks = pl.row_blocks;
  p.scale_log2e = a.scale * 1.4426950408889634f;
  p.part = (float*)a.workspace;
  p.stat = p.part + (int64_t)pl.shares * pl.row_blocks * 2 * pl.block_rows * a.head_dim;
  if (f32) launch_dh<FORGE_KV_SAME, float>(p, pl, a.head_dim, s);
  else if (a.type == FORGE_KV_SAME) launch_dh<FORGE_KV_SAME, bf16>(p, pl, a.head_dim, s);
  else if (a.type == FORGE_KV_INT8) launch_dh<FORGE_KV_INT8, bf16>(p, pl, a.head_dim, s);
  else launch_dh<FORGE_KV_FP8, bf16>(p, pl, a.head_dim, s);
  if (!pl.dealt) return launch_status();
  if (hipGetLastError() != hipSuccess) return FORGE_ERR_HIP;
  if (f32) launch_merge<float>(p, pl.block_rows, a.head_dim, s);
  else launch_merge<bf16>(p, pl.block_rows, a.head_dim, s);
  return launch_status();
}

}  // namespace forge
