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
#include <float.h>
#include <math.h>
#include "tree.hpp"
#include "tree_plan.hpp"

namespace forge {
namespace {

constexpr int NW = 4;                     // waves per block

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

// ---- how cache rows become matrix operands -------------------------------------------------------------------
// Raw: the operands of a 32-row tile.  k[f]: rows of half f in the A layout (lane = row l % 16, 16 bytes per 64 contiguous
// ones); v[i]: columns c (DH / 16) .. of row 8 (l / 16) + i, c = l % 16.
// Neither layout is read from memory: a wave-wide load of 16 rows x 16 bytes a quarter costs a line lookup per lane, and the
// lookups, not the bytes, then bound the kernel (int8, 64 ragged sequences up to 2049 rows of 8 heads: 45 us, the address unit
// busy throughout).  A tile comes in whole 1 KB pieces into registers, a tile ahead or two, and goes through LDS of its wave alone.
template <int BYTES, int DH>
struct Raw {
  static constexpr int KL = DH * BYTES / 64;                 // 16-byte pieces of a K row per lane
  static constexpr int VW = DH / 16 * BYTES / 4;             // words of a V row per lane
  u32x4 k[2][KL];
  uint32_t v[8][VW];
};
template <int BYTES, int DH>
struct Patch {                                               // a wave's tile in LDS
  static constexpr int ROW = DH * BYTES, STRIDE = ROW + 16;  // (rows 16 bytes apart in the banks: reads of either layout are free of conflicts)
  static constexpr int LOADS = TILE * ROW / 1024, PER = 1024 / ROW;      // pieces of K or V, rows of one
  static constexpr int SCALES = 2 * TILE * STRIDE, BYTES_ALL = SCALES + 256;
  // K rows in the order of the operands: half f holds rows r with bit 2 of r == f
  static __host__ __device__ constexpr int k_slot(int r) { return (r >> 3) * 4 + (r & 3) + 16 * ((r >> 2) & 1); }
};

template <int W> struct Words;
template <> struct Words<1> { typedef uint32_t type; };
template <> struct Words<2> { typedef u32x2 type; };
template <> struct Words<4> { typedef u32x4 type; };

template <int VW>
__device__ inline void load_words(const char* p, uint32_t (&w)[VW]) {
  constexpr int W = VW > 4 ? 4 : VW;
#pragma unroll
  for (int o = 0; o < VW; o += W) {
    const auto t = *reinterpret_cast<const typename Words<W>::type*>(p + o * 4);
    if constexpr (W == 1) w[o] = t;
    else {
#pragma unroll
      for (int i = 0; i < W; ++i) w[o + i] = t[i];
    }
  }
}

template <forge_kv_type S, typename T> struct Store;

// bf16 operands of v_mfma_f32_16x16x32_bf16
template <> struct Store<FORGE_KV_SAME, bf16> {
  static constexpr int BYTES = 2;
  template <int DH> static __device__ inline bf16x8 k(const Raw<2, DH>& r, int f, int j) {
    return __builtin_bit_cast(bf16x8, r.k[f][j]);
  }
  template <int DH> static __device__ inline u32x4 v(const Raw<2, DH>& r, int m) {
    u32x4 o;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      o[t] = __builtin_amdgcn_perm(r.v[2 * t + 1][m / 2], r.v[2 * t][m / 2], m & 1 ? 0x07060302 : 0x05040100);
    return o;
  }
  // first of the query elements that MFMA j contracts for lane group kg
  static __device__ inline int q_at(int j, int kg) { return 32 * j + 8 * kg; }
  // all ones in the place of the elements of this word that are infinite or NaN
  static __device__ inline uint32_t odd(uint32_t w) { return ((((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu; }
  static __device__ inline void values4(const char* p, float* f) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
    f[0] = bf_lo(w[0]); f[1] = bf_hi(w[0]); f[2] = bf_lo(w[1]); f[3] = bf_hi(w[1]);
  }
};
template <> struct Store<FORGE_KV_INT8, bf16> {
  static constexpr int BYTES = 1;
  static __device__ inline float byte(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }
  template <int DH> static __device__ inline bf16x8 k(const Raw<1, DH>& r, int f, int j) {
    u32x4 o;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint32_t w = r.k[f][j / 2][2 * (j & 1) + t / 2];
      o[t] = pack_bf2(byte(w, 2 * (t & 1)), byte(w, 2 * (t & 1) + 1));
    }
    return __builtin_bit_cast(bf16x8, o);
  }
  template <int DH> static __device__ inline u32x4 v(const Raw<1, DH>& r, int m) {
    u32x4 o;
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = pack_bf2(byte(r.v[2 * t][m / 4], m & 3), byte(r.v[2 * t + 1][m / 4], m & 3));
    return o;
  }
  static __device__ inline int q_at(int j, int kg) { return 64 * (j / 2) + 16 * kg + 8 * (j & 1); }
  static __device__ inline uint32_t odd(uint32_t) { return 0; }          // (codes are finite)
  static __device__ inline void values4(const char* p, float* f) { Codes<FORGE_KV_INT8>::unpack(*reinterpret_cast<const uint32_t*>(p), f); }
};
template <> struct Store<FORGE_KV_FP8, bf16> {
  static constexpr int BYTES = 1;
  static __device__ inline uint32_t pair(uint32_t w, bool hi) {     // bytes 2 hi, 2 hi + 1 as bf16
    return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
  }
  template <int DH> static __device__ inline bf16x8 k(const Raw<1, DH>& r, int f, int j) {
    u32x4 o;
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = pair(r.k[f][j / 2][2 * (j & 1) + t / 2], t & 1);
    return __builtin_bit_cast(bf16x8, o);
  }
  template <int DH> static __device__ inline u32x4 v(const Raw<1, DH>& r, int m) {
    u32x4 o;
#pragma unroll
    for (int t = 0; t < 4; ++t)       // (the pairs of columns m and m ^ 1 are the same instructions)
      o[t] = __builtin_amdgcn_perm(pair(r.v[2 * t + 1][m / 4], m & 2), pair(r.v[2 * t][m / 4], m & 2),
                                   m & 1 ? 0x07060302 : 0x05040100);
    return o;
  }
  static __device__ inline int q_at(int j, int kg) { return 64 * (j / 2) + 16 * kg + 8 * (j & 1); }
  static __device__ inline uint32_t odd(uint32_t w) { return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu; }
  static __device__ inline void values4(const char* p, float* f) { Codes<FORGE_KV_FP8>::unpack(*reinterpret_cast<const uint32_t*>(p), f); }
};
template <> struct Store<FORGE_KV_SAME, float> {
  static constexpr int BYTES = 4;
  static __device__ inline uint32_t odd(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u ? ~0u : 0u; }
  static __device__ inline void values4(const char* p, float* f) {
    const floatx4 w = *reinterpret_cast<const floatx4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = w[i];
  }
};

__device__ inline float lanes_max(float x) {       // over lanes l, l ^ 16, l ^ 32, l ^ 48
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ inline float lanes_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}

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

template <typename T> __device__ inline void store4(T* p, floatx4 v);
template <> __device__ inline void store4<float>(float* p, floatx4 v) { *reinterpret_cast<floatx4*>(p) = v; }
template <> __device__ inline void store4<bf16>(bf16* p, floatx4 v) {
  *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
}

__device__ inline int position_of(const TreeParams& p, int b) {
  return p.seq_pos != nullptr ? min(max(p.seq_pos[b], 0), p.max_pos) : p.max_pos;
}
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }      // into a scalar register
__device__ inline int units_of(const TreeParams& p, int pos) { return (pos + p.n + UNIT - 1) / UNIT; }

// Units of the sequences, a lane each and 64 at a time: how many there are before one, and whose one is
struct Deal {
  uint32_t before[MAX_DEALT / 64], units[MAX_DEALT / 64], total;      // per cache head
  __device__ inline explicit Deal(const TreeParams& p) {
    const int lane = threadIdx.x & 63;
    total = 0;
#pragma unroll
    for (int k = 0; k < MAX_DEALT / 64; ++k) {
      units[k] = 64 * k + lane < p.batch ? units_of(p, position_of(p, 64 * k + lane)) : 0;
    }
#pragma unroll
    for (int k = 0; k < MAX_DEALT / 64; ++k) {
      before[k] = 0xffffffffu;
      if (64 * k >= p.batch) continue;
      int v = units[k];                                  // running sum over the lanes
      v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);     // row_shr:1, 2, 4, 8
      v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
      v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
      v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
      v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);    // row_bcast:15 into rows 1 and 3
      v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);    // row_bcast:31 into rows 2 and 3
      before[k] = total + v - units[k];
      total += __builtin_amdgcn_readlane(v, 63);
    }
  }
  // of sequence b
  __device__ inline void of(int b, uint32_t& first, uint32_t& count) const {
    first = count = 0;
#pragma unroll
    for (int k = 0; k < MAX_DEALT / 64; ++k)
      if (b / 64 == k) {
        first = __builtin_amdgcn_readlane(before[k], b & 63);
        count = __builtin_amdgcn_readlane(units[k], b & 63);
      }
  }
  // the sequence that holds unit x of the heads side by side (x < total * heads)
  __device__ inline int holder(uint32_t x, int heads) const {
    int b = -1;
#pragma unroll
    for (int k = 0; k < MAX_DEALT / 64; ++k)
      b += __popcll(__ballot(before[k] != 0xffffffffu && units[k] != 0 && before[k] * heads <= x));
    return b;
  }
};
// The shares that the units are dealt over: of a batch that is shorter than the host had to expect no more than units, so that none between
// two shares of a pair is empty.  The first unit of share i, and the share that holds unit x:
__device__ inline uint32_t shares_of(const TreeParams& p, uint32_t units) { return min((uint32_t)p.shares, units); }
__device__ inline uint32_t share_begin(uint32_t i, uint32_t units, uint32_t shares) { return (uint32_t)((uint64_t)i * units / shares); }
__device__ inline uint32_t share_of(uint32_t x, uint32_t units, uint32_t shares) {
  return (uint32_t)((((uint64_t)x + 1) * shares - 1) / units);       // the largest i with floor(i units / shares) <= x
}

// Whole pairs, longest sequences first, every other round of the chip backwards (the last one forwards), so that each CU gets about
// the same number of rows: the pair of block i.  At most 64 sequences.
__device__ inline int by_length(const TreeParams& p, int i) {
  const int lane = threadIdx.x & 63, all = p.shares;
  const int mine = lane < p.batch ? position_of(p, lane) : -1;
  const int first = i - i % p.by_length;
  const int at = ((all - 1) / p.by_length - i / p.by_length) & 1 ? 2 * first + min(all - first, p.by_length) - 1 - i : i;
  int place = 0;                                     // sequences before this lane's
  for (int j = 0; j < p.batch; ++j) {
    const int other = __builtin_amdgcn_readlane(mine, j);
    place += other > mine || (other == mine && j < lane);
  }
  const int b = __ffsll((unsigned long long)__ballot(lane < p.batch && place == at / p.kv_heads)) - 1;
  return b * p.kv_heads + at % p.kv_heads;
}

// What a block works through: cache rows [begin, stop) of one (sequence, cache head) at a time
struct Piece {
  int b, g, pos, begin, stop;
  int which;            // partials: 1 the rows' beginning, 0 a continuation; -1: all rows, the output is written
};
struct Share {
  int i, rb;            // share, block of query rows
  uint32_t left;        // units still to do
  int b, g, unit;       // where the next piece begins
  int pos;              // of sequence b; a vector register, not waited for before the piece is taken
  // false: nothing to do.  Blocks go round-robin over the 8 XCDs: those of one share are 8 apart, so that its rows come into one L2
  // A block (or, of `of` shares a block, this wave)
  __device__ inline bool start(const TreeParams& p, int of = 1, int wave = 0) {
    i = blockIdx.x;
    rb = 0;
    if (p.row_blocks > 1) {
      const int turn = blockIdx.x / (8 * p.row_blocks), in = blockIdx.x % (8 * p.row_blocks);
      i = turn * 8 + in % 8;
      rb = in / 8;
    }
    i = i * of + wave;
    if (i >= p.shares) return false;
    unit = 0;
    if (!p.dealt) {
      const int at = p.by_length > 0 ? by_length(p, i) : i;
      b = uniform(at / p.kv_heads);
      g = uniform(at % p.kv_heads);
      left = 0x7fffffffu;
    } else {
      const Deal d(p);
      const uint32_t all = d.total * p.kv_heads, shares = shares_of(p, all);
      if ((uint32_t)i >= shares) return false;
      const uint32_t x = share_begin(i, all, shares);
      left = uniform(share_begin(i + 1, all, shares) - x);
      b = uniform(d.holder(x, p.kv_heads));
      uint32_t first, count;
      d.of(b, first, count);
      g = uniform((x - first * p.kv_heads) / count);
      unit = uniform((x - first * p.kv_heads) % count);
    }
    pos = position_of(p, b);
    return true;
  }
  __device__ inline Piece next(const TreeParams& p) {
    const int here = uniform(pos), count = units_of(p, here);
    const int stop = min(count, unit + (int)left);
    const Piece w = {b, g, here, unit * UNIT, min(stop * UNIT, here + p.n), unit == 0 ? (stop == count ? -1 : 1) : 0};
    left = p.dealt ? left - (stop - unit) : 0;
    unit = 0;
    if (left > 0 && ++g == p.kv_heads) {
      g = 0;
      pos = position_of(p, ++b);
    }
    return w;
  }
};
// where the partials of a share's query row r go (r < rows of a block)
__device__ inline int64_t slot_of(const TreeParams& p, int i, int rb, int which, int block_rows) {
  return ((int64_t)(i * p.row_blocks + rb) * 2 + which) * block_rows;
}
template <typename T>
__device__ inline T* out_row(const TreeParams& p, int b, int g, int row, int dh) {
  const int tok = row / p.group, hh = g * p.group + row % p.group;
  return reinterpret_cast<T*>(p.out) + (((int64_t)b * p.n + tok) * p.q_heads + hh) * dh;
}

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
  Share share;
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

  Share share;
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

// 2^x, the weight of a share that lies -x below the largest; one that would round to 0 is the smallest positive number, so that an infinity that was
// put back there stays one
__device__ inline float share_weight(float x) { return fmaxf(__builtin_amdgcn_exp2f(x), __uint_as_float(1)); }

// The shares of a query row in order, 4 a round trip: DH / 4 lanes a row.  Rows that one share held whole are there already.
// SPLIT: all lanes of the block for one row, the shares in as many runs, added in their order at the end (32 shares a pair, 4 rows of 8 pairs: 8 -> 4 us).
template <typename T, int DH, bool SPLIT>
__global__ __launch_bounds__(256) void attn_tree_merge(TreeParams p, int block_rows) {
  constexpr int LPR = DH / 4, PER = 256 / LPR;
  __shared__ floatx4 so[SPLIT ? PER : 1][LPR];
  __shared__ float sm[SPLIT ? PER : 1][2];
  const int pair = blockIdx.y, b = pair / p.kv_heads, g = pair % p.kv_heads;
  const int run = threadIdx.x / LPR, row = SPLIT ? blockIdx.x : blockIdx.x * PER + run, at = threadIdx.x % LPR, d = at * 4;
  const Deal deal(p);
  uint32_t first, count;
  deal.of(b, first, count);
  const uint32_t all = deal.total * p.kv_heads, x = first * p.kv_heads + g * count;
  const uint32_t shares = shares_of(p, all);
  const int i0 = share_of(x, all, shares), i1 = share_of(x + count - 1, all, shares);
  if (i0 == i1 || row >= p.rows) return;
  const int rb = row / block_rows, r = row % block_rows;
  const int each = SPLIT ? ceil_div(i1 - i0 + 1, PER) : 0;
  const int from = SPLIT ? min(i0 + run * each, i1 + 1) : i0, to = SPLIT ? min(from + each, i1 + 1) : i1 + 1;
  float mx = -FLT_MAX, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int z0 = from; z0 < to; z0 += 4) {
    float mz[4], lz[4];
    floatx4 oz[4];
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const int i = min(z0 + z, to - 1);
      const int64_t slot = slot_of(p, i, rb, i == i0, block_rows) + r;
      mz[z] = p.stat[slot * 2];
      lz[z] = p.stat[slot * 2 + 1];
      oz[z] = *reinterpret_cast<const floatx4*>(p.part + slot * DH + d);
    }
    float mn = mx;
#pragma unroll
    for (int z = 0; z < 4; ++z) mn = fmaxf(mn, mz[z]);
    const float a = share_weight(mx - mn);
    mx = mn;
    l *= a;
    o *= a;
#pragma unroll
    for (int z = 0; z < 4; ++z)
      if (z0 + z < to) {
        const float w = share_weight(mz[z] - mn);
        l += lz[z] * w;
        o += oz[z] * w;
      }
  }
  if constexpr (SPLIT) {
    so[run][at] = o;
    if (at == 0) { sm[run][0] = mx; sm[run][1] = l; }
    __syncthreads();
    if (run > 0) return;
    float top = mx;
#pragma unroll
    for (int w = 1; w < PER; ++w) top = fmaxf(top, sm[w][0]);
    const float a = share_weight(mx - top);
    l *= a;
    o *= a;
#pragma unroll
    for (int w = 1; w < PER; ++w) {
      const float k = share_weight(sm[w][0] - top);
      l += sm[w][1] * k;
      o += so[w][at] * k;
    }
  }
  store4<T>(out_row<T>(p, b, g, row, DH) + d, o * (l == 0.f ? 0.f : 1.f / l));
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
  if (head_dim == 64) split ? attn_tree_merge<T, 64, true><<<grid, 256, 0, s>>>(p, block_rows) : attn_tree_merge<T, 64, false><<<grid, 256, 0, s>>>(p, block_rows);
  else split ? attn_tree_merge<T, 128, true><<<grid, 256, 0, s>>>(p, block_rows) : attn_tree_merge<T, 128, false><<<grid, 256, 0, s>>>(p, block_rows);
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
