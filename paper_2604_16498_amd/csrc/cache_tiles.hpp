// Attention over the rows of a cache, in 16 or 32 bits, int8 or fp8: how a tile of rows becomes matrix operands, how the rows of all
// (sequence, cache head) pairs are dealt over blocks, and how the blocks' shares are merged.  Shared by the kernels over one
// run of rows per sequence and over pages.  Internal to the library.
#pragma once
#include <float.h>
#include <math.h>
#include "tree.hpp"
#include "tree_plan.hpp"

namespace forge {
namespace {

constexpr int NW = 4;                     // waves per block

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

template <typename T> __device__ inline void store4(T* p, floatx4 v);
template <> __device__ inline void store4<float>(float* p, floatx4 v) { *reinterpret_cast<floatx4*>(p) = v; }
template <> __device__ inline void store4<bf16>(bf16* p, floatx4 v) {
  *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
}

__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }      // into a scalar register
// The parameters P of a kernel that deals have batch, kv_heads, group, rows (query rows of a pair), q_heads, n, out, shares, dealt,
// by_length and row_blocks, and functions of their own: position_of(p, b), the cached rows of sequence b before its n new ones;
// units_of(p, position), the units that these and the new ones are; next_sequence(p, b), which moves b on to the next one that has any, and
// gives its position.

// Units of the sequences, a lane each and 64 at a time: how many there are before one, and whose one is
template <typename P>
struct Deal {
  uint32_t before[MAX_DEALT / 64], units[MAX_DEALT / 64], total;      // per cache head
  __device__ inline explicit Deal(const P& p) {
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
  // the sequence that holds unit x of the heads side by side (x < total * heads): the last one with units that begins at or before it
  __device__ inline int holder(uint32_t x, int heads) const {
    int b = 0;
#pragma unroll
    for (int k = 0; k < MAX_DEALT / 64; ++k) {
      const uint64_t m = __ballot(before[k] != 0xffffffffu && units[k] != 0 && before[k] * heads <= x);
      if (m != 0) b = 64 * k + 63 - __builtin_clzll((unsigned long long)m);
    }
    return b;
  }
};
// The shares that the units are dealt over: of a batch that is shorter than the host had to expect no more than units, so that none between
// two shares of a pair is empty.  The first unit of share i, and the share that holds unit x:
template <typename P> __device__ inline uint32_t shares_of(const P& p, uint32_t units) { return min((uint32_t)p.shares, units); }
__device__ inline uint32_t share_begin(uint32_t i, uint32_t units, uint32_t shares) { return (uint32_t)((uint64_t)i * units / shares); }
__device__ inline uint32_t share_of(uint32_t x, uint32_t units, uint32_t shares) {
  return (uint32_t)((((uint64_t)x + 1) * shares - 1) / units);       // the largest i with floor(i units / shares) <= x
}

// Whole pairs, longest sequences first, every other round of the chip backwards (the last one forwards), so that each CU gets about
// the same number of rows: the pair of block i.  At most 64 sequences.
template <typename P>
__device__ inline int by_length(const P& p, int i) {
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
template <typename P>
struct Share {
  int i, rb;            // share, block of query rows
  uint32_t left;        // units still to do
  int b, g, unit;       // where the next piece begins
  int pos;              // of sequence b; a vector register, not waited for before the piece is taken
  // false: nothing to do.  Blocks go round-robin over the 8 XCDs: those of one share are 8 apart, so that its rows come into one L2
  // A block (or, of `of` shares a block, this wave)
  __device__ inline bool start(const P& p, int of = 1, int wave = 0) {
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
      const Deal<P> d(p);
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
  __device__ inline Piece next(const P& p) {
    const int here = uniform(pos), count = units_of(p, here);
    const int stop = min(count, unit + (int)left);
    const Piece w = {b, g, here, unit * UNIT, min(stop * UNIT, here + p.n), unit == 0 ? (stop == count ? -1 : 1) : 0};
    left = p.dealt ? left - (stop - unit) : 0;
    unit = 0;
    if (left > 0 && ++g == p.kv_heads) {
      g = 0;
      pos = next_sequence(p, b);
    }
    return w;
  }
};
// where the partials of a share's query row r go (r < rows of a block)
template <typename P>
__device__ inline int64_t slot_of(const P& p, int i, int rb, int which, int block_rows) {
  return ((int64_t)(i * p.row_blocks + rb) * 2 + which) * block_rows;
}
template <typename T, typename P>
__device__ inline T* out_row(const P& p, int b, int g, int row, int dh) {
  const int tok = row / p.group, hh = g * p.group + row % p.group;
  return reinterpret_cast<T*>(p.out) + (((int64_t)b * p.n + tok) * p.q_heads + hh) * dh;
}

// 2^x, the weight of a share that lies -x below the largest; one that would round to 0 is the smallest positive number, so that an infinity that was
// put back there stays one
__device__ inline float share_weight(float x) { return fmaxf(__builtin_amdgcn_exp2f(x), __uint_as_float(1)); }

// The shares of a query row in order, 4 a round trip: DH / 4 lanes a row.  Rows that one share held whole are there already.
// SPLIT: all lanes of the block for one row, the shares in as many runs, added in their order at the end (32 shares a pair, 4 rows of 8 pairs: 8 -> 4 us).
template <typename T, int DH, bool SPLIT, typename P>
__global__ __launch_bounds__(256) void attn_merge_kernel(P p, int block_rows) {
  constexpr int LPR = DH / 4, PER = 256 / LPR;
  __shared__ floatx4 so[SPLIT ? PER : 1][LPR];
  __shared__ float sm[SPLIT ? PER : 1][2];
  const int pair = blockIdx.y, b = pair / p.kv_heads, g = pair % p.kv_heads;
  const int run = threadIdx.x / LPR, row = SPLIT ? blockIdx.x : blockIdx.x * PER + run, at = threadIdx.x % LPR, d = at * 4;
  const Deal<P> deal(p);
  uint32_t first, count;
  deal.of(b, first, count);
  if (count == 0) {                    // (a sequence without rows)
    if (row < p.rows && (!SPLIT || run == 0)) store4<T>(out_row<T>(p, b, g, row, DH) + d, floatx4{0.f, 0.f, 0.f, 0.f});
    return;
  }
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


}  // namespace
}  // namespace forge
