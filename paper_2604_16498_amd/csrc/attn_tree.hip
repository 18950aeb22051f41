// Attention of 1 .. 64 new tokens per sequence over a cache in 16 or 32 bits, int8 or fp8, each of the new tokens seeing the
// cached rows and its own ancestors among the new ones.
//
// The G = Hq / Hkv query heads of a cache head and the n tokens are one set of G n query rows (row = token * G + head), taken in
// tiles of 16.  A block of 4 waves owns RT such tiles of one (sequence, cache head) and one range of cache rows; its waves take
// the 32-row tiles of the range in turn, and nothing but the final merge goes through LDS:
//   scores   S^T = K . Q^T (v_mfma_f32_16x16x32_bf16): K rows are the A operand, loaded from memory in its layout, 16 bytes a
//            lane (the order of the contraction is free, Q follows it).  Row r of the 16-row half f of a tile is cache row
//            8 (r / 4) + r % 4 + 4 f, so that a lane ends up with the scores of 8 consecutive cache rows for its query row ...
//   softmax  ... and with their weights as the B operand of the second product, without moving them.  Running maximum per
//            query row, held back until a tile exceeds it by 2^8 (fp32 sums have room for that, and rescaling becomes rare).
//   P . V    O^T = V^T . P^T: the lane that holds columns c (DH / 16) .. of its 8 cache rows, loaded in whole
//            pieces of the rows, forms the transposed operand with the packing that the conversion needs anyway.
// Rows in 8 bits become bf16 exactly (int8 and e4m3 both fit its 8 significant bits); their scales multiply the scores
// and the weights in fp32.  fp32 caches run the same way on v_mfma_f32_16x16x4_f32, all operands in fp32.
// Several ranges per (sequence, head): fp32 partials in the workspace, merged in range order by a second kernel.  No atomics.
#include <float.h>
#include "tree.hpp"

namespace forge {
namespace {

constexpr int TILE = 32;                  // cache rows per step of a wave
constexpr int NW = 4;                     // waves per block
constexpr int GRAIN = TILE * NW;          // ranges are multiples of this many rows
constexpr int MAX_RANGES = 64;

struct TreeParams {
  CacheView c;
  Heads q;
  char* out;
  float* part;             // [pairs, ranges, rows, DH] unnormalised outputs, then [.., 2] (maximum, sum)
  float* stat;
  const int* seq_pos;
  const uint64_t* visible;
  int q_heads, kv_heads, group, n, rows, max_pos;      // rows = group * n
  int ranges, rows_per_range, row_blocks;
  float scale_log2e;
};

// ---- how cache rows become matrix operands -------------------------------------------------------------------
// Raw: the registers of a 32-row tile.  k[f]: rows of half f in the A layout (lane = row l % 16, 16 bytes per 64 contiguous
// ones); v[i]: columns c (DH / 16) .. of row 8 (l / 16) + i, c = l % 16.
template <int BYTES, int DH>
struct Raw {
  static constexpr int KL = DH * BYTES / 64;                 // 16-byte loads per K row and lane
  static constexpr int VW = DH / 16 * BYTES / 4;             // words of a V row per lane
  u32x4 k[2][KL];
  uint32_t v[8][VW];
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

// infinities and NaN of an operand taken out: what is left, and where there was something positive or negative infinite (NaN: both)
__device__ inline bool split_bf16(uint32_t w, uint32_t& fin, uint32_t& pos, uint32_t& neg) {
  fin = pos = neg = 0;
  bool any = false;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t x = w >> (16 * i) & 0xffffu, mag = x & 0x7fffu;
    const bool bad = mag >= 0x7f80u, nan = mag > 0x7f80u;
    any |= bad;
    if (!bad) fin |= x << (16 * i);
    if (bad && (nan || !(x & 0x8000u))) pos |= 0x3f80u << (16 * i);
    if (bad && (nan || (x & 0x8000u))) neg |= 0x3f80u << (16 * i);
  }
  return any;
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
};
__device__ inline uint32_t pack_pair(float a, float b) { return pack_bf2(a, b); }
template <> struct Store<FORGE_KV_INT8, bf16> {
  static constexpr int BYTES = 1;
  static __device__ inline float byte(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }
  template <int DH> static __device__ inline bf16x8 k(const Raw<1, DH>& r, int f, int j) {
    u32x4 o;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint32_t w = r.k[f][j / 2][2 * (j & 1) + t / 2];
      o[t] = pack_pair(byte(w, 2 * (t & 1)), byte(w, 2 * (t & 1) + 1));
    }
    return __builtin_bit_cast(bf16x8, o);
  }
  template <int DH> static __device__ inline u32x4 v(const Raw<1, DH>& r, int m) {
    u32x4 o;
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = pack_pair(byte(r.v[2 * t][m / 4], m & 3), byte(r.v[2 * t + 1][m / 4], m & 3));
    return o;
  }
  static __device__ inline int q_at(int j, int kg) { return 64 * (j / 2) + 16 * kg + 8 * (j & 1); }
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
};
template <> struct Store<FORGE_KV_SAME, float> {
  static constexpr int BYTES = 4;
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

// the block's place: (range, cache head, sequence) and which RT tiles of its query rows.  Blocks go round-robin over the 8 XCDs:
// those that read the same cache rows are 8 apart, so that they share an L2.
struct Place { int range, g, b, rb; };
__device__ inline bool place_of(const TreeParams& p, int pairs, Place& at) {
  int pair = blockIdx.x, rb = 0;
  if (p.row_blocks > 1) {
    const int turn = blockIdx.x / (8 * p.row_blocks), in = blockIdx.x % (8 * p.row_blocks);
    pair = turn * 8 + in % 8;
    rb = in / 8;
    if (pair >= pairs) return false;
  }
  at.rb = rb;
  at.range = pair % p.ranges;
  at.g = pair / p.ranges % p.kv_heads;
  at.b = pair / p.ranges / p.kv_heads;
  return true;
}

template <forge_kv_type S, typename T, int DH, int RT>
__global__ __launch_bounds__(NW * 64, RT >= 4 ? 1 : 2) void attn_tree_kernel(TreeParams p, int pairs) {
  typedef Store<S, T> St;
  constexpr int BYTES = St::BYTES;
  constexpr bool F32 = sizeof(T) == 4, SCALED = S != FORGE_KV_SAME;
  constexpr int NJ = F32 ? DH / 4 : DH / 32;       // MFMAs of a score tile
  constexpr int NM = DH / 16;                      // 16-column tiles of the output
  constexpr int NBUF = F32 || RT == 4 ? 1 : 2;     // tiles in registers
  typedef Raw<BYTES, DH> R;
  constexpr int PAD = DH + 4;
  __shared__ __attribute__((aligned(16))) float sm[NW][16][PAD];
  __shared__ float sml[NW][16][2];

  Place at;
  if (!place_of(p, pairs, at)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = lane & 15, kg = lane >> 4;
  const int pos = p.seq_pos != nullptr ? min(max(p.seq_pos[at.b], 0), p.max_pos) : p.max_pos;
  const int end = pos + p.n;                                   // rows behind the last one
  const int begin = at.range * p.rows_per_range, stop = min(end, begin + p.rows_per_range);
  const int last = end - 1;

  const int64_t head = at.b * p.c.bs + at.g * p.c.hs;          // elements
  const char* kb = p.c.k + head * BYTES;
  const char* vb = p.c.v + head * BYTES;
  const float* ksb = SCALED ? p.c.ks + head / DH : nullptr;
  const float* vsb = SCALED ? p.c.vs + head / DH : nullptr;

  // query rows of this lane's column: fragments and the drafts they see
  u32x4 qf[RT][F32 ? DH / 16 : DH / 32];
  uint64_t bits[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int row = (at.rb * RT + i) * 16 + c;
    const bool real = row < p.rows;
    const int t = real ? row / p.group : 0, hh = at.g * p.group + (real ? row % p.group : 0);
    const T* qr = reinterpret_cast<const T*>(p.q.p) + at.b * p.q.bs + t * p.q.ts + hh * p.q.hs;
#pragma unroll
    for (int j = 0; j < (F32 ? DH / 16 : DH / 32); ++j) {
      u32x4 x = {0, 0, 0, 0};
      if constexpr (F32) { if (real) x = *reinterpret_cast<const u32x4*>(qr + 16 * j + 4 * kg); }
      else { if (real) x = *reinterpret_cast<const u32x4*>(qr + St::q_at(j, kg)); }
      qf[i][j] = x;
    }
    bits[i] = !real ? 0 : p.visible != nullptr ? p.visible[(int64_t)at.b * p.n + t] : (2ull << t) - 1;
  }

  R raw[NBUF];
  float ks[NBUF][SCALED ? 8 : 1], vs[NBUF][SCALED ? 8 : 1];
  auto tile_base = [&](int t) { return begin + (t * NW + wave) * TILE; };
  const int ntile = stop > begin + wave * TILE ? ceil_div(stop - begin - wave * TILE, NW * TILE) : 0;
  // rows past the end read the last one again (cut below); a tile past a wave's last one is requested, not used
  auto load_tile = [&](int t, R& r, float* ksr, float* vsr) {
    const int base = tile_base(t);
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const char* kr = kb + (int64_t)min(base + 8 * (c >> 2) + (c & 3) + 4 * f, last) * (DH * BYTES) + 16 * kg;
#pragma unroll
      for (int j = 0; j < R::KL; ++j) r.k[f][j] = *reinterpret_cast<const u32x4*>(kr + 64 * j);
    }
    if constexpr (SCALED) {
      // 8 consecutive scales; where a tile passes the end they are clamped one by one
      const int r0 = base + 8 * kg;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ksr[i] = ksb[min(r0 + i, last)];
        vsr[i] = vsb[min(r0 + i, last)];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      load_words<R::VW>(vb + (int64_t)min(base + 8 * kg + i, last) * (DH * BYTES) + c * (R::VW * 4), r.v[i]);
  };
#pragma unroll
  for (int u = 0; u < NBUF; ++u) load_tile(u, raw[u], ks[u], vs[u]);

  float m_run[RT], l_run[RT];
  floatx4 acc[RT][NM];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    m_run[i] = -FLT_MAX;
    l_run[i] = 0.f;
#pragma unroll
    for (int m = 0; m < NM; ++m) acc[i][m] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  auto step = [&](int t, R& r, const float* ksr, const float* vsr) {
    const int base = tile_base(t), first = base + 8 * kg;      // this lane's 8 cache rows
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
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        seen[i] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = first + e, d = j - pos;
          const bool sees = d < 0 || (j < end && (bits[i] >> (d & 63) & 1));
          seen[i] |= (uint32_t)sees << e;
          s[i][e] = sees ? s[i][e] : -INFINITY;
        }
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
    if constexpr (F32) {
      bool bad = false;
      if (edge)
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int m = 0; m < NM; ++m) bad |= (r.v[e][m] & 0x7fffffffu) >= 0x7f800000u;
      if (edge && __any(bad)) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int m = 0; m < NM; ++m) {
            floatx4 up = {0.f, 0.f, 0.f, 0.f}, down = up;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t x = r.v[e][m], mag = x & 0x7fffffffu;
              const bool off = mag >= 0x7f800000u, nan = mag > 0x7f800000u, sign = x >> 31;
              const float sees = seen[i] >> e & 1 ? 1.f : 0.f;
              acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(off ? 0.f : __uint_as_float(x), s[i][e], acc[i][m], 0, 0, 0);
              up = __builtin_amdgcn_mfma_f32_16x16x4f32(off && (nan || !sign) ? 1.f : 0.f, sees, up, 0, 0, 0);
              down = __builtin_amdgcn_mfma_f32_16x16x4f32(off && (nan || sign) ? 1.f : 0.f, sees, down, 0, 0, 0);
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[i][m][v] += (up[v] > 0.f ? INFINITY : 0.f) + (down[v] > 0.f ? -INFINITY : 0.f);
          }
        return;
      }
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
        u32x4 x = St::v(r, m);
        if constexpr (S != FORGE_KV_INT8) {              // (int8 codes are finite)
          if (edge) {
            u32x4 fin, up, down;
            bool bad = false;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              uint32_t a, b, d;
              bad |= split_bf16(x[w], a, b, d);
              fin[w] = a; up[w] = b; down[w] = d;
            }
            if (__any(bad)) {
#pragma unroll
              for (int i = 0; i < RT; ++i) {
                u32x4 sw;
#pragma unroll
                for (int w = 0; w < 4; ++w)
                  sw[w] = (seen[i] >> (2 * w) & 1 ? 0x3f80u : 0u) | (seen[i] >> (2 * w + 1) & 1 ? 0x3f800000u : 0u);
                const bf16x8 see = __builtin_bit_cast(bf16x8, sw);
                const floatx4 none = {0.f, 0.f, 0.f, 0.f};
                const floatx4 u = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, up), see, none, 0, 0, 0);
                const floatx4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, down), see, none, 0, 0, 0);
#pragma unroll
                for (int v = 0; v < 4; ++v)
                  acc[i][m][v] += (u[v] > 0.f ? INFINITY : 0.f) + (d[v] > 0.f ? -INFINITY : 0.f);
              }
              x = fin;
            }
          }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i)
          acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), pf[i], acc[i][m], 0, 0, 0);
      }
    }
  };

  for (int t0 = 0; t0 < ntile; t0 += NBUF) {
#pragma unroll
    for (int u = 0; u < NBUF; ++u) {
      if (t0 + u < ntile) step(t0 + u, raw[u], ks[u], vs[u]);
      load_tile(t0 + u + NBUF, raw[u], ks[u], vs[u]);
    }
  }

  // ---- the waves' shares, added in wave order, 16 query rows at a time ---------------------------------------
  const int64_t slot = (int64_t)((at.b * p.kv_heads + at.g) * p.ranges + at.range) * p.rows;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const float l = lanes_sum(l_run[i]);
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int m = 0; m < NM; m += 4)
        *reinterpret_cast<floatx4*>(&sm[wave][c][(4 * kg + v) * NM + m]) =
            floatx4{acc[i][m][v], acc[i][m + 1][v], acc[i][m + 2][v], acc[i][m + 3][v]};
    if (kg == 0) { sml[wave][c][0] = m_run[i]; sml[wave][c][1] = l; }
    lds_barrier();
    for (int idx = tid; idx < 16 * (DH / 4); idx += NW * 64) {
      const int r = idx / (DH / 4), d = idx % (DH / 4) * 4, row = (at.rb * RT + i) * 16 + r;
      if (row >= p.rows) continue;
      float mn = sml[0][r][0];
#pragma unroll
      for (int w = 1; w < NW; ++w) mn = fmaxf(mn, sml[w][r][0]);
      floatx4 o = {0.f, 0.f, 0.f, 0.f};
      float lt = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float a = __builtin_amdgcn_exp2f(sml[w][r][0] - mn);
        o += *reinterpret_cast<const floatx4*>(&sm[w][r][d]) * a;
        lt += sml[w][r][1] * a;
      }
      if (p.ranges == 1) {
        const int tok = row / p.group, hh = at.g * p.group + row % p.group;
        const float inv = lt == 0.f ? 0.f : 1.f / lt;
        store4<T>(reinterpret_cast<T*>(p.out) + (((int64_t)at.b * p.n + tok) * p.q_heads + hh) * DH + d, o * inv);
      } else {
        *reinterpret_cast<floatx4*>(p.part + (slot + row) * DH + d) = o;
        if (d == 0) { p.stat[(slot + row) * 2] = mn; p.stat[(slot + row) * 2 + 1] = lt; }
      }
    }
    lds_barrier();
  }
}

// The ranges of a query row, in range order, 8 a round trip: DH / 4 lanes a row
template <typename T, int DH>
__global__ __launch_bounds__(256) void attn_tree_merge(TreeParams p, int64_t total) {
  constexpr int LPR = DH / 4;
  const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPR;       // (sequence, cache head, row)
  if (id >= total) return;
  const int d = threadIdx.x % LPR * 4;
  const int64_t pair = id / p.rows;
  const int row = (int)(id % p.rows), g = (int)(pair % p.kv_heads);
  const int64_t b = pair / p.kv_heads;
  const int64_t first = pair * p.ranges * p.rows + row;
  float mx = -FLT_MAX, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int z0 = 0; z0 < p.ranges; z0 += 8) {
    float mz[8], lz[8];
    floatx4 oz[8];
#pragma unroll
    for (int z = 0; z < 8; ++z) {
      const int64_t at = first + (int64_t)min(z0 + z, p.ranges - 1) * p.rows;
      mz[z] = p.stat[at * 2];
      lz[z] = p.stat[at * 2 + 1];
      oz[z] = *reinterpret_cast<const floatx4*>(p.part + at * DH + d);
    }
    float mn = mx;
#pragma unroll
    for (int z = 0; z < 8; ++z) mn = fmaxf(mn, mz[z]);
    const float a = __builtin_amdgcn_exp2f(mx - mn);
    mx = mn;
    l *= a;
    o *= a;
#pragma unroll
    for (int z = 0; z < 8; ++z)
      if (z0 + z < p.ranges) {
        const float w = __builtin_amdgcn_exp2f(mz[z] - mn);
        l += lz[z] * w;
        o += oz[z] * w;
      }
  }
  const int hh = g * p.group + row % p.group, tok = row / p.group;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  store4<T>(reinterpret_cast<T*>(p.out) + ((b * p.n + tok) * p.q_heads + hh) * DH + d, o * inv);
}

// ---- how the work is cut ---------------------------------------------------------------------------------------
// 16-row tiles of query rows per block
inline int tiles_per_block(int rows, bool f32) { return f32 || rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }
inline int most_ranges(int64_t blocks, int len, int rt) {
  const int64_t want = (rt == 4 ? 1 : 2) * (int64_t)compute_units();
  const int64_t by_blocks = want / blocks, by_rows = len / 256;
  const int64_t r = by_blocks < by_rows ? by_blocks : by_rows;
  return (int)(r < 1 ? 1 : r > MAX_RANGES ? MAX_RANGES : r);
}

struct TreePlan { int rt, row_blocks, ranges, rows_per_range; };
TreePlan plan_tree(int batch, int q_heads, int kv_heads, int n, int len, bool f32) {
  TreePlan pl;
  const int rows = q_heads / kv_heads * n;
  pl.rt = tiles_per_block(rows, f32);
  pl.row_blocks = ceil_div(rows, 16 * pl.rt);
  const int most = most_ranges((int64_t)batch * kv_heads * pl.row_blocks, len, pl.rt);
  pl.rows_per_range = ceil_div(ceil_div(len, most), GRAIN) * GRAIN;
  pl.ranges = ceil_div(len, pl.rows_per_range);
  return pl;
}

template <forge_kv_type S, typename T, int DH>
void launch_rt(const TreeParams& p, const TreePlan& pl, int pairs, hipStream_t s) {
  const unsigned blocks = pl.row_blocks > 1 ? (unsigned)(ceil_div(pairs, 8) * 8 * pl.row_blocks) : (unsigned)pairs;
  if (pl.rt == 1) attn_tree_kernel<S, T, DH, 1><<<blocks, NW * 64, 0, s>>>(p, pairs);
  if constexpr (sizeof(T) == 2) {
    if (pl.rt == 2) attn_tree_kernel<S, T, DH, 2><<<blocks, NW * 64, 0, s>>>(p, pairs);
    if (pl.rt == 4) attn_tree_kernel<S, T, DH, 4><<<blocks, NW * 64, 0, s>>>(p, pairs);
  }
}
template <forge_kv_type S, typename T>
void launch_dh(const TreeParams& p, const TreePlan& pl, int pairs, int head_dim, hipStream_t s) {
  if (head_dim == 64) launch_rt<S, T, 64>(p, pl, pairs, s);
  else launch_rt<S, T, 128>(p, pl, pairs, s);
}
template <typename T>
void launch_merge(const TreeParams& p, int64_t total, int head_dim, hipStream_t s) {
  const unsigned blocks = (unsigned)ceil_div64(total * (head_dim / 4), 256);
  if (head_dim == 64) attn_tree_merge<T, 64><<<blocks, 256, 0, s>>>(p, total);
  else attn_tree_merge<T, 128><<<blocks, 256, 0, s>>>(p, total);
}

}  // namespace

// room for the ranges of any shorter cache too: their number only falls with the length
size_t attn_tree_workspace_bytes(int batch, int q_heads, int kv_heads, int head_dim, int n, int max_pos, bool f32) {
  const int rows = q_heads / kv_heads * n, rt = tiles_per_block(rows, f32);
  const int most = most_ranges((int64_t)batch * kv_heads * ceil_div(rows, 16 * rt), max_pos + n, rt);
  return most > 1 ? (size_t)batch * kv_heads * most * rows * (head_dim + 2) * sizeof(float) : 0;
}

forge_status launch_attn_tree(const TreeArgs& a, hipStream_t s) {
  const TreePlan pl = plan_tree(a.batch, a.q_heads, a.kv_heads, a.n, a.max_pos + a.n, a.dt == FORGE_F32);
  TreeParams p;
  p.c = a.c;
  p.q = a.q;
  p.out = (char*)a.out;
  p.seq_pos = a.seq_pos;
  p.visible = a.visible;
  p.q_heads = a.q_heads;
  p.kv_heads = a.kv_heads;
  p.group = a.q_heads / a.kv_heads;
  p.n = a.n;
  p.rows = p.group * a.n;
  p.max_pos = a.max_pos;
  p.ranges = pl.ranges;
  p.rows_per_range = pl.rows_per_range;
  p.row_blocks = pl.row_blocks;
  p.scale_log2e = a.scale * 1.4426950408889634f;
  const int pairs = a.batch * a.kv_heads * pl.ranges;
  p.part = (float*)a.workspace;
  p.stat = p.part + (int64_t)pairs * p.rows * a.head_dim;
  if (a.dt == FORGE_F32) launch_dh<FORGE_KV_SAME, float>(p, pl, pairs, a.head_dim, s);
  else if (a.type == FORGE_KV_SAME) launch_dh<FORGE_KV_SAME, bf16>(p, pl, pairs, a.head_dim, s);
  else if (a.type == FORGE_KV_INT8) launch_dh<FORGE_KV_INT8, bf16>(p, pl, pairs, a.head_dim, s);
  else launch_dh<FORGE_KV_FP8, bf16>(p, pl, pairs, a.head_dim, s);
  if (pl.ranges == 1) return launch_status();
  if (hipGetLastError() != hipSuccess) return FORGE_ERR_HIP;
  const int64_t total = (int64_t)a.batch * a.kv_heads * p.rows;
  if (a.dt == FORGE_F32) launch_merge<float>(p, total, a.head_dim, s);
  else launch_merge<bf16>(p, total, a.head_dim, s);
  return launch_status();
}

}  // namespace forge
