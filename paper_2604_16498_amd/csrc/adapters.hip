// Low-rank adapters of many requests: y = base + scale * B (A x) per row, the row's own A and B.
//
// Two launches: t = A x into fp32 planes (K in `splits` ranges), then y from their sum in order.  Both work on tiles of 16 rows of x with
// matrix instructions, one adapter of a tile at a time: rows of other requests are multiplied along, their results dropped (so that no
// infinity of one request's adapter reaches another's rows).  Neighbours in a batch of requests have different adapters, so a tile's adapters are dealt
// over blocks (`lanes`) where there are few tiles; the rows of a prompt share one, and blocks then take several tiles.
// An adapter is read once per tile that has it, which is what bounds a decode step; the rows of x, base and y bound a prompt.
#include "paged.hpp"

namespace forge {
namespace {

constexpr int JT = 4;          // 16-wide tiles of the inner index a block works on
constexpr int COLS = 256;      // columns of y per block, 64 a wave

// Operands of 16 rows x 64 bytes: lane l has 16 bytes of row l % 16 at 16 (l / 16)
template <typename T> struct Mma;
template <> struct Mma<bf16> {
  static constexpr int STEP = 32;          // elements of 64 bytes
  static __device__ inline floatx4 go(u32x4 a, u32x4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mma<float> {
  static constexpr int STEP = 16;
  static __device__ inline floatx4 go(u32x4 a, u32x4 b, floatx4 c) {      // (the order of a contraction is free)
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
    return c;
  }
};

// The adapters of a block's rows (at most 64, one a lane): the lanes that are the first with theirs
struct Rows {
  int id;                // of this lane's row, -1: none
  uint64_t leaders;
  __device__ inline Rows(const AdapterArgs& p, int64_t m0, int rows) {
    const int lane = threadIdx.x & 63;
    id = lane < rows && m0 + lane < p.M ? p.ids[m0 + lane] : -1;
    if ((uint32_t)id >= (uint32_t)p.n_adapters) id = -1;
    bool first = id >= 0;
    for (int j = 0; j < rows; ++j) first = first && !(j < lane && __builtin_amdgcn_readlane(id, j) == id);
    leaders = __ballot(first);
  }
};

struct Cut { int tiles, splits, chunks, lanes; };

// t of 16 RT rows and 64 inner columns over one range of K, shared out among the waves 128 bytes of a row at a time
template <typename T, int RT>
__global__ __launch_bounds__(256, RT == 1 ? 4 : 2) void adapters_inner_kernel(AdapterArgs p, Cut cut) {
  typedef Mma<T> M;
  constexpr int UNIT = 2 * M::STEP;
  __shared__ __attribute__((aligned(16))) floatx4 red[4][RT][JT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, kg = lane >> 4;
  const int inner = p.parts * p.rank;
  const int64_t m0 = (int64_t)blockIdx.x * (16 * RT);
  const int split = blockIdx.y / cut.chunks, j0 = blockIdx.y % cut.chunks * (16 * JT);
  const Rows rows(p, m0, 16 * RT);
  const int units = ceil_div(p.K, UNIT);
  const int u0 = (int)((int64_t)units * split / cut.splits), u1 = (int)((int64_t)units * (split + 1) / cut.splits);
  const T* xr[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int64_t m = m0 + 16 * i + c;
    xr[i] = reinterpret_cast<const T*>(p.x) + (m < p.M ? m : p.M - 1) * p.K + kg * (16 / (int)sizeof(T));
  }
  uint64_t left = rows.leaders;
  for (int s = 0; left != 0; ++s, left &= left - 1) {
    if (s % cut.lanes != (int)blockIdx.z) continue;
    const int id = __builtin_amdgcn_readlane(rows.id, __ffsll((unsigned long long)left) - 1);
    const T* ar[JT];
#pragma unroll
    for (int j = 0; j < JT; ++j) {
      const int at = j0 + 16 * j + c;
      ar[j] = reinterpret_cast<const T*>(p.a) + ((int64_t)id * inner + (at < inner ? at : inner - 1)) * p.K + kg * (16 / (int)sizeof(T));
    }
    floatx4 acc[RT][JT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < JT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    u32x4 xf[2][RT][2], af[2][JT][2];
    auto load = [&](int u, int buf) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = u * UNIT + h * M::STEP;
        const bool in = k + kg * (16 / (int)sizeof(T)) < p.K;
        const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < RT; ++i) xf[buf][i][h] = in ? *reinterpret_cast<const u32x4*>(xr[i] + k) : zero;
#pragma unroll
        for (int j = 0; j < JT; ++j)
          if (j0 + 16 * j < inner) af[buf][j][h] = in ? *reinterpret_cast<const u32x4*>(ar[j] + k) : zero;
      }
    };
    auto multiply = [&](int buf) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < JT; ++j)
          if (j0 + 16 * j < inner)
#pragma unroll
            for (int i = 0; i < RT; ++i) acc[i][j] = M::go(af[buf][j][h], xf[buf][i][h], acc[i][j]);
    };
    int u = u0 + wave;
    if (u < u1) load(u, 0);
    for (; u < u1; u += 8) {
      if (u + 4 < u1) load(u + 4, 1);
      multiply(0);
      if (u + 8 < u1) load(u + 8, 0);
      if (u + 4 < u1) multiply(1);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < JT; ++j) red[wave][i][j][lane] = acc[i][j];
    lds_barrier();
    const int at = j0 + 16 * wave + 4 * kg;                    // a wave adds up one tile: 4 inner indices of a row a lane
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const floatx4 t = red[0][i][wave][lane] + red[1][i][wave][lane] + red[2][i][wave][lane] + red[3][i][wave][lane];
      const int mine = __shfl(rows.id, 16 * i + c, 64);
      if (mine == id && at < inner)
        *reinterpret_cast<floatx4*>(reinterpret_cast<float*>(p.workspace) + ((int64_t)split * p.M + m0 + 16 * i + c) * inner + at) = t;
    }
    lds_barrier();
  }
}

// 16 consecutive elements of a row as fp32
template <typename T>
__device__ inline void load16(const T* p, float (&v)[16]) {
  float a[8], b[8];
  Vec8<T>::load(p, a);
  Vec8<T>::load(p + 8, b);
#pragma unroll
  for (int i = 0; i < 8; ++i) { v[i] = a[i]; v[8 + i] = b[i]; }
}
template <typename T>
__device__ inline void store16(T* p, const float (&v)[16]) {
  float a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { a[i] = v[i]; b[i] = v[8 + i]; }
  Vec8<T>::store(p, a);
  Vec8<T>::store(p + 8, b);
}

// y of 16 RT rows and 64 columns a wave.  The rows of b in tile i of its 64 columns are 16 (r / 4) + 4 i + r % 4, so that a lane ends up with 16
// consecutive columns of its row.  bf16: t as the sum of two bf16 numbers, 16 bits of it, in two products.  NS: steps of the rank.
template <typename T, int RT, int NS>
__global__ __launch_bounds__(256, 2) void adapters_outer_kernel(AdapterArgs p, Cut cut) {
  typedef Mma<T> M;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int PER = 16 / sizeof(T);      // elements of a lane's 16 bytes
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, kg = lane >> 4;
  const int inner = p.parts * p.rank;
  const int chunks = ceil_div(p.N, COLS);
  const int64_t m0 = (int64_t)(blockIdx.x / chunks) * (16 * RT);
  const int n0 = blockIdx.x % chunks * COLS + 64 * wave;
  if (n0 >= p.N) return;
  const Rows rows(p, m0, 16 * RT);
  const bool whole = n0 + 16 * kg + 16 <= p.N && p.ldy % 8 == 0;       // this lane's 16 columns, at addresses for wide accesses
  auto finish = [&](int i, const float (&add)[16], const float (&old)[16]) {
    const int64_t at = (m0 + 16 * i + c) * p.ldy + n0 + 16 * kg;
    T* y = reinterpret_cast<T*>(p.y) + at;
    if (whole) {
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = old[e] + add[e];
      store16<T>(y, v);
    } else {
      const T* b = reinterpret_cast<const T*>(p.base) + at;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (n0 + 16 * kg + e < p.N) y[e] = from_f32<T>(to_f32<T>(b[e]) + add[e]);
    }
  };
  auto old_of = [&](int i, float (&old)[16]) {
    if (whole) load16<T>(reinterpret_cast<const T*>(p.base) + (m0 + 16 * i + c) * p.ldy + n0 + 16 * kg, old);
  };
  if (blockIdx.y == 0 && p.y != p.base) {                      // rows without an adapter
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int mine = __shfl(rows.id, 16 * i + c, 64);
      if (mine >= 0 || m0 + 16 * i + c >= p.M) continue;
      const float none[16] = {};
      float old[16];
      old_of(i, old);
      finish(i, none, old);
    }
  }
  int part0 = 0, part1 = 0;                                    // the parts that these columns belong to
  const int last = min(n0 + 63, p.N - 1);
  while (n0 >= p.part_end[part0]) ++part0;
  while (last >= p.part_end[part1]) ++part1;
  int my_part = part0;                                         // of this lane's 16 columns
  while (my_part < part1 && n0 + 16 * kg >= p.part_end[my_part]) ++my_part;

  uint64_t left = rows.leaders;
  for (int s = 0; left != 0; ++s, left &= left - 1) {
    if (s % cut.lanes != (int)blockIdx.y) continue;
    const int id = __builtin_amdgcn_readlane(rows.id, __ffsll((unsigned long long)left) - 1);
    const float scale = p.scale != nullptr ? p.scale[id] : 1.f;
    u32x4 bf[4][NS];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = min(n0 + 16 * (c >> 2) + 4 * i + (c & 3), p.N - 1);
      const T* b = reinterpret_cast<const T*>(p.b) + ((int64_t)id * p.N + n) * p.rank;
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const int r = st * M::STEP + kg * PER;
        bf[i][st] = r < p.rank ? *reinterpret_cast<const u32x4*>(b + r) : u32x4{0, 0, 0, 0};
      }
    }
#pragma unroll 1
    for (int part = part0; part <= part1; ++part) {
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const int mine = __shfl(rows.id, 16 * i + c, 64);
        const bool here = mine == id && part == my_part;
        if (__ballot(mine == id) == 0) continue;
        float old[16];
        if (here) old_of(i, old);
        const int64_t m = m0 + 16 * i + c;
        const float* t0 = reinterpret_cast<const float*>(p.workspace) + (mine == id ? m : m0 + __ffsll((unsigned long long)left) - 1) * inner + part * p.rank;
        floatx4 acc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
        float t[NS][PER];
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
          for (int e = 0; e < PER; ++e) t[st][e] = 0.f;
        for (int z = 0; z < cut.splits; ++z) {
          const float* tz = t0 + (int64_t)z * p.M * inner;
#pragma unroll
          for (int st = 0; st < NS; ++st) {
            const int r = st * M::STEP + kg * PER;
            if (r < p.rank)
#pragma unroll
              for (int e = 0; e < PER; e += 4) {
                const floatx4 v = *reinterpret_cast<const floatx4*>(tz + r + e);
#pragma unroll
                for (int q = 0; q < 4; ++q) t[st][e + q] += v[q];
              }
          }
        }
#pragma unroll
        for (int st = 0; st < NS; ++st) {
          u32x4 hi, lo;
          if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) hi[e] = __float_as_uint(t[st][e] * scale);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float a = t[st][2 * e] * scale, b = t[st][2 * e + 1] * scale;
              hi[e] = pack_bf2(a, b);
              lo[e] = pack_bf2(a - bf_lo(hi[e]), b - bf_hi(hi[e]));
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            acc[j] = M::go(bf[j][st], hi, acc[j]);
            if constexpr (!F32) acc[j] = M::go(bf[j][st], lo, acc[j]);
          }
        }
        if (here) {
          float add[16];
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) add[4 * j + e] = acc[j][e];
          finish(i, add, old);
        }
      }
    }
  }
}

// Blocks of one tile until two rounds of the chip are full of tiles; K in ranges of 4 units (one a wave) at least
Cut cut_of(int M, int K, int inner, forge_dtype dt, int rt) {
  const int cus = compute_units(), units = ceil_div(K, dt == FORGE_BF16 ? 64 : 32);
  Cut c;
  c.tiles = ceil_div(M, 16 * rt);
  c.chunks = ceil_div(inner, 16 * JT);
  const int64_t blocks = (int64_t)c.tiles * c.chunks;
  const int want = (int)ceil_div64(2 * cus, blocks), most = units < 4 ? 1 : units / 4;
  c.splits = want < 1 ? 1 : want < most ? want : most;
  c.lanes = 1;
  return c;
}
int tiles_per_block(int M) { return M >= 1024 ? 4 : 1; }

template <typename T, int RT>
forge_status launch_rt(const AdapterArgs& a, hipStream_t s) {
  const int cus = compute_units(), inner = a.parts * a.rank;
  Cut c = cut_of(a.M, a.K, inner, a.dt, RT);
  auto lanes = [&](int64_t blocks) {                           // a tile of 16 rows has at most 16 adapters
    const int64_t l = ceil_div64(8 * cus, blocks);
    const int most = RT > 1 ? 1 : a.M < 16 ? a.M : 16;
    return (int)(l < 1 ? 1 : l < most ? l : most);
  };
  c.lanes = lanes((int64_t)c.tiles * c.chunks * c.splits);
  adapters_inner_kernel<T, RT><<<dim3(c.tiles, c.chunks * c.splits, c.lanes), 256, 0, s>>>(a, c);
  if (hipGetLastError() != hipSuccess) return FORGE_ERR_HIP;
  const int64_t blocks = (int64_t)c.tiles * ceil_div(a.N, COLS);
  c.lanes = lanes(blocks);
  const dim3 grid((unsigned)blocks, c.lanes);
  const int steps = ceil_div(a.rank, Mma<T>::STEP);
  if (steps == 1) adapters_outer_kernel<T, RT, 1><<<grid, 256, 0, s>>>(a, c);
  else if (steps == 2) adapters_outer_kernel<T, RT, 2><<<grid, 256, 0, s>>>(a, c);
  else if (steps <= 4) adapters_outer_kernel<T, RT, 4><<<grid, 256, 0, s>>>(a, c);
  else adapters_outer_kernel<T, RT, 8><<<grid, 256, 0, s>>>(a, c);
  return launch_status();
}
template <typename T>
forge_status launch(const AdapterArgs& a, hipStream_t s) {
  return tiles_per_block(a.M) == 4 ? launch_rt<T, 4>(a, s) : launch_rt<T, 1>(a, s);
}

}  // namespace

// Room for any smaller M too: of m rows in `tiles` tiles the planes are at most units / 4, and at most 2 cus / (tiles chunks) + 1, times m rows
size_t adapters_workspace_bytes(int M, int N, int K, int rank, int parts, forge_dtype dt) {
  const int inner = parts * rank, rt = tiles_per_block(M), units = ceil_div(K, dt == FORGE_BF16 ? 64 : 32);
  const int64_t most = (int64_t)(units < 4 ? 1 : units / 4) * M;
  const int64_t full = ceil_div(2 * compute_units() * 16 * rt, ceil_div(inner, 16 * JT)) + (int64_t)M;
  return (size_t)(most < full ? most : full) * inner * sizeof(float);
}

forge_status launch_adapters(const AdapterArgs& a, hipStream_t s) {
  return a.dt == FORGE_F32 ? launch<float>(a, s) : launch<bf16>(a, s);
}

}  // namespace forge
