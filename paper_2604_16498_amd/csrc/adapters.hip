// Low-rank adapters of many requests: y = base + scale * B (A x) per row, the row's own A and B.
//
// Two launches: t = A x into fp32 planes (K in `splits` ranges), then y from their sum in order.  Both work on tiles of 16 rows of x with
// matrix instructions, one adapter of a tile at a time: rows of other requests are multiplied along, their results dropped (so that no
// infinity of one request's adapter reaches another's rows).  Neighbours in a batch of requests have different adapters, so a tile's adapters are dealt
// over blocks (`lanes`) where there are few tiles; the rows of a prompt share one, and blocks then take 64 of them.
// An adapter is read once per tile that has it: with the chain adapter number, adapter, sum of each launch that bounds a decode step (61 rows, 49 adapters
// of rank 16 beside q, k and v of 4096: 8 + 8 us for 19 + 10 MB of adapters).  The rows of x, base and y bound a prompt (4096 rows of 5 requests, rank 64,
// 4096 x 4096: 15.8 + 21.3 us for 34 + 67 MB; one row of 768 in fp32 4.4 + 4.6).
#include "paged.hpp"
#include "adapters_plan.hpp"

namespace forge {
namespace {

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
  // what a block asks for first (a wait is for everything that was asked for before)
  static __device__ inline int request(const AdapterArgs& p, int64_t m0, int rows) {
    const int lane = threadIdx.x & 63;
    return lane < rows && m0 + lane < p.M ? p.ids[m0 + lane] : -1;
  }
  __device__ inline Rows(const AdapterArgs& p, int requested) : id(requested) {
    if ((uint32_t)id >= (uint32_t)p.n_adapters) id = -1;
    uint64_t todo = __ballot(id >= 0);
    leaders = 0;
    while (todo != 0) {                  // (an adapter a turn)
      const int l = __ffsll((unsigned long long)todo) - 1;
      leaders |= 1ull << l;
      todo &= ~__ballot(id == __builtin_amdgcn_readlane(id, l));
    }
  }
};

// t of 16 RT rows and 64 inner columns over one range of K, in units of 512 bytes a row: a load of a block is 8 rows x 512 bytes (a kernel that only
// read 4096 rows of 8 KB took 7.9 us so, 12.0 in lines of 128 bytes), two units of x and of the adapter are on their way in registers, and a unit
// goes through LDS.  Wave w multiplies inner columns 16 w .. with all rows.
template <typename T, int RT>
__global__ __launch_bounds__(256, 2) void adapters_inner_kernel(AdapterArgs p, Cut cut) {
  typedef Mma<T> M;
  constexpr int PER = 16 / sizeof(T), UNIT = 32 * PER, ROW = 528, XN = 2 * RT, AN = 2 * JT;      // (rows 16 bytes apart in the banks)
  __shared__ __attribute__((aligned(16))) char lds[(16 * RT + 16 * JT) * ROW];                   // rows of x, then of the adapter
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, kg = lane >> 4;
  const int inner = p.parts * p.rank, line = tid >> 5, at16 = (tid & 31) * PER;
  const int64_t m0 = (int64_t)blockIdx.x * (16 * RT);
  const int split = blockIdx.y / cut.chunks, j0 = blockIdx.y % cut.chunks * (16 * JT);
  const int tiles = min(JT, ceil_div(inner - j0, 16));                   // of the inner index that there are here
  const int units = ceil_div(p.K, UNIT);
  const int u0 = (int)((int64_t)units * split / cut.splits), u1 = (int)((int64_t)units * (split + 1) / cut.splits);
  const T* xs[XN];
#pragma unroll
  for (int i = 0; i < XN; ++i) {
    const int64_t m = m0 + 8 * i + line;
    xs[i] = reinterpret_cast<const T*>(p.x) + (m < p.M ? m : p.M - 1) * p.K;
  }
  u32x4 xf[2][XN], af[2][AN];
  auto offset = [&](int u) { return min(u * UNIT + at16, p.K - PER); };  // (what lies past the end of K is 0 in LDS)
  auto load_x = [&](int u, u32x4 (&r)[XN]) {
    const int k = offset(u);
#pragma unroll
    for (int i = 0; i < XN; ++i) r[i] = *reinterpret_cast<const u32x4*>(xs[i] + k);
  };
  int ids = 0;                             // (ahead of x where x is long; few rows wait less for x first: 61 rows 15.5 | 15.9 us)
  if (RT > 1) ids = Rows::request(p, m0, 16 * RT);
  bool again = blockIdx.z > 0;             // x not requested yet: few tiles have many adapters
  if (!again) {
    load_x(u0, xf[0]);
    if (u0 + 1 < u1) load_x(u0 + 1, xf[1]);
  }
  if (RT == 1) ids = Rows::request(p, m0, 16);
  const Rows rows(p, ids);
  uint64_t left = rows.leaders;
  for (int s = 0; left != 0; ++s, left &= left - 1) {
    if (s % cut.lanes != (int)blockIdx.z) continue;
    const int id = __builtin_amdgcn_readlane(rows.id, __ffsll((unsigned long long)left) - 1);
    const T* as[AN];
#pragma unroll
    for (int i = 0; i < AN; ++i) as[i] = reinterpret_cast<const T*>(p.a) + ((int64_t)id * inner + min(j0 + 8 * i + line, inner - 1)) * p.K;
    auto load_a = [&](int u, u32x4 (&r)[AN]) {
      const int k = offset(u);
#pragma unroll
      for (int i = 0; i < AN; ++i)
        if (i < 2 * tiles) r[i] = *reinterpret_cast<const u32x4*>(as[i] + k);
    };
    load_a(u0, af[0]);
    if (again) load_x(u0, xf[0]);
    if (u0 + 1 < u1) {
      load_a(u0 + 1, af[1]);
      if (again) load_x(u0 + 1, xf[1]);
    }
    again = true;
    floatx4 acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto step = [&](int u, u32x4 (&x)[XN], u32x4 (&a)[AN]) {
      const bool in = u * UNIT + at16 < p.K;
      char* const to = lds + line * ROW + (tid & 31) * 16;
      const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < XN; ++i) *reinterpret_cast<u32x4*>(to + 8 * i * ROW) = in ? x[i] : zero;
#pragma unroll
      for (int i = 0; i < AN; ++i)
        if (i < 2 * tiles) *reinterpret_cast<u32x4*>(to + (16 * RT + 8 * i) * ROW) = in ? a[i] : zero;
      if (u + 2 < u1) {
        load_x(u + 2, x);
        load_a(u + 2, a);
      }
      lds_barrier();
      if (wave < tiles) {
        const char* const from = lds + c * ROW + kg * 16;
#pragma unroll
        for (int h = 0; h < 8; ++h) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(from + (16 * RT + 16 * wave) * ROW + h * 64);
#pragma unroll
          for (int i = 0; i < RT; ++i) acc[i] = M::go(w, *reinterpret_cast<const u32x4*>(from + 16 * i * ROW + h * 64), acc[i]);
        }
      }
      lds_barrier();
    };
    for (int u = u0; u < u1; u += 2) {
      step(u, xf[0], af[0]);
      if (u + 1 < u1) step(u + 1, xf[1], af[1]);
    }
    const int at = j0 + 16 * wave + 4 * kg;                    // 4 inner indices of a row a lane
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int mine = __shfl(rows.id, 16 * i + c, 64);
      if (mine == id && at < inner)
        *reinterpret_cast<floatx4*>(reinterpret_cast<float*>(p.workspace) + ((int64_t)split * p.M + m0 + 16 * i + c) * inner + at) = acc[i];
    }
  }
}

// 4 elements of a row of y
template <typename T> struct Four;
template <> struct Four<float> {
  typedef u32x4 type;
  static __device__ inline u32x4 added(u32x4 w, const floatx4& v) { return __builtin_bit_cast(u32x4, __builtin_bit_cast(floatx4, w) + v); }
};
template <> struct Four<bf16> {
  typedef u32x2 type;
  static __device__ inline u32x2 added(u32x2 w, const floatx4& v) {
    return u32x2{pack_bf2(bf_lo(w[0]) + v[0], bf_hi(w[0]) + v[1]), pack_bf2(bf_lo(w[1]) + v[2], bf_hi(w[1]) + v[3])};
  }
};

// t of ROWS rows of one part, added up over the ranges: fours of a row's inner indices, thread q % 256 has four q
template <typename T, int NS, int ROWS>
struct Inner {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int QUADS = NS * (Mma<T>::STEP / 4), ALL = ROWS * QUADS, EACH = (ALL + 255) / 256;
  static constexpr int ROW = NS * 64 + 16, PLANE = ROWS * ROW, BYTES = (F32 ? 1 : 2) * PLANE;      // in LDS (rows apart in the banks)
  floatx4 t[EACH];
  static __device__ inline bool mine(const AdapterArgs& p, int q) { return q < ALL && q % QUADS < p.rank / 4; }
  static __device__ inline const float* first_range(const AdapterArgs& p, int64_t m0, int rows_left, int part, int q) {
    return reinterpret_cast<const float*>(p.workspace) + (m0 + min(q / QUADS, rows_left - 1)) * (p.parts * p.rank) + part * p.rank + 4 * (q % QUADS);
  }
  __device__ inline void load(const AdapterArgs& p, int splits, int64_t m0, int rows_left, int part) {
    const int64_t plane = (int64_t)p.M * p.parts * p.rank;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int q = (int)threadIdx.x + 256 * i;
      t[i] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (!mine(p, q)) continue;
      const float* from = first_range(p, m0, rows_left, part, q);
      constexpr int AT_ONCE = EACH > 2 ? 4 : 8;
      for (int z = 0; z < splits; z += AT_ONCE) {
        floatx4 v[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
          if (z + k < splits) v[k] = *reinterpret_cast<const floatx4*>(from + (z + k) * plane);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
          if (z + k < splits) t[i] += v[k];
      }
    }
  }
  // bf16: as the sum of two bf16 numbers, 16 bits of it
  template <typename Scale>
  __device__ inline void store(char* lds, Scale scale) const {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int q = (int)threadIdx.x + 256 * i;
      if (q >= ALL) continue;
      const floatx4 v = t[i] * scale(q / QUADS);
      char* to = lds + q / QUADS * ROW + q % QUADS * (int)(4 * sizeof(T));
      if constexpr (F32) *reinterpret_cast<floatx4*>(to) = v;
      else {
        const u32x2 hi = {pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
        *reinterpret_cast<u32x2*>(to) = hi;
        // (an infinity has no second part: it would take it back)
        auto rest = [](float v, float hi) { return fabsf(hi) < INFINITY ? v - hi : 0.f; };
        *reinterpret_cast<u32x2*>(to + PLANE) = u32x2{pack_bf2(rest(v[0], bf_lo(hi[0])), rest(v[1], bf_hi(hi[0]))),
                                                      pack_bf2(rest(v[2], bf_lo(hi[1])), rest(v[3], bf_hi(hi[1])))};
      }
    }
  }
};

// The same in two: requested, and added up once what is requested next is under way (4096 x 4096, rank 64: 39.2 | 36.6 us for both launches; blocks of
// 16 rows lose by it what the registers cost, 61 rows 15.5 | 16.4 us)
template <typename T, int NS, int ROWS>
struct InnerAhead : Inner<T, NS, ROWS> {
  typedef Inner<T, NS, ROWS> I;
  static constexpr int FIRST = I::EACH > 4 ? 1 : I::EACH == 4 && NS == 4 ? 2 : 4;      // ranges at once, as registers allow
  floatx4 v[I::EACH][FIRST];
  const float* from[I::EACH];
  __device__ inline void ranges(const AdapterArgs& p, int splits, int z) {
    const int64_t plane = (int64_t)p.M * p.parts * p.rank;
#pragma unroll
    for (int k = 0; k < FIRST; ++k)
      if (z + k < splits) {
#pragma unroll
        for (int i = 0; i < I::EACH; ++i)
          if (I::mine(p, (int)threadIdx.x + 256 * i)) v[i][k] = *reinterpret_cast<const floatx4*>(from[i] + (z + k) * plane);
      }
  }
  __device__ inline void request(const AdapterArgs& p, int splits, int64_t m0, int part) {
#pragma unroll
    for (int i = 0; i < I::EACH; ++i) from[i] = I::first_range(p, m0, ROWS, part, (int)threadIdx.x + 256 * i);
    ranges(p, splits, 0);
  }
  __device__ inline void sum(const AdapterArgs& p, int splits) {
#pragma unroll
    for (int i = 0; i < I::EACH; ++i) this->t[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int z = 0; z < splits; z += FIRST) {
      if (z > 0) ranges(p, splits, z);
#pragma unroll
      for (int k = 0; k < FIRST; ++k)
        if (z + k < splits) {
#pragma unroll
          for (int i = 0; i < I::EACH; ++i)
            if (I::mine(p, (int)threadIdx.x + 256 * i)) this->t[i] += v[i][k];
        }
    }
  }
};

// Column c of product j is column 4 c + j of a wave's 64, so that a lane ends up with 4 columns of four rows and a wave's accesses to base and y are
// whole lines: rows n0 + 4 c + j of b, 16 bytes of a step at 16 (l / 16).
template <typename T, int NS>
__device__ inline void load_b(u32x4 (&bf)[4][NS], const AdapterArgs& p, int id, int n0) {
  const int c = threadIdx.x & 15, kg = threadIdx.x >> 4 & 3;
  constexpr int PER = 16 / sizeof(T), STEP = Mma<T>::STEP;
  const T* const bm = reinterpret_cast<const T*>(p.b) + (int64_t)id * p.N * p.rank;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const T* b = bm + (int64_t)min(n0 + 4 * c + j, p.N - 1) * p.rank;
#pragma unroll
    for (int st = 0; st < NS; ++st) {
      const int r = st * STEP + kg * PER;
      bf[j][st] = *reinterpret_cast<const u32x4*>(b + (r < p.rank ? r : 0));
    }
  }
}
// (inner indices past the rank: t is 0 there, and an infinity must not meet it)
template <typename T, int NS>
__device__ inline void trim_b(u32x4 (&bf)[4][NS], int rank) {
  const int kg = threadIdx.x >> 4 & 3;
  constexpr int PER = 16 / sizeof(T), STEP = Mma<T>::STEP;
  if (rank == NS * STEP) return;
#pragma unroll
  for (int st = NS / 2; st < NS; ++st)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) bf[j][st][e] = st * STEP + kg * PER < rank ? bf[j][st][e] : 0u;
}
template <typename T, int NS, int ROWS>
__device__ inline void products(floatx4 (&acc)[4], const u32x4 (&bf)[4][NS], const char* lds, int tile) {
  typedef Inner<T, NS, ROWS> I;
  const int c = threadIdx.x & 15, kg = threadIdx.x >> 4 & 3;
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int st = 0; st < NS; ++st) {
    const char* from = lds + (16 * tile + c) * I::ROW + st * 64 + kg * 16;
#pragma unroll
    for (int h = 0; h < (I::F32 ? 1 : 2); ++h) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(from + h * I::PLANE);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = Mma<T>::go(x, bf[j][st], acc[j]);
    }
  }
}

// y of 16 rows from m0 on and columns b0 .. b1 - 1, 64 a wave at a time; of the rows' adapters every `lanes`-th from `lane0` on
template <typename T, int NS>
__device__ inline void outer_rows(const AdapterArgs& p, const Cut& cut, int lanes, int lane0, int64_t m0, int b0, int b1, char* tl) {
  typedef typename Four<T>::type F;
  typedef Inner<T, NS, 16> I;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, kg = lane >> 4;
  const int rows_left = (int)min((int64_t)16, p.M - m0);
  int part0 = 0, part1 = 0;                                    // the parts that these columns belong to
  while (b0 >= p.part_end[part0]) ++part0;
  while (b1 - 1 >= p.part_end[part1]) ++part1;
  I t;
  t.load(p, cut.splits, m0, rows_left, part0);
  int have = part0;
  const Rows rows(p, Rows::request(p, m0, 16));
  const T* const base = reinterpret_cast<const T*>(p.base) + m0 * p.ldy;
  T* const y = reinterpret_cast<T*>(p.y) + m0 * p.ldy;
  const bool wide = p.ldy % 4 == 0;        // rows at addresses for wide accesses
  if (lane0 == 0 && p.y != p.base) {                           // rows without an adapter
    const uint32_t none = (uint32_t)__ballot(rows.id < 0) & ((1u << rows_left) - 1);
    for (int n = b0 + 4 * lane; n < b1; n += 256) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t at = (int64_t)(4 * i + wave) * p.ldy + n;
        if (!(none >> (4 * i + wave) & 1)) continue;
        if (wide && n + 4 <= b1) *reinterpret_cast<F*>(y + at) = *reinterpret_cast<const F*>(base + at);
        else
          for (int j = 0; j < 4 && n + j < b1; ++j) y[at + j] = base[at + j];
      }
    }
  }
  uint64_t left = rows.leaders;
  for (int s = 0; left != 0; ++s, left &= left - 1) {
    if (s % lanes != lane0) continue;
    const int id = __builtin_amdgcn_readlane(rows.id, __ffsll((unsigned long long)left) - 1);
    const float scale = p.scale != nullptr ? p.scale[id] : 1.f;
    const uint32_t here = (uint32_t)__ballot(rows.id == id);   // this adapter's rows; t of the others is multiplied along
    for (int part = part0; part <= part1; ++part) {
      const int first = max(b0, part == 0 ? 0 : p.part_end[part - 1]) + 64 * wave, end = min(b1, p.part_end[part]);
      u32x4 bf[4][NS];
      F old[4];
      auto request = [&](int n0) {
        load_b<T, NS>(bf, p, id, n0);
        if (!wide || n0 + 4 * c + 4 > end) return;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((here >> e & 0x1111) != 0)                       // (one of rows e, 4 + e, 8 + e, 12 + e)
            old[e] = *reinterpret_cast<const F*>(base + (int64_t)min(4 * kg + e, rows_left - 1) * p.ldy + n0 + 4 * c);
      };
      if (first < end) request(first);
      if (part != have) t.load(p, cut.splits, m0, rows_left, have = part);
      t.store(tl, [&](int) { return scale; });
      lds_barrier();
      for (int n0 = first; n0 < end; n0 += 256) {
        if (n0 != first) request(n0);
        trim_b<T, NS>(bf, p.rank);
        floatx4 acc[4];
        products<T, NS, 16>(acc, bf, tl, 0);
        const int n = n0 + 4 * c;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((here >> e & 0x1111) == 0) continue;
          if (!(here >> (4 * kg + e) & 1)) continue;
          const floatx4 v = {acc[0][e], acc[1][e], acc[2][e], acc[3][e]};
          const int64_t at = (int64_t)(4 * kg + e) * p.ldy + n;
          if (wide && n + 4 <= end) *reinterpret_cast<F*>(y + at) = Four<T>::added(old[e], v);
          else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (n + j < end) y[at + j] = from_f32<T>(to_f32<T>(base[at + j]) + v[j]);
          }
        }
      }
      lds_barrier();
    }
  }
}
template <typename T, int NS>
__global__ __launch_bounds__(256, 2) void adapters_outer_kernel(AdapterArgs p, Cut cut) {
  __shared__ __attribute__((aligned(16))) char tl[Inner<T, NS, 16>::BYTES];
  const int cols = 64 * cut.groups, chunks = ceil_div(p.N, cols);
  const int b0 = blockIdx.x % chunks * cols;
  outer_rows<T, NS>(p, cut, cut.lanes, blockIdx.y, (int64_t)(blockIdx.x / chunks) * 16, b0, min(b0 + cols, p.N), tl);
}

// Many rows: 64 of them and 256 columns of one part, all there, 64 columns a wave.  Most share an adapter: base, b and t are requested at once and no
// row is tested (beside memory, instructions bound these blocks), and a row's accesses are one offset a lane from one address a row, past the caches
// (4096 x 4096, rank 64: 24.0 | 20.4 us).  Where they do not, one adapter after another.
template <typename T, int NS>
__global__ __launch_bounds__(256, 2) void adapters_outer_many_kernel(AdapterArgs p, Cut cut) {
  typedef typename Four<T>::type F;
  typedef InnerAhead<T, NS, 64> I;
  __shared__ __attribute__((aligned(16))) char tl[I::BYTES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, kg = lane >> 4;
  const int chunks = p.N / 256;
  const int turn = blockIdx.x / 8;         // of the XCDs: each works on whole rows
  const int tile0 = (turn / chunks * 8 + (int)blockIdx.x % 8) * 64;
  if (tile0 >= p.M) return;
  const int64_t m0 = min(tile0, p.M - 64);           // (the last one begins among the rows of the one before, which are not its own)
  const uint64_t own = ~0ull << (tile0 - (int)m0);
  const int b0 = turn % chunks * 256;
  int part = 0;
  while (b0 >= p.part_end[part]) ++part;
  const int n0 = b0 + 64 * wave;
  const int64_t row = p.ldy * (int64_t)sizeof(T);
  const uint32_t at = 4 * kg * (uint32_t)row + 4 * c * (uint32_t)sizeof(T);      // (ldy is at most 2^24)
  const char* const base = reinterpret_cast<const char*>(p.base) + m0 * row + n0 * (int64_t)sizeof(T);
  char* const y = reinterpret_cast<char*>(p.y) + m0 * row + n0 * (int64_t)sizeof(T);
  const int ids = Rows::request(p, m0, 64);
  F old[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) old[i][e] = __builtin_nontemporal_load(reinterpret_cast<const F*>(base + (16 * i + e) * row + at));
  I t;
  t.request(p, cut.splits, m0, part);
  const Rows rows(p, own >> lane & 1 ? ids : -1);
  const uint64_t none = __ballot(rows.id < 0) & own;
  int id = __builtin_amdgcn_readlane(rows.id, rows.leaders != 0 ? __ffsll((unsigned long long)rows.leaders) - 1 : 0);
  u32x4 bf[4][NS];
  if (rows.leaders != 0) load_b<T, NS>(bf, p, id, n0);
  if (none != 0 && p.y != p.base) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (none >> (16 * i + 4 * kg + e) & 1) *reinterpret_cast<F*>(y + (16 * i + e) * row + at) = old[i][e];
  }
  if (rows.leaders == 0) return;
  t.sum(p, cut.splits);
  t.store(tl, [&](int r) {
    const int whose = __shfl(rows.id, r, 64);
    return p.scale != nullptr ? p.scale[max(whose, 0)] : 1.f;
  });
  lds_barrier();
  for (uint64_t left = rows.leaders;;) {
    const uint64_t here = __ballot(rows.id == id);
    trim_b<T, NS>(bf, p.rank);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __builtin_amdgcn_sched_barrier(0);   // (a tile's operands at a time, or they fill the registers)
      floatx4 acc[4];
      products<T, NS, 64>(acc, bf, tl, i);
      if (here == ~0ull) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          __builtin_nontemporal_store(Four<T>::added(old[i][e], floatx4{acc[0][e], acc[1][e], acc[2][e], acc[3][e]}), reinterpret_cast<F*>(y + (16 * i + e) * row + at));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (here >> (16 * i + 4 * kg + e) & 1)
            __builtin_nontemporal_store(Four<T>::added(old[i][e], floatx4{acc[0][e], acc[1][e], acc[2][e], acc[3][e]}), reinterpret_cast<F*>(y + (16 * i + e) * row + at));
      }
    }
    left &= left - 1;
    if (left == 0) break;
    id = __builtin_amdgcn_readlane(rows.id, __ffsll((unsigned long long)left) - 1);
    load_b<T, NS>(bf, p, id, n0);
  }
}

template <typename T, int NS>
forge_status launch_outer(const AdapterArgs& a, Cut c, bool many, hipStream_t s) {
  if (many && adapters_whole(a.ldy, a.parts, a.part_end)) {
    adapters_outer_many_kernel<T, NS><<<(unsigned)(ceil_div(ceil_div(a.M, 64), 8) * 8 * (a.N / 256)), 256, 0, s>>>(a, c);
    return launch_status();
  }
  c.groups = a.N <= 256 ? 4 : 8;
  const int64_t blocks = (int64_t)ceil_div(a.M, 16) * ceil_div(a.N, 64 * c.groups);
  c.lanes = adapters_lanes(blocks, a.M, compute_units());
  adapters_outer_kernel<T, NS><<<dim3((unsigned)blocks, c.lanes), 256, 0, s>>>(a, c);
  return launch_status();
}
template <typename T>
forge_status launch(const AdapterArgs& a, hipStream_t s) {
  constexpr bool F32 = sizeof(T) == 4;
  const int inner = a.parts * a.rank;
  const bool many = adapters_many(a.M, a.N, inner, F32);
  const Cut c = adapters_cut(a.M, a.K, inner, many, F32, compute_units());
  const dim3 grid(c.tiles, c.chunks * c.splits, c.lanes);
  if (many) adapters_inner_kernel<T, 4><<<grid, 256, 0, s>>>(a, c);
  else adapters_inner_kernel<T, 1><<<grid, 256, 0, s>>>(a, c);
  if (hipGetLastError() != hipSuccess) return FORGE_ERR_HIP;
  const int steps = adapters_steps(a.rank, F32);
  if (steps == 1) return launch_outer<T, 1>(a, c, many, s);
  if (steps == 2) return launch_outer<T, 2>(a, c, many, s);
  if constexpr (F32) {
    if (steps == 8) return launch_outer<T, 8>(a, c, many, s);
  }
  return launch_outer<T, 4>(a, c, many, s);
}

}  // namespace

size_t adapters_workspace_bytes(int M, int K, int rank, int parts, forge_dtype dt) {
  return adapters_room(M, K, parts * rank, dt == FORGE_F32, compute_units());
}

forge_status launch_adapters(const AdapterArgs& a, hipStream_t s) {
  return a.dt == FORGE_F32 ? launch<float>(a, s) : launch<bf16>(a, s);
}

}  // namespace forge
