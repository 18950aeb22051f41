// The bookkeeping of a step over a paged cache: pages given back, pages taken, and a slot for every new token.
//
// With n rows before and n' after, request b has ceil(n / P) and ceil(n' / P) pages; what is given back and taken goes to and comes from the
// stack at the running sums of these differences over the requests, and token j's slot is page * P + (n + j) % P of the page that holds row
// n + j.  All of it is prefix sums and whole numbers: a block walks over the requests a chunk at a time, a thread each, and deals what the
// chunk's requests have together (pages, tokens) to its threads by a search in their running sums.
// Latency, not bytes, bounds it: a chain of loads (lengths and changes; then old and new page numbers together, the new ones from the
// stack rather than from the table), few steps between them, one wave where the requests fit one.  3 requests that add a token 2.7 us, 256 that
// grow and end with a prompt among them, 8192 tokens, 10.2.
#include "paged.hpp"

namespace forge {
namespace {

constexpr int CHUNK = 1024;

// Running sum over the lanes of a wave, on the vector ALU
__device__ inline uint32_t wave_scan(uint32_t v) {
  int x = (int)v;
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);     // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);    // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);    // row_bcast:31 into rows 2 and 3
  return (uint32_t)x;
}

// Running sums over the threads of a block: of the threads before this one, and of all.  64 values stay below 2^32 (a request's at most 2^25 + 1,
// see the limits of the entry point), a block's are added in 64 bits.
template <bool ONE>
__device__ inline int64_t before(uint32_t v, int64_t& all, uint32_t* waves) {
  const uint32_t sum = wave_scan(v);
  if constexpr (ONE) {
    all = (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
    return sum - v;
  }
  const int wave = threadIdx.x >> 6, n = blockDim.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) waves[wave] = sum;
  __syncthreads();
  int64_t first = 0;
  all = 0;
  for (int w = 0; w < n; ++w) {
    const uint32_t x = waves[w];
    if (w < wave) first += x;
    all += x;
  }
  return first + sum - v;
}

// the last of n running sums that is at most x
__device__ inline int holder(const uint32_t* first, int n, uint32_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
template <typename F>
__device__ inline void each(int64_t n, F f) {
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) f(i);
}

__device__ inline void put_token(const PagesArgs& p, int64_t t, int slot, int row, int b) {
  p.slots[t] = slot;
  p.positions[t] = row;
  p.owners[t] = b;
}
__device__ inline int slot_in(const PagesArgs& p, int page, int row) {
  return (uint32_t)page < (uint32_t)p.n_pages ? (page << p.shift) + (row & ((1 << p.shift) - 1)) : -1;
}

// ONE: a block of one wave for at most 64 requests
template <bool ONE>
__global__ __launch_bounds__(ONE ? 64 : CHUNK) void pages_assign_kernel(PagesArgs p, int with_tokens) {
  constexpr int N = ONE ? 64 : CHUNK;
  __shared__ uint32_t waves[N / 64], first[N], tok0[N];
  __shared__ int col0[N], row0[N];         // (col0: -1 for a request that gets nothing)
  __shared__ int taken;
  const int tid = threadIdx.x, P = 1 << p.shift, per = blockDim.x;
  const int room = p.cols << p.shift;
  auto request = [&](int b, int& n, int& c) {
    n = b < p.batch ? min(max(p.lengths[b], 0), room) : 0;
    c = b < p.batch ? max(p.change[b], -n) : 0;
  };
  auto pages_of = [&](int64_t rows) { return (int)((rows + P - 1) >> p.shift); };
  int n0, c0;                              // of the first chunk
  request(tid, n0, c0);
  const int count = min(max(*p.free_count, 0), p.n_pages);
  if (tid == 0) taken = 0;

  // ---- pages that are no longer needed ----------------------------------------------------------
  int64_t back = 0;
  for (int b0 = 0; b0 < p.batch; b0 += per) {
    int n = n0, c = c0;
    if (b0 > 0) request(b0 + tid, n, c);
    const int keep = pages_of(n + min(c, 0));
    int64_t all;
    const int64_t mine = before<ONE>(pages_of(n) - keep, all, waves);
    if (all == 0) continue;
    first[tid] = (uint32_t)min(mine, (int64_t)UINT32_MAX);
    col0[tid] = keep;
    __syncthreads();
    each(min(all, (int64_t)UINT32_MAX), [&](int64_t i) {
      const int j = holder(first, per, (uint32_t)i);
      int* at = p.table + (int64_t)(b0 + j) * p.cols + col0[j] + (i - first[j]);
      const int64_t to = count + back + i;
      if (to < p.n_pages) p.free_pages[to] = *at;
      *at = -1;
    });
    back += all;
    __syncthreads();
  }
  const int64_t avail = min(count + back, (int64_t)p.n_pages);

  // ---- pages for new rows, and the rows' slots ----------------------------------------------------
  int64_t tokens = 0, wants = 0;
  for (int b0 = 0; b0 < p.batch; b0 += per) {
    const int b = b0 + tid;
    int n = n0, c = c0;
    if (b0 > 0) request(b, n, c);
    int64_t all_tokens, all_wants;
    const uint32_t asked = (uint32_t)min(max(c, 0), p.max_tokens + 1);        // (more would not be granted either)
    const int64_t t0 = tokens + before<ONE>(asked, all_tokens, waves), t1 = t0 + asked;
    bool grows = c > 0 && (int64_t)n + c <= room && t1 <= p.max_tokens;
    const int have = pages_of(n), want = grows ? pages_of((int64_t)n + c) - have : 0;
    const int64_t w0 = wants + before<ONE>(want, all_wants, waves);
    if (want > 0 && w0 + want > avail) grows = false;
    if (grows && want > 0) atomicMax(&taken, (int)(w0 + want));      // (the granted ones are the first of those that want any)
    first[tid] = (uint32_t)min(w0 - wants, (int64_t)UINT32_MAX);
    tok0[tid] = (uint32_t)min(t0 - tokens, (int64_t)UINT32_MAX);
    col0[tid] = grows ? have : -1;
    row0[tid] = n;
    __syncthreads();
    each(min(all_wants, avail - wants), [&](int64_t i) {
      const int j = holder(first, per, (uint32_t)i);
      if (col0[j] >= 0) p.table[(int64_t)(b0 + j) * p.cols + col0[j] + (i - first[j])] = p.free_pages[avail - 1 - (wants + i)];
    });
    if (with_tokens)
      each(min(all_tokens, p.max_tokens - tokens), [&](int64_t i) {
        const int j = holder(tok0, per, (uint32_t)i), row = row0[j] + (int)(i - tok0[j]), col = row >> p.shift;
        int slot = -1;
        if (col0[j] >= 0)          // (a new page's number from where the table has it from)
          slot = slot_in(p, col < col0[j] ? p.table[(int64_t)(b0 + j) * p.cols + col]
                                          : p.free_pages[avail - 1 - (wants + first[j] + (col - col0[j]))], row);
        put_token(p, tokens + i, slot, row, b0 + j);
      });
    if (b < p.batch) {
      const int change = c > 0 && !grows ? 0 : c;
      p.lengths_out[b] = n + change;
      p.granted[b] = change;
      p.starts[b] = (int)min(t0, (int64_t)p.max_tokens);
      if (b == p.batch - 1) p.starts[p.batch] = (int)min(t1, (int64_t)p.max_tokens);
    }
    tokens += all_tokens;
    wants += all_wants;
    __syncthreads();
  }
  if (tid == 0) *p.free_count = (int)(avail - taken);
  if (with_tokens)
    for (int64_t t = min(tokens, (int64_t)p.max_tokens) + tid; t < p.max_tokens; t += per) put_token(p, t, -1, 0, -1);
}

// The slots of many tokens, after the tables are made
constexpr int SEARCHED = 2048;             // running sums that a block holds
__global__ __launch_bounds__(256) void pages_slots_kernel(PagesArgs p) {
  __shared__ uint32_t first[SEARCHED];
  const int t = blockIdx.x * 256 + threadIdx.x;
  const bool held = p.batch <= SEARCHED;
  if (held) {
    for (int b = threadIdx.x; b < p.batch; b += 256) first[b] = (uint32_t)p.starts[b];
    __syncthreads();
  }
  if (t >= p.max_tokens) return;
  if (t >= p.starts[p.batch]) {
    put_token(p, t, -1, 0, -1);
    return;
  }
  // the last request that starts at or before t (empty ones before it start there too)
  const int b = held ? holder(first, p.batch, (uint32_t)t) : holder(reinterpret_cast<const uint32_t*>(p.starts), p.batch, (uint32_t)t);
  // granted: its rows end at its length; refused: they would begin there
  const int granted = p.granted[b], row = p.lengths_out[b] - max(granted, 0) + t - p.starts[b];
  put_token(p, t, granted > 0 ? slot_in(p, p.table[(int64_t)b * p.cols + (row >> p.shift)], row) : -1, row, b);
}

}  // namespace

forge_status launch_pages_assign(const PagesArgs& a, hipStream_t s) {
  // the tokens' slots by a launch of its own where one block would take longer (256 requests, 8192 tokens: 6.5 + 3.7 us, in one 14.5)
  const bool apart = a.max_tokens > 4096;
  if (a.batch <= 64 && a.max_tokens <= 256) {
    pages_assign_kernel<true><<<1, 64, 0, s>>>(a, 1);
    return launch_status();
  }
  const int threads = apart || a.max_tokens <= 256 ? (a.batch <= 256 ? 256 : CHUNK) : CHUNK;
  pages_assign_kernel<false><<<1, threads, 0, s>>>(a, !apart);
  if (!apart) return launch_status();
  if (hipGetLastError() != hipSuccess) return FORGE_ERR_HIP;
  pages_slots_kernel<<<ceil_div(a.max_tokens, 256), 256, 0, s>>>(a);
  return launch_status();
}

}  // namespace forge
