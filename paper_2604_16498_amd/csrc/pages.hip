// The bookkeeping of a step over a paged cache: pages given back, pages taken, and a slot for every new token.
//
// With n rows before and n' after, request b has ceil(n / P) and ceil(n' / P) pages; what is given back and taken goes to and comes from the
// stack at the running sums of these differences over the requests, and token j's slot is table[(n + j) / P] * P + (n + j) % P.  All of it is
// prefix sums and whole numbers: a block walks over the requests a chunk at a time, a thread each, and deals what the
// chunk's requests have together (pages, tokens) to its threads by a search in their running sums.  Latency, not bytes, bounds it.
#include "paged.hpp"

namespace forge {
namespace {

constexpr int CHUNK = 1024;

// Running sums over the threads of a block: of the threads before this one, and of all
struct Sums {
  int64_t wave[CHUNK / 64];
};
__device__ inline int64_t before(int64_t v, int64_t& all, Sums& lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int64_t sum = v;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int64_t other = __shfl_up(sum, o, 64);
    if (lane >= o) sum += other;
  }
  __syncthreads();
  if (lane == 63) lds.wave[wave] = sum;
  __syncthreads();
  int64_t first = 0;
  all = 0;
  for (int w = 0; w < waves; ++w) {
    const int64_t x = lds.wave[w];
    if (w < wave) first += x;
    all += x;
  }
  return first + sum - v;
}

// the last request of the chunk whose running sum is at most x
__device__ inline int holder(const int* first, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ inline void token_slot(const PagesArgs& p, int t, int b, int row, bool ok) {
  const int page = ok ? p.table[(int64_t)b * p.cols + (row >> p.shift)] : -1;
  p.slots[t] = (uint32_t)page < (uint32_t)p.n_pages ? (page << p.shift) + (row & ((1 << p.shift) - 1)) : -1;
  p.positions[t] = row;
  p.owners[t] = b;
}

__global__ __launch_bounds__(CHUNK) void pages_assign_kernel(PagesArgs p, int with_tokens) {
  __shared__ Sums lds;
  __shared__ int first[CHUNK], col0[CHUNK], ok[CHUNK], row0[CHUNK];
  __shared__ int taken;
  const int tid = threadIdx.x, P = 1 << p.shift;
  const int room = p.cols << p.shift;
  const int count = min(max(*p.free_count, 0), p.n_pages);
  if (tid == 0) taken = 0;
  auto request = [&](int b, int& n, int& c) {
    n = b < p.batch ? min(max(p.lengths[b], 0), room) : 0;
    c = b < p.batch ? max(p.change[b], -n) : 0;
  };
  auto pages_of = [&](int64_t rows) { return (int)((rows + P - 1) >> p.shift); };

  // ---- pages that are no longer needed ----------------------------------------------------------
  int64_t back = 0;
  for (int b0 = 0; b0 < p.batch; b0 += blockDim.x) {
    int n, c;
    request(b0 + tid, n, c);
    const int keep = pages_of(n + min(c, 0));
    int64_t all;
    const int64_t mine = before(pages_of(n) - keep, all, lds);
    if (all == 0) continue;
    first[tid] = (int)min(mine, (int64_t)INT32_MAX);
    col0[tid] = keep;
    __syncthreads();
    for (int64_t i = tid; i < all && i < INT32_MAX; i += blockDim.x) {
      const int j = holder(first, blockDim.x, (int)i);
      int* at = p.table + (int64_t)(b0 + j) * p.cols + col0[j] + (i - first[j]);
      const int64_t to = count + back + i;
      if (to < p.n_pages) p.free_pages[to] = *at;
      *at = -1;
    }
    back += all;
  }
  const int64_t avail = min(count + back, (int64_t)p.n_pages);
  __syncthreads();

  // ---- pages for new rows, and the rows' slots ----------------------------------------------------
  int64_t tokens = 0, wants = 0;
  for (int b0 = 0; b0 < p.batch; b0 += blockDim.x) {
    const int b = b0 + tid;
    int n, c;
    request(b, n, c);
    int64_t all_tokens, all_wants;
    const int64_t t0 = tokens + before(max(c, 0), all_tokens, lds), t1 = t0 + max(c, 0);
    bool grows = c > 0 && (int64_t)n + c <= room && t1 <= p.max_tokens;
    const int have = pages_of(n), want = grows ? pages_of((int64_t)n + c) - have : 0;
    const int64_t w0 = wants + before(want, all_wants, lds);
    if (want > 0 && w0 + want > avail) grows = false;
    if (grows && want > 0) atomicMax(&taken, (int)(w0 + want));      // (the granted ones are the first of those that want any)
    if (b < p.batch) {
      const int change = c > 0 && !grows ? 0 : c;
      p.lengths_out[b] = n + change;
      p.granted[b] = change;
      p.starts[b] = (int)min(t0, (int64_t)p.max_tokens);
      if (b == p.batch - 1) p.starts[p.batch] = (int)min(t1, (int64_t)p.max_tokens);
    }
    first[tid] = (int)min(w0 - wants, (int64_t)INT32_MAX);
    col0[tid] = have;
    row0[tid] = n;
    ok[tid] = grows;
    __syncthreads();
    const int64_t fresh = min(all_wants, avail - wants);
    for (int64_t i = tid; i < fresh; i += blockDim.x) {
      const int j = holder(first, blockDim.x, (int)i);
      if (ok[j]) p.table[(int64_t)(b0 + j) * p.cols + col0[j] + (i - first[j])] = p.free_pages[avail - 1 - (wants + i)];
    }
    __syncthreads();
    if (with_tokens) {
      first[tid] = (int)min(t0 - tokens, (int64_t)INT32_MAX);
      __syncthreads();
      const int64_t here = min(all_tokens, p.max_tokens - tokens);
      for (int64_t i = tid; i < here; i += blockDim.x) {
        const int j = holder(first, blockDim.x, (int)i);
        token_slot(p, (int)(tokens + i), b0 + j, row0[j] + (int)(i - first[j]), ok[j]);
      }
    }
    tokens += all_tokens;
    wants += all_wants;
    __syncthreads();
  }
  if (tid == 0) *p.free_count = (int)(avail - taken);
  if (with_tokens)
    for (int64_t t = min(tokens, (int64_t)p.max_tokens) + tid; t < p.max_tokens; t += blockDim.x) {
      p.slots[t] = -1;
      p.positions[t] = 0;
      p.owners[t] = -1;
    }
}

// The slots of many tokens, after the tables are made
__global__ __launch_bounds__(256) void pages_slots_kernel(PagesArgs p) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= p.max_tokens) return;
  if (t >= p.starts[p.batch]) {
    p.slots[t] = -1;
    p.positions[t] = 0;
    p.owners[t] = -1;
    return;
  }
  int lo = 0, hi = p.batch - 1;           // the last request that starts at or before t (empty ones before it start there too)
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.starts[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  // granted: its rows end at its length; refused: they would begin there
  const int after = p.lengths_out[lo], granted = p.granted[lo];
  token_slot(p, t, lo, after - max(granted, 0) + t - p.starts[lo], granted > 0);
}

}  // namespace

forge_status launch_pages_assign(const PagesArgs& a, hipStream_t s) {
  const bool apart = a.max_tokens > 4096;
  const int threads = CHUNK;
  pages_assign_kernel<<<1, threads, 0, s>>>(a, !apart);
  if (!apart) return launch_status();
  if (hipGetLastError() != hipSuccess) return FORGE_ERR_HIP;
  pages_slots_kernel<<<ceil_div(a.max_tokens, 256), 256, 0, s>>>(a);
  return launch_status();
}

}  // namespace forge
