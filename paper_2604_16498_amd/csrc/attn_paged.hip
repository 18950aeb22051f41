// Attention of one new token per request over a cache in pages.
#include <math.h>
#include "paged.hpp"

namespace forge {
namespace {

template <forge_kv_type S, typename T>
__device__ inline float element(const char* rows, const float* scales, int64_t e, int dh) {
  if constexpr (S == FORGE_KV_SAME) return to_f32<T>(reinterpret_cast<const T*>(rows)[e]);
  else {
    float f[4];
    Codes<S>::unpack((uint8_t)rows[e], f);
    return f[0] * scales[e / dh];
  }
}

// A wave per query head: a lane per column, one cache row after another.
template <forge_kv_type S, typename T, int DH>
__global__ __launch_bounds__(64) void attn_paged_kernel(PagedAttnArgs p) {
  const int b = blockIdx.y, h = blockIdx.x, g = h / (p.q_heads / p.kv_heads), lane = threadIdx.x;
  constexpr int N = DH / 64;
  const CacheView& c = p.cache.c;
  const int len = min(max(p.lengths[b], 0), p.max_len);
  const T* q = reinterpret_cast<const T*>(p.q.p) + b * p.q.bs + h * p.q.hs;
  float m = -INFINITY, l = 0.f, o[N] = {}, x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = to_f32<T>(q[lane + 64 * i]) * p.scale;
  for (int r = 0; r < len; ++r) {
    const int page = min(max(p.table[(int64_t)b * p.table_cols + (r >> p.cache.shift)], 0), p.cache.n_pages - 1);
    const int64_t e = page * c.bs + g * c.hs + (int64_t)(r & ((1 << p.cache.shift) - 1)) * DH;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s += x[i] * element<S, T>(c.k, c.ks, e + lane + 64 * i, DH);
    s = wave_sum(s);
    const float mn = fmaxf(m, s), a = __expf(m - mn), w = __expf(s - mn);
    m = mn;
    l = l * a + w;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = o[i] * a + w * element<S, T>(c.v, c.vs, e + lane + 64 * i, DH);
  }
  T* out = reinterpret_cast<T*>(p.out) + ((int64_t)b * p.q_heads + h) * DH;
#pragma unroll
  for (int i = 0; i < N; ++i) out[lane + 64 * i] = from_f32<T>(l > 0.f ? o[i] / l : 0.f);
}

template <forge_kv_type S, typename T>
void launch_dh(const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid(a.q_heads, a.batch);
  if (a.head_dim == 64) attn_paged_kernel<S, T, 64><<<grid, 64, 0, s>>>(a);
  else attn_paged_kernel<S, T, 128><<<grid, 64, 0, s>>>(a);
}

}  // namespace

size_t attn_paged_workspace_bytes(int, int, int, int, int) { return 0; }

forge_status launch_attn_paged(const PagedAttnArgs& a, hipStream_t s) {
  if (a.dt == FORGE_F32) launch_dh<FORGE_KV_SAME, float>(a, s);
  else if (a.type == FORGE_KV_SAME) launch_dh<FORGE_KV_SAME, bf16>(a, s);
  else if (a.type == FORGE_KV_INT8) launch_dh<FORGE_KV_INT8, bf16>(a, s);
  else launch_dh<FORGE_KV_FP8, bf16>(a, s);
  return launch_status();
}

}  // namespace forge
