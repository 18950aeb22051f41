// Low-rank adapters of many requests: y = base + scale * B (A x) per row, the row's own A and B.
#include "paged.hpp"

namespace forge {
namespace {

// A wave per (row, inner index): t[m, j] = scale * a[id, j, :] . x[m, :]
template <typename T>
__global__ __launch_bounds__(64) void adapters_inner_kernel(AdapterArgs p) {
  const int64_t m = blockIdx.x;
  const int inner = p.parts * p.rank, j = blockIdx.y, id = p.ids[m];
  if ((uint32_t)id >= (uint32_t)p.n_adapters) return;
  const T* x = reinterpret_cast<const T*>(p.x) + m * p.K;
  const T* a = reinterpret_cast<const T*>(p.a) + ((int64_t)id * inner + j) * p.K;
  float s = 0.f;
  for (int k = threadIdx.x; k < p.K; k += 64) s += to_f32<T>(x[k]) * to_f32<T>(a[k]);
  s = wave_sum(s);
  if (threadIdx.x == 0) reinterpret_cast<float*>(p.workspace)[m * inner + j] = s * (p.scale != nullptr ? p.scale[id] : 1.f);
}

template <typename T>
__global__ __launch_bounds__(256) void adapters_outer_kernel(AdapterArgs p) {
  const int n = blockIdx.y * 256 + threadIdx.x;
  const int64_t m = blockIdx.x;
  if (n >= p.N) return;
  const int id = p.ids[m];
  const int64_t at = m * p.ldy + n;
  float y = to_f32<T>(reinterpret_cast<const T*>(p.base)[at]);
  if ((uint32_t)id < (uint32_t)p.n_adapters) {
    int part = 0;
    while (n >= p.part_end[part]) ++part;
    const T* b = reinterpret_cast<const T*>(p.b) + ((int64_t)id * p.N + n) * p.rank;
    const float* t = reinterpret_cast<const float*>(p.workspace) + m * p.parts * p.rank + part * p.rank;
    float s = 0.f;
    for (int r = 0; r < p.rank; ++r) s += t[r] * to_f32<T>(b[r]);
    y += s;
  }
  reinterpret_cast<T*>(p.y)[at] = from_f32<T>(y);
}

template <typename T>
forge_status launch(const AdapterArgs& a, hipStream_t s) {
  adapters_inner_kernel<T><<<dim3(a.M, a.parts * a.rank), 64, 0, s>>>(a);
  if (hipGetLastError() != hipSuccess) return FORGE_ERR_HIP;
  adapters_outer_kernel<T><<<dim3(a.M, ceil_div(a.N, 256)), 256, 0, s>>>(a);
  return launch_status();
}

}  // namespace

size_t adapters_workspace_bytes(int M, int, int, int rank, int parts, forge_dtype) { return (size_t)M * parts * rank * sizeof(float); }

forge_status launch_adapters(const AdapterArgs& a, hipStream_t s) {
  return a.dt == FORGE_F32 ? launch<float>(a, s) : launch<bf16>(a, s);
}

}  // namespace forge
