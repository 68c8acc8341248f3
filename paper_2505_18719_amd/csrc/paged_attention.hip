// Attention of one new token per environment over a paged KV cache of any length (vla_paged_attention).
#include <hip/hip_runtime.h>

#include "cache.h"
#include "common.h"

namespace vla {
namespace {

template <CacheType T>
__device__ __forceinline__ float to_f32(bf16_t h) {
  if constexpr (T == kBf16) return bf2f(h);
  else return (float)__builtin_bit_cast(_Float16, h);
}
template <CacheType T>
__device__ __forceinline__ bf16_t from_f32(float f) {
  if constexpr (T == kBf16) return f2bf(f);
  else return __builtin_bit_cast(bf16_t, (_Float16)f);
}

constexpr int kAttnThreads = 256, kAttnWaves = kAttnThreads / kWave;

// One workgroup per (environment, head); wave w takes keys w, w + 4, ... with a running maximum and sum, a lane holding
// features lane, lane + 64, ...; the waves are joined in LDS.
template <int HD, CacheType T>
__global__ __launch_bounds__(kAttnThreads) void paged_attn_kernel(PagedAttnArgs a) {
  constexpr int N = HD / kWave;
  __shared__ float ms[kAttnWaves], ls[kAttnWaves], os[kAttnWaves][HD];
  const int head = blockIdx.x, env = blockIdx.y, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int kvh = head / (a.n_heads / a.n_kv_heads);
  const long long len = a.lens[env];
  const bool bad = len < 0 || len > (long long)a.max_pages * kPage;
  const int32_t* pt = a.page_table + env * a.ld_table;
  float q[N], o[N], m = -INFINITY, l = bad ? __builtin_nanf("") : 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    q[i] = to_f32<T>(a.q[env * a.ld_q + head * HD + lane + 64 * i]);
    o[i] = 0.f;
  }
  for (long long key = w; !bad && key < len; key += kAttnWaves) {
    const int page = pt[key / kPage], slot = (int)(key % kPage);
    if (page < 0 || page >= a.n_pages) {
      l = __builtin_nanf("");
      break;
    }
    const size_t at = (size_t)page * a.n_kv_heads + kvh;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s += q[i] * to_f32<T>(a.pages.k[(at * kPage + slot) * HD + lane + 64 * i]);
    s = wave_sum(s) * a.scale;
    const float mn = fmaxf(m, s), c = m == -INFINITY ? 0.f : expf(m - mn), p = mn == -INFINITY ? 0.f : expf(s - mn);
    l = l * c + p;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = o[i] * c + p * to_f32<T>(a.pages.v[(at * HD + lane + 64 * i) * kPage + slot]);
    m = mn;
  }
  if (lane == 0) {
    ms[w] = m;
    ls[w] = l;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) os[w][lane + 64 * i] = o[i];
  __syncthreads();
  float mm = -INFINITY, ll = 0.f;
#pragma unroll
  for (int u = 0; u < kAttnWaves; ++u) mm = fmaxf(mm, ms[u]);
#pragma unroll
  for (int u = 0; u < kAttnWaves; ++u) ll += ls[u] * (ms[u] == -INFINITY ? 0.f : expf(ms[u] - mm));
  for (int f = threadIdx.x; f < HD; f += kAttnThreads) {
    float v = 0.f;
#pragma unroll
    for (int u = 0; u < kAttnWaves; ++u) v += os[u][f] * (ms[u] == -INFINITY ? 0.f : expf(ms[u] - mm));
    a.o[env * a.ld_o + head * HD + f] = from_f32<T>(ll == 0.f ? 0.f : v / ll);
  }
  if (a.lse && threadIdx.x == 0) a.lse[(size_t)env * a.n_heads + head] = mm + logf(ll);
}

template <CacheType T>
hipError_t launch_t(const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid(a.n_heads, a.n_env), block(kAttnThreads);
  if (a.head_dim == 64) hipLaunchKernelGGL((paged_attn_kernel<64, T>), grid, block, 0, s, a);
  else if (a.head_dim == 128) hipLaunchKernelGGL((paged_attn_kernel<128, T>), grid, block, 0, s, a);
  else if (a.head_dim == 256) hipLaunchKernelGGL((paged_attn_kernel<256, T>), grid, block, 0, s, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

size_t paged_attn_bytes(int, int, int, int, int) { return 256; }

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  return a.type == kBf16 ? launch_t<kBf16>(a, s) : launch_t<kF16>(a, s);
}

}  // namespace vla
