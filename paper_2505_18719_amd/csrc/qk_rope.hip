// Norms of queries and keys per head with their rotation and the append to the paged cache, and the gradient of the norms
// and the rotation (vla_qk_norm_rope, vla_qk_norm_rope_backward).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"
#include "common.h"

namespace vla {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <CacheType T>
__device__ __forceinline__ void unpack(const uint4& v, float* f) {
  if constexpr (T == kBf16) {
    unpack8(v, f);
  } else {
    const f16x8 h = __builtin_bit_cast(f16x8, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)h[i];
  }
}

template <CacheType T>
__device__ __forceinline__ uint4 pack(const float* f) {
  if constexpr (T == kBf16) {
    return make_uint4(pack2bf(f[0], f[1]), pack2bf(f[2], f[3]), pack2bf(f[4], f[5]), pack2bf(f[6], f[7]));
  } else {
    f16x8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (_Float16)f[i];
    return __builtin_bit_cast(uint4, h);
  }
}

// Sum over the N lanes (4, 8 or 16) that share lane / N.
template <int N>
__device__ __forceinline__ float group_sum(float v) {
  v += dpp_mov<0xB1>(v, v);                          // lane ^ 1
  v += dpp_mov<0x4E>(v, v);                          // lane ^ 2
  if constexpr (N >= 8) v += dpp_mov<0x141>(v, v);   // mirrored within 8: the other quad
  if constexpr (N >= 16) v += dpp_mov<0x140>(v, v);  // mirrored within 16: the other 8
  return v;
}

// A head vector is held by head_dim / 16 lanes, two 8-feature chunks each, so that both features of every pair are in one
// lane: in the half layout lane j < rot / 16 takes chunks j and j + rot / 16, every other lane two neighbouring chunks.
struct Chunks {
  int lo, hi;   // the lane's chunks
  bool turned;  // whether they are rotated
};
__device__ __forceinline__ Chunks lane_chunks(int j, int rot_dim, int layout) {
  const int np = rot_dim >> 4;
  const bool half = layout == 0 && j < np;
  return {half ? j : 2 * j, half ? j + np : 2 * j + 1, j < np};
}

// cos and sin, times `scale`, of the lane's 8 pairs at position p: the turns p f / (2 pi) are reduced in 64 bits, so that far
// positions lose nothing.
__device__ __forceinline__ void lane_angles(const double* freqs, int layout, int j, int p, float scale, float* cs, float* sn) {
  constexpr double kTurn = 0.15915494309189533577;  // 1 / (2 pi)
  const int i0 = 8 * j;  // both layouts: pairs 8 j .. 8 j + 7 (interleaved: 4 of chunk 2 j, 4 of chunk 2 j + 1)
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double t = (double)p * freqs[i0 + e] * kTurn;
    const float x = (float)(t - rint(t));
    sincospif(2.f * x, sn + e, cs + e);
    cs[e] *= scale;
    sn[e] *= scale;
  }
}

// Rotates the lane's features y[0 .. 8) (chunk lo) and y[8 .. 16) (chunk hi); sgn = -1 rotates back.
__device__ __forceinline__ void turn(float* y, int layout, const float* cs, const float* sn, float sgn) {
  if (layout == 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = y[e], b = y[8 + e], s = sgn * sn[e];
      y[e] = fmaf(a, cs[e], -(b * s));
      y[8 + e] = fmaf(b, cs[e], a * s);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = y[2 * e], b = y[2 * e + 1], s = sgn * sn[e];
      y[2 * e] = fmaf(a, cs[e], -(b * s));
      y[2 * e + 1] = fmaf(b, cs[e], a * s);
    }
  }
}

constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / kWave;

__device__ __forceinline__ bool live_slot(const int32_t* row_slot, int row, int n_pages, int& slot) {
  slot = row_slot ? row_slot[row] : 0;
  return !row_slot || (slot >= 0 && slot < (long long)n_pages * kPage);
}

// One wave per row and run of head vectors (a row's runs are `parts` waves), the angles computed once per wave.
template <int HD, CacheType T>
__device__ __forceinline__ void rope_rows(const QkRopeArgs& a, long long wave, int parts) {
  constexpr int LPH = HD / 16, HPW = kWave / LPH;  // lanes per head vector, head vectors per pass of a wave
  const int lane = threadIdx.x & 63, j = lane % LPH;
  const long long row = wave / parts;
  if (row >= a.rows) return;
  int slot;
  if (!live_slot(a.row_slot, (int)row, a.n_pages, slot)) return;
  const int heads = a.n_heads + a.n_kv_heads;
  const Chunks ch = lane_chunks(j, a.rot_dim, a.layout);
  float cs[8], sn[8];
  if (ch.turned) lane_angles(a.freqs, a.layout, j, a.row_pos[row], a.rope_scale, cs, sn);
  for (int h0 = (int)(wave % parts) * HPW; h0 < heads; h0 += parts * HPW) {
    const int h = h0 + lane / LPH;
    if (h >= heads) continue;
    const bool is_q = h < a.n_heads;
    const int hh = is_q ? h : h - a.n_heads;
    const bf16_t* x = (is_q ? a.q.p + row * a.q.ld : a.k.p + row * a.k.ld) + hh * HD;
    const uint4 v0 = *reinterpret_cast<const uint4*>(x + 8 * ch.lo), v1 = *reinterpret_cast<const uint4*>(x + 8 * ch.hi);
    float y[16];
    unpack<T>(v0, y);
    unpack<T>(v1, y + 8);
    const bf16_t* gain = is_q ? a.q_gain : a.k_gain;
    if (gain) {
      float g[16], ss = 0.f;
      unpack<T>(*reinterpret_cast<const uint4*>(gain + 8 * ch.lo), g);
      unpack<T>(*reinterpret_cast<const uint4*>(gain + 8 * ch.hi), g + 8);
#pragma unroll
      for (int e = 0; e < 16; ++e) ss = fmaf(y[e], y[e], ss);
      const float r = 1.f / sqrtf(group_sum<LPH>(ss) * (1.f / HD) + a.eps);
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = y[e] * r * g[e];
    }
    if (ch.turned) turn(y, a.layout, cs, sn, 1.f);
    const uint4 o0 = pack<T>(y), o1 = pack<T>(y + 8);
    if (is_q) {
      bf16_t* o = a.q_out.p + row * a.q_out.ld + hh * HD;
      *reinterpret_cast<uint4*>(o + 8 * ch.lo) = o0;
      *reinterpret_cast<uint4*>(o + 8 * ch.hi) = o1;
    } else {
      if (a.k_out.p) {
        bf16_t* o = a.k_out.p + row * a.k_out.ld + hh * HD;
        *reinterpret_cast<uint4*>(o + 8 * ch.lo) = o0;
        *reinterpret_cast<uint4*>(o + 8 * ch.hi) = o1;
      }
      if (a.pages.k) {
        bf16_t* o = a.pages.k + (((long long)(slot / kPage) * a.n_kv_heads + hh) * kPage + slot % kPage) * HD;
        *reinterpret_cast<uint4*>(o + 8 * ch.lo) = o0;
        *reinterpret_cast<uint4*>(o + 8 * ch.hi) = o1;
      }
    }
  }
}

// Values of 16 rows and one key head to their transposed pages: through LDS, so that the lanes of 16 consecutive slots of a
// feature store next to each other.
template <int HD>
__device__ __forceinline__ void append_v(const QkRopeArgs& a, int tile, bf16_t (*lds)[HD + 8], int* slots) {
  const int tid = threadIdx.x, head = tile % a.n_kv_heads;
  const long long row0 = (long long)(tile / a.n_kv_heads) * 16;
  if (tid < 16) {
    int slot = -1;
    if (row0 + tid < a.rows && !live_slot(a.row_slot, (int)(row0 + tid), a.n_pages, slot)) slot = -1;
    slots[tid] = slot;
  }
  __syncthreads();
  for (int i = tid; i < 16 * HD / 8; i += kRopeThreads) {
    const int r = i / (HD / 8), c = i % (HD / 8);
    if (slots[r] >= 0)
      *reinterpret_cast<uint4*>(&lds[r][8 * c]) =
          *reinterpret_cast<const uint4*>(a.v.p + (row0 + r) * a.v.ld + head * HD + 8 * c);
  }
  __syncthreads();
  for (int i = tid; i < 16 * HD; i += kRopeThreads) {
    const int r = i % 16, f = i / 16, slot = slots[r];
    if (slot >= 0) a.pages.v[(((long long)(slot / kPage) * a.n_kv_heads + head) * HD + f) * kPage + slot % kPage] = lds[r][f];
  }
}

template <int HD, CacheType T>
__global__ __launch_bounds__(kRopeThreads) void qk_rope_kernel(QkRopeArgs a, int qk_groups, int parts) {
  __shared__ __align__(16) bf16_t lds[16][HD + 8];
  __shared__ int slots[16];
  if ((int)blockIdx.x < qk_groups)
    rope_rows<HD, T>(a, (long long)blockIdx.x * kRopeWaves + (threadIdx.x >> 6), parts);
  else
    append_v<HD>(a, blockIdx.x - qk_groups, lds, slots);
}

// ------------------------------------------------------------------ backward
constexpr int kBwdGroups = 512;

// A wave goes over rows w, w + W, ...; the gains' gradients of its lanes' features stay in registers, are joined over the
// workgroup and left in part[group][q or k][feature].
template <int HD, CacheType T>
__global__ __launch_bounds__(kRopeThreads) void qk_rope_bwd_kernel(QkRopeBwdArgs a) {
  constexpr int LPH = HD / 16, HPW = kWave / LPH;
  __shared__ float red[kRopeWaves][2][HD];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, j = lane % LPH;
  const int heads = a.n_heads + a.n_kv_heads;
  const Chunks ch = lane_chunks(j, a.rot_dim, a.layout);
  float dg[2][16];
#pragma unroll
  for (int e = 0; e < 16; ++e) dg[0][e] = dg[1][e] = 0.f;
  for (long long row = (long long)blockIdx.x * kRopeWaves + w; row < a.rows; row += (long long)gridDim.x * kRopeWaves) {
    float cs[8], sn[8];
    if (ch.turned) lane_angles(a.freqs, a.layout, j, a.row_pos[row], a.rope_scale, cs, sn);
    for (int h0 = 0; h0 < heads; h0 += HPW) {
      const int h = h0 + lane / LPH;
      if (h >= heads) continue;
      const bool is_q = h < a.n_heads;
      const int hh = is_q ? h : h - a.n_heads;
      const bf16_t* d = (is_q ? a.dq_out.p + row * a.dq_out.ld : a.dk_out.p + row * a.dk_out.ld) + hh * HD;
      float y[16];
      unpack<T>(*reinterpret_cast<const uint4*>(d + 8 * ch.lo), y);
      unpack<T>(*reinterpret_cast<const uint4*>(d + 8 * ch.hi), y + 8);
      if (ch.turned) turn(y, a.layout, cs, sn, -1.f);
      const bf16_t* gain = is_q ? a.q_gain : a.k_gain;
      if (gain) {
        const bf16_t* xp = (is_q ? a.q.p + row * a.q.ld : a.k.p + row * a.k.ld) + hh * HD;
        float g[16], x[16], ss = 0.f;
        unpack<T>(*reinterpret_cast<const uint4*>(gain + 8 * ch.lo), g);
        unpack<T>(*reinterpret_cast<const uint4*>(gain + 8 * ch.hi), g + 8);
        unpack<T>(*reinterpret_cast<const uint4*>(xp + 8 * ch.lo), x);
        unpack<T>(*reinterpret_cast<const uint4*>(xp + 8 * ch.hi), x + 8);
#pragma unroll
        for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
        const float r = 1.f / sqrtf(group_sum<LPH>(ss) * (1.f / HD) + a.eps);
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[e] *= r;
          const float t = x[e] * y[e];
          if (is_q) dg[0][e] += t;
          else dg[1][e] += t;
          y[e] *= g[e];
          dot = fmaf(x[e], y[e], dot);
        }
        dot = group_sum<LPH>(dot) * (1.f / HD);
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = r * fmaf(-x[e], dot, y[e]);
      }
      bf16_t* o = (is_q ? a.dq.p + row * a.dq.ld : a.dk.p + row * a.dk.ld) + hh * HD;
      *reinterpret_cast<uint4*>(o + 8 * ch.lo) = pack<T>(y);
      *reinterpret_cast<uint4*>(o + 8 * ch.hi) = pack<T>(y + 8);
    }
  }
  if (!a.q_gain && !a.k_gain) return;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = dg[t][e];
#pragma unroll
      for (int o = LPH; o < kWave; o <<= 1) v += __shfl_xor(v, o, kWave);
      if (lane < LPH) red[w][t][8 * (e < 8 ? ch.lo : ch.hi) + e % 8] = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * HD; i += kRopeThreads) {
    float v = 0.f;
#pragma unroll
    for (int u = 0; u < kRopeWaves; ++u) v += red[u][i / HD][i % HD];
    a.part[(size_t)blockIdx.x * 2 * HD + i] = v;
  }
}

// Sums the groups' parts in order: 64 columns per workgroup, its waves each a run of groups.
constexpr int kFinishWaves = 16;
__global__ __launch_bounds__(64 * kFinishWaves) void qk_rope_gain_kernel(QkRopeBwdArgs a, int groups) {
  __shared__ float red[kFinishWaves][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, cols = 2 * a.head_dim, c = blockIdx.x * 64 + lane;
  float v = 0.f;
  for (int g = w; g < groups; g += kFinishWaves) v += a.part[(size_t)g * cols + c];
  red[w][lane] = v;
  __syncthreads();
  if (w > 0) return;
  v = 0.f;
#pragma unroll
  for (int u = 0; u < kFinishWaves; ++u) v += red[u][lane];
  float* out = c < a.head_dim ? a.dq_gain : a.dk_gain;
  if (c < a.head_dim ? a.q_gain != nullptr : a.k_gain != nullptr) out[c % a.head_dim] = v;
}

template <int HD, CacheType T>
hipError_t launch_fwd(const QkRopeArgs& a, hipStream_t s) {
  const int per = kWave / (HD / 16), runs = (a.n_heads + a.n_kv_heads + per - 1) / per;
  const int parts = a.rows >= 2048 ? 1 : runs;
  const long long qk = ((long long)a.rows * parts + kRopeWaves - 1) / kRopeWaves;
  const long long v = a.pages.v ? ((long long)a.rows + 15) / 16 * a.n_kv_heads : 0;
  if (qk + v > 0x7fffffffll) return hipErrorInvalidValue;
  hipLaunchKernelGGL((qk_rope_kernel<HD, T>), dim3((unsigned)(qk + v)), dim3(kRopeThreads), 0, s, a, (int)qk, parts);
  return hipGetLastError();
}

template <int HD, CacheType T>
hipError_t launch_bwd(const QkRopeBwdArgs& a, hipStream_t s) {
  const int groups = std::min(kBwdGroups, (a.rows + kRopeWaves - 1) / kRopeWaves);
  if (groups > 0) hipLaunchKernelGGL((qk_rope_bwd_kernel<HD, T>), dim3(groups), dim3(kRopeThreads), 0, s, a);
  if (a.q_gain || a.k_gain)
    hipLaunchKernelGGL(qk_rope_gain_kernel, dim3(2 * HD / 64), dim3(64 * kFinishWaves), 0, s, a, groups);
  return hipGetLastError();
}

template <template <int, CacheType> class F, class A>
hipError_t by_type(const A& a, hipStream_t s) {
  const bool b = a.type == kBf16;
  if (a.head_dim == 64) return b ? F<64, kBf16>::run(a, s) : F<64, kF16>::run(a, s);
  if (a.head_dim == 128) return b ? F<128, kBf16>::run(a, s) : F<128, kF16>::run(a, s);
  if (a.head_dim == 256) return b ? F<256, kBf16>::run(a, s) : F<256, kF16>::run(a, s);
  return hipErrorInvalidValue;
}
template <int HD, CacheType T>
struct Fwd {
  static hipError_t run(const QkRopeArgs& a, hipStream_t s) { return launch_fwd<HD, T>(a, s); }
};
template <int HD, CacheType T>
struct Bwd {
  static hipError_t run(const QkRopeBwdArgs& a, hipStream_t s) { return launch_bwd<HD, T>(a, s); }
};

}  // namespace

size_t qk_rope_bwd_floats(int head_dim) { return (size_t)kBwdGroups * 2 * head_dim; }
hipError_t launch_qk_rope(const QkRopeArgs& a, hipStream_t s) { return by_type<Fwd>(a, s); }
hipError_t launch_qk_rope_bwd(const QkRopeBwdArgs& a, hipStream_t s) { return by_type<Bwd>(a, s); }

}  // namespace vla
