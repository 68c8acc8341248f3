// Keys and values to a paged cache of 8-bit numbers and back (vla_kv_append_f8, vla_kv_read_f8).
//
// A head of a token is stored as 8-bit numbers x 448 / top, with top the largest size among its elements, and the scale top / 448.
// Bound: HBM, 2 bytes of each element and 1 of its 8-bit number; for few rows, a launch's latency.  A page holds a feature's 16 tokens
// together: rows that fill pages go through LDS, from where 16 bytes are written (or to where they are read) at once.
#include <hip/hip_runtime.h>

#include "cache.h"
#include "common.h"

namespace vla {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
constexpr int kThreads = 256;
constexpr float kF8Max = 448.f, kLeast = 0x1p-100f;

template <CacheType T>
__device__ __forceinline__ float2 two(uint32_t v) {
  if constexpr (T == kBf16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  const f16x2 h = __builtin_bit_cast(f16x2, v);
  return make_float2((float)h[0], (float)h[1]);
}
template <CacheType T>
__device__ __forceinline__ uint32_t two_of(float lo, float hi) {
  if constexpr (T == kBf16) return pack2bf(lo, hi);
  else return __builtin_bit_cast(uint32_t, (f16x2){(_Float16)lo, (_Float16)hi});
}

// Largest v of the N lanes (8, 16 or 32, aligned) that hold a head; NaN if one is.
template <int N>
__device__ __forceinline__ float head_max(float v) {
  auto larger = [](float a, float b) { return a > b || __builtin_isnan(a) ? a : b; };
#pragma unroll
  for (int d = N / 2; d > 0; d /= 2) v = larger(v, __shfl_xor(v, d, kWave));
  return v;
}

// The 8-bit numbers of this lane's eight elements, of a head held by HD / 8 lanes, and its scale.  The quotient x 448 / top is
// rounded to fp32 as a division rounds it (a product with the reciprocal of top's mantissa, corrected once), so that what lies half
// way between two 8-bit numbers stays there.
template <int HD, CacheType T>
__device__ __forceinline__ uint2 encode(const uint4& x, float& scale) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  float f[8], top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = two<T>(w[i]);
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
  bool nan = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    top = fmaxf(top, fabsf(f[i]));
    nan |= __builtin_isnan(f[i]);
  }
  top = head_max<HD / 8>(nan ? __builtin_nanf("") : top);
  if (__builtin_isinf(top)) top = __builtin_nanf("");  // an infinite element: no scale holds the others
  top = top < kLeast ? kLeast : top;
  scale = top / kF8Max;
  const int e = __builtin_amdgcn_frexp_expf(top);
  const float m = __builtin_amdgcn_frexp_mantf(top), r = 1.f / m, up = ldexpf(kF8Max, -e);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float n = f[i] * up, q = n * r;  // the first product is exact
    y[i] = copysignf(fmaf(fmaf(-q, m, n), r, q), q);  // of zeros, too
  }
  uint2 out;
  out.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  out.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], out.x, true);
  out.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  out.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], out.y, true);
  return out;
}
template <CacheType T>
__device__ __forceinline__ uint4 decode(const uint2& c, float s) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, true);
  const auto d = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, false), e = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, true);
  return make_uint4(two_of<T>(a[0] * s, a[1] * s), two_of<T>(b[0] * s, b[1] * s), two_of<T>(d[0] * s, d[1] * s), two_of<T>(e[0] * s, e[1] * s));
}

// One thread per eight features of a row's head, of keys and values both.
template <int HD, CacheType T, bool READ>
__global__ __launch_bounds__(kThreads) void kv_f8_kernel(KvF8Args a) {
  constexpr int CH = HD / 8;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int c = i % CH;
  const int64_t j = i / CH;
  const int head = j % a.n_kv_heads, row = (int)(j / a.n_kv_heads);
  if (row >= a.rows) return;  // whole heads: their lanes return together
  const int slot = a.row_slot[row];
  if ((unsigned)slot >= (unsigned)a.n_pages * kPage) return;
  const int64_t at = (int64_t)(slot / kPage) * a.n_kv_heads + head;  // the page's head
  const int s = slot % kPage;
  bf16_t* k = a.k.p + row * a.k.ld + head * HD + 8 * c;
  bf16_t* v = a.v.p + row * a.v.ld + head * HD + 8 * c;
  uint8_t* kp = a.k_pages + (at * kPage + s) * HD + 8 * c;
  uint8_t* vp = a.v_pages + (at * HD + 8 * c) * kPage + s;
  if constexpr (READ) {
    const float ks = a.k_scales[at * kPage + s], vs = a.v_scales[at * kPage + s];
    *reinterpret_cast<uint4*>(k) = decode<T>(*reinterpret_cast<const uint2*>(kp), ks);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int f = 0; f < 8; ++f) w[f / 4] |= (uint32_t)vp[f * kPage] << 8 * (f % 4);
    *reinterpret_cast<uint4*>(v) = decode<T>(make_uint2(w[0], w[1]), vs);
  } else {
    float ks, vs;
    const uint4 kx = *reinterpret_cast<const uint4*>(k), vx = *reinterpret_cast<const uint4*>(v);
    *reinterpret_cast<uint2*>(kp) = encode<HD, T>(kx, ks);
    const uint2 w = encode<HD, T>(vx, vs);
#pragma unroll
    for (int f = 0; f < 8; ++f) vp[f * kPage] = (f < 4 ? w.x : w.y) >> 8 * (f % 4);
    if (c == 0) {
      a.k_scales[at * kPage + s] = ks;
      a.v_scales[at * kPage + s] = vs;
    }
  }
}

// Bytes of four rows' four features, and back: x[r] byte f becomes byte r of x[f].
__device__ __forceinline__ void transpose4(uint32_t (&x)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602);
  const uint32_t c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602);
  x[0] = __builtin_amdgcn_perm(c, a, 0x05040100);
  x[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
  x[2] = __builtin_amdgcn_perm(d, b, 0x05040100);
  x[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}

// One workgroup per 64 rows of a head.  Rows whose slots are a whole page in order, or a quarter of one, move their values by 16 or 4
// bytes a feature; the others by single ones.
constexpr int kRows = 64;
template <int HD, CacheType T, bool READ>
__global__ __launch_bounds__(kThreads) void kv_f8_rows_kernel(KvF8Args a) {
  constexpr int CH = HD / 8, RPP = kThreads / CH, NW = kThreads / kWave;  // rows a pass
  __shared__ __align__(16) uint8_t codes[kRows][HD];
  __shared__ int slots[kRows];
  __shared__ unsigned long long runs[3];  // first rows of pages, quarters and single slots
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.x % a.n_kv_heads, r0 = blockIdx.x / a.n_kv_heads * kRows;
  if (wave == 0) {
    int s = r0 + lane < a.rows ? a.row_slot[r0 + lane] : -1;
    if ((unsigned)s >= (unsigned)a.n_pages * kPage) s = -1;
    slots[lane] = s;
    const int after = __shfl_down(s, 1, kWave);
    const unsigned long long next = __ballot(s >= 0 && lane < 63 && after == s + 1) >> lane;
    const unsigned long long pages = __ballot(s >= 0 && s % kPage == 0 && (next & 0x7fff) == 0x7fff);
    unsigned long long taken = pages;
    taken |= taken << 1;
    taken |= taken << 2;
    taken |= taken << 4;
    taken |= taken << 8;
    const unsigned long long quarters = __ballot(s >= 0 && s % 4 == 0 && (next & 7) == 7) & ~taken;
    taken |= quarters | quarters << 1 | quarters << 2 | quarters << 3;
    const unsigned long long singles = __ballot(s >= 0) & ~taken;
    if (lane == 0) {
      runs[0] = pages;
      runs[1] = quarters;
      runs[2] = singles;
    }
  }
  __syncthreads();
  auto page_head = [&](int slot) { return (int64_t)(slot / kPage) * a.n_kv_heads + head; };
  // Rows' 8-bit values between LDS and the pages, each run by one wave, a lane four features.
  auto move = [&] {
    int nth = 0;
    for (unsigned long long m = runs[0]; m; m &= m - 1, ++nth) {
      if (nth % NW != wave || 4 * lane >= HD) continue;
      const int i = __builtin_ctzll(m);
      uint4* to = reinterpret_cast<uint4*>(a.v_pages + (page_head(slots[i]) * HD + 4 * lane) * kPage);
      uint32_t x[4][4];  // by feature: four rows each
      if constexpr (READ) {
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const uint4 v = to[f];
          x[f][0] = v.x, x[f][1] = v.y, x[f][2] = v.z, x[f][3] = v.w;
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = READ ? x[e][q] : *reinterpret_cast<const uint32_t*>(&codes[i + 4 * q + e][4 * lane]);
        transpose4(y);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (READ) *reinterpret_cast<uint32_t*>(&codes[i + 4 * q + e][4 * lane]) = y[e];
          else x[e][q] = y[e];
        }
      }
      if constexpr (!READ) {
#pragma unroll
        for (int f = 0; f < 4; ++f) to[f] = make_uint4(x[f][0], x[f][1], x[f][2], x[f][3]);
      }
    }
    for (unsigned long long m = runs[1]; m; m &= m - 1, ++nth) {
      if (nth % NW != wave || 4 * lane >= HD) continue;
      const int i = __builtin_ctzll(m), s = slots[i];
      uint8_t* to = a.v_pages + (page_head(s) * HD + 4 * lane) * kPage + s % kPage;
      uint32_t y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        y[e] = READ ? *reinterpret_cast<const uint32_t*>(to + e * kPage) : *reinterpret_cast<const uint32_t*>(&codes[i + e][4 * lane]);
      transpose4(y);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (READ) *reinterpret_cast<uint32_t*>(&codes[i + e][4 * lane]) = y[e];
        else *reinterpret_cast<uint32_t*>(to + e * kPage) = y[e];
      }
    }
    for (unsigned long long m = runs[2]; m; m &= m - 1, ++nth) {
      if (nth % NW != wave || 4 * lane >= HD) continue;
      const int i = __builtin_ctzll(m), s = slots[i];
      uint8_t* to = a.v_pages + (page_head(s) * HD + 4 * lane) * kPage + s % kPage;
      uint32_t y = 0;
      if constexpr (READ) {
#pragma unroll
        for (int e = 0; e < 4; ++e) y |= (uint32_t)to[e * kPage] << 8 * e;
        *reinterpret_cast<uint32_t*>(&codes[i][4 * lane]) = y;
      } else {
        y = *reinterpret_cast<const uint32_t*>(&codes[i][4 * lane]);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e * kPage] = y >> 8 * e;
      }
    }
  };
  if constexpr (READ) {
    move();
    __syncthreads();
  }
  const int c = tid % CH;
#pragma unroll
  for (int i = 0; i < kRows / RPP; ++i) {
    const int r = i * RPP + tid / CH, slot = slots[r];  // whole heads: their lanes go on together
    if (slot < 0) continue;
    const int64_t row = r0 + r, at = page_head(slot);
    const int s = slot % kPage;
    bf16_t* k = a.k.p + row * a.k.ld + head * HD + 8 * c;
    bf16_t* v = a.v.p + row * a.v.ld + head * HD + 8 * c;
    uint2* kp = reinterpret_cast<uint2*>(a.k_pages + (at * kPage + s) * HD + 8 * c);
    uint2* mine = reinterpret_cast<uint2*>(&codes[r][8 * c]);
    float& ks = a.k_scales[at * kPage + s];
    float& vs = a.v_scales[at * kPage + s];
    if constexpr (READ) {
      *reinterpret_cast<uint4*>(k) = decode<T>(*kp, ks);
      *reinterpret_cast<uint4*>(v) = decode<T>(*mine, vs);
    } else {
      float kt, vt;
      *kp = encode<HD, T>(*reinterpret_cast<const uint4*>(k), kt);
      *mine = encode<HD, T>(*reinterpret_cast<const uint4*>(v), vt);
      if (c == 0) {
        ks = kt;
        vs = vt;
      }
    }
  }
  if constexpr (!READ) {
    __syncthreads();
    move();
  }
}

template <int HD, CacheType T, bool READ>
hipError_t launch(const KvF8Args& a, hipStream_t s) {
  const int64_t n = (int64_t)a.rows * a.n_kv_heads * (HD / 8), groups = (int64_t)(a.rows + kRows - 1) / kRows * a.n_kv_heads;
  // Rows one by one where they are few, whole workgroups of them where those fill the GPU (us, 8 heads of 128, one by one / 64 together:
  // append of 1024 rows in order 8.6 / 7.8, 4096 25.2 / 10.9, read back 4.4 / 5.4 and 13.0 / 7.3; of 64 rows 3.8 / 7.3 and 3.0 / 5.0;
  // of 4096 rows in slots apart 25.5 / 31.2 and 15.4 / 17.8)
  if (groups >= (READ ? 256 : 192)) hipLaunchKernelGGL((kv_f8_rows_kernel<HD, T, READ>), dim3((unsigned)groups), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((kv_f8_kernel<HD, T, READ>), dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}
template <CacheType T, bool READ>
hipError_t launch_heads(const KvF8Args& a, hipStream_t s) {
  if (a.head_dim == 64) return launch<64, T, READ>(a, s);
  if (a.head_dim == 128) return launch<128, T, READ>(a, s);
  if (a.head_dim == 256) return launch<256, T, READ>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace

bool kv_f8_fits(int rows, int n_kv_heads, int head_dim) {  // threads below 2^32
  return (int64_t)rows * n_kv_heads * (head_dim / 8) < (int64_t)(1ll << 32) - kThreads;
}
hipError_t launch_kv_append_f8(const KvF8Args& a, hipStream_t s) {
  return a.type == kBf16 ? launch_heads<kBf16, false>(a, s) : launch_heads<kF16, false>(a, s);
}
hipError_t launch_kv_read_f8(const KvF8Args& a, hipStream_t s) {
  return a.type == kBf16 ? launch_heads<kBf16, true>(a, s) : launch_heads<kF16, true>(a, s);
}

}  // namespace vla
