// Attention of one new token per environment over a paged KV cache of any length (vla_paged_attention).
//
// Bound: HBM, every cached key and value once (4 head_dim bytes a key and key head), against 4 flops per byte and query head
// of a group.  A wave takes steps of 32 keys, two pages, for up to 16 or 32 query heads of one key head, all on 16x16x32
// MFMAs: S^T = K Q^T with the keys on the rows, placed so that lane group g = lane / 16 ends up with the scores of keys
// 8 g .. 8 g + 7 of the step for head lane % 16, which is the B operand of O^T += V^T P^T as it stands; the transposed value
// pages give the A operand by one 16-byte load per lane.  Nothing goes through LDS but the joins.  Softmax by a running
// maximum and sum per head in fp32 (base 2); the weights enter the second product as a pair of numbers of the cache's type
// (hi + lo, 16 bits or more), so that their rounding stays below the output's.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"
#include "common.h"
#include "lds_limit.h"

namespace vla {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kStep = 32;  // keys of a wave's step
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

template <CacheType T>
__device__ __forceinline__ f32x4 mfma(const uint4& a, const uint4& b, const f32x4& c) {
  if constexpr (T == kBf16) return mfma16(as_bf16x8(a), as_bf16x8(b), c);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <CacheType T>
__device__ __forceinline__ bf16_t from_f32(float f) {
  if constexpr (T == kBf16) return f2bf(f);
  else return __builtin_bit_cast(bf16_t, (_Float16)f);
}

// Those of the two numbers in x that are infinite or NaN, 0 in the place of the others.
template <CacheType T>
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {
  constexpr uint32_t kExp = T == kBf16 ? 0x7f80 : 0x7c00;
  return ((x & kExp) == kExp ? x & 0xffffu : 0u) | ((x & kExp << 16) == kExp << 16 ? x & 0xffff0000u : 0u);
}
// What the sums under a base-2 maximum m are worth under a larger one: at least 2^-149, so that an infinity among them stays one
// (finite sums lose nothing: 2^-149 of them does not show).
__device__ __forceinline__ float worth(float m, float larger) { return fmaxf(__builtin_amdgcn_exp2f(m - larger), 0x1p-149f); }

// hi + lo = p[0 .. 8) to the precision of two numbers of the type
template <CacheType T>
__device__ __forceinline__ void split_weights(const float* p, uint4& hi, uint4& lo) {
  if constexpr (T == kBf16) {
    uint32_t h[4], r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[i] = pack2bf(p[2 * i], p[2 * i + 1]);
      r[i] = pack2bf(p[2 * i] - __uint_as_float(h[i] << 16), p[2 * i + 1] - __uint_as_float(h[i] & 0xffff0000u));
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(r[0], r[1], r[2], r[3]);
  } else {
    f16x8 h, r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[i] = (_Float16)p[i];
      r[i] = (_Float16)(p[i] - (float)h[i]);
    }
    hi = __builtin_bit_cast(uint4, h);
    lo = __builtin_bit_cast(uint4, r);
  }
}
// Half-precision weights are held 2^15 times as large: the largest stays below 65504, and a weight is lost only below 2^-40
// of it, where even 2^18 such keys do not show.
template <CacheType T>
constexpr float kWeightExp = T == kBf16 ? 0.f : 15.f;

// log of the sum of weights l relative to the base-2 maximum m
template <CacheType T>
__device__ __forceinline__ float log_sum(float m, float l) {
  return (m - kWeightExp<T> + __builtin_amdgcn_logf(l)) * kLn2;
}

// Max / sum over the lanes that share lane % 16.
__device__ __forceinline__ float column_max(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float column_sum(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// One block of up to 16 QT query heads of a key head.
struct HeadBlock {
  int kvh, head0, n;  // key head, first query head, query heads
};
template <int QT>
__host__ __device__ __forceinline__ int head_blocks(int group) { return (group + 16 * QT - 1) / (16 * QT); }
template <int QT>
__device__ __forceinline__ HeadBlock head_block(const PagedAttnArgs& a, int hb) {
  const int group = a.n_heads / a.n_kv_heads, qb = head_blocks<QT>(group);
  const int kvh = hb / qb, first = hb % qb * 16 * QT;
  return {kvh, kvh * group + first, min(group - first, 16 * QT)};
}

// What a wave holds of its keys: per head (lane % 16, tile t) the running maximum m of the base-2 scores, this lane's part
// of the sum l of weights, and O^T: features 16 i + 4 (lane / 16) + r in o[t][i][r].
template <int HD, int QT>
struct Running {
  float m[QT], l[QT];
  f32x4 o[QT][HD / 16];
};

// 16 bytes of a page: past the caches where the pool is larger than they keep (STREAM).
template <bool STREAM>
__device__ __forceinline__ uint4 load_page(const bf16_t* p) {
  const u32x4* src = reinterpret_cast<const u32x4*>(p);
  const u32x4 v = STREAM ? __builtin_nontemporal_load(src) : *src;
  return make_uint4(v.x, v.y, v.z, v.w);
}

// The pages of step s; entries up to the table's end may be read before the length is known.
__device__ __forceinline__ int2 step_pages(const int32_t* pt, int max_pages, int s) {
  return make_int2(pt[min(2 * s, max_pages - 1)], pt[min(2 * s + 1, max_pages - 1)]);
}

// A wave at its steps.
template <int HD, CacheType T, int QT, bool STREAM>
struct Wave {
  static constexpr int KC = HD / 32, VC = HD / 16;
  const PagedAttnArgs& a;
  int m16, g;
  float scale;
  size_t page_elems;
  uint4 q[QT][KC], k[2][KC], v[VC];
  Running<HD, QT> run;
  bool bad;  // a page outside the pool among the keys since begin()

  __device__ __forceinline__ explicit Wave(const PagedAttnArgs& args)
      : a(args), m16(threadIdx.x & 15), g((threadIdx.x & 63) >> 4), scale(args.scale * kLog2e),
        page_elems((size_t)args.n_kv_heads * kPage * HD) {}

  __device__ __forceinline__ void begin() {
    bad = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      run.m[t] = -INFINITY;
      run.l[t] = 0.f;
#pragma unroll
      for (int i = 0; i < VC; ++i) run.o[t][i] = {0.f, 0.f, 0.f, 0.f};
    }
  }

  __device__ __forceinline__ void load_q(int env, const HeadBlock& b) {  // columns past the block's heads repeat its last one
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < KC; ++i)
        q[t][i] = *reinterpret_cast<const uint4*>(a.q + env * a.ld_q + (size_t)(b.head0 + min(16 * t + m16, b.n - 1)) * HD + 32 * i + 8 * g);
  }

  // The pages to read for step s of `len` keys, of which `ids` are the table's: no page past the last one, none outside the
  // pool (`outside` then).
  __device__ __forceinline__ int2 usable(int2 ids, int len, int s, bool& outside) const {
    if (2 * s + 1 > (len - 1) / kPage) ids.y = ids.x;
    outside = (unsigned)ids.x >= (unsigned)a.n_pages || (unsigned)ids.y >= (unsigned)a.n_pages;
    return outside ? make_int2(0, 0) : ids;
  }
  // K operand: row lane % 16 of tile t is page m16 / 8 of the step, slot 8 (m16 / 4 % 2) + 4 t + m16 % 4
  __device__ __forceinline__ void load_k(int2 ids, int kvh) {
    const bf16_t* p = a.pages.k + ((size_t)kvh * kPage + 8 * ((m16 >> 2) & 1) + (m16 & 3)) * HD + 8 * g + (m16 < 8 ? ids.x : ids.y) * page_elems;
#pragma unroll
    for (int i = 0; i < KC; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) k[t][i] = load_page<STREAM>(p + 4 * t * HD + 32 * i);
  }
  __device__ __forceinline__ const bf16_t* v_at(int2 ids, int kvh) const {
    return a.pages.v + ((size_t)kvh * HD + m16) * kPage + 8 * (g & 1) + (g < 2 ? ids.x : ids.y) * page_elems;
  }
  __device__ __forceinline__ void load_v(const bf16_t* p) {
#pragma unroll
    for (int i = 0; i < VC; ++i) v[i] = load_page<STREAM>(p + 16 * i * kPage);
  }

  // p = base-2 scores of the step's keys; k is free afterwards
  __device__ __forceinline__ void scores(float (&p)[QT][8]) {
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KC; ++i) c = mfma<T>(k[u][i], q[t][i], c);
#pragma unroll
        for (int r = 0; r < 4; ++r) p[t][4 * u + r] = c[r] * scale;
      }
  }
  // Takes the step's keys, of which `left` (< 32: the last step) count, into the running sums; v is free afterwards.  APART:
  // values that are infinite or NaN are taken by weights of 1 (0 at scores of -inf), apart from the finite ones: an infinity
  // times a weight's lo part of 0 or below is no part of the sum, nor is one times a weight that rounds to 0.
  template <bool APART>
  __device__ __forceinline__ void weigh(float (&p)[QT][8], int left) {
    uint4 hi[QT], lo[QT], one[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (left < kStep) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (8 * g + j >= left) p[t][j] = -INFINITY;
      }
      float mx = p[t][0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx = fmaxf(mx, p[t][j]);
      mx = fmaxf(run.m[t], column_max(mx));
      if (__any(mx > run.m[t])) {  // seldom after the first steps
        const float c = run.m[t] == -INFINITY ? 1.f : worth(run.m[t], mx);  // nothing to scale yet: 1
        run.l[t] *= c;
#pragma unroll
        for (int i = 0; i < VC; ++i) run.o[t][i] *= c;
        run.m[t] = mx;
      }
      if constexpr (APART) {
        constexpr uint32_t k1 = T == kBf16 ? 0x3f80 : 0x3c00;
        uint32_t d[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = (p[t][2 * j] > -INFINITY ? k1 : 0) | (p[t][2 * j + 1] > -INFINITY ? k1 << 16 : 0);
        one[t] = make_uint4(d[0], d[1], d[2], d[3]);
      }
      const float base = run.m[t] == -INFINITY ? 0.f : run.m[t] - kWeightExp<T>;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        p[t][j] = __builtin_amdgcn_exp2f(p[t][j] - base);
        sum += p[t][j];
      }
      run.l[t] += sum;
      split_weights<T>(p[t], hi[t], lo[t]);
    }
    if (left < kStep) {  // slots past the length hold anything: 0 weights must multiply finite values
      uint32_t keep[4];
#pragma unroll
      for (int d = 0; d < 4; ++d)
        keep[d] = (8 * g + 2 * d < left ? 0xffffu : 0u) | (8 * g + 2 * d + 1 < left ? 0xffff0000u : 0u);
#pragma unroll
      for (int i = 0; i < VC; ++i) v[i] = make_uint4(v[i].x & keep[0], v[i].y & keep[1], v[i].z & keep[2], v[i].w & keep[3]);
    }
#pragma unroll
    for (int i = 0; i < VC; ++i) {
      uint4 rest;
      if constexpr (APART) {
        rest = make_uint4(not_finite<T>(v[i].x), not_finite<T>(v[i].y), not_finite<T>(v[i].z), not_finite<T>(v[i].w));
        v[i] = make_uint4(v[i].x ^ rest.x, v[i].y ^ rest.y, v[i].z ^ rest.z, v[i].w ^ rest.w);
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        run.o[t][i] = mfma<T>(v[i], hi[t], run.o[t][i]);
        run.o[t][i] = mfma<T>(v[i], lo[t], run.o[t][i]);
        if constexpr (APART) run.o[t][i] = mfma<T>(rest, one[t], run.o[t][i]);
      }
    }
  }
  // l over all keys since begin(), in every lane of its column
  __device__ __forceinline__ void end() {
#pragma unroll
    for (int t = 0; t < QT; ++t) run.l[t] = bad ? __builtin_nanf("") : column_sum(run.l[t]);
  }
  // After end(): whether a sum is NaN though its weights are not, as infinite or NaN values make it.  Only then is a piece taken
  // again with them apart: the check costs 0.1 us of a call, taking them apart at once would cost every step.
  __device__ __forceinline__ bool spoiled() const {
    bool nan = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      f32x4 c[2] = {run.o[t][0], run.o[t][1]};  // NaN where one of its terms is
#pragma unroll
      for (int i = 2; i < VC; ++i) c[i % 2] += run.o[t][i];
      c[0] += c[1];
      nan |= __builtin_isnan((c[0][0] + c[0][1]) + (c[0][2] + c[0][3])) && !__builtin_isnan(run.l[t]);
    }
    return __any(nan);
  }
  // One step by itself, with infinite and NaN values apart.
  __device__ __forceinline__ void step_apart(const int32_t* pt, int len, int s, int kvh) {
    bool outside;
    const int2 ids = usable(step_pages(pt, a.max_pages, s), len, s, outside);
    bad |= outside;
    load_k(ids, kvh);
    load_v(v_at(ids, kvh));
    float p[QT][8];
    scores(p);
    weigh<true>(p, len - kStep * s);
  }
};

// Where a joined result goes: the output, or a partial (o fp32 [rows][HD], m and l [rows] each).
struct Partial {
  float* o;
  float* ml;
  int rows;
};

// Parts of a head block's result in LDS, one after the other: per part and head the sums O (HD + 4 floats, padded by a
// 16-byte bank group), m and l.
template <int HD>
struct Parts {
  float* o;   // [parts][rows][HD + 4]
  float* ml;  // [parts][2][rows]
  int rows;
  static size_t bytes(int parts, int rows) { return (size_t)parts * rows * (HD + 4 + 2) * sizeof(float); }
  __device__ __forceinline__ Parts(float* lds, int parts, int n) : o(lds), ml(lds + (size_t)parts * n * (HD + 4)), rows(n) {}
  template <int QT>
  __device__ __forceinline__ void put(int part, const Running<HD, QT>& run, int heads) {
    const int lane = threadIdx.x & 63, m16 = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int h = 16 * t + m16;
      if (h < heads) {
        if (g == 0) {
          ml[part * 2 * rows + h] = run.m[t];
          ml[(part * 2 + 1) * rows + h] = run.l[t];
        }
#pragma unroll
        for (int i = 0; i < HD / 16; ++i)
          *reinterpret_cast<f32x4*>(o + (size_t)(part * rows + h) * (HD + 4) + 16 * i + 4 * g) = run.o[t][i];
      }
    }
  }
};

// 1 / l, or 0 where no score is above -inf; then the output is zeros, also where a value times its weight of 0 is NaN.
__device__ __forceinline__ float reciprocal(float l) { return l == 0.f ? 0.f : 1.f / l; }
template <CacheType T>
__device__ __forceinline__ bf16_t output(float o, float r) { return from_f32<T>(r == 0.f ? 0.f : o * r); }
template <CacheType T>
__device__ __forceinline__ void store4(bf16_t* p, const f32x4& v, float r) {
  bf16_t h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = output<T>(v[e], r);
  *reinterpret_cast<uint2*>(p) = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
}

// Adds parts first, first + step, ... (N of them) by the whole workgroup.  True where an output is NaN though its weights are
// not, as infinite or NaN values make it.
template <int HD, CacheType T, int N>
__device__ __forceinline__ bool join_parts(const PagedAttnArgs& a, int env, const HeadBlock& b, const Parts<HD>& ps, int first,
                                           int n, int second, int step, const Partial& to) {
  bool spoiled = false;
  for (int i = threadIdx.x; i < b.n * (HD / 4); i += blockDim.x) {
    const int h = i / (HD / 4), f = 4 * (i % (HD / 4));
    float mu[N], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int p = u == 0 ? first : second + (u - 1) * step;
      mu[u] = u < n ? ps.ml[p * 2 * ps.rows + h] : -INFINITY;
      m = fmaxf(m, mu[u]);
    }
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if (u >= n) break;
      const int p = u == 0 ? first : second + (u - 1) * step;
      const float c = mu[u] == -INFINITY ? 1.f : worth(mu[u], m);  // a part without keys adds zeros
      l = fmaf(ps.ml[(p * 2 + 1) * ps.rows + h], c, l);
      const f32x4 o = *reinterpret_cast<const f32x4*>(ps.o + (size_t)(p * ps.rows + h) * (HD + 4) + f);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(o[e], c, v[e]);
    }
    if (to.o) {
      *reinterpret_cast<f32x4*>(to.o + h * HD + f) = v;
      if (f == 0) {
        to.ml[h] = m;
        to.ml[to.rows + h] = l;
      }
    } else {
      store4<T>(a.o + env * a.ld_o + (size_t)(b.head0 + h) * HD + f, v, reciprocal(l));
      if (a.lse && f == 0) a.lse[(size_t)env * a.n_heads + b.head0 + h] = log_sum<T>(m, l);
      spoiled |= __builtin_isnan((v[0] + v[1]) + (v[2] + v[3])) && !__builtin_isnan(l);
    }
  }
  return spoiled;
}

// An environment's number of steps; 0 for one that gets zeros or NaN.
__device__ __forceinline__ int steps_of(const PagedAttnArgs& a, int len) {
  const bool bad = len < 0 || len > (long long)a.max_pages * kPage || a.n_pages == 0;
  return bad ? 0 : (len + kStep - 1) / kStep;
}

// The rows of a head block of an environment without steps: zeros for length 0, else NaN.
template <int HD, CacheType T>
__device__ __forceinline__ void no_keys(const PagedAttnArgs& a, int env, int head0, int n, int len) {
  const float v = len == 0 ? 0.f : __builtin_nanf("");
  for (int i = threadIdx.x; i < n * HD; i += blockDim.x) a.o[env * a.ld_o + (size_t)head0 * HD + i] = from_f32<T>(v);
  if (a.lse)  // n may be all heads of an environment, more than there are threads
    for (int i = threadIdx.x; i < n; i += blockDim.x) a.lse[(size_t)env * a.n_heads + head0 + i] = len == 0 ? -INFINITY : v;
}

// One workgroup of W waves per (head block, environment); wave w takes steps w, w + W, ...
template <int HD, CacheType T, int QT, bool STREAM, int W>
__global__ __launch_bounds__(64 * W) void attn_whole_kernel(PagedAttnArgs a, int rows) {
  extern __shared__ __align__(16) float lds[];
  __shared__ int again;
  const int env = blockIdx.y, len = __builtin_amdgcn_readfirstlane(a.lens[env]), steps = steps_of(a, len);
  const HeadBlock b = head_block<QT>(a, blockIdx.x);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t* pt = a.page_table + env * a.ld_table;
  int2 ids = a.max_pages > 0 ? step_pages(pt, a.max_pages, w) : make_int2(0, 0);
  if (steps == 0) return no_keys<HD, T>(a, env, b.head0, b.n, len);
  Wave<HD, T, QT, STREAM> wave(a);
  wave.begin();
  if (w < steps) {
    bool outside;
    wave.load_q(env, b);
    ids = wave.usable(ids, len, w, outside);
    wave.bad |= outside;
    wave.load_k(ids, b.kvh);
    wave.load_v(wave.v_at(ids, b.kvh));
    ids = step_pages(pt, a.max_pages, w + W);
    for (int s = w; s < steps; s += W) {
      float p[QT][8];
      wave.scores(p);
      const bool more = s + W < steps;
      const bf16_t* next_v = nullptr;
      if (more) {
        ids = wave.usable(ids, len, s + W, outside);
        wave.bad |= outside;
        wave.load_k(ids, b.kvh);
        next_v = wave.v_at(ids, b.kvh);
        ids = step_pages(pt, a.max_pages, s + 2 * W);
      }
      wave.template weigh<false>(p, len - kStep * s);
      if (more) wave.load_v(next_v);
    }
  }
  wave.end();
  Parts<HD> ps(lds, W, rows);
  ps.put(w, wave.run, b.n);
  if (threadIdx.x == 0) again = 0;
  __syncthreads();
  if (join_parts<HD, T, W>(a, env, b, ps, 0, W, 1, 1, {nullptr, nullptr, 0})) again = 1;
  __syncthreads();
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(again) == 0, 1)) return;
  wave.begin();  // once more with infinite and NaN values apart; the queries are still there
#pragma nounroll
  for (int s = w; s < steps; s += W) wave.step_apart(pt, len, s, b.kvh);
  wave.end();
  ps.put(w, wave.run, b.n);
  __syncthreads();
  join_parts<HD, T, W>(a, env, b, ps, 0, W, 1, 1, {nullptr, nullptr, 0});
}

// ------------------------------------------------------------------ split over the keys
// The steps of all environments and head blocks lie in one line, environment by environment, head block by head block (a
// piece is one environment and head block); a persistent grid takes the line in runs of equal length, one per wave, so that
// ragged lengths cost nothing.  A wave goes from piece to piece without a pause: the next step's pages are on their way
// while a step is taken, whatever piece it belongs to.  A piece inside a wave's run is written by the wave; what runs past
// the run's ends is left in LDS, joined there with the neighbouring waves' parts, and what runs past the workgroup's ends
// goes to the workspace: slot 2 w + 1 of workgroup w if the piece began there, else 2 w.  Who began a piece notes it down
// for the kernel that then adds its partials in order.
// Workgroups that the registers leave room for at once (64 x 4096 keys, 16 heads of 64: 254 us with 512, 174 with 1024).
template <int HD, int QT>
constexpr int kRunGroups = HD == 256 || (HD == 128 && QT == 2) ? 256 : HD == 64 && QT == 1 ? 1024 : 512;
constexpr int kRunWaves = 4, kRunThreads = 64 * kRunWaves;  // the grid may be smaller than kRunGroups where the lengths cannot need it

// Steps of a wave's run.
template <int HD, int QT>
__device__ __forceinline__ long long run_steps(long long units) {
  constexpr unsigned kWavesAll = kRunGroups<HD, QT> * kRunWaves;
  return max((long long)(((unsigned long long)units + kWavesAll - 1) / kWavesAll), 1ll);
}

struct SplitSpace {
  int4* begun;  // [groups] the piece that workgroup w began and did not end: environment, head block, last workgroup; or -1
  float* o;     // [2 groups][rows][HD]
  float* ml;    // [2 groups][2][rows]
};
template <int HD, int QT>
SplitSpace split_space(void* ws, int rows) {
  char* p = static_cast<char*>(ws);
  float* o = reinterpret_cast<float*>(p + kRunGroups<HD, QT> * sizeof(int4));
  return {reinterpret_cast<int4*>(p), o, o + (size_t)2 * kRunGroups<HD, QT> * rows * HD};
}
template <int HD, int QT>
size_t split_bytes(int rows) {
  return kRunGroups<HD, QT> * (sizeof(int4) + (size_t)2 * rows * (HD + 2) * sizeof(float));
}

// Sum over this lane and those before it.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // the lane 1, 2, 4, 8 before in its 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // lane 15 to the second 16 (47 to the fourth)
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // lane 31 to the second 32
  return v;
}

// A step in the line.
struct Place {
  int env, hb, s, len, steps;
};
__device__ __forceinline__ Place after(const PagedAttnArgs& a, const int32_t* lens, Place p, int blocks) {
  if (++p.s < p.steps) return p;
  p.s = 0;
  if (++p.hb < blocks) return p;
  p.hb = 0;
  do {
    p.len = __builtin_amdgcn_readfirstlane(lens[++p.env]);
    p.steps = steps_of(a, p.len);
  } while (p.steps == 0);
  return p;
}

template <int HD, CacheType T, int QT, bool STREAM>
__global__ __launch_bounds__(kRunThreads) void attn_run_kernel(PagedAttnArgs a, const int32_t* __restrict__ lens,
                                                              const int32_t* __restrict__ table, SplitSpace sp, int blocks, int rows) {
  extern __shared__ __align__(16) float lds[];
  __shared__ int4 ends[kRunWaves][2];  // per wave and part: environment, head block, steps past the run, valid
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), me = blockIdx.x;
  if (lane == 0) ends[w][0] = ends[w][1] = make_int4(0, 0, 0, 0);  // by the lane that notes parts down later
  // every wave adds up the steps of all environments, each lane those of a run of them, and finds its place in the line
  const int per = (a.n_env + kWave - 1) / kWave, e0 = min(a.n_env, lane * per), e1 = min(a.n_env, e0 + per);
  const int len0 = e0 < e1 ? lens[e0] : 0;
  int mine = 0;
  bool empty = false;  // an environment without steps
  for (int e = e0; e < e1; ++e) {
    const int n = steps_of(a, e == e0 ? len0 : lens[e]);
    mine += n;
    empty |= n == 0;
  }
  const int upto = wave_scan(mine);
  const long long units = (long long)__builtin_amdgcn_readlane(upto, kWave - 1) * blocks;
  const long long run = run_steps<HD, QT>(units);
  const long long u0 = ((long long)me * kRunWaves + w) * run, first = (long long)(upto - mine) * blocks;
  const int n = __builtin_amdgcn_readfirstlane((int)max(0ll, min(run, units - u0)));
  int e = e0, len = len0;
  long long at = first;
  const bool here = first <= u0 && u0 < (long long)upto * blocks;
  if (here)
    for (;;) {
      const long long m = (long long)steps_of(a, len) * blocks;
      if (u0 < at + m) break;
      at += m;
      len = lens[++e];
    }
  const int holder = n > 0 ? __builtin_ctzll(__ballot(here)) : 0;
  const int env0 = __builtin_amdgcn_readlane(e, holder), len_0 = __builtin_amdgcn_readlane(len, holder);
  const unsigned into = __builtin_amdgcn_readlane((int)(u0 - at), holder);  // steps from the environment's first to u0
  Parts<HD> ps(lds, 2 * kRunWaves, rows);
  if (n > 0) {
    Place cur = {env0, 0, 0, len_0, steps_of(a, len_0)};
    cur.hb = into / (unsigned)cur.steps;
    cur.s = into - cur.hb * cur.steps;
    const int s0 = cur.s;
    bool began = cur.s == 0, outside;  // whether the piece began in this run
    int left = 0;  // steps of the run from a spoiled piece on
    HeadBlock b = head_block<QT>(a, cur.hb);
    Wave<HD, T, QT, STREAM> wave(a);
    // What the run holds of a piece up to p, its last step in the run: all of it to the output, or a part to LDS.
    auto all_of = [&](const Place& p, bool began) { return began && p.s == p.steps - 1; };
    auto write = [&](const Place& p, const HeadBlock& b) {
      const int m16 = lane & 15, g = lane >> 4;
#pragma unroll
      for (int t = 0; t < QT; ++t)
        if (16 * t + m16 < b.n) {
          bf16_t* o = a.o + p.env * a.ld_o + (size_t)(b.head0 + 16 * t + m16) * HD + 4 * g;
          const float r = reciprocal(wave.run.l[t]);
#pragma unroll
          for (int j = 0; j < HD / 16; ++j) store4<T>(o + 16 * j, wave.run.o[t][j], r);
          if (a.lse && g == 0) a.lse[(size_t)p.env * a.n_heads + b.head0 + 16 * t + m16] = log_sum<T>(wave.run.m[t], wave.run.l[t]);
        }
    };
    auto keep = [&](const Place& p, const HeadBlock& b, bool began) {
      ps.put(2 * w + began, wave.run, b.n);
      if (lane == 0) ends[w][began] = make_int4(p.env, p.hb, p.steps - 1 - p.s, 1);
    };
    wave.begin();
    int2 ids = step_pages(table + cur.env * a.ld_table, a.max_pages, cur.s);
    wave.load_q(cur.env, b);
    ids = wave.usable(ids, cur.len, cur.s, outside);
    wave.bad |= outside;
    wave.load_k(ids, b.kvh);
    wave.load_v(wave.v_at(ids, b.kvh));
    Place next = cur;
    if (n > 1) {
      next = after(a, lens, cur, blocks);
      ids = step_pages(table + next.env * a.ld_table, a.max_pages, next.s);
    }
    for (int i = 0; i < n; ++i) {
      float p[QT][8];
      wave.scores(p);
      const bool more = i + 1 < n, ends_here = !more || next.s == 0;
      const bf16_t* next_v = nullptr;
      HeadBlock nb = b;
      Place third = next;
      if (more) {
        if (ends_here) {
          nb = head_block<QT>(a, next.hb);
          wave.load_q(next.env, nb);
        }
        ids = wave.usable(ids, next.len, next.s, outside);
        wave.load_k(ids, nb.kvh);
        next_v = wave.v_at(ids, nb.kvh);
        if (i + 2 < n) {
          third = after(a, lens, next, blocks);
          ids = step_pages(table + third.env * a.ld_table, a.max_pages, third.s);
        }
      }
      wave.template weigh<false>(p, cur.len - kStep * cur.s);
      if (more) wave.load_v(next_v);
      if (ends_here) {
        wave.end();
        const bool all = all_of(cur, began);
        if (!all) keep(cur, b, began);  // its writes go on while the sums are looked at
        if (__builtin_expect(wave.spoiled(), 0)) {
          left = n - i + cur.s - (began ? 0 : s0);
          cur.s = began ? 0 : s0;
          break;
        }
        if (all) write(cur, b);
        if (more) {
          wave.begin();
          began = true;
        }
      }
      wave.bad |= more && outside;
      cur = next;
      next = third;
      b = nb;
    }
    if (__builtin_expect(left > 0, 0)) {  // that piece once more and the others after it
      bool first = true;
#pragma nounroll
      do {
        b = head_block<QT>(a, cur.hb);
        if (first || cur.s == 0) {
          wave.begin();
          wave.load_q(cur.env, b);
        }
        first = false;
        wave.step_apart(table + cur.env * a.ld_table, cur.len, cur.s, b.kvh);
        next = --left > 0 ? after(a, lens, cur, blocks) : cur;
        if (left == 0 || next.s == 0) {
          wave.end();
          if (all_of(cur, began)) write(cur, b);
          else keep(cur, b, began);
          began = true;
        }
        cur = next;
      } while (left > 0);
    }
  }
  __syncthreads();
  // the pieces with parts in LDS: one that began before the workgroup's run, and those that began in a wave's run
  int4 head[kRunWaves], tail[kRunWaves], begun = make_int4(-1, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < kRunWaves; ++i) {
    head[i] = ends[i][0];
    tail[i] = ends[i][1];
  }
#pragma unroll
  for (int w0 = -1; w0 < kRunWaves; ++w0) {
    const bool earlier = w0 < 0;
    int4 end = earlier ? head[0] : tail[max(w0, 0)];
    if (!__builtin_amdgcn_readfirstlane(end.w)) continue;
    const HeadBlock b = head_block<QT>(a, __builtin_amdgcn_readfirstlane(end.y));
    const int env = __builtin_amdgcn_readfirstlane(end.x), i0 = max(w0, 0);
    int parts = 1;
#pragma unroll
    for (int i = i0 + 1; i < kRunWaves; ++i)  // the waves that went on
      if (parts == i - i0 && end.z > 0 && head[i].w) {
        end = head[i];
        ++parts;
      }
    Partial to = {nullptr, nullptr, rows};
    if (earlier || end.z > 0) {
      const size_t slot = 2 * (size_t)me + !earlier;
      to.o = sp.o + slot * rows * HD;
      to.ml = sp.ml + slot * 2 * rows;
      if (!earlier) begun = make_int4(env, end.y, me + 1 + (int)((unsigned)(end.z - 1) / (unsigned)(run * kRunWaves)), 0);
    }
    join_parts<HD, T, kRunWaves>(a, env, b, ps, earlier ? 0 : 2 * w0 + 1, __builtin_amdgcn_readfirstlane(parts), 2 * (i0 + 1), 2, to);
  }
  if (tid == 0) sp.begun[me] = begun;
  if (!__any(empty)) return;
  for (int e = me; e < a.n_env; e += gridDim.x) {
    const int len = lens[e];
    if (steps_of(a, len) == 0) no_keys<HD, T>(a, e, 0, a.n_heads, len);
  }
}

// Adds the partials of a piece that workgroups w0 .. w0 + parts - 1 left, for row `row` of its head block and FW features
// from f0 on.
constexpr int kJoinThreads = 256;
template <int HD, CacheType T, int QT, int FW>
__device__ __forceinline__ void join_piece(const PagedAttnArgs& a, const SplitSpace& sp, int rows, int env, const HeadBlock& b, int row,
                                           int w0, int parts, int f0) {
  constexpr int PG = kJoinThreads * 4 / FW, NW = kJoinThreads / kWave;  // PG runs of partials are added side by side
  constexpr int PT = kRunGroups<HD, QT> / kJoinThreads;                 // partials per thread
  static_assert(kRunGroups<HD, QT> % kJoinThreads == 0, "partials are dealt out evenly");
  __shared__ __align__(16) float so[PG][FW];
  __shared__ float sc[kRunGroups<HD, QT>], sm[NW], sl[NW];
  const int tid = threadIdx.x;
  auto slot = [&](int i) { return 2 * (size_t)(w0 + i) + (i == 0 ? 1 : 0); };
  float mp[PT], lp[PT], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int j = 0; j < PT; ++j) {
    const int i = tid + j * kJoinThreads;
    mp[j] = -INFINITY;
    lp[j] = 0.f;
    if (i < parts) {
      const float* ml = sp.ml + slot(i) * 2 * rows;
      mp[j] = ml[row];
      lp[j] = ml[rows + row];
    }
    m = fmaxf(m, mp[j]);
  }
  m = wave_max(m);
  if ((tid & 63) == 0) sm[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) m = fmaxf(m, sm[i]);
#pragma unroll
  for (int j = 0; j < PT; ++j) {
    const float c = mp[j] == -INFINITY ? 1.f : worth(mp[j], m);
    sc[tid + j * kJoinThreads] = c;
    l = fmaf(lp[j], c, l);
  }
  l = wave_sum(l);
  if ((tid & 63) == 0) sl[tid >> 6] = l;
  __syncthreads();
  const int f = 4 * (tid % (FW / 4)), pg = tid / (FW / 4);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int i = pg; i < parts; i += PG) {
    const f32x4 o = *reinterpret_cast<const f32x4*>(sp.o + (slot(i) * rows + row) * HD + f0 + f);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(o[e], sc[i], v[e]);
  }
  *reinterpret_cast<f32x4*>(&so[pg][f]) = v;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) l += sl[i];
  const float r = reciprocal(l);
  if (tid < FW) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < PG; ++i) t += so[i][tid];
    a.o[env * a.ld_o + (size_t)(b.head0 + row) * HD + f0 + tid] = output<T>(t, r);
  }
  if (a.lse && tid == 0 && f0 == 0) a.lse[(size_t)env * a.n_heads + b.head0 + row] = log_sum<T>(m, l);
}

// Where there are many pieces: one workgroup per workgroup of the run kernel and row of a head block, for the piece that it
// began.
template <int HD, CacheType T, int QT>
__global__ __launch_bounds__(kJoinThreads) void attn_join_begun_kernel(PagedAttnArgs a, SplitSpace sp, int rows) {
  const int w0 = blockIdx.x, row = blockIdx.y;
  const int4 piece = sp.begun[w0];
  if (piece.x < 0) return;
  const HeadBlock b = head_block<QT>(a, piece.y);
  if (row < b.n) join_piece<HD, T, QT, HD>(a, sp, rows, piece.x, b, row, w0, piece.z - w0 + 1, 0);
}

// Where there are few: one workgroup per piece, row of its head block and 64 features, which finds the piece's workgroups from
// the lengths.
template <int HD, CacheType T, int QT>
__global__ __launch_bounds__(kJoinThreads) void attn_join_piece_kernel(PagedAttnArgs a, SplitSpace sp, int blocks, int rows) {
  const int lane = threadIdx.x & 63, env = blockIdx.x / blocks, hb = blockIdx.x - env * blocks, row = blockIdx.y;
  int all = 0, before = 0;
  for (int e = lane; e < a.n_env; e += kWave) {
    const int n = steps_of(a, a.lens[e]);
    all += n;
    before += e < env ? n : 0;
  }
  const int steps = steps_of(a, a.lens[env]);
  const HeadBlock b = head_block<QT>(a, hb);
  if (steps == 0 || row >= b.n) return;
  all = __builtin_amdgcn_readlane(wave_scan(all), kWave - 1);
  before = __builtin_amdgcn_readlane(wave_scan(before), kWave - 1);
  const unsigned long long per = (unsigned long long)run_steps<HD, QT>((long long)all * blocks) * kRunWaves;
  const unsigned long long u0 = (unsigned long long)before * blocks + (unsigned long long)hb * steps;
  const int w0 = (int)(u0 / per), w1 = (int)((u0 + steps - 1) / per);
  if (w0 < w1) join_piece<HD, T, QT, 64>(a, sp, rows, env, b, row, w0, w1 - w0 + 1, 64 * blockIdx.z);
}

// ------------------------------------------------------------------ host
int query_rows(int group, int tiles) { return std::min(16 * tiles, group); }

template <int HD, CacheType T, int QT, bool STREAM, int W>
hipError_t launch_whole(const PagedAttnArgs& a, int blocks, int rows, hipStream_t s) {
  static LdsLimit limit;
  const auto kernel = attn_whole_kernel<HD, T, QT, STREAM, W>;
  const hipError_t e = limit.allow((const void*)kernel, Parts<HD>::bytes(W, 16 * QT));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(blocks, a.n_env), dim3(64 * W), Parts<HD>::bytes(W, rows), s, a, rows);
  return hipGetLastError();
}

template <int HD, CacheType T, int QT, bool STREAM>
hipError_t launch_run(const PagedAttnArgs& a, int blocks, int rows, hipStream_t s) {
  static LdsLimit limit;
  const auto kernel = attn_run_kernel<HD, T, QT, STREAM>;
  const hipError_t e = limit.allow((const void*)kernel, Parts<HD>::bytes(2 * kRunWaves, 16 * QT));
  if (e != hipSuccess) return e;
  const SplitSpace sp = split_space<HD, QT>(a.ws, rows);
  const long long most = (long long)a.n_env * blocks * ((a.max_pages + 1) / 2);  // steps of full lengths
  const int groups = (int)std::min((long long)kRunGroups<HD, QT>, (most + kRunWaves - 1) / kRunWaves);
  hipLaunchKernelGGL(kernel, dim3(groups), dim3(kRunThreads), Parts<HD>::bytes(2 * kRunWaves, rows), s, a, a.lens, a.page_table, sp,
                     blocks, rows);
  // Few pieces have many partials each (us of the join, by pieces / from the list: 2 pieces of 120 partials, heads of 256, 4.7 /
  // 14.5; 8 of 64 4.4 / 5.7); of 512 pieces most workgroups would find nothing to do (64 x 4096 tokens in all 176 / 172).
  const long long pieces = (long long)a.n_env * blocks;
  if (pieces <= kRunGroups<HD, QT> / 4)
    hipLaunchKernelGGL((attn_join_piece_kernel<HD, T, QT>), dim3((unsigned)pieces, rows, HD / 64), dim3(kJoinThreads), 0, s, a, sp, blocks, rows);
  else
    hipLaunchKernelGGL((attn_join_begun_kernel<HD, T, QT>), dim3(groups, rows), dim3(kJoinThreads), 0, s, a, sp, rows);
  return hipGetLastError();
}

// Whether the keys are split, of `pieces` environments and head blocks.  Short keys are taken whole: the split's second launch
// and its way through the workspace cost more than they save (GPU us, whole / split: 1 x 278 tokens, 32 pieces, 6.3 / 10.5; 1 x
// 512, 8 pieces, 7.6 / 9.5), up to 1024 tokens where there are pieces enough to fill half the GPU (32 x 700 tokens, 256 pieces,
// 18.2 / 26.1; 16 of up to 1024, 128 pieces, 12.8 / 15.3; but 8 x 1024, 64 pieces, 18.2 / 14.5).  Beyond, the split is about as
// fast where pieces abound (64 x 4096, 512 pieces, 169 / 172.5) and faster where they are few or uneven (1 x 1024, 8 pieces, 12.0 /
// 9.8; 8 x 3000, 8 pieces, 29.6 / 11.4; 64 of up to 2048 56.5 / 54.0).
bool split_keys(long long pieces, int max_pages) { return max_pages > (pieces >= 128 ? 64 : 32); }

template <int HD, CacheType T, int QT, bool STREAM>
hipError_t launch_blocks(const PagedAttnArgs& a, hipStream_t s) {
  const int group = a.n_heads / a.n_kv_heads, blocks = head_blocks<QT>(group) * a.n_kv_heads, rows = query_rows(group, QT);
  const long long pieces = (long long)a.n_env * blocks;
  if (split_keys(pieces, a.max_pages)) return launch_run<HD, T, QT, STREAM>(a, blocks, rows, s);
  // One wave per piece where those fill the GPU, else four (us, one / four: 512 x 30 tokens, 8 key heads 16 / 28; 512 x 128
  // 47 / 53; 64 x 300, 32 key heads 52.9 / 54; 512 pieces of 300 tokens 16.9 / 16.2, 256 of 64 5.2 / 4.7)
  if (pieces >= 1024) return launch_whole<HD, T, QT, STREAM, 1>(a, blocks, rows, s);
  return launch_whole<HD, T, QT, STREAM, 4>(a, blocks, rows, s);
}

// Query heads of a group by tiles of 16: up to head_dim 128 two share a step's keys in registers (at 256 two tiles' sums do
// not fit), further ones read the keys again.
int query_tiles(int group, int head_dim) { return head_dim < 256 && group > 16 ? 2 : 1; }

// A pool of up to 32 MB, the L2s' size, may be in the caches from one step to the next (278 tokens, 32 key heads: 6.3 us with
// cached loads; in a larger pool, past the caches, 7.9); beyond, reads past the caches are faster (64 x 4096: 191 and 173 us).
bool stream_pool(const PagedAttnArgs& a) {
  return (size_t)a.n_pages * a.n_kv_heads * kPage * a.head_dim * 2 * sizeof(bf16_t) > (size_t)32 << 20;
}

template <int HD, CacheType T, int QT>
hipError_t launch_tiles(const PagedAttnArgs& a, hipStream_t s) {
  return stream_pool(a) ? launch_blocks<HD, T, QT, true>(a, s) : launch_blocks<HD, T, QT, false>(a, s);
}
template <int HD, CacheType T>
hipError_t launch_heads(const PagedAttnArgs& a, hipStream_t s) {
  if constexpr (HD < 256)
    if (query_tiles(a.n_heads / a.n_kv_heads, HD) == 2) return launch_tiles<HD, T, 2>(a, s);
  return launch_tiles<HD, T, 1>(a, s);
}
template <CacheType T>
hipError_t launch_type(const PagedAttnArgs& a, hipStream_t s) {
  if (a.head_dim == 64) return launch_heads<64, T>(a, s);
  if (a.head_dim == 128) return launch_heads<128, T>(a, s);
  if (a.head_dim == 256) return launch_heads<256, T>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace

size_t paged_attn_bytes(int n_env, int n_heads, int n_kv_heads, int head_dim, int max_pages) {
  const int group = n_heads / n_kv_heads, tiles = query_tiles(group, head_dim), rows = query_rows(group, tiles);
  const int blocks = (tiles == 1 ? head_blocks<1>(group) : head_blocks<2>(group)) * n_kv_heads;
  if (!split_keys((long long)n_env * blocks, max_pages)) return 256;
  if (head_dim == 64) return tiles == 1 ? split_bytes<64, 1>(rows) : split_bytes<64, 2>(rows);
  if (head_dim == 128) return tiles == 1 ? split_bytes<128, 1>(rows) : split_bytes<128, 2>(rows);
  return split_bytes<256, 1>(rows);
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  return a.type == kBf16 ? launch_type<kBf16>(a, s) : launch_type<kF16>(a, s);
}

}  // namespace vla
