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

typedef unsigned u32x4v __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const bf16_t* p) {  // past the caches: a page is read by one wave
  const u32x4v v = __builtin_nontemporal_load(reinterpret_cast<const u32x4v*>(p));
  return make_uint4(v.x, v.y, v.z, v.w);
}

// The pages of step s; entries up to the table's end may be read before the length is known.
__device__ __forceinline__ int2 step_pages(const PagedAttnArgs& a, const int32_t* pt, int s) {
  return make_int2(pt[min(2 * s, a.max_pages - 1)], pt[min(2 * s + 1, a.max_pages - 1)]);
}

// Steps s0, s0 + stride, ... below s1 of environment `env`, of `len` keys, for head block b; `ids` are step s0's pages.  A
// step's keys are requested as soon as the step before has used its own, its values likewise, so that a wave always has one
// step's pages on the way.
template <int HD, CacheType T, int QT>
__device__ __forceinline__ void attend(const PagedAttnArgs& a, int env, const HeadBlock& b, int len, int s0, int s1, int stride,
                                       int2 ids, Running<HD, QT>& run) {
  constexpr int KC = HD / 32, VC = HD / 16;
  const int lane = threadIdx.x & 63, m16 = lane & 15, g = lane >> 4;
  const float scale = a.scale * kLog2e;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    run.m[t] = -INFINITY;
    run.l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < VC; ++i) run.o[t][i] = {0.f, 0.f, 0.f, 0.f};
  }
  if (s0 >= s1) return;
  uint4 q[QT][KC];  // columns past the block's heads repeat its last one; nothing reads what becomes of them
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int i = 0; i < KC; ++i)
      q[t][i] = *reinterpret_cast<const uint4*>(a.q + env * a.ld_q + (size_t)(b.head0 + min(16 * t + m16, b.n - 1)) * HD + 32 * i + 8 * g);
  const int32_t* pt = a.page_table + env * a.ld_table;
  const int last = (len - 1) / kPage;
  const size_t page_elems = (size_t)a.n_kv_heads * kPage * HD;
  // row lane % 16 of the K operand of tile t: page m16 / 8 of the step, slot 8 (m16 / 4 % 2) + 4 t + m16 % 4
  const bf16_t* kb = a.pages.k + ((size_t)b.kvh * kPage + 8 * ((m16 >> 2) & 1) + (m16 & 3)) * HD + 8 * g;
  const bf16_t* vb = a.pages.v + ((size_t)b.kvh * HD + m16) * kPage + 8 * (g & 1);
  bool bad = false;
  auto check = [&](int s) {  // a bad page is not read: NaN from there on
    if (2 * s + 1 > last) ids.y = ids.x;
    if ((unsigned)ids.x >= (unsigned)a.n_pages || (unsigned)ids.y >= (unsigned)a.n_pages) {
      ids = make_int2(0, 0);
      bad = true;
    }
  };
  uint4 k[2][KC], v[VC];
  auto load_k = [&] {
    const bf16_t* kp = kb + (m16 < 8 ? ids.x : ids.y) * page_elems;
#pragma unroll
    for (int i = 0; i < KC; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) k[t][i] = load_once(kp + 4 * t * HD + 32 * i);
  };
  auto load_v = [&](const bf16_t* vp) {
#pragma unroll
    for (int i = 0; i < VC; ++i) v[i] = load_once(vp + 16 * i * kPage);
  };
  check(s0);
  load_k();
  load_v(vb + (g < 2 ? ids.x : ids.y) * page_elems);
  int2 after = step_pages(a, pt, s0 + stride);  // of the next step
  for (int s = s0; s < s1; s += stride) {
    const bool more = s + stride < s1;
    const int left = len - kStep * s;  // keys of the step that count
    float p[QT][8];
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
    const bf16_t* next_v = vb;
    if (more) {
      ids = after;
      check(s + stride);
      load_k();
      next_v = vb + (g < 2 ? ids.x : ids.y) * page_elems;
      after = step_pages(a, pt, s + 2 * stride);
    }
    uint4 hi[QT], lo[QT];
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
        const float c = run.m[t] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(run.m[t] - mx);  // nothing to scale yet: 1
        run.l[t] *= c;
#pragma unroll
        for (int i = 0; i < VC; ++i) run.o[t][i] *= c;
        run.m[t] = mx;
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
    for (int i = 0; i < VC; ++i)
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        run.o[t][i] = mfma<T>(v[i], hi[t], run.o[t][i]);
        run.o[t][i] = mfma<T>(v[i], lo[t], run.o[t][i]);
      }
    if (more) load_v(next_v);
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) run.l[t] = bad ? __builtin_nanf("") : column_sum(run.l[t]);
}

// Where the joined result of a head block goes: the output, or a partial (o fp32 [16 QT][HD], m and l [16 QT] each).
struct Partial {
  float* o;
  float* ml;
};

// LDS of the join of W waves: the rows of a head block, padded by one 16-byte bank group.
template <int HD, int QT, int W>
constexpr size_t kJoinBytes = (size_t)W * 16 * QT * (HD + 4 + 2) * sizeof(float);

// Joins the W waves' parts through LDS and writes the output rows (part.o == null) or the partial.
template <int HD, CacheType T, int QT, int W>
__device__ __forceinline__ void join_waves(const PagedAttnArgs& a, int env, const HeadBlock& b, Running<HD, QT>& run, Partial part) {
  extern __shared__ __align__(16) float lds[];
  float* so = lds;                                  // [W][16 QT][HD + 4]
  float* sm = lds + (size_t)W * 16 * QT * (HD + 4);  // [W][16 QT]
  float* sl = sm + W * 16 * QT;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, m16 = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int h = w * 16 * QT + 16 * t + m16;
    if (16 * t + m16 < b.n) {
      if (g == 0) {
        sm[h] = run.m[t];
        sl[h] = run.l[t];
      }
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) *reinterpret_cast<f32x4*>(so + (size_t)h * (HD + 4) + 16 * i + 4 * g) = run.o[t][i];
    }
  }
  __syncthreads();
  for (int i = tid; i < b.n * (HD / 4); i += 64 * W) {
    const int h = i / (HD / 4), f = 4 * (i % (HD / 4));
    float mu[W], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int u = 0; u < W; ++u) {
      mu[u] = sm[u * 16 * QT + h];
      m = fmaxf(m, mu[u]);
    }
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < W; ++u) {
      const float c = mu[u] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mu[u] - m);  // a wave without keys adds zeros
      l = fmaf(sl[u * 16 * QT + h], c, l);
      const f32x4 o = *reinterpret_cast<const f32x4*>(so + (size_t)(u * 16 * QT + h) * (HD + 4) + f);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(o[e], c, v[e]);
    }
    if (part.o) {
      *reinterpret_cast<f32x4*>(part.o + h * HD + f) = v;
      if (f == 0) {
        part.ml[h] = m;
        part.ml[16 * QT + h] = l;
      }
    } else {
      const float r = l == 0.f ? 0.f : 1.f / l;  // no key with a score above -inf: zeros
      bf16_t h4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) h4[e] = from_f32<T>(v[e] * r);
      *reinterpret_cast<uint2*>(a.o + env * a.ld_o + (size_t)(b.head0 + h) * HD + f) =
          make_uint2(h4[0] | (uint32_t)h4[1] << 16, h4[2] | (uint32_t)h4[3] << 16);
      if (a.lse && f == 0) a.lse[(size_t)env * a.n_heads + b.head0 + h] = log_sum<T>(m, l);
    }
  }
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
  if (a.lse && (int)threadIdx.x < n) a.lse[(size_t)env * a.n_heads + head0 + threadIdx.x] = len == 0 ? -INFINITY : v;
}

// One workgroup of W waves per (head block, environment).
template <int HD, CacheType T, int QT, int W>
__global__ __launch_bounds__(64 * W) void attn_whole_kernel(PagedAttnArgs a) {
  const int env = blockIdx.y, len = __builtin_amdgcn_readfirstlane(a.lens[env]), steps = steps_of(a, len);
  const HeadBlock b = head_block<QT>(a, blockIdx.x);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int2 ids = a.max_pages > 0 ? step_pages(a, a.page_table + env * a.ld_table, w) : make_int2(0, 0);
  if (steps == 0) return no_keys<HD, T>(a, env, b.head0, b.n, len);
  Running<HD, QT> run;
  attend<HD, T, QT>(a, env, b, len, w, steps, W, ids, run);
  join_waves<HD, T, QT, W>(a, env, b, run, {nullptr, nullptr});
}

// ------------------------------------------------------------------ split over the keys
// The steps of all environments and head blocks lie in one line, environment by environment, head block by head block; a
// persistent grid of workgroups takes runs of equal length.  A workgroup's first and last piece (of one environment and head
// block) may be a part: then it leaves a partial, in slot 2 w + 1 of the workspace if it began the piece, else in 2 w, and
// who began a piece notes it down for attn_join_kernel, which adds its partials in order.
template <int HD>
constexpr int kSplitGroups = HD == 256 ? 256 : 512;
constexpr int kSplitWaves = 4;

// Units of a workgroup: whole rounds of its waves.
template <int HD>
__device__ __forceinline__ long long units_per_group(long long units) {
  const long long n = (units + kSplitGroups<HD> - 1) / kSplitGroups<HD>;
  return max((n + kSplitWaves - 1) / kSplitWaves, 1ll) * kSplitWaves;
}

struct SplitSpace {
  int4* begun;  // [groups] the piece that workgroup w began and did not end: environment, head block, last workgroup; or -1
  float* o;     // [2 groups][16 QT][HD]
  float* ml;    // [2 groups][2][16 QT]
};
template <int HD, int QT>
SplitSpace split_space(void* ws) {
  char* p = static_cast<char*>(ws);
  float* o = reinterpret_cast<float*>(p + kSplitGroups<HD> * sizeof(int4));
  return {reinterpret_cast<int4*>(p), o, o + (size_t)2 * kSplitGroups<HD> * 16 * QT * HD};
}
template <int HD>
size_t split_bytes(int tiles) {
  return kSplitGroups<HD> * (sizeof(int4) + (size_t)2 * 16 * tiles * (HD + 2) * sizeof(float));
}

template <int HD, CacheType T, int QT>
__global__ __launch_bounds__(64 * kSplitWaves) void attn_split_kernel(PagedAttnArgs a, SplitSpace sp, int blocks) {
  constexpr int NT = 64 * kSplitWaves;
  __shared__ long long sums[kSplitWaves];
  __shared__ long long found_base;
  __shared__ int found_env, found_len;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), me = blockIdx.x;
  // every workgroup adds up the steps of all environments, thread t those of a run of them
  const int per = (a.n_env + NT - 1) / NT, e0 = min(a.n_env, tid * per), e1 = min(a.n_env, e0 + per);
  long long mine = 0;
  const int len0 = e0 < e1 ? a.lens[e0] : 0;
  for (int e = e0; e < e1; ++e) mine += steps_of(a, e == e0 ? len0 : a.lens[e]);
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const long long v = __shfl_up(upto, o, kWave);
    if (lane >= o) upto += v;
  }
  if (lane == 63) sums[w] = upto;
  __syncthreads();
  long long units = 0;
#pragma unroll
  for (int i = 0; i < kSplitWaves; ++i) {
    if (i < w) upto += sums[i];
    units += sums[i];
  }
  units *= blocks;
  const long long per_group = units_per_group<HD>(units), begin = min(me * per_group, units), u1 = min(begin + per_group, units);
  long long u = begin;
  if ((upto - mine) * blocks <= u && u < upto * blocks) {
    long long at = (upto - mine) * blocks;
    int e = e0, len = len0;
    for (;;) {
      const long long n = (long long)steps_of(a, len) * blocks;
      if (u < at + n) break;
      at += n;
      len = a.lens[++e];
    }
    found_base = at;
    found_env = e;
    found_len = len;
  }
  int4 begun = make_int4(-1, 0, 0, 0);
  __syncthreads();
  if (u < u1) {
    long long base = found_base;
    int env = __builtin_amdgcn_readfirstlane(found_env), len = __builtin_amdgcn_readfirstlane(found_len);
    while (u < u1) {
      const int steps = steps_of(a, len);
      const long long end = base + (long long)steps * blocks;
      while (u < u1 && u < end) {
        const int hb = __builtin_amdgcn_readfirstlane((int)((unsigned)(u - base) / (unsigned)steps));
        const int s0 = __builtin_amdgcn_readfirstlane((int)((u - base) - (long long)hb * steps));
        const int n = __builtin_amdgcn_readfirstlane((int)min((long long)(steps - s0), u1 - u));
        const HeadBlock b = head_block<QT>(a, hb);
        const int2 ids = step_pages(a, a.page_table + env * a.ld_table, s0 + w);
        Running<HD, QT> run;
        attend<HD, T, QT>(a, env, b, len, s0 + w, s0 + n, kSplitWaves, ids, run);
        Partial part = {nullptr, nullptr};
        if (n < steps) {
          const bool began = u - s0 >= begin;
          const size_t slot = 2 * (size_t)me + began;
          part = {sp.o + slot * 16 * QT * HD, sp.ml + slot * 2 * 16 * QT};
          if (began) begun = make_int4(env, hb, me + (int)((unsigned)(u - s0 + steps - 1 - begin) / (unsigned)per_group), 0);
        }
        __syncthreads();  // the last join's reads of LDS
        join_waves<HD, T, QT, kSplitWaves>(a, env, b, run, part);
        u += n;
      }
      base = end;
      if (u < u1) len = __builtin_amdgcn_readfirstlane(a.lens[++env]);
    }
  }
  if (tid == 0) sp.begun[me] = begun;
  for (int e = me; e < a.n_env; e += kSplitGroups<HD>) {
    const int len = a.lens[e];
    if (steps_of(a, len) == 0) no_keys<HD, T>(a, e, 0, a.n_heads, len);
  }
}

// One workgroup per (workgroup of the split, row of a head block): joins the piece that it began.
constexpr int kJoinThreads = 256;
template <int HD, CacheType T, int QT>
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(PagedAttnArgs a, SplitSpace sp) {
  constexpr int PG = kJoinThreads * 4 / HD, NW = kJoinThreads / kWave;  // PG runs of partials are added side by side
  constexpr int PT = kSplitGroups<HD> / kJoinThreads;                   // partials per thread
  static_assert(kSplitGroups<HD> % kJoinThreads == 0, "partials are dealt out evenly");
  __shared__ __align__(16) float so[PG][HD];
  __shared__ float sc[kSplitGroups<HD>], sm[NW], sl[NW];
  const int w0 = blockIdx.x, row = blockIdx.y, tid = threadIdx.x;
  const int4 piece = sp.begun[w0];
  if (piece.x < 0) return;
  const HeadBlock b = head_block<QT>(a, piece.y);
  if (row >= b.n) return;
  const int parts = piece.z - w0 + 1;
  auto slot = [&](int i) { return 2 * (size_t)(w0 + i) + (i == 0 ? 1 : 0); };
  float mp[PT], lp[PT], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int j = 0; j < PT; ++j) {
    const int i = tid + j * kJoinThreads;
    mp[j] = -INFINITY;
    lp[j] = 0.f;
    if (i < parts) {
      const float* ml = sp.ml + slot(i) * 2 * 16 * QT;
      mp[j] = ml[row];
      lp[j] = ml[16 * QT + row];
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
    const float c = mp[j] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mp[j] - m);
    sc[tid + j * kJoinThreads] = c;
    l = fmaf(lp[j], c, l);
  }
  l = wave_sum(l);
  if ((tid & 63) == 0) sl[tid >> 6] = l;
  __syncthreads();
  const int f = 4 * (tid % (HD / 4)), pg = tid / (HD / 4);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int i = pg; i < parts; i += PG) {
    const f32x4 o = *reinterpret_cast<const f32x4*>(sp.o + slot(i) * 16 * QT * HD + row * HD + f);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(o[e], sc[i], v[e]);
  }
  *reinterpret_cast<f32x4*>(&so[pg][f]) = v;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) l += sl[i];
  const float r = l == 0.f ? 0.f : 1.f / l;
  if (tid < HD) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < PG; ++i) t += so[i][tid];
    a.o[piece.x * a.ld_o + (size_t)(b.head0 + row) * HD + tid] = from_f32<T>(t * r);
  }
  if (a.lse && tid == 0) a.lse[(size_t)piece.x * a.n_heads + b.head0 + row] = log_sum<T>(m, l);
}

// ------------------------------------------------------------------ host
bool split_keys(int max_pages) { return max_pages > 32; }

template <int HD, CacheType T, int QT, int W>
hipError_t launch_whole(const PagedAttnArgs& a, int blocks, hipStream_t s) {
  static LdsLimit limit;
  constexpr size_t lds = kJoinBytes<HD, QT, W>;
  const hipError_t e = limit.allow((const void*)attn_whole_kernel<HD, T, QT, W>, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attn_whole_kernel<HD, T, QT, W>), dim3(blocks, a.n_env), dim3(64 * W), lds, s, a);
  return hipGetLastError();
}

template <int HD, CacheType T, int QT>
hipError_t launch_blocks(const PagedAttnArgs& a, hipStream_t s) {
  const int blocks = head_blocks<QT>(a.n_heads / a.n_kv_heads) * a.n_kv_heads;
  if (!split_keys(a.max_pages)) return launch_whole<HD, T, QT, 4>(a, blocks, s);
  static LdsLimit limit;
  constexpr size_t lds = kJoinBytes<HD, QT, kSplitWaves>;
  const hipError_t e = limit.allow((const void*)attn_split_kernel<HD, T, QT>, lds);
  if (e != hipSuccess) return e;
  const SplitSpace sp = split_space<HD, QT>(a.ws);
  const int rows = std::min(16 * QT, a.n_heads / a.n_kv_heads);
  hipLaunchKernelGGL((attn_split_kernel<HD, T, QT>), dim3(kSplitGroups<HD>), dim3(64 * kSplitWaves), lds, s, a, sp, blocks);
  hipLaunchKernelGGL((attn_join_kernel<HD, T, QT>), dim3(kSplitGroups<HD>, rows), dim3(kJoinThreads), 0, s, a, sp);
  return hipGetLastError();
}

// Query heads of a group by tiles of 16: up to head_dim 128 two share a step's keys in registers (at 256 two tiles' sums do
// not fit), further ones read the keys again.
int query_tiles(int n_heads, int n_kv_heads, int head_dim) { return head_dim < 256 && n_heads / n_kv_heads > 16 ? 2 : 1; }

template <int HD, CacheType T>
hipError_t launch_heads(const PagedAttnArgs& a, hipStream_t s) {
  if constexpr (HD < 256)
    if (query_tiles(a.n_heads, a.n_kv_heads, HD) == 2) return launch_blocks<HD, T, 2>(a, s);
  return launch_blocks<HD, T, 1>(a, s);
}
template <CacheType T>
hipError_t launch_type(const PagedAttnArgs& a, hipStream_t s) {
  if (a.head_dim == 64) return launch_heads<64, T>(a, s);
  if (a.head_dim == 128) return launch_heads<128, T>(a, s);
  if (a.head_dim == 256) return launch_heads<256, T>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace

size_t paged_attn_bytes(int, int n_heads, int n_kv_heads, int head_dim, int max_pages) {
  if (!split_keys(max_pages)) return 256;
  const int tiles = query_tiles(n_heads, n_kv_heads, head_dim);
  return head_dim == 64 ? split_bytes<64>(tiles) : head_dim == 128 ? split_bytes<128>(tiles) : split_bytes<256>(tiles);
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  return a.type == kBf16 ? launch_type<kBf16>(a, s) : launch_type<kF16>(a, s);
}

}  // namespace vla
