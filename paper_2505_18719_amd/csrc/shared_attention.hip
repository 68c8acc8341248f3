// Attention of one new token per environment where groups of environments share their first pages (vla_shared_attention).
//
// Bound: HBM and the matrix units: the shared keys and values once for a group, 4 head_dim flops a query and key.  Three parts:
//   shared  a workgroup takes 32 columns a wave, a column being one query head of one environment of a group, over a run of the
//           group's shared pages, which pass through LDS in tiles of four as in attention over whole prompts, and leaves its
//           columns' maximum, sum of weights and sum of weighted values
//   own     a workgroup takes an environment's remaining pages, as attention without sharing does, and joins the parts; where
//           there are few environments, a run of them, and leaves another part
//   join    then adds the parts
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged_dev.h"
#include "prompt_dev.h"

namespace vla {
namespace {

struct Plan {
  bool share;      // else vla_paged_attention's kernels
  int waves;       // of a workgroup of the shared part
  int parts, own;  // runs of the shared pages, and of an environment's own
};

// The parts of all columns: sums of weighted values [part][environment][head][HD], maxima (to base 2) and sums of weights.
struct PartSpace {
  float* o;
  float2* ml;
  size_t columns;  // n_env * n_heads
};
PartSpace part_space(void* ws, const PagedAttnArgs& a, int parts) {
  const size_t columns = (size_t)a.n_env * a.n_heads;
  float* o = static_cast<float*>(ws);
  return {o, reinterpret_cast<float2*>(o + (size_t)parts * columns * a.head_dim), columns};
}

// Items of the groups, as seq_items: C columns each.
template <int C>
__device__ __forceinline__ bool find_group(const SharedArgs& s, int item, int group, int& e0, int& n_col, int& c0, int& pages) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = s.n_groups;
  auto first = [&](int g) { return (int)((long long)min(max(s.group_start[g], 0), s.a.n_env) * group / C) + g; };
  for (;;) {
    const int step = (n + kWave - 1) / kWave, at = lo + lane * step;
    const int found = __popcll(__ballot(lane * step < n && first(min(at, s.n_groups)) <= item));
    if (found == 0) return false;
    lo += (found - 1) * step;
    n = min(step, n - (found - 1) * step);
    if (step == 1) break;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  e0 = __builtin_amdgcn_readfirstlane(s.group_start[lo]);
  const int e1 = __builtin_amdgcn_readfirstlane(s.group_start[lo + 1]);
  if (e0 < 0 || e1 <= e0 || e1 > s.a.n_env) return false;
  n_col = (e1 - e0) * group;
  c0 = (item - first(lo)) * C;
  pages = min(__builtin_amdgcn_readfirstlane(s.shared_pages[lo]), s.a.max_pages);
  return c0 < n_col && pages > 0;
}
// Pages that environment env shares with its group.
__device__ __forceinline__ int shared_of(const SharedArgs& s, int env) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = s.n_groups;
  for (;;) {
    const int step = (n + kWave - 1) / kWave, at = lo + lane * step;
    const int found = __popcll(__ballot(lane * step < n && s.group_start[min(at, s.n_groups)] <= env));
    if (found == 0) return 0;
    lo += (found - 1) * step;
    n = min(step, n - (found - 1) * step);
    if (step == 1) break;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const int e0 = s.group_start[lo], e1 = s.group_start[lo + 1];
  if (e0 < 0 || e0 > env || e1 <= env || e1 > s.a.n_env) return 0;
  return __builtin_amdgcn_readfirstlane(min(max(s.shared_pages[lo], 0), s.a.max_pages));
}

__host__ __device__ __forceinline__ int run_of(int n, int parts) { return (n + parts - 1) / parts; }

// ------------------------------------------------------------------ shared pages
template <int HD, CacheType T, int NW>
__global__ __launch_bounds__(64 * NW, HD == 256 ? 1 : 2) void attn_shared_kernel(SharedArgs args, PartSpace sp, int parts) {
  using namespace tiles;
  extern __shared__ __align__(16) char lds[];
  constexpr int C = 32 * NW, CH = HD / 8, RPK = 64 / CH, PK = kPage / RPK;  // chunks of a row, rows of a copy, copies of a page
  const PagedAttnArgs& a = args.a;
  const int kvh = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads, part = rest % parts, group = a.n_heads / a.n_kv_heads;
  int e0, n_col, c0, pages;
  if (!find_group<C>(args, rest / parts, group, e0, n_col, c0, pages)) return;
  const int n_tiles = (pages + 3) / 4, run = run_of(n_tiles, parts), j0 = part * run, j1 = min(j0 + run, n_tiles);
  if (j0 >= j1) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = c0 + 32 * wave + (lane & 31), c = min(col, n_col - 1), env = e0 + c / group, head = kvh * group + c % group;
  Queries<HD, T> w;
  w.load(a.q + env * a.ld_q + (int64_t)head * HD, a.scale);
  const TileLane<HD, true> at;
  const int32_t* pt = a.page_table + e0 * a.ld_table;
  auto tile = [&](int j, int which) { return lds + (2 * (j & 1) + which) * kTileBytes<HD>; };
  bool bad = false;
  // This lane's place in a copy of keys: of rows, in their turned order.
  const uint32_t row = lane / CH;
  const uint32_t lb = (uint32_t)(uintptr_t)((lds_ptr_t*)lds);
  const int page_bytes = kPage * HD * 2;
  // Pages of tile j, one in a lane of four; those behind the last are it once more.
  auto ids_of = [&](int j) { return pt[min(4 * j + (lane & 3), pages - 1)]; };
  auto copy = [&](int j, int id) {
    const bool outside = (unsigned)id >= (unsigned)a.n_pages;
    bad |= outside;
    if (outside) id = 0;
#pragma unroll
    for (int i = 0; i < (8 * PK + NW - 1) / NW; ++i) {
      const int n = i * NW + wave;  // keys' copies first, then the values'
      if (8 * PK % NW != 0 && n >= 8 * PK) break;
      const int p = n / PK % 4, k = n % PK, values = n / (4 * PK);
      const int page = __builtin_amdgcn_readlane(id, p);
      const char* from = reinterpret_cast<const char*>(values ? a.pages.v : a.pages.k) + ((int64_t)page * a.n_kv_heads + kvh) * page_bytes;
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)from, (short)0, page_bytes, 0x00020000);
      const uint32_t R = k * RPK + row;
      const uint32_t voff = values ? k * 1024 + 16 * lane : R * HD * 2 + 16 * ((lane % CH) ^ swz<HD>(R));
      const uint32_t to = lb + (2 * (j & 1) + values) * kTileBytes<HD> + p * page_bytes + k * 1024;
      lds_dma16(__builtin_amdgcn_readfirstlane(to), voff, rs, 0);
    }
  };
  copy(j0, ids_of(j0));
  int id = ids_of(min(j0 + 1, n_tiles - 1));
  WAIT_VMCNT(0);
  __syncthreads();
  const bool some = c0 + 32 * wave < n_col;
  for (int j = j0; j < j1; ++j) {
    if (j + 1 < j1) {
      copy(j + 1, id);
      id = ids_of(min(j + 2, n_tiles - 1));
    }
    if (some) {
      f32x16 s[2];
      w.scores(at, tile(j, 0), s);
      if (kPage * pages - kTile * j < kTile) w.template mask<true>(s, kPage * pages - 1 - kTile * j);
      w.follow(s);
      w.weigh(s);
      w.add(at, tile(j, 1), s);
    }
    WAIT_VMCNT(0);
    __syncthreads();
  }
  __shared__ int any_bad;
  if (threadIdx.x == 0) any_bad = 0;
  __syncthreads();
  if (bad) any_bad = 1;
  __syncthreads();
  if (col >= n_col) return;
  const float l = any_bad ? __builtin_nanf("") : half_sum(w.l);
  const size_t to = part * sp.columns + (size_t)env * a.n_heads + head;
  // in half precision the weights are held at another power of two than those of the own pages
  if (lane < 32) sp.ml[to] = make_float2(w.m == -INFINITY ? -INFINITY : w.m * w.scale + (kWeightExp<T> - tiles::kHeldExp<T>), l);
  float* o = sp.o + to * HD + 4 * (lane >> 5);
#pragma unroll
  for (int mb = 0; mb < HD / 32; ++mb)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(o + 32 * mb + 8 * i) = {w.o[mb][4 * i], w.o[mb][4 * i + 1], w.o[mb][4 * i + 2], w.o[mb][4 * i + 3]};
}

// ------------------------------------------------------------------ own pages, and the join
// What an environment's length says: its own keys, their steps, and what the rows are without any part.
struct Own {
  int skip, len, steps;  // pages shared, own keys, their steps
  bool zeros, bad;
};
template <CacheType T>
__device__ __forceinline__ Own own_of(const SharedArgs& s, int env) {
  const int len = __builtin_amdgcn_readfirstlane(s.a.lens[env]), skip = shared_of(s, env);
  Own o = {skip, 0, 0, len == 0, false};
  o.bad = len < 0 || len > (long long)s.a.max_pages * kPage || (len > 0 && len < (long long)skip * kPage);
  if (o.bad || o.zeros) return o;
  o.len = len - skip * kPage;
  o.steps = (o.len + kStep<T> - 1) / kStep<T>;
  return o;
}

// Four features from f on of one head: parts of the shared pages (n of them), parts of its own (from `first` on, m of them), and N
// parts in LDS.
template <int HD, CacheType T, int N>
__device__ __forceinline__ void join_column(const PagedAttnArgs& a, const PartSpace& sp, int env, int head, int f, int n, int first, int m,
                                            const Parts<HD>* ps, int h) {
  const size_t at = (size_t)env * a.n_heads + head;
  auto part = [&](int i) { return i < n ? i : first + i - n; };
  float mx = -INFINITY;
#pragma unroll
  for (int u = 0; u < N; ++u) mx = fmaxf(mx, ps->ml[u * 2 * ps->rows + h]);
  for (int i = 0; i < n + m; ++i) mx = fmaxf(mx, sp.ml[part(i) * sp.columns + at].x);
  float l = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const float mu = ps->ml[u * 2 * ps->rows + h], c = mu == -INFINITY ? 1.f : worth(mu, mx);
    l = fmaf(ps->ml[(u * 2 + 1) * ps->rows + h], c, l);
    const f32x4 o = *reinterpret_cast<const f32x4*>(ps->o + (size_t)(u * ps->rows + h) * (HD + 4) + f);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(o[e], c, v[e]);
  }
#pragma unroll 4
  for (int i = 0; i < n + m; ++i) {
    const size_t p = part(i) * sp.columns + at;
    const float2 ml = sp.ml[p];
    const float c = ml.x == -INFINITY ? 1.f : worth(ml.x, mx);
    l = fmaf(ml.y, c, l);
    const f32x4 o = *reinterpret_cast<const f32x4*>(sp.o + p * HD + f);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(o[e], c, v[e]);
  }
  store4<T>(a.o + env * a.ld_o + (size_t)head * HD + f, v, reciprocal(l));
  if (a.lse && f == 0) a.lse[at] = log_sum<T>(mx, l);
}
// Runs of the shared pages that there are parts of.
__device__ __forceinline__ int shared_parts(int skip, int parts) {
  const int n = (skip + 3) / 4;
  return n == 0 ? 0 : (n + run_of(n, parts) - 1) / run_of(n, parts);
}
template <int HD, CacheType T>
__device__ __forceinline__ void fill_rows(const PagedAttnArgs& a, int env, int head0, int n, bool zeros) {
  const float v = zeros ? 0.f : __builtin_nanf("");
  for (int i = threadIdx.x; i < n * HD; i += blockDim.x) a.o[env * a.ld_o + (size_t)head0 * HD + i] = from_f32<T>(v);
  if (a.lse)
    for (int i = threadIdx.x; i < n; i += blockDim.x) a.lse[(size_t)env * a.n_heads + head0 + i] = zeros ? -INFINITY : v;
}

template <int HD, CacheType T, int QT, int W>
__global__ __launch_bounds__(64 * W) void attn_own_kernel(SharedArgs args, PartSpace sp, int parts, int runs, int rows) {
  extern __shared__ __align__(16) float own_lds[];
  const PagedAttnArgs& a = args.a;
  const int env = blockIdx.y, run = blockIdx.x % runs;
  const HeadBlock b = head_block<QT>(a, blockIdx.x / runs);
  const Own own = own_of<T>(args, env);
  if (own.zeros || own.bad) {
    if (runs == 1) fill_rows<HD, T>(a, env, b.head0, b.n, own.zeros);
    return;
  }
  const int per = run_of(own.steps, runs), s0 = run * per, s1 = min(s0 + per, own.steps);
  if (runs > 1 && s0 >= s1) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), max_pages = a.max_pages - own.skip;
  const int32_t* pt = a.page_table + env * a.ld_table + own.skip;
  Wave<HD, T, QT, false> wave(a);
  wave.begin();
  if (s0 + w < s1) {
    bool outside;
    wave.load_q(env, b);
    StepPages<T> ids(pt, max_pages, s0 + w);
    ids = wave.usable(ids, own.len, s0 + w, outside);
    wave.bad |= outside;
    wave.load_k(ids, b.kvh);
    wave.load_v(wave.v_at(ids, b.kvh));
    ids = StepPages<T>(pt, max_pages, s0 + w + W);
    for (int s = s0 + w; s < s1; s += W) {
      float p[QT][Wave<HD, T, QT, false>::S];
      wave.scores(p);
      const bool more = s + W < s1;
      typename Wave<HD, T, QT, false>::ValuesAt next_v = {nullptr, 0};
      if (more) {
        ids = wave.usable(ids, own.len, s + W, outside);
        wave.bad |= outside;
        wave.load_k(ids, b.kvh);
        next_v = wave.v_at(ids, b.kvh);
        ids = StepPages<T>(pt, max_pages, s + 2 * W);
      }
      wave.template weigh<false>(p, own.len - kStep<T> * s);
      if (more) wave.load_v(next_v);
    }
    wave.end();
    if (__builtin_expect(wave.spoiled(), 0)) {  // once more with infinite and NaN values apart
      wave.begin();
#pragma nounroll
      for (int s = s0 + w; s < s1; s += W) {
        bool out;
        const StepPages<T> again = wave.usable(StepPages<T>(pt, max_pages, s), own.len, s, out);
        wave.bad |= out;
        wave.load_k(again, b.kvh);
        wave.load_v(wave.v_at(again, b.kvh));
        float p[QT][Wave<HD, T, QT, false>::S];
        wave.scores(p);
        wave.template weigh<true>(p, own.len - kStep<T> * s);
      }
      wave.end();
    }
  }
  Parts<HD> ps(own_lds, W, rows);
  ps.put(w, wave.run, b.n);
  __syncthreads();
  if (runs == 1) {
    const int n = shared_parts(own.skip, parts);
    for (int i = threadIdx.x; i < b.n * (HD / 4); i += blockDim.x)
      join_column<HD, T, W>(a, sp, env, b.head0 + i / (HD / 4), 4 * (i % (HD / 4)), n, 0, 0, &ps, i / (HD / 4));
    return;
  }
  const size_t to = (parts + run) * sp.columns + (size_t)env * a.n_heads + b.head0;
  for (int i = threadIdx.x; i < b.n * (HD / 4); i += blockDim.x) {
    const int h = i / (HD / 4), f = 4 * (i % (HD / 4));
    float mx = -INFINITY, l = 0.f;
#pragma unroll
    for (int u = 0; u < W; ++u) mx = fmaxf(mx, ps.ml[u * 2 * rows + h]);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < W; ++u) {
      const float mu = ps.ml[u * 2 * rows + h], c = mu == -INFINITY ? 1.f : worth(mu, mx);
      l = fmaf(ps.ml[(u * 2 + 1) * rows + h], c, l);
      const f32x4 o = *reinterpret_cast<const f32x4*>(ps.o + (size_t)(u * rows + h) * (HD + 4) + f);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(o[e], c, v[e]);
    }
    *reinterpret_cast<f32x4*>(sp.o + (to + h) * HD + f) = v;
    if (f == 0) sp.ml[to + h] = make_float2(mx, l);
  }
}

// One wave per head (HD 64: a quarter of it; 256: all).
template <int HD, CacheType T>
__global__ __launch_bounds__(64) void attn_parts_kernel(SharedArgs args, PartSpace sp, int parts, int runs) {
  const PagedAttnArgs& a = args.a;
  const int env = blockIdx.y, head = blockIdx.x;
  const Own own = own_of<T>(args, env);
  if (own.zeros || own.bad) return fill_rows<HD, T>(a, env, head, 1, own.zeros);
  const int m = own.steps == 0 ? 0 : (own.steps + run_of(own.steps, runs) - 1) / run_of(own.steps, runs);
  if (4 * threadIdx.x < HD) join_column<HD, T, 0>(a, sp, env, head, 4 * threadIdx.x, shared_parts(own.skip, parts), parts, m, nullptr, 0);
}

// ------------------------------------------------------------------ host
Plan plan(int n_env, int n_groups, int n_heads, int n_kv_heads, int head_dim, int max_pages) {
  const int group = n_heads / n_kv_heads;
  Plan p = {false, 2, 1, 1};
  if (n_groups == 0 || max_pages == 0 || n_env < 2 * n_groups) return p;
  p.share = true;
  const long long columns = (long long)n_env * group / n_groups;  // of a group and key head, in the mean
  p.waves = columns > 128 && head_dim < 256 ? 8 : columns > 64 ? 4 : 2;
  const long long items = ((long long)n_env * group / (32 * p.waves) + n_groups) * n_kv_heads;
  p.parts = (int)std::max(1ll, std::min({(512 + items - 1) / items, (max_pages + 7ll) / 8, 64ll}));
  if (items * p.parts * 64 * p.waves >= 1ll << 32) return {false, 2, 1, 1};  // more threads than a launch takes
  const int tiles = query_tiles(group, head_dim);
  const long long pieces = (long long)n_env * (tiles == 1 ? head_blocks<1>(group) : head_blocks<2>(group)) * n_kv_heads;
  p.own = (int)std::max(1ll, std::min({(256 + pieces - 1) / pieces, (max_pages + 31ll) / 32, 32ll}));
  return p;
}

template <int HD, CacheType T, int NW>
hipError_t launch_shared(const SharedArgs& s, const PartSpace& sp, const Plan& p, hipStream_t stream) {
  static LdsLimit limit;
  const auto kernel = attn_shared_kernel<HD, T, NW>;
  constexpr int kLds = 4 * tiles::kTileBytes<HD>;
  const hipError_t e = limit.allow((const void*)kernel, kLds);
  if (e != hipSuccess) return e;
  const int group = s.a.n_heads / s.a.n_kv_heads;
  const long long items = (long long)s.a.n_env * group / (32 * NW) + s.n_groups;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(items * s.a.n_kv_heads * p.parts)), dim3(64 * NW), kLds, stream, s, sp, p.parts);
  return hipGetLastError();
}
template <int HD, CacheType T, int QT>
hipError_t launch_own(const SharedArgs& s, const PartSpace& sp, const Plan& p, hipStream_t stream) {
  constexpr int W = 4;
  static LdsLimit limit;
  const auto kernel = attn_own_kernel<HD, T, QT, W>;
  hipError_t e = limit.allow((const void*)kernel, Parts<HD>::bytes(W, 16 * QT));
  if (e != hipSuccess) return e;
  const int group = s.a.n_heads / s.a.n_kv_heads, blocks = head_blocks<QT>(group) * s.a.n_kv_heads, rows = query_rows(group, QT);
  hipLaunchKernelGGL(kernel, dim3(blocks * p.own, s.a.n_env), dim3(64 * W), Parts<HD>::bytes(W, rows), stream, s, sp, p.parts, p.own, rows);
  e = hipGetLastError();
  if (e != hipSuccess || p.own == 1) return e;
  hipLaunchKernelGGL((attn_parts_kernel<HD, T>), dim3(s.a.n_heads, s.a.n_env), dim3(64), 0, stream, s, sp, p.parts, p.own);
  return hipGetLastError();
}
int all_parts(const Plan& p) { return p.parts + (p.own > 1 ? p.own : 0); }

template <int HD, CacheType T>
hipError_t launch_both(const SharedArgs& s, const Plan& p, hipStream_t stream) {
  const PartSpace sp = part_space(s.a.ws, s.a, all_parts(p));
  hipError_t e = hipErrorInvalidValue;
  if (p.waves == 2) e = launch_shared<HD, T, 2>(s, sp, p, stream);
  if (p.waves == 4) e = launch_shared<HD, T, 4>(s, sp, p, stream);
  if constexpr (HD < 256)
    if (p.waves == 8) e = launch_shared<HD, T, 8>(s, sp, p, stream);
  if (e != hipSuccess) return e;
  if constexpr (HD < 256)
    if (query_tiles(s.a.n_heads / s.a.n_kv_heads, HD) == 2) return launch_own<HD, T, 2>(s, sp, p, stream);
  return launch_own<HD, T, 1>(s, sp, p, stream);
}
template <CacheType T>
hipError_t launch_dims(const SharedArgs& s, const Plan& p, hipStream_t stream) {
  if (s.a.head_dim == 64) return launch_both<64, T>(s, p, stream);
  if (s.a.head_dim == 128) return launch_both<128, T>(s, p, stream);
  if (s.a.head_dim == 256) return launch_both<256, T>(s, p, stream);
  return hipErrorInvalidValue;
}

}  // namespace

size_t shared_attn_bytes(int n_env, int n_groups, int n_heads, int n_kv_heads, int head_dim, int max_pages) {
  const Plan p = plan(n_env, n_groups, n_heads, n_kv_heads, head_dim, max_pages);
  const size_t plain = paged_attn_bytes(n_env, n_heads, n_kv_heads, head_dim, max_pages);  // also where there are no pages
  if (!p.share) return plain;
  return std::max(plain, ((size_t)all_parts(p) * n_env * n_heads * (head_dim + 2) * sizeof(float) + 255) / 256 * 256);
}

hipError_t launch_shared_attn(const SharedArgs& s, hipStream_t stream) {
  const Plan p = plan(s.a.n_env, s.n_groups, s.a.n_heads, s.a.n_kv_heads, s.a.head_dim, s.a.max_pages);
  if (!p.share || s.a.n_pages == 0) return launch_paged_attn(s.a, stream);
  return s.a.type == kBf16 ? launch_dims<kBf16>(s, p, stream) : launch_dims<kF16>(s, p, stream);
}

}  // namespace vla
