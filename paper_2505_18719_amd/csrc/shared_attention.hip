// Attention of one new token per environment where groups of environments share their first pages (vla_shared_attention).
//
// Bound: HBM and the matrix units: the shared keys and values once for a group, 4 head_dim flops a query and key.  One launch of two
// kinds of workgroups, and a join:
//   shared  takes 32 columns a wave, a column being one query head of one environment of a group, over a run of the group's shared
//           pages, which pass through LDS in tiles of four as in attention over whole prompts
//   own     takes an environment's remaining pages, or a run of them, as attention without sharing does
// Each leaves its columns' maxima, sums of weights and sums of weighted values, and own ones say which parts there are none of, so
// that the join has no lengths or groups to look up (its time for 128 environments of 8 groups: 4.8 us, was 6.6).  What bounds it
// in earnest is a wave's way through a tile, 1.7 us with its SIMD to itself or shared with one (50 environments, 16384 shared
// tokens, 28 on 4 heads of 128: 36 us, of which ten tiles a workgroup 17, the start 8, the parts' way through memory 5 and their
// sum 7; unshared 244): scores, maximum, weights and their product with the values follow one another.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged_dev.h"
#include "prompt_dev.h"

namespace vla {
namespace {

struct Plan {
  bool share;      // else vla_paged_attention's kernels
  int parts, own;  // runs of the shared pages, and of an environment's own
  int all() const { return parts + own; }
};

// The parts of all columns: sums of weighted values [part][environment][head][HD], maxima (to base 2) and sums of weights.  In place of a
// sum of weights, kNone: there is no such part.  kZeros, in the first part of the own keys: an environment without tokens.
constexpr float kNone = -1.f, kZeros = -2.f;
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

// The last group g with key(g) <= x: its environments e0 .. e1 - 1 and shared pages, as far as they are usable.  Each lane looks at one
// group of 64 at a time, at its pages together with its start.
struct Group {
  int g, e0, e1, pages;
};
template <class F>
__device__ __forceinline__ bool find_group(const SharedArgs& s, long long x, F key, Group& out) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = s.n_groups;
  for (;;) {
    const int step = (n + kWave - 1) / kWave, at = min(lo + lane * step, s.n_groups), start = s.group_start[at];
    const int pages = s.shared_pages[min(at, s.n_groups - 1)];
    const int found = __popcll(__ballot(lane * step < n && key(start, at) <= x));
    if (found == 0) return false;
    lo += (found - 1) * step;
    n = min(step, n - (found - 1) * step);
    if (step > 1) continue;
    out.g = __builtin_amdgcn_readfirstlane(lo);
    out.e0 = __builtin_amdgcn_readlane(start, found - 1);
    out.e1 = __builtin_amdgcn_readfirstlane(found < kWave ? __builtin_amdgcn_readlane(start, found) : s.group_start[min(lo + 1, s.n_groups)]);
    out.pages = min(max(__builtin_amdgcn_readlane(pages, found - 1), 0), s.a.max_pages);
    return out.e0 >= 0 && out.e1 > out.e0 && out.e1 <= s.a.n_env;
  }
}
// Items of the groups, C columns each: group g has items first_of(group_start[g], g) and on, as many as it needs or more.
template <int C>
__device__ __forceinline__ long long first_of(const SharedArgs& s, int start, int g, int group) {
  return (long long)min(max(start, 0), s.a.n_env) * group / C + g;
}
// Pages that environment env shares with its group.
__device__ __forceinline__ int shared_of(const SharedArgs& s, int env) {
  Group g;
  const bool found = find_group(s, env, [](int start, int) { return start; }, g);
  return found && g.e1 > env ? g.pages : 0;
}

__host__ __device__ __forceinline__ int run_of(int n, int parts) { return (n + parts - 1) / parts; }

// ------------------------------------------------------------------ shared pages
template <int HD, CacheType T, int NW>
__device__ __forceinline__ void shared_part(const SharedArgs& args, const PartSpace& sp, int parts, int block, char* lds) {
  using namespace tiles;
  constexpr int C = 32 * NW, CH = HD / 8, RPK = 64 / CH, PK = kPage / RPK;  // chunks of a row, rows of a copy, copies of a page
  const PagedAttnArgs& a = args.a;
  const int kvh = block % a.n_kv_heads, rest = block / a.n_kv_heads, part = rest % parts, item = rest / parts;
  const int group = a.n_heads / a.n_kv_heads;
  Group of;
  if (!find_group(args, item, [&](int start, int g) { return first_of<C>(args, start, g, group); }, of)) return;
  const int e0 = of.e0, n_col = (of.e1 - e0) * group, c0 = (int)(item - first_of<C>(args, e0, of.g, group)) * C, pages = of.pages;
  if (c0 >= n_col || pages == 0) return;
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

// Runs of the shared pages that there are parts of.
__device__ __forceinline__ int shared_parts(int skip, int parts) {
  const int n = (skip + 3) / 4;
  return n == 0 ? 0 : (n + run_of(n, parts) - 1) / run_of(n, parts);
}
template <int HD, CacheType T, int QT, int W>
__device__ __forceinline__ void own_part(const SharedArgs& args, const PartSpace& sp, int parts, int runs, int rows, int block, float* lds) {
  const PagedAttnArgs& a = args.a;
  const int blocks = head_blocks<QT>(a.n_heads / a.n_kv_heads) * a.n_kv_heads, run = block % runs, env = block / runs / blocks;
  const HeadBlock b = head_block<QT>(a, block / runs % blocks);
  const Own own = own_of<T>(args, env);
  const int per = run_of(own.steps, runs), s0 = run * per, s1 = min(s0 + per, own.steps);
  const size_t to = (parts + run) * sp.columns + (size_t)env * a.n_heads + b.head0;
  if (run == 0)  // the runs of shared pages that there are none of
    for (int i = threadIdx.x, n = shared_parts(own.skip, parts); i < (parts - n) * b.n; i += blockDim.x)
      sp.ml[(n + i / b.n) * sp.columns + (size_t)env * a.n_heads + b.head0 + i % b.n] = make_float2(-INFINITY, kNone);
  if (s0 >= s1) {
    const float l = run > 0 ? kNone : own.bad ? __builtin_nanf("") : own.zeros ? kZeros : kNone;
    if ((int)threadIdx.x < b.n) sp.ml[to + threadIdx.x] = make_float2(-INFINITY, l);
    return;
  }
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
  Parts<HD> ps(lds, W, rows);
  ps.put(w, wave.run, b.n);
  __syncthreads();
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

template <int HD, CacheType T, int QT, int NW>
__global__ __launch_bounds__(64 * NW, HD == 256 || (HD == 128 && QT == 2) ? 1 : 2) void attn_parts_kernel(SharedArgs args, PartSpace sp, int shared_blocks,
                                                                                                         int parts, int runs, int rows) {
  extern __shared__ __align__(16) char lds[];
  if ((int)blockIdx.x < shared_blocks) shared_part<HD, T, NW>(args, sp, parts, blockIdx.x, lds);
  else own_part<HD, T, QT, NW>(args, sp, parts, runs, rows, blockIdx.x - shared_blocks, reinterpret_cast<float*>(lds));
}

// One workgroup per head of an environment: each thread first takes a part's maximum and sum, then every HD / 4 threads add a share
// of the parts, four features each.
constexpr int kMostParts = 128, kSumThreads = 256;
template <int HD, CacheType T>
__global__ __launch_bounds__(kSumThreads) void attn_sum_kernel(PagedAttnArgs a, PartSpace sp, int parts, int own) {
  constexpr int CH = HD / 4, PG = kSumThreads / CH, NW = kSumThreads / kWave;
  __shared__ float weight[kMostParts], top[NW], total[NW];
  __shared__ __align__(16) f32x4 sums[PG][CH];
  const int env = blockIdx.y, head = blockIdx.x, tid = threadIdx.x;
  const size_t at = (size_t)env * a.n_heads + head;
  const float2 ml = tid < parts + own ? sp.ml[tid * sp.columns + at] : make_float2(-INFINITY, kNone);
  const bool some = !(ml.y < 0.f);  // NaN is some
  float mx = wave_max(some ? ml.x : -INFINITY);
  if ((tid & 63) == 0) top[tid >> 6] = mx;
  const bool zeros = __syncthreads_or(tid == parts && ml.y == kZeros);
#pragma unroll
  for (int i = 0; i < NW; ++i) mx = fmaxf(mx, top[i]);
  const float c = !some ? kNone : ml.x == -INFINITY ? 1.f : worth(ml.x, mx);  // a part all of whose scores are -inf adds zeros
  if (tid < kMostParts) weight[tid] = c;
  const float sum = wave_sum(some ? ml.y * c : 0.f);
  if ((tid & 63) == 0) total[tid >> 6] = sum;
  __syncthreads();
  const int f = tid % CH, pg = tid / CH;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = pg; i < parts + own; i += PG) {
    const float w = weight[i];
    if (w < 0.f) continue;
    const f32x4 o = *reinterpret_cast<const f32x4*>(sp.o + (i * sp.columns + at) * HD + 4 * f);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(o[e], w, v[e]);
  }
  sums[pg][f] = v;
  __syncthreads();
  if (pg != 0) return;
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) l += total[i];
#pragma unroll
  for (int i = 1; i < PG; ++i) v += sums[i][f];
  if (zeros) v = f32x4{0.f, 0.f, 0.f, 0.f};
  store4<T>(a.o + env * a.ld_o + (size_t)head * HD + 4 * f, v, zeros ? 1.f : reciprocal(l));
  if (a.lse && f == 0) a.lse[at] = zeros ? -INFINITY : log_sum<T>(mx, l);
}

// ------------------------------------------------------------------ host
constexpr int kSharedWaves = 4;
long long shared_items(int n_env, int n_groups, int group) { return (long long)n_env * group / (32 * kSharedWaves) + n_groups; }

// Workgroups of both kinds are to run at once, two to a CU: what the environments' own pages leave of 512 goes to the shared ones.
Plan plan(int n_env, int n_groups, int n_heads, int n_kv_heads, int head_dim, int max_pages) {
  const int group = n_heads / n_kv_heads;
  const Plan none = {false, 1, 1};
  if (n_groups == 0 || max_pages == 0 || n_env < 2 * n_groups) return none;
  const int tiles = query_tiles(group, head_dim);
  const long long pieces = (long long)n_env * (tiles == 1 ? head_blocks<1>(group) : head_blocks<2>(group)) * n_kv_heads;
  const long long own = std::max(1ll, std::min({256 / pieces, (max_pages + 31ll) / 32, 32ll}));
  const long long items = shared_items(n_env, n_groups, group) * n_kv_heads, left = 512 - std::min(pieces * own, 256ll);
  const long long parts = std::max(1ll, std::min({left / items, (max_pages + 7ll) / 8, 64ll}));
  // more threads than a launch takes: not shared
  return (items * parts + pieces * own) * 64 * kSharedWaves < 1ll << 32 ? Plan{true, (int)parts, (int)own} : none;
}

template <int HD, CacheType T, int QT>
hipError_t launch_parts(const SharedArgs& s, const PartSpace& sp, const Plan& p, hipStream_t stream) {
  constexpr int NW = kSharedWaves;
  static LdsLimit limit;
  const auto kernel = attn_parts_kernel<HD, T, QT, NW>;
  const int group = s.a.n_heads / s.a.n_kv_heads, rows = query_rows(group, QT);
  const size_t shared = 4 * tiles::kTileBytes<HD>, most = std::max(shared, Parts<HD>::bytes(NW, 16 * QT));
  const hipError_t e = limit.allow((const void*)kernel, most);
  if (e != hipSuccess) return e;
  const long long blocks = shared_items(s.a.n_env, s.n_groups, group) * s.a.n_kv_heads * p.parts;
  const long long pieces = (long long)s.a.n_env * head_blocks<QT>(group) * s.a.n_kv_heads * p.own;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks + pieces)), dim3(64 * NW), std::max(shared, Parts<HD>::bytes(NW, rows)), stream, s, sp,
                     (int)blocks, p.parts, p.own, rows);
  return hipGetLastError();
}

template <int HD, CacheType T, int QT>
hipError_t launch_both(const SharedArgs& s, const Plan& p, hipStream_t stream) {
  const PartSpace sp = part_space(s.a.ws, s.a, p.all());
  const hipError_t e = launch_parts<HD, T, QT>(s, sp, p, stream);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attn_sum_kernel<HD, T>), dim3(s.a.n_heads, s.a.n_env), dim3(kSumThreads), 0, stream, s.a, sp, p.parts, p.own);
  return hipGetLastError();
}
template <int HD, CacheType T>
hipError_t launch_group(const SharedArgs& s, const Plan& p, hipStream_t stream) {
  if constexpr (HD < 256)
    if (query_tiles(s.a.n_heads / s.a.n_kv_heads, HD) == 2) return launch_both<HD, T, 2>(s, p, stream);
  return launch_both<HD, T, 1>(s, p, stream);
}
template <CacheType T>
hipError_t launch_dims(const SharedArgs& s, const Plan& p, hipStream_t stream) {
  if (s.a.head_dim == 64) return launch_group<64, T>(s, p, stream);
  if (s.a.head_dim == 128) return launch_group<128, T>(s, p, stream);
  if (s.a.head_dim == 256) return launch_group<256, T>(s, p, stream);
  return hipErrorInvalidValue;
}

}  // namespace

size_t shared_attn_bytes(int n_env, int n_groups, int n_heads, int n_kv_heads, int head_dim, int max_pages) {
  const Plan p = plan(n_env, n_groups, n_heads, n_kv_heads, head_dim, max_pages);
  const size_t plain = paged_attn_bytes(n_env, n_heads, n_kv_heads, head_dim, max_pages);  // also where there are no pages
  if (!p.share) return plain;
  return std::max(plain, ((size_t)p.all() * n_env * n_heads * (head_dim + 2) * sizeof(float) + 255) / 256 * 256);
}

hipError_t launch_shared_attn(const SharedArgs& s, hipStream_t stream) {
  const Plan p = plan(s.a.n_env, s.n_groups, s.a.n_heads, s.a.n_kv_heads, s.a.head_dim, s.a.max_pages);
  if (!p.share || s.a.n_pages == 0) return launch_paged_attn(s.a, stream);
  return s.a.type == kBf16 ? launch_dims<kBf16>(s, p, stream) : launch_dims<kF16>(s, p, stream);
}

}  // namespace vla
