// Causal attention over whole prompts (vla_prompt_attention).
//
// Bound: the matrix units, 4 head_dim flops a query-key pair, and beside them the vector units, which take an exponential, a
// product, a maximum, a sum and a rounding of each pair's score.  A wave holds 32 queries of one head as MFMA columns, its
// workgroup's waves 32 queries each further on; tiles of 64 keys and values pass through LDS, the next on its way while one is
// used.  S^T = K Q^T leaves a query's scores in two lanes, so that the running maximum costs one exchange, and the weights are the B
// operand of O^T += V^T P^T as they stand.  The tiles are taken from the last one back: the first that a wave takes is the one part
// of which is masked, all others are whole.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lds_limit.h"
#include "prompt.h"
#include "prompt_dev.h"

namespace vla {
namespace {

using namespace tiles;

template <int HD, CacheType T, int NW>
__global__ __launch_bounds__(64 * NW, HD == 256 ? 1 : 2) void prompt_attn_kernel(PromptArgs a) {
  extern __shared__ __align__(16) char lds[];
  constexpr int M = 32 * NW;
  const int head = blockIdx.x % a.n_heads, item = blockIdx.x / a.n_heads;
  SeqTile st;
  if (!find_tile<M>(a.row_start, a.n_seq, a.rows, item, st)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = head / (a.n_heads / a.n_kv_heads);
  const SeqRows k = {a.k.p + st.row0 * a.k.ld + kvh * HD, a.k.ld}, v = {a.v.p + st.row0 * a.v.ld + kvh * HD, a.v.ld};
  const int q0 = M * st.tile + 32 * wave;  // this wave's first query
  const int qi = q0 + (lane & 31);
  const bool mine = qi < st.len;
  const int64_t row = st.row0 + (int64_t)min(qi, st.len - 1);
  Queries<HD, T> w;
  w.load(a.q.p + row * a.q.ld + head * HD, a.scale);
  const TileLane<HD> at;
  const int last = (min(M * (st.tile + 1), st.len) - 1) / kTile;  // tile of the workgroup's last query
  const int own = q0 < st.len ? q0 / kTile : -1;                  // of this wave's queries
  auto keys = [&](int j) { return lds + (j & 1) * kTileBytes<HD>; };
  auto values = [&](int j) { return lds + (2 + (j & 1)) * kTileBytes<HD>; };
  auto copy_keys = [&](int j) { if (j >= 0) copy_tile<HD, NW>(keys(j), k, kTile * j, st.len, wave); };
  auto copy_values = [&](int j) { if (j >= 0) copy_tile<HD, NW>(values(j), v, kTile * j, st.len, wave); };
  auto arrived = [&] {
    WAIT_VMCNT(0);
    __syncthreads();
  };
  // Scores are a tile ahead of the weights, so that the matrix units have the next ones' products while the vector units take the
  // weights: at tile j its scores are there, as are keys j - 1 and values j in LDS, and keys j - 2 and values j - 1 are on their way.
  f32x16 s[2];
  copy_keys(last);
  copy_values(last);
  copy_keys(last - 1);
  arrived();
  if (own == last) w.scores(at, keys(last), s);
  __syncthreads();
  int j = last;
  for (; j > own; --j) {  // tiles of the workgroup's later queries only
    copy_keys(j - 2);
    copy_values(j - 1);
    if (j - 1 == own) w.scores(at, keys(own), s);
    arrived();
  }
  if (own < 0) return;
  copy_keys(j - 2);
  copy_values(j - 1);
  w.template mask<false>(s, qi - kTile * j);
  w.follow(s);
  {
    f32x16 p[2] = {s[0], s[1]};
    w.weigh(p);
    w.add(at, values(j), p);
  }
  if (__builtin_expect(any_nan(w.o), 0)) {  // a masked value may have spoiled the sums: once more without it
    const float l = w.l;
    w.weigh(s);
    w.l = l;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) w.o[i] = zeros16();
#pragma unroll
    for (int t = 0; t < 2; ++t) add_apart<HD, T>(w.o, s[t], values(j), 32 * t, [&](int key) { return kTile * j + key <= qi; });
  }
  if (j > 0) w.scores(at, keys(j - 1), s);
  arrived();
  for (--j; j > 0; --j) {
    copy_keys(j - 2);
    copy_values(j - 1);
    w.follow(s);
    f32x16 next[2];
    w.scores(at, keys(j - 1), next);
    w.weigh(s);
    w.add(at, values(j), s);
    s[0] = next[0];
    s[1] = next[1];
    arrived();
  }
  if (j == 0) {
    w.follow(s);
    w.weigh(s);
    w.add(at, values(0), s);
  }
  const float l = half_sum(w.l), r = l == 0.f ? 0.f : 1.f / l;
  if (l == 0.f) {  // no score above -inf: zeros whatever the values
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) w.o[i] = zeros16();
  }
  store_row<HD, T>(a.o.p + row * a.o.ld + head * HD, w.o, r, mine);
  if (a.lse && mine && lane < 32) a.lse[row * a.n_heads + head] = ((w.m * w.scale - kHeldExp<T>) + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int HD, CacheType T, int NW>
hipError_t launch(const PromptArgs& a, hipStream_t s) {
  static LdsLimit limit;
  const auto kernel = prompt_attn_kernel<HD, T, NW>;
  const hipError_t e = limit.allow((const void*)kernel, 4 * kTileBytes<HD>);
  if (e != hipSuccess) return e;
  const long long groups = seq_items(a.rows, a.n_seq, 32 * NW) * a.n_heads;
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * NW), 4 * kTileBytes<HD>, s, a);
  return hipGetLastError();
}

template <int HD, CacheType T>
hipError_t launch_rows(const PromptArgs& a, hipStream_t s) {
  auto groups = [&](int waves) { return seq_items(a.rows, a.n_seq, 32 * waves) * a.n_heads; };
  if (groups(4) >= 512) return launch<HD, T, 4>(a, s);
  return launch<HD, T, 2>(a, s);
}

template <CacheType T>
hipError_t launch_type(const PromptArgs& a, hipStream_t s) {
  if (a.head_dim == 64) return launch_rows<64, T>(a, s);
  if (a.head_dim == 128) return launch_rows<128, T>(a, s);
  if (a.head_dim == 256) return launch_rows<256, T>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace

bool prompt_fits(int rows, int n_seq, int n_heads) {  // the smallest workgroups have 64 rows, none more than 512 threads
  return n_seq < 1 << 26 && tiles::seq_items(rows, n_seq, 64) * n_heads * 512 < 1ll << 32;
}

hipError_t launch_prompt_attn(const PromptArgs& a, hipStream_t s) {
  return a.type == kBf16 ? launch_type<kBf16>(a, s) : launch_type<kF16>(a, s);
}

}  // namespace vla
