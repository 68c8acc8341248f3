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
  auto tile = [&](int j, int which) { return lds + (2 * (j & 1) + which) * kTileBytes<HD>; };
  copy_tile<HD, NW>(tile(last, 0), k, kTile * last, st.len, wave);
  copy_tile<HD, NW>(tile(last, 1), v, kTile * last, st.len, wave);
  WAIT_VMCNT(0);
  __syncthreads();
  for (int j = last; j >= 0; --j) {
    if (j > 0) {
      copy_tile<HD, NW>(tile(j - 1, 0), k, kTile * (j - 1), st.len, wave);
      copy_tile<HD, NW>(tile(j - 1, 1), v, kTile * (j - 1), st.len, wave);
    }
    if (j <= own) {
      f32x16 s[2];
      w.scores(at, tile(j, 0), s);
      if (j == own) w.template mask<false>(s, qi - kTile * j);
      w.weigh(s);
      w.add(at, tile(j, 1), s);
      if (j == own && __builtin_expect(any_nan(w.o), 0)) {  // a masked value may have spoiled the sums: once more without it
        const float m = w.m, l = w.l;
        w.scores(at, tile(j, 0), s);
        w.template mask<false>(s, qi - kTile * j);
        w.weigh(s);
        w.m = m;
        w.l = l;
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) w.o[i] = zeros16();
#pragma unroll
        for (int t = 0; t < 2; ++t) add_apart<HD, T>(w.o, s[t], tile(j, 1), 32 * t, [&](int key) { return kTile * j + key <= qi; });
      }
    }
    WAIT_VMCNT(0);
    __syncthreads();
  }
  const float l = half_sum(w.l), r = l == 0.f ? 0.f : 1.f / l;
  if (own < 0) return;
  if (l == 0.f) {  // no score above -inf: zeros whatever the values
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) w.o[i] = zeros16();
  }
  store_row<HD, T>(a.o.p + row * a.o.ld + head * HD, w.o, r, mine);
  if (a.lse && mine && lane < 32) a.lse[row * a.n_heads + head] = ((w.m * w.scale - kWeightExp<T>) + __builtin_amdgcn_logf(l)) * kLn2;
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
  if constexpr (HD < 256)
    if (groups(8) >= 512) return launch<HD, T, 8>(a, s);
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
