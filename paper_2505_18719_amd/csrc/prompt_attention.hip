// Causal attention over whole prompts (vla_prompt_attention).
//
// Bound: the matrix units, 4 head_dim flops a query-key pair, and beside them the vector units, which take an exponential, a
// product, a maximum, a sum and a rounding of each pair's score (8190 rows, 28 on 4 heads of 128: 0.9 to 1.0 PFLOP/s, where a large
// product reaches 1.5; matrix units and vector units busy 57 % of the time each).  Short sequences are bound by a workgroup's way
// in and out: of 117 us for 64 of 272 to 304 rows, 32 on 8 heads, 39 are queries and first tiles, 30 the outputs.  A wave holds 32
// queries of one head as MFMA columns, its workgroup's waves 32 queries each further on; tiles of 64 keys and values pass through
// LDS, the next on its way while one is used.  S^T = K Q^T leaves a query's scores in two lanes, so that the running maximum costs
// one exchange, and the weights are the B operand of O^T += V^T P^T as they stand.  The tiles are taken from the last one back: the
// first that a wave takes is the one part of which is masked, all others are whole.
#include <hip/hip_runtime.h>

#include "lds_limit.h"
#include "prompt.h"
#include "prompt_dev.h"

namespace vla {
namespace {

using namespace tiles;

// Waves that a SIMD is to hold: 3 have 168 registers each, 2 have 256, 1 has 512.
template <int HD>
constexpr int kWavesPerSimd = HD == 256 ? 1 : HD == 64 ? 3 : 2;

template <int HD, CacheType T, int NW>
__global__ __launch_bounds__(64 * NW, kWavesPerSimd<HD>) void prompt_attn_kernel(PromptArgs a) {
  extern __shared__ __align__(16) char lds[];
  const int kvh = blockIdx.x % a.n_kv_heads, item = blockIdx.x / a.n_kv_heads, group = a.n_heads / a.n_kv_heads;
  SeqItem st;
  if (!find_item<NW>(a.row_start, a.n_seq, a.rows, group, item, st)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const SeqRows k = {a.k.p + st.row0 * a.k.ld + kvh * HD, a.k.ld}, v = {a.v.p + st.row0 * a.v.ld + kvh * HD, a.v.ld};
  const int line = NW * st.nth + wave;  // this wave's place in the sequence's line
  const int q0 = 32 * (line / group), head = kvh * group + line % group;
  const int qi = q0 + (lane & 31);
  const bool mine = qi < st.len;
  const int64_t row = st.row0 + (int64_t)min(qi, st.len - 1);
  Queries<HD, T> w;
  w.load(a.q.p + row * a.q.ld + head * HD, a.scale);
  const TileLane<HD> at;
  const int last = (min(32 * ((NW * (st.nth + 1) - 1) / group) + 32, st.len) - 1) / kTile;  // tile of the workgroup's last query
  const int halves = q0 % kTile / 32 + 1;  // of its own tile, those with keys that some query sees
  const int own = q0 < st.len ? q0 / kTile : -1;                                          // of this wave's queries
  // Buffers by the parity of the tile, at places that the loop over pairs of tiles knows beforehand.
  auto keys = [&](int parity) { return lds + parity * kTileBytes<HD>; };
  auto values = [&](int parity) { return lds + (2 + parity) * kTileBytes<HD>; };
  auto copy_keys = [&](int j, int parity) { if (j >= 0) copy_tile<HD, NW>(keys(parity), k, kTile * j, st.len, wave); };
  auto copy_values = [&](int j, int parity) { if (j >= 0) copy_tile<HD, NW>(values(parity), v, kTile * j, st.len, wave); };
  // Every wave comes to last + 1 barriers behind the first two: one with the end of each tile but the first of the sequence, and one
  // before the outputs; those without queries have one with the end of each tile.
  auto arrived = [&] {
    WAIT_VMCNT(0);
    __syncthreads();
  };
  // Scores are a tile ahead of the weights, so that the matrix units have the next ones' products while the vector units take the
  // weights: at tile j its scores are there, as are keys j - 1 and values j in LDS, and keys j - 2 and values j - 1 are on their way.
  typename Queries<HD, T>::Scores s, next;
  copy_keys(last, last & 1);
  copy_values(last, last & 1);
  copy_keys(last - 1, ~last & 1);
  arrived();
  if (own == last) w.scores(at, keys(last & 1), s, halves);
  __syncthreads();
  int j = last;
  for (; j > own; --j) {  // tiles of the workgroup's later queries only
    copy_keys(j - 2, j & 1);
    copy_values(j - 1, ~j & 1);
    if (j - 1 == own) w.scores(at, keys(~j & 1), s, halves);
    arrived();
  }
  if (own < 0) return;
  copy_keys(j - 2, j & 1);
  copy_values(j - 1, ~j & 1);
  w.template mask<false>(s, qi - kTile * j);
  w.follow(s);
#pragma unroll
  for (int t = 0; t < kTile / 32; ++t) next[t] = s[t];
  w.weigh(next);
  w.add(at, values(j & 1), next, halves);
  if (__builtin_expect(any_nan(w.o), 0)) {  // a masked value may have spoiled the sums: once more without it
    const float l = w.l;
    w.weigh(s);
    w.l = l;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) w.o[i] = zeros16();
#pragma unroll
    for (int t = 0; t < kTile / 32; ++t) add_apart<HD, T>(w.o, s[t], values(j & 1), 32 * t, [&](int key) { return kTile * j + key <= qi; });
  }
  if (j > 0) {
    w.scores(at, keys(~j & 1), s);
    arrived();
  }
  auto tile = [&](int j, int parity, typename Queries<HD, T>::Scores& s, typename Queries<HD, T>::Scores& next) {
    copy_keys(j - 2, parity);
    copy_values(j - 1, 1 - parity);
    w.follow(s);
    w.scores(at, keys(1 - parity), next);
    w.weigh(s);
    w.add(at, values(parity), s);
    arrived();
  };
  if (--j > 0 && j % 2 == 1) {
    tile(j, 1, s, next);
#pragma unroll
    for (int t = 0; t < kTile / 32; ++t) s[t] = next[t];
    --j;
  }
  for (; j > 0; j -= 2) {
    tile(j, 0, s, next);
    tile(j - 1, 1, next, s);
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
  __syncthreads();  // the tiles have been used
  constexpr int kShare = 4 * kTileBytes<HD> / NW;
  store_rows<HD, T, kShare>(lds + wave * kShare, a.o.p + (st.row0 + (int64_t)q0) * a.o.ld + head * HD, a.o.ld, min(st.len - q0, 32), w.o, r);
  if (a.lse && mine && lane < 32) a.lse[row * a.n_heads + head] = ((w.m * w.scale - kHeldExp<T>) + __builtin_amdgcn_logf(l)) * kLn2;
}

// Four waves share a tile's way through LDS, two workgroups a CU (64 x 272 to 304 rows, 32 heads of 128: 117 us, with two waves 179,
// with eight 133; up to 8190 rows, 28 heads: 526, 775 and 513; one of 278: 10.6, 10.9 and 12.3; of 1400, 32 heads of 256: 70, with two
// waves 115, which are faster only there and up to 100 rows, 8.2 for 9.1).
constexpr int kWaves = 4;

template <int HD, CacheType T>
hipError_t launch(const PromptArgs& a, hipStream_t s) {
  static LdsLimit limit;
  const auto kernel = prompt_attn_kernel<HD, T, kWaves>;
  constexpr int kLds = 4 * kTileBytes<HD>;
  const hipError_t e = limit.allow((const void*)kernel, kLds);
  if (e != hipSuccess) return e;
  const long long groups = seq_items<kWaves>(a.rows, a.n_seq, a.n_heads / a.n_kv_heads) * a.n_kv_heads;
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * kWaves), kLds, s, a);
  return hipGetLastError();
}

template <CacheType T>
hipError_t launch_type(const PromptArgs& a, hipStream_t s) {
  if (a.head_dim == 64) return launch<64, T>(a, s);
  if (a.head_dim == 128) return launch<128, T>(a, s);
  if (a.head_dim == 256) return launch<256, T>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace

bool prompt_fits(int rows, int n_seq, int n_heads) {  // threads of the most workgroups of any of the kernels, below 2^32
  return n_seq < 1 << 26 && (tiles::seq_items<2>(rows, n_seq, 1) + n_seq) * n_heads * 128 < 1ll << 32;
}

hipError_t launch_prompt_attn(const PromptArgs& a, hipStream_t s) {
  return a.type == kBf16 ? launch_type<kBf16>(a, s) : launch_type<kF16>(a, s);
}

}  // namespace vla
