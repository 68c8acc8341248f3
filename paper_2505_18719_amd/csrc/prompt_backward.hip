// Gradient of causal attention over whole prompts (vla_prompt_attention_backward), in two passes that share nothing but D and the
// log-sum-exps, so that no sum depends on the order of workgroups:
//   queries: a wave holds 32 queries as MFMA columns, tiles of keys and values pass through LDS: S^T = K Q^T, dP^T = V dO^T - D,
//            dQ^T += K^T dS^T
//   keys:    a wave holds 32 keys as columns and goes over the queries behind them, of every head that reads the keys:
//            S = Q K^T, dP = dO V^T - D, dV^T += dO^T P, dK^T += Q^T dS
// Bound: the matrix units.  The gradient is 10 head_dim flops a query-key pair; scores and dP are computed in both passes and dS
// enters dQ as a pair, which makes 16 (3001 to 5003 rows, 16 on 4 heads of 128: 0.83 PFLOP/s of those, 0.52 of the 10).  Each tile
// lies in LDS once, read by rows for one product and transposed for the other.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lds_limit.h"
#include "prompt.h"
#include "prompt_dev.h"

namespace vla {
namespace {

using namespace tiles;

// A query's log-sum-exp to base 2; kNoWeight where it has no score above -inf.  Its weights are 0, and it is left out of all sums,
// whatever its elements are.
constexpr float kNoWeight = INFINITY;
__device__ __forceinline__ float lse_base2(float lse) { return lse == -INFINITY ? kNoWeight : lse * kLog2e; }

// Products with a column's weights, of any size, in the type's range.  In bf16 as they are.  Half precision has 5 bits of exponent:
// each column's weights are held times a power of two that keeps the largest so far below 2^15 (and at first within a factor of four
// of it), and what is summed follows when that changes.
template <int HD, CacheType T>
struct Column {
  f32x16 sum[HD / 32];
  float unit;
  __device__ __forceinline__ void begin() {
    unit = T == kBf16 ? 1.f : 0x1p120f;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) sum[i] = zeros16();
  }
  __device__ __forceinline__ void fit(f32x16& w) {
    if constexpr (T == kF16) {
      float mx = fabsf(w[0]);
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, fabsf(w[r]));
      mx = half_max(mx);
      const bool grown = mx * unit > 0x1p15f && mx < INFINITY;
      if (__any(grown)) {
        const float u = grown ? ldexpf(1.f, min(max(14 - __builtin_amdgcn_frexp_expf(mx), -120), 120)) : unit;
        const float c = u / unit;
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) sum[i] *= c;
        unit = u;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) w[r] *= unit;
    }
  }
  // sum += x^T w over the 32 rows of a tile from 32 t on, w rounded to the type: a relative 2^-9 (2^-12), of either sign, of each
  // term at most, beside the output's own rounding.  PAIR: w as hi + lo of the type, twice the bits.
  template <bool PAIR = false>
  __device__ __forceinline__ void add(const TileLane<HD>& at, const char* tile, int t, const f32x16& w) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      uint32_t p[4], rest[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 8 * b + 2 * e;
        p[e] = pack2<T>(w[r], w[r + 1]);
        if constexpr (PAIR) {
          const float2 hi = unpack2<T>(p[e]);
          rest[e] = pack2<T>(w[r] - hi.x, w[r + 1] - hi.y);
        }
      }
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {
        const uint4 x = at.cols(tile, 2 * t + b, i);
        sum[i] = mma32<T>(x, make_uint4(p[0], p[1], p[2], p[3]), sum[i]);
        if constexpr (PAIR) sum[i] = mma32<T>(x, make_uint4(rest[0], rest[1], rest[2], rest[3]), sum[i]);
      }
    }
  }
  // The same with only the rows of the tile that are to be kept.
  template <class F>
  __device__ __forceinline__ void add_only(const char* tile, int t, const f32x16& w, F keep) {
    add_apart<HD, T>(sum, w, tile, 32 * t, keep);
  }
};

// ------------------------------------------------------------------ queries
template <int HD, CacheType T, int NW>
__global__ __launch_bounds__(64 * NW, HD == 256 ? 1 : 2) void prompt_dq_kernel(PromptBwdArgs b, float2* stats) {
  extern __shared__ __align__(16) char lds[];
  constexpr int KS = HD / 16;
  const PromptArgs& a = b.fwd;
  const int kvh = blockIdx.x % a.n_kv_heads, item = blockIdx.x / a.n_kv_heads, group = a.n_heads / a.n_kv_heads;
  SeqItem st;
  if (!find_item<NW>(a.row_start, a.n_seq, a.rows, group, item, st)) return;
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const SeqRows k = {a.k.p + st.row0 * a.k.ld + kvh * HD, a.k.ld}, v = {a.v.p + st.row0 * a.v.ld + kvh * HD, a.v.ld};
  const int line = NW * st.nth + wave;  // this wave's place in the sequence's line
  const int q0 = 32 * (line / group), head = kvh * group + line % group, qi = q0 + (lane & 31);
  const bool mine = qi < st.len;
  const int64_t row = st.row0 + (int64_t)min(qi, st.len - 1);
  const ScoreScale sc(a.scale);
  uint4 q[KS], go[KS];
  float d = 0.f;
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    const int f = head * HD + 16 * i + 8 * h;
    q[i] = *reinterpret_cast<const uint4*>(a.q.p + row * a.q.ld + f);
    go[i] = *reinterpret_cast<const uint4*>(b.dout.p + row * b.dout.ld + f);
    const uint4 o = *reinterpret_cast<const uint4*>(a.o.p + row * a.o.ld + f);
    const uint32_t x[4] = {go[i].x, go[i].y, go[i].z, go[i].w}, y[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 u = unpack2<T>(x[e]), w = unpack2<T>(y[e]);
      d = fmaf(u.x, w.x, fmaf(u.y, w.y, d));
    }
  }
  d = half_sum(d);
  const float lse = lse_base2(a.lse[row * a.n_heads + head]);
  const bool none = lse == kNoWeight;
  if (none) d = 0.f;
  sc.template turn<T>(q);
  Column<HD, T> dq;
  dq.begin();
  const TileLane<HD> at;
  const int last = (min(32 * ((NW * (st.nth + 1) - 1) / group) + 32, st.len) - 1) / kTile, own = q0 < st.len ? q0 / kTile : -1;
  auto keys = [&](int parity) { return lds + parity * kTileBytes<HD>; };
  auto values = [&](int parity) { return lds + (2 + parity) * kTileBytes<HD>; };
  auto copy = [&](int j, int parity) {
    if (j < 0) return;
    copy_tile<HD, NW>(keys(parity), k, kTile * j, st.len, wave);
    copy_tile<HD, NW>(values(parity), v, kTile * j, st.len, wave);
  };
  auto arrived = [&] {
    WAIT_VMCNT(0);
    __syncthreads();
  };
  // A row's dS add up to 0 but for what the rounding of its output made of D: the keys' pass gets D with that taken back.  This pass
  // cannot wait for it but for the first rows, where dS is smallest beside D, and holds dS in pairs of numbers of the type instead
  // (errors relative to the gradient of bf16 inputs of 279 rows, whose own rounding is 1.66e-3: of dk 2.7e-3 with neither, 2.3e-3 with
  // D; of dq 2.8e-3 with neither, 2.2e-3 with pairs).
  float excess = 0.f;
  // dS of the 32 keys from 32 t on of the tile in buffer `parity`, before the scale; keys behind `to` (from the tile's first) none
  auto ds_of = [&](int parity, int t, int to, bool count) {
    f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
    for (int i = 0; i < KS; ++i) s = mma32<T>(at.rows(keys(parity), 32 * t, i), q[i], s);
#pragma unroll
    for (int i = 0; i < KS; ++i) dp = mma32<T>(at.rows(values(parity), 32 * t, i), go[i], dp);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sc.base2, -lse)) * (dp[r] - d);
      if (to < kTile && 32 * t + mma_row(r, h) > to) s[r] = 0.f;
    }
    if (count) {
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[r & 1] += s[r];
      excess += sum[0] + sum[1];
    }
    return s;
  };
  copy(last, last & 1);
  arrived();
  int j = last;
  for (; j > own; --j) {  // tiles of the workgroup's later queries only
    copy(j - 1, ~j & 1);
    arrived();
  }
  if (own < 0) return;
  copy(j - 1, ~j & 1);
  const int to = min(qi - kTile * j, kTile - 1), halves = q0 % kTile / 32 + 1;  // of the own tile, those with keys that some query sees
  if (j == 0) {  // all keys of these queries: D is exact before dS is taken
#pragma nounroll
    for (int t = 0; t < halves; ++t) ds_of(j & 1, t, to, true);
    d += half_sum(excess);
    excess = 0.f;
  }
#pragma nounroll
  for (int t = 0; t < halves; ++t) {
    f32x16 s = ds_of(j & 1, t, to, true);
    dq.fit(s);
    dq.template add<true>(at, keys(j & 1), t, s);
  }
  if (__builtin_expect(any_nan(dq.sum), 0)) {  // a masked key may have spoiled the sums: once more without it
    dq.begin();
#pragma nounroll
    for (int t = 0; t < halves; ++t) {
      f32x16 s = ds_of(j & 1, t, to, false);
      dq.fit(s);
      dq.add_only(keys(j & 1), t, s, [&](int key) { return key <= to; });
    }
  }
  arrived();
  auto tile = [&](int j, int parity) {
    copy(j - 1, 1 - parity);
#pragma nounroll
    for (int t = 0; t < 2; ++t) {
      f32x16 s = ds_of(parity, t, kTile, true);
      dq.fit(s);
      dq.template add<true>(at, keys(parity), t, s);
    }
    arrived();
  };
  if (--j >= 0 && j % 2 == 0) {
    tile(j, 0);
    --j;
  }
  for (; j >= 0; j -= 2) {
    tile(j, 1);
    tile(j - 1, 0);
  }
  excess = half_sum(excess);
  if (mine && lane < 32) stats[(int64_t)head * a.rows + row] = make_float2(lse, none ? 0.f : d + excess);
  if (__any(none)) {  // weights of 0 times keys of any size
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq.sum[i][r] = none ? 0.f : dq.sum[i][r];
  }
  constexpr int kShare = 4 * kTileBytes<HD> / NW;
  store_rows<HD, T, kShare>(lds + wave * kShare, b.dq.p + (st.row0 + (int64_t)q0) * b.dq.ld + head * HD, b.dq.ld, min(st.len - q0, 32), dq.sum,
                            a.scale / dq.unit);
}

// ------------------------------------------------------------------ keys
// Where one workgroup per 128 keys would leave the GPU empty, each has `parts`, which take turns at the queries and leave fp32 sums.
struct KeyParts {
  int parts;
  float* sums;  // [parts][2][rows][n_kv_heads][head_dim], unused with one part
};

// WHAT: 1 dK, 2 dV, 3 both.  At head_dim 256 the sums of one alone fill half the registers: each has a launch of its own there, and
// scores are computed once more.
//
// Returns whether this wave's sums have a NaN; then they are not stored.  A weight of 0 times an infinite or NaN element may have
// spoiled them: of a masked query, or of one without weight.  CAREFUL, for waves that are to go `again`, leaves such queries out: the
// keys' own tiles are taken apart, and those behind if there is one without weight.
template <int HD, CacheType T, int NW, int WHAT, bool CAREFUL>
__device__ __forceinline__ bool keys_pass(const PromptBwdArgs& b, const float2* stats, const KeyParts& kp, char* lds, bool again) {
  constexpr int M = 32 * NW, KS = HD / 16;
  constexpr bool DK = WHAT & 1, DV = WHAT & 2;
  const PromptArgs& a = b.fwd;
  const int kvh = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads, part = rest % kp.parts, item = rest / kp.parts;
  const int group = a.n_heads / a.n_kv_heads;
  SeqItem st;
  if (!find_sorted<NW>(a.row_start, a.n_seq, a.rows, 1, item, st)) return false;
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nth = (st.len + M - 1) / M - 1 - st.nth;  // the first keys have the most queries
  const int k0 = M * nth + 32 * wave, kj = k0 + (lane & 31);
  const int64_t row = st.row0 + (int64_t)min(kj, st.len - 1);
  const ScoreScale sc(a.scale);
  uint4 k[KS], v[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    k[i] = *reinterpret_cast<const uint4*>(a.k.p + row * a.k.ld + kvh * HD + 16 * i + 8 * h);
    v[i] = *reinterpret_cast<const uint4*>(a.v.p + row * a.v.ld + kvh * HD + 16 * i + 8 * h);
  }
  sc.template turn<T>(k);
  Column<HD, T> dk, dv;
  const TileLane<HD> at;
  // Tiles of queries: those with the workgroup's keys' own, of which one has pairs of this wave's that are masked, and those behind.
  const int first = M * nth / kTile, behind = (min(M * (nth + 1), st.len) - 1) / kTile + 1, end = (st.len + kTile - 1) / kTile;
  const int own = k0 < st.len ? k0 / kTile : end;
  auto tile = [&](int n, int which) { return lds + (2 * (n & 1) + which) * kTileBytes<HD>; };
  auto stat = [&](int n) { return reinterpret_cast<float*>(lds + 4 * kTileBytes<HD>) + (n & 1) * 2 * kTile; };  // log-sum-exps, then D
  // Halves of tile j that have queries.
  auto halves = [&](int j) { return kTile * j + 32 < st.len ? 2 : 1; };
  // Tile j of head `head` into buffer n.  Its rows' statistics pass through a register of the first wave, which puts them there after
  // the tile before has been used: rows behind the last have weights of 0.  (Their lanes load too: where a branch leaves lanes out, the
  // compiler has been seen to save registers of all lanes before it takes them in again.)
  float2 x = make_float2(kNoWeight, 0.f);
  int n_stat = 0;
  auto copy = [&](int n, int head, int j) {
    const SeqRows q = {a.q.p + st.row0 * a.q.ld + head * HD, a.q.ld};
    const SeqRows go = {b.dout.p + st.row0 * b.dout.ld + head * HD, b.dout.ld};
    copy_tile<HD, NW>(tile(n, 0), q, kTile * j, st.len, wave);
    copy_tile<HD, NW>(tile(n, 1), go, kTile * j, st.len, wave);
    n_stat = st.len - kTile * j;
    if (wave == 0) x = stats[(int64_t)head * a.rows + st.row0 + min(kTile * j + lane, st.len - 1)];
  };
  auto arrived = [&](int n) {
    if (wave == 0) {
      stat(n)[lane] = lane < n_stat ? x.x : kNoWeight;
      stat(n)[kTile + lane] = lane < n_stat ? x.y : 0.f;
    }
    WAIT_VMCNT(0);
    __syncthreads();
  };
  // Weights p (times 2^15 in half precision) and ds of the 32 queries from 32 t on of the tile in buffer n; those before `from` (from
  // the tile's first) do not see the lane's key.
  auto weights = [&](int n, int t, int from, bool masked, f32x16& p, f32x16& ds) {
    p = ds = zeros16();
#pragma unroll
    for (int i = 0; i < KS; ++i) p = mma32<T>(at.rows(tile(n, 0), 32 * t, i), k[i], p);
    if constexpr (DK) {
#pragma unroll
      for (int i = 0; i < KS; ++i) ds = mma32<T>(at.rows(tile(n, 1), 32 * t, i), v[i], ds);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 lse = *reinterpret_cast<const f32x4*>(stat(n) + 32 * t + mma_row(4 * i, h));
      const f32x4 d = *reinterpret_cast<const f32x4*>(stat(n) + kTile + 32 * t + mma_row(4 * i, h));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * i + e;
        p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], sc.base2, kWeightExp<T> - lse[e]));
        ds[r] = p[r] * (ds[r] - d[e]);
        if (masked && 32 * t + mma_row(r, h) < from) p[r] = ds[r] = 0.f;
      }
    }
  };
  // All heads' tiles j0 .. j1 - 1 in turn, or this part's share of them.
  auto over = [&](int j0, int j1, auto&& take) {
    const int all = group * (j1 - j0), s0 = (int)((long long)all * part / kp.parts), n = (int)((long long)all * (part + 1) / kp.parts) - s0;
    if (n <= 0) return;
    int head = kvh * group + s0 / (j1 - j0), j = j0 + s0 % (j1 - j0);
    copy(0, head, j);
    arrived(0);
    for (int i = 0; i < n; ++i) {
      const int now = j;
      if (++j == j1) {
        j = j0;
        ++head;
      }
      if (i + 1 < n) copy(i + 1, head, j);
      if (now >= own) take(i, now);
      arrived(i + 1);
    }
  };
  auto add = [&](int n, int t, const f32x16& p, f32x16& ds) {
    if constexpr (DV) dv.add(at, tile(n, 1), t, p);
    if constexpr (DK) {
      dk.fit(ds);
      dk.add(at, tile(n, 0), t, ds);
    }
  };
  auto apart = [&](int n, int j) {
    if (!again) return;
    const int from = kj - kTile * j;
    auto keep = [&](int k) { return k >= from && stat(n)[k] != kNoWeight; };
#pragma nounroll
    for (int t = 0; t < halves(j); ++t) {
      f32x16 p, ds;
      weights(n, t, from, true, p, ds);
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i] = keep(32 * t + mma_row(i, h)) ? ds[i] : 0.f;
      if constexpr (DV) dv.add_only(tile(n, 1), t, p, keep);
      if constexpr (DK) {
        dk.fit(ds);
        dk.add_only(tile(n, 0), t, ds, keep);
      }
    }
  };
  auto whole = [&](int n, int j) {
    if (CAREFUL && !again) return;
#pragma nounroll
    for (int t = 0; t < halves(j); ++t) {
      f32x16 p, ds;
      weights(n, t, 0, false, p, ds);
      add(n, t, p, ds);
    }
  };
  dk.begin();
  dv.begin();
  if constexpr (CAREFUL) {
    over(first, behind, apart);
    bool none = false;  // a query without weight behind the keys
    for (int head = kvh * group; head < (kvh + 1) * group; ++head)
      for (int i = kTile * behind + (int)threadIdx.x; i < st.len; i += 64 * NW) none |= stats[(int64_t)head * a.rows + st.row0 + i].x == kNoWeight;
    if (__builtin_amdgcn_readfirstlane(__syncthreads_or(none))) over(behind, end, apart);
    else over(behind, end, whole);
    if (!again) return false;
  } else {
    over(first, behind, [&](int n, int j) {
#pragma nounroll
      for (int t = 0; t < halves(j); ++t) {
        f32x16 p, ds;
        weights(n, t, kj - kTile * j, true, p, ds);
        add(n, t, p, ds);
      }
    });
    over(behind, end, whole);
  }
  if (own == end) return false;
  if (!CAREFUL && __builtin_expect((DK && any_nan(dk.sum)) || (DV && any_nan(dv.sum)), 0)) return true;
  constexpr float kUnit = T == kBf16 ? 1.f : 0x1p-15f;
  const int64_t first_row = st.row0 + (int64_t)k0;
  const int n = min(st.len - k0, 32);
  const float mul = a.scale * kUnit / dk.unit;
  if (kp.parts == 1) {
    constexpr int kShare = 4 * kTileBytes<HD> / NW;
    if constexpr (DK) store_rows<HD, T, kShare>(lds + wave * kShare, b.dk.p + first_row * b.dk.ld + kvh * HD, b.dk.ld, n, dk.sum, mul);
    if constexpr (DV) store_rows<HD, T, kShare>(lds + wave * kShare, b.dv.p + first_row * b.dv.ld + kvh * HD, b.dv.ld, n, dv.sum, kUnit);
    return false;
  }
  if ((lane & 31) >= n) return false;
  const int64_t width = (int64_t)a.n_kv_heads * HD;
  float* to = kp.sums + (2 * (int64_t)part * a.rows + row) * width + kvh * HD + 4 * h;
#pragma unroll
  for (int mb = 0; mb < HD / 32; ++mb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 u, w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        u[e] = dk.sum[mb][4 * i + e] * mul;
        w[e] = dv.sum[mb][4 * i + e] * kUnit;
      }
      if constexpr (DK) *reinterpret_cast<f32x4*>(to + 32 * mb + 8 * i) = u;
      if constexpr (DV) *reinterpret_cast<f32x4*>(to + a.rows * width + 32 * mb + 8 * i) = w;
    }
  return false;
}

// By a call, so that the pass that all take has not its registers: at head_dim 128 and 256 it spilled 22 to 227 with the tiles taken
// apart in the same function, now 13 and none (64 sequences of 279 to 311 rows, 32 on 8 heads of 128: 375 us, was 391).  At 64 there
// are enough, and the call's stack would cost 1 to 6 us.
typedef __attribute__((address_space(3))) char shared_char;
template <class S>
__device__ __forceinline__ S uniform(const S& s) {  // a call's arguments come in vector registers
  uint32_t w[sizeof(S) / 4];
  __builtin_memcpy(w, &s, sizeof(S));
#pragma unroll
  for (int i = 0; i < (int)(sizeof(S) / 4); ++i) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
  S u;
  __builtin_memcpy(&u, w, sizeof(S));
  return u;
}
template <int HD, CacheType T, int NW, int WHAT>
__device__ __attribute__((noinline)) void keys_again(PromptBwdArgs b, const float2* stats, KeyParts kp, shared_char* lds, bool again) {
  keys_pass<HD, T, NW, WHAT, true>(uniform(b), uniform(stats), uniform(kp), (char*)uniform(lds), __builtin_amdgcn_readfirstlane(again));
}
template <int HD, CacheType T, int NW, int WHAT>
__global__ __launch_bounds__(64 * NW, HD <= 128 ? 2 : 1) void prompt_dkv_kernel(PromptBwdArgs b, const float2* stats, KeyParts kp) {
  extern __shared__ __align__(16) char lds[];
  const bool again = keys_pass<HD, T, NW, WHAT, false>(b, stats, kp, lds, false);
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(__syncthreads_or(again)), 0)) {
    if constexpr (HD == 64) keys_pass<HD, T, NW, WHAT, true>(b, stats, kp, lds, again);
    else keys_again<HD, T, NW, WHAT>(b, stats, kp, (shared_char*)lds, again);
  }
}

// Adds the parts' sums in order, four features a thread, of the rows of sequences.
constexpr int kSumThreads = 256;
template <CacheType T>
__global__ __launch_bounds__(kSumThreads) void prompt_sum_kernel(PromptBwdArgs b, KeyParts kp, int width) {
  const PromptArgs& a = b.fwd;
  const int64_t i = (int64_t)blockIdx.x * kSumThreads + threadIdx.x, row = i / (width / 4);
  const int f = 4 * (int)(i % (width / 4));
  if (row >= a.rows) return;
  bool in = false;  // a row of a sequence (fewer than 410 of them: more fill the GPU, and their keys have one part)
  for (int s = 0, start = a.row_start[0]; s < a.n_seq; s += 8) {
    int end[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) end[i] = a.row_start[min(s + 1 + i, a.n_seq)];  // behind the last: an empty one
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      in |= start >= 0 && start <= row && row < end[i] && end[i] <= a.rows;
      start = end[i];
    }
  }
  if (!in) return;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < kp.parts; ++p) s += *reinterpret_cast<const f32x4*>(kp.sums + ((2 * p + w) * (int64_t)a.rows + row) * width + f);
    const HeadRows& to = w == 0 ? b.dk : b.dv;
    *reinterpret_cast<uint2*>(to.p + row * to.ld + f) = make_uint2(pack2<T>(s[0], s[1]), pack2<T>(s[2], s[3]));
  }
}

// ------------------------------------------------------------------ host
constexpr int kWaves = 4;

// Parts of each 128 keys' queries.  Where the keys' workgroups leave CUs idle, as many as fill the GPU once, with two tiles each or more
// (the whole gradient of 16 sequences of 54 to 108 rows, 16 on 2 heads of 256: 74 us, in one part 157, in ten 95; 1400 rows of 8 heads of
// 128: 88, in one part 113, in two 97, in ten 109).  Long ones, eight tiles or more to a part, fill it twice over, as the first keys of a sequence have many times the work of the last ones.
int key_parts(int rows, int n_seq, int n_heads, int n_kv_heads) {
  const long long groups = seq_items<kWaves>(rows, n_seq, 1) * n_kv_heads;
  const long long steps = ((long long)rows / n_seq / kTile + 1) * (n_heads / n_kv_heads);  // of a workgroup, about
  const long long once = steps < 6 ? 1 : std::min(512 / groups, steps / 2), twice = std::min(1024 / groups, steps / 8);
  return (int)std::max(1ll, std::min(std::max(once, twice), 16ll));
}
size_t stat_bytes(int rows, int n_heads) { return ((size_t)rows * n_heads * sizeof(float2) + 255) / 256 * 256; }

template <int HD, CacheType T, int WHAT>
hipError_t launch_dkv(const PromptBwdArgs& b, long long groups, const float2* stats, const KeyParts& kp, hipStream_t s) {
  constexpr int kLds = 4 * kTileBytes<HD> + 4 * kTile * (int)sizeof(float);
  static LdsLimit limit;
  const auto kernel = prompt_dkv_kernel<HD, T, kWaves, WHAT>;
  const hipError_t e = limit.allow((const void*)kernel, kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * kWaves), kLds, s, b, stats, kp);
  return hipGetLastError();
}

template <int HD, CacheType T>
hipError_t launch(const PromptBwdArgs& b, hipStream_t s) {
  constexpr int NW = kWaves, kDq = 4 * kTileBytes<HD>;
  static LdsLimit limit;
  const auto dq = prompt_dq_kernel<HD, T, NW>;
  hipError_t e = limit.allow((const void*)dq, kDq);
  if (e != hipSuccess) return e;
  const PromptArgs& a = b.fwd;
  const long long items = seq_items<NW>(a.rows, a.n_seq, 1);
  const long long lines = seq_items<NW>(a.rows, a.n_seq, a.n_heads / a.n_kv_heads);
  float2* stats = static_cast<float2*>(b.ws);
  const KeyParts kp = {key_parts(a.rows, a.n_seq, a.n_heads, a.n_kv_heads),
                       reinterpret_cast<float*>(static_cast<char*>(b.ws) + stat_bytes(a.rows, a.n_heads))};
  hipLaunchKernelGGL(dq, dim3((unsigned)(lines * a.n_kv_heads)), dim3(64 * NW), kDq, s, b, stats);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const long long groups = items * a.n_kv_heads * kp.parts;
  if constexpr (HD == 256) {
    e = launch_dkv<HD, T, 1>(b, groups, stats, kp, s);
    if (e == hipSuccess) e = launch_dkv<HD, T, 2>(b, groups, stats, kp, s);
  } else {
    e = launch_dkv<HD, T, 3>(b, groups, stats, kp, s);
  }
  if (e != hipSuccess || kp.parts == 1) return e;
  const int width = a.n_kv_heads * HD;
  const long long threads = (long long)a.rows * (width / 4);
  hipLaunchKernelGGL(prompt_sum_kernel<T>, dim3((unsigned)((threads + kSumThreads - 1) / kSumThreads)), dim3(kSumThreads), 0, s, b, kp, width);
  return hipGetLastError();
}

template <CacheType T>
hipError_t launch_type(const PromptBwdArgs& b, hipStream_t s) {
  if (b.fwd.head_dim == 64) return launch<64, T>(b, s);
  if (b.fwd.head_dim == 128) return launch<128, T>(b, s);
  if (b.fwd.head_dim == 256) return launch<256, T>(b, s);
  return hipErrorInvalidValue;
}

}  // namespace

size_t prompt_bwd_bytes(int rows, int n_seq, int n_heads, int n_kv_heads, int head_dim) {
  if (rows == 0 || n_seq == 0) return 0;
  const int parts = key_parts(rows, n_seq, n_heads, n_kv_heads);
  return stat_bytes(rows, n_heads) + (parts == 1 ? 0 : (size_t)parts * 2 * rows * n_kv_heads * head_dim * sizeof(float));
}

hipError_t launch_prompt_attn_bwd(const PromptBwdArgs& b, hipStream_t s) {
  return b.fwd.type == kBf16 ? launch_type<kBf16>(b, s) : launch_type<kF16>(b, s);
}

}  // namespace vla
