// Norms of queries and keys per head with their rotation and the append to the paged cache, and the gradient of the norms
// and the rotation (vla_qk_norm_rope, vla_qk_norm_rope_backward).
//
// Bound: HBM, every feature read once and written once (the gradient: two read, one written).  A head vector is held by
// head_dim / 16 lanes, 16 features each, placed so that both features of every pair are in one lane: the norm is a sum over
// 4, 8 or 16 lanes by DPP, the rotation needs no exchange.  Measured at 32 + 8 heads of 128: 18432 rows appended in 82 us, 453
// MB, 5.5 TB/s (a copy of 1 GiB past the caches, as these accesses are: 6.0); the gradient of 18880 rows 109 us and 5 for the
// gains, 580 MB, 5.1 TB/s; one row 3.1 us.
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

// 16 bytes from or to memory, past the caches where a call moves more than they hold (STREAM).
template <bool STREAM>
__device__ __forceinline__ uint4 load16(const bf16_t* p) {
  const u32x4* s = reinterpret_cast<const u32x4*>(p);
  const u32x4 v = STREAM ? __builtin_nontemporal_load(s) : *s;
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <bool STREAM>
__device__ __forceinline__ void store16(bf16_t* p, const uint4& v) {
  const u32x4 u = {v.x, v.y, v.z, v.w};
  if (STREAM) __builtin_nontemporal_store(u, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = u;
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

// Lane j of a head holds two 8-feature chunks, chosen so that pairs stay together and neighbouring lanes' chunks are
// neighbours in memory: interleaved, chunks j and j + N of the 2 N; in the half layout the n = rot / 16 first lanes hold j and
// j + n (both halves of their pairs), the others j + n and j + N.  pair0, pair1: the first pairs of the lane's two sets of
// four, turned0, turned1: whether they are rotated.
template <int HD, int LAYOUT>
struct Chunks {
  int lo, hi;  // first features of the chunks
  int pair0, pair1;
  bool turned0, turned1;
  __device__ __forceinline__ Chunks(int j, int rot_dim) {
    constexpr int N = HD / 16;
    const int n = rot_dim >> 4;
    constexpr bool half = LAYOUT == 0;
    const bool first = half && j < n;
    lo = 8 * (half && !first ? j + n : j);
    hi = 8 * (first ? j + n : j + N);
    pair0 = half ? 8 * j : lo / 2;
    pair1 = half ? 8 * j + 4 : hi / 2;
    turned0 = half ? first : lo < rot_dim;
    turned1 = half ? first : hi < rot_dim;
  }
};

// Rotates four pairs: a, b by the angles of cosine c and sine s.
__device__ __forceinline__ void turn_pair(float& a, float& b, float c, float s) {
  const float x = a, y = b;
  a = fmaf(x, c, -(y * s));
  b = fmaf(y, c, x * s);
}
// Rotates the lane's features y[0 .. 8) (chunk lo) and y[8 .. 16) (chunk hi) by the angles of its two sets of pairs.
template <int HD, int LAYOUT>
__device__ __forceinline__ void turn(float (&y)[16], const Chunks<HD, LAYOUT>& ch, const float (&c)[8], const float (&s)[8]) {
  if constexpr (LAYOUT == 0) {
    if (ch.turned0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) turn_pair(y[e], y[8 + e], c[e], s[e]);
    }
  } else {
    if (ch.turned0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) turn_pair(y[2 * e], y[2 * e + 1], c[e], s[e]);
    }
    if (ch.turned1) {
#pragma unroll
      for (int e = 4; e < 8; ++e) turn_pair(y[2 * e], y[2 * e + 1], c[e], s[e]);
    }
  }
}

// The turns p f / (2 pi) are reduced in 64 bits, so that far positions lose nothing; the hardware's sine and cosine of a
// fraction of a turn are within 2^-22.9.
__device__ __forceinline__ void angle(double turns_per_position, int pos, float scale, float& c, float& s) {
  const float x = (float)__builtin_amdgcn_fract((double)pos * turns_per_position);
  c = scale * __builtin_amdgcn_cosf(x);
  s = scale * __builtin_amdgcn_sinf(x);
}
constexpr double kTurns = 0.15915494309189533577;  // per radian

constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / kWave;

// Slot of a row, -1 where it is outside the pool or there is no such row.
__device__ __forceinline__ int slot_of(const QkRopeArgs& a, long long row) {
  const int s = row >= 0 && row < a.rows ? a.row_slot[row] : -1;
  return s < (long long)a.n_pages * kPage ? max(s, -1) : -1;
}

// A wave takes passes `part`, part + parts, ... of a row's head vectors, 64 / (HD / 16) a pass; the angles are the same for
// all of them.  One pass at a time: eight waves per SIMD keep more on the way than unrolled passes (two together 103 us, four
// over tiles of rows with the angles in LDS 112, where this takes 97, all with cached accesses).
template <int HD, CacheType T, int LAYOUT, bool STREAM>
__device__ __forceinline__ void rope_row(const QkRopeArgs& a, long long row, int part, int parts) {
  constexpr int LPH = HD / 16, HPW = kWave / LPH;
  const int lane = threadIdx.x & 63, j = lane % LPH, heads = a.n_heads + a.n_kv_heads;
  int slot = 0;
  if (a.row_slot) {
    slot = slot_of(a, row);
    if (slot < 0) return;
  }
  const Chunks<HD, LAYOUT> ch(j, a.rot_dim);
  float c[8] = {}, s[8] = {};
  if (ch.turned0 || ch.turned1) {
    const int pos = a.row_pos[row], last = a.rot_dim / 2 - 4;
    const double* f0 = a.freqs + min(ch.pair0, last);  // a set that is not rotated is not used
    const double* f1 = a.freqs + min(ch.pair1, last);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      angle(f0[e] * kTurns, pos, a.rope_scale, c[e], s[e]);
      angle(f1[e] * kTurns, pos, a.rope_scale, c[4 + e], s[4 + e]);
    }
  }
  for (int h0 = part * HPW; h0 < heads; h0 += parts * HPW) {
    const int h = h0 + lane / LPH;
    if (h >= heads) continue;
    const bool is_q = h < a.n_heads;
    const int hh = is_q ? h : h - a.n_heads;
    const bf16_t* x = (is_q ? a.q.p + row * a.q.ld : a.k.p + row * a.k.ld) + hh * HD;
    const uint4 v0 = load16<STREAM>(x + ch.lo), v1 = load16<STREAM>(x + ch.hi);
    float y[16];
    unpack<T>(v0, y);
    unpack<T>(v1, y + 8);
    const bf16_t* gain = is_q ? a.q_gain : a.k_gain;
    if (gain) {
      float g[16], ss = 0.f;
      unpack<T>(*reinterpret_cast<const uint4*>(gain + ch.lo), g);
      unpack<T>(*reinterpret_cast<const uint4*>(gain + ch.hi), g + 8);
#pragma unroll
      for (int e = 0; e < 16; ++e) ss = fmaf(y[e], y[e], ss);
      const float r = rsqrtf(group_sum<LPH>(ss) * (1.f / HD) + a.eps);
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = y[e] * r * g[e];
    }
    turn(y, ch, c, s);
    const uint4 o0 = pack<T>(y), o1 = pack<T>(y + 8);
    bf16_t* o = is_q ? a.q_out.p + row * a.q_out.ld + hh * HD : a.k_out.p ? a.k_out.p + row * a.k_out.ld + hh * HD : nullptr;
    if (o) {
      store16<STREAM>(o + ch.lo, o0);
      store16<STREAM>(o + ch.hi, o1);
    }
    if (!is_q && a.pages.k) {
      o = a.pages.k + (((long long)(slot / kPage) * a.n_kv_heads + hh) * kPage + slot % kPage) * HD;
      store16<STREAM>(o + ch.lo, o0);
      store16<STREAM>(o + ch.hi, o1);
    }
  }
}

// 64 features of a key head's values to their transposed pages, by one wave through its own LDS.  Rows whose slots follow one
// another go together in groups that end where a slot is a multiple of 8: 8 features' slots are one 16-byte store then.  The
// wave takes the groups that begin in rows row0 .. row0 + n - 1, up to 7 rows past them; shorter groups (a decode step's
// rows) are stored 2 bytes a feature.  `first`: the features' number among all of the row.
constexpr int kTileRows = 16, kTileSpan = kTileRows + 8, kSlice = 64;
struct ValueTile {
  bf16_t x[kTileSpan][kSlice + 8];
};
template <int HD>
__device__ __forceinline__ void append_v(const QkRopeArgs& a, long long row0, int n, int first, ValueTile& tile) {
  const int lane = threadIdx.x & 63;
  // lane i: row row0 + i
  const int slot = lane < n + 8 ? slot_of(a, row0 + lane) : -1, prev = lane <= n + 8 ? slot_of(a, row0 + lane - 1) : -1;
  const unsigned long long lives = __ballot(slot >= 0), ends = __ballot(prev < 0 || slot != prev + 1 || slot % 8 == 0) | ~lives;
  const unsigned long long begins = ends & lives & ((1ull << n) - 1);
  if (!begins) return;
  const int r0 = __builtin_ctzll(begins), r1 = 64 - __builtin_clzll(begins);  // rows from r0 on; the last group begins at r1 - 1
  const int end = r1 + __builtin_ctzll(ends >> r1);                           // at most n + 8: lanes from there on are no rows
  const bf16_t* src = a.v.p + (row0 + lane / 8) * a.v.ld + first + 8 * (lane % 8);
#pragma unroll
  for (int i = 0; i < kTileSpan / 8; ++i) {
    const int r = lane / 8 + i * 8;
    if (r >= r0 && r < end && (lives >> r & 1)) *reinterpret_cast<uint4*>(&tile.x[r][8 * (lane % 8)]) = load16<false>(src + i * 8 * a.v.ld);
  }
  // written by other lanes and as another type: the reads below stay behind the writes (no instruction, LDS is in order)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // feature `first` of slot s: head first / HD, its feature first % HD
  auto at = [&](int s) { return a.pages.v + ((long long)(s / kPage) * a.n_kv_heads * HD + first) * kPage + s % kPage; };
  unsigned long long todo = begins;
  while (todo) {
    // two groups at a time, every other lane one, so that the two halves of a page are stored side by side
    const int i0 = __builtin_ctzll(todo);
    todo &= todo - 1;
    const int i1 = todo ? __builtin_ctzll(todo) : i0;
    const int len0 = __builtin_ctzll(ends >> (i0 + 1)) + 1, len1 = __builtin_ctzll(ends >> (i1 + 1)) + 1;
    if (len0 == 8) {
      const bool both = i1 != i0 && len1 == 8, second = lane & 1;
      if (both) todo &= todo - 1;
      if (second && !both) continue;
      const int i = second ? i1 : i0;
      bf16_t* dst = second ? at(__builtin_amdgcn_readlane(slot, i1)) : at(__builtin_amdgcn_readlane(slot, i0));
#pragma unroll
      for (int f0 = 0; f0 < kSlice; f0 += 32) {
        const int f = f0 + lane / 2;
        uint32_t d[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) d[r] = tile.x[i + 2 * r][f] | (uint32_t)tile.x[i + 2 * r + 1][f] << 16;
        store16<false>(dst + f * kPage, make_uint4(d[0], d[1], d[2], d[3]));
      }
    } else {
      bf16_t* dst = at(__builtin_amdgcn_readlane(slot, i0)) + lane * kPage;
      for (int r = 0; r < len0; ++r) dst[r] = tile.x[i0 + r][lane];
    }
  }
}

// The first workgroups take queries and keys, the others the values of a tile of rows and four 64-feature slices.
template <int HD, CacheType T, int LAYOUT, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void qk_rope_kernel(QkRopeArgs a, int groups, int parts, int tile) {
  __shared__ __align__(16) ValueTile values[kRopeWaves];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x < groups) {
    const long long wave = (long long)blockIdx.x * kRopeWaves + w, row = parts == 1 ? wave : wave / parts;
    if (row < a.rows) rope_row<HD, T, LAYOUT, STREAM>(a, row, (int)(wave - row * parts), parts);
  } else {
    const int slices = a.n_kv_heads * (HD / kSlice), quads = (slices + kRopeWaves - 1) / kRopeWaves;
    const int i = blockIdx.x - groups, row0 = i / quads * tile, slice = i % quads * kRopeWaves + w;
    if (slice < slices) append_v<HD>(a, row0, min(tile, a.rows - row0), slice * kSlice, values[w]);
  }
}

// ------------------------------------------------------------------ backward
// n / d for n < 2^16 and d <= 2^12, given div_magic(d): with e = d ceil(2^32 / d) - 2^32 < d, n e < 2^32.
__host__ __device__ __forceinline__ unsigned div_magic(unsigned d) { return (unsigned)(0xffffffffull / d + 1); }  // 0 for 1
__device__ __forceinline__ int div_by(int n, unsigned magic) { return magic ? (int)__umulhi((unsigned)n, magic) : n; }

// Cosines and sines of a tile's rows and pairs.
template <int HD>
struct Angles {
  float c[kTileRows][HD / 2], s[kTileRows][HD / 2];
  __device__ __forceinline__ void fill(const double* freqs, const int32_t* row_pos, int pairs, float scale, long long row0, int rows) {
    const int p = threadIdx.x % (HD / 2);
    if (p >= pairs) return;
    const double f = freqs[p] * kTurns;
    for (int r = threadIdx.x / (HD / 2); r < rows; r += kRopeThreads / (HD / 2)) angle(f, row_pos[row0 + r], scale, c[r][p], s[r][p]);
  }
  // Rotates the lane's features back.
  template <int LAYOUT>
  __device__ __forceinline__ void turn_back(float (&y)[16], const Chunks<HD, LAYOUT>& ch, int r) const {
    float cs[8] = {}, sn[8] = {};
    if (ch.turned0 || ch.turned1) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int p = i == 0 ? ch.pair0 : ch.turned1 ? ch.pair1 : ch.pair0;
        const f32x4 a = *reinterpret_cast<const f32x4*>(&c[r][p]), b = *reinterpret_cast<const f32x4*>(&s[r][p]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          cs[4 * i + e] = a[e];
          sn[4 * i + e] = -b[e];
        }
      }
    }
    turn(y, ch, cs, sn);
  }
};
// Workgroups of the gradient: two per CU, each with its sums in registers (us of 18880 and 4096 rows, 512 / 768 / 1024: 117.8,
// 31.5 / 121.1, 33.9 / 129.2, 38.3).
constexpr int kBwdGroups = 512;

// The gradient of a tile's queries or of its keys.
template <int HD, CacheType T, int LAYOUT, bool STREAM>
struct Backward {
  static constexpr int LPH = HD / 16, VPP = kRopeThreads / LPH;  // lanes per head vector, vectors per pass
  // What a lane holds of a vector: the gradient and the input.
  struct Vector {
    uint4 d[2], x[2];
    int row, head;
  };
  const Chunks<HD, LAYOUT>& ch;
  HeadRows in, dout, out;
  const bf16_t* gain;
  int heads;
  unsigned magic;
  float eps;

  __device__ __forceinline__ void load(Vector& u, long long row0, int v) const {
    u.row = div_by(v, magic);
    u.head = v - u.row * heads;
    const bf16_t* p = dout.p + (row0 + u.row) * dout.ld + u.head * HD;
    u.d[0] = load16<STREAM>(p + ch.lo);
    u.d[1] = load16<STREAM>(p + ch.hi);
    if (gain) {
      p = in.p + (row0 + u.row) * in.ld + u.head * HD;
      u.x[0] = load16<STREAM>(p + ch.lo);
      u.x[1] = load16<STREAM>(p + ch.hi);
    }
  }
  // The first pass's vector of a tile, on its way before the tile's angles are known.
  __device__ __forceinline__ void start(Vector& u, long long row0, int rows) const {
    const int v = threadIdx.x / LPH;
    if (v < rows * heads) load(u, row0, v);
  }
  // All passes from `cur` on; the next pass's vector is on its way while one is taken.
  __device__ __forceinline__ void tile(Vector cur, const Angles<HD>& angles, long long row0, int rows, float (&dg)[16]) const {
    const int vectors = rows * heads;
    uint4 w[2];
    if (gain) {
      w[0] = *reinterpret_cast<const uint4*>(gain + ch.lo);
      w[1] = *reinterpret_cast<const uint4*>(gain + ch.hi);
    }
    for (int v = threadIdx.x / LPH; v < vectors; v += VPP) {
      Vector next = cur;
      if (v + VPP < vectors) load(next, row0, v + VPP);
      float y[16];
      unpack<T>(cur.d[0], y);
      unpack<T>(cur.d[1], y + 8);
      angles.turn_back(y, ch, cur.row);
      if (gain) {
        float g[16], h[16], ss = 0.f;
        unpack<T>(w[0], g);
        unpack<T>(w[1], g + 8);
        unpack<T>(cur.x[0], h);
        unpack<T>(cur.x[1], h + 8);
#pragma unroll
        for (int e = 0; e < 16; ++e) ss = fmaf(h[e], h[e], ss);
        const float r = rsqrtf(group_sum<LPH>(ss) * (1.f / HD) + eps);
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          h[e] *= r;
          dg[e] = fmaf(h[e], y[e], dg[e]);
          y[e] *= g[e];
          dot = fmaf(h[e], y[e], dot);
        }
        dot = group_sum<LPH>(dot) * (1.f / HD);
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = r * fmaf(-h[e], dot, y[e]);
      }
      bf16_t* o = out.p + (row0 + cur.row) * out.ld + cur.head * HD;
      store16<STREAM>(o + ch.lo, pack<T>(y));
      store16<STREAM>(o + ch.hi, pack<T>(y + 8));
      cur = next;
    }
  }
};

// Sum over the lanes that share lane % N (N = 4, 8, 16).
template <int N>
__device__ __forceinline__ float across_sum(float v) {
  if constexpr (N <= 8) v += dpp_mov<0x128>(v, v);  // 8 lanes on in the 16
  if constexpr (N <= 4) v += dpp_mov<0x124>(v, v);  // 4 lanes on
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A workgroup goes over tiles of rows, all of them side by side in memory; the gains' gradients of its lanes' features stay
// in registers, are joined over the workgroup and left in part[group][q or k][feature].  A tile's first queries are
// requested before its angles are made (18880 and 300 rows of 32 + 8 heads: 117.5 -> 115.6, 12.3 -> 10.7 us).
template <int HD, CacheType T, int LAYOUT, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void qk_rope_bwd_kernel(QkRopeBwdArgs a, int tile, unsigned magic_q, unsigned magic_k) {
  using B = Backward<HD, T, LAYOUT, STREAM>;
  __shared__ Angles<HD> angles;
  __shared__ float red[kRopeWaves][2][HD];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, j = threadIdx.x % B::LPH;
  const Chunks<HD, LAYOUT> ch(j, a.rot_dim);
  const B q = {ch, a.q, a.dq_out, a.dq, a.q_gain, a.n_heads, magic_q, a.eps};
  const B k = {ch, a.k, a.dk_out, a.dk, a.k_gain, a.n_kv_heads, magic_k, a.eps};
  float dg[2][16];
#pragma unroll
  for (int e = 0; e < 16; ++e) dg[0][e] = dg[1][e] = 0.f;
  for (long long row0 = (long long)blockIdx.x * tile; row0 < a.rows; row0 += (long long)gridDim.x * tile) {
    const int rows = (int)min((long long)tile, a.rows - row0);
    typename B::Vector vq, vk;
    q.start(vq, row0, rows);
    if (a.rot_dim > 0) {
      __syncthreads();  // the last tile's angles have been read
      angles.fill(a.freqs, a.row_pos, a.rot_dim / 2, a.rope_scale, row0, rows);
      __syncthreads();
    }
    q.tile(vq, angles, row0, rows, dg[0]);
    k.start(vk, row0, rows);
    k.tile(vk, angles, row0, rows, dg[1]);
  }
  if (!a.q_gain && !a.k_gain) return;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float v = across_sum<B::LPH>(dg[t][e]);
      if (lane < B::LPH) red[w][t][(e < 8 ? ch.lo : ch.hi) + e % 8] = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * HD; i += kRopeThreads) {
    float v = 0.f;
#pragma unroll
    for (int u = 0; u < kRopeWaves; ++u) v += red[u][i / HD][i % HD];
    a.part[(size_t)blockIdx.x * 2 * HD + i] = v;
  }
}

// Sums the groups' parts in a fixed order: 64 columns per workgroup, its waves every 16th group each.
constexpr int kFinishWaves = 16;
__global__ __launch_bounds__(64 * kFinishWaves) void qk_rope_gain_kernel(QkRopeBwdArgs a, int groups) {
  __shared__ float red[kFinishWaves][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, cols = 2 * a.head_dim, c = blockIdx.x * 64 + lane;
  float v = 0.f;
#pragma unroll 8
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

// ------------------------------------------------------------------ host
// Past the caches from 64 MB a call on, where each access covers whole cache lines (18432 rows of 32 + 8 heads of 128: 97.7 ->
// 86.4 us, 4096 rows 26.0 -> 22.6; 2048 rows 11.6 -> 14.3; heads of 64, of which an access covers half a line, 53.8 -> 57.2).
constexpr size_t kStreamBytes = (size_t)64 << 20;
template <int HD, int LAYOUT>
bool whole_lines(int rot_dim) {
  return HD >= 128 && (LAYOUT == 1 || rot_dim == HD || rot_dim == 0);
}

// The forward's launch: workgroups for queries and keys, `parts` waves a row, then those for tiles of values.
struct FwdGrid {
  int parts, tile;
  long long groups, all;
};
FwdGrid fwd_grid(int rows, int n_heads, int n_kv_heads, int head_dim, bool cache) {
  const int per_wave = kWave / (head_dim / 16), heads = n_heads + n_kv_heads;
  FwdGrid g;
  g.parts = rows >= 2048 ? 1 : (heads + per_wave - 1) / per_wave;
  g.tile = std::min(kTileRows, std::max(1, rows / 512));
  g.groups = ((long long)rows * g.parts + kRopeWaves - 1) / kRopeWaves;
  const long long tiles = (rows - 1) / g.tile + 1, quads = cache ? (n_kv_heads * (head_dim / kSlice) + kRopeWaves - 1) / kRopeWaves : 0;
  g.all = g.groups + tiles * quads;
  return g;
}

template <int HD, CacheType T, int LAYOUT>
struct Fwd {
  static hipError_t run(const QkRopeArgs& a, hipStream_t s) {
    const FwdGrid g = fwd_grid(a.rows, a.n_heads, a.n_kv_heads, HD, a.pages.v != nullptr);
    const dim3 grid((unsigned)g.all), block(kRopeThreads);
    const size_t bytes = (size_t)a.rows * (a.n_heads + 2 * a.n_kv_heads) * HD * 4;
    const bool stream = whole_lines<HD, LAYOUT>(a.rot_dim) && bytes > kStreamBytes;
    if (stream) hipLaunchKernelGGL((qk_rope_kernel<HD, T, LAYOUT, true>), grid, block, 0, s, a, (int)g.groups, g.parts, g.tile);
    else hipLaunchKernelGGL((qk_rope_kernel<HD, T, LAYOUT, false>), grid, block, 0, s, a, (int)g.groups, g.parts, g.tile);
    return hipGetLastError();
  }
};

template <int HD, CacheType T, int LAYOUT>
struct Bwd {
  static hipError_t run(const QkRopeBwdArgs& a, hipStream_t s) {
    // tiles of equal size, as many for each workgroup, no smaller than what fills its lanes with queries
    constexpr int VPP = Backward<HD, T, LAYOUT, false>::VPP;
    const long long rounds = ((long long)a.rows + kBwdGroups * kTileRows - 1) / (kBwdGroups * kTileRows), per = std::max(rounds, 1ll) * kBwdGroups;
    const int tile = std::min(kTileRows, std::max((VPP + a.n_heads - 1) / a.n_heads, (int)((a.rows + per - 1) / per)));
    const int groups = a.rows > 0 ? std::min(kBwdGroups, (a.rows - 1) / tile + 1) : 0;
    const unsigned mq = div_magic(a.n_heads), mk = div_magic(a.n_kv_heads);
    const bool stream = whole_lines<HD, LAYOUT>(a.rot_dim) && (size_t)a.rows * (a.n_heads + a.n_kv_heads) * HD * 6 > kStreamBytes;
    const dim3 grid(groups), block(kRopeThreads);
    if (groups > 0) {
      if (stream) hipLaunchKernelGGL((qk_rope_bwd_kernel<HD, T, LAYOUT, true>), grid, block, 0, s, a, tile, mq, mk);
      else hipLaunchKernelGGL((qk_rope_bwd_kernel<HD, T, LAYOUT, false>), grid, block, 0, s, a, tile, mq, mk);
    }
    if (a.q_gain || a.k_gain)
      hipLaunchKernelGGL(qk_rope_gain_kernel, dim3(2 * HD / 64), dim3(64 * kFinishWaves), 0, s, a, groups);
    return hipGetLastError();
  }
};

template <template <int, CacheType, int> class F, int HD, class A>
hipError_t by_type(const A& a, hipStream_t s) {
  if (a.type == kBf16) return a.layout == 0 ? F<HD, kBf16, 0>::run(a, s) : F<HD, kBf16, 1>::run(a, s);
  return a.layout == 0 ? F<HD, kF16, 0>::run(a, s) : F<HD, kF16, 1>::run(a, s);
}
template <template <int, CacheType, int> class F, class A>
hipError_t by_head(const A& a, hipStream_t s) {
  if (a.head_dim == 64) return by_type<F, 64>(a, s);
  if (a.head_dim == 128) return by_type<F, 128>(a, s);
  if (a.head_dim == 256) return by_type<F, 256>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace

bool qk_rope_fits(int rows, int n_heads, int n_kv_heads, int head_dim, bool cache) {
  return fwd_grid(rows, n_heads, n_kv_heads, head_dim, cache).all * kRopeThreads < 1ll << 32;
}
size_t qk_rope_bwd_floats(int head_dim) { return (size_t)kBwdGroups * 2 * head_dim; }
hipError_t launch_qk_rope(const QkRopeArgs& a, hipStream_t s) { return by_head<Fwd>(a, s); }
hipError_t launch_qk_rope_bwd(const QkRopeBwdArgs& a, hipStream_t s) { return by_head<Bwd>(a, s); }

}  // namespace vla
