// Device code that attention over whole prompts and its gradient share: tiles of rows in LDS, 32x32x16 MFMA operands from them,
// and the way from a workgroup to its sequence.
//
// Every product has the softmax's own index on the MFMA's columns: a wave holds 32 queries (or keys) as columns, lane % 32, and
// the other index on the rows, of which lane half h = lane / 32 has rows 8 i + 4 h + e, i, e = 0 .. 3, in registers 4 i + e.  Eight
// of these (i = 2 b, 2 b + 1) are the B operand of step b of the next product, if its A operand's k are taken in the same order:
// two transposed reads of 4 rows each, 4 h .. and 8 + 4 h .. of the step's 16.  So weights never leave their registers.
#pragma once

#include "cache.h"
#include "common.h"

namespace vla {
namespace tiles {

constexpr int kTile = 64;  // rows of a tile in LDS
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <CacheType T>
__device__ __forceinline__ f32x16 mma32(const uint4& a, const uint4& b, const f32x16& c) {
  if constexpr (T == kBf16) return mfma32(as_bf16x8(a), as_bf16x8(b), c);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// Two numbers of the type, to nearest even.
template <CacheType T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const f32x2 v = {lo, hi};  // as a pair: one conversion of both
  if constexpr (T == kBf16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}
template <CacheType T>
__device__ __forceinline__ float2 unpack2(uint32_t v) {
  if constexpr (T == kBf16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  const f16x2 h = __builtin_bit_cast(f16x2, v);
  return make_float2((float)h[0], (float)h[1]);
}
// The scale of the scores to base 2, positive: its sign goes into one of the factors, and a scale of 0 makes that factor 0, or NaN
// where it is infinite or NaN, so that the largest product has the largest score and a masked one's -inf stays -inf.
struct ScoreScale {
  float base2;
  uint32_t sign;
  bool zero;
  __device__ __forceinline__ explicit ScoreScale(float s)
      : base2(s == 0.f ? 1.f : fabsf(s) * kLog2e), sign(s < 0.f ? 0x80008000u : 0u), zero(s == 0.f) {}
  // After all loads of x: a branch between them would have each waited for (64 sequences of 272 to 304 rows: 163 us, not 115).
  template <CacheType T, int N>
  __device__ __forceinline__ void turn(uint4 (&x)[N]) const {
    if (__builtin_expect(zero, 0)) {
      auto two = [](uint32_t v) {
        constexpr uint32_t kExp = T == kBf16 ? 0x7f80 : 0x7c00;
        return ((v & kExp) == kExp ? 0x7fffu : 0u) | ((v & kExp << 16) == kExp << 16 ? 0x7fff0000u : 0u);
      };
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = make_uint4(two(x[i].x), two(x[i].y), two(x[i].z), two(x[i].w));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = make_uint4(x[i].x ^ sign, x[i].y ^ sign, x[i].z ^ sign, x[i].w ^ sign);
  }
};
// Half-precision weights are held 2^15 times as large: the largest stays below 65504, and one is rounded to fewer than 11 bits only
// below 2^-29 of the largest.
template <CacheType T>
constexpr float kWeightExp = T == kBf16 ? 0.f : 15.f;
// The running maximum follows the scores only where they pass it by a factor of 2^4 of the weights: 17 products of what is summed per
// tile are saved at most of them.  Weights are then up to 16, and half-precision ones held 2^11 times as large.
constexpr float kSlack = 4.f;
template <CacheType T>
constexpr float kHeldExp = T == kBf16 ? 0.f : kWeightExp<T> - kSlack;
__device__ __forceinline__ f32x16 zeros16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// Max / sum over the two lanes that share lane % 32.
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// MFMA row of register r in lane half h.
__device__ __forceinline__ constexpr int mma_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// ------------------------------------------------------------------ tiles in LDS
// Row R of a tile lies at R * 2 HD bytes, its 16-byte chunk j at place j ^ swz(R).  Both ways to read then spread over all
// banks: the same chunk of 16 consecutive rows (128-bit reads), and 64 bytes of 4 consecutive rows (transposed reads).
template <int HD>
__device__ __forceinline__ int swz(int R) {
  return HD == 64 ? ((R >> 1 & 1) << 2 | (R >> 2 & 3)) : ((R & 3) << 2 | (R >> 2 & 3));
}
template <int HD>
constexpr int kTileBytes = kTile * HD * 2;

// Rows of four pages of a cache as a tile: MFMA row m is the pages' token page_row(m), so that lane half h holds tokens 8 h .. 8 h + 7
// of page b in registers 8 b .. 8 b + 7, which meet the 16 bytes of a feature's values there as they lie.
__device__ __forceinline__ constexpr int page_row(int m) { return (m & 19) | (m >> 2 & 1) << 3 | (m >> 3 & 1) << 2; }

// Lane addresses into a tile.
template <int HD, bool PAGES = false>
struct TileLane {
  uint32_t row;   // chunk 0 of the lane's row, before its place is turned
  uint32_t turn;  // 16 (lane / 32 ^ swz of that row)
  uint32_t col;   // first transposed read of features 0 .. 31; PAGES: this lane's feature of the first 32 in a page
  __device__ __forceinline__ TileLane() {
    const int lane = threadIdx.x & 63, h = lane >> 5, i = lane & 15, m = PAGES ? page_row(lane & 31) : lane & 31;
    row = m * HD * 2;
    turn = 16 * (h ^ swz<HD>(m));
    if constexpr (PAGES) {
      col = 32 * (lane & 31) + 16 * h;
      return;
    }
    const int r = 4 * h + (i >> 2);
    col = r * HD * 2 + 16 * ((2 * (lane >> 4 & 1) + (i >> 1 & 1)) ^ swz<HD>(r)) + 8 * (i & 1);
  }
  // Row lane % 32 of the 32 from r0 on (0 or 32), features 16 ks + 8 (lane / 32) .. + 8.
  __device__ __forceinline__ uint4 rows(const char* tile, int r0, int ks) const {
    return *reinterpret_cast<const uint4*>(tile + r0 * HD * 2 + row + (turn ^ 32 * ks));
  }
  // Features 32 mb + lane % 32, rows 16 b + 4 (lane / 32) .. + 4 and 8 more on; PAGES: of page b's values [HD][16], tokens
  // 8 (lane / 32) .. + 8.
  __device__ __forceinline__ uint4 cols(const char* tile, int b, int mb) const {
    if constexpr (PAGES) return *reinterpret_cast<const uint4*>(tile + (b * HD + 32 * mb) * 32 + col);
    // eight rows on, bit 1 of the place turns; 32 features on, bits 2 and up
    const char* p = tile + 16 * b * HD * 2;
    return __builtin_bit_cast(uint4, lds_read_tr(p + (col ^ 64 * mb), p + 8 * HD * 2 + (col ^ 32 ^ 64 * mb)));
  }
};

// The rows of one head of a sequence, from its first on.
struct SeqRows {
  const bf16_t* p;
  int64_t ld;
};
// Copies rows r0 .. r0 + 63 of a sequence of `len` rows into a tile (rows behind its last: that one), 1 KB per wave and
// instruction; the waves of the workgroup share them.
template <int HD, int NW>
__device__ __forceinline__ void copy_tile(char* tile, const SeqRows& x, int r0, int len, int wave) {
  constexpr int CH = HD / 8, RPK = 64 / CH, N = kTile / RPK;  // chunks of a row, rows of a copy, copies
  const int lane = threadIdx.x & 63;
  const uint32_t lb = (uint32_t)(uintptr_t)((lds_ptr_t*)tile);
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc((void*)(x.p + (int64_t)r0 * x.ld), (short)0, 0x7fffffff, 0x00020000);
#pragma unroll
  for (int i = 0; i < (N + NW - 1) / NW; ++i) {
    const int j = i * NW + wave;
    if (N % NW != 0 && j >= N) break;
    const int R = j * RPK + lane / CH;
    lds_dma16(__builtin_amdgcn_readfirstlane(lb + j * 1024), (uint32_t)(min(R, len - 1 - r0) * (int)x.ld + 8 * ((lane % CH) ^ swz<HD>(R))) * 2, rs, 0);
  }
}

// acc[mb][r] += sum over the 32 rows k of a tile from r0 on of w[k] x[k][feature], features 32 mb + mma_row(r): one product on the
// vector units, with every term for which keep(k) is false left out whatever x[k] is.  w: the weights of this lane's column, as
// the two halves hold them.  Only where infinite or NaN elements lie in a tile part of whose pairs are masked.
template <int HD, CacheType T, class F>
__device__ __forceinline__ void add_apart(f32x16 (&acc)[HD / 32], f32x16 w, const char* tile, int r0, F keep) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma nounroll
  for (int n = 0; n < 32; ++n) {  // row n's weight is in half n / 4 % 2, register 4 (n / 8) + n % 4
    float p = w[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) p = 4 * (n >> 3) + (n & 3) == r ? w[r] : p;
    p = __shfl(p, (lane & 31) + 32 * (n >> 2 & 1), kWave);
    const int k = r0 + n;
    const bool use = keep(k);
#pragma unroll
    for (int mb = 0; mb < HD / 32; ++mb)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint2 x = *reinterpret_cast<const uint2*>(tile + k * HD * 2 + 16 * ((4 * mb + c) ^ swz<HD>(k)) + 8 * h);
        const float2 lo = unpack2<T>(x.x), hi = unpack2<T>(x.y);
        const float v[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[mb][4 * c + f] = use ? fmaf(p, v[f], acc[mb][4 * c + f]) : acc[mb][4 * c + f];
      }
  }
}

// Whether an element of acc is NaN, in any lane.
template <int N>
__device__ __forceinline__ bool any_nan(const f32x16 (&acc)[N]) {
  float s[4] = {0.f, 0.f, 0.f, 0.f};  // NaN where a term is
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r & 3] += acc[i][r];
  return __any(__builtin_isnan((s[0] + s[1]) + (s[2] + s[3])));
}

// Writes the columns of acc, times each lane's `mul`, as `n` rows (at most 32) of HD numbers of the type: through BYTES of LDS of the
// wave's own, so that a store writes whole rows (stores straight from the columns write 32 bytes of 32 rows).
template <int HD, CacheType T, int BYTES>
__device__ __forceinline__ void store_rows(char* lds, bf16_t* row, int64_t ld, int n, const f32x16 (&acc)[HD / 32], float mul) {
  constexpr int F = BYTES / 64 < HD ? BYTES / 64 : HD, CH = F / 8, RPI = 64 / CH;  // features at a time, their 16-byte chunks, rows a store
  static_assert(F % 32 == 0, "whole blocks of features");
  const int lane = threadIdx.x & 63, h = lane >> 5, r = lane & 31;
#pragma unroll
  for (int f0 = 0; f0 < HD; f0 += F) {
#pragma unroll
    for (int mb = 0; mb < F / 32; ++mb)
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const f32x16& x = acc[f0 / 32 + mb];
        uint32_t a[2], b[2];  // features 8 i + 4 h .. + 4, and eight on
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          a[e] = pack2<T>(x[4 * i + 2 * e] * mul, x[4 * i + 2 * e + 1] * mul);
          b[e] = pack2<T>(x[4 * i + 4 + 2 * e] * mul, x[4 * i + 5 + 2 * e] * mul);
        }
        // lane half 0 gets features 8 i .. + 8, half 1 those eight on
        const auto u = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
        const auto v = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
        *reinterpret_cast<uint4*>(lds + r * (F * 2) + 16 * ((4 * mb + i + h) ^ (r & (CH - 1)))) = make_uint4(u[0], v[0], u[1], v[1]);
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 32 / RPI; ++k) {
      const int R = k * RPI + lane / CH, c = lane % CH;
      const uint4 x = *reinterpret_cast<const uint4*>(lds + R * (F * 2) + 16 * (c ^ (R & (CH - 1))));
      if (R < n) *reinterpret_cast<uint4*>(row + R * ld + f0 + 8 * c) = x;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ------------------------------------------------------------------ 32 queries of a wave
template <int HD, CacheType T>
struct Queries {
  static constexpr int KS = HD / 16, MB = HD / 32, N = kTile / 32;  // steps of the products with keys, blocks of features, of keys
  typedef f32x16 Scores[N];
  uint4 q[KS];
  f32x16 o[MB];
  float m, l;   // of this lane's query: largest score, this lane's part of the weights' sum
  float scale;  // ScoreScale's

  __device__ __forceinline__ void load(const bf16_t* row, float s) {
    const int h = (threadIdx.x & 63) >> 5;
    const ScoreScale sc(s);
#pragma unroll
    for (int i = 0; i < KS; ++i) q[i] = *reinterpret_cast<const uint4*>(row + 16 * i + 8 * h);
    sc.template turn<T>(q);
    scale = sc.base2;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < MB; ++i) o[i] = zeros16();
  }

  // s = scores of the tile's keys, or of its first `n` times 32
  template <bool PAGES>
  __device__ __forceinline__ void scores(const TileLane<HD, PAGES>& at, const char* k, Scores& s, int n = N) {
#pragma unroll
    for (int t = 0; t < N; ++t) {
      s[t] = zeros16();
      if (t >= n) continue;
#pragma unroll
      for (int i = 0; i < KS; ++i) s[t] = mma32<T>(at.rows(k, 32 * t, i), q[i], s[t]);
    }
  }
  // Scores of keys behind `last` (from the tile's first) count as -inf.
  template <bool PAGES>
  __device__ __forceinline__ void mask(Scores& s, int last) {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (32 * t + (PAGES ? page_row(mma_row(r, h)) : mma_row(r, h)) > last) s[t][r] = -INFINITY;
  }
  // The maximum follows scores that pass it by kSlack, and l and o the maximum.
  __device__ __forceinline__ void follow(const Scores& s) {
    float mx = s[0][0];
#pragma unroll
    for (int r = 1; r < 16 * N; ++r) mx = __builtin_elementwise_maximum(mx, s[r / 16][r % 16]);
    mx = half_max(mx);
    const bool passed = (mx - m) * scale > kSlack || (m == -INFINITY && mx > m);
    if (__any(passed)) {
      const float c = !passed ? 1.f : m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mx) * scale);
      l *= c;
#pragma unroll
      for (int i = 0; i < MB; ++i) o[i] *= c;
      m = passed ? mx : m;
    }
  }
  // s = weights under the maximum
  __device__ __forceinline__ void weigh(Scores& s) {
    const float base = (m == -INFINITY ? 0.f : m * scale) - kHeldExp<T>;
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], scale, -base));
        sum[r & 1] += s[t][r];
      }
    l += sum[0] + sum[1];
  }
  template <bool PAGES>
  __device__ __forceinline__ void add(const TileLane<HD, PAGES>& at, const char* v, const Scores& s, int n = N) {
#pragma unroll
    for (int b = 0; b < 2 * N; ++b) {
      if (b >= 2 * n) continue;
      const f32x16& p = s[b >> 1];
      const int r = 8 * (b & 1);
      // rounded to the type: 2^-9 (2^-12 in half precision) of a weight at most, of either sign, where the output's own rounding
      // is as much of their weighted mean
      const uint4 w = make_uint4(pack2<T>(p[r], p[r + 1]), pack2<T>(p[r + 2], p[r + 3]), pack2<T>(p[r + 4], p[r + 5]),
                                 pack2<T>(p[r + 6], p[r + 7]));
#pragma unroll
      for (int i = 0; i < MB; ++i) o[i] = mma32<T>(at.cols(v, b, i), w, o[i]);
    }
  }
};

// ------------------------------------------------------------------ from a workgroup to its rows
// A wave takes a block of 32 rows of one of `group` heads: a sequence's blocks and heads lie in a line, block by block, of which
// a workgroup takes NW, an item, so that its waves have keys alike, and none idles but for a sequence's last item.  A sequence whose
// bounds descend or lie outside [0, rows] has no items.  Up to kListed * 64 sequences are all looked at by every wave, so that such
// bounds cost the others nothing.  Of more, sequence s has
// items first_item(row_start[s], s) and on, enough of them and none of the next sequence's if the bounds ascend, so that a workgroup
// finds its sequence by a search of row_start; the items in between are empty.
struct SeqItem {
  int row0, len, nth;  // first row and rows of the sequence, the item's place in it from the last one back
};
template <int NW>
__host__ __device__ __forceinline__ long long first_item(int start, int s, int group) {
  return ((long long)(start / 32) + s) * group / NW + s;
}
// Items of a launch: of sequences that share no row never fewer than there are, whatever their order.
template <int NW>
long long seq_items(int rows, int n_seq, int group) { return first_item<NW>(rows, n_seq, group); }
template <int NW>
__device__ __forceinline__ int items_of(int len, int group) {  // 32 bits: prompt_fits
  return (int)(((unsigned)(len + 31) / 32 * (unsigned)group + NW - 1) / NW);
}

// Sum over the lanes up to each, and over all.
__device__ __forceinline__ unsigned wave_upto(unsigned v) {
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);  // the lane 1, 2, 4, 8 before in its 16
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);  // lane 15 to the second 16 (47 to the fourth)
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);  // lane 31 to the second 32
  return v;
}
__device__ __forceinline__ unsigned wave_total(unsigned v) { return (unsigned)__builtin_amdgcn_readlane(wave_upto(v), kWave - 1); }

// Sequences 64 p + lane, p = 0 .. kListed - 1: rows (none of one to be passed over) and items.
constexpr int kListed = 8, kListedSeqs = kListed * kWave;
constexpr int kMostItems = 1 << 25;  // above every item of a launch (prompt_fits): sums of lanes' items, held to it, fit 32 bits
struct SeqList {
  int start[kListed], len[kListed], items[kListed];
};
template <int NW>
__device__ __forceinline__ void list_sequences(const int32_t* row_start, int n_seq, int rows, int group, SeqList& q) {
  auto look = [&](int p) {
    const int s = p * kWave + (threadIdx.x & 63), from = row_start[min(s, n_seq)], to = row_start[min(s + 1, n_seq)];
    const bool usable = s < n_seq && from >= 0 && from < to && to <= rows;
    q.start[p] = from;
    q.len[p] = usable ? to - from : 0;
    q.items[p] = items_of<NW>(q.len[p], group);
  };
  look(0);
#pragma unroll
  for (int p = 1; p < kListed; ++p) q.start[p] = q.len[p] = q.items[p] = 0;
  if (n_seq > kWave) {
#pragma unroll
    for (int p = 1; p < kListed; ++p) look(p);
  }
}

template <int NW>
__device__ __forceinline__ bool find_item(const int32_t* row_start, int n_seq, int rows, int group, int item, SeqItem& t) {
  const int lane = threadIdx.x & 63;
  if (n_seq <= kListedSeqs) {  // items lane by lane
    SeqList q;
    list_sequences<NW>(row_start, n_seq, rows, group, q);
    int mine = q.items[0];
#pragma unroll
    for (int p = 1; p < kListed; ++p) mine = min(mine + q.items[p], kMostItems);
    const unsigned upto = wave_upto(mine);
    const int l = __popcll(__ballot(upto <= (unsigned)item));
    if (l == kWave) return false;
    int left = item - (int)(__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));  // items from the lane's first on
    int start = q.start[0], len = q.len[0], items = __builtin_amdgcn_readlane(q.items[0], l);
    if (n_seq > kWave) {
#pragma unroll
      for (int p = 1; p < kListed; ++p) {
        if (left < items) continue;
        left -= items;
        start = q.start[p];
        len = q.len[p];
        items = __builtin_amdgcn_readlane(q.items[p], l);
      }
    }
    t.row0 = __builtin_amdgcn_readlane(start, l);
    t.len = __builtin_amdgcn_readlane(len, l);
    t.nth = items - 1 - left;  // the longest rows of a sequence first
    return true;
  }
  int lo = 0, n = n_seq, start, end;
  for (;;) {
    const int step = (n + kWave - 1) / kWave, at = min(lo + lane * step, n_seq), v = row_start[at];
    const bool before = lane * step < n && first_item<NW>(min(max(v, 0), rows), at, group) <= item;
    const int found = __popcll(__ballot(before));
    if (found == 0) return false;
    lo += (found - 1) * step;
    n = min(step, n - (found - 1) * step);
    if (step > 1) continue;
    start = __builtin_amdgcn_readlane(v, found - 1);
    end = found < kWave ? __builtin_amdgcn_readlane(v, found) : row_start[min(lo + 1, n_seq)];
    break;
  }
  t.row0 = __builtin_amdgcn_readfirstlane(start);
  end = __builtin_amdgcn_readfirstlane(end);
  if (t.row0 < 0 || end <= t.row0 || end > rows) return false;
  t.len = end - t.row0;
  const int items = items_of<NW>(t.len, group);
  const int nth = item - (int)first_item<NW>(t.row0, __builtin_amdgcn_readfirstlane(lo), group);
  t.nth = items - 1 - nth;
  return nth >= 0 && nth < items;
}

// As find_item, but of up to kListedSeqs sequences the items of all in the order of their length, the longest first, so that no long
// one starts late: an item's place in its sequence says how long it is, and every sequence has one of each length up to its number of
// items.  Costs a workgroup about 1 us: worth it where a workgroup takes many times that.
template <int NW>
__device__ __forceinline__ bool find_sorted(const int32_t* row_start, int n_seq, int rows, int group, int item, SeqItem& t) {
  if (n_seq > kListedSeqs) return find_item<NW>(row_start, n_seq, rows, group, item, t);
  const int lane = threadIdx.x & 63;
  SeqList q;
  list_sequences<NW>(row_start, n_seq, rows, group, q);
  int most = 0;
#pragma unroll
  for (int p = 0; p < kListed; ++p) most = max(most, q.items[p]);
  // items of length w or more
  auto from_length = [&](int w) {
    int n = 0;
#pragma unroll
    for (int p = 0; p < kListed; ++p)
      if (p * kWave < n_seq) n = min(n + max(q.items[p] - w + 1, 0), kMostItems);
    return wave_total(n);
  };
  if (from_length(1) <= (unsigned)item) return false;
  int w = 1, hi = 1;
  while (__any(most >= 2 * hi)) hi *= 2;
  for (int bit = hi; bit > 0; bit /= 2)
    if (from_length(w + bit) > (unsigned)item) w += bit;
  int rank = item - (int)from_length(w + 1);
  bool found = false;
#pragma unroll
  for (int p = 0; p < kListed; ++p) {
    if (p * kWave >= n_seq || found) continue;
    const unsigned long long has = __ballot(q.items[p] >= w);
    if (rank >= __popcll(has)) {
      rank -= __popcll(has);
      continue;
    }
    const bool it = q.items[p] >= w && __popcll(has & ((1ull << lane) - 1)) == rank;
    const int l = __builtin_ctzll(__ballot(it));
    t.row0 = __builtin_amdgcn_readlane(q.start[p], l);
    t.len = __builtin_amdgcn_readlane(q.len[p], l);
    found = true;
  }
  t.nth = w - 1;
  return found;
}

}  // namespace tiles
}  // namespace vla
