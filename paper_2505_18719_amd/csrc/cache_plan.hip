// Pages, rows and cache slots of a step's new tokens from the environments' lengths (vla_kv_plan).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"
#include "common.h"

namespace vla {
namespace {

// a + b, or 2^32 - 1 where that is more: what is asked for beyond that has no room in any case.
__device__ __forceinline__ unsigned add_sat(unsigned a, unsigned b) { return __builtin_elementwise_add_sat(a, b); }

// Sum over this lane and those before it, 4 steps within 16 lanes and 2 across them.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned scan_step(unsigned v) {
  return add_sat(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ unsigned wave_scan(unsigned v) {
  v = scan_step<0x111, 0xF>(v);
  v = scan_step<0x112, 0xF>(v);
  v = scan_step<0x114, 0xF>(v);
  v = scan_step<0x118, 0xF>(v);
  v = scan_step<0x142, 0xA>(v);
  return scan_step<0x143, 0xC>(v);
}
// Sum over this thread of the workgroup and those before it; `total` receives that over all.
template <int W>
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned (&sums)[W], unsigned& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_scan(v);
  if (lane == 63) sums[w] = v;
  __syncthreads();
  total = 0;
  unsigned before = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if (i < w) before = add_sat(before, sums[i]);
    total = add_sat(total, sums[i]);
  }
  return add_sat(v, before);
}

// One launch: every workgroup adds up the lengths of the environments up to its own rows, in tiles of one environment per
// thread (the lengths are a few KB that the caches hold; a second launch and the way of the sums through memory would cost
// more), and looks its rows' environments up in the tile.  Workgroup 0 goes through all tiles and writes what belongs to
// environments.  A new page's table entry is written by the row at its first slot, which is always a new row; rows read only
// entries of pages that were there before, so no workgroup reads what another writes.  Bound: the latency of three dependent
// loads and five barriers (64 environments 3.5 us, 256 environments with 130000 rows 5.6 us).
template <int NT>
__global__ __launch_bounds__(NT) void kv_plan_kernel(KvPlanArgs a, int rows_per_wg) {
  constexpr int W = NT / kWave;
  __shared__ unsigned sums[2][W];
  __shared__ int s_start[NT];   // first row of the tile's environments
  __shared__ int s_cached[NT];
  __shared__ int s_page[NT];    // index into free_pages of the first new page, or -1: refused
  __shared__ int s_refused[W];
  __shared__ unsigned s_taken[W];
  const int tid = threadIdx.x;
  const unsigned max_rows = a.max_rows, r0 = min((long long)max_rows, (long long)blockIdx.x * rows_per_wg), r1 = min((long long)max_rows, (long long)r0 + rows_per_wg);
  const bool first = blockIdx.x == 0;
  const int head = a.free_head ? *a.free_head : 0;
  const unsigned avail = head >= 0 && head <= a.n_free ? a.n_free - head : 0;
  unsigned row = 0, page = 0, taken = 0;  // rows and pages asked for before the tile; pages given out
  int refused = 0;
  const unsigned n_env = a.n_env;  // the last tile may end past 2^31 - 1
  for (unsigned t0 = 0; t0 < n_env; t0 += NT) {
    if (!first && row >= r1) break;
    const unsigned e = t0 + tid;
    const bool in = e < n_env;
    const int c = in ? a.cached[e] : 0, w = in ? a.added[e] : 0;
    unsigned tile_rows, tile_pages;
    const unsigned rows = max(w, 0), end = add_sat(row, block_scan<W>(rows, sums[0], tile_rows));
    const unsigned start = end == ~0u ? max_rows : end - rows;  // past the last row where the sum has no room
    const bool fits = in && c >= 0 && w >= 0 && (long long)c + w <= (long long)a.max_pages * kPage && end <= max_rows;
    const int held = (int)(((long long)c + kPage - 1) / kPage);
    const unsigned need = fits ? (int)(((long long)c + w + kPage - 1) / kPage) - held : 0;
    const unsigned upto = add_sat(page, block_scan<W>(need, sums[1], tile_pages));
    const bool ok = fits && (need == 0 || upto <= avail);
    s_start[tid] = min(start, max_rows);
    s_cached[tid] = c;
    s_page[tid] = ok ? (need ? head + (int)(upto - need) : 0) : -1;
    if (first && in) {
      a.lens[e] = ok ? c + w : max(c, 0);
      a.row_start[e] = min(start, max_rows);
      if (ok && need > 0) taken = max(taken, upto);
      refused += !ok;
    }
    __syncthreads();
    const unsigned lo = max(r0, row), hi = min(r1, add_sat(row, tile_rows));
    for (unsigned r = lo + tid; r < hi; r += NT) {
      int i = 0;  // last environment of the tile whose rows start at or before r (one without rows ends where it starts)
#pragma unroll
      for (int step = NT / 2; step > 0; step >>= 1)
        if ((unsigned)s_start[i + step] <= r) i += step;
      const long long pos = (long long)s_cached[i] + (r - (unsigned)s_start[i]);
      int slot = -1;
      if (s_page[i] >= 0) {
        int32_t* entry = a.page_table + (long long)(t0 + i) * a.ld_table + pos / kPage;
        const int fresh = (int)(pos / kPage) - (s_cached[i] + kPage - 1) / kPage;
        const int p = fresh >= 0 ? a.free_pages[s_page[i] + fresh] : *entry;
        if (fresh >= 0 && pos % kPage == 0) *entry = p;
        if (p >= 0 && p < a.n_pages) slot = p * kPage + (int)(pos % kPage);
      }
      a.row_pos[r] = (int)min(max(pos, 0ll), 0x7fffffffll);
      a.row_env[r] = (int)(t0 + i);
      a.row_slot[r] = slot;
    }
    row = add_sat(row, tile_rows);
    page = add_sat(page, tile_pages);
    __syncthreads();  // the tile's arrays and sums are free again
  }
  const unsigned rows = min(row, max_rows);
  // a workgroup that left the loop early has all its rows below `row`
  for (unsigned r = max(r0, rows) + tid; r < r1; r += NT) {
    a.row_pos[r] = 0;
    a.row_env[r] = -1;
    a.row_slot[r] = -1;
  }
  if (!first) return;
  // pages given out are those of a first run of environments: the largest running count of one that got its pages
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    taken = max(taken, (unsigned)__shfl_xor((int)taken, o, kWave));
    refused += __shfl_xor(refused, o, kWave);
  }
  if ((tid & 63) == 0) {
    s_taken[tid >> 6] = taken;
    s_refused[tid >> 6] = refused;
  }
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < W; ++i) {
      taken = max(taken, s_taken[i]);
      refused += s_refused[i];
    }
    a.row_start[a.n_env] = rows;
    a.stats[0] = head + (int)taken;
    a.stats[1] = rows;
    a.stats[2] = refused;
  }
}

template <int NT>
void launch_plan(const KvPlanArgs& a, hipStream_t s) {
  constexpr int kRows = 1024, kMaxGroups = 512;  // rows of a workgroup at least; workgroups at most
  const int per = kRows * std::max(1, (a.max_rows - 1) / (kRows * kMaxGroups) + 1);
  const int groups = a.max_rows > 0 ? (a.max_rows - 1) / per + 1 : 1;
  hipLaunchKernelGGL(kv_plan_kernel<NT>, dim3(groups), dim3(NT), 0, s, a, per);
}

}  // namespace

hipError_t launch_kv_plan(const KvPlanArgs& a, hipStream_t s) {
  // a tile of 256 environments has fewer waves to wait for than one of 1024, but more than one tile costs more than they
  if (a.n_env <= 256) launch_plan<256>(a, s);
  else launch_plan<1024>(a, s);
  return hipGetLastError();
}

}  // namespace vla
