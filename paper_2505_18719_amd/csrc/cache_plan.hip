// Pages, rows and cache slots of a step's new tokens from the environments' lengths (vla_kv_plan).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"
#include "common.h"

namespace vla {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;

__device__ __forceinline__ long long wave_scan(long long v, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const long long u = __shfl_up(v, o, kWave);
    if (lane >= o) v += u;
  }
  return v;
}

// Inclusive scan over the workgroup; `total` receives the sum.
__device__ __forceinline__ long long block_scan(long long v, long long (&sums)[kPlanWaves], long long& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_scan(v, lane);
  if (lane == 63) sums[w] = v;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kPlanWaves; ++i) {
    const long long s = sums[i];
    if (i < w) before += s;
    all += s;
  }
  total = all;
  return v + before;
}

// One launch: every workgroup scans the lengths of the environments up to its own rows, in tiles of one environment per
// thread (the lengths are a few KB that the caches hold; a second launch and the way of the sums through memory would
// cost more), and looks its rows' environments up in the tile.  Workgroup 0 goes through all tiles and writes what
// belongs to environments.  A new page's table entry is written by the row at its first slot, which is always a new row;
// rows read only entries of pages that were there before, so no workgroup reads what another writes.
__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(KvPlanArgs a, int rows_per_wg) {
  __shared__ long long sums[2][kPlanWaves];
  __shared__ int s_start[kPlanThreads + 1];  // first row of the tile's environments, and the row after the last
  __shared__ int s_cached[kPlanThreads];
  __shared__ long long s_page[kPlanThreads];  // index into free_pages of the first new page, or -1: refused
  const int tid = threadIdx.x;
  const long long r0 = (long long)blockIdx.x * rows_per_wg, r1 = min((long long)a.max_rows, r0 + rows_per_wg);
  const bool first = blockIdx.x == 0;
  const long long head = a.free_head ? *a.free_head : 0;
  const long long avail = head >= 0 && head <= a.n_free ? a.n_free - head : 0;
  long long row = 0, page = 0, taken = 0;  // rows and pages asked for before the tile; pages given out
  int refused = 0;
  for (int t0 = 0; t0 < a.n_env; t0 += kPlanThreads) {
    if (!first && row >= r1) break;
    const int e = t0 + tid;
    const bool in = e < a.n_env;
    const long long c = in ? a.cached[e] : 0, w = in ? a.added[e] : 0;
    long long tile_rows, tile_pages;
    const long long end = row + block_scan(max(w, 0ll), sums[0], tile_rows);
    const bool fits = in && c >= 0 && w >= 0 && c + w <= (long long)a.max_pages * kPage && end <= a.max_rows;
    const long long need = fits ? (c + w + kPage - 1) / kPage - (c + kPage - 1) / kPage : 0;
    const long long upto = page + block_scan(need, sums[1], tile_pages);
    const bool ok = fits && (need == 0 || upto <= avail);
    const long long start = end - max(w, 0ll);
    s_start[tid] = (int)min(start, (long long)a.max_rows);
    if (tid == kPlanThreads - 1) s_start[kPlanThreads] = (int)min(end, (long long)a.max_rows);
    s_cached[tid] = (int)c;
    s_page[tid] = ok ? head + upto - need : -1;
    if (first && in) {
      a.lens[e] = (int)(ok ? c + w : max(c, 0ll));
      a.row_start[e] = (int)min(start, (long long)a.max_rows);
      if (ok && need > 0) taken = max(taken, upto);
      refused += !ok;
    }
    __syncthreads();
    const long long lo = max(r0, row), hi = min(r1, row + tile_rows);
    for (long long r = lo + tid; r < hi; r += kPlanThreads) {
      int i = 0;  // last environment of the tile whose rows start at or before r (one without rows ends where it starts)
#pragma unroll
      for (int step = kPlanThreads / 2; step > 0; step >>= 1)
        if (s_start[i + step] <= r) i += step;
      const long long pos = (long long)s_cached[i] + (r - s_start[i]);
      int slot = -1;
      if (s_page[i] >= 0) {
        const int32_t* entry = a.page_table + (long long)(t0 + i) * a.ld_table + pos / kPage;
        const long long fresh = pos / kPage - (s_cached[i] + kPage - 1) / kPage;
        const int p = fresh >= 0 ? a.free_pages[s_page[i] + fresh] : *entry;
        if (fresh >= 0 && pos % kPage == 0) *const_cast<int32_t*>(entry) = p;
        if (p >= 0 && p < a.n_pages) slot = p * kPage + (int)(pos % kPage);
      }
      a.row_pos[r] = (int)min(max(pos, 0ll), 0x7fffffffll);
      a.row_env[r] = t0 + i;
      a.row_slot[r] = slot;
    }
    row += tile_rows;
    page += tile_pages;
    __syncthreads();  // the tile's arrays and sums are free again
  }
  const int rows = (int)min(row, (long long)a.max_rows);
  // a workgroup that left the loop early has all its rows below `row`
  for (long long r = max(r0, (long long)rows) + tid; r < r1; r += kPlanThreads) {
    a.row_pos[r] = 0;
    a.row_env[r] = -1;
    a.row_slot[r] = -1;
  }
  if (!first) return;
  // pages given out are those of a first run of environments: the largest running count of one that got its pages
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    taken = max(taken, (long long)__shfl_xor(taken, o, kWave));
    refused += __shfl_xor(refused, o, kWave);
  }
  if ((tid & 63) == 0) {
    sums[0][tid >> 6] = taken;
    sums[1][tid >> 6] = refused;
  }
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < kPlanWaves; ++i) {
      taken = max(taken, sums[0][i]);
      refused += (int)sums[1][i];
    }
    a.row_start[a.n_env] = rows;
    a.stats[0] = (int)(head + taken);
    a.stats[1] = rows;
    a.stats[2] = refused;
  }
}

}  // namespace

hipError_t launch_kv_plan(const KvPlanArgs& a, hipStream_t s) {
  constexpr int kMaxGroups = 512;
  const int per = kPlanThreads * std::max(1, (a.max_rows - 1) / (kPlanThreads * kMaxGroups) + 1);
  const int groups = a.max_rows > 0 ? (a.max_rows - 1) / per + 1 : 1;
  hipLaunchKernelGGL(kv_plan_kernel, dim3(groups), dim3(kPlanThreads), 0, s, a, per);
  return hipGetLastError();
}

}  // namespace vla
