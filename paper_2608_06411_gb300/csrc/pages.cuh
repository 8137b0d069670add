// Shared by the bookkeeping calls on a cache's pages (cache.cu, evict.cu): one CTA does a whole call's.
#pragma once
#include "handoff.h"

namespace mapk {

constexpr int kMaxSeqs = 262144;

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMaxEntries = 4096;
constexpr int kMaxFree = 1 << 20;

// Exclusive prefix sums of v over the block, and their total (every thread gets it).
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  if (lane == 31) warp_sums[warp] = s;
  __syncthreads();
  int w = warp_sums[lane];                 // every warp scans the 32 sums for itself
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += u;
  }
  __syncthreads();
  *total = __shfl_sync(0xffffffffu, w, 31);
  const int before = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
  return (warp > 0 ? before : 0) + s - v;
}

// Last i in [0, n) with start[i] <= x (start ascending, start[0] = 0).
__device__ __forceinline__ int entry_of(const int* start, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// The total lowest free pages, each with one holder: the r-th into *entry(r).  False, and all counts as they were, if there are
// fewer.  The first pages' counts are read ahead of the entries (HeadCounts): most calls need no others.
constexpr int kPagesEach = 4;              // neighbouring pages a thread looks at
struct HeadCounts {
  int v[kPagesEach];
  __device__ __forceinline__ void load(const map_cache& c, int p) {
#pragma unroll
    for (int k = 0; k < kPagesEach; ++k) v[k] = p + k < c.pages ? c.refs[p + k] : 1;
  }
};
template <typename Entry>
__device__ __forceinline__ bool take_pages(const map_cache& c, int total, HeadCounts& counts, int* warp_sums, const Entry& entry) {
  int found = 0;
  for (int p0 = 0; p0 < c.pages && found < total; p0 += kPlanThreads * kPagesEach) {
    const int p = p0 + threadIdx.x * kPagesEach;
    int mine = 0, got;
    if (p0 > 0) counts.load(c, p);
#pragma unroll
    for (int k = 0; k < kPagesEach; ++k) mine += counts.v[k] == 0;
    int r = found + block_scan(mine, warp_sums, &got);
#pragma unroll
    for (int k = 0; k < kPagesEach; ++k)
      if (counts.v[k] == 0) {
        if (r < total) {
          *entry(r) = p + k;
          c.refs[p + k] = 1;
        }
        ++r;
      }
    found += got;
  }
  __syncthreads();
  if (found >= total) return true;
  for (int r = threadIdx.x; r < found; r += kPlanThreads) c.refs[*entry(r)] = 0;
  return false;
}

// The same into the table: need r of entry i (start[i] <= r < start[i + 1]) is column col[i] + r - start[i] of row seq[i].
__device__ bool take_pages(const map_cache& c, const int* start, const int* col, const int* seq, int n, int total,
                           HeadCounts& counts, int* warp_sums) {
  return take_pages(c, total, counts, warp_sums, [&](int r) {
    const int i = entry_of(start, n, r);
    return c.table + static_cast<long long>(seq[i]) * c.max_pages + col[i] + r - start[i];
  });
}

// Shared memory of a bookkeeping call (extend_kernel's; fork_plan_kernel takes a word less): five words an entry, a bit a
// sequence.
constexpr size_t plan_smem(size_t n, size_t seqs) { return (5 * n + 2 + (seqs + 31) / 32) * 4; }

// The limit belongs to all threads of the process: every call that needs one sets the same, the largest, so that none lowers it
// between another's setting and its launch.  What a kernel has without asking, 48 KB, holds its fixed words too.
cudaError_t allow_smem(const void* kern, size_t bytes) {
  constexpr size_t fixed = 256;            // warp_sums and error are 132
  if (bytes + fixed <= 48 * 1024) return cudaSuccess;
  return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(plan_smem(kMaxEntries, kMaxSeqs)));
}

}  // namespace
}  // namespace mapk
