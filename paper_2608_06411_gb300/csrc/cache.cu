// Pages of a language model's key/value cache: rows appended (map_cache_extend), sequences forked whole or with the
// kept visual tokens of a question (map_cache_fork), and freed (map_cache_free).
//
// Bookkeeping runs on the device, so that a kept set or a count computed there needs no trip to the host and
// every call can be captured.  One CTA does it for a whole call: the entries' needs are added up in shared memory, the
// free pages are those with a reference count of zero, and the r-th lowest of them goes to the r-th need.  Nothing but
// the counts says what is free, so results follow from the state alone, and a fork that is freed leaves it as it was.
// A call is checked whole before it changes a length; until then it writes only table entries past a length, and counts
// that it puts back where the pages do not suffice.
// A bookkeeping call is a chain of loads that depend on one another (entries, lengths, counts, table: about 0.7 us each),
// so entries are read once, all together, and nothing that is known is read back.
#include "handoff.h"

namespace mapk {

static constexpr int kMaxSeqs = 262144;

int check_cache(const map_cache* c) {
  if (!c || !c->pool || !c->table || !c->len || !c->refs || !c->status) return MAP_EINVAL;
  if (c->type != MAP_BF16 && c->type != MAP_F16) return MAP_EINVAL;
  if (c->layers < 1 || c->pages < 1 || c->heads < 1 || c->page < 1 || c->dh < 1 || c->seqs < 1 || c->max_pages < 1)
    return MAP_EINVAL;
  if (!aligned16(c->pool)) return MAP_EINVAL;
  if (c->dh % 8 || c->dh > kMaxHead || c->page > 1024 || c->seqs > kMaxSeqs) return MAP_EUNSUPPORTED;
  if (c->pages > (1 << 20)) return MAP_EUNSUPPORTED;            // block_scan adds 1024 needs of at most so many pages
  if (static_cast<long long>(c->max_pages) * c->page >= (1ll << 31)) return MAP_EUNSUPPORTED;
  if (c->heads > 65535 || 2ll * c->layers * c->heads > (1 << 24)) return MAP_EUNSUPPORTED;      // units of a page: 32 bits
  return MAP_OK;
}

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMaxEntries = 4096;
constexpr int kMaxFree = 1 << 20;

// What a fork makes of a parent: rows kept as they are, shared whole pages, length.
struct ForkShape { int base, span, k, shared, len; };
__device__ __forceinline__ ForkShape fork_shape(int parent_len, int page, bool kept, int base, int span, int k) {
  if (!kept) return {parent_len, 0, 0, parent_len / page, parent_len};
  return {base, span, k, base / page, parent_len - span + k};
}

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

// The total lowest free pages into the table, each with one holder: need r of entry i (start[i] <= r < start[i + 1]) is
// column col[i] + r - start[i] of row seq[i].  False, and all counts as they were, if there are fewer.
// The first pages' counts are read ahead of the entries (HeadCounts): most calls need no others.
constexpr int kPagesEach = 4;              // neighbouring pages a thread looks at
struct HeadCounts {
  int v[kPagesEach];
  __device__ __forceinline__ void load(const map_cache& c, int p) {
#pragma unroll
    for (int k = 0; k < kPagesEach; ++k) v[k] = p + k < c.pages ? c.refs[p + k] : 1;
  }
};
__device__ bool take_pages(const map_cache& c, const int* start, const int* col, const int* seq, int n, int total,
                           HeadCounts& counts, int* warp_sums) {
  const auto entry = [&](int r) {
    const int i = entry_of(start, n, r);
    return c.table + static_cast<long long>(seq[i]) * c.max_pages + col[i] + r - start[i];
  };
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

// counts[i] more rows for sequence seqs[i], and their slots.  Without counts entry i has row i, padding or not.  Latency-bound
// (a few KB): one CTA, since every entry's pages depend on the needs of those before it.  16 entries of 200 rows and the call
// that frees them take 8.5 us one after the other, 64 decoding rows and theirs 7.0 (with 512 threads 10.2 and 8.1).
__global__ void __launch_bounds__(kPlanThreads) extend_kernel(const map_cache c, const int32_t* __restrict__ seqs,
                                                              const int32_t* __restrict__ counts, int n, int rows,
                                                              int32_t* __restrict__ slots) {
  extern __shared__ int sh[];
  int* start = sh;                         // [n + 1] pages needed before entry i
  int* row0 = start + n + 1;               // [n + 1] rows before entry i
  int* col = row0 + n + 1;                 // [n] first new page
  int* seq = col + n;                      // [n]
  int* old = seq + n;                      // [n] length before, -1: padding
  unsigned* seen = reinterpret_cast<unsigned*>(old + n);   // bitmap of the sequences
  __shared__ int warp_sums[kPlanThreads / 32];
  __shared__ int error;
  pdl_enter();
  for (int i = threadIdx.x; i < (c.seqs + 31) / 32; i += kPlanThreads) seen[i] = 0;
  if (threadIdx.x == 0) error = 0;
  HeadCounts head;
  head.load(c, threadIdx.x * kPagesEach);
  __syncthreads();
  int pages0 = 0, rows0 = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int need = 0, add = 0;
    if (i < n) {
      const int s = seqs[i];
      seq[i] = col[i] = 0;
      old[i] = -1;
      add = counts ? (s == -1 ? 0 : counts[i]) : 1;
      if (s != -1) {
        if (s < 0 || s >= c.seqs || add < 0 || add > rows ||
            (atomicOr(&seen[s >> 5], 1u << (s & 31)) >> (s & 31) & 1u)) {
          atomicOr(&error, ST_BADINDEX);
          add = 0;
        } else {
          const int len = c.len[s];
          const unsigned pages = (static_cast<unsigned>(len) + add + c.page - 1) / c.page;     // below 2^31 + 2^20 + 2^10 rows
          if (!good_len(c, len)) {
            atomicOr(&error, ST_BADINDEX);
            add = 0;
          } else if (pages > static_cast<unsigned>(c.max_pages)) {
            atomicOr(&error, ST_NOPAGES);
            add = 0;
          } else {
            seq[i] = s;
            old[i] = len;
            col[i] = pieces_of(len, c.page);
            need = static_cast<int>(pages) - col[i];
          }
        }
      }
    }
    int all;
    const int rs = rows0 + block_scan(add, warp_sums, &all);
    if (i < n) row0[i] = rs;
    rows0 += all;                          // 1024 counts of at most 2^20 rows
    const int ps = pages0 + block_scan(need, warp_sums, &all);
    if (i < n) start[i] = ps;
    pages0 += all;
    if (rows0 > rows) {
      if (threadIdx.x == 0) atomicOr(&error, ST_BADINDEX);
      rows0 = pages0 = 0;
    }
  }
  if (threadIdx.x == 0) { start[n] = pages0; row0[n] = rows0; }
  __syncthreads();
  const bool ok = error == 0;
  const bool enough = ok && take_pages(c, start, col, seq, n, pages0, head, warp_sums);
  if (!enough) {
    if (threadIdx.x == 0) atomicOr(c.status, ok ? ST_NOPAGES : error);
    for (int r = threadIdx.x; r < rows; r += kPlanThreads) slots[r] = -1;
    return;
  }
  for (int i = threadIdx.x; i < n; i += kPlanThreads)
    if (old[i] >= 0) c.len[seq[i]] = old[i] + row0[i + 1] - row0[i];
  constexpr int kEach = 4;                 // table entries a thread reads at once
  for (int r0 = threadIdx.x; r0 < rows; r0 += kEach * kPlanThreads) {
    int page[kEach], in_page[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int r = r0 + k * kPlanThreads;
      page[k] = -1;
      if (r < rows0) {
        const int i = entry_of(row0, n, r), t = old[i] + r - row0[i];
        in_page[k] = t % c.page;
        if (old[i] >= 0) page[k] = c.table[static_cast<long long>(seq[i]) * c.max_pages + t / c.page];
        if (old[i] >= 0 && !good_page(c, page[k])) {
          atomicOr(c.status, ST_BADINDEX);
          page[k] = -1;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k)
      if (r0 + k * kPlanThreads < rows) slots[r0 + k * kPlanThreads] = page[k] < 0 ? -1 : page[k] * c.page + in_page[k];
  }
}

// Tables, counts and lengths of the children.  status[1]: whether fork_copy_kernel is to copy.  Latency-bound like
// extend_kernel, and one CTA for the same reason: of the 64 us of 8 questions' forks on a cached image and their free call the
// copy takes 53 to 55.
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(const map_cache c, const int32_t* __restrict__ parents,
                                                                 const int32_t* __restrict__ children, int n, int kept,
                                                                 int k, const int32_t* __restrict__ base,
                                                                 const int32_t* __restrict__ span) {
  extern __shared__ int sh[];
  int* start = sh;                         // [n + 1] pages needed before entry i
  int* col = start + n + 1;                // [n] pages shared with the parent
  int* seq = col + n;                      // [n] child
  int* len = seq + n;                      // [n] its length
  int* par = len + n;                      // [n]
  unsigned* seen = reinterpret_cast<unsigned*>(par + n);
  __shared__ int warp_sums[kPlanThreads / 32];
  __shared__ int error;
  pdl_enter();
  for (int i = threadIdx.x; i < (c.seqs + 31) / 32; i += kPlanThreads) seen[i] = 0;
  if (threadIdx.x == 0) error = 0;
  HeadCounts head;
  head.load(c, threadIdx.x * kPagesEach);
  __syncthreads();
  int pages0 = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int need = 0;
    if (i < n) {
      const int p = parents[i], s = children[i];
      par[i] = seq[i] = col[i] = len[i] = 0;
      if (p < 0 || p >= c.seqs || s < 0 || s >= c.seqs || c.len[s] != 0 ||
          (atomicOr(&seen[s >> 5], 1u << (s & 31)) >> (s & 31) & 1u)) {
        atomicOr(&error, ST_BADINDEX);
      } else {
        const int plen = c.len[p], b = kept ? base[i] : 0, sp = kept ? span[i] : 0;
        if (!good_len(c, plen) || b < 0 || sp < 0 || static_cast<long long>(b) + sp > plen) {
          atomicOr(&error, ST_BADINDEX);
        } else {
          // a child longer than its parent (keep may repeat rows) can pass its table row, or 2^31
          // (needs beyond the pool are refused here: 1024 of them could pass 2^31 in their sum)
          const unsigned pages = (static_cast<unsigned>(plen) - sp + (kept ? k : 0) + c.page - 1) / c.page;   // below 2^32 rows
          const ForkShape f = fork_shape(plen, c.page, kept, b, sp, k);
          if (pages > static_cast<unsigned>(c.max_pages) || static_cast<int>(pages) - f.shared > c.pages) {
            atomicOr(&error, ST_NOPAGES);
          } else {
            par[i] = p;
            seq[i] = s;
            col[i] = f.shared;
            len[i] = f.len;
            need = static_cast<int>(pages) - f.shared;
          }
        }
      }
    }
    int all;
    const int ps = pages0 + block_scan(need, warp_sums, &all);
    if (i < n) start[i] = ps;
    pages0 += all;
    if (pages0 > c.pages) {                // more than there are: no sum past this one
      if (threadIdx.x == 0) atomicOr(&error, ST_NOPAGES);
      pages0 = 0;
    }
  }
  if (threadIdx.x == 0) start[n] = pages0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlanThreads)       // no child may be a parent
    if (seen[par[i] >> 5] >> (par[i] & 31) & 1u && error == 0) atomicOr(&error, ST_BADINDEX);
  __syncthreads();
  const bool ok = error == 0;
  const bool enough = ok && take_pages(c, start, col, seq, n, pages0, head, warp_sums);
  if (threadIdx.x == 0) {
    c.status[1] = enough;
    if (!enough) atomicOr(c.status, ok ? ST_NOPAGES : error);
  }
  if (!enough) return;
  for (int i = threadIdx.x >> 5; i < n; i += kPlanThreads / 32) {        // a warp an entry
    const int32_t* from = c.table + static_cast<long long>(par[i]) * c.max_pages;
    int32_t* to = c.table + static_cast<long long>(seq[i]) * c.max_pages;
    for (int j = threadIdx.x & 31; j < col[i]; j += 32) {
      const int page = from[j];
      to[j] = page;
      if (good_page(c, page)) atomicAdd(&c.refs[page], 1);
      else atomicOr(c.status, ST_BADINDEX);
    }
    if ((threadIdx.x & 31) == 0) c.len[seq[i]] = len[i];
  }
}

// The rows of the children's own pages, each read once and written once in every plane (K or V of a layer).  A unit is one
// head of one new page in one plane, a slab of page * dh elements; a block takes an equal run of the units, page by page, so
// that it looks a page's source rows up once.  Full occupancy with one vector a thread in flight: 53 us for 8 questions on an
// image in 32 layers, 171 MB copied (two in flight 56, four with six CTAs an SM 60).  Of those 342 MB DRAM sees 261 in that
// time, 4.7 TB/s, 0.7 of what a copy reaches: each row is 256 bytes at a place of its own, and rows that several children keep
// (32 of the 171 MB) are read by each, page by page of one child, mostly from L2.
// What comes before griddepcontrol.wait (shapes, the parents' tables) fork_plan_kernel only reads, and so runs beside it.
constexpr int kCopyThreads = 256, kCopyGrid = 152 * 8;
__global__ void __launch_bounds__(kCopyThreads, 8) fork_copy_kernel(const map_cache c, const int32_t* __restrict__ parents,
                                                                    const int32_t* __restrict__ children, int n,
                                                                    const int32_t* __restrict__ keep, int k,
                                                                    const int32_t* __restrict__ base,
                                                                    const int32_t* __restrict__ span) {
  extern __shared__ int sh[];
  int* start = sh;                         // [n + 1] new pages before entry i
  int* from = sh + n + 1;                  // [page] source slot of each row: -1 none, -2 a bad index
  __shared__ int warp_sums[kCopyThreads / 32];
  const bool kept = base != nullptr;
  const auto shape = [&](int i) {
    const int p = parents[i], plen = p >= 0 && p < c.seqs && good_len(c, c.len[p]) ? c.len[p] : 0;
    return fork_shape(plen, c.page, kept, kept ? base[i] : 0, kept ? span[i] : 0, k);
  };
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // a thread counts a run of the entries (a refused call may have any numbers here: nothing is copied for it)
  const int each = (n + kCopyThreads - 1) / kCopyThreads, e0 = threadIdx.x * each, e1 = min(n, e0 + each);
  int mine = 0;
  for (int i = e0; i < e1; ++i) {
    const ForkShape f = shape(i);
    start[i] = mine;
    mine += max(0, pieces_of(f.len, c.page) - f.shared);
  }
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, incl, o);
    if ((threadIdx.x & 31) >= o) incl += u;
  }
  if ((threadIdx.x & 31) == 31) warp_sums[threadIdx.x >> 5] = incl;
  __syncthreads();
  int before = incl - mine;
  for (int w = 0; w < static_cast<int>(threadIdx.x >> 5); ++w) before += warp_sums[w];
  for (int i = e0; i < e1; ++i) start[i] += before;
  if (threadIdx.x == kCopyThreads - 1) start[n] = before + mine;
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (c.status[1] == 0) return;

  const int vec = c.dh / 8, slab = c.page * vec, of_page = 2 * c.layers * c.heads;
  const long long units = static_cast<long long>(start[n]) * of_page, plane = static_cast<long long>(c.pages) * c.heads * slab;
  const long long u1 = units * (blockIdx.x + 1) / gridDim.x;
  uint4* pool = static_cast<uint4*>(c.pool);
  // threads beyond a slab take further units
  const int lanes = min(slab, kCopyThreads), subs = kCopyThreads / lanes, sub = threadIdx.x / lanes;
  for (long long u = units * blockIdx.x / gridDim.x; u < u1;) {
    const int r = static_cast<int>(u / of_page), a0 = static_cast<int>(u % of_page);
    const int a1 = static_cast<int>(min(static_cast<long long>(of_page), a0 + u1 - u)), i = entry_of(start, n, r);
    const int32_t* ptab = c.table + static_cast<long long>(parents[i]) * c.max_pages;
    const ForkShape f = shape(i);
    const int colm = f.shared + r - start[i];
    const int to_page = c.table[static_cast<long long>(children[i]) * c.max_pages + colm];
    __syncthreads();
    for (int t = threadIdx.x; t < c.page; t += kCopyThreads) {
      const int j = colm * c.page + t;
      int src = j;
      bool bad = false;
      if (j >= f.base && kept) {
        if (j < f.base + k) {
          const int x = keep[static_cast<long long>(i) * k + j - f.base];
          bad = x < 0 || x >= f.span;
          src = f.base + x;
        } else {
          src = j - k + f.span;
        }
      }
      const int page = j < f.len && !bad ? ptab[src / c.page] : 0;
      bad = bad || !good_page(c, page);
      if (j >= f.len) from[t] = -1;
      else if (bad) { from[t] = -2; atomicOr(c.status, ST_BADINDEX); }
      else from[t] = page * c.page + src % c.page;
    }
    __syncthreads();
    if (sub < subs) {
      for (int e = threadIdx.x % lanes; e < slab; e += lanes) {
        const int t = e / vec, s = from[t];
        if (s == -1) continue;
        const uint4* src = pool + static_cast<long long>(s < 0 ? 0 : s / c.page) * c.heads * slab + (s < 0 ? 0 : s % c.page * vec + e % vec);
        uint4* dst = pool + static_cast<long long>(to_page) * c.heads * slab + e;
        // unit b = (plane b / heads, head b % heads) lies `at` past the first
        int h = (a0 + sub) % c.heads;
        long long at = (a0 + sub) / c.heads * plane + h * slab;
        for (int b = a0 + sub; b < a1; b += subs) {
          dst[at] = s < 0 ? make_uint4(0, 0, 0, 0) : src[at];
          at += subs * slab;
          for (h += subs; h >= c.heads; h -= c.heads) at += plane - c.heads * slab;
        }
      }
    }
    u += a1 - a0;
  }
}

// A warp a sequence; the first to take its length frees its pages.  Latency-bound: three loads that depend on one another,
// 5 us by itself with cold caches, 1.2 behind another call.
__global__ void __launch_bounds__(256) free_kernel(const map_cache c, const int32_t* __restrict__ seqs, int n) {
  pdl_enter();
  const int i = (blockIdx.x * 256 + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  if (i >= n) return;
  const int s = seqs[i];
  if (s < 0 || s >= c.seqs) {
    if (s != -1 && lane == 0) atomicOr(c.status, ST_BADINDEX);
    return;
  }
  int len = lane == 0 ? atomicExch(&c.len[s], 0) : 0;
  len = __shfl_sync(0xffffffffu, len, 0);
  if (!good_len(c, len)) {                 // as it was: the sequence is not empty (another entry that names it finds the same, or 0)
    if (lane == 0) {
      atomicExch(&c.len[s], len);
      atomicOr(c.status, ST_BADINDEX);
    }
    return;
  }
  const int32_t* row = c.table + static_cast<long long>(s) * c.max_pages;
  for (int j = lane; j < pieces_of(len, c.page); j += 32) {
    const int page = row[j];
    if (good_page(c, page)) atomicSub(&c.refs[page], 1);
    else atomicOr(c.status, ST_BADINDEX);
  }
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

int launch_err(cudaError_t e) {
  if (e == cudaSuccess) return MAP_OK;
  cudaGetLastError();
  return MAP_ECUDA;
}

}  // namespace
}  // namespace mapk

using namespace mapk;

extern "C" {

int map_cache_extend(const map_cache* c, const int32_t* seqs, const int32_t* counts, int n, long long rows,
                     int32_t* slots, void* stream) {
  const int rc = check_cache(c);
  if (rc != MAP_OK) return rc;
  if (n < 0 || rows < 0 || (n > 0 && !seqs) || (rows > 0 && !slots)) return MAP_EINVAL;
  if (n > kMaxEntries || rows > (1 << 20)) return MAP_EUNSUPPORTED;
  if (n == 0 && rows == 0) return MAP_OK;
  const size_t smem = plan_smem(n, c->seqs);
  cudaError_t e = allow_smem(reinterpret_cast<const void*>(extend_kernel), smem);
  if (e == cudaSuccess)
    e = launch_k(extend_kernel, dim3(1), dim3(kPlanThreads), smem, static_cast<cudaStream_t>(stream), *c, seqs, counts,
                 n, static_cast<int>(rows), slots);
  return launch_err(e);
}

int map_cache_fork(const map_cache* c, const int32_t* parents, const int32_t* children, int n, const int32_t* keep,
                   int k, const int32_t* base, const int32_t* span, void* stream) {
  const int rc = check_cache(c);
  if (rc != MAP_OK) return rc;
  if (n < 0 || k < 0) return MAP_EINVAL;
  if (n == 0) return MAP_OK;
  if (!parents || !children) return MAP_EINVAL;
  if ((base == nullptr) != (span == nullptr) || (keep && !base) || (k > 0 && !keep)) return MAP_EINVAL;
  if (n > kMaxEntries || k > (1 << 24)) return MAP_EUNSUPPORTED;
  const size_t smem = plan_smem(n, c->seqs);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = allow_smem(reinterpret_cast<const void*>(fork_plan_kernel), smem);
  if (e == cudaSuccess)
    e = launch_k(fork_plan_kernel, dim3(1), dim3(kPlanThreads), smem, st, *c, parents, children, n,
                 base != nullptr ? 1 : 0, k, base, span);
  if (e == cudaSuccess)
    e = launch_k(fork_copy_kernel, dim3(kCopyGrid), dim3(kCopyThreads), (n + 1 + static_cast<size_t>(c->page)) * 4, st, *c,
                 parents, children, n, keep, k, base, span);
  return launch_err(e);
}

int map_cache_free(const map_cache* c, const int32_t* seqs, int n, void* stream) {
  const int rc = check_cache(c);
  if (rc != MAP_OK) return rc;
  if (n < 0 || (n > 0 && !seqs)) return MAP_EINVAL;
  if (n > kMaxFree) return MAP_EUNSUPPORTED;
  if (n == 0) return MAP_OK;
  return launch_err(launch_k(free_kernel, dim3((n + 7) / 8), dim3(256), 0, static_cast<cudaStream_t>(stream), *c, seqs, n));
}

int map_cache_status(const map_cache* c, void* stream) {
  const int rc = check_cache(c);
  if (rc != MAP_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t bits = 0;
  cudaError_t e = cudaMemcpyAsync(&bits, c->status, sizeof(bits), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && bits) {
    e = cudaMemsetAsync(c->status, 0, sizeof(bits), st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  }
  if (e != cudaSuccess) return launch_err(e);
  return bits & ST_BADINDEX ? MAP_EINTERNAL : bits & ST_NOPAGES ? MAP_ENOMEM : bits ? MAP_EINTERNAL : MAP_OK;
}

}  // extern "C"
