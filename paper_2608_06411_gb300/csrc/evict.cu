// Rows that leave a cache by their weights (map_cache_evict): of each entry's rows first .. len - last - 1 the k of greatest
// weight stay, chosen for every layer and key head by itself, in their order.
//
// Mathematics.  The k-th greatest weight of a (layer, head) by a radix select on the weights as ordered 32-bit keys (11, 11 and
// 10 bits a pass, ending early where a digit's rows all stay), then one pass in row order: a row stays if its key is greater, or
// equal and among the first of the equals that are needed.
// Bound: HBM, the candidates' weights once and the rows that move once read and once written.  In place: a kept row's new place is
// never behind its old one, and places rise with the rows, so a CTA that goes through a (layer, head)'s rows in order, reading
// a batch whole before it writes it, overwrites nothing that is still to be read.  Pages that other sequences hold as well are
// replaced by new ones (evict_plan_kernel), from which nothing is read.
#include <algorithm>

#include "pages.cuh"

namespace mapk {
namespace {

// An entry of a call: its sequence (-1: nothing of it changes), rows before, first row that may leave, rows after.
struct Eviction { int seq, len, first, left; };
constexpr int kReplaced = 1 << 30;         // of a page in EvictArgs::was: the table has another in its place now

struct EvictArgs {
  map_cache c;
  float* weights;
  const int32_t *seqs, *first, *last;
  int n, k;
  Eviction* entries;                       // [n]
  int32_t* was;                            // [n, max_pages]: pages before the call, of the columns that rows move to
  int32_t* taken;                          // [pages]
};

// Checks, lengths, pages.  Latency-bound, one CTA (see extend_kernel); the columns of all entries form one list.
__global__ void __launch_bounds__(kPlanThreads) evict_plan_kernel(const EvictArgs a) {
  extern __shared__ int sh[];
  const map_cache& c = a.c;
  int* start = sh;                         // [n + 1] columns before entry i
  int* seq = start + a.n + 1;              // [n]
  int* len = seq + a.n;
  int* first = len + a.n;
  int* left = first + a.n;
  unsigned* seen = reinterpret_cast<unsigned*>(left + a.n);   // bitmap of the sequences
  __shared__ int warp_sums[kPlanThreads / 32];
  __shared__ int error;
  pdl_enter();
  for (int i = threadIdx.x; i < (c.seqs + 31) / 32; i += kPlanThreads) seen[i] = 0;
  if (threadIdx.x == 0) error = 0;
  HeadCounts head;
  head.load(c, threadIdx.x * kPagesEach);
  __syncthreads();
  int cols = 0;
  for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int mine = 0;
    if (i < a.n) {
      const int s = a.seqs[i], f = a.first ? a.first[i] : 0, l = a.last ? a.last[i] : 0;
      seq[i] = -1;
      if (s != -1) {
        if (s < 0 || s >= c.seqs || f < 0 || l < 0 || (atomicOr(&seen[s >> 5], 1u << (s & 31)) >> (s & 31) & 1u)) {
          atomicOr(&error, ST_BADINDEX);
        } else if (const int n = c.len[s]; !good_len(c, n)) {
          atomicOr(&error, ST_BADINDEX);
        } else if (const long long window = static_cast<long long>(n) - f - l; window > a.k) {
          seq[i] = s;
          len[i] = n;
          first[i] = f;
          left[i] = n - static_cast<int>(window) + a.k;
          mine = pieces_of(n, c.page) - f / c.page;
        }
      }
    }
    int all;
    const int at = cols + block_scan(mine, warp_sums, &all);
    if (i < a.n) start[i] = at;
    cols += all;
  }
  if (threadIdx.x == 0) start[a.n] = cols;
  __syncthreads();
  // column x of the list: its entry, the table's word; whether rows move there
  const auto column = [&](int x, int& i, int32_t*& word) {
    i = entry_of(start, a.n, x);
    const int col = first[i] / c.page + x - start[i];
    word = c.table + static_cast<long long>(seq[i]) * c.max_pages + col;
    return col < pieces_of(left[i], c.page) ? a.was + static_cast<long long>(i) * c.max_pages + col : nullptr;
  };
  int need = 0;
  for (int x0 = 0; x0 < cols; x0 += kPlanThreads) {
    const int x = x0 + threadIdx.x;
    int replaced = 0;
    if (x < cols) {
      int i;
      int32_t *word, *was = column(x, i, word);
      const int page = *word;
      if (!good_page(c, page)) {
        atomicOr(&error, ST_BADINDEX);
      } else if (was) {
        replaced = c.refs[page] > 1;
        *was = replaced ? page | kReplaced : page;
      }
    }
    need += __syncthreads_count(replaced);     // (at most what a list of 2^31 columns has)
  }
  const bool ok = error == 0;
  const bool enough = ok && need <= c.pages && take_pages(c, need, head, warp_sums, [&](int r) { return a.taken + r; });
  if (!enough && threadIdx.x == 0) atomicOr(c.status, ok ? ST_NOPAGES : error);
  for (int i = threadIdx.x; i < a.n; i += kPlanThreads) {
    const int s = enough ? seq[i] : -1;
    a.entries[i] = s < 0 ? Eviction{-1, 0, 0, 0} : Eviction{s, len[i], first[i], left[i]};
    if (s >= 0) c.len[s] = left[i];
  }
  if (!enough) return;
  __syncthreads();                             // the new pages are there
  int before = 0;
  for (int x0 = 0; x0 < cols; x0 += kPlanThreads) {
    const int x = x0 + threadIdx.x;
    int replaced = 0, page = 0;
    int32_t* word = nullptr;
    bool gone = false;
    if (x < cols) {
      int i;
      const int32_t* was = column(x, i, word);
      page = was ? *was : *word;
      replaced = was && (page & kReplaced) != 0;
      page &= ~kReplaced;
      gone = !was || replaced;
    }
    int all;
    const int r = before + block_scan(replaced, warp_sums, &all);
    before += all;
    if (replaced) *word = a.taken[r];
    if (gone) atomicSub(&c.refs[page], 1);
  }
}

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kEach = 4, kChunk = kThreads * kEach;      // candidates looked at together
constexpr int kList = 2 * kChunk;                        // rows that move, at most so many at a time
constexpr int kBins = 2048;

// Weights in ascending order as unsigned numbers; NaN of either sign is the greatest, zeros are equal.
__device__ __forceinline__ uint32_t key_of(float w) {
  const uint32_t b = __float_as_uint(w + 0.f);
  return isnan(w) ? 0xffffffffu : b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive prefix sums over the block's threads, and the total.
__device__ __forceinline__ uint32_t scan_block(uint32_t v, uint32_t* sums, uint32_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  __syncthreads();                             // the sums of the last call have been read
  if (lane == 31) sums[warp] = s;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const uint32_t x = sums[w];
    before += w < warp ? x : 0;
    all += x;
  }
  *total = all;
  return before + s - v;
}

__global__ void __launch_bounds__(kThreads, 3) evict_kernel(const EvictArgs a) {
  __shared__ union {
    int hist[kBins];
    struct { long long from[kList], to[kList]; } list;   // vectors of a plane
  } sh;
  __shared__ uint32_t sums[kWarps];
  __shared__ uint32_t pick_bin;
  __shared__ int pick_want, pick_size;
  pdl_enter();
  const map_cache& c = a.c;
  const int tid = threadIdx.x, vec = c.dh / 8, max_rows = c.max_pages * c.page;
  const long long plane = static_cast<long long>(c.pages) * c.heads * c.page * vec;
  const long long units = static_cast<long long>(a.n) * c.layers * c.heads;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int head = static_cast<int>(u % c.heads), layer = static_cast<int>(u / c.heads % c.layers);
    const int i = static_cast<int>(u / c.heads / c.layers);
    const int4 en = __ldcg(reinterpret_cast<const int4*>(a.entries + i));
    const int seq = en.x, len = en.y, first = en.z, left = en.w;
    if (seq < 0) continue;
    const int window = len - left + a.k, tail = left - first - a.k;
    float* w = a.weights + ((static_cast<long long>(layer) * c.seqs + seq) * c.heads + head) * max_rows;

    // the least key that stays, and how many rows with it
    uint32_t least = 0xffffffffu;
    int want = 0;
    if (a.k > 0) {
      uint32_t prefix = 0;                     // of the keys' bits above `shift`
      want = a.k;
      int shift = 32;
#pragma unroll 1
      while (shift > 0) {
        const int bits = shift > 10 ? 11 : 10, down = shift - bits;
        __syncthreads();
        for (int b = tid; b < kBins; b += kThreads) sh.hist[b] = 0;
        __syncthreads();
        for (int t = tid; t < window; t += kThreads) {
          const uint32_t key = key_of(w[first + t]);
          if (shift == 32 || key >> shift == prefix) atomicAdd(&sh.hist[key >> down & ((1 << bits) - 1)], 1);
        }
        __syncthreads();
        // from the greatest digit on: a thread counts eight
        constexpr int kOwn = kBins / kThreads;
        int mine = 0;
#pragma unroll
        for (int b = 0; b < kOwn; ++b) mine += sh.hist[kBins - 1 - tid * kOwn - b];
        uint32_t all;
        int above = static_cast<int>(scan_block(mine, sums, &all));
        if (above < want && want <= above + mine)
          for (int b = kBins - 1 - tid * kOwn;; --b) {
            if (want <= above + sh.hist[b]) {
              pick_bin = b;
              pick_want = want - above;
              pick_size = sh.hist[b];
              break;
            }
            above += sh.hist[b];
          }
        __syncthreads();
        prefix = shift == 32 ? pick_bin : prefix << bits | pick_bin;
        want = pick_want;
        shift = down;
        if (pick_size == want) break;          // all of the digit's rows stay
      }
      least = prefix << shift;
      if (pick_size == want) { --least; want = 0; }        // (no weight has a key of zero)
    }

    const int32_t* row = c.table + static_cast<long long>(seq) * c.max_pages;
    const int32_t* was = a.was + static_cast<long long>(i) * c.max_pages;
    const int moved_to = pieces_of(left, c.page);
    const auto place = [&](int page, int t) { return ((static_cast<long long>(page) * c.heads + head) * c.page + t % c.page) * vec; };
    const auto push = [&](int at, int from, int to) {
      const int cf = from / c.page;
      sh.list.from[at] = place(cf < moved_to ? was[cf] & ~kReplaced : row[cf], from);
      sh.list.to[at] = place(row[to / c.page], to);
    };
    uint4* pk = static_cast<uint4*>(c.pool) + 2 * layer * plane;
    uint4* pv = pk + plane;
    int listed = 0;
    const auto flush = [&]() {
      __syncthreads();
      const int vecs = listed * vec;
      for (int e0 = tid; e0 - tid < vecs; e0 += kThreads * kEach) {
        uint4 kx[kEach], vx[kEach];
        long long to[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          const int e = e0 + j * kThreads, r = e / vec, x = e % vec;
          to[j] = -1;
          if (e < vecs && sh.list.from[r] != sh.list.to[r]) {
            const long long from = sh.list.from[r] + x;
            to[j] = sh.list.to[r] + x;
            kx[j] = pk[from];
            vx[j] = pv[from];
          }
        }
        __syncthreads();                       // the batch has been read
#pragma unroll
        for (int j = 0; j < kEach; ++j)
          if (to[j] >= 0) {
            pk[to[j]] = kx[j];
            pv[to[j]] = vx[j];
          }
      }
      listed = 0;
      __syncthreads();
    };

    // rows before the first that may leave, in its page: they move where the page is replaced
    __syncthreads();
    const int at0 = first / c.page * c.page;
    for (int t = at0 + tid; t < first; t += kThreads) push(t - at0, t, t);
    listed = first - at0;
    int kept = 0, equals = 0;                  // rows so far that stay, and with the least key
    for (int t0 = 0; t0 < window; t0 += kChunk) {
      float x[kEach];
      uint32_t key[kEach], mine = 0;
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int t = t0 + tid * kEach + j;
        x[j] = t < window ? w[first + t] : 0.f;
        key[j] = t < window ? key_of(x[j]) : 0u;
        mine += key[j] > least ? 1u : key[j] == least ? 0x10000u : 0u;
      }
      uint32_t all, at = scan_block(mine, sums, &all);       // (the chunk has been read behind it)
      int greater = at & 0xffff, eq = equals + (at >> 16);
      const int eq0 = min(equals, want);
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int here = greater + min(eq, want) - eq0;
        const bool same = key[j] == least && t0 + tid * kEach + j < window;
        if (key[j] > least || (same && eq < want)) {
          push(listed + here, first + t0 + tid * kEach + j, first + kept + here);
          w[first + kept + here] = x[j];
        }
        greater += key[j] > least;
        eq += same;
      }
      equals += all >> 16;
      const int stay = (all & 0xffff) + min(equals, want) - eq0;
      kept += stay;
      listed += stay;
      if (listed > kList - kChunk) flush();
    }
    for (int t0 = 0; t0 < tail; t0 += kChunk) {
      const int from = len - tail + t0, to = left - tail + t0, rows = min(kChunk, tail - t0);
      float x[kEach];
#pragma unroll
      for (int j = 0; j < kEach; ++j)
        if (tid + j * kThreads < rows) x[j] = w[from + tid + j * kThreads];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int r = tid + j * kThreads;
        if (r < rows) {
          w[to + r] = x[j];
          push(listed + r, from + r, to + r);
        }
      }
      listed += rows;
      if (listed > kList - kChunk) flush();
    }
    flush();
    for (int t = left + tid; t < len; t += kThreads) w[t] = 0.f;
  }
}

struct EvictSpace { size_t was, taken, bytes; };
EvictSpace evict_space(const map_cache* c, long long n) {
  EvictSpace s;
  s.was = static_cast<size_t>(n) * sizeof(Eviction);
  s.taken = s.was + static_cast<size_t>(n) * c->max_pages * 4;
  s.bytes = s.taken + static_cast<size_t>(c->pages) * 4;
  return s;
}
bool evict_fits(const map_cache* c, int n) { return n <= kMaxEntries && static_cast<long long>(n) * c->max_pages < (1ll << 31); }

}  // namespace
}  // namespace mapk

using namespace mapk;

extern "C" {

size_t map_cache_evict_workspace(const map_cache* c, int n) {
  return check_cache(c) == MAP_OK && n >= 0 && evict_fits(c, n) ? evict_space(c, n).bytes : 0;
}

int map_cache_evict(const map_cache* c, float* weights, const int32_t* seqs, int n, const int32_t* first, const int32_t* last,
                    int k, void* ws, void* stream) {
  const int rc = check_cache(c);
  if (rc != MAP_OK) return rc;
  if (n < 0 || k < 0) return MAP_EINVAL;
  if (!evict_fits(c, n)) return MAP_EUNSUPPORTED;
  if (n == 0) return MAP_OK;
  if (!seqs || !weights || (reinterpret_cast<uintptr_t>(weights) & 3) || !ws || !aligned16(ws)) return MAP_EINVAL;
  const EvictSpace s = evict_space(c, n);
  char* p = static_cast<char*>(ws);
  const EvictArgs a{*c, weights, seqs, first, last, n, k, reinterpret_cast<Eviction*>(p),
                    reinterpret_cast<int32_t*>(p + s.was), reinterpret_cast<int32_t*>(p + s.taken)};
  const size_t smem = plan_smem(n, c->seqs);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = allow_smem(reinterpret_cast<const void*>(evict_plan_kernel), smem);
  if (e == cudaSuccess) e = launch_k(evict_plan_kernel, dim3(1), dim3(kPlanThreads), smem, st, a);
  const long long units = static_cast<long long>(n) * c->layers * c->heads;
  if (e == cudaSuccess)
    e = launch_k(evict_kernel, dim3(static_cast<unsigned>(std::min<long long>(units, 152 * 6))), dim3(kThreads), 0, st, a);
  return launch_err(e);
}

}  // extern "C"
