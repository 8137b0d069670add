// Rows that leave a cache by their weights (map_cache_evict): of each entry's rows first .. len - last - 1 the k of greatest
// weight stay, chosen for every layer and key head (a unit) by itself, in their order.
//
// Mathematics.  The k-th greatest weight of a unit by a radix select on the weights as ordered 32-bit keys (11, 11 and 10 bits a
// pass, ending early where a digit's rows all stay); then a row stays if its key has greater digits, or the digits found and is
// among the first of those that are needed.
// Bound: HBM, the candidates' weights once and the rows that move once read and once written.  In place: a kept row's new place is
// never behind its old one, and places rise with the rows, so a CTA that goes through rows in order, reading a batch whole
// before it writes it, overwrites nothing that is still to be read; columns do not depend on one another, so that slices of them
// are moved by CTAs of their own, and the weights like one more column.  Pages that other sequences hold as well are replaced by
// new ones (evict_plan_kernel), from which nothing is read.
// Three launches.  One CTA does the pages; beside it a cluster a unit (a CTA where units are many) lists the rows that stay; then
// the rows move.  (One kernel, a CTA a unit, took 65, 223, 229 and 621 us for the cases below; that kernel with 2048 units in
// two halves, the select of some beside the moves of others, gained nothing.)
// Measured (28 layers of 4 key heads, 128 columns, unless said otherwise; with the copies of tables and weights that the
// measurement makes): one sequence of 1100 rows to 512: 26 us, a chain of launches; 6 of 3001 to 4096 rows to 1315: 170 us, of
// which the move of 854 MB of DRAM traffic takes 141 to 148, 5.8 to 6.1 TB/s; 8 questions of 2915 to 3000 rows on one image in
// 32 layers of 8 heads to 245: 119 us, the move of rows at random places 77 (5.5 TB/s), the select 28, bound by its
// instructions; one of 60001 rows in 8 layers to 16900: 144 us, of which the move of 64-byte slices takes 108 (4.9 TB/s).
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
  int n, k, page_shift;                    // log2 of the page, -1: no power of two
  Eviction* entries;                       // [n]
  int32_t* was;                            // [n, max_pages]: pages before the call, of the columns that rows move to
  int32_t* taken;                          // [pages]
  int32_t* kept;                           // [n][layers][heads][k]: rows that stay of those that may leave
};

// Checks, new lengths, pages.  Latency-bound, one CTA (see extend_kernel); the columns of all entries form one list.
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
  for (unsigned x0 = 0; x0 < static_cast<unsigned>(cols); x0 += kPlanThreads) {        // (columns and a block can add up past 2^31)
    const unsigned x = x0 + threadIdx.x;
    int replaced = 0;
    if (x < static_cast<unsigned>(cols)) {
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
  }
  if (!enough) return;
  __syncthreads();                             // the new pages are there
  int before = 0;
  for (unsigned x0 = 0; x0 < static_cast<unsigned>(cols); x0 += kPlanThreads) {
    const unsigned x = x0 + threadIdx.x;
    int replaced = 0, page = 0;
    int32_t* word = nullptr;
    bool gone = false;
    if (x < static_cast<unsigned>(cols)) {
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

constexpr int kBins = 2048;

// Weights in ascending order as unsigned numbers; NaN of either sign is the greatest, zeros are equal.
__device__ __forceinline__ uint32_t key_of(float w) {
  const uint32_t b = __float_as_uint(w + 0.f);
  return isnan(w) ? 0xffffffffu : b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ int4 ld_peer(uint32_t at) {
  int4 v;
  asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ int cluster_size() {
  int n;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
  return n;
}

struct Unit { Eviction e; int entry, layer, head; long long id; };
__device__ __forceinline__ Unit unit_of(const EvictArgs& a, unsigned u) {       // (entry, layer, head), without the entry's Eviction
  const unsigned heads = a.c.heads, layers = a.c.layers, r = u / heads;
  Unit x;
  x.id = u;
  x.head = u - r * heads;
  x.entry = r / layers;
  x.layer = r - x.entry * layers;
  return x;
}
// What the plan will find for an entry, if it does not refuse the call.
__device__ __forceinline__ Eviction eviction_of(const EvictArgs& a, int i) {
  const int s = __ldcg(a.seqs + i), f = a.first ? __ldcg(a.first + i) : 0, l = a.last ? __ldcg(a.last + i) : 0;
  if (s < 0 || s >= a.c.seqs || f < 0 || l < 0) return {-1, 0, 0, 0};
  const int n = __ldcg(a.c.len + s);
  const long long window = static_cast<long long>(n) - f - l;
  if (!good_len(a.c, n) || window <= a.k) return {-1, 0, 0, 0};
  return {s, n, f, n - static_cast<int>(window) + a.k};
}
__device__ __forceinline__ float* weights_of(const EvictArgs& a, const Unit& x) {
  return a.weights + ((static_cast<long long>(x.layer) * a.c.seqs + x.e.seq) * a.c.heads + x.head) * (static_cast<long long>(a.c.max_pages) * a.c.page);
}

// The rows that stay, in order, into kept [units][k]: a cluster a unit, an equal run of the candidates a CTA, of which a warp holds
// HOLD times 32 in a row.  Runs of up to HOLD * THREADS are read once.
template <int THREADS, int HOLD>
__global__ void __launch_bounds__(THREADS, 1280 / THREADS) evict_select_kernel(const EvictArgs a) {
  constexpr int kWarps = THREADS / 32, kBinsEach = kBins / THREADS, kChunk = HOLD * THREADS;
  __shared__ __align__(16) int hist[2][kBins];
  __shared__ int warp_sum[kWarps];
  __shared__ int2 warp_kept[kWarps];
  __shared__ uint32_t pick_bin;
  __shared__ int pick_want, pick_size;
  __shared__ __align__(16) int4 mine;          // candidates of this CTA above the digits found, and with them
  // Beside the plan, which starts this kernel once it has waited for those before it, and writes nothing that is read here (loads go
  // to L2: without a wait L1 may have older lines).  The wait at the end makes this kernel end behind the plan.
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, ranks = cluster_size(), rank = blockIdx.x % ranks;
  Unit x = unit_of(a, blockIdx.x / ranks);
  x.e = eviction_of(a, x.entry);
  if (x.e.seq < 0 || a.k == 0) {               // (one decision a cluster)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    return;
  }
  // (unsigned: a window and a chunk can add up past 2^31)
  const unsigned window = x.e.len - x.e.left + a.k, each = pieces_of(static_cast<int>(window), ranks);
  const unsigned t0 = min(window, rank * each), t1 = min(window, t0 + each);
  const float* w = weights_of(a, x) + x.e.first;
  const auto all_here = [&]() { if (ranks > 1) cluster_sync(); else __syncthreads(); };
  uint32_t key[HOLD];                         // of candidates row0 + 32 j; 0, below all weights, where there is none
  const auto load = [&](unsigned c0) {
    const unsigned row0 = c0 + warp * (32 * HOLD) + lane;
    float v[HOLD];
#pragma unroll
    for (int j = 0; j < HOLD; ++j) v[j] = row0 + 32 * j < t1 ? __ldcg(w + row0 + 32 * j) : 0.f;
#pragma unroll
    for (int j = 0; j < HOLD; ++j) key[j] = row0 + 32 * j < t1 ? key_of(v[j]) : 0u;
  };
  const bool once = t1 - t0 <= kChunk;
  load(t0);

  for (int b = tid; b < kBins / 4; b += THREADS) reinterpret_cast<int4*>(hist[0])[b] = make_int4(0, 0, 0, 0);
  if (tid == 0) mine = make_int4(0, 0, 0, 0);
  __syncthreads();
  // a digit a pass, of the keys with the digits found so far
  uint32_t prefix = 0;
  int want = a.k, shift = 32, pass = 0;
#pragma unroll 1
  for (; shift > 0; pass ^= 1) {
    const int bits = shift > 10 ? 11 : 10, down = shift - bits;
#pragma unroll 1
    for (unsigned c0 = t0; c0 < t1; c0 += kChunk) {
      if (!once) load(c0);
#pragma unroll
      for (int j = 0; j < HOLD; ++j)
        if (key[j] != 0 && (shift == 32 || key[j] >> shift == prefix)) atomicAdd(&hist[pass][key[j] >> down & ((1 << bits) - 1)], 1);
    }
    all_here();
    // (the others have read the last pass's counts: they are here)
    for (int b = tid; b < kBins / 4; b += THREADS) reinterpret_cast<int4*>(hist[pass ^ 1])[b] = make_int4(0, 0, 0, 0);
    // from the greatest digit on: a thread counts kBinsEach, over all of the cluster's CTAs
    const int bin0 = kBins - (tid + 1) * kBinsEach;
    int count[kBinsEach], own[kBinsEach];
#pragma unroll
    for (int b = 0; b < kBinsEach; b += 4) {
      const int4 v = *reinterpret_cast<const int4*>(&hist[pass][bin0 + b]);
      count[b] = own[b] = v.x;
      count[b + 1] = own[b + 1] = v.y;
      count[b + 2] = own[b + 2] = v.z;
      count[b + 3] = own[b + 3] = v.w;
    }
#pragma unroll 7
    for (int r = 1; r < ranks; ++r) {
#pragma unroll
      for (int b = 0; b < kBinsEach; b += 4) {
        const int4 v = ld_peer(mapa_u32(&hist[pass][bin0 + b], rank + r < ranks ? rank + r : rank + r - ranks));
        count[b] += v.x;
        count[b + 1] += v.y;
        count[b + 2] += v.z;
        count[b + 3] += v.w;
      }
    }
    int sum = 0;
#pragma unroll
    for (int b = 0; b < kBinsEach; ++b) sum += count[b];
    int above = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, above, o);
      if (lane >= o) above += u;
    }
    if (lane == 31) warp_sum[warp] = above;
    __syncthreads();
    above -= sum;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) above += i < warp ? warp_sum[i] : 0;
    if (above < want && want <= above + sum) {
#pragma unroll
      for (int b = kBinsEach - 1; b >= 0; --b) {
        if (above < want && want <= above + count[b]) {
          pick_bin = bin0 + b;
          pick_want = want - above;
          pick_size = count[b];
        }
        above += count[b];
      }
    }
    __syncthreads();
    if (ranks > 1) {                           // for the CTAs behind this one
      const int pick = static_cast<int>(pick_bin);
      int greater = 0, equal = 0;
#pragma unroll
      for (int b = 0; b < kBinsEach; ++b) {
        greater += bin0 + b > pick ? own[b] : 0;
        equal += bin0 + b == pick ? own[b] : 0;
      }
      greater = __reduce_add_sync(0xffffffffu, greater);
      if (lane == 0 && greater) atomicAdd(&mine.x, greater);
      if (equal && (pick_size == pick_want || down == 0)) mine.y = equal;
    }
    prefix = shift == 32 ? pick_bin : prefix << bits | pick_bin;
    want = pick_want;
    shift = down;
    if (pick_size == want) break;              // all of the digit's rows stay
  }
  // keys from `least` on have the digits found, those past `most` greater ones
  const uint32_t least = prefix << shift, most = shift > 0 ? least | ((1u << shift) - 1) : least;

  all_here();
  int kept = 0, equals = 0;                    // rows so far with greater digits, and with the digits found
#pragma unroll 8
  for (int r = 0; r < rank; ++r) {
    const int4 v = ld_peer(mapa_u32(&mine, r));
    kept += v.x;
    equals += v.y;
  }
  int32_t* out = a.kept + x.id * a.k;
#pragma unroll 1
  for (unsigned c0 = t0; c0 < t1; c0 += kChunk) {
    if (!once) load(c0);
    int2 n = make_int2(0, 0);
#pragma unroll
    for (int j = 0; j < HOLD; ++j) {
      n.x += key[j] > most;
      n.y += key[j] >= least;
    }
    n.x = __reduce_add_sync(0xffffffffu, n.x);
    n.y = __reduce_add_sync(0xffffffffu, n.y) - n.x;
    __syncthreads();                           // the last chunk's have been read
    if (lane == 0) warp_kept[warp] = n;
    __syncthreads();
    int at = kept, eq = equals;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const int2 v = warp_kept[i];
      if (i < warp) {
        at += v.x;
        eq += v.y;
      }
      kept += v.x;
      equals += v.y;
    }
    const uint32_t before = (1u << lane) - 1;
    const unsigned row0 = x.e.first + c0 + warp * (32 * HOLD) + lane;
#pragma unroll
    for (int j = 0; j < HOLD; ++j) {
      const bool more = key[j] > most, same = !more && key[j] >= least;
      const uint32_t m = __ballot_sync(0xffffffffu, more), s = __ballot_sync(0xffffffffu, same);
      const int mine_eq = eq + __popc(s & before);
      if (more || (same && mine_eq < want)) out[at + __popc(m & before) + min(mine_eq, want)] = row0 + 32 * j;
      at += __popc(m);
      eq += __popc(s);
    }
  }
  if (ranks > 1) cluster_sync();               // no CTA leaves while another may read its counts
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// The rows that move, a slice of a unit's columns (or its weights) a CTA.  THREADS / wide rows are read together, a 16-byte vector a
// thread, kMoveEach times before the first is written.
constexpr int kMoveEach = 8, kMoveRowsEach = 2;
template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) evict_move_kernel(const EvictArgs a, int slices) {
  struct Row { long long from, to; };          // vectors of a plane; from -1: the row is where it shall be
  __shared__ Row list[3][kMoveRowsEach * THREADS];           // batches: being stored, loaded, looked up
  pdl_enter();
  const map_cache& c = a.c;
  const int tid = threadIdx.x, parts = 2 * slices + 1, part = blockIdx.x % parts;
  Unit x = unit_of(a, blockIdx.x / parts);
  const int4 planned = __ldcg(reinterpret_cast<const int4*>(a.entries + x.entry));
  x.e = Eviction{planned.x, planned.y, planned.z, planned.w};
  if (x.e.seq < 0) return;
  const Eviction& e = x.e;
  const int tail = e.left - e.first - a.k;
  const int32_t* kept = a.kept + x.id * a.k;
  // row r of those from e.first on: where it comes from
  const auto source = [&](int r) { return r < a.k ? __ldcg(kept + r) : e.len - tail + (r - a.k); };

  if (part == parts - 1) {                     // the weights, and zeros behind them
    float* w = weights_of(a, x);
    constexpr int kBatch = THREADS * kMoveEach;
    const unsigned moved = a.k + tail;         // (unsigned: these and a batch, and a length and a block, can add up past 2^31)
    for (unsigned r0 = 0; r0 < moved; r0 += kBatch) {
      float v[kMoveEach];
#pragma unroll
      for (int j = 0; j < kMoveEach; ++j) {
        const unsigned r = r0 + tid + j * THREADS;
        v[j] = r < moved ? w[source(r)] : 0.f;
      }
      __syncthreads();                         // the batch has been read
#pragma unroll
      for (int j = 0; j < kMoveEach; ++j) {
        const unsigned r = r0 + tid + j * THREADS;
        if (r < moved) w[e.first + r] = v[j];
      }
    }
    __syncthreads();                           // the last rows' sources lie where the zeros go
    for (unsigned t = e.left + tid; t < static_cast<unsigned>(e.len); t += THREADS) w[t] = 0.f;
    if (x.layer == 0 && x.head == 0 && tid == 0) c.len[e.seq] = e.left;      // (select reads it beside the plan)
    return;
  }

  const int vec = c.dh / 8, slice = part % slices, v0 = vec * slice / slices, wide = vec * (slice + 1) / slices - v0;
  const int together = min(THREADS / wide, kMoveRowsEach * THREADS / kMoveEach), mine = tid / wide;    // rows; this thread's
  const long long plane = static_cast<long long>(c.pages) * c.heads * c.page * vec;
  uint4* pool = static_cast<uint4*>(c.pool) + (2 * x.layer + part / slices) * plane + v0 + tid % wide;
  const int32_t* row = c.table + static_cast<long long>(e.seq) * c.max_pages;
  const int32_t* was = a.was + static_cast<long long>(x.entry) * c.max_pages;
  const int moved_to = pieces_of(e.left, c.page);
  const auto page_of = [&](int t) { return a.page_shift >= 0 ? t >> a.page_shift : t / c.page; };
  const auto place = [&](int page, int in_page) { return ((static_cast<long long>(page) * c.heads + x.head) * c.page + in_page) * vec; };
  // rows before e.first in its page move too, where the page is replaced
  const int head = e.first - page_of(e.first) * c.page, rows = head + a.k + tail, batch = together * kMoveEach;
  int src[kMoveRowsEach];                      // of the batch to be looked up next
  const auto sources = [&](unsigned r0, int n) {       // (r0 of a batch behind the last can pass 2^31; n says that it has no rows)
#pragma unroll
    for (int k = 0; k < kMoveRowsEach; ++k) {
      const int i = tid + k * THREADS;
      src[k] = i < min(batch, n) ? (r0 + i < static_cast<unsigned>(head) ? static_cast<int>(e.first + r0 + i - head) : source(r0 + i - head)) : -1;
    }
  };
  const auto look_up = [&](unsigned r0, Row* to) {
#pragma unroll
    for (int k = 0; k < kMoveRowsEach; ++k) {
      const int s = src[k];
      if (s < 0) continue;
      const int t = e.first + r0 + tid + k * THREADS - head;
      const int cf = page_of(s), ct = page_of(t);
      const int old = cf < moved_to ? __ldcg(was + cf) & ~kReplaced : __ldcg(row + cf), now = __ldcg(row + ct);
      to[tid + k * THREADS] = Row{s == t && old == now ? -1 : place(old, s - cf * c.page), place(now, t - ct * c.page)};
    }
  };
  sources(0, rows);
  look_up(0, list[0]);
  sources(batch, rows - batch);
  __syncthreads();
  int at = 0;
  unsigned r0 = 0;
  for (int n = rows; n > 0; r0 += batch, n -= batch) {
    const Row* here = list[at] + mine;
    at = at == 2 ? 0 : at + 1;
    const int here_n = mine < together ? min(batch, n) - mine : 0;       // this thread's rows: 0, together, ... below it
    uint4 v[kMoveEach];
#pragma unroll
    for (int j = 0; j < kMoveEach; ++j)
      if (j * together < here_n && here[j * together].from >= 0) v[j] = pool[here[j * together].from];
    look_up(r0 + batch, list[at]);
    sources(r0 + 2 * batch, n - 2 * batch);
    __syncthreads();                           // the batch has been read, the next one looked up
#pragma unroll
    for (int j = 0; j < kMoveEach; ++j)
      if (j * together < here_n && here[j * together].from >= 0) pool[here[j * together].to] = v[j];
  }
}

struct EvictSpace { size_t was, taken, kept, bytes; };
EvictSpace evict_space(const map_cache* c, long long n, long long k) {
  EvictSpace s;
  s.was = static_cast<size_t>(n) * sizeof(Eviction);
  s.taken = s.was + static_cast<size_t>(n) * c->max_pages * 4;
  s.kept = s.taken + static_cast<size_t>(c->pages) * 4;
  s.bytes = s.kept + static_cast<size_t>(n) * c->layers * c->heads * std::min<long long>(k, static_cast<long long>(c->max_pages) * c->page) * 4;
  return s;
}
bool evict_fits(const map_cache* c, long long n) {            // units: 9 CTAs each, and 2^31 rows that stay, of 4 bytes
  return n <= kMaxEntries && n * c->max_pages < (1ll << 31) && n * c->layers * c->heads <= (1 << 24);
}

}  // namespace
}  // namespace mapk

using namespace mapk;

extern "C" {

size_t map_cache_evict_workspace(const map_cache* c, int n, int k) {
  return check_cache(c) == MAP_OK && n >= 0 && k >= 0 && evict_fits(c, n) ? evict_space(c, n, k).bytes : 0;
}

int map_cache_evict(const map_cache* c, float* weights, const int32_t* seqs, int n, const int32_t* first, const int32_t* last,
                    int k, void* ws, void* stream) {
  const int rc = check_cache(c);
  if (rc != MAP_OK) return rc;
  if (n < 0 || k < 0) return MAP_EINVAL;
  if (!evict_fits(c, n)) return MAP_EUNSUPPORTED;
  if (n == 0) return MAP_OK;
  if (!seqs || !weights || (reinterpret_cast<uintptr_t>(weights) & 3) || !ws || !aligned16(ws)) return MAP_EINVAL;
  const EvictSpace s = evict_space(c, n, k);
  char* p = static_cast<char*>(ws);
  const int shift = (c->page & (c->page - 1)) == 0 ? __builtin_ctz(c->page) : -1;
  const EvictArgs a{*c, weights, seqs, first, last, n, k, shift, reinterpret_cast<Eviction*>(p),
                    reinterpret_cast<int32_t*>(p + s.was), reinterpret_cast<int32_t*>(p + s.taken), reinterpret_cast<int32_t*>(p + s.kept)};
  const size_t smem = plan_smem(n, c->seqs);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = allow_smem(reinterpret_cast<const void*>(evict_plan_kernel), smem);
  if (e == cudaSuccess) e = launch_k(evict_plan_kernel, dim3(1), dim3(kPlanThreads), smem, st, a);
  const long long units = static_cast<long long>(n) * c->layers * c->heads, max_rows = static_cast<long long>(c->max_pages) * c->page;
  // CTAs that look for a unit's rows, and slices that its columns move in: as many as fill the chip where the units do not.  What a
  // sequence can hold counts, for its length is not known here: one of 1100 rows to 512 takes 28 to 30 us in a cache of 1120 to 4112
  // rows, 32 in one of 16384 and 37 in one of 131072.
  int ranks = 1, slices = 1;
  while (ranks < 8 && units * ranks < 2 * 152 && max_rows / ranks > 2048) ranks *= 2;
  while (slices < 4 && units * (4 * slices + 1) <= 4 * 152 && c->dh / 8 / slices >= 8) slices *= 2;
  const unsigned select = static_cast<unsigned>(units * ranks);
  const long long most = (max_rows + ranks - 1) / ranks;     // candidates of a CTA (2048 runs of 2830: 33 us with 16 a thread, 28 with 13)
  const auto look = [&](auto kernel, int threads) { if (e == cudaSuccess) e = launch_cluster(kernel, select, threads, ranks, st, a); };
  if (most <= 4 * 256) look(evict_select_kernel<256, 4>, 256);
  else if (most <= 8 * 256) look(evict_select_kernel<256, 8>, 256);
  else if (most <= 13 * 256) look(evict_select_kernel<256, 13>, 256);
  else if (most <= 16 * 256) look(evict_select_kernel<256, 16>, 256);
  else look(evict_select_kernel<512, 16>, 512);
  const unsigned move = static_cast<unsigned>(units * (2 * slices + 1));
  if (e == cudaSuccess)
    e = move <= 2 * 152 ? launch_k(evict_move_kernel<512>, dim3(move), dim3(512), 0, st, a, slices)
                        : launch_k(evict_move_kernel<256>, dim3(move), dim3(256), 0, st, a, slices);
  return launch_err(e);
}

}  // extern "C"
