// Attention of single tokens for groups of sequences that begin with the same pages (map_cache_attend_shared).
//
// Mathematics.  The rows t < S of a group are the same for all of its sequences, so that their part of every member's attention
// (m, l, o: largest score, sum of weights, unnormalised output) is a product of all the members' queries of a key head with one
// set of keys and values; the rows from S on are each member's own (attend's kernel), and the parts join as in attend.
//
// Bound: HBM, a group's shared rows once and the others once a sequence; 4 S dh operations a query head beside them, which is
// what limits it from about 100 query heads a key head on (224: 22 us of tensor time against 18 of loads, below).
// Four launches: what is shared (a CTA a group compares the members' table rows), the shared rows, the sequences' own, the join.
#include <type_traits>

#include "attend.cuh"

namespace mapk {
namespace {

// A group: entries first .. first + count - 1, whose sequences' first `rows` rows are those of sequence `seq`.
struct Group { int first, count, rows, seq; };

struct SharedArgs {
  AttendArgs a;
  const int32_t* starts;
  int groups;
  Group* group;                                // [groups]
  int32_t* of;                                 // [n] an entry's group, -1: none
  int32_t* skip;                               // [n] rows that it shares
  long long* tile0;                            // [groups + 1] tiles before a group, and all (the list of shared_kernel)
  float* parts;                                // [grid][2] parts of items that several CTAs share
  float2* whole_stats;                         // the others': (m, l) [n][q.heads]
  float* whole;                                //         o [n][q.heads][dh]
  int grid;                                    // of shared_kernel
};

constexpr int kPlan = 512;

// What a group shares: the pages that all its sequences with rows hold in front, as far as all are full.
__global__ void __launch_bounds__(kPlan) shared_plan_kernel(const __grid_constant__ SharedArgs p) {
  const AttendArgs& a = p.a;
  __shared__ int least, lead, valid;
  pdl_enter();
  const int g = blockIdx.x, tid = threadIdx.x;
  if (tid == 0) {
    least = a.c.max_pages;
    lead = a.n;
    valid = 0;
  }
  bool bad = false;                            // (every CTA looks at all of it: no more than 65536 numbers)
  for (int i = tid; i <= p.groups; i += kPlan) {
    const int s = __ldg(p.starts + i), next = i < p.groups ? __ldg(p.starts + i + 1) : a.n;
    bad |= s > next || (i == 0 && s != 0) || (i == p.groups && s != a.n);
  }
  if (__syncthreads_or(bad)) {
    if (g == 0 && tid == 0) atomicOr(a.c.status, ST_BADINDEX);
    for (int i = g * kPlan + tid; i < a.n; i += static_cast<int>(gridDim.x) * kPlan) {
      p.of[i] = -1;
      p.skip[i] = 0;
    }
    if (tid == 0) p.group[g] = Group{0, 0, 0, 0};
    return;
  }
  const int first = __ldg(p.starts + g), last = __ldg(p.starts + g + 1);
  int mine = 0;
  for (int i = first + tid; i < last; i += kPlan) {
    const int len = seq_len(a, i);
    if (len == 0) continue;
    ++mine;
    atomicMin(&lead, i);
    atomicMin(&least, len / a.c.page);
  }
  if (mine) atomicAdd(&valid, mine);
  __syncthreads();
  const int of = lead, full = valid > 1 ? least : 0;
  __syncthreads();
  int same = full;
  if (full > 0) {
    const int32_t* row = a.c.table + static_cast<long long>(__ldg(a.seqs + of)) * a.c.max_pages;
    for (int i = first + tid / 32; i < last; i += kPlan / 32) {          // a warp a member
      if (seq_len(a, i) == 0) continue;
      const int32_t* other = a.c.table + static_cast<long long>(__ldg(a.seqs + i)) * a.c.max_pages;
#pragma unroll 8
      for (int j = tid % 32; j < full; j += 32)
        if (__ldg(other + j) != __ldg(row + j)) same = min(same, j);
    }
    atomicMin(&least, same);
  }
  __syncthreads();
  const int rows = full > 0 ? least * a.c.page : 0;
  for (int i = first + tid; i < last; i += kPlan) {
    p.of[i] = g;
    p.skip[i] = seq_len(a, i) > 0 ? rows : 0;
  }
  if (tid == 0) p.group[g] = Group{first, last - first, rows, rows > 0 ? __ldg(a.seqs + of) : 0};
}

// ---- the shared rows.  An item is up to 128 rows of queries (member, head) of one key head and group: the M of a
// tcgen05.mma.  64 keys are the N of the scores' product and the K of the values', whose first operand, the weights as two halves
// of T, lies in TMEM.  Warps 0-3 do the softmax, a row a thread; 4 and 5 load keys, 6 and 7 values, each with a ring of its own;
// a thread of warp 8 issues the products: scores of a tile while the last one's weights are made.
constexpr int kM = 128, kN = 64;
constexpr int kSharedThreads = 288, kKeyRing = 3, kValueRing = 2;

template <int DH>
struct Shape {
  static constexpr int kBlocks = (DH + 63) / 64;             // boxes of 64 columns, 128 bytes a row, 16-byte units exchanged by the row's low bits
  static constexpr int kTileBytes = kBlocks * kN * 128, kQBytes = kBlocks * kM * 128;
  static constexpr int kTiles = kQBytes + (kKeyRing + kValueRing) * kTileBytes, kSmem = kTiles + 512;    // the barriers behind the tiles
  static constexpr int kCtas = DH <= 128 ? 2 : 1;
  static constexpr int kHi = kN, kLo = kN + kN / 2, kO = 2 * kN;       // TMEM columns: scores at 0
  static constexpr int kCols = kO + DH <= 256 ? 256 : 512;
  static constexpr int kPart = kM * (DH + 2);                // floats: m [128], l [128], o [DH / 4][128] float4
  static_assert(kCtas * kCols <= 512 && kCtas * (kSmem + 1024) <= 228 * 1024, "TMEM and shared memory");
};

constexpr uint32_t kBf16Types = (1u << 7) | (1u << 10);      // of an instruction descriptor: A and B
template <typename T>
__host__ __device__ constexpr uint32_t idesc_of(int m, int n) {
  return std::is_same<T, __half>::value ? idesc_bf16(m, n) & ~kBf16Types : idesc_bf16(m, n);
}

// D[tmem] (+)= A[tmem] * B[smem]: A's 16-bit columns two to a 32-bit one.
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Where a run of the list (group, key head, rows of queries, tile) is.
struct SharedPlace {
  Group gr;
  int g, item, items, tiles, t;
  __device__ __forceinline__ void enter(const SharedArgs& p, int from) {
    tiles = 0;
    for (g = from; g < p.groups; ++g) {
      const int4 x = __ldcg(reinterpret_cast<const int4*>(p.group + g));
      gr = Group{x.x, x.y, x.z, x.w};
      if (gr.rows > 0) break;
    }
    if (g >= p.groups) return;
    tiles = pieces_of(gr.rows, kN);
    items = p.a.c.heads * blocks(p);
  }
  __device__ __forceinline__ int blocks(const SharedArgs& p) const { return (gr.count * p.a.group + kM - 1) / kM; }
  __device__ __forceinline__ bool next(const SharedArgs& p) {          // whether another item begins
    if (++t < tiles) return false;
    t = 0;
    if (++item < items) return true;
    item = 0;
    enter(p, g + 1);
    return true;
  }
};

struct SharedBars {
  uint64_t k_full[kKeyRing], k_empty[kKeyRing], v_full[kValueRing], v_empty[kValueRing], q_full, s_full, s_free, p_full, o_done, drain;
  uint32_t tmem;
  int abort, group;
  long long tile;
  long long red[kSharedThreads / 32];
};
static_assert(sizeof(SharedBars) <= 512, "behind the tiles");

template <typename T, int DH>
__global__ void __launch_bounds__(kSharedThreads, Shape<DH>::kCtas) shared_kernel(const __grid_constant__ SharedArgs p) {
  using S = Shape<DH>;
  constexpr int VPR = DH / 8;
  extern __shared__ __align__(1024) unsigned char sh[];
  SharedBars& b = *reinterpret_cast<SharedBars*>(sh + S::kTiles);
  pdl_enter();
  const AttendArgs& a = p.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

  // this CTA's run of the list, and where it begins: a thread counts a run of the groups
  const auto tiles_of = [&](int g) -> long long {
    SharedPlace x;
    const int4 v = __ldcg(reinterpret_cast<const int4*>(p.group + g));
    x.gr = Group{v.x, v.y, v.z, v.w};
    return x.gr.rows > 0 ? static_cast<long long>(pieces_of(x.gr.rows, kN)) * a.c.heads * x.blocks(p) : 0;
  };
  const int each = (p.groups + kSharedThreads - 1) / kSharedThreads, g0 = min(p.groups, tid * each), g1 = min(p.groups, g0 + each);
  long long mine = 0, total;
  for (int g = g0; g < g1; ++g) mine += tiles_of(g);
  long long at0 = block_prefix<kSharedThreads / 32>(mine, b.red, &total);
  const long long per = (total + gridDim.x - 1) / gridDim.x, t0 = per * blockIdx.x;
  if (blockIdx.x == 0) {
    long long at = at0;
    for (int g = g0; g < g1; ++g) {
      p.tile0[g] = at;
      at += tiles_of(g);
    }
    if (tid == 0) p.tile0[p.groups] = total;
  }
  if (t0 >= total) return;
  if (smem_u32(sh) & 1023) {                   // (never: the alignment that its declaration asks for)
    if (tid == 0) atomicOr(a.c.status, ST_INTERNAL);
    return;
  }
  const int run = static_cast<int>(t0 + per <= total ? per : total - t0);
  if (at0 <= t0 && t0 < at0 + mine) {
    for (int g = g0;; ++g) {
      const long long k = tiles_of(g);
      if (t0 < at0 + k) {
        b.group = g;
        b.tile = t0 - at0;
        break;
      }
      at0 += k;
    }
  }
  if (tid == 0) {
    for (int i = 0; i < kKeyRing; ++i) {
      mbar_init(&b.k_full[i], 64);
      mbar_init(&b.k_empty[i], 1);
    }
    for (int i = 0; i < kValueRing; ++i) {
      mbar_init(&b.v_full[i], 64);
      mbar_init(&b.v_empty[i], 1);
    }
    mbar_init(&b.q_full, 128);
    mbar_init(&b.s_full, 1);
    mbar_init(&b.s_free, 4);
    mbar_init(&b.p_full, 4);
    mbar_init(&b.o_done, 1);
    mbar_init(&b.drain, 1);
    b.abort = 0;
    fence_mbar_init();
  }
  if (warp == 8) {
    tmem_alloc(&b.tmem, S::kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = b.tmem;
  const uint32_t base = smem_u32(sh), keys = base + S::kQBytes, values = keys + kKeyRing * S::kTileBytes;
  volatile int* stop = &b.abort;
  const auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity & 1, a.c.status, stop); };

  SharedPlace pl;
  pl.enter(p, b.group);
  pl.item = static_cast<int>(b.tile / pl.tiles);
  pl.t = static_cast<int>(b.tile % pl.tiles);

  if (warp < 4) {
    // ---- softmax: row `tid` of the item's queries
    const uint32_t mine_at = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    const float lift = kLift<T>;
    float m = -INFINITY, l = 0.f;
    bool begins = true, from_start = pl.t == 0;
    int have = 0, q0 = 0, kh = 0;
    for (int n = 0; n < run; ++n) {
      if (begins) {
        const int mb = pl.blocks(p);
        kh = pl.item / mb;
        q0 = pl.item % mb * kM;                // of the group's rows (member, head)
        have = min(kM, pl.gr.count * a.group - q0);
        // (the last item's scores are done with the queries)
        const T* q = static_cast<const T*>(a.q.p) + kh * a.group * a.q.head;
        for (int e = tid; e < kM * VPR; e += 128) {
          const int r = e / VPR, x = e % VPR, i = (q0 + r) / a.group, h = (q0 + r) % a.group;
          const bool on = r < have;
          cp_async16_or_zero(base + (x >> 3) * (kM * 128) + r * 128 + (((x & 7) ^ (r & 7)) << 4),
                             q + (on ? static_cast<long long>(pl.gr.first + i) * a.q.row + h * a.q.head : 0) + x * 8, on);
        }
        cp_async_commit();
        cp_async_wait_group<0>();
        fence_proxy_async_smem();
        mbar_arrive(&b.q_full);
        m = -INFINITY;
        l = 0.f;
      }
      if (!wait(&b.s_full, n)) break;
      tc_fence_after();
      const bool busy = warp * 32 < have;      // rows of this warp hold queries
      uint32_t z[kN];
      if (busy) {
        tmem_ld32(mine_at, *reinterpret_cast<uint32_t(*)[32]>(z));
        tmem_ld32(mine_at + 32, *reinterpret_cast<uint32_t(*)[32]>(z + 32));
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.s_free);
      float f = 1.f;
      if (busy) {
        const int valid = pl.gr.rows - pl.t * kN;
        float top = m;
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          float x = __uint_as_float(z[j]) * a.scale2;
          if (valid < kN && j >= valid) x = -INFINITY;
          z[j] = __float_as_uint(x);
          top = fmaxf(top, x);
        }
        const float at = top == -INFINITY ? 0.f : top;
        f = exp2_fast(m - at);
        m = top;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < kN; j += 2) {
          const float x = exp2_fast(__uint_as_float(z[j]) - (at - lift)), y = exp2_fast(__uint_as_float(z[j + 1]) - (at - lift));
          sum += x + y;
          split_weights(x, y, z[j], z[j + 1], T());
        }
        l = l * f + sum;
      }
      // the last tile's product is done: its sums can be scaled, its weights overwritten
      if (n > 0 && !wait(&b.o_done, n - 1)) break;
      tc_fence_after();
      if (busy) {
        if (!begins && __any_sync(0xffffffffu, f != 1.f)) {
#pragma unroll 1
          for (int x = 0; x < DH; x += 16) {
            uint32_t o[16];
            tmem_ld16(mine_at + S::kO + x, o);
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
            tmem_st16(mine_at + S::kO + x, o);
          }
        }
        uint32_t w[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) w[j] = z[2 * j];
        tmem_st32(mine_at + S::kHi, w);
#pragma unroll
        for (int j = 0; j < 32; ++j) w[j] = z[2 * j + 1];
        tmem_st32(mine_at + S::kLo, w);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.p_full);

      const bool ends = pl.t + 1 == pl.tiles;
      if (ends || n + 1 == run) {
        if (!wait(&b.o_done, n)) break;
        tc_fence_after();
        const bool done = ends && from_start, on = tid < have;
        const int i = pl.gr.first + (q0 + tid) / a.group, head = kh * a.group + (q0 + tid) % a.group;
        const long long at = static_cast<long long>(i) * a.q.heads + head;
        float* part = p.parts + static_cast<long long>(2 * blockIdx.x + (from_start ? 1 : 0)) * S::kPart;
        if (busy) {
#pragma unroll 1
          for (int x = 0; x < DH; x += 16) {
            uint32_t o[16];
            tmem_ld16(mine_at + S::kO + x, o);
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
              const float4 v = make_float4(__uint_as_float(o[j]), __uint_as_float(o[j + 1]), __uint_as_float(o[j + 2]), __uint_as_float(o[j + 3]));
              if (!on) continue;
              if (done) *reinterpret_cast<float4*>(p.whole + at * DH + x + j) = v;
              else *reinterpret_cast<float4*>(part + 2 * kM + ((x + j) / 4 * kM + tid) * 4) = v;
            }
          }
          if (on && done) p.whole_stats[at] = make_float2(m, l);
          if (on && !done) {
            part[tid] = m;
            part[kM + tid] = l;
          }
        }
        tc_fence_before();
      }
      begins = pl.next(p);
      if (begins) from_start = true;
    }
  } else if (warp < 8) {
    // ---- loads: the rows 32 w .. 32 w + 31 of each tile a warp, a row's page by the lane of that number
    const bool of_keys = warp < 6;
    const int w = warp & 1, stages = of_keys ? kKeyRing : kValueRing;
    uint64_t *full = of_keys ? b.k_full : b.v_full, *empty = of_keys ? b.k_empty : b.v_empty;
    const uint32_t ring = of_keys ? keys : values;
    const T* from = static_cast<const T*>(a.pk) + (of_keys ? 0 : a.plane);
    const auto page_of = [&]() -> int {
      const int tok = pl.t * kN + w * 32 + lane;
      if (pl.g >= p.groups || tok >= pl.gr.rows) return 0;
      return __ldg(a.c.table + static_cast<long long>(pl.gr.seq) * a.c.max_pages + (a.page_shift >= 0 ? tok >> a.page_shift : tok / a.c.page));
    };
    int pid = page_of(), slot = 0, last = 0;
    uint32_t turn = 1;                         // parity of `empty`: the first pass finds the slots free
    bool ok = true;
    for (int n = 0; n < run; ++n) {
      ok = wait(&empty[slot], turn);
      if (!ok) break;
      const int tok = pl.t * kN + w * 32 + lane, valid = pl.gr.rows - pl.t * kN - w * 32;
      const int kh = pl.item / pl.blocks(p);
      if (tok < pl.gr.rows && !good_page(a.c, pid)) {
        atomicOr(a.c.status, ST_BADINDEX);
        pid = 0;
      }
      const int in_page = a.page_shift >= 0 ? tok & (a.c.page - 1) : tok % a.c.page;
      const long long row = lane < valid ? ((static_cast<long long>(pid) * a.c.heads + kh) * a.c.page + in_page) * DH : 0;
      pl.next(p);
      pid = page_of();
      const uint32_t dst = ring + slot * S::kTileBytes + w * 32 * 128;
#pragma unroll
      for (int j = 0; j < VPR; ++j) {
        const int e = lane + 32 * j, r = e / VPR, x = e % VPR;
        const long long src = __shfl_sync(0xffffffffu, row, r) + x * 8;
        cp_async16_or_zero(dst + (x >> 3) * (kN * 128) + r * 128 + (((x & 7) ^ (r & 7)) << 4), from + src, r < valid);
      }
      cp_async_commit();
      if (n > 0) {
        cp_async_wait_group<1>();
        fence_proxy_async_smem();
        mbar_arrive(&full[last]);
      }
      last = slot;
      if (++slot == stages) {
        slot = 0;
        turn ^= 1;
      }
    }
    cp_async_wait_group<0>();
    fence_proxy_async_smem();
    if (ok) mbar_arrive(&full[last]);
  } else if (elect_one()) {
    // ---- products
    constexpr uint32_t kScores = idesc_of<T>(kM, kN), kSums = idesc_of<T>(kM, DH) | 1u << 16;
    const uint64_t qd = desc_sw128(base), kd = desc_sw128(0), vd = desc_sw128_mn(0);
    bool ok = true, first = true;              // of an item's tiles in this run
    int vslot = 0;
    uint32_t vturn = 0;
    const auto weigh = [&](int n) {            // sums += weights of tile n * values
      ok = ok && wait(&b.p_full, n) && wait(&b.v_full[vslot], vturn);
      if (!ok) return;
      tc_fence_after();
      const uint32_t at = values + vslot * S::kTileBytes;
#pragma unroll
      for (int k = 0; k < kN / 16; ++k) umma_ts(tmem + S::kO, tmem + S::kHi + 8 * k, vd + ((at + k * 2048) >> 4), kSums, !first || k != 0);
#pragma unroll
      for (int k = 0; k < kN / 16; ++k) umma_ts(tmem + S::kO, tmem + S::kLo + 8 * k, vd + ((at + k * 2048) >> 4), kSums, 1);
      first = false;
      umma_commit(&b.v_empty[vslot]);
      umma_commit(&b.o_done);
      if (++vslot == kValueRing) {
        vslot = 0;
        vturn ^= 1;
      }
    };
    int kslot = 0, item = 0;
    uint32_t kturn = 0;
    bool begins = true;
    for (int n = 0; n < run && ok; ++n) {
      if (begins) {
        if (n > 0) weigh(n - 1);
        first = true;
        ok = ok && wait(&b.q_full, item++);
      }
      ok = ok && (n == 0 || wait(&b.s_free, n - 1)) && wait(&b.k_full[kslot], kturn);
      if (!ok) break;
      tc_fence_after();
      const uint32_t at = keys + kslot * S::kTileBytes;
#pragma unroll
      for (int k = 0; k < DH / 16; ++k)
        umma_bf16(tmem, qd + (((k >> 2) * (kM * 128) + (k & 3) * 32) >> 4), kd + ((at + (k >> 2) * (kN * 128) + (k & 3) * 32) >> 4), kScores, k != 0);
      umma_commit(&b.k_empty[kslot]);
      umma_commit(&b.s_full);
      if (++kslot == kKeyRing) {
        kslot = 0;
        kturn ^= 1;
      }
      if (!begins) weigh(n - 1);
      begins = pl.next(p);
    }
    if (ok) weigh(run - 1);
    umma_commit(&b.drain);                     // all products have ended, whatever came before
    mbar_wait(&b.drain, 0, a.c.status, nullptr);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kCols);
  }
}

// ---- the join: 8 rows (entry, head of a key head) by dh / 4 pieces of four columns a block.
template <typename T>
__global__ void __launch_bounds__(512) shared_join_kernel(const __grid_constant__ SharedArgs p) {
  pdl_enter();
  const AttendArgs& a = p.a;
  const int dh = a.c.dh, kh = blockIdx.y, x = 4 * (threadIdx.x / 8);
  const long long row = static_cast<long long>(blockIdx.x) * 8 + threadIdx.x % 8;
  if (row >= static_cast<long long>(a.n) * a.group) return;
  const int i = static_cast<int>(row / a.group), head = kh * a.group + static_cast<int>(row % a.group);
  T* out = static_cast<T*>(a.out.p) + i * a.out.row + head * a.out.head + x;
  const int s = __ldg(a.seqs + i);
  if (s < 0 || s >= a.c.seqs) {
    if (s != -1 && x == 0) atomicOr(a.c.status, ST_BADINDEX);
    return;
  }
  const int len = seq_len(a, i), skip = __ldcg(p.skip + i);
  if (len == 0) {
    if (x == 0 && __ldg(a.c.len + s) != 0) atomicOr(a.c.status, ST_BADINDEX);
    store4(out, make_float4(0.f, 0.f, 0.f, 0.f));
    return;
  }
  const long long at = static_cast<long long>(i) * a.q.heads + head;
  float top = -INFINITY, l = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto add = [&](float m, float sum, float4 y) {
    const float next = fmaxf(top, m), by = next == -INFINITY ? 0.f : next, f = exp2_fast(top - by), h = exp2_fast(m - by);
    top = next;
    l = l * f + sum * h;
    v = make_float4(v.x * f + y.x * h, v.y * f + y.y * h, v.z * f + y.z * h, v.w * f + y.w * h);
  };
  if (skip > 0) {
    const int g = __ldcg(p.of + i);
    const int4 gr = __ldcg(reinterpret_cast<const int4*>(p.group + g));
    const int tiles = pieces_of(gr.z, kN), blocks = (gr.y * a.group + kM - 1) / kM;
    const int q = (i - gr.x) * a.group + static_cast<int>(row % a.group), r = q % kM;
    const long long total = __ldcg(p.tile0 + p.groups), per = (total + p.grid - 1) / p.grid;
    const long long tile = __ldcg(p.tile0 + g) + static_cast<long long>(kh * blocks + q / kM) * tiles;
    const int c0 = static_cast<int>(tile / per), c1 = static_cast<int>((tile + tiles - 1) / per);
    if (c0 == c1) {
      const float2 st = __ldcg(p.whole_stats + at);
      add(st.x, st.y, __ldcg(reinterpret_cast<const float4*>(p.whole + at * dh + x)));
    } else {
      const long long size = static_cast<long long>(kM) * (dh + 2);
#pragma unroll 4
      for (int c = c0; c <= c1; ++c) {
        const float* part = p.parts + (2ll * c + (c == c0 ? 1 : 0)) * size;
        add(__ldcg(part + r), __ldcg(part + kM + r), __ldcg(reinterpret_cast<const float4*>(part + 2 * kM + (x / 4 * kM + r) * 4)));
      }
    }
  }
  if (len > skip) {
    const float2 st = __ldcg(a.stats + at);
    add(st.x, st.y, __ldcg(reinterpret_cast<const float4*>(a.own + at * dh + x)));
  }
  store4(out, make_float4(v.x / l, v.y / l, v.z / l, v.w / l));
}

template <typename T, int DH>
cudaError_t launch_shared_width(const SharedArgs& p, cudaStream_t st) {
  using S = Shape<DH>;
  cudaError_t e = cudaFuncSetAttribute(shared_kernel<T, DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
  if (e == cudaSuccess) e = launch_k(shared_kernel<T, DH>, dim3(p.grid), dim3(kSharedThreads), S::kSmem, st, p);
  return e;
}
template <typename T>
cudaError_t launch_shared(const SharedArgs& p, cudaStream_t st) {
  switch (p.a.c.dh) {
    case 64: return launch_shared_width<T, 64>(p, st);
    case 80: return launch_shared_width<T, 80>(p, st);
    case 96: return launch_shared_width<T, 96>(p, st);
    case 128: return launch_shared_width<T, 128>(p, st);
    case 192: return launch_shared_width<T, 192>(p, st);
    default: return launch_shared_width<T, 256>(p, st);
  }
}

constexpr int shared_grid(int dh) { return 152 * (dh <= 128 ? 2 : 1); }

struct SharedSpace { size_t group, of, skip, tile0, stats, own, whole_stats, whole, parts, bytes; };
SharedSpace shared_space(const map_cache* c, long long heads, long long n, long long groups) {
  SharedSpace s;
  size_t at = (map_cache_attend_workspace(c) + 255) / 256 * 256;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  s.group = take(groups * sizeof(Group));
  s.of = take(n * 4);
  s.skip = take(n * 4);
  s.tile0 = take((groups + 1) * 8);
  s.stats = take(n * heads * sizeof(float2));
  s.own = take(n * heads * c->dh * 4);
  s.whole_stats = take(n * heads * sizeof(float2));
  s.whole = take(n * heads * c->dh * 4);
  s.parts = take(2ull * shared_grid(c->dh) * kM * (c->dh + 2) * 4);
  s.bytes = at;
  return s;
}

}  // namespace
}  // namespace mapk

using namespace mapk;

extern "C" {

size_t map_cache_attend_shared_workspace(const map_cache* c, int heads, int n, int groups) {
  if (check_cache(c) != MAP_OK || heads < 1 || heads > 65535 || n < 0 || n > 65535 || groups < 1 || groups > 65535) return 0;
  return shared_space(c, heads, n, groups).bytes;
}

int map_cache_attend_shared(const map_cache* c, int layer, const map_heads* q, const int32_t* seqs, int n, const int32_t* starts,
                            int groups, float scale, const map_heads* out, void* ws, void* stream) {
  SharedArgs p{};
  AttendArgs& a = p.a;
  const int rc = attend_args(c, layer, q, seqs, n, scale, out, ws, a);
  if (rc != MAP_OK) return rc;
  if (groups < 1) return MAP_EINVAL;
  if (groups > 65535) return MAP_EUNSUPPORTED;
  if (a.n == 0) return MAP_OK;
  if (!starts) return MAP_EINVAL;
  const SharedSpace s = shared_space(c, q->heads, n, groups);
  char* w = static_cast<char*>(ws);
  p.starts = starts;
  p.groups = groups;
  p.group = reinterpret_cast<Group*>(w + s.group);
  p.of = reinterpret_cast<int32_t*>(w + s.of);
  p.skip = reinterpret_cast<int32_t*>(w + s.skip);
  p.tile0 = reinterpret_cast<long long*>(w + s.tile0);
  p.parts = reinterpret_cast<float*>(w + s.parts);
  p.whole_stats = reinterpret_cast<float2*>(w + s.whole_stats);
  p.whole = reinterpret_cast<float*>(w + s.whole);
  p.grid = shared_grid(c->dh);
  a.skip = p.skip;
  a.stats = reinterpret_cast<float2*>(w + s.stats);
  a.own = reinterpret_cast<float*>(w + s.own);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool half = c->type == MAP_F16;
  cudaError_t e = launch_k(shared_plan_kernel, dim3(groups), dim3(kPlan), 0, st, p);
  if (e == cudaSuccess) e = half ? launch_shared<__half>(p, st) : launch_shared<__nv_bfloat16>(p, st);
  if (e == cudaSuccess) e = launch_attend<kOwn>(a, st);
  if (e == cudaSuccess) {
    const dim3 grid(static_cast<unsigned>((static_cast<long long>(n) * a.group + 7) / 8), c->heads), block(8 * (c->dh / 4));
    e = half ? launch_k(shared_join_kernel<__half>, grid, block, 0, st, p) : launch_k(shared_join_kernel<__nv_bfloat16>, grid, block, 0, st, p);
  }
  return launch_err(e);
}

}  // extern "C"
