// Attention of single tokens for groups of sequences that begin with the same pages (map_cache_attend_shared).
//
// Mathematics.  The rows t < S of a group are the same for all of its sequences, so that their part of every member's attention
// (m, l, o: largest score, sum of weights, unnormalised output) is a product of all the members' queries of a key head with one
// set of keys and values; the rows from S on are each member's own (attend's kernel), and the parts join as in attend.
//
// Bound: HBM, a group's shared rows once and the others once a sequence; 4 S dh operations a query head beside them (6 with the
// weights in two halves), on the tensor cores as much as the loads from about 200 query heads a key head on; for groups of a few
// sequences the chain of four launches.
// The launches: what is shared, the shared rows, the sequences' own rows, the join.  The own rows' kernel starts on the SMs that the
// shared rows leave free.  (The other order took 3 us more for 64 questions and 6 more for the video below.)
// Measured, 128 columns: 4 questions on 611 rows, 32 heads over 32: 22 us (plan 4, shared rows 9, join 5, launches); 64 questions on
// 2915 rows, 32 over 8: 42.5 us (plan 6, shared rows done at 22 and own rows at 30, join 7 of 17 MB of parts); 8 groups of 8 on up to
// 1315 rows, 28 over 4: 33 us; 32 answers on 60001 rows, 28 over 4, fp16: 69 us, of which the shared rows take 48, 123 MB at
// 2.5 TB/s and tensor cores 48 % busy.
#include <type_traits>

#include "attend.cuh"

namespace mapk {
namespace {

// A group: entries first .. first + count - 1, whose sequences' first `rows` rows are those of sequence `seq`.  Below 0: nothing is
// shared here, nor in the next -rows - 1 groups (skip_groups).
struct Group { int first, count, rows, seq; };

struct SharedArgs {
  AttendArgs a;
  const int32_t* starts;
  int groups;
  Group* group;                                // [groups]
  Entry* entries;                              // [n]
  long long* tile0;                            // [groups + 1] tiles before a group, and those of a CTA (the list of shared_kernel)
  float* parts;                                // [grid][2] parts of items that several CTAs share
  float2* whole_stats;                         // the others': (m, l) [n][q.heads]
  float* whole;                                //         o [n][q.heads][dh]
  int grid, m, box;                            // of shared_kernel: its CTAs, query rows of an item, rows of a TMA box (0: none)
};

constexpr int kPlan = 1024, kPlanEach = 8;

// An entry's sequence (-1: padding, a bad one, or no entry) and its rows (0 where the length is bad).
struct Member { int seq, len; bool bad; };
__device__ __forceinline__ Member member(const AttendArgs& a, int i, int last) {
  const int s = i < last ? __ldg(a.seqs + i) : -1;
  if (s < 0 || s >= a.c.seqs) return {-1, 0, s != -1};
  const int len = __ldg(a.c.len + s);
  return good_len(a.c, len) ? Member{s, len, false} : Member{s, 0, true};
}

// What a group shares: the pages that all its sequences with rows hold in front, as far as all are full.  Latency: a cluster a group;
// every CTA looks all of the group's sequences up, together, and compares a part of their pages.
__global__ void __launch_bounds__(kPlan) shared_plan_kernel(const __grid_constant__ SharedArgs p, int ranks) {
  const AttendArgs& a = p.a;
  __shared__ int least, lead, valid;
  __shared__ int seq[kPlan];                   // of kPlan members; -1: without rows
  pdl_enter();
  const int g = blockIdx.x / ranks, rank = blockIdx.x % ranks, tid = threadIdx.x;
  if (tid == 0) {
    least = a.c.max_pages;
    lead = a.n;
    valid = 0;
  }
  int first = __ldg(p.starts + g), last = __ldg(p.starts + g + 1);
  bool bad = false;                            // (every CTA looks at all of it: no more than 65536 numbers)
  for (int i = tid; i <= p.groups; i += kPlan) {
    const int s = __ldg(p.starts + i), next = i < p.groups ? __ldg(p.starts + i + 1) : a.n;
    bad |= s > next || (i == 0 && s != 0) || (i == p.groups && s != a.n);
  }
  const bool refused = __syncthreads_or(bad) != 0;           // nothing is shared then
  if (refused && blockIdx.x == 0 && tid == 0) atomicOr(a.c.status, ST_BADINDEX);
  if (refused) first = last = 0;
  Member own = member(a, first + tid, last);   // of the first kPlan, which most groups do not pass
  seq[tid] = own.len > 0 ? own.seq : -1;
  int mine = 0, from = a.n, pages = a.c.max_pages;
  for (int i = first + tid; i < last; i += kPlan) {
    const int len = i == first + tid ? own.len : member(a, i, last).len;
    if (len <= 0) continue;
    ++mine;
    from = min(from, i);
    pages = min(pages, len / a.c.page);
  }
  mine = __reduce_add_sync(0xffffffffu, mine);
  from = __reduce_min_sync(0xffffffffu, from);
  pages = __reduce_min_sync(0xffffffffu, pages);
  if (tid % 32 == 0 && mine) {
    atomicAdd(&valid, mine);
    atomicMin(&lead, from);
    atomicMin(&least, pages);
  }
  __syncthreads();
  const int of = lead, full = valid > 1 ? least : 0;
  const int lead_seq = full == 0 ? 0 : of < first + kPlan ? seq[of - first] : __ldg(a.seqs + of);
  __syncthreads();
  if (full > 0) {
    int same = full;
    const int32_t* row = a.c.table + static_cast<long long>(lead_seq) * a.c.max_pages;
    for (int i0 = first; i0 < last; i0 += kPlan) {
      const int count = min(kPlan, last - i0);
      if (i0 > first) {
        __syncthreads();
        const Member m = member(a, i0 + tid, last);
        seq[tid] = m.len > 0 ? m.seq : -1;
        __syncthreads();
      }
      const long long all = static_cast<long long>(count) * full;
      for (long long x0 = rank * kPlan + tid; x0 < all; x0 += kPlan * kPlanEach * ranks) {
        int j[kPlanEach], page[kPlanEach], other[kPlanEach];
#pragma unroll
        for (int k = 0; k < kPlanEach; ++k) {
          const long long x = x0 + k * kPlan * ranks;
          const int m = x < all ? (all < (1ll << 31) ? static_cast<int>(x) / full : static_cast<int>(x / full)) : 0;
          const int s = x < all ? seq[m] : -1;
          j[k] = static_cast<int>(x - static_cast<long long>(m) * full);
          page[k] = other[k] = 0;
          if (s >= 0) {
            page[k] = __ldg(a.c.table + static_cast<long long>(s) * a.c.max_pages + j[k]);
            other[k] = __ldg(row + j[k]);
          }
        }
#pragma unroll
        for (int k = 0; k < kPlanEach; ++k)
          if (page[k] != other[k]) same = min(same, j[k]);
      }
    }
    same = __reduce_min_sync(0xffffffffu, same);
    if (tid % 32 == 0) atomicMin(&least, same);
  }
  int shared = 0;
  if (ranks > 1) {                             // (full is the same in all of the cluster)
    cluster_sync();
    shared = a.c.max_pages;
    for (int r = 0; r < ranks; ++r) {
      int v;
      asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(mapa_u32(&least, r)) : "memory");
      shared = min(shared, v);
    }
    cluster_sync();                            // no CTA leaves while another may read
  } else {
    __syncthreads();
    shared = least;
  }
  const int rows = full > 0 ? shared * a.c.page : 0;
  // entries of the group; all of them where nothing is shared because the groups are bad
  const int e0 = refused ? 0 : first, e1 = refused ? a.n : last;
  const int block = refused ? static_cast<int>(blockIdx.x) : rank, blocks = refused ? static_cast<int>(gridDim.x) : ranks;
  for (int i = e0 + block * kPlan + tid; i < e1; i += blocks * kPlan) {
    const Member m = i == first + tid && !refused ? own : member(a, i, e1);
    Entry e{rows, g, m.len - rows, 0};
    if (m.len <= 0) e = Entry{m.seq < 0 ? -2 : -1, 0, 0, 0};
    if (m.bad) atomicOr(a.c.status, ST_BADINDEX);
    *reinterpret_cast<int4*>(p.entries + i) = make_int4(e.skip, e.group, e.own, 0);
  }
  if (tid == 0 && rank == 0) p.group[g] = Group{first, last - first, rows, lead_seq};
}

// ---- the shared rows.  An item is up to M = 128 MT rows of queries (member, head) of one key head and group, 128 the M of a
// tcgen05.mma.  64 keys are the N of the scores' product and the K of the values', whose first operand, the weights as two halves
// of T, lies in TMEM.  Four warps for each 128 rows do the softmax, a row a thread (two threads a row, twice the warps: no
// faster); a warp loads keys and one values, each with a ring of its own; a thread of a warp for each 128 rows issues the
// products: a tile's scores while the last one's weights are made, which take the place of theirs.
constexpr int kM = 128, kN = 64;

template <int DH, int MT>
struct Shape {
  static constexpr int kThreads = 128 * MT + 128;
  static constexpr int kBlocks = (DH + 63) / 64;             // boxes of 64 columns, 128 bytes a row, 16-byte units exchanged by the row's low bits
  static constexpr int kTileBytes = kBlocks * kN * 128, kQBytes = kBlocks * MT * kM * 128;
  static constexpr int kCtas = MT == 1 && DH <= 128 ? 2 : 1;
  static constexpr int kRing = (227 * 1024 / kCtas - 3 * 1024 - kQBytes) / kTileBytes;           // tiles that fit
  static constexpr int kKeyRing = kRing >= 8 ? 4 : (kRing + 1) / 2, kValueRing = kRing >= 8 ? 4 : kRing / 2;
  static constexpr int kTiles = kQBytes + (kKeyRing + kValueRing) * kTileBytes;
  static constexpr int kSmem = kTiles + 512 + MT * kM * 8;   // the barriers and the queries' places behind the tiles
  static constexpr int kLo = kN / 2, kO = 2 * kN;            // TMEM columns of 128 rows: two tiles' scores, weights in their place; sums
  static constexpr int kCols = kO + DH <= 256 ? 256 : 512;
  static_assert(kKeyRing <= 4 && kValueRing >= 2 && kCtas * (kSmem + 1024) <= 228 * 1024 && kCtas * MT * kCols <= 512, "an SM");
};

constexpr uint32_t kBf16Types = (1u << 7) | (1u << 10);      // of an instruction descriptor: A and B
template <typename T>
__host__ __device__ constexpr uint32_t idesc_of(int m, int n) {
  return std::is_same<T, __half>::value ? idesc_bf16(m, n) & ~kBf16Types : idesc_bf16(m, n);
}

// A descriptor's low half, which has the address; the high half is the same for all (desc_sw128, desc_sw128_mn).  The 64-bit sums
// of an address cost more to issue than the product takes.
__device__ __forceinline__ uint32_t desc_low(uint32_t at) { return static_cast<uint32_t>(desc_sw128(0)) | at >> 4; }
__device__ __forceinline__ uint32_t desc_low_mn(uint32_t at) { return static_cast<uint32_t>(desc_sw128_mn(0)) | at >> 4; }
__device__ __forceinline__ uint32_t desc_high() { return static_cast<uint32_t>(desc_sw128(0) >> 32); }

// D[tmem] (+)= A[smem] * B[smem].
template <bool ACC>
__device__ __forceinline__ void umma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tmov.b64 x, {%1, %4};\n\tmov.b64 y, {%2, %4};\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(desc_high()), "n"(ACC)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: A's 16-bit columns two to a 32-bit one.
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tmov.b64 y, {%2, %4};\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(desc_high()), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}

// 8 columns of the warp's 32 TMEM lanes, completed by tmem_wait_st.
__device__ __forceinline__ void tmem_put8(uint32_t at, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two fp32 at once: half the instructions.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// Weights as two halves like split_weights, two at once: both halves of a weight above zero are raised to their type's smallest
// number, those of a weight of zero are zero.  Weights are 2^kLift times what they are to the row's base, which the largest score
// passes by kSlack at most: sums are scaled only then, not whenever a tile has a greater score.  fp16 has room for a little less
// than 2^16, so that a half that is raised adds 2^-39 of the base's weight there as in split_weights.  (A smaller lift under a
// slack of 4 and halves raised whatever the weight took 4 to 5 us less of the video's 69 above and added 2^-34 a row.)
template <typename T> constexpr float kSlack = 8.f;
template <> constexpr float kSlack<__half> = 0.99f;
__device__ __forceinline__ uint32_t min_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ void halves(float2 x, uint32_t& hi, uint32_t& lo, __nv_bfloat16) {
  const uint32_t a = __float_as_uint(x.x), b = __float_as_uint(x.y);
  hi = __byte_perm(a, b, 0x7632);
  const uint32_t least = min_u16x2(hi, 0x00800080u);         // 2^-126 where x is above zero (ex2 gives no subnormal numbers)
  const float2 rest = fma2(make_float2(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u)), make_float2(-1.f, -1.f), x);
  const __nv_bfloat162 r = __hmax2(__floats2bfloat162_rn(rest.x, rest.y), *reinterpret_cast<const __nv_bfloat162*>(&least));
  lo = *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ void halves(float2 x, uint32_t& hi, uint32_t& lo, __half) {
  asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(x.y), "f"(x.x));
  const uint32_t some = min_u16x2(__byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x7632), 0x00010001u);     // 2^-24 likewise
  const __half2 least = *reinterpret_cast<const __half2*>(&some), h = __hmax2_nan(*reinterpret_cast<const __half2*>(&hi), least);
  const float2 rest = fma2(__half22float2(h), make_float2(-1.f, -1.f), x);
  const __half2 r = __hmax2(__floats2half2_rn(rest.x, rest.y), least);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  lo = *reinterpret_cast<const uint32_t*>(&r);
}

// Where a run of the list (group, key head, rows of queries, tile) is.
struct SharedPlace {
  Group gr;
  int g, item, items, tiles, t;
  __device__ __forceinline__ void enter(const SharedArgs& p, int from) {
    tiles = 0;
    for (g = from; g < p.groups; g += max(1, -gr.rows)) {
      const int4 x = __ldcg(reinterpret_cast<const int4*>(p.group + g));
      gr = Group{x.x, x.y, x.z, x.w};
      if (gr.rows > 0) break;
    }
    if (g >= p.groups) return;
    tiles = pieces_of(gr.rows, kN);
    items = p.a.c.heads * blocks(p);
  }
  __device__ __forceinline__ int blocks(const SharedArgs& p) const { return (gr.count * p.a.group + p.m - 1) / p.m; }
  // query rows of the item
  __device__ __forceinline__ int have(const SharedArgs& p) const { return min(p.m, gr.count * p.a.group - item % blocks(p) * p.m); }
  __device__ __forceinline__ bool next(const SharedArgs& p) {          // whether another item begins
    if (++t < tiles) return false;
    t = 0;
    if (++item < items) return true;
    item = 0;
    enter(p, g + 1);
    return true;
  }
};

// Of more groups than kWalked every CTA notes, behind each of its run that shares rows, how many that do not come next; going through them
// one at a time takes 0.3 us each.  (Of 1000 groups three share: 51 us, 289 without; of 60000: 3.5 ms, of which the plan is the
// most, and 19.5.  Done in line for 1 to 8 groups it took 0.8 us more.)  A thread has groups g0 .. g1 - 1, in the run or not;
// `lead` is a word a warp.
constexpr int kWalked = 8;
__device__ __noinline__ void skip_groups(Group* group, int groups, int g0, int g1, bool in_run, int* lead) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int first = groups, behind = groups;         // that share rows: of this thread's, behind them
  for (int g = g1 - 1; g >= g0; --g)
    if (__ldcg(&group[g].rows) > 0) first = g;
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_down_sync(0xffffffffu, first, o);
    if (lane + o < 32) {
      behind = min(behind, u);
      first = min(first, u);
    }
  }
  if (lane == 0) lead[warp] = first;
  __syncthreads();
  if (!in_run) return;
  for (int w = warp + 1; w < warps; ++w) behind = min(behind, lead[w]);
  for (int g = g1 - 1; g >= g0; --g)
    if (__ldcg(&group[g].rows) > 0) {
      if (behind > g + 1) group[g + 1].rows = g + 1 - behind;          // (CTAs that write it write the same, and who reads it looks for rows above 0)
      behind = g;
    }
}

struct SharedBars {
  uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4], q_full[2], s_full[2][2], p_full[2][2], o_done[2][2], drain;
  uint32_t tmem;
  int abort, group;
  long long tile;
  long long red[12];
  int lead[12];
};
static_assert(sizeof(SharedBars) <= 512, "behind the tiles");

template <typename T, int DH, int MT>
__global__ void __launch_bounds__(Shape<DH, MT>::kThreads, Shape<DH, MT>::kCtas)
    shared_kernel(const __grid_constant__ SharedArgs p, const __grid_constant__ CUtensorMap map) {
  using S = Shape<DH, MT>;
  constexpr int VPR = DH / 8, kWarpsAll = S::kThreads / 32, kKeys = 4 * MT, kValues = kKeys + 1, kProducts = kKeys + 2;
  extern __shared__ __align__(1024) unsigned char tile_mem[];
  SharedBars& b = *reinterpret_cast<SharedBars*>(tile_mem + S::kTiles);
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
  const int each = (p.groups + S::kThreads - 1) / S::kThreads, g0 = min(p.groups, tid * each), g1 = min(p.groups, g0 + each);
  long long mine = 0, total;
  for (int g = g0; g < g1; ++g) mine += tiles_of(g);
  long long at0 = block_prefix<kWarpsAll>(mine, b.red, &total);
  const long long per = (total + gridDim.x - 1) / gridDim.x, t0 = per * blockIdx.x;
  if (blockIdx.x == 0) {
    long long at = at0;
    for (int g = g0; g < g1; ++g) {
      p.tile0[g] = at;
      at += tiles_of(g);
    }
    if (tid == 0) p.tile0[p.groups] = per;
  }
  if (t0 >= total || (smem_u32(tile_mem) & 1023) != 0) {           // (the alignment is what its declaration asks for)
    if (t0 < total && tid == 0) atomicOr(a.c.status, ST_INTERNAL);
    return;
  }
  const int run = static_cast<int>(t0 + per <= total ? per : total - t0);
  if (p.groups > kWalked) skip_groups(p.group, p.groups, g0, g1, mine > 0 && at0 < t0 + run && t0 < at0 + mine, b.lead);
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
    for (int i = 0; i < 4; ++i) {
      mbar_init(&b.k_full[i], p.box > 0 ? 1 : 32);
      mbar_init(&b.k_empty[i], MT);
      mbar_init(&b.v_full[i], p.box > 0 ? 1 : 32);
      mbar_init(&b.v_empty[i], MT);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&b.q_full[i], 128);
      for (int j = 0; j < 2; ++j) {            // (scores, and some of the warps, can be a tile ahead of the others: by the tile's parity)
        mbar_init(&b.s_full[i][j], 1);
        mbar_init(&b.p_full[i][j], 4);
        mbar_init(&b.o_done[i][j], 1);
      }
    }
    mbar_init(&b.drain, MT);
    b.abort = 0;
    fence_mbar_init();
  }
  if (warp == kProducts) {
    tmem_alloc(&b.tmem, MT * S::kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = b.tmem;
  const uint32_t base = smem_u32(tile_mem), keys = base + S::kQBytes, values = keys + S::kKeyRing * S::kTileBytes;
  volatile int* stop = &b.abort;
  const auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity & 1, a.c.status, stop); };

  SharedPlace pl;
  pl.enter(p, b.group);
  pl.item = static_cast<int>(b.tile / pl.tiles);
  pl.t = static_cast<int>(b.tile % pl.tiles);

  if (warp < kKeys) {
    // ---- softmax: row `tid` of the item's queries
    const int mt = MT > 1 ? warp >> 2 : 0;
    const uint32_t mine_at = tmem + mt * S::kCols + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    long long* q_at = reinterpret_cast<long long*>(tile_mem + S::kTiles + 512);    // where the rows' queries are
    float m = -INFINITY, l = 0.f;
    bool begins = true, from_start = pl.t == 0;
    int have = 0, q0 = 0, kh = 0;
    uint32_t count = 0;                        // tiles of these 128 rows so far
    for (int n = 0; n < run; ++n) {
      if (begins) {
        const int mb = pl.blocks(p);
        kh = pl.item / mb;
        q0 = pl.item % mb * p.m;               // of the group's rows (member, head)
        have = pl.have(p);
        if (mt * kM < have) {                  // (these rows' last scores are done with the queries)
          const int i = pl.gr.first + (q0 + tid) / a.group, h = kh * a.group + (q0 + tid) % a.group;
          q_at[tid] = tid < have ? i * a.q.row + h * a.q.head : -1;
          asm volatile("bar.sync %0, 128;" ::"r"(1 + mt) : "memory");
          const T* q = static_cast<const T*>(a.q.p);
#pragma unroll 4
          for (int j = 0; j < VPR; ++j) {
            const int e = (tid & 127) + 128 * j, row = e / VPR, x = e % VPR;
            const long long at = q_at[mt * kM + row];
            cp_async16_or_zero(base + mt * (S::kQBytes / MT) + (x >> 3) * (kM * 128) + row * 128 + (((x & 7) ^ (row & 7)) << 4),
                               q + (at < 0 ? 0 : at) + x * 8, at >= 0);
          }
          cp_async_commit();
          cp_async_wait_group<0>();
          fence_proxy_async_smem();
          mbar_arrive(&b.q_full[mt]);
        }
        m = -INFINITY;
        l = 0.f;
      }
      if (mt * kM < have) {
        const bool busy = warp * 32 < have;    // rows of this warp hold queries
        wait(&b.s_full[mt][count & 1], count >> 1); // (one that gave up stops all others; the barriers between warps need every pass)
        tc_fence_after();
        uint32_t z[kN];
        float f = 1.f;
        bool grows = false;
        if (busy) {
          const uint32_t scores = mine_at + (count & 1) * kN;
          tmem_ld32(scores, *reinterpret_cast<uint32_t(*)[32]>(z));
          tmem_ld32(scores + 32, *reinterpret_cast<uint32_t(*)[32]>(z + 32));
          const int valid = pl.gr.rows - pl.t * kN;
          float mul = a.scale2;
          if (valid < kN) {
#pragma unroll
            for (int j = 0; j < kN; ++j) z[j] = __float_as_uint(j < valid ? __uint_as_float(z[j]) * mul : -INFINITY);
            mul = 1.f;
          }
          // the largest score: the least where the factor is below zero
          float top = __uint_as_float(z[0]), other = __uint_as_float(z[1]);
          if (mul >= 0.f) {
#pragma unroll
            for (int j = 2; j < kN; j += 2) {
              top = fmaxf(top, __uint_as_float(z[j]));
              other = fmaxf(other, __uint_as_float(z[j + 1]));
            }
            top = fmaxf(top, other);
          } else {
#pragma unroll
            for (int j = 2; j < kN; j += 2) {
              top = fminf(top, __uint_as_float(z[j]));
              other = fminf(other, __uint_as_float(z[j + 1]));
            }
            top = fminf(top, other);
          }
          top *= mul;
          if (top > m + kSlack<T>) {           // (a row's result does not depend on the other rows, which may be padding)
            f = exp2_fast(m - top);
            m = top;
          }
          grows = __any_sync(0xffffffffu, f != 1.f);
          const float base_at = m == -INFINITY ? 0.f : m;
          // The base is a rounded product, the scores below are not: 2^-17 off up to here, whole powers of two for large scores.
          // From here on they are rounded alike, so that equal scores have equal weights, in other tiles and kernels too.
          if (fabsf(base_at) >= 256.f) {
#pragma unroll
            for (int j = 0; j < kN; ++j) z[j] = __float_as_uint(__fmul_rn(__uint_as_float(z[j]), mul));
            mul = 1.f;
          }
          const float add = kLift<T> - base_at;
          float2 sum = make_float2(0.f, 0.f);
#pragma unroll
          for (int j = 0; j < kN; j += 2) {
            float2 x = fma2(make_float2(__uint_as_float(z[j]), __uint_as_float(z[j + 1])), make_float2(mul, mul), make_float2(add, add));
            x = make_float2(exp2_fast(x.x), exp2_fast(x.y));
            sum = add2(sum, x);
            halves(x, z[j], z[j + 1], T());
          }
          l = l * f + (sum.x + sum.y);
        }
        if (!begins && grows) {                // the sums so far, once the last tile's product is done
          wait(&b.o_done[mt][(count - 1) & 1], (count - 1) >> 1);
          tc_fence_after();
#pragma unroll 1
          for (int x = 0; x < DH / 16; ++x) {
            uint32_t o[16];
            tmem_ld16(mine_at + S::kO + 16 * x, o);
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
            tmem_st16(mine_at + S::kO + 16 * x, o);
          }
        }
        if (busy) {
          const uint32_t weights = mine_at + (count & 1) * kN;
#pragma unroll
          for (int j = 0; j < kN / 16; ++j) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = z[16 * j + 2 * i];
            tmem_put8(weights + 8 * j, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = z[16 * j + 2 * i + 1];
            tmem_put8(weights + S::kLo + 8 * j, w);
          }
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.p_full[mt][count & 1]);
        ++count;

        const bool ends = pl.t + 1 == pl.tiles;
        if (ends || n + 1 == run) {
          wait(&b.o_done[mt][(count - 1) & 1], (count - 1) >> 1);
          tc_fence_after();
          const bool done = ends && from_start, on = tid < have;
          const int i = pl.gr.first + (q0 + tid) / a.group, head = kh * a.group + (q0 + tid) % a.group;
          const long long at = static_cast<long long>(i) * a.q.heads + head;
          float* part = p.parts + static_cast<long long>(2 * blockIdx.x + (from_start ? 1 : 0)) * (MT * kM * (DH + 2));
          if (busy) {
#pragma unroll 1
            for (int x = 0; x < DH / 16; ++x) {
              uint32_t o[16];
              tmem_ld16(mine_at + S::kO + 16 * x, o);
#pragma unroll
              for (int j = 0; j < 16; j += 4) {
                const float4 v = make_float4(__uint_as_float(o[j]), __uint_as_float(o[j + 1]), __uint_as_float(o[j + 2]),
                                             __uint_as_float(o[j + 3]));
                if (!on) continue;
                if (done) *reinterpret_cast<float4*>(p.whole + at * DH + 16 * x + j) = v;
                else *reinterpret_cast<float4*>(part + 2 * MT * kM + ((4 * x + j / 4) * (MT * kM) + tid) * 4) = v;
              }
            }
            if (on && done) p.whole_stats[at] = make_float2(m, l);
            if (on && !done) {
              part[tid] = m;
              part[MT * kM + tid] = l;
            }
          }
          tc_fence_before();
        }
      }
      begins = pl.next(p);
      if (begins) from_start = true;
    }
  } else if (warp <= kValues) {
    // ---- loads.  Boxes of `box` rows, in one page each, by TMA where a page is a multiple of 8 rows, a box a lane; else 16 bytes a
    // lane, a row's page by the lane of its number, rows 32 .. 63 by the same lanes.
    constexpr int kAtOnce = 8;
    const bool of_keys = warp == kKeys;
    const int stages = of_keys ? S::kKeyRing : S::kValueRing;
    uint64_t *full = of_keys ? b.k_full : b.v_full, *empty = of_keys ? b.k_empty : b.v_empty;
    const uint32_t ring = of_keys ? keys : values;
    int slot = 0;
    uint32_t turn = 1;                         // parity of `empty`: the first pass finds the slots free
    if (p.box > 0) {
      const int past = a.c.pages * a.c.heads * a.c.page;     // rows from here on read as zeros
      const auto page_of = [&]() {
        const int tok = pl.t * kN + lane * p.box;
        if (pl.g >= p.groups || lane * p.box >= kN || tok >= pl.gr.rows) return -1;
        const int page = a.page_shift >= 0 ? tok >> a.page_shift : tok / a.c.page;
        return __ldg(a.c.table + static_cast<long long>(pl.gr.seq) * a.c.max_pages + page);
      };
      int pid = page_of(), issued = 0;
      for (; issued < run; ++issued) {
        const int tok = pl.t * kN + lane * p.box, kh = pl.item / pl.blocks(p);
        const bool on = lane * p.box < kN && tok < pl.gr.rows;
        if (on && !good_page(a.c, pid)) {
          atomicOr(a.c.status, ST_BADINDEX);
          pid = 0;
        }
        const int row = on ? (pid * a.c.heads + kh) * a.c.page + (a.page_shift >= 0 ? tok & (a.c.page - 1) : tok % a.c.page) : past;
        pl.next(p);
        pid = page_of();
        if (!__all_sync(0xffffffffu, wait(&empty[slot], turn))) break;       // (the warp gives up as one)
        if (lane == 0) mbar_arrive_expect_tx(&full[slot], S::kTileBytes);
        __syncwarp();
        if (lane * p.box < kN) {
#pragma unroll
          for (int x = 0; x < S::kBlocks; ++x)
            tma_load_3d(ring + slot * S::kTileBytes + x * (kN * 128) + lane * p.box * 128, &map, &full[slot], x * 64, row, of_keys ? 0 : 1);
        }
        if (++slot == stages) {
          slot = 0;
          turn ^= 1;
        }
      }
      for (int i = 0; i < stages && i < issued; ++i)         // none is in flight at the end, whatever came before
        mbar_wait(&full[i], (issued - 1 - i) / stages & 1, a.c.status, nullptr);
    } else {
      const T* from = static_cast<const T*>(a.pk) + (of_keys ? 0 : a.plane);
      int last = 0, pid[2];
      const auto pages_of = [&]() {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int tok = pl.t * kN + h * 32 + lane;
          pid[h] = pl.g < p.groups && tok < pl.gr.rows
                       ? __ldg(a.c.table + static_cast<long long>(pl.gr.seq) * a.c.max_pages + (a.page_shift >= 0 ? tok >> a.page_shift : tok / a.c.page))
                       : 0;
        }
      };
      pages_of();
      bool ok = true;
      for (int n = 0; n < run; ++n) {
        const int valid = pl.gr.rows - pl.t * kN, kh = pl.item / pl.blocks(p);
        long long row[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int tok = pl.t * kN + h * 32 + lane, in_page = a.page_shift >= 0 ? tok & (a.c.page - 1) : tok % a.c.page;
          if (h * 32 + lane < valid && !good_page(a.c, pid[h])) {
            atomicOr(a.c.status, ST_BADINDEX);
            pid[h] = 0;
          }
          row[h] = h * 32 + lane < valid ? ((static_cast<long long>(pid[h]) * a.c.heads + kh) * a.c.page + in_page) * DH : 0;
        }
        pl.next(p);
        pages_of();
        ok = __all_sync(0xffffffffu, wait(&empty[slot], turn));
        if (!ok) break;
        const uint32_t dst = ring + slot * S::kTileBytes;
#pragma unroll 1
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j0 = 0; j0 < VPR; j0 += kAtOnce) {
            long long src[kAtOnce];              // (so many: a copy would wait for its own row's address otherwise)
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) src[j] = __shfl_sync(0xffffffffu, row[h], (lane + 32 * (j0 + j)) / VPR & 31);
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
              const int e = lane + 32 * (j0 + j), r = e / VPR, x = e % VPR;
              if (j0 + j < VPR)
                cp_async16_or_zero(dst + h * (32 * 128) + (x >> 3) * (kN * 128) + r * 128 + (((x & 7) ^ (r & 7)) << 4),
                                   from + src[j] + x * 8, h * 32 + r < valid);
            }
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
    }
  } else if (warp < kProducts + MT && elect_one()) {
    // ---- products, of 128 rows a warp
    constexpr uint32_t kScores = idesc_of<T>(kM, kN), kSums = idesc_of<T>(kM, DH) | 1u << 16;
    const int mt = MT > 1 ? warp - kProducts : 0;
    const uint32_t tm = tmem + mt * S::kCols, qd = desc_low(base + mt * (S::kQBytes / MT));
    bool ok = true, first = true, active = false;            // first of an item's tiles in this run; whether it has queries here
    int vslot = 0, kslot = 0;
    uint32_t vturn = 0, kturn = 0, items = 0, scored = 0, weighed = 0;
    const auto weigh = [&]() {                 // sums += weights of the last tile * values
      ok = ok && wait(&b.v_full[vslot], vturn) && (!active || wait(&b.p_full[mt][weighed & 1], weighed >> 1));
      if (!ok) return;
      if (active) {
        tc_fence_after();
        const uint32_t vd = desc_low_mn(values + vslot * S::kTileBytes), w = tm + (weighed & 1) * kN;
#pragma unroll
        for (int k = 0; k < kN / 16; ++k) umma_ts(tm + S::kO, w + 8 * k, vd + k * (2048 >> 4), kSums, !first || k != 0);
#pragma unroll
        for (int k = 0; k < kN / 16; ++k) umma_ts(tm + S::kO, w + S::kLo + 8 * k, vd + k * (2048 >> 4), kSums, 1);
        first = false;
        umma_commit(&b.o_done[mt][weighed & 1]);
        ++weighed;
        umma_commit(&b.v_empty[vslot]);
      } else {
        mbar_arrive(&b.v_empty[vslot]);
      }
      if (++vslot == S::kValueRing) {
        vslot = 0;
        vturn ^= 1;
      }
    };
    bool begins = true;
    for (int n = 0; n < run && ok; ++n) {
      if (begins) {
        if (n > 0) weigh();
        first = true;
        active = mt * kM < pl.have(p);
        ok = ok && (!active || wait(&b.q_full[mt], items++));
      }
      ok = ok && wait(&b.k_full[kslot], kturn) && (!active || scored < 2 || wait(&b.o_done[mt][scored & 1], (scored - 2) >> 1));
      if (!ok) break;
      if (active) {
        tc_fence_after();
        const uint32_t to = tm + (scored & 1) * kN;          // (free: the weights there have been used)
        const uint32_t kd = desc_low(keys + kslot * S::kTileBytes);
#pragma unroll
        for (int k = 0; k < DH / 16; ++k) {
          const uint32_t qk = qd + (((k >> 2) * (kM * 128) + (k & 3) * 32) >> 4), kk = kd + (((k >> 2) * (kN * 128) + (k & 3) * 32) >> 4);
          if (k == 0) umma_ss<false>(to, qk, kk, kScores);
          else umma_ss<true>(to, qk, kk, kScores);
        }
        umma_commit(&b.s_full[mt][scored & 1]);
        ++scored;
        umma_commit(&b.k_empty[kslot]);
      } else {
        mbar_arrive(&b.k_empty[kslot]);
      }
      if (++kslot == S::kKeyRing) {
        kslot = 0;
        kturn ^= 1;
      }
      if (!begins) weigh();
      begins = pl.next(p);
    }
    if (ok) weigh();
    umma_commit(&b.drain);                     // all products have ended, whatever came before
    mbar_wait(&b.drain, 0, a.c.status, nullptr);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kProducts) {
    tc_fence_after();
    tmem_dealloc(tmem, MT * S::kCols);
  }
}

// ---- the join: 8 rows (entry, head of a key head) by dh / 4 pieces of four columns by a few runs of their parts a block.  Latency:
// an entry, then its group and places in the lists, then its parts, kJoinEach of them together.
constexpr int kJoinEach = 3;                   // (six, and with them fewer threads: 1 to 3 us more)
// CTAs whose runs of `per` tiles have those from `tile` on.
__device__ __forceinline__ void runs_of(long long tile, int tiles, long long per, int& first, int& last) {
  if (tile + tiles < (1ll << 31)) {            // (a 64-bit division takes four times as long)
    first = static_cast<int>(tile) / static_cast<int>(per);
    last = static_cast<int>(tile + tiles - 1) / static_cast<int>(per);
  } else {
    first = static_cast<int>(tile / per);
    last = static_cast<int>((tile + tiles - 1) / per);
  }
}
template <typename T>
__global__ void __launch_bounds__(1024) shared_join_kernel(const __grid_constant__ SharedArgs p) {
  extern __shared__ __align__(16) float js[];  // (m, l) and four sums of each run but the first
  pdl_enter();
  const AttendArgs& a = p.a;
  const int dh = a.c.dh, kh = blockIdx.y, cells = 2 * dh, cell = threadIdx.x % cells, split = threadIdx.x / cells, x = 4 * (cell / 8);
  const int splits = blockDim.x / cells;
  const long long row = static_cast<long long>(blockIdx.x) * 8 + cell % 8;
  const bool real = row < static_cast<long long>(a.n) * a.group;
  const int i = real ? static_cast<int>(row / a.group) : 0, h = static_cast<int>(row - static_cast<long long>(i) * a.group), head = kh * a.group + h;
  const int4 e = real ? __ldcg(reinterpret_cast<const int4*>(p.entries + i)) : make_int4(-2, 0, 0, 0);
  const long long at = static_cast<long long>(i) * a.q.heads + head;
  // the CTAs that have parts of the shared rows (c0 .. c1) and of the others (d0 .. d1); one has all
  int c0 = 0, c1 = -1, d0 = 0, d1 = -1, r = 0;
  if (e.z > 0) {
    const int tiles = pieces_of(e.z, kTile);
    runs_of(__ldcg(a.tile0 + i) + static_cast<long long>(kh * a.subs + h / kRows) * tiles, tiles, __ldcg(a.tile0 + a.n), d0, d1);
  }
  if (e.x > 0) {
    const int4 gr = __ldcg(reinterpret_cast<const int4*>(p.group + e.y));
    const int tiles = pieces_of(gr.z, kN), blocks = (gr.y * a.group + p.m - 1) / p.m, q = (i - gr.x) * a.group + h;
    r = q % p.m;
    runs_of(__ldcg(p.tile0 + e.y) + static_cast<long long>(kh * blocks + q / p.m) * tiles, tiles, __ldcg(p.tile0 + p.groups), c0, c1);
  }
  const int shared = c1 - c0 + 1, all = shared + d1 - d0 + 1;
  float top = -INFINITY, l = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto add = [&](float m, float sum, float4 y) {
    const float next = fmaxf(top, m), by = next == -INFINITY ? 0.f : next, f = exp2_fast(top - by), g = exp2_fast(m - by);
    top = next;
    l = l * f + sum * g;
    v = make_float4(v.x * f + y.x * g, v.y * f + y.y * g, v.z * f + y.z * g, v.w * f + y.w * g);
  };
  for (int k0 = split; k0 < all; k0 += splits * kJoinEach) {
    float m[kJoinEach], sum[kJoinEach];
    float4 y[kJoinEach];
#pragma unroll
    for (int k = 0; k < kJoinEach; ++k) {
      const int part = k0 + k * splits;
      const bool on = part < all, own = part >= shared;
      const float *pm, *pl, *po;
      if (own ? d0 == d1 : c0 == c1) {
        pm = reinterpret_cast<const float*>((own ? a.stats : p.whole_stats) + at);
        pl = pm + 1;
        po = (own ? a.own : p.whole) + at * dh + x;
      } else if (own) {
        const int d = d0 + part - shared;
        pm = a.ws + (2ll * d + (d == d0 ? 1 : 0)) * part_floats(dh) + h % kRows;
        pl = pm + kRows;
        po = pm + 2 * kRows + (h % kRows) * (dh - 1) + x;
      } else {
        const int c = c0 + part;
        const float* base = p.parts + (2ll * c + (c == c0 ? 1 : 0)) * (static_cast<long long>(p.m) * (dh + 2));
        pm = base + r;
        pl = pm + p.m;
        po = base + 2 * p.m + (x / 4 * p.m + r) * 4;
      }
      m[k] = on ? __ldcg(pm) : -INFINITY;
      sum[k] = on ? __ldcg(pl) : 0.f;
      y[k] = on ? __ldcg(reinterpret_cast<const float4*>(po)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int k = 0; k < kJoinEach; ++k) add(m[k], sum[k], y[k]);
  }
  if (split > 0) {
    float2* mine = reinterpret_cast<float2*>(js + ((split - 1) * cells + cell) * 6);
    mine[0] = make_float2(top, l);
    mine[1] = make_float2(v.x, v.y);
    mine[2] = make_float2(v.z, v.w);
  }
  __syncthreads();
  if (split > 0 || e.x == -2) return;
  T* out = static_cast<T*>(a.out.p) + i * a.out.row + head * a.out.head + x;
  if (e.x == -1) {
    store4(out, make_float4(0.f, 0.f, 0.f, 0.f));
    return;
  }
  for (int k = 1; k < splits; ++k) {
    const float2* other = reinterpret_cast<const float2*>(js + ((k - 1) * cells + cell) * 6);
    add(other[0].x, other[0].y, make_float4(other[1].x, other[1].y, other[2].x, other[2].y));
  }
  store4(out, make_float4(v.x / l, v.y / l, v.z / l, v.w / l));
}

template <typename T, int DH, int MT>
cudaError_t launch_shared_rows(const SharedArgs& p, const CUtensorMap& map, cudaStream_t st) {
  using S = Shape<DH, MT>;
  const cudaError_t e = cudaFuncSetAttribute(shared_kernel<T, DH, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
  return e != cudaSuccess ? e : launch_k(shared_kernel<T, DH, MT>, dim3(p.grid), dim3(S::kThreads), S::kSmem, st, p, map);
}
template <typename T, int DH>
cudaError_t launch_shared_width(const SharedArgs& p, const CUtensorMap& map, cudaStream_t st) {
  if constexpr (DH <= 128)
    if (p.m > kM) return launch_shared_rows<T, DH, 2>(p, map, st);
  return launch_shared_rows<T, DH, 1>(p, map, st);
}
template <typename T>
cudaError_t launch_shared(const SharedArgs& p, const CUtensorMap& map, cudaStream_t st) {
  switch (p.a.c.dh) {
    case 64: return launch_shared_width<T, 64>(p, map, st);
    case 80: return launch_shared_width<T, 80>(p, map, st);
    case 96: return launch_shared_width<T, 96>(p, map, st);
    case 128: return launch_shared_width<T, 128>(p, map, st);
    case 192: return launch_shared_width<T, 192>(p, map, st);
    default: return launch_shared_width<T, 256>(p, map, st);
  }
}

// Keys and values of the layer as [2][rows][dh], boxes of `box` rows of 64 columns.  0: a page is no multiple of 8 rows, or there are
// more rows than a coordinate holds.
int shared_box(const AttendArgs& a, CUtensorMap* map) {
  const long long rows = static_cast<long long>(a.c.pages) * a.c.heads * a.c.page;
  const int box = std::min(kN, a.c.page & -a.c.page);
  const auto encode = tensor_map_encoder();
  if (box < 8 || rows >= (1ll << 31) || !encode) return 0;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(a.c.dh), static_cast<cuuint64_t>(rows), 2};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(a.c.dh) * 2, static_cast<cuuint64_t>(a.plane) * 2};
  const cuuint32_t sides[3] = {64, static_cast<cuuint32_t>(box), 1}, steps[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void*>(a.pk), dims, strides, sides, steps,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? box : 0;
}

// Rows of an item: 256, on an SM of its own, where groups have more than 128 on average (32 answers of 7 heads a key head on a
// video took a third more with 128, which read the keys and values twice).
int shared_rows(const map_cache* c, long long heads, long long n, long long groups) {
  return c->dh <= 128 && n * (heads / c->heads) > kM * groups ? 2 * kM : kM;
}
int shared_grid(const map_cache* c, int m) { return m == kM && c->dh <= 128 ? 2 * 152 : 152; }

struct SharedSpace { size_t group, entries, tile0, own_tile0, stats, own, whole_stats, whole, parts, bytes; };
SharedSpace shared_space(const map_cache* c, long long heads, long long n, long long groups) {
  SharedSpace s;
  size_t at = (map_cache_attend_workspace(c) + 255) / 256 * 256;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  s.group = take(groups * sizeof(Group));
  s.entries = take(n * sizeof(Entry));
  s.tile0 = take((groups + 1) * 8);
  s.own_tile0 = take((n + 1) * 8);
  s.stats = take(n * heads * sizeof(float2));
  s.own = take(n * heads * c->dh * 4);
  s.whole_stats = take(n * heads * sizeof(float2));
  s.whole = take(n * heads * c->dh * 4);
  s.parts = take(2ull * 2 * 152 * kM * (c->dh + 2) * 4);      // (152 CTAs of 256 rows or 304 of 128)
  s.bytes = at;
  return s;
}

}  // namespace
}  // namespace mapk

using namespace mapk;

extern "C" {

size_t map_cache_attend_shared_workspace(const map_cache* c, int heads, int n, int groups) {
  if (check_cache(c) != MAP_OK || heads < 1 || heads > 65535 || n < 0 || n > 65535 || groups < 1 || groups > 65535) return 0;
  if (static_cast<long long>(n) * heads >= (1ll << 31)) return 0;
  return shared_space(c, heads, n, groups).bytes;
}

int map_cache_attend_shared(const map_cache* c, int layer, const map_heads* q, const int32_t* seqs, int n, const int32_t* starts,
                            int groups, float scale, const map_heads* out, void* ws, void* stream) {
  SharedArgs p{};
  AttendArgs& a = p.a;
  const int rc = attend_args(c, layer, q, seqs, n, scale, out, ws, a);
  if (rc != MAP_OK) return rc;
  if (groups < 1) return MAP_EINVAL;
  if (groups > 65535 || static_cast<long long>(n) * q->heads >= (1ll << 31)) return MAP_EUNSUPPORTED;      // a group's rows of queries: 32 bits
  if (a.n == 0) return MAP_OK;
  if (!starts) return MAP_EINVAL;
  const SharedSpace s = shared_space(c, q->heads, n, groups);
  char* w = static_cast<char*>(ws);
  p.starts = starts;
  p.groups = groups;
  p.group = reinterpret_cast<Group*>(w + s.group);
  p.entries = reinterpret_cast<Entry*>(w + s.entries);
  p.tile0 = reinterpret_cast<long long*>(w + s.tile0);
  p.parts = reinterpret_cast<float*>(w + s.parts);
  p.whole_stats = reinterpret_cast<float2*>(w + s.whole_stats);
  p.whole = reinterpret_cast<float*>(w + s.whole);
  p.m = shared_rows(c, q->heads, n, groups);
  p.grid = shared_grid(c, p.m);
  CUtensorMap map{};
  p.box = shared_box(a, &map);
  a.entries = p.entries;
  a.tile0 = reinterpret_cast<long long*>(w + s.own_tile0);
  a.stats = reinterpret_cast<float2*>(w + s.stats);
  a.own = reinterpret_cast<float*>(w + s.own);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool half = c->type == MAP_F16;
  // (a cluster a group where they have many sequences on average)
  const int ranks = n / groups >= 16 ? 8 : 1;
  cudaError_t e = launch_cluster(shared_plan_kernel, static_cast<unsigned>(groups * ranks), kPlan, ranks, st, p, ranks);
  if (e == cudaSuccess) e = half ? launch_shared<__half>(p, map, st) : launch_shared<__nv_bfloat16>(p, map, st);
  if (e == cudaSuccess) e = launch_attend<kOwn>(a, st);
  if (e == cudaSuccess) {
    // (as many runs as one wave of threads allows; 64 questions on an image took 4 us longer with twice as many)
    const int cells = 2 * c->dh;
    int splits = 1;
    while (splits < 4 && 2 * splits * cells <= 1024 && static_cast<long long>(n) * q->heads * (c->dh / 4) * 2 * splits <= 152 * 1024) splits *= 2;
    const dim3 grid(static_cast<unsigned>((static_cast<long long>(n) * a.group + 7) / 8), c->heads), block(splits * cells);
    const size_t smem = static_cast<size_t>(splits - 1) * cells * 6 * 4;
    e = half ? launch_k(shared_join_kernel<__half>, grid, block, smem, st, p) : launch_k(shared_join_kernel<__nv_bfloat16>, grid, block, smem, st, p);
  }
  return launch_err(e);
}

}  // extern "C"
