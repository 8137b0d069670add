// Attention of single tokens over a cache's pages (map_cache_attend).
//
// Mathematics.  out = sum_t p_t v_t / sum_t p_t with p_t = 2^(z_t - m), z_t = scale log2(e) <q, k_t>, m the largest
// score, in one pass: a part of the rows gives (m, l = sum p, o = sum p v), and two parts join as m' = max, each
// part's l and o times 2^(m - m').
//
// Bound: HBM, the rows of K and V once (2 G multiply-adds per element for G query heads a key head; on the tensor cores
// that is below the loads for any G up to 16).  Split: an item is a sequence and up to 16 query heads of one key
// head; the 64-row tiles of all items form one list, and every CTA takes an equal run of it (the lengths are read on the
// device, so one long sequence and many short ones fill the chip alike).  A CTA's four warps take 16 rows of a tile
// each, with a ring of tiles of their own filled by cp.async, and join once an item ends (one barrier; 64 columns at a time
// through a smaller buffer took eight, and 53 us where 50 are taken now): no barrier in the loop over
// tiles.  Runs that begin or end inside an item leave (m, l, o) in the workspace; the last CTA of an item to do so
// (counted in the cache's status words) joins them in list order, so results do not depend on timing.  (A second
// kernel for that took 7 to 8 us; this way the join takes 3 to 4.)
// Measured, dh = 128 in bf16: 64 sequences of 200 to 1600 rows, 32 heads over 8: 50.2 us, 5.0 TB/s, where the loads alone,
// in this order and without any use, take 45.7; one sequence of 120001 rows, 28 heads over 4: 51.0 us, loads alone 42.5.
// Short sequences are bound by an item's own latency, about 2 us on a CTA: 1024 of 64 rows 76 us, 4000 of one row 217.
#include <algorithm>
#include <cmath>

#include "handoff.h"

namespace mapk {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kTok = 16;                       // rows a warp takes of a tile
constexpr int kTile = kWarps * kTok;
constexpr int kRows = 16;                      // query heads of an item: the M of an mma.m16n8k16
constexpr int kMaxGrid = 456;                  // three CTAs for each of 152 SMs
constexpr int kGroup = 10;                     // parts that one CTA joins
static_assert(2 + 2 * kMaxGrid <= MAP_CACHE_STATUS_WORDS, "counters of an item's groups and of their parts");

// CTAs that an SM is to hold, by the registers and the ring that a head's width takes, and the largest grid.
__host__ __device__ constexpr int ctas_of(int dh) { return dh <= 80 ? 3 : dh <= 192 ? 2 : 1; }
constexpr int max_grid(int dh) { return kMaxGrid / 3 * ctas_of(dh); }

// A partial result: m [16], l [16], o [16][dh].
__host__ __device__ constexpr int part_floats(int dh) { return kRows * (dh + 2); }

struct AttendArgs {
  map_cache c;
  const void* pk;                              // plane of the layer's keys; values `plane` elements on
  long long plane;
  map_heads q, out;
  const int32_t* seqs;
  int n, group, subs;                          // query heads a key head, items a key head
  int page_shift;                              // log2 of the page, -1: no power of two
  float scale2;                                // scale log2(e)
  float* ws;
};

__device__ __forceinline__ int seq_len(const AttendArgs& a, int i) {
  const int s = __ldg(a.seqs + i);
  const int len = s >= 0 && s < a.c.seqs ? __ldg(a.c.len + s) : 0;
  return good_len(a.c, len) ? len : 0;
}

__device__ __forceinline__ int seq_tiles(const AttendArgs& a, int i) { return pieces_of(seq_len(a, i), kTile); }

// Sum over the block's threads before this one, and over all (red: kWarps words).
__device__ __forceinline__ long long block_prefix(long long v, long long* red, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  if (lane == 31) red[warp] = s;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    before += w < warp ? red[w] : 0;
    all += red[w];
  }
  *total = all;
  return before + s - v;
}

__device__ __forceinline__ void cp_async16_at(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {       // 2 ulp; 0 at -inf
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T> __device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
               "{%0, %1, %2, %3};" : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
               "{%0, %1, %2, %3};" : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Weights as two halves of T, 16 bits of them and more: one half alone would add an error as large as the output's own
// rounding.  The first is cut, so that the second is not negative.  Both halves of a weight above zero are kept above zero, and
// those of a weight of zero are zero: an infinite v is infinite in the sum as far as fp32 knows its weight, and scores that
// are all minus infinity add up to nothing.  (A half that is raised adds its type's smallest number at most: 2^-39 of the
// largest weight.)  kLift: weights are taken 2^kLift times too large, l and o with them, where T's range needs it.
template <typename T> constexpr float kLift = 0.f;
template <> constexpr float kLift<__half> = 15.f;            // 2^15 down to 2^-24
__device__ __forceinline__ float at_least(float least, float x) { return x > 0.f ? least : 0.f; }
__device__ __forceinline__ void split_weights(float x, float y, uint32_t& hi, uint32_t& lo, __nv_bfloat16) {
  const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
  hi = __byte_perm(a, b, 0x7632);              // above zero where x is: ex2 gives no subnormal numbers
  const __nv_bfloat162 r = __hmax2(__floats2bfloat162_rn(x - __uint_as_float(a & 0xffff0000u), y - __uint_as_float(b & 0xffff0000u)),
                                   __floats2bfloat162_rn(at_least(0x1p-126f, x), at_least(0x1p-126f, y)));
  lo = *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ void split_weights(float x, float y, uint32_t& hi, uint32_t& lo, __half) {
  asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(y), "f"(x));
  const __half2 cut = *reinterpret_cast<const __half2*>(&hi), least = __floats2half2_rn(at_least(0x1p-24f, x), at_least(0x1p-24f, y));
  const __half2 h = __hmax2_nan(cut, least);                 // (not a number where x is none)
  const __half2 r = __hmax2(__floats2half2_rn(x - __low2float(cut), y - __high2float(cut)), least);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  lo = *reinterpret_cast<const uint32_t*>(&r);
}

template <typename T>
__device__ __forceinline__ void store4(T* p, float4 v) {      // 8-byte aligned: strides are multiples of 8, columns of 4
  alignas(8) const T x[4] = {from_f32<T>(v.x), from_f32<T>(v.y), from_f32<T>(v.z), from_f32<T>(v.w)};
  *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(x);
}

// Place in the list: tile t of item `item` (key head * subs + sub) of entry i.
struct Place {
  int i, s, len, tiles, item, t;
  __device__ __forceinline__ void enter(const AttendArgs& a, int entry) {
    for (i = entry; i < a.n; ++i) {
      len = seq_len(a, i);
      if (len > 0) break;
    }
    if (i < a.n) s = __ldg(a.seqs + i);
    tiles = pieces_of(len, kTile);
  }
  __device__ __forceinline__ void next(const AttendArgs& a, int items) {
    if (++t < tiles) return;
    t = 0;
    if (++item < items) return;
    item = 0;
    enter(a, i + 1);
  }
};

// A row of a tile in shared memory, 16 bytes longer than its columns: eight rows' vector x meet distinct banks.  (An
// exclusive or of the vector with the row saves the padding but its addresses are not constants: 58 against 53 us.)
template <int DH>
struct Tile {
  static constexpr int kVecs = DH / 8;
  static constexpr int kRow = DH * 2 + 16;
  static constexpr int kStage = 2 * kTok * kRow;             // K and V rows of one warp's part of a tile
  static constexpr int kSum = DH + 8;                        // floats of a row of sums: four rows' halves meet distinct banks
  static_assert(kRows * kSum * 4 <= kStage, "sums take the place of a tile");
  static __device__ __forceinline__ uint32_t at(int row, int x) { return row * kRow + x * 16; }
};
// Joins `count` parts, of CTAs c, c + stride, ... (the first one's slot `slot0`, the others' slot 0), in order: into out,
// or into the first part where out is nullptr.  All of the block's threads, two pieces of four columns of a row each, with
// kGroup parts of both in flight, for all that a join takes is latency.
template <typename T, int DH>
__device__ __noinline__ void join_parts(const AttendArgs& a, int c, int stride, int slot0, int count, int have, T* out,
                                        float* tops, float* sums) {
  const auto part = [&](int p) { return a.ws + (2 * static_cast<long long>(c + p * stride) + (p == 0 ? slot0 : 0)) * part_floats(DH); };
  const int pieces = have * (DH / 4);
  for (int e0 = threadIdx.x; e0 < pieces; e0 += 2 * kThreads) {
    float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
    float4 v[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int p0 = 0; p0 < count; p0 += kGroup) {
      float4 y[2][kGroup];
      float m[2][kGroup], l[2][kGroup];
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int e = e0 + d * kThreads, r = e / (DH / 4), x = 4 * (e % (DH / 4));
#pragma unroll
        for (int k = 0; k < kGroup; ++k) {
          const bool on = p0 + k < count && e < pieces;
          const float* q = part(p0 + k < count ? p0 + k : 0);
          m[d][k] = on ? __ldcg(q + r) : -INFINITY;
          l[d][k] = on ? __ldcg(q + kRows + r) : 0.f;
          y[d][k] = on ? __ldcg(reinterpret_cast<const float4*>(q + 2 * kRows + r * DH + x)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        float next = top[d];
#pragma unroll
        for (int k = 0; k < kGroup; ++k) next = fmaxf(next, m[d][k]);
        const float at = next == -INFINITY ? 0.f : next, f0 = exp2_fast(top[d] - at);
        top[d] = next;
        sum[d] *= f0;
        v[d] = make_float4(v[d].x * f0, v[d].y * f0, v[d].z * f0, v[d].w * f0);
#pragma unroll
        for (int k = 0; k < kGroup; ++k) {
          const float f = exp2_fast(m[d][k] - at);
          sum[d] = fmaf(f, l[d][k], sum[d]);
          v[d].x = fmaf(f, y[d][k].x, v[d].x);
          v[d].y = fmaf(f, y[d][k].y, v[d].y);
          v[d].z = fmaf(f, y[d][k].z, v[d].z);
          v[d].w = fmaf(f, y[d][k].w, v[d].w);
        }
      }
    }
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const int e = e0 + d * kThreads, r = e / (DH / 4), x = 4 * (e % (DH / 4));
      if (e >= pieces) break;
      if (out) {
        T* o = out + r * a.out.head + x;
        store4(o, make_float4(v[d].x / sum[d], v[d].y / sum[d], v[d].z / sum[d], v[d].w / sum[d]));
      } else {
        *reinterpret_cast<float4*>(part(0) + 2 * kRows + r * DH + x) = v[d];
        if (x == 0) {
          tops[r] = top[d];
          sums[r] = sum[d];
        }
      }
    }
  }
  if (out) return;
  __syncthreads();                             // the first part's m and l have been read
  if (threadIdx.x < have) {
    part(0)[threadIdx.x] = tops[threadIdx.x];
    part(0)[kRows + threadIdx.x] = sums[threadIdx.x];
  }
}

// Whether this block is the last of `count` to come here after writing a part.  The barriers order every thread's writes
// before, and reads after, thread 0's add, which releases them to the last block and acquires theirs.  The counter is zero
// between uses.
__device__ __forceinline__ bool is_last(int* counter, int count, int* flag) {
  __syncthreads();
  if (threadIdx.x == 0) {
    bool last = true;
    if (count > 1) {
      int old;
      asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(old) : "l"(counter) : "memory");
      last = old == count - 1;
      if (last) *counter = 0;
    }
    *flag = last;
  }
  __syncthreads();
  return *flag;
}

template <typename T, int DH, int STAGES>
__global__ void __launch_bounds__(kThreads, ctas_of(DH)) attend_kernel(const __grid_constant__ AttendArgs a) {
  using R = Tile<DH>;
  constexpr int VPR = R::kVecs, KSTEPS = DH / 16;
  constexpr bool QREG = DH <= 128;             // query fragments stay in registers
  extern __shared__ __align__(16) unsigned char sh[];
  __shared__ float sm[kWarps][kRows], sl[kWarps][kRows];
  __shared__ long long red[kWarps + kRows / 2];  // and 16 floats
  __shared__ int first_entry;
  __shared__ long long first_tile;
  __shared__ int last_part;
  pdl_enter();
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);              // one value a warp, as the compiler then knows
  const int rows = min(a.group, kRows), items = a.c.heads * a.subs;

  // this CTA's run of the list, and where it begins: a thread counts a run of the entries
  const int each = (a.n + kThreads - 1) / kThreads, e0 = tid * each, e1 = min(a.n, e0 + each);
  long long mine = 0, total;
  for (int e = e0; e < e1; ++e) mine += static_cast<long long>(seq_tiles(a, e)) * items;
  long long at0 = block_prefix(mine, red, &total);
  const long long per = (total + gridDim.x - 1) / gridDim.x, t0 = per * blockIdx.x;
  for (int e = blockIdx.x; e < a.n; e += gridDim.x) {                  // sequences without rows; bad ones
    const int s = __ldg(a.seqs + e);
    if (s < 0 || s >= a.c.seqs) {
      if (s != -1 && tid == 0) atomicOr(a.c.status, ST_BADINDEX);
    } else if (const int len = __ldg(a.c.len + s); len == 0 || !good_len(a.c, len)) {
      if (len != 0 && tid == 0) atomicOr(a.c.status, ST_BADINDEX);
      T* out = static_cast<T*>(a.out.p) + e * a.out.row;
      for (int x = tid; x < a.out.heads * DH; x += kThreads) out[x / DH * a.out.head + x % DH] = from_f32<T>(0.f);
    }
  }
  if (t0 >= total) return;
  const int run = static_cast<int>(t0 + per <= total ? per : total - t0);
  if (at0 <= t0 && t0 < at0 + mine) {
    for (int e = e0;; ++e) {
      const long long k = static_cast<long long>(seq_tiles(a, e)) * items;
      if (t0 < at0 + k) {
        first_entry = e;
        first_tile = t0 - at0;
        break;
      }
      at0 += k;
    }
  }
  __syncthreads();
  Place ld;
  ld.enter(a, first_entry);
  ld.item = static_cast<int>(first_tile / ld.tiles);
  ld.t = static_cast<int>(first_tile % ld.tiles);
  Place cp = ld;

  const uint32_t ring = smem_u32(sh) + warp * STAGES * R::kStage;
  const uint32_t qbuf = smem_u32(sh) + kWarps * STAGES * R::kStage;                        // [STAGES][rows] tile rows
  const T* pk = static_cast<const T*>(a.pk);
  const T* pv = pk + a.plane;
  const bool whole = a.c.page % kTok == 0;     // a warp's 16 rows lie in one page
  const auto page_at = [&](int tok) { return a.page_shift >= 0 ? tok >> a.page_shift : tok / a.c.page; };
  const auto row_in_page = [&](int tok) { return a.page_shift >= 0 ? tok & (a.c.page - 1) : tok % a.c.page; };

  // ---- loads.  pid: page of the warp's first row (whole), else of row lane & 15, read a tile ahead.
  const auto page_of = [&](const Place& p) -> int {
    if (p.i >= a.n) return 0;
    const int tok = p.t * kTile + warp * kTok + (whole ? 0 : lane & 15);
    return tok < p.len ? __ldg(a.c.table + static_cast<long long>(p.s) * a.c.max_pages + page_at(tok)) : 0;
  };
  int pid = page_of(ld), ld_seg = 0;
  bool ld_new = true;
  const auto load = [&](int slot) {
    const int kh = ld.item / a.subs;
    if (ld_new) {                              // the item's queries: a quarter a warp
      const int g0 = (ld.item % a.subs) * kRows, have = min(kRows, a.group - g0);
      const T* q = static_cast<const T*>(a.q.p) + ld.i * a.q.row + (kh * a.group + g0) * a.q.head;
      for (int e = tid; e < rows * VPR; e += kThreads) {
        const int r = e / VPR, x = e % VPR;
        cp_async16_or_zero(qbuf + (ld_seg % STAGES) * rows * R::kRow + R::at(r, x), q + (r < have ? r : 0) * a.q.head + x * 8, r < have);
      }
    }
    const int tok0 = ld.t * kTile + warp * kTok, valid = ld.len - tok0;
    if (valid > 0) {
      if (!good_page(a.c, pid)) {              // (here, a tile after it was asked for: a check there would wait for it)
        atomicOr(a.c.status, ST_BADINDEX);
        pid = 0;
      }
      const uint32_t dst = ring + slot * R::kStage;
      if (whole) {
        const long long first = ((static_cast<long long>(pid) * a.c.heads + kh) * a.c.page + row_in_page(tok0)) * DH;
        const T* k = pk + first + lane * 8;
        const T* v = pv + first + lane * 8;
        if (valid >= kTok) {
#pragma unroll
          for (int j = 0; j < VPR / 2; ++j) {
            const int e = lane + 32 * j;
            cp_async16_at(dst + R::at(e / VPR, e % VPR), k + 256 * j);
            cp_async16_at(dst + R::at(kTok + e / VPR, e % VPR), v + 256 * j);
          }
        } else {
#pragma unroll
          for (int j = 0; j < VPR / 2; ++j) {
            const int e = lane + 32 * j;
            cp_async16_or_zero(dst + R::at(e / VPR, e % VPR), k + 256 * j, e / VPR < valid);
            cp_async16_or_zero(dst + R::at(kTok + e / VPR, e % VPR), v + 256 * j, e / VPR < valid);
          }
        }
      } else {
        const long long mine = ((static_cast<long long>(pid) * a.c.heads + kh) * a.c.page + row_in_page(tok0 + (lane & 15))) * DH;
#pragma unroll
        for (int j = 0; j < VPR / 2; ++j) {
          const int e = lane + 32 * j, r = e / VPR, x = e % VPR;
          const long long from = __shfl_sync(0xffffffffu, mine, r) + x * 8;
          cp_async16_or_zero(dst + R::at(r, x), pk + from, r < valid);
          cp_async16_or_zero(dst + R::at(kTok + r, x), pv + from, r < valid);
        }
      }
    }
    const int item = ld.item, i = ld.i;
    ld.next(a, items);
    ld_new = ld.item != item || ld.i != i;
    ld_seg += ld_new;
    pid = page_of(ld);
  };

  float o[DH / 8][4], m[2], l[2];
  uint32_t qf[QREG ? KSTEPS : 1][4];
  auto reset = [&]() {
#pragma unroll
    for (int j = 0; j < DH / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  };
  reset();
  // ldmatrix rows: queries and values by (lane & 15, lane / 16), keys by ((lane & 7) + 8 (lane / 16), lane / 8 % 2)
  const int q_row = min(lane & 15, rows - 1), k_row = (lane & 7) + ((lane >> 4) << 3), k_vec = (lane >> 3) & 1;
  const bool two = rows > 8;                   // rows 8 .. 15 hold heads too

  int loaded = 0;
  for (; loaded < STAGES - 1; ++loaded) {
    if (loaded < run) load(loaded);
    cp_async_commit();
  }
  bool begins = true;                          // the next tile is the first of a new item (or of the run)
  bool from_start = cp.t == 0;                 // the run of this item begins with its first tile
  int seg = 0;
  for (int n = 0; n < run; ++n) {
    cp_async_wait_group<STAGES - 2>();
    if (begins) __syncthreads(); else __syncwarp();
    const uint32_t qa = qbuf + (seg % STAGES) * rows * R::kRow;
    if (QREG && begins) {
#pragma unroll
      for (int k = 0; k < KSTEPS; ++k) ldsm4(qf[QREG ? k : 0], qa + R::at(q_row, 2 * k + (lane >> 4)));
    }
    if (n + STAGES - 1 < run) load((n + STAGES - 1) % STAGES);
    cp_async_commit();

    const int valid = cp.len - cp.t * kTile - warp * kTok;
    if (valid > 0) {
      const uint32_t st = ring + (n % STAGES) * R::kStage;
      float z[2][4] = {};
#pragma unroll
      for (int k = 0; k < KSTEPS; ++k) {
        uint32_t b[4];
        ldsm4(b, st + R::at(k_row, 2 * k + k_vec));
        if (QREG) {
          mma16<T>(z[0], qf[QREG ? k : 0], b[0], b[1]);
          mma16<T>(z[1], qf[QREG ? k : 0], b[2], b[3]);
        } else {
          uint32_t f[4];
          ldsm4(f, qa + R::at(q_row, 2 * k + (lane >> 4)));
          mma16<T>(z[0], f, b[0], b[1]);
          mma16<T>(z[1], f, b[2], b[3]);
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[j][e] *= a.scale2;
      if (valid < kTok) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (j * 8 + 2 * (lane & 3) + (e & 1) >= valid) z[j][e] = -INFINITY;
      }
      float f[2] = {1.f, 1.f};
      uint32_t hi[4] = {}, lo[4] = {};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (h == 1 && !two) break;
        float mx = fmaxf(fmaxf(z[0][2 * h], z[0][2 * h + 1]), fmaxf(z[1][2 * h], z[1][2 * h + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        mx = fmaxf(mx, m[h]);
        const float at = mx == -INFINITY ? 0.f : mx;
        f[h] = exp2_fast(m[h] - at);
        m[h] = mx;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float x = exp2_fast(z[j][2 * h] - (at - kLift<T>)), y = exp2_fast(z[j][2 * h + 1] - (at - kLift<T>));
          sum += x + y;
          split_weights(x, y, hi[2 * j + h], lo[2 * j + h], T());
        }
        l[h] = l[h] * f[h] + sum;
      }
      if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) {
          o[j][0] *= f[0];
          o[j][1] *= f[0];
          o[j][2] *= f[1];
          o[j][3] *= f[1];
        }
      }
#pragma unroll
      for (int j = 0; j < DH / 16; ++j) {
        uint32_t b[4];
        ldsm4_t(b, st + R::at(kTok + (lane & 15), 2 * j + (lane >> 4)));
        mma16<T>(o[2 * j], hi, b[0], b[1]);
        mma16<T>(o[2 * j + 1], hi, b[2], b[3]);
        mma16<T>(o[2 * j], lo, b[0], b[1]);
        mma16<T>(o[2 * j + 1], lo, b[2], b[3]);
      }
    }

    const bool ends = cp.t + 1 == cp.tiles;
    if (ends || n + 1 == run) {
      // join the warps: each lays its sums down where its rows of this tile were, which nothing but itself has read and
      // the next load to write there is behind the next barrier
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        if ((lane & 3) == 0) {
          sm[warp][(lane >> 2) + 8 * h] = m[h];
          sl[warp][(lane >> 2) + 8 * h] = l[h];
        }
      }
      __syncwarp();
      float* sums = reinterpret_cast<float*>(sh + (n % STAGES) * R::kStage);     // of warp 0
      float* own = sums + warp * (STAGES * R::kStage / 4) + (lane >> 2) * R::kSum + 2 * (lane & 3);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if ((lane >> 2) + 8 * h < rows)
#pragma unroll
          for (int j = 0; j < DH / 8; ++j)
            *reinterpret_cast<float2*>(own + 8 * h * R::kSum + 8 * j) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
      __syncthreads();
      const int kh = cp.item / a.subs, g0 = (cp.item % a.subs) * kRows, have = min(kRows, a.group - g0);
      const bool done = ends && from_start;
      float* part = a.ws + static_cast<long long>(2 * blockIdx.x + (from_start ? 1 : 0)) * part_floats(DH);
      T* out = static_cast<T*>(a.out.p) + cp.i * a.out.row + (kh * a.group + g0) * a.out.head;
      for (int e = tid; e < have * (DH / 4); e += kThreads) {                    // four columns of a row
        const int r = e / (DH / 4), x = 4 * (e % (DH / 4));
        const float top = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r])), at = top == -INFINITY ? 0.f : top;
        float lr = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = exp2_fast(sm[w][r] - at);
          const float4 y = *reinterpret_cast<const float4*>(sums + w * (STAGES * R::kStage / 4) + r * R::kSum + x);
          lr = fmaf(f, sl[w][r], lr);
          v = make_float4(fmaf(f, y.x, v.x), fmaf(f, y.y, v.y), fmaf(f, y.z, v.z), fmaf(f, y.w, v.w));
        }
        if (done) {
          store4(out + r * a.out.head + x, make_float4(v.x / lr, v.y / lr, v.z / lr, v.w / lr));
        } else {
          *reinterpret_cast<float4*>(part + 2 * kRows + r * DH + x) = v;
          if (x == 0) {
            part[r] = top;
            part[kRows + r] = lr;
          }
        }
      }
      if (!done) {
        // the item's parts: CTAs c0 (whose run begins it) to c0 + parts - 1, in groups of kGroup.  The last CTA of a
        // group joins the group, the last group's the groups.  Counters: a group's at its first CTA, the groups' at c0;
        // a group of one needs none, so the next item's first group may begin where this one's last does.
        const long long tile = t0 + n - cp.t;
        const int c0 = static_cast<int>(tile / per), parts = static_cast<int>((tile + cp.tiles - 1) / per) - c0 + 1;
        const int g = (static_cast<int>(blockIdx.x) - c0) / kGroup, groups = (parts + kGroup - 1) / kGroup;
        const int first = c0 + g * kGroup, count = min(kGroup, parts - g * kGroup);
        float* scratch = reinterpret_cast<float*>(red + kWarps);
        if (is_last(a.c.status + 2 + first, count, &last_part)) {
          if (groups == 1 || count > 1) join_parts<T, DH>(a, first, 1, g == 0, count, have, groups == 1 ? out : nullptr, sm[0], scratch);
          if (groups > 1 && is_last(a.c.status + 2 + kMaxGrid + c0, groups, &last_part))
            join_parts<T, DH>(a, c0, kGroup, 1, groups, have, out, sm[0], scratch);
        }
        __syncthreads();
      }
      reset();
    }
    const int item = cp.item, i = cp.i;
    cp.next(a, items);
    begins = cp.item != item || cp.i != i;
    if (begins) { from_start = true; ++seg; }
  }
}

template <int DH>
constexpr size_t smem_of(int stages, int rows) {
  return static_cast<size_t>(kWarps) * stages * Tile<DH>::kStage + stages * rows * Tile<DH>::kRow;
}

// The kernel's limit of shared memory belongs to all threads of the process: every call sets the same one, the largest, so that
// none lowers it between another's setting and its launch.
template <typename T, int DH, int STAGES>
cudaError_t launch_run(const AttendArgs& a, size_t smem, int grid, cudaStream_t st) {
  constexpr int most = static_cast<int>(smem_of<DH>(STAGES, kRows));
  const cudaError_t e = cudaFuncSetAttribute(attend_kernel<T, DH, STAGES>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  return e != cudaSuccess ? e : launch_k(attend_kernel<T, DH, STAGES>, dim3(grid), dim3(kThreads), smem, st, a);
}

// Tiles in a ring and CTAs an SM: two tiles ahead and two CTAs where they fit (dh = 128, without the join: one sequence of
// 120001 rows 45 us, with one ahead and three CTAs 53; 64 of 200 to 1600 rows 53 and 58), three CTAs up to 80 columns.
// At 192 columns two rings of two tiles fit with up to 15 query heads a key head; with 16 they are 512 bytes too large, and an
// SM holds one CTA of three tiles.
template <typename T, int DH>
cudaError_t launch_width(const AttendArgs& a, int sms, cudaStream_t st) {
  constexpr size_t kSm = 228 * 1024, kOwn = 1024 + 768;      // an SM's shared memory; what a CTA takes beside its dynamic part
  const int rows = a.group < kRows ? a.group : kRows;
  constexpr int kWant = ctas_of(DH);
  const int deep = static_cast<int>(kSm / (smem_of<DH>(3, rows) + kOwn)), flat = static_cast<int>(kSm / (smem_of<DH>(2, rows) + kOwn));
  const bool three = deep >= kWant || deep >= flat;
  const int ctas = std::min(kWant, three ? deep : flat);
  const long long most = static_cast<long long>(a.n) * a.c.heads * a.subs *
                         ((static_cast<long long>(a.c.max_pages) * a.c.page + kTile - 1) / kTile);
  const int grid = static_cast<int>(std::min<long long>(most, std::min(ctas * sms, max_grid(DH))));
  // (64 and 96 columns have room for three with any number of rows)
  if constexpr (kSm / (smem_of<DH>(3, kRows) + kOwn) < kWant)
    if (!three) return launch_run<T, DH, 2>(a, smem_of<DH>(2, rows), grid, st);
  return launch_run<T, DH, 3>(a, smem_of<DH>(3, rows), grid, st);
}

template <typename T>
cudaError_t launch_attend(const AttendArgs& a, int sms, cudaStream_t st) {
  switch (a.c.dh) {
    case 64: return launch_width<T, 64>(a, sms, st);
    case 80: return launch_width<T, 80>(a, sms, st);
    case 96: return launch_width<T, 96>(a, sms, st);
    case 128: return launch_width<T, 128>(a, sms, st);
    case 192: return launch_width<T, 192>(a, sms, st);
    default: return launch_width<T, 256>(a, sms, st);
  }
}

}  // namespace
}  // namespace mapk

using namespace mapk;

extern "C" {

size_t map_cache_attend_workspace(const map_cache* c) {
  return check_cache(c) == MAP_OK ? static_cast<size_t>(2) * max_grid(c->dh) * part_floats(c->dh) * sizeof(float) : 0;
}

int map_cache_attend(const map_cache* c, int layer, const map_heads* q, const int32_t* seqs, int n, float scale,
                     const map_heads* out, void* ws, void* stream) {
  const int rc = check_cache(c);
  if (rc != MAP_OK) return rc;
  if (layer < 0 || layer >= c->layers || !q || !out || n < 0 || !std::isfinite(scale)) return MAP_EINVAL;
  for (const map_heads* h : {q, out})
    if ((!h->p && n > 0) || !aligned16(h->p) || h->heads < 1 || h->row < 0 || h->head < 0 || h->row % 8 || h->head % 8)
      return MAP_EINVAL;
  if (q->heads != out->heads || q->heads % c->heads || !distinct_vectors(out->row, n, out->head, out->heads, c->dh))
    return MAP_EINVAL;
  if (c->dh != 64 && c->dh != 80 && c->dh != 96 && c->dh != 128 && c->dh != 192 && c->dh != 256) return MAP_EUNSUPPORTED;
  if (n > 65535 || q->heads > 65535) return MAP_EUNSUPPORTED;
  if (n == 0) return MAP_OK;
  if (!seqs || !ws || !aligned16(ws)) return MAP_EINVAL;
  AttendArgs a{};
  a.c = *c;
  a.plane = static_cast<long long>(c->pages) * c->heads * c->page * c->dh;
  a.pk = static_cast<const uint16_t*>(c->pool) + 2 * layer * a.plane;
  a.q = *q;
  a.out = *out;
  a.seqs = seqs;
  a.n = n;
  a.group = q->heads / c->heads;
  a.subs = (a.group + kRows - 1) / kRows;
  a.page_shift = -1;
  for (int k = 0; k < 11; ++k)
    if (c->page == 1 << k) a.page_shift = k;
  a.scale2 = scale * 1.4426950408889634f;
  a.ws = static_cast<float*>(ws);
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (e == cudaSuccess) e = c->type == MAP_F16 ? launch_attend<__half>(a, sms, st) : launch_attend<__nv_bfloat16>(a, sms, st);
  if (e == cudaSuccess) return MAP_OK;
  cudaGetLastError();
  return MAP_ECUDA;
}

}  // extern "C"
