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
// each, with a ring of tiles of their own filled by cp.async, and join once an item ends: no barrier in the loop over
// tiles.  Runs that begin or end inside an item leave (m, l, o) in the workspace and a second kernel joins them in
// list order, so results do not depend on timing.
#include <cmath>

#include "handoff.h"

namespace mapk {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kTok = 16;                       // rows a warp takes of a tile
constexpr int kTile = kWarps * kTok;
constexpr int kRows = 16;                      // query heads of an item: the M of an mma.m16n8k16
constexpr int kMaxGrid = 304;                  // two CTAs for each of 152 SMs

// A partial result: m [16], l [16], o [16][dh].
__host__ __device__ constexpr int part_floats(int dh) { return kRows * (dh + 2); }

struct AttendArgs {
  map_cache c;
  const void* pk;                              // plane of the layer's keys; values `plane` elements on
  long long plane;
  map_heads q, out;
  const int32_t* seqs;
  int n, group, subs;                          // query heads a key head, items a key head
  float scale2;                                // scale log2(e)
  float* ws;
};

__device__ __forceinline__ int seq_len(const AttendArgs& a, int i) {
  const int s = __ldg(a.seqs + i);
  return s >= 0 && s < a.c.seqs ? max(0, __ldg(a.c.len + s)) : 0;
}

// Tiles before entry i (i = n: all) of the list, per item; all threads call it.
__device__ __forceinline__ long long tiles_before(const AttendArgs& a, int i, long long* red) {
  long long sum = 0;
  for (int e = threadIdx.x; e < i; e += kThreads) sum += (seq_len(a, e) + kTile - 1) / kTile;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
  __syncthreads();
  sum = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) sum += red[w];
  return sum;
}

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
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
// rounding.  The first is cut, so that the second is not negative, and the second is never zero: an infinite v stays
// infinite.  kLift: weights are taken 2^kLift times too large, l and o with them, where T's range needs it.
template <typename T> constexpr float kLift = 0.f;
template <> constexpr float kLift<__half> = 15.f;            // 2^15 down to 2^-24
__device__ __forceinline__ void split_weights(float x, float y, uint32_t& hi, uint32_t& lo, __nv_bfloat16) {
  const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
  hi = __byte_perm(a, b, 0x7632);
  const __nv_bfloat162 r = __hmax2(__floats2bfloat162_rn(x - __uint_as_float(a & 0xffff0000u), y - __uint_as_float(b & 0xffff0000u)),
                                   __floats2bfloat162_rn(0x1p-126f, 0x1p-126f));
  lo = *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ void split_weights(float x, float y, uint32_t& hi, uint32_t& lo, __half) {
  asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(y), "f"(x));
  const __half2 h = *reinterpret_cast<const __half2*>(&hi);
  const __half2 r = __hmax2(__floats2half2_rn(x - __low2float(h), y - __high2float(h)), __floats2half2_rn(0x1p-24f, 0x1p-24f));
  lo = *reinterpret_cast<const uint32_t*>(&r);
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
    tiles = (len + kTile - 1) / kTile;
  }
  __device__ __forceinline__ void next(const AttendArgs& a, int items) {
    if (++t < tiles) return;
    t = 0;
    if (++item < items) return;
    item = 0;
    enter(a, i + 1);
  }
};

template <typename T, int DH, int STAGES>
__global__ void __launch_bounds__(kThreads) attend_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int RS = DH * 2 + 16;              // row of a tile in shared memory: eight rows meet distinct banks
  constexpr int VPR = DH / 8;                  // 16-byte vectors of a row
  constexpr int KSTEPS = DH / 16;
  constexpr bool QREG = DH <= 128;             // query fragments stay in registers
  constexpr int kStage = 2 * kTok * RS;        // K and V rows of one warp's part of a tile
  extern __shared__ __align__(16) unsigned char sh[];
  __shared__ float sm[kWarps][kRows], sl[kWarps][kRows];
  __shared__ long long red[kWarps];
  __shared__ int first_entry;
  __shared__ long long first_tile;
  pdl_enter();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rows = min(a.group, kRows), items = a.c.heads * a.subs;

  // this CTA's run of the list
  const long long total = tiles_before(a, a.n, red) * items;
  const long long per = (total + gridDim.x - 1) / gridDim.x, t0 = per * blockIdx.x;
  if (t0 >= total) return;
  const int run = static_cast<int>(t0 + per <= total ? per : total - t0);
  {
    // entry of tile t0: a thread's entries are a run of the list, found by the prefix of the threads' sums
    const int each = (a.n + kThreads - 1) / kThreads, e0 = tid * each;
    long long mine = 0;
    for (int e = e0; e < min(a.n, e0 + each); ++e) mine += static_cast<long long>((seq_len(a, e) + kTile - 1) / kTile) * items;
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    __syncthreads();
    if (lane == 31) red[warp] = incl;
    __syncthreads();
    for (int w = 0; w < warp; ++w) incl += red[w];
    long long at = incl - mine;
    if (at <= t0 && t0 < incl) {
      int e = e0;
      for (;; ++e) {
        const long long k = static_cast<long long>((seq_len(a, e) + kTile - 1) / kTile) * items;
        if (t0 < at + k) break;
        at += k;
      }
      first_entry = e;
      first_tile = t0 - at;
    }
    __syncthreads();
  }
  Place ld;
  ld.enter(a, first_entry);
  ld.item = static_cast<int>(first_tile / ld.tiles);
  ld.t = static_cast<int>(first_tile % ld.tiles);
  Place cp = ld;

  unsigned char* ring = sh + warp * STAGES * kStage;
  unsigned char* qbuf = sh + kWarps * STAGES * kStage;                 // [3][rows][RS]
  float* join = reinterpret_cast<float*>(qbuf + 3 * rows * RS);        // [2][rows][64]
  const T* pk = static_cast<const T*>(a.pk);
  const bool whole = a.c.page % kTok == 0;     // a warp's 16 rows lie in one page

  // ---- loads.  pid: page of the warp's first row (whole), else of row lane & 15, read a tile ahead.
  auto page_of = [&](const Place& p) -> int {
    if (p.i >= a.n) return 0;
    const int tok = p.t * kTile + warp * kTok + (whole ? 0 : lane & 15);
    return tok < p.len ? __ldg(a.c.table + static_cast<long long>(p.s) * a.c.max_pages + tok / a.c.page) : 0;
  };
  int pid = page_of(ld), ld_seg = 0;
  bool ld_new = true;
  auto load = [&](int slot) {
    const int kh = ld.item / a.subs;
    if (ld_new) {                              // the item's queries: a quarter a warp
      const int g0 = (ld.item % a.subs) * kRows, have = min(kRows, a.group - g0);
      const T* q = static_cast<const T*>(a.q.p) + ld.i * a.q.row + (kh * a.group + g0) * a.q.head;
      for (int e = tid; e < rows * VPR; e += kThreads) {
        const int r = e / VPR, x = e % VPR;
        cp_async16_or_zero(smem_u32(qbuf + ((ld_seg % 3) * rows + r) * RS + x * 16), q + (r < have ? r : 0) * a.q.head + x * 8, r < have);
      }
    }
    const int tok0 = ld.t * kTile + warp * kTok, valid = ld.len - tok0;
    if (valid > 0) {
      const uint32_t dst = smem_u32(ring + slot * kStage);
      if (whole) {
        const T* src = pk + ((static_cast<long long>(pid) * a.c.heads + kh) * a.c.page + tok0 % a.c.page) * DH;
#pragma unroll
        for (int j = 0; j < VPR / 2; ++j) {
          const int e = lane + 32 * j, r = e / VPR, x = e % VPR;
          cp_async16_or_zero(dst + r * RS + x * 16, src + e * 8, r < valid);
          cp_async16_or_zero(dst + (kTok + r) * RS + x * 16, src + a.plane + e * 8, r < valid);
        }
      } else {
        const long long mine = ((static_cast<long long>(pid) * a.c.heads + kh) * a.c.page + (tok0 + (lane & 15)) % a.c.page) * DH;
#pragma unroll
        for (int j = 0; j < VPR / 2; ++j) {
          const int e = lane + 32 * j, r = e / VPR, x = e % VPR;
          const T* src = pk + __shfl_sync(0xffffffffu, mine, r) + x * 8;
          cp_async16_or_zero(dst + r * RS + x * 16, src, r < valid);
          cp_async16_or_zero(dst + (kTok + r) * RS + x * 16, src + a.plane, r < valid);
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
  const uint32_t q_at = min(lane & 15, rows - 1) * RS + (lane >> 4) * 16;
  const uint32_t k_at = ((lane & 7) + ((lane >> 4) << 3)) * RS + ((lane >> 3) & 1) * 16;
  const uint32_t v_at = (kTok + (lane & 15)) * RS + (lane >> 4) * 16;
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
    const uint32_t qa = smem_u32(qbuf + (seg % 3) * rows * RS) + q_at;
    if (QREG && begins) {
#pragma unroll
      for (int k = 0; k < KSTEPS; ++k) ldsm4(qf[QREG ? k : 0], qa + k * 32);
    }
    if (n + STAGES - 1 < run) load((n + STAGES - 1) % STAGES);
    cp_async_commit();

    const int valid = cp.len - cp.t * kTile - warp * kTok;
    if (valid > 0) {
      const uint32_t st = smem_u32(ring + (n % STAGES) * kStage);
      float z[2][4] = {};
#pragma unroll
      for (int k = 0; k < KSTEPS; ++k) {
        uint32_t b[4];
        ldsm4(b, st + k_at + k * 32);
        if (QREG) {
          mma16<T>(z[0], qf[QREG ? k : 0], b[0], b[1]);
          mma16<T>(z[1], qf[QREG ? k : 0], b[2], b[3]);
        } else {
          uint32_t f[4];
          ldsm4(f, qa + k * 32);
          mma16<T>(z[0], f, b[0], b[1]);
          mma16<T>(z[1], f, b[2], b[3]);
        }
      }
      float f[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (h == 1 && !two) { f[1] = 1.f; z[0][2] = z[0][3] = z[1][2] = z[1][3] = 0.f; continue; }
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& x = z[j][2 * h + e];
            x = j * 8 + 2 * (lane & 3) + e < valid ? x * a.scale2 : -INFINITY;
            mx = fmaxf(mx, x);
          }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        mx = fmaxf(mx, m[h]);
        const float at = mx == -INFINITY ? 0.f : mx;
        f[h] = exp2f(m[h] - at);
        m[h] = mx;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            z[j][2 * h + e] = exp2f(z[j][2 * h + e] - (at - kLift<T>));
            sum += z[j][2 * h + e];
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
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) split_weights(z[e >> 1][2 * (e & 1)], z[e >> 1][2 * (e & 1) + 1], hi[e], lo[e], T());
#pragma unroll
      for (int j = 0; j < DH / 16; ++j) {
        uint32_t b[4];
        ldsm4_t(b, st + v_at + j * 32);
        mma16<T>(o[2 * j], hi, b[0], b[1]);
        mma16<T>(o[2 * j + 1], hi, b[2], b[3]);
        mma16<T>(o[2 * j], lo, b[0], b[1]);
        mma16<T>(o[2 * j + 1], lo, b[2], b[3]);
      }
    }

    const bool ends = cp.t + 1 == cp.tiles;
    if (ends || n + 1 == run) {
      // join the warps
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        if ((lane & 3) == 0) {
          sm[warp][(lane >> 2) + 8 * h] = m[h];
          sl[warp][(lane >> 2) + 8 * h] = l[h];
        }
      }
      __syncthreads();
      float top[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = (lane >> 2) + 8 * h;
        top[h] = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r]));
        const float f = exp2f(m[h] - (top[h] == -INFINITY ? 0.f : top[h]));
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) {
          o[j][2 * h] *= f;
          o[j][2 * h + 1] *= f;
        }
      }
      const int kh = cp.item / a.subs, g0 = (cp.item % a.subs) * kRows, have = min(kRows, a.group - g0);
      const bool done = ends && from_start;
      float* part = a.ws + static_cast<long long>(2 * blockIdx.x + (from_start ? 1 : 0)) * part_floats(DH);
      T* out = static_cast<T*>(a.out.p) + cp.i * a.out.row + (kh * a.group + g0) * a.out.head;
#pragma unroll
      for (int c0 = 0; c0 < DH; c0 += 64) {
        // warps 0 and 2 lay down 64 columns, 1 and 3 add theirs, all threads add the two
        float* buf = join + (warp >> 1) * rows * 64;
#pragma unroll
        for (int turn = 0; turn < 2; ++turn) {
          if ((warp & 1) == turn) {
#pragma unroll
            for (int jj = 0; jj < 8; ++jj)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int r = (lane >> 2) + 8 * h, j = c0 / 8 + jj;
                if (j >= DH / 8 || r >= rows) continue;
                float2* x = reinterpret_cast<float2*>(buf + r * 64 + jj * 8 + 2 * (lane & 3));
                float2 v = make_float2(o[j][2 * h], o[j][2 * h + 1]);
                if (turn) { v.x += x->x; v.y += x->y; }
                *x = v;
              }
          }
          __syncthreads();
        }
        const int width = DH - c0 < 64 ? DH - c0 : 64;
        for (int e = tid; e < have * 64; e += kThreads) {
          const int r = e >> 6, x = e & 63;
          if (x >= width) continue;
          const float v = join[r * 64 + x] + join[(rows + r) * 64 + x];
          if (done) {
            const float mr = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r])), at = mr == -INFINITY ? 0.f : mr;
            const float lr = sl[0][r] * exp2f(sm[0][r] - at) + sl[1][r] * exp2f(sm[1][r] - at) +
                             sl[2][r] * exp2f(sm[2][r] - at) + sl[3][r] * exp2f(sm[3][r] - at);
            out[r * a.out.head + c0 + x] = from_f32<T>(v / lr);
          } else {
            part[2 * kRows + r * DH + c0 + x] = v;
          }
        }
        __syncthreads();
      }
      if (!done && tid < have) {
        const float mr = fmaxf(fmaxf(sm[0][tid], sm[1][tid]), fmaxf(sm[2][tid], sm[3][tid])), at = mr == -INFINITY ? 0.f : mr;
        part[tid] = mr;
        part[kRows + tid] = sl[0][tid] * exp2f(sm[0][tid] - at) + sl[1][tid] * exp2f(sm[1][tid] - at) +
                            sl[2][tid] * exp2f(sm[2][tid] - at) + sl[3][tid] * exp2f(sm[3][tid] - at);
      }
      reset();
    }
    const int item = cp.item, i = cp.i;
    cp.next(a, items);
    begins = cp.item != item || cp.i != i;
    if (begins) { from_start = true; ++seg; }
  }
}

// Joins the parts of the items that several CTAs' runs share; zeros for sequences without rows.  A CTA a query head:
// its warps take every fourth part, a lane the columns 4 lane .. (and 128 on).
template <typename T>
__global__ void __launch_bounds__(kThreads) attend_join_kernel(const __grid_constant__ AttendArgs a, int grid) {
  __shared__ long long red[kWarps];
  __shared__ float w[kMaxGrid], stat[2][kWarps];
  __shared__ float4 acc[kWarps][kMaxHead / 4];
  pdl_enter();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, i = blockIdx.y, h = blockIdx.x, dh = a.c.dh;
  const int s = __ldg(a.seqs + i);
  if (s < 0 || s >= a.c.seqs) {
    if (s != -1 && tid == 0) atomicOr(a.c.status, ST_BADINDEX);
    return;
  }
  const int kh = h / a.group, g = h % a.group, items = a.c.heads * a.subs, item = kh * a.subs + g / kRows, r = g % kRows;
  T* out = static_cast<T*>(a.out.p) + i * a.out.row + h * a.out.head;
  const int tiles = (seq_len(a, i) + kTile - 1) / kTile;
  if (tiles == 0) {
    for (int d = tid; d < dh; d += kThreads) out[d] = from_f32<T>(0.f);
    return;
  }
  const long long total = tiles_before(a, a.n, red) * items, per = (total + grid - 1) / grid;
  const long long first = tiles_before(a, i, red) * items + static_cast<long long>(item) * tiles;
  const int c0 = static_cast<int>(first / per), c1 = static_cast<int>((first + tiles - 1) / per), parts = c1 - c0 + 1;
  if (parts == 1) return;
  // part p: CTA c0 + p; the first is that CTA's second slot (its run begins the item)
  const auto part = [&](int p) { return a.ws + (2 * static_cast<long long>(c0 + p) + (p == 0)) * part_floats(dh); };
  float top = -INFINITY;
  for (int p = tid; p < parts; p += kThreads) top = fmaxf(top, part(p)[r]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) stat[0][warp] = top;
  __syncthreads();
  top = fmaxf(fmaxf(stat[0][0], stat[0][1]), fmaxf(stat[0][2], stat[0][3]));
  const float at = top == -INFINITY ? 0.f : top;
  float l = 0.f;
  for (int p = tid; p < parts; p += kThreads) {
    w[p] = exp2f(part(p)[r] - at);
    l = fmaf(w[p], part(p)[kRows + r], l);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  if (lane == 0) stat[1][warp] = l;
  __syncthreads();
  l = (stat[1][0] + stat[1][1]) + (stat[1][2] + stat[1][3]);
  for (int v = lane; v < dh / 4; v += 32) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = warp; p < parts; p += kWarps) {
      const float4 y = *reinterpret_cast<const float4*>(part(p) + 2 * kRows + r * dh + 4 * v);
      x.x = fmaf(w[p], y.x, x.x);
      x.y = fmaf(w[p], y.y, x.y);
      x.z = fmaf(w[p], y.z, x.z);
      x.w = fmaf(w[p], y.w, x.w);
    }
    acc[warp][v] = x;
  }
  __syncthreads();
  const float* f = reinterpret_cast<const float*>(acc);
  for (int d = tid; d < dh; d += kThreads)
    out[d] = from_f32<T>(((f[d] + f[kMaxHead + d]) + (f[2 * kMaxHead + d] + f[3 * kMaxHead + d])) / l);
}

size_t attend_smem(int dh, int stages, int rows) {
  return static_cast<size_t>(kWarps) * stages * 2 * kTok * (dh * 2 + 16) + 3 * rows * (dh * 2 + 16) + 2 * rows * 64 * 4;
}

template <typename T, int DH, int STAGES>
cudaError_t launch_run(const AttendArgs& a, size_t smem, int grid, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(attend_kernel<T, DH, STAGES>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e == cudaSuccess) e = launch_k(attend_kernel<T, DH, STAGES>, dim3(grid), dim3(kThreads), smem, st, a);
  if (e == cudaSuccess) e = launch_k(attend_join_kernel<T>, dim3(a.q.heads, a.n), dim3(kThreads), 0, st, a, grid);
  return e;
}

// Two CTAs an SM where two stages of both fit its 227 KB, else one; three stages where they fit then.
template <typename T, int DH>
cudaError_t launch_width(const AttendArgs& a, int sms, cudaStream_t st) {
  constexpr size_t kHalf = 113 * 1024, kWhole = 226 * 1024;
  const int rows = a.group < kRows ? a.group : kRows;
  const size_t three = attend_smem(DH, 3, rows), two = attend_smem(DH, 2, rows);
  const int ctas = two <= kHalf ? 2 : 1;
  const long long most = static_cast<long long>(a.n) * a.c.heads * a.subs *
                         ((static_cast<long long>(a.c.max_pages) * a.c.page + kTile - 1) / kTile);
  int grid = ctas * sms < kMaxGrid ? ctas * sms : kMaxGrid;
  if (most < grid) grid = static_cast<int>(most);
  if constexpr (DH > 96)                       // up to 96 columns three stages always fit
    if (three > (ctas == 2 ? kHalf : kWhole)) return launch_run<T, DH, 2>(a, two, grid, st);
  return launch_run<T, DH, 3>(a, three, grid, st);
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
  return check_cache(c) == MAP_OK ? static_cast<size_t>(2) * kMaxGrid * part_floats(c->dh) * sizeof(float) : 0;
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
