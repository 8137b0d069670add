// Queries and keys before a language model's attention: the RMS norm of each head and the rotation
// by position on up to four axes, in one pass (map_qk_rotate), its gradient (map_qk_rotate_grad), and the
// form whose keys and values go to a cache's pages (map_qk_rotate_append).
//
// Mathematics.  Per head x of dh columns: r = (mean x^2 + eps)^(-1/2), z = x r w; pair (a, b) turned by
// t = pos[axis] inv_freq:  y_a = z_a cos t - z_b sin t, y_b = z_b cos t + z_a sin t.  Backward, with g the
// pair turned back (t -> -t) and n = x r:  dx = r (g w - n mean(g w n)),  dw = sum over rows and heads of g n.
//
// Angles.  inv_freq / 2 pi is held as a 64-bit binary fraction of a turn, the nearest one; that times a position is taken
// modulo 2^64, which drops whole turns exactly.  The fraction is off by 2^-65 turns (frequencies up to 2^40), its multiple by
// |pos| times as much, at most 2^-34; the 32 bits that are kept of it are cut, 2^-32 at most: together under 2^-29 radians at
// any position.  cos and sin come from those bits in fp32.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cuda_fp16.h>
#include <new>

#include "../../include/map_gb300.h"
#include "handoff.h"

struct map_rope {
  mapk::RopeTab tab;
};

namespace mapk {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kRotateCtas = 3, kGradCtas = 2;  // CTAs an SM
constexpr int kGradBlocks = 152 * kGradCtas;   // blocks of a gradient's sides, each with a partial sum of dw

struct Side {                        // one tensor's heads: input, output, norm weight
  const void* x; long long xrow, xhead;
  void* y; long long yrow, yhead;
  const void* w;
  const void* g; long long grow, ghead;   // backward: gradient of the output
  float* part;                       // backward: this side's partial sums
  int heads;
  int kind;                          // kRowsOut: y is a tensor; kKeys, kValues: slots of a cache's plane y
};
enum Kind { kRowsOut = 0, kKeys = 1, kValues = 2 };

// Up to three tensors of one launch; side i takes blocks first[i] .. first[i + 1] - 1, its warps runs of run[i] passes.
struct Job {
  Side s[3];
  unsigned first[4], run[3];
  const int32_t* pos;
  long long rows;
  const int32_t* slots;              // append: a row's slot
  int page, pages;
  int* status;
};

__device__ __forceinline__ int side_of_block(const Job& job) {
  return (blockIdx.x >= job.first[1] ? 1 : 0) + (blockIdx.x >= job.first[2] ? 1 : 0);
}

// cos and sin of a 32-bit fraction of a turn: the nearest quarter turn off, the rest x (|x| <= pi / 4) by the Taylor
// series of both to x^9 and x^10, whose next terms are below 2e-9 and 2e-10; fp32 roundings add up to 2^-23.
__device__ __forceinline__ float2 cos_sin(uint32_t turn) {
  const uint32_t quarter = (turn + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int>(turn - (quarter << 30))) * 1.46291807926715968e-9f;   // 2 pi 2^-32
  const float y = x * x;
  float s = fmaf(y, 2.75573192e-6f, -1.98412698e-4f);
  s = fmaf(s, y, 8.33333333e-3f);
  s = fmaf(s, y, -1.66666667e-1f);
  s = fmaf(s * y, x, x);
  float c = fmaf(y, -2.75573192e-7f, 2.48015873e-5f);
  c = fmaf(c, y, -1.38888889e-3f);
  c = fmaf(c, y, 4.16666667e-2f);
  c = fmaf(c, y, -0.5f);
  c = fmaf(c, y, 1.f);
  const float co = quarter & 1 ? s : c, si = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -co : co, quarter & 2 ? -si : si);
}

// Whether a row is written: not for slot -1 (padding), nor for one outside the pool, which is reported.
__device__ __forceinline__ bool good_slot(const Job& job, int slot) {
  if (slot >= 0 && slot < job.pages * job.page) return true;
  if (slot != -1) atomicOr(job.status, ST_BADINDEX);
  return false;
}
// ------------------------------------------------------------------ vectors of V columns: a warp a row's heads
// (Scalar instructions: the two-wide ones took as many moves between registers as they saved, and 0.92 of the speed.)
__device__ __forceinline__ float2 neg2(float2 a) { return make_float2(-a.x, -a.y); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }

// V columns as one access (16 bytes; 8 for V = 4 of a 16-bit type), and as V / 2 pairs of floats.
template <typename T, int V> struct Vec;
template <> struct Vec<float, 4> {
  float4 r;
  __device__ __forceinline__ void load(const void* p) { r = *static_cast<const float4*>(p); }
  __device__ __forceinline__ void get(float2 (&v)[2]) const { v[0] = make_float2(r.x, r.y); v[1] = make_float2(r.z, r.w); }
  static __device__ __forceinline__ void store(float* p, const float2 (&v)[2]) {
    const float2 a = v[0], b = v[1];
    *reinterpret_cast<float4*>(p) = make_float4(a.x, a.y, b.x, b.y);
  }
};
__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
__device__ __forceinline__ uint32_t pack2(float2 v, __nv_bfloat16) {
  const __nv_bfloat162 h = __float22bfloat162_rn(v);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float2 v, __half) {
  const __half2 h = __float22half2_rn(v);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T> struct Vec<T, 8> {
  uint4 r;
  __device__ __forceinline__ void load(const void* p) { r = *static_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float2 (&v)[4]) const {
    v[0] = unpack2(r.x, T());
    v[1] = unpack2(r.y, T());
    v[2] = unpack2(r.z, T());
    v[3] = unpack2(r.w, T());
  }
  static __device__ __forceinline__ void store(T* p, const float2 (&v)[4]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(v[0], T()), pack2(v[1], T()), pack2(v[2], T()), pack2(v[3], T()));
  }
};
template <typename T> struct Vec<T, 4> {
  uint2 r;
  __device__ __forceinline__ void load(const void* p) { r = *static_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(float2 (&v)[2]) const { v[0] = unpack2(r.x, T()); v[1] = unpack2(r.y, T()); }
  static __device__ __forceinline__ void store(T* p, const float2 (&v)[2]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], T()), pack2(v[1], T()));
  }
};

// A lane holds two vectors of a head, those of its V pairs: V columns from a and V from b, pairs (a + i, b + i), or for
// adjacent pairs 2 V columns in a row.  2^shift lanes (the last ones may be without columns) share a head, 32 >> shift
// heads a warp.
struct Lane { int j, a, b, turned; bool on, two; };     // turned: how many of the lane's pairs turn
template <int V, bool ADJ>
__device__ __forceinline__ Lane lane_of(const RopeTab& t, int shift) {
  Lane l;
  const int nr = ADJ ? 0 : t.rot / (2 * V);
  l.j = threadIdx.x & ((1 << shift) - 1);
  l.turned = ADJ ? min(V, max(0, (t.rot >> 1) - l.j * V)) : l.j < nr ? V : 0;
  l.a = l.j < nr ? l.j * V : 2 * l.j * V;
  l.b = l.j < nr ? (t.rot >> 1) + l.j * V : l.a + V;
  l.on = l.a < t.dh;
  l.two = l.b < t.dh;
  return l;
}

// The plan's frequencies and axes where lanes read different ones at once (the parameter bank serves one a cycle).
struct Freqs {
  unsigned long long turn[kMaxHead / 2];
  int axis[kMaxHead / 2];
};
__device__ __forceinline__ void fill_freqs(Freqs& f, const RopeTab& t) {
  for (int p = threadIdx.x; p < t.rot >> 1; p += kThreads) {
    f.turn[p] = t.turn[p];
    f.axis[p] = t.axis[p];
  }
  __syncthreads();
}

// cos and sin of the lane's V pairs at one row, two pairs at a time.  A warp computes each pair once (a head's
// lanes would repeat it for every head of the warp) and hands them round through its part of shared memory.
template <int V>
struct Turns {
  float2 c[V / 2], s[V / 2];
  // at: the row's position on axis `lane` (lane < axes)
  __device__ __forceinline__ void make(const RopeTab& t, const Freqs& f, int at, int lane, const Lane& ln, float* buf) {
    const int half = t.rot >> 1;
    __syncwarp();
    for (int p0 = 0; p0 < half; p0 += 32) {
      const int p = p0 + lane;
      const int x = __shfl_sync(0xffffffffu, at, p < half ? f.axis[p] : 0);
      if (p >= half) break;                            // (in the last round only)
      const unsigned long long ph = f.turn[p] * static_cast<unsigned long long>(static_cast<long long>(x));
      const float2 cs = cos_sin(static_cast<uint32_t>(ph >> 32));
      buf[(p >> 1) * 4 + (p & 1)] = cs.x;              // (c, c, s, s) of two pairs
      buf[(p >> 1) * 4 + 2 + (p & 1)] = cs.y;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const int at = min(ln.j * (V / 2) + i, kMaxHead / 4 - 1);
      const float4 x = reinterpret_cast<const float4*>(buf)[at];
      c[i] = make_float2(x.x, x.y);
      s[i] = make_float2(x.z, x.w);
    }
  }
  // The lane's pairs turned (SIGN = 1) or turned back (-1); columns past rot are left as they are.
  template <bool ADJ, int SIGN>
  __device__ __forceinline__ void turn(float2 (&a)[V / 2], float2 (&b)[V / 2], int turned, bool all) const {
    if constexpr (!ADJ) {
      if (!all && turned == 0) return;
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const float2 u = fma2(a[i], c[i], mul2(b[i], SIGN > 0 ? neg2(s[i]) : s[i]));
        b[i] = fma2(b[i], c[i], mul2(a[i], SIGN > 0 ? s[i] : neg2(s[i])));
        a[i] = u;
      }
    } else {
#pragma unroll
      for (int q = 0; q < V; ++q) {
        if (q >= turned) continue;
        const float co = q & 1 ? c[q / 2].y : c[q / 2].x, si = SIGN * (q & 1 ? s[q / 2].y : s[q / 2].x);
        float2& v = q < V / 2 ? a[q] : b[q - V / 2];
        const float2 x = v;
        v = make_float2(x.x * co - x.y * si, x.y * co + x.x * si);
      }
    }
  }
};

template <int N>
__device__ __forceinline__ float dot2(const float2 (&a)[N], const float2 (&b)[N], float add) {
  float2 s = make_float2(add, 0.f);
#pragma unroll
  for (int i = 0; i < N; ++i) s = fma2(a[i], b[i], s);
  return s.x + s.y;
}
// Sum over the lanes of a head, of what a lane gives times `part` = 2^(shift - 5): always five steps, for those past the
// head's lanes, which add a lane's sum to itself, cost less than branches around them.  What they double is taken out
// before: squares that add up to less than 2^128 do not pass it on the way.
struct LaneSum {
  int m[5];
  float part;
  __device__ __forceinline__ explicit LaneSum(int shift) : part(static_cast<float>(1 << shift) * 0.03125f) {
#pragma unroll
    for (int i = 0; i < 5; ++i) m[i] = i < shift ? 1 << i : 0;
  }
  __device__ __forceinline__ float operator()(float x) const {
#pragma unroll
    for (int i = 0; i < 5; ++i) x += __shfl_xor_sync(0xffffffffu, x, m[i]);
    return x;
  }
};

// A norm weight as floats in shared memory: a pass reads it from there, for registers are what its heads need.
template <typename T>
__device__ __forceinline__ void fill_weight(float* to, const T* w, int dh) {
  if (w)
    for (int c = threadIdx.x; c < dh; c += kThreads) to[c] = to_f32(w[c]);
}
template <int V>
__device__ __forceinline__ void weight_at(const float* w, float2 (&v)[V / 2]) {
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    const float4 x = reinterpret_cast<const float4*>(w)[i];
    v[2 * i] = make_float2(x.x, x.y);
    v[2 * i + 1] = make_float2(x.z, x.w);
  }
}

// Loads in flight, without registers: a lane copies its vectors to places of its own in shared memory (no other lane
// reads them, so no barrier is needed), kAhead passes ahead.  Places that a lane never fills hold zeros.
// (Predicated: with branches around the copies the gradient took 82 us, not 80.)
template <int BYTES>
__device__ __forceinline__ void copy_vec(uint32_t dst, const char* src, bool on) {
  if (BYTES == 16)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}"
                 ::"r"(dst), "l"(src), "r"(static_cast<int>(on)) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p cp.async.ca.shared.global [%0], [%1], 8;\n\t}"
                 ::"r"(dst), "l"(src), "r"(static_cast<int>(on)) : "memory");
}
__device__ __forceinline__ void copy_int(uint32_t dst, const int32_t* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
constexpr int kStages = 4, kAhead = kStages - 1;

// A pass is 32 >> shift heads of one row.  A warp takes runs of `run` passes of a row, the runs first, first + stride,
// ...: it makes the row's turns once a run, and from pass to pass only adds to its addresses.
struct Passes {
  unsigned row, k, end, at, rows, of_row, run, of_run, drow, dat;
  __device__ __forceinline__ Passes(unsigned first, unsigned stride, long long rows_, unsigned of_row_, unsigned run_)
      : rows(static_cast<unsigned>(rows_)), of_row(of_row_), run(run_) {
    of_run = (of_row + run - 1) / run;
    row = first / of_run;
    at = first % of_run;
    drow = stride / of_run;
    dat = stride % of_run;
    enter();
  }
  __device__ __forceinline__ void enter() {
    k = at * run;
    end = min(k + run, of_row);
  }
  __device__ __forceinline__ bool left() const { return row < rows; }
  // The next pass; whether it begins a run.
  __device__ __forceinline__ bool next() {
    if (++k < end) return false;
    row += drow;
    at += dat;
    if (at >= of_run) { at -= of_run; ++row; }
    enter();
    return true;
  }
  __device__ __forceinline__ void next_run() {
    k = end - 1;
    next();
  }
};

// Addresses in bytes of a lane's first vector of a head.
struct Heads {
  const char* p; long long row, head;
  template <typename T>
  __device__ __forceinline__ Heads(const void* base, long long row_, long long head_, int a, T)
      : p(static_cast<const char*>(base) + a * static_cast<int>(sizeof(T))), row(row_ * static_cast<int>(sizeof(T))),
        head(head_ * static_cast<int>(sizeof(T))) {}
  __device__ __forceinline__ const char* at(unsigned r, int h) const { return p + r * row + h * head; }
};
template <typename T, int V>
__device__ __forceinline__ void store_vec(const char* y, const float2 (&v)[V / 2]) {
  Vec<T, V>::store(reinterpret_cast<T*>(const_cast<char*>(y)), v);
}

// A block's warps take the passes of one side.  HBM-bound (q and k once in, once out): 18944 rows of 32 and 32 heads of
// 128 in bf16 take 101 us, 6.1 TB/s where a copy reaches 6.8, with issue slots 76 % busy; 3 CTAs an SM, for 80 registers hold
// a lane's 16 columns and their turns, and the loads in flight need none.
template <typename T, int V, bool ADJ, bool APPEND>
__global__ void __launch_bounds__(kThreads, kRotateCtas) rotate_kernel(const __grid_constant__ RopeTab tab,
                                                                       const __grid_constant__ Job job, int shift) {
  constexpr int VB = V * sizeof(T);
  __shared__ Freqs freqs;
  __shared__ __align__(16) float turns_buf[kWarps][kMaxHead];
  __shared__ __align__(16) float weight[kMaxHead];
  __shared__ int row_buf[kWarps][kStages][8];  // positions on up to 4 axes, slot
  extern __shared__ uint4 stages[];            // [kWarps][kStages][2][32]
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = 32 >> shift;
  const int si = side_of_block(job);
  const Side& sd = job.s[si];
  const Lane ln = lane_of<V, ADJ>(tab, shift);
  const unsigned blk = blockIdx.x - job.first[si], blocks = job.first[si + 1] - job.first[si];
  const bool values = APPEND && sd.kind == kValues, paged = APPEND && sd.kind != kRowsOut, norm = sd.w != nullptr;
  const int heads = ln.on ? sd.heads : 0;      // of this lane
  const int heads2 = ln.two ? heads : 0;
  const int gap = (ln.b - ln.a) * static_cast<int>(sizeof(T));
  uint4* mine = stages + warp * (kStages * 64) + lane;
#pragma unroll
  for (int n = 0; n < 2 * kStages; ++n) mine[n * 32] = make_uint4(0, 0, 0, 0);
  __syncthreads();                             // before the copies to the same places
  const uint32_t mine_at = smem_u32(mine), row_at = smem_u32(row_buf[warp][0]);
  const Heads in(sd.x, sd.xrow, sd.xhead, ln.a, T());
  const Heads out(sd.y, paged ? 0 : sd.yrow, paged ? static_cast<long long>(job.page) * tab.dh : sd.yhead, ln.a, T());
  const long long in_step = per * in.head, out_step = per * out.head;
  Passes ld(warp * blocks + blk, blocks * kWarps, job.rows, (sd.heads + per - 1) / per, job.run[si]), cp = ld;
  int lh = 0, ch = 0;                          // head of the lane in the pass loaded and in the one computed
  const char* lx = nullptr;
  char* cy = nullptr;
  bool enter = true;
  const auto load = [&](int stage) {
    if (enter && !ld.left()) { enter = false; lh = 1 << 30; }          // no passes left: no heads either
    if (enter) {
      lh = ld.k * per + (lane >> shift);
      lx = in.at(ld.row, lh);
      if (lane < tab.axes && tab.rot > 0 && !values) copy_int(row_at + (stage * 8 + lane) * 4, job.pos + lane * job.rows + ld.row);
      if (APPEND && lane == 4) copy_int(row_at + (stage * 8 + 4) * 4, job.slots + ld.row);
    }
    copy_vec<VB>(mine_at + stage * 1024, lx, lh < heads);
    copy_vec<VB>(mine_at + stage * 1024 + 512, lx + gap, lh < heads2);
    lh += per;
    lx += in_step;
    if (ld.left()) enter = ld.next();
    cp_async_commit();
  };
#pragma unroll
  for (int n = 0; n < kAhead; ++n) load(n);
  fill_weight(weight, static_cast<const T*>(sd.w), tab.dh);
  fill_freqs(freqs, tab);                      // and a barrier
  const float* w_a = weight + (ln.on ? ln.a : 0);
  const float* w_b = weight + (ln.two ? ln.b : 0);
  const LaneSum lane_sum(shift);
  const float inv = tab.inv_dh;
  Turns<V> turns;
  unsigned turned_row = 0xffffffffu;
  bool begins = true, write = true;
  for (int stage = 0; cp.left(); stage = stage + 1 == kStages ? 0 : stage + 1) {
    cp_async_wait_group<kAhead - 1>();
    load(stage == 0 ? kStages - 1 : stage - 1);        // read by this lane in the round before
    if (begins) {
      const int at = lane < 8 ? row_buf[warp][stage][lane] : 0;  // lanes read what they copied
      ch = cp.k * per + (lane >> shift);
      cy = const_cast<char*>(out.at(cp.row, ch));
      if (APPEND) {
        const int slot = __shfl_sync(0xffffffffu, at, 4);
        write = good_slot(job, slot);
        if (paged && write)
          cy += (static_cast<long long>(slot / job.page) * sd.heads * job.page + slot % job.page) * tab.dh * static_cast<int>(sizeof(T));
      }
      if (!values && cp.row != turned_row) {
        turns.make(tab, freqs, at, lane, ln, turns_buf[warp]);
        turned_row = cp.row;
      }
    }
    if (!APPEND || write) {
      Vec<T, V> va, vb;
      va.load(mine + stage * 64);
      vb.load(mine + stage * 64 + 32);
      float2 a[V / 2], b[V / 2];
      va.get(a);
      vb.get(b);
      if (norm) {
        const float ss = lane_sum(dot2(a, a, dot2(b, b, 0.f)) * lane_sum.part);
        const float r = rsqrtf(fmaf(ss, inv, tab.eps));
        const float2 r2 = make_float2(r, r);
        float2 wa[V / 2], wb[V / 2];
        weight_at<V>(w_a, wa);
        weight_at<V>(w_b, wb);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          a[i] = mul2(a[i], mul2(r2, wa[i]));
          b[i] = mul2(b[i], mul2(r2, wb[i]));
        }
      }
      if (!values) turns.template turn<ADJ, 1>(a, b, ln.turned, tab.rot == tab.dh);
      if (ch < heads) store_vec<T, V>(cy, a);
      if (ch < heads2) store_vec<T, V>(cy + gap, b);
    }
    ch += per;
    cy += out_step;
    begins = cp.next();
  }
}

// The same passes; the lanes' sums of g n stay in registers until the end (two CTAs an SM, 128 registers).  HBM's work is q, k
// and the gradients of both once in, their gradients once out; bound by instructions and by the warps that hide their
// latency: 16171 rows of 28 and 4 heads of 128 in bf16 take 80 us with the sums of dw, 5.0 TB/s, issue slots 65 % busy.
// (8-byte vectors and three CTAs 128 us; x, w and turns read again from shared memory, three CTAs, 134.)
template <typename T, int V, bool ADJ>
__global__ void __launch_bounds__(kThreads, kGradCtas) grad_kernel(const __grid_constant__ RopeTab tab,
                                                                   const __grid_constant__ Job job, int shift) {
  constexpr int VB = V * sizeof(T);
  __shared__ Freqs freqs;
  __shared__ __align__(16) float turns_buf[kWarps][kMaxHead];
  __shared__ __align__(16) float weight[kMaxHead];
  __shared__ int row_buf[kWarps][kStages][4];
  extern __shared__ uint4 stages[];            // [kWarps][kStages][4][32]
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = 32 >> shift;
  const int si = side_of_block(job);
  const Side& sd = job.s[si];
  const Lane ln = lane_of<V, ADJ>(tab, shift);
  const unsigned blk = blockIdx.x - job.first[si], blocks = job.first[si + 1] - job.first[si];
  const bool norm = sd.w != nullptr;
  const int heads = ln.on ? sd.heads : 0, heads2 = ln.two ? heads : 0;
  const int gap = (ln.b - ln.a) * static_cast<int>(sizeof(T));
  uint4* mine = stages + warp * (kStages * 128) + lane;
#pragma unroll
  for (int n = 0; n < 4 * kStages; ++n) mine[n * 32] = make_uint4(0, 0, 0, 0);
  // behind a row's turns too: a lane without columns turns its zeros by what stands there and adds them to its head's sums,
  // which an earlier kernel's words could make NaN
  for (int c = tab.rot + lane; c < kMaxHead; c += 32) turns_buf[warp][c] = 0.f;
  __syncthreads();                             // before the copies to the same places
  const uint32_t mine_at = smem_u32(mine), row_at = smem_u32(row_buf[warp][0]);
  const Heads ing(sd.g, sd.grow, sd.ghead, ln.a, T()), inx(sd.x, sd.xrow, sd.xhead, ln.a, T()), out(sd.y, sd.yrow, sd.yhead, ln.a, T());
  const long long g_step = per * ing.head, x_step = per * inx.head, out_step = per * out.head;
  Passes ld(warp * blocks + blk, blocks * kWarps, job.rows, (sd.heads + per - 1) / per, job.run[si]), cp = ld;
  int lh = 0, ch = 0;
  const char *lg = nullptr, *lx = nullptr;
  char* cy = nullptr;
  bool enter = true;
  const auto load = [&](int stage) {
    if (enter && !ld.left()) { enter = false; lh = 1 << 30; }          // no passes left: no heads either
    if (enter) {
      lh = ld.k * per + (lane >> shift);
      lg = ing.at(ld.row, lh);
      lx = inx.at(ld.row, lh);
      if (lane < tab.axes && tab.rot > 0) copy_int(row_at + (stage * 4 + lane) * 4, job.pos + lane * job.rows + ld.row);
    }
    const uint32_t to = mine_at + stage * 2048;
    copy_vec<VB>(to, lg, lh < heads);
    copy_vec<VB>(to + 512, lg + gap, lh < heads2);
    copy_vec<VB>(to + 1024, lx, lh < heads && norm);
    copy_vec<VB>(to + 1536, lx + gap, lh < heads2 && norm);
    lh += per;
    lg += g_step;
    lx += x_step;
    if (ld.left()) enter = ld.next();
    cp_async_commit();
  };
#pragma unroll
  for (int n = 0; n < kAhead; ++n) load(n);
  fill_weight(weight, static_cast<const T*>(sd.w), tab.dh);
  fill_freqs(freqs, tab);                      // and a barrier
  const float* w_a = weight + (ln.on ? ln.a : 0);
  const float* w_b = weight + (ln.two ? ln.b : 0);
  float2 da[V / 2], db[V / 2];
#pragma unroll
  for (int i = 0; i < V / 2; ++i) da[i] = db[i] = make_float2(0.f, 0.f);
  const LaneSum lane_sum(shift);
  const float inv = tab.inv_dh, minus = -inv * lane_sum.part;
  Turns<V> turns;
  unsigned turned_row = 0xffffffffu;
  bool begins = true;
  for (int stage = 0; cp.left(); stage = stage + 1 == kStages ? 0 : stage + 1) {
    cp_async_wait_group<kAhead - 1>();
    load(stage == 0 ? kStages - 1 : stage - 1);        // read by this lane in the round before
    if (begins) {
      ch = cp.k * per + (lane >> shift);
      cy = const_cast<char*>(out.at(cp.row, ch));
      if (cp.row != turned_row) {
        turns.make(tab, freqs, lane < 4 ? row_buf[warp][stage][lane] : 0, lane, ln, turns_buf[warp]);
        turned_row = cp.row;
      }
    }
    const uint4* from = mine + stage * 128;
    Vec<T, V> va, vb;
    va.load(from);
    vb.load(from + 32);
    float2 a[V / 2], b[V / 2];
    va.get(a);
    vb.get(b);
    turns.template turn<ADJ, -1>(a, b, ln.turned, tab.rot == tab.dh);
    if (norm) {
      float2 na[V / 2], nb[V / 2], ha[V / 2], hb[V / 2];     // x, later n = x r; g w
      va.load(from + 64);
      vb.load(from + 96);
      va.get(na);
      vb.get(nb);
      weight_at<V>(w_a, ha);
      weight_at<V>(w_b, hb);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        ha[i] = mul2(a[i], ha[i]);
        hb[i] = mul2(b[i], hb[i]);
      }
      const float ss = lane_sum(dot2(na, na, dot2(nb, nb, 0.f)) * lane_sum.part);
      const float r = rsqrtf(fmaf(ss, inv, tab.eps));
      const float m = lane_sum(dot2(ha, na, dot2(hb, nb, 0.f)) * minus) * r;       // -mean(g w n)
      const float2 r2 = make_float2(r, r), m2 = make_float2(m, m);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        na[i] = mul2(na[i], r2);
        nb[i] = mul2(nb[i], r2);
        if (ch < heads) {                      // elsewhere n may be 0 times an infinite r
          da[i] = fma2(a[i], na[i], da[i]);
          db[i] = fma2(b[i], nb[i], db[i]);
        }
        a[i] = mul2(r2, fma2(na[i], m2, ha[i]));
        b[i] = mul2(r2, fma2(nb[i], m2, hb[i]));
      }
    }
    if (ch < heads) store_vec<T, V>(cy, a);
    if (ch < heads2) store_vec<T, V>(cy + gap, b);
    ch += per;
    cy += out_step;
    begins = cp.next();
  }
  if (!norm) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V / 2; ++i) {
    float2 fa = da[i], fb = db[i];
    for (int o = 16; o >= 1 << shift; o >>= 1) {
      fa.x += __shfl_xor_sync(0xffffffffu, fa.x, o);
      fa.y += __shfl_xor_sync(0xffffffffu, fa.y, o);
      fb.x += __shfl_xor_sync(0xffffffffu, fb.x, o);
      fb.y += __shfl_xor_sync(0xffffffffu, fb.y, o);
    }
    if (lane >> shift == 0 && ln.on) {
      turns_buf[warp][ln.a + 2 * i] = fa.x;
      turns_buf[warp][ln.a + 2 * i + 1] = fa.y;
      if (ln.two) {
        turns_buf[warp][ln.b + 2 * i] = fb.x;
        turns_buf[warp][ln.b + 2 * i + 1] = fb.y;
      }
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < tab.dh; c += kThreads) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) s += turns_buf[k][c];
    sd.part[static_cast<long long>(blk) * tab.dh + c] = s;
  }
}

// ------------------------------------------------------------------ any width, any alignment: a lane S pairs
// Pair j's columns; b = -1 where a has no partner.
struct Pair { int a, b; bool turned; };
__device__ __forceinline__ Pair pair_of(const RopeTab& t, int j) {
  Pair p;
  const int half = t.rot >> 1;
  p.turned = j < half;
  if (p.turned && !t.adjacent) { p.a = j; p.b = half + j; return p; }
  p.a = 2 * j;
  p.b = 2 * j + 1 < t.dh ? 2 * j + 1 : -1;
  return p;
}

// A lane's pairs j0 + 2^shift i of a head, with what does not change from head to head.
template <typename T, int S>
struct Pairs {
  int a[S], b[S];                      // -1: none
  bool turned[S];
  float wa[S], wb[S], c[S], s[S];
  unsigned long long turn[S];
  const int32_t* pos[S];
  __device__ __forceinline__ Pairs(const RopeTab& t, const Job& job, const T* w, int j0, int shift) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int j = j0 + (i << shift);
      const bool on = j < (t.dh + 1) >> 1;
      const Pair p = pair_of(t, on ? j : 0);
      a[i] = on ? p.a : -1;
      b[i] = on ? p.b : -1;
      turned[i] = on && p.turned;
      wa[i] = w && a[i] >= 0 ? to_f32(w[a[i]]) : 1.f;
      wb[i] = w && b[i] >= 0 ? to_f32(w[b[i]]) : 1.f;
      turn[i] = turned[i] ? t.turn[j] : 0;
      pos[i] = turned[i] ? job.pos + t.axis[j] * job.rows : nullptr;
      c[i] = 1.f;
      s[i] = 0.f;
    }
  }
  __device__ __forceinline__ void make(unsigned row) {
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (turned[i]) {
        const unsigned long long ph = turn[i] * static_cast<unsigned long long>(static_cast<long long>(__ldg(pos[i] + row)));
        const float2 cs = cos_sin(static_cast<uint32_t>(ph >> 32));
        c[i] = cs.x;
        s[i] = cs.y;
      }
  }
  // Without conditions, so that all of a lane's loads are under way before the first is waited for: column 0 stands
  // for one that is not there.
  __device__ __forceinline__ void load(const T* x, T (&va)[S], T (&vb)[S]) const {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      va[i] = x[max(a[i], 0)];
      vb[i] = x[max(b[i], 0)];
    }
  }
  __device__ __forceinline__ void get(const T (&va)[S], const T (&vb)[S], float (&fa)[S], float (&fb)[S]) const {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      fa[i] = a[i] >= 0 ? to_f32(va[i]) : 0.f;
      fb[i] = b[i] >= 0 ? to_f32(vb[i]) : 0.f;
    }
  }
  __device__ __forceinline__ void store(T* y, const float (&va)[S], const float (&vb)[S]) const {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      if (a[i] >= 0) y[a[i]] = from_f32<T>(va[i]);
      if (b[i] >= 0) y[b[i]] = from_f32<T>(vb[i]);
    }
  }
  template <int SIGN>
  __device__ __forceinline__ void turn_all(float (&va)[S], float (&vb)[S]) const {
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (turned[i]) {
        const float u = va[i] * c[i] - SIGN * vb[i] * s[i];
        vb[i] = vb[i] * c[i] + SIGN * va[i] * s[i];
        va[i] = u;
      }
  }
};
constexpr int kAnyPairs = 8;         // pairs that a lane loads at once
template <int S> constexpr int kAnyCtas = S == 4 ? kGradCtas : kRotateCtas;      // 256 columns: 283 us, three CTAs 404

// For what vectors cannot take: passes as above, turns once a run, but loads of single elements, kAnyPairs / S passes of
// them in registers at once.  Bound by instructions (issue slots 60 % busy at a third of the warps): 18944 rows of 32 and
// 32 heads of 128 that begin on odd elements take 197 us by themselves, aligned ones 111; 12000 rows of 56 and 8 heads of
// 36, 18 pairs, 73 (floor 16).  With a warp a head and its turns made anew they took 1186 and 279.  Two pairs a lane up to
// 128 columns (one: 91 us for the heads of 36; four: 99), four beyond.
template <typename T, int S, bool APPEND>
__global__ void __launch_bounds__(kThreads, kAnyCtas<S>) rotate_any_kernel(const __grid_constant__ RopeTab tab,
                                                                        const __grid_constant__ Job job, int shift) {
  constexpr int U = kAnyPairs / S;
  pdl_enter();
  const int lane = threadIdx.x & 31, sub = lane >> shift, per = 32 >> shift;
  const int si = side_of_block(job);
  const Side& sd = job.s[si];
  const unsigned blk = blockIdx.x - job.first[si], blocks = job.first[si + 1] - job.first[si];
  const bool values = APPEND && sd.kind == kValues, paged = APPEND && sd.kind != kRowsOut, norm = sd.w != nullptr;
  const long long yhead = paged ? static_cast<long long>(job.page) * tab.dh : sd.yhead;
  Pairs<T, S> pairs(tab, job, static_cast<const T*>(sd.w), lane & ((1 << shift) - 1), shift);
  const LaneSum lane_sum(shift);
  const float inv = tab.inv_dh;
  for (Passes at((threadIdx.x >> 5) * blocks + blk, blocks * kWarps, job.rows, (sd.heads + per - 1) / per, job.run[si]); at.left(); at.next_run()) {
    const T* x = static_cast<const T*>(sd.x) + at.row * sd.xrow;
    T* y = static_cast<T*>(sd.y) + (paged ? 0 : at.row * sd.yrow);
    if (APPEND) {
      const int slot = __ldg(job.slots + at.row);
      if (!good_slot(job, slot)) continue;
      if (paged) y += (static_cast<long long>(slot / job.page) * sd.heads * job.page + slot % job.page) * tab.dh;
    }
    if (!values) pairs.make(at.row);
    for (unsigned k = at.k; k < at.end; k += U) {
      T ra[U][S], rb[U][S];
#pragma unroll
      for (int u = 0; u < U; ++u) pairs.load(x + min(static_cast<int>(min(k + u, at.end - 1)) * per + sub, sd.heads - 1) * sd.xhead, ra[u], rb[u]);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k + u >= at.end) break;
        const int h = (k + u) * per + sub;
        float a[S], b[S];
        pairs.get(ra[u], rb[u], a, b);
        if (norm) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < S; ++i) ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
          const float r = rsqrtf(fmaf(lane_sum(ss * lane_sum.part), inv, tab.eps));
#pragma unroll
          for (int i = 0; i < S; ++i) {
            a[i] *= r * pairs.wa[i];
            b[i] *= r * pairs.wb[i];
          }
        }
        if (!values) pairs.template turn_all<1>(a, b);
        if (h < sd.heads) pairs.store(y + h * yhead, a, b);
      }
    }
  }
}

// Its gradient: dx, and this block's sum of g n per column into part[block of the side][dh].  The same rows of 32 and 32
// heads take 310 us (aligned 156), of 56 and 8 heads of 36 columns 110 (floor 25).
template <typename T, int S>
__global__ void __launch_bounds__(kThreads, kGradCtas) grad_any_kernel(const __grid_constant__ RopeTab tab,
                                                                       const __grid_constant__ Job job, int shift) {
  constexpr int U = kAnyPairs / S;
  __shared__ float red[kWarps][kMaxHead];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane >> shift, per = 32 >> shift;
  const int si = side_of_block(job);
  const Side& sd = job.s[si];
  const unsigned blk = blockIdx.x - job.first[si], blocks = job.first[si + 1] - job.first[si];
  const bool norm = sd.w != nullptr;
  Pairs<T, S> pairs(tab, job, static_cast<const T*>(sd.w), lane & ((1 << shift) - 1), shift);
  const LaneSum lane_sum(shift);
  const float inv = tab.inv_dh;
  float da[S] = {}, db[S] = {};
  for (Passes at(warp * blocks + blk, blocks * kWarps, job.rows, (sd.heads + per - 1) / per, job.run[si]); at.left(); at.next_run()) {
    const T* g = static_cast<const T*>(sd.g) + at.row * sd.grow;
    const T* x = static_cast<const T*>(sd.x) + at.row * sd.xrow;
    T* y = static_cast<T*>(sd.y) + at.row * sd.yrow;
    pairs.make(at.row);
    for (unsigned k = at.k; k < at.end; k += U) {
      T ga[U][S], gb[U][S], xa[U][S], xb[U][S];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = min(static_cast<int>(min(k + u, at.end - 1)) * per + sub, sd.heads - 1);
        pairs.load(g + h * sd.ghead, ga[u], gb[u]);
        if (norm) pairs.load(x + h * sd.xhead, xa[u], xb[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k + u >= at.end) break;
        const int h = (k + u) * per + sub;
        float a[S], b[S], na[S], nb[S];
        pairs.get(ga[u], gb[u], a, b);
        pairs.template turn_all<-1>(a, b);
        if (norm) {
          float ss = 0.f, dot = 0.f;
          pairs.get(xa[u], xb[u], na, nb);
#pragma unroll
          for (int i = 0; i < S; ++i) {
            ss = fmaf(na[i], na[i], fmaf(nb[i], nb[i], ss));
            dot = fmaf(a[i] * pairs.wa[i], na[i], fmaf(b[i] * pairs.wb[i], nb[i], dot));
          }
          const float r = rsqrtf(fmaf(lane_sum(ss * lane_sum.part), inv, tab.eps));
          const float m = lane_sum(dot * lane_sum.part) * r * inv;             // mean(g w n)
#pragma unroll
          for (int i = 0; i < S; ++i) {
            na[i] *= r;
            nb[i] *= r;
            if (h < sd.heads) {                                // the others are the last head again
              da[i] = fmaf(a[i], na[i], da[i]);
              db[i] = fmaf(b[i], nb[i], db[i]);
            }
            a[i] = r * (a[i] * pairs.wa[i] - na[i] * m);
            b[i] = r * (b[i] * pairs.wb[i] - nb[i] * m);
          }
        }
        if (h < sd.heads) pairs.store(y + h * sd.yhead, a, b);
      }
    }
  }
  if (!norm) return;
#pragma unroll
  for (int i = 0; i < S; ++i) {
    for (int o = 16; o >= 1 << shift; o >>= 1) {
      da[i] += __shfl_xor_sync(0xffffffffu, da[i], o);
      db[i] += __shfl_xor_sync(0xffffffffu, db[i], o);
    }
    if (sub == 0 && pairs.a[i] >= 0) red[warp][pairs.a[i]] = da[i];
    if (sub == 0 && pairs.b[i] >= 0) red[warp][pairs.b[i]] = db[i];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < tab.dh; c += kThreads) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) s += red[k][c];
    sd.part[static_cast<long long>(blk) * tab.dh + c] = s;
  }
}

// dw[c] = sum over a side's blocks of part[b][c], in a fixed order: 32 columns a CTA, every 32nd block a warp.  Latency
// only (156 KB a side): 7.5 us by itself with cold caches; the gradient of 16171 rows took 80 us with eight warps, 79 with 32.
constexpr int kSumWarps = 32;         // as many as columns
struct Sums { const float* part[2]; float* dw[2]; int blocks[2]; };
__global__ void __launch_bounds__(32 * kSumWarps) grad_sum_kernel(const __grid_constant__ Sums g, int dh) {
  __shared__ float red[kSumWarps][33];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, side = blockIdx.y;
  float s = 0.f;
  if (c < dh) {
#pragma unroll 10
    for (int b = warp; b < g.blocks[side]; b += kSumWarps) s += g.part[side][static_cast<long long>(b) * dh + c];
  }
  red[warp][lane] = s;
  __syncthreads();
  // warp w adds the warps' sums of column w
  s = red[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0 && blockIdx.x * 32 + warp < dh && g.dw[side]) g.dw[side][blockIdx.x * 32 + warp] = s;
}

// f / 2 pi modulo 1 in units of 2^-64, rounded: f times 1 / 2 pi as a double p and the rest of it (1 / 2 pi in two doubles,
// the product's own rest exact by fma), whole turns dropped from both before they are added.  (fmod: a compiler that
// contracts p - floor(p) to one fma would take p's rest in twice.)
unsigned long long turn_of(double f) {
  constexpr double hi = 0.15915494309189535, lo = -9.839338337591243e-18;
  const double p = f * hi, rest = std::fma(f, hi, -p) + f * lo;
  const double a = std::ldexp(std::fmod(p, 1.0), 64), whole = std::floor(a);     // below 2^64
  double b = std::ldexp(rest - std::nearbyint(rest), 64);                        // half a turn at most
  if (b >= 0x1p63) b -= 0x1p64;
  return static_cast<unsigned long long>(whole) + static_cast<unsigned long long>(std::llrint(a - whole + b));
}

int elem_size(int type) { return type == MAP_F32 ? 4 : 2; }
bool good_type(int type) { return type == MAP_BF16 || type == MAP_F16 || type == MAP_F32; }
bool absent(const map_heads* h) { return !h || h->heads == 0; }

// A side as input: present, its strides not negative, aligned to its elements.
bool good_in(const map_heads* h, int type, long long rows) {
  return (h->p || rows == 0) && h->heads > 0 && h->row >= 0 && h->head >= 0 &&
         reinterpret_cast<uintptr_t>(h->p) % elem_size(type) == 0 && rows * h->heads < (1ll << 31);
}
// As output too: no two of its vectors overlap.
bool good_out(const map_heads* h, int type, long long rows, int dh, int heads) {
  if (!h || h->heads != heads || !good_in(h, type, rows)) return false;
  return distinct_vectors(h->row, rows, h->head, heads, dh);
}

int check_rotation(const map_rope* r, int type, long long rows, const int32_t* pos) {
  if (!r || !good_type(type) || rows < 0) return MAP_EINVAL;
  if (r->tab.rot > 0 && rows > 0 && !pos) return MAP_EINVAL;
  if (rows > 0x7fffffffll) return MAP_EUNSUPPORTED;
  return MAP_OK;
}

Side side_of(const map_heads* in, const map_heads* out, const void* w) {
  Side s{};
  s.x = in->p;
  s.xrow = in->row;
  s.xhead = in->head;
  if (out) {
    s.y = out->p;
    s.yrow = out->row;
    s.yhead = out->head;
  }
  s.w = w;
  s.heads = in->heads;
  return s;
}

// Whether `bytes` (16 or 8) is the alignment of every vector that a job touches, in elements of `size` bytes.
bool aligned_to(const Job& job, int sides, size_t bytes, int size) {
  uintptr_t all = 0;
  for (int i = 0; i < sides; ++i) {
    const Side& s = job.s[i];
    all |= reinterpret_cast<uintptr_t>(s.x) | reinterpret_cast<uintptr_t>(s.y) | reinterpret_cast<uintptr_t>(s.w) |
           reinterpret_cast<uintptr_t>(s.g);
    all |= static_cast<uintptr_t>(s.xrow | s.xhead | s.yrow | s.yhead | s.grow | s.ghead) * size;
  }
  return all % bytes == 0;
}

// Columns of a vector: the widest that the columns of a head, of its rotated half and every address are multiples of;
// 0: the kernels for any alignment.
int vector_of(const RopeTab& t, const Job& job, int sides, int size) {
  for (int v = size == 4 ? 4 : 8; v >= 4; v >>= 1)
    if (t.dh % v == 0 && (t.adjacent || t.rot / 2 % v == 0) && aligned_to(job, sides, v * size, size)) return v;
  return 0;
}

int shift_of(const RopeTab& t, int v) {
  const int np = ((t.dh + 1) / 2 + v - 1) / v;
  int s = 0;
  while ((1 << s) < np) ++s;
  return s;
}

// Passes of a run: the split of a row that ends first where its runs are dealt to `warps` warps and the row's turns cost
// as much as a pass.  (At least four runs a warp instead: a prompt's append 33.7 us, not 31.8.)
unsigned run_of(long long rows, long long of_row, long long warps) {
  long long best = 0;
  unsigned run = 1;
  for (long long parts = 1; parts <= std::min(of_row, 64ll); ++parts) {
    const long long r = (of_row + parts - 1) / parts, runs = rows * ((of_row + r - 1) / r);
    const long long end = (runs + warps - 1) / warps * (r + 1);
    if (parts == 1 || end < best) {
      best = end;
      run = static_cast<unsigned>(r);
    }
  }
  return run;
}

// Blocks of the sides: `limit` in proportion to what a row of them costs, at most one for kWarps passes of `per` heads.
// In thirds of a pass: a pass 3 (of values, which are copied, 2), a row's turns 2.  (By passes alone the keys of grouped
// heads, with a pass a row, were the last to end: the gradient of 16171 rows of 28 and 4 heads took 100 us, not 82.)
void spread_blocks(Job& job, int sides, int per, int limit) {
  long long of_row[3] = {}, cost[3] = {}, all = 0;
  for (int i = 0; i < sides; ++i) {
    of_row[i] = (job.s[i].heads + per - 1) / per;
    all += cost[i] = job.rows * (job.s[i].kind == kValues ? 2 * of_row[i] : 3 * of_row[i] + 2);
  }
  unsigned at = 0;
  for (int i = 0; i < 4; ++i) {
    job.first[i] = at;
    if (i >= sides) continue;
    const long long share = std::max(1ll, limit * cost[i] / all), most = (job.rows * of_row[i] + kWarps - 1) / kWarps;
    const long long blocks = std::min(share, most);
    job.run[i] = run_of(job.rows, of_row[i], blocks * kWarps);
    at += static_cast<unsigned>(blocks);
  }
}

template <typename T, int V, bool ADJ, bool APPEND>
cudaError_t run_rotate(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int shift = shift_of(t, V);
  spread_blocks(job, sides, 32 >> shift, 152 * kRotateCtas);
  constexpr size_t smem = kWarps * kStages * 64 * sizeof(uint4);
  static_assert(smem <= 34 * 1024, "with 12 KB of fixed arrays within what a kernel has without asking");
  return launch_k(rotate_kernel<T, V, ADJ, APPEND>, dim3(job.first[3]), dim3(kThreads), smem, st, t, job, shift);
}

template <typename T, int S, bool APPEND>
cudaError_t run_rotate_any(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int shift = shift_of(t, S);
  spread_blocks(job, sides, 32 >> shift, 152 * kAnyCtas<S>);
  return launch_k(rotate_any_kernel<T, S, APPEND>, dim3(job.first[3]), dim3(kThreads), 0, st, t, job, shift);
}

template <typename T, int V, bool APPEND>
cudaError_t rotate_width(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  return t.adjacent ? run_rotate<T, V, true, APPEND>(t, job, sides, st) : run_rotate<T, V, false, APPEND>(t, job, sides, st);
}

template <typename T, bool APPEND>
cudaError_t rotate_job(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int v = vector_of(t, job, sides, sizeof(T));
  if (v == 4) return rotate_width<T, 4, APPEND>(t, job, sides, st);
  if constexpr (sizeof(T) == 2)
    if (v == 8) return rotate_width<T, 8, APPEND>(t, job, sides, st);
  return t.dh <= 128 ? run_rotate_any<T, 2, APPEND>(t, job, sides, st) : run_rotate_any<T, 4, APPEND>(t, job, sides, st);
}

template <typename T, int V, bool ADJ>
cudaError_t run_grad(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int shift = shift_of(t, V);
  spread_blocks(job, sides, 32 >> shift, kGradBlocks);
  constexpr size_t smem = kWarps * kStages * 128 * sizeof(uint4);
  const cudaError_t e = cudaFuncSetAttribute(grad_kernel<T, V, ADJ>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_k(grad_kernel<T, V, ADJ>, dim3(job.first[3]), dim3(kThreads), smem, st, t, job, shift);
}

template <typename T, int S>
cudaError_t run_grad_any(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int shift = shift_of(t, S);
  spread_blocks(job, sides, 32 >> shift, kGradBlocks);
  return launch_k(grad_any_kernel<T, S>, dim3(job.first[3]), dim3(kThreads), 0, st, t, job, shift);
}

template <typename T>
cudaError_t grad_job(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int v = vector_of(t, job, sides, sizeof(T));
  if (v == 4) return t.adjacent ? run_grad<T, 4, true>(t, job, sides, st) : run_grad<T, 4, false>(t, job, sides, st);
  if constexpr (sizeof(T) == 2)
    if (v == 8) return t.adjacent ? run_grad<T, 8, true>(t, job, sides, st) : run_grad<T, 8, false>(t, job, sides, st);
  return t.dh <= 128 ? run_grad_any<T, 2>(t, job, sides, st) : run_grad_any<T, 4>(t, job, sides, st);
}

}  // namespace
}  // namespace mapk

using namespace mapk;

extern "C" {

int map_rope_init(int dh, int rot, int adjacent, int n_axes, const double* inv_freq, const int32_t* axis, double eps,
                  map_rope** out) {
  if (!out) return MAP_EINVAL;
  *out = nullptr;
  if (dh < 1 || dh > kMaxHead || rot < 0 || rot > dh || rot % 2 || n_axes < 1 || n_axes > 4) return MAP_EINVAL;
  if ((adjacent != 0 && adjacent != 1) || !(eps >= 0.0) || !std::isfinite(eps) || (rot > 0 && !inv_freq)) return MAP_EINVAL;
  for (int i = 0; i < rot / 2; ++i) {
    if (!std::isfinite(inv_freq[i])) return MAP_EINVAL;
    if (axis && (axis[i] < 0 || axis[i] >= n_axes)) return MAP_EINVAL;
  }
  map_rope* r = new (std::nothrow) map_rope();
  if (!r) return MAP_ENOMEM;
  RopeTab& t = r->tab;
  t.dh = dh;
  t.rot = rot;
  t.adjacent = adjacent;
  t.axes = n_axes;
  t.eps = static_cast<float>(eps);
  t.inv_dh = 1.f / static_cast<float>(dh);
  for (int i = 0; i < rot / 2; ++i) {
    const unsigned long long turn = turn_of(std::fabs(inv_freq[i]));
    t.turn[i] = inv_freq[i] < 0 ? 0 - turn : turn;
    t.axis[i] = static_cast<uint8_t>(axis ? axis[i] : 0);
  }
  *out = r;
  return MAP_OK;
}

void map_rope_destroy(map_rope* r) { delete r; }

int map_qk_rotate(const map_rope* rope, int type, long long rows, const int32_t* pos, const map_heads* q,
                  const map_heads* k, const void* wq, const void* wk, const map_heads* q_out, const map_heads* k_out,
                  void* stream) {
  const int rc = check_rotation(rope, type, rows, pos);
  if (rc != MAP_OK) return rc;
  if (absent(q) && absent(k)) return MAP_EINVAL;
  const RopeTab& t = rope->tab;
  const map_heads* in[2] = {q, k};
  const map_heads* out[2] = {q_out, k_out};
  const void* w[2] = {wq, wk};
  Job job{};
  int sides = 0;
  for (int i = 0; i < 2; ++i) {
    if (absent(in[i])) continue;
    if (!good_in(in[i], type, rows) || !good_out(out[i], type, rows, t.dh, in[i]->heads)) return MAP_EINVAL;
    job.s[sides++] = side_of(in[i], out[i], w[i]);
  }
  if (rows == 0) return MAP_OK;
  job.pos = pos;
  job.rows = rows;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return launch_err(type == MAP_F32   ? rotate_job<float, false>(t, job, sides, st)
                    : type == MAP_F16 ? rotate_job<__half, false>(t, job, sides, st)
                                      : rotate_job<__nv_bfloat16, false>(t, job, sides, st));
}

size_t map_qk_rotate_grad_workspace(const map_rope* rope) {
  return rope ? static_cast<size_t>(2) * kGradBlocks * rope->tab.dh * sizeof(float) : 0;
}

int map_qk_rotate_grad(const map_rope* rope, int type, long long rows, const int32_t* pos, const map_heads* dq_out,
                       const map_heads* dk_out, const map_heads* q, const map_heads* k, const void* wq, const void* wk,
                       const map_heads* dq, const map_heads* dk, float* dwq, float* dwk, void* ws, void* stream) {
  const int rc = check_rotation(rope, type, rows, pos);
  if (rc != MAP_OK) return rc;
  if (absent(dq_out) && absent(dk_out)) return MAP_EINVAL;
  const RopeTab& t = rope->tab;
  const map_heads* g[2] = {dq_out, dk_out};
  const map_heads* x[2] = {q, k};
  const map_heads* out[2] = {dq, dk};
  const void* w[2] = {wq, wk};
  float* dw[2] = {dwq, dwk};
  Job job{};
  Sums sums{};
  int sides = 0;
  bool norm = false;
  for (int i = 0; i < 2; ++i) {
    if (absent(g[i])) {
      if (g[i] && w[i] && dw[i]) {             // no heads: a sum of nothing, in the place behind the one side that has some
        sums.dw[1] = dw[i];
        norm = true;
      }
      continue;
    }
    if (!good_in(g[i], type, rows) || !good_out(out[i], type, rows, t.dh, g[i]->heads)) return MAP_EINVAL;
    if (w[i] && (absent(x[i]) || !good_in(x[i], type, rows) || x[i]->heads != g[i]->heads || !dw[i] || !ws ||
                 !aligned16(ws)))
      return MAP_EINVAL;
    Side& s = job.s[sides];
    s = side_of(w[i] ? x[i] : g[i], out[i], w[i]);
    s.g = g[i]->p;
    s.grow = g[i]->row;
    s.ghead = g[i]->head;
    if (w[i]) {
      s.part = static_cast<float*>(ws) + static_cast<size_t>(sides) * kGradBlocks * t.dh;
      sums.part[sides] = s.part;
      sums.dw[sides] = dw[i];
      norm = true;
    }
    ++sides;
  }
  job.pos = pos;
  job.rows = rows;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (rows > 0)
    e = type == MAP_F32   ? grad_job<float>(t, job, sides, st)
        : type == MAP_F16 ? grad_job<__half>(t, job, sides, st)
                          : grad_job<__nv_bfloat16>(t, job, sides, st);
  for (int i = 0; i < 2; ++i) sums.blocks[i] = i < sides && sums.part[i] ? static_cast<int>(job.first[i + 1] - job.first[i]) : 0;
  if (e == cudaSuccess && norm) e = launch_k(grad_sum_kernel, dim3((t.dh + 31) / 32, 2), dim3(32 * kSumWarps), 0, st, sums, t.dh);
  return launch_err(e);
}

int map_qk_rotate_append(const map_rope* rope, const map_cache* c, int layer, long long rows, const int32_t* pos,
                         const int32_t* slots, const map_heads* q, const map_heads* k, const map_heads* v,
                         const void* wq, const void* wk, const map_heads* q_out, void* stream) {
  int rc = check_cache(c);
  if (rc != MAP_OK) return rc;
  rc = check_rotation(rope, c->type, rows, pos);
  if (rc != MAP_OK) return rc;
  const RopeTab& t = rope->tab;
  if (layer < 0 || layer >= c->layers || t.dh != c->dh) return MAP_EINVAL;
  if (!k || !v || k->heads != c->heads || v->heads != c->heads) return MAP_EINVAL;
  if (!good_in(k, c->type, rows) || !good_in(v, c->type, rows)) return MAP_EINVAL;
  if (!absent(q) && (!good_in(q, c->type, rows) || !good_out(q_out, c->type, rows, t.dh, q->heads))) return MAP_EINVAL;
  const int hq = absent(q) ? 0 : q->heads;
  if (rows == 0) return MAP_OK;
  if (!slots) return MAP_EINVAL;
  if (rows * (hq + 2ll * c->heads) >= (1ll << 31)) return MAP_EUNSUPPORTED;
  const long long plane = static_cast<long long>(c->pages) * c->heads * c->page * c->dh;
  uint16_t* keys = static_cast<uint16_t*>(c->pool) + 2 * layer * plane;
  Job job{};
  int sides = 0;
  if (hq) job.s[sides++] = side_of(q, q_out, wq);
  job.s[sides] = side_of(k, nullptr, wk);
  job.s[sides].y = keys;
  job.s[sides++].kind = kKeys;
  job.s[sides] = side_of(v, nullptr, nullptr);
  job.s[sides].y = keys + plane;
  job.s[sides++].kind = kValues;
  job.pos = pos;
  job.rows = rows;
  job.slots = slots;
  job.page = c->page;
  job.pages = c->pages;
  job.status = c->status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return launch_err(c->type == MAP_F16 ? rotate_job<__half, true>(t, job, sides, st)
                                       : rotate_job<__nv_bfloat16, true>(t, job, sides, st));
}

}  // extern "C"
