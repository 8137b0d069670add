// Queries and keys before a language model's attention: the RMS norm of each head and the rotation
// by position on up to four axes, in one pass (map_qk_rotate), its gradient (map_qk_rotate_grad), and the
// form whose keys and values go to a cache's pages (map_qk_rotate_append).
//
// Mathematics.  Per head x of dh columns: r = (mean x^2 + eps)^(-1/2), z = x r w; pair (a, b) turned by
// t = pos[axis] inv_freq:  y_a = z_a cos t - z_b sin t, y_b = z_b cos t + z_a sin t.  Backward, with g the
// pair turned back (t -> -t) and n = x r:  dx = r (g w - n mean(g w n)),  dw = sum over rows and heads of g n.
//
// Angles.  inv_freq / 2 pi is held as a 64-bit binary fraction of a turn; its product with a position is taken
// modulo 2^64, which drops whole turns exactly, so an angle is as exact at position 2^31 as at 1 (2^-33 turns from
// the 32 bits kept, plus 2^-53 of the frequency).  cos and sin come from the fraction's upper 32 bits in fp32.
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
constexpr int kGradBlocks = 608;     // partial sums of dw: at most this many blocks a side (4 for each of 152 SMs)

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

// Up to three tensors of one launch; side i takes blocks first[i] .. first[i + 1] - 1.
struct Job {
  Side s[3];
  unsigned first[4];
  const int32_t* pos;
  long long rows;
  const int32_t* slots;              // append: a row's slot
  int page, pages;
  int* status;
};

__device__ __forceinline__ int side_of_block(const Job& job) {
  return (blockIdx.x >= job.first[1] ? 1 : 0) + (blockIdx.x >= job.first[2] ? 1 : 0);
}

__device__ __forceinline__ float2 turn_of(const RopeTab& t, int pair, const int32_t* __restrict__ pos, long long rows,
                                          long long row) {
  const unsigned long long ph =
      t.turn[pair] * static_cast<unsigned long long>(static_cast<long long>(__ldg(pos + t.axis[pair] * rows + row)));
  float s, c;
  sincospif(static_cast<float>(static_cast<int>(ph >> 32)) * 0x1p-31f, &s, &c);
  return make_float2(c, s);
}

// Where head h of row `row` goes; nullptr: nowhere (a padding row, or a slot outside the pool).
template <typename T, bool APPEND>
__device__ __forceinline__ T* out_of(const RopeTab& tab, const Job& job, const Side& sd, long long row, int h) {
  if (APPEND) {
    const int slot = __ldg(job.slots + row);
    if (slot < 0 || slot >= job.pages * job.page) {
      if (slot != -1) atomicOr(job.status, ST_BADINDEX);
      return nullptr;
    }
    if (sd.kind != kRowsOut)
      return static_cast<T*>(sd.y) +
             ((static_cast<long long>(slot / job.page) * sd.heads + h) * job.page + slot % job.page) * tab.dh;
  }
  return static_cast<T*>(sd.y) + row * sd.yrow + h * sd.yhead;
}

// ------------------------------------------------------------------ any width, any alignment: a warp a head
// Columns of pair j (lane + 32 i, 4 of them a lane): b = -1 where a has no partner.
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

template <typename T, bool APPEND>
__global__ void __launch_bounds__(kThreads) rotate_any_kernel(const __grid_constant__ RopeTab tab,
                                                              const __grid_constant__ Job job) {
  pdl_enter();
  const int si = side_of_block(job);
  const Side& sd = job.s[si];
  const long long item = static_cast<long long>(blockIdx.x - job.first[si]) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (item >= job.rows * sd.heads) return;
  const long long row = item / sd.heads;
  const int h = static_cast<int>(item - row * sd.heads);
  const T* x = static_cast<const T*>(sd.x) + row * sd.xrow + h * sd.xhead;
  T* y = out_of<T, APPEND>(tab, job, sd, row, h);
  if (y == nullptr) return;
  const T* w = static_cast<const T*>(sd.w);
  const int np = (tab.dh + 1) >> 1;
  float a[4], b[4], ss = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = lane + 32 * i;
    a[i] = b[i] = 0.f;
    if (j < np) {
      const Pair p = pair_of(tab, j);
      a[i] = to_f32(x[p.a]);
      if (p.b >= 0) b[i] = to_f32(x[p.b]);
    }
    ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
  }
  float r = 1.f;
  if (w) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    r = rsqrtf(ss / static_cast<float>(tab.dh) + tab.eps);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = lane + 32 * i;
    if (j >= np) continue;
    const Pair p = pair_of(tab, j);
    float za = a[i], zb = b[i];
    if (w) {
      za *= r * to_f32(w[p.a]);
      if (p.b >= 0) zb *= r * to_f32(w[p.b]);
    }
    if (p.turned && sd.kind != kValues) {
      const float2 cs = turn_of(tab, j, job.pos, job.rows, row);
      const float u = za * cs.x - zb * cs.y;
      zb = zb * cs.x + za * cs.y;
      za = u;
    }
    y[p.a] = from_f32<T>(za);
    if (p.b >= 0) y[p.b] = from_f32<T>(zb);
  }
}

// dx, and this block's sum of g n per column into part[block of the side][dh].
template <typename T>
__global__ void __launch_bounds__(kThreads) grad_any_kernel(const __grid_constant__ RopeTab tab,
                                                            const __grid_constant__ Job job) {
  __shared__ float red[kWarps][kMaxHead];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, np = (tab.dh + 1) >> 1;
  const int si = side_of_block(job);
  const Side& sd = job.s[si];
  const unsigned blk = blockIdx.x - job.first[si], blocks = job.first[si + 1] - job.first[si];
  const T* w = static_cast<const T*>(sd.w);
  float da[4] = {}, db[4] = {};
  for (long long item = static_cast<long long>(blk) * kWarps + warp; item < job.rows * sd.heads;
       item += static_cast<long long>(blocks) * kWarps) {
    const long long row = item / sd.heads;
    const int h = static_cast<int>(item - row * sd.heads);
    const T* g = static_cast<const T*>(sd.g) + row * sd.grow + h * sd.ghead;
    const T* x = w ? static_cast<const T*>(sd.x) + row * sd.xrow + h * sd.xhead : nullptr;
    T* y = static_cast<T*>(sd.y) + row * sd.yrow + h * sd.yhead;
    float ga[4], gb[4], xa[4], xb[4], ss = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = lane + 32 * i;
      ga[i] = gb[i] = xa[i] = xb[i] = 0.f;
      if (j >= np) continue;
      const Pair p = pair_of(tab, j);
      const float u = to_f32(g[p.a]), v = p.b >= 0 ? to_f32(g[p.b]) : 0.f;
      ga[i] = u;
      gb[i] = v;
      if (p.turned) {
        const float2 cs = turn_of(tab, j, job.pos, job.rows, row);
        ga[i] = u * cs.x + v * cs.y;
        gb[i] = v * cs.x - u * cs.y;
      }
      if (w) {
        xa[i] = to_f32(x[p.a]);
        if (p.b >= 0) xb[i] = to_f32(x[p.b]);
        ss = fmaf(xa[i], xa[i], fmaf(xb[i], xb[i], ss));
        dot = fmaf(ga[i] * to_f32(w[p.a]), xa[i], dot);
        if (p.b >= 0) dot = fmaf(gb[i] * to_f32(w[p.b]), xb[i], dot);
      }
    }
    float r = 1.f, m = 0.f;
    if (w) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        ss += __shfl_xor_sync(0xffffffffu, ss, o);
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
      }
      r = rsqrtf(ss / static_cast<float>(tab.dh) + tab.eps);
      m = dot * r / static_cast<float>(tab.dh);              // mean(g w n)
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = lane + 32 * i;
      if (j >= np) continue;
      const Pair p = pair_of(tab, j);
      float oa = ga[i], ob = gb[i];
      if (w) {
        const float na = xa[i] * r, nb = xb[i] * r;
        da[i] = fmaf(ga[i], na, da[i]);
        db[i] = fmaf(gb[i], nb, db[i]);
        oa = r * (ga[i] * to_f32(w[p.a]) - na * m);
        if (p.b >= 0) ob = r * (gb[i] * to_f32(w[p.b]) - nb * m);
      }
      y[p.a] = from_f32<T>(oa);
      if (p.b >= 0) y[p.b] = from_f32<T>(ob);
    }
  }
  if (!w) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = lane + 32 * i;
    if (j >= np) continue;
    const Pair p = pair_of(tab, j);
    red[warp][p.a] = da[i];
    if (p.b >= 0) red[warp][p.b] = db[i];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < tab.dh; c += kThreads) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) s += red[k][c];
    sd.part[static_cast<long long>(blk) * tab.dh + c] = s;
  }
}

// ------------------------------------------------------------------ vectors of V columns
// V columns as one access (16 bytes; 8 for V = 4 of a 16-bit type).
template <typename T, int V> struct Vec;
template <> struct Vec<float, 4> {
  float4 r;
  __device__ __forceinline__ void load(const float* p) { r = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ uint32_t pack2(float x, float y, __nv_bfloat16) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float x, float y, __half) {
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T> struct Vec<T, 8> {
  uint4 r;
  __device__ __forceinline__ void load(const T* p) { r = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack2(w[i], T());
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ void store(T* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()), pack2(v[4], v[5], T()), pack2(v[6], v[7], T()));
  }
};
template <typename T> struct Vec<T, 4> {
  uint2 r;
  __device__ __forceinline__ void load(const T* p) { r = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(float (&v)[4]) const {
    const float2 a = unpack2(r.x, T()), b = unpack2(r.y, T());
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
  }
  static __device__ __forceinline__ void store(T* p, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()));
  }
};

// A lane holds two vectors of a head, those of its pairs: V columns from a and V from b, pairs (a + i, b + i), or for
// adjacent pairs 2 V columns in a row.  `lanes` (a power of two, the last ones without columns) share a head.
struct Lane { int a, b, turned; bool on, two; };       // turned: how many of the lane's V pairs turn
template <int V, bool ADJ>
__device__ __forceinline__ Lane lane_of(const RopeTab& t, int shift) {
  Lane l;
  const int j = threadIdx.x & ((1 << shift) - 1), nr = ADJ ? 0 : t.rot / (2 * V);
  l.turned = ADJ ? min(V, max(0, (t.rot >> 1) - j * V)) : j < nr ? V : 0;
  l.a = j < nr ? j * V : 2 * j * V;
  l.b = j < nr ? (t.rot >> 1) + j * V : l.a + V;
  l.on = l.a < t.dh;
  l.two = l.b < t.dh;
  return l;
}

// (cos, sin) of the pairs of `n` rows from row0 on, where the lanes of a
// warp read them without bank conflicts: pair j V + i of row r is entry ((r V / 2 + i / 2) np + j) 2 + i % 2.  They are
// computed once a block, not once a head: a head takes 16 instructions a pair without them.
template <int V>
__device__ __forceinline__ void fill_turns(float2* cs, const RopeTab& t, const Job& job, long long row0, int n, int np) {
  const int half = t.rot >> 1;
  for (int e = threadIdx.x; e < n * half; e += kThreads) {
    const int r = e / half, p = e - r * half, j = p / V, i = p % V;
    if (row0 + r < job.rows) cs[((r * (V / 2) + i / 2) * np + j) * 2 + i % 2] = turn_of(t, p, job.pos, job.rows, row0 + r);
  }
}

// The lane's pairs turned by row r's entries (SIGN = 1) or back (-1); columns past rot are left as they are.
template <int V, bool ADJ, int SIGN>
__device__ __forceinline__ void turn_pairs(float (&a)[V], float (&b)[V], const float2* cs, int r, int np, int j, int turned) {
  if (turned == 0) return;
  const float4* c4 = reinterpret_cast<const float4*>(cs) + r * (V / 2) * np + j;
#pragma unroll
  for (int i = 0; i < V; i += 2) {
    const float4 c = c4[(i / 2) * np];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int q = i + k;
      if (ADJ && q >= turned) continue;
      const float co = k ? c.z : c.x, si = SIGN * (k ? c.w : c.y);
      float& x = ADJ ? (q < V / 2 ? a[2 * q] : b[2 * q - V]) : a[q];
      float& y = ADJ ? (q < V / 2 ? a[2 * q + 1] : b[2 * q + 1 - V]) : b[q];
      const float u = x * co - y * si;
      y = y * co + x * si;
      x = u;
    }
  }
}

// U heads a lane, all loaded before the turns are computed.
template <typename T, int V, bool ADJ, int U, bool APPEND>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const __grid_constant__ RopeTab tab,
                                                          const __grid_constant__ Job job, int shift, int turn_rows) {
  extern __shared__ float2 cs[];
  pdl_enter();
  const int si = side_of_block(job);
  const Side& sd = job.s[si];
  const Lane ln = lane_of<V, ADJ>(tab, shift);
  const unsigned per = kThreads >> shift, heads = sd.heads, base = (blockIdx.x - job.first[si]) * (per * U);
  const unsigned total = static_cast<unsigned>(job.rows) * heads, row0 = base / heads;
  const int j = threadIdx.x & ((1 << shift) - 1), np = (tab.dh / V + 1) >> 1;
  Vec<T, V> va[U], vb[U];
  unsigned row[U], h[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const unsigned hv = base + u * per + (threadIdx.x >> shift);
    row[u] = hv / heads;
    h[u] = hv - row[u] * heads;
    va[u].r = {};
    vb[u].r = {};
    if (hv < total && ln.on) {
      const T* x = static_cast<const T*>(sd.x) + row[u] * sd.xrow + h[u] * sd.xhead;
      va[u].load(x + ln.a);
      if (ln.two) vb[u].load(x + ln.b);
    }
  }
  const bool turns = sd.kind != kValues;
  if (turns) {
    fill_turns<V>(cs, tab, job, row0, turn_rows, np);
    __syncthreads();
  }
  const T* w = static_cast<const T*>(sd.w);
  float wa[V], wb[V];
  if (w && ln.on) {
    Vec<T, V> t;
    t.load(w + ln.a);
    t.get(wa);
    if (ln.two) t.load(w + ln.b);
    t.get(wb);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float a[V], b[V];
    va[u].get(a);
    vb[u].get(b);
    if (w) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
      for (int o = 1 << shift >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float r = rsqrtf(ss / static_cast<float>(tab.dh) + tab.eps);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        a[i] *= r * wa[i];
        b[i] *= r * wb[i];
      }
    }
    if (base + u * per + (threadIdx.x >> shift) >= total || !ln.on) continue;
    T* y = out_of<T, APPEND>(tab, job, sd, row[u], h[u]);
    if (y == nullptr) continue;
    if (turns) turn_pairs<V, ADJ, 1>(a, b, cs, row[u] - row0, np, j, ln.turned);
    Vec<T, V>::store(y + ln.a, a);
    if (ln.two) Vec<T, V>::store(y + ln.b, b);
  }
}

// A block takes every blocks-th group of heads of its side; its lanes keep their columns, so the sums of g n stay in
// registers until the end.
template <typename T, int V, bool ADJ>
__global__ void __launch_bounds__(kThreads) grad_kernel(const __grid_constant__ RopeTab tab,
                                                        const __grid_constant__ Job job, int shift, int turn_rows) {
  extern __shared__ float2 cs[];               // two groups' turns
  __shared__ float red[kWarps][kMaxHead];
  pdl_enter();
  const int si = side_of_block(job);
  const Side& sd = job.s[si];
  const Lane ln = lane_of<V, ADJ>(tab, shift);
  const unsigned blk = blockIdx.x - job.first[si], blocks = job.first[si + 1] - job.first[si];
  const unsigned per = kThreads >> shift, heads = sd.heads, total = static_cast<unsigned>(job.rows) * heads;
  const int j = threadIdx.x & ((1 << shift) - 1), np = (tab.dh / V + 1) >> 1;
  const T* w = static_cast<const T*>(sd.w);
  float wa[V], wb[V], da[V] = {}, db[V] = {};
  if (w && ln.on) {
    Vec<T, V> t;
    t.load(w + ln.a);
    t.get(wa);
    if (ln.two) t.load(w + ln.b);
    t.get(wb);
  }
  int side = 0;
  for (unsigned long long base64 = static_cast<unsigned long long>(blk) * per; base64 < total;
       base64 += static_cast<unsigned long long>(blocks) * per, side ^= 1) {
    const unsigned base = static_cast<unsigned>(base64), row0 = base / heads, hv = base + (threadIdx.x >> shift);
    const unsigned row = hv / heads, h = hv - row * heads;
    const bool on = hv < total && ln.on;
    Vec<T, V> ga, gb, xa, xb;
    ga.r = {}; gb.r = {}; xa.r = {}; xb.r = {};
    if (on) {
      const T* g = static_cast<const T*>(sd.g) + row * sd.grow + h * sd.ghead;
      ga.load(g + ln.a);
      if (ln.two) gb.load(g + ln.b);
      if (w) {
        const T* x = static_cast<const T*>(sd.x) + row * sd.xrow + h * sd.xhead;
        xa.load(x + ln.a);
        if (ln.two) xb.load(x + ln.b);
      }
    }
    float2* c = cs + side * turn_rows * np * V;
    fill_turns<V>(c, tab, job, row0, turn_rows, np);
    __syncthreads();                           // the other half is read by no one past this barrier
    float a[V], b[V];
    ga.get(a);
    gb.get(b);
    if (on) turn_pairs<V, ADJ, -1>(a, b, c, row - row0, np, j, ln.turned);
    if (w) {
      float na[V], nb[V], ss = 0.f, dot = 0.f;
      xa.get(na);
      xb.get(nb);
#pragma unroll
      for (int i = 0; i < V; ++i) ss = fmaf(na[i], na[i], fmaf(nb[i], nb[i], ss));
      if (on) {
#pragma unroll
        for (int i = 0; i < V; ++i) dot = fmaf(a[i] * wa[i], na[i], fmaf(b[i] * (ln.two ? wb[i] : 0.f), nb[i], dot));
      }
      for (int o = 1 << shift >> 1; o > 0; o >>= 1) {
        ss += __shfl_xor_sync(0xffffffffu, ss, o);
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
      }
      if (on) {
        const float r = rsqrtf(ss / static_cast<float>(tab.dh) + tab.eps), m = dot * r / static_cast<float>(tab.dh);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          na[i] *= r;
          nb[i] *= r;
          da[i] = fmaf(a[i], na[i], da[i]);
          db[i] = fmaf(b[i], nb[i], db[i]);
          a[i] = r * (a[i] * wa[i] - na[i] * m);
          b[i] = r * (b[i] * wb[i] - nb[i] * m);
        }
      }
    }
    if (on) {
      T* y = static_cast<T*>(sd.y) + row * sd.yrow + h * sd.yhead;
      Vec<T, V>::store(y + ln.a, a);
      if (ln.two) Vec<T, V>::store(y + ln.b, b);
    }
  }
  if (!w) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    for (int o = 16; o >= 1 << shift; o >>= 1) {
      da[i] += __shfl_xor_sync(0xffffffffu, da[i], o);
      db[i] += __shfl_xor_sync(0xffffffffu, db[i], o);
    }
    if ((threadIdx.x & 31) >> shift == 0 && ln.on) {
      red[threadIdx.x >> 5][ln.a + i] = da[i];
      if (ln.two) red[threadIdx.x >> 5][ln.b + i] = db[i];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < tab.dh; c += kThreads) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) s += red[k][c];
    sd.part[static_cast<long long>(blk) * tab.dh + c] = s;
  }
}

// dw[c] = sum over a side's blocks of part[b][c], in a fixed order: 32 columns a CTA, every 8th block a warp.
struct Sums { const float* part[2]; float* dw[2]; int blocks[2]; };
__global__ void __launch_bounds__(kThreads) grad_sum_kernel(const __grid_constant__ Sums g, int dh) {
  __shared__ float red[kWarps][32];
  pdl_enter();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5, side = blockIdx.y;
  float s = 0.f;
  if (c < dh) {
#pragma unroll 8
    for (int b = warp; b < g.blocks[side]; b += kWarps) s += g.part[side][static_cast<long long>(b) * dh + c];
  }
  red[warp][threadIdx.x & 31] = s;
  __syncthreads();
  if (warp == 0 && c < dh && g.dw[side]) {
    s = red[0][threadIdx.x];
#pragma unroll
    for (int k = 1; k < kWarps; ++k) s += red[k][threadIdx.x];
    g.dw[side][c] = s;
  }
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

int launch_err(cudaError_t e) {
  if (e == cudaSuccess) return MAP_OK;
  cudaGetLastError();
  return MAP_ECUDA;
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
  const int np = (t.dh / v + 1) / 2;
  int s = 0;
  while ((1 << s) < np) ++s;
  return s;
}

// Rows whose turns a group of `vectors` heads of a side needs.
int rows_spanned(int vectors, int heads, long long rows) {
  const long long n = (vectors - 1) / heads + 2;
  return static_cast<int>(n < rows ? n : rows);
}

template <typename T, int V, bool ADJ, int U, bool APPEND>
cudaError_t run_rotate(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int shift = shift_of(t, V), per = (kThreads >> shift) * U;
  unsigned blocks = 0;
  int rows = 0;
  for (int i = 0; i < 3; ++i) {
    job.first[i] = blocks;
    if (i >= sides) continue;
    blocks += static_cast<unsigned>((job.rows * job.s[i].heads + per - 1) / per);
    if (job.s[i].kind != kValues) rows = std::max(rows, rows_spanned(per, job.s[i].heads, job.rows));
  }
  job.first[3] = blocks;
  for (int i = sides; i < 3; ++i) job.first[i] = blocks;
  const size_t smem = static_cast<size_t>(rows) * ((t.dh / V + 1) / 2) * V * sizeof(float2);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(rotate_kernel<T, V, ADJ, U, APPEND>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
  return launch_k(rotate_kernel<T, V, ADJ, U, APPEND>, dim3(blocks), dim3(kThreads), smem, st, t, job, shift, rows);
}

template <typename T, bool APPEND>
cudaError_t run_rotate_any(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  unsigned blocks = 0;
  for (int i = 0; i < 4; ++i) {
    job.first[i] = blocks;
    if (i < sides) blocks += static_cast<unsigned>((job.rows * job.s[i].heads + kWarps - 1) / kWarps);
  }
  return launch_k(rotate_any_kernel<T, APPEND>, dim3(blocks), dim3(kThreads), 0, st, t, job);
}

template <typename T, int V, bool APPEND>
cudaError_t rotate_width(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  return t.adjacent ? run_rotate<T, V, true, 2, APPEND>(t, job, sides, st) : run_rotate<T, V, false, 2, APPEND>(t, job, sides, st);
}

template <typename T, bool APPEND>
cudaError_t rotate_job(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int v = vector_of(t, job, sides, sizeof(T));
  if (v == 4) return rotate_width<T, 4, APPEND>(t, job, sides, st);
  if constexpr (sizeof(T) == 2)
    if (v == 8) return rotate_width<T, 8, APPEND>(t, job, sides, st);
  return run_rotate_any<T, APPEND>(t, job, sides, st);
}

// Blocks of a gradient's sides: in proportion to their heads, at most kGradBlocks a side and one a group.
void grad_blocks(Job& job, int sides, int per) {
  long long heads = 0;
  for (int i = 0; i < sides; ++i) heads += job.s[i].heads;
  unsigned at = 0;
  for (int i = 0; i < 4; ++i) {
    job.first[i] = at;
    if (i >= sides) continue;
    const long long groups = (job.rows * job.s[i].heads + per - 1) / per;
    const long long share = (kGradBlocks * job.s[i].heads + heads - 1) / heads;
    at += static_cast<unsigned>(std::min(groups, share));
  }
}

template <typename T, int V, bool ADJ>
cudaError_t run_grad(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int shift = shift_of(t, V), per = kThreads >> shift;
  grad_blocks(job, sides, per);
  int rows = 0;
  for (int i = 0; i < sides; ++i) rows = std::max(rows, rows_spanned(per, job.s[i].heads, job.rows));
  const size_t smem = 2 * static_cast<size_t>(rows) * ((t.dh / V + 1) / 2) * V * sizeof(float2);
  if (smem > 40 * 1024) {                       // beside 8 KB of static shared memory
    const cudaError_t e = cudaFuncSetAttribute(grad_kernel<T, V, ADJ>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
  return launch_k(grad_kernel<T, V, ADJ>, dim3(job.first[3]), dim3(kThreads), smem, st, t, job, shift, rows);
}

template <typename T>
cudaError_t grad_job(const RopeTab& t, Job& job, int sides, cudaStream_t st) {
  const int v = vector_of(t, job, sides, sizeof(T));
  if (v == 4) return t.adjacent ? run_grad<T, 4, true>(t, job, sides, st) : run_grad<T, 4, false>(t, job, sides, st);
  if constexpr (sizeof(T) == 2)
    if (v == 8) return t.adjacent ? run_grad<T, 8, true>(t, job, sides, st) : run_grad<T, 8, false>(t, job, sides, st);
  grad_blocks(job, sides, kWarps);
  return launch_k(grad_any_kernel<T>, dim3(job.first[3]), dim3(kThreads), 0, st, t, job);
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
  for (int i = 0; i < rot / 2; ++i) {
    const double turns = inv_freq[i] * 0.15915494309189533577;     // 1 / 2 pi
    t.turn[i] = static_cast<unsigned long long>(std::ldexp(turns - std::floor(turns), 64));
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
    if (absent(g[i])) continue;
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
  if (e == cudaSuccess && norm) e = launch_k(grad_sum_kernel, dim3((t.dh + 31) / 32, 2), dim3(kThreads), 0, st, sums, t.dh);
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
