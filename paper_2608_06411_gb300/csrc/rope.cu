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

constexpr int kThreads = 256;
constexpr int kGradBlocks = 608;     // partial sums of dw: at most this many blocks a side (4 for each of 152 SMs)

struct Side {                        // one tensor's heads: input, output, norm weight
  const void* x; long long xrow, xhead;
  void* y; long long yrow, yhead;
  const void* w;
  const void* g; long long grow, ghead;   // backward: gradient of the output
  int heads;
};

__device__ __forceinline__ float2 turn_of(const RopeTab& t, int pair, const int32_t* __restrict__ pos, long long rows,
                                          long long row) {
  const unsigned long long ph =
      t.turn[pair] * static_cast<unsigned long long>(static_cast<long long>(__ldg(pos + t.axis[pair] * rows + row)));
  float s, c;
  sincospif(static_cast<float>(static_cast<int>(ph >> 32)) * 0x1p-31f, &s, &c);
  return make_float2(c, s);
}

// Column pairs of lane l (every 32nd one): (a, b) columns, b = -1 where a has no partner.
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

// One warp a head: 4 column pairs a lane.
template <typename T>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const __grid_constant__ RopeTab tab, const Side sd,
                                                          const int32_t* __restrict__ pos, long long rows) {
  pdl_enter();
  const long long item = static_cast<long long>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (item >= rows * sd.heads) return;
  const long long row = item / sd.heads;
  const int h = static_cast<int>(item - row * sd.heads);
  const T* x = static_cast<const T*>(sd.x) + row * sd.xrow + h * sd.xhead;
  T* y = static_cast<T*>(sd.y) + row * sd.yrow + h * sd.yhead;
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
    float2 cs = make_float2(1.f, 0.f);
    if (p.turned) cs = turn_of(tab, j, pos, rows, row);
    y[p.a] = from_f32<T>(za * cs.x - zb * cs.y);
    if (p.b >= 0) y[p.b] = from_f32<T>(zb * cs.x + za * cs.y);
  }
}

// dx, and this block's sum of g n per column into part[blockIdx.x][dh].
template <typename T>
__global__ void __launch_bounds__(kThreads) rotate_grad_kernel(const __grid_constant__ RopeTab tab, const Side sd,
                                                               const int32_t* __restrict__ pos, long long rows,
                                                               float* __restrict__ part) {
  __shared__ float red[kThreads / 32][256];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, np = (tab.dh + 1) >> 1;
  const T* w = static_cast<const T*>(sd.w);
  float da[4] = {}, db[4] = {};
  for (long long item = static_cast<long long>(blockIdx.x) * (kThreads / 32) + warp; item < rows * sd.heads;
       item += static_cast<long long>(gridDim.x) * (kThreads / 32)) {
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
      float2 cs = make_float2(1.f, 0.f);
      if (p.turned) cs = turn_of(tab, j, pos, rows, row);
      const float u = to_f32(g[p.a]), v = p.b >= 0 ? to_f32(g[p.b]) : 0.f;
      ga[i] = u * cs.x + v * cs.y;
      gb[i] = v * cs.x - u * cs.y;
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
    for (int k = 0; k < kThreads / 32; ++k) s += red[k][c];
    part[static_cast<long long>(blockIdx.x) * tab.dh + c] = s;
  }
}

// dw[c] = sum over nb blocks of part[b][c], in block order.
__global__ void grad_sum_kernel(const float* __restrict__ part, int nb, int dh, float* __restrict__ dw) {
  pdl_enter();
  const int c = threadIdx.x;
  if (c >= dh) return;
  float s = 0.f;
  for (int b = 0; b < nb; ++b) s += part[static_cast<long long>(b) * dh + c];
  dw[c] = s;
}

// Rotated keys and copied values into their slots, rotated queries to q_out: one warp a head of q, k or v.
template <typename T>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ RopeTab tab, const Side q,
                                                          const Side k, const Side v, const int32_t* __restrict__ pos,
                                                          const int32_t* __restrict__ slots, long long rows,
                                                          T* __restrict__ plane_k, T* __restrict__ plane_v, int page,
                                                          int pages, int* status) {
  pdl_enter();
  const int heads = q.heads + 2 * k.heads;
  const long long item = static_cast<long long>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (item >= rows * heads) return;
  const long long row = item / heads;
  int h = static_cast<int>(item - row * heads);
  const int slot = __ldg(slots + row);
  if (slot < 0 || slot >= pages * page) {
    if (slot != -1 && lane == 0) atomicOr(status, ST_BADINDEX);
    return;
  }
  const bool isq = h < q.heads, isv = h >= q.heads + k.heads;
  const Side& sd = isq ? q : isv ? v : k;
  h -= isq ? 0 : isv ? q.heads + k.heads : q.heads;
  const T* x = static_cast<const T*>(sd.x) + row * sd.xrow + h * sd.xhead;
  T* y = isq ? static_cast<T*>(sd.y) + row * sd.yrow + h * sd.yhead
             : (isv ? plane_v : plane_k) +
                   ((static_cast<long long>(slot / page) * k.heads + h) * page + slot % page) * tab.dh;
  if (isv) {
    for (int c = lane; c < tab.dh; c += 32) y[c] = x[c];
    return;
  }
  const T* w = static_cast<const T*>(sd.w);
  const int np = (tab.dh + 1) >> 1;
  float ss = 0.f, r = 1.f;
  if (w) {
    for (int c = lane; c < tab.dh; c += 32) ss = fmaf(to_f32(x[c]), to_f32(x[c]), ss);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    r = rsqrtf(ss / static_cast<float>(tab.dh) + tab.eps);
  }
  for (int j = lane; j < np; j += 32) {
    const Pair p = pair_of(tab, j);
    float za = to_f32(x[p.a]), zb = p.b >= 0 ? to_f32(x[p.b]) : 0.f;
    if (w) {
      za *= r * to_f32(w[p.a]);
      if (p.b >= 0) zb *= r * to_f32(w[p.b]);
    }
    float2 cs = make_float2(1.f, 0.f);
    if (p.turned) cs = turn_of(tab, j, pos, rows, row);
    y[p.a] = from_f32<T>(za * cs.x - zb * cs.y);
    if (p.b >= 0) y[p.b] = from_f32<T>(zb * cs.x + za * cs.y);
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

template <typename T>
cudaError_t rotate_side(const RopeTab& t, const Side& s, const int32_t* pos, long long rows, cudaStream_t st) {
  const long long blocks = (rows * s.heads + kThreads / 32 - 1) / (kThreads / 32);
  return launch_k(rotate_kernel<T>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, t, s, pos, rows);
}

template <typename T>
cudaError_t grad_side(const RopeTab& t, const Side& s, const int32_t* pos, long long rows, float* part, float* dw,
                      cudaStream_t st) {
  const long long want = (rows * s.heads + kThreads / 32 - 1) / (kThreads / 32);
  const int blocks = static_cast<int>(want < kGradBlocks ? want : kGradBlocks);
  cudaError_t e = cudaSuccess;
  if (blocks > 0) e = launch_k(rotate_grad_kernel<T>, dim3(blocks), dim3(kThreads), 0, st, t, s, pos, rows, part);
  if (e == cudaSuccess && s.w)
    e = launch_k(grad_sum_kernel, dim3(1), dim3(256), 0, st, static_cast<const float*>(part), blocks, t.dh, dw);
  return e;
}

Side side_of(const map_heads* in, const map_heads* out, const void* w) {
  return Side{in ? in->p : nullptr, in ? in->row : 0, in ? in->head : 0, out ? out->p : nullptr, out ? out->row : 0,
              out ? out->head : 0, w, nullptr, 0, 0, in ? in->heads : 0};
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
  for (int i = 0; i < 2; ++i)
    if (!absent(in[i]) && (!good_in(in[i], type, rows) || !good_out(out[i], type, rows, t.dh, in[i]->heads)))
      return MAP_EINVAL;
  if (rows == 0) return MAP_OK;
  for (int i = 0; i < 2; ++i) {
    if (absent(in[i])) continue;
    const Side s = side_of(in[i], out[i], w[i]);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = type == MAP_F32   ? rotate_side<float>(t, s, pos, rows, st)
                          : type == MAP_F16 ? rotate_side<__half>(t, s, pos, rows, st)
                                            : rotate_side<__nv_bfloat16>(t, s, pos, rows, st);
    if (e != cudaSuccess) return launch_err(e);
  }
  return MAP_OK;
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
  for (int i = 0; i < 2; ++i) {
    if (absent(g[i])) continue;
    if (!good_in(g[i], type, rows) || !good_out(out[i], type, rows, t.dh, g[i]->heads)) return MAP_EINVAL;
    if (w[i] && (absent(x[i]) || !good_in(x[i], type, rows) || x[i]->heads != g[i]->heads || !dw[i] || !ws ||
                 !aligned16(ws)))
      return MAP_EINVAL;
  }
  for (int i = 0; i < 2; ++i) {
    if (absent(g[i])) continue;
    Side s = side_of(w[i] ? x[i] : g[i], out[i], w[i]);
    s.g = g[i]->p;
    s.grow = g[i]->row;
    s.ghead = g[i]->head;
    float* part = static_cast<float*>(ws) + (ws ? static_cast<size_t>(i) * kGradBlocks * t.dh : 0);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = type == MAP_F32   ? grad_side<float>(t, s, pos, rows, part, dw[i], st)
                          : type == MAP_F16 ? grad_side<__half>(t, s, pos, rows, part, dw[i], st)
                                            : grad_side<__nv_bfloat16>(t, s, pos, rows, part, dw[i], st);
    if (e != cudaSuccess) return launch_err(e);
  }
  return MAP_OK;
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
  Side sq = hq ? side_of(q, q_out, wq) : Side{};
  const Side sk = side_of(k, nullptr, wk), sv = side_of(v, nullptr, nullptr);
  const long long blocks = (rows * (hq + 2 * c->heads) + kThreads / 32 - 1) / (kThreads / 32);
  const size_t plane = static_cast<size_t>(c->pages) * c->heads * c->page * c->dh;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (c->type == MAP_F16) {
    __half* p = static_cast<__half*>(c->pool) + 2 * layer * plane;
    e = launch_k(append_kernel<__half>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, t, sq, sk, sv, pos,
                 slots, rows, p, p + plane, c->page, c->pages, c->status);
  } else {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(c->pool) + 2 * layer * plane;
    e = launch_k(append_kernel<__nv_bfloat16>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, t, sq, sk,
                 sv, pos, slots, rows, p, p + plane, c->page, c->pages, c->status);
  }
  return launch_err(e);
}

}  // extern "C"
