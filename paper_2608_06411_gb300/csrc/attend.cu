// Attention of single tokens over a cache's pages (map_cache_attend).
//
// Mathematics.  out = sum_t p_t v_t / sum_t p_t with p_t = exp(scale <q, k_t> - m), m the largest score, in one pass:
// a part of the rows gives (m, l = sum p, o = sum p v), and two parts join as m' = max, each part's l and o times
// exp(m - m').
#include <cmath>

#include "handoff.h"

namespace mapk {
namespace {

constexpr int kThreads = 128;

// One CTA a query head: scores of 128 rows, a thread each, then a thread a column of v.
template <typename T>
__global__ void __launch_bounds__(kThreads) attend_kernel(const map_cache c, const T* __restrict__ pk,
                                                          const T* __restrict__ pv, const map_heads q,
                                                          const map_heads out, const int32_t* __restrict__ seqs,
                                                          float scale) {
  __shared__ float qs[kMaxHead], p[kThreads], red[kThreads];
  pdl_enter();
  const int i = blockIdx.y, h = blockIdx.x, hk = h / (q.heads / c.heads), tid = threadIdx.x;
  const int s = seqs[i];
  if (s < 0 || s >= c.seqs) {
    if (s != -1 && tid == 0) atomicOr(c.status, ST_BADINDEX);
    return;
  }
  const T* qp = static_cast<const T*>(q.p) + i * q.row + h * q.head;
  T* o = static_cast<T*>(out.p) + i * out.row + h * out.head;
  const int32_t* table = c.table + static_cast<long long>(s) * c.max_pages;
  const int len = c.len[s];
  for (int d = tid; d < c.dh; d += kThreads) qs[d] = to_f32(qp[d]);
  float m = -INFINITY, l = 0.f, acc[kMaxHead / kThreads] = {};
  for (int t0 = 0; t0 < len; t0 += kThreads) {
    __syncthreads();
    const int t = t0 + tid, cnt = min(kThreads, len - t0);
    float z = -INFINITY;
    if (t < len) {
      const T* k = pk + ((static_cast<long long>(table[t / c.page]) * c.heads + hk) * c.page + t % c.page) * c.dh;
      z = 0.f;
      for (int d = 0; d < c.dh; ++d) z = fmaf(qs[d], to_f32(k[d]), z);
      z *= scale;
    }
    red[tid] = z;
    __syncthreads();
    float mx = m;
    for (int j = 0; j < cnt; ++j) mx = fmaxf(mx, red[j]);
    p[tid] = t < len ? expf(z - mx) : 0.f;
    __syncthreads();
    const float f = m == -INFINITY ? 0.f : expf(m - mx);
    l *= f;
    for (int j = 0; j < cnt; ++j) l += p[j];
#pragma unroll
    for (int e = 0; e < kMaxHead / kThreads; ++e) {
      const int d = tid + e * kThreads;
      if (d >= c.dh) continue;
      acc[e] *= f;
      for (int j = 0; j < cnt; ++j) {
        const int tj = t0 + j;
        acc[e] = fmaf(p[j], to_f32(pv[((static_cast<long long>(table[tj / c.page]) * c.heads + hk) * c.page + tj % c.page) * c.dh + d]), acc[e]);
      }
    }
    m = mx;
  }
#pragma unroll
  for (int e = 0; e < kMaxHead / kThreads; ++e)
    if (tid + e * kThreads < c.dh) o[tid + e * kThreads] = from_f32<T>(len > 0 ? acc[e] / l : 0.f);
}

template <typename T>
cudaError_t launch_attend(const map_cache& c, int layer, const map_heads& q, const map_heads& out, const int32_t* seqs,
                          int n, float scale, cudaStream_t st) {
  const size_t plane = static_cast<size_t>(c.pages) * c.heads * c.page * c.dh;
  const T* pk = static_cast<const T*>(c.pool) + 2 * layer * plane;
  return launch_k(attend_kernel<T>, dim3(q.heads, n), dim3(kThreads), 0, st, c, pk, pk + plane, q, out, seqs, scale);
}

}  // namespace
}  // namespace mapk

using namespace mapk;

extern "C" {

size_t map_cache_attend_workspace(const map_cache* c) { return check_cache(c) == MAP_OK ? 16 : 0; }

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
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = c->type == MAP_F16 ? launch_attend<__half>(*c, layer, *q, *out, seqs, n, scale, st)
                                           : launch_attend<__nv_bfloat16>(*c, layer, *q, *out, seqs, n, scale, st);
  if (e == cudaSuccess) return MAP_OK;
  cudaGetLastError();
  return MAP_ECUDA;
}

}  // extern "C"
