// Attention of single tokens over a cache's pages with the sums of its weights (map_cache_attend_weigh).
//
// Mathematics.  weights[t] += sum_h 2^(z_ht - m_h) / l_h over the query heads h of a key head, with attend's scores z, largest
// score m and sum l: known only once a head's last row has been seen.
// Bound: HBM, the rows of K and V once and a row's sum read and written (8 bytes a key head against 512 at 128 columns).  The
// scores are kept in fp32 (4 bytes a head, 16 to 32 a row against the 256 of reading its key again for a second product; mostly
// they do not leave L2), and a second kernel turns them into weights: equal runs of a list of 512-row pieces a CTA, four
// neighbouring rows a thread, eight heads' scores in flight.
// A sequence's sums are added up by one thread a row, over its rows of the call in their order: no atomics, one result.
// Measured, bf16 or fp16: one sequence of 701 rows, 28 heads over 4 of 128: 16 us, latency; 64 of 200 to 1600 rows, 32 over 8:
// 57 us, 4.0 TB/s (attend alone 50); one of 120001 rows, 28 over 4: 68 us, 3.7 TB/s (attend alone 51: its scores' stores cost 4,
// the second kernel 9 to 13); 7 of up to 5001 rows, 40 heads over 10 of 96, pages of 24 rows: 27 us.
#include "attend.cuh"

namespace mapk {
namespace {

constexpr int kRowsEach = 4, kPiece = kRowsEach * kThreads, kHeadsEach = 8;      // neighbouring rows of a thread; heads at once

__global__ void __launch_bounds__(kThreads) weigh_kernel(const __grid_constant__ AttendArgs a, float* __restrict__ weights,
                                                         int max_rows) {
  __shared__ long long red[kWarps];
  __shared__ int first_entry;
  __shared__ long long first_piece;
  pdl_enter();
  const int tid = threadIdx.x;
  const auto pieces = [&](int e) { return pieces_of(seq_len(a, e), kPiece); };
  // this CTA's run of the list (entry, key head, piece): a thread counts a run of the entries
  const int each = (a.n + kThreads - 1) / kThreads, e0 = tid * each, e1 = min(a.n, e0 + each);
  long long mine = 0, total;
  for (int e = e0; e < e1; ++e) mine += static_cast<long long>(pieces(e)) * a.c.heads;
  long long at0 = block_prefix(mine, red, &total);
  const long long per = (total + gridDim.x - 1) / gridDim.x, t0 = per * blockIdx.x, t1 = min(total, t0 + per);
  if (t0 >= t1) return;
  if (at0 <= t0 && t0 < at0 + mine) {
    for (int e = e0;; ++e) {
      const long long k = static_cast<long long>(pieces(e)) * a.c.heads;
      if (t0 < at0 + k) {
        first_entry = e;
        first_piece = t0 - at0;
        break;
      }
      at0 += k;
    }
  }
  __syncthreads();
  long long at = first_piece;                  // within the entry
  int e = first_entry;
  for (long long t = t0; t < t1; ++e, at = 0) {
    const int len = seq_len(a, e), count = pieces_of(len, kPiece);
    const long long last = min(static_cast<long long>(count) * a.c.heads, at + t1 - t);
    if (count == 0) continue;
    // the first of a sequence's rows adds up for all of them
    const int s = __ldg(a.seqs + e);
    int twice = 0;                             // 1: it is named before, 2: behind
    for (int j = tid; j < a.n && a.n > 1; j += kThreads)
      if (__ldg(a.seqs + j) == s && j != e) twice |= j < e ? 1 : 2;
    if (a.n > 1) {
      const int before = __syncthreads_or(twice & 1);
      twice = __syncthreads_or(twice & 2);
      if (before) twice = -1;
    }
    t += last - at;
    if (twice < 0) continue;
    for (; at < last; ++at) {
      const int kh = static_cast<int>(at / count), row0 = static_cast<int>(at % count) * kPiece + tid * kRowsEach;
      float* w = weights + (static_cast<long long>(s) * a.c.heads + kh) * max_rows + row0;
      float sum[kRowsEach], was[kRowsEach];
#pragma unroll
      for (int k = 0; k < kRowsEach; ++k) {
        sum[k] = 0.f;
        was[k] = row0 + k < len ? w[k] : 0.f;
      }
      for (int j = e; j < a.n; ++j) {
        if (j != e && __ldg(a.seqs + j) != s) continue;
        const long long head0 = static_cast<long long>(j) * a.q.heads + kh * a.group;
        for (int g0 = 0; g0 < a.group; g0 += kHeadsEach) {   // (loads of several heads in flight)
          float2 st[kHeadsEach];
          float4 z[kHeadsEach];
#pragma unroll
          for (int g = 0; g < kHeadsEach; ++g) {
            const bool on = g0 + g < a.group && row0 < len;  // (scores come 16 at a time, those past the last row -inf)
            st[g] = on ? __ldcg(a.stats + head0 + g0 + g) : make_float2(0.f, 0.f);
            z[g] = on ? __ldcg(reinterpret_cast<const float4*>(a.z + (head0 + g0 + g) * a.z_row + row0))
                      : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
          }
#pragma unroll
          for (int g = 0; g < kHeadsEach; ++g) {
            if (g0 + g >= a.group) break;
            const float y[kRowsEach] = {z[g].x, z[g].y, z[g].z, z[g].w};
#pragma unroll
            for (int k = 0; k < kRowsEach; ++k) sum[k] = fmaf(exp2_fast(y[k] - st[g].x), st[g].y, sum[k]);
          }
        }
        if (!twice) break;
      }
#pragma unroll
      for (int k = 0; k < kRowsEach; ++k)
        if (row0 + k < len) w[k] = was[k] + sum[k];
    }
  }
}

// Parts of the workspace: attend's, then (m, 1 / l) of each head, then the scores, whole tiles a head.
struct WeighSpace {
  size_t stats, z, bytes;
  long long z_row;
};
bool weigh_space(const map_cache* c, long long heads, long long n, WeighSpace* w) {
  const long long rows = static_cast<long long>(c->max_pages) * c->page;
  w->z_row = (rows + kTile - 1) / kTile * kTile;
  w->stats = (map_cache_attend_workspace(c) + 255) / 256 * 256;
  w->z = w->stats + (static_cast<size_t>(heads * n) * sizeof(float2) + 255) / 256 * 256;
  if (heads * n > (1ll << 46) / (w->z_row * 4)) return false;
  w->bytes = w->z + static_cast<size_t>(heads * n) * w->z_row * 4;
  return true;
}

}  // namespace
}  // namespace mapk

using namespace mapk;

extern "C" {

size_t map_cache_attend_weigh_workspace(const map_cache* c, int heads, int n) {
  WeighSpace w;
  if (check_cache(c) != MAP_OK || heads < 1 || heads > 65535 || n < 0 || n > 65535) return 0;
  return weigh_space(c, heads, n, &w) ? w.bytes : 0;
}

int map_cache_attend_weigh(const map_cache* c, int layer, const map_heads* q, const int32_t* seqs, int n, float scale,
                           const map_heads* out, float* weights, void* ws, void* stream) {
  AttendArgs a;
  const int rc = attend_args(c, layer, q, seqs, n, scale, out, ws, a);
  if (rc != MAP_OK || a.n == 0) return rc;
  if (!weights || reinterpret_cast<uintptr_t>(weights) & 3) return MAP_EINVAL;
  WeighSpace w;
  if (!weigh_space(c, q->heads, n, &w)) return MAP_EUNSUPPORTED;
  a.stats = reinterpret_cast<float2*>(static_cast<char*>(ws) + w.stats);
  a.z = reinterpret_cast<float*>(static_cast<char*>(ws) + w.z);
  a.z_row = w.z_row;
  const int max_rows = c->max_pages * c->page;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = launch_attend<kWeigh>(a, st);
  const long long most = static_cast<long long>(n) * c->heads * pieces_of(max_rows, kPiece);
  if (e == cudaSuccess)
    e = launch_k(weigh_kernel, dim3(static_cast<unsigned>(std::min<long long>(most, 152 * 8))), dim3(kThreads), 0, st, a,
                 weights + static_cast<long long>(layer) * c->seqs * c->heads * max_rows, max_rows);
  return launch_err(e);
}

}  // extern "C"
