// Shared by the language-model hand-off (rope.cu, cache.cu, evict.cu, attend*.cu): element types, checks.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/map_gb300.h"
#include "ptx.cuh"

namespace mapk {

constexpr int kMaxHead = 256;        // widest head (dh)

// Rotation plan, a kernel parameter: the fraction of a turn per position (2^-64 units) and the axis of each pair.
struct RopeTab {
  unsigned long long turn[kMaxHead / 2];
  uint8_t axis[kMaxHead / 2];
  int dh, rot, adjacent, axes;
  float eps, inv_dh;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Whether rows * heads vectors of dh elements, `row` and `head` elements apart, are disjoint: the inner of the two
// strides covers a vector, the outer one the inner's whole extent.
inline bool distinct_vectors(long long row, long long rows, long long head, long long heads, long long dh) {
  if (rows <= 1 && heads <= 1) return true;
  if (rows <= 1) return head >= dh;
  if (heads <= 1) return row >= dh;
  return (head >= dh && row >= (heads - 1) * head + dh) || (row >= dh && head >= (rows - 1) * row + dh);
}

// Whether a table entry is a page of the pool, and a length one that a table row can hold: what a call finds in the
// caller's arrays is checked before it becomes an address.
__device__ __forceinline__ bool good_page(const map_cache& c, int page) {
  return static_cast<unsigned>(page) < static_cast<unsigned>(c.pages);
}
__device__ __forceinline__ bool good_len(const map_cache& c, int len) { return len >= 0 && len <= c.max_pages * c.page; }
// Pieces of `size` rows that hold `len` (a good length; it and a piece can add up past 2^31).
__host__ __device__ __forceinline__ int pieces_of(int len, int size) { return static_cast<int>((static_cast<unsigned>(len) + size - 1) / size); }

// MAP_OK, MAP_EINVAL or MAP_EUNSUPPORTED for a cache's description (host values only).
int check_cache(const map_cache* c);

// launch_k of clusters of `ranks` CTAs.
template <typename... P, typename... Args>
cudaError_t launch_cluster(void (*kern)(P...), unsigned grid, unsigned threads, int ranks, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = pdl_disabled() ? 0 : 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = ranks;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

// A launch's status as a call's, the runtime's sticky copy of it cleared.
inline int launch_err(cudaError_t e) {
  if (e == cudaSuccess) return MAP_OK;
  cudaGetLastError();
  return MAP_ECUDA;
}

}  // namespace mapk
