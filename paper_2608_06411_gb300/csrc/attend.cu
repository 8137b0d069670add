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
#include "attend.cuh"

using namespace mapk;

extern "C" {

size_t map_cache_attend_workspace(const map_cache* c) {
  return check_cache(c) == MAP_OK ? static_cast<size_t>(2) * max_grid(c->dh) * part_floats(c->dh) * sizeof(float) : 0;
}

int map_cache_attend(const map_cache* c, int layer, const map_heads* q, const int32_t* seqs, int n, float scale,
                     const map_heads* out, void* ws, void* stream) {
  AttendArgs a;
  const int rc = attend_args(c, layer, q, seqs, n, scale, out, ws, a);
  if (rc != MAP_OK || a.n == 0) return rc;
  return launch_err(launch_attend<kOut>(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
