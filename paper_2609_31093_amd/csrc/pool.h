// Means of leaf blocks and of pyramid nodes, shared by the pyramid's kernels
// (pool.hip) and the 8-bit cache's append (qcache.hip), so that both give the
// same bits.
#pragma once

#include <hip/hip_runtime.h>

#include "common.h"

namespace pisa {

// Mean of a leaf block's `nrows` rows computed by one wavefront: 16 lanes cover
// a key row, the 4 row groups take every 4th row; the lanes of every row group
// return the D/16 means of their column slice.  `row(r)` is the address of this
// lane's slice of row r.
template <typename T, int D, typename R>
__device__ __forceinline__ void leaf_mean_rows(R row, int nrows, int rg, float (&m)[D / 16]) {
  constexpr int DPL = D / 16;
  float acc[DPL];
#pragma unroll
  for (int e = 0; e < DPL; ++e) acc[e] = 0.f;
  int r = rg;
  for (; r + 12 < nrows; r += 16) {
    float x0[DPL], x1[DPL], x2[DPL], x3[DPL];
    load_row_part<T, DPL>(row(r), x0);
    load_row_part<T, DPL>(row(r + 4), x1);
    load_row_part<T, DPL>(row(r + 8), x2);
    load_row_part<T, DPL>(row(r + 12), x3);
#pragma unroll
    for (int e = 0; e < DPL; ++e) acc[e] += (x0[e] + x1[e]) + (x2[e] + x3[e]);
  }
  for (; r < nrows; r += 4) {
    float x0[DPL];
    load_row_part<T, DPL>(row(r), x0);
#pragma unroll
    for (int e = 0; e < DPL; ++e) acc[e] += x0[e];
  }
#pragma unroll
  for (int e = 0; e < DPL; ++e) {
    acc[e] += __shfl_xor(acc[e], 16);
    acc[e] += __shfl_xor(acc[e], 32);
  }
  const float inv = 1.0f / static_cast<float>(nrows);
#pragma unroll
  for (int e = 0; e < DPL; ++e) m[e] = acc[e] * inv;
}

// Leaf block `leaf` (rows [leaf*C, min((leaf+1)*C, N))) of contiguous keys.
template <typename T, int D>
__device__ __forceinline__ void leaf_mean(const T* __restrict__ kb, const Geo& geo, int leaf, int sub, int rg,
                                          float (&m)[D / 16]) {
  const int64_t row0 = static_cast<int64_t>(leaf) * geo.C;
  const int nrows = min(geo.C, geo.N - static_cast<int>(row0));
  const T* base = kb + row0 * D + sub * (D / 16);
  leaf_mean_rows<T, D>([&](int r) { return base + static_cast<int64_t>(r) * D; }, nrows, rg, m);
}

// Node `node` of level lv (>= 2): the mean of its existing children, summed
// in index order; `child(ch, col)` reads column col of child ch.
template <typename F>
__device__ __forceinline__ float node_mean(const Geo& geo, int lv, int node, int col, F child) {
  const int c0 = node * geo.g;
  const int c1 = min(c0 + geo.g, geo.M[lv - 1]);
  float s = 0.f;
  for (int ch = c0; ch < c1; ++ch) s += child(ch, col);
  return s / static_cast<float>(c1 - c0);
}

}  // namespace pisa
