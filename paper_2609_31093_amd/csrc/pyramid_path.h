// The path update of the mean pyramid (qcache.hip, drafts.hip): only the last one or
// two leaf blocks changed.
#pragma once

#include "common.h"

namespace pisa {

// Most stored levels: 65535 leaf blocks, two children to a node.
constexpr int kMaxStored = 16;

// Leaf blocks whose ancestors path_levels updates, 0 where it does not.  Two more
// blocks add one level at most (its two nodes are then the last ones of all).
inline int path_leaves(const Geo& geo, int n_old) {
  const int n = geo.M[1] - n_old / geo.C;
  return n_old > 0 && n <= 2 ? n : 0;
}

// Thread d (of at least D) of a workgroup whose other wavefronts write the means of
// the last LEAVES blocks into `mean` and then join its barrier: sums the unchanged
// children of the blocks' ancestors meanwhile, all levels' loads in flight at once,
// and takes the means up from there (node_mean's order: children by index, changed
// ones last).  Two changed nodes of a level are its last ones; as long as they have
// parents of their own, the second is an only child.  grown: the topmost level is new,
// and its first node too where no changed block is below it.  (12 levels, 5 rows past a
// border into the 8-bit cache: 14.4 us with two copies, 27.5 in launches of their own.)
template <int D, int LEAVES>
__device__ __forceinline__ void path_levels(const Geo& geo, float* pb, const float (&mean)[LEAVES][D], int d, bool grown) {
  float sum[kMaxStored + 1], x[kMaxStored + 1];
  bool two[kMaxStored + 1];  // does the level have two changed nodes?
  two[1] = LEAVES == 2;
  int top = 0;  // first changed node of the topmost level
#pragma unroll
  for (int lv = 2; lv <= kMaxStored; ++lv) {
    sum[lv] = 0.f;
    two[lv] = LEAVES == 2 && lv <= geo.Lstore && two[lv - 1] && (geo.M[lv] - 1) * geo.g == geo.M[lv - 1] - 1;
    if (lv == geo.Lstore) top = geo.M[lv] - 1 - two[lv];
  }
  if (d < D) {
    for (int j = 0; j < geo.g - 1; ++j) {
#pragma unroll
      for (int lv = 2; lv <= kMaxStored; ++lv) {
        const int c0 = (geo.M[lv] - 1 - two[lv]) * geo.g + j;
        const bool have = lv <= geo.Lstore && c0 < geo.M[lv - 1] - 1 - two[lv - 1];
        x[lv] = pb[(geo.off[1] + (have ? geo.off[lv - 1] - geo.off[1] + c0 : 0)) * D + d];
        x[lv] = have ? x[lv] : 0.f;
      }
#pragma unroll
      for (int lv = 2; lv <= kMaxStored; ++lv) sum[lv] += x[lv];
    }
    if (grown && top > 0) {
      const float* child = pb + geo.off[geo.Lstore - 1] * D + d;
      float all = 0.f;
#pragma unroll 4
      for (int j = 0; j < geo.g; ++j) all += child[j * D];
      pb[geo.off[geo.Lstore] * D + d] = all / static_cast<float>(geo.g);
    }
  }
  __syncthreads();
  if (d < D) {
    float v = mean[0][d], w = mean[LEAVES - 1][d];
#pragma unroll
    for (int lv = 2; lv <= kMaxStored; ++lv) {
      if (lv <= geo.Lstore) {
        float* node = pb + (geo.off[lv] + geo.M[lv] - 1) * D + d;
        v = sum[lv] + v;
        if (two[lv - 1] && !two[lv]) v += w;
        v /= static_cast<float>(two[lv] ? geo.g : geo.M[lv - 1] - (geo.M[lv] - 1) * geo.g);
        if (two[lv]) {
          w += 0.f;  // the mean of one child
          *node = w;
        }
        node[two[lv] ? -D : 0] = v;
      }
    }
  }
}

}  // namespace pisa
