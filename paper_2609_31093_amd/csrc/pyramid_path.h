// The path update of the mean pyramid (qcache.hip, drafts.hip): only the last leaf
// block changed and no level is new.
#pragma once

#include "common.h"

namespace pisa {

// Most stored levels: 65535 leaf blocks, two children to a node.
constexpr int kMaxStored = 16;

// Thread d (of at least D) of a workgroup whose other wavefronts write the changed
// block's mean into `mean` and then join its barrier: sums the unchanged children of
// the block's ancestors meanwhile, all levels' loads in flight at once, and takes the
// mean up from there (node_mean's order: children by index, the changed one last).
template <int D>
__device__ __forceinline__ void path_levels(const Geo& geo, float* pb, const float* mean, int d) {
  float sum[kMaxStored + 1], x[kMaxStored + 1];
#pragma unroll
  for (int lv = 2; lv <= kMaxStored; ++lv) sum[lv] = 0.f;
  if (d < D) {
    for (int j = 0; j < geo.g - 1; ++j) {
#pragma unroll
      for (int lv = 2; lv <= kMaxStored; ++lv) {
        const int c0 = (geo.M[lv] - 1) * geo.g + j;
        const bool have = lv <= geo.Lstore && c0 < geo.M[lv - 1] - 1;
        x[lv] = pb[(geo.off[1] + (have ? geo.off[lv - 1] - geo.off[1] + c0 : 0)) * D + d];
        x[lv] = have ? x[lv] : 0.f;
      }
#pragma unroll
      for (int lv = 2; lv <= kMaxStored; ++lv) sum[lv] += x[lv];
    }
  }
  __syncthreads();
  if (d < D) {
    float v = mean[d];
#pragma unroll
    for (int lv = 2; lv <= kMaxStored; ++lv) {
      if (lv <= geo.Lstore) {
        v = (sum[lv] + v) / static_cast<float>(geo.M[lv - 1] - (geo.M[lv] - 1) * geo.g);
        pb[(geo.off[lv] + geo.M[lv] - 1) * D + d] = v;
      }
    }
  }
}

}  // namespace pisa
