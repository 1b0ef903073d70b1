// Trees of drafted tokens: the masks and positions that a tree's parents give, and
// the accepted rows' way into a cache of the problem's type.
#include "common.h"
#include "kernels.h"
#include "pyramid_path.h"

namespace pisa {

// A workgroup per tree and word of the mask, a thread per token.  After round r token
// i knows its word of its nearest 2^r ancestors, how many they are, and the one behind
// them; the next round adds what that one knows.  So a chain of T tokens takes log2(T)
// rounds of two LDS reads (777 tokens that follow one of the last eight: 6.6 us, where
// walking each token's ancestors one by one took 21).
__global__ __launch_bounds__(1024) void draft_layout_kernel(const int32_t* __restrict__ parents, int T, int n,
                                                            uint64_t* __restrict__ mask, int32_t* __restrict__ positions) {
  __shared__ uint64_t bits[1024];
  __shared__ int next[1024], above[1024];  // the ancestor behind those that are known (-1: none), and their number
  const int b = blockIdx.y, word = blockIdx.x, i = threadIdx.x;
  const int64_t row = static_cast<int64_t>(b) * T + i;
  int up = -2;
  if (i < T) {
    up = parents[row];
    bits[i] = (i >> 6) == word ? uint64_t(1) << (i & 63) : 0;
    next[i] = up < T ? max(up, -1) : -1;
    above[i] = next[i] >= 0 ? 1 : 0;
  }
  __syncthreads();
  for (int span = 1; span < T; span *= 2) {
    uint64_t more = 0;
    int j = -1, k = 0;
    if (i < T && next[i] >= 0) {
      const int at = next[i];
      more = bits[at];
      j = next[at];
      k = above[at];
    }
    __syncthreads();
    if (i < T) {
      bits[i] |= more;
      next[i] = j;
      above[i] += k;
    }
    if (!__syncthreads_or(j >= 0)) break;  // every token knows all of its ancestors
  }
  if (i >= T) return;
  mask[row * gridDim.x + word] = up < -1 ? 0 : bits[i];
  if (positions && word == 0) positions[row] = n + (up < -1 ? 0 : min(above[i], T - 1));
}

hipError_t launch_draft_layout(const int32_t* parents, int B, int T, int n, uint64_t* mask, int32_t* positions, hipStream_t st) {
  const int W = (T + 63) / 64;
  ProfScope ps("draft_layout", st);
  draft_layout_kernel<<<dim3(W, B), W * 64, 0, st>>>(parents, T, n, mask, positions);
  return hipGetLastError();
}

namespace {

// Rows of one block as a wavefront sees them: 16 lanes cover a row, the four row
// groups take every fourth (the order of pool.hip's leaf_mean, to the same bits).
template <typename T, int D, bool PICK>
struct BlockRows {
  T* cache;             // the (batch, KV head)'s rows from the block's first on, at this lane's columns
  const T* fresh;       // its drafted rows, likewise
  const int32_t* rows;  // PICK: which drafted row each appended one is; otherwise one after another
  int64_t stride;       // between drafted rows
  int had, at, n_rows;  // rows of the block that the cache has; place of the block's first row among the appended ones
  __device__ __forceinline__ const T* source(int r) const {
    const int i = max(at + r, 0);
    uintptr_t drafted = reinterpret_cast<uintptr_t>(fresh + (PICK ? picked_row(rows, i, n_rows) : i) * stride);
    asm volatile("" : "+v"(drafted));  // a choice between two addresses, no branch
    return r < had ? cache + static_cast<int64_t>(r) * D : reinterpret_cast<const T*>(drafted);
  }
};

template <typename T, int DPL>
struct RowPart {
  static constexpr int W = DPL * sizeof(T) / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (W == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[0] = x.x, w[1] = x.y;
    } else {
#pragma unroll
      for (int j = 0; j < W; j += 4) {
        const uint4 x = reinterpret_cast<const uint4*>(p)[j / 4];
        w[j] = x.x, w[j + 1] = x.y, w[j + 2] = x.z, w[j + 3] = x.w;
      }
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (W == 2) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (int j = 0; j < W; j += 4) reinterpret_cast<uint4*>(p)[j / 4] = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
    }
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float((e & 1) ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
};

// Copies the block's appended rows into the cache.  KEYS with a pyramid: reads all
// of its rows and returns their mean (in every lane).
template <typename T, int D, bool MEAN, bool PICK>
__device__ __forceinline__ void append_block(const BlockRows<T, D, PICK>& src, int nrows, int rg, float (&m)[D / 16]) {
  constexpr int DPL = D / 16;
  if constexpr (MEAN) {
#pragma unroll
    for (int e = 0; e < DPL; ++e) m[e] = 0.f;
  }
  // the rows that are only read are left out where no mean is wanted
  int r = MEAN ? rg : src.had / 16 * 16 + rg;
  for (; r < nrows; r += 16) {
    RowPart<T, DPL> x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i].load(src.source(min(r + 4 * i, nrows - 1)));
    if constexpr (MEAN) {
      if (r + 12 < nrows) {
#pragma unroll
        for (int e = 0; e < DPL; ++e) m[e] += (x[0].at(e) + x[1].at(e)) + (x[2].at(e) + x[3].at(e));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (r + 4 * i < nrows) {
#pragma unroll
            for (int e = 0; e < DPL; ++e) m[e] += x[i].at(e);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int rr = r + 4 * i;
      if (rr >= src.had && rr < nrows) x[i].store(src.cache + static_cast<int64_t>(rr) * D);
    }
  }
  if constexpr (MEAN) {
    const float f = 1.0f / static_cast<float>(nrows);
#pragma unroll
    for (int e = 0; e < DPL; ++e) {
      m[e] += __shfl_xor(m[e], 16);
      m[e] += __shfl_xor(m[e], 32);
      m[e] *= f;
    }
  }
}

}  // namespace

// A wavefront per changed block and side.  PATH (one or two blocks change): a workgroup
// per (batch, KV head), a wavefront for the keys and one for the values of each block,
// and two for the levels, as qcache_append_kernel has it.  A prompt is bound by HBM
// (131072 rows of 8 heads of 128 in bf16: 207 us, 229 with the pyramid; a copy of both
// 183), a tree's rows by the chain of rows, mean and levels (4 x 9 rows 6.5 us, where
// the levels in launches of their own took 13.3).
template <typename T, int D, int PATH, bool PICK>
__global__ __launch_bounds__(PATH == 2 ? 384 : 256) void cache_append_kernel(CacheAppend a, Geo geo, bool grown) {
  constexpr int DPL = D / 16;
  __shared__ __align__(16) float mean[PATH ? PATH : 1][D];
  const int C = geo.C;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sub = lane & 15, rg = lane >> 4;
  const int bh = blockIdx.y, b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int first = a.n_old / C, last = (geo.N - 1) / C;
  const int unit = PATH ? wave : static_cast<int>(blockIdx.x) * 4 + wave;
  const int leaf = first + unit / 2;
  const bool keys = unit % 2 == 0;
  float* pb = a.pyr + static_cast<int64_t>(bh) * geo.R * D;
  if (PATH ? wave < 2 * PATH : leaf <= last) {
    BlockRows<T, D, PICK> src;
    src.cache = static_cast<T*>(keys ? a.k : a.v) + (static_cast<int64_t>(bh) * geo.Nkv + static_cast<int64_t>(leaf) * C) * D +
                sub * DPL;
    src.fresh = static_cast<const T*>(keys ? a.k_new : a.v_new) + b * (keys ? a.ksb : a.vsb) + h * (keys ? a.ksh : a.vsh) + sub * DPL;
    src.rows = PICK ? a.rows + static_cast<int64_t>(b) * (geo.N - a.n_old) : nullptr;
    src.stride = keys ? a.ksn : a.vsn;
    src.had = max(0, a.n_old - leaf * C);
    src.at = leaf * C - a.n_old;
    src.n_rows = a.n_rows;
    const int nrows = min(C, geo.N - leaf * C);
    float m[DPL];
    if (keys && a.pyr) {
      append_block<T, D, true>(src, nrows, rg, m);
      if (rg == 0) {
        float* dst = pb + (geo.off[1] + leaf) * D + sub * DPL;
#pragma unroll
        for (int e = 0; e < DPL; e += 4) {
          const float4 v4 = make_float4(m[e], m[e + 1], m[e + 2], m[e + 3]);
          *reinterpret_cast<float4*>(dst + e) = v4;
          if constexpr (PATH > 0) *reinterpret_cast<float4*>(&mean[unit / 2][sub * DPL + e]) = v4;
        }
      }
    } else {
      append_block<T, D, false>(src, nrows, rg, m);
    }
    if (PATH && a.pyr) __syncthreads();
  } else if constexpr (PATH > 0) {
    if (a.pyr) path_levels<D, PATH>(geo, pb, mean, threadIdx.x - 128 * PATH, grown);
  }
}

template <typename T, int D, bool PICK>
static hipError_t launch_append(const Geo& geo, const Geo& geo_old, int BH, const CacheAppend& a, hipStream_t st) {
  const int nleaf = geo.M[1] - a.n_old / geo.C, path = path_leaves(geo, a.n_old);
  const bool grown = geo_old.Lstore != geo.Lstore;  // (n_old > 0)
  {
    ProfScope ps("cache_append", st);
    if (path == 1)
      cache_append_kernel<T, D, 1, PICK><<<dim3(1, BH), 256, 0, st>>>(a, geo, grown);
    else if (path == 2)
      cache_append_kernel<T, D, 2, PICK><<<dim3(1, BH), 384, 0, st>>>(a, geo, grown);
    else
      cache_append_kernel<T, D, 0, PICK><<<dim3((nleaf + 1) / 2, BH), 256, 0, st>>>(a, geo, grown);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || path || !a.pyr) return e;
  return launch_pyramid_levels(geo, BH, D, a.pyr, a.n_old, st);
}

template <typename T, int D>
static hipError_t launch_append_rows(const Geo& geo, const Geo& geo_old, int BH, const CacheAppend& a, hipStream_t st) {
  return a.rows ? launch_append<T, D, true>(geo, geo_old, BH, a, st) : launch_append<T, D, false>(geo, geo_old, BH, a, st);
}

hipError_t launch_cache_append(const Geo& geo, const Geo& geo_old, int BH, int D, bool bf16, const CacheAppend& a, hipStream_t st) {
  if (bf16)
    return D == 128 ? launch_append_rows<uint16_t, 128>(geo, geo_old, BH, a, st)
                    : launch_append_rows<uint16_t, 64>(geo, geo_old, BH, a, st);
  return D == 128 ? launch_append_rows<float, 128>(geo, geo_old, BH, a, st) : launch_append_rows<float, 64>(geo, geo_old, BH, a, st);
}

}  // namespace pisa
