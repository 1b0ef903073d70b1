// 8-bit key/value cache: quantising appended rows, and the mean pyramid of the
// raw keys with it.
//
// A block of C tokens of one KV head has one scale 2^e, the smallest with
// max|x| <= 448 * 2^e (448: the largest e4m3), keys and values apart.  A power
// of two makes x / 2^e and code * 2^e exact, so the only rounding is the one to
// e4m3, and every later reader (fp32 or bf16) sees the same numbers.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "pool.h"

namespace pisa {

namespace {

constexpr int kLeastExp = -100;

// Magnitude bits of a finite value, 0 for an infinity or NaN.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}

// Exponent of the scale for the largest magnitude `u` (as bits): 448 = 1.75 * 2^8,
// so e = floor(log2) - 8, one more where the mantissa is past 1.75.
__device__ __forceinline__ int scale_exp(uint32_t u) {
  const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, kLeastExp);
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// e4m3 codes of two values in the low (or high) half of a word; infinities and
// NaN become the NaN code.
__device__ __forceinline__ float nan_if_not_finite(float x) {
  return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : x;
}
template <bool HI>
__device__ __forceinline__ int pack2_e4m3(float a, float b, int old) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(nan_if_not_finite(a), nan_if_not_finite(b), old, HI);
}

}  // namespace

// One workgroup per changed block, for its keys (blockIdx.z = 0) or its values.
// PATH: only the last block changed and no level is new, so the keys'
// workgroup also walks the block's ancestors up (as pool_append_path_kernel).
template <typename T, int D, bool PATH>
__global__ __launch_bounds__(256) void qcache_append_kernel(QAppend a, Geo geo) {
  constexpr int DPL = D / 16;
  extern __shared__ __align__(16) uint8_t lds[];  // values: codes [D][C]; keys with PATH: [D] mean, siblings
  __shared__ uint32_t s_max[4];
  const int C = geo.C;
  const int bh = blockIdx.y, b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int first = a.n_old / C, last = (geo.N - 1) / C;
  const int leaf = first + static_cast<int>(blockIdx.x);
  const bool keys = blockIdx.z == 0;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int grp = tid >> 4, sub = tid & 15;
  const int tok0 = leaf * C;
  const int nrows = min(C, geo.N - tok0);
  const int had = max(0, a.n_old - tok0);  // rows that are in the open block
  T* open = static_cast<T*>(keys ? a.k_open : a.v_open) + static_cast<int64_t>(bh) * C * D;
  const int64_t sn = keys ? a.ksn : a.vsn;
  const T* fresh = static_cast<const T*>(keys ? a.k_new : a.v_new) + b * (keys ? a.ksb : a.vsb) + h * (keys ? a.ksh : a.vsh);
  auto row = [&](int r) -> const T* {  // this lane's slice of the block's row r
    return (r < had ? open + r * D : fresh + (tok0 + r - a.n_old) * sn) + sub * DPL;
  };

  if constexpr (PATH) {
    if (keys && a.pyr && wave > 0) {
      // siblings of each ancestor's changed child, fetched while the rows are
      float* sib = reinterpret_cast<float*>(lds) + D;
      const float* pb = a.pyr + static_cast<int64_t>(bh) * geo.R * D;
      for (int lv = 2; lv <= geo.Lstore; ++lv) {
        const int c0 = (geo.M[lv] - 1) * geo.g, ns = geo.M[lv - 1] - 1 - c0;
        float* dst = sib + (lv - 2) * (geo.g - 1) * D;
        for (int e = tid - 64; e < ns * D; e += 192) dst[e] = pb[(geo.off[lv - 1] + c0) * D + e];
      }
    }
  }

  uint32_t big = 0;
  for (int r = grp; r < nrows; r += 16) {
    float x[DPL];
    load_row_part<T, DPL>(row(r), x);
#pragma unroll
    for (int e = 0; e < DPL; ++e) big = max(big, finite_bits(x[e]));
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) big = max(big, static_cast<uint32_t>(__shfl_xor(static_cast<int>(big), o)));
  if (lane == 0) s_max[wave] = big;
  __syncthreads();
  const int ex = scale_exp(max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3])));
  const float inv = exp2i(-ex);
  const int64_t blk = static_cast<int64_t>(bh) * a.c.M + leaf;
  if (tid == 0) (keys ? a.c.k_scale : a.c.v_scale)[blk] = exp2i(ex);

  if (keys) {
    uint8_t* dst = a.c.k + blk * C * D + sub * DPL;
    for (int r = grp; r < C; r += 16) {
      uint2 w = make_uint2(0, 0);
      if (r < nrows) {
        float x[DPL];
        load_row_part<T, DPL>(row(r), x);
        w.x = pack2_e4m3<true>(x[2] * inv, x[3] * inv, pack2_e4m3<false>(x[0] * inv, x[1] * inv, 0));
        if constexpr (DPL == 8)
          w.y = pack2_e4m3<true>(x[6] * inv, x[7] * inv, pack2_e4m3<false>(x[4] * inv, x[5] * inv, 0));
      }
      if constexpr (DPL == 8)
        *reinterpret_cast<uint2*>(dst + static_cast<int64_t>(r) * D) = w;
      else
        *reinterpret_cast<uint32_t*>(dst + static_cast<int64_t>(r) * D) = w.x;
    }
  } else {
    for (int r = grp; r < C; r += 16) {
      float x[DPL];
#pragma unroll
      for (int e = 0; e < DPL; ++e) x[e] = 0.f;
      if (r < nrows) load_row_part<T, DPL>(row(r), x);
#pragma unroll
      for (int e = 0; e < DPL; ++e)
        lds[(sub * DPL + e) * C + r] = static_cast<uint8_t>(pack2_e4m3<false>(x[e] * inv, 0.f, 0));
    }
    __syncthreads();
    uint4* dst = reinterpret_cast<uint4*>(a.c.v + blk * C * D);
    for (int e = tid; e < C * D / 16; e += 256) dst[e] = reinterpret_cast<const uint4*>(lds)[e];
  }

  if (keys && a.pyr) {
    float* pb = a.pyr + static_cast<int64_t>(bh) * geo.R * D;
    float* val = reinterpret_cast<float*>(lds);
    if (wave == 0) {
      const int rg = lane >> 4;
      float m[DPL];
      leaf_mean_rows<T, D>(row, nrows, rg, m);
      if (rg == 0) {
        float* dst = pb + (geo.off[1] + leaf) * D + sub * DPL;
#pragma unroll
        for (int e = 0; e < DPL; e += 4) {
          const float4 v4 = make_float4(m[e], m[e + 1], m[e + 2], m[e + 3]);
          *reinterpret_cast<float4*>(dst + e) = v4;
          if constexpr (PATH) *reinterpret_cast<float4*>(val + sub * DPL + e) = v4;
        }
      }
    }
    if constexpr (PATH) {
      __syncthreads();
      if (tid < D) {
        float x = val[tid];
        for (int lv = 2; lv <= geo.Lstore; ++lv) {
          const int ns = geo.M[lv - 1] - 1 - (geo.M[lv] - 1) * geo.g;
          const float* sv = val + D + (lv - 2) * (geo.g - 1) * D + tid;
          float sum = 0.f;
          for (int j = 0; j < ns; ++j) sum += sv[j * D];
          sum += x;
          x = sum / static_cast<float>(ns + 1);
          pb[(geo.off[lv] + geo.M[lv] - 1) * D + tid] = x;
        }
      }
    }
  }

  // The last block's raw rows become the open ones.  The first block's
  // workgroup writes them, after its own reads of the old ones.
  if (blockIdx.x == 0) {
    __syncthreads();
    const int l0 = last * C;
    for (int r = grp; r < geo.N - l0; r += 16) {
      if (l0 + r < a.n_old) continue;  // already there
      const T* src = fresh + (l0 + r - a.n_old) * sn + sub * DPL;
      T* dst = open + r * D + sub * DPL;
      if constexpr (sizeof(T) * DPL == 8)
        *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(src);
      else
#pragma unroll
        for (int e = 0; e < DPL; e += 16 / sizeof(T))
          *reinterpret_cast<uint4*>(dst + e) = *reinterpret_cast<const uint4*>(src + e);
    }
  }
}

template <typename T, int D>
static hipError_t launch_append(const Geo& geo, const Geo& geo_old, int BH, const QAppend& a, hipStream_t st) {
  const int first = a.n_old / geo.C, nleaf = geo.M[1] - first;
  const bool path = a.n_old > 0 && nleaf == 1 && geo_old.Lstore == geo.Lstore;
  const dim3 grid(nleaf, BH, 2);
  const size_t codes = static_cast<size_t>(geo.C) * D;
  {
    ProfScope ps("qcache_append", st);
    if (path) {
      const size_t sib = (static_cast<size_t>(D) + static_cast<size_t>(geo.Lstore) * (geo.g - 1) * D) * sizeof(float);
      qcache_append_kernel<T, D, true><<<grid, 256, std::max(codes, sib), st>>>(a, geo);
    } else {
      qcache_append_kernel<T, D, false><<<grid, 256, codes, st>>>(a, geo);
    }
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || path || !a.pyr) return e;
  return launch_pyramid_levels(geo, BH, D, a.pyr, a.n_old, st);
}

hipError_t launch_qcache_append(const Geo& geo, const Geo& geo_old, int BH, int D, bool bf16, const QAppend& a,
                                hipStream_t st) {
  if (bf16) return D == 128 ? launch_append<uint16_t, 128>(geo, geo_old, BH, a, st) : launch_append<uint16_t, 64>(geo, geo_old, BH, a, st);
  return D == 128 ? launch_append<float, 128>(geo, geo_old, BH, a, st) : launch_append<float, 64>(geo, geo_old, BH, a, st);
}

}  // namespace pisa
