// 8-bit key/value cache: quantising appended rows, and the mean pyramid of the
// raw keys with it.
//
// A block of C tokens of one KV head has one scale 2^e, the smallest with
// max|x| <= 448 * 2^e (448: the largest e4m3), keys and values apart.  A power
// of two makes x / 2^e and code * 2^e exact, so the only rounding is the one to
// e4m3, and every later reader (fp32 or bf16) sees the same numbers.
#include "common.h"
#include "kernels.h"

namespace pisa {

namespace {

constexpr int kLeastExp = -100;

// Exponent of the scale for the largest magnitude `u` (as bits): 448 = 1.75 * 2^8,
// so e = floor(log2) - 8, one more where the mantissa is past 1.75.
__device__ __forceinline__ int scale_exp(uint32_t u) {
  const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, kLeastExp);
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// One lane's part of up to R rows: DPL = D/16 columns of each, as loaded.
template <typename T, int D, int R>
struct Rows {
  static constexpr int DPL = D / 16;
  static constexpr int W = DPL * sizeof(T) / 4;  // words of a row part
  uint32_t w[R][W];

  template <typename F>
  __device__ __forceinline__ void load(F row) {  // row(i): address of row i's part
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const T* p = row(i);
      if constexpr (W == 2) {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        w[i][0] = x.x, w[i][1] = x.y;
      } else {
#pragma unroll
        for (int j = 0; j < W; j += 4) {
          const uint4 x = reinterpret_cast<const uint4*>(p)[j / 4];
          w[i][j] = x.x, w[i][j + 1] = x.y, w[i][j + 2] = x.z, w[i][j + 3] = x.w;
        }
      }
    }
  }
  __device__ __forceinline__ void store(int i, T* p) const {
    if constexpr (W == 2) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[i][0], w[i][1]);
    } else {
#pragma unroll
      for (int j = 0; j < W; j += 4) reinterpret_cast<uint4*>(p)[j / 4] = make_uint4(w[i][j], w[i][j + 1], w[i][j + 2], w[i][j + 3]);
    }
  }
  __device__ __forceinline__ float at(int i, int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i][e]);
    else return __uint_as_float((e & 1) ? w[i][e / 2] & 0xFFFF0000u : w[i][e / 2] << 16);
  }
  // largest magnitude as the bits of a float, of all values (an infinity or NaN
  // comes out at or past 0x7F800000) or of the finite ones
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        if constexpr (sizeof(T) == 4) big = max(big, w[i][j] & 0x7FFFFFFFu);
        else big = max_u16x2(big, w[i][j] & 0x7FFF7FFFu);
      }
    }
    return sizeof(T) == 4 ? big : max(big & 0xFFFF0000u, big << 16);
  }
  __device__ __forceinline__ uint32_t largest_finite() const {
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
      for (int e = 0; e < DPL; ++e) {
        const uint32_t u = __float_as_uint(at(i, e)) & 0x7FFFFFFFu;
        big = max(big, u < 0x7F800000u ? u : 0u);
      }
    }
    return big;
  }
};

// e4m3 codes of two values times inv in the low (or high) half of a word.  ODD:
// infinities are about, and become NaN.
template <bool HI, bool ODD>
__device__ __forceinline__ int pack2_e4m3(float a, float b, float inv, int old) {
  if constexpr (ODD) {
    const float nan = __uint_as_float(0x7FC00000u);
    a = (__float_as_uint(a) & 0x7F800000u) == 0x7F800000u ? nan : a;
    b = (__float_as_uint(b) & 0x7F800000u) == 0x7F800000u ? nan : b;
  }
  return __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, old, HI);
}
template <bool ODD>
__device__ __forceinline__ uint32_t pack4_e4m3(float a, float b, float c, float d, float inv) {
  return static_cast<uint32_t>(pack2_e4m3<true, ODD>(c, d, inv, pack2_e4m3<false, ODD>(a, b, inv, 0)));
}

// What a wavefront needs to know of the block it quantises.
template <typename T, int D>
struct Source {
  const T* open;   // the (batch, KV head)'s raw rows, at this lane's columns
  const T* fresh;  // its appended rows, likewise
  int64_t stride;  // between appended rows
  int tok0, nrows, had, n_old;
  __device__ __forceinline__ const T* row(int r) const {
    return r < had ? open + r * D : fresh + (tok0 + r - n_old) * stride;
  }
};

// Lane (sub, rg) of a wavefront: columns sub * D/16 .. of row(i) of CH rows from
// `base` on: every fourth row for keys (a store covers whole rows, and the mean
// is summed in the order of pool.hip's leaf_mean, to the same bits), CH/4 consecutive ones for values (their
// codes of one column are consecutive bytes).
template <bool KEYS, int CH>
__device__ __forceinline__ int row_at(int base, int rg, int i) {
  return KEYS ? base + rg + 4 * i : base + rg * (CH / 4) + i;
}

// Codes of the chunk's rows below C; those of rows from nrows on are 0.
template <typename T, int D, bool KEYS, int CH, bool ODD>
__device__ __forceinline__ void store_codes(const Rows<T, D, CH / 4>& x, uint8_t* dst, int C, int nrows, int base, int sub,
                                            int rg, float inv) {
  constexpr int DPL = D / 16, R = CH / 4;
  if constexpr (KEYS) {  // [C][D]
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = row_at<true, CH>(base, rg, i);
      if (r < C) {
        uint8_t* p = dst + r * D + sub * DPL;
        const uint32_t live = r < nrows ? ~0u : 0u;
        const uint32_t lo = live & pack4_e4m3<ODD>(x.at(i, 0), x.at(i, 1), x.at(i, 2), x.at(i, 3), inv);
        if constexpr (DPL == 8)
          *reinterpret_cast<uint2*>(p) = make_uint2(lo, live & pack4_e4m3<ODD>(x.at(i, 4), x.at(i, 5), x.at(i, 6), x.at(i, 7), inv));
        else
          *reinterpret_cast<uint32_t*>(p) = lo;
      }
    }
  } else {  // [D][C]; C is a multiple of 32 and so of the 8 rows that each store covers
#pragma unroll
    for (int i = 0; i < R; i += 8) {
      const int r = row_at<false, CH>(base, rg, i);
      if (r < C) {
        const int n = nrows - r;  // rows that exist: bytes to keep
        const uint32_t lo = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
        const uint32_t hi = n >= 8 ? ~0u : n <= 4 ? 0u : (1u << (8 * n - 32)) - 1u;
#pragma unroll
        for (int e = 0; e < DPL; ++e) {
          uint2 w;
          w.x = lo & pack4_e4m3<ODD>(x.at(i, e), x.at(i + 1, e), x.at(i + 2, e), x.at(i + 3, e), inv);
          w.y = hi & pack4_e4m3<ODD>(x.at(i + 4, e), x.at(i + 5, e), x.at(i + 6, e), x.at(i + 7, e), inv);
          *reinterpret_cast<uint2*>(dst + (sub * DPL + e) * C + r) = w;
        }
      }
    }
  }
}

// One block's keys or values by one wavefront.  CH rows are held in registers:
// the whole block where C <= CH, read once; larger blocks are read twice, the
// second time from the cache.  Keys: means(m) is called with the means of the
// raw rows before any code is stored.
template <typename T, int D, bool KEYS, int CH, typename F>
__device__ __forceinline__ void quantise_block(const Source<T, D>& src, int C, uint8_t* dst, float* scale, int lane, F means) {
  constexpr int DPL = D / 16, R = CH / 4;
  const int sub = lane & 15, rg = lane >> 4;
  Rows<T, D, R> x;
  auto load = [&](int base) {  // rows past the last one are read as the last one
    const int r0 = row_at<KEYS, CH>(base, rg, 0), step = KEYS ? 4 : 1;
    const T* fresh = src.fresh + (src.tok0 - src.n_old + r0) * src.stride;
    const T* end = src.row(src.nrows - 1);
    x.load([&](int i) {
      const int r = r0 + i * step;
      const T* p = r < src.had ? src.open + r * D : fresh + i * step * src.stride;
      return r < src.nrows ? p : end;
    });
  };
  auto lanes_max = [&](uint32_t v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o)));
    return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v)));
  };
  uint32_t big = 0;
  float m[DPL];
#pragma unroll
  for (int e = 0; e < DPL; ++e) m[e] = 0.f;
  for (int base = 0; base < C; base += CH) {
    load(base);
    big = max(big, x.largest());
    if constexpr (KEYS) {
#pragma unroll
      for (int i = 0; i < R; i += 4) {
        const int r = base + rg + 4 * i;
        if (r + 12 < src.nrows) {
#pragma unroll
          for (int e = 0; e < DPL; ++e) m[e] += (x.at(i, e) + x.at(i + 1, e)) + (x.at(i + 2, e) + x.at(i + 3, e));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (r + 4 * j < src.nrows) {
#pragma unroll
              for (int e = 0; e < DPL; ++e) m[e] += x.at(i + j, e);
            }
          }
        }
      }
    }
  }
  if constexpr (KEYS) {
    const float f = 1.0f / static_cast<float>(src.nrows);
#pragma unroll
    for (int e = 0; e < DPL; ++e) {
      m[e] += __shfl_xor(m[e], 16);
      m[e] += __shfl_xor(m[e], 32);
      m[e] *= f;
    }
    means(m);
  }
  big = lanes_max(big);
  const bool odd = big >= 0x7F800000u;
  if (odd) {
    big = 0;
    for (int base = 0; base < C; base += CH) {
      if (C > CH) load(base);
      big = max(big, x.largest_finite());
    }
    big = lanes_max(big);
  }
  const int ex = scale_exp(big);
  const float inv = exp2i(-ex);
  if (lane == 0) *scale = exp2i(ex);
  for (int base = 0; base < C; base += CH) {
    if (C > CH) load(base);
    if (odd)
      store_codes<T, D, KEYS, CH, true>(x, dst, C, src.nrows, base, sub, rg, inv);
    else
      store_codes<T, D, KEYS, CH, false>(x, dst, C, src.nrows, base, sub, rg, inv);
  }
}

// The rows of the last block that were appended now, into the raw rows.  Called
// by the wavefront that read the old raw rows, after it used them.
template <typename T, int D>
__device__ __forceinline__ void keep_raw(const Source<T, D>& src, T* open, int last0, int N, int lane) {
  constexpr int R = 8;
  const int rg = lane >> 4, n = N - last0;
  for (int r0 = max(0, src.n_old - last0); r0 < n; r0 += 4 * R) {
    Rows<T, D, R> x;
    x.load([&](int i) { return src.fresh + (last0 + min(r0 + rg + 4 * i, n - 1) - src.n_old) * src.stride; });
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = r0 + rg + 4 * i;
      if (r < n) x.store(i, open + r * D);
    }
  }
}

// Most stored levels: 65535 leaf blocks, two children to a node.
constexpr int kMaxStored = 16;

}  // namespace

// A wavefront per changed block and side.  PATH (only the last block changed and
// no level is new): a workgroup per (batch, KV head), wavefront 0 for the keys, 1
// for the values; the others sum the unchanged children of the block's ancestors
// meanwhile, all levels' loads in flight at once, and take the mean up from
// there (node_mean's order: children by index, the changed one last).  Otherwise
// four wavefronts on their own: blocks x {keys, values}.
template <typename T, int D, int CH, bool PATH>
__global__ __launch_bounds__(256) void qcache_append_kernel(QAppend a, Geo geo) {
  constexpr int DPL = D / 16;
  __shared__ __align__(16) float mean[D];
  const int C = geo.C;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sub = lane & 15, rg = lane >> 4;
  const int bh = blockIdx.y, b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int first = a.n_old / C, last = (geo.N - 1) / C;
  const int unit = PATH ? wave : static_cast<int>(blockIdx.x) * 4 + wave;
  const int leaf = first + unit / 2;
  const bool keys = unit % 2 == 0;
  float* pb = a.pyr + static_cast<int64_t>(bh) * geo.R * D;

  if (PATH ? wave < 2 : leaf <= last) {
    Source<T, D> src;
    T* open = static_cast<T*>(keys ? a.k_open : a.v_open) + static_cast<int64_t>(bh) * C * D + sub * DPL;
    src.open = open;
    src.fresh = static_cast<const T*>(keys ? a.k_new : a.v_new) + b * (keys ? a.ksb : a.vsb) + h * (keys ? a.ksh : a.vsh) + sub * DPL;
    src.stride = keys ? a.ksn : a.vsn;
    src.tok0 = leaf * C;
    src.nrows = min(C, geo.N - src.tok0);
    src.n_old = a.n_old;
    src.had = max(0, a.n_old - src.tok0);
    const int64_t blk = static_cast<int64_t>(bh) * a.c.M + leaf;
    if (keys) {
      quantise_block<T, D, true, CH>(src, C, a.c.k + blk * C * D, a.c.k_scale + blk, lane, [&](const float (&m)[DPL]) {
        if (!a.pyr) return;
        if (rg == 0) {
          float* dst = pb + (geo.off[1] + leaf) * D + sub * DPL;
#pragma unroll
          for (int e = 0; e < DPL; e += 4) {
            const float4 v4 = make_float4(m[e], m[e + 1], m[e + 2], m[e + 3]);
            *reinterpret_cast<float4*>(dst + e) = v4;
            if constexpr (PATH) *reinterpret_cast<float4*>(mean + sub * DPL + e) = v4;
          }
        }
        if constexpr (PATH) __syncthreads();
      });
    } else {
      if constexpr (PATH)
        if (a.pyr) __syncthreads();
      quantise_block<T, D, false, CH>(src, C, a.c.v + blk * C * D, a.c.v_scale + blk, lane, [](const float (&)[DPL]) {});
    }
    if (leaf == first) keep_raw<T, D>(src, open, last * C, geo.N, lane);
  } else if (PATH && a.pyr) {
    const int d = threadIdx.x - 128;
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
}

template <typename T, int D, int CH>
static hipError_t launch_append(const Geo& geo, const Geo& geo_old, int BH, const QAppend& a, hipStream_t st) {
  const int first = a.n_old / geo.C, nleaf = geo.M[1] - first;
  const bool path = a.n_old > 0 && nleaf == 1 && geo_old.Lstore == geo.Lstore;
  {
    ProfScope ps("qcache_append", st);
    if (path) {
      qcache_append_kernel<T, D, CH, true><<<dim3(1, BH), 256, 0, st>>>(a, geo);
    } else {
      qcache_append_kernel<T, D, CH, false><<<dim3((nleaf + 1) / 2, BH), 256, 0, st>>>(a, geo);
    }
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || path || !a.pyr) return e;
  return launch_pyramid_levels(geo, BH, D, a.pyr, a.n_old, st);
}

// Rows in registers: 64 are 64 registers a lane in bf16 with d = 128 (128 in
// fp32); bf16 blocks of more than 64 tokens get 128.
template <typename T, int D>
static hipError_t launch_append_ch(const Geo& geo, const Geo& geo_old, int BH, const QAppend& a, hipStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (geo.C > 64) return launch_append<T, D, 128>(geo, geo_old, BH, a, st);
  return launch_append<T, D, 64>(geo, geo_old, BH, a, st);
}

hipError_t launch_qcache_append(const Geo& geo, const Geo& geo_old, int BH, int D, bool bf16, const QAppend& a,
                                hipStream_t st) {
  if (bf16)
    return D == 128 ? launch_append_ch<uint16_t, 128>(geo, geo_old, BH, a, st) : launch_append_ch<uint16_t, 64>(geo, geo_old, BH, a, st);
  return D == 128 ? launch_append_ch<float, 128>(geo, geo_old, BH, a, st) : launch_append_ch<float, 64>(geo, geo_old, BH, a, st);
}

}  // namespace pisa
