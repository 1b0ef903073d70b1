// Sparse attention over the 8-bit cache (qcache.hip).
//
// A wavefront takes KU keys of one selected block (KU = 64, or 32 where C is no
// multiple of 64) for the up to 16 query heads of a KV head, straight from the
// cache into matrix operands: no LDS.  With v_mfma_f32_16x16x32_bf16 (A lane l:
// row l%16, k 8*(l/16)..+7; B lane l: k 8*(l/16)..+7, column l%16; D lane l:
// rows 4*(l/16)..+3, column l%16):
//   S^T = K q^T      rows: keys, columns: heads.  Row r of tile mt is key
//                    (r/4)*(KU/4) + 4*mt + r%4, so that lane group r/4 ends up
//                    with the logits of KU/4 consecutive keys, and the dimensions
//                    are dealt so that a lane reads D/4 consecutive bytes.
//   O^T += V^T P^T   the same keys: a lane reads KU/4 consecutive tokens of one
//                    dimension, which is why the cache keeps values transposed.
// e4m3 times a power of two is exact in bf16, and so are its products with q in
// fp32.  32-bit queries are split into three bf16 terms that add up to them
// exactly, and so are their weights; bf16 queries' weights are rounded to bf16
// (relative 2^-8 at most each, as in the other attention kernels), their sum is not.
#include <algorithm>

#include "attn_shared.h"
#include "common.h"
#include "kernels.h"

namespace pisa {

namespace {

struct QAttnArgs {
  QCache c;
  const void* q;
  const int32_t* idx;
  void* o;
  float* lse;
  // splits > 1: unnormalised sums [rows][splits][G][D], and maximum and sum
  // [rows][G][splits]
  float* part_o;
  float2* part_ml;
  int H, Hkv, G, Nq, N, C, K, causal, M1;
  int BH, splits;
  int row0;  // first row of this launch
  float qscale2;
};

// Four e4m3 codes times 2^e as four bf16.
__device__ __forceinline__ uint2 codes4_bf16(uint32_t w, float scale) {
  const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
  const bf16x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}
__device__ __forceinline__ bf16x8a codes8_bf16(uint32_t w0, uint32_t w1, float scale) {
  const uint2 a = codes4_bf16(w0, scale), b = codes4_bf16(w1, scale);
  return u4_as_bf16x8(make_uint4(a.x, a.y, b.x, b.y));
}

// bf16 terms of 8 floats: x = term 0 + term 1 + term 2 exactly (NT = 3), or its
// rounding (NT = 1).  A term of an infinity or NaN is followed by zeros.
template <int NT>
__device__ __forceinline__ void split_terms(const float (&x)[8], bf16x8a (&t)[NT]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = pack2_bf16(r[2 * i], r[2 * i + 1]);
      if (j + 1 < NT) {
        const float a = __uint_as_float(w[i] << 16), b = __uint_as_float(w[i] & 0xFFFF0000u);
        r[2 * i] = __builtin_isfinite(a) ? r[2 * i] - a : 0.f;
        r[2 * i + 1] = __builtin_isfinite(b) ? r[2 * i + 1] - b : 0.f;
      }
    }
    t[j] = u4_as_bf16x8(make_uint4(w[0], w[1], w[2], w[3]));
  }
}

// Word w of codes at token `at`: those of tokens >= limit cleared.
__device__ __forceinline__ uint32_t keep_below(uint32_t w, int at, int limit) {
  const int n = limit - at;
  return n >= 4 ? w : n <= 0 ? 0u : w & ((1u << (8 * n)) - 1u);
}

}  // namespace

// A key unit's codes and scales, as a wavefront's lanes hold them.
template <int D, int KU>
struct Unit {
  static constexpr int MT = KU / 16;  // key tiles
  static constexpr int DT = D / 16;   // dimension tiles of O
  static constexpr int KW = D / 16;   // words of a lane's part of a key (D/4 bytes)
  static constexpr int VW = KU / 16;  // words of a lane's part of a dimension (KU/4 tokens)
  uint32_t kw[MT][KW], vw[DT][VW];
  float ksc, vsc;
  int nkeys;  // visible keys, from the first on

  __device__ __forceinline__ void load(const QCache& c, int64_t cell, int C, int u, int visible, int col, int grp) {
    const uint8_t* kp = c.k + (cell * C + u * KU) * D + grp * (D / 4);
    const uint8_t* vp = c.v + cell * C * D + u * KU + grp * (KU / 4);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int key = (col >> 2) * (KU / 4) + mt * 4 + (col & 3);
#pragma unroll
      for (int i = 0; i < KW; i += 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(kp + key * D + i * 4);
        kw[mt][i] = x.x, kw[mt][i + 1] = x.y, kw[mt][i + 2] = x.z, kw[mt][i + 3] = x.w;
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const uint8_t* p = vp + (dt * 16 + col) * C;
      if constexpr (VW == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        vw[dt][0] = x.x, vw[dt][1] = x.y, vw[dt][2] = x.z, vw[dt][3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        vw[dt][0] = x.x, vw[dt][1] = x.y;
      }
    }
    ksc = c.k_scale[cell];
    vsc = c.v_scale[cell];
    nkeys = visible;
  }
};

// Running softmax of a wavefront's 16 columns over key units.
template <int D, int KU, int NT>
struct Softmax {
  using U = Unit<D, KU>;
  static constexpr int KS = D / 32;  // k-steps of S
  f32x4a oacc[U::DT];
  float m = -INFINITY, l = 0.f;

  __device__ __forceinline__ Softmax() {
#pragma unroll
    for (int dt = 0; dt < U::DT; ++dt) oacc[dt] = f32x4a{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void add(U& u, const bf16x8a (&qt)[KS][NT], float qscale2, int grp) {
    f32x4a s[U::MT];
#pragma unroll
    for (int mt = 0; mt < U::MT; ++mt) {
      s[mt] = f32x4a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8a kv = codes8_bf16(u.kw[mt][2 * ks], u.kw[mt][2 * ks + 1], u.ksc);
#pragma unroll
        for (int j = 0; j < NT; ++j) s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv, qt[ks][j], s[mt], 0, 0, 0);
      }
    }
    // lane (col, grp) holds keys grp*KU/4 + 4*mt + i; hidden ones: weight 0, and
    // their codes are cleared (0 times a NaN code would not be 0)
    const int k0 = grp * (KU / 4);
    if (u.nkeys < KU) {
#pragma unroll
      for (int mt = 0; mt < U::MT; ++mt) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[mt][i] = k0 + 4 * mt + i < u.nkeys ? s[mt][i] : -INFINITY;
      }
#pragma unroll
      for (int dt = 0; dt < U::DT; ++dt) {
#pragma unroll
        for (int i = 0; i < U::VW; ++i) u.vw[dt][i] = keep_below(u.vw[dt][i], k0 + 4 * i, u.nkeys);
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < U::MT; ++mt) mx = fmaxf(mx, fmaxf(fmaxf(s[mt][0], s[mt][1]), fmaxf(s[mt][2], s[mt][3])));
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float mn = fmaxf(m, mx * qscale2);
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float corr = fast_exp2(m - ref);
    m = mn;
    float sum = 0.f;
#pragma unroll
    for (int mt = 0; mt < U::MT; ++mt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[mt][i] = fast_exp2(fmaf(s[mt][i], qscale2, -ref));
        sum += s[mt][i];
      }
    }
    l = l * corr + sum;
#pragma unroll
    for (int dt = 0; dt < U::DT; ++dt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) oacc[dt][i] *= corr;
    }
#pragma unroll
    for (int st = 0; st < U::MT / 2; ++st) {
      const float p[8] = {s[2 * st][0], s[2 * st][1], s[2 * st][2], s[2 * st][3],
                          s[2 * st + 1][0], s[2 * st + 1][1], s[2 * st + 1][2], s[2 * st + 1][3]};
      bf16x8a pt[NT];
      split_terms<NT>(p, pt);
#pragma unroll
      for (int dt = 0; dt < U::DT; ++dt) {
        const bf16x8a vv = codes8_bf16(u.vw[dt][2 * st], u.vw[dt][2 * st + 1], u.vsc);
#pragma unroll
        for (int j = 0; j < NT; ++j) oacc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pt[j], oacc[dt], 0, 0, 0);
      }
    }
  }
};

// One workgroup of NW wavefronts per (row, KV head, split of its key units).
template <typename T, int D, int KU, int NW>
__global__ __launch_bounds__(NW * 64, 2) void qcache_attn_kernel(QAttnArgs a) {
  constexpr int NT = sizeof(T) == 4 ? 3 : 1;  // bf16 terms of a query and of a weight
  constexpr int KS = D / 32;
  constexpr int DT = D / 16;
  extern __shared__ __align__(16) float red[];  // [NW][G][D + 2]

  const int64_t w = blockIdx.x;
  const int bh = static_cast<int>(w % a.BH);
  const int row = a.row0 + static_cast<int>(w / a.BH);
  const int split = blockIdx.y;
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, grp = lane >> 4;
  const int t = a.N - a.Nq + row;
  const int end = a.causal ? min(a.N, t + 1) : a.N;  // tokens from here on are hidden

  // the row's blocks, one per lane (K <= 128); queries: column col is head col,
  // dimensions grp*D/4 .. +D/4-1
  const int32_t* sel = a.idx + (static_cast<int64_t>(bh) * a.Nq + row) * a.K;
  const int sel0 = lane < a.K ? sel[lane] : -1, sel1 = lane + 64 < a.K ? sel[lane + 64] : -1;
  float qx[KS][8];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
    for (int i = 0; i < 8; ++i) qx[ks][i] = 0.f;
    if (col < a.G)
      load_row_part<T, 8>(static_cast<const T*>(a.q) + ((static_cast<int64_t>(b) * a.H + h * a.G + col) * a.Nq + row) * D +
                              grp * (D / 4) + ks * 8, qx[ks]);
  }

  const int per = a.C / KU;  // key units of a block
  const int ntask = a.K * per, step = a.splits * NW;
  // the next unit from `task` on with a visible key: loaded into u; ntask at the end
  auto fetch = [&](int task, Unit<D, KU>& u) {
    for (; task < ntask; task += step) {
      const int slot = task / per, part = task - slot * per;
      const int blk = __builtin_amdgcn_readlane(slot < 64 ? sel0 : sel1, slot & 63);
      if (static_cast<uint32_t>(blk) >= static_cast<uint32_t>(a.M1)) continue;  // padding
      const int visible = min(KU, end - (blk * a.C + part * KU));
      if (visible <= 0) continue;
      u.load(a.c, static_cast<int64_t>(bh) * a.c.M + blk, a.C, part, visible, col, grp);
      break;
    }
    return task;
  };
  Unit<D, KU> ua, ub;
  int ta = fetch(split * NW + wave, ua);
  bf16x8a qt[KS][NT];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) split_terms<NT>(qx[ks], qt[ks]);
  Softmax<D, KU, NT> sm;
  while (ta < ntask) {  // the next unit's loads are in flight while one is added
    const int tb = fetch(ta + step, ub);
    sm.add(ua, qt, a.qscale2, grp);
    if (tb >= ntask) break;
    ta = fetch(tb + step, ua);
    sm.add(ub, qt, a.qscale2, grp);
  }
  auto& oacc = sm.oacc;
  const float m = sm.m;
  float l = sm.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // the wavefronts' states of every head meet in LDS
  constexpr int W = D + 2;
  if (col < a.G) {
    float* mine = red + (wave * a.G + col) * W;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) mine[dt * 16 + grp * 4 + i] = oacc[dt][i];
    }
    if (grp == 0) {
      mine[D] = m;
      mine[D + 1] = l;
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.G * D; e += NW * 64) {
    const int hh = e / D, dd = e - hh * D;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NW; ++i) top = fmaxf(top, red[(i * a.G + hh) * W + D]);
    const float ref = top == -INFINITY ? 0.f : top;
    float ll = 0.f, oo = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float* r = red + (i * a.G + hh) * W;
      const float f = fast_exp2(r[D] - ref);
      ll += r[D + 1] * f;
      oo += r[dd] * f;
    }
    if (a.splits == 1) {
      const int64_t orow = (static_cast<int64_t>(b) * a.H + h * a.G + hh) * a.Nq + row;
      const float res = ll == 0.f ? 0.f : oo / ll;
      if constexpr (sizeof(T) == 2)
        static_cast<uint16_t*>(a.o)[orow * D + dd] = f32_to_bf16_rne(res);
      else
        static_cast<float*>(a.o)[orow * D + dd] = res;
      if (a.lse && dd == 0) a.lse[orow] = ll == 0.f ? -INFINITY : (ref + fast_log2(ll)) * kLn2;
    } else {
      a.part_o[((w * a.splits + split) * a.G + hh) * D + dd] = oo;
      if (dd == 0) a.part_ml[(w * a.G + hh) * a.splits + split] = make_float2(top, ll);
    }
  }
}

// The splits' states of one (row, head): a wavefront, lane i < splits holding
// split i's weight.
constexpr int kMaxSplits = 16;
template <typename T, int D>
__global__ __launch_bounds__(64) void qcache_merge_kernel(QAttnArgs a) {
  constexpr int E = D / 64;
  const int64_t w = blockIdx.x;
  const int hh = blockIdx.y, lane = threadIdx.x;
  const float2 ml = lane < a.splits ? a.part_ml[(w * a.G + hh) * a.splits + lane] : make_float2(-INFINITY, 0.f);
  float x[kMaxSplits][E];
#pragma unroll
  for (int i = 0; i < kMaxSplits; ++i) {
    if (i < a.splits) {
      const float* p = a.part_o + ((w * a.splits + i) * a.G + hh) * D + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) x[i][e] = p[e];
    }
  }
  float top = ml.x;
#pragma unroll
  for (int o = 1; o < kMaxSplits; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float ref = top == -INFINITY ? 0.f : top;
  const float f = fast_exp2(ml.x - ref);
  float ll = ml.y * f;
#pragma unroll
  for (int o = 1; o < kMaxSplits; o <<= 1) ll += __shfl_xor(ll, o);
  ll = __shfl(ll, 0);
  const float inv = ll == 0.f ? 0.f : 1.f / ll;
  float oo[E] = {};
#pragma unroll
  for (int i = 0; i < kMaxSplits; ++i) {
    if (i < a.splits) {
      const float fi = __shfl(f, i);
#pragma unroll
      for (int e = 0; e < E; ++e) oo[e] += x[i][e] * fi;
    }
  }
  const int bh = static_cast<int>(w % a.BH);
  const int row = a.row0 + static_cast<int>(w / a.BH);
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int64_t orow = (static_cast<int64_t>(b) * a.H + h * a.G + hh) * a.Nq + row;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if constexpr (sizeof(T) == 2)
      static_cast<uint16_t*>(a.o)[orow * D + lane * E + e] = f32_to_bf16_rne(oo[e] * inv);
    else
      static_cast<float*>(a.o)[orow * D + lane * E + e] = oo[e] * inv;
  }
  if (a.lse && lane == 0) a.lse[orow] = ll == 0.f ? -INFINITY : (ref + fast_log2(ll)) * kLn2;
}

namespace {

// How many wavefronts share a row's key units, NW of them in a workgroup and
// `splits` workgroups.  The device holds 2048 wavefronts of these kernels (two
// on each of 1024 SIMDs), so a row gets one per unit while that many fit, and
// never more than its share of 2048.  Up to 8 meet in one workgroup's LDS; more
// are spread over workgroups, since one CU takes about 50 GB/s, at the price of
// a second launch (16 units of 64 keys, d = 128, 8 rows: 2 x 8 7.3 us, 4 x 4 8.1,
// 8 x 2 9.3, all in one workgroup of 8 10.2; 64 units, 16 rows: 4 x 16 10.2,
// 4 x 4 15.5, 4 x 1 33).  With enough rows a wavefront takes a row alone and no
// states meet (16 units, 16384 rows: 1 361 us, 2 373, 4 403, 8 591).
struct Spread {
  int nw, splits;
};
Spread spread(const Shape& s, int ku) {
  const int64_t rows = static_cast<int64_t>(s.BH()) * s.Nq, units = static_cast<int64_t>(s.K) * (s.C / ku);
  int w = 1;
  while (w < units && w < 64 && 2 * w * rows <= 2048) w *= 2;
  if (w <= 8) return {w, 1};
  const int nw = w == 16 ? 2 : 4;
  return {nw, w / nw};
}

// Keys of a unit: 64 where the block allows it; with three terms of 128
// dimensions the registers hold 32.
int unit_keys(const Shape& s) { return s.C % 64 == 0 && (s.bf16 || s.D == 64) ? 64 : 32; }

template <typename T, int D, int KU, int NW>
hipError_t launch(const Shape& s, const QAttnArgs& a, hipStream_t st) {
  const size_t lds = static_cast<size_t>(NW) * s.G * (D + 2) * sizeof(float);  // 65 KB for 8 x 16 heads of 128
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(qcache_attn_kernel<T, D, KU, NW>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
    if (e != hipSuccess) return e;
  }
  // a launch's threads fit 32 bits; several rows per KV head in each (workgroup
  // w takes KV head w % BH, so that an XCD's workgroups share KV heads)
  const int most = std::max(1, (1 << 22) / s.BH());
  QAttnArgs c = a;
  for (c.row0 = 0; c.row0 < s.Nq; c.row0 += most) {
    const unsigned n = static_cast<unsigned>(std::min(most, s.Nq - c.row0)) * static_cast<unsigned>(s.BH());
    {
      ProfScope ps("qcache_attn", st);
      qcache_attn_kernel<T, D, KU, NW><<<dim3(n, a.splits), NW * 64, lds, st>>>(c);
    }
    if (a.splits > 1) {
      ProfScope ps("qcache_merge", st);
      qcache_merge_kernel<T, D><<<dim3(n, s.G), 64, 0, st>>>(c);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, int D, int KU>
hipError_t launch_nw(const Shape& s, const QAttnArgs& a, int nw, hipStream_t st) {
  switch (nw) {
    case 1: return launch<T, D, KU, 1>(s, a, st);
    case 2: return launch<T, D, KU, 2>(s, a, st);
    case 4: return launch<T, D, KU, 4>(s, a, st);
    default: return launch<T, D, KU, 8>(s, a, st);
  }
}

}  // namespace

static size_t part_ml_at(const Shape& s, int splits) {
  return (static_cast<size_t>(s.BH()) * s.Nq * splits * s.G * s.D * sizeof(float) + 255) & ~static_cast<size_t>(255);
}

size_t qcache_attn_ws(const Shape& s, const Geo&) {
  const int splits = spread(s, unit_keys(s)).splits;
  return splits > 1 ? part_ml_at(s, splits) + static_cast<size_t>(s.BH()) * s.Nq * splits * s.G * sizeof(float2) : 0;
}

hipError_t launch_qcache_attn(const Shape& s, const Geo& geo, const QCache& c, const void* q, const int32_t* idx, void* o,
                              float* lse, void* ws, hipStream_t st) {
  const int ku = unit_keys(s);
  const Spread sp = spread(s, ku);
  char* base = static_cast<char*>(ws);
  QAttnArgs a{c, q, idx, o, lse, reinterpret_cast<float*>(base), nullptr, s.H, s.Hkv, s.G, s.Nq, s.N, s.C, s.K, s.causal,
              geo.M[1], s.BH(), sp.splits, 0, kLog2e / sqrtf(static_cast<float>(s.D))};
  if (sp.splits > 1) a.part_ml = reinterpret_cast<float2*>(base + part_ml_at(s, sp.splits));
  if (s.bf16) {
    if (s.D == 128)
      return ku == 64 ? launch_nw<uint16_t, 128, 64>(s, a, sp.nw, st) : launch_nw<uint16_t, 128, 32>(s, a, sp.nw, st);
    return ku == 64 ? launch_nw<uint16_t, 64, 64>(s, a, sp.nw, st) : launch_nw<uint16_t, 64, 32>(s, a, sp.nw, st);
  }
  if (s.D == 128) return launch_nw<float, 128, 32>(s, a, sp.nw, st);
  return ku == 64 ? launch_nw<float, 64, 64>(s, a, sp.nw, st) : launch_nw<float, 64, 32>(s, a, sp.nw, st);
}

}  // namespace pisa
