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
  float* part;  // [rows][splits][G][D + 2]: unnormalised sums, maximum, sum (splits > 1)
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

// One workgroup of NW wavefronts per (row, KV head, split of its key units).
template <typename T, int D, int KU, int NW>
__global__ __launch_bounds__(NW * 64) void qcache_attn_kernel(QAttnArgs a) {
  constexpr int NT = sizeof(T) == 4 ? 3 : 1;  // bf16 terms of a query and of a weight
  constexpr int KS = D / 32;                  // k-steps of S
  constexpr int MT = KU / 16;                 // key tiles
  constexpr int DT = D / 16;                  // dimension tiles of O
  constexpr int KW = D / 16;                  // words of a lane's part of a key (D/4 bytes)
  constexpr int VW = KU / 16;                 // words of a lane's part of a dimension (KU/4 tokens)
  extern __shared__ __align__(16) float red[];  // [NW][G][D + 2]

  const int64_t w = blockIdx.x;
  const int bh = static_cast<int>(w % a.BH);
  const int row = a.row0 + static_cast<int>(w / a.BH);
  const int split = blockIdx.y;
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, grp = lane >> 4;
  const int t = a.N - a.Nq + row;
  const int32_t* sel = a.idx + (static_cast<int64_t>(bh) * a.Nq + row) * a.K;

  // queries: column col is head col, dimensions grp*D/4 .. +D/4-1
  bf16x8a qt[KS][NT];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    if (col < a.G)
      load_row_part<T, 8>(static_cast<const T*>(a.q) + ((static_cast<int64_t>(b) * a.H + h * a.G + col) * a.Nq + row) * D +
                              grp * (D / 4) + ks * 8, x);
    split_terms<NT>(x, qt[ks]);
  }

  float m = -INFINITY, l = 0.f;
  f32x4a oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x4a{0.f, 0.f, 0.f, 0.f};

  const int per = a.C / KU;  // key units of a block
  for (int task = split * NW + wave; task < a.K * per; task += a.splits * NW) {
    const int slot = task / per, u = task - slot * per;
    const int blk = __builtin_amdgcn_readfirstlane(sel[slot]);
    if (blk < 0 || blk >= a.M1) continue;
    const int tok0 = blk * a.C + u * KU;
    const int end = a.causal ? min(a.N, t + 1) : a.N;
    const int nkeys = min(KU, end - tok0);  // visible ones
    if (nkeys <= 0) continue;
    const int64_t cell = static_cast<int64_t>(bh) * a.c.M + blk;
    const uint8_t* kp = a.c.k + (cell * a.C + u * KU) * D + grp * (D / 4);
    const uint8_t* vp = a.c.v + cell * a.C * D + u * KU + grp * (KU / 4);
    uint32_t kw[MT][KW], vw[DT][VW];
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
      const uint8_t* p = vp + (dt * 16 + col) * a.C;
      if constexpr (VW == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        vw[dt][0] = x.x, vw[dt][1] = x.y, vw[dt][2] = x.z, vw[dt][3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        vw[dt][0] = x.x, vw[dt][1] = x.y;
      }
    }
    const float ksc = a.c.k_scale[cell], vsc = a.c.v_scale[cell];

    f32x4a s[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      s[mt] = f32x4a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8a kv = codes8_bf16(kw[mt][2 * ks], kw[mt][2 * ks + 1], ksc);
#pragma unroll
        for (int j = 0; j < NT; ++j) s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv, qt[ks][j], s[mt], 0, 0, 0);
      }
    }
    // lane (col, grp) holds keys grp*KU/4 + 4*mt + i; hidden ones: weight 0, and
    // their codes are cleared (0 times a NaN code would not be 0)
    const int k0 = grp * (KU / 4);
    if (nkeys < KU) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[mt][i] = k0 + 4 * mt + i < nkeys ? s[mt][i] : -INFINITY;
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
        for (int i = 0; i < VW; ++i) vw[dt][i] = keep_below(vw[dt][i], k0 + 4 * i, nkeys);
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[mt][i] *= a.qscale2;
        mx = fmaxf(mx, s[mt][i]);
      }
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float mn = fmaxf(m, mx);
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float corr = fast_exp2(m - ref);
    m = mn;
    float sum = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[mt][i] = fast_exp2(s[mt][i] - ref);
        sum += s[mt][i];
      }
    }
    l = l * corr + sum;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) oacc[dt][i] *= corr;
    }
#pragma unroll
    for (int st = 0; st < MT / 2; ++st) {
      const float p[8] = {s[2 * st][0], s[2 * st][1], s[2 * st][2], s[2 * st][3],
                          s[2 * st + 1][0], s[2 * st + 1][1], s[2 * st + 1][2], s[2 * st + 1][3]};
      bf16x8a pt[NT];
      split_terms<NT>(p, pt);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8a vv = codes8_bf16(vw[dt][2 * st], vw[dt][2 * st + 1], vsc);
#pragma unroll
        for (int j = 0; j < NT; ++j) oacc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pt[j], oacc[dt], 0, 0, 0);
      }
    }
  }
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
      float* p = a.part + ((w * a.splits + split) * a.G + hh) * W;
      p[dd] = oo;
      if (dd == 0) {
        p[D] = top;
        p[D + 1] = ll;
      }
    }
  }
}

// The splits' states of one row and KV head.
template <typename T, int D>
__global__ __launch_bounds__(256) void qcache_merge_kernel(QAttnArgs a) {
  constexpr int W = D + 2;
  const int64_t w = blockIdx.x;
  const int bh = static_cast<int>(w % a.BH);
  const int row = a.row0 + static_cast<int>(w / a.BH);
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  for (int e = threadIdx.x; e < a.G * D; e += 256) {
    const int hh = e / D, dd = e - hh * D;
    const float* p = a.part + (w * a.splits * a.G + hh) * W;
    float top = -INFINITY;
    for (int i = 0; i < a.splits; ++i) top = fmaxf(top, p[static_cast<int64_t>(i) * a.G * W + D]);
    const float ref = top == -INFINITY ? 0.f : top;
    float ll = 0.f, oo = 0.f;
    for (int i = 0; i < a.splits; ++i) {
      const float* r = p + static_cast<int64_t>(i) * a.G * W;
      const float f = fast_exp2(r[D] - ref);
      ll += r[D + 1] * f;
      oo += r[dd] * f;
    }
    const int64_t orow = (static_cast<int64_t>(b) * a.H + h * a.G + hh) * a.Nq + row;
    const float res = ll == 0.f ? 0.f : oo / ll;
    if constexpr (sizeof(T) == 2)
      static_cast<uint16_t*>(a.o)[orow * D + dd] = f32_to_bf16_rne(res);
    else
      static_cast<float*>(a.o)[orow * D + dd] = res;
    if (a.lse && dd == 0) a.lse[orow] = ll == 0.f ? -INFINITY : (ref + fast_log2(ll)) * kLn2;
  }
}

namespace {

constexpr int kQWaves = 4;

int qcache_splits(const Shape& s) {
  (void)s;
  return 1;
}

template <typename T, int D, int KU>
hipError_t launch(const Shape& s, const QAttnArgs& a, hipStream_t st) {
  const size_t lds = static_cast<size_t>(kQWaves) * s.G * (D + 2) * sizeof(float);
  // a launch's threads fit 32 bits; several rows per KV head in each (workgroup
  // w takes KV head w % BH, so that an XCD's workgroups share KV heads)
  const int most = std::max(1, (1 << 22) / s.BH());
  QAttnArgs c = a;
  for (c.row0 = 0; c.row0 < s.Nq; c.row0 += most) {
    const unsigned n = static_cast<unsigned>(std::min(most, s.Nq - c.row0)) * static_cast<unsigned>(s.BH());
    {
      ProfScope ps("qcache_attn", st);
      qcache_attn_kernel<T, D, KU, kQWaves><<<dim3(n, a.splits), kQWaves * 64, lds, st>>>(c);
    }
    if (a.splits > 1) {
      ProfScope ps("qcache_merge", st);
      qcache_merge_kernel<T, D><<<n, 256, 0, st>>>(c);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t launch_t(const Shape& s, const QAttnArgs& a, hipStream_t st) {
  if (s.D == 128) return s.C % 64 == 0 ? launch<T, 128, 64>(s, a, st) : launch<T, 128, 32>(s, a, st);
  return s.C % 64 == 0 ? launch<T, 64, 64>(s, a, st) : launch<T, 64, 32>(s, a, st);
}

}  // namespace

size_t qcache_attn_ws(const Shape& s, const Geo&) {
  const int splits = qcache_splits(s);
  return splits > 1 ? static_cast<size_t>(s.BH()) * s.Nq * splits * s.G * (s.D + 2) * sizeof(float) : 0;
}

hipError_t launch_qcache_attn(const Shape& s, const Geo& geo, const QCache& c, const void* q, const int32_t* idx, void* o,
                              float* lse, void* ws, hipStream_t st) {
  QAttnArgs a{c, q, idx, o, lse, static_cast<float*>(ws), s.H, s.Hkv, s.G, s.Nq, s.N, s.C, s.K, s.causal, geo.M[1],
              s.BH(), qcache_splits(s), 0, kLog2e / sqrtf(static_cast<float>(s.D))};
  return s.bf16 ? launch_t<uint16_t>(s, a, st) : launch_t<float>(s, a, st);
}

}  // namespace pisa
