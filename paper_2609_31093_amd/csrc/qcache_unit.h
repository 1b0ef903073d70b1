// Keys and values of the 8-bit cache as matrix operands (qcache_attn.hip,
// draft_attn.hip).
#pragma once

#include "attn_shared.h"
#include "common.h"
#include "kernels.h"

namespace pisa {

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

// Weights as the values' operands: fp16, or with NT = 3 bf16 terms, and four
// codes (unscaled) to go with them.
typedef _Float16 f16x2a __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8a __attribute__((ext_vector_type(8)));
__device__ __forceinline__ uint32_t pack2_f16(float a, float b) {
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2a));
}
template <int NT>
struct Weights {
  bf16x8a t[NT];
  __device__ __forceinline__ void set(const float (&p)[8]) { split_terms<NT>(p, t); }
  static __device__ __forceinline__ bf16x8a codes(uint32_t w0, uint32_t w1) { return codes8_bf16(w0, w1, 1.f); }
  __device__ __forceinline__ f32x4a times(bf16x8a v, f32x4a acc) const {
#pragma unroll
    for (int j = 0; j < NT; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, t[j], acc, 0, 0, 0);
    return acc;
  }
};
template <>
struct Weights<1> {
  f16x8a t;
  __device__ __forceinline__ void set(const float (&p)[8]) {
    t = __builtin_bit_cast(f16x8a, make_uint4(pack2_f16(p[0], p[1]), pack2_f16(p[2], p[3]), pack2_f16(p[4], p[5]), pack2_f16(p[6], p[7])));
  }
  static __device__ __forceinline__ uint2 codes4(uint32_t w) {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true)));
  }
  static __device__ __forceinline__ f16x8a codes(uint32_t w0, uint32_t w1) {
    const uint2 a = codes4(w0), b = codes4(w1);
    return __builtin_bit_cast(f16x8a, make_uint4(a.x, a.y, b.x, b.y));
  }
  __device__ __forceinline__ f32x4a times(f16x8a v, f32x4a acc) const {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(v, t, acc, 0, 0, 0);
  }
};

// Word w of codes at token `at`: those of tokens >= limit cleared.
__device__ __forceinline__ uint32_t keep_below(uint32_t w, int at, int limit) {
  const int n = limit - at;
  return n >= 4 ? w : n <= 0 ? 0u : w & ((1u << (8 * n)) - 1u);
}

// A key unit's codes and scales, as a wavefront's lanes hold them.
template <int D, int KU>
struct Unit {
  static constexpr int MT = KU / 16;  // key tiles
  static constexpr int DT = D / 16;   // dimension tiles of O
  static constexpr int KW = D / 16;   // words of a lane's part of a key (D/4 bytes)
  static constexpr int VW = KU / 16;  // words of a lane's part of a dimension (KU/4 tokens)
  uint32_t kw[MT][KW], vw[DT][VW];
  float ksc, vsc;

  __device__ __forceinline__ void load(const QCache& c, int64_t cell, int C, int u, int col, int grp) {
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
  }
  // Keeps the compiler from turning all codes into operands ahead of a loop,
  // which its registers could not hold.
  __device__ __forceinline__ void pin() {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int i = 0; i < KW; ++i) asm volatile("" : "+v"(kw[mt][i]));
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int i = 0; i < VW; ++i) asm volatile("" : "+v"(vw[dt][i]));
    }
  }
  // Clears the values' codes of tokens from `limit` on (0 times a NaN code would
  // not be 0).
  __device__ __forceinline__ void clear_from(int limit, int grp) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int i = 0; i < VW; ++i) vw[dt][i] = keep_below(vw[dt][i], grp * (KU / 4) + 4 * i, limit);
    }
  }
  __device__ __forceinline__ bf16x8a key(int mt, int ks) const { return codes8_bf16(kw[mt][2 * ks], kw[mt][2 * ks + 1], ksc); }
  template <int NT>
  __device__ __forceinline__ auto value(int st, int dt) const { return Weights<NT>::codes(vw[dt][2 * st], vw[dt][2 * st + 1]); }
  template <int NT>
  __device__ __forceinline__ auto value_below(int st, int dt, int limit, int grp) const {
    const int at = grp * (KU / 4) + 8 * st;
    return Weights<NT>::codes(keep_below(vw[dt][2 * st], at, limit), keep_below(vw[dt][2 * st + 1], at + 4, limit));
  }
  __device__ __forceinline__ bool nan_value() const {  // among any lane's values
    uint32_t any = 0;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int i = 0; i < VW; ++i) any |= ((vw[dt][i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    }
    return __any(any != 0);
  }
};

}  // namespace pisa
