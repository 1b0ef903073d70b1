// Loads, stores and angles of the rotary kernels (rope.hip, norm_rope.hip).
#pragma once

#include "common.h"
#include "kernels.h"

namespace pisa {

// 8 consecutive values from an address that may be aligned to the element only.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  T raw[8];
  __builtin_memcpy(raw, p, sizeof(raw));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(T) == 2) x[i] = bf16_to_f32(raw[i]);
    else x[i] = raw[i];
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint4 w = make_uint4(pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]), pack2_bf16(x[4], x[5]), pack2_bf16(x[6], x[7]));
    __builtin_memcpy(p, &w, 16);
  } else {
    __builtin_memcpy(p, x, 32);
  }
}

template <typename T>
__device__ __forceinline__ void store1(T* p, float x) {
  if constexpr (sizeof(T) == 2) *p = static_cast<T>(pack2_bf16(x, x));
  else *p = x;
}

// Cosine and sine, times the amplitude, of pairs p0 .. p0 + 7 (the last pair's for
// those behind it) of row n of batch b; how exact they are is said in rope.hip.
__device__ __forceinline__ void rope_angles(const RopeArgs& a, int b, int n, int p0, int pairs, float (&c)[8], float (&s)[8]) {
  const int64_t t = a.positions ? static_cast<int64_t>(a.positions[b * a.pos_bstride + n]) : static_cast<int64_t>(a.pos0) + n;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double turns = static_cast<double>(t) * a.turn[min(p0 + i, pairs - 1)];
    float sn, cs;
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &sn, &cs);
    c[i] = a.amplitude * cs;
    s[i] = a.amplitude * sn * a.sign;
  }
}

}  // namespace pisa
