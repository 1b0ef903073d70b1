// Rotary positions of queries and keys, and their gradients.
//
// Pair (a, b) of a row at position t becomes amplitude * (a cos - b sin,
// b cos + a sin) with the angle t * freq; the gradient is the transposed map,
// the same with -sin.  A thread owns 8 pairs of one (batch, row) and walks the
// heads with one set of sines, so the angles cost little and the kernel is bound
// by reading and writing each value once (1.07 GB in 192 us, 5.6 TB/s, where a
// large copy moves 4.9).
//
// The angle is taken in turns: t * (freq / 2 pi) in 64 bits, its fraction in
// 32.  Position 2^20 times a frequency of 1 would lose 2^-4 radians in 32 bits;
// here the fraction is off by at most 2^-26 turns, and by 2^-51 of all the turns
// (2^-28 after 2^23 of them) that the roundings in 64 bits leave.  With 32 bits
// the sines stay 32-bit ones; fp32 results are then 5.6e-8 from the exact ones
// (relative, 8192 positions from 2^20 on), where 64-bit sines leave 4.2e-8.
#include "common.h"
#include "kernels.h"

namespace pisa {

namespace {

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

}  // namespace

template <typename T, bool HALF>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  const int units = a.d / 16;  // threads of a row
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t row = at / units;
  const int u = static_cast<int>(at - row * units);
  if (row >= static_cast<int64_t>(a.B) * a.N) return;
  const int b = static_cast<int>(row / a.N), n = static_cast<int>(row - static_cast<int64_t>(b) * a.N);
  const int pairs = a.rot / 2;

  float c[8], s[8];
  const int64_t t = a.positions ? static_cast<int64_t>(a.positions[b * a.pos_bstride + n]) : static_cast<int64_t>(a.pos0) + n;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double turns = static_cast<double>(t) * a.turn[min(8 * u + i, pairs - 1)];
    float sn, cs;
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &sn, &cs);
    c[i] = a.amplitude * cs;
    s[i] = a.amplitude * sn * a.sign;
  }

  const int h1 = min(a.HH, (static_cast<int>(blockIdx.y) + 1) * a.heads);
  for (int hh = blockIdx.y * a.heads; hh < h1; ++hh) {
    const bool is_q = hh < a.H;
    const RopeSide& io = is_q ? a.q : a.k;
    const int h = is_q ? hh : hh - a.H;
    const T* src = static_cast<const T*>(io.in) + b * io.ib + h * io.ih + n * io.in_n;
    T* dst = static_cast<T*>(io.out) + b * io.ob + h * io.oh + n * io.on;
    if constexpr (HALF) {
      // pairs (i, i + rot/2): two runs of 8 values, the second aligned to the
      // element only where rot/2 is no multiple of 8
      if (8 * u < pairs) {
        float x[8], y[8], p[8], q[8];
        load8(src + 8 * u, x);  // within the row: 8u + 7 < d / 2
        load8(src + pairs + 8 * u, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = x[i] * c[i] - y[i] * s[i];
          q[i] = y[i] * c[i] + x[i] * s[i];
        }
        if (8 * u + 8 <= pairs) {
          store8(dst + 8 * u, p);
          store8(dst + pairs + 8 * u, q);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (8 * u + i < pairs) {
              store1(dst + 8 * u + i, p[i]);
              store1(dst + pairs + 8 * u + i, q[i]);
            }
          }
        }
      }
      for (int e = a.rot + u; e < a.d; e += units) dst[e] = src[e];
    } else {
      // pairs (2i, 2i + 1): 16 values of its own per thread
      float x[8], y[8];
      load8(src + 16 * u, x);
      load8(src + 16 * u + 8, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (8 * u + i < pairs) {
          const float x0 = x[2 * i], x1 = x[2 * i + 1];
          x[2 * i] = x0 * c[i] - x1 * s[i];
          x[2 * i + 1] = x1 * c[i] + x0 * s[i];
        }
        if (8 * u + 4 + i < pairs) {
          const float y0 = y[2 * i], y1 = y[2 * i + 1];
          y[2 * i] = y0 * c[4 + i] - y1 * s[4 + i];
          y[2 * i + 1] = y1 * c[4 + i] + y0 * s[4 + i];
        }
      }
      store8(dst + 16 * u, x);
      store8(dst + 16 * u + 8, y);
    }
  }
}

hipError_t launch_rope(const RopeArgs& args, bool bf16, bool half, hipStream_t st) {
  RopeArgs a = args;
  const int64_t threads = static_cast<int64_t>(a.B) * a.N * (a.d / 16);
  // One set of sines serves 4 heads where that leaves 1024 workgroups, four on
  // each CU (16 heads at 131072 rows of 128 in bf16: 1 head a thread 232 us, 2
  // 188, 4 192, all 204; 20 heads at 30011 rows, written back into rows of 20
  // heads: 75, 66, 63, 68), fewer with fewer rows (4 heads at 4099 rows of 64 in
  // fp32, 256 workgroups at one head: 5.4, 5.3, 6.5; one row: 3.3, 3.6, 4.2).
  const int64_t groups = (threads + 255) / 256 * a.HH;
  a.heads = groups >= 4 * 1024 ? 4 : groups >= 2 * 1024 ? 2 : 1;
  const dim3 grid(static_cast<unsigned>((threads + 255) / 256), static_cast<unsigned>((a.HH + a.heads - 1) / a.heads));
  ProfScope ps("rope", st);
  if (bf16) {
    if (half)
      rope_kernel<uint16_t, true><<<grid, 256, 0, st>>>(a);
    else
      rope_kernel<uint16_t, false><<<grid, 256, 0, st>>>(a);
  } else {
    if (half)
      rope_kernel<float, true><<<grid, 256, 0, st>>>(a);
    else
      rope_kernel<float, false><<<grid, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace pisa
