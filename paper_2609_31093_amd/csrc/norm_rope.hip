// Root-mean-square norms of queries and keys, head by head, with their rotary
// positions in the same pass, and the gradients of both.
//
//   r = 1 / sqrt(mean(x^2) + eps),  y = R (x r w)
// with w the learned weights (plus an offset) and R the rotation of rope.hip.
// With u = R^T dy (R^T turns back and has the same amplitude):
//   dw = sum over rows and heads of u x r
//   dx = r (u w - x r mean(u w x r))
//
// d/16 lanes share a row; each holds 16 of its values, two runs of 8 (`lo`, `hi`),
// among them both values of each of its pairs, so that the rotation stays in the
// lane and the sums over the head are three (two) exchanges between neighbours.
// Everything is held in fp32 and rounded once.  Each value is read once and
// written once, which bounds the kernels: 131072 rows of 16 heads of 128 in bf16 take
// 189 to 192 us (5.6 TB/s; a copy has 5.2; workgroups that go on to other rows 208 with 4096
// of them), gradients of 30011 rows of 20 heads 100 us (4.6 TB/s, 3 us of it the
// weights' sums).
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "rope_shared.h"

namespace pisa {

namespace {

// How pairs lie: (2i, 2i + 1); (i, i + pairs) with a lane's all before or all behind the
// border of what is rotated, 16 dimensions of lane u from 16 u on behind it; and the
// same with the border among a lane's pairs (pairs no multiple of 8).
constexpr int kPairs = 0, kHalves = 1, kMixed = 2;

bool mixed_pairs(bool half, int rot) { return half && rot % 16 != 0; }

// Where a lane's values are: dimensions lo .. lo + 7 and hi .. hi + 7.  The lane with
// the border (kMixed) has r < 8 pairs; its `hi` runs on into the dimensions behind the
// rotated ones, and its `lo` has from value r on those that follow, lo2 + r ...
// lo2 + 7.  So three runs are loaded and one value chosen from two (131072 rows of 16
// heads: 308 us, 192 without a border; each value loaded on its own 782).
template <int LAY>
struct Slots {
  int lo, hi, lo2, r, p0;

  __device__ __forceinline__ Slots(int u, int pairs) : lo(16 * u), hi(16 * u + 8), lo2(16 * u), r(8), p0(8 * u) {
    if (LAY != kPairs && p0 < pairs) {
      lo = lo2 = p0;
      hi = p0 + pairs;
      if (LAY == kMixed && p0 + 8 > pairs) {
        r = pairs - p0;
        lo2 = 2 * pairs + 8 - 2 * r;
      }
    }
  }
  __device__ __forceinline__ int lo_at(int j) const { return (LAY == kMixed && j >= r ? lo2 : lo) + j; }
  __device__ __forceinline__ int hi_at(int j) const { return hi + j; }
};

template <int LAY, typename T>
__device__ __forceinline__ void load16(const T* p, const Slots<LAY>& s, float (&lo)[8], float (&hi)[8]) {
  load8(p + s.lo, lo);
  load8(p + s.hi, hi);
  if constexpr (LAY == kMixed) {
    float more[8];
    load8(p + s.lo2, more);
#pragma unroll
    for (int j = 0; j < 8; ++j) lo[j] = j < s.r ? lo[j] : more[j];
  }
}
template <int LAY, typename T>
__device__ __forceinline__ void store16(T* p, const Slots<LAY>& s, const float (&lo)[8], const float (&hi)[8]) {
  store8(p + s.hi, hi);
  if (LAY != kMixed || s.r == 8) {
    store8(p + s.lo, lo);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) store1(p + s.lo_at(j), lo[j]);
  }
}

__device__ __forceinline__ void turn2(float& x, float& y, float c, float s) {
  const float a = x, b = y;
  x = a * c - b * s;
  y = b * c + a * s;
}
template <int LAY>
__device__ __forceinline__ void turn(float (&lo)[8], float (&hi)[8], const float (&c)[8], const float (&s)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (LAY != kPairs) turn2(lo[j], hi[j], c[j], s[j]);
    else if (j < 4) turn2(lo[2 * j], lo[2 * j + 1], c[j], s[j]);
    else turn2(hi[2 * j - 8], hi[2 * j - 7], c[j], s[j]);
  }
}

// Sum over the lanes of a row.
template <int UNITS>
__device__ __forceinline__ float row_sum(float v) {
  v += dpp_f<0xB1>(v);                              // quad_perm [1,0,3,2]
  v += dpp_f<0x4E>(v);                              // quad_perm [2,3,0,1]
  if constexpr (UNITS == 8) v += dpp_f<0x141>(v);   // row_half_mirror
  return v;
}

// Weights of a lane's values (1 where there are none).
template <int LAY>
__device__ __forceinline__ void load_weights(const NormArgs& m, const void* w, const Slots<LAY>& s, float (&lo)[8], float (&hi)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) lo[j] = hi[j] = 1.f;
  if (!w) return;
  if (m.w_bf16) load16<LAY>(static_cast<const uint16_t*>(w), s, lo, hi);
  else load16<LAY>(static_cast<const float*>(w), s, lo, hi);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo[j] += m.offset;
    hi[j] += m.offset;
  }
}

// The heads of workgroup column y: `heads` of the queries', or of the keys'.
struct HeadRange {
  bool is_q;
  int first, end;
};
__device__ __forceinline__ HeadRange heads_of(const RopeArgs& a, int y) {
  const int gq = (a.H + a.heads - 1) / a.heads, Hkv = a.HH - a.H;
  const bool is_q = y < gq;
  const int first = (is_q ? y : y - gq) * a.heads;
  return {is_q, first, min(first + a.heads, is_q ? a.H : Hkv)};
}

template <typename T>
__device__ __forceinline__ const T* row_in(const RopeSide& io, int b, int h, int n) {
  return static_cast<const T*>(io.in) + b * io.ib + h * io.ih + n * io.in_n;
}
template <typename T>
__device__ __forceinline__ T* row_out(const RopeSide& io, int b, int h, int n) {
  return static_cast<T*>(io.out) + b * io.ob + h * io.oh + n * io.on;
}

// Angles of a lane's pairs; those behind the border turn by nothing.
__device__ __forceinline__ void lane_angles(const RopeArgs& a, int b, int n, int p0, int pairs, float (&c)[8], float (&s)[8]) {
  rope_angles(a, b, n, p0, pairs, c, s);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    c[j] = p0 + j < pairs ? c[j] : 1.f;
    s[j] = p0 + j < pairs ? s[j] : 0.f;
  }
}

}  // namespace

// Workgroups (rows, heads): 256 threads take 256 / UNITS rows; bf16 kMixed ones go on to
// others.
template <typename T, int D, int LAY>
__global__ __launch_bounds__(256) void norm_rope_kernel(RopeArgs a, NormArgs m) {
  constexpr int UNITS = D / 16, ROWS = 256 / UNITS;
  const int u = threadIdx.x % UNITS, pairs = a.rot / 2;
  const Slots<LAY> at(u, pairs);
  const HeadRange heads = heads_of(a, blockIdx.y);
  const RopeSide& io = heads.is_q ? a.q : a.k;
  float wlo[8], whi[8];
  load_weights<LAY>(m, heads.is_q ? m.q_weight : m.k_weight, at, wlo, whi);
  int row = static_cast<int>(blockIdx.x) * ROWS + threadIdx.x / UNITS;
  if (row >= a.B * a.N) return;
  do {
    const int b = row / a.N, n = row - b * a.N;
    float c[8], s[8];
    lane_angles(a, b, n, 8 * u, pairs, c, s);
    for (int h = heads.first; h < heads.end; ++h) {
      float lo[8], hi[8];
      load16<LAY>(row_in<T>(io, b, h, n), at, lo, hi);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += lo[j] * lo[j] + hi[j] * hi[j];
      const float r = rsqrtf(row_sum<UNITS>(sum) * (1.f / D) + m.eps);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        lo[j] = lo[j] * r * wlo[j];  // (r w may be past fp32's range where x r w is not)
        hi[j] = hi[j] * r * whi[j];
      }
      turn<LAY>(lo, hi, c, s);
      store16<LAY>(row_out<T>(io, b, h, n), at, lo, hi);
    }
  } while (LAY == kMixed && sizeof(T) == 2 && (row += static_cast<int>(gridDim.x) * ROWS) < a.B * a.N);
}

// A lane's 16 values of a row as they lie in memory.
template <typename T, int LAY>
struct Raw16 {
  static constexpr int W = 2 * sizeof(T), V = 4 / sizeof(T);  // words of 8 values, values of a word
  uint32_t lo[W], hi[W], more[LAY == kMixed ? W : 1];
  __device__ __forceinline__ void load(const T* p, const Slots<LAY>& s) {
    __builtin_memcpy(lo, p + s.lo, sizeof(lo));
    __builtin_memcpy(hi, p + s.hi, sizeof(hi));
    if constexpr (LAY == kMixed) __builtin_memcpy(more, p + s.lo2, sizeof(more));
  }
  static __device__ __forceinline__ float at(uint32_t w, int j) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w);
    else return __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
  }
  __device__ __forceinline__ void values(const Slots<LAY>& s, float (&x)[8], float (&y)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = at(lo[j / V], j);
      y[j] = at(hi[j / V], j);
      if constexpr (LAY == kMixed) x[j] = j < s.r ? x[j] : at(more[j / V], j);
    }
  }
};

// Workgroups of the gradients that a CU holds at once, by their registers (four spill).
constexpr int held(bool bf16, bool mixed) { return bf16 && !mixed ? 3 : 2; }

// The next head's values are on their way while one is worked on (without: 139 us for
// 30011 rows of 20 heads, with 95), which takes the registers of held() wavefronts on a
// SIMD.  The weights'
// gradients: each thread sums its rows', then the workgroup's meet in LDS, and
// norm_rope_weights_kernel adds the workgroups' in their order.
template <typename T, int D, int LAY>
__global__ __launch_bounds__(256, held(sizeof(T) == 2, LAY == kMixed)) void norm_rope_bwd_kernel(RopeArgs a, NormArgs m,
                                                                                              RopeSide dq, RopeSide dk) {
  constexpr int UNITS = D / 16, ROWS = 256 / UNITS;
  __shared__ float part[4][D];
  const int u = threadIdx.x % UNITS, pairs = a.rot / 2;
  const Slots<LAY> at(u, pairs);
  const HeadRange heads = heads_of(a, blockIdx.y);
  const RopeSide& io = heads.is_q ? a.q : a.k;   // in: x
  const RopeSide& gr = heads.is_q ? dq : dk;     // in: dy, out: dx
  float wlo[8], whi[8], dlo[8], dhi[8], c[8], s[8];
  load_weights<LAY>(m, heads.is_q ? m.q_weight : m.k_weight, at, wlo, whi);
#pragma unroll
  for (int j = 0; j < 8; ++j) dlo[j] = dhi[j] = 0.f;
  const int rows = a.B * a.N, step = static_cast<int>(gridDim.x) * ROWS;
  int row = static_cast<int>(blockIdx.x) * ROWS + threadIdx.x / UNITS, h = heads.first;
  int b = row / a.N, n = row - b * a.N;
  Raw16<T, LAY> x0, u0, x1, u1;

  // works on row `row`, head h, and moves on to the next ones
  auto pass = [&](const Raw16<T, LAY>& xr, const Raw16<T, LAY>& ur, Raw16<T, LAY>& xn, Raw16<T, LAY>& un) {
    if (h == heads.first) lane_angles(a, b, n, 8 * u, pairs, c, s);
    T* out = row_out<T>(gr, b, h, n);
    if (++h == heads.end) {
      h = heads.first;
      row += step;
      b = row / a.N;
      n = row - b * a.N;
    }
    if (row < rows) {
      xn.load(row_in<T>(io, b, h, n), at);
      un.load(row_in<T>(gr, b, h, n), at);
    }
    float lo[8], hi[8], ulo[8], uhi[8];
    xr.values(at, lo, hi);
    ur.values(at, ulo, uhi);
    turn<LAY>(ulo, uhi, c, s);
    float sum = 0.f, dot = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += lo[j] * lo[j] + hi[j] * hi[j];
    const float r = rsqrtf(row_sum<UNITS>(sum) * (1.f / D) + m.eps);
#pragma unroll
    for (int j = 0; j < 8; ++j) {  // (u w x may be past fp32's range where u w x r is not)
      lo[j] *= r;
      hi[j] *= r;
      dot += ulo[j] * wlo[j] * lo[j] + uhi[j] * whi[j] * hi[j];
    }
    const float along = row_sum<UNITS>(dot) * (1.f / D);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dlo[j] = fmaf(ulo[j], lo[j], dlo[j]);
      dhi[j] = fmaf(uhi[j], hi[j], dhi[j]);
      lo[j] = r * (ulo[j] * wlo[j] - lo[j] * along);
      hi[j] = r * (uhi[j] * whi[j] - hi[j] * along);
    }
    store16<LAY>(out, at, lo, hi);
  };
  if (row < rows) {
    x0.load(row_in<T>(io, b, h, n), at);
    u0.load(row_in<T>(gr, b, h, n), at);
  }
  while (row < rows) {
    pass(x0, u0, x1, u1);
    if (row >= rows) break;
    pass(x1, u1, x0, u0);
  }

  if (!(heads.is_q ? m.d_q_weight : m.d_k_weight)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int o = UNITS; o < 64; o <<= 1) {
      dlo[j] += __shfl_xor(dlo[j], o);
      dhi[j] += __shfl_xor(dhi[j], o);
    }
    if (lane < UNITS) {
      part[wave][at.lo_at(j)] = dlo[j];
      part[wave][at.hi_at(j)] = dhi[j];
    }
  }
  __syncthreads();
  if (threadIdx.x < D) {
    const int e = threadIdx.x;
    m.parts[(static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * D + e] =
        (part[0][e] + part[1][e]) + (part[2][e] + part[3][e]);
  }
}

// Sums of the parts: a workgroup for 16 dimensions of a side, 256 threads for each
// four of them, whose loads are four at a time on their way.
template <int D>
__global__ __launch_bounds__(1024) void norm_rope_weights_kernel(const float* __restrict__ parts, int nq, int nk, float* d_q,
                                                                 float* d_k) {
  __shared__ float4 sums[256][4];
  const bool is_q = blockIdx.y == 0;
  float* out = is_q ? d_q : d_k;
  if (!out) return;
  const int quad = threadIdx.x & 3, t = threadIdx.x >> 2, n = is_q ? nq : nk;
  const float* p = parts + (is_q ? 0 : static_cast<int64_t>(nq) * D) + blockIdx.x * 16 + quad * 4;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = t; i < n; i += 1024) {
    float4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const float4*>(p + static_cast<int64_t>(min(i + 256 * j, n - 1)) * D);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i + 256 * j < n) v.x += x[j].x, v.y += x[j].y, v.z += x[j].z, v.w += x[j].w;
    }
  }
  sums[t][quad] = v;
  for (int o = 128; o >= 1; o >>= 1) {
    __syncthreads();
    if (t < o) {
      const float4 x = sums[t + o][quad];
      v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
      sums[t][quad] = v;
    }
  }
  if (t == 0) *reinterpret_cast<float4*>(out + blockIdx.x * 16 + quad * 4) = v;
}

namespace {

// Workgroups of a pass: heads to a workgroup and workgroups along the rows.
struct Grid {
  int heads, gx, gq, gk;
};
Grid grid_of(int B, int N, int H, int Hkv, int d, bool bf16, bool mixed, bool bwd) {
  const int64_t rows = static_cast<int64_t>(B) * N, groups = (rows * (d / 16) + 255) / 256;
  Grid g{};
  g.heads = groups * (H + Hkv) >= 4 * 1024 ? 4 : groups * (H + Hkv) >= 2 * 1024 ? 2 : 1;
  g.gq = (H + g.heads - 1) / g.heads;
  g.gk = (Hkv + g.heads - 1) / g.heads;
  g.gx = static_cast<int>(groups);
  // gradients: as few workgroups (and parts of the weights' sums) as the device holds
  // at once, each the same number of rows (20 heads at 30011 rows, bf16: 640 workgroups
  // 108 us, 768 100, 1024 110, 4096 109; kMixed 512 130 us, 768 136)
  if (bwd) {
    const int64_t most = 256 * held(bf16, mixed), rounds = (groups * (g.gq + g.gk) + most - 1) / most;
    g.gx = static_cast<int>((groups + rounds - 1) / rounds);
  } else if (mixed && bf16) {
    // workgroups that go on to other rows (131072 rows of 16 heads: 308 us, with a row to
    // a lane group 334; fp32 710 and 706)
    g.gx = static_cast<int>(std::min<int64_t>(groups, std::max(1, 4096 / (g.gq + g.gk))));
  }
  return g;
}

template <typename T, int D, int LAY>
hipError_t launch(const RopeArgs& a, const NormArgs& m, const RopeSide* dq, const RopeSide* dk, const Grid& g, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(g.gx), static_cast<unsigned>(g.gq + g.gk));
  if (!dq) {
    ProfScope ps("norm_rope", st);
    norm_rope_kernel<T, D, LAY><<<grid, 256, 0, st>>>(a, m);
    return hipGetLastError();
  }
  {
    ProfScope ps("norm_rope_bwd", st);
    norm_rope_bwd_kernel<T, D, LAY><<<grid, 256, 0, st>>>(a, m, *dq, *dk);
  }
  if (m.d_q_weight || m.d_k_weight) {
    ProfScope ps("norm_rope_weights", st);
    norm_rope_weights_kernel<D><<<dim3(D / 16, 2), 1024, 0, st>>>(m.parts, g.gx * g.gq, g.gx * g.gk, m.d_q_weight, m.d_k_weight);
  }
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_layout(const RopeArgs& a, const NormArgs& m, const RopeSide* dq, const RopeSide* dk, const Grid& g, bool half,
                         hipStream_t st) {
  if (!half) return launch<T, D, kPairs>(a, m, dq, dk, g, st);
  return !mixed_pairs(half, a.rot) ? launch<T, D, kHalves>(a, m, dq, dk, g, st) : launch<T, D, kMixed>(a, m, dq, dk, g, st);
}

}  // namespace

size_t norm_rope_bwd_ws(int B, int N, int H, int Hkv, int d, int rot, bool bf16, bool half) {
  const Grid g = grid_of(B, N, H, Hkv, d, bf16, mixed_pairs(half, rot), true);
  return static_cast<size_t>(g.gx) * (g.gq + g.gk) * d * sizeof(float);
}

hipError_t launch_norm_rope(const RopeArgs& args, const NormArgs& m, const RopeSide* dq, const RopeSide* dk, bool bf16, bool half,
                            hipStream_t st) {
  RopeArgs a = args;
  const Grid g = grid_of(a.B, a.N, a.H, a.HH - a.H, a.d, bf16, mixed_pairs(half, a.rot), dq != nullptr);
  a.heads = g.heads;
  if (bf16)
    return a.d == 128 ? launch_layout<uint16_t, 128>(a, m, dq, dk, g, half, st) : launch_layout<uint16_t, 64>(a, m, dq, dk, g, half, st);
  return a.d == 128 ? launch_layout<float, 128>(a, m, dq, dk, g, half, st) : launch_layout<float, 64>(a, m, dq, dk, g, half, st);
}

}  // namespace pisa
