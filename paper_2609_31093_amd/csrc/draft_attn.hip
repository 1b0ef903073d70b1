// Attention of drafted tokens over their selected blocks of a cache and over each
// other, as a tree's mask has it.
//
// A wavefront's 16 matrix columns are the G query heads of 16 / G drafted tokens of
// one KV head.  Tokens of one tree look for nearly the same blocks, so a workgroup
// first makes the list of the blocks that any of its rows selected, and its
// wavefronts walk that list: a block is read and multiplied once for all rows, and
// the columns whose row did not select it are masked.  (16 tokens of one head, 16
// blocks each: 50 blocks together, not 256.)
//
// The products are those of qcache_attn.hip:
//   S^T = K q^T      row r of key tile mt is key (r/4) (KU/4) + 4 mt + r%4 of the unit,
//                    so that lane group grp gets the logits of KU/4 consecutive keys
//   O^T += V^T P^T   over those keys.  Row r of dimension tile dt is dimension
//                    r D/16 + dt: a lane then needs D/16 consecutive values of each of
//                    its keys, 16 lanes a whole row, and turns eight keys' values into
//                    operands by itself (a byte permutation for two of them); 8-bit
//                    values lie by dimension already.
// Keys, and the 8-bit values, go through the wavefront's own LDS (KeyRows), the next
// unit's being loaded meanwhile.  The drafted rows, and a bf16 cache, are units of 32
// keys on v_mfma_f32_16x16x32_bf16 (weights as two bf16 terms); fp32 ones take
// v_mfma_f32_16x16x4_f32, whose operands are one value a lane.  The 8-bit cache is
// multiplied as qcache_attn.hip does it, with two fp16 terms of a weight.
//
// What bounds it: few tokens the chain of latencies (the list 1.2 us, a unit's loads
// 1.5 and products 1.6, the wavefronts' sums 1.2; 11.0 us with the second launch for 16
// tokens of 8 heads over 131071 in 8 bits); many a unit's vector instructions, half of
// them conversions and the sums' rescaling, and what two wavefronts to a SIMD leave
// unhidden of its waits (256 tokens of 8 heads on 2 over 523776: 37.1 us, in which the
// two issue vector instructions in 54% of a SIMD's cycles and each waits in 37% of its
// own; with operands straight from the cache, whose scattered pieces a CU takes in at 13
// bytes a clock, 48 before the weights' second term).
//
// The running maximum is that of the products before the softmax's scale.  Sums of
// weights times values are held in units of kUnit, so that values up to the type's
// largest do not overflow before they are divided (values below 2^-109 lose bits).
#include <algorithm>
#include <atomic>

#include "attn_shared.h"
#include "common.h"
#include "kernels.h"
#include "qcache_unit.h"

namespace pisa {

namespace {

struct DraftAttnArgs {
  QCache c;             // 8-bit
  const void *k, *v;    // otherwise [BH, Nkv, D]
  const void *k_new, *v_new;
  int64_t ksb, ksh, ksn, vsb, vsh, vsn;  // strides of the drafted rows, in elements
  const uint64_t* mask;
  int64_t mask_bstride;
  const void* q;
  const int32_t* idx;
  void* o;
  float* lse;
  // splits > 1: unnormalised sums [tiles][BH][splits][columns][D], and the largest
  // logit and sum of weights [tiles][BH][columns][splits]
  float* part_o;
  float2* part_ml;
  int H, Hkv, G, T, n, C, K, Nkv;
  int M;               // blocks of the n cached tokens
  int R;               // rows of a tile
  int KS;              // wavefronts of a workgroup
  int W;               // words of a mask row
  int BH, splits;
  int tile0;           // first tile of this launch
  int list;            // entries of the block list, at most
  float qscale2;
};

// log2 of the largest weight: fp16 weights (bf16 queries on 8-bit values) are taken up
// to 2^14, so that ones of 2^-28 of the largest are still normal numbers.
template <typename T, bool Q8>
constexpr float kHead = !Q8 ? -16.f : sizeof(T) == 2 ? 14.f : 0.f;
// What weights are multiplied by besides, so that they add up to less than 1 (a row has
// less than 2^16 tokens).
template <typename T, bool Q8>
constexpr float kUnit = !Q8 ? 1.f : sizeof(T) == 2 ? 0x1p-30f : 0x1p-16f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A value at a wavefront's address plus a lane's offset, which the load adds by itself.
template <typename V>
__device__ __forceinline__ V value_at(const void* base, uint32_t off) {
  return *reinterpret_cast<const V*>(static_cast<const char*>(base) + off);
}
// Row strides up to which a unit's rows are within a 32-bit offset.
constexpr int64_t kNear = 1 << 24;

// Key rows of RB bytes on their way to matrix operands.  An operand's lane holds a part
// of one key's row, 16 lanes 16 rows: loaded like that, each lane's 16 bytes are a
// request of their own and a CU takes in 13 bytes a clock.  So a wavefront loads 1 KB in
// a row, puts it into its own LDS and reads operands from there; a row's pieces are
// placed so that 8 lanes' reads of 8 rows, as operand() makes them, meet 8 banks.
template <int RB, int KU>
struct KeyRows {
  static constexpr int NP = RB / 16, NL = KU * NP / 64, BYTES = KU * RB;
  u32x4 r[NL];

  // Piece p of a row is at place p ^ turn(row) of it.
  static __device__ __forceinline__ int turn(int row) {
    const int run = (row / (KU / 4)) & 1;
    return NP >= 8 ? (row & 3) | run << 2 : ((row >> 1) & 1) | run << 1;
  }
  // ptr(i): row i of the unit
  template <typename F>
  __device__ __forceinline__ void load(F ptr, int lane) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int n = i * 64 + lane;
      r[i] = reinterpret_cast<const u32x4*>(ptr(n / NP))[n % NP];
    }
  }
  // rows 0 .. KU - 1, `stride` bytes from one to the next
  __device__ __forceinline__ void load_all(const void* base, uint32_t stride, int lane) {
    const uint32_t off = lane / NP * stride + lane % NP * 16;
#pragma unroll
    for (int i = 0; i < NL; ++i) r[i] = value_at<u32x4>(static_cast<const char*>(base) + i * (64 / NP) * stride, off);
  }
  // (Load i has rows i 64/NP + lane/NP, whose turns differ from lane/NP's in bits that
  // depend on i alone.)
  __device__ __forceinline__ void stage(u32x4* lds, int lane) const {
    const int first = lane ^ turn(lane / NP);
#pragma unroll
    for (int i = 0; i < NL; ++i) lds[i * 64 + (first ^ turn(i * (64 / NP)))] = r[i];
  }
  // piece i of lane (col, grp)'s part of key tile mt (a turn depends on the column alone,
  // and a lane's pieces differ in their lowest bits)
  static __device__ __forceinline__ u32x4 operand(const u32x4* lds, int mt, int i, int col, int grp) {
    const int row = (col >> 2) * (KU / 4) + (col & 3);
    return lds[row * NP + mt * 4 * NP + ((grp * (NP / 4)) ^ turn(row) ^ i)];
  }
};

// 32 keys and values in bf16.
template <int D>
struct Unit16 {
  static constexpr int KU = 32, MT = 2, DT = D / 16, KS = D / 32;
  static constexpr int VW = DT / 2;  // words of a lane's part of a value row
  using Query = bf16x8a[KS][1];
  using Keys = KeyRows<2 * D, KU>;
  static constexpr int BYTES = Keys::BYTES;  // of LDS
  Keys keys;
  uint32_t next[8][VW], vw[8][VW];

  // key(i), value(i): addresses of row i of the unit.  Values: 16 lanes read a row.
  template <typename FK, typename FV>
  __device__ __forceinline__ void load(FK key, FV value, int lane) {
    const int col = lane & 15, grp = lane >> 4;
    keys.load(key, lane);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint16_t* p = value(grp * 8 + j) + col * DT;
      if constexpr (VW == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        next[j][0] = x.x, next[j][1] = x.y, next[j][2] = x.z, next[j][3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        next[j][0] = x.x, next[j][1] = x.y;
      }
    }
  }
  // The same where all rows are there, with their strides in elements (at most kNear).
  __device__ __forceinline__ void load_all(const uint16_t* k, uint32_t ks, const uint16_t* v, uint32_t vs, int lane) {
    keys.load_all(k, 2 * ks, lane);
    const uint32_t off = (lane >> 4) * 8 * 2 * vs + (lane & 15) * DT * 2;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (VW == 4) {
        const u32x4 x = value_at<u32x4>(v + j * vs, off);
#pragma unroll
        for (int i = 0; i < 4; ++i) next[j][i] = x[i];
      } else {
        const u32x2 x = value_at<u32x2>(v + j * vs, off);
        next[j][0] = x[0], next[j][1] = x[1];
      }
    }
  }
  // What was loaded becomes the unit that is worked on: its first n keys.
  __device__ __forceinline__ void stage(u32x4* lds, int lane, int n) {
    keys.stage(lds, lane);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
      for (int i = 0; i < VW; ++i) vw[j][i] = next[j][i];
    }
    if (n < KU) {  // 0 times a NaN would not be 0
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t live = (lane >> 4) * 8 + j < n ? ~0u : 0u;
#pragma unroll
        for (int i = 0; i < VW; ++i) vw[j][i] &= live;
      }
    }
  }
  __device__ __forceinline__ void logits(const u32x4* lds, const Query& q, f32x4a (&s)[MT], int col, int grp) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      s[mt] = f32x4a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8a, Keys::operand(lds, mt, ks, col, grp)), q[ks][0],
                                                        s[mt], 0, 0, 0);
    }
  }
  // Keeps the compiler from making operands of all values ahead of the weights, which
  // its registers could not hold.
  __device__ __forceinline__ void pin() {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
      for (int i = 0; i < VW; ++i) asm volatile("" : "+v"(vw[j][i]));
    }
  }
  __device__ __forceinline__ bool odd() const {  // an infinity or NaN among any lane's values
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
      for (int i = 0; i < VW; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vw[j][i] & 0x7FFF7FFFu));
    }
    return __any(top.x >= 0x7F80 || top.y >= 0x7F80);
  }
  // The weights p of this lane's keys, times `unit`, as operands, and the values' sums
  // of dimension tile dt for them.  Two bf16 terms for a weight: with one the result was
  // 1.25 times as far from the exact one as its rounding (2.1e-3 and 1.7e-3 relative, 64
  // tokens of 16 heads on 4), for 3% less time.  The first term is the largest one below
  // the weight, so that the second is above 0 too and an infinite value stays what it is
  // (a second term of 0, or of the other sign, would make it NaN).
  struct Operand {
    bf16x8a t[2];
  };
  __device__ __forceinline__ Operand operand(const float (&p)[8], float unit) const {
    uint32_t w0[4], w1[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = unit == 1.f ? p[2 * i] : p[2 * i] * unit, y = unit == 1.f ? p[2 * i + 1] : p[2 * i + 1] * unit;
      const uint32_t xb = __builtin_elementwise_sub_sat(__float_as_uint(x), 1u), yb = __builtin_elementwise_sub_sat(__float_as_uint(y), 1u);
      w0[i] = __builtin_amdgcn_perm(yb, xb, 0x07060302u);
      w1[i] = pack2_bf16(x - __uint_as_float(xb & 0xFFFF0000u), y - __uint_as_float(yb & 0xFFFF0000u));
    }
    return {{u4_as_bf16x8(make_uint4(w0[0], w0[1], w0[2], w0[3])), u4_as_bf16x8(make_uint4(w1[0], w1[1], w1[2], w1[3]))}};
  }
  // bits: this lane group's keys whose values count
  __device__ __forceinline__ f32x4a tile(const u32x4*, int dt, const Operand& p, int, int, uint32_t bits = ~0u) const {
    const uint32_t sel = dt & 1 ? 0x07060302u : 0x05040100u;  // high or low halves
    uint32_t a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = __builtin_amdgcn_perm(vw[2 * i + 1][dt / 2], vw[2 * i][dt / 2], sel);
      a[i] &= (bits >> (2 * i) & 1u ? 0xFFFFu : 0u) | (bits >> (2 * i) & 2u ? 0xFFFF0000u : 0u);
    }
    const bf16x8a v = u4_as_bf16x8(make_uint4(a[0], a[1], a[2], a[3]));
    const f32x4a x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p.t[1], f32x4a{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p.t[0], x, 0, 0, 0);
  }
};

// The same in fp32: 16 keys of 128 dimensions, or 32 of 64.
template <int D>
struct Unit32 {
  static constexpr int KU = D == 128 ? 16 : 32, MT = KU / 16, DT = D / 16, KS = D / 4;
  static constexpr int VT = KU / 4;  // keys of a lane group
  using Query = float[KS];
  using Keys = KeyRows<4 * D, KU>;
  static constexpr int BYTES = Keys::BYTES;
  Keys keys;
  float next[VT][DT], vw[VT][DT];

  template <typename FK, typename FV>
  __device__ __forceinline__ void load(FK key, FV value, int lane) {
    const int col = lane & 15, grp = lane >> 4;
    keys.load(key, lane);
#pragma unroll
    for (int j = 0; j < VT; ++j) {
      const float4* p = reinterpret_cast<const float4*>(value(grp * VT + j) + col * DT);
#pragma unroll
      for (int i = 0; i < DT; i += 4) {
        const float4 x = p[i / 4];
        next[j][i] = x.x, next[j][i + 1] = x.y, next[j][i + 2] = x.z, next[j][i + 3] = x.w;
      }
    }
  }
  __device__ __forceinline__ void load_all(const float* k, uint32_t ks, const float* v, uint32_t vs, int lane) {
    keys.load_all(k, 4 * ks, lane);
    const uint32_t off = (lane >> 4) * VT * 4 * vs + (lane & 15) * DT * 4;
#pragma unroll
    for (int j = 0; j < VT; ++j) {
#pragma unroll
      for (int i = 0; i < DT; i += 4) {
        const f32x4a x = value_at<f32x4a>(v + j * vs + i, off);
#pragma unroll
        for (int e = 0; e < 4; ++e) next[j][i + e] = x[e];
      }
    }
  }
  __device__ __forceinline__ void stage(u32x4* lds, int lane, int n) {
    keys.stage(lds, lane);
#pragma unroll
    for (int j = 0; j < VT; ++j) {
#pragma unroll
      for (int i = 0; i < DT; ++i) vw[j][i] = next[j][i];
    }
    if (n < KU) {
#pragma unroll
      for (int j = 0; j < VT; ++j) {
        const bool live = (lane >> 4) * VT + j < n;
#pragma unroll
        for (int i = 0; i < DT; ++i) vw[j][i] = live ? vw[j][i] : 0.f;
      }
    }
  }
  __device__ __forceinline__ void logits(const u32x4* lds, const Query& q, f32x4a (&s)[MT], int col, int grp) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      s[mt] = f32x4a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS / 4; ++i) {
        const u32x4 x = Keys::operand(lds, mt, i, col, grp);
        const float k[4] = {__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w)};
#pragma unroll
        for (int e = 0; e < 4; ++e) s[mt] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], q[4 * i + e], s[mt], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void pin() {}
  __device__ __forceinline__ bool odd() const {
    bool any = false;
#pragma unroll
    for (int j = 0; j < VT; ++j) {
#pragma unroll
      for (int i = 0; i < DT; ++i) any |= (__float_as_uint(vw[j][i]) & 0x7F800000u) == 0x7F800000u;
    }
    return __any(any);
  }
  struct Operand {
    float t[VT];
  };
  __device__ __forceinline__ Operand operand(const float (&p)[VT], float unit) const {
    Operand w;
#pragma unroll
    for (int j = 0; j < VT; ++j) w.t[j] = unit == 1.f ? p[j] : p[j] * unit;
    return w;
  }
  __device__ __forceinline__ f32x4a tile(const u32x4*, int dt, const Operand& p, int, int, uint32_t bits = ~0u) const {
    f32x4a x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < VT; ++j)
      x = __builtin_amdgcn_mfma_f32_16x16x4f32(bits >> j & 1u ? vw[j][dt] : 0.f, p.t[j], x, 0, 0, 0);
    return x;
  }
};

// Weights of a bf16 problem over 8-bit values: two fp16 terms, off by 2^-22 (codes are
// exact in fp16).  One term, off by 2^-11, left the result 1.71e-3 from the exact one where
// rounding to bf16 leaves 1.70e-3, and further where values cancel (256 tokens of 8 heads
// on 2 over 523776: 34.9 us with one, 37.1 with two; 16 tokens 11.0 either way).
struct WeightPair {
  f16x8a t[2];
  __device__ __forceinline__ void set(const float (&p)[8]) {
    uint32_t w0[4], w1[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w0[i] = pack2_f16(p[2 * i], p[2 * i + 1]);
      const f16x2a first = __builtin_bit_cast(f16x2a, w0[i]);
      w1[i] = pack2_f16(p[2 * i] - static_cast<float>(first[0]), p[2 * i + 1] - static_cast<float>(first[1]));
    }
    t[0] = __builtin_bit_cast(f16x8a, make_uint4(w0[0], w0[1], w0[2], w0[3]));
    t[1] = __builtin_bit_cast(f16x8a, make_uint4(w1[0], w1[1], w1[2], w1[3]));
  }
  static __device__ __forceinline__ f16x8a codes(uint32_t w0, uint32_t w1) { return Weights<1>::codes(w0, w1); }
  __device__ __forceinline__ f32x4a times(f16x8a v, f32x4a acc) const {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, t[1], acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(v, t[0], acc, 0, 0, 0);
  }
};

// KU keys of the 8-bit cache, keys and values by way of LDS; NT bf16 terms of a query
// (qcache_unit.h), and of a weight where that is more than one.  Row r of the values'
// dimension tile dt is dimension r D/16 + dt, as above.
template <int D, int KU8, int NT>
struct Unit8 {
  using Weight = std::conditional_t<NT == 1, WeightPair, Weights<NT>>;
  static constexpr int KU = KU8, MT = KU / 16, DT = D / 16, KS = D / 32;
  static constexpr int NP = KU / 16, NL = D * NP / 64;  // pieces of a dimension's codes
  using Query = bf16x8a[KS][NT];
  using Keys = KeyRows<D, KU>;
  static constexpr int BYTES = Keys::BYTES + D * KU;
  Keys keys;
  u32x4 codes[NL];
  float ksc, vsc, ksc_next, vsc_next;

  // Piece p of a dimension is at place (NP dim + p) ^ (dim / DT % 8), so that 16 lanes'
  // dimensions lie on different banks.  (Load i's places, and dimension tile dt's, differ
  // from the first ones in bits that depend on i or dt alone.)
  static constexpr int kFirst = Keys::BYTES / 16, kRun = NP * DT;

  __device__ __forceinline__ void load(const QCache& c, int64_t cell, int C, int u, int lane) {
    const uint8_t* kp = c.k + (cell * C + u * KU) * D;
    const uint8_t* vp = c.v + cell * C * D + u * KU;
    keys.load_all(kp, D, lane);
    const uint32_t off = lane / NP * C + lane % NP * 16;
#pragma unroll
    for (int i = 0; i < NL; ++i) codes[i] = value_at<u32x4>(vp + i * (64 / NP) * C, off);
    ksc_next = c.k_scale[cell];
    vsc_next = c.v_scale[cell];
  }
  __device__ __forceinline__ void stage(u32x4* lds, int lane, int n) {
    keys.stage(lds, lane);
    ksc = ksc_next;
    vsc = vsc_next;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int m = i * 64 + lane, p = m % NP;
      u32x4 x = codes[i];
      if (n < KU) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = keep_below(x[e], p * 16 + 4 * e, n);
      }
      lds[kFirst + i * 64 + ((lane ^ ((lane / kRun) & 7)) ^ ((i * 64 / kRun) & 7))] = x;
    }
  }
  __device__ __forceinline__ void pin() {}
  __device__ __forceinline__ void logits(const u32x4* lds, const Query& q, f32x4a (&s)[MT], int col, int grp) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      s[mt] = f32x4a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS / 2; ++i) {
        const u32x4 x = Keys::operand(lds, mt, i, col, grp);
        const bf16x8a k0 = codes8_bf16(x.x, x.y, ksc), k1 = codes8_bf16(x.z, x.w, ksc);
#pragma unroll
        for (int j = 0; j < NT; ++j) s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[2 * i][j], s[mt], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < NT; ++j) s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[2 * i + 1][j], s[mt], 0, 0, 0);
      }
    }
  }
  struct Operand {
    Weight t[KU / 32];
    float scale;
  };
  __device__ __forceinline__ Operand operand(const float (&p)[KU / 4], float unit) const {
    Operand w;
#pragma unroll
    for (int st = 0; st < KU / 32; ++st) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = p[8 * st + i];
      w.t[st].set(x);
    }
    w.scale = vsc * unit;
    return w;
  }
  __device__ __forceinline__ f32x4a tile(const u32x4* lds, int dt, const Operand& p, int col, int grp, uint32_t = ~0u) const {
    f32x4a x = {0.f, 0.f, 0.f, 0.f};
    const int far = kFirst + col * kRun + dt * NP / 8 * 8, near = (col & 7) ^ (dt * NP % 8);
    if constexpr (KU == 64) {
      const u32x4 v = lds[far + (near ^ grp)];
      x = p.t[0].times(Weight::codes(v.x, v.y), x);
      x = p.t[1].times(Weight::codes(v.z, v.w), x);
    } else {
      const uint2 v = reinterpret_cast<const uint2*>(lds + far + (near ^ (grp >> 1)))[grp & 1];
      x = p.t[0].times(Weight::codes(v.x, v.y), x);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= p.scale;
    return x;
  }
};

// The largest of the four lane groups' values of a column.
__device__ __forceinline__ float max_of_groups(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Running softmax of a wavefront's 16 columns.
template <typename T, int D, bool Q8>
struct Columns {
  static constexpr int DT = D / 16;
  f32x4a o[DT];
  float m = -INFINITY, l = 0.f;  // largest logit (before its scale), this lane's sum of weights

  __device__ __forceinline__ Columns() {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4a{0.f, 0.f, 0.f, 0.f};
  }
  // s: masked logits of a unit.  Leaves the weights in p and returns the factor for
  // what was summed before.
  template <int MT>
  __device__ __forceinline__ float weigh(const f32x4a (&s)[MT], float qscale2, float (&p)[4 * MT]) {
    float mx = m;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) mx = fmaxf(mx, fmaxf(fmaxf(s[mt][0], s[mt][1]), fmaxf(s[mt][2], s[mt][3])));
    mx = max_of_groups(mx);
    const float ref = mx == -INFINITY ? 0.f : mx;
    const float corr = fast_exp2((m - ref) * qscale2);
    m = mx;
    l *= corr;
#pragma unroll
    for (int i = 0; i < 4 * MT; ++i) {
      p[i] = fast_exp2(fmaf(s[i / 4][i % 4] - ref, qscale2, kHead<T, Q8>));
      l += p[i];
    }
    return corr;
  }
  // A unit's values with their weights p.  Columns that see none of the unit keep
  // their sums (their weights of 0 do not hide an infinity or NaN).
  template <typename U>
  __device__ __forceinline__ void add(const U& u, const u32x4* lds, const typename U::Operand& p, float corr, bool sees, int col,
                                      int grp, uint32_t bits = ~0u) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const f32x4a x = u.tile(lds, dt, p, col, grp, bits);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y = fmaf(o[dt][i], corr, x[i]);
        o[dt][i] = sees ? y : o[dt][i];
      }
    }
  }
};

__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// Drafted keys j0 .. j0 + KU - 1.
template <typename U, typename T>
__device__ __forceinline__ void load_drafted(U& u, const DraftAttnArgs& a, const T* kn, const T* vn, int j0, int lane) {
  if (j0 + U::KU <= a.T && a.ksn <= kNear && a.vsn <= kNear) {
    u.load_all(kn + j0 * a.ksn, static_cast<uint32_t>(a.ksn), vn + j0 * a.vsn, static_cast<uint32_t>(a.vsn), lane);
    return;
  }
  const int last = a.T - 1;
  u.load([&](int i) { return kn + min(j0 + i, last) * a.ksn; }, [&](int i) { return vn + min(j0 + i, last) * a.vsn; }, lane);
}
// bits: those that this column sees.
template <typename U, typename T, int D, bool Q8>
__device__ __forceinline__ void add_drafted(Columns<T, D, Q8>& cs, U& u, const u32x4* lds, float qscale2, uint32_t bits,
                                            const typename U::Query& q, int col, int grp) {
  f32x4a s[U::MT];
  u.logits(lds, q, s, col, grp);
#pragma unroll
  for (int mt = 0; mt < U::MT; ++mt) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[mt][i] = (bits >> (grp * (U::KU / 4) + 4 * mt + i)) & 1u ? s[mt][i] : -INFINITY;
  }
  float p[4 * U::MT];
  const float corr = cs.template weigh<U::MT>(s, qscale2, p);
  const typename U::Operand w = u.operand(p, kUnit<T, Q8>);
  u.pin();
  if (u.odd()) {  // a column at a time, without the values that it does not see
#pragma unroll 1
    for (int c = 0; c < 16; ++c) {
      u.pin();
      cs.add(u, lds, w, corr, bits != 0 && col == c, col, grp,
             static_cast<uint32_t>(__builtin_amdgcn_readlane(bits, c)) >> (grp * (U::KU / 4)));
    }
  } else {
    cs.add(u, lds, w, corr, bits != 0, col, grp);
  }
}

// A cached unit of which the first `visible` keys exist.
template <typename U, typename T, int D, bool Q8>
__device__ __forceinline__ void add_cached(Columns<T, D, Q8>& cs, U& u, const u32x4* lds, float qscale2, int visible, bool sees,
                                           const typename U::Query& q, int col, int grp) {
  f32x4a s[U::MT];
  u.logits(lds, q, s, col, grp);
  if (__any(!sees) || visible < U::KU) {
#pragma unroll
    for (int mt = 0; mt < U::MT; ++mt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[mt][i] = sees && grp * (U::KU / 4) + 4 * mt + i < visible ? s[mt][i] : -INFINITY;
    }
  }
  float p[4 * U::MT];
  const float corr = cs.template weigh<U::MT>(s, qscale2, p);
  const typename U::Operand w = u.operand(p, kUnit<T, Q8>);
  u.pin();
  cs.add(u, lds, w, corr, sees, col, grp);
}

// Most wavefronts of a workgroup; LDS of a CU, the most a wavefront's unit takes of it,
// and the list (65535 blocks, 16 rows of 128 at most, since fanout * K <= 256).
constexpr int kMaxWaves = 8;
constexpr size_t kMaxLds = 160 * 1024, kStageMost = 16 * 1024, kListMost = (2048 + 16 * (kMaxCand / 2)) * 8;
static_assert(kMaxWaves * kStageMost + kListMost <= kMaxLds);

// 16-byte pieces of LDS that the list takes.
__host__ __device__ __forceinline__ int list_pieces(int M, int list) { return ((M + 31) / 32 + list + 1) / 2; }

// LDS of a wavefront's unit.
template <typename T, int D, bool Q8, int KU>
constexpr int kStage = Q8 ? (Unit8<D, KU, 1>::BYTES > (sizeof(T) == 4 ? Unit32<D>::BYTES : Unit16<D>::BYTES)
                                 ? Unit8<D, KU, 1>::BYTES
                                 : (sizeof(T) == 4 ? Unit32<D>::BYTES : Unit16<D>::BYTES))
                          : (sizeof(T) == 4 ? Unit32<D>::BYTES : Unit16<D>::BYTES);
static_assert(kStage<uint16_t, 128, true, 64> <= kStageMost && kStage<float, 128, false, 16> <= kStageMost);

// The blocks that any of a tile's rows selected, ascending, and for each the rows
// that did, in LDS: a bitmap of the cache's blocks, its words' running counts, and
// each entry's place from both.  Returns their number.
__device__ __forceinline__ int union_list(const DraftAttnArgs& a, int bh, int row0, int rows, uint32_t* lds, uint32_t*& blocks,
                                          uint32_t*& who) {
  const int words = (a.M + 31) / 32, nt = static_cast<int>(blockDim.x), lane = threadIdx.x & 63;
  uint32_t *bitmap = lds, *before = lds + words;
  blocks = before + words;
  who = blocks + a.list;
  const int32_t* sel = a.idx + (static_cast<int64_t>(bh) * a.T + row0) * a.K;
  const int entries = rows * a.K;
  constexpr int KEEP = 4;  // entries that a thread reads once
  int kept[KEEP];
#pragma unroll
  for (int i = 0; i < KEEP; ++i) {
    const int e = threadIdx.x + i * nt;
    kept[i] = e < entries ? sel[e] : -1;
  }
  for (int i = threadIdx.x; i < words; i += nt) bitmap[i] = 0;
  for (int i = threadIdx.x; i < a.list; i += nt) who[i] = 0;
  __syncthreads();
  auto mark = [&](int blk) {
    if (static_cast<uint32_t>(blk) < static_cast<uint32_t>(a.M)) atomicOr(&bitmap[blk >> 5], 1u << (blk & 31));
  };
#pragma unroll
  for (int i = 0; i < KEEP; ++i) mark(kept[i]);
  for (int e = threadIdx.x + KEEP * nt; e < entries; e += nt) mark(sel[e]);
  __syncthreads();
  int total = 0;
  for (int base = 0; base < words; base += 64) {  // every wavefront counts; the first one writes
    const int c = base + lane < words ? __popc(bitmap[base + lane]) : 0;
    int incl = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(incl, o);
      incl += lane >= o ? y : 0;
    }
    if (threadIdx.x < 64 && base + lane < words) before[base + lane] = static_cast<uint32_t>(total + incl - c);
    total += __shfl(incl, 63);
  }
  __syncthreads();
  auto place = [&](int blk, int e) {
    if (static_cast<uint32_t>(blk) < static_cast<uint32_t>(a.M)) {
      const uint32_t at = before[blk >> 5] + __popc(bitmap[blk >> 5] & ((1u << (blk & 31)) - 1u));
      blocks[at] = static_cast<uint32_t>(blk);
      atomicOr(&who[at], 1u << (e / a.K));
    }
  };
#pragma unroll
  for (int i = 0; i < KEEP; ++i) place(kept[i], threadIdx.x + i * nt);
  for (int e = threadIdx.x + KEEP * nt; e < entries; e += nt) place(sel[e], e);
  __syncthreads();
  return total;
}

// A lane's dimensions of a query as a unit's operand: as they are, in three bf16 terms
// (8-bit units of fp32 queries), or each a value (fp32 units).
template <typename T, int QW, int KS, int NT>
__device__ __forceinline__ void make_query(const uint4 (&qw)[QW], bf16x8a (&q)[KS][NT]) {
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    if constexpr (sizeof(T) == 2) {
      q[ks][0] = u4_as_bf16x8(qw[ks]);
    } else {
      const uint4 a = qw[2 * ks], b = qw[2 * ks + 1];
      const float x[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                          __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
      split_terms<NT>(x, q[ks]);
    }
  }
}
template <typename T, int QW, int KS>
__device__ __forceinline__ void make_query(const uint4 (&qw)[QW], float (&q)[KS]) {
#pragma unroll
  for (int i = 0; i < QW; ++i) {
    q[4 * i] = __uint_as_float(qw[i].x);
    q[4 * i + 1] = __uint_as_float(qw[i].y);
    q[4 * i + 2] = __uint_as_float(qw[i].z);
    q[4 * i + 3] = __uint_as_float(qw[i].w);
  }
}

__device__ __forceinline__ int uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(static_cast<int>(x)); }

template <typename T, bool Q8>
__device__ __forceinline__ float row_lse(float ref, float sum, float qscale2) {
  constexpr float unit = kHead<T, Q8> == 14.f ? 0x1p-14f : kHead<T, Q8> == 0.f ? 1.f : 0x1p16f;  // 2^-kHead
  return sum == 0.f ? -INFINITY : fmaf(ref, qscale2, fast_log2(sum * unit)) * kLn2;
}

template <typename T>
__device__ __forceinline__ void store_out(void* o, int64_t at, float x) {
  if constexpr (sizeof(T) == 2) static_cast<uint16_t*>(o)[at] = f32_to_bf16_rne(x);
  else static_cast<float*>(o)[at] = x;
}
template <typename T>
__device__ __forceinline__ void store_out4(void* o, int64_t at, const float (&x)[4]) {
  if constexpr (sizeof(T) == 2) {
    uint2 w;
    w.x = f32_to_bf16_rne(x[0]) | static_cast<uint32_t>(f32_to_bf16_rne(x[1])) << 16;
    w.y = f32_to_bf16_rne(x[2]) | static_cast<uint32_t>(f32_to_bf16_rne(x[3])) << 16;
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(o) + at) = w;
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(o) + at) = make_float4(x[0], x[1], x[2], x[3]);
  }
}

// Where column c (of R G) of a tile is kept: its row of the outputs, or its place among
// the partials.
struct Place {
  int64_t row, part;
};
__device__ __forceinline__ Place place_of(const DraftAttnArgs& a, int tile, int bh, int c) {
  const int b = bh / a.Hkv, h = bh - b * a.Hkv, r = c / a.G;
  const int64_t at = static_cast<int64_t>(tile) * a.BH + bh;
  return {(static_cast<int64_t>(b) * a.H + h * a.G + (c - r * a.G)) * a.T + tile * a.R + r,
          at * (a.R * a.G) + c};
}

// Four dimensions from dd on of a column's sums, and with the first ones its state.
template <typename T, int D, bool Q8>
__device__ __forceinline__ void finish(const DraftAttnArgs& a, const Place& pl, int dd, const float (&x)[4], float top, float l,
                                       int split) {
  if (a.splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / (l * kUnit<T, Q8>);
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = l == 0.f ? 0.f : x[i] * inv;
    store_out4<T>(a.o, pl.row * D + dd, y);
    if (a.lse && dd == 0) a.lse[pl.row] = row_lse<T, Q8>(top == -INFINITY ? 0.f : top, l, a.qscale2);
  } else {
    const int64_t at = pl.part * a.splits + split;
    *reinterpret_cast<float4*>(a.part_o + at * D + dd) = make_float4(x[0], x[1], x[2], x[3]);
    if (dd == 0) a.part_ml[at] = make_float2(top, l);
  }
}

}  // namespace

// A workgroup of KS wavefronts per (tile, KV head, split of its units).  The splits of
// a tile are ranges of its ascending list and neighbours in the grid, which the device
// deals to its 8 XCDs in turn: where tiles look for the same blocks, an XCD's L2 holds
// those of its range (256 rows of 8 heads on 2, 32 blocks of 128 each, 13 MB together:
// 47 us; splits that take every fourth unit 48).
template <typename T, int D, bool Q8, int KU>
__global__ __launch_bounds__(kMaxWaves * 64, 2) void draft_attn_kernel(DraftAttnArgs a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NT = F32 ? 3 : 1, DT = D / 16;
  using Drafted = std::conditional_t<F32, Unit32<D>, Unit16<D>>;
  using Cached = std::conditional_t<Q8, Unit8<D, KU, NT>, Drafted>;
  extern __shared__ __align__(16) uint32_t lds[];

  const int split = static_cast<int>(blockIdx.x % a.splits), w = static_cast<int>(blockIdx.x / a.splits);
  const int bh = w % a.BH, tile = a.tile0 + w / a.BH;
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int row0 = tile * a.R, rows = min(a.R, a.T - row0), live = rows * a.G;
  const int r = col / a.G, hh = col - r * a.G, row = row0 + min(r, rows - 1);
  const bool on = col < live;

  // queries: dimensions grp D/4 .. of this column's row and head, as loaded
  constexpr int QW = D / 4 * sizeof(T) / 16;
  uint4 qw[QW];
  {
    const T* q = static_cast<const T*>(a.q) + ((static_cast<int64_t>(b) * a.H + h * a.G + hh) * a.T + row) * D + grp * (D / 4);
#pragma unroll
    for (int i = 0; i < QW; ++i) qw[i] = on ? reinterpret_cast<const uint4*>(q)[i] : make_uint4(0, 0, 0, 0);
  }

  const int chunks = (a.T + Drafted::KU - 1) / Drafted::KU;
  const uint64_t* mask = a.mask + b * a.mask_bstride + static_cast<int64_t>(row) * a.W;
  const T* kn = static_cast<const T*>(a.k_new) + b * a.ksb + h * a.ksh;
  const T* vn = static_cast<const T*>(a.v_new) + b * a.vsb + h * a.vsh;
  auto seen = [&](int j0) {  // drafted keys from j0 on that this column sees
    return on ? static_cast<uint32_t>(mask[j0 >> 6] >> (j0 & 63)) & low_bits(min(Drafted::KU, a.T - j0)) : 0u;
  };
  // units are the drafted keys', then the list's; the first ones are on their way while
  // the list is made
  Drafted ud;
  uint32_t bits = 0;
  const bool early = split == 0 && wave < chunks;
  if (early) {
    bits = seen(wave * Drafted::KU);
    load_drafted(ud, a, kn, vn, wave * Drafted::KU, lane);
  }

  uint32_t *blocks, *who;
  const int nblk = uniform(union_list(a, bh, row0, rows, lds, blocks, who));
  u32x4* stage = reinterpret_cast<u32x4*>(lds) + list_pieces(a.M, a.list) + wave * (kStage<T, D, Q8, KU> / 16);
  const int per = a.C / KU, all = chunks + nblk * per, step = a.KS;
  const int begin = static_cast<int>(static_cast<int64_t>(all) * split / a.splits);
  const int end = static_cast<int>(static_cast<int64_t>(all) * (split + 1) / a.splits);

  Columns<T, D, Q8> cs;
  int t = begin + wave;
  const int drafts = min(chunks, end);
  if (t < drafts) {
    typename Drafted::Query q;
    make_query<T>(qw, q);
    if (!early) {
      bits = seen(t * Drafted::KU);
      load_drafted(ud, a, kn, vn, t * Drafted::KU, lane);
    }
    for (;;) {
      if (__any(bits != 0)) {
        wave_sync();
        ud.stage(stage, lane, a.T - t * Drafted::KU);
        wave_sync();
        add_drafted<Drafted, T, D, Q8>(cs, ud, stage, a.qscale2, bits, q, col, grp);
      }
      do {  // on to the next ones that any column sees
        t += step;
        bits = t < drafts ? seen(t * Drafted::KU) : 0u;
      } while (t < drafts && !__any(bits != 0));
      if (t >= drafts) break;
      load_drafted(ud, a, kn, vn, t * Drafted::KU, lane);
    }
  }

  {
    typename Cached::Query q;
    make_query<T>(qw, q);
    Cached u;
    int next_visible = 0;
    bool next_sees = false;
    // loads the cached unit of task t: its visible keys, and whether this column sees it
    auto fetch = [&](int t) {
      next_visible = 0;
      if (t >= end) return;
      const int slot = (t - chunks) / per, part = t - chunks - slot * per;
      const int blk = uniform(blocks[slot]);
      const uint32_t rows_in = static_cast<uint32_t>(uniform(who[slot]));
      const int key0 = blk * a.C + part * KU;
      next_sees = ((rows_in >> r) & 1u) || !on;
      next_visible = min(KU, a.n - key0);
      if (next_visible <= 0) return;  // the last block's end
      if constexpr (Q8) {
        u.load(a.c, static_cast<int64_t>(bh) * a.c.M + blk, a.C, part, lane);
      } else {
        const int64_t first = (static_cast<int64_t>(bh) * a.Nkv + key0) * D;
        const T *kb = static_cast<const T*>(a.k) + first, *vb = static_cast<const T*>(a.v) + first;
        if (next_visible == KU) {
          u.load_all(kb, D, vb, D, lane);
          return;
        }
        const int last = next_visible - 1;
        u.load([&](int i) { return kb + static_cast<uint32_t>(min(i, last) * D); },
               [&](int i) { return vb + static_cast<uint32_t>(min(i, last) * D); }, lane);
      }
    };
    fetch(t);
    while (t < end) {  // the next unit's loads are in flight while one is added
      const int visible = next_visible;
      const bool sees = next_sees;
      if (visible > 0) {
        wave_sync();
        u.stage(stage, lane, visible);
        wave_sync();
      }
      t += step;
      fetch(t);
      if (visible > 0) add_cached<Cached, T, D, Q8>(cs, u, stage, a.qscale2, visible, sees, q, col, grp);
    }
  }

  float l = cs.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  if (a.KS == 1) {
    if (!on) return;
    const Place pl = place_of(a, tile, bh, col);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int dt = 0; dt < DT; dt += 4) {
        const float x[4] = {cs.o[dt][i], cs.o[dt + 1][i], cs.o[dt + 2][i], cs.o[dt + 3][i]};
        finish<T, D, Q8>(a, pl, (grp * 4 + i) * DT + dt, x, cs.m, l, split);
      }
    }
    return;
  }

  // the wavefronts' states of every column meet in LDS, where the list was
  constexpr int LW = D + 4;
  const int cols = a.R * a.G;
  float* red = reinterpret_cast<float*>(lds);
  __syncthreads();
  if (on) {
    float* mine = red + (wave * cols + col) * LW;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int dt = 0; dt < DT; dt += 4)
        *reinterpret_cast<float4*>(mine + (grp * 4 + i) * DT + dt) =
            make_float4(cs.o[dt][i], cs.o[dt + 1][i], cs.o[dt + 2][i], cs.o[dt + 3][i]);
    }
    if (grp == 0) {
      mine[D] = cs.m;
      mine[D + 1] = l;
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < live * (D / 4); e += static_cast<int>(blockDim.x)) {
    const int c = e / (D / 4), dd = (e - c * (D / 4)) * 4, next = cols * LW;  // to the next wavefront's
    const float* x = red + c * LW;
    float2 ml[kMaxWaves];  // all of them asked for at once; the last one's again for those that are not there
    f32x4a y[kMaxWaves];
#pragma unroll
    for (int i = 0; i < kMaxWaves; ++i) {
      const float* xi = x + min(i, a.KS - 1) * next;
      ml[i] = *reinterpret_cast<const float2*>(xi + D);
      y[i] = *reinterpret_cast<const f32x4a*>(xi + dd);
    }
    float top = ml[0].x;
#pragma unroll
    for (int i = 1; i < kMaxWaves; ++i) top = fmaxf(top, ml[i].x);
    const float ref = top == -INFINITY ? 0.f : top;
    float ll = 0.f, oo[4] = {};
#pragma unroll
    for (int i = 0; i < kMaxWaves; ++i) {
      if (i < a.KS) {
        const float f = fast_exp2((ml[i].x - ref) * a.qscale2);
        ll += ml[i].y * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) oo[e] += y[i][e] * f;
      }
    }
    finish<T, D, Q8>(a, place_of(a, tile, bh, c), dd, oo, top, ll, split);
  }
}

// The splits' states of one column: a wavefront, lane i < splits holding split i's
// weight.  All of its loads are asked for at once: one latency and the launch, 2.4 to
// 4.8 us.
constexpr int kMaxSplits = 16;  // 64 wavefronts, four to a workgroup
template <typename T, int D, bool Q8>
__global__ __launch_bounds__(64) void draft_merge_kernel(DraftAttnArgs a) {
  constexpr int E = D / 64;
  const int w = static_cast<int>(blockIdx.x), c = static_cast<int>(blockIdx.y), lane = threadIdx.x;
  const int bh = w % a.BH, tile = a.tile0 + w / a.BH;
  if (tile * a.R + c / a.G >= a.T) return;
  const Place pl = place_of(a, tile, bh, c);
  const float2 ml = lane < a.splits ? a.part_ml[pl.part * a.splits + lane] : make_float2(-INFINITY, 0.f);
  const float* p = a.part_o + pl.part * a.splits * D + lane * E;
  float x[kMaxSplits][E];
#pragma unroll
  for (int i = 0; i < kMaxSplits; ++i) {
    if (i < a.splits) {
#pragma unroll
      for (int e = 0; e < E; ++e) x[i][e] = p[i * D + e];
    }
  }
  float top = ml.x;
#pragma unroll
  for (int o = 1; o < kMaxSplits; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  top = __shfl(top, 0);
  const float ref = top == -INFINITY ? 0.f : top;
  const float f = fast_exp2((ml.x - ref) * a.qscale2);
  float ll = ml.y * f;
#pragma unroll
  for (int o = 1; o < kMaxSplits; o <<= 1) ll += __shfl_xor(ll, o);
  ll = __shfl(ll, 0);
  const float inv = ll == 0.f ? 0.f : 1.f / (ll * kUnit<T, Q8>);
  float oo[E] = {};
#pragma unroll
  for (int i = 0; i < kMaxSplits; ++i) {
    if (i < a.splits) {
      const float fi = __shfl(f, i);
#pragma unroll
      for (int e = 0; e < E; ++e) oo[e] += x[i][e] * fi;
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) store_out<T>(a.o, pl.row * D + lane * E + e, oo[e] * inv);
  if (a.lse && lane == 0) a.lse[pl.row] = row_lse<T, Q8>(ref, ll, a.qscale2);
}

namespace {

int tile_rows(const Shape& s) { return std::max(1, 16 / s.G); }

// Keys of a cached unit.
int unit_keys(const Shape& s, bool q8) {
  if (!q8) return s.bf16 || s.D == 64 ? 32 : 16;
  return s.C % 64 == 0 && (s.bf16 || s.D == 64) ? 64 : 32;
}

// How a tile's units are spread: over the wavefronts of a workgroup, and workgroups.
// A SIMD holds two of these wavefronts (three in bf16 of 64 dimensions), so a CU one
// workgroup of five to eight, or two (three) of up to four.  With more tiles than CUs
// they are of four at most (bf16 of 128 dimensions, 32 heads on 2, 400 tiles: 16.4 us,
// seven 22; 64 dimensions, 280 tiles: 11.7, eight 14.6), and share units more finely
// where the device does not hold them at once.  Otherwise a unit to a wavefront is best,
// with as many to spare as rows may want other blocks, up to 64 and where that is much
// more than one workgroup can do: the second launch that joins workgroups costs what 32
// units of bf16 and 64 dimensions do in eight wavefronts (12 units of 64 dimensions, 118
// tiles: 8.0 us in one workgroup, 10.6 in two; 50 of 128, 8 tiles: 34 in one, 12.2 in
// eight of eight wavefronts, 11.4 in sixteen of four).  Workgroups of four where that
// leaves at most one to a CU (above), of eight elsewhere (64 tiles of 32: 13.8 and 15.4),
// and no more of these than CUs (64 dimensions, 128 tiles of 4 blocks: 12.1 in two each,
// 16.1 in three).
struct Spread {
  int ks, splits;
};
struct Units {
  int64_t tiles, held, w;  // a tile's wavefronts: those that the device holds, those wanted
  bool split;              // more than one workgroup to a tile
};
// M: blocks that there are.
Units units_of(const Shape& s, bool q8, int64_t M) {
  Units u{};
  const int R = tile_rows(s);
  u.tiles = static_cast<int64_t>(s.BH()) * ((s.Nq + R - 1) / R);
  // blocks that the rows of a tile select together, about (a tree's rows: 1.6 times one
  // row's for four, 2.5 times for sixteen), and units
  int lg = 0;
  while ((2 << lg) <= R) ++lg;
  const int64_t blocks = std::min<int64_t>(M, static_cast<int64_t>(s.K) * (8 + 3 * lg) / 8);
  const int64_t units = blocks * (s.C / unit_keys(s, q8)) + (s.Nq + 31) / 32;
  u.held = (kDeviceCUs * (s.bf16 && s.D == 64 ? 12 : 8) + u.tiles / 2) / u.tiles;
  u.w = std::max<int64_t>(1, std::min<int64_t>({u.held, 64, units * 7 / 5}));
  u.split = u.w > kMaxWaves && units * (s.D / 64) * (s.bf16 ? 1 : 3) > 32;
  return u;
}
Spread spread(const Shape& s, bool q8) {
  const Units u = units_of(s, q8, (s.N - s.Nq + s.C - 1) / s.C);
  if (u.tiles > kDeviceCUs) return {static_cast<int>(std::min<int64_t>(u.w, 4)), 1};
  if (!u.split) return {static_cast<int>(std::min<int64_t>(u.w, kMaxWaves)), 1};
  const int ks = u.tiles * ((u.w + 3) / 4) <= kDeviceCUs ? 4 : kMaxWaves;
  return {ks, static_cast<int>(std::min((u.w + ks - 1) / ks, kDeviceCUs / u.tiles))};
}
// Most splits that spread() takes whatever the cache holds, so that one workspace serves
// a cache that grows.
int most_splits(const Shape& s, bool q8) {
  const Units u = units_of(s, q8, INT32_MAX);
  return u.split ? static_cast<int>(std::max<int64_t>(1, std::min((u.w + 3) / 4, kDeviceCUs / u.tiles))) : 1;
}

size_t al256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

int tiles_of(const Shape& s) { return (s.Nq + tile_rows(s) - 1) / tile_rows(s); }

// Columns of the partials.
size_t part_cols(const Shape& s, int splits) {
  return static_cast<size_t>(s.BH()) * tiles_of(s) * tile_rows(s) * s.G * splits;
}

template <typename T, int D, bool Q8, int KU>
hipError_t launch(const Shape& s, const DraftAttnArgs& a, hipStream_t st) {
  const int tiles = tiles_of(s);
  size_t lds = static_cast<size_t>(list_pieces(a.M, a.list)) * 16 + static_cast<size_t>(a.KS) * kStage<T, D, Q8, KU>;
  if (a.KS > 1) lds = std::max(lds, static_cast<size_t>(a.KS) * a.R * s.G * (D + 4) * 4);
  if (lds > 65536) {
    static std::atomic<uint64_t> allowed{0};  // devices that were told
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = uint64_t(1) << (dev & 63);
    if (dev > 63 || !(allowed.load(std::memory_order_acquire) & bit)) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(draft_attn_kernel<T, D, Q8, KU>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMaxLds));
      if (e != hipSuccess) return e;
      if (dev <= 63) allowed.fetch_or(bit, std::memory_order_release);
    }
  }
  const int most = std::max(1, (1 << 22) / (s.BH() * a.splits));  // a launch's threads fit 32 bits
  DraftAttnArgs c = a;
  for (c.tile0 = 0; c.tile0 < tiles; c.tile0 += most) {
    const unsigned n = static_cast<unsigned>(std::min(most, tiles - c.tile0)) * static_cast<unsigned>(s.BH());
    {
      ProfScope ps("draft_attn", st);
      draft_attn_kernel<T, D, Q8, KU><<<n * a.splits, a.KS * 64, lds, st>>>(c);
    }
    if (a.splits > 1) {
      ProfScope ps("draft_merge", st);
      draft_merge_kernel<T, D, Q8><<<dim3(n, a.R * s.G), 64, 0, st>>>(c);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t draft_attn_ws(const Shape& s, bool q8) {
  const int splits = most_splits(s, q8);
  if (splits == 1) return 0;
  const size_t n = part_cols(s, splits);
  return al256(n * s.D * sizeof(float)) + n * sizeof(float2);
}

hipError_t launch_draft_attn(const Shape& s, const DraftAttn& d, const void* q, const int32_t* idx, void* o, float* lse, void* ws,
                             hipStream_t st) {
  const bool q8 = d.k == nullptr;
  const Spread sp = spread(s, q8);
  const int n = s.N - s.Nq, ku = unit_keys(s, q8);
  char* base = static_cast<char*>(ws);
  DraftAttnArgs a{};
  a.c = d.c;
  a.k = d.k;
  a.v = d.v;
  a.k_new = d.k_new;
  a.v_new = d.v_new;
  a.ksb = d.ksb, a.ksh = d.ksh, a.ksn = d.ksn;
  a.vsb = d.vsb, a.vsh = d.vsh, a.vsn = d.vsn;
  a.mask = d.mask;
  a.mask_bstride = d.mask_bstride;
  a.q = q;
  a.idx = idx;
  a.o = o;
  a.lse = lse;
  a.H = s.H, a.Hkv = s.Hkv, a.G = s.G, a.T = s.Nq, a.n = n, a.C = s.C, a.K = s.K, a.Nkv = s.Nkv;
  a.M = (n + s.C - 1) / s.C;
  a.R = tile_rows(s);
  a.KS = sp.ks;
  a.W = (s.Nq + 63) / 64;
  a.BH = s.BH();
  a.splits = sp.splits;
  a.list = std::min(a.R * s.K, a.M);
  a.qscale2 = kLog2e / sqrtf(static_cast<float>(s.D));
  if (sp.splits > 1) {
    a.part_o = reinterpret_cast<float*>(base);
    a.part_ml = reinterpret_cast<float2*>(base + al256(part_cols(s, sp.splits) * s.D * sizeof(float)));
  }
  if (q8) {
    if (s.bf16) {
      if (s.D == 128)
        return ku == 64 ? launch<uint16_t, 128, true, 64>(s, a, st) : launch<uint16_t, 128, true, 32>(s, a, st);
      return ku == 64 ? launch<uint16_t, 64, true, 64>(s, a, st) : launch<uint16_t, 64, true, 32>(s, a, st);
    }
    if (s.D == 128) return launch<float, 128, true, 32>(s, a, st);
    return ku == 64 ? launch<float, 64, true, 64>(s, a, st) : launch<float, 64, true, 32>(s, a, st);
  }
  if (s.bf16) return s.D == 128 ? launch<uint16_t, 128, false, 32>(s, a, st) : launch<uint16_t, 64, false, 32>(s, a, st);
  return s.D == 128 ? launch<float, 128, false, 16>(s, a, st) : launch<float, 64, false, 32>(s, a, st);
}

}  // namespace pisa
