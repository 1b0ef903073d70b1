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
// The products are those of qcache_attn.hip, with keys and values straight from the
// cache into operands, no LDS:
//   S^T = K q^T      row r of key tile mt is key (r/4) (KU/4) + 4 mt + r%4 of the unit,
//                    so that lane group grp gets the logits of KU/4 consecutive keys
//   O^T += V^T P^T   over those keys.  Row r of dimension tile dt is dimension
//                    r D/16 + dt: a lane then reads D/16 consecutive values of each of
//                    its keys, 16 lanes a whole row, and turns eight keys' values into
//                    operands by itself (a byte permutation for two of them).
// The drafted rows, and a bf16 cache, are units of 32 keys on v_mfma_f32_16x16x32_bf16
// (weights as bf16); fp32 ones take v_mfma_f32_16x16x4_f32, whose operands are one
// value a lane.  The 8-bit cache is multiplied as qcache_attn.hip does it.
//
// The running maximum is that of the products before the softmax's scale.  Sums of
// weights times values are held in units of kUnit, so that values up to the type's
// largest do not overflow before they are divided (values below 2^-109 lose bits).
#include <algorithm>

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
  int W;               // words of a mask row
  int BH, splits;
  int tile0;           // first tile of this launch
  int list;            // entries of the block list, at most
  float qscale2;
};

// log2 of the largest weight: fp16 weights (bf16 queries on 8-bit values) are taken up
// to 2^14, so that ones of 2^-28 of the largest are still normal numbers.
template <typename T, bool Q8>
constexpr float kHead = Q8 && sizeof(T) == 2 ? 14.f : 0.f;
// Units of the sums: 1 / (the largest weight times the tokens of a row, below 2^16).
template <typename T, bool Q8>
constexpr float kUnit = Q8 && sizeof(T) == 2 ? 0x1p-30f : 0x1p-16f;

// 32 keys and values in bf16 as a wavefront's lanes hold them.
template <int D>
struct Unit16 {
  static constexpr int KU = 32, MT = 2, DT = D / 16, KS = D / 32;
  static constexpr int VW = DT / 2;  // words of a lane's part of a value row
  using Query = bf16x8a[KS][1];
  uint4 kw[MT][KS];
  uint32_t vw[8][VW];

  // key(i), value(i): addresses of row i of the unit
  template <typename FK, typename FV>
  __device__ __forceinline__ void load(FK key, FV value, int col, int grp) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const uint4* p = reinterpret_cast<const uint4*>(key((col >> 2) * 8 + mt * 4 + (col & 3)) + grp * (D / 4));
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kw[mt][ks] = p[ks];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint16_t* p = value(grp * 8 + j) + col * DT;
      if constexpr (VW == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        vw[j][0] = x.x, vw[j][1] = x.y, vw[j][2] = x.z, vw[j][3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        vw[j][0] = x.x, vw[j][1] = x.y;
      }
    }
  }
  __device__ __forceinline__ void logits(const Query& q, f32x4a (&s)[MT]) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      s[mt] = f32x4a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u4_as_bf16x8(kw[mt][ks]), q[ks][0], s[mt], 0, 0, 0);
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
  // Clears the values of keys that `bits` does not have.
  __device__ __forceinline__ void keep(uint32_t bits, int grp) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t live = (bits >> (grp * 8 + j)) & 1u ? ~0u : 0u;
#pragma unroll
      for (int i = 0; i < VW; ++i) vw[j][i] &= live;
    }
  }
  __device__ __forceinline__ bool odd() const {  // an infinity or NaN among any lane's values
    uint32_t any = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
      for (int i = 0; i < VW; ++i) any |= ((vw[j][i] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
    }
    return __any(any != 0);
  }
  // The weights p of this lane's keys, times `unit`, as operands, and the values' sums
  // of dimension tile dt for them.
  struct Operand {
    bf16x8a t;
  };
  __device__ __forceinline__ Operand operand(const float (&p)[8], float unit) const {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack2_bf16(p[2 * i] * unit, p[2 * i + 1] * unit);
    return {u4_as_bf16x8(make_uint4(w[0], w[1], w[2], w[3]))};
  }
  // bits: this lane group's keys whose values count
  __device__ __forceinline__ f32x4a tile(int dt, const Operand& p, uint32_t bits = ~0u) const {
    const uint32_t sel = dt & 1 ? 0x07060302u : 0x05040100u;  // high or low halves
    uint32_t a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = __builtin_amdgcn_perm(vw[2 * i + 1][dt / 2], vw[2 * i][dt / 2], sel);
      a[i] &= (bits >> (2 * i) & 1u ? 0xFFFFu : 0u) | (bits >> (2 * i) & 2u ? 0xFFFF0000u : 0u);
    }
    const f32x4a zero = {0.f, 0.f, 0.f, 0.f};
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(u4_as_bf16x8(make_uint4(a[0], a[1], a[2], a[3])), p.t, zero, 0, 0, 0);
  }
};

// The same in fp32: 16 keys of 128 dimensions, or 32 of 64.
template <int D>
struct Unit32 {
  static constexpr int KU = D == 128 ? 16 : 32, MT = KU / 16, DT = D / 16, KS = D / 4;
  static constexpr int VT = KU / 4;  // keys of a lane group
  using Query = float[KS];
  float kw[MT][KS], vw[VT][DT];

  template <typename FK, typename FV>
  __device__ __forceinline__ void load(FK key, FV value, int col, int grp) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float4* p = reinterpret_cast<const float4*>(key((col >> 2) * VT + mt * 4 + (col & 3)) + grp * KS);
#pragma unroll
      for (int i = 0; i < KS; i += 4) {
        const float4 x = p[i / 4];
        kw[mt][i] = x.x, kw[mt][i + 1] = x.y, kw[mt][i + 2] = x.z, kw[mt][i + 3] = x.w;
      }
    }
#pragma unroll
    for (int j = 0; j < VT; ++j) {
      const float4* p = reinterpret_cast<const float4*>(value(grp * VT + j) + col * DT);
#pragma unroll
      for (int i = 0; i < DT; i += 4) {
        const float4 x = p[i / 4];
        vw[j][i] = x.x, vw[j][i + 1] = x.y, vw[j][i + 2] = x.z, vw[j][i + 3] = x.w;
      }
    }
  }
  __device__ __forceinline__ void logits(const Query& q, f32x4a (&s)[MT]) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      s[mt] = f32x4a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS; ++i) s[mt] = __builtin_amdgcn_mfma_f32_16x16x4f32(kw[mt][i], q[i], s[mt], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void pin() {}
  __device__ __forceinline__ void keep(uint32_t bits, int grp) {
#pragma unroll
    for (int j = 0; j < VT; ++j) {
      const bool live = (bits >> (grp * VT + j)) & 1u;
#pragma unroll
      for (int i = 0; i < DT; ++i) vw[j][i] = live ? vw[j][i] : 0.f;
    }
  }
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
    for (int j = 0; j < VT; ++j) w.t[j] = p[j] * unit;
    return w;
  }
  __device__ __forceinline__ f32x4a tile(int dt, const Operand& p, uint32_t bits = ~0u) const {
    f32x4a x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < VT; ++j)
      x = __builtin_amdgcn_mfma_f32_16x16x4f32(bits >> j & 1u ? vw[j][dt] : 0.f, p.t[j], x, 0, 0, 0);
    return x;
  }
};

// KU8 keys of the 8-bit cache (qcache_unit.h); NT bf16 terms of a query and a weight.
template <int D, int KU8, int NT>
struct Unit8 {
  static constexpr int KU = KU8, MT = KU / 16, DT = D / 16, KS = D / 32;
  using Query = bf16x8a[KS][NT];
  Unit<D, KU, true> u;

  __device__ __forceinline__ void pin() { u.pin(); }
  __device__ __forceinline__ void logits(const Query& q, f32x4a (&s)[MT]) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      s[mt] = f32x4a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8a kv = u.key(mt, ks);
#pragma unroll
        for (int j = 0; j < NT; ++j) s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv, q[ks][j], s[mt], 0, 0, 0);
      }
    }
  }
  struct Operand {
    Weights<NT> t[KU / 32];
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
    w.scale = u.vsc * unit;
    return w;
  }
  __device__ __forceinline__ f32x4a tile(int dt, const Operand& p, uint32_t = ~0u) const {
    f32x4a x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < KU / 32; ++st) x = p.t[st].times(u.template value<NT>(st, dt), x);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= p.scale;
    return x;
  }
};

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
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
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
  __device__ __forceinline__ void add(const U& u, const typename U::Operand& p, float corr, bool sees, uint32_t bits = ~0u) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const f32x4a x = u.tile(dt, p, bits);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y = fmaf(o[dt][i], corr, x[i]);
        o[dt][i] = sees ? y : o[dt][i];
      }
    }
  }
};

__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// Drafted keys j0 .. j0 + KU - 1; bits: those that this column sees.
template <typename U, typename T, int D, bool Q8>
__device__ __forceinline__ void add_drafted(Columns<T, D, Q8>& cs, const DraftAttnArgs& a, const T* kn, const T* vn, int j0,
                                            uint32_t bits, const typename U::Query& q, int col, int grp) {
  U u;
  const int last = a.T - 1;
  u.load([&](int i) { return kn + min(j0 + i, last) * a.ksn; }, [&](int i) { return vn + min(j0 + i, last) * a.vsn; }, col, grp);
  const uint32_t real = low_bits(a.T - j0);
  u.keep(real, grp);
  f32x4a s[U::MT];
  u.logits(q, s);
#pragma unroll
  for (int mt = 0; mt < U::MT; ++mt) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[mt][i] = (bits >> (grp * (U::KU / 4) + 4 * mt + i)) & 1u ? s[mt][i] : -INFINITY;
  }
  float p[4 * U::MT];
  const float corr = cs.template weigh<U::MT>(s, a.qscale2, p);
  const typename U::Operand w = u.operand(p, kUnit<T, Q8>);
  u.pin();
  if (u.odd()) {  // a column at a time, without the values that it does not see
#pragma unroll 1
    for (int c = 0; c < 16; ++c) {
      u.pin();
      cs.add(u, w, corr, bits != 0 && col == c, static_cast<uint32_t>(__builtin_amdgcn_readlane(bits, c)) >> (grp * (U::KU / 4)));
    }
  } else {
    cs.add(u, w, corr, bits != 0);
  }
}

// A cached unit of which the first `visible` keys exist.
template <typename U, typename T, int D, bool Q8>
__device__ __forceinline__ void add_cached(Columns<T, D, Q8>& cs, U& u, float qscale2, int visible, bool sees,
                                           const typename U::Query& q, int grp) {
  f32x4a s[U::MT];
  u.logits(q, s);
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
  cs.add(u, w, corr, sees);
}

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
  for (int i = threadIdx.x; i < words; i += nt) bitmap[i] = 0;
  for (int i = threadIdx.x; i < a.list; i += nt) who[i] = 0;
  __syncthreads();
  for (int e = threadIdx.x; e < rows * a.K; e += nt) {
    const int blk = sel[e];
    if (static_cast<uint32_t>(blk) < static_cast<uint32_t>(a.M)) atomicOr(&bitmap[blk >> 5], 1u << (blk & 31));
  }
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
  for (int e = threadIdx.x; e < rows * a.K; e += nt) {
    const int blk = sel[e];
    if (static_cast<uint32_t>(blk) < static_cast<uint32_t>(a.M)) {
      const uint32_t at = before[blk >> 5] + __popc(bitmap[blk >> 5] & ((1u << (blk & 31)) - 1u));
      blocks[at] = static_cast<uint32_t>(blk);
      atomicOr(&who[at], 1u << (e / a.K));
    }
  }
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
  constexpr float unit = kHead<T, Q8> == 14.f ? 0x1p-14f : 1.f;  // the headroom leaves the sum before its logarithm
  return sum == 0.f ? -INFINITY : fmaf(ref, qscale2, fast_log2(sum * unit)) * kLn2;
}

template <typename T>
__device__ __forceinline__ void store_out(void* o, int64_t at, float x) {
  if constexpr (sizeof(T) == 2) static_cast<uint16_t*>(o)[at] = f32_to_bf16_rne(x);
  else static_cast<float*>(o)[at] = x;
}

}  // namespace

// A workgroup of NW wavefronts per (tile of R rows, KV head, split of its units).
template <typename T, int D, bool Q8, int KU, int NW>
__global__ __launch_bounds__(NW * 64, 2) void draft_attn_kernel(DraftAttnArgs a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NT = F32 ? 3 : 1, DT = D / 16;
  using Drafted = std::conditional_t<F32, Unit32<D>, Unit16<D>>;
  using Cached = std::conditional_t<Q8, Unit8<D, KU, NT>, Drafted>;
  extern __shared__ __align__(16) uint32_t lds[];

  const int64_t w = blockIdx.x;
  const int bh = static_cast<int>(w % a.BH), tile = a.tile0 + static_cast<int>(w / a.BH);
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

  uint32_t *blocks, *who;
  const int nblk = union_list(a, bh, row0, rows, lds, blocks, who);

  const int chunks = (a.T + Drafted::KU - 1) / Drafted::KU;
  const int per = a.C / KU, ntask = chunks + nblk * per, step = a.splits * NW;
  int task = static_cast<int>(blockIdx.y) * NW + wave;
  Columns<T, D, Q8> cs;

  {  // drafted keys
    typename Drafted::Query q;
    make_query<T>(qw, q);
    const uint64_t* mask = a.mask + b * a.mask_bstride + static_cast<int64_t>(row) * a.W;
    const T* kn = static_cast<const T*>(a.k_new) + b * a.ksb + h * a.ksh;
    const T* vn = static_cast<const T*>(a.v_new) + b * a.vsb + h * a.vsh;
    for (; task < chunks; task += step) {
      const int j0 = task * Drafted::KU;
      const uint32_t word = static_cast<uint32_t>(mask[j0 >> 6] >> (j0 & 63));
      const uint32_t bits = on ? word & low_bits(min(Drafted::KU, a.T - j0)) : 0u;
      if (__any(bits != 0)) add_drafted<Drafted, T, D, Q8>(cs, a, kn, vn, j0, bits, q, col, grp);
    }
  }

  {  // cached keys
    typename Cached::Query q;
    make_query<T>(qw, q);
    // the unit of task t: its codes or rows, its visible keys, and whether this column sees it
    auto fetch = [&](int t, Cached& u, int& visible, bool& sees) {
      if (t >= ntask) return;
      const int e = t - chunks, slot = e / per, part = e - slot * per;
      const int blk = uniform(blocks[slot]);
      const uint32_t rows_in = static_cast<uint32_t>(uniform(who[slot]));
      const int key0 = blk * a.C + part * KU;
      visible = min(KU, a.n - key0);
      sees = on && ((rows_in >> r) & 1u);
      if (visible <= 0) return;  // the last block's end
      if constexpr (Q8) {
        u.u.load(a.c, static_cast<int64_t>(bh) * a.c.M + blk, a.C, part, col, grp);
      } else {
        const int64_t first = (static_cast<int64_t>(bh) * a.Nkv + key0) * D;
        const T *kb = static_cast<const T*>(a.k) + first, *vb = static_cast<const T*>(a.v) + first;
        const int last = visible - 1;
        u.load([&](int i) { return kb + static_cast<uint32_t>(min(i, last) * D); },
               [&](int i) { return vb + static_cast<uint32_t>(min(i, last) * D); }, col, grp);
      }
    };
    auto add = [&](Cached& u, int visible, bool sees) {
      if (visible <= 0) return;
      if (visible < KU) {
        if constexpr (Q8) u.u.clear_from(visible, grp);
        else u.keep(low_bits(visible), grp);
      }
      add_cached<Cached, T, D, Q8>(cs, u, a.qscale2, visible, sees || !on, q, grp);
    };
    Cached ua;
    int na = 0;
    bool sa = false;
    fetch(task, ua, na, sa);
    if constexpr (F32 && !Q8 && D == 128) {  // two units and their sums are more than the registers hold
      for (; task < ntask; task += step) {
        add(ua, na, sa);
        fetch(task + step, ua, na, sa);
      }
    } else {
      Cached ub;
      int nb = 0;
      bool sb = false;
      while (task < ntask) {  // the next unit's loads are in flight while one is added
        fetch(task + step, ub, nb, sb);
        add(ua, na, sa);
        task += step;
        if (task >= ntask) break;
        fetch(task + step, ua, na, sa);
        add(ub, nb, sb);
        task += step;
      }
    }
  }

  float l = cs.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // the wavefronts' states of every column meet in LDS, where the list was
  constexpr int LW = D + 2;
  const int cols = a.R * a.G;
  float* red = reinterpret_cast<float*>(lds);
  __syncthreads();
  if (on) {
    float* mine = red + (wave * cols + col) * LW;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) mine[(grp * 4 + i) * DT + dt] = cs.o[dt][i];
    }
    if (grp == 0) {
      mine[D] = cs.m;
      mine[D + 1] = l;
    }
  }
  __syncthreads();
  const int64_t at = static_cast<int64_t>(tile) * a.BH + bh;
  for (int e = threadIdx.x; e < live * D; e += NW * 64) {
    const int c = e / D, dd = e - c * D;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NW; ++i) top = fmaxf(top, red[(i * cols + c) * LW + D]);
    const float ref = top == -INFINITY ? 0.f : top;
    float ll = 0.f, oo = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float* x = red + (i * cols + c) * LW;
      const float f = fast_exp2((x[D] - ref) * a.qscale2);
      ll += x[D + 1] * f;
      oo += x[dd] * f;
    }
    if (a.splits == 1) {
      const int cr = c / a.G;
      const int64_t orow = (static_cast<int64_t>(b) * a.H + h * a.G + (c - cr * a.G)) * a.T + row0 + cr;
      store_out<T>(a.o, orow * D + dd, ll == 0.f ? 0.f : oo / (ll * kUnit<T, Q8>));
      if (a.lse && dd == 0) a.lse[orow] = row_lse<T, Q8>(ref, ll, a.qscale2);
    } else {
      a.part_o[((at * a.splits + blockIdx.y) * cols + c) * D + dd] = oo;
      if (dd == 0) a.part_ml[(at * cols + c) * a.splits + blockIdx.y] = make_float2(top, ll);
    }
  }
}

// The splits' states of one column: a wavefront, lane i < splits holding split i's
// weight.
constexpr int kMaxSplits = 16;
template <typename T, int D, bool Q8>
__global__ __launch_bounds__(64) void draft_merge_kernel(DraftAttnArgs a) {
  constexpr int E = D / 64;
  const int64_t w = blockIdx.x;
  const int c = blockIdx.y, lane = threadIdx.x, cols = a.R * a.G;
  const int bh = static_cast<int>(w % a.BH), tile = a.tile0 + static_cast<int>(w / a.BH);
  const int64_t at = static_cast<int64_t>(tile) * a.BH + bh;
  const int cr = c / a.G, row = tile * a.R + cr;
  if (row >= a.T) return;
  const float2 ml = lane < a.splits ? a.part_ml[(at * cols + c) * a.splits + lane] : make_float2(-INFINITY, 0.f);
  float x[kMaxSplits][E];
#pragma unroll
  for (int i = 0; i < kMaxSplits; ++i) {
    if (i < a.splits) {
      const float* p = a.part_o + ((at * a.splits + i) * cols + c) * D + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) x[i][e] = p[e];
    }
  }
  float top = ml.x;
#pragma unroll
  for (int o = 1; o < kMaxSplits; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
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
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int64_t orow = (static_cast<int64_t>(b) * a.H + h * a.G + (c - cr * a.G)) * a.T + row;
#pragma unroll
  for (int e = 0; e < E; ++e) store_out<T>(a.o, orow * D + lane * E + e, oo[e] * inv);
  const float top0 = __shfl(ref, 0);
  if (a.lse && lane == 0) a.lse[orow] = row_lse<T, Q8>(top0, ll, a.qscale2);
}

namespace {

int tile_rows(const Shape& s) { return std::max(1, 16 / s.G); }

// Keys of a cached unit.
int unit_keys(const Shape& s, bool q8) {
  if (!q8) return s.bf16 || s.D == 64 ? 32 : 16;
  return s.C % 64 == 0 && (s.bf16 || s.D == 64) ? 64 : 32;
}

// Wavefronts that share a tile's units: nw of a workgroup, splits of them.  As in
// qcache_attn.hip the device holds 2048 of these wavefronts.
struct Spread {
  int nw, splits;
};
Spread spread(const Shape& s, bool q8) {
  const int R = tile_rows(s);
  const int64_t tiles = static_cast<int64_t>(s.BH()) * ((s.Nq + R - 1) / R);
  const int64_t units = static_cast<int64_t>(s.K) * (s.C / unit_keys(s, q8)) * (R > 1 ? 2 : 1);
  int w = 1;
  while (w < units && w < 64 && 2 * w * tiles <= 2048) w *= 2;
  if (w <= 8) return {w, 1};
  const int nw = w == 16 ? 2 : 4;
  return {nw, w / nw};
}

size_t al256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

size_t part_ml_at(const Shape& s, int splits) {
  const int R = tile_rows(s);
  return al256(static_cast<size_t>(s.BH()) * ((s.Nq + R - 1) / R) * splits * R * s.G * s.D * sizeof(float));
}

template <typename T, int D, bool Q8, int KU, int NW>
hipError_t launch(const Shape& s, const DraftAttnArgs& a, hipStream_t st) {
  const int tiles = (s.Nq + a.R - 1) / a.R;
  const size_t words = (a.M + 31) / 32;
  const size_t lds = std::max((2 * words + 2 * static_cast<size_t>(a.list)) * 4, static_cast<size_t>(NW) * a.R * s.G * (D + 2) * 4);
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(draft_attn_kernel<T, D, Q8, KU, NW>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
    if (e != hipSuccess) return e;
  }
  // a launch's threads fit 32 bits; workgroup w takes KV head w % BH, so that an
  // XCD's workgroups share KV heads
  const int most = std::max(1, (1 << 22) / s.BH());
  DraftAttnArgs c = a;
  for (c.tile0 = 0; c.tile0 < tiles; c.tile0 += most) {
    const unsigned n = static_cast<unsigned>(std::min(most, tiles - c.tile0)) * static_cast<unsigned>(s.BH());
    {
      ProfScope ps("draft_attn", st);
      draft_attn_kernel<T, D, Q8, KU, NW><<<dim3(n, a.splits), NW * 64, lds, st>>>(c);
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

template <typename T, int D, bool Q8, int KU>
hipError_t launch_nw(const Shape& s, const DraftAttnArgs& a, int nw, hipStream_t st) {
  switch (nw) {
    case 1: return launch<T, D, Q8, KU, 1>(s, a, st);
    case 2: return launch<T, D, Q8, KU, 2>(s, a, st);
    case 4: return launch<T, D, Q8, KU, 4>(s, a, st);
    default: return launch<T, D, Q8, KU, 8>(s, a, st);
  }
}

}  // namespace

size_t draft_attn_ws(const Shape& s, bool q8) {
  const int splits = spread(s, q8).splits, R = tile_rows(s);
  if (splits == 1) return 0;
  return part_ml_at(s, splits) + static_cast<size_t>(s.BH()) * ((s.Nq + R - 1) / R) * splits * R * s.G * sizeof(float2);
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
  a.W = (s.Nq + 63) / 64;
  a.BH = s.BH();
  a.splits = sp.splits;
  a.list = std::min(a.R * s.K, a.M);
  a.qscale2 = kLog2e / sqrtf(static_cast<float>(s.D));
  if (sp.splits > 1) {
    a.part_o = reinterpret_cast<float*>(base);
    a.part_ml = reinterpret_cast<float2*>(base + part_ml_at(s, sp.splits));
  }
  if (q8) {
    if (s.bf16) {
      if (s.D == 128)
        return ku == 64 ? launch_nw<uint16_t, 128, true, 64>(s, a, sp.nw, st) : launch_nw<uint16_t, 128, true, 32>(s, a, sp.nw, st);
      return ku == 64 ? launch_nw<uint16_t, 64, true, 64>(s, a, sp.nw, st) : launch_nw<uint16_t, 64, true, 32>(s, a, sp.nw, st);
    }
    if (s.D == 128) return launch_nw<float, 128, true, 32>(s, a, sp.nw, st);
    return ku == 64 ? launch_nw<float, 64, true, 64>(s, a, sp.nw, st) : launch_nw<float, 64, true, 32>(s, a, sp.nw, st);
  }
  if (s.bf16) return s.D == 128 ? launch_nw<uint16_t, 128, false, 32>(s, a, sp.nw, st) : launch_nw<uint16_t, 64, false, 32>(s, a, sp.nw, st);
  return s.D == 128 ? launch_nw<float, 128, false, 16>(s, a, sp.nw, st) : launch_nw<float, 64, false, 32>(s, a, sp.nw, st);
}

}  // namespace pisa
