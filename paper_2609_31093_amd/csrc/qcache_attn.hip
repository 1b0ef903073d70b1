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
// An e4m3 key times its power of two is exact in bf16, and so are its products
// with q in fp32.  32-bit queries are split into three bf16 terms that add up to
// them exactly, and so are their weights.  bf16 queries' weights are rounded to
// fp16 (relative 2^-11; bf16's 2^-8 left the result 1.3 times as far from the
// exact one as rounding it does), in which value codes are exact too; the values'
// scale is applied to the product in fp32.  Those weights are taken up to 2^14
// (kHeadroom), so that ones of 2^-28 of the largest are still normal numbers.
// Sums of weights are not rounded.  (A second fp16 term for what the first leaves
// of a weight brings a token's result over 131072 to what rounding it to bf16
// alone leaves, 1.666e-3 from the exact one instead of 1.673e-3, and took 7.80 us
// instead of 7.57, 8 drafted rows over 524288 10.2 instead of 9.65.)
//
// The running maximum is that of the products S themselves, and the softmax's
// scale (with log2 e) multiplies differences from it: a large logit that is
// rounded with its scale first is off by more than fp16's last two octaves.  The
// sums over a row are held in units of kRowUnit, so that values up to the type's
// largest do not overflow before they are divided by the weights' sum.
#include <algorithm>

#include "attn_shared.h"
#include "common.h"
#include "kernels.h"
#include "qcache_unit.h"

namespace pisa {

namespace {

struct QAttnArgs {
  QCache c;
  const void* q;
  const int32_t* idx;
  void* o;
  float* lse;
  // splits > 1: unnormalised sums [rows][splits][G][D], and the largest logit and
  // sum of weights [rows][G][splits]
  float* part_o;
  float2* part_ml;
  int H, Hkv, G, Nq, N, C, K, causal, M1;
  int BH, splits;
  int row0;  // first row of this launch
  float qscale2;
};

// log2 of the largest weight.
template <int NT>
constexpr float kHeadroom = NT == 1 ? 14.f : 0.f;

// A row's sums of weights times values, and of weights before they divide them,
// are taken times this: 1 / (the largest weight times a row's 128 * 256 tokens at
// most).  A power of two, so nothing is rounded by it; the least value, 2^-109,
// leaves a sum of 2^-124, which still has all its bits.
template <int NT>
constexpr float kRowUnit = NT == 1 ? 0x1p-29f : 0x1p-15f;

}  // namespace

// Logits of a unit for 16 columns, masked: s[mt][i] is key grp*KU/4 + 4*mt + i.
// nkeys: this column's visible keys, from the first on.
template <int D, int KU, int NT>
__device__ __forceinline__ void unit_logits(const Unit<D, KU>& u, const bf16x8a (&qt)[D / 32][NT], bool partial, int nkeys, int grp,
                                            f32x4a (&s)[KU / 16]) {
#pragma unroll
  for (int mt = 0; mt < KU / 16; ++mt) {
    s[mt] = f32x4a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      const bf16x8a kv = u.key(mt, ks);
#pragma unroll
      for (int j = 0; j < NT; ++j) s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv, qt[ks][j], s[mt], 0, 0, 0);
    }
  }
  if (partial) {
#pragma unroll
    for (int mt = 0; mt < KU / 16; ++mt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[mt][i] = grp * (KU / 4) + 4 * mt + i < nkeys ? s[mt][i] : -INFINITY;
    }
  }
}
// A column's largest logit.
template <int MT>
__device__ __forceinline__ float column_max(const f32x4a (&s)[MT]) {
  float mx = -INFINITY;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) mx = fmaxf(mx, fmaxf(fmaxf(s[mt][0], s[mt][1]), fmaxf(s[mt][2], s[mt][3])));
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  return fmaxf(mx, __shfl_xor(mx, 32));
}
// Logits to weights 2^((s - ref) * qscale2 + headroom), as operands, for ref the
// largest of them or larger; returns this lane's sum.
template <int MT, int NT>
__device__ __forceinline__ float weights(const f32x4a (&s)[MT], float qscale2, float ref, Weights<NT> (&pt)[MT / 2]) {
  float sum = 0.f;
#pragma unroll
  for (int st = 0; st < MT / 2; ++st) {
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = fast_exp2(fmaf(s[2 * st + i / 4][i % 4] - ref, qscale2, kHeadroom<NT>));
      sum += p[i];
    }
    pt[st].set(p);
  }
  return sum;
}
// Dimension tile dt of the weights times the value codes.
template <int D, int KU, int NT>
__device__ __forceinline__ f32x4a value_tile(const Unit<D, KU>& u, int dt, const Weights<NT> (&pt)[KU / 32]) {
  f32x4a acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int st = 0; st < KU / 32; ++st) acc = pt[st].times(u.template value<NT>(st, dt), acc);
  return acc;
}
// The same where a NaN value is seen by some columns and hidden from others (a
// weight of 0 does not hide it): a product for each column, without the codes
// that this column does not see.
template <int D, int KU, int NT>
__device__ __forceinline__ f32x4a value_tile_by_column(const Unit<D, KU>& u, int dt, const Weights<NT> (&pt)[KU / 32], int nkeys,
                                                       int grp) {
  f32x4a kept = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int c = 0; c < 16; ++c) {
    const int limit = __builtin_amdgcn_readlane(nkeys, c);
    f32x4a x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < KU / 32; ++st) x = pt[st].times(u.template value_below<NT>(st, dt, limit, grp), x);
#pragma unroll
    for (int i = 0; i < 4; ++i) kept[i] = (threadIdx.x & 15) == c ? x[i] : kept[i];
  }
  return kept;
}

// Running softmax of a wavefront's 16 columns over key units.  MIXED: the
// columns' visible keys differ (otherwise the hidden values' codes are cleared),
// and the units are of one block, whose values' scale is left to the caller;
// otherwise the values' sums are in units of kRowUnit.
template <int D, int KU, int NT>
struct Softmax {
  using U = Unit<D, KU>;
  f32x4a oacc[U::DT];
  float m = -INFINITY, l = 0.f;  // largest logit (before its scale), sum of weights

  __device__ __forceinline__ Softmax() {
#pragma unroll
    for (int dt = 0; dt < U::DT; ++dt) oacc[dt] = f32x4a{0.f, 0.f, 0.f, 0.f};
  }
  template <bool MIXED>
  __device__ __forceinline__ void add(U& u, const bf16x8a (&qt)[D / 32][NT], float qscale2, int nkeys, int grp) {
    const bool partial = MIXED ? __any(nkeys < KU) : nkeys < KU;
    if (!MIXED && partial) u.clear_from(nkeys, grp);
    f32x4a s[U::MT];
    unit_logits<D, KU, NT>(u, qt, partial, nkeys, grp, s);
    const float mn = fmaxf(m, column_max<U::MT>(s));
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float corr = fast_exp2((m - ref) * qscale2);
    m = mn;
    Weights<NT> pt[U::MT / 2];
    l = l * corr + weights<U::MT, NT>(s, qscale2, ref, pt);
    const bool by_column = MIXED && partial && u.nan_value();
    const float scale = MIXED ? 1.f : u.vsc * kRowUnit<NT>;
#pragma unroll
    for (int dt = 0; dt < U::DT; ++dt) {
      const f32x4a x = MIXED && by_column ? value_tile_by_column<D, KU, NT>(u, dt, pt, nkeys, grp) : value_tile<D, KU, NT>(u, dt, pt);
#pragma unroll
      for (int i = 0; i < 4; ++i) oacc[dt][i] = fmaf(x[i], scale, oacc[dt][i] * corr);
    }
  }
};

// Natural log of a row's sum of exponentials: largest logit, sum of weights.  The
// headroom leaves the sum before its logarithm, which is then that of a number from
// 1 on and keeps its bits.
template <int NT>
__device__ __forceinline__ float row_lse(float ref, float sum, float qscale2) {
  constexpr float unit = NT == 1 ? 0x1p-14f : 1.f;
  static_assert(unit * (1 << static_cast<int>(kHeadroom<NT>)) == 1.f);
  return sum == 0.f ? -INFINITY : fmaf(ref, qscale2, fast_log2(sum * unit)) * kLn2;
}

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
  auto fetch = [&](int task, Unit<D, KU>& u, int& visible) {
    for (; task < ntask; task += step) {
      const int slot = task / per, part = task - slot * per;
      const int blk = __builtin_amdgcn_readlane(slot < 64 ? sel0 : sel1, slot & 63);
      if (static_cast<uint32_t>(blk) >= static_cast<uint32_t>(a.M1)) continue;  // padding
      visible = min(KU, end - (blk * a.C + part * KU));
      if (visible <= 0) continue;
      u.load(a.c, static_cast<int64_t>(bh) * a.c.M + blk, a.C, part, col, grp);
      break;
    }
    return task;
  };
  Unit<D, KU> ua, ub;
  int na = 0, nb = 0;
  int ta = fetch(split * NW + wave, ua, na);
  bf16x8a qt[KS][NT];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) split_terms<NT>(qx[ks], qt[ks]);
  Softmax<D, KU, NT> sm;
  while (ta < ntask) {  // the next unit's loads are in flight while one is added
    const int tb = fetch(ta + step, ub, nb);
    sm.template add<false>(ua, qt, a.qscale2, na, grp);
    if (tb >= ntask) break;
    ta = fetch(tb + step, ua, na);
    sm.template add<false>(ub, qt, a.qscale2, nb, grp);
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
      const float f = fast_exp2((r[D] - ref) * a.qscale2);
      ll += r[D + 1] * f;
      oo += r[dd] * f;
    }
    if (a.splits == 1) {
      const int64_t orow = (static_cast<int64_t>(b) * a.H + h * a.G + hh) * a.Nq + row;
      const float res = ll == 0.f ? 0.f : oo / (ll * kRowUnit<NT>);
      if constexpr (sizeof(T) == 2)
        static_cast<uint16_t*>(a.o)[orow * D + dd] = f32_to_bf16_rne(res);
      else
        static_cast<float*>(a.o)[orow * D + dd] = res;
      if (a.lse && dd == 0) a.lse[orow] = row_lse<NT>(ref, ll, a.qscale2);
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
  constexpr int NT = sizeof(T) == 4 ? 3 : 1;
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
  const float f = fast_exp2((ml.x - ref) * a.qscale2);
  float ll = ml.y * f;
#pragma unroll
  for (int o = 1; o < kMaxSplits; o <<= 1) ll += __shfl_xor(ll, o);
  ll = __shfl(ll, 0);
  const float inv = ll == 0.f ? 0.f : 1.f / (ll * kRowUnit<NT>);
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
  if (a.lse && lane == 0) a.lse[orow] = row_lse<NT>(ref, ll, a.qscale2);
}

// Many rows (bf16): the (row, slot) pairs are grouped by key block, and a
// wavefront's 16 columns are the heads of 16 / G pairs of one block instead of
// one row's G heads: the block's codes are read once and turned into operands
// once for all of them.  Each pair leaves its own softmax of the block, normalised,
// in units of the values' scale (so at most 448) and rounded to fp16 (relative
// 2^-11; its largest logit and sum stay in fp32, apart: the logarithm of the sum
// would be lost in a large logit), and qcache_combine_kernel merges a row's K.
//   part_o [KV heads of the pass][its rows][K][G][D], within each 32 dimensions in the order
//   [grp][dimension tile 0..1][4], so that a lane stores 16 bytes at a time
constexpr int kBlockTiles = 8;  // tiles of a wavefront, at most

struct QBlockArgs {
  QAttnArgs a;
  const int32_t *offs, *toffs, *pairs;  // launch_cluster
  int64_t ncl;
  uint16_t* part_o;
  float2* part_ml;  // [KV heads][rows][K][G]: largest logit, sum of weights
  int nrows;  // rows of this pass, from a.row0 on
  int bh0;    // its first KV head of [0, BH)
  int chunk;  // pairs of one block per workgroup, at most
};

// WHOLE: a unit is a block, whose codes stay in registers (158 in all, three
// wavefronts on a SIMD; with the operands there instead, 256 and two, 4096 rows of
// 16 heads on 4 took 157 us in this kernel against 126 at that time); otherwise its
// units are read again, from the cache, for every tile.  What bounds it there (120
// us) is the partials' 268 MB out and the queries' 268 MB in, 4.5 TB/s; the vector
// units are busy 45% of that time and the matrix cores 12%.
template <int D, int KU, bool WHOLE>
__global__ __launch_bounds__(64, WHOLE ? (D == 128 ? 3 : 4) : 2) void qcache_block_kernel(QBlockArgs p) {
  constexpr int KS = D / 32, DT = D / 16;
  const QAttnArgs& a = p.a;
  int64_t cl;
  int beg, end;
  if (!cluster_chunk(p.offs, p.toffs, p.ncl, blockIdx.x, p.chunk, cl, beg, end)) return;
  const int pbh = static_cast<int>(cl / a.M1), blk = static_cast<int>(cl - static_cast<int64_t>(pbh) * a.M1);
  const int bh = p.bh0 + pbh;
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int col = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const int ppt = 16 / a.G;                // pairs of a tile
  const int cp = col / a.G, hh = col - cp * a.G;  // this column's pair and head
  const bool head = cp < ppt;
  const int per = a.C / KU;
  const int64_t cell = static_cast<int64_t>(bh) * a.c.M + blk;
  const int tok0 = blk * a.C;

  // the tiles' pairs are read up front, and the next tile's queries while one is
  // computed
  const int ntile = (end - beg + ppt - 1) / ppt;
  int words[kBlockTiles];
#pragma unroll
  for (int j = 0; j < kBlockTiles; ++j) {
    const int at = beg + j * ppt + cp;
    words[j] = head && at < end ? p.pairs[at] : -1;
  }
  Unit<D, KU> whole;
  if constexpr (WHOLE) whole.load(a.c, cell, a.C, 0, col, grp);
  uint4 qn[KS];
  auto gather = [&](int word) {
    const uint16_t* q = static_cast<const uint16_t*>(a.q) +
                        ((static_cast<int64_t>(b) * a.H + h * a.G + hh) * a.Nq + a.row0 + (word >> 8)) * D + grp * (D / 4);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qn[ks] = make_uint4(0, 0, 0, 0);
      if (word >= 0) qn[ks] = *reinterpret_cast<const uint4*>(q + ks * 8);
    }
  };
  gather(words[0]);
  if constexpr (WHOLE) {
    whole.clear_from(a.N - tok0, grp);
  }
#pragma unroll 1
  for (int j = 0; j < ntile; ++j) {
    bf16x8a qt[KS][1];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qt[ks][0] = u4_as_bf16x8(qn[ks]);
    const int word = words[0];
    const bool live = word >= 0;
    const int rr = live ? word >> 8 : 0, slot = word & 255;
    const int t = a.N - a.Nq + a.row0 + rr;
    const int visible = live ? (a.causal ? min(a.N, t + 1) : a.N) - tok0 : a.C;  // keys of the block
#pragma unroll
    for (int i = 0; i + 1 < kBlockTiles; ++i) words[i] = words[i + 1];
    if (j + 1 < ntile) gather(words[0]);
    uint16_t* dst = nullptr;
    const int64_t pidx = ((static_cast<int64_t>(pbh) * p.nrows + rr) * a.K + slot) * a.G + hh;
    if (live) dst = p.part_o + pidx * D + grp * 8;
    auto store = [&](int j, f32x4a x, f32x4a y, float inv) {  // dimension tiles 2j and 2j + 1
      uint4 w;
      w.x = pack2_f16(x[0] * inv, x[1] * inv);
      w.y = pack2_f16(x[2] * inv, x[3] * inv);
      w.z = pack2_f16(y[0] * inv, y[1] * inv);
      w.w = pack2_f16(y[2] * inv, y[3] * inv);
      if (live) *reinterpret_cast<uint4*>(dst + j * 32) = w;
    };
    float m, l, inv;
    auto close = [&] {  // the column's sum over its four lanes
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      inv = l == 0.f ? 0.f : 1.f / l;
    };
    if constexpr (WHOLE) {
      // one softmax per tile: its sum is known before the values, whose tiles are
      // stored as they come
      whole.pin();
      const int nkeys = min(KU, visible);
      const bool partial = __any(nkeys < KU);
      f32x4a s[KU / 16];
      unit_logits<D, KU, 1>(whole, qt, partial, nkeys, grp, s);
      m = column_max<KU / 16>(s);
      Weights<1> pt[KU / 32];
      l = weights<KU / 16, 1>(s, a.qscale2, m == -INFINITY ? 0.f : m, pt);
      close();
      if (partial && whole.nan_value()) {
#pragma unroll
        for (int dj = 0; dj < DT / 2; ++dj)
          store(dj, value_tile_by_column<D, KU, 1>(whole, 2 * dj, pt, nkeys, grp),
                value_tile_by_column<D, KU, 1>(whole, 2 * dj + 1, pt, nkeys, grp), inv);
      } else {
#pragma unroll
        for (int dj = 0; dj < DT / 2; ++dj)
          store(dj, value_tile<D, KU, 1>(whole, 2 * dj, pt), value_tile<D, KU, 1>(whole, 2 * dj + 1, pt), inv);
      }
    } else {
      Softmax<D, KU, 1> sm;
      for (int part = 0; part < per; ++part) {
        Unit<D, KU> u;
        u.load(a.c, cell, a.C, part, col, grp);
        u.clear_from(a.N - tok0 - part * KU, grp);
        sm.template add<true>(u, qt, a.qscale2, min(KU, visible - part * KU), grp);
      }
      m = sm.m;
      l = sm.l;
      close();
#pragma unroll
      for (int dj = 0; dj < DT / 2; ++dj) store(dj, sm.oacc[2 * dj], sm.oacc[2 * dj + 1], inv);
    }
    if (live && grp == 0) p.part_ml[pidx] = make_float2(m, l);
  }
}

// One wavefront per (row, head): 16 lanes hold a partial (8 values each for
// d = 128), so four slots at a time, and SPL rounds of them asked for before the
// first is used (4096 rows of 16 heads, 16 blocks: 64 us, 277 MB; with each
// round's values converted as they came, and so waited for, 89).
template <int D>
__global__ __launch_bounds__(256) void qcache_combine_kernel(QBlockArgs p) {
  constexpr int E = D / 16;
  constexpr int SPL = 4;  // rounds in flight
  const QAttnArgs& a = p.a;
  const int lane = threadIdx.x & 63;
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);  // heads of a row side by side, as its partials
  const int rr = static_cast<int>(e / a.G), hh = static_cast<int>(e - static_cast<int64_t>(rr) * a.G);
  if (rr >= p.nrows) return;
  const int grp = lane >> 4, sub = lane & 15;
  const int bh = p.bh0 + static_cast<int>(blockIdx.y), b = bh / a.Hkv;
  const int hq = (bh - b * a.Hkv) * a.G + hh;
  const int row = a.row0 + rr;
  const int32_t* sel = a.idx + (static_cast<int64_t>(bh) * a.Nq + row) * a.K;
  const int64_t base = (static_cast<int64_t>(blockIdx.y) * p.nrows + rr) * a.K;
  float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int s0 = grp; s0 < a.K; s0 += 4 * SPL) {
    int blk[SPL];
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
      const int x = s0 + 4 * i < a.K ? sel[s0 + 4 * i] : -1;
      blk[i] = static_cast<uint32_t>(x) < static_cast<uint32_t>(a.M1) ? x : -1;  // padding left no partial
    }
    float2 ml[SPL];
    float sc[SPL];
    uint32_t raw[SPL][E / 2];  // converted when all of them are asked for
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
      ml[i] = make_float2(-INFINITY, 0.f);
      sc[i] = 0.f;
#pragma unroll
      for (int e = 0; e < E / 2; ++e) raw[i][e] = 0;
      if (blk[i] >= 0) {
        const int64_t at = (base + s0 + 4 * i) * a.G + hh;
        ml[i] = p.part_ml[at];
        sc[i] = a.c.v_scale[static_cast<int64_t>(bh) * a.c.M + blk[i]];
        __builtin_memcpy(raw[i], __builtin_assume_aligned(p.part_o + at * D + sub * E, 2 * E), 2 * E);
      }
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < SPL; ++i) top = fmaxf(top, ml[i].x);
    const float ref = top == -INFINITY ? 0.f : top;
    const float f = fast_exp2((m - ref) * a.qscale2);
    l *= f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= f;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
      const float w = ml[i].y * fast_exp2((ml[i].x - ref) * a.qscale2);
      l += w;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const _Float16 x = __builtin_bit_cast(f16x2a, raw[i][e / 2])[e % 2];
        o[e] = fmaf(w * (sc[i] * kRowUnit<1>), static_cast<float>(x), o[e]);
      }
    }
    m = top;
  }
#pragma unroll
  for (int msk = 16; msk <= 32; msk <<= 1) {
    const float m2 = __shfl_xor(m, msk), l2 = __shfl_xor(l, msk);
    const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
    const float f = fast_exp2((m - ref) * a.qscale2), f2 = fast_exp2((m2 - ref) * a.qscale2);
    l = l * f + l2 * f2;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + __shfl_xor(o[e], msk) * f2;
    m = top;
  }
  if (grp == 0) {
    const float inv = l == 0.f ? 0.f : 1.f / (l * kRowUnit<1>);
    const int64_t orow = (static_cast<int64_t>(b) * a.H + hq) * a.Nq + row;
    uint16_t* dst = static_cast<uint16_t*>(a.o) + orow * D;
    // value i of this lane's part is at position sub*E + i of the stored order
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const int pos = sub * E + e;
      const int d = pos / 32 * 32 + (pos & 4) * 4 + (pos % 32) / 8 * 4;
      *reinterpret_cast<uint2*>(dst + d) = make_uint2(pack2_bf16(o[e] * inv, o[e + 1] * inv), pack2_bf16(o[e + 2] * inv, o[e + 3] * inv));
    }
    if (a.lse && sub == 0) a.lse[orow] = row_lse<1>(m, l, a.qscale2);
  }
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

static size_t al256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// Partials of one pass take about 1 GB.  A pass takes all rows of some KV heads,
// so that their blocks are grouped once, and only where those of one KV head are
// more than that does it take a part of them.  (Passes over a part of the rows of
// every KV head group all blocks each time: 2048 rows of 32 x 8 KV heads over
// 131072 keys took 26.5 ms that way, 7.4 this way.)
constexpr size_t kPartialBytes = size_t(1) << 30;
struct BlockPass {
  int heads, rows;       // of a pass, at most
  int hpasses, rpasses;  // passes over KV heads, and over the rows of each
};
static BlockPass block_pass(const Shape& s) {
  const size_t row = static_cast<size_t>(s.K) * s.G * (s.D * 2 + 4);  // a KV head's row
  const int most = static_cast<int>(std::max<size_t>(kPartialBytes / row, 1));
  auto div_up = [](int x, int y) { return (x + y - 1) / y; };
  BlockPass b{};
  b.rpasses = div_up(s.Nq, most);
  b.rows = div_up(s.Nq, b.rpasses);
  b.hpasses = div_up(s.BH(), std::max(1, most / s.Nq));
  b.heads = div_up(s.BH(), b.hpasses);
  return b;
}

// Does grouping the rows by block pay?  A row alone reads its K blocks, of 2 C D
// bytes, at about 10 TB/s over all; grouped, a block is read once for many rows,
// but each (row, slot) writes and reads back a partial of 2 D bytes a head (0.25
// ns per KB and 64 keys of the block), a pass costs 36 us, and the grouping 2.5 ns
// per block of every KV head, again for each part of its rows.  Measured, alone
// and grouped (us): 128-wide heads, 16 blocks of 64 keys, 32768 keys, 4 heads to a
// KV head: 2048 rows x KV heads 62 and 56, 4096 109 and 69, 16384 373 and 203; 1
// head: 2048 58 and 51, 16384 367 and 78; 8 heads: 2048 63 and 67, 8192 207 and
// 187; 16 heads of 64, 8 blocks: 8192 61 and 131; over 524288 keys, 4 heads: 4096
// 135 and 194, 16384 481 and 317.  Several passes, 4 heads, 131072 keys: 2048 rows
// of 32 x 8 KV heads (9 passes) 21105 and 7436, 512 of 64 x 8 (5) 11620 and 7746,
// 32768 of 8 (8) 6066 and 3221.  Over 177 shapes of 256 to 524288 rows the mean
// time is 0.3% above that of the faster choice for each.
static bool use_blocks(const Shape& s, const Geo& geo) {
  if (!s.bf16 || geo.M[1] > 16384) return false;  // the grouping's LDS histogram
  if (static_cast<int64_t>(s.BH()) * geo.M[1] > (1 << 23)) return false;  // a workgroup per block fits one launch
  const double rows = static_cast<double>(s.BH()) * s.Nq;
  const double saved = rows * s.K * s.D / 1024 * (0.2 * s.C - s.G * std::max(1.0, s.C / 64.0));
  const BlockPass b = block_pass(s);
  return saved >= b.rpasses * (36000.0 * b.hpasses + 2.5 * s.BH() * geo.M[1]);
}

// Rows per workgroup of the grouping: about 4096 pairs (262144 pairs on 4 KV heads:
// 21 us for the grouping, 35 with 1024 rows).
static int group_rows(const Shape& s) { return std::max(64, 4096 / s.K); }
// Pairs of one block per wavefront.  Workgroups of one (4096 rows of 8 heads on 8,
// 16 blocks of 131072 keys: 103 us in this kernel; 4 wavefronts of 4 tiles 150, 2 of
// 8 113, one of 16 106).
static int pair_chunk(const Shape& s) { return 16 / s.G * kBlockTiles; }
struct BlockWs {
  size_t part_o, part_ml, cl, total;
};
static BlockWs block_layout(const Shape& s, const Geo& geo) {
  const BlockPass b = block_pass(s);
  const size_t np = static_cast<size_t>(b.heads) * b.rows * s.K;
  BlockWs w{};
  w.part_ml = al256(np * s.G * s.D * 2);
  w.cl = w.part_ml + al256(np * s.G * sizeof(float2));
  w.total = w.cl + al256(cluster_ws(b.heads, geo.M[1], static_cast<int64_t>(np), b.rows, group_rows(s)));
  return w;
}

template <int D>
static hipError_t launch_blocks(const Shape& s, const Geo& geo, const QAttnArgs& a, char* base, int ku, hipStream_t st) {
  const BlockWs w = block_layout(s, geo);
  const BlockPass bp = block_pass(s);
  QBlockArgs p{};
  p.a = a;
  p.part_o = reinterpret_cast<uint16_t*>(base + w.part_o);
  p.part_ml = reinterpret_cast<float2*>(base + w.part_ml);
  p.chunk = pair_chunk(s);
  for (int bh0 = 0; bh0 < s.BH(); bh0 += bp.heads) {
    const int heads = std::min(bp.heads, s.BH() - bh0);
    p.bh0 = bh0;
    for (int row0 = 0; row0 < s.Nq; row0 += bp.rows) {
      p.a.row0 = row0;
      p.nrows = std::min(bp.rows, s.Nq - row0);
      ClusterArgs ca{a.idx + static_cast<int64_t>(bh0) * s.Nq * s.K, nullptr, s.K, s.Nq, s.N, s.C, s.K, s.causal, geo.M[1],
                     kClusterAttn, row0, p.nrows, s.g};
      ca.chunk_rows = group_rows(s);
      ClusterOut co{};
      hipError_t e = launch_cluster(ca, heads, base + w.cl, &co, st, p.chunk);
      if (e != hipSuccess) return e;
      p.offs = co.offs;
      p.toffs = co.toffs;
      p.pairs = co.pairs;
      p.ncl = co.ncl;
      {
        ProfScope ps("qcache_block", st);
        const unsigned grid = static_cast<unsigned>(
            cluster_max_chunks(heads, geo.M[1], static_cast<int64_t>(heads) * p.nrows * s.K, p.chunk));
        if (s.C == 64)
          qcache_block_kernel<D, 64, true><<<grid, 64, 0, st>>>(p);
        else if (s.C == 32)
          qcache_block_kernel<D, 32, true><<<grid, 64, 0, st>>>(p);
        else if (ku == 64)
          qcache_block_kernel<D, 64, false><<<grid, 64, 0, st>>>(p);
        else
          qcache_block_kernel<D, 32, false><<<grid, 64, 0, st>>>(p);
      }
      {
        ProfScope ps("qcache_combine", st);
        qcache_combine_kernel<D><<<dim3(static_cast<unsigned>((static_cast<int64_t>(p.nrows) * s.G + 3) / 4), heads), 256, 0, st>>>(p);
      }
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

static size_t part_ml_at(const Shape& s, int splits) {
  return (static_cast<size_t>(s.BH()) * s.Nq * splits * s.G * s.D * sizeof(float) + 255) & ~static_cast<size_t>(255);
}

size_t qcache_attn_ws(const Shape& s, const Geo& geo) {
  if (use_blocks(s, geo)) return block_layout(s, geo).total;
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
  if (use_blocks(s, geo))
    return s.D == 128 ? launch_blocks<128>(s, geo, a, base, ku, st) : launch_blocks<64>(s, geo, a, base, ku, st);
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
