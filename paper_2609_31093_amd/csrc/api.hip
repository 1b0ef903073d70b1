// C ABI of libpisa: argument validation, hierarchy geometry, workspace sizing
// and dispatch to the kernels.  Nothing is enqueued before every argument has
// been checked; no call allocates device memory or synchronises.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <iterator>
#include <mutex>

#include "../../include/pisa.h"
#include "common.h"
#include "kernels.h"

namespace {

thread_local char g_last_error[512] = "";

int fail(int status, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
  va_end(ap);
  return status;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Level sizes M[1..L] of an N-token hierarchy (Sec. 3.2 eq. key_hierarchy);
// returns L or a negative status.
int level_sizes(int64_t N, int32_t C, int32_t g, int32_t* M) {
  int64_t m = (N + C - 1) / C;
  int L = 1;
  M[1] = static_cast<int32_t>(m);
  while (m > 1) {
    m = (m + g - 1) / g;
    ++L;
    if (L > pisa::kMaxLevels) return PISA_ERR_UNSUPPORTED;
    M[L] = static_cast<int32_t>(m);
  }
  return L;
}

// Geometry of an N-token problem whose pyramid (and k/v rows) are laid out
// for cap >= N tokens.
int compute_geo(int32_t N, int32_t C, int32_t g, pisa::Geo* geo, int32_t cap = 0) {
  if (N < 1 || C < 1 || g < 2) return PISA_ERR_INVALID_ARG;
  if (cap == 0) cap = N;
  if (cap < N) return PISA_ERR_INVALID_ARG;
  pisa::Geo G{};
  G.N = N;
  G.Nkv = cap;
  G.C = C;
  G.g = g;
  const int L = level_sizes(N, C, g, G.M);
  if (L < 0) return L;
  int32_t Mc[pisa::kMaxLevels + 1] = {};
  const int Lc = level_sizes(cap, C, g, Mc);
  if (Lc < 0) return Lc;
  G.L = L;
  G.Lstore = L > 1 ? L - 1 : 1;
  G.lg = -1;
  for (int b = 0; b < 31; ++b)
    if ((1 << b) == g) G.lg = b;
  G.gpow[1] = 1;
  G.gp[1] = 1;
  for (int l = 2; l <= pisa::kMaxLevels; ++l)
    G.gp[l] = G.gp[l - 1] > (1 << 26) ? (1 << 30) : G.gp[l - 1] * g;
  for (int l = 2; l <= pisa::kMaxLevels; ++l)  // saturate beyond the root
    G.gpow[l] = G.gpow[l - 1] > (int64_t(1) << 40) ? G.gpow[l - 1] : G.gpow[l - 1] * g;
  // Row offsets of the capacity layout: levels 1 .. max(1, Lc - 1) of a
  // cap-token hierarchy (which contain the stored levels of N).
  const int Lcs = Lc > 1 ? Lc - 1 : 1;
  G.off[1] = 0;
  for (int l = 1; l <= pisa::kMaxLevels; ++l) G.off[l + 1] = G.off[l] + (l <= Lcs ? Mc[l] : 0);
  G.R = G.off[Lcs + 1];
  if (geo) *geo = G;
  return L;
}

// Leaf blocks of the capacity (Ncap tokens) a problem may reserve.
constexpr int32_t kMaxLeafBlocks = 65535;

// Full validation of a problem; fills the kernel view on success.
int check_problem(const pisa_problem* p, pisa::Shape* s, pisa::Geo* geo) {
  if (!p) return fail(PISA_ERR_INVALID_ARG, "problem is NULL");
  if (p->B < 1 || p->H < 1 || p->Hkv < 1)
    return fail(PISA_ERR_INVALID_ARG, "B, H and Hkv must be >= 1 (got %d, %d, %d)", p->B, p->H, p->Hkv);
  if (p->H % p->Hkv != 0)
    return fail(PISA_ERR_INVALID_ARG, "H (%d) must be a multiple of Hkv (%d)", p->H, p->Hkv);
  if (p->N < 1 || p->Nq < 1 || p->Nq > p->N)
    return fail(PISA_ERR_INVALID_ARG, "need 1 <= Nq <= N (got Nq=%d, N=%d)", p->Nq, p->N);
  if (p->C < 1 || p->fanout < 2 || p->K < 1)
    return fail(PISA_ERR_INVALID_ARG, "need C >= 1, fanout >= 2, K >= 1 (got %d, %d, %d)", p->C, p->fanout,
                p->K);
  if (p->causal != 0 && p->causal != 1) return fail(PISA_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (p->causal && p->K < 3)
    return fail(PISA_ERR_INVALID_ARG, "causal selection keeps the first, previous and current blocks: K >= 3");
  if (p->dtype != PISA_DTYPE_F32 && p->dtype != PISA_DTYPE_BF16)
    return fail(PISA_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  if (p->schedule < PISA_SCHEDULE_AUTO || p->schedule > PISA_SCHEDULE_SPLIT)
    return fail(PISA_ERR_INVALID_ARG, "unknown schedule %d", p->schedule);
  if (p->d != 64 && p->d != 128) return fail(PISA_ERR_UNSUPPORTED, "head dim %d (supported: 64, 128)", p->d);
  if (p->C % 32 != 0 || p->C > pisa::kMaxLeafKeys)
    return fail(PISA_ERR_UNSUPPORTED, "block size %d (supported: multiples of 32 up to 256)", p->C);
  if (p->fanout > 16) return fail(PISA_ERR_UNSUPPORTED, "fanout %d (supported: 2..16)", p->fanout);
  const int G = p->H / p->Hkv;
  if (G > 16) return fail(PISA_ERR_UNSUPPORTED, "group size H/Hkv = %d (supported: <= 16)", G);
  if (static_cast<int64_t>(p->fanout) * p->K > pisa::kMaxCand)
    return fail(PISA_ERR_UNSUPPORTED, "fanout*K = %lld exceeds %d", static_cast<long long>(p->fanout) * p->K,
                pisa::kMaxCand);
  if (static_cast<int64_t>(p->fanout) * p->fanout * p->K * G > 2048)
    return fail(PISA_ERR_UNSUPPORTED, "fanout^2*K*G = %lld exceeds 2048",
                static_cast<long long>(p->fanout) * p->fanout * p->K * G);
  if (p->Nq >= (1 << 23)) return fail(PISA_ERR_UNSUPPORTED, "Nq %d exceeds 2^23-1", p->Nq);
  if (static_cast<int64_t>(p->B) * p->Hkv > 65535 || static_cast<int64_t>(p->B) * p->H > 65535)
    return fail(PISA_ERR_UNSUPPORTED, "B*H must be <= 65535");
  if (p->score < PISA_SCORE_LSE || p->score > PISA_SCORE_MEAN_VAR)
    return fail(PISA_ERR_INVALID_ARG, "unknown score %d", p->score);
  if (p->Ncap != 0 && p->Ncap < p->N)
    return fail(PISA_ERR_INVALID_ARG, "Ncap (%d) must be 0 or >= N (%d)", p->Ncap, p->N);
  pisa::Geo g{};
  const int L = compute_geo(p->N, p->C, p->fanout, &g, p->Ncap);
  if (L < 0) return fail(L, "hierarchy too deep");
  if ((static_cast<int64_t>(g.Nkv) + p->C - 1) / p->C > kMaxLeafBlocks)
    return fail(PISA_ERR_UNSUPPORTED, "more than %d leaf blocks", kMaxLeafBlocks);
  if (s) {
    s->B = p->B;
    s->H = p->H;
    s->Hkv = p->Hkv;
    s->G = G;
    s->Nq = p->Nq;
    s->N = p->N;
    s->D = p->d;
    s->C = p->C;
    s->g = p->fanout;
    s->K = p->K;
    s->causal = p->causal;
    s->Nkv = g.Nkv;
    s->score = p->score;
    s->bf16 = p->dtype == PISA_DTYPE_BF16;
  }
  if (geo) *geo = g;
  return PISA_OK;
}

int check_ptr(const void* ptr, const char* name, bool nullable = false) {
  if (!ptr) return nullable ? PISA_OK : fail(PISA_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned16(ptr)) return fail(PISA_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return PISA_OK;
}

// The same for what kernels read or write a value at a time.
int check_values(const void* ptr, const char* name, unsigned size, bool nullable = false) {
  if (!ptr) return nullable ? PISA_OK : fail(PISA_ERR_INVALID_ARG, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(ptr) % size) return fail(PISA_ERR_INVALID_ARG, "%s is not %u-byte aligned", name, size);
  return PISA_OK;
}

bool aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }

int check_ws(void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return PISA_OK;
  if (ws_bytes < need)
    return fail(PISA_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", ws_bytes, need);
  if (!ws) return fail(PISA_ERR_WORKSPACE, "workspace is NULL, need %zu bytes", need);
  if (!aligned256(ws)) return fail(PISA_ERR_INVALID_ARG, "workspace not 256-byte aligned");
  return PISA_OK;
}

int device_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return PISA_OK;
  return fail(PISA_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

// The cluster histogram of the two-stage schedule lives in LDS (one int per
// leaf block).
constexpr int kMaxClusterBins = 16384;

// Rows (query rows x batch x KV heads) up to which the automatic schedule
// spreads each row's leaf candidates over workgroups of their own.
constexpr int64_t kSplitMaxRows = 2048;

// Fewer rows than kTwoStageRows: does grouping the leaf pairs by key block
// pay?  Only rows of one (batch, KV head) share its key blocks, and the
// grouping costs 30 us and more, the longer the more pairs a head has (few
// workgroups count and place them), against leaf scores that the split
// schedule (up to 2048 rows) or the fused one spreads over the device.
//   * pairs, those of one head, against its key blocks.  One row to a
//     block is enough where several heads of the row want it too, two for a
//     single head; half a row above the split schedule's range.  Decode, however
//     many sequences, has no two (512 KV heads x 1 row of 4 heads, 131072 keys:
//     127 us split, 1508 grouped; 16 x 64 rows, 32768 keys: 155 and 122).
//   * work = keys x dims x heads of one row's scored candidates, over the KV
//     heads: many short lists are spread widely either way (d = 64, g*K = 16,
//     4000 rows of one head on one KV head: 33 us fused, 100 grouped), long or
//     wide ones are not (2048 rows of 4 heads on one KV head, g*K = 128,
//     128-key blocks over 131072 keys: 1562 split, 527 grouped).  Up to 1024
//     rows of one KV head are counted by so few workgroups that it takes four
//     times the work (4 heads, g*K = 32, 8192 keys, 1024 rows: 131 and 203;
//     2048: 247 and 218).
//   * Lists of at most 16 candidates (8 with more than four heads) have fused
//     kernels of their own and want more of both (g*K = 8, d = 128, 2 x 1050
//     rows of 4 heads: 45 fused, 129 grouped; 128 x 17 of 16: 423 and 81).
//   * More than four heads, where no other kernel shares loads among them: above
//     the split schedule's range already where a third of a head per block is
//     shared (16 heads, g*K = 16, 2100 KV heads x 1 row over 33, 129 and 513
//     blocks: 1096, 1226 and 1370 fused, 537, 876 and 1959 grouped).
// Over 7298 shapes of 512 to 4095 rows (1 to 300 KV heads, 8 to 256 candidates,
// 32- to 256-key blocks) the mean time is 1.0% above that of the faster
// schedule for each; grouping them all is 6.2% above it.
bool two_stage_pays(const pisa::Shape& s, const pisa::Geo& g, int64_t rows) {
  const int64_t M1 = g.M[1], scored = std::min<int64_t>(s.gK(), M1) - s.K;
  if (scored <= 0) return false;
  const int64_t pairs = s.Nq * scored, work = static_cast<int64_t>(s.BH()) * s.G * s.C * s.D * scored;
  if (rows <= kSplitMaxRows) {
    if (s.G > 4 || rows * s.G < kSplitMaxRows) return false;
    const int64_t least = (s.G <= 2 ? 224 << 10 : 384 << 10) * (s.BH() == 1 && rows <= 1024 ? 4 : 1);
    return pairs >= (s.G == 1 ? 2 : 1) * M1 && work >= least;
  }
  if (s.gK() <= (s.G <= 4 ? 16 : 8)) return pairs >= 2 * M1 && work >= (s.G <= 4 ? 2 << 20 : 4 << 20);
  if (s.G > 4) return 3 * s.G * pairs >= M1;
  return 2 * pairs >= M1 && work >= 64 << 10;
}

// From this many rows the automatic schedule insists on the two-stage
// workspace; below it a smaller one gets the other schedules.
constexpr int64_t kTwoStageRows = 4096;

// small_ws: the choice for a caller without the two-stage workspace.
int pick_schedule(const pisa_problem* p, const pisa::Shape& s, const pisa::Geo& g, bool small_ws = false) {
  if (p->schedule != PISA_SCHEDULE_AUTO) return p->schedule;
  const int64_t rows = static_cast<int64_t>(s.Nq) * s.BH();
  if (s.bf16 && g.M[1] <= kMaxClusterBins && (rows >= kTwoStageRows || (!small_ws && two_stage_pays(s, g, rows))))
    return PISA_SCHEDULE_TWO_STAGE;
  return rows <= kSplitMaxRows ? PISA_SCHEDULE_SPLIT : PISA_SCHEDULE_FUSED;
}

size_t select_ws(int sched, const pisa::Shape& s, const pisa::Geo& g) {
  if (sched == PISA_SCHEDULE_TWO_STAGE) return pisa::select_two_stage_ws(s, g);
  if (sched == PISA_SCHEDULE_SPLIT) return pisa::select_split_ws(s, g);
  return 0;
}

// The workspace that the call insists on (a split selection is faster with
// all of select_ws()).
size_t select_ws_min(int sched, const pisa::Shape& s, const pisa::Geo& g) {
  return sched == PISA_SCHEDULE_SPLIT ? pisa::select_split_ws_min(s) : select_ws(sched, s, g);
}

// Settles the schedule for a workspace with ws_bytes of use (none where it is
// NULL or misaligned), and how its stage 1 runs.
int schedule_for_ws(const pisa_problem* p, pisa::Shape* s, const pisa::Geo& g, int sched, size_t ws_bytes) {
  if (ws_bytes < select_ws_min(sched, *s, g)) sched = pick_schedule(p, *s, g, true);
  s->plain_stage1 = p->schedule == PISA_SCHEDULE_AUTO && static_cast<int64_t>(s->Nq) * s->BH() < kTwoStageRows;
  return sched;
}

#define PISA_TRY(x)           \
  do {                        \
    const int _st = (x);      \
    if (_st != PISA_OK) return _st; \
  } while (0)

// Argument checks of pisa_select and pisa_select_static (everything except
// the workspace); fills the kernel view and the schedule.
int check_select(const pisa_problem* p, const void* q, const void* k, const float* pyramid, const int32_t* block_idx,
                 const float* block_score, pisa::Shape* s, pisa::Geo* g, int* sched) {
  PISA_TRY(check_problem(p, s, g));
  PISA_TRY(check_ptr(q, "q"));
  PISA_TRY(check_ptr(k, "k"));
  PISA_TRY(check_ptr(pyramid, "pyramid"));
  PISA_TRY(check_ptr(block_idx, "block_idx"));
  PISA_TRY(check_ptr(block_score, "block_score", true));
  *sched = pick_schedule(p, *s, *g);
  const bool two = *sched == PISA_SCHEDULE_TWO_STAGE;
  if (two && !s->bf16)
    return fail(PISA_ERR_UNSUPPORTED, "the two-stage schedule runs on bf16 inputs (use the fused schedule)");
  if (two && g->M[1] > kMaxClusterBins)
    return fail(PISA_ERR_UNSUPPORTED, "the two-stage schedule needs N/C <= %d", kMaxClusterBins);
  return PISA_OK;
}

int run_select(const pisa::Shape& s, const pisa::Geo& g, int sched, const void* q, const void* k,
               const float* pyramid, int32_t* block_idx, float* block_score, void* ws, size_t ws_bytes,
               hipStream_t st, const char* who) {
  hipError_t e;
  if (sched == PISA_SCHEDULE_TWO_STAGE)
    e = pisa::launch_select_two_stage(s, g, q, k, pyramid, block_idx, block_score, ws, st);
  else if (sched == PISA_SCHEDULE_SPLIT)
    e = pisa::launch_select_split(s, g, q, k, pyramid, block_idx, block_score, ws, ws_bytes, st);
  else
    e = pisa::launch_select_fused(s, g, q, k, pyramid, block_idx, block_score, st);
  return device_status(e, who);
}

// Per-device address of the static scratch of pisa_select_static, taken once
// per device (with that device current) on its first call there.
constexpr int kMaxDevices = 64;
std::once_flag g_scratch_once[kMaxDevices];
void* g_scratch_ptr[kMaxDevices];
hipError_t g_scratch_err[kMaxDevices];

}  // namespace

namespace pisa {
// Scratch of pisa_select_static: one copy per device, held while the library
// is loaded.  Host code never passes this name to a kernel or a copy (on the
// host it only names the symbol); it uses the device address from
// hipGetSymbolAddress instead.
__device__ __align__(256) unsigned char scratch[PISA_STATIC_SCRATCH_BYTES];
}  // namespace pisa

namespace {

int static_scratch(void** out) {
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return device_status(e, "hipGetDevice");
  if (dev < 0 || dev >= kMaxDevices) return fail(PISA_ERR_UNSUPPORTED, "device %d (supported: < %d)", dev, kMaxDevices);
  std::call_once(g_scratch_once[dev], [dev] {
    void* ptr = nullptr;
    g_scratch_err[dev] = hipGetSymbolAddress(&ptr, HIP_SYMBOL(pisa::scratch));
    g_scratch_ptr[dev] = ptr;
  });
  if (g_scratch_err[dev] != hipSuccess) return device_status(g_scratch_err[dev], "hipGetSymbolAddress(scratch)");
  if (!aligned256(g_scratch_ptr[dev]))
    return fail(PISA_ERR_DEVICE, "static scratch is not 256-byte aligned");
  *out = g_scratch_ptr[dev];
  return PISA_OK;
}

// Are there two rows of d values less than d apart?  They are `off` plus, for each
// dimension from `at` on (largest stride first), its stride times a difference of
// indexes within [lo, hi].  `same`: no difference so far, where a row is not to be
// compared with itself.  Where no stride is less than what the smaller ones span,
// each dimension leaves a few differences to look at; after `steps` of them the
// rows count as meeting.
struct IndexRange {
  int64_t stride, lo, hi;
};
bool rows_meet(const IndexRange (&dim)[3], int at, __int128 off, int d, bool same, int* steps) {
  if (at == 3) return off > -d && off < d && !same;
  __int128 reach = d - 1;  // of the dimensions behind this one
  for (int i = at + 1; i < 3; ++i) reach += static_cast<__int128>(dim[i].stride) * std::max(-dim[i].lo, dim[i].hi);
  const int64_t st = dim[at].stride;
  int64_t lo = dim[at].lo, hi = dim[at].hi;
  if (reach + (off < 0 ? -off : off) < st) {  // the usual case, without divisions
    lo = std::max<int64_t>(lo, 0);
    hi = std::min<int64_t>(hi, 0);
  } else if (st > 0) {
    auto floor_div = [&](__int128 x) { return x >= 0 ? x / st : -((-x + st - 1) / st); };
    lo = static_cast<int64_t>(std::max<__int128>(lo, -floor_div(reach + off)));
    hi = static_cast<int64_t>(std::min<__int128>(hi, floor_div(reach - off)));
  }
  for (int64_t i = lo; i <= hi; ++i)
    if (--*steps < 0 || rows_meet(dim, at + 1, off + static_cast<__int128>(st) * i, d, same && i == 0, steps)) return true;
  return false;
}
constexpr int kMeetSteps = 10000;

// Strides of a [B, heads, rows, d] tensor (the contiguous ones where NULL).
// Written tensors keep their rows apart.
int check_strides(const pisa_strides* in, const char* name, int64_t B, int64_t heads, int64_t rows, int d, int dtype,
                  bool written, pisa_strides* out) {
  if (!in) {
    *out = pisa_strides{heads * rows * d, rows * d, d};
    return PISA_OK;
  }
  const int unit = dtype == PISA_DTYPE_BF16 ? 8 : 4;
  for (const int64_t x : {in->b, in->h, in->n})
    if (x < 0 || x % unit != 0)
      return fail(PISA_ERR_INVALID_ARG, "strides of %s must be non-negative multiples of 16 bytes (got %lld elements)", name,
                  static_cast<long long>(x));
  if (written) {
    IndexRange dim[3] = {{in->b, 1 - B, B - 1}, {in->h, 1 - heads, heads - 1}, {in->n, 1 - rows, rows - 1}};
    std::sort(dim, dim + 3, [](const IndexRange& x, const IndexRange& y) { return x.stride > y.stride; });
    int steps = kMeetSteps;
    if (rows_meet(dim, 0, 0, d, true, &steps)) return fail(PISA_ERR_INVALID_ARG, "strides of %s make its rows overlap", name);
  }
  *out = *in;
  return PISA_OK;
}

int check_rope(const pisa_rope* r) {
  if (!r) return fail(PISA_ERR_INVALID_ARG, "rope is NULL");
  if (r->B < 1 || r->H < 1 || r->Hkv < 1 || r->N < 1)
    return fail(PISA_ERR_INVALID_ARG, "B, H, Hkv and N must be >= 1 (got %d, %d, %d, %d)", r->B, r->H, r->Hkv, r->N);
  if (r->d != 64 && r->d != 128) return fail(PISA_ERR_UNSUPPORTED, "head dim %d (supported: 64, 128)", r->d);
  if (r->rot < 2 || r->rot > r->d || r->rot % 2 != 0)
    return fail(PISA_ERR_INVALID_ARG, "rot must be even and in [2, d] (got %d, d=%d)", r->rot, r->d);
  if (r->layout != PISA_ROPE_HALF && r->layout != PISA_ROPE_INTERLEAVED)
    return fail(PISA_ERR_INVALID_ARG, "unknown layout %d", r->layout);
  if (r->dtype != PISA_DTYPE_F32 && r->dtype != PISA_DTYPE_BF16)
    return fail(PISA_ERR_INVALID_ARG, "unknown dtype %d", r->dtype);
  if (r->reserved != 0) return fail(PISA_ERR_INVALID_ARG, "reserved must be 0");
  if (r->pos_bstride < 0) return fail(PISA_ERR_INVALID_ARG, "pos_bstride must be >= 0");
  if (!isfinite(r->amplitude)) return fail(PISA_ERR_INVALID_ARG, "amplitude is not finite");
  for (int i = 0; i < r->rot / 2; ++i)
    if (!(fabs(r->freq[i]) <= 1e6)) return fail(PISA_ERR_INVALID_ARG, "freq[%d] is not a number within 10^6", i);
  if (static_cast<int64_t>(r->pos0) + r->N > INT32_MAX) return fail(PISA_ERR_UNSUPPORTED, "positions past 2^31-1");
  if (static_cast<int64_t>(r->B) * r->N > (int64_t(1) << 28)) return fail(PISA_ERR_UNSUPPORTED, "B*N exceeds 2^28");
  if (static_cast<int64_t>(r->H) + r->Hkv > 65535) return fail(PISA_ERR_UNSUPPORTED, "H + Hkv exceeds 65535");
  return PISA_OK;
}

// One side (queries or keys) of a rotation; both pointers NULL leave it out.
int check_rope_side(const pisa_rope* r, const char* name, int heads, const void* in, const pisa_strides* is, void* out,
                    const pisa_strides* os, pisa::RopeSide* side) {
  if (!in && !out) return PISA_OK;
  char nout[32];
  snprintf(nout, sizeof(nout), "%s (output)", name);
  PISA_TRY(check_ptr(in, name));
  PISA_TRY(check_ptr(out, nout));
  pisa_strides si, so;
  PISA_TRY(check_strides(is, name, r->B, heads, r->N, r->d, r->dtype, false, &si));
  PISA_TRY(check_strides(os, nout, r->B, heads, r->N, r->d, r->dtype, true, &so));
  if (in == out && ((r->B > 1 && si.b != so.b) || (heads > 1 && si.h != so.h) || (r->N > 1 && si.n != so.n)))
    return fail(PISA_ERR_INVALID_ARG, "%s in place needs the same strides for input and output", name);
  *side = pisa::RopeSide{in, out, si.b, si.h, si.n, so.b, so.h, so.n};
  return PISA_OK;
}

// A [B, heads, rows, d] tensor where it lies.
struct Placed {
  const void* ptr;
  pisa_strides s;
  int64_t B, heads, rows;
};
// Do two tensors share memory?  Those whose spans meet but whose strides are
// alike (two parts of a packed projection) are compared row by row as rows_meet
// does; other strides count as sharing.
bool share(const Placed& x, const Placed& y, int d, int64_t esz) {
  auto span = [&](const Placed& t) {
    return (static_cast<__int128>(t.B - 1) * t.s.b + static_cast<__int128>(t.heads - 1) * t.s.h +
            static_cast<__int128>(t.rows - 1) * t.s.n + d) * esz;
  };
  const __int128 at = static_cast<__int128>(reinterpret_cast<uintptr_t>(y.ptr)) - reinterpret_cast<uintptr_t>(x.ptr);
  if (at >= span(x) || -at >= span(y)) return false;
  IndexRange dim[3];
  const int64_t ex[3] = {x.B, x.heads, x.rows}, ey[3] = {y.B, y.heads, y.rows};
  const int64_t sx[3] = {x.s.b, x.s.h, x.s.n}, sy[3] = {y.s.b, y.s.h, y.s.n};
  for (int i = 0; i < 3; ++i) {
    if (ex[i] > 1 && ey[i] > 1 && sx[i] != sy[i]) return true;
    dim[i] = {ex[i] > 1 ? sx[i] : sy[i], 1 - ex[i], ey[i] - 1};
  }
  std::sort(dim, dim + 3, [](const IndexRange& a, const IndexRange& b) { return a.stride > b.stride; });
  int steps = kMeetSteps;
  return rows_meet(dim, 0, at / esz, d, false, &steps);
}

// What a rotation's kernels take from its descriptor; sides are filled in already.
void fill_rope(const pisa_rope* r, const int32_t* positions, float sign, pisa::RopeArgs* a) {
  a->positions = positions;
  a->pos_bstride = r->pos_bstride;
  a->B = r->B;
  a->H = a->q.in ? r->H : 0;
  a->HH = a->H + (a->k.in ? r->Hkv : 0);
  a->N = r->N;
  a->d = r->d;
  a->rot = r->rot;
  a->pos0 = r->pos0;
  a->amplitude = static_cast<float>(r->amplitude);
  a->sign = sign;
  for (int i = 0; i < r->rot / 2; ++i) a->turn[i] = r->freq[i] / 6.283185307179586476925286766559;
}

// Rows are read and written in one launch, in any order: an output (side i's) meets
// no input, but its own in place, and no other output.
int check_rope_overlaps(const pisa_rope* r, const pisa::RopeSide (&side)[2], const char* const (&names)[2]) {
  const int heads[2] = {r->H, r->Hkv};
  const int64_t esz = r->dtype == PISA_DTYPE_BF16 ? 2 : 4;
  Placed in[2], out[2];
  for (int i = 0; i < 2; ++i) {
    in[i] = Placed{side[i].in, pisa_strides{side[i].ib, side[i].ih, side[i].in_n}, r->B, heads[i], r->N};
    out[i] = Placed{side[i].out, pisa_strides{side[i].ob, side[i].oh, side[i].on}, r->B, heads[i], r->N};
  }
  for (int i = 0; i < 2; ++i) {
    if (!out[i].ptr) continue;
    for (int j = 0; j < 2; ++j) {
      if (in[j].ptr && !(i == j && in[j].ptr == out[i].ptr) && share(out[i], in[j], r->d, esz))
        return fail(PISA_ERR_INVALID_ARG, "%s (output) overlaps %s", names[i], names[j]);
    }
  }
  if (out[0].ptr && out[1].ptr && share(out[0], out[1], r->d, esz))
    return fail(PISA_ERR_INVALID_ARG, "%s (output) overlaps %s (output)", names[0], names[1]);
  return PISA_OK;
}

int check_positions(const int32_t* positions) {
  if (reinterpret_cast<uintptr_t>(positions) & 3u) return fail(PISA_ERR_INVALID_ARG, "positions is not 4-byte aligned");
  return PISA_OK;
}

int run_rope(const pisa_rope* r, const void* q, const pisa_strides* qs, const void* k, const pisa_strides* ks,
             const int32_t* positions, void* qo, const pisa_strides* qos, void* ko, const pisa_strides* kos, float sign,
             pisa_stream_t stream, const char* who) {
  PISA_TRY(check_rope(r));
  pisa::RopeArgs a{};
  PISA_TRY(check_rope_side(r, "q", r->H, q, qs, qo, qos, &a.q));
  PISA_TRY(check_rope_side(r, "k", r->Hkv, k, ks, ko, kos, &a.k));
  if (!q && !k) return fail(PISA_ERR_INVALID_ARG, "neither q nor k given");
  PISA_TRY(check_positions(positions));
  PISA_TRY(check_rope_overlaps(r, {a.q, a.k}, {"q", "k"}));
  fill_rope(r, positions, sign, &a);
  return device_status(pisa::launch_rope(a, r->dtype == PISA_DTYPE_BF16, r->layout == PISA_ROPE_HALF,
                                         static_cast<hipStream_t>(stream)),
                       who);
}

// A norm's descriptor for a rotation of these sides.
int check_norm(const pisa_rope* r, const pisa_qk_norm* m, pisa::NormArgs* out) {
  if (!m) return fail(PISA_ERR_INVALID_ARG, "norm is NULL");
  PISA_TRY(check_ptr(m->q_weight, "q_weight", true));
  PISA_TRY(check_ptr(m->k_weight, "k_weight", true));
  if (m->weight_dtype != PISA_DTYPE_F32 && m->weight_dtype != PISA_DTYPE_BF16)
    return fail(PISA_ERR_INVALID_ARG, "unknown weight_dtype %d", m->weight_dtype);
  if (m->reserved != 0) return fail(PISA_ERR_INVALID_ARG, "reserved of the norm must be 0");
  if (!(m->eps >= 1e-30 && m->eps <= 1e30)) return fail(PISA_ERR_INVALID_ARG, "eps must be in [1e-30, 1e30]");
  if (!(fabs(m->offset) <= 1e30)) return fail(PISA_ERR_INVALID_ARG, "offset is not a number within 10^30");
  *out = pisa::NormArgs{m->q_weight, m->k_weight, nullptr, nullptr, nullptr, static_cast<float>(m->eps),
                        static_cast<float>(m->offset), m->weight_dtype == PISA_DTYPE_BF16};
  return PISA_OK;
}

// Bytes from a tensor's first value to its last (at most 2^62).
size_t span_of(const pisa_strides& x, int64_t B, int64_t heads, int64_t rows, int d, size_t esz) {
  const __int128 n = (static_cast<__int128>(B - 1) * x.b + static_cast<__int128>(heads - 1) * x.h +
                      static_cast<__int128>(rows - 1) * x.n + d) * static_cast<__int128>(esz);
  return static_cast<size_t>(std::min<__int128>(n, int64_t(1) << 62));
}

struct Region {
  const void* ptr;
  size_t bytes;
  const char* name;
};
bool meet(const Region& x, const Region& y) {
  const uintptr_t u = reinterpret_cast<uintptr_t>(x.ptr), w = reinterpret_cast<uintptr_t>(y.ptr);
  return x.bytes && y.bytes && u < w + y.bytes && w < u + x.bytes;
}

// Rows that an append reads, against what it writes.
int check_append_regions(const Region* fresh, int nfresh, const Region* held, int nheld, const char* clash) {
  for (int i = 0; i < nfresh; ++i) {
    for (int j = 0; j < nheld; ++j)
      if (meet(fresh[i], held[j])) return fail(PISA_ERR_INVALID_ARG, "%s overlaps the %s", fresh[i].name, held[j].name);
  }
  for (int i = 1; i < nheld; ++i) {
    for (int j = 0; j < i; ++j)
      if (meet(held[i], held[j])) return fail(PISA_ERR_INVALID_ARG, "%s", clash);
  }
  return PISA_OK;
}

// The list of rows of an append: which of n_rows each of the appended ones is.
int check_rows(const int32_t* rows, int32_t n_rows, int32_t appended) {
  if (n_rows < 1) return fail(PISA_ERR_INVALID_ARG, "n_rows must be >= 1 (got %d)", n_rows);
  if (reinterpret_cast<uintptr_t>(rows) & 3u) return fail(PISA_ERR_INVALID_ARG, "rows is not 4-byte aligned");
  if (!rows && n_rows < appended)
    return fail(PISA_ERR_INVALID_ARG, "without rows, n_rows (%d) must be >= N - n_old (%d)", n_rows, appended);
  return PISA_OK;
}

int check_qcache(const pisa_qcache* c, const pisa::Geo& g, pisa::QCache* out) {
  if (!c) return fail(PISA_ERR_INVALID_ARG, "cache is NULL");
  PISA_TRY(check_ptr(c->k, "cache k"));
  PISA_TRY(check_ptr(c->v, "cache v"));
  PISA_TRY(check_ptr(c->k_scale, "k_scale"));
  PISA_TRY(check_ptr(c->v_scale, "v_scale"));
  *out = pisa::QCache{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale,
                      (g.Nkv + g.C - 1) / g.C};
  return PISA_OK;
}

int check_n_old(const pisa_problem* p, int32_t n_old) {
  if (n_old < 0 || n_old > p->N) return fail(PISA_ERR_INVALID_ARG, "need 0 <= n_old <= N (got %d, N=%d)", n_old, p->N);
  return PISA_OK;
}

int run_qcache_append(const pisa_problem* p, const pisa_qcache* c, const void* k_new, const pisa_strides* k_strides,
                      const void* v_new, const pisa_strides* v_strides, const int32_t* rows, int32_t n_rows, int32_t n_old,
                      float* pyramid, pisa_stream_t stream, const char* who) {
  pisa::Shape s{};
  pisa::Geo g{};
  pisa::QAppend a{};
  PISA_TRY(check_problem(p, &s, &g));
  PISA_TRY(check_qcache(c, g, &a.c));
  PISA_TRY(check_ptr(c->k_open, "k_open"));
  PISA_TRY(check_ptr(c->v_open, "v_open"));
  PISA_TRY(check_ptr(pyramid, "pyramid", true));
  PISA_TRY(check_n_old(p, n_old));
  PISA_TRY(check_rows(rows, n_rows, p->N - n_old));
  if (n_old == p->N) return PISA_OK;
  PISA_TRY(check_ptr(k_new, "k_new"));
  PISA_TRY(check_ptr(v_new, "v_new"));
  const int32_t have = rows ? n_rows : p->N - n_old;  // rows that may be read
  // without a list the contiguous layout is that of the rows that are appended
  const int32_t wide = n_rows == INT32_MAX ? have : n_rows;
  pisa_strides ks, vs;
  PISA_TRY(check_strides(k_strides, "k_new", p->B, p->Hkv, wide, p->d, p->dtype, false, &ks));
  PISA_TRY(check_strides(v_strides, "v_new", p->B, p->Hkv, wide, p->d, p->dtype, false, &vs));
  // the appended rows are read while the cache is written
  const size_t esz = s.bf16 ? 2 : 4, codes = pisa_qcache_bytes(p), open = static_cast<size_t>(s.BH()) * s.C * s.D * esz;
  const size_t scales = static_cast<size_t>(s.BH()) * a.c.M * sizeof(float);
  const size_t levels = static_cast<size_t>(s.BH()) * g.R * s.D * sizeof(float);
  const Region fresh[] = {{k_new, span_of(ks, p->B, p->Hkv, have, p->d, esz), "k_new"},
                          {v_new, span_of(vs, p->B, p->Hkv, have, p->d, esz), "v_new"},
                          {rows, rows ? static_cast<size_t>(p->B) * (p->N - n_old) * 4 : 0, "rows"}};
  const Region held[] = {{c->k, codes, "cache"},        {c->v, codes, "cache"},        {c->k_open, open, "cache"},
                         {c->v_open, open, "cache"},    {c->k_scale, scales, "cache"}, {c->v_scale, scales, "cache"},
                         {pyramid, pyramid ? levels : 0, "pyramid"}};
  PISA_TRY(check_append_regions(fresh, 3, held, 7, "buffers of the cache or the pyramid overlap"));
  a.k_new = k_new;
  a.v_new = v_new;
  a.ksb = ks.b;
  a.ksh = ks.h;
  a.ksn = ks.n;
  a.vsb = vs.b;
  a.vsh = vs.h;
  a.vsn = vs.n;
  a.k_open = c->k_open;
  a.v_open = c->v_open;
  a.pyr = pyramid;
  a.Hkv = p->Hkv;
  a.n_old = n_old;
  a.rows = rows;
  a.n_rows = n_rows;
  pisa::Geo g_old{};
  if (n_old > 0) compute_geo(n_old, p->C, p->fanout, &g_old, g.Nkv);
  return device_status(pisa::launch_qcache_append(g, g_old, s.BH(), s.D, s.bf16, a, static_cast<hipStream_t>(stream)), who);
}

// The input of one side of a norm's gradient.
int check_rope_input(const pisa_rope* r, const char* name, int heads, const void* in, const pisa_strides* is, pisa::RopeSide* side) {
  if (!in) return PISA_OK;
  PISA_TRY(check_ptr(in, name));
  pisa_strides si;
  PISA_TRY(check_strides(is, name, r->B, heads, r->N, r->d, r->dtype, false, &si));
  *side = pisa::RopeSide{in, nullptr, si.b, si.h, si.n, 0, 0, 0};
  return PISA_OK;
}

// A norm's gradient reads its inputs while the gradients are written.
int check_inputs_apart(const pisa_rope* r, const pisa::RopeSide (&x)[2], const pisa::RopeSide (&d)[2]) {
  const int heads[2] = {r->H, r->Hkv};
  const char* const names[2] = {"q", "k"};
  const int64_t esz = r->dtype == PISA_DTYPE_BF16 ? 2 : 4;
  for (int i = 0; i < 2; ++i) {
    for (int j = 0; j < 2; ++j) {
      if (!x[i].in || !d[j].out) continue;
      const Placed in{x[i].in, pisa_strides{x[i].ib, x[i].ih, x[i].in_n}, r->B, heads[i], r->N};
      const Placed out{d[j].out, pisa_strides{d[j].ob, d[j].oh, d[j].on}, r->B, heads[j], r->N};
      if (share(out, in, r->d, esz)) return fail(PISA_ERR_INVALID_ARG, "d_%s overlaps %s", names[j], names[i]);
    }
  }
  return PISA_OK;
}

// What a norm writes against what it reads, but for the tensors that check_rope_overlaps
// and check_inputs_apart compare row by row (by what lies between a tensor's first value
// and its last).  out: the sides' outputs; in, dy: the sides' inputs (of a gradient).
int check_norm_overlaps(const pisa_rope* r, const pisa_qk_norm* m, const int32_t* positions, const pisa::RopeSide (&out)[2],
                        const pisa::RopeSide (&in)[2], const float* d_q_weight, const float* d_k_weight, const void* ws,
                        size_t ws_bytes) {
  const size_t w = static_cast<size_t>(r->d) * (m->weight_dtype == PISA_DTYPE_BF16 ? 2 : 4), dw = static_cast<size_t>(r->d) * 4;
  const size_t esz = r->dtype == PISA_DTYPE_BF16 ? 2 : 4;
  const int heads[2] = {r->H, r->Hkv};
  auto bytes = [](const void* p, size_t n) { return p ? n : 0; };
  auto reads = [&](const pisa::RopeSide& x, int i, const char* name) {
    return Region{x.in, bytes(x.in, span_of({x.ib, x.ih, x.in_n}, r->B, heads[i], r->N, r->d, esz)), name};
  };
  auto writes = [&](const pisa::RopeSide& x, int i, const char* name) {
    return Region{x.out, bytes(x.out, span_of({x.ob, x.oh, x.on}, r->B, heads[i], r->N, r->d, esz)), name};
  };
  const Region small_in[] = {{m->q_weight, bytes(m->q_weight, w), "q_weight"},
                             {m->k_weight, bytes(m->k_weight, w), "k_weight"},
                             {positions, bytes(positions, span_of({r->pos_bstride, 0, 1}, r->B, 1, r->N, 1, 4)), "positions"}};
  const Region small_out[] = {{d_q_weight, bytes(d_q_weight, dw), "d_q_weight"},
                              {d_k_weight, bytes(d_k_weight, dw), "d_k_weight"},
                              {ws, bytes(ws, ws_bytes), "workspace"}};
  const Region large_in[] = {reads(in[0], 0, "q"), reads(in[1], 1, "k"), reads(out[0], 0, "d_q_out"), reads(out[1], 1, "d_k_out")};
  const Region large_out[] = {writes(out[0], 0, "q (output)"), writes(out[1], 1, "k (output)")};
  auto apart = [](const Region& x, const Region& y) {
    return meet(x, y) ? fail(PISA_ERR_INVALID_ARG, "%s overlaps %s", x.name, y.name) : PISA_OK;
  };
  for (const Region& y : small_in) {
    for (const Region& x : small_out) PISA_TRY(apart(x, y));
    for (const Region& x : large_out) PISA_TRY(apart(x, y));
  }
  for (int i = 0; i < 3; ++i) {
    for (const Region& y : large_in) PISA_TRY(apart(small_out[i], y));
    for (const Region& y : large_out) PISA_TRY(apart(small_out[i], y));
    for (int j = 0; j < i; ++j) PISA_TRY(apart(small_out[i], small_out[j]));
  }
  return PISA_OK;
}

// Drafted rows of a problem with Nq of them behind N - Nq cached ones.
int check_draft(const pisa_problem* p, pisa::Shape* s, pisa::Geo* g) {
  PISA_TRY(check_problem(p, s, g));
  if (p->Nq > PISA_DRAFT_MAX) return fail(PISA_ERR_UNSUPPORTED, "%d drafted rows (supported: <= %d)", p->Nq, PISA_DRAFT_MAX);
  return PISA_OK;
}

size_t draft_ws(const pisa_problem* p, bool q8) {
  pisa::Shape s{};
  pisa::Geo g{};
  return check_draft(p, &s, &g) == PISA_OK ? pisa::draft_attn_ws(s, q8) : 0;
}

// What both attentions of drafted rows check and launch alike; d has the cache, held
// its buffers.
int run_draft_attn(const pisa_problem* p, const pisa::Shape& s, pisa::DraftAttn d, const Region* held, int nheld,
                   const void* q, const int32_t* block_idx, const void* k_new, const pisa_strides* k_strides, const void* v_new,
                   const pisa_strides* v_strides, const uint64_t* mask, int64_t mask_bstride, void* o, float* lse, void* ws,
                   size_t ws_bytes, pisa_stream_t stream, const char* who) {
  PISA_TRY(check_ptr(q, "q"));
  PISA_TRY(check_ptr(block_idx, "block_idx"));
  PISA_TRY(check_ptr(k_new, "k_new"));
  PISA_TRY(check_ptr(v_new, "v_new"));
  PISA_TRY(check_values(mask, "mask", 8));
  PISA_TRY(check_ptr(o, "o"));
  PISA_TRY(check_ptr(lse, "lse", true));
  const int64_t W = (p->Nq + 63) / 64;
  if (mask_bstride != 0 && mask_bstride < p->Nq * W)
    return fail(PISA_ERR_INVALID_ARG, "mask_bstride must be 0 (one mask) or >= Nq * ceil(Nq / 64) (got %lld)",
                static_cast<long long>(mask_bstride));
  pisa_strides ks, vs;
  PISA_TRY(check_strides(k_strides, "k_new", p->B, p->Hkv, p->Nq, p->d, p->dtype, false, &ks));
  PISA_TRY(check_strides(v_strides, "v_new", p->B, p->Hkv, p->Nq, p->d, p->dtype, false, &vs));
  const size_t need = pisa::draft_attn_ws(s, d.k == nullptr);
  PISA_TRY(check_ws(ws, ws_bytes, need));
  // what is written against what is read meanwhile
  const size_t esz = s.bf16 ? 2 : 4, rows = static_cast<size_t>(p->B) * p->H * p->Nq;
  const Region out[] = {{o, rows * p->d * esz, "o"}, {lse, lse ? rows * 4 : 0, "lse"}, {ws, need, "workspace"}};
  const Region in[] = {{q, rows * p->d * esz, "q"},
                       {block_idx, static_cast<size_t>(s.BH()) * p->Nq * p->K * 4, "block_idx"},
                       {k_new, span_of(ks, p->B, p->Hkv, p->Nq, p->d, esz), "k_new"},
                       {v_new, span_of(vs, p->B, p->Hkv, p->Nq, p->d, esz), "v_new"},
                       {mask, span_of({mask_bstride, 0, W}, p->B, 1, p->Nq, static_cast<int>(W), 8), "mask"}};
  for (int i = 0; i < 3; ++i) {
    for (const Region& x : in)
      if (meet(out[i], x)) return fail(PISA_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, x.name);
    for (int j = 0; j < nheld; ++j)
      if (meet(out[i], held[j])) return fail(PISA_ERR_INVALID_ARG, "%s overlaps the %s", out[i].name, held[j].name);
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return fail(PISA_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, out[j].name);
  }
  d.k_new = k_new;
  d.v_new = v_new;
  d.ksb = ks.b, d.ksh = ks.h, d.ksn = ks.n;
  d.vsb = vs.b, d.vsh = vs.h, d.vsn = vs.n;
  d.mask = mask;
  d.mask_bstride = mask_bstride;
  return device_status(pisa::launch_draft_attn(s, d, q, block_idx, o, lse, ws, static_cast<hipStream_t>(stream)), who);
}

// Whichever sides a call has.
size_t norm_rope_ws(const pisa_rope* r) {
  const bool bf16 = r->dtype == PISA_DTYPE_BF16;
  auto bytes = [&](int H, int Hkv) { return pisa::norm_rope_bwd_ws(r->B, r->N, H, Hkv, r->d, r->rot, bf16, r->layout == PISA_ROPE_HALF); };
  return std::max({bytes(r->H, r->Hkv), bytes(r->H, 0), bytes(0, r->Hkv)});
}

}  // namespace

extern "C" {

int pisa_num_levels(int32_t N, int32_t C, int32_t fanout) {
  const int L = compute_geo(N, C, fanout, nullptr);
  if (L < 0) return fail(L, "invalid N, C or fanout");
  return L;
}

int pisa_pyramid_layout(const pisa_problem* p, int64_t* level_row_offset, int64_t* rows_R) {
  pisa::Geo g{};
  PISA_TRY(check_problem(p, nullptr, &g));
  if (!level_row_offset || !rows_R) return fail(PISA_ERR_INVALID_ARG, "output pointers must be non-NULL");
  for (int l = 1; l <= g.L; ++l) level_row_offset[l - 1] = l <= g.Lstore ? g.off[l] : g.R;
  *rows_R = g.R;
  return g.L;
}

size_t pisa_pyramid_bytes(const pisa_problem* p) {
  pisa::Geo g{};
  if (check_problem(p, nullptr, &g) != PISA_OK) return 0;
  return static_cast<size_t>(p->B) * p->Hkv * g.R * p->d * sizeof(float);
}

size_t pisa_select_workspace_bytes(const pisa_problem* p) {
  pisa::Shape s{};
  pisa::Geo g{};
  if (check_problem(p, &s, &g) != PISA_OK) return 0;
  return select_ws(pick_schedule(p, s, g), s, g);
}

size_t pisa_bsa_workspace_bytes(const pisa_problem* p) {
  pisa::Shape s{};
  pisa::Geo g{};
  if (check_problem(p, &s, &g) != PISA_OK) return 0;
  return pisa::bsa_ws(s, g);
}

size_t pisa_attn_workspace_bytes(const pisa_problem* p) {
  pisa::Shape s{};
  pisa::Geo g{};
  if (check_problem(p, &s, &g) != PISA_OK) return 0;
  return pisa::attn_ws(s, g);
}

int pisa_build_pyramid(const pisa_problem* p, const void* k, float* pyramid, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  PISA_TRY(check_problem(p, &s, &g));
  PISA_TRY(check_ptr(k, "k"));
  PISA_TRY(check_ptr(pyramid, "pyramid"));
  return device_status(pisa::launch_build_pyramid(g, s.BH(), s.D, s.bf16, k, pyramid,
                                                  static_cast<hipStream_t>(stream)),
                       "pisa_build_pyramid");
}

int pisa_pyramid_append(const pisa_problem* p, const void* k, float* pyramid, int32_t n_old, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  PISA_TRY(check_problem(p, &s, &g));
  PISA_TRY(check_ptr(k, "k"));
  PISA_TRY(check_ptr(pyramid, "pyramid"));
  if (n_old < 0 || n_old > p->N) return fail(PISA_ERR_INVALID_ARG, "need 0 <= n_old <= N (got %d, N=%d)", n_old, p->N);
  if (n_old == p->N) return PISA_OK;
  pisa::Geo g_old{};
  if (n_old > 0) compute_geo(n_old, p->C, p->fanout, &g_old, g.Nkv);
  return device_status(pisa::launch_pyramid_append(g, g_old, s.BH(), s.D, s.bf16, k, pyramid, n_old,
                                                   static_cast<hipStream_t>(stream)),
                       "pisa_pyramid_append");
}

int32_t pisa_cache_capacity(int32_t cap, int32_t need, int32_t C) {
  if (cap < 0 || need < 1 || C < 1) return fail(PISA_ERR_INVALID_ARG, "need cap >= 0, need >= 1, C >= 1");
  if (need <= cap) return cap;
  const int64_t grown = std::max<int64_t>(need, static_cast<int64_t>(cap) + (static_cast<int64_t>(cap) + 1) / 2);
  const int64_t rounded = (grown + C - 1) / C * C;
  const int64_t limit = static_cast<int64_t>(kMaxLeafBlocks) * C;
  if (rounded <= limit && rounded <= INT32_MAX) return static_cast<int32_t>(rounded);
  if (need <= limit && need <= INT32_MAX) return static_cast<int32_t>(std::min<int64_t>(limit, INT32_MAX));
  return fail(PISA_ERR_UNSUPPORTED, "a cache of %d tokens exceeds %d leaf blocks of %d", need, kMaxLeafBlocks, C);
}

int pisa_cache_grow(const pisa_problem* p, int32_t new_cap, const float* pyr_old, float* pyr_new, const void* k_old,
                    void* k_new, const void* v_old, void* v_new, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  PISA_TRY(check_problem(p, &s, &g));
  if (new_cap < g.Nkv)
    return fail(PISA_ERR_INVALID_ARG, "new_cap (%d) is below the current capacity (%d)", new_cap, g.Nkv);
  pisa_problem pn = *p;
  pn.Ncap = new_cap;
  pisa::Geo gn{};
  PISA_TRY(check_problem(&pn, nullptr, &gn));
  PISA_TRY(check_ptr(pyr_old, "pyr_old"));
  PISA_TRY(check_ptr(pyr_new, "pyr_new"));
  const bool kv = k_old || k_new || v_old || v_new;
  if (kv) {
    PISA_TRY(check_ptr(k_old, "k_old"));
    PISA_TRY(check_ptr(k_new, "k_new"));
    PISA_TRY(check_ptr(v_old, "v_old"));
    PISA_TRY(check_ptr(v_new, "v_new"));
  }
  const int64_t BH = s.BH();
  const size_t esz = s.bf16 ? 2 : 4;
  auto overlap = [](const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
  };
  const size_t pyr_old_bytes = static_cast<size_t>(BH) * g.R * s.D * 4;
  const size_t pyr_new_bytes = static_cast<size_t>(BH) * gn.R * s.D * 4;
  if (overlap(pyr_old, pyr_old_bytes, pyr_new, pyr_new_bytes))
    return fail(PISA_ERR_INVALID_ARG, "pyr_old and pyr_new overlap");
  if (kv) {
    const size_t kv_old_bytes = static_cast<size_t>(BH) * g.Nkv * s.D * esz;
    const size_t kv_new_bytes = static_cast<size_t>(BH) * gn.Nkv * s.D * esz;
    if (overlap(k_old, kv_old_bytes, k_new, kv_new_bytes) || overlap(v_old, kv_old_bytes, v_new, kv_new_bytes) ||
        overlap(k_new, kv_new_bytes, v_new, kv_new_bytes) || overlap(k_old, kv_old_bytes, v_new, kv_new_bytes) ||
        overlap(v_old, kv_old_bytes, k_new, kv_new_bytes))
      return fail(PISA_ERR_INVALID_ARG, "old and new key/value buffers overlap");
  }
  // 16-byte units: a summary row is D floats (16 or 32 units), a key row D
  // elements of esz bytes (8/16 units in bf16, 16/32 in fp32)
  const int64_t pu = s.D / 4, ku = s.D * static_cast<int64_t>(esz) / 16;
  pisa::GrowArgs a{};
  int64_t end = 0;
  for (int l = 1; l <= g.Lstore; ++l) {
    end += static_cast<int64_t>(g.M[l]) * pu;
    a.lev_end[l - 1] = end;
    a.off_old[l - 1] = g.off[l] * pu;
    a.off_new[l - 1] = gn.off[l] * pu;
  }
  a.pyr_units = end;
  a.kv_units = kv ? static_cast<int64_t>(s.N) * ku : 0;
  a.pyr_old_stride = g.R * pu;
  a.pyr_new_stride = gn.R * pu;
  a.kv_old_stride = static_cast<int64_t>(g.Nkv) * ku;
  a.kv_new_stride = static_cast<int64_t>(gn.Nkv) * ku;
  return device_status(pisa::launch_cache_grow(a, static_cast<int>(BH), pyr_old, pyr_new, k_old, k_new, v_old, v_new,
                                               static_cast<hipStream_t>(stream)),
                       "pisa_cache_grow");
}

int pisa_select(const pisa_problem* p, const void* q, const void* k, const float* pyramid, int32_t* block_idx,
                float* block_score, void* ws, size_t ws_bytes, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  int sched = 0;
  PISA_TRY(check_select(p, q, k, pyramid, block_idx, block_score, &s, &g, &sched));
  sched = schedule_for_ws(p, &s, g, sched, ws && aligned256(ws) ? ws_bytes : 0);
  PISA_TRY(check_ws(ws, ws_bytes, select_ws_min(sched, s, g)));
  return run_select(s, g, sched, q, k, pyramid, block_idx, block_score, ws, ws_bytes, static_cast<hipStream_t>(stream),
                    "pisa_select");
}

int pisa_select_static(const pisa_problem* p, const void* q, const void* k, const float* pyramid,
                       int32_t* block_idx, float* block_score, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  int sched = 0;
  PISA_TRY(check_select(p, q, k, pyramid, block_idx, block_score, &s, &g, &sched));
  sched = schedule_for_ws(p, &s, g, sched, PISA_STATIC_SCRATCH_BYTES);
  const size_t need = select_ws_min(sched, s, g);
  if (need > PISA_STATIC_SCRATCH_BYTES)
    return fail(PISA_ERR_WORKSPACE,
                "pisa_select_static: this selection needs %zu bytes of scratch, the static scratch holds %zu "
                "(call pisa_select with a workspace instead)",
                need, static_cast<size_t>(PISA_STATIC_SCRATCH_BYTES));
  void* ws = nullptr;
  if (need > 0) PISA_TRY(static_scratch(&ws));
  return run_select(s, g, sched, q, k, pyramid, block_idx, block_score, ws, PISA_STATIC_SCRATCH_BYTES,
                    static_cast<hipStream_t>(stream), "pisa_select_static");
}

int pisa_select_flat_bsa(const pisa_problem* p, const void* q, const float* pyramid, int32_t* block_idx, void* ws,
                         size_t ws_bytes, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  PISA_TRY(check_problem(p, &s, &g));
  PISA_TRY(check_ptr(q, "q"));
  PISA_TRY(check_ptr(pyramid, "pyramid"));
  PISA_TRY(check_ptr(block_idx, "block_idx"));
  const bool mfma_bsa = s.bf16 && s.K <= 32;
  if (!mfma_bsa && (static_cast<int64_t>(g.M[1]) + s.K) * 4 > 65536)
    return fail(PISA_ERR_UNSUPPORTED, "flat BSA on fp32 or K > 32 keeps one score per leaf block in LDS: N/C < 16384");
  PISA_TRY(check_ws(ws, ws_bytes, pisa::bsa_ws(s, g)));
  return device_status(pisa::launch_flat_bsa(s, g, q, pyramid, block_idx, ws, static_cast<hipStream_t>(stream)),
                       "pisa_select_flat_bsa");
}

int pisa_sparse_attn_fwd(const pisa_problem* p, const void* q, const void* k, const void* v,
                         const int32_t* block_idx, void* o, float* lse, void* ws, size_t ws_bytes,
                         pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  PISA_TRY(check_problem(p, &s, &g));
  PISA_TRY(check_ptr(q, "q"));
  PISA_TRY(check_ptr(k, "k"));
  PISA_TRY(check_ptr(v, "v"));
  PISA_TRY(check_ptr(block_idx, "block_idx"));
  PISA_TRY(check_ptr(o, "o"));
  PISA_TRY(check_ptr(lse, "lse", true));
  PISA_TRY(check_ws(ws, ws_bytes, pisa::attn_ws(s, g)));
  return device_status(
      pisa::launch_attention(s, g, q, k, v, block_idx, o, lse, ws, static_cast<hipStream_t>(stream)),
      "pisa_sparse_attn_fwd");
}

size_t pisa_attn_bwd_workspace_bytes(const pisa_problem* p) {
  pisa::Shape s{};
  pisa::Geo g{};
  if (check_problem(p, &s, &g) != PISA_OK || !pisa::attn_bwd_supported(s)) return 0;
  return pisa::attn_bwd_ws(s, g);
}

int pisa_sparse_attn_bwd(const pisa_problem* p, const void* q, const void* k, const void* v,
                         const int32_t* block_idx, const void* o, const float* lse, const void* d_o, void* dq,
                         void* dk, void* dv, void* ws, size_t ws_bytes, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  PISA_TRY(check_problem(p, &s, &g));
  PISA_TRY(check_ptr(q, "q"));
  PISA_TRY(check_ptr(k, "k"));
  PISA_TRY(check_ptr(v, "v"));
  PISA_TRY(check_ptr(block_idx, "block_idx"));
  PISA_TRY(check_ptr(o, "o"));
  PISA_TRY(check_ptr(lse, "lse"));
  PISA_TRY(check_ptr(d_o, "d_o"));
  PISA_TRY(check_ptr(dq, "dq"));
  PISA_TRY(check_ptr(dk, "dk"));
  PISA_TRY(check_ptr(dv, "dv"));
  if (!pisa::attn_bwd_supported(s))
    return fail(PISA_ERR_UNSUPPORTED, "the attention backward runs on bf16 with d in {64,128} and C in {32,64,96,128}");
  PISA_TRY(check_ws(ws, ws_bytes, pisa::attn_bwd_ws(s, g)));
  return device_status(pisa::launch_attention_bwd(s, g, q, k, v, block_idx, o, lse, d_o, dq, dk, dv, ws,
                                                  static_cast<hipStream_t>(stream)),
                       "pisa_sparse_attn_bwd");
}

size_t pisa_quality_workspace_bytes(const pisa_problem* p, int32_t n_rows) {
  pisa::Shape s{};
  pisa::Geo g{};
  if (check_problem(p, &s, &g) != PISA_OK || n_rows < 1) return 0;
  return pisa::quality_ws(s, n_rows);
}

int pisa_selection_quality(const pisa_problem* p, const void* q, const void* k, const int32_t* block_idx,
                           const int32_t* rows, int32_t n_rows, float* metrics, int32_t* ref_idx, void* ws,
                           size_t ws_bytes, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  PISA_TRY(check_problem(p, &s, &g));
  PISA_TRY(check_ptr(q, "q"));
  PISA_TRY(check_ptr(k, "k"));
  PISA_TRY(check_ptr(block_idx, "block_idx"));
  PISA_TRY(check_ptr(rows, "rows"));
  PISA_TRY(check_ptr(metrics, "metrics"));
  PISA_TRY(check_ptr(ref_idx, "ref_idx", true));
  if (n_rows < 1 || n_rows > (1 << 24)) return fail(PISA_ERR_INVALID_ARG, "n_rows %d out of [1, 2^24]", n_rows);
  if (!pisa::quality_supported(s))
    return fail(PISA_ERR_UNSUPPORTED, "the quality diagnostic runs on bf16 with C in {32,64,96,128}, N/C <= 16384, K <= 64");
  PISA_TRY(check_ws(ws, ws_bytes, pisa::quality_ws(s, n_rows)));
  return device_status(pisa::launch_quality(s, q, k, block_idx, rows, n_rows, metrics, ref_idx, ws,
                                            static_cast<hipStream_t>(stream)),
                       "pisa_selection_quality");
}

int pisa_rope_frequencies(pisa_rope* r, double base, int32_t scaling, double factor, int32_t ctx, double fast,
                          double slow) {
  if (!r) return fail(PISA_ERR_INVALID_ARG, "rope is NULL");
  if (r->rot < 2 || r->rot > 2 * PISA_ROPE_MAX_PAIRS || r->rot % 2 != 0)
    return fail(PISA_ERR_INVALID_ARG, "rot must be even and in [2, %d] (got %d)", 2 * PISA_ROPE_MAX_PAIRS, r->rot);
  if (!(base > 1.0) || !isfinite(base)) return fail(PISA_ERR_INVALID_ARG, "base must be > 1");
  if (!(factor >= 1.0) || !isfinite(factor)) return fail(PISA_ERR_INVALID_ARG, "factor must be >= 1");
  if (scaling < PISA_ROPE_SCALE_NONE || scaling > PISA_ROPE_SCALE_PARTS)
    return fail(PISA_ERR_INVALID_ARG, "unknown scaling %d", scaling);
  if (scaling == PISA_ROPE_SCALE_BASE && r->rot == 2)
    return fail(PISA_ERR_INVALID_ARG, "scaling the base needs rot > 2");
  const bool parts = scaling == PISA_ROPE_SCALE_PARTS;
  if (parts && (ctx < 1 || !(slow >= 0.0) || !(fast > slow) || !isfinite(fast)))
    return fail(PISA_ERR_INVALID_ARG, "scaling by parts needs ctx >= 1 and fast > slow >= 0");
  const int pairs = r->rot / 2;
  if (scaling == PISA_ROPE_SCALE_BASE) base *= pow(factor, static_cast<double>(r->rot) / (r->rot - 2));
  for (int i = 0; i < PISA_ROPE_MAX_PAIRS; ++i) {
    double f = i < pairs ? pow(base, -2.0 * i / r->rot) : 0.0;
    if (scaling == PISA_ROPE_SCALE_LINEAR) f /= factor;
    if (parts) {
      const double y = std::min(1.0, std::max(0.0, (ctx * f / 6.283185307179586476925286766559 - slow) / (fast - slow)));
      f *= y + (1.0 - y) / factor;
    }
    r->freq[i] = f;
  }
  r->amplitude = parts ? 0.1 * log(factor) + 1.0 : 1.0;
  return PISA_OK;
}

int pisa_rope_fwd(const pisa_rope* r, const void* q, const pisa_strides* q_strides, const void* k,
                  const pisa_strides* k_strides, const int32_t* positions, void* q_out,
                  const pisa_strides* q_out_strides, void* k_out, const pisa_strides* k_out_strides,
                  pisa_stream_t stream) {
  return run_rope(r, q, q_strides, k, k_strides, positions, q_out, q_out_strides, k_out, k_out_strides, 1.f, stream,
                  "pisa_rope_fwd");
}

int pisa_rope_bwd(const pisa_rope* r, const void* d_q_out, const pisa_strides* d_q_out_strides, const void* d_k_out,
                  const pisa_strides* d_k_out_strides, const int32_t* positions, void* d_q,
                  const pisa_strides* d_q_strides, void* d_k, const pisa_strides* d_k_strides, pisa_stream_t stream) {
  return run_rope(r, d_q_out, d_q_out_strides, d_k_out, d_k_out_strides, positions, d_q, d_q_strides, d_k, d_k_strides,
                  -1.f, stream, "pisa_rope_bwd");
}

int32_t pisa_qcache_blocks(const pisa_problem* p) {
  pisa::Geo g{};
  PISA_TRY(check_problem(p, nullptr, &g));
  return (g.Nkv + g.C - 1) / g.C;
}

size_t pisa_qcache_bytes(const pisa_problem* p) {
  pisa::Geo g{};
  if (check_problem(p, nullptr, &g) != PISA_OK) return 0;
  return static_cast<size_t>(p->B) * p->Hkv * ((g.Nkv + g.C - 1) / g.C) * g.C * p->d;
}

int pisa_qcache_append(const pisa_problem* p, const pisa_qcache* c, const void* k_new, const pisa_strides* k_strides,
                       const void* v_new, const pisa_strides* v_strides, int32_t n_old, float* pyramid,
                       pisa_stream_t stream) {
  return run_qcache_append(p, c, k_new, k_strides, v_new, v_strides, nullptr, INT32_MAX, n_old, pyramid, stream,
                           "pisa_qcache_append");
}

int pisa_qcache_append_rows(const pisa_problem* p, const pisa_qcache* c, const void* k_new, const pisa_strides* k_strides,
                            const void* v_new, const pisa_strides* v_strides, const int32_t* rows, int32_t n_rows,
                            int32_t n_old, float* pyramid, pisa_stream_t stream) {
  return run_qcache_append(p, c, k_new, k_strides, v_new, v_strides, rows, n_rows, n_old, pyramid, stream,
                           "pisa_qcache_append_rows");
}

int pisa_cache_append_rows(const pisa_problem* p, void* k, void* v, const void* k_new, const pisa_strides* k_strides,
                           const void* v_new, const pisa_strides* v_strides, const int32_t* rows, int32_t n_rows,
                           int32_t n_old, float* pyramid, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  PISA_TRY(check_problem(p, &s, &g));
  PISA_TRY(check_ptr(k, "k"));
  PISA_TRY(check_ptr(v, "v"));
  PISA_TRY(check_ptr(pyramid, "pyramid", true));
  PISA_TRY(check_n_old(p, n_old));
  PISA_TRY(check_rows(rows, n_rows, p->N - n_old));
  if (n_old == p->N) return PISA_OK;
  PISA_TRY(check_ptr(k_new, "k_new"));
  PISA_TRY(check_ptr(v_new, "v_new"));
  const int32_t have = rows ? n_rows : p->N - n_old;  // rows that may be read
  pisa_strides ks, vs;
  PISA_TRY(check_strides(k_strides, "k_new", p->B, p->Hkv, n_rows, p->d, p->dtype, false, &ks));
  PISA_TRY(check_strides(v_strides, "v_new", p->B, p->Hkv, n_rows, p->d, p->dtype, false, &vs));
  const size_t esz = s.bf16 ? 2 : 4, cache = static_cast<size_t>(s.BH()) * g.Nkv * s.D * esz;
  const Region fresh[] = {{k_new, span_of(ks, p->B, p->Hkv, have, p->d, esz), "k_new"},
                          {v_new, span_of(vs, p->B, p->Hkv, have, p->d, esz), "v_new"},
                          {rows, rows ? static_cast<size_t>(p->B) * (p->N - n_old) * 4 : 0, "rows"}};
  const Region held[] = {{k, cache, "cache"}, {v, cache, "cache"},
                         {pyramid, pyramid ? static_cast<size_t>(s.BH()) * g.R * s.D * 4 : 0, "pyramid"}};
  PISA_TRY(check_append_regions(fresh, 3, held, 3, "k, v and the pyramid overlap"));
  pisa::CacheAppend a{k, v, k_new, v_new, ks.b, ks.h, ks.n, vs.b, vs.h, vs.n, pyramid, p->Hkv, n_old, rows, n_rows};
  pisa::Geo g_old{};
  if (n_old > 0) compute_geo(n_old, p->C, p->fanout, &g_old, g.Nkv);
  return device_status(pisa::launch_cache_append(g, g_old, s.BH(), s.D, s.bf16, a, static_cast<hipStream_t>(stream)),
                       "pisa_cache_append_rows");
}

int pisa_draft_layout(int32_t B, int32_t T, const int32_t* parents, int32_t n, uint64_t* mask, int32_t* positions,
                      pisa_stream_t stream) {
  if (B < 1 || B > 65535) return fail(PISA_ERR_INVALID_ARG, "B must be in [1, 65535] (got %d)", B);
  if (T < 1 || T > PISA_DRAFT_MAX) return fail(PISA_ERR_INVALID_ARG, "T must be in [1, %d] (got %d)", PISA_DRAFT_MAX, T);
  if (n < 0 || n > INT32_MAX - T) return fail(PISA_ERR_INVALID_ARG, "need 0 <= n <= 2^31 - 1 - T (got %d)", n);
  PISA_TRY(check_values(parents, "parents", 4));
  PISA_TRY(check_values(mask, "mask", 8));
  PISA_TRY(check_values(positions, "positions", 4, true));
  const size_t row = static_cast<size_t>(B) * T;
  const Region r[] = {{parents, row * 4, "parents"}, {mask, row * 8 * ((T + 63) / 64), "mask"},
                      {positions, positions ? row * 4 : 0, "positions"}};
  for (int i = 1; i < 3; ++i) {
    for (int j = 0; j < i; ++j)
      if (meet(r[i], r[j])) return fail(PISA_ERR_INVALID_ARG, "%s overlaps %s", r[i].name, r[j].name);
  }
  return device_status(pisa::launch_draft_layout(parents, B, T, n, mask, positions, static_cast<hipStream_t>(stream)),
                       "pisa_draft_layout");
}

size_t pisa_draft_attn_workspace_bytes(const pisa_problem* p) { return draft_ws(p, false); }
size_t pisa_qcache_draft_attn_workspace_bytes(const pisa_problem* p) { return draft_ws(p, true); }

int pisa_draft_attn_fwd(const pisa_problem* p, const void* q, const void* k, const void* v, const int32_t* block_idx,
                        const void* k_new, const pisa_strides* k_strides, const void* v_new, const pisa_strides* v_strides,
                        const uint64_t* mask, int64_t mask_bstride, void* o, float* lse, void* ws, size_t ws_bytes,
                        pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  PISA_TRY(check_draft(p, &s, &g));
  PISA_TRY(check_ptr(k, "k"));
  PISA_TRY(check_ptr(v, "v"));
  pisa::DraftAttn d{};
  d.k = k;
  d.v = v;
  const size_t rows = static_cast<size_t>(s.BH()) * g.Nkv * s.D * (s.bf16 ? 2 : 4);
  const Region held[] = {{k, rows, "cache"}, {v, rows, "cache"}};
  return run_draft_attn(p, s, d, held, 2, q, block_idx, k_new, k_strides, v_new, v_strides, mask, mask_bstride, o, lse, ws,
                        ws_bytes, stream, "pisa_draft_attn_fwd");
}

int pisa_qcache_draft_attn_fwd(const pisa_problem* p, const pisa_qcache* c, const void* q, const int32_t* block_idx,
                               const void* k_new, const pisa_strides* k_strides, const void* v_new,
                               const pisa_strides* v_strides, const uint64_t* mask, int64_t mask_bstride, void* o, float* lse,
                               void* ws, size_t ws_bytes, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  pisa::DraftAttn d{};
  PISA_TRY(check_draft(p, &s, &g));
  PISA_TRY(check_qcache(c, g, &d.c));
  const size_t codes = pisa_qcache_bytes(p), scales = static_cast<size_t>(s.BH()) * d.c.M * sizeof(float);
  const Region held[] = {{c->k, codes, "cache"}, {c->v, codes, "cache"}, {c->k_scale, scales, "cache"}, {c->v_scale, scales, "cache"}};
  return run_draft_attn(p, s, d, held, 4, q, block_idx, k_new, k_strides, v_new, v_strides, mask, mask_bstride, o, lse, ws,
                        ws_bytes, stream, "pisa_qcache_draft_attn_fwd");
}

int pisa_norm_rope_fwd(const pisa_rope* r, const pisa_qk_norm* m, const void* q, const pisa_strides* q_strides, const void* k,
                       const pisa_strides* k_strides, const int32_t* positions, void* q_out,
                       const pisa_strides* q_out_strides, void* k_out, const pisa_strides* k_out_strides,
                       pisa_stream_t stream) {
  PISA_TRY(check_rope(r));
  pisa::RopeArgs a{};
  pisa::NormArgs na{};
  PISA_TRY(check_norm(r, m, &na));
  PISA_TRY(check_rope_side(r, "q", r->H, q, q_strides, q_out, q_out_strides, &a.q));
  PISA_TRY(check_rope_side(r, "k", r->Hkv, k, k_strides, k_out, k_out_strides, &a.k));
  if (!q && !k) return fail(PISA_ERR_INVALID_ARG, "neither q nor k given");
  PISA_TRY(check_positions(positions));
  PISA_TRY(check_rope_overlaps(r, {a.q, a.k}, {"q", "k"}));
  PISA_TRY(check_norm_overlaps(r, m, positions, {a.q, a.k}, {}, nullptr, nullptr, nullptr, 0));
  fill_rope(r, positions, 1.f, &a);
  return device_status(pisa::launch_norm_rope(a, na, nullptr, nullptr, r->dtype == PISA_DTYPE_BF16, r->layout == PISA_ROPE_HALF,
                                              static_cast<hipStream_t>(stream)),
                       "pisa_norm_rope_fwd");
}

size_t pisa_norm_rope_bwd_workspace_bytes(const pisa_rope* r) {
  if (check_rope(r) != PISA_OK) return 0;
  return norm_rope_ws(r);
}

int pisa_norm_rope_bwd(const pisa_rope* r, const pisa_qk_norm* m, const void* q, const pisa_strides* q_strides, const void* k,
                       const pisa_strides* k_strides, const void* d_q_out, const pisa_strides* d_q_out_strides,
                       const void* d_k_out, const pisa_strides* d_k_out_strides, const int32_t* positions, void* d_q,
                       const pisa_strides* d_q_strides, void* d_k, const pisa_strides* d_k_strides, float* d_q_weight,
                       float* d_k_weight, void* ws, size_t ws_bytes, pisa_stream_t stream) {
  PISA_TRY(check_rope(r));
  pisa::RopeArgs a{};
  pisa::NormArgs na{};
  pisa::RopeSide dq{}, dk{};
  PISA_TRY(check_norm(r, m, &na));
  if ((!q) != (!d_q) || (!k) != (!d_k))
    return fail(PISA_ERR_INVALID_ARG, "a side needs its input, its output's gradient and its gradient, or none of them");
  PISA_TRY(check_rope_side(r, "d_q_out", r->H, d_q_out, d_q_out_strides, d_q, d_q_strides, &dq));
  PISA_TRY(check_rope_side(r, "d_k_out", r->Hkv, d_k_out, d_k_out_strides, d_k, d_k_strides, &dk));
  if (!q && !k) return fail(PISA_ERR_INVALID_ARG, "neither q nor k given");
  PISA_TRY(check_rope_input(r, "q", r->H, q, q_strides, &a.q));
  PISA_TRY(check_rope_input(r, "k", r->Hkv, k, k_strides, &a.k));
  PISA_TRY(check_positions(positions));
  PISA_TRY(check_ptr(d_q_weight, "d_q_weight", true));
  PISA_TRY(check_ptr(d_k_weight, "d_k_weight", true));
  if ((d_q_weight && !q) || (d_k_weight && !k)) return fail(PISA_ERR_INVALID_ARG, "a weight's gradient needs its side");
  PISA_TRY(check_rope_overlaps(r, {dq, dk}, {"d_q_out", "d_k_out"}));
  // the inputs against the gradients that are written
  PISA_TRY(check_inputs_apart(r, {a.q, a.k}, {dq, dk}));
  const size_t need = d_q_weight || d_k_weight ? norm_rope_ws(r) : 0;
  PISA_TRY(check_ws(ws, ws_bytes, need));
  PISA_TRY(check_norm_overlaps(r, m, positions, {dq, dk}, {a.q, a.k}, d_q_weight, d_k_weight, need ? ws : nullptr, need));
  na.d_q_weight = d_q_weight;
  na.d_k_weight = d_k_weight;
  na.parts = static_cast<float*>(ws);
  fill_rope(r, positions, -1.f, &a);
  return device_status(pisa::launch_norm_rope(a, na, &dq, &dk, r->dtype == PISA_DTYPE_BF16, r->layout == PISA_ROPE_HALF,
                                              static_cast<hipStream_t>(stream)),
                       "pisa_norm_rope_bwd");
}

size_t pisa_qcache_attn_workspace_bytes(const pisa_problem* p) {
  pisa::Shape s{};
  pisa::Geo g{};
  if (check_problem(p, &s, &g) != PISA_OK) return 0;
  return pisa::qcache_attn_ws(s, g);
}

int pisa_qcache_attn_fwd(const pisa_problem* p, const pisa_qcache* c, const void* q, const int32_t* block_idx, void* o,
                         float* lse, void* ws, size_t ws_bytes, pisa_stream_t stream) {
  pisa::Shape s{};
  pisa::Geo g{};
  pisa::QCache qc{};
  PISA_TRY(check_problem(p, &s, &g));
  PISA_TRY(check_qcache(c, g, &qc));
  PISA_TRY(check_ptr(q, "q"));
  PISA_TRY(check_ptr(block_idx, "block_idx"));
  PISA_TRY(check_ptr(o, "o"));
  PISA_TRY(check_ptr(lse, "lse", true));
  PISA_TRY(check_ws(ws, ws_bytes, pisa::qcache_attn_ws(s, g)));
  return device_status(pisa::launch_qcache_attn(s, g, qc, q, block_idx, o, lse, ws, static_cast<hipStream_t>(stream)),
                       "pisa_qcache_attn_fwd");
}

const char* pisa_status_string(int status) {
  switch (status) {
    case PISA_OK: return "ok";
    case PISA_ERR_INVALID_ARG: return "invalid argument";
    case PISA_ERR_UNSUPPORTED: return "unsupported shape";
    case PISA_ERR_WORKSPACE: return "workspace too small";
    case PISA_ERR_DEVICE: return "device error";
    default: return "unknown status";
  }
}

const char* pisa_last_error(void) { return g_last_error; }

}  // extern "C"
