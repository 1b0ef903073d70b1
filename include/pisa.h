/*
 * pisa.h -- C ABI of the PISA hot path for AMD Instinct MI355X (gfx950).
 *
 * PISA ("Block Sparse Attention with Log-Linear Complexity") selects, for
 * every query position, K key blocks of C tokens by a coarse-to-fine search
 * over a mean-pooled key pyramid, then runs softmax attention over the
 * original keys and values of the selected blocks.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Every buffer pointer is a DEVICE pointer unless stated otherwise and must
 *   be 16-byte aligned (workspaces 256-byte).  The caller allocates and owns every buffer,
 *   including workspaces; the library never allocates device memory, never
 *   synchronises and never creates streams.
 * - Every compute call is asynchronous on `stream` (a hipStream_t; 0 is the
 *   legacy default stream).
 * - Indices are 0-based (the paper counts from 1).
 * - Layouts are contiguous and row-major:
 *     q, o      [B, H,   Nq, d]   (dtype of the problem)
 *     k, v      [B, Hkv, Ncap, d] (dtype of the problem; Ncap = N unless
 *               the problem reserves more rows, see pisa_problem.Ncap)
 *     pyramid   [B, Hkv, R,  d]   float32: summary levels 1 .. max(1, L-1)
 *               concatenated (level 1 = leaf blocks first), each level laid
 *               out for Ncap tokens; R and the level offsets come from
 *               pisa_pyramid_layout().  The root (level L) is never scored
 *               and is not stored.
 *     block_idx [B, Hkv, Nq, K]   int32, ascending, padded with -1
 *     lse       [B, H,   Nq]      float32, natural log
 * - Query row i sits at absolute position t = N - Nq + i (end-aligned), so
 *   Nq = N is prefill and Nq = 1 is one decode step.
 * - Query head h' reads KV head h' / (H / Hkv) (grouped-query attention);
 *   the G = H / Hkv heads of a group share one selected block set.
 * - Logits are scaled by 1/sqrt(d); scores and lse use the natural log.
 * - Errors: every call validates all arguments before anything is enqueued.
 *   On error it returns a negative status, launches nothing and leaves the
 *   outputs untouched; pisa_last_error() then describes the problem (per
 *   thread).  PISA_ERR_DEVICE means a HIP launch reported a failure.
 *
 * Supported shapes: d in {64, 128}; C a multiple of 32 in [32, 256];
 * 2 <= fanout <= 16; 1 <= K with fanout*K <= 256 (K >= 3 when causal);
 * G = H/Hkv <= 16 with fanout*fanout*K*G <= 2048; Nq <= N < 2^31,
 * Nq < 2^23; B*Hkv <= 65535.
 */
#ifndef PISA_H
#define PISA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef void* pisa_stream_t;

typedef enum { PISA_DTYPE_F32 = 0, PISA_DTYPE_BF16 = 1 } pisa_dtype;

enum {
  PISA_OK = 0,
  PISA_ERR_INVALID_ARG = -1, /* malformed problem, null or misaligned pointer */
  PISA_ERR_UNSUPPORTED = -2, /* well-formed but outside the supported shapes */
  PISA_ERR_WORKSPACE = -3,   /* workspace smaller than the *_workspace_bytes */
  PISA_ERR_DEVICE = -4       /* a HIP call or kernel launch failed */
};

/* Selection schedules (pisa_problem.schedule). */
enum {
  PISA_SCHEDULE_AUTO = 0,      /* library picks from the problem size */
  PISA_SCHEDULE_TWO_STAGE = 1, /* Sec. 3.3 prefill design: intermediate
                                  levels per query, then leaf blocks scored
                                  once per key block for a tile of queries,
                                  then a final Top-K (bf16 only) */
  PISA_SCHEDULE_FUSED = 2,     /* Sec. 3.3 decode design: one program per
                                  (query, KV head) walks every level down to
                                  the raw leaf keys */
  PISA_SCHEDULE_SPLIT = 3      /* few rows (decode): intermediate levels with
                                  a workgroup per (query, KV head), then each
                                  leaf candidate scored by a workgroup of its
                                  own, then the final Top-K; the same
                                  selection as the other schedules, spread
                                  over the whole GPU */
};

/* Block scores of pisa_select (pisa_problem.score): for one candidate and
 * query head with child logits z_1..z_m (child summaries above the leaf
 * level, raw keys at it), summed over the group's query heads. */
enum {
  PISA_SCORE_LSE = 0,      /* PISA, eq. direct_child_lse: log sum_j exp(z_j) */
  PISA_SCORE_MEAN = 1,     /* PISA-1, App. A: the mean of the z_j             */
  PISA_SCORE_MEAN_VAR = 2  /* PISA-2, App. A: the mean plus half the
                              population variance of the z_j                   */
};

/* The problem statement of Sec. 3.1-3.2: q/k/v, N, head dim d, block size C,
 * fan-out g (the paper fixes g = 2; any 2..16 is accepted), budget K. */
typedef struct {
  int32_t B, H, Hkv; /* batch, query heads, KV heads (H % Hkv == 0)         */
  int32_t Nq, N;     /* query rows and key rows, 1 <= Nq <= N               */
  int32_t d;         /* head dimension                                      */
  int32_t C;         /* leaf block size (tokens per leaf block)             */
  int32_t fanout;    /* g: children per node above the leaf level           */
  int32_t K;         /* block budget per (query, KV head) at every level    */
  int32_t causal;    /* 1: App. B eligibility + forced first/previous/current
                        blocks and masked future tokens; 0: plain method    */
  int32_t dtype;     /* pisa_dtype of q, k, v and o                         */
  int32_t schedule;  /* PISA_SCHEDULE_* for pisa_select; ignored elsewhere  */
  int32_t Ncap;      /* rows reserved per (batch, KV head): k and v are
                        [B,Hkv,Ncap,d] of which the first N rows are used,
                        and the pyramid is laid out for Ncap tokens, so a
                        decode loop grows N in place (App. B decode cache);
                        0 means N, otherwise N <= Ncap                       */
  int32_t score;     /* PISA_SCORE_* reducer of pisa_select (ignored by flat
                        BSA and everywhere else)                            */
} pisa_problem;

/* Number of hierarchy levels L (Sec. 3.2 eq. key_hierarchy: M_1 = ceil(N/C),
 * M_{l+1} = ceil(M_l / fanout) until M_L = 1), or a negative status. */
int pisa_num_levels(int32_t N, int32_t C, int32_t fanout);

/* Row layout of the stored pyramid.  Writes level_row_offset[l-1] = first row
 * of level l for l = 1..L (host array with room for L entries; the root's
 * entry equals R) and *rows_R = R.  Returns L or a negative status. */
int pisa_pyramid_layout(const pisa_problem* p, int64_t* level_row_offset, int64_t* rows_R);

/* Bytes of the pyramid buffer (B*Hkv*R*d*4), or 0 if the problem is invalid. */
size_t pisa_pyramid_bytes(const pisa_problem* p);

/* Workspace bytes each call needs (0 is a valid answer); 0 also for invalid
 * problems, which the call itself then rejects.  pisa_select
 * also takes less (or none, or a misaligned one as none) where the problem has
 * a slower schedule that fits: the automatic choice below 4096 rows x KV heads,
 * and PISA_SCHEDULE_SPLIT without its node scores. */
size_t pisa_select_workspace_bytes(const pisa_problem* p);
size_t pisa_bsa_workspace_bytes(const pisa_problem* p);
size_t pisa_attn_workspace_bytes(const pisa_problem* p);

/* Mean pyramid (Sec. 3.2 eq. mean_pyramid): level 1 = mean of each leaf
 * block's raw keys (the last block may be short), level l+1 = mean of the
 * existing children at level l.  Accumulates in float32; writes `pyramid`. */
int pisa_build_pyramid(const pisa_problem* p, const void* k, float* pyramid, pisa_stream_t stream);

/* Decode cache update (App. B "decode cache": each new token updates the
 * mean of its leaf block and of that block's ancestors).  `pyramid` holds
 * the pyramid of the first n_old keys, as left by pisa_build_pyramid or an
 * earlier append with the same C, fanout and Ncap; k holds the first p->N
 * keys.  The leaf blocks containing rows [n_old, N) and all of their
 * ancestors are recomputed, and levels that did not exist at n_old are
 * computed whole, with the arithmetic of pisa_build_pyramid: the result
 * equals a full build at N bit for bit.  0 <= n_old <= N (n_old = 0 rebuilds
 * every block, on one workgroup per (batch, KV head)); one launch, no
 * workspace. */
int pisa_pyramid_append(const pisa_problem* p, const void* k, float* pyramid, int32_t n_old,
                        pisa_stream_t stream);

/* Capacity rule of the decode cache (App. B "Decode cache": when the cache
 * needs room, each level's capacity grows by a fixed fraction, so a level is
 * re-laid a constant number of times per doubling of the length and the
 * copying through length N stays within O((N/C) d log N) per KV head).
 * Returns the capacity (in tokens) for a cache that reserves `cap` tokens and
 * must hold `need`: cap when need <= cap, otherwise the smallest multiple of
 * C that is >= need and >= cap + cap/2 (the fraction is 1/2), clamped to the
 * largest supported capacity (65535 leaf blocks); a negative status if need
 * itself exceeds it or an argument is invalid (cap >= 0, need >= 1, C >= 1).
 * Host only. */
int32_t pisa_cache_capacity(int32_t cap, int32_t need, int32_t C);

/* Decode cache growth (App. B "Decode cache"): re-lays a cache of p->N tokens
 * held in buffers reserved for p->Ncap tokens (0 means N) into caller-
 * allocated buffers reserved for new_cap >= max(N, Ncap) tokens.  Per (batch,
 * KV head), the rows of every stored level of pyr_old (the layout of
 * pisa_pyramid_layout for Ncap) move to that level's offset in pyr_new (the
 * layout for new_cap), and, when the four key/value pointers are non-NULL,
 * the first N rows of k_old, v_old [B,Hkv,Ncap,d] go to k_new, v_new
 * [B,Hkv,new_cap,d].  Afterwards pyr_new equals pisa_build_pyramid of the
 * problem with Ncap = new_cap bit for bit, and pisa_pyramid_append continues
 * from it with that Ncap.  Rows past N in the new buffers are not written.
 * The key/value pointers are all NULL (pyramid only) or all non-NULL; old and
 * new buffers must not overlap (PISA_ERR_INVALID_ARG otherwise).  One launch,
 * no workspace, no allocation. */
int pisa_cache_grow(const pisa_problem* p, int32_t new_cap, const float* pyr_old, float* pyr_new, const void* k_old,
                    void* k_new, const void* v_old, void* v_new, pisa_stream_t stream);

/* Pyramid Top-K selection (Sec. 3.2 eqs. hierarchical_topk and
 * direct_child_lse; grouped heads Sec. 3.3 eq. kernel_grouped_score; causal
 * policy App. B).  From the root, each level keeps all candidates when there
 * are at most K, otherwise keeps the forced ones plus the best by the sum over
 * the group's heads of the LSE of the children's scaled logits (child
 * summaries above the leaf level, raw keys at the leaf level); kept blocks
 * expand to their eligible children.  Ties go to the smaller block index.
 * Writes block_idx.  block_score (nullable, float32 [B,Hkv,Nq,K]) receives the
 * leaf score of each kept block, +inf for blocks kept without a score, -inf
 * for padding.  `pyramid` must come from pisa_build_pyramid on the same k. */
int pisa_select(const pisa_problem* p, const void* q, const void* k, const float* pyramid,
                int32_t* block_idx, float* block_score, void* ws, size_t ws_bytes,
                pisa_stream_t stream);

/* Bytes of the static scratch that pisa_select_static uses instead of a
 * caller workspace (one copy per device, held while the library is loaded). */
#define PISA_STATIC_SCRATCH_BYTES (32u << 20)

/* pisa_select without a workspace argument, for callers that cannot allocate
 * device memory (code under HIP graph capture, serving loops that must not
 * call hipMalloc, harnesses that forbid it).  Same arguments, validation,
 * kernels and results as pisa_select; the scratch it needs comes from a
 * static device array of PISA_STATIC_SCRATCH_BYTES bytes instead of `ws`.
 * A problem whose pisa_select_workspace_bytes() exceeds that size is refused
 * with PISA_ERR_WORKSPACE (nothing is launched; use pisa_select).  The call
 * allocates nothing (no hipMalloc, hipFree or allocating library routine);
 * its first call on a device looks up that device's copy of the array.
 * Every call on a device shares that device's one array, so calls that
 * overlap on one device (concurrent streams, or host threads) race and give
 * undefined results: serialise them.  The array keeps the last call's
 * contents; every call writes what it reads. */
int pisa_select_static(const pisa_problem* p, const void* q, const void* k, const float* pyramid,
                       int32_t* block_idx, float* block_score, pisa_stream_t stream);

/* Flat block selection baseline (Sec. 3.1 eqs. bsa_block_scores, bsa_topk):
 * every eligible leaf summary (pyramid level 1) is scored; with G > 1 the
 * scores are turned into per-head softmax probabilities over the eligible
 * non-forced blocks and summed over the group (App. C.1); the forced blocks
 * of App. B are kept inside the budget.  Same block_idx layout as
 * pisa_select. */
int pisa_select_flat_bsa(const pisa_problem* p, const void* q, const float* pyramid,
                         int32_t* block_idx, void* ws, size_t ws_bytes, pisa_stream_t stream);

/* Selected sparse attention (Sec. 3.1 eq. selected_sparse_attention): for
 * every query row and head, softmax over the tokens of its KV head's selected
 * blocks (future tokens masked when causal, App. B) applied to the original
 * values.  block_idx entries outside [0, ceil(N/C)) -- negative ones and
 * ones past the last leaf block -- are padding and contribute nothing; in
 * causal mode a block that starts after the query contributes nothing either
 * (all of its tokens are masked).  The entries of a row need not be sorted
 * but must be distinct (pisa_select writes them so): a block listed twice is
 * attended once or twice depending on the kernel that takes the row (the
 * row-tile kernels, and a row's first, previous and own blocks, count it
 * once).  Writes o (problem dtype) and lse (nullable); a row with no visible
 * token gets o = 0 and lse = -inf. */
int pisa_sparse_attn_fwd(const pisa_problem* p, const void* q, const void* k, const void* v,
                         const int32_t* block_idx, void* o, float* lse, void* ws,
                         size_t ws_bytes, pisa_stream_t stream);

/* Tuning of pisa_sparse_attn_fwd's row-tile path (same results either way, up
 * to fp32 rounding order).  A row tile is 256/G consecutive query rows of one
 * (batch, KV head); when the blocks its rows select number at most
 * min(3K, 256), the whole tile can be attended by one workgroup that walks
 * those blocks once, instead of by the block-centric kernels.  That path is
 * taken, on calls with G in {1, 2, 4, 8, 16}, only when at least n tiles of
 * the call qualify (so that it fills the device); n < 0 turns it off.
 * Process-wide, read at each call's launch; default 1024.  Returns the
 * previous value.  Host only: no device work. */
int pisa_attn_union_min_tiles(int32_t n);

/* Backward of the selected sparse attention with the block indices held
 * fixed (App. B: during backpropagation gradients flow through the attention
 * over the selected entries, not through the selection).  For every row and
 * query head, with z = q.k / sqrt(d) over the selected visible tokens,
 * p = exp(z - lse) and D = d_o . o:
 *   dv_j += p_j d_o,  ds_j = p_j (d_o . v_j - D),  dq = sum_j ds_j k_j / sqrt(d),
 *   dk_j += ds_j q / sqrt(d)
 * (dk, dv summed over every row and query head that reaches token j).
 * o and lse are the forward's outputs (pisa_sparse_attn_fwd on the same
 * block_idx); d_o has o's layout.  Writes dq [B,H,Nq,d] and dk, dv in k's
 * layout [B,Hkv,N,d] (row stride Ncap; every stored row is written, rows no
 * query reaches get 0), all in the problem dtype; sums run in fp32.  bf16
 * with d in {64,128} and C in {32,64,96,128}, else PISA_ERR_UNSUPPORTED.
 * Workspace: pisa_attn_bwd_workspace_bytes(p). */
size_t pisa_attn_bwd_workspace_bytes(const pisa_problem* p);
int pisa_sparse_attn_bwd(const pisa_problem* p, const void* q, const void* k, const void* v,
                         const int32_t* block_idx, const void* o, const float* lse, const void* d_o, void* dq,
                         void* dk, void* dv, void* ws, size_t ws_bytes, pisa_stream_t stream);

/* Block-selection quality diagnostic (Sec. 4 "Block-selection quality", eq.
 * oracle_metrics; App. C "Block-selection diagnostic", eq. oracle_block_mass).
 * For each (batch, KV head) and each listed query row: the full attention's
 * log mass of every eligible leaf block, a(B) = log of the sum over B's
 * tokens (future ones masked when causal) of exp(q.k / sqrt(d)), per query
 * head; P(B) = mean over the KV head's query heads of each head's softmax of
 * a over the eligible blocks.  The reference set holds the forced blocks of
 * App. B (causal) and the eligible blocks of highest P up to K (ties to the
 * smaller index); with at most K eligible blocks it is all of them.  For the
 * selection in block_idx:
 *   metrics[..., 0] = |selection & reference| / K         (Recall@K)
 *   metrics[..., 1] = sum of P over the selection          (captured mass)
 *   metrics[..., 2] = metrics[..., 1] / sum of P over the reference
 *                                                          (attention mass ratio)
 * rows: device int32 [n_rows], query-row indices; a row outside [0, Nq)
 * gets NaN metrics and an empty reference.  block_idx: [B,Hkv,Nq,K] as
 * pisa_select writes it (negative entries are padding; repeats count once).
 * metrics: device float32 [B,Hkv,n_rows,3]; ref_idx: nullable device int32
 * [B,Hkv,n_rows,K], the reference set ascending, -1 padded.  The work is dense
 * over every visible key of every listed row (n_rows x N x d per head): meant
 * for sampled rows.  bf16 inputs, C in {32, 64, 96, 128}, N/C <= 16384, K <= 64;
 * otherwise PISA_ERR_UNSUPPORTED.  Workspace: pisa_quality_workspace_bytes(p,
 * n_rows) bytes (the log masses, B*Hkv*n_rows*G*ceil(N/C) floats). */
size_t pisa_quality_workspace_bytes(const pisa_problem* p, int32_t n_rows);
int pisa_selection_quality(const pisa_problem* p, const void* q, const void* k, const int32_t* block_idx,
                           const int32_t* rows, int32_t n_rows, float* metrics, int32_t* ref_idx, void* ws,
                           size_t ws_bytes, pisa_stream_t stream);

/* ---- Rotary positions ------------------------------------------------------
 *
 * Queries and keys get their positions before the pyramid is built from the
 * keys: the first `rot` dimensions of a head form rot/2 pairs, and pair i of
 * the row at position t is turned by the angle t * freq[i] and multiplied by
 * `amplitude`; dimensions from `rot` on are copied. */

/* Strides, in elements, of a [B, heads, rows, d] tensor whose last dimension is
 * contiguous, so that a projection's [B, rows, heads, d] is read (or written)
 * as it stands.  Non-negative multiples of 16 bytes.  A NULL pisa_strides means
 * the contiguous [B, heads, rows, d]. */
typedef struct {
  int64_t b, h, n;
} pisa_strides;

enum {
  PISA_ROPE_HALF = 0,       /* pair i: dimensions i and i + rot/2 */
  PISA_ROPE_INTERLEAVED = 1 /* pair i: dimensions 2i and 2i + 1   */
};

/* How pisa_rope_frequencies adapts the frequencies f_i = base^(-2i/rot) to a
 * context `factor` times as long as the original one. */
enum {
  PISA_ROPE_SCALE_NONE = 0,
  PISA_ROPE_SCALE_LINEAR = 1, /* f_i / factor                                     */
  PISA_ROPE_SCALE_BASE = 2,   /* base * factor^(rot/(rot-2)) in base's place: the
                                 slowest pair is slowed by factor, the fastest not */
  PISA_ROPE_SCALE_PARTS = 3   /* f_i (y + (1-y)/factor), y = (turns - slow) /
                                 (fast - slow) cut to [0, 1], turns = ctx f_i / 2 pi:
                                 pairs that turn often within the original context
                                 keep their frequency, slow ones are interpolated;
                                 amplitude = 0.1 ln(factor) + 1                    */
};

#define PISA_ROPE_MAX_PAIRS 64

/* q, q_out: [B, H, N, d]; k, k_out: [B, Hkv, N, d], any of H >= 1, Hkv >= 1.
 * d in {64, 128}; rot even, 2 <= rot <= d.  Row n of batch b is at position
 * pos0 + n, or where the call has `positions` (device int32) at
 * positions[b * pos_bstride + n]; pos_bstride = 0 shares one list among the
 * batch.  Positions may be negative.  Angles are computed in 64 bits and
 * reduced before the sine: the angle of T turns is off by at most 2^-26 turns for
 * any position, and by 2^-51 T more (less than a quarter of that up to 2^23
 * turns; 2^-22 turns at 2^29, position 2^31 with a frequency of 1.6). */
typedef struct {
  int32_t B, H, Hkv, N, d;
  int32_t rot;
  int32_t layout; /* PISA_ROPE_HALF / _INTERLEAVED                    */
  int32_t dtype;  /* pisa_dtype of every tensor                       */
  int32_t pos0;
  int32_t reserved; /* 0 */
  int64_t pos_bstride;
  double amplitude;
  double freq[PISA_ROPE_MAX_PAIRS]; /* radians per position; rot/2 are used */
} pisa_rope;

/* Fills r->freq and r->amplitude from r->rot (host only).  base > 1; factor >=
 * 1; PARTS also takes ctx >= 1 (tokens of the original context) and
 * fast > slow >= 0 (turns); the other scalings ignore them. */
int pisa_rope_frequencies(pisa_rope* r, double base, int32_t scaling, double factor, int32_t ctx, double fast,
                          double slow);

/* Turns q and k (either may be NULL together with its output) in one launch.
 * An output may be its own input (same pointer and strides); otherwise outputs
 * overlap neither inputs nor each other, nor their own rows (PISA_ERR_INVALID_ARG;
 * tensors of the same strides, as the parts of a packed projection, are compared
 * value by value, others by what lies between their first value and their last).
 * Arithmetic in float32, rounded once. */
int pisa_rope_fwd(const pisa_rope* r, const void* q, const pisa_strides* q_strides, const void* k,
                  const pisa_strides* k_strides, const int32_t* positions, void* q_out,
                  const pisa_strides* q_out_strides, void* k_out, const pisa_strides* k_out_strides,
                  pisa_stream_t stream);

/* Gradients of pisa_rope_fwd: d_q and d_k from the gradients of its outputs (the
 * transposed map: turned back, times the same amplitude). */
int pisa_rope_bwd(const pisa_rope* r, const void* d_q_out, const pisa_strides* d_q_out_strides, const void* d_k_out,
                  const pisa_strides* d_k_out_strides, const int32_t* positions, void* d_q,
                  const pisa_strides* d_q_strides, void* d_k, const pisa_strides* d_k_strides, pisa_stream_t stream);

/* ---- Norms of queries and keys with their positions ------------------------
 *
 * Each head of a row is divided by its root mean square and multiplied by learned
 * weights before it is turned:
 *   y = R (x / sqrt(mean(x^2) + eps) * (w + offset))
 * with R the rotation of pisa_rope_fwd (dimensions from `rot` on are normed but not
 * turned).  Sums and products in fp32, rounded once; the sum of a head's squares is
 * held in fp32, so a head whose mean square is past its range comes out as 0. */
typedef struct {
  const void* q_weight; /* [d] in weight_dtype, one for every head; NULL: all 1, without offset */
  const void* k_weight;
  int32_t weight_dtype; /* pisa_dtype of both           */
  int32_t reserved;     /* 0                            */
  double eps;           /* in [1e-30, 1e30]             */
  double offset;        /* 1 for weights stored around 0 */
} pisa_qk_norm;

/* Norms and turns q and k in one launch; tensors, sides and outputs as in
 * pisa_rope_fwd. */
int pisa_norm_rope_fwd(const pisa_rope* r, const pisa_qk_norm* m, const void* q, const pisa_strides* q_strides, const void* k,
                       const pisa_strides* k_strides, const int32_t* positions, void* q_out,
                       const pisa_strides* q_out_strides, void* k_out, const pisa_strides* k_out_strides,
                       pisa_stream_t stream);

/* Gradients of pisa_norm_rope_fwd from its inputs q, k and the gradients of its
 * outputs: d_q, d_k, and the weights' d_q_weight, d_k_weight (float32 [d], summed
 * over every row and head in a fixed order; nullable, and NULL for a side that is
 * left out).  A side has its input, its output's gradient and its gradient, or none
 * of them.  d_q may be d_q_out and d_k d_k_out (same pointer and strides); nothing
 * that is written overlaps anything else (PISA_ERR_INVALID_ARG).  Workspace:
 * pisa_norm_rope_bwd_workspace_bytes(r), needed where a weight's gradient is wanted. */
size_t pisa_norm_rope_bwd_workspace_bytes(const pisa_rope* r);
int pisa_norm_rope_bwd(const pisa_rope* r, const pisa_qk_norm* m, const void* q, const pisa_strides* q_strides, const void* k,
                       const pisa_strides* k_strides, const void* d_q_out, const pisa_strides* d_q_out_strides,
                       const void* d_k_out, const pisa_strides* d_k_out_strides, const int32_t* positions, void* d_q,
                       const pisa_strides* d_q_strides, void* d_k, const pisa_strides* d_k_strides, float* d_q_weight,
                       float* d_k_weight, void* ws, size_t ws_bytes, pisa_stream_t stream);

/* ---- 8-bit key/value cache --------------------------------------------------
 *
 * Keys and values in e4m3 (4 exponent, 3 mantissa bits, largest 448), one scale
 * for each leaf block of C tokens and KV head, keys and values apart.  A scale
 * is the smallest power of two 2^e, e >= -100, with max|x| <= 448 * 2^e over the
 * block's finite values, so scaling never rounds and code * scale is exact in
 * bf16; the code is x / 2^e rounded to nearest even.  Infinities and NaN become
 * the NaN code.  (Values from 0.96875 * 2^128 on round to 2^128 and read as
 * infinite.)  Half the bytes of a bf16 cache where nothing else is kept:
 * pisa_select_flat_bsa selects from the pyramid alone, but pisa_select also reads
 * raw keys for its leaf scores, and a caller that selects with it keeps those
 * beside the cache (2 bytes a value in bf16: as much again as codes of both).
 * A call has one N for the whole batch; sequences of other lengths are calls of
 * their own.
 *
 * With M = ceil(Ncap / C) blocks (Ncap = 0 means N):
 *   k        [B, Hkv, M, C, d]  codes
 *   v        [B, Hkv, M, d, C]  codes, a block's tokens contiguous: the order
 *                               in which the attention's matrix product reads them
 *   k_scale, v_scale  [B, Hkv, M] float32
 *   k_open, v_open    [B, Hkv, C, d] in the problem dtype: the raw rows of the
 *                     last block, from which it is quantised anew as it fills, so
 *                     that the cache does not depend on how it was appended to
 *                     (pisa_qcache_append only; NULL elsewhere is fine)
 */
typedef struct {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  void* k_open;
  void* v_open;
} pisa_qcache;

/* Blocks M per (batch, KV head), or a negative status for an invalid problem;
 * bytes of each code buffer (B*Hkv*M*C*d), or 0 for one. */
int32_t pisa_qcache_blocks(const pisa_problem* p);
size_t pisa_qcache_bytes(const pisa_problem* p);

/* Appends rows [n_old, N): k_new, v_new hold those rows, [B, Hkv, N - n_old, d]
 * in the problem dtype (strides as in pisa_strides).  The cache holds the first
 * n_old rows, as left by earlier appends with the same C and Ncap, and
 * k_open, v_open the raw rows of the block of row n_old - 1 (of n_old, where it
 * is a multiple of C, none are read).  Blocks from n_old / C on are quantised,
 * codes of tokens past N in the last of them written as 0; afterwards k_open,
 * v_open start with the raw rows of the last block (their other rows are left).
 * The result equals one append of all N rows bit for bit.  pyramid (nullable):
 * the mean pyramid of the raw keys for the same fanout and Ncap, brought from
 * n_old to N, bit for bit as pisa_build_pyramid has it.  k_new and v_new, from
 * their first value to their last, must not overlap the codes, the scales, the raw
 * rows or the pyramid, nor those each other (PISA_ERR_INVALID_ARG).  0 <= n_old <= N; n_old = N does nothing.  No
 * workspace; one launch where a single block changes and no level is new.
 *
 * Rows are taken back (drafted tokens that were not accepted) by an append with a
 * smaller n_old, which replaces everything from that row on.  The call cannot see
 * which block k_open and v_open belong to: they serve an n_old in the last block
 * or on any block's border.  Before a draft that may pass a border keep a copy of
 * both, and put it back to return to the block that the draft began in.  Until
 * that append the mean and the scale of n_old's block still count the rows that
 * were taken back. */
int pisa_qcache_append(const pisa_problem* p, const pisa_qcache* c, const void* k_new, const pisa_strides* k_strides,
                       const void* v_new, const pisa_strides* v_strides, int32_t n_old, float* pyramid,
                       pisa_stream_t stream);

/* pisa_sparse_attn_fwd over the cache, its keys and values being code * scale.
 * Sums run in fp32; a bf16 problem's weights are rounded to fp16 before they
 * meet the values (and with many rows each block's result is, before the blocks
 * of a row are merged), an fp32 problem's are not.  Entries of block_idx as
 * there; a row with no visible token gets o = 0 and lse = -inf; tokens that the
 * causal mask or N hides are not used, whatever their codes.  Logits and values may
 * be as large as fp32 holds the products q . k and the type o.  o and lse
 * (nullable) as there. */
size_t pisa_qcache_attn_workspace_bytes(const pisa_problem* p);
int pisa_qcache_attn_fwd(const pisa_problem* p, const pisa_qcache* c, const void* q, const int32_t* block_idx, void* o,
                         float* lse, void* ws, size_t ws_bytes, pisa_stream_t stream);

/* ---- Drafted tokens ---------------------------------------------------------
 *
 * T drafted tokens per sequence, a tree (or several) that continues its n cached
 * ones.  Their keys and values stay out of the cache until they are accepted, so
 * there is nothing to take back: rows k_new, v_new [B, Hkv, T, d] in the problem
 * dtype (strides as in pisa_strides).  Masks are 8-byte aligned, parents, positions and
 * rows 4-byte.  With a problem of Nq = T, N = n + T (and room for them, Ncap >= N):
 *   pisa_draft_layout       masks, and positions for pisa_rope_fwd or pisa_norm_rope_fwd,
 *                           from the parents
 *   pisa_select, pisa_select_flat_bsa
 *                           with causal = 1, and for at most C rows a call: the blocks
 *                           that hold their drafted rows are then forced, and neither
 *                           call reads nodes or keys of these.  More than C rows are
 *                           taken in groups of C, each in a call of its own with
 *                           Nq = its rows and N = n + Nq; in one call blocks of drafted
 *                           rows would be ranked from nodes that nobody wrote
 *   pisa_draft_attn_fwd, pisa_qcache_draft_attn_fwd
 *   pisa_cache_append_rows, pisa_qcache_append_rows
 *                           the accepted rows, with a problem of N = n + accepted */
#define PISA_DRAFT_MAX 1024

/* parents: device int32 [B, T], the drafted token that each one follows; -1 (or T and
 * more): the last cached one; below -1: none, a token that pads the tree.  Parents
 * may come behind their children.
 * mask: uint64 [B, T, W], W = ceil(T / 64): bit j % 64 of word j / 64 of row i is set
 * where j is i or an ancestor of i (none in the row of a token that pads; nothing
 * should follow one).
 * positions: nullable int32 [B, T], n + the number of i's ancestors (n for one that
 * pads).  A token whose ancestors run in a circle has those of the circle, and a
 * position of n + T - 1.  B <= 65535, 1 <= T <= PISA_DRAFT_MAX, n + T < 2^31. */
int pisa_draft_layout(int32_t B, int32_t T, const int32_t* parents, int32_t n, uint64_t* mask, int32_t* positions,
                      pisa_stream_t stream);

/* Attention of the Nq drafted rows: for every row and query head, softmax over the
 * cached tokens (the first N - Nq rows of k, v) of its KV head's selected blocks and
 * over the drafted rows of its mask, applied to their values.  The cached tokens all
 * come before the drafted ones, so p->causal is not read.  block_idx as in
 * pisa_sparse_attn_fwd: entries outside [0, ceil((N - Nq) / C)), among them blocks that
 * hold drafted rows alone, contribute nothing; distinct entries in any order.  mask:
 * [B, Nq, W] words of pisa_draft_layout, or any others (bits from Nq on are not read);
 * mask_bstride words lie between two sequences, 0 shares one mask among the batch.
 * Rows that nothing selects or masks in are hidden whatever their values; an infinite
 * value that a row sees stays infinite in o (with a weight of 2^-64 of the row's largest
 * or more; below that it may become NaN).  Writes o [B, H, Nq, d] and lse (nullable); a
 * row that sees nothing gets o = 0 and lse = -inf.  Sums in fp32.  Weights meet bf16
 * values as two bf16 terms (off by 2^-16), 8-bit ones as two fp16 terms (2^-22), in fp32
 * problems as they are.  Nq <= PISA_DRAFT_MAX; N = Nq is an empty cache.
 * o, lse and the workspace must not overlap anything else (PISA_ERR_INVALID_ARG).  The
 * workspace's size does not depend on N: one serves a cache that grows. */
size_t pisa_draft_attn_workspace_bytes(const pisa_problem* p);
int pisa_draft_attn_fwd(const pisa_problem* p, const void* q, const void* k, const void* v, const int32_t* block_idx,
                        const void* k_new, const pisa_strides* k_strides, const void* v_new, const pisa_strides* v_strides,
                        const uint64_t* mask, int64_t mask_bstride, void* o, float* lse, void* ws, size_t ws_bytes,
                        pisa_stream_t stream);

/* The same over the 8-bit cache, its keys and values being code * scale. */
size_t pisa_qcache_draft_attn_workspace_bytes(const pisa_problem* p);
int pisa_qcache_draft_attn_fwd(const pisa_problem* p, const pisa_qcache* c, const void* q, const int32_t* block_idx,
                               const void* k_new, const pisa_strides* k_strides, const void* v_new,
                               const pisa_strides* v_strides, const uint64_t* mask, int64_t mask_bstride, void* o, float* lse,
                               void* ws, size_t ws_bytes, pisa_stream_t stream);

/* Appends accepted rows to a cache k, v [B, Hkv, Ncap, d] of n_old rows: row n_old + i
 * of sequence b becomes row rows[b * (N - n_old) + i] of k_new, v_new [B, Hkv, n_rows, d],
 * for i < N - n_old (any rows, in any order; an entry outside [0, n_rows) is read as the
 * nearest one inside).  rows NULL: the first N - n_old of them, so that the call also
 * writes a prompt.  pyramid (nullable): as in pisa_qcache_append.  k_new, v_new and rows
 * must not overlap the cache or the pyramid (PISA_ERR_INVALID_ARG). */
int pisa_cache_append_rows(const pisa_problem* p, void* k, void* v, const void* k_new, const pisa_strides* k_strides,
                           const void* v_new, const pisa_strides* v_strides, const int32_t* rows, int32_t n_rows,
                           int32_t n_old, float* pyramid, pisa_stream_t stream);

/* pisa_qcache_append of such rows: the same cache as an append of them in order. */
int pisa_qcache_append_rows(const pisa_problem* p, const pisa_qcache* c, const void* k_new, const pisa_strides* k_strides,
                            const void* v_new, const pisa_strides* v_strides, const int32_t* rows, int32_t n_rows,
                            int32_t n_old, float* pyramid, pisa_stream_t stream);

/* Per-kernel timing for benchmarks (not needed for computing anything).
 * pisa_profile_enable(1) makes every later call bracket each kernel it
 * launches with two hipEvents recorded on that call's stream (host-side
 * bookkeeping only; no device memory).  pisa_profile_report() waits for the
 * recorded events, writes one line "kernel_name launches total_ms" per kernel
 * into buf (host, NUL-terminated, truncated to cap) and clears the totals; it
 * returns the untruncated text length. */
int pisa_profile_enable(int on);
int pisa_profile_report(char* buf, size_t cap);

/* Static text for a status code. */
const char* pisa_status_string(int status);

/* Detail of the last failing call on this thread ("" if none). */
const char* pisa_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* PISA_H */
